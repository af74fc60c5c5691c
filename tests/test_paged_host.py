"""Host checks of the operators over a page pool (no GPU): what the entry points
refuse (tests/native/paged_refusals_check.cpp, their sources with launches that
only count), how attention's work is dealt out (tests/native/paged_schedule_check.cpp:
every key tile of every unit once over 4000 ragged batches), and what the Python
binding refuses before it calls the library."""
import types

import pytest
import torch

import paper_2609_30884_amd as crf
from tests.test_schedule_host import _build_and_run


def test_entry_points_refuse_before_they_launch(tmp_path):
    assert _build_and_run(tmp_path, "paged_refusals_check") > 150


def test_attention_computes_every_key_tile_once(tmp_path):
    assert _build_and_run(tmp_path, "paged_schedule_check") > 3900


def _ctx():
    return types.SimpleNamespace(dims=crf.make_dims(2, 128, 4, 2, 64, 64), lib=None, handle=None, device=0)


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _state(rows=6):
    pools = [torch.zeros(2, 8, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)]
    x = dict(pool=crf.page_pool(*pools, 16), batch=crf.seq_batch(_i32(4), _i32(3), _i32(3, 2), rows),
             q=torch.zeros(rows, 4, 64, dtype=torch.bfloat16), k=torch.zeros(rows, 2, 64, dtype=torch.bfloat16),
             v=torch.zeros(rows, 128, dtype=torch.bfloat16))
    return types.SimpleNamespace(**x)


@pytest.mark.parametrize("change,status", [
    (dict(q=torch.zeros(6, 4, 64)), 1),                                          # another type
    (dict(q=torch.zeros(5, 4, 64, dtype=torch.bfloat16)), 2),                    # too few rows
    (dict(q=torch.zeros(6, 4, 64, dtype=torch.bfloat16).transpose(1, 2)), 2),
    (dict(q=torch.zeros(4, 6, 64, dtype=torch.bfloat16).transpose(0, 1)), 2),    # heads are not next to each other
    (dict(k=torch.zeros(6, 4, 64, dtype=torch.bfloat16)), 2),
    (dict(v=torch.zeros(6, 256, dtype=torch.bfloat16)[:, ::2]), 2),
    (dict(positions=torch.zeros(6)), 2),
    (dict(positions=_i32(5)), 2),
    (dict(layer=2), 3),
])
def test_rope_append_refuses_tensors(change, status):
    s = _state()
    a = {**dict(q=s.q, k=s.k, v=s.v, layer=0, positions=None), **change}
    with pytest.raises(crf.CrfError) as e:
        crf.rope_append(_ctx(), crf.rope(64, 1e6), s.batch, a["q"], a["k"], a["v"], s.pool, a["layer"], s.q, a["positions"])
    assert e.value.status == status


@pytest.mark.parametrize("change,status", [
    (dict(out=torch.zeros(6, 4, 64)), 1), (dict(out=torch.zeros(6, 128, dtype=torch.bfloat16)), 2),
    (dict(lse=torch.zeros(6, 4, dtype=torch.bfloat16)), 2), (dict(lse=torch.zeros(4, 6).t()), 2), (dict(layer=-2), 3)])
def test_paged_attention_refuses_tensors(change, status):
    s = _state()
    a = {**dict(out=s.q, lse=None, layer=0), **change}
    with pytest.raises(crf.CrfError) as e:
        crf.paged_attention(_ctx(), s.batch, s.q, s.pool, a["layer"], a["out"], lse=a["lse"])
    assert e.value.status == status


def test_pools_and_maps_refuse_tensors():
    k = torch.zeros(2, 8, 2, 16, 64, dtype=torch.bfloat16)
    for a, b, page in ((k, k.float(), 16), (k, k[:1], 16), (k, k, 8), (k[0], k[0], 16),
                       (k.transpose(2, 3), k.transpose(2, 3), 2)):
        with pytest.raises(crf.CrfError):
            crf.page_pool(a, b, page)
    for args in ((_i32(3), _i32(3), _i32(3, 2), 5), (_i32(4), _i32(3).long(), _i32(3, 2), 5),
                 (_i32(4), _i32(3), _i32(2, 3).t(), 5), (_i32(8)[::2], _i32(3), _i32(3, 2), 5)):
        with pytest.raises(crf.CrfError):
            crf.seq_batch(*args)
    for args in ((_i32(8).long(), _i32(3, 2), _i32(3)), (_i32(8), _i32(3, 2), _i32(2)), (_i32(8), _i32(6), _i32(3))):
        with pytest.raises(crf.CrfError):
            crf.page_map(*args, 16)
    s, m = _state(), crf.page_map(_i32(8), _i32(3, 2), _i32(3), 16)
    wrong = types.SimpleNamespace(dims=crf.make_dims(2, 128, 4, 4, 64, 64), lib=None, handle=None, device=0)
    for call in (lambda: crf.pages_fork(wrong, s.pool, m, _i32(1), _i32(1)),
                 lambda: crf.pages_fork(_ctx(), s.pool, m, _i32(2), _i32(1)),
                 lambda: crf.pages_extend(_ctx(), m, _i32(2)),
                 lambda: crf.pages_free(_ctx(), m, torch.zeros(2)),
                 lambda: crf.pages_copy(_ctx(), s.pool, _i32(1), _i32(2)),
                 lambda: crf.pages_copy(_ctx(), s.pool, _i32(1), _i32(1), 1, 2),
                 lambda: crf.pages_compact(_ctx(), s.pool, m, m, _i32(7), _i32(2))):
        with pytest.raises(crf.CrfError):
            call()


def test_host_tensors_are_refused():
    """Right in shape and type, but on the host: nothing reaches the library (lib is None)."""
    s, m = _state(), crf.page_map(_i32(8), _i32(3, 2), _i32(3), 16)
    for call in (lambda: crf.rope_append(_ctx(), crf.rope(64, 1e6), s.batch, s.q, s.k, s.v, s.pool, 0, s.q),
                 lambda: crf.paged_attention(_ctx(), s.batch, s.q, s.pool, 0, s.q),
                 lambda: crf.pages_copy(_ctx(), s.pool, _i32(1), _i32(1)),
                 lambda: crf.pages_fork(_ctx(), s.pool, m, _i32(1), _i32(1)),
                 lambda: crf.pages_extend(_ctx(), m, _i32(3)), lambda: crf.pages_free(_ctx(), m, _i32(1)),
                 lambda: crf.pages_compact(_ctx(), s.pool, m, m, _i32(8), _i32(2))):
        with pytest.raises(crf.CrfError) as e:
            call()
        assert e.value.status == 1 and "host" in str(e.value)


def test_rope_plans():
    r = crf.rope(64, 1e4)
    assert r.mscale == 1.0 and r.freq[0] == 1.0 and abs(r.freq[31] - 1e4 ** (-62 / 64)) < 1e-16
    for args in (dict(rotary_dim=40), dict(layout="other"), dict(scaling="other"), dict(theta=-1.0),
                 dict(scaling="linear", factor=0.0), dict(scaling="parts", factor=2.0)):
        with pytest.raises(crf.CrfError):
            crf.rope(**{**dict(rotary_dim=64, theta=1e4), **args})


def test_rope_plans_are_finite():
    for args in (dict(theta=1e-320), dict(scaling="base", factor=1e-320), dict(mscale=1e300), dict(mscale=float("nan"))):
        with pytest.raises(crf.CrfError):
            crf.rope(**{**dict(rotary_dim=128, theta=1e4), **args})


def test_tables_whose_rows_overlap():
    """One table for several sequences is no table of several rows: its stride would read past it."""
    one = _i32(1, 5)
    with pytest.raises(crf.CrfError):
        crf.seq_batch(_i32(4), _i32(3), one.expand(3, 5), 3)
    with pytest.raises(crf.CrfError):
        crf.page_map(_i32(8), torch.as_strided(_i32(9), (3, 5), (2, 1)), _i32(3), 16)
    assert crf.seq_batch(_i32(2), _i32(1), one.expand(1, 5), 3).table_stride == 5
    assert crf.page_map(_i32(8), _i32(3, 9)[:, :5], _i32(3), 16).table_stride == 9
    empty = torch.zeros(2, 0, 2, 16, 64, dtype=torch.bfloat16)
    assert crf.page_pool(empty, empty, 16).n_pages == 0

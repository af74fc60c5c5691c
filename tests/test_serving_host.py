"""Host checks of a server step's further operators (no GPU): what the entry points
refuse (tests/native/serving_refusals_check.cpp, their sources with launches that
only count), how the work of attention with sinks is dealt out
(tests/native/sink_schedule_check.cpp), and what the Python binding refuses before it
calls the library, or hands to it."""
import types

import pytest
import torch

import paper_2609_30884_amd as crf
from tests.test_schedule_host import _build_and_run

BF = torch.bfloat16


def test_entry_points_refuse_before_they_launch(tmp_path):
    assert _build_and_run(tmp_path, "serving_refusals_check") > 100


def test_sinks_and_windows_are_computed_once(tmp_path):
    assert _build_and_run(tmp_path, "sink_schedule_check") > 2500


def _i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def _ctx(device=0, lib=None):
    return types.SimpleNamespace(dims=crf.make_dims(2, 128, 4, 2, 64, 64), lib=lib, handle=None, device=device)


def _state(rows=6):
    pools = [torch.zeros(2, 8, 2, 16, 64, dtype=BF) for _ in range(2)]
    x = dict(pool=crf.page_pool(*pools, 16), batch=crf.seq_batch(_i32(4), _i32(3), _i32(3, 2), rows),
             q=torch.zeros(rows, 4, 64, dtype=BF), k=torch.zeros(rows, 2, 64, dtype=BF),
             v=torch.zeros(rows, 128, dtype=BF), gain=torch.ones(64, dtype=BF))
    return types.SimpleNamespace(**x)


@pytest.mark.parametrize("change,status", [
    (dict(q_norm=torch.ones(64)), 1), (dict(k_norm=torch.ones(64)), 1), (dict(k_norm=torch.ones(128, dtype=BF)), 2),
    (dict(q_norm=torch.ones(128, dtype=BF)[::2]), 2), (dict(q_norm=torch.ones(1, 64, dtype=BF)), 2),
    (dict(q=torch.zeros(6, 4, 64)), 1), (dict(k=torch.zeros(6, 4, 64, dtype=BF)), 2), (dict(positions=_i32(5)), 2),
    (dict(layer=2), 3)])
def test_norm_rope_append_refuses_tensors(change, status):
    s = _state()
    a = {**dict(q=s.q, k=s.k, q_norm=s.gain, k_norm=s.gain, layer=0, positions=None), **change}
    with pytest.raises(crf.CrfError) as e:
        crf.norm_rope_append(_ctx(), crf.rope(64, 1e6), s.batch, a["q"], a["k"], s.v, a["q_norm"], a["k_norm"], s.pool,
                             a["layer"], s.q, a["positions"])
    assert e.value.status == status


@pytest.mark.parametrize("change,status", [
    (dict(out=torch.zeros(6, 4, 64)), 1), (dict(out=torch.zeros(6, 128, dtype=BF)), 2),
    (dict(lse=torch.zeros(6, 4, dtype=BF)), 2), (dict(layer=-2), 3)])
def test_attention_refuses_tensors(change, status):
    s, groups = _state(), crf.seq_groups(_i32(3), _i32(2))
    a = {**dict(out=s.q, lse=None, layer=0), **change}
    for call in (lambda: crf.sink_attention(_ctx(), s.batch, s.q, s.pool, a["layer"], a["out"], 5, 2, lse=a["lse"]),
                 lambda: crf.shared_attention(_ctx(), s.batch, groups, s.q, s.pool, a["layer"], a["out"], lse=a["lse"])):
        with pytest.raises(crf.CrfError) as e:
            call()
        assert e.value.status == status


def test_groups_refuse_tensors():
    for args in ((_i32(3), _i32(3)), (_i32(4).long(), _i32(3)), (_i32(8)[::2], _i32(3)), (_i32(4), torch.zeros(3)),
                 (_i32(2, 2), _i32(3))):
        with pytest.raises(crf.CrfError):
            crf.seq_groups(*args)
    assert crf.seq_groups(_i32(1), _i32(0)).n_groups == 0


@pytest.mark.parametrize("change,status", [
    (dict(logits=torch.zeros(4, 50, dtype=torch.float16)), 2), (dict(logits=torch.zeros(50, 4).t()), 2),
    (dict(logits=torch.zeros(4, 50, 1)), 2), (dict(logits=torch.zeros(4, 100)[:, ::2]), 2),
    (dict(tokens=_i32(5, 2)), 2), (dict(tokens=_i32(4, 2).long()), 2), (dict(tokens=None), 1), (dict(logprob=None), 1),
    (dict(logprob=torch.zeros(4, 3)), 2), (dict(logprob=torch.zeros(4, 2, dtype=BF)), 2),
    (dict(entropy=torch.zeros(5)), 2), (dict(lse=torch.zeros(8)[::2]), 2), (dict(top_token=None), 1),
    (dict(top_token=_i32(4)), 2), (dict(top_token=_i32(5, 3)), 2), (dict(top_token=_i32(4, 3).long()), 2),
    (dict(top_logprob=torch.zeros(4, 2)), 2)])
def test_token_logprobs_refuses_tensors(change, status):
    a = {**dict(logits=torch.zeros(4, 50), tokens=_i32(4, 2), logprob=torch.zeros(4, 2), entropy=torch.zeros(4),
                lse=torch.zeros(4), top_token=_i32(4, 3), top_logprob=torch.zeros(4, 3)), **change}
    with pytest.raises(crf.CrfError) as e:
        crf.token_logprobs(_ctx(), **a)
    assert e.value.status == status


def test_host_tensors_are_refused():
    """Right in shape and type, but on the host: nothing reaches the library (lib is None)."""
    s = _state()
    for call in (lambda: crf.norm_rope_append(_ctx(), crf.rope(64, 1e6), s.batch, s.q, s.k, s.v, s.gain, s.gain, s.pool, 0,
                                              s.q),
                 lambda: crf.sink_attention(_ctx(), s.batch, s.q, s.pool, 0, s.q, 5, 2),
                 lambda: crf.shared_attention(_ctx(), s.batch, crf.seq_groups(_i32(2), _i32(1)), s.q, s.pool, 0, s.q),
                 lambda: crf.token_logprobs(_ctx(), torch.zeros(4, 50), lse=torch.zeros(4))):
        with pytest.raises(crf.CrfError) as e:
            call()
        assert e.value.status == 1 and "host" in str(e.value)


@pytest.mark.parametrize("given,taken", [(5, 5), (1 << 31, (1 << 31) - 1), ((1 << 32) + 5, (1 << 31) - 1), (-1, -1),
                                         (-(1 << 32) + 7, -1)])
def test_numbers_of_keys_past_an_int(given, taken):
    """Not their low 32 bits: past the longest sequence all keys are meant, and negative ones stay so."""
    got = []
    ctx = _ctx(-1, types.SimpleNamespace(crf_sink_attention=lambda *a: got.append(a[7:9]) or 0,
                                         crf_paged_attention=lambda *a: got.append(a[7]) or 0))
    s = _state()
    crf.sink_attention(ctx, s.batch, s.q, s.pool, 0, s.q, given, given, stream=1)
    crf.paged_attention(ctx, s.batch, s.q, s.pool, 0, s.q, window=given, stream=1)
    assert got == [(taken, taken), taken]

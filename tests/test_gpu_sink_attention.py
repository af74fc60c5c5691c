"""crf_sink_attention against softmax attention in 64 bits: windows and sinks of
every size next to each other, both schedules, pages, strides, values that are no
numbers where nobody sees them; and against crf_paged_attention where they agree."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EDGES = [0, 1, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 511]


def _check(b, window, sinks, what, scale=0.0, ctx=None):
    import paper_2609_30884_amd as crf
    from tests.paged import assert_within, context
    from tests.serving import masked_reference, sink_mask
    ctx = ctx or context(b.nq, b.nkv, b.hd, b.dtype)
    out = torch.full((b.n_rows, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda")
    lse = torch.full((b.n_rows, b.nq), 7.0, device="cuda")
    crf.sink_attention(ctx, b.batch, b.q, b.pool, 1, out, window, sinks, lse=lse, scale=scale)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 0
    ref, rl, bo, bl = masked_reference(b, sink_mask(window, sinks), scale)
    n = b.rows
    assert_within(out[:n], ref[:n], bo[:n], what)
    assert_within(lse[:n], rl[:n], bl[:n], what + " lse")
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()  # rows of nobody
    return out, lse


@pytest.mark.parametrize("dtype,hd,nq,nkv,page", [(BF, 128, 12, 2, 16), (BF, 64, 4, 2, 1), (BF, 128, 28, 4, 32),
                                                  (F32, 64, 4, 2, 16), (F32, 128, 3, 1, 5)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (64, 4), (100, 33), (30, 200), (128, 128), (600, 4)])
def test_steps(dtype, hd, nq, nkv, page, window, sinks):
    from tests.paged import Batch
    print(f"[case] sinks steps {dtype} hd {hd} {nq}/{nkv} page {page} window {window} sinks {sinks}", flush=True)
    _check(Batch([(1, c) for c in EDGES], nq, nkv, hd, dtype, page=page, seed=3), window, sinks, "steps")


@pytest.mark.parametrize("dtype,hd,nq,nkv,page,seqs", [
    (BF, 128, 12, 2, 16, [(5, 0), (1, 700), (0, 40), (3, 129), (2, 64)]),      # drafts: keys shared out
    (BF, 128, 28, 4, 16, [(5, 3), (40, 0), (0, 0), (129, 77), (1, 1000)]),     # tiles of 128 rows
    (BF, 64, 12, 2, 1, [(130, 40), (300, 500)]),
    (BF, 128, 5, 1, 9, [(100, 31), (60, 500)]),
    (F32, 64, 4, 2, 8, [(64, 300), (1, 31), (17, 0), (0, 9), (130, 77)]),
    (F32, 128, 2, 2, 3, [(16, 40), (33, 300)]),
])
@pytest.mark.parametrize("window,sinks", [(1, 3), (50, 1), (50, 70), (200, 129)])
def test_ragged_chunks(dtype, hd, nq, nkv, page, seqs, window, sinks):
    from tests.paged import Batch
    print(f"[case] sinks chunks {dtype} hd {hd} {nq}/{nkv} page {page} window {window} sinks {sinks}", flush=True)
    _check(Batch(seqs, nq, nkv, hd, dtype, page=page, seed=5, pad=4), window, sinks, "chunks")


@pytest.mark.parametrize("dtype,hd,nq,nkv,page,seqs,window,sinks", [
    (BF, 128, 28, 4, 16, [(1, 20000)], 12000, 5000),               # sinks and window split over many workgroups
    (BF, 128, 12, 2, 16, [(1, 9000), (2, 50), (1, 4000)], 3000, 4),
    (BF, 128, 2, 1, 1, [(1, 7000), (1, 2100)], 4500, 2300),        # one-token pages: the staged table refills
    (BF, 64, 12, 2, 16, [(200, 8003)], 2500, 700),
    (BF, 128, 12, 2, 1, [(150, 6500)], 2200, 2300),
    (BF, 128, 12, 2, 16, [(1500, 3000), (40, 6000)], 1000, 16),
    (BF, 64, 12, 2, 16, [(4096, 0)], 300, 64),
    (F32, 64, 4, 2, 16, [(1, 9000), (1, 3)], 2000, 1500),
    (F32, 64, 4, 2, 1, [(70, 4500)], 700, 2500),
])
def test_long(dtype, hd, nq, nkv, page, seqs, window, sinks):
    from tests.paged import Batch
    print(f"[case] sinks long {dtype} hd {hd} page {page} {seqs} window {window} sinks {sinks}", flush=True)
    _check(Batch(seqs, nq, nkv, hd, dtype, page=page, seed=7), window, sinks, "long", scale=0.2)


@pytest.mark.parametrize("dtype,seqs", [(BF, [(1, 900), (1, 40), (1, 0)]), (BF, [(90, 900), (200, 40), (1, 0)]),
                                        (F32, [(90, 300), (1, 40)])])
def test_agrees_with_paged_attention(dtype, seqs):
    """Without sinks, without a window, or with either past every key: the same attention, the first to the bit."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, context
    print(f"[case] sinks as paged attention {dtype} {seqs}", flush=True)
    b = Batch(seqs, 12, 2, 64, dtype, seed=11)
    ctx, out, want = context(12, 2, 64, dtype), torch.zeros_like(b.q), torch.zeros_like(b.q)
    for window, sinks, plain in ((70, 0, 70), (0, 9, 0), (0, 0, 0), (1 << 40, 9, 0)):
        crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, want, window=plain)
        crf.sink_attention(ctx, b.batch, b.q, b.pool, 1, out, window, sinks)
        torch.cuda.synchronize()
        if plain == window:
            assert torch.equal(out, want)
        _check(b, window, sinks, f"window {window} sinks {sinks}", ctx=ctx)
    for window, sinks in ((10, 1 << 40), (10, (1 << 31) - 1), ((1 << 31) - 1, (1 << 31) - 1), ((1 << 31) - 5, 7)):
        _check(b, window, sinks, f"window {window} sinks {sinks}", ctx=ctx)
    assert ctx.device_errors() == 0


@pytest.mark.parametrize("dtype,page", [(BF, 16), (F32, 8), (BF, 5)])
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("odd", [math.nan, math.inf])
def test_what_nobody_sees_has_no_influence(dtype, page, new, odd):
    """Keys between the sinks and the windows, slots past the end, and rows that see none of a bad value."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, context
    print(f"[case] sinks unseen {dtype} page {page} new {new} {odd}", flush=True)
    window, sinks = 60, 7
    b = Batch([(new, 400), (new, 3)], 4, 2, 64, dtype, page=page, seed=13)
    ctx, out, want = context(4, 2, 64, dtype), torch.zeros_like(b.q), torch.zeros_like(b.q)
    crf.sink_attention(ctx, b.batch, b.q, b.pool, 1, want, window, sinks)
    used = torch.zeros(b.n_pages, page, dtype=torch.bool, device="cuda")
    for s, t in enumerate(b.total):
        first = t - b.new[s] - window + 1
        j = torch.arange(t)
        pg, sl = b.places(s, j[(j < sinks) | (j >= first)])
        used[pg, sl] = True
    for pool in (b.k_pool, b.v_pool):
        pool[1].permute(0, 2, 1, 3)[~used] = odd
    crf.sink_attention(ctx, b.batch, b.q, b.pool, 1, out, window, sinks)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    # a value that one row's window alone has (the first row's first key) counts there only
    pg, sl = b.places(0, torch.tensor([400 - window + 1]))
    b.v_pool[1, pg, 0, sl, 9] = odd
    crf.sink_attention(ctx, b.batch, b.q, b.pool, 1, out, window, sinks)
    torch.cuda.synchronize()
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[0, :2, 9] = True
    assert torch.equal(out[~hit], want[~hit]) and not torch.isfinite(out[hit]).any()
    assert ctx.device_errors() == 0


def test_pages_out_of_range():
    """Between sinks and window they are never looked at; among the sinks nobody sees their keys."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, assert_within, context
    from tests.serving import masked_reference
    print("[case] sinks, bad pages", flush=True)
    b = Batch([(1, 1000), (100, 1000)], 12, 2, 128, BF, seed=17)
    ctx, out = context(12, 2, 128, BF), torch.zeros_like(b.q)
    window, sinks = 100, 40
    b.tables[:, 10:40] = -1
    for bad in (False, True):
        if bad:
            b.tables[:, 1] = b.n_pages  # tokens 16 .. 31
        crf.sink_attention(ctx, b.batch, b.q, b.pool, 1, out, window, sinks)
        torch.cuda.synchronize()
        assert ctx.device_errors() == int(bad)

        def seen(s, pos, key):
            return (key <= pos) & ((key > pos - window) | (key < sinks)) & ~((key // 16 == 1) & bad)
        ref, _, bo, _ = masked_reference(b, seen)
        assert_within(out, ref, bo, "bad pages" if bad else "unread pages")

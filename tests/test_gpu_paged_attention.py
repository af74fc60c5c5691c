"""crf_paged_attention against softmax attention in 64 bits: lengths from one
token to long ones, page sizes, head layouts, windows, strides, both schedules."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = "bf16", "f32"


def _dt(name):
    return torch.bfloat16 if name == BF else torch.float32


def _run(b, ctx=None, lse=True, **kw):
    import paper_2609_30884_amd as crf
    from tests.paged import context
    ctx = ctx or context(b.nq, b.nkv, b.hd, b.dtype)
    out = torch.full((b.n_rows, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda")
    ls = torch.full((b.n_rows, b.nq), 7.0, dtype=torch.float32, device="cuda") if lse else None
    crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out, lse=ls, **kw)
    torch.cuda.synchronize()
    return out, ls, ctx


def _check(b, what, flags=0, hidden=None, **kw):
    from tests.paged import assert_within, attention_reference
    out, lse, ctx = _run(b, **kw)
    assert ctx.device_errors() == flags
    ref, rl, bo, bl = attention_reference(b, hidden=hidden, **kw)
    n = b.rows
    assert_within(out[:n], ref[:n], bo[:n], what)
    assert_within(lse[:n], rl[:n], bl[:n], what + " lse")
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()  # rows of nobody
    return out, lse, ctx


EDGES = [0, 1, 15, 30, 31, 32, 33, 62, 63, 64, 126, 127, 128, 129, 255, 256, 511]


@pytest.mark.parametrize("dtype,hd,nq,nkv,page", [
    (BF, 128, 12, 2, 16), (BF, 128, 28, 4, 16), (BF, 64, 4, 2, 16), (BF, 128, 3, 3, 8), (BF, 64, 32, 2, 1),
    (BF, 128, 28, 1, 32), (BF, 64, 10, 2, 7), (BF, 128, 2, 1, 48), (F32, 64, 4, 2, 16), (F32, 128, 3, 1, 16),
    (F32, 64, 6, 6, 1), (F32, 128, 8, 2, 5), (F32, 64, 16, 1, 64)])
def test_steps_of_every_short_length(dtype, hd, nq, nkv, page):
    from tests.paged import Batch
    print(f"[case] steps {dtype} hd {hd} heads {nq}/{nkv} page {page}", flush=True)
    _check(Batch([(1, c) for c in EDGES], nq, nkv, hd, _dt(dtype), page=page, seed=3), "steps")


@pytest.mark.parametrize("dtype,hd,nq,nkv,page,seqs", [
    (BF, 128, 12, 2, 16, [(5, 0), (1, 700), (0, 40), (3, 129), (2, 64)]),          # drafts: keys shared out
    (BF, 64, 4, 4, 16, [(32, 0), (31, 33), (32, 500), (7, 1)]),                    # 32 rows of one head
    (BF, 128, 28, 4, 16, [(5, 3), (40, 0), (0, 0), (129, 77), (1, 1000)]),         # tiles of 128 rows
    (BF, 128, 12, 2, 32, [(200, 1000), (21, 0), (22, 0), (64, 64), (1, 0)]),
    (BF, 64, 12, 2, 1, [(130, 40), (300, 0)]),
    (BF, 128, 5, 1, 9, [(100, 31), (60, 500)]),
    (BF, 64, 80, 2, 16, [(33, 100), (4, 64)]),                                     # more heads than rows of 32
    (F32, 64, 4, 2, 8, [(64, 300), (1, 31), (17, 0), (0, 9), (130, 77)]),
    (F32, 128, 3, 1, 16, [(50, 0), (12, 200), (1, 1)]),
    (F32, 128, 2, 2, 3, [(16, 40), (33, 100)]),
])
@pytest.mark.parametrize("window", [0, 1, 50])
def test_ragged_chunks(dtype, hd, nq, nkv, page, seqs, window):
    from tests.paged import Batch
    print(f"[case] chunks {dtype} hd {hd} heads {nq}/{nkv} page {page} window {window} {seqs}", flush=True)
    _check(Batch(seqs, nq, nkv, hd, _dt(dtype), page=page, seed=5, pad=4), "chunks", window=window)


@pytest.mark.parametrize("dtype,hd,nq,nkv,page,seqs,window", [
    (BF, 128, 28, 4, 16, [(1, 20000)], 0),                     # one long step over all units
    (BF, 128, 12, 2, 16, [(1, 9000), (2, 50), (1, 4000)], 0),
    (BF, 128, 2, 1, 1, [(1, 5000), (1, 2100)], 0),             # one-token pages: the staged table refills
    (BF, 64, 12, 2, 16, [(200, 8003)], 0),                     # few tiles over a long prefix
    (BF, 128, 12, 2, 1, [(150, 4500)], 0),
    (BF, 128, 12, 2, 16, [(1500, 3000), (40, 6000)], 1000),
    (BF, 128, 12, 2, 16, [(4096, 0)], 0),                      # a window's shape
    (F32, 64, 4, 2, 16, [(1, 9000), (1, 3)], 0),
    (F32, 128, 4, 2, 16, [(100, 3000)], 0),
    (F32, 64, 4, 2, 1, [(70, 2500)], 700),
])
def test_long_prefixes(dtype, hd, nq, nkv, page, seqs, window):
    from tests.paged import Batch
    print(f"[case] long {dtype} hd {hd} heads {nq}/{nkv} page {page} window {window} {seqs}", flush=True)
    _check(Batch(seqs, nq, nkv, hd, _dt(dtype), page=page, seed=7), "long", window=window)


def test_many_units():
    """More units than four to a resident workgroup: one unit a workgroup, none split."""
    from tests.paged import Batch
    print("[case] many sequences", flush=True)
    _check(Batch([(1, (37 * i) % 300) for i in range(700)], 8, 4, 64, torch.bfloat16, seed=9), "many steps")
    print("[case] many row tiles", flush=True)
    _check(Batch([(3000, 10), (1, 2), (2900, 0)], 32, 8, 64, torch.bfloat16, seed=9), "many tiles")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_scale_and_strides(dtype):
    """Queries and outputs as slices of wider rows, a padded pool, and a scale of the caller's."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, assert_within, attention_reference, context
    print(f"[case] strides {dtype}", flush=True)
    dt = _dt(dtype)
    b = Batch([(9, 100), (1, 33), (40, 0)], 4, 2, 64, dt, seed=11, wide=3)
    wide = torch.randn(b.n_rows, 4 * 64 + 2 * 2 * 64, device="cuda").to(dt)
    wide[:, :256] = b.q.reshape(b.n_rows, 256)
    big = torch.zeros(3, b.n_pages + 2, 2 * 16 * 64 + 64, dtype=dt, device="cuda")
    kp, vp = big[:2, :b.n_pages], big.clone()[:2, :b.n_pages]
    kp[..., :2048] = b.k_pool.reshape(2, b.n_pages, -1)
    vp[..., :2048] = b.v_pool.reshape(2, b.n_pages, -1)
    split = lambda t: t[..., :2048].unflatten(-1, (2, 16, 64))  # noqa: E731
    pool = crf.page_pool(split(kp), split(vp), 16)
    ctx = context(4, 2, 64, dt)
    out = torch.zeros(b.n_rows, 4 * 64 + 8, dtype=dt, device="cuda")
    crf.paged_attention(ctx, b.batch, wide[:, :256], pool, 1, out[:, :256], scale=0.3)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 0
    ref, _, bo, _ = attention_reference(b, scale=0.3)
    assert_within(out[:, :256].reshape(b.n_rows, 4, 64), ref, bo, "strides")
    assert (out[:, 256:] == 0).all()
    # in place
    crf.paged_attention(ctx, b.batch, b.q, pool, 1, b.q, scale=0.3)
    torch.cuda.synchronize()
    assert torch.equal(b.q.reshape(b.n_rows, 256), out[:, :256])


@pytest.mark.parametrize("dtype,hd,nq,seqs", [
    (BF, 128, 12, [(60, 1500), (200, 700)]), (BF, 64, 12, [(130, 900), (64, 333)]), (F32, 64, 4, [(150, 700)]),
    (F32, 128, 4, [(130, 400)]), (BF, 128, 12, [(1, 1500), (2, 900), (1, 40)]), (F32, 64, 4, [(1, 1500), (3, 200)])])
def test_keys_that_outweigh_all_before(dtype, hd, nq, seqs):
    """A few keys score 40 times the others, in the first and the second half of tiles of 64 and of 128: the reference
    rises in the middle of a prefix, for some rows of a tile and not for others, or falls behind at once."""
    from tests.paged import Batch
    print(f"[case] spikes {dtype} hd {hd} {seqs}", flush=True)
    b = Batch(seqs, nq, 2, hd, _dt(dtype), seed=23)
    for s, t in enumerate(b.total):
        spikes = (3, 37, 70, 101, 135, 200, 230, 290, 355, 420, 500, 707, 1100)
        pg, sl = b.places(s, torch.tensor([x for x in spikes if x < t]))
        b.k_pool[1, pg, :, sl] *= 40
    _check(b, "spikes")


@pytest.mark.parametrize("dtype,hd,seqs", [(BF, 128, [(40, 2000), (100, 900)]), (BF, 64, [(1, 2000), (2, 500)]),
                                           (F32, 64, [(90, 1500)])])
def test_values_near_the_largest(dtype, hd, seqs):
    """Weights that rise by 2^15 along the keys times values of 2^109: the sums pass the
    range unless the reference follows the scores."""
    from tests.paged import Batch
    print(f"[case] large values {dtype} hd {hd}", flush=True)
    b = Batch(seqs, 4, 2, hd, _dt(dtype), seed=21)
    b.q.fill_(1.0)
    for s, t in enumerate(b.total):
        pg, sl = b.places(s)
        rise = torch.arange(t, device="cuda") * (15 * math.log(2) / t) * hd ** -0.5
        b.k_pool[1, pg, :, sl] = rise[:, None, None].to(b.dtype).expand(t, 2, hd)
    b.v_pool.copy_(b.v_pool.abs() * 2.0 ** 109)
    _check(b, "large values")


@pytest.mark.parametrize("dtype,nq,nkv", [(BF, 12, 2), (F32, 4, 2)])
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see(dtype, nq, nkv, odd):
    """Unused slots and spare pages hold no numbers, and neither does a late token: rows before it are as without."""
    from tests.paged import Batch
    print(f"[case] unseen {dtype} {odd}", flush=True)
    b = Batch([(1, 40), (50, 90), (6, 0), (1, 200)], nq, nkv, 64, _dt(dtype), seed=13, fill=odd)
    _check(b, "unused slots")
    clean, _, _ = _run(b)
    pg, sl = b.places(1, torch.tensor([110]))
    b.k_pool[1, pg, :, sl] = odd
    b.v_pool[1, pg, 0, sl] = odd
    b.v_pool[1, pg, 1, sl, 3] = odd
    got, lse, _ = _run(b)
    first, at = b.starts[1], b.starts[1] + 110 - 90
    keep = torch.ones(b.n_rows, dtype=torch.bool, device="cuda")
    keep[at:first + 50] = False
    assert torch.equal(got[keep], clean[keep])
    assert torch.isfinite(lse[keep]).all()
    # only values odd: the definition's infinities and NaN where the key is seen
    b.k_pool[1, pg, :, sl] = 0.5
    _check(b, "odd values")


def test_pages_out_of_range():
    """Keys on bad pages are seen by nobody; a row that sees none gets zeros and -inf; the flag says so."""
    from tests.paged import Batch
    for dtype, nq in ((BF, 12), (F32, 4)):
        for seqs in ([(1, 100), (1, 5), (2, 300)], [(60, 100), (1, 5), (20, 300)]):
            print(f"[case] bad pages {dtype} {seqs}", flush=True)
            b = Batch(seqs, nq, 2, 64, _dt(dtype), seed=17)
            bad = b.tables.clone()
            bad[0, 3], bad[1, 0], bad[2, 0], bad[2, 17] = -1, b.n_pages, 1 << 30, -(1 << 31)
            b.tables.copy_(bad)
            gone = {0: [3], 1: [0], 2: [0, 17]}

            def hidden(s):
                page = torch.arange(b.total[s], device="cuda") // b.page
                return (page[:, None] == torch.tensor(gone[s], device="cuda")).any(1)

            out, lse, _ = _check(b, "bad pages", flags=1, hidden=hidden)
            r = b.starts[1]
            assert (out[r] == 0).all() and (lse[r] == -math.inf).all()


def test_sequences_that_contradict_the_batch():
    from tests.paged import Batch, context
    print("[case] contradictions", flush=True)
    b = Batch([(3, 20), (2, 30), (1, 40), (4, 10)], 4, 2, 64, torch.bfloat16, seed=19)
    ctx = context(4, 2, 64, torch.bfloat16)
    good, _, _ = _run(b, ctx)
    for change in ("short", "long", "order", "past"):
        length, start = b.length.clone(), b.row_start.clone()
        if change == "short":
            length[1] = 1          # fewer tokens than new ones
        elif change == "long":
            length[1] = 1 << 20    # past its table
        elif change == "order":
            start[2] = 2           # sequence 1 has -1 rows (and sequence 2 one of sequence 0's)
        else:
            start[4] = 1000        # rows past the tensors
        keep_l, keep_s = b.length.clone(), b.row_start.clone()
        b.length.copy_(length)
        b.row_start.copy_(start)
        out, _, _ = _run(b, ctx)
        assert ctx.device_errors() & 2, change
        rows = [0, 1] + ([2, 5] if change != "order" else []) + (list(range(6, 10)) if change != "past" else [])
        assert torch.equal(out[rows], good[rows]), change
        b.length.copy_(keep_l)
        b.row_start.copy_(keep_s)
    assert ctx.device_errors() == 0


@pytest.mark.parametrize("seqs", [[(1, 6000), (1, 100)], [(300, 3000), (1, 77)]])
def test_same_bits_twice_and_on_another_stream(seqs):
    from tests.paged import Batch
    print(f"[case] repeat {seqs}", flush=True)
    b = Batch(seqs, 12, 2, 128, torch.bfloat16, seed=23)
    out, lse, ctx = _run(b)
    for _ in range(5):
        o2, l2, _ = _run(b, ctx)
        assert torch.equal(out, o2) and torch.equal(lse, l2)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        o2, l2, _ = _run(b, ctx)
    assert torch.equal(out, o2) and torch.equal(lse, l2)


def test_captured_step_follows_lengths():
    """One captured step, replayed as the sequence grows: each replay equals the eager call."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, context
    print("[case] captured", flush=True)
    b = Batch([(1, 3000), (1, 10), (1, 500)], 12, 2, 128, torch.bfloat16, seed=29)
    ctx = context(12, 2, 128, torch.bfloat16)
    out = torch.zeros_like(b.q)
    crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out)
    for i, lens in enumerate(([3001, 11, 501], [1, 1, 1], [2500, 7, 333], [3001, 2, 64])):
        b.length.copy_(torch.tensor(lens, dtype=torch.int32))
        b.q.normal_()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.zero_()
        crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out)
        torch.cuda.synchronize()
        assert torch.equal(got, out), i
        b.total = lens
        eager, lse, _ = _check(b, f"replay {i}")
        assert torch.equal(eager, got)
    assert ctx.device_errors() == 0


def test_offsets_past_4_gib():
    """A layer of 4.7 GiB a pool: pages at its end are found."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, assert_within, attention_reference, context
    print("[case] large pool", flush=True)
    b = Batch([(1, 90), (70, 200)], 12, 2, 128, torch.bfloat16, page=16, seed=31)
    n = 600000
    pools = [torch.empty(1, n, 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    tables = b.tables.clone()
    for s, t in enumerate(b.total):
        held = -(-t // 16)
        old = b.tables[s, :held].long()
        new = n - 1 - 3 * old
        tables[s, :held] = new.int()
        for big, small in zip(pools, (b.k_pool, b.v_pool)):
            big[0, new] = small[1, old]
    ctx = context(12, 2, 128, torch.bfloat16)
    batch = crf.seq_batch(b.row_start, b.length, tables, b.n_rows, 70)
    out = torch.zeros_like(b.q)
    crf.paged_attention(ctx, batch, b.q, crf.page_pool(*pools, 16), 0, out)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 0
    ref, _, bo, _ = attention_reference(b)
    assert_within(out, ref, bo, "large pool")

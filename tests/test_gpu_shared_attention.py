"""crf_shared_attention against softmax attention in 64 bits: groups of every size
and shared length, sequences of no group, contradicting groups, pages, strides,
values that are no numbers; and captured."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Grouped:
    """groups: (shared tokens, [(new, own cached) ...]); alone: (new, cached) behind them.  A Batch whose group members'
    first pages are the first member's (a begun page is a copy, as a fork leaves it).  Tables are as wide as it takes
    for the batch not to count as a small one, whose sequences read their keys by themselves (small: as they are)."""

    def __new__(cls, groups, nq, nkv, hd, dtype, alone=(), page=16, seed=0, pad=0, max_new=None, ahead=(), small=False):
        import paper_2609_30884_amd as crf
        from tests.paged import Batch
        seqs, start, shared = list(ahead), [len(ahead)], []
        for doc, members in groups:
            seqs += [(n, doc + own) for n, own in members]
            start.append(len(seqs))
            shared.append(doc)
        seqs += list(alone)
        one = page * nkv * hd * 2 * (2 if dtype == BF else 4)  # bytes of a page
        wide = 0 if small else (41 << 20) // (one * len(seqs)) + 1
        b = Batch(seqs, nq, nkv, hd, dtype, page=page, seed=seed, pad=pad, max_new=max_new, wide=wide)
        for g, doc in enumerate(shared):
            first = start[g]
            for s in range(first + 1, start[g + 1]):
                b.tables_h[s, :doc // page] = b.tables_h[first, :doc // page]
                if doc % page:
                    a, c = (int(b.tables_h[i, doc // page]) for i in (first, s))
                    for pool in (b.k_pool, b.v_pool):
                        pool[1, c, :, :doc % page] = pool[1, a, :, :doc % page]
        b.tables.copy_(b.tables_h)
        b.seq_start, b.shared = _i32(start), _i32(shared)
        b.groups = crf.seq_groups(b.seq_start, b.shared)
        return b


def _run(b, ctx, scale=0.0):
    import paper_2609_30884_amd as crf
    out = torch.full((b.n_rows, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda")
    lse = torch.full((b.n_rows, b.nq), 7.0, device="cuda")
    crf.shared_attention(ctx, b.batch, b.groups, b.q, b.pool, 1, out, lse=lse, scale=scale)
    torch.cuda.synchronize()
    return out, lse


def _check(b, what, scale=0.0, flags=0, ctx=None, skip=()):
    from tests.paged import assert_within, context
    from tests.serving import masked_reference, sink_mask
    ctx = ctx or context(b.nq, b.nkv, b.hd, b.dtype)
    out, lse = _run(b, ctx, scale)
    assert ctx.device_errors() == flags
    ref, rl, bo, bl = masked_reference(b, sink_mask(0, 0), scale)
    keep = torch.ones(b.n_rows, dtype=torch.bool, device="cuda")
    keep[b.rows:] = False
    for s in skip:
        keep[b.starts[s]:b.starts[s + 1]] = False
    assert_within(out[keep], ref[keep], bo[keep], what)
    assert_within(lse[keep], rl[keep], bl[keep], what + " lse")
    assert (out[~keep] == 7.0).all() and (lse[~keep] == 7.0).all()  # rows of nobody
    return out, lse, ctx


@pytest.mark.parametrize("dtype,hd,nq,nkv,page", [
    (BF, 128, 12, 2, 16), (BF, 128, 28, 4, 16), (BF, 64, 4, 2, 1), (BF, 128, 3, 3, 8), (BF, 64, 32, 2, 32),
    (BF, 128, 28, 1, 48), (F32, 64, 4, 2, 16), (F32, 128, 3, 1, 5), (F32, 64, 16, 1, 64)])
@pytest.mark.parametrize("docs", [(0, 1, 15), (16, 63, 64), (65, 128, 500)])
def test_steps(dtype, hd, nq, nkv, page, docs):
    print(f"[case] shared steps {dtype} hd {hd} {nq}/{nkv} page {page} {docs}", flush=True)
    own = [0, 1, 15, 16, 33, 70, 200]
    groups = [(docs[0], [(1, o) for o in own]), (docs[1], [(1, 3)]), (docs[2], [(1, o) for o in own[::-1]] * 3)]
    _check(Grouped(groups, nq, nkv, hd, dtype, alone=[(1, 90), (1, 0)], page=page, seed=3, pad=2), "steps")


@pytest.mark.parametrize("dtype,hd,nq,nkv,page", [(BF, 128, 12, 2, 16), (BF, 64, 4, 4, 7), (F32, 64, 4, 2, 16),
                                                  (F32, 128, 2, 2, 1)])
def test_drafts_and_idle_sequences(dtype, hd, nq, nkv, page):
    print(f"[case] shared drafts {dtype} hd {hd} {nq}/{nkv} page {page}", flush=True)
    groups = [(300, [(0, 4), (5, 0), (20, 31), (0, 0), (1, 64)]), (77, [(0, 9), (0, 0)]), (40, [(21, 2)] * 9),
              (1000, [(1, 0)] * 40)]
    _check(Grouped(groups, nq, nkv, hd, dtype, ahead=[(3, 5), (0, 7)], alone=[(21, 0), (1, 500)], page=page, seed=5,
                   pad=5), "drafts")


@pytest.mark.parametrize("dtype,hd,nq,nkv,page,groups", [
    (BF, 128, 28, 4, 16, [(16384, [(1, 20 * i) for i in range(16)]), (9000, [(1, 100)] * 3)]),
    (BF, 128, 2, 1, 1, [(5000, [(1, 3000), (2, 2100)])]),            # one-token pages: the staged table refills
    (BF, 64, 12, 2, 16, [(7000, [(4, 3000)] * 4), (40, [(10, 9000)])]),
    (F32, 64, 4, 2, 8, [(6000, [(1, 900)] * 5)]),
])
def test_long(dtype, hd, nq, nkv, page, groups):
    print(f"[case] shared long {dtype} hd {hd} {nq}/{nkv} page {page}", flush=True)
    b = Grouped(groups, nq, nkv, hd, dtype, page=page, seed=7)
    first = _check(b, "long", scale=0.15)
    again = _run(b, first[2], 0.15)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_many_groups_and_sequences():
    print("[case] shared many", flush=True)
    import random
    r = random.Random(3)
    groups = [(r.randrange(0, 90), [(r.randrange(0, 3), r.randrange(0, 40)) for _ in range(r.randrange(1, 6))])
              for _ in range(90)]
    _check(Grouped(groups, 8, 4, 64, BF, page=8, seed=9, pad=1), "many")
    _check(Grouped([(50, [(1, i % 30) for i in range(600)])], 8, 4, 64, BF, seed=9), "many in one")
    _check(Grouped([(20, [(1, i % 7)]) for i in range(1100)], 2, 2, 64, BF, seed=9), "more groups than are shared")


def test_what_the_plain_kernels_take():
    """Small batches, sequences that fill tiles by themselves, and a batch whose parts the workspace does not hold."""
    import paper_2609_30884_amd as crf
    from tests.paged import context
    print("[case] shared chunks", flush=True)
    ctx = context(12, 2, 64, BF)
    for what, b in (("small", Grouped([(300, [(1, 20), (2, 0)])], 12, 2, 64, BF, seed=11, small=True)),
                    ("chunks", Grouped([(300, [(70, 20), (200, 0)])], 12, 2, 64, BF, seed=11))):
        out, _, _ = _check(b, what, ctx=ctx)
        want = torch.zeros_like(out)
        crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    b = Grouped([(300, [(1, 20), (2, 0)])], 12, 2, 64, BF, seed=11)
    assert not torch.equal(_check(b, "shared", ctx=ctx)[0], torch.zeros_like(b.q))
    b = Grouped([(30, [(9, 0)] * 900)], 28, 4, 128, BF, seed=11)  # 226800 rows of heads
    _check(b, "no room", ctx=context(28, 4, 128, BF))


def test_groups_that_contradict():
    """Flagged; nothing is shared by them, and every row that is a sequence's is right."""
    print("[case] shared contradictions", flush=True)

    def batch(**kw):
        return Grouped([(64, [(1, 3), (2, 40)]), (80, [(1, 0), (0, 9), (3, 5)])], 4, 2, 64, BF, alone=[(1, 30)], seed=13,
                       pad=2, **kw)
    for start in ([0, 2, 9], [-1, 2, 5], [3, 2, 5], [0, 2, 1], [0, 2, 1 << 30], [5, 5, 1]):
        b = batch()
        b.seq_start.copy_(_i32(start))
        _check(b, f"start {start}", flags=2)
    for shared in ([64, 82], [-1, 80], [1 << 30, 80], [64, -(1 << 31)]):
        b = batch()
        b.shared.copy_(_i32(shared))
        _check(b, f"shared {shared}", flags=2)
    # a member that does not reach behind what is shared sees what is before it: no contradiction
    b = Grouped([(64, [(1, 30), (2, 0)])], 4, 2, 64, BF, seed=15)
    b.shared.copy_(_i32([65]))
    b.tables_h[1, 4] = b.tables_h[0, 4]
    b.tables.copy_(b.tables_h)
    _check(b, "shared past a member's own")
    # a sequence that contradicts the batch has no rows, the others of its group keep theirs
    b = batch()
    b.length[1] = 1
    _check(b, "short", flags=2, skip=[1])
    b = batch()
    b.length[0] = 50  # the first one is shorter than what is shared: nothing is
    b.total[0] = 50
    _check(b, "short first", flags=2)


def test_a_contradicting_sequence_among_many():
    """Row starts out of range in a batch of more sequences than a workgroup has threads: two have no rows, all others
    of the group are right."""
    print("[case] shared contradiction among many", flush=True)
    b = Grouped([(40, [(1, i % 5) for i in range(600)])], 4, 2, 64, BF, seed=18, pad=2, max_new=1)
    b.row_start[10] = 1 << 30
    _check(b, "row start out of range", flags=2, skip=[9, 10])


def test_rows_claimed_over_and_over():
    """Row starts that go back and forth claim more rows than there are: flagged, and no row is written out of range."""
    import paper_2609_30884_amd as crf
    from tests.paged import context
    print("[case] shared rows claimed twice", flush=True)
    b = Grouped([(32, [(1, 3)] * 8)], 28, 4, 128, BF, seed=17, max_new=4)
    ctx, n = context(28, 4, 128, BF), 2600
    guard = torch.full((b.n_rows + 8, 28, 128), 7.0, dtype=BF, device="cuda")
    back = _i32([4 * (i % 2) for i in range(n + 1)])
    batch = crf.seq_batch(back, b.length[:1].repeat(n), b.tables[:1, :40].repeat(n, 1), b.n_rows, 4)
    crf.shared_attention(ctx, batch, b.groups, b.q, b.pool, 1, guard[4:-4])
    torch.cuda.synchronize()
    assert ctx.device_errors() == 2
    assert (guard[:4] == 7.0).all() and (guard[-4:] == 7.0).all()
    _check(b, "after", ctx=ctx)


@pytest.mark.parametrize("dtype,page", [(BF, 16), (F32, 8), (BF, 5)])
@pytest.mark.parametrize("odd", [math.nan, math.inf])
def test_values_that_are_no_numbers(dtype, page, odd):
    """Unseen ones change nothing; one in a sequence's own keys counts in its rows alone, one in the shared ones in all
    of the group's."""
    from tests.paged import context
    print(f"[case] shared no numbers {dtype} page {page} {odd}", flush=True)
    b = Grouped([(100, [(2, 30), (1, 7), (3, 0)]), (40, [(1, 9), (1, 0)])], 4, 2, 64, dtype, page=page, seed=19)
    ctx = context(4, 2, 64, dtype)
    want, _ = _run(b, ctx)
    used = torch.zeros(b.n_pages, page, dtype=torch.bool, device="cuda")
    for s in range(len(b.new)):
        pg, sl = b.places(s)
        used[pg, sl] = True
    for pool in (b.k_pool, b.v_pool):
        pool[1].permute(0, 2, 1, 3)[~used] = odd
    out, _ = _run(b, ctx)
    assert torch.equal(out, want)
    hit = torch.zeros_like(out, dtype=torch.bool)
    for s, key, rows in ((0, 110, slice(1, 2)), (3, 20, slice(6, 8))):
        if s == 0:
            key = b.total[0] - 1  # its last token: the second of its two new ones sees it
        pg, sl = b.places(s, torch.tensor([key]))
        b.v_pool[1, pg, 1, sl, 33] = odd
        hit[rows, 2:, 33] = True
    out, _ = _run(b, ctx)
    assert torch.equal(out[~hit], want[~hit]) and not torch.isfinite(out[hit]).any()
    assert ctx.device_errors() == 0


def test_pages_out_of_range():
    from tests.paged import assert_within, context
    from tests.serving import masked_reference
    print("[case] shared, bad pages", flush=True)
    b = Grouped([(160, [(1, 30), (4, 9), (1, 0)])], 12, 2, 128, BF, seed=21)
    b.tables[0, 3] = -1            # of the shared pages, as the first sequence names them
    b.tables[1, 10] = b.n_pages    # the second one's own tokens 160 .. 172
    ctx = context(12, 2, 128, BF)
    out, _ = _run(b, ctx)
    assert ctx.device_errors() == 1

    def seen(s, pos, key):
        bad = (key // 16 == 3) | ((key // 16 == 10) if s == 1 else key < 0)
        return (key <= pos) & ~bad
    ref, _, bo, _ = masked_reference(b, seen)
    assert_within(out, ref, bo, "bad pages")


@pytest.mark.parametrize("dtype", [BF, F32])
def test_strides_in_place_and_captured(dtype):
    """Queries and outputs as slices of wider rows, in place; captured once and replayed with other lengths and groups."""
    import paper_2609_30884_amd as crf
    from tests.paged import assert_within, context
    from tests.serving import masked_reference, sink_mask
    print(f"[case] shared captured {dtype}", flush=True)
    b = Grouped([(96, [(1, 30)] * 5), (64, [(1, 11), (1, 2)])], 4, 2, 64, dtype, seed=23)
    ctx = context(4, 2, 64, dtype)
    wide = torch.zeros(b.n_rows, 256 + 16, dtype=dtype, device="cuda")
    q = b.q.reshape(b.n_rows, 256)

    def step():
        wide[:, :256].copy_(q)
        crf.shared_attention(ctx, b.batch, b.groups, wide[:, :256], b.pool, 1, wide[:, :256])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, (start, shared, shorter) in enumerate([([0, 5, 7], [96, 64], 0), ([0, 3, 5], [96, 96], 1), ([1, 5, 7], [32, 0], 2),
                                                  ([0, 5, 7], [80, 64], 3)]):
        b.seq_start.copy_(_i32(start))
        b.shared.copy_(_i32(shared))
        b.total = [t - shorter if j % 2 else t for j, t in enumerate([127] * 5 + [76, 67])]
        b.length.copy_(_i32(b.total))
        q.copy_(torch.randn(q.shape, generator=b.gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = wide.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, wide)
        ref, _, bo, _ = masked_reference(b, sink_mask(0, 0))
        assert_within(got[:, :256].unflatten(1, (4, 64)), ref, bo, f"replay {i}")
    assert ctx.device_errors() == 0

"""crf_paged_attention with values that are no finite numbers: keys that a row does
not see leave its result as it is to the bit, and keys that it sees count however
little they weigh."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = "bf16", "f32"


def _dt(name):
    return torch.bfloat16 if name == BF else torch.float32


def _run(b, ctx):
    import paper_2609_30884_amd as crf
    out = torch.full((b.n_rows, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda")
    lse = torch.full((b.n_rows, b.nq), 7.0, dtype=torch.float32, device="cuda")
    crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out, lse=lse)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 0
    return out, lse


# (new tokens, cached ones): steps and drafts, whose keys the waves share out, and chunks of
# tiles of 128 rows; prefixes long enough that a row's scores pass 2^4 and 2^16 of its first ones
SEEN = [
    (BF, 128, 12, 2, 16, [(3, 1500), (1, 700)], 1), (BF, 64, 8, 2, 7, [(8, 2100)], 4),
    (F32, 64, 4, 2, 16, [(6, 1200)], 2), (F32, 128, 3, 1, 16, [(9, 1100)], 5),
    (BF, 128, 12, 2, 16, [(150, 1500), (60, 900)], 90), (BF, 64, 12, 2, 1, [(260, 1100)], 200),
    (BF, 128, 28, 4, 16, [(400, 3000)], 333), (F32, 64, 4, 2, 16, [(300, 1600)], 140),
    (F32, 128, 4, 2, 16, [(200, 1800)], 150),
]


@pytest.mark.parametrize("dtype,hd,nq,nkv,page,seqs,first", SEEN)
@pytest.mark.parametrize("scale", [2.0, 4.0])
def test_rows_before_a_key_are_as_without_it(dtype, hd, nq, nkv, page, seqs, first, scale):
    """Token `first` of sequence 0's new ones is no number, in K, V or both: the rows before it keep every bit."""
    from tests.paged import Batch, context
    print(f"[case] unseen {dtype} hd {hd} heads {nq}/{nkv} {seqs} queries x {scale}", flush=True)
    b = Batch(seqs, nq, nkv, hd, _dt(dtype), page=page, seed=41)
    b.q.mul_(scale)
    ctx = context(nq, nkv, hd, b.dtype)
    clean, clean_lse = _run(b, ctx)
    pg, sl = b.places(0, torch.tensor([seqs[0][1] + first]))
    keep = torch.ones(b.n_rows, dtype=torch.bool, device="cuda")
    keep[first:seqs[0][0]] = False
    pools = [b.k_pool.clone(), b.v_pool.clone()]
    for odd in (math.nan, math.inf, -math.inf):
        for which in ("k", "v", "some of v"):
            if which == "k":
                b.k_pool[1, pg, :, sl] = odd
            elif which == "v":
                b.v_pool[1, pg, :, sl] = odd
            else:
                b.v_pool[1, pg, 0, sl, 5::7] = odd
            got, lse = _run(b, ctx)
            assert torch.equal(got[keep], clean[keep]), (odd, which)
            assert torch.equal(lse[keep], clean_lse[keep]), (odd, which)
            b.k_pool.copy_(pools[0])
            b.v_pool.copy_(pools[1])


@pytest.mark.parametrize("dtype,hd,nq,seqs", [
    (BF, 128, 12, [(2, 900), (1, 40)]), (BF, 64, 4, [(4, 2500)]), (F32, 64, 4, [(2, 1500)]), (F32, 128, 4, [(3, 500)]),
    (BF, 128, 12, [(60, 900), (150, 30)]), (BF, 64, 4, [(100, 2500)]), (F32, 64, 4, [(90, 1500)]),
    (F32, 128, 4, [(70, 1500)])])
@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("order", ["before", "after"])
def test_values_that_weigh_next_to_nothing(dtype, hd, nq, seqs, odd, order):
    """A value at a key that is seen counts, also where its weight is e^-400, which no fp32 holds: at the head of a
    prefix, whose later keys raise the reference, and at its end, in a block of keys that outweigh it."""
    from tests.paged import Batch, assert_within, attention_reference, context
    print(f"[case] weightless {dtype} hd {hd} {seqs} {odd} {order}", flush=True)
    b = Batch(seqs, nq, 2, hd, _dt(dtype), seed=43)
    b.q.fill_(1.0)
    b.k_pool.mul_(0.1)
    low = -400.0 / math.sqrt(hd)  # of every element of a key: a score of -400
    for s, (n, t) in enumerate(zip(b.new, b.total)):
        if order == "before":  # blocks of nothing but such keys, of long prefixes whole parts
            lows, odds = range(t // 2 if t >= 1400 else min(32, t - n)), [0, 20]
        else:
            lows = odds = [t - n - 1]
        pg, sl = b.places(s, torch.tensor(list(lows)))
        b.k_pool[1, pg, :, sl] = low
        pg, sl = b.places(s, torch.tensor(odds))
        b.v_pool[1, pg, :, sl, 3::5] = odd
    ctx = context(nq, 2, hd, b.dtype)
    out, lse = _run(b, ctx)
    ref, rl, bo, bl = attention_reference(b)
    assert not torch.isfinite(ref).all() and torch.isfinite(ref).any()
    assert_within(out, ref, bo, "weightless")
    assert_within(lse, rl, bl, "weightless lse")


@pytest.mark.parametrize("dtype,hd,heads", [(BF, 64, 8), (F32, 64, 4)])
def test_bad_pages_of_unit_after_unit(dtype, hd, heads):
    """Units dealt out whole, several to a workgroup, taken twice for values that are no numbers, some with pages out of
    range: what one finds out about its pages is not the next one's."""
    from tests.paged import Batch, assert_within, attention_reference, context
    print(f"[case] bad pages of units {dtype}", flush=True)
    b = Batch([(130 + s % 3, 20 + 7 * (s % 5)) for s in range(260)], heads, heads, hd, _dt(dtype), seed=47)
    bad, gone = b.tables.clone(), {}
    for s in range(260):
        pg, sl = b.places(s, torch.tensor([5, 100]))
        b.v_pool[1, pg, :, sl, s % 3::11] = math.inf
        gone[s] = [[], [2], [0, 9], []][s % 4]
        for j in gone[s]:
            bad[s, j] = (-1, b.n_pages)[s % 2]
    b.tables.copy_(bad)

    def hidden(s):
        page = torch.arange(b.total[s], device="cuda") // b.page
        return (page[:, None] == torch.tensor(gone[s] or [-1], device="cuda")).any(1)

    import paper_2609_30884_amd as crf
    ctx = context(heads, heads, hd, b.dtype)
    out = torch.zeros(b.n_rows, heads, hd, dtype=b.dtype, device="cuda")
    for _ in range(3):
        crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 1
    ref, _, bound, _ = attention_reference(b, hidden=hidden)
    assert_within(out, ref, bound, "units")

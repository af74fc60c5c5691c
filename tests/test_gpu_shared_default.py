"""crf_shared_attention of a batch whose caller does not bound the new tokens
(max_new 0): the same kernels, to the bit, as with the bound that it could give."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _both(groups, nq, nkv, hd, dtype, alone, pad, bound):
    """With max_new `bound` and 0, and crf_paged_attention's."""
    import paper_2609_30884_amd as crf
    from tests.paged import context
    from tests.test_gpu_shared_attention import Grouped, _check
    ctx, got = context(nq, nkv, hd, dtype), []
    for most in (bound, 0):
        b = Grouped(groups, nq, nkv, hd, dtype, alone=alone, seed=51, pad=pad, max_new=most)
        got.append(_check(b, f"max_new {most}", ctx=ctx)[:2])
    out, lse = torch.full_like(got[0][0], 7.0), torch.full_like(got[0][1], 7.0)
    crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out, lse=lse)
    torch.cuda.synchronize()
    return *got, (out, lse)


@pytest.mark.parametrize("dtype,nq,nkv,hd", [(BF, 28, 4, 128), (BF, 12, 2, 64), (F32, 8, 2, 64)])
@pytest.mark.parametrize("new", [1, 2])
def test_short_sequences(dtype, nq, nkv, hd, new):
    print(f"[case] shared default {dtype} {nq}/{nkv} of {hd}, {new} tokens", flush=True)
    groups = [(300, [(new, 7 * i) for i in range(40)]), (200, [(new, 60 + i) for i in range(30)])]
    given, default, plain = _both(groups, nq, nkv, hd, dtype, [(new, 90)], 0, new)
    assert all(torch.equal(a, b) for a, b in zip(given, default))
    assert not torch.equal(default[0], plain[0])  # (joined from other parts, in other last bits)


def test_what_may_be_long():
    """More than two tokens a sequence on average, of which one may have nearly all."""
    print("[case] shared default, long", flush=True)
    groups = [(300, [(3, 7 * i) for i in range(30)])]
    given, default, plain = _both(groups, 12, 2, 64, BF, [(200, 90)], 3, 200)
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(given, default, plain))


@pytest.mark.parametrize("dtype,nq,nkv,hd,page", [(BF, 28, 4, 128, 16), (BF, 12, 2, 64, 7), (F32, 8, 2, 64, 16),
                                                  (F32, 4, 4, 128, 16)])
def test_chunks_among_single_tokens(dtype, nq, nkv, hd, page):
    """Not bounded, and short on average: chunks of several tiles of rows in a group and alone, some begun within what is
    shared."""
    import paper_2609_30884_amd as crf
    from tests.paged import context
    from tests.test_gpu_shared_attention import Grouped, _check, _run
    print(f"[case] shared default, chunks {dtype} {nq}/{nkv} of {hd}", flush=True)
    ctx = context(nq, nkv, hd, dtype)
    singles = [(1, 5 * i) for i in range(60)]
    groups = [(300, singles + [(43, 31)]), (77, [(25, 0)] + singles[:50]), (500, [(1, 2), (1, 0), (0, 40)])]
    b = Grouped(groups, nq, nkv, hd, dtype, ahead=[(20, 0)], alone=[(33, 700), (1, 90)], page=page, seed=53, pad=2,
                max_new=0)
    assert b.n_rows > 1.5 * len(b.new) and b.n_rows <= 2 * len(b.new)
    out, lse, _ = _check(b, "chunks", ctx=ctx)
    plain = torch.full_like(out, 7.0)
    crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, plain)
    torch.cuda.synchronize()
    assert not torch.equal(out, plain)
    again = _run(b, ctx)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    # the second group shares 100 tokens, which most of its members do not reach
    b.shared.copy_(torch.tensor([300, 100, 500], dtype=torch.int32))
    first = b.tables_h[b.seq_start[1].item()]
    for s in range(b.seq_start[1].item() + 1, b.seq_start[2].item()):
        for p in range(77 // page, -(-100 // page)):
            lo, hi = max(77, p * page), min(100, (p + 1) * page, b.total[s])
            if lo < hi and p < -(-b.total[s] // page):
                for pool in (b.k_pool, b.v_pool):
                    pool[1, int(b.tables_h[s, p]), :, lo - p * page:hi - p * page] = \
                        pool[1, int(first[p]), :, lo - p * page:hi - p * page]
    _check(b, "shared past a member's own", ctx=ctx)

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

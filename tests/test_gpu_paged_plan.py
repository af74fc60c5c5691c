"""How crf_paged_attention's launches are planned, by results: windows that no
sequence reaches."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _run(b, ctx, window=0):
    import paper_2609_30884_amd as crf
    out = torch.full((b.n_rows, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda")
    lse = torch.full((b.n_rows, b.nq), 7.0, dtype=torch.float32, device="cuda")
    crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out, lse=lse, window=window)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 0
    return out, lse


@pytest.mark.parametrize("dtype,hd,nq,nkv,seqs", [
    (torch.bfloat16, 128, 12, 2, [(200, 8003), (40, 700)]), (torch.bfloat16, 64, 12, 2, [(1, 9000), (3, 20)]),
    (torch.float32, 64, 4, 2, [(150, 4000)])])
def test_windows_that_no_sequence_reaches(dtype, hd, nq, nkv, seqs):
    """They are no window: the same bits, from the same plan, up to the largest int."""
    from tests.paged import Batch, context
    print(f"[case] wide windows {dtype} {seqs}", flush=True)
    b = Batch(seqs, nq, nkv, hd, dtype, seed=51)
    ctx = context(nq, nkv, hd, dtype)
    none = _run(b, ctx)
    for window in (max(b.total), 1 << 30, (1 << 31) - 129, (1 << 31) - 100, (1 << 31) - 1):
        got = _run(b, ctx, window)
        assert torch.equal(got[0], none[0]) and torch.equal(got[1], none[1]), window

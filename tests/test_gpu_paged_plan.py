"""How crf_paged_attention's launches are planned, by results: windows that no
sequence reaches, and launches of more workgroups than stay resident."""
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


@pytest.mark.parametrize("nq,nkv,hd,seqs,pad,window", [
    (32, 8, 64, [(4000, 10), (3500, 0)], 0, 0),        # 1888 row tiles as the launch counts them, 512 resident workgroups
    (32, 8, 64, [(4000, 10), (3500, 0)], 0, 700),
    (28, 4, 128, [(7200, 100)], 3, 0),                 # 1576, 504
    (12, 2, 128, [(200, 8003), (40, 6000)], 17000, 0),  # 1620 with the rows of nobody; 24 real units, which are split
    (12, 2, 64, [(130, 5000), (1, 9000), (0, 7)], 19000, 2500),
])
def test_more_workgroups_than_stay_resident(nq, nkv, hd, seqs, pad, window):
    """From three row tiles to a resident workgroup on, a launch has a workgroup to each row tile: whole units, one
    each, or, where the device finds few units, stretches to as many workgroups as before and nothing to the others."""
    from tests.paged import Batch, assert_within, attention_reference, context
    print(f"[case] wide launches {nq}/{nkv} x {hd} {seqs} and {pad} rows of nobody, window {window}", flush=True)
    b = Batch(seqs, nq, nkv, hd, torch.bfloat16, seed=53, pad=pad)
    g, slots = nq // nkv, 512 if hd == 64 else 504
    assert (b.n_rows * g // 128 + len(seqs)) * nkv >= 3 * slots
    ctx = context(nq, nkv, hd, torch.bfloat16)
    out, lse = _run(b, ctx, window)
    ref, rl, bo, bl = attention_reference(b, window=window)
    n = b.rows
    assert_within(out[:n], ref[:n], bo[:n], "wide")
    assert_within(lse[:n], rl[:n], bl[:n], "wide lse")
    assert (out[n:] == 7.0).all() and (lse[n:] == 7.0).all()
    again = _run(b, ctx, window)
    assert torch.equal(again[0], out) and torch.equal(again[1], lse)

"""crf_shared_attention: the positions of a tile's tokens are those of the item's own
sequences, whatever row starts others have (batches whose row starts descend)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype,n,back,nq,nkv,hd,page", [(BF, 100, 50, 12, 2, 128, 16), (BF, 400, 30, 4, 2, 64, 7),
                                                         (F32, 100, 70, 4, 2, 64, 16)])
def test_a_row_that_two_sequences_claim_is_the_last_ones(dtype, n, back, nq, nkv, hd, page):
    """The same to the bit each time, and right: not up to the position that the other one's token has."""
    from tests.paged import context
    from tests.test_gpu_shared_contradictions import Claims
    print(f"[case] shared positions {dtype} {n} from {back}", flush=True)
    c, ctx = Claims(n, back, nq, nkv, hd, dtype, page), context(nq, nkv, hd, dtype)
    out, lse = c.run(ctx)
    c.check(out, lse, list(c.owner), "all rows")
    for _ in range(3):
        again = c.run(ctx)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_rows_that_one_sequence_goes_back_to():
    """A group of more sequences than a workgroup has threads goes back to rows whose first claimants contradict the batch
    (no token): the later ones alone have them, and see what the group shares."""
    import paper_2609_30884_amd as crf
    from tests.paged import assert_within, context
    from tests.serving import masked_reference, sink_mask
    from tests.test_gpu_shared_attention import Grouped, _i32
    print("[case] shared positions gone back", flush=True)
    ctx = context(4, 2, 64, BF)
    # sequences 0 .. 399 on rows 0 .. 399, 400 descends to row 100, 401 .. 600 on rows 100 .. 299
    b = Grouped([(96, [(1, 7 + s % 50) for s in range(601)])], 4, 2, 64, BF, seed=43)
    starts = list(range(401)) + list(range(100, 301))
    gone = range(100, 128)
    q = torch.randn(403, 4, 64, generator=b.gen, device="cuda").to(BF)
    for s in range(601):
        b.q[s] = q[starts[s]]
    want, _, bo, _ = masked_reference(b, sink_mask(0, 0))
    length, row_start = _i32([t if s not in gone else 0 for s, t in enumerate(b.total)]), _i32(starts)
    batch = crf.seq_batch(row_start, length, b.tables, 403, 1)
    out = torch.full((403, 4, 64), 7.0, dtype=BF, device="cuda")
    crf.shared_attention(ctx, batch, b.groups, q, b.pool, 1, out)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 2 and (out[400:] == 7.0).all()
    owner = {r: r for r in range(400)} | {100 + i: 401 + i for i in range(200)}
    seqs = [owner[r] for r in range(400)]
    assert_within(out[:400], want[seqs], bo[seqs], "gone back")

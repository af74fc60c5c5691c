"""crf_rope_append and crf_norm_rope_append of batches whose row starts descend, so that
two sequences claim a row: flagged; the row is one of theirs, at its own position and
on its own pages, and no other slot is written."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


# (past 2048 rows a workgroup takes four tokens)
@pytest.mark.parametrize("dtype,n,back", [(BF, 100, 50), (F32, 100, 20), (BF, 1500, 700)])
@pytest.mark.parametrize("norm", [False, True])
def test_rows_that_two_sequences_claim(dtype, n, back, norm):
    import paper_2609_30884_amd as crf
    from tests.paged import context
    print(f"[case] append claims {dtype} {n} from {back} norm {norm}", flush=True)
    page, nq, nkv, hd = 4, 4, 2, 64
    ctx, rope = context(nq, nkv, hd, dtype), crf.rope(hd, 1e4)
    g = torch.Generator().manual_seed(n + back)
    starts = list(range(n + 1)) + list(range(back, back + n + 1))  # sequence n descends
    seqs, rows = 2 * n + 1, back + n
    claims = [[s for s in range(seqs) if starts[s] == r and starts[s + 1] > r] for r in range(rows)]
    length = torch.randint(1, 33, (seqs,), generator=g).int()
    # every entry names a page; a sequence's are its own, those behind them some that nobody has
    tables = torch.arange(8 * seqs, dtype=torch.int32).view(seqs, 8)
    rand = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()  # noqa: E731
    q, k, v, gain = rand(rows + 2, nq, hd), rand(rows + 2, nkv, hd), rand(rows + 2, nkv, hd), rand(hd)

    def call(row_start, length, tables, flags):
        pools = [torch.full((1, 8 * seqs, nkv, page, hd), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
        pool = crf.page_pool(*pools, page)
        out = torch.full_like(q, 7.0)
        held = [torch.tensor(row_start, dtype=torch.int32).cuda(), length.cuda(), tables.cuda()]
        batch = crf.seq_batch(*held, rows + 2, 1)
        if norm:
            crf.norm_rope_append(ctx, rope, batch, q, k, v, gain, gain, pool, 0, out)
        else:
            crf.rope_append(ctx, rope, batch, q, k, v, pool, 0, out)
        torch.cuda.synchronize()
        assert ctx.device_errors() == flags
        return [out, *pools]
    def alone(whose):  # as a batch of these sequences, a row each
        out, *pools = call(list(range(rows + 1)), length[whose], tables[whose], 0)
        at = length[whose].long() - 1
        pages = tables[whose].long()[torch.arange(rows), at // page]
        return out, [p[0, pages, :, at % page] for p in pools], pages, at % page
    first, last = alone([c[0] for c in claims]), alone([c[-1] for c in claims])
    assert any(len(c) == 2 for c in claims)
    for _ in range(3):
        out, *pools = call(starts, length, tables, 2)
        written = torch.zeros(8 * seqs, page, dtype=torch.bool)
        for r in range(rows):
            fits = False
            for o, kv, pages, slots in (first, last):
                got = [p[0, pages[r], :, slots[r]] for p in pools]
                if torch.equal(out[r], o[r]) and all(torch.equal(a, b[r]) for a, b in zip(got, kv)):
                    fits = True
                    written[pages[r], slots[r]] = True
                    break
            assert fits, f"row {r}"
        assert (out[rows:] == 7.0).all()
        for p in pools:
            assert (p[0].permute(0, 2, 1, 3)[~written] == 7.0).all()

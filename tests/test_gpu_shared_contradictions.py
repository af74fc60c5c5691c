"""crf_shared_attention of batches whose row starts descend, so that several sequences
claim a row: flagged, inside their parts, and every row right that one of them has."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


class Claims:
    """n sequences of one token on rows 0 .. n-1, a sequence whose rows descend, and n more on rows back .. back+n-1; the
    first and the last third of them share a prompt.  want(s): row s of the attention of sequence s by itself."""

    def __init__(self, n, back, nq, nkv, hd, dtype, page):
        import paper_2609_30884_amd as crf
        from tests.serving import masked_reference, sink_mask
        from tests.test_gpu_shared_attention import Grouped, _i32
        third = (2 * n + 1) // 3
        own = lambda s: 20 + (53 * s) % 380  # noqa: E731
        b = Grouped([(64, [(1, own(s)) for s in range(third)]), (0, [(1, own(s)) for s in range(third, 2 * n + 1 - third)]),
                     (48, [(1, own(s)) for s in range(third)])], nq, nkv, hd, dtype, page=page, seed=41)
        starts = list(range(n + 1)) + list(range(back, back + n + 1))
        self.rows, self.owner = back + n, {}
        for s in range(2 * n + 1):
            if starts[s + 1] > starts[s]:
                self.owner.setdefault(starts[s], []).append(s)
        self.n_rows = self.rows + 3
        q = torch.randn(self.n_rows, nq, hd, generator=b.gen, device="cuda").to(dtype)
        for s in range(2 * n + 1):
            b.q[s] = q[starts[s]]
        self.b, self.q, self.starts = b, q, _i32(starts)
        self.batch = crf.seq_batch(self.starts, b.length, b.tables, self.n_rows, 1)
        self.want = masked_reference(b, sink_mask(0, 0))

    def run(self, ctx):
        import paper_2609_30884_amd as crf
        b = self.b
        out = torch.full((self.n_rows, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda")
        lse = torch.full((self.n_rows, b.nq), 7.0, device="cuda")
        crf.shared_attention(ctx, self.batch, b.groups, self.q, b.pool, 1, out, lse=lse)
        torch.cuda.synchronize()
        assert ctx.device_errors() == 2
        assert (out[self.rows:] == 7.0).all() and (lse[self.rows:] == 7.0).all()
        return out, lse

    def check(self, out, lse, rows, what):
        """Those rows are those of the last sequence that claims them."""
        from tests.paged import assert_within
        seqs = [self.owner[r][-1] for r in rows]
        ref, rl, bo, bl = (x[seqs] for x in self.want)
        assert_within(out[rows], ref, bo, what)
        assert_within(lse[rows], rl, bl, what + " lse")


@pytest.mark.parametrize("dtype,n,back,nq,nkv,hd,page", [(BF, 100, 50, 12, 2, 128, 16), (BF, 400, 30, 4, 2, 64, 7),
                                                         (F32, 100, 70, 4, 2, 64, 16)])
def test_rows_that_two_sequences_claim(dtype, n, back, nq, nkv, hd, page):
    """The two lie in different waves of the workgroup that looks for a row's parts: it takes one's, not a mixture."""
    from tests.paged import context
    print(f"[case] shared claims {dtype} {n} from {back}", flush=True)
    c, ctx = Claims(n, back, nq, nkv, hd, dtype, page), context(nq, nkv, hd, dtype)
    for _ in range(3):
        out, lse = c.run(ctx)
        c.check(out, lse, [r for r in c.owner if len(c.owner[r]) == 1], "one claim")
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()

"""Shared by the tests of the operators over a page pool: ragged batches on
shuffled pages, and plain references in 64 bits with their error bounds."""
import math

import torch

import paper_2609_30884_amd as crf

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # half a step, relative


def context(nq, nkv, hd, dtype, layers=2):
    if dtype == torch.bfloat16:
        d, f = 128, 64
    else:
        d, f = 64, 64
    return crf.Context(crf.make_dims(layers, d, nq, nkv, hd, f, dtype="bf16" if dtype == torch.bfloat16 else "f32"),
                       1, 0)


class Batch:
    """Sequences of (new tokens, cached tokens) with their pages shuffled over pools of two layers."""

    def __init__(self, seqs, nq, nkv, hd, dtype, page=16, seed=0, pad=0, spare=3, fill=None, max_new=None, wide=0):
        g = torch.Generator().manual_seed(seed)
        self.new = [n for n, _ in seqs]
        self.total = [n + c for n, c in seqs]
        self.nq, self.nkv, self.hd, self.dtype, self.page = nq, nkv, hd, dtype, page
        need = [-(-t // page) for t in self.total]
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g)
        # entries past a sequence's pages are never to be read
        self.tables_h = torch.full((len(seqs), max(max(need), 1) + wide), 1 << 30, dtype=torch.int32)
        at = 0
        for s, k in enumerate(need):
            self.tables_h[s, :k] = order[at:at + k].int()
            at += k
        self.starts = [0]
        for n in self.new:
            self.starts.append(self.starts[-1] + n)
        self.rows = self.starts[-1]
        self.n_rows = self.rows + pad
        self.row_start = torch.tensor(self.starts, dtype=torch.int32).cuda()
        self.length = torch.tensor(self.total, dtype=torch.int32).cuda()
        self.tables = self.tables_h.cuda()
        gen = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.gen = gen
        shape = (2, self.n_pages, nkv, page, hd)
        rand = lambda *sh: torch.randn(*sh, generator=gen, device="cuda").to(dtype)  # noqa: E731
        self.k_pool = rand(*shape) if fill is None else torch.full(shape, fill, dtype=dtype, device="cuda")
        self.v_pool = rand(*shape) if fill is None else torch.full(shape, fill, dtype=dtype, device="cuda")
        if fill is not None:  # numbers only where a sequence has tokens
            for s, t in enumerate(self.total):
                pg, sl = self.places(s)
                self.k_pool[1, pg, :, sl] = rand(t, nkv, hd)
                self.v_pool[1, pg, :, sl] = rand(t, nkv, hd)
        self.q = rand(max(self.n_rows, 1), nq, hd)[:self.n_rows]
        self.pool = crf.page_pool(self.k_pool, self.v_pool, page)
        self.batch = crf.seq_batch(self.row_start, self.length, self.tables, self.n_rows,
                                   max(self.new) if max_new is None else max_new)

    def places(self, s, tokens=None):
        j = torch.arange(self.total[s]) if tokens is None else tokens
        return self.tables_h[s].long()[j // self.page].cuda(), (j % self.page).cuda()

    def cached(self, s):
        pg, sl = self.places(s)
        return self.k_pool[1, pg, :, sl], self.v_pool[1, pg, :, sl]  # [tokens, nkv, hd]


def attention_reference(b: Batch, scale=None, window=0, hidden=None):
    """(out, lse, bound of out, bound of lse) in 64 bits; hidden(s): bool [tokens] of keys that nobody sees.

    Bounds: a score is a sum of hd products, off by (hd + 2) steps of 2^-24 of the
    sum of their magnitudes (the factor to log2 units included), a weight by that
    (twice: numerator and sum) and 2 steps of the exponential; the sums of n terms
    add n steps; then the weights' rounding to the storage type before the second
    product and the output's own rounding, in bf16 2^-8 each."""
    scale = scale or b.hd ** -0.5
    g = b.nq // b.nkv
    u32, u = 2.0 ** -24, U[b.dtype]
    out = torch.zeros(b.n_rows, b.nq, b.hd, dtype=torch.float64, device="cuda")
    lse = torch.full((b.n_rows, b.nq), -math.inf, dtype=torch.float64, device="cuda")
    bo, bl = torch.zeros_like(out), torch.zeros_like(lse)
    for s, (n, t) in enumerate(zip(b.new, b.total)):
        if n == 0:
            continue
        kk, vv = b.cached(s)
        kk, vv = kk.double().permute(1, 2, 0).contiguous(), vv.double().permute(1, 0, 2).contiguous()
        key = torch.arange(t, device="cuda")
        for r0 in range(0, n, 2048):
            r1 = min(n, r0 + 2048)
            pos = torch.arange(t - n + r0, t - n + r1, device="cuda")[:, None]
            seen = key <= pos
            if window:
                seen = seen & (key > pos - window)
            if hidden is not None:
                seen = seen & ~hidden(s)
            some = seen.any(1)
            rows = slice(b.starts[s] + r0, b.starts[s] + r1)
            for h in range(b.nq):
                q = b.q[rows, h].double()
                sc = torch.where(seen, scale * (q @ kk[h // g]), -math.inf)
                mag = scale * (q.abs() @ torch.where(torch.isfinite(kk[h // g]), kk[h // g].abs(), 0.0))
                delta = ((b.hd + 2) * u32 * torch.where(seen, mag, 0.0)).amax(1) + 4 * u32 * \
                    torch.where(seen, sc.abs(), 0.0).amax(1)
                m = torch.where(some, sc.amax(1), 0.0)
                p = (sc - m[:, None]).exp()
                z = p.sum(1)
                v = vv[h // g]
                w = p / torch.where(some, z, 1.0)[:, None]
                # (a value that is not a number counts where its key is seen)
                fine = torch.isfinite(v)
                out[rows, h] = w @ torch.where(fine, v, 0.0)
                mean = w @ torch.where(fine, v.abs(), 0.0)
                if not bool(fine.all()):
                    odd = (~fine).any(1)
                    for j in torch.nonzero(odd).squeeze(1).tolist():
                        out[rows, h] += torch.where(seen[:, j, None] & ~fine[j], v[j], 0.0)
                rel = 2 * delta + (t + 4) * u32 + u * (1 if b.dtype == torch.bfloat16 else 0)
                bo[rows, h] = mean * (rel[:, None] + u) * (1 + 2.0 ** -6)
                lse[rows, h] = torch.where(some, m + z.log(), -math.inf)
                bl[rows, h] = delta + (t + 4) * u32 + 4 * u32 * torch.where(some, lse[rows, h].abs(), 0.0)
    return out, lse, bo, bl


def assert_within(got, ref, bound, what):
    """Element by element, non-finite values equal."""
    got = got.double()
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), fine), f"{what}: finite elsewhere"
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN elsewhere"
    assert torch.equal(got[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)]), f"{what}: infinities"
    err = torch.where(fine, (got - ref).abs() - bound, torch.zeros_like(ref))
    worst = float(err.max()) if err.numel() else 0.0
    share = float((torch.where(fine, (got - ref).abs(), 0.0) / bound.clamp(min=1e-300)).max()) if err.numel() else 0.0
    print(f"[{what}] largest error {share:.3f} of its bound", flush=True)
    assert worst <= 0.0, f"{what}: {worst:.3e} over its bound"

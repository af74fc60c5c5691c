"""The operators over a page pool together, as a server uses them: sequences grow,
their tokens are appended and attended to, they branch, leave, and the pool is
compacted; step by step and as captured steps."""
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LAYERS = 2


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Cache:
    """A pool with its map, and what each sequence's tokens were given, in the order of the tokens."""

    def __init__(self, n_seqs, n_pages, width, dtype, nq, nkv, hd, page, max_rows):
        import paper_2609_30884_amd as crf
        from tests.paged import context
        self.crf, self.nq, self.nkv, self.hd, self.dtype, self.page = crf, nq, nkv, hd, dtype, page
        self.ctx = context(nq, nkv, hd, dtype, layers=LAYERS)
        self.k, self.v = (torch.zeros(LAYERS, n_pages, nkv, page, hd, dtype=dtype, device="cuda") for _ in range(2))
        self.refs, self.lengths = _i32([0] * n_pages), _i32([0] * n_seqs)
        self.tables = torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
        self.map = crf.page_map(self.refs, self.tables, self.lengths, page)
        self.pool = crf.page_pool(self.k, self.v, page)
        self.rope = crf.rope(hd // 2, 1e4, "interleaved")
        # what a step reads and writes, in place
        self.n_new, self.row_start = _i32([0] * n_seqs), _i32([0] * (n_seqs + 1))
        rows = lambda heads: torch.zeros(max_rows, heads, hd, dtype=dtype, device="cuda")  # noqa: E731
        self.q_in, self.k_in, self.v_in = ([rows(n) for _ in range(LAYERS)] for n in (nq, nkv, nkv))
        self.q_rot, self.out = ([rows(nq) for _ in range(LAYERS)] for _ in range(2))
        self.batch = crf.seq_batch(self.row_start, self.lengths, self.tables, max_rows, max_rows)
        self.history = [[[] for _ in range(n_seqs)] for _ in range(LAYERS)]

    def feed(self, new, gen):
        self.new = new
        self.n_new.copy_(_i32(new))
        self.row_start.copy_(_i32([0] + list(itertools.accumulate(new))))
        for t in self.q_in + self.k_in + self.v_in:
            t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))

    def step(self):
        """One step of every layer: nothing but calls on the current stream."""
        self.crf.pages_extend(self.ctx, self.map, self.n_new)
        for l in range(LAYERS):
            self.crf.rope_append(self.ctx, self.rope, self.batch, self.q_in[l], self.k_in[l], self.v_in[l], self.pool, l,
                                 q_out=self.q_rot[l])
            self.crf.paged_attention(self.ctx, self.batch, self.q_rot[l], self.pool, l, self.out[l])

    def tokens(self, layer, s):
        n = int(self.lengths[s])
        j = torch.arange(n)
        pg, sl = self.tables[s].cpu().long()[j // self.page].cuda(), (j % self.page).cuda()
        return self.k[layer, pg, :, sl], self.v[layer, pg, :, sl]

    def record(self):
        for l in range(LAYERS):
            for s, n in enumerate(self.new):
                if n:
                    k, v = self.tokens(l, s)
                    self.history[l][s].append((k[-n:].clone(), v[-n:].clone()))

    def check(self):
        """Every token of every sequence is where the map says; attention over them is right."""
        from tests.paged import assert_within, attention_reference
        torch.cuda.synchronize()
        assert self.ctx.device_errors() == 0
        starts = self.row_start.tolist()
        for l in range(LAYERS):
            cached = [[torch.cat(p) for p in zip(*h)] if h else [self.k[0, 0].new_zeros(0, self.nkv, self.hd)] * 2
                      for h in self.history[l]]
            for s, kv in enumerate(cached):
                for got, want in zip(self.tokens(l, s), kv):
                    assert torch.equal(got, want), f"layer {l} sequence {s}"

            class Seen:
                new, total = self.new, [len(kv[0]) for kv in cached]
                nq, nkv, hd, dtype, q, n_rows = self.nq, self.nkv, self.hd, self.dtype, self.q_rot[l], len(self.q_rot[l])
            Seen.starts, Seen.cached = starts, staticmethod(cached.__getitem__)
            ref, _, bound, _ = attention_reference(Seen)
            n = starts[-1]
            assert_within(self.out[l][:n], ref[:n], bound[:n], f"layer {l}")

    def fork(self, parents, children):
        self.crf.pages_fork(self.ctx, self.pool, self.map, _i32(parents), _i32(children))
        for h in self.history:
            for a, b in zip(parents, children):
                h[b] = list(h[a])

    def free(self, seqs):
        self.crf.pages_free(self.ctx, self.map, _i32(seqs))
        for h in self.history:
            for s in seqs:
                h[s] = []

    def compact(self):
        remap, counts = torch.zeros_like(self.refs), _i32([0, 0])
        self.crf.pages_compact(self.ctx, self.pool, self.map, self.map, remap, counts)
        return counts


SHAPES = [(torch.bfloat16, 12, 2, 128, 16), (torch.bfloat16, 8, 8, 64, 8), (torch.float32, 4, 2, 64, 16),
          (torch.float32, 6, 1, 128, 5)]


@pytest.mark.parametrize("dtype,nq,nkv,hd,page", SHAPES)
def test_a_servers_life(dtype, nq, nkv, hd, page):
    print(f"[case] serving {dtype} {nq}/{nkv} x {hd} page {page}", flush=True)
    c = Cache(6, 1200 // page, 600 // page, dtype, nq, nkv, hd, page, 160)
    gen = torch.Generator(device="cuda").manual_seed(hd + page)

    def grow(*new):
        c.feed(list(new), gen)
        c.step()
        c.record()
        c.check()
    grow(37, 100, 0, 1, 0, 0)            # prompts
    grow(1, 1, 64, 1, 0, 0)              # steps beside a prompt
    c.fork([0, 2], [4, 5])
    for _ in range(3):
        grow(1, 1, 1, 1, 1, 1)
    c.fork([], [])
    c.free([1, 3])
    held = int((c.refs > 0).sum())
    assert c.compact().tolist()[0] == held
    grow(1, 0, 5, 0, 3, 1)               # a draft for some
    before = [t.clone() for t in c.out]
    # a layer's pages are saved, overwritten and brought back
    used = torch.nonzero(c.refs > 0).flatten().int()
    spare = [torch.zeros_like(c.k[:1, :len(used)]) for _ in range(2)]
    store, at = c.crf.page_pool(*spare, page), torch.arange(len(used), device="cuda", dtype=torch.int32)
    c.crf.pages_copy(c.ctx, c.pool, used, at, 1, 1, store, 0)
    c.k[1].fill_(1e4)
    c.v[1].fill_(-1.0)
    c.crf.pages_copy(c.ctx, store, at, used, 0, 1, c.pool, 1)
    c.crf.paged_attention(c.ctx, c.batch, c.q_rot[1], c.pool, 1, c.out[1])
    c.check()
    assert torch.equal(c.out[1], before[1])
    grow(1, 120, 1, 30, 1, 1)            # the freed ones again
    c.free([0, 1, 2, 3, 4, 5])
    assert c.compact().tolist() == [0, 0] and int(c.refs.abs().sum()) == 0


@pytest.mark.parametrize("dtype,nq,nkv,hd,page", SHAPES)
def test_captured_steps(dtype, nq, nkv, hd, page):
    """A step, a branch and a departure captured once and replayed, against the same calls made one by one."""
    print(f"[case] captured {dtype} {nq}/{nkv} x {hd} page {page}", flush=True)
    a, b = (Cache(6, 1200 // page, 600 // page, dtype, nq, nkv, hd, page, 24) for _ in range(2))
    gens = [torch.Generator(device="cuda").manual_seed(3) for _ in range(2)]
    lists = [[_i32([0, 2]), _i32([4, 5]), torch.zeros_like(x.refs), _i32([0, 0])] for x in (a, b)]

    def branch(x, v):
        x.crf.pages_fork(x.ctx, x.pool, x.map, v[0], v[1])

    def leave(x, v):
        x.crf.pages_free(x.ctx, x.map, v[1])
        x.crf.pages_compact(x.ctx, x.pool, x.map, x.map, v[2], v[3])
    for x, g in ((a, gens[0]), (b, gens[1])):
        x.feed([20, 0, 3, 0, 0, 0], g)
        x.step()
    torch.cuda.synchronize()
    graphs = []
    for call in (a.step, lambda: branch(a, lists[0]), lambda: leave(a, lists[0])):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call()

    def same(flags=0):
        torch.cuda.synchronize()
        for x, y in ((a.k, b.k), (a.v, b.v), (a.refs, b.refs), (a.tables, b.tables), (a.lengths, b.lengths),
                     *zip(a.out, b.out), *zip(a.q_rot, b.q_rot), *zip(lists[0], lists[1])):
            assert torch.equal(x, y)
        assert a.ctx.device_errors() == b.ctx.device_errors() == flags
    for i, new in enumerate([[1, 0, 1, 0, 0, 0], [1, 0, 1, 0, 1, 1], [1, 3, 1, 0, 7, 1], [0, 1, 5, 9, 1, 1]] * 2):
        if i % 2:
            taken = bool((b.lengths[4:] != 0).any())  # (such a child is skipped, and that is flagged)
            graphs[1].replay()
            branch(b, lists[1])
            same(2 if taken else 0)
        a.feed(new, gens[0])
        b.feed(new, gens[1])
        graphs[0].replay()
        b.step()
        same()
        if i % 2:
            graphs[2].replay()
            leave(b, lists[1])
            same()


def test_two_servers_at_once():
    """Two contexts, each on a stream of its own, at the same time: each as if alone."""
    print("[case] two servers", flush=True)
    out = []
    for together in (False, True):
        caches = [Cache(6, 300, 60, torch.bfloat16, 12, 2, 128, 16, 300) for _ in range(2)]
        streams = [torch.cuda.Stream() if together else torch.cuda.current_stream() for _ in caches]
        for i, c in enumerate(caches):
            c.feed([100, 50, 0, 150, 0, 0], torch.Generator(device="cuda").manual_seed(i))
        torch.cuda.synchronize()
        for _ in range(4):
            for c, s in zip(caches, streams):
                with torch.cuda.stream(s):
                    c.step()
                    c.crf.pages_fork(c.ctx, c.pool, c.map, c.n_new[4:5], c.row_start[1:2] * 0 + 4)
                    c.crf.pages_free(c.ctx, c.map, c.n_new[4:5] + 4)
        torch.cuda.synchronize()
        assert all(c.ctx.device_errors() == 0 for c in caches)
        out.append([[t.clone() for t in (c.k, c.v, c.refs, c.lengths, *c.out)] for c in caches])
    for x, y in zip(*out):
        assert all(torch.equal(p, q) for p, q in zip(x, y))

"""A server's step as it uses the operators together: documents are read, branches
forked from them, each step appends normed and rotated keys, attends (one layer over
the shared prefixes, one in a window with sinks), and the logits of its rows are
scored.  Step by step against 64 bits, captured and replayed, two servers at once."""
import itertools

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
LAYERS, WINDOW, SINKS, VOCAB, EPS = 2, 50, 5, 3001, 1e-6


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Server:
    """Two documents with branches: sequence 0 and its branches 1 .. 3, sequence 4 and its branches 5 .. 7; 8 alone."""

    def __init__(self, dtype, nq, nkv, hd, page, seed, max_rows=200):
        import paper_2609_30884_amd as crf
        from tests.paged import context
        self.crf, self.dtype, self.nq, self.nkv, self.hd, self.page = crf, dtype, nq, nkv, hd, page
        self.ctx, self.seqs = context(nq, nkv, hd, dtype, layers=LAYERS), 9
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        # tables so wide that a batch counts as a large one
        width = max(800 // page, (41 << 20) // (page * nkv * hd * 2 * (2 if dtype == BF else 4) * self.seqs) + 1)
        pages = 2400 // page
        self.k, self.v = (torch.zeros(LAYERS, pages, nkv, page, hd, dtype=dtype, device="cuda") for _ in range(2))
        self.refs, self.lengths = _i32([0] * pages), _i32([0] * self.seqs)
        self.tables = torch.full((self.seqs, width), -1, dtype=torch.int32, device="cuda")
        self.map, self.pool = crf.page_map(self.refs, self.tables, self.lengths, page), crf.page_pool(self.k, self.v, page)
        self.rope = crf.rope(hd, 1e4)
        self.n_new, self.row_start = _i32([0] * self.seqs), _i32([0] * (self.seqs + 1))
        self.seq_start, self.shared_len = _i32([0, 4, 8]), _i32([0, 0])
        self.groups = crf.seq_groups(self.seq_start, self.shared_len)
        self.batch = crf.seq_batch(self.row_start, self.lengths, self.tables, max_rows, 128 // (nq // nkv))
        rand = lambda *s: torch.randn(*s, generator=self.gen, device="cuda")  # noqa: E731
        self.gains = [(1 + 0.2 * rand(2, hd)).to(dtype) for _ in range(LAYERS)]
        self.head = (rand(nq * hd, VOCAB) * 0.05).to(dtype)
        rows = lambda h: torch.zeros(max_rows, h, hd, dtype=dtype, device="cuda")  # noqa: E731
        self.qkv = [[rows(h) for h in (nq, nkv, nkv)] for _ in range(LAYERS)]
        self.q, self.out = ([rows(nq) for _ in range(LAYERS)] for _ in range(2))
        self.logits = torch.zeros(max_rows, VOCAB, device="cuda")
        self.tokens = torch.zeros(max_rows, 1, dtype=torch.int32, device="cuda")
        f = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
        self.scores = dict(logprob=f(max_rows, 1), entropy=f(max_rows), lse=f(max_rows),
                           top_token=torch.zeros(max_rows, 4, dtype=torch.int32, device="cuda"), top_logprob=f(max_rows, 4))
        self.given = [[] for _ in range(self.seqs)]  # raw k and v of every token, by layer

    def feed(self, new):
        self.new = new
        self.n_new.copy_(_i32(new))
        self.row_start.copy_(_i32([0] + list(itertools.accumulate(new))))
        for t in itertools.chain(*self.qkv):
            t.copy_(torch.randn(t.shape, generator=self.gen, device="cuda") * 2)
        self.tokens.copy_(torch.randint(VOCAB, self.tokens.shape, generator=self.gen, device="cuda"))

    def step(self):
        """Nothing but calls on the current stream."""
        crf = self.crf
        crf.pages_extend(self.ctx, self.map, self.n_new)
        for l in range(LAYERS):
            crf.norm_rope_append(self.ctx, self.rope, self.batch, *self.qkv[l], *self.gains[l], self.pool, l, self.q[l])
            if l == 0:
                crf.shared_attention(self.ctx, self.batch, self.groups, self.q[l], self.pool, l, self.out[l])
            else:
                crf.sink_attention(self.ctx, self.batch, self.q[l], self.pool, l, self.out[l], WINDOW, SINKS)
        self.logits.copy_(self.out[1].flatten(1) @ self.head)
        crf.token_logprobs(self.ctx, self.logits, self.tokens, **self.scores)

    def record(self):
        starts = [0] + list(itertools.accumulate(self.new))
        for s, n in enumerate(self.new):
            for i in range(n):
                self.given[s].append([(self.qkv[l][1][starts[s] + i].clone(), self.qkv[l][2][starts[s] + i].clone())
                                      for l in range(LAYERS)])

    def check(self):
        from tests.paged import assert_within
        from tests.serving import masked_reference, normed, rotated, sink_mask
        torch.cuda.synchronize()
        assert self.ctx.device_errors() == 0
        starts = [0] + list(itertools.accumulate(self.new))
        n = starts[-1]
        freq = [1e4 ** (-2 * i / self.hd) for i in range(self.hd // 2)]
        assert [len(x) for x in self.given] == self.lengths.tolist()
        for l in range(LAYERS):
            cached = []
            for s in range(self.seqs):
                t = len(self.given[s])
                if not t:
                    cached.append((self.k[l, 0, :, :0].transpose(0, 1), self.v[l, 0, :, :0].transpose(0, 1)))
                    continue
                j = torch.arange(t)
                pg, sl = self.tables[s].cpu().long()[j // self.page].cuda(), (j % self.page).cuda()
                cached.append((self.k[l, pg, :, sl], self.v[l, pg, :, sl]))
                k, v = (torch.stack([x[l][i] for x in self.given[s]]) for i in range(2))
                ref, bound = rotated(*normed(k, self.gains[l][1], EPS), freq, j.cuda(), "half", self.dtype)
                assert_within(cached[-1][0], ref, bound, f"keys {l} {s}")
                assert torch.equal(cached[-1][1], v)

            class Seen:
                new, total = self.new, [len(x) for x in self.given]
                nq, nkv, hd, dtype, q, n_rows = self.nq, self.nkv, self.hd, self.dtype, self.q[l], len(self.q[l])
            Seen.starts, Seen.cached = starts, staticmethod(cached.__getitem__)
            ref, _, bound, _ = masked_reference(Seen, sink_mask(WINDOW if l else 0, SINKS))
            assert_within(self.out[l][:n], ref[:n], bound[:n], f"layer {l}")
        # (sums of 3001 terms, values below 100: 2^-16 of them is far above fp32's steps)
        z = self.logits.double()
        lp = torch.log_softmax(z, 1)
        got = self.scores
        assert torch.equal(got["top_token"], torch.sort(z, dim=1, descending=True, stable=True).indices[:, :4].int())
        for name, want in (("lse", torch.logsumexp(z, 1)), ("entropy", -(lp.exp() * lp).sum(1)),
                           ("logprob", lp.gather(1, self.tokens.long())),
                           ("top_logprob", lp.gather(1, got["top_token"].long()))):
            assert_within(got[name], want, 2.0 ** -16 * (1 + want.abs()), name)

    def branch(self):
        """The documents' branches, which share their full pages and a copy of the begun one."""
        self.crf.pages_fork(self.ctx, self.pool, self.map, _i32([0, 0, 0, 4, 4, 4]), _i32([1, 2, 3, 5, 6, 7]))
        for s in range(self.seqs - 1):
            if s % 4:
                self.given[s] = list(self.given[s - s % 4])
        self.shared_len.copy_(self.lengths[0:8:4])


SHAPES = [(BF, 12, 2, 128, 16), (BF, 8, 8, 64, 8), (F32, 4, 2, 64, 16), (F32, 6, 1, 128, 5)]


@pytest.mark.parametrize("dtype,nq,nkv,hd,page", SHAPES)
def test_documents_and_branches(dtype, nq, nkv, hd, page):
    print(f"[case] step {dtype} {nq}/{nkv} x {hd} page {page}", flush=True)
    c = Server(dtype, nq, nkv, hd, page, hd + page)

    def grow(*new):
        c.feed(list(new))
        c.step()
        c.record()
        c.check()
    for _ in range(8):  # the documents, in chunks
        grow(20, 0, 0, 0, 13, 0, 0, 0, 1)
    c.branch()
    grow(1, 1, 1, 1, 1, 1, 1, 1, 1)
    grow(0, 1, 4, 0, 0, 2, 0, 1, 3)      # drafts beside idle ones
    grow(1, 1, 1, 1, 1, 1, 1, 1, 0)


@pytest.mark.parametrize("dtype,nq,nkv,hd,page", SHAPES[:3])
def test_captured(dtype, nq, nkv, hd, page):
    """A step captured once and replayed over growing sequences, eager work between, against the same calls one by one."""
    print(f"[case] captured step {dtype} {nq}/{nkv} x {hd} page {page}", flush=True)
    a, b = (Server(dtype, nq, nkv, hd, page, 3, 60) for _ in range(2))
    for x in (a, b):
        x.feed([20, 0, 0, 0, 17, 0, 0, 0, 3])
        x.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    for i, new in enumerate([[15, 0, 0, 0, 9, 0, 0, 0, 1]] * 2 + [[1] * 9, [1, 0, 3, 1, 1, 1, 1, 5, 0], [1] * 9]):
        if i == 2:
            a.branch()
            b.branch()
        a.feed(new)
        b.feed(new)
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for x, y in ((a.k, b.k), (a.v, b.v), (a.lengths, b.lengths), *zip(a.out, b.out), (a.logits, b.logits),
                     *((a.scores[k], b.scores[k]) for k in a.scores)):
            assert torch.equal(x, y)
    assert a.ctx.device_errors() == b.ctx.device_errors() == 0


def test_two_servers_at_once():
    """Two contexts, each on a stream of its own: each as if alone."""
    print("[case] two servers' steps", flush=True)
    out = []
    for together in (False, True):
        servers = [Server(BF, 12, 2, 128, 16, i) for i in range(2)]
        streams = [torch.cuda.Stream() if together else torch.cuda.current_stream() for _ in servers]
        torch.cuda.synchronize()
        for i in range(6):
            for c, s in zip(servers, streams):
                with torch.cuda.stream(s):
                    c.feed([1] * 9 if i > 2 else [20, 0, 0, 0, 20, 0, 0, 0, 1])
                    c.step()
                    if i == 2:
                        c.branch()
        torch.cuda.synchronize()
        assert all(c.ctx.device_errors() == 0 for c in servers)
        out.append([[t.clone() for t in (c.k, c.v, *c.out, c.logits, *c.scores.values())] for c in servers])
    for x, y in zip(*out):
        assert all(torch.equal(p, q) for p, q in zip(x, y))

"""crf_token_logprobs against log-softmax in 64 bits: vocabularies and rows of every
alignment, rows shared out to many workgroups, ties, tokens ruled out, rows of no
numbers, orders that fill the lists of the most likely."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24


def _ctx():
    from tests.paged import context
    return context(2, 2, 64, BF)


def _call(ctx, z, tokens, top):
    import paper_2609_30884_amd as crf
    n = z.shape[0]
    f = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
    out = {"entropy": f(n), "lse": f(n)}
    if tokens is not None:
        out["logprob"] = f(*tokens.shape)
    if top:
        out["top_token"] = torch.full((n, top), -7, dtype=torch.int32, device="cuda")
        out["top_logprob"] = f(n, top)
    crf.token_logprobs(ctx, z, tokens, **out)
    torch.cuda.synchronize()
    return out


def _reference(z, tokens, top):
    """Values and bounds in 64 bits.  z - m is off by one step of 2^-24 of itself, the factor to log2 units by 2 and the
    exponential by 2 of its own: each weight is off by (3 |z - m| + 2) steps, weighted; sums of n terms add at most
    n / 256 + 40 (a thread's own, then trees of 6 + 2 + 6 and rescalings); the logarithm 2 of itself; the rest is roundings."""
    z = z.double()
    n, v = z.shape
    none = (z == -math.inf).all(1)
    odd = torch.isnan(z).any(1) | (z == math.inf).any(1)
    m = torch.where(none | odd, 0.0, z.amax(1))
    d = z - m[:, None]
    e = torch.where(d > -math.inf, d.exp(), 0.0)
    s = e.sum(1)
    ls = s.log()
    steps = v / 256 + 40
    dd = torch.where(e > 0, d, 0.0)
    spread = (e * (3 * dd.abs() + 2)).sum(1) / torch.where(none, 1.0, s) + steps
    b_ls = (spread + 3 * ls.abs()) * U32
    lse = torch.where(none, -math.inf, torch.where(odd, math.nan, m + ls))
    b_lse = b_ls + 2 * U32 * lse.abs()
    p = e / torch.where(none, 1.0, s)[:, None]
    ent = torch.where(none, 0.0, torch.where(odd, math.nan, ls - (p * dd).sum(1)))
    b_ent = 2 * b_ls + ((p * dd.abs() * (3 * dd.abs() + 4 + 2 * steps)).sum(1) + 3 * ent.abs()) * U32
    out, bound = {"lse": lse, "entropy": ent}, {"lse": b_lse, "entropy": b_ent}

    def log_p(x):
        lp = (x - m[:, None]) - ls[:, None]  # (64 bits do not hold lse next to a type's lowest value)
        lp = torch.where(none[:, None], -math.inf, torch.where(odd[:, None], math.nan, lp))
        return lp, b_ls[:, None] + U32 * ((x - m[:, None]).abs() + 2 * lp.abs())
    if tokens is not None:
        t = tokens.long().view(n, -1)
        lp, b = log_p(z.gather(1, t.clamp(0, v - 1)))
        lp = torch.where(t >= v, -math.inf, lp)
        out["logprob"], bound["logprob"] = (torch.where(t < 0, 0.0, x).view(tokens.shape) for x in (lp, b))
    if top:
        order = torch.where(torch.isnan(z), math.inf, z)
        # NaN above +inf, the lowest index among equals
        rank = torch.sort(torch.isnan(z).to(torch.int8), dim=1, descending=True, stable=True).indices
        first = torch.sort(order.gather(1, rank), dim=1, descending=True, stable=True).indices
        idx = rank.gather(1, first)[:, :top]
        out["top_token"] = idx.int()
        out["top_logprob"], bound["top_logprob"] = log_p(z.gather(1, idx))
    return out, bound


def _check(z, tokens, top, what, flags=0, ctx=None):
    from tests.paged import assert_within
    ctx = ctx or _ctx()
    got = _call(ctx, z, tokens, top)
    assert ctx.device_errors() == flags
    ref, bound = _reference(z, tokens, top)
    if top:
        assert torch.equal(got["top_token"], ref.pop("top_token")), what
    for name, r in ref.items():
        b = torch.where(torch.isfinite(r), bound[name], 0.0)
        assert_within(got[name], r, b, f"{what} {name}")
    return got


def _logits(rows, vocab, dtype, seed, pad=0, off=0, scale=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g, device="cuda") * scale
    flat = torch.full((rows * (vocab + pad) + off,), math.nan, dtype=dtype, device="cuda")
    view = torch.as_strided(flat, (rows, vocab), (vocab + pad, 1), off)
    view.copy_(z)
    tokens = torch.randint(-1, vocab, (rows, 3), generator=g, device="cuda").int()
    return view, tokens


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 63, 64, 65, 511, 1000, 2047, 2048, 2049, 4099, 32003])
def test_vocabularies(dtype, vocab):
    print(f"[case] logprobs {dtype} vocab {vocab}", flush=True)
    ctx = _ctx()
    for rows, pad, off, top in ((1, 0, 0, 1), (5, 0, 1, 5), (3, 1, 3, 32), (9, 13, 7, 0), (2, 0, 2, 20)):
        z, tokens = _logits(rows, vocab, dtype, vocab + rows, pad, off)
        _check(z, tokens, min(top, vocab), f"{rows} x {vocab} + {pad} at {off}", ctx=ctx)


@pytest.mark.parametrize("dtype,rows,vocab,top", [(F32, 1, 152064, 5), (BF, 1, 152064, 32), (BF, 64, 152064, 20),
                                                  (F32, 33, 152063, 1), (BF, 700, 40000, 8), (BF, 1500, 20001, 32),
                                                  (F32, 3, 1 << 20, 20), (BF, 2100, 3000, 0)])
def test_sizes(dtype, rows, vocab, top):
    print(f"[case] logprobs {dtype} {rows} x {vocab} top {top}", flush=True)
    z, tokens = _logits(rows, vocab, dtype, 3, pad=5)
    ctx = _ctx()
    first = _check(z, tokens[:, 0].contiguous(), top, "rows", ctx=ctx)
    for _ in range(3):  # the same to the bit
        again = _call(ctx, z, tokens[:, 0].contiguous(), top)
        assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("top", [1, 20, 32])
def test_orders_and_ties(dtype, top):
    """Ascending rows, where every element is among the largest so far; all equal; two values; signed zeros."""
    print(f"[case] logprobs orders {dtype} top {top}", flush=True)
    v = 30011
    up = torch.linspace(-20, 20, v, device="cuda")
    rows = [up, -up, torch.zeros(v, device="cuda"), (torch.arange(v, device="cuda") % 7 == 3).float(),
            torch.where(torch.arange(v, device="cuda") % 2 == 0, -0.0, 0.0), torch.round(up),
            torch.where(torch.arange(v, device="cuda") < 29000, -0.0, up), up.roll(5000)]
    z = torch.stack(rows).to(dtype)
    tokens = torch.tensor([[0, v - 1]] * len(rows), dtype=torch.int32, device="cuda")
    _check(z, tokens, top, "split rows")
    _check(z.repeat(150, 1), tokens.repeat(150, 1), top, "whole rows")


@pytest.mark.parametrize("top", [1, 20, 32])
def test_values_that_differ_in_their_last_bits(top):
    """All values of a row have the same leading 16 bits, which bound what may be among the largest."""
    print(f"[case] logprobs last bits top {top}", flush=True)
    v = 30011
    g = torch.Generator(device="cuda").manual_seed(8)
    up = 1 + torch.arange(v, device="cuda") * 2.0**-23
    shuffled = up[torch.randperm(v, generator=g, device="cuda")]
    few = 1 + torch.randint(0, 40, (v,), generator=g, device="cuda") * 2.0**-23
    z = torch.stack([up, up.flip(0), -up, shuffled, -shuffled, few, -few, 1e30 * shuffled])
    tokens = torch.tensor([[0, v - 1]] * len(z), dtype=torch.int32, device="cuda")
    _check(z, tokens, top, "split rows")
    _check(z.repeat(150, 1), tokens.repeat(150, 1), top, "whole rows")


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("many", [1, 200])
def test_values_at_the_ends(dtype, many):
    """Tokens ruled out, rows of nothing else, the type's lowest and largest values, NaN and infinities."""
    print(f"[case] logprobs ends {dtype} x {many}", flush=True)
    v, inf = 5003, math.inf
    g = torch.Generator(device="cuda").manual_seed(5)
    base = torch.randn(14, v, generator=g, device="cuda") * 4
    low = torch.finfo(dtype).min
    base[0, torch.randperm(v, generator=g, device="cuda")[:4980]] = -inf   # fewer left than asked for
    base[1] = -inf
    base[2] = -inf
    base[2, 4001] = -3.0
    base[3] = low
    base[4] = low
    base[4, 17] = 0.0
    base[5, 3] = torch.finfo(dtype).max
    base[6, 4000] = math.nan
    base[7, 9] = inf
    base[8, 9], base[8, 8] = inf, math.nan
    base[9] = math.nan
    base[10] += 60000.0
    base[11] *= 1e4
    base[12, :2500] = -inf
    base[13] = inf
    z = base.to(dtype).repeat(many, 1)
    tokens = torch.tensor([[0, 17, 4001, -1, 9]] * len(z), dtype=torch.int32, device="cuda")
    _check(z, tokens, 32, "ends")


def test_tokens_past_the_vocabulary():
    print("[case] logprobs tokens", flush=True)
    z, _ = _logits(6, 3000, F32, 9)
    tokens = torch.tensor([[0, 2999, 3000], [-1, -5, -(1 << 31)], [(1 << 31) - 1, 1, 1]] * 2, dtype=torch.int32, device="cuda")
    got = _check(z, tokens, 3, "tokens", flags=8)
    assert got["logprob"][0, 2] == -math.inf and (got["logprob"][1] == 0).all()


def test_what_is_not_asked_for():
    """Every output is optional; logits of one row, of no row; none is written past its rows."""
    import paper_2609_30884_amd as crf
    print("[case] logprobs outputs", flush=True)
    ctx = _ctx()
    z, tokens = _logits(4, 1003, BF, 11, pad=2)
    ref, _ = _reference(z, tokens, 4)
    lse = torch.full((6,), 7.0, device="cuda")
    crf.token_logprobs(ctx, z, lse=lse[:4])
    top, lp = torch.zeros(4, 4, dtype=torch.int32, device="cuda"), torch.zeros(4, 4, device="cuda")
    crf.token_logprobs(ctx, z, top_token=top, top_logprob=lp)
    one = torch.zeros(1, device="cuda")
    crf.token_logprobs(ctx, z[2], entropy=one)
    crf.token_logprobs(ctx, z)
    crf.token_logprobs(ctx, z[:0], tokens[:0], torch.zeros(0, 3, device="cuda"), lse=lse[:0])
    torch.cuda.synchronize()
    assert (lse[4:] == 7.0).all() and (lse[:4] - ref["lse"]).abs().max() < 1e-5
    assert torch.equal(top, ref["top_token"]) and (lp - ref["top_logprob"]).abs().max() < 1e-5
    assert abs(one.item() - ref["entropy"][2].item()) < 1e-5 and ctx.device_errors() == 0


def test_after_a_decoding_step_captured():
    """As a step's end: logits made by other work of the graph, replayed with others, eager calls between."""
    print("[case] logprobs captured", flush=True)
    import paper_2609_30884_amd as crf
    ctx = _ctx()
    g = torch.Generator(device="cuda").manual_seed(3)
    src = torch.randn(8, 50000, generator=g, device="cuda") * 3
    z, tokens = torch.zeros(8, 50000, dtype=BF, device="cuda"), torch.zeros(8, 1, dtype=torch.int32, device="cuda")
    out = {"logprob": torch.zeros(8, 1, device="cuda"), "entropy": torch.zeros(8, device="cuda"),
           "lse": torch.zeros(8, device="cuda"), "top_token": torch.zeros(8, 9, dtype=torch.int32, device="cuda"),
           "top_logprob": torch.zeros(8, 9, device="cuda")}

    def step():
        z.copy_(src)
        crf.token_logprobs(ctx, z, tokens, **out)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(5):
        src.copy_(torch.randn(8, 50000, generator=g, device="cuda") * (1 + i))
        tokens.fill_(i * 1000)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: v.clone() for k, v in out.items()}
        want = _call(ctx, src.to(BF), tokens, 9)
        assert all(torch.equal(got[k], want[k]) for k in got)
    assert ctx.device_errors() == 0

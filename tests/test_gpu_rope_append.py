"""crf_rope_append against the rotation in 64 bits: layouts, parts of a head,
scalings, far positions, strides, ragged batches."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = "bf16", "f32"


def _dt(name):
    return torch.bfloat16 if name == BF else torch.float32


def _rotate(x, freq, m, pos, layout):
    """(result, bound): pairs as complex numbers times m e^(i pos freq)."""
    from tests.paged import U
    r = 2 * len(freq)
    d = x.double()
    out = d.clone()
    ang = pos.double()[:, None, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    i0 = torch.arange(r // 2, device="cuda") * (2 if layout == "interleaved" else 1)
    i1 = i0 + (1 if layout == "interleaved" else r // 2)
    a, b = d[..., i0], d[..., i1]
    out[..., i0] = m * (a * ang.cos() - b * ang.sin())
    out[..., i1] = m * (b * ang.cos() + a * ang.sin())
    # the angle in half turns is rounded to 24 bits (at most 2^-25 of pi), cosine and
    # sine are within 2 steps, the products and their sum within one each
    slack = torch.zeros_like(d)
    slack[..., i0] = slack[..., i1] = 2.0 ** -21 * m * (a.abs() + b.abs())
    return out, torch.where(slack > 0, slack + U[x.dtype] * (out.abs() + slack), 0.0)


def _case(b, rope, freq, m, layout, positions=None, ctx=None, with_q=True):
    import paper_2609_30884_amd as crf
    from tests.paged import assert_within, context
    ctx = ctx or context(b.nq, b.nkv, b.hd, b.dtype)
    n, w = b.n_rows, (b.nq + 2 * b.nkv) * b.hd
    qkv = torch.randn(n, w, generator=b.gen, device="cuda").to(b.dtype)
    q = qkv[:, :b.nq * b.hd].unflatten(1, (b.nq, b.hd))
    k = qkv[:, b.nq * b.hd:(b.nq + b.nkv) * b.hd].unflatten(1, (b.nkv, b.hd))
    v = qkv[:, (b.nq + b.nkv) * b.hd:]
    q_out = torch.full((n, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda") if with_q else None
    kp, vp = b.k_pool.clone(), b.v_pool.clone()
    crf.rope_append(ctx, rope, b.batch, q if with_q else None, k, v, b.pool, 1, q_out, positions)
    torch.cuda.synchronize()
    for s, (new, total) in enumerate(zip(b.new, b.total)):
        if new == 0:
            continue
        rows = slice(b.starts[s], b.starts[s + 1])
        tok = torch.arange(total - new, total)
        pos = tok.cuda() if positions is None else positions[rows]
        pg, sl = b.places(s, tok)
        ref, bound = _rotate(k[rows], freq, m, pos, layout)
        assert_within(b.k_pool[1, pg, :, sl], ref, bound, f"k {s}")
        assert torch.equal(b.v_pool[1, pg, :, sl], v[rows].unflatten(1, (b.nkv, b.hd)))
        kp[1, pg, :, sl], vp[1, pg, :, sl] = b.k_pool[1, pg, :, sl], b.v_pool[1, pg, :, sl]
        if with_q:
            ref, bound = _rotate(q[rows], freq, m, pos, layout)
            assert_within(q_out[rows], ref, bound, f"q {s}")
    assert torch.equal(kp, b.k_pool) and torch.equal(vp, b.v_pool)  # nothing else was written
    if with_q:
        assert (q_out[b.rows:] == 7.0).all()
    return ctx


SEQS = [(1, 100), (17, 0), (0, 5), (3, 4000), (1, 0), (40, 31)]


@pytest.mark.parametrize("dtype,nq,nkv,hd,page", [(BF, 12, 2, 128, 16), (BF, 4, 2, 64, 1), (F32, 4, 2, 64, 8),
                                                  (F32, 3, 1, 128, 7), (BF, 28, 4, 128, 32)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rotary", [0, 16, 48, -1])
def test_layouts(dtype, nq, nkv, hd, page, layout, rotary):
    import paper_2609_30884_amd as crf
    from tests.paged import Batch
    r = hd if rotary < 0 else rotary
    print(f"[case] rope {dtype} {nq}/{nkv} hd {hd} {layout} rotary {r} page {page}", flush=True)
    b = Batch(SEQS, nq, nkv, hd, _dt(dtype), page=page, seed=3, pad=2)
    freq = [1e4 ** (-2 * i / r) for i in range(r // 2)]
    ctx = _case(b, crf.rope(r, 1e4, layout=layout), freq, 1.0, layout)
    assert ctx.device_errors() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("base", 8.0), ("parts", 4.0), ("parts", 1.0)])
def test_scalings(dtype, scaling, factor):
    import paper_2609_30884_amd as crf
    from tests.paged import Batch
    print(f"[case] rope {dtype} {scaling} {factor}", flush=True)
    r, length, lo, hi = 64, 4096, 1.0, 32.0
    theta = 1e4 * factor ** (r / (r - 2)) if scaling == "base" else 1e4
    freq = [theta ** (-2 * i / r) for i in range(r // 2)]
    if scaling == "linear":
        freq = [f / factor for f in freq]
    if scaling == "parts":
        keep = [min(1.0, max(0.0, (f * length / (2 * math.pi) - lo) / (hi - lo))) for f in freq]
        assert 0.0 in keep and 1.0 in keep and any(0 < k < 1 for k in keep)
        freq = [k * f + (1 - k) * f / factor for f, k in zip(freq, keep)]
    m = float(torch.tensor(0.1 * math.log(factor) + 1.0 if scaling == "parts" else 1.0, dtype=torch.float32))
    plan = crf.rope(r, 1e4, scaling=scaling, factor=factor, original_len=length)
    assert plan.mscale == m
    for f, g in zip(freq, plan.freq):
        assert abs(f - g) <= 1e-13 * f
    _case(Batch(SEQS, 4, 2, 128, _dt(dtype), seed=5), plan, list(plan.freq[:r // 2]), m, "half")


def test_far_positions_and_many_rows():
    import paper_2609_30884_amd as crf
    from tests.paged import Batch
    print("[case] rope far, many rows", flush=True)
    for dtype, nq in ((BF, 12), (F32, 3)):
        b = Batch([(1500, 20), (0, 3), (701, 0), (2, 9)], nq, 1, 128, _dt(dtype), seed=7, pad=5)
        freq = [1e6 ** (-2 * i / 128) for i in range(64)]
        plan = crf.rope(128, 1e6)
        pos = torch.arange(b.n_rows, dtype=torch.int32, device="cuda")
        ctx = _case(b, plan, freq, 1.0, "half", positions=pos + (1 << 20))
        _case(b, plan, freq, 1.0, "half", positions=(1 << 31) - 1 - pos, ctx=ctx)
        _case(b, plan, freq, 1.0, "half", ctx=ctx)
        _case(b, plan, freq, 1.0, "half", ctx=ctx, with_q=False)
        assert ctx.device_errors() == 0


def test_more_rows_than_a_launch_takes():
    """Tokens behind four million rows of nobody are appended as if alone."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, context
    print("[case] rope behind 2^22 rows", flush=True)
    b = Batch([(3, 20)], 2, 2, 64, torch.bfloat16, seed=3)
    ctx, plan, far = context(2, 2, 64, torch.bfloat16), crf.rope(64, 1e4), (1 << 22) + 9
    x = torch.zeros(far + 3, 6, 64, dtype=torch.bfloat16, device="cuda")
    x[far:] = torch.randn(3, 6, 64, device="cuda")
    some = [x[:, 2 * i:2 * i + 2] for i in range(3)]
    outs, pools = [], []
    for first in (far, 0):
        t = [y[far - first:] for y in some]
        batch = crf.seq_batch(b.row_start + first, b.length, b.tables, first + 3, 3)
        out = torch.zeros(first + 3, 2, 64, dtype=torch.bfloat16, device="cuda")
        crf.rope_append(ctx, plan, batch, *t, b.pool, 1, out)
        torch.cuda.synchronize()
        assert (out[:first] == 0).all() and out[first:].any()
        outs.append(out[first:].clone())
        pools.append([b.k_pool.clone(), b.v_pool.clone()])
        b.k_pool.zero_()
        b.v_pool.zero_()
    pg, sl = b.places(0, torch.tensor([20, 21, 22]))
    assert torch.equal(outs[0], outs[1])
    for p, q in zip(*pools):
        assert torch.equal(p[1, pg, :, sl], q[1, pg, :, sl]) and q[1, pg, :, sl].any()
    assert ctx.device_errors() == 0


def test_in_place_and_pages_out_of_range():
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, context
    print("[case] rope in place, bad pages", flush=True)
    b = Batch([(5, 30), (2, 0), (40, 3)], 12, 2, 64, torch.bfloat16, seed=9)
    ctx, plan = context(12, 2, 64, torch.bfloat16), crf.rope(64, 1e6)
    k, v = (torch.randn(b.n_rows, 128, device="cuda").bfloat16() for _ in range(2))
    out = torch.zeros_like(b.q)
    crf.rope_append(ctx, plan, b.batch, b.q, k, v, b.pool, 1, out)
    kp, vp = b.k_pool.clone(), b.v_pool.clone()
    keep = [b.tables[2, 1].clone(), b.tables[1, 0].clone()]
    pages = [int(x) for x in keep]
    b.tables[2, 1], b.tables[1, 0] = b.n_pages, -5
    b.k_pool.zero_()
    b.v_pool.zero_()
    crf.rope_append(ctx, plan, b.batch, b.q, k, v, b.pool, 1, b.q)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 1
    assert torch.equal(b.q, out)
    wrote = torch.zeros(b.n_pages, dtype=torch.bool, device="cuda")
    for s, (n, t) in enumerate(zip(b.new, b.total)):
        for j in range(t - n, t):
            page, slot = int(b.tables_h[s, j // 16]), j % 16
            if page not in pages:
                assert torch.equal(b.k_pool[1, page, :, slot], kp[1, page, :, slot])
                assert torch.equal(b.v_pool[1, page, :, slot], vp[1, page, :, slot])
                wrote[page] = True
    assert (b.k_pool[1, ~wrote] == 0).all() and (b.k_pool[0] == 0).all()


def test_appended_keys_are_the_windows():
    """The rotation that a window writes into the cache and the append's agree: positions, pairs and base."""
    import paper_2609_30884_amd as crf
    from tests.paged import assert_within, context
    print("[case] rope as the windows rotate", flush=True)
    n, hd = 50, 64
    dims = crf.make_dims(1, 64, 2, 1, hd, 64, rope_theta=1e6, dtype="f32")
    ctx = crf.Context(dims, n, 0)
    w = {"attn_norm": torch.ones(64), "mlp_norm": torch.ones(64), "w_q": torch.zeros(128, 64),
         "w_k": torch.eye(64), "w_v": torch.eye(64), "w_o": torch.zeros(64, 128), "w_gate": torch.zeros(64, 64),
         "w_up": torch.zeros(64, 64), "w_down": torch.zeros(64, 64)}
    w = {k: v.cuda() for k, v in w.items()}
    h = torch.randn(n, 64, device="cuda")
    pools = [torch.zeros(1, 4, 1, 16, hd, device="cuda") for _ in range(4)]
    table = torch.tensor([[2, 0, 3, 1]], dtype=torch.int32, device="cuda")
    crf.recompute_window(ctx, dims, h, crf.layer_weights_array([w]), None, 0, 1,
                         crf.kv_cache(pools[0], pools[1], table[0], n, 16))
    x = pools[1][0, table[0].long()].permute(0, 2, 1, 3).reshape(64, hd)[:n].contiguous()  # V: the rows before rotation
    batch = crf.seq_batch(torch.tensor([0, n], dtype=torch.int32, device="cuda"),
                          torch.tensor([n], dtype=torch.int32, device="cuda"), table, n)
    crf.rope_append(ctx, crf.rope(hd, 1e6), batch, None, x, x, crf.page_pool(pools[2], pools[3], 16), 0)
    torch.cuda.synchronize()
    assert torch.equal(pools[3], pools[1])
    # both round cosines, sines, products: 2^-20 of the pair's magnitudes each
    mag = x.abs() + x.abs().roll(32, 1)
    bound = torch.zeros(64, hd, device="cuda", dtype=torch.float64)
    bound[:n] = 2.0 ** -19 * mag.double()
    flat = lambda p: p[0, table[0].long()].permute(0, 2, 1, 3).reshape(64, hd)  # noqa: E731
    assert_within(flat(pools[2]), flat(pools[0]).double(), bound, "window")

"""crf_norm_rope_append against RMSNorm and rotation in 64 bits: layouts, parts of
a head, strides, ragged batches, heads of zeros, of huge and of no numbers."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6  # of tests.paged.context's dims
SEQS = [(1, 100), (17, 0), (0, 5), (3, 4000), (1, 0), (40, 31)]


def _inputs(b, size=None):
    n, heads = b.n_rows, b.nq + 2 * b.nkv
    x = torch.randn(n, heads, b.hd, generator=b.gen, device="cuda")
    x = x * torch.exp(2 * torch.randn(heads, 1, generator=b.gen, device="cuda"))  # heads of different sizes
    qkv = x.to(b.dtype).view(n, -1)
    q = qkv[:, :b.nq * b.hd].unflatten(1, (b.nq, b.hd))
    k = qkv[:, b.nq * b.hd:(b.nq + b.nkv) * b.hd].unflatten(1, (b.nkv, b.hd))
    v = qkv[:, (b.nq + b.nkv) * b.hd:]
    gains = [(1 + 0.3 * torch.randn(b.hd, generator=b.gen, device="cuda")).to(b.dtype) for _ in range(2)]
    return q, k, v, gains


def _case(b, theta=1e4, rotary=None, layout="half", positions=None, with_q=True):
    import paper_2609_30884_amd as crf
    from tests.paged import assert_within, context
    from tests.serving import normed, rotated
    r = b.hd if rotary is None else rotary
    freq = [theta ** (-2 * i / r) for i in range(r // 2)]
    ctx = context(b.nq, b.nkv, b.hd, b.dtype)
    q, k, v, (gq, gk) = _inputs(b)
    q_out = torch.full((b.n_rows, b.nq, b.hd), 7.0, dtype=b.dtype, device="cuda") if with_q else None
    kp, vp = b.k_pool.clone(), b.v_pool.clone()
    crf.norm_rope_append(ctx, crf.rope(r, theta, layout=layout), b.batch, q if with_q else None, k, v,
                         gq if with_q else None, gk, b.pool, 1, q_out, positions)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 0
    for s, (new, total) in enumerate(zip(b.new, b.total)):
        if new == 0:
            continue
        rows = slice(b.starts[s], b.starts[s + 1])
        tok = torch.arange(total - new, total)
        pos = tok.cuda() if positions is None else positions[rows]
        pg, sl = b.places(s, tok)
        ref, bound = rotated(*normed(k[rows], gk, EPS), freq, pos, layout, b.dtype)
        assert_within(b.k_pool[1, pg, :, sl], ref, bound, f"k {s}")
        assert torch.equal(b.v_pool[1, pg, :, sl], v[rows].unflatten(1, (b.nkv, b.hd)))
        kp[1, pg, :, sl], vp[1, pg, :, sl] = b.k_pool[1, pg, :, sl], b.v_pool[1, pg, :, sl]
        if with_q:
            ref, bound = rotated(*normed(q[rows], gq, EPS), freq, pos, layout, b.dtype)
            assert_within(q_out[rows], ref, bound, f"q {s}")
    assert torch.equal(kp, b.k_pool) and torch.equal(vp, b.v_pool)  # nothing else was written
    if with_q:
        assert (q_out[b.rows:] == 7.0).all()


@pytest.mark.parametrize("dtype,nq,nkv,hd,page", [(BF, 12, 2, 128, 16), (BF, 4, 2, 64, 1), (F32, 4, 2, 64, 8),
                                                  (F32, 3, 1, 128, 7), (BF, 28, 4, 128, 32), (BF, 10, 2, 64, 9)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rotary", [0, 16, 48, -1])
def test_layouts(dtype, nq, nkv, hd, page, layout, rotary):
    from tests.paged import Batch
    print(f"[case] norm {dtype} {nq}/{nkv} hd {hd} {layout} rotary {rotary} page {page}", flush=True)
    _case(Batch(SEQS, nq, nkv, hd, dtype, page=page, seed=3, pad=2), rotary=hd if rotary < 0 else rotary, layout=layout)


@pytest.mark.parametrize("dtype,nq", [(BF, 12), (F32, 3)])
def test_many_rows_and_positions(dtype, nq):
    from tests.paged import Batch
    print(f"[case] norm many rows {dtype}", flush=True)
    b = Batch([(1500, 20), (0, 3), (701, 0), (2, 9)], nq, 1, 128, dtype, seed=7, pad=5)
    pos = torch.arange(b.n_rows, dtype=torch.int32, device="cuda") + (1 << 20)
    _case(b, theta=1e6)
    _case(b, theta=1e6, positions=pos)
    _case(b, theta=1e6, with_q=False)


@pytest.mark.parametrize("dtype", [BF, F32])
def test_heads_of_zeros_huge_and_no_numbers(dtype):
    """A head's norm is its own: zeros give zeros, values whose squares pass the range of fp32 their right
    result, a head with an infinity or NaN changes no other."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, assert_within, context
    from tests.serving import normed, rotated
    print(f"[case] norm extremes {dtype}", flush=True)
    nq, nkv, hd = 6, 2, 64
    b = Batch([(3, 2), (2, 40)], nq, nkv, hd, dtype, seed=5)
    q, k, v, (gq, gk) = _inputs(b)
    q, k = q.clone(), k.clone()
    q[0, 0] = 0
    q[0, 1] *= 1e36 / q[0, 1].abs().max().item()
    q[0, 2] *= 1e-25 / q[0, 2].abs().max().item()
    q[0, 3] = 0
    q[0, 3, 5] = 3e38  # one value that holds the whole norm
    q[1, 4, 3], q[2, 5, 63] = math.inf, math.nan
    k[3, 0] *= 2e19 / k[3, 0].abs().max().item()
    k[1, 1, 0] = -math.inf
    ctx, plan, freq = context(nq, nkv, hd, dtype), crf.rope(hd, 1e4), [1e4 ** (-2 * i / hd) for i in range(hd // 2)]
    out = torch.zeros_like(q)
    crf.norm_rope_append(ctx, plan, b.batch, q, k, v, gq, gk, b.pool, 1, out)
    torch.cuda.synchronize()
    pos = torch.tensor([2, 3, 4, 40, 41], device="cuda")
    odd_q, odd_k = torch.zeros(5, nq, dtype=torch.bool, device="cuda"), torch.zeros(5, nkv, dtype=torch.bool, device="cuda")
    odd_q[1, 4] = odd_q[2, 5] = odd_k[1, 1] = True
    ref, bound = rotated(*normed(q, gq, EPS), freq, pos, "half", dtype)
    assert_within(out[~odd_q], ref[~odd_q], bound[~odd_q], "q")
    assert (out[0, 0] == 0).all() and torch.isnan(out[2, 5]).all() and torch.isnan(out[1, 4]).any()
    ref, bound = rotated(*normed(k, gk, EPS), freq, pos, "half", dtype)
    at = [b.places(0, torch.arange(2, 5)), b.places(1, torch.arange(40, 42))]
    got = torch.cat([b.k_pool[1, pg, :, sl] for pg, sl in at])
    assert_within(got[~odd_k], ref[~odd_k], bound[~odd_k], "k")
    assert torch.isnan(got[1, 1]).any() and ctx.device_errors() == 0


@pytest.mark.parametrize("dtype", [BF, F32])
def test_without_eps(dtype):
    """rms_eps 0: a head's norm does not depend on its size, down to values whose squares fp32 does not hold."""
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, assert_within
    from tests.serving import normed, rotated
    print(f"[case] norm without eps {dtype}", flush=True)
    b = Batch([(4, 3)], 6, 2, 64, dtype, seed=5)
    dims = crf.make_dims(2, 128 if dtype == BF else 64, 6, 2, 64, 64, rms_eps=0.0, dtype="bf16" if dtype == BF else "f32")
    ctx, freq = crf.Context(dims, 1, 0), [1e4 ** (-2 * i / 64) for i in range(32)]
    q, k, v, (gq, gk) = _inputs(b)
    q = (q.float() * torch.tensor([1.0, 1e-18, 1e-25, 1e-30, 1e18, 1e30], device="cuda")[:, None]).to(dtype)
    out = torch.zeros_like(q)
    crf.norm_rope_append(ctx, crf.rope(64, 1e4), b.batch, q, k, v, gq, gk, b.pool, 1, out)
    torch.cuda.synchronize()
    ref, bound = rotated(*normed(q, gq, 0.0), freq, torch.arange(3, 7, device="cuda"), "half", dtype)
    assert_within(out, ref, bound, "q")
    assert ctx.device_errors() == 0


def test_in_place_bad_pages_and_a_contradicting_sequence():
    import paper_2609_30884_amd as crf
    from tests.paged import Batch, context
    print("[case] norm in place, bad pages", flush=True)
    b = Batch([(5, 30), (2, 0), (40, 3)], 12, 2, 64, BF, seed=9)
    ctx, plan = context(12, 2, 64, BF), crf.rope(64, 1e6)
    q, k, v, (gq, gk) = _inputs(b)
    q = q.contiguous()
    out = torch.zeros_like(q)
    crf.norm_rope_append(ctx, plan, b.batch, q, k, v, gq, gk, b.pool, 1, out)
    kp = b.k_pool.clone()
    torch.cuda.synchronize()
    assert ctx.device_errors() == 0
    b.k_pool.zero_()
    bad = int(b.tables[2, 1])
    b.tables[2, 1] = b.n_pages
    b.length[0] = 4  # five new tokens of four
    crf.norm_rope_append(ctx, plan, b.batch, q, k, v, gq, gk, b.pool, 1, q)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 3
    assert torch.equal(q[5:], out[5:]) and not torch.equal(q[:5], out[:5])
    for s, (n, t) in ((1, (2, 2)), (2, (40, 43))):
        for j in range(t - n, t):
            page = int(b.tables_h[s, j // 16])
            want = 0 * kp[1, page, :, j % 16] if page == bad else kp[1, page, :, j % 16]
            assert torch.equal(b.k_pool[1, page, :, j % 16], want)
    pg, sl = b.places(0)
    assert (b.k_pool[1, pg, :, sl] == 0).all()

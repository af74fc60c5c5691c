"""crf_shared_attention where every workgroup takes several units: up to 256 sequences
and groups (a thread holds one) over many heads, with drafts, pages out of range and
values that are no numbers in late units."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _batch(dtype, nq, nkv, page):
    from tests.test_gpu_shared_attention import Grouped
    own = lambda g: [((1, 1, 3, 1, 2)[i % 5], 40 + (37 * i + 11 * g) % 260) for i in range(48)]  # noqa: E731
    groups = [(doc, own(g)) for g, doc in enumerate((700, 333, 64, 1000))]
    return Grouped(groups, nq, nkv, 64, dtype, alone=[(2, 90)] * 8, page=page, seed=31, pad=3)


# 200 sequences and 4 groups over 8 heads are at least 1632 units; no more than 512 workgroups stay on 256 CUs
@pytest.mark.parametrize("dtype,nq,nkv,page", [(BF, 16, 8, 16), (BF, 24, 8, 7), (F32, 8, 8, 16)])
def test_rounds_of_units(dtype, nq, nkv, page):
    from tests.paged import assert_within, context
    from tests.serving import masked_reference
    from tests.test_gpu_shared_attention import _check, _run
    print(f"[case] shared rounds {dtype} {nq}/{nkv} page {page}", flush=True)
    b, ctx = _batch(dtype, nq, nkv, page), context(nq, nkv, 64, dtype)
    want, wl, _ = _check(b, "rounds", ctx=ctx)
    for _ in range(3):
        again = _run(b, ctx)
        assert torch.equal(want, again[0]) and torch.equal(wl, again[1])
    # NaN among the own values of late sequences: their rows' alone
    hit = torch.zeros_like(want, dtype=torch.bool)
    for s in (150, 178, 199):
        pg, sl = b.places(s, torch.tensor([b.total[s] - b.new[s]]))  # (the first new token, which all of them see)
        b.v_pool[1, pg, 2, sl, 11] = math.nan
        g = nq // nkv
        hit[b.starts[s]:b.starts[s + 1], 2 * g:3 * g, 11] = True
    out, lse = _run(b, ctx)
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse, wl) and torch.isnan(out[hit]).all()
    assert ctx.device_errors() == 0
    # and pages out of range among their own keys
    b = _batch(dtype, nq, nkv, page)
    gone = {s: (b.total[s] - b.new[s] - 20) // page for s in (60, 149, 177, 197)}
    for s, p in gone.items():
        b.tables[s, p] = b.n_pages
    out, lse = _run(b, ctx)
    assert ctx.device_errors() == 1

    def seen(s, pos, key):
        return (key <= pos) & ((key // page != gone[s]) if s in gone else key >= 0)
    ref, rl, bo, bl = masked_reference(b, seen)
    assert_within(out[:b.rows], ref[:b.rows], bo[:b.rows], "bad pages")
    assert_within(lse[:b.rows], rl[:b.rows], bl[:b.rows], "bad pages lse")

"""crf_paged_attention with values that are no finite numbers."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = "bf16", "f32"


def _dt(name):
    return torch.bfloat16 if name == BF else torch.float32


@pytest.mark.parametrize("dtype,hd,heads", [(BF, 64, 8), (F32, 64, 4)])
def test_bad_pages_of_unit_after_unit(dtype, hd, heads):
    """Units dealt out whole, several to a workgroup, taken twice for values that are no numbers, some with pages out of
    range: what one finds out about its pages is not the next one's."""
    from tests.paged import Batch, assert_within, attention_reference, context
    print(f"[case] bad pages of units {dtype}", flush=True)
    b = Batch([(130 + s % 3, 20 + 7 * (s % 5)) for s in range(260)], heads, heads, hd, _dt(dtype), seed=47)
    bad, gone = b.tables.clone(), {}
    for s in range(260):
        pg, sl = b.places(s, torch.tensor([5, 100]))
        b.v_pool[1, pg, :, sl, s % 3::11] = math.inf
        gone[s] = [[], [2], [0, 9], []][s % 4]
        for j in gone[s]:
            bad[s, j] = (-1, b.n_pages)[s % 2]
    b.tables.copy_(bad)

    def hidden(s):
        page = torch.arange(b.total[s], device="cuda") // b.page
        return (page[:, None] == torch.tensor(gone[s] or [-1], device="cuda")).any(1)

    import paper_2609_30884_amd as crf
    ctx = context(heads, heads, hd, b.dtype)
    out = torch.zeros(b.n_rows, heads, hd, dtype=b.dtype, device="cuda")
    for _ in range(3):
        crf.paged_attention(ctx, b.batch, b.q, b.pool, 1, out)
    torch.cuda.synchronize()
    assert ctx.device_errors() == 1
    ref, _, bound, _ = attention_reference(b, hidden=hidden)
    assert_within(out, ref, bound, "units")

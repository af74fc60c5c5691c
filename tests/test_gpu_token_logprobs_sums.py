"""crf_token_logprobs: sums over long rows do not drift.  A row of zeros and of one
other value whose weight a long running sum rounds to the same side every time."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
U32 = 2.0 ** -24


# (one after the other into one sum of 32 bits, the 594 terms of a thread leave ln S off by 8.5e-6 for the first value and
# by 1.1e-5 for the second, whose entropy is off by 2.3e-5)
@pytest.mark.parametrize("dtype,held", [(F32, 4), (BF, 8)])
@pytest.mark.parametrize("z", [-63 / 128 * 2.0 ** -15, -230 / 64])
def test_long_rows(dtype, held, z):
    """Weights e^z: z is exact, the factor to log2 units and the exponential leave each off by 3 |z| + 2 steps of 2^-24.
    A sum adds a step for each addition on a term's way into it: within a load of 16 bytes, four loads in flight, the
    rounds of those (256 threads), 6 + 2 over lanes and waves, 4 more for changes of the reference.  ln S: the sum's own
    error, and 3 steps of the logarithm.  The weighted sum's terms have one step more, the quotient another."""
    import paper_2609_30884_amd as crf
    from tests.paged import context
    print(f"[case] logprobs sums {dtype} {z}", flush=True)
    ctx, rows, vocab, zeros = context(2, 2, 64, BF), 520, 152064, 4096  # (so many rows are not shared out)
    logits = torch.full((rows, vocab), z, device="cuda").to(dtype)
    assert float(logits[0, 0]) == z
    logits[:, :zeros] = 0.0
    lse, ent = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
    tokens, lp = torch.full((rows,), vocab - 1, dtype=torch.int32, device="cuda"), torch.zeros(rows, device="cuda")
    crf.token_logprobs(ctx, logits, tokens, lp, entropy=ent, lse=lse)
    torch.cuda.synchronize()
    s, w = zeros + (vocab - zeros) * math.exp(z), (vocab - zeros) * math.exp(z) * z
    ln_s = math.log(s)
    steps = held + 4 + math.ceil(vocab / (256 * 4 * held)) + 12
    weight = 3 * abs(z) + 2
    b_ln = (steps + weight + 3 * ln_s) * U32
    for name, got, want, bound in (
            ("lse", lse, ln_s, b_ln), ("logprob", lp, z - ln_s, b_ln + 2 * abs(z - ln_s) * U32),
            ("entropy", ent, ln_s - w / s,
             b_ln + (abs(w / s) * (2 * (steps + weight) + 2) + abs(ln_s - w / s)) * U32)):
        off = float((got.double() - want).abs().max())
        print(f"[{name}] off by {off:.2e}, bound {bound:.2e}", flush=True)
        assert off <= bound, name
    assert ctx.device_errors() == 0

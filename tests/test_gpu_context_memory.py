"""What contexts need: device memory (free before and after), and nothing of torch."""
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_second_workspace_of_a_batch_holds_no_partials_of_paged_attention():
    """An fp32 context's second workspace, made by its first batch of several caches, serves windows alone."""
    import paper_2609_30884_amd as crf
    print("[case] second workspace", flush=True)
    n, hd = 50, 64
    dims = crf.make_dims(1, 64, 2, 1, hd, 64, dtype="f32")
    w = {"attn_norm": (64,), "mlp_norm": (64,), "w_q": (128, 64), "w_k": (64, 64), "w_v": (64, 64), "w_o": (64, 128),
         "w_gate": (64, 64), "w_up": (64, 64), "w_down": (64, 64)}
    w = {k: torch.randn(*s, device="cuda") * 0.1 for k, s in w.items()}
    layers = crf.layer_weights_array([w])
    table = torch.tensor([2, 0, 3, 1], dtype=torch.int32, device="cuda")
    hidden = [torch.randn(n, 64, device="cuda") for _ in range(2)]

    def batch(ctx, pools):
        kvs = [crf.kv_cache(k, v, table, n, 16) for k, v in pools]
        crf.recompute_window_batched(ctx, dims, layers, [crf.window_item(h, None, 0, 1, kv)
                                                         for h, kv in zip(hidden, kvs)])
        torch.cuda.synchronize()

    def pools():
        return [[torch.zeros(1, 4, 1, 16, hd, device="cuda") for _ in range(2)] for _ in range(2)]

    first, ctx = crf.Context(dims, n, 0), crf.Context(dims, n, 0)
    a, b, c = pools(), pools(), pools()
    batch(first, a)  # (kernels, queues)
    before = torch.cuda.mem_get_info()[0]
    batch(ctx, b)
    grown = before - torch.cuda.mem_get_info()[0]
    assert grown < 16 << 20, f"{grown / 2 ** 20:.0f} MiB"
    # and what it computes is what the context alone computes
    for h, (k, v) in zip(hidden, c):
        crf.recompute_window(ctx, dims, h, layers, None, 0, 1, crf.kv_cache(k, v, table, n, 16))
    torch.cuda.synchronize()
    for x, y, z in zip(a, b, c):
        assert all(torch.equal(p, q) and torch.equal(p, r) for p, q, r in zip(x, y, z))
    assert ctx.device_errors() == 0
    del first, ctx


def test_contexts_of_programs_without_torch():
    """A program that hands pointers of its own to the library makes contexts without importing torch."""
    print("[case] no torch", flush=True)
    code = ("import sys, paper_2609_30884_amd as crf\n"
            "c = crf.Context(crf.make_dims(2, 128, 2, 2, 64, 64), 16, 0)\n"
            "assert c.device_errors() == 0 and 'torch' not in sys.modules\n"
            "c.close()\nprint('made')")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=60,
                       cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0 and r.stdout.strip() == "made", r.stdout + r.stderr

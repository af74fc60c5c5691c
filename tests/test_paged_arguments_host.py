"""Arguments of the page-pool operators at the ends of their ranges (no GPU)."""
import types

import pytest
import torch

import paper_2609_30884_amd as crf


@pytest.mark.parametrize("factor", [1e308, 1e300])
def test_a_base_that_passes_the_range_is_refused(factor):
    """theta * factor^(r / (r - 2)) infinite: every frequency but the first would come out as zero."""
    with pytest.raises(crf.CrfError) as e:
        crf.rope(16, 1e10, scaling="base", factor=factor)
    assert e.value.status == 2
    assert crf.rope(16, 1e10, scaling="base", factor=1e200).freq[7] > 0


@pytest.mark.parametrize("window", [1, 500, (1 << 31) - 1, 1 << 31, (1 << 32) + 5, 1 << 62])
def test_windows_past_the_largest_int_are_none(window):
    """A Python int that 32 bits do not hold is a window that no sequence reaches, not its low bits."""
    got = []
    lib = types.SimpleNamespace(crf_paged_attention=lambda *a: got.append(a[7]) or 0)
    ctx = types.SimpleNamespace(dims=crf.make_dims(2, 128, 4, 2, 64, 64), lib=lib, handle=None, device=-1)
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)  # noqa: E731
    pools = [torch.zeros(2, 8, 2, 16, 64, dtype=torch.bfloat16) for _ in range(2)]
    q = torch.zeros(6, 4, 64, dtype=torch.bfloat16)
    crf.paged_attention(ctx, crf.seq_batch(i32(4), i32(3), i32(3, 2), 6), q, crf.page_pool(*pools, 16), 0, q, window=window,
                        stream=1)
    assert got == [min(window, (1 << 31) - 1)]

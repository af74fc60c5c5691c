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

"""What the paged cache's binding refuses by itself, before the library or a GPU is reached."""
import pytest
import torch

from paper_2505_14260_gb300 import msd

WIDTHS = dict(layers=1, heads=4, kv_heads=2, head_dim=64, page_size=16, n_pages=4, max_seqs=2, max_pages=3)


@pytest.mark.parametrize("dtype", ["bfloat16", "fp32", "float32", "BF16", "", None, torch.bfloat16])
def test_other_words_for_a_type_are_refused(dtype):
    with pytest.raises(ValueError, match="bf16"):
        msd.Pages(dtype=dtype, **WIDTHS)

"""What the paged cache's binding refuses by itself, before the library or a GPU is reached."""
import pytest
import torch

from paper_2505_14260_gb300 import build, msd

WIDTHS = dict(layers=1, heads=4, kv_heads=2, head_dim=64, page_size=16, n_pages=4, max_seqs=2, max_pages=3)


@pytest.mark.parametrize("dtype", ["bfloat16", "fp32", "float32", "BF16", "", None, torch.bfloat16])
def test_other_words_for_a_type_are_refused(dtype):
    with pytest.raises(ValueError, match="bf16"):
        msd.Pages(dtype=dtype, **WIDTHS)


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


class Listed:
    """Stands for a batch of two sequences of one row each."""
    n = rows = 2
    seqs = ints(2)


@pytest.fixture
def pool():
    """A pool's binding without the pool behind it: nothing here reaches a GPU."""
    build.build()
    p = msd.Pages.__new__(msd.Pages)
    p.ptr, p.dtype, p._H, p._K, p._hd, p._dev = None, torch.bfloat16, 4, 2, 64, 0
    return p


def test_host_tensors_are_refused(pool):
    """Their addresses mean nothing to a kernel."""
    on_host = torch.zeros(2, 256, dtype=torch.bfloat16)
    b = Listed()
    b.c = lambda: None
    for call in (lambda: msd.Batch(ints(2), ints(3), 2),
                 lambda: msd.Pages(dtype="bf16", device="cpu", **WIDTHS),
                 lambda: pool.fork(ints(1), ints(1)),
                 lambda: pool.free(ints(1)),
                 lambda: pool.compact(b, None, ints(2)),
                 lambda: pool.positions(b, None, None, ints(3, 2)),
                 lambda: pool.rope_append(0, b, on_host, on_host[:, :128], on_host[:, :128], ints(1, 2), on_host),
                 lambda: pool.attention(0, b, on_host, on_host),
                 lambda: pool.attention(0, b, on_host, on_host, lse=torch.zeros(2, 4)),
                 lambda: pool.attention(0, b, on_host, on_host, tree=msd.Tree(2, 1, device="cpu"))):
        with pytest.raises(ValueError, match="on the GPU"):
            call()

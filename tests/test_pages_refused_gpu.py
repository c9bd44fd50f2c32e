"""What the paged cache does when a call cannot be carried out, is given lists or tables that are wrong, or
meets sizes at its limits: nothing that other sequences hold changes, and the caller is told."""
import pytest
import torch

from paper_2505_14260_gb300 import build, msd
from tests.pages_support import batch, i32, pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def state(p):
    return [t.clone() for t in (p.table, p.lens, p.refs, p.kv.nan_to_num())]


def same(p, before):
    return all(torch.equal(a, b) for a, b in zip(before, (p.table, p.lens, p.refs, p.kv.nan_to_num())))


def reported(p, status):
    """The next call reports an earlier one's error and does nothing."""
    torch.cuda.synchronize()
    with pytest.raises(msd.MsdError) as e:
        p.restore()
    assert e.value.status == status


# ---------------------------------------------------------------------------
# Lists that are refused whole
# ---------------------------------------------------------------------------
def test_free_takes_a_list_whole_or_not_at_all():
    p = pool([20, 40, 33], extra_seqs=2)
    for bad in ([0, 77], [77, 0, 1], [1, -1, 2]):
        before = state(p)
        p.free(i32(bad))
        reported(p, msd.MSD_ERR_DEVICE)
        assert same(p, before)
    for length in (-7, p.cfg.max_pages * 16 + 1):
        keep = int(p.lens[1])
        p.lens[1] = length
        before = state(p)
        p.free(i32([0, 1, 2]))
        reported(p, msd.MSD_ERR_DEVICE)
        assert same(p, before)
        p.lens[1] = keep
    p.free(i32([2, 0, 4, 2, 0]))
    torch.cuda.synchronize()
    assert p.lens.tolist() == [0, 40, 0, 0, 0] and int(p.refs.sum()) == 3
    p.restore()


def test_free_of_a_long_list():
    n = 4000
    p = msd.Pages(dtype="bf16", layers=1, heads=1, kv_heads=1, head_dim=64, page_size=16, n_pages=3 * n, max_seqs=n,
                  max_pages=3)
    b = batch(list(range(n)), [1 + i % 48 for i in range(n)])
    p.reserve(b)
    torch.cuda.synchronize()
    before = state(p)
    p.free(i32(list(range(n - 1)) + [n]))
    reported(p, msd.MSD_ERR_DEVICE)
    assert same(p, before)
    p.free(b.seqs)
    torch.cuda.synchronize()
    assert not p.refs.any() and not p.lens.any() and (p.table == -1).all()

"""What the paged cache refuses before it touches a GPU, and the binding's structs."""
import ctypes

import pytest

from paper_2505_14260_gb300 import build, msd
from tests.test_abi_cpu import _header_struct_fields


@pytest.fixture(scope="module")
def lib():
    build.build()
    return msd.lib()


GOOD = dict(dtype=1, n_layers=2, n_heads=8, n_kv_heads=2, head_dim=128, page_size=64, n_pages=100, max_seqs=4,
            max_pages=50, rot_dim=128, rot_section=(24, 20, 20), rot_interleaved=0, rope_base=10000.0)


def config(**kw):
    c = dict(GOOD, **kw)
    c["rot_section"] = (ctypes.c_int32 * 3)(*c["rot_section"])
    return msd.msd_pages_config(**c)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(n_layers=0), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=9), dict(n_heads=130, n_kv_heads=2),
    dict(head_dim=96), dict(head_dim=256), dict(page_size=8), dict(page_size=48), dict(page_size=256), dict(n_pages=0),
    dict(max_seqs=0), dict(max_seqs=70000), dict(max_pages=0), dict(max_pages=(1 << 24) + 1), dict(n_pages=1 << 30),
    dict(rot_dim=130), dict(rot_dim=127), dict(rot_dim=-2), dict(rot_section=(24, 20, 19)), dict(rot_section=(-1, 45, 20)),
    dict(rot_interleaved=2), dict(rot_interleaved=1, rot_section=(16, 24, 24)), dict(rope_base=0.5),
    dict(rope_base=float("inf")), dict(rope_base=float("nan"))])
def test_create_refuses_bad_configurations(lib, kw):
    buf, out = msd.msd_pages_buffers(16, 16, 16, 16), ctypes.c_void_p()
    assert lib.msd_pages_create(ctypes.byref(config(**kw)), ctypes.byref(buf), ctypes.byref(out)) == msd.MSD_ERR_INVALID
    assert not out.value


def test_create_refuses_null_and_unaligned_arrays(lib):
    out, cfg = ctypes.c_void_p(), config()
    for at in range(4):
        buf = msd.msd_pages_buffers(*[0 if i == at else 256 for i in range(4)])
        assert lib.msd_pages_create(ctypes.byref(cfg), ctypes.byref(buf), ctypes.byref(out)) == msd.MSD_ERR_INVALID
    buf = msd.msd_pages_buffers(264, 256, 256, 256)
    assert lib.msd_pages_create(ctypes.byref(cfg), ctypes.byref(buf), ctypes.byref(out)) == msd.MSD_ERR_INVALID
    assert lib.msd_pages_create(None, ctypes.byref(buf), ctypes.byref(out)) == msd.MSD_ERR_INVALID
    assert lib.msd_pages_create(ctypes.byref(cfg), None, ctypes.byref(out)) == msd.MSD_ERR_INVALID


def test_null_pools_are_refused(lib):
    b = ctypes.byref(msd.msd_batch(1, 16, 16, 1))
    assert lib.msd_pages_restore(None, None) == msd.MSD_ERR_INVALID
    assert lib.msd_pages_reserve(None, b, None) == msd.MSD_ERR_INVALID
    assert lib.msd_pages_fork(None, 1, 16, 16, 0, None) == msd.MSD_ERR_INVALID
    assert lib.msd_pages_compact(None, b, None, 0, 16, None) == msd.MSD_ERR_INVALID
    assert lib.msd_pages_free(None, 1, 16, None) == msd.MSD_ERR_INVALID
    assert lib.msd_rope_positions(None, b, None, None, 0, None, 16, 1, None, None) == msd.MSD_ERR_INVALID
    assert lib.msd_pages_destroy(None) == msd.MSD_OK
    assert lib.msd_pages_last_error(None) == b"null pool"


@pytest.mark.parametrize("name", ["msd_pages_buffers", "msd_batch"])
def test_binding_structs_match_the_header(name):
    names = [n.split()[-1].lstrip("*") for n in _header_struct_fields(name)]        # (const int32_t *x: the last word)
    assert [f for f, _ in getattr(msd, name)._fields_] == names


def test_binding_config_matches_the_header():
    names = [n.split("[")[0] for n in _header_struct_fields("msd_pages_config")]
    assert names == [f for f, _ in msd.msd_pages_config._fields_]

"""Query rows that would be written over each other, or over rows that are still to be read: refused by the append calls
on the host, before any device call (no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2607_05708_gb300 import _build, load_library
    _build.build()
    return load_library()


def _statuses(lib, n, heads, width=64, **kw):
    """What both append calls say (4: no device here, the arguments were taken)."""
    from paper_2607_05708_gb300 import _KVConfig, _LatentConfig, _Rotation
    r = dict(positions=16, cos=16, sin=16, table_rows=4, rotary_dim=64, q=1 << 20, q_row_stride=heads * width,
             q_head_stride=width, q_heads=heads, q_out=1 << 30, q_out_row_stride=heads * width, q_out_head_stride=width)
    r = ctypes.byref(_Rotation(**{**r, **kw}))
    kv = ctypes.byref(_KVConfig(4, 2, width, 64, 8, 1 << 20))
    latent = ctypes.byref(_LatentConfig(512, 64, 64, 0, 8, 1 << 20))
    a = lib.akashic_mem_kv_append(kv, 16, None, 16, 128, 64, 16, 128, 64, 0, n, 16, None, r, None, None)
    b = lib.akashic_mem_latent_append(latent, 16, None, 16, 512, 16, 64, 0, n, 16, None, r, None, None)
    return a, b


SAME = dict(q_out=1 << 20)
BAD = [dict(q_out_head_stride=0), dict(q_out_row_stride=0), dict(q_out_head_stride=56), dict(q_out_row_stride=-63),
       dict(q_head_stride=0, q_out_head_stride=0, **SAME), dict(q_row_stride=0, q_out_row_stride=0, **SAME),
       dict(q_out_row_stride=256, **SAME), dict(q_out_head_stride=256, **SAME), dict(q_row_stride=0, **SAME)]
GOOD = [dict(), SAME, dict(q_row_stride=0), dict(q_head_stride=0, q_row_stride=0), dict(q_out_row_stride=64,
        q_out_head_stride=5 * 64), dict(q_out_row_stride=200), dict(q_row_stride=-192, q_out_row_stride=-192, **SAME)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_overlapping_rows_are_refused(lib, bad):
    assert _statuses(lib, 5, 3, **bad) == (1, 1)


@pytest.mark.parametrize("good", GOOD, ids=str)
def test_rows_apart_are_taken(lib, good):
    assert _statuses(lib, 5, 3, **good) == (4, 4)


def test_strides_of_single_rows_and_heads_do_not_count(lib):
    assert _statuses(lib, 1, 3, q_out_row_stride=0) == (4, 4)
    assert _statuses(lib, 1, 3, q_out_row_stride=7, **SAME) == (4, 4)
    assert _statuses(lib, 5, 1, q_out_head_stride=0) == (4, 4)
    assert _statuses(lib, 5, 1, q_head_stride=0, **SAME) == (4, 4)

"""Sizes of the expanded latent attention whose products pass 64 bits: refused on the host, before any device call
(no GPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2607_05708_gb300 import _build, load_library
    _build.build()
    return load_library()


def _refused(lib, cfg, **kw):
    from paper_2607_05708_gb300 import _LatentAttend
    R = kw.pop("R")
    a = dict(q=16, blocks=16, out=16, scale=1.0, w_k=16, w_v=16, w_k_head_stride=128 * R, w_k_row_stride=R,
             w_v_head_stride=128 * R, w_v_row_stride=R, nope_dim=128, value_dim=128)
    a = ctypes.byref(_LatentAttend(**{**a, **kw}))
    size = ctypes.c_int64(-7)
    assert lib.akashic_mem_latent_expanded_scratch(cfg, a, ctypes.byref(size)) == 1
    assert b"expanded_scratch" in lib.akashic_mem_last_error()
    assert size.value == -7
    assert lib.akashic_mem_latent_attend_expanded(cfg, 16, a, 16, 1 << 62, None, None) == 1


def _config(block_tokens=64, R=128):
    from paper_2607_05708_gb300 import _LatentConfig
    return ctypes.byref(_LatentConfig(R, 32, block_tokens, 0, 8, 0))


# sequences and blocks of 4096 tokens a list: 2^55 tokens (times 512 bytes: 2^64); just 2^31; one token's
# list of 128 a sequence
@pytest.mark.parametrize("n_seq,max_blocks", [(1 << 25, 1 << 18), (1 << 24, 1 << 18), ((1 << 31) - 1, 1 << 18),
                                              (1 << 12, 1 << 7), (4, 1 << 17), (1 << 24, 0), ((1 << 31) - 1, 0)])
def test_more_tokens_than_the_scratch_can_number(lib, n_seq, max_blocks):
    _refused(lib, _config(4096), R=128, n_q=n_seq, q_heads=1, n_seq=n_seq, max_blocks=max_blocks)


@pytest.mark.parametrize("name", ["w_k_head_stride", "w_v_head_stride"])
@pytest.mark.parametrize("stride,heads", [(128 << 55, 513), (128 << 54, 1024), ((1 << 63) - 128, 3), (128 << 31, 2)])
def test_head_strides_beyond_64_bits(lib, name, stride, heads):
    _refused(lib, _config(), R=128, n_q=1, q_heads=heads, n_seq=1, max_blocks=1, **{name: stride})


def test_nothing_to_do_is_no_error(lib):
    from paper_2607_05708_gb300 import _LatentAttend
    a = ctypes.byref(_LatentAttend(n_q=0, q_heads=1, n_seq=1 << 25, max_blocks=1 << 18, scale=1.0, w_k_head_stride=128,
                                   w_k_row_stride=128, w_v_head_stride=128, w_v_row_stride=128, nope_dim=64,
                                   value_dim=64))
    assert lib.akashic_mem_latent_attend_expanded(_config(4096), None, a, None, 0, None, None) == 0

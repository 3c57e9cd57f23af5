"""What the append calls and the latent cache's calls refuse on the host, before any device
call, and the test oracle's own pins (no GPU)."""
import ctypes

import numpy as np
import pytest

import _latent_oracle as orc


@pytest.fixture(scope="module")
def lib():
    from paper_2607_05708_gb300 import _build, load_library
    _build.build()
    return load_library()


def _kv():
    from paper_2607_05708_gb300 import _KVConfig
    return ctypes.byref(_KVConfig(4, 2, 128, 64, 8, 0))


def _config(**kw):
    from paper_2607_05708_gb300 import _LatentConfig
    c = dict(latent_dim=512, rope_dim=64, block_tokens=64, dtype=0, n_blocks=8, device=0)
    c.update(kw)
    return ctypes.byref(_LatentConfig(*(c[k] for k in ("latent_dim", "rope_dim", "block_tokens", "dtype", "n_blocks",
                                                       "device"))))


def _rotation(**kw):
    from paper_2607_05708_gb300 import _Rotation
    r = dict(positions=16, cos=16, sin=16, table_rows=4, rotary_dim=64)
    r.update(kw)
    return ctypes.byref(_Rotation(**r))


BAD = [dict(latent_dim=64), dict(latent_dim=384), dict(latent_dim=0), dict(rope_dim=0), dict(rope_dim=48),
       dict(rope_dim=128), dict(block_tokens=0), dict(block_tokens=24), dict(block_tokens=8192), dict(dtype=2),
       dict(dtype=-1), dict(n_blocks=0), dict(n_blocks=1 << 25), dict(device=-1)]


@pytest.mark.parametrize("bad", BAD, ids=lambda b: "_".join(f"{k}{v}" for k, v in b.items()))
def test_bad_configs(lib, bad):
    from paper_2607_05708_gb300 import _LatentAttend
    size = ctypes.c_int64()
    assert lib.akashic_mem_latent_cache_bytes(_config(**bad), ctypes.byref(size)) == 1
    assert b"latent_cache_bytes" in lib.akashic_mem_last_error()
    assert lib.akashic_mem_latent_append(_config(**bad), 16, None, 16, 1, 16, 1, 0, 1, 16, None, None, None, None) == 1
    a = ctypes.byref(_LatentAttend(n_q=1, q_heads=2, n_seq=1, max_blocks=1, scale=1.0))
    for call in (lib.akashic_mem_latent_attend, lib.akashic_mem_latent_attend_expanded):
        assert call(_config(**bad), 16, a, 16, 1 << 30, None, None) == 1


def test_cache_bytes(lib):
    size = ctypes.c_int64()
    assert lib.akashic_mem_latent_cache_bytes(_config(block_tokens=48, n_blocks=5), ctypes.byref(size)) == 0
    assert size.value == 576 * 2 * 48 * 5
    assert lib.akashic_mem_latent_cache_bytes(_config(), None) == 1
    assert lib.akashic_mem_latent_cache_bytes(None, ctypes.byref(size)) == 1


ROT = [dict(rotary_dim=0), dict(rotary_dim=16), dict(rotary_dim=48), dict(rotary_dim=160), dict(table_rows=0),
       dict(positions=None), dict(cos=None), dict(sin=None), dict(cos=20), dict(sin=8), dict(positions=20),
       dict(q=16), dict(q_out=16), dict(q=16, q_out=16, q_heads=0), dict(q=17, q_out=16, q_heads=1),
       dict(q=16, q_out=17, q_heads=1)]


@pytest.mark.parametrize("bad", ROT, ids=lambda b: "_".join(f"{k}{v}" for k, v in b.items()))
def test_bad_rotations(lib, bad):
    assert lib.akashic_mem_kv_append(_kv(), 16, None, 16, 8, 8, 16, 8, 8, 0, 1, 16, None, _rotation(**bad), None,
                                     None) == 1
    assert b"kv_append" in lib.akashic_mem_last_error()
    assert lib.akashic_mem_latent_append(_config(), 16, None, 16, 8, 16, 8, 0, 1, 16, None, _rotation(**bad), None,
                                         None) == 1


def test_bad_rows(lib):
    k = lib.akashic_mem_kv_append
    assert k(_kv(), 16, None, 16, 1, 1, 16, 1, 1, 0, 1, 16, None, None, None, None) == 1         # no rotation
    assert k(_kv(), 16, None, 16, 1, 1, 16, 1, 1, 3, 1, 16, None, _rotation(), None, None) == 1
    assert k(_kv(), 16, None, 16, 1, 1, 16, 1, 1, 0, -1, 16, None, _rotation(), None, None) == 1
    assert k(_kv(), None, None, 16, 1, 1, 16, 1, 1, 0, 1, 16, None, _rotation(), None, None) == 1
    assert k(_kv(), 16, None, 16, 1, 1, 16, 1, 1, 0, 1, 16, 16, _rotation(), None, None) == 1     # tags
    assert k(_kv(), None, None, None, 1, 1, None, 1, 1, 0, 0, None, None, _rotation(), None, None) == 0
    a = lib.akashic_mem_latent_append
    assert a(_config(), 16, None, 16, 1, 16, 1, 3, 1, 16, None, None, None, None) == 1
    assert a(_config(), 16, None, 16, 1, 16, 1, 0, 1 << 31, 16, None, None, None, None) == 1
    assert a(_config(), 16, None, None, 1, 16, 1, 0, 1, 16, None, None, None, None) == 1
    assert a(_config(), 8, None, 16, 1, 16, 1, 0, 1, 16, None, None, None, None) == 1
    assert a(_config(), 16, None, 17, 1, 16, 1, 0, 1, 16, None, None, None, None) == 1
    assert a(_config(), 16, None, 16, 1, 16, 1, 0, 1, 20, None, None, None, None) == 1
    assert a(_config(), 16, None, 16, 1, 16, 1, 0, 1, 16, 16, None, None, None) == 1
    assert a(_config(rope_dim=32), 16, None, 16, 1, 16, 1, 0, 1, 16, None, _rotation(), None, None) == 1
    assert a(_config(), None, None, None, 1, None, 1, 0, 0, None, None, None, None, None) == 0


GOOD = dict(n_q=2, q_heads=4, n_seq=2, max_blocks=3, q=16, blocks=16, out=16, scale=1.0)
WEIGHTS = dict(w_k=16, w_v=16, w_k_head_stride=64 * 512, w_k_row_stride=512, w_v_head_stride=64 * 512,
               w_v_row_stride=512, nope_dim=64, value_dim=64)
ATTEND = [dict(q_heads=0), dict(q_heads=1025), dict(n_seq=-1), dict(n_q=-1), dict(max_blocks=-1),
          dict(max_blocks=1 << 26), dict(n_q=3), dict(n_q=1 << 28, q_heads=16), dict(scale=0.0),
          dict(scale=float("nan")), dict(scale=float("inf")), dict(tags=16), dict(q_tags=16)]
EXPANDED = [dict(nope_dim=32), dict(value_dim=96), dict(w_k_row_stride=504), dict(w_v_row_stride=516),
            dict(w_k_head_stride=64 * 512 + 8), dict(w_v_head_stride=-512), dict(lse=16),
            dict(w_k_head_stride=512 << 33)]


@pytest.mark.parametrize("bad", ATTEND + EXPANDED, ids=lambda b: "_".join(f"{k}{v}" for k, v in b.items()))
def test_bad_attention(lib, bad):
    from paper_2607_05708_gb300 import _LatentAttend
    size = ctypes.c_int64()
    a = ctypes.byref(_LatentAttend(**{**GOOD, **WEIGHTS, **bad}))
    forms = [(lib.akashic_mem_latent_attend_expanded, lib.akashic_mem_latent_expanded_scratch)]
    if bad in ATTEND:
        forms.append((lib.akashic_mem_latent_attend, lib.akashic_mem_latent_attend_scratch))
    for call, scratch in forms:
        assert scratch(_config(), a, ctypes.byref(size)) == 1
        assert call(_config(), 16, a, 16, 1 << 40, None, None) == 1
        assert b"latent" in lib.akashic_mem_last_error()


def test_bad_attention_pointers(lib):
    from paper_2607_05708_gb300 import _LatentAttend
    for call, extra in ((lib.akashic_mem_latent_attend, {}), (lib.akashic_mem_latent_attend_expanded, WEIGHTS)):
        more = [dict(w_k=None), dict(w_v=None), dict(w_k=24)] if extra else [dict(lse=2)]
        for bad in [dict(q=None), dict(out=None), dict(blocks=None), dict(q=17), dict(out=18), dict(blocks=20),
                    dict(kv_len=18), dict(q_start=2), dict(prefix_len=2), dict(tags=20, q_tags=16)] + more:
            a = _LatentAttend(**{**GOOD, **extra, **bad})
            assert call(_config(), 16, ctypes.byref(a), 16, 1 << 40, None, None) == 1, bad
        a = _LatentAttend(**{**GOOD, **extra})
        assert call(_config(), None, ctypes.byref(a), 16, 1 << 40, None, None) == 1
        assert call(_config(), 8, ctypes.byref(a), 16, 1 << 40, None, None) == 1
        assert call(_config(), 16, ctypes.byref(a), 8, 1 << 40, None, None) == 1
        assert call(_config(), 16, None, 16, 1 << 40, None, None) == 1
        for none in (dict(n_q=0), dict(n_seq=0, n_q=0)):      # nothing to do
            a = _LatentAttend(**{**GOOD, **extra, **none, "q": None, "out": None, "blocks": None})
            assert call(_config(), None, ctypes.byref(a), None, 0, None, None) == 0


# ------------------------------------------------------------------ the oracle's pins
def test_rotation_by_hand():
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    cos, sin = np.array([[1.0, 1], [0, 1]]), np.array([[0.0, 0], [1, 0]])
    assert (orc.rotate(x, [0], cos, sin, False) == x).all()
    got = orc.rotate(x, [1], cos, sin, False)[0, 0]            # (1, 3) a quarter turn, (2, 4) none
    assert got.tolist() == [-3, 2, 1, 4, 5, 6, 7, 8]
    got = orc.rotate(x, [1], cos, sin, True)[0, 0]             # (1, 2) a quarter turn
    assert got.tolist() == [-2, 1, 3, 4, 5, 6, 7, 8]


def test_attention_by_hand():
    """Equal keys: the mean of the values seen; one key: its value; none: nothing; the forms are the same function."""
    rows = np.zeros((32, 6))
    rows[:, 0] = np.arange(32.0)
    q = np.zeros((3, 1, 6))
    r = orc.attend(q, rows, [[0, 1]], 16, [20], [0, 3], 1.0, True, 4)
    assert np.allclose(r["out"][:, 0, 0], [np.arange(18).mean(), np.arange(19).mean(), np.arange(20).mean()])
    assert np.allclose(r["lse"][:, 0], np.log([18, 19, 20]))
    r = orc.attend(q, rows, [[0, -1]], 16, [20], [0, 3], 1.0, True, 4, causal=False)
    assert np.allclose(r["out"][:, 0, 0], np.arange(16).mean())
    r = orc.attend(q, rows, [[0, 1]], 16, [2], [0, 3], 1.0, True, 4)
    assert (r["out"][0] == 0).all() and np.isneginf(r["lse"][0]).all() and np.allclose(r["out"][1], 0)
    rng = np.random.default_rng(0)
    rows, q = rng.standard_normal((32, 6)), rng.standard_normal((3, 2, 5))
    wk, wv = rng.standard_normal((2, 3, 4)), rng.standard_normal((2, 7, 4))
    e = orc.attend(q, rows, [[1, 0]], 16, [25], [0, 3], 0.7, True, 4, w_k=wk, w_v=wv)
    lat = np.concatenate((np.einsum("bhn,hnr->bhr", q[..., :3], wk), q[..., 3:]), -1)
    a = orc.attend(lat, rows, [[1, 0]], 16, [25], [0, 3], 0.7, True, 4)
    assert np.allclose(np.einsum("bhr,hvr->bhv", a["out"], wv), e["out"])

"""What the quantised cache's calls refuse on the host, before any device call, and the
test oracle's own pins (no GPU)."""
import ctypes

import numpy as np
import pytest

import _kv_oracle as orc


@pytest.fixture(scope="module")
def lib():
    from paper_2607_05708_gb300 import _build, load_library
    _build.build()
    return load_library()


def _config(**kw):
    from paper_2607_05708_gb300 import _KVConfig
    c = dict(bits=4, heads=2, head_dim=128, block_tokens=64, n_blocks=8, device=0)
    c.update(kw)
    return ctypes.byref(_KVConfig(c["bits"], c["heads"], c["head_dim"], c["block_tokens"],
                                  c["n_blocks"], c["device"]))


BAD = [dict(bits=3), dict(bits=0), dict(heads=0), dict(heads=1025), dict(head_dim=96),
       dict(head_dim=0), dict(head_dim=512), dict(block_tokens=0), dict(block_tokens=24),
       dict(block_tokens=4112), dict(block_tokens=-16), dict(n_blocks=0), dict(n_blocks=-1),
       dict(n_blocks=1 << 40), dict(n_blocks=1 << 28, heads=1024), dict(device=-1)]


@pytest.mark.parametrize("bad", BAD, ids=lambda b: "_".join(f"{k}{v}" for k, v in b.items()))
def test_bad_configs(lib, bad):
    from paper_2607_05708_gb300 import _KVAttend
    size = ctypes.c_int64()
    assert lib.akashic_mem_kv_cache_bytes(_config(**bad), ctypes.byref(size)) == 1
    assert b"kv_cache_bytes" in lib.akashic_mem_last_error()
    assert lib.akashic_mem_kv_write(_config(**bad), 16, None, 16, 1, 1, 16, 1, 1, 0, 1, 16, None,
                                    None, None) == 1
    assert lib.akashic_mem_kv_read(_config(**bad), 16, 16, 1, 0, 16, 16, None, None) == 1
    a = _KVAttend(dtype=0, n_q=1, q_heads=2, n_seq=1, max_blocks=1)
    assert lib.akashic_mem_kv_attend(_config(**bad), 16, ctypes.byref(a), 16, 1 << 30, None, None) == 1


@pytest.mark.parametrize("bits,dim,token", [(4, 64, 74), (4, 128, 146), (4, 256, 290), (8, 64, 132),
                                            (8, 128, 260), (8, 256, 516)])
def test_cache_bytes(lib, bits, dim, token):
    """Codes, scales and exponents of keys and values: so many bytes a token and head."""
    size = ctypes.c_int64()
    assert lib.akashic_mem_kv_cache_bytes(_config(bits=bits, head_dim=dim, heads=3, n_blocks=5,
                                                  block_tokens=48), ctypes.byref(size)) == 0
    assert size.value == token * 3 * 5 * 48
    assert lib.akashic_mem_kv_cache_bytes(_config(), None) == 1


def test_bad_rows(lib):
    w, r = lib.akashic_mem_kv_write, lib.akashic_mem_kv_read
    c = _config()
    assert w(c, 16, None, 16, 1, 1, 16, 1, 1, 3, 1, 16, None, None, None) == 1     # dtype
    assert w(c, 16, None, 16, 1, 1, 16, 1, 1, 0, -1, 16, None, None, None) == 1    # n
    assert w(c, 16, None, 16, 1, 1, 16, 1, 1, 0, 1 << 31, 16, None, None, None) == 1
    assert w(c, None, None, 16, 1, 1, 16, 1, 1, 0, 1, 16, None, None, None) == 1   # NULL
    assert w(c, 16, None, 16, 1, 1, 16, 1, 1, 0, 1, None, None, None, None) == 1
    assert w(c, 24, None, 16, 1, 1, 16, 1, 1, 0, 1, 16, None, None, None) == 1     # alignment
    assert w(c, 16, None, 17, 1, 1, 16, 1, 1, 0, 1, 16, None, None, None) == 1
    assert w(c, 16, None, 16, 1, 1, 18, 1, 1, 2, 1, 16, None, None, None) == 1
    assert w(c, 16, None, 16, 1, 1, 16, 1, 1, 0, 1, 20, None, None, None) == 1
    assert w(c, 16, None, 16, 1, 1, 16, 1, 1, 0, 1, 16, 16, None, None) == 1       # tags
    assert w(c, None, None, None, 1, 1, None, 1, 1, 0, 0, None, None, None, None) == 0
    assert r(c, 16, 16, 1, 7, 16, 16, None, None) == 1
    assert r(c, 16, 16, -1, 0, 16, 16, None, None) == 1
    assert r(c, 16, 16, 1, 0, None, 16, None, None) == 1
    assert r(c, 16, 12, 1, 0, 16, 16, None, None) == 1
    assert r(c, None, None, 0, 0, None, None, None, None) == 0


ATTEND = [dict(dtype=2), dict(dtype=-1), dict(q_heads=0), dict(q_heads=3), dict(q_heads=4096),
          dict(n_seq=-1), dict(n_q=-1), dict(max_blocks=-1), dict(max_blocks=1 << 26),
          dict(n_q=3, n_seq=2), dict(n_q=1 << 28, q_heads=16), dict(scale=float("nan")),
          dict(scale=float("inf")), dict(cap=-1.0), dict(cap=1e-39), dict(cap=float("inf")), dict(cap=float("nan")),
          dict(tags=16), dict(q_tags=16)]


@pytest.mark.parametrize("bad", ATTEND, ids=lambda b: "_".join(f"{k}{v}" for k, v in b.items()))
def test_bad_attention(lib, bad):
    from paper_2607_05708_gb300 import _KVAttend
    kw = dict(dtype=0, n_q=2, q_heads=4, n_seq=2, max_blocks=3, q=16, blocks=16, out=16)
    kw.update(bad)
    a = _KVAttend(**kw)
    size = ctypes.c_int64()
    assert lib.akashic_mem_kv_attend_scratch(_config(), ctypes.byref(a), ctypes.byref(size)) == 1
    assert lib.akashic_mem_kv_attend(_config(), 16, ctypes.byref(a), 16, 1 << 40, None, None) == 1
    assert lib.akashic_mem_last_error()


def test_bad_attention_pointers(lib):
    from paper_2607_05708_gb300 import _KVAttend
    good = dict(dtype=0, n_q=2, q_heads=4, n_seq=2, max_blocks=3, q=16, blocks=16, out=16)
    call = lib.akashic_mem_kv_attend
    for bad in (dict(q=None), dict(out=None), dict(blocks=None), dict(q=17), dict(out=18),
                dict(blocks=20), dict(kv_len=18), dict(lse=2), dict(tags=20, q_tags=16)):
        a = _KVAttend(**{**good, **bad})
        assert call(_config(), 16, ctypes.byref(a), 16, 1 << 40, None, None) == 1, bad
    a = _KVAttend(**good)
    assert call(_config(), None, ctypes.byref(a), 16, 1 << 40, None, None) == 1
    assert call(_config(), 8, ctypes.byref(a), 16, 1 << 40, None, None) == 1
    assert call(_config(), 16, ctypes.byref(a), None, 1 << 40, None, None) == 1
    assert call(_config(), 16, ctypes.byref(a), 8, 1 << 40, None, None) == 1
    assert call(_config(), 16, None, 16, 1 << 40, None, None) == 1
    for none in (dict(n_q=0), dict(n_seq=0, n_q=0)):      # nothing to do
        a = _KVAttend(**{**good, **none, "q": None, "out": None, "blocks": None})
        assert call(_config(), None, ctypes.byref(a), None, 0, None, None) == 0


# ------------------------------------------------------------------ the oracle's pins
def test_stored_values_by_hand():
    x = np.zeros(64)
    x[:16] = 7.0                       # T = 0, e = 1: exact
    x[16], x[17] = 3.5, -0.25          # e = 1/2: 7 and -1/2 -> 0 (even)
    x[32] = 0.7                        # e = 0.1 -> 13/128, code 7
    got = orc.stored(x, 4)
    assert (got[:16] == 7).all() and got[16] == 3.5 and got[17] == 0 and got[32] == 7 * 13 / 128
    y = np.array([127.0, 63.5, -0.5, 1.5] + [0.0] * 60)
    assert orc.stored(y, 8)[:4].tolist() == [127.0, 64.0, 0.0, 2.0]


@pytest.mark.parametrize("bits", [4, 8])
def test_stored_values_are_near_and_kept(bits):
    """At most half a step of its group away; what is stored twice stays."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 64)) * np.exp2(rng.integers(-20, 20, (50, 1)))
    y = orc.stored(x, bits)
    if bits == 4:       # step: largest of the group / 7, times 1 + 2^-5 as the scale is rounded
        top = np.abs(x.reshape(50, 4, 16)).max(-1)
        step = np.repeat(top, 16, -1) / 7 * (1 + 2.0 ** -5)
    else:
        step = np.abs(x).max(-1, keepdims=True) / 127 * (1 + 2.0 ** -8)
    assert (np.abs(x - y) <= step / 2 * (1 + 2.0 ** -4)).all()
    assert (np.abs(orc.stored(y, bits) - y) <= step / 2 * (1 + 2.0 ** -4)).all()


def test_attention_oracle_closed_forms():
    """Equal keys: the mean of the values seen; one key: its value; none: nothing."""
    k = np.ones((32, 1, 64))
    v = np.arange(32.0)[:, None, None] * np.ones((1, 1, 64))
    q = np.ones((3, 1, 64))
    r = orc.attend(q, k, v, [[0, 1]], 16, [20], [0, 3], causal=True)
    assert np.allclose(r["out"][:, 0, 0], [np.arange(18).mean(), np.arange(19).mean(), np.arange(20).mean()])
    assert np.allclose(r["lse"][:, 0], 8 + np.log([18, 19, 20]))
    r = orc.attend(q, k, v, [[0, -1]], 16, [20], [0, 3], causal=False, prefix=[1])
    assert np.allclose(r["out"], np.arange(16).mean())
    r = orc.attend(q, k, v, [[0, 1]], 16, [2], [0, 3], causal=True)
    assert (r["out"][0] == 0).all() and np.isneginf(r["lse"][0]).all() and np.allclose(r["out"][1], 0)
    r = orc.attend(q, k, v, [[0, 1]], 16, [32], [0, 3], causal=False, slopes=[5.0], cap=2.0)
    w = np.exp(-5.0 * np.abs(np.array([29, 30, 31])[:, None] - np.arange(32)))
    assert np.allclose(r["out"][:, 0, 0], (w / w.sum(1, keepdims=True)) @ np.arange(32))

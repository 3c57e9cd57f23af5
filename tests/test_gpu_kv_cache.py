"""The quantised key and value cache on the GPU, against 64-bit restatements:
what is written and read back exactly, attention within bounds derived from the
kernels' roundings (_kv_oracle.tolerances)."""
import numpy as np
import pytest

import _kv_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2607_05708_gb300 import _build
    _build.build()


def _cache(*a, **k):
    from paper_2607_05708_gb300 import KVCache
    return KVCache(*a, **k)


def _gpu(a, dtype=None):
    t = torch.as_tensor(a)
    return (t if dtype is None else t.to(dtype)).cuda()


def _values(rng, n, heads, dim, dtype):
    """Rows of different sizes with large channels, rounded to dtype; float64 too."""
    x = rng.standard_normal((n, heads, dim)) * np.exp2(rng.integers(-3, 4, (n, heads, 1)))
    x *= np.where(rng.random((1, heads, dim)) < 0.06, 6.0, 1.0)
    t = torch.from_numpy(x).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def _expect(x, dtype):
    return torch.from_numpy(x).to(DT[dtype])


# ------------------------------------------------------------------ write and read
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bits", [4, 8])
def test_written_rows_read_back_as_the_format_says(bits, dim, dtype):
    rng = np.random.default_rng(bits * 1000 + dim)
    n, heads, T = 53, 3, 32
    c = _cache(5, heads, dim, block_tokens=T, bits=bits)
    k, k64 = _values(rng, n, heads, dim, dtype)
    v, v64 = _values(rng, n, heads, dim, dtype)
    slots = rng.permutation(5 * T)[:n]
    c.write(k, v, _gpu(slots))
    for out in ("bf16", "fp16", "fp32"):
        rk, rv = c.read(_gpu(slots), dtype=DT[out])
        assert torch.equal(rk.cpu(), _expect(orc.stored(k64, bits), out))
        assert torch.equal(rv.cpu(), _expect(orc.stored(v64, bits), out))
    c.sync()


def _special_rows(dim, rng):
    rows = [np.zeros(dim), np.full(dim, 1e-38), np.full(dim, 3.4e38), np.full(dim, -1.0)]
    r = rng.standard_normal(dim)
    r[3], r[20], r[40] = np.inf, -np.inf, np.nan
    rows.append(r)
    r = np.zeros(dim)
    r[5] = 2.0 ** -149                      # the smallest fp32
    rows.append(r)
    r = rng.standard_normal(dim) * 1e-20
    r[0] = 1e20                             # all but one group vanish beside it
    rows.append(r)
    rows.append(np.arange(dim) / 2.0)       # many exact halves of a step
    rows.append(np.where(np.arange(dim) % 16 == 0, 28.0, 27.0) * np.exp2(np.arange(dim) // 16))
    r = np.repeat([7 * (1 + m / 16 + 1 / 32) * 2.0 ** -e for m, e in
                   zip(range(16), range(16))], max(1, dim // 16))[:dim]
    r[0] = 13.0                             # scales halfway between two of the format's
    rows.append(r)
    rows.append(np.full(dim, np.nan))
    rows += [rng.standard_normal(dim) * 2.0 ** e for e in (-110, -102, -99, 60, 120)]
    # just below and above where the exponent steps
    rows += [np.full(dim, np.nextafter(np.float32(7 * 2.0 ** e), np.float32(s * 1e30)))
             for e in (-3, 0, 9) for s in (-1, 1)]
    return np.stack(rows).astype(np.float32)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("bits", [4, 8])
def test_special_rows(bits, dim):
    """Zeros, infinities, NaN, subnormals, exact half steps, the range's ends."""
    x = _special_rows(dim, np.random.default_rng(3))[:, None]
    n = len(x)
    c = _cache(3, 1, dim, block_tokens=16, bits=bits)
    slots = _gpu(np.arange(n))
    c.write(_gpu(x), _gpu(x[::-1].copy()), slots)
    k, v = c.read(slots, dtype=torch.float32)
    want = torch.from_numpy(orc.stored(x.astype(np.float64), bits)).float()
    assert torch.equal(k.cpu(), want)
    assert torch.equal(v.cpu(), want.flip(0))


@pytest.mark.parametrize("bits,dim", [(4, 128), (8, 64)])
def test_strided_and_unaligned_rows(bits, dim):
    """Any strides of the first two dimensions: heads first, rows inside a wider
    projection, an odd offset, a broadcast row."""
    rng = np.random.default_rng(9)
    n, heads = 21, 2
    c = _cache(4, heads, dim, block_tokens=16, bits=bits)
    base, _ = _values(rng, heads, n, dim, "bf16")
    wide, _ = _values(rng, n, 1, 2 * heads * dim + 3, "bf16")
    wide = wide.view(n, -1)
    one, _ = _values(rng, 1, heads, dim, "bf16")
    views = [base.transpose(0, 1),
             wide[:, :heads * dim].unflatten(1, (heads, dim)),
             wide[:, 3:3 + heads * dim].unflatten(1, (heads, dim)),
             one.expand(n, heads, dim),
             base.transpose(0, 1).flip(0)]
    slots = _gpu(rng.permutation(64)[:n])
    for a in views:
        for b in views:
            c.write(a, b, slots)
            k, v = c.read(slots, dtype=torch.float32)
            assert torch.equal(k.cpu(), torch.from_numpy(orc.stored(a.double().cpu().numpy(), bits)).float())
            assert torch.equal(v.cpu(), torch.from_numpy(orc.stored(b.double().cpu().numpy(), bits)).float())


@pytest.mark.parametrize("bits,dim,dtype", [(4, 64, "fp16"), (4, 128, "bf16"), (8, 256, "fp32")])
def test_skipped_rows_and_other_slots_stay(bits, dim, dtype):
    """Slot -1 writes nothing and reads zeros; slots not named keep their rows; tags
    follow their rows; n = 0 and n = 1."""
    rng = np.random.default_rng(4)
    heads, T, nb = 3, 16, 6
    c = _cache(nb, heads, dim, block_tokens=T, bits=bits, tagged=True)
    every = _gpu(np.arange(nb * T))
    k0, _ = _values(rng, nb * T, heads, dim, dtype)
    v0, _ = _values(rng, nb * T, heads, dim, dtype)
    tags0 = _gpu(np.arange(nb * T), torch.int32)
    c.write(k0, v0, every, tags=tags0)
    rk0, rv0 = c.read(every, dtype=torch.float32)
    for n in (0, 1, 37):
        k1, k64 = _values(rng, n, heads, dim, dtype)
        v1, v64 = _values(rng, n, heads, dim, dtype)
        slots = rng.permutation(nb * T)[:n]
        skip = rng.random(n) < 0.4
        given = np.where(skip, -1, slots)
        c.write(k1, v1, _gpu(given), tags=_gpu(np.full(n, 500 + n), torch.int32))
        rk, rv = c.read(_gpu(given), dtype=torch.float32)
        wk, wv = orc.stored(k64, bits), orc.stored(v64, bits)
        wk[skip] = 0
        wv[skip] = 0
        assert torch.equal(rk.cpu(), torch.from_numpy(wk).float().view_as(rk.cpu()))
        assert torch.equal(rv.cpu(), torch.from_numpy(wv).float().view_as(rv.cpu()))
        keep = np.setdiff1d(np.arange(nb * T), slots[~skip])
        ak, av = c.read(every, dtype=torch.float32)
        assert torch.equal(ak[keep], rk0[keep]) and torch.equal(av[keep], rv0[keep])
        want = tags0.clone()
        want[slots[~skip]] = 500 + n
        assert torch.equal(c.tags, want)
        c.write(k0, v0, every, tags=tags0)
    c.write(k0, v0, every)
    assert int(c.tags.abs().max()) == 0
    c.sync()


# ------------------------------------------------------------------ attention
def _problem(seed, *, bits=4, dim=128, heads=2, group=4, T=16, kv=(100,), nq=None, dtype="bf16",
             causal=True, prefix=None, cap=0.0, slopes=False, docs=0, holes=False, tail=0,
             kv_given=True, size=1.0, scale=0.0):
    """A cache with the sequences' tokens in shuffled blocks, the call's arguments, and
    the oracle's answer."""
    rng = np.random.default_rng(seed)
    S = len(kv)
    nq = nq or (1,) * S
    need = [-(-n // T) for n in kv]
    width = max(need + [1]) + 1
    nb = sum(need) + 3
    order = rng.permutation(nb)
    blocks = np.full((S, width), -1, np.int64)
    at = 0
    for s in range(S):
        blocks[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
    if holes:
        blocks[rng.random(blocks.shape) < 0.3] = -1
    c = _cache(nb, heads, dim, block_tokens=T, bits=bits, tagged=bool(docs))
    # what was there before must not matter: every byte pattern
    c.data.copy_(torch.from_numpy(rng.integers(0, 256, c.data.numel(), dtype=np.uint8)))
    k, k64 = _values(rng, nb * T, heads, dim, dtype)
    v, v64 = _values(rng, nb * T, heads, dim, dtype)
    used = np.zeros(nb * T, bool)
    for s in range(S):
        for j in range(kv[s]):
            if blocks[s, j // T] >= 0:
                used[blocks[s, j // T] * T + j % T] = True
    tags = np.where(used, rng.integers(0, max(docs, 1), nb * T), -1).astype(np.int32)
    if docs:
        used &= rng.random(nb * T) < 0.9
        tags[~used] = -1
    slots = np.where(used, np.arange(nb * T), -1)
    c.write(k, v, _gpu(slots), tags=_gpu(tags) if docs else None)
    n_q = sum(nq) + tail
    q = torch.from_numpy(rng.standard_normal((n_q, heads * group, dim)) * size).to(DT[dtype])
    q_start = np.cumsum([0] + list(nq)).astype(np.int32)
    args = dict(causal=causal, cap=cap, scale=scale)
    ref = dict(causal=causal, cap=cap, scale=scale)
    if kv_given:
        args["kv_len"] = _gpu(np.array(kv, np.int32))
        lens = kv
    else:
        lens = [width * T] * S
    if len(set(nq)) > 1 or tail:
        args["q_start"] = _gpu(q_start)
    if prefix is not None:
        args["prefix_len"] = _gpu(np.array(prefix, np.int32))
        ref["prefix"] = prefix
    if slopes:
        sl = np.exp2(-np.arange(1, heads * group + 1) * 8.0 / (heads * group)).astype(np.float32)
        args["slopes"] = _gpu(sl)
        ref["slopes"] = sl.astype(np.float64)
    if docs:
        qt = rng.integers(-1, docs, n_q).astype(np.int32)
        args["q_tags"] = _gpu(qt)
        ref.update(tags=tags, q_tags=qt)
    want = orc.attend(q.double().numpy(), orc.stored(k64, bits), orc.stored(v64, bits), blocks, T,
                      lens, q_start, **ref)
    return c, q.cuda(), _gpu(blocks), args, want


def _compare(got, want, dim, dtype, bits, rows=None):
    out, lse = (x.double().cpu().numpy()[:rows] for x in got)
    want = {k: v[:rows] for k, v in want.items()}
    t_out, t_lse = orc.tolerances(want, dim, torch.finfo(DT[dtype]).eps / 2, bits)
    empty = np.isneginf(want["lse"])
    assert (out[empty] == 0).all() and np.isneginf(lse[empty]).all()
    assert np.isfinite(out).all() and np.isfinite(lse[~empty]).all()
    worst = (np.abs(out - want["out"]) / t_out).max(initial=0)
    assert worst <= 1, f"out is {worst:.2f} of its bound"
    worst = (np.abs(lse[~empty] - want["lse"][~empty]) / t_lse[~empty]).max(initial=0)
    assert worst <= 1, f"lse is {worst:.2f} of its bound"


CASES = {
    "one_token": dict(kv=(1,)),
    "fifteen": dict(kv=(15,)),
    "sixteen": dict(kv=(16,)),
    "seventeen": dict(kv=(17,)),
    "long": dict(kv=(1900,), heads=1),
    "ragged": dict(kv=(5, 300, 64, 1, 129), T=32),
    "none_at_all": dict(kv=(0, 40, 0)),
    "group1": dict(kv=(200, 90), group=1, heads=3),
    "group7": dict(kv=(77, 210), group=7, heads=1, T=64),
    "group9": dict(kv=(77, 310), group=9, heads=1),
    "group20": dict(kv=(150,), group=20, heads=2),
    "draft3": dict(kv=(60, 200), nq=(3, 3)),
    "draft_ragged": dict(kv=(60, 200, 9, 33), nq=(3, 1, 0, 5), tail=2),
    "more_rows_than_keys": dict(kv=(3, 2), nq=(5, 5)),
    "prompt": dict(kv=(70, 41), nq=(70, 41), group=2),
    "prompt_prefix": dict(kv=(90, 41, 30), nq=(30, 41, 30), prefix=(60, 20, 0)),
    "not_causal": dict(kv=(50, 33), nq=(7, 7), causal=False),
    "cap": dict(kv=(120,), cap=4.0, size=3.0),
    "slopes": dict(kv=(140, 35), nq=(2, 2), slopes=True),
    "prefix_slopes_cap": dict(kv=(100,), nq=(9,), slopes=True, cap=20.0, prefix=(95,)),
    "documents": dict(kv=(130, 47), nq=(4, 4), docs=3),
    "documents_prefix": dict(kv=(130, 47), nq=(4, 20), docs=2, prefix=(130, 33), holes=True),
    "holes": dict(kv=(170, 300), holes=True, T=16),
    "all_listed": dict(kv=(64, 48), kv_given=False, causal=False, docs=2),
    "sharp": dict(kv=(500,), size=12.0),
    "scaled": dict(kv=(90,), scale=-0.03),
    "block128": dict(kv=(300, 129), T=128),
    "long_prompt": dict(kv=(400,), nq=(400,), heads=1, group=1, T=64),
    "wide_group": dict(kv=(333, 40), nq=(90, 90), heads=1, group=3, T=32, causal=False),
    "few_of_many": dict(kv=(700, 530), nq=(20, 20), heads=1, group=2, T=64),
    "mixed_rows": dict(kv=(300, 90, 200, 31, 150), nq=(1, 90, 3, 31, 150), heads=1, group=2, tail=3),
    "long_documents": dict(kv=(520,), nq=(300,), heads=1, group=1, docs=2, prefix=(300,)),
    "long_cap_slopes": dict(kv=(300,), nq=(140,), heads=1, group=2, cap=6.0, slopes=True, size=2.0),
    "many": dict(kv=tuple(range(1, 300, 7)), heads=1),
}


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("bits,dim,dtype", [(4, 128, "bf16"), (4, 64, "fp16"), (4, 256, "bf16"),
                                            (8, 128, "fp16"), (8, 64, "bf16"), (8, 256, "fp16")])
def test_attention(name, bits, dim, dtype):
    kw = dict(CASES[name])
    c, q, blocks, args, want = _problem(sum(map(ord, name)), bits=bits, dim=dim, dtype=dtype, **kw)
    n = sum(kw.get("nq") or (1,) * len(kw["kv"]))
    got = c.attend(q, blocks, **args)
    c.sync()
    _compare(got, want, dim, dtype, bits, rows=n)


LONG = {   # many steps for every worker: rings go round, several items in a row, items shared
    "prompt": dict(kv=(1400, 900), nq=(1400, 700), heads=2, group=2, T=64),
    "prompt_packed": dict(kv=(2100,), nq=(2100,), heads=2, group=3, T=32, docs=5, prefix=(900,)),
    "prompt_cap_slopes": dict(kv=(1500, 60), nq=(1200, 60), heads=2, group=2, T=128, cap=9.0,
                              slopes=True),
    "mixed": dict(kv=(3000, 800, 1, 1300, 2500), nq=(1, 800, 1, 1, 600), heads=2, group=4, T=32),
    "decode_long": dict(kv=(60_000, 33, 21_000), heads=3, group=5, T=64),
    "decode_many": dict(kv=tuple(900 + 37 * i for i in range(60)), heads=4, group=2, T=16),
    "decode_tags": dict(kv=(20_000, 5_000, 17_777), heads=4, group=1, T=64, docs=3, holes=True),
    "draft_long": dict(kv=(30_000, 11_111), nq=(3, 3), heads=4, group=4, T=64, slopes=True, cap=15.0),
}


@pytest.mark.parametrize("name", LONG)
@pytest.mark.parametrize("bits,dim,dtype", [(4, 128, "bf16"), (8, 64, "fp16"), (4, 256, "fp16"),
                                            (8, 128, "bf16"), (4, 64, "bf16"), (8, 256, "bf16")])
def test_attention_with_many_steps(name, bits, dim, dtype):
    kw = LONG[name]
    c, q, blocks, args, want = _problem(sum(map(ord, name)), bits=bits, dim=dim, dtype=dtype, **kw)
    got = c.attend(q, blocks, **args)
    c.sync()
    _compare(got, want, dim, dtype, bits, rows=sum(kw.get("nq") or (1,) * len(kw["kv"])))


def test_attention_rounds_no_small_rows_away():
    """Values of very different sizes between tokens, the small ones with the weight."""
    rng = np.random.default_rng(8)
    T, n, dim = 16, 96, 128
    c = _cache(6, 1, dim, block_tokens=T)
    k = rng.standard_normal((n, 1, dim))
    v = rng.standard_normal((n, 1, dim)) * np.where(np.arange(n) % 5 == 0, 1.0, 2.0 ** -12)[:, None, None]
    q = rng.standard_normal((1, 1, dim))
    k[np.arange(n) % 5 == 0] -= 4 * q / np.linalg.norm(q) ** 2 * dim ** 0.5
    kt, vt, qt = (torch.from_numpy(x).bfloat16() for x in (k, v, q))
    c.write(kt.cuda(), vt.cuda(), _gpu(np.arange(n)))
    blocks = np.arange(6)[None]
    got = c.attend(qt.cuda(), _gpu(blocks))
    want = orc.attend(qt.double().numpy(), orc.stored(kt.double().numpy(), 4),
                      orc.stored(vt.double().numpy(), 4), blocks, T, [n], [0, 1])
    _compare(got, want, dim, "bf16", 4)

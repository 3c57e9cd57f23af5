"""Rows rotated to their positions on the way into the caches, against 64-bit and 32-bit
restatements: what is stored and the query rows, exactly."""
import numpy as np
import pytest

import _kv_oracle as kv
import _latent_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_05708_gb300 import _build
    _build.build()


def _gpu(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def _rand(rng, shape, dtype):
    return torch.from_numpy(rng.standard_normal(shape)).to(DT[dtype])


def _table(rng, rows, half):
    angle = rng.uniform(-4, 4, (rows, half))
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


def _error(c):
    from paper_2607_05708_gb300 import AkashicError
    with pytest.raises(AkashicError) as e:
        c.sync()
    c.sync()                               # cleared
    return e.value.code


def _turned(x, positions, cos, sin, pairs, dtype=None):
    y = torch.from_numpy(orc.rotate(x.float().numpy(), positions, cos, sin, pairs))
    return y if dtype is None else y.to(dtype)


@pytest.mark.parametrize("n,heads,qh,dim,bits,dtype,rotary,pairs", [
    (1, 8, 32, 128, 4, "bf16", 128, False), (1, 1, 1, 64, 8, "fp16", 64, True),
    (37, 3, 6, 64, 4, "fp32", 32, True), (129, 5, 5, 256, 4, "fp16", 256, True),
    (300, 2, 14, 128, 8, "bf16", 64, False), (65, 1, 7, 256, 8, "fp32", 96, False),
    (17, 40, 40, 64, 4, "bf16", 64, True), (2000, 2, 4, 128, 4, "fp32", 128, False)])
def test_stored_values_and_queries(n, heads, qh, dim, bits, dtype, rotary, pairs):
    from paper_2607_05708_gb300 import KVCache
    rng = np.random.default_rng(n + dim)
    c = KVCache(-(-n // 16) + 2, heads, dim, block_tokens=16, bits=bits, tagged=True)
    k, v = _rand(rng, (n, heads, dim), dtype) * 3, _rand(rng, (n, heads, dim), dtype)
    q = _rand(rng, (n, qh, dim), dtype)
    cos, sin = _table(rng, 500, rotary // 2)
    pos = rng.integers(0, 500, n)
    pos[0] = 499
    slots = rng.permutation(c.n_blocks * 16)[:n]
    slots[2::5] = -1
    pos[2::5] = -77                        # not read
    real = slots >= 0
    tags = rng.integers(0, 9, n).astype(np.int32)
    out = c.append(k.cuda(), v.cuda(), _gpu(slots), _gpu(pos), _gpu(cos), _gpu(sin), q=q.cuda(),
                   interleaved=pairs, tags=_gpu(tags))
    c.sync()
    safe = np.where(real, pos, 0)
    want = _turned(q, safe, cos, sin, pairs, DT[dtype])
    want[~torch.from_numpy(real)] = 0
    assert torch.equal(out.cpu(), want)
    rk, rv = c.read(_gpu(slots), dtype=torch.float32)
    kw = kv.stored(_turned(k, safe, cos, sin, pairs).double().numpy(), bits)
    vw = kv.stored(v.double().numpy(), bits)
    kw[~real], vw[~real] = 0, 0
    assert torch.equal(rk.cpu(), torch.from_numpy(kw).float())
    assert torch.equal(rv.cpu(), torch.from_numpy(vw).float())
    got = c.tags.cpu().numpy()
    assert (got[slots[real]] == tags[real]).all() and (np.delete(got, slots[real]) == -1).all()


def test_angle_zero_is_write():
    """The same bytes as write() where every angle is 0."""
    from paper_2607_05708_gb300 import KVCache
    rng = np.random.default_rng(0)
    k, v = _rand(rng, (90, 4, 128), "bf16").cuda(), _rand(rng, (90, 4, 128), "bf16").cuda()
    cos, sin = torch.ones(2, 64).cuda(), torch.zeros(2, 64).cuda()
    slots, pos = torch.arange(90).cuda(), torch.ones(90, dtype=torch.int64).cuda()
    a, b = KVCache(6, 4, 128, block_tokens=16), KVCache(6, 4, 128, block_tokens=16)
    a.data.zero_(), b.data.zero_()
    a.write(k, v, slots)
    assert b.append(k, v, slots, pos, cos, sin) is None
    assert torch.equal(a.data, b.data)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_strided_and_in_place(pairs, shift):
    """q, k and v are slices of one projection; q is turned where it lies (shift: off 16-byte
    alignment)."""
    from paper_2607_05708_gb300 import KVCache
    rng = np.random.default_rng(3)
    n, hq, h, d = 50, 6, 2, 64
    flat = torch.zeros(n * (hq + 2 * h) * d + 8, dtype=torch.bfloat16)
    flat[:] = _rand(rng, flat.shape, "bf16")
    dev = flat.cuda()
    host = flat[shift:shift + n * (hq + 2 * h) * d].view(n, hq + 2 * h, d)
    proj = dev[shift:shift + n * (hq + 2 * h) * d].view(n, hq + 2 * h, d)
    cos, sin = _table(rng, 60, d // 2)
    pos, slots = np.arange(n) + 3, np.arange(n) * 2
    c = KVCache(7, h, d, block_tokens=16, bits=8)
    q = proj[:, :hq]
    assert c.append(proj[:, hq:hq + h], proj[:, hq + h:], _gpu(slots), _gpu(pos), _gpu(cos), _gpu(sin), q=q,
                    q_out=q, interleaved=pairs) is q
    assert torch.equal(q.cpu(), _turned(host[:, :hq], pos, cos, sin, pairs, torch.bfloat16))
    assert torch.equal(proj[:, hq:].cpu(), host[:, hq:])       # not touched
    rk, rv = c.read(_gpu(slots), dtype=torch.float32)
    k = _turned(host[:, hq:hq + h], pos, cos, sin, pairs).double().numpy()
    assert torch.equal(rk.cpu(), torch.from_numpy(kv.stored(k, 8)).float())
    assert torch.equal(rv.cpu(), torch.from_numpy(kv.stored(host[:, hq + h:].double().numpy(), 8)).float())


def test_bad_positions_and_slots_are_reported_and_skipped():
    from paper_2607_05708_gb300 import KVCache, LatentCache
    rng = np.random.default_rng(4)
    cos, sin = _table(rng, 10, 32)
    k = _rand(rng, (3, 2, 64), "bf16")
    for bad_slot, bad_pos in ((5, 10), (5, -1), (5, 1 << 40), (48, 3), (-2, 3), (1 << 34, 3)):
        c = KVCache(3, 2, 64, block_tokens=16, tagged=True)
        c.write(torch.zeros_like(k).cuda().expand(3, 2, 64), torch.zeros_like(k).cuda(), _gpu(np.array([4, 5, 6])))
        slots, pos = np.array([4, bad_slot, 6]), np.array([1, bad_pos, 2])
        out = c.append(k.cuda(), k.cuda(), _gpu(slots), _gpu(pos), _gpu(cos), _gpu(sin), q=k.cuda(),
                       tags=_gpu(np.array([7, 8, 9], np.int32)))
        assert _error(c) == "EDEVICE"
        want = _turned(k, np.array([1, 0, 2]), cos, sin, False, torch.bfloat16)
        want[1] = 0
        assert torch.equal(out.cpu(), want)
        rk, _ = c.read(_gpu(np.array([4, 5, 6])), dtype=torch.float32)
        assert (rk[1] == 0).all() and (rk[0] != 0).any() and c.tags[5] == 0 and c.tags[4] == 7
        m = LatentCache(3, 128, 64, block_tokens=16, tagged=True)
        lat = _rand(rng, (3, 128), "bf16")
        out = m.append(lat.cuda(), k[:, 0].cuda(), _gpu(slots), _gpu(pos), _gpu(cos), _gpu(sin), q=k.cuda(),
                       tags=_gpu(np.array([7, 8, 9], np.int32)))
        assert _error(m) == "EDEVICE"
        assert torch.equal(out.cpu(), want)
        data = m.data.cpu()
        assert torch.equal(data[[4, 6], :128], lat[[0, 2]]) and (data[5] == 0).all()
        assert m.tags[4] == 7 and m.tags[5] == -1


def test_what_is_not_finite():
    """As write(): NaN is stored as 0, infinities as the largest value."""
    from paper_2607_05708_gb300 import KVCache, LatentCache
    k = torch.ones(2, 1, 64)
    k[0, 0, 0], k[0, 0, 40], k[1, 0, 5] = float("inf"), float("nan"), -float("inf")
    cos, sin = torch.ones(1, 32).cuda(), torch.zeros(1, 32).cuda()
    pos, slots = torch.zeros(2, dtype=torch.int64).cuda(), torch.arange(2).cuda()
    c = KVCache(1, 1, 64, block_tokens=16, bits=8)
    c.append(k.cuda(), k.cuda(), slots, pos, cos, sin)
    rk, _ = c.read(slots, dtype=torch.float32)
    assert torch.isfinite(rk).all()
    for dt, most in ((torch.bfloat16, 3.3895313892515355e38), (torch.float16, 65504.0)):
        m = LatentCache(1, 128, 64, block_tokens=16, dtype=dt)
        lat = torch.ones(2, 128)
        lat[0, 0], lat[0, 1], lat[1, 2], lat[1, 3] = float("inf"), float("nan"), -float("inf"), 3.4e38
        m.append(lat.cuda(), k[:, 0].cuda(), slots)
        d = m.data.float().cpu()
        assert d[0, 0] == most and d[0, 1] == 0 and d[1, 2] == -most and d[1, 3] == most
        assert d[0, 128] == most and d[0, 168] == 0 and d[1, 133] == -most and torch.isfinite(d).all()


@pytest.mark.parametrize("n,R,P,qh,dtype,stored,pairs", [
    (1, 512, 64, 16, "bf16", "bf16", True), (1, 128, 32, 1, "fp32", "fp16", False),
    (37, 256, 64, 5, "fp16", "fp16", False), (300, 512, 32, 32, "bf16", "fp16", True),
    (1001, 128, 64, 3, "fp32", "bf16", True), (48, 512, 64, 64, "bf16", "bf16", False)])
def test_latent_rows(n, R, P, qh, dtype, stored, pairs):
    from paper_2607_05708_gb300 import LatentCache
    rng = np.random.default_rng(n + R)
    c = LatentCache(-(-n // 48) + 2, R, P, block_tokens=48, dtype=DT[stored], tagged=True)
    both = _rand(rng, (n, R + P + 3), dtype)           # slices of one projection, unaligned
    lat, k, q = both[:, 1:R + 1], both[:, R + 1:R + P + 1], _rand(rng, (n, qh, P + 16), dtype)[..., 5:5 + P]
    cos, sin = _table(rng, 99, P // 2)
    pos, slots = rng.integers(0, 99, n), rng.permutation(c.n_blocks * 48)[:n]
    slots[1::4] = -1
    real = slots >= 0
    dev, qd = both.cuda(), q.cuda()
    out = c.append(dev[:, 1:R + 1], dev[:, R + 1:R + P + 1], _gpu(slots), _gpu(pos), _gpu(cos), _gpu(sin),
                   q=qd, interleaved=pairs)
    c.sync()
    want = _turned(q, pos, cos, sin, pairs, DT[dtype])
    want[~torch.from_numpy(real)] = 0
    assert torch.equal(out.cpu(), want)
    rows = torch.zeros(c.n_blocks * 48, R + P, dtype=DT[stored])
    turned = _turned(k[:, None], pos, cos, sin, pairs)[:, 0]
    rows[slots[real]] = torch.cat((lat.float(), turned), 1).to(DT[stored])[real]
    assert torch.equal(c.data.cpu(), rows)
    assert (c.tags.cpu().numpy()[slots[real]] == 0).all() and int((c.tags == -1).sum()) == c.n_blocks * 48 - real.sum()
    # without rotation
    c.append(lat.cuda(), k.cuda(), _gpu(slots))
    rows[slots[real], R:] = k.float().to(DT[stored])[real]
    assert torch.equal(c.data.cpu(), rows)


def test_graphs_and_streams():
    """Captured and replayed with other inputs in the same tensors; on a stream of its own."""
    from paper_2607_05708_gb300 import KVCache
    rng = np.random.default_rng(8)
    c = KVCache(4, 2, 64, block_tokens=16)
    k, v, q = (torch.zeros(9, h, 64, dtype=torch.bfloat16, device="cuda") for h in (2, 2, 4))
    slots, pos = torch.zeros(9, dtype=torch.int64, device="cuda"), torch.zeros(9, dtype=torch.int64, device="cuda")
    cos, sin = _table(rng, 30, 32)
    dc, ds, out = _gpu(cos), _gpu(sin), torch.empty_like(q)
    slots.copy_(torch.arange(9))
    c.append(k, v, slots, pos, dc, ds, q=q, q_out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.append(k, v, slots, pos, dc, ds, q=q, q_out=out)
    for _ in range(2):
        new = [_rand(rng, tuple(t.shape), "bf16") for t in (k, v, q)]
        for t, x in zip((k, v, q), new):
            t.copy_(x)
        s, p = rng.permutation(64)[:9], rng.integers(0, 30, 9)
        slots.copy_(torch.from_numpy(s)), pos.copy_(torch.from_numpy(p))
        g.replay()
        assert torch.equal(out.cpu(), _turned(new[2], p, cos, sin, False, torch.bfloat16))
        rk, _ = c.read(slots, dtype=torch.float32)
        assert torch.equal(rk.cpu(), torch.from_numpy(kv.stored(_turned(new[0], p, cos, sin, False).double().numpy(), 4)).float())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = c.append(k, v, slots, pos, dc, ds, q=q, stream=st)
    c.sync(st)
    assert torch.equal(got, out)


def test_nothing_to_append():
    from paper_2607_05708_gb300 import KVCache, LatentCache
    e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")         # noqa: E731
    i = torch.empty(0, dtype=torch.int64, device="cuda")
    t = torch.ones(1, 32, device="cuda")
    assert KVCache(1, 2, 64).append(e(0, 2, 64), e(0, 2, 64), i, i, t, t, q=e(0, 4, 64)).shape == (0, 4, 64)
    assert LatentCache(1, 128, 64).append(e(0, 128), e(0, 64), i, i, t, t, q=e(0, 4, 64)).shape == (0, 4, 64)


def test_tensors_that_are_refused():
    from paper_2607_05708_gb300 import KVCache, LatentCache
    c, m = KVCache(2, 2, 64, block_tokens=16), LatentCache(2, 128, 64, block_tokens=16)
    e = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d, device="cuda")    # noqa: E731
    slots, pos, t = torch.arange(3).cuda(), torch.zeros(3, dtype=torch.int64).cuda(), torch.ones(4, 32).cuda()
    good = dict(k=e(3, 2, 64), v=e(3, 2, 64), slots=slots, positions=pos, cos=t, sin=t)
    c.append(**good)
    for bad in (dict(k=e(3, 3, 64)), dict(v=e(2, 2, 64)), dict(v=e(3, 2, 64, d=torch.float16)), dict(cos=t[:3]),
                dict(cos=None), dict(positions=pos[:2]), dict(positions=None), dict(q=e(2, 4, 64)), dict(q=e(3, 4, 32)),
                dict(q=e(3, 4, 64, d=torch.float32)), dict(q_out=e(3, 4, 64)), dict(slots=slots.cpu()),
                dict(q=e(3, 4, 64), q_out=e(3, 5, 64)), dict(tags=slots.int()), dict(cos=t.t(), sin=t.t())):
        with pytest.raises((ValueError, TypeError)):
            c.append(**{**good, **bad})
    from paper_2607_05708_gb300 import AkashicError
    for half in (8, 24, 64):               # not a multiple of 32, or wider than the head
        w = torch.ones(4, half).cuda()
        with pytest.raises(AkashicError):
            c.append(**{**good, "cos": w, "sin": w})
    good = dict(latent=e(3, 128), k_rope=e(3, 64), slots=slots)
    m.append(**good)
    for bad in (dict(latent=e(3, 64)), dict(k_rope=e(3, 32)), dict(k_rope=e(2, 64)), dict(positions=pos),
                dict(q=e(3, 2, 64)), dict(k_rope=e(3, 64, d=torch.float32)), dict(tags=slots.int())):
        with pytest.raises((ValueError, TypeError)):
            m.append(**{**good, **bad})
    for half in (16, 64):
        w = torch.ones(4, half).cuda()
        with pytest.raises(AkashicError):
            m.append(**good, positions=pos, cos=w, sin=w)

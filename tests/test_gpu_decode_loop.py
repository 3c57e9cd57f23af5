"""Decoding as it runs in an engine: a captured step that appends one token of every request, its key
and query rows rotated, and attends over what is there, replayed while the requests grow; against
64-bit restatements."""
import numpy as np
import pytest

import _kv_oracle as kv
import _latent_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_05708_gb300 import _build
    _build.build()


def _gpu(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _rand(rng, shape, dt):
    return torch.from_numpy(rng.standard_normal(shape)).to(DT[dt])


def _turn(x, pos, cos, sin, pairs, dtype=None):
    y = torch.from_numpy(orc.rotate(x.float().numpy(), pos, cos, sin, pairs))
    return y if dtype is None else y.to(dtype)


class Requests:
    """Requests of `start` tokens, their blocks in an order of their own, and the tensors that a step
    reads: slots, positions and lengths."""

    def __init__(self, rng, start, T, steps, half):
        self.len, self.T = list(start), T
        need = [-(-(n + steps) // T) for n in start]
        order = rng.permutation(sum(need) + 2)
        self.n_blocks = len(order)
        self.blocks = np.full((len(start), max(need)), -1, np.int64)
        at = 0
        for i, m in enumerate(need):
            self.blocks[i, :m] = order[at:at + m]
            at += m
        angle = np.arange(max(start) + steps)[:, None] * 100.0 ** (-np.arange(half) / half)
        self.cos, self.sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
        self.slots, self.pos = (torch.zeros(len(start), dtype=torch.int64, device="cuda") for _ in range(2))
        self.kv_len = torch.zeros(len(start), dtype=torch.int32, device="cuda")

    def slot(self, i, j):
        return self.blocks[i, j // self.T] * self.T + j % self.T

    def all_slots(self):
        return (np.array([self.slot(i, j) for i, n in enumerate(self.len) for j in range(n)]),
                np.array([j for n in self.len for j in range(n)]))

    def grow(self):
        slots, pos = np.array([self.slot(i, n) for i, n in enumerate(self.len)]), np.array(self.len)
        self.len = [n + 1 for n in self.len]
        self.slots.copy_(torch.from_numpy(slots)), self.pos.copy_(torch.from_numpy(pos))
        self.kv_len.copy_(torch.tensor(self.len, dtype=torch.int32))
        return slots, pos


def _capture(step):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                             # once before the capture
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    return g, out


@pytest.mark.parametrize("dt,R,heads,pairs", [("bf16", 512, 40, True), ("fp16", 128, 16, False)])
def test_latent(dt, R, heads, pairs):
    from paper_2607_05708_gb300 import LatentCache
    rng = np.random.default_rng(R)
    P, T, start, steps = 64, 16, [5, 63, 130, 1], 4
    r = Requests(rng, start, T, steps, P // 2)
    c = LatentCache(r.n_blocks, R, P, block_tokens=T, dtype=DT[dt])
    cos, sin, B = _gpu(r.cos), _gpu(r.sin), len(start)
    slots, pos = r.all_slots()
    lat, k = _rand(rng, (len(slots), R), dt), _rand(rng, (len(slots), P), dt)
    c.append(lat.cuda(), k.cuda(), _gpu(slots), _gpu(pos), cos, sin, interleaved=pairs)
    rows = torch.zeros(r.n_blocks * T, R + P, dtype=DT[dt])
    rows[slots] = torch.cat((lat, _turn(k[:, None], pos, r.cos, r.sin, pairs, DT[dt])[:, 0]), 1)
    x, q = (torch.zeros(B, w, dtype=DT[dt], device="cuda") for w in (R + P, heads * (R + P)))
    q, lists, scale = q.view(B, heads, R + P), _gpu(r.blocks), (R + P) ** -0.5

    def step():
        c.append(x[:, :R], x[:, R:], r.slots, r.pos, cos, sin, q=q[..., R:], q_out=q[..., R:], interleaved=pairs)
        return c.attend(q, lists, scale, kv_len=r.kv_len)

    r.slots.fill_(-1)                      # (the call before the capture stores nothing)
    g, (out, lse) = _capture(step)
    for _ in range(steps):
        nx, nq = _rand(rng, (B, R + P), dt), _rand(rng, (B, heads, R + P), dt)
        slots, pos = r.grow()
        x.copy_(nx), q.copy_(nq)
        g.replay()
        c.sync()
        rows[slots] = torch.cat((nx[:, :R], _turn(nx[:, None, R:], pos, r.cos, r.sin, pairs, DT[dt])[:, 0]), 1)
        assert torch.equal(c.data.cpu(), rows)
        nq[..., R:] = _turn(nq[..., R:], pos, r.cos, r.sin, pairs, DT[dt])
        assert torch.equal(q.cpu(), nq)
        want = orc.attend(nq.double().numpy(), rows.double().numpy(), r.blocks, T, r.len, np.arange(B + 1), scale,
                          dt == "bf16", R)
        assert (np.abs(out.double().cpu().numpy() - want["out"]) <= want["tol"]).all()
        assert (np.abs(lse.double().cpu().numpy() - want["lse"]) <= want["tol_lse"]).all()


@pytest.mark.parametrize("bits,dim,heads,q_heads,pairs", [(4, 128, 2, 14, False), (8, 64, 3, 3, True)])
def test_keys_and_values(bits, dim, heads, q_heads, pairs):
    from paper_2607_05708_gb300 import KVCache
    rng = np.random.default_rng(bits)
    T, start, steps = 16, [5, 63, 130, 1], 4
    r = Requests(rng, start, T, steps, dim // 2)
    c = KVCache(r.n_blocks, heads, dim, block_tokens=T, bits=bits)
    cos, sin, B = _gpu(r.cos), _gpu(r.sin), len(start)
    slots, pos = r.all_slots()
    k, v = (_rand(rng, (len(slots), heads, dim), "bf16") for _ in range(2))
    c.append(k.cuda(), v.cuda(), _gpu(slots), _gpu(pos), cos, sin, interleaved=pairs)
    keys, values = (np.zeros((r.n_blocks * T, heads, dim)) for _ in range(2))
    keys[slots] = kv.stored(_turn(k, pos, r.cos, r.sin, pairs).double().numpy(), bits)
    values[slots] = kv.stored(v.double().numpy(), bits)
    new = torch.zeros(2, B, heads, dim, dtype=torch.bfloat16, device="cuda")
    q, lists = torch.zeros(B, q_heads, dim, dtype=torch.bfloat16, device="cuda"), _gpu(r.blocks)

    def step():
        c.append(new[0], new[1], r.slots, r.pos, cos, sin, q=q, q_out=q, interleaved=pairs)
        return c.attend(q, lists, kv_len=r.kv_len)

    r.slots.fill_(-1)
    g, (out, lse) = _capture(step)
    for _ in range(steps):
        nk, nv, nq = (_rand(rng, (B, h, dim), "bf16") for h in (heads, heads, q_heads))
        slots, pos = r.grow()
        new.copy_(torch.stack((nk, nv))), q.copy_(nq)
        g.replay()
        c.sync()
        keys[slots] = kv.stored(_turn(nk, pos, r.cos, r.sin, pairs).double().numpy(), bits)
        values[slots] = kv.stored(nv.double().numpy(), bits)
        nq = _turn(nq, pos, r.cos, r.sin, pairs, torch.bfloat16)
        assert torch.equal(q.cpu(), nq)
        want = kv.attend(nq.double().numpy(), keys, values, r.blocks, T, r.len, np.arange(B + 1))
        t_out, t_lse = kv.tolerances(want, dim, 2.0 ** -8, bits)
        assert (np.abs(out.double().cpu().numpy() - want["out"]) <= t_out).all()
        assert (np.abs(lse.double().cpu().numpy() - want["lse"]) <= t_lse).all()

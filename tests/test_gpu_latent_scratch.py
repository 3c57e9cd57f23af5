"""The latent attention's calls with scratch as the C ABI promises it: 16-byte aligned, no larger than asked
for, whatever stands in it, and nothing written around it."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2607_05708_gb300 import _build, load_library
    _build.build()
    return load_library()


def _problem(dt, nope, value, tags, kv, nq, listed, H=3, R=128, P=32, T=32):
    from paper_2607_05708_gb300 import LatentCache
    rng = np.random.default_rng(31)
    S, n_blocks = len(kv), 48
    c = LatentCache(n_blocks, R, P, block_tokens=T, dtype=dt, tagged=tags)
    rows = torch.from_numpy(rng.standard_normal((n_blocks * T, R + P))).to(dt).cuda()
    c.append(rows[:, :R], rows[:, R:], torch.arange(n_blocks * T, device="cuda"),
             tags=torch.from_numpy(rng.integers(0, 2, n_blocks * T).astype(np.int32)).cuda() if tags else None)
    blocks = np.full((S, listed), -1, np.int64)
    for i, n in enumerate(kv):
        m = -(-n // T)
        blocks[i, :m] = rng.permutation(n_blocks)[:m]
    n_q = sum(nq)
    q = torch.from_numpy(rng.standard_normal((n_q, H, nope + P))).to(dt).cuda()
    wide = torch.from_numpy(rng.standard_normal((n_q, H, R + P))).to(dt).cuda()
    w = torch.from_numpy(rng.standard_normal((H, nope + value, R)) * R ** -0.5).to(dt).cuda()
    up = lambda x: torch.from_numpy(np.array(x, np.int32)).cuda()               # noqa: E731
    args = dict(kv_len=up(kv), q_start=up(np.concatenate(([0], np.cumsum(nq)))),
                q_tags=up(rng.integers(0, 2, n_q)) if tags else None)
    return c, q, wide, w, torch.from_numpy(blocks).cuda(), args


@pytest.mark.parametrize("case", [
    dict(dt="bf16", nope=64, value=64, tags=False, kv=[300, 0, 77], nq=[40, 1, 3], listed=12),
    dict(dt="fp16", nope=64, value=128, tags=True, kv=[300, 200], nq=[300, 9], listed=10),
    dict(dt="bf16", nope=128, value=64, tags=False, kv=[500], nq=[2], listed=16),
    dict(dt="bf16", nope=128, value=128, tags=True, kv=[1000], nq=[700], listed=264, R=256),
    dict(dt="fp16", nope=128, value=128, tags=False, kv=[900, 700], nq=[600, 520], listed=3200, R=256),
], ids=lambda c: f"{c['dt']}_{c['nope']}_{c['value']}_{c['listed']}")
def test_expanded_scratch_at_16_bytes(lib, case):
    """Keys and values are stored 32 bytes at a time, wherever the scratch begins.  (The wide lists take pairs of
    CTAs.)"""
    kw = dict(case, dt={"bf16": torch.bfloat16, "fp16": torch.float16}[case["dt"]])
    c, q, _, w, blocks, args = _problem(**kw)
    N = case["nope"]
    good = c.attend_expanded(q, w[:, :N], w[:, N:], blocks, **args)
    c.sync()

    def run(out, a, size):
        for at in (0, 16, 32, 48, 112):
            buffer = torch.full((size + 1024,), 0xAB, dtype=torch.uint8, device="cuda")
            first = buffer.data_ptr() % 256
            assert first == 0
            out.fill_(9)
            assert lib.akashic_mem_latent_attend_expanded(c._cfg, c._data_ptr, a, buffer.data_ptr() + 512 + at, size,
                                                          c._status_ptr, torch.cuda.current_stream().cuda_stream) == 0
            c.sync()
            assert torch.equal(out, good), at
            assert (buffer[:512 + at] == 0xAB).all() and (buffer[512 + at + size:] == 0xAB).all()

    _call(lib.akashic_mem_latent_expanded_scratch, c, q, blocks, args, good, run, (N + c.rope_dim) ** -0.5,
          w_k=w.data_ptr(), w_v=w[:, N:].data_ptr(), w_k_head_stride=w.stride(0), w_k_row_stride=w.stride(1),
          w_v_head_stride=w.stride(0), w_v_row_stride=w.stride(1), nope_dim=N, value_dim=case["value"])


def _call(scratch, c, q, blocks, args, good, run, scale, **more):
    from paper_2607_05708_gb300 import _LatentAttend
    ptr = lambda t: None if t is None else t.data_ptr()                         # noqa: E731
    out = torch.empty_like(good)
    a = ctypes.byref(_LatentAttend(
        q=q.data_ptr(), q_row_stride=q.stride(0), q_head_stride=q.stride(1), n_q=q.shape[0], q_heads=q.shape[1],
        n_seq=blocks.shape[0], q_start=ptr(args["q_start"]), kv_len=ptr(args["kv_len"]), blocks=blocks.data_ptr(),
        max_blocks=blocks.shape[1], causal=1, scale=scale, tags=c._tags_ptr if args["q_tags"] is not None else None,
        q_tags=ptr(args["q_tags"]), out=out.data_ptr(), **more))
    size = ctypes.c_int64()
    assert scratch(c._cfg, a, ctypes.byref(size)) == 0
    run(out, a, size.value)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
def test_absorbed_scratch_at_16_bytes(lib, dt):
    c, _, q, _, blocks, args = _problem(dt=getattr(torch, {"bf16": "bfloat16", "fp16": "float16"}[dt]), nope=64,
                                        value=64, tags=True, kv=[900, 700, 3], nq=[3, 20, 1], listed=40)
    good, _ = c.attend(q, blocks, 0.1, **args)
    c.sync()

    def run(out, a, size):
        assert size > 0
        for at in (0, 16, 48):
            buffer = torch.full((size + 1024,), 0xAB, dtype=torch.uint8, device="cuda")
            assert buffer.data_ptr() % 256 == 0
            out.fill_(9)
            assert lib.akashic_mem_latent_attend(c._cfg, c._data_ptr, a, buffer.data_ptr() + 512 + at, size,
                                                 c._status_ptr, torch.cuda.current_stream().cuda_stream) == 0
            c.sync()
            assert torch.equal(out, good), at
            assert (buffer[:512 + at] == 0xAB).all() and (buffer[512 + at + size:] == 0xAB).all()

    _call(lib.akashic_mem_latent_attend_scratch, c, q, blocks, args, good, run, 0.1)

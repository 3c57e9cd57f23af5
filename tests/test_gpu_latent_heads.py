"""Absorbed attention of the most heads over contexts that many CTAs share: items of several row tiles, each in
parts."""
import numpy as np
import pytest

import _latent_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("R,heads,kv,nq", [(512, 128, [5003, 0, 1029], [1, 1, 1]), (512, 128, [3100], [2]),
                                           (256, 128, [4099, 700], [1, 3]), (512, 200, [2500], [1]),
                                           (128, 1024, [900, 1], [1, 1]), (512, 1, [6001, 3], [129, 1])])
def test_many_heads_over_long_contexts(R, heads, kv, nq, dt):
    from paper_2607_05708_gb300 import LatentCache
    T, P = 64, 64
    rng = np.random.default_rng(61)
    n_blocks = sum(-(-n // T) for n in kv) + 1
    order = rng.permutation(n_blocks)
    blocks = np.full((len(kv), max(-(-n // T) for n in kv)), -1, np.int64)
    at = 0
    for i, n in enumerate(kv):
        m = -(-n // T)
        blocks[i, :m] = order[at:at + m]
        at += m
    make = lambda *s: torch.from_numpy(rng.standard_normal(s)).to(DT[dt])      # noqa: E731
    rows, q = make(n_blocks * T, R + P), make(sum(nq), heads, R + P)
    c = LatentCache(n_blocks, R, P, block_tokens=T, dtype=DT[dt])
    c.append(rows[:, :R].cuda(), rows[:, R:].cuda(), torch.arange(n_blocks * T).cuda())
    starts = np.concatenate(([0], np.cumsum(nq)))
    up = lambda x: torch.from_numpy(np.array(x, np.int32)).cuda()               # noqa: E731
    args = dict(kv_len=up(kv), q_start=up(starts))
    scale = (R + P) ** -0.5
    out, lse = c.attend(q.cuda(), torch.from_numpy(blocks).cuda(), scale, **args)
    again, _ = c.attend(q.cuda(), torch.from_numpy(blocks).cuda(), scale, **args)
    c.sync()
    assert torch.equal(out, again)
    want = orc.attend(q.double().numpy(), rows.double().numpy(), blocks, T, kv, starts, scale, dt == "bf16", R)
    assert (np.abs(out.double().cpu().numpy() - want["out"]) <= want["tol"]).all()
    e, fine = lse.double().cpu().numpy(), np.isfinite(want["lse"])
    assert (np.isneginf(e) == ~fine).all()
    assert (np.abs(e[fine] - want["lse"][fine]) <= want["tol_lse"][fine]).all()

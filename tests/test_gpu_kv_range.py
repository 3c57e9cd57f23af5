"""Attention at the ends of fp32's range: keys and values that are stored infinities, scores and
sums that are nearly as large."""
import numpy as np
import pytest

import _kv_oracle as orc
from test_gpu_kv_cache import DT, _built, _cache, _gpu  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FORMS = [(4, 128), (8, 64), (4, 256), (8, 128), (4, 64), (8, 256)]
# 1 row: a CTA an item; 3 rows of a long list: parts that are joined; 300 rows: the kernel for
# many, whose parts are joined too
SHAPES = [(1, 90), (3, 9000), (300, 9000)]


def _attend(bits, dim, q, k, v, T=16, **args):
    """Attention over all of k, v [kv, 1, dim] (fp32) for q [nq, heads, dim] bf16."""
    n = -(-len(k) // T)
    c = _cache(n, 1, dim, block_tokens=T, bits=bits)
    c.write(k.cuda(), v.cuda(), torch.arange(len(k), device="cuda"))
    got = c.attend(q.cuda(), torch.arange(n, device="cuda")[None],
                   kv_len=_gpu(np.array([len(k)], np.int32)), causal=False, **args)
    c.sync()
    return got


def _normal(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape)).bfloat16().float()


@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim", FORMS)
def test_infinite_keys_that_are_seen(bits, dim, nq, kv):
    """A key that is infinite in one dim is stored as the largest fp32 there and 0 elsewhere.
    Queries of 0 there score it 0; of either sign, all or nothing."""
    q, k, v = _normal(1, nq, 2, dim), _normal(2, kv, 1, dim), _normal(3, kv, 1, dim)
    k[40, 0], k[40, 0, 5] = 0, float("inf")
    q[:, 0, 5] = 0
    out, lse = _attend(bits, dim, q.bfloat16(), k, v)
    k0 = k.clone()
    k0[40] = 0                                  # the same scores for head 0
    want, wlse = _attend(bits, dim, q.bfloat16(), k0, v)
    assert torch.equal(out[:, 0], want[:, 0]) and torch.equal(lse[:, 0], wlse[:, 0])
    # head 1, positive: that token's value; its score is q max / sqrt(dim)
    q[:, 1, 5] = 0.5
    out, lse = _attend(bits, dim, q.bfloat16(), k, v)
    value = torch.from_numpy(orc.stored(v[40].double().numpy(), bits))[0]
    key = float(orc.stored(k[40].double().numpy(), bits)[0, 5])
    assert torch.equal(out[:, 1].cpu(), value.bfloat16().expand(nq, dim))
    assert torch.allclose(lse[:, 1].double().cpu(), torch.tensor(0.5 * key / dim ** 0.5, dtype=torch.float64), rtol=1e-6)
    # negative: as if the token were not there
    q[:, 1, 5] = -0.5
    out, lse = _attend(bits, dim, q.bfloat16(), k, v)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    keep = torch.arange(kv) != 40
    want, wlse = _attend(bits, dim, q.bfloat16(), k[keep], v[keep])
    # (tokens in other places: two roundings of the result, of weights and of scores)
    assert (out[:, 1].double() - want[:, 1].double()).abs().max() <= 2.0 ** -7 * float(v.abs().max())
    assert (lse[:, 1] - wlse[:, 1]).abs().max() <= 2.0 ** -14


@pytest.mark.parametrize("size", [1e37, 3e38])
@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim", FORMS)
def test_values_near_the_largest_fp32(bits, dim, nq, kv, size):
    """Their weighted mean is in range, so the result is, whatever their sum."""
    q, k = _normal(5, nq, 2, dim) * 0.25, _normal(6, kv, 1, dim)
    v = torch.full((kv, 1, dim), size)
    v[:, :, 1::2] *= -0.5
    out, lse = _attend(bits, dim, q.bfloat16(), k, v)
    value = torch.from_numpy(orc.stored(v[:1].double().numpy(), bits))[0, 0]
    assert torch.isfinite(out).all()
    # all values alike: weights' roundings and the result's
    assert ((out.double().cpu() - value).abs() <= (2.0 ** -11 + 2.0 ** -8 + 2.0 ** -17) * value.abs()).all()
    assert torch.isfinite(lse).all()


@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim", FORMS)
def test_scores_far_below_zero(bits, dim, nq, kv):
    """All scores -6.6e36 or -1.5e32: equal weights all the same."""
    for size in (1e32, 4.2e36):
        q, k, v = torch.zeros(nq, 2, dim), torch.zeros(kv, 1, dim), _normal(4, kv, 1, dim)
        q[:, :, 3], k[:, :, 3] = -1.5, size
        out, lse = _attend(bits, dim, q.bfloat16(), k, v, scale=1.0)
        stored = orc.stored(v.double().numpy(), bits)[:, 0]
        mean = torch.from_numpy(stored.mean(0))
        # weights equal and exact; values rounded to 2^-17 of their row's largest; fp32 sums, the result
        bound = 2.0 ** -17 * np.abs(stored).max(1).mean() + 2.0 ** -18 * np.abs(stored).max() + 2.0 ** -8 * mean.abs()
        assert ((out.double().cpu() - mean).abs() <= bound).all()
        key = orc.stored(k[:1].double().numpy(), bits)[0, 0, 3]
        assert torch.allclose(lse.double().cpu(), torch.tensor(-1.5 * key, dtype=torch.float64), rtol=1e-6)

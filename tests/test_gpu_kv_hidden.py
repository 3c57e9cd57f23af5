"""What a row does not see changes nothing of its result, whatever it is: keys and values of
other tags and of later tokens that are infinite, NaN or far larger than those seen.  The same bits
are asked for: a result is a sum over the seen keys alone."""
import numpy as np
import pytest

import _kv_oracle as orc
from test_gpu_kv_cache import DT, _built, _cache, _gpu  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FORMS = [(4, 128, "bf16"), (8, 64, "fp16"), (4, 256, "fp16"), (8, 128, "bf16"), (4, 64, "bf16"), (8, 256, "bf16")]
# 1 row: a CTA an item; 3 rows of a long list: parts that are joined; 300: the kernel for many
SHAPES = [(1, 90), (3, 9000), (300, 700)]


def _fill(rng, n, dim, dtype):
    x = rng.standard_normal((n, 1, dim)) * np.exp2(rng.integers(-2, 3, (n, 1, 1)))
    return torch.from_numpy(x).to(DT[dtype]).float()


def _extreme(what, x, rng):
    """x with rows that are infinite (of either sign, in some dims or all), NaN, or larger."""
    y = x.clone()
    n = len(y)
    if what == "inf":
        y[0::3] = float("inf")
        y[1::3, :, 3] = -float("inf")
        y[2::3, :, 5::7] = float("nan")
        y[2::3, :, 1] = float("inf")
    elif what == "1e30":
        y *= torch.from_numpy(np.where(rng.random((n, 1, 1)) < 0.5, 1e30, -1e30)).float()
    else:
        y *= float(what)
    return y


class _Call:
    """One sequence of kv tokens in shuffled blocks, nq query rows of two heads on one."""

    def __init__(self, seed, bits, dim, dtype, nq, kv, docs, T=16, **args):
        rng = self.rng = np.random.default_rng(seed)
        nb = -(-kv // T) + 2
        order = rng.permutation(nb)
        self.blocks = _gpu(order[None, :-2].copy())
        self.slots = order[np.arange(kv) // T] * T + np.arange(kv) % T
        self.cache = _cache(nb, 1, dim, block_tokens=T, bits=bits, tagged=bool(docs))
        self.k, self.v = (_fill(rng, kv, dim, dtype) for _ in "kv")
        self.q = torch.from_numpy(rng.standard_normal((nq, 2, dim))).to(DT[dtype]).cuda()
        self.tags = rng.integers(0, docs, kv).astype(np.int32) if docs else None
        self.args = dict(kv_len=_gpu(np.array([kv], np.int32)), **args)

    def __call__(self, k, v):
        tags = None if self.tags is None else _gpu(self.tags)
        self.cache.write(k.cuda(), v.cuda(), _gpu(self.slots), tags=tags)
        out, lse = self.cache.attend(self.q, self.blocks, **self.args)
        self.cache.sync()
        return out, lse


def _by_tags(bits, dim, dtype, nq, kv, which, what):
    """Tokens of tag 1 are replaced; rows of tag 0 stay, beside rows of tag 1 and without them."""
    for mixed in (False, True):
        c = _Call(nq + kv, bits, dim, dtype, nq, kv, 2, causal=False)
        qt = np.arange(nq) % 2 if mixed else np.zeros(nq)
        c.args["q_tags"] = _gpu(qt.astype(np.int32))
        a = c(c.k, c.v)
        hide = torch.from_numpy(c.tags == 1)
        k, v = c.k.clone(), c.v.clone()
        if which != "values":
            k[hide] = _extreme(what, k[hide], c.rng)
        if which != "keys":
            v[hide] = _extreme(what, v[hide], c.rng)
        b = c(k, v)
        rows = _gpu(np.flatnonzero(qt == 0))
        assert torch.isfinite(a[0]).all() and a[0].abs().max() > 0
        assert torch.equal(a[0][rows], b[0][rows]) and torch.equal(a[1][rows], b[1][rows])


def _by_time(bits, dim, dtype, nq, kv, which, what):
    """Tokens from row nq / 2's successor on are replaced; the rows before stay."""
    c = _Call(nq + kv + 1, bits, dim, dtype, nq, kv, 0, causal=True)
    a = c(c.k, c.v)
    first = nq // 2 + 1                        # first row that sees a replaced token
    at = kv - nq + first
    k, v = c.k.clone(), c.v.clone()
    if which != "values":
        k[at:] = _extreme(what, k[at:], c.rng)
    if which != "keys":
        v[at:] = _extreme(what, v[at:], c.rng)
    b = c(k, v)
    assert torch.isfinite(a[0]).all()
    assert torch.equal(a[0][:first], b[0][:first]) and torch.equal(a[1][:first], b[1][:first])


@pytest.mark.parametrize("what", ["inf", "1e30", "65536"])
@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim,dtype", FORMS)
def test_hidden_keys_change_nothing(bits, dim, dtype, nq, kv, what):
    if nq > 1:
        _by_time(bits, dim, dtype, nq, kv, "keys", what)
    _by_tags(bits, dim, dtype, nq, kv, "keys", what)


@pytest.mark.parametrize("what", ["inf", "1e30", "65536"])
@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim,dtype", FORMS)
def test_hidden_values_change_nothing(bits, dim, dtype, nq, kv, what):
    if nq > 1:
        _by_time(bits, dim, dtype, nq, kv, "values", what)
    _by_tags(bits, dim, dtype, nq, kv, "values", what)


@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim,dtype", FORMS[:3])
def test_hidden_tokens_behind_a_prefix_and_a_bias(bits, dim, dtype, nq, kv):
    """Both at once, under a prefix and a distance bias."""
    if nq > 1:
        c = _Call(nq + kv + 2, bits, dim, dtype, nq, kv, 0, causal=True,
                  prefix_len=_gpu(np.array([kv // 2], np.int32)), slopes=_gpu(np.array([0.5, 0.01], np.float32)))
        a = c(c.k, c.v)
        at = kv - nq + 1                       # row 0 sees none of these
        k, v = c.k.clone(), c.v.clone()
        k[at:], v[at:] = _extreme("inf", k[at:], c.rng), _extreme("inf", v[at:], c.rng)
        b = c(k, v)
        assert torch.equal(a[0][0], b[0][0]) and torch.equal(a[1][0], b[1][0])
    _by_tags(bits, dim, dtype, nq, kv, "both", "inf")


@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim,dtype", FORMS)
def test_hidden_tokens_under_a_cap(bits, dim, dtype, nq, kv):
    """Which of its two forms a capped score takes goes by the warp's largest, so that here
    a score may differ by the forms' difference, 2^-21 of the cap and less."""
    c = _Call(nq + kv + 3, bits, dim, dtype, nq, kv, 2, causal=False, cap=5.0)
    qt = np.arange(nq) % 2
    c.args["q_tags"] = _gpu(qt.astype(np.int32))
    a = c(c.k, c.v)
    hide = torch.from_numpy(c.tags == 1)
    k, v = c.k.clone(), c.v.clone()
    k[hide], v[hide] = _extreme("inf", k[hide], c.rng), _extreme("inf", v[hide], c.rng)
    b = c(k, v)
    rows = _gpu(np.flatnonzero(qt == 0))
    # scores off by t: weights by 2 t relative and by another rounding to fp16 (a step is
    # 2^-10); the result is rounded twice
    t = 5 * 2.0 ** -20
    size = float(c.v[~hide].abs().max())
    far = (a[0][rows].double() - b[0][rows].double()).abs().max()
    assert far <= (2 * t + 2.0 ** -10 + torch.finfo(DT[dtype]).eps) * size
    assert (a[1][rows] - b[1][rows]).abs().max() <= 2 * t

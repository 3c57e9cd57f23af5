"""Errors of the attention against bounds by what a row sees (_kv_seen.tolerances): no key or
value that its mask hides, and no value of little weight, takes part in them."""
import numpy as np
import pytest

import _kv_oracle as orc
import _kv_seen
from test_gpu_kv_cache import CASES, DT, LONG, _built, _problem  # noqa: F401
from test_gpu_kv_hidden import FORMS, SHAPES, _Call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _seen_problem(monkeypatch, *a, **kw):
    """_problem, its answer with what the bounds by seen tokens need."""
    plain = orc.attend
    monkeypatch.setattr(orc, "attend", lambda *x, **y: _kv_seen.add(plain(*x, **y), *x, **y))
    return _problem(*a, **kw)


def _close(got, want, dim, dtype, bits, rows=None):
    out, lse = (x.double().cpu().numpy()[:rows] for x in got)
    want = {k: v[:rows] for k, v in want.items()}
    t_out, t_lse = _kv_seen.tolerances(want, dim, torch.finfo(DT[dtype]).eps / 2, bits, dtype)
    empty = np.isneginf(want["lse"])
    assert (out[empty] == 0).all() and np.isneginf(lse[empty]).all()
    assert np.isfinite(out).all() and np.isfinite(lse[~empty]).all()
    worst = (np.abs(out - want["out"]) / t_out).max(initial=0)
    assert worst <= 1, f"out is {worst:.2f} of its bound"
    worst = (np.abs(lse[~empty] - want["lse"][~empty]) / t_lse[~empty]).max(initial=0)
    assert worst <= 1, f"lse is {worst:.2f} of its bound"


@pytest.mark.parametrize("name", CASES)
@pytest.mark.parametrize("bits,dim,dtype", [FORMS[0], FORMS[1], FORMS[2]])
def test_errors_within_what_is_seen(monkeypatch, name, bits, dim, dtype):
    kw = CASES[name]
    c, q, blocks, args, want = _seen_problem(monkeypatch, sum(map(ord, name)) + 1, bits=bits, dim=dim,
                                             dtype=dtype, **kw)
    got = c.attend(q, blocks, **args)
    c.sync()
    _close(got, want, dim, dtype, bits, rows=sum(kw.get("nq") or (1,) * len(kw["kv"])))


@pytest.mark.parametrize("gap", [12, 16, 20, 40])
@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim,dtype", [FORMS[0], FORMS[3], FORMS[4]])
def test_seen_values_of_very_different_sizes(bits, dim, dtype, nq, kv, gap):
    """Every fifth value is 2^gap times the others, and its weight 2^-2 gap or so: the others
    make the result."""
    rng = np.random.default_rng(gap)
    c = _Call(nq + kv + gap, bits, dim, dtype, nq, kv, 0, causal=True)
    big = rng.random(kv) < 0.2
    u = rng.choice([-1.0, 1.0], dim)           # every row's keys and queries along u
    keys = rng.standard_normal((kv, 1, dim)) * 0.05 + u / dim
    keys[big] -= u * (2 * gap * np.log(2) + 3) / np.sqrt(dim)
    q = rng.standard_normal((nq, 2, dim)) * 0.05 + u
    values = rng.standard_normal((kv, 1, dim)) * np.where(big, 2.0 ** gap, 1.0)[:, None, None]
    k, v, q = (torch.from_numpy(x).to(DT[dtype]) for x in (keys, values, q))
    c.q = q.cuda()
    got = c(k.float(), v.float())
    a = (q.double().numpy(), orc.stored(k.double().numpy(), bits), orc.stored(v.double().numpy(), bits),
         np.arange(-(-kv // 16))[None], 16, [kv], [0, nq])
    want = _kv_seen.add(orc.attend(*a), *a)
    _close(got, want, dim, dtype, bits)
    # what the large values add is no more than a tenth of the result, which is not lost
    assert np.median(np.abs(got[0].double().cpu().numpy() - want["out"])) <= 0.05 * np.median(np.abs(want["out"]))


@pytest.mark.parametrize("size", [-20, -11, -8, 4, 6, 9, "mixed"])
@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim,dtype", [FORMS[0], FORMS[1], FORMS[2]])
def test_keys_and_values_of_any_size(bits, dim, dtype, nq, kv, size):
    """Powers of two apart, all alike or from token to token; queries that make the scores
    ordinary."""
    rng = np.random.default_rng(nq)
    c = _Call(nq + kv, bits, dim, dtype, nq, kv, 0, causal=True)
    if size == "mixed":
        ke, ve = rng.integers(-14, 3, (kv, 1, 1)), rng.integers(-14, 9, (kv, 1, 1))
        qe = 0
    else:
        ke = ve = np.full((kv, 1, 1), size)
        qe = -size if dtype == "bf16" else np.clip(-size, -8, 8)
    k = torch.from_numpy(rng.standard_normal((kv, 1, dim)) * np.exp2(ke)).float()
    v = torch.from_numpy(rng.standard_normal((kv, 1, dim)) * np.exp2(ve)).float()
    q = torch.from_numpy(rng.standard_normal((nq, 2, dim)) * np.exp2(qe)).to(DT[dtype])
    c.q = q.cuda()
    got = c(k, v)
    a = (q.double().numpy(), orc.stored(k.double().numpy(), bits), orc.stored(v.double().numpy(), bits),
         np.arange(-(-kv // 16))[None], 16, [kv], [0, nq])
    _close(got, _kv_seen.add(orc.attend(*a), *a), dim, dtype, bits)


@pytest.mark.parametrize("nq,kv", SHAPES)
@pytest.mark.parametrize("bits,dim,dtype", FORMS)
def test_an_infinite_value_that_is_seen(bits, dim, dtype, nq, kv):
    """One token's value is infinite (stored as the largest fp32) in one dim, and comes
    early, in the middle or last: that dim of the rows that see it is as large as its
    weight says, and the total as it was."""
    for at in (1, kv // 2, kv - 1):
        c = _Call(nq + kv + at, bits, dim, "bf16", nq, kv, 0, causal=False)
        v = c.v.clone()
        v[at, 0, 9] = float("inf")
        plain, ref = c(c.k, c.v), orc.stored(v.double().numpy(), bits)
        got = c(c.k, v)
        # the exponent less the maximum and R, at most 2^8 in size, is rounded: 2^-17 a weight; sums 2^-20
        assert (plain[1] - got[1]).abs().max() <= 2.0 ** -16
        a = (c.q.double().cpu().numpy(), orc.stored(c.k.double().numpy(), bits), ref,
             np.arange(-(-kv // 16))[None], 16, [kv], [0, nq])
        want = _kv_seen.add(orc.attend(*a, causal=False), *a, causal=False)
        out = got[0].double().cpu().numpy()
        t_out, _ = _kv_seen.tolerances(want, dim, torch.finfo(torch.bfloat16).eps / 2, bits, "bf16")
        assert np.isfinite(out).all()
        assert (np.abs(out - want["out"]) <= t_out).all()

"""The expanded form with keys and values that are no numbers: of weights that are not finite, of sums of infinities of
both signs.  Rows that see such a token are NaN, and nothing else changes by a bit."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_05708_gb300 import _build
    _build.build()


def _problem(dt, N, V, kv, nq, listed=0, H=3, R=128, P=32, T=32):
    from paper_2607_05708_gb300 import LatentCache
    rng = np.random.default_rng(51)
    n_blocks = sum(-(-n // T) for n in kv) + 1
    c = LatentCache(n_blocks, R, P, block_tokens=T, dtype=DT[dt])
    rows = torch.from_numpy(rng.standard_normal((n_blocks * T, R + P))).to(DT[dt]).cuda()
    c.append(rows[:, :R], rows[:, R:], torch.arange(n_blocks * T, device="cuda"))
    blocks = np.full((len(kv), max(max(-(-n // T) for n in kv), listed // T)), -1, np.int64)
    at = 0
    for i, n in enumerate(kv):
        m = -(-n // T)
        blocks[i, :m] = np.arange(at, at + m)
        at += m
    q = torch.from_numpy(rng.standard_normal((sum(nq), H, N + P))).to(DT[dt]).cuda()
    w = torch.from_numpy(rng.standard_normal((H, N + V, R)) * R ** -0.5).to(DT[dt]).cuda()
    up = lambda x: torch.from_numpy(np.array(x, np.int32)).cuda()               # noqa: E731
    args = dict(kv_len=up(kv), q_start=up(np.concatenate(([0], np.cumsum(nq)))))
    lists = torch.from_numpy(blocks).cuda()
    return c, w, lambda w: c.attend_expanded(q, w[:, :N], w[:, N:], lists, **args)


# the second sequence's first rows see nothing: more rows than tokens
SHAPES = {"64_64": (64, 64, [300, 40], [7, 60], 0), "64_128": (64, 128, [300, 40], [200, 60], 0),
          "128_64": (128, 64, [140, 40], [3, 60], 0), "128_128": (128, 128, [300, 40], [290, 60], 0),
          "pairs": (128, 128, [700, 500], [600, 520], 8224)}


@pytest.mark.parametrize("bad", [NAN, INF, -INF], ids=["nan", "inf", "minus_inf"])
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_weights_that_are_not_finite(shape, dt, bad):
    N, V, kv, nq, listed = SHAPES[shape]
    c, w, call = _problem(dt, N, V, kv, nq, listed)
    good = call(w)
    blind = torch.zeros(sum(nq), dtype=torch.bool, device="cuda")
    blind[nq[0]:sum(nq) - kv[1]] = True
    assert int(blind.sum()) == 20 and torch.isfinite(good).all() and (good[blind] == 0).all()
    for row in (0, N - 1, N, N + V - 1):       # keys' first and last, values' first and last
        spoilt = w.clone()
        spoilt[1, row, 77] = bad
        out = call(spoilt)
        c.sync()
        assert torch.equal(out[:, 0], good[:, 0]) and torch.equal(out[:, 2], good[:, 2]), row
        assert (out[blind, 1] == 0).all(), row
        assert torch.isnan(out[~blind, 1]).all(), row


@pytest.mark.parametrize("shape", SHAPES)
def test_sums_that_are_no_numbers_are_their_tokens(shape):
    """One token whose latent values make products beyond fp32 of both signs: rows that do not see it keep their
    bits."""
    N, V, kv, nq, listed = SHAPES[shape]
    c, w, call = _problem("bf16", N, V, kv, nq, listed)
    good = call(w)
    at = kv[0] - 2                             # a token of the first sequence that its last two rows see
    for part in (slice(0, N), slice(N, None)):
        spoilt = w.clone()
        spoilt[1, part, 0], spoilt[1, part, 64] = 4.0, -4.0
        c.data[:, [0, 64]] = 0
        even = call(spoilt)                    # (weights of values that are 0 count nowhere)
        c.data[at, [0, 64]] = torch.finfo(torch.bfloat16).max
        out = call(spoilt)
        c.sync()
        sees = torch.zeros(len(out), dtype=torch.bool, device="cuda")
        sees[nq[0] - 2:nq[0]] = True           # (in the other heads a key and a value like others, but large)
        assert torch.isfinite(even).all()
        assert torch.equal(out[~sees], even[~sees])
        assert torch.isnan(out[sees, 1]).all()
    assert torch.isfinite(good).all()

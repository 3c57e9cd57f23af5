"""The expanded form's query rows and weights in every layout that it takes, by CTAs and by pairs of them: the
same bits as from contiguous ones, and what the definition gives."""
import numpy as np
import pytest

import _latent_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_05708_gb300 import _build
    _build.build()


def _layouts(q):
    """Aligned views of the values of q [n, heads, width] whose rows are spaced otherwise."""
    n, h, w = q.shape
    e = lambda *s: torch.full(s, float("nan"), dtype=q.dtype, device="cuda")   # noqa: E731
    yield "padded", e(n, h, w + 24)[..., 8:8 + w]
    yield "head_major", e(h, n, w).transpose(0, 1)
    yield "head_major_padded", e(h, n + 5, w + 8)[:, 3:3 + n, 8:].transpose(0, 1)
    yield "among_others", e(n, 3 * h + 1, w)[:, 1:1 + h]
    yield "every_second_head", e(n, 2 * h, w)[:, ::2]
    yield "every_second_row", e(2 * n, h, w)[::2]
    yield "heads_together", e(n, h, 2, w)[:, :, 1]


def _misaligned(q):
    n, h, w = q.shape
    e = lambda *s: torch.full(s, float("nan"), dtype=q.dtype, device="cuda")   # noqa: E731
    yield "one_off", e(n, h, w + 8)[..., 1:1 + w]
    yield "odd_rows", e(n, h, w + 3)[..., :w]
    yield "odd_heads", e(h, n * w + 1).as_strided((n, h, w), (w, n * w + 1, 1))


# sequences' contexts and rows; lists of 8256 tokens and 512 rows a sequence: pairs of CTAs
SHAPES = {
    "ctas": dict(kv=[200, 260], nq=[3, 140], heads=3, nope=64, value=128, listed=320, R=128, P=32),
    "ctas_one_head": dict(kv=[400], nq=[300], heads=1, nope=128, value=128, listed=448, R=256, P=64),
    "pairs": dict(kv=[700, 1300], nq=[700, 600], heads=2, nope=128, value=128, listed=8256, R=128, P=32),
    "pairs_one_head": dict(kv=[1500], nq=[1030], heads=1, nope=128, value=128, listed=8256, R=128, P=64),
}


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_query_rows_and_weights_in_any_layout(shape, dt):
    from paper_2607_05708_gb300 import LatentCache
    s = SHAPES[shape]
    kv, nq, H, N, V, R, P, T = s["kv"], s["nq"], s["heads"], s["nope"], s["value"], s["R"], s["P"], 64
    rng = np.random.default_rng(41)
    n_blocks = 24
    blocks = np.full((len(kv), s["listed"] // T), -1, np.int64)
    for i, n in enumerate(kv):
        m = -(-n // T)
        blocks[i, :m] = rng.permutation(n_blocks)[:m]
    make = lambda *z: torch.from_numpy(rng.standard_normal(z)).to(DT[dt])      # noqa: E731
    rows, q, w = make(n_blocks * T, R + P), make(sum(nq), H, N + P), (make(H, N + V, R).float() * R ** -0.5).to(DT[dt])
    c = LatentCache(n_blocks, R, P, block_tokens=T, dtype=DT[dt])
    c.append(rows[:, :R].cuda(), rows[:, R:].cuda(), torch.arange(n_blocks * T).cuda())
    starts = np.concatenate(([0], np.cumsum(nq)))
    up = lambda x: torch.from_numpy(np.array(x, np.int32)).cuda()               # noqa: E731
    args = dict(kv_len=up(kv), q_start=up(starts))
    lists, wk, wv = torch.from_numpy(blocks).cuda(), w[:, :N].contiguous().cuda(), w[:, N:].contiguous().cuda()
    want = orc.attend(q.double().numpy(), rows.double().numpy(), blocks, T, kv, starts, (N + P) ** -0.5, dt == "bf16", R,
                      w_k=w[:, :N].double().numpy(), w_v=w[:, N:].double().numpy())

    def fits(out, name):
        o = out.double().cpu().numpy()
        assert np.isfinite(o).all(), name
        assert (np.abs(o - want["out"]) <= want["tol"]).all(), name

    good = c.attend_expanded(q.cuda(), wk, wv, lists, **args)
    fits(good, "contiguous")
    for name, view in _layouts(q):
        view.copy_(q)
        assert torch.equal(c.attend_expanded(view, wk, wv, lists, **args), good), name
    for name, view in _misaligned(q):          # (never by pairs: bits may be others)
        view.copy_(q)
        fits(c.attend_expanded(view, wk, wv, lists, **args), name)
    # weights: halves of one projection, rows apart, heads apart by whole rows
    both = w.cuda()
    assert torch.equal(c.attend_expanded(q.cuda(), both[:, :N], both[:, N:], lists, **args), good)
    apart = torch.full((H, N + V + 5, R + 40), float("nan"), dtype=DT[dt], device="cuda")
    apart[:, 2:2 + N + V, 8:8 + R] = both
    assert torch.equal(c.attend_expanded(q.cuda(), apart[:, 2:2 + N, 8:8 + R], apart[:, 2 + N:2 + N + V, 8:8 + R], lists,
                                         **args), good)
    c.sync()

"""The warps of the kernel for many rows keep together whatever order items come in: second row
tiles with and without rows, items of one step and of many, shared between CTAs or not."""
import numpy as np
import pytest

from test_gpu_kv_cache import _built, _compare, _problem  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,dim,dtype", [(4, 128, "bf16"), (8, 64, "fp16"), (4, 64, "bf16"), (8, 128, "fp16"),
                                            (4, 256, "fp16")])
@pytest.mark.parametrize("order", ["by_turns", "few_then_one", "random"])
def test_second_row_tiles_that_come_and_go(order, bits, dim, dtype):
    """Sequences of 65 to 128 rows, whose items leave the second row tile without rows, among ones of
    up to 256 and more."""
    rng = np.random.default_rng(len(order))
    S = 60
    if order == "by_turns":
        nq = np.where(np.arange(S) % 2, 200, 100)
    elif order == "few_then_one":
        nq = np.where(np.arange(S) % 7 == 6, 256, 128)
    else:
        nq = rng.integers(65, 300, S)
    kv = np.maximum(rng.integers(1, 700, S), np.where(np.arange(S) % 5 == 0, nq, 1))
    c, q, blocks, args, want = _problem(91, kv=tuple(kv), nq=tuple(nq), heads=3, group=1, bits=bits, dim=dim,
                                        dtype=dtype, T=64)
    first = [x.clone() for x in c.attend(q, blocks, **args)]
    c.sync()
    _compare(first, want, dim, dtype, bits)
    for _ in range(20):
        got = c.attend(q, blocks, **args)
        assert torch.equal(got[0], first[0]) and torch.equal(got[1], first[1])
    c.sync()

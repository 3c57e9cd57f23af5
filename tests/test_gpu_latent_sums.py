"""Many keys of nearly the row's largest score, with values near the type's largest: their mean is finite, however many
there are, and whatever the first of them were."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_05708_gb300 import _build
    _build.build()


def _cache(dt, n, R, quiet, value):
    """n tokens with the same latent vector, the first `quiet` of score 0, the others of 7.48 (log2): not enough for
    the reference of the first tile to be raised."""
    from paper_2607_05708_gb300 import LatentCache
    c = LatentCache(-(-n // 64), R, 32, dtype=DT[dt])
    rows = torch.zeros(n, R + 32, dtype=DT[dt])
    rows[:, 1:R:2] = value
    rows[quiet:, R] = 5.1875                   # 7.484 in log2
    c.append(rows[:, :R].cuda(), rows[:, R:].cuda(), torch.arange(n).cuda())
    return c, rows, torch.arange(-(-n // 64)).cuda()


def _value(dt):
    # three quarters of the largest, exactly a value of the type: weights and the result are rounded by half a step
    # each, (1 + eps / 2)^2, which keeps the result below the type's largest
    return {"bf16": 1.5 * 2.0 ** 127, "fp16": 1.5 * 2.0 ** 15}[dt]


def _check(out, want, dt):
    eps = torch.finfo(DT[dt]).eps
    assert torch.isfinite(out).all()
    # sums of thousands of equal terms in fp32 besides: 2^-12
    assert ((out.double() - want).abs() <= (1.01 * eps + 2.0 ** -12) * want.abs()).all()


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("R,n,quiet,seqs,heads", [(128, 768, 128, 1, 3), (256, 768, 128, 1, 16), (512, 2000, 64, 200, 16),
                                                  (512, 1200, 64, 160, 33), (128, 120_000, 0, 1, 16),
                                                  (128, 500_000, 1000, 1, 40), (512, 3000, 2, 200, 1)])
def test_absorbed(dt, R, n, quiet, seqs, heads):
    c, rows, blocks = _cache(dt, n, R, quiet, _value(dt))
    q = torch.zeros(seqs, heads, R + 32, dtype=DT[dt])
    q[..., R] = 1.0
    kv = torch.full((seqs,), n, dtype=torch.int32).cuda()
    out, lse = c.attend(q.cuda(), blocks[None].expand(seqs, -1).contiguous(), 1.0, kv_len=kv)
    c.sync()
    _check(out, rows[0, :R].double().cuda(), dt)
    want = torch.logsumexp(rows[:, R].double(), 0).cuda()
    # totals: fp32 sums in many lanes, 2^-13; the exponential and the logarithm
    assert ((lse.double() - want).abs() <= 2.0 ** -12 + 2.0 ** -20 * want.abs()).all()


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("n,quiet,seqs,rows_of,heads,width,listed", [
    (768, 64, 200, 1, 4, 64, 0), (2000, 10, 100, 3, 4, 128, 0), (120_000, 0, 1, 2, 1, 64, 0),
    (1500, 64, 12, 600, 8, 128, 8256), (60_000, 0, 2, 520, 1, 128, 0)])
def test_expanded(dt, n, quiet, seqs, rows_of, heads, width, listed):
    R, V = 128, _value(dt)
    c, rows, blocks = _cache(dt, n, R, quiet, V)
    lists = torch.full((seqs, max(len(blocks), listed // 64)), -1, dtype=torch.int64, device="cuda")
    lists[:, :len(blocks)] = blocks
    q = torch.zeros(seqs * rows_of, heads, width + 32, dtype=DT[dt])
    q[..., width] = 1.0
    w = torch.zeros(heads, 2 * width, R, dtype=DT[dt])
    w[:, width::2, 1] = 1.0
    kv = torch.full((seqs,), n, dtype=torch.int32).cuda()
    out = c.attend_expanded(q.cuda(), w[:, :width].cuda(), w[:, width:].cuda(), lists, scale=1.0, kv_len=kv,
                            causal=False)
    c.sync()
    want = torch.zeros(width, dtype=torch.float64)
    want[::2] = V
    _check(out, want.cuda(), dt)


def _leaning(dt, n):
    """Scores of n tokens: every 64th 0, the others such that a weight, a power of two times that, is rounded up by
    three quarters of half a step (bf16 0.0033, fp16 0.0004 of itself; from the middle between the type's largest and
    the next power of two on, 0.002 and 0.00025 above the largest, a result would round to infinity)."""
    eps = torch.finfo(DT[dt]).eps
    z = torch.log(torch.tensor((1 + 0.58 * eps) / 2, dtype=torch.float64))
    a = z.to(DT[dt])
    b = (z - a.double()).to(DT[dt])
    rope = torch.zeros(n, 32, dtype=DT[dt])
    rope[:, 0], rope[:, 1] = a, b
    rope[::64] = 0
    w = torch.exp(rope.double().sum(1)[1])
    up = float((w.to(DT[dt]).double() - w) / w)
    assert up > 1.3 * eps / 4 / (2 - eps) * 2
    return rope


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("form", ["absorbed", "absorbed_joined", "expanded", "expanded_pairs"])
def test_means_of_the_largest_are_finite(form, dt, sign):
    from paper_2607_05708_gb300 import LatentCache
    R, n, most = 128, 700, torch.finfo(DT[dt]).max
    c = LatentCache(-(-n // 64), R, 32, dtype=DT[dt])
    rows = torch.zeros(n, R + 32, dtype=DT[dt])
    rows[:, 1:R:2] = sign * most
    rows[:, R:] = _leaning(dt, n)
    c.append(rows[:, :R].cuda(), rows[:, R:].cuda(), torch.arange(n).cuda())
    blocks = torch.arange(-(-n // 64)).cuda()
    if form.startswith("absorbed"):
        # 151 whole items on as many CTAs, or two tiles of rows that all CTAs share
        seqs, rows_of, heads, listed = (151, 1, 16, 0) if form == "absorbed" else (1, 40, 3, 4096)
        wide, want = R, rows[0, :R].double()
    else:
        seqs, rows_of, heads, listed = (200, 1, 4, 0) if form == "expanded" else (12, 600, 8, 8256)
        wide = 128
        want = torch.zeros(wide, dtype=torch.float64)
        want[::2] = sign * most
    lists = torch.full((seqs, max(len(blocks), listed // 64)), -1, dtype=torch.int64, device="cuda")
    lists[:, :len(blocks)] = blocks
    kv = torch.full((seqs,), n, dtype=torch.int32).cuda()
    q = torch.zeros(seqs * rows_of, heads, wide + 32, dtype=DT[dt])
    q[..., wide:wide + 2] = 1.0
    if form.startswith("absorbed"):
        out = c.attend(q.cuda(), lists, 1.0, kv_len=kv, causal=False)[0]
    else:
        w = torch.zeros(heads, 2 * wide, R, dtype=DT[dt])
        w[:, wide::2, 1] = 1.0
        out = c.attend_expanded(q.cuda(), w[:, :wide].cuda(), w[:, wide:].cuda(), lists, scale=1.0, kv_len=kv, causal=False)
    c.sync()
    _check(out, want.cuda(), dt)

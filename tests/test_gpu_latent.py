"""Attention over the latent cache, both forms, against 64 bits (bounds: _latent_oracle.py); lists,
lengths, masks, streams, graphs, offsets past 32 bits, retrieval and attention together."""
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


def _gpu(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def _error(c):
    from paper_2607_05708_gb300 import AkashicError
    with pytest.raises(AkashicError) as e:
        c.sync()
    c.sync()                               # cleared
    return e.value.code


def _round(x, dt):
    t = torch.from_numpy(x).to(DT[dt])
    return t, t.double().numpy()


def problem(seed, kv, nq, heads=4, R=256, P=64, T=64, dt="bf16", form="absorbed", nope=64, value=64, causal=True,
            prefix=None, tags=0, holes=False, tail=0, gain=1.0, tag_rows=None, listed=0):
    """A cache, a call on it and what it should give."""
    from paper_2607_05708_gb300 import LatentCache
    rng = np.random.default_rng(seed)
    need = [-(-n // T) for n in kv]
    n_blocks, S, width = sum(need) + 2, len(kv), max(max(need), 1, listed // T)
    order = rng.permutation(n_blocks)
    blocks = np.full((S, width), -1, np.int64)
    at = 0
    for i, m in enumerate(need):
        blocks[i, :m] = order[at:at + m]
        at += m
    if holes:
        blocks[rng.random(blocks.shape) < 0.3] = -1
    rows, rows64 = _round(gain * rng.standard_normal((n_blocks * T, R + P)), dt)
    c = LatentCache(n_blocks, R, P, block_tokens=T, dtype=DT[dt], tagged=bool(tags))
    slot_tags = rng.integers(-1, tags, n_blocks * T).astype(np.int32) if tags else None
    c.append(rows[:, :R].cuda(), rows[:, R:].cuda(), torch.arange(n_blocks * T).cuda(),
             tags=None if slot_tags is None else _gpu(slot_tags))
    n_q = sum(nq) + tail
    q_start = np.concatenate(([0], np.cumsum(nq))).astype(np.int32)
    q_tags = None
    if tags:
        # among them one that no slot has
        q_tags = rng.integers(0, tags + 1, n_q).astype(np.int32) if tag_rows is None else tag_rows
    wide = (R if form == "absorbed" else nope) + P
    q, q64 = _round(rng.standard_normal((n_q, heads, wide)), dt)
    scale = wide ** -0.5
    args = dict(kv_len=_gpu(np.array(kv, np.int32)), q_start=_gpu(q_start), causal=causal,
                prefix_len=None if prefix is None else _gpu(np.array(prefix, np.int32)),
                q_tags=None if q_tags is None else _gpu(q_tags))
    kw = {}
    if form == "absorbed":
        call = lambda **o: c.attend(q.cuda(), _gpu(blocks), scale, **{**args, **o})              # noqa: E731
    else:
        w, w64 = _round(rng.standard_normal((heads, nope + value, R)) * R ** -0.5, dt)
        w = w.cuda()
        kw = dict(w_k=w64[:, :nope], w_v=w64[:, nope:])
        call = lambda **o: c.attend_expanded(q.cuda(), w[:, :nope], w[:, nope:], _gpu(blocks),  # noqa: E731
                                             **{**args, **o})
    want = orc.attend(q64[:sum(nq)], rows64, blocks, T, kv, q_start, scale, dt == "bf16", R, causal=causal,
                      prefix=prefix, tags=slot_tags, q_tags=q_tags, **kw)
    return c, call, want, dict(q=q, blocks=blocks, rows=rows, scale=scale, args=args, q64=q64, rows64=rows64)


def compare(got, want, n=None):
    out, lse = got if isinstance(got, tuple) else (got, None)
    o = out.double().cpu().numpy()[:n]
    assert np.isfinite(o).all()
    worst = (np.abs(o - want["out"][:n]) / want["tol"][:n]).max(initial=0)
    assert worst <= 1, f"out: {worst} of the bound"
    if lse is not None:
        e, w = lse.double().cpu().numpy()[:n], want["lse"][:n]
        assert (np.isneginf(e) == np.isneginf(w)).all()
        fine = np.isfinite(w)
        worst = (np.abs(e[fine] - w[fine]) / want["tol_lse"][:n][fine]).max(initial=0)
        assert worst <= 1, f"lse: {worst} of the bound"


FORMS = ["absorbed", "expanded"]
# context lengths and query rows of the sequences, and what else
CASES = {
    "one": dict(kv=[1], nq=[1], heads=1),
    "none": dict(kv=[0, 5, 0], nq=[1, 2, 3]),
    "nothing_listed": dict(kv=[0], nq=[2]),
    "edges": dict(kv=[15, 16, 17, 127, 128, 129, 255, 256, 257], nq=[1] * 9, T=16),
    "ragged": dict(kv=[700, 3, 64, 401], nq=[1, 1, 1, 1], heads=16, T=32),
    "drafts": dict(kv=[300, 77, 6], nq=[5, 5, 5], heads=5, T=48),
    "more_rows_than_keys": dict(kv=[3, 140], nq=[9, 150], heads=3),
    "uneven": dict(kv=[300, 260, 20, 130], nq=[1, 40, 0, 7], heads=12, tail=3),
    "prompt": dict(kv=[333], nq=[333], heads=2, T=16),
    "tall": dict(kv=[400, 300], nq=[290, 257], heads=2, T=128),
    "bidirectional": dict(kv=[300, 140], nq=[7, 3], heads=9, causal=False),
    "prefix": dict(kv=[300, 260, 50], nq=[30, 260, 4], heads=3, prefix=[200, 100, 80]),
    "tags": dict(kv=[300, 270], nq=[6, 33], heads=6, tags=3, causal=False),
    "tags_causal": dict(kv=[200, 270], nq=[150, 33], heads=2, tags=2, T=16),
    "holes": dict(kv=[700, 300], nq=[3, 20], heads=4, T=32, holes=True),
    "holes_tags_prefix": dict(kv=[500, 300], nq=[3, 200], heads=2, T=16, holes=True, tags=2, prefix=[400, 10]),
    "long": dict(kv=[3001], nq=[2], heads=2),
    "loud": dict(kv=[500, 300], nq=[2, 130], heads=4, gain=8.0),
    "faint": dict(kv=[300], nq=[3], heads=4, gain=2.0 ** -6),
}


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("case", CASES)
def test_masks_and_lengths(form, case):
    c, call, want, _ = problem(1, form=form, **CASES[case])
    got = call()
    c.sync()
    compare(got, want, len(want["out"]))


@pytest.mark.parametrize("R,P", [(128, 32), (128, 64), (256, 32), (256, 64), (512, 32), (512, 64)])
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("heads", [1, 8, 16, 17, 32, 40, 64, 128])
def test_absorbed_shapes(R, P, dt, heads):
    c, call, want, _ = problem(2, kv=[290, 33], nq=[2, 1], heads=heads, R=R, P=P, dt=dt, tags=2, causal=True)
    got = call()
    c.sync()
    compare(got, want)


@pytest.mark.parametrize("R,P", [(128, 32), (256, 64), (512, 32), (512, 64)])
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("nope,value", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_expanded_shapes(R, P, dt, nope, value):
    c, call, want, _ = problem(3, kv=[330, 33], nq=[200, 3], heads=3, R=R, P=P, dt=dt, form="expanded", nope=nope,
                               value=value, prefix=[100, 0])
    got = call()
    c.sync()
    compare(got, want)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
@pytest.mark.parametrize("form", FORMS)
def test_scores_that_rise(dt, form):
    """Keys grow along the context, so that the running maximum is raised many times, then
    fall."""
    c, call, want, x = problem(4, kv=[900], nq=[3], heads=4, dt=dt, form=form, R=128, P=32)
    rows = x["rows64"]
    order = [b * 64 + t for b in x["blocks"][0] for t in range(64)]
    size = np.concatenate((np.linspace(0.1, 12, 600), np.linspace(12, 0.1, len(order) - 600)))
    rows[order] *= size[:, None]
    t, r64 = _round(rows, dt)
    c.append(t[:, :128].cuda(), t[:, 128:].cuda(), torch.arange(len(t)).cuda())
    # the oracle again with these rows
    kw = {}
    if form == "expanded":
        rng = np.random.default_rng(4)
        rng.permutation(len(x["rows"]) // 64), rng.standard_normal(x["rows"].shape), rng.standard_normal(x["q"].shape)
        _, w = _round(rng.standard_normal((4, 128, 128)) * 128 ** -0.5, dt)
        kw = dict(w_k=w[:, :64], w_v=w[:, 64:])
    want = orc.attend(x["q64"], r64, x["blocks"], 64, [900], [0, 3], x["scale"], dt == "bf16", 128, **kw)
    compare(call(), want)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
def test_hidden_rows_change_no_bit(form, dt):
    """What no row sees (another tag's tokens, tokens behind kv_len, other blocks) may hold the
    type's largest values."""
    kw = dict(kv=[300, 270], nq=[6, 150], heads=3, tags=2, form=form, dt=dt, R=128, P=32)
    rows = np.zeros(156, np.int32)
    c, call, want, x = problem(5, tag_rows=rows, **kw)
    good = call()
    first = good[0] if form == "absorbed" else good
    compare(good, want)
    hidden = (c.tags != 0).cpu()
    for b, n in ((0, 300), (1, 270)):
        for j in range(n, 5 * 64):
            blk = x["blocks"][b][j // 64]
            if blk >= 0:
                hidden[blk * 64 + j % 64] = True
    assert 100 < int(hidden.sum()) < len(hidden) - 100
    most = torch.finfo(DT[dt]).max
    sign = torch.where(torch.arange(160) % 2 == 0, most, -most).to(DT[dt]).cuda()
    c.data[hidden.cuda()] = sign
    again = call()
    c.sync()
    assert torch.equal(first, again[0] if form == "absorbed" else again)


@pytest.mark.parametrize("form", FORMS)
def test_bad_lists_and_lengths_are_reported_and_bounded(form):
    c, call, want, x = problem(6, kv=[300, 310, 290], nq=[2, 2, 2], form=form, heads=2)
    first = (lambda g: g[0]) if form == "absorbed" else (lambda g: g)
    good = first(call()).clone()
    c.sync()
    for bad in (c.n_blocks, 1 << 40, -7):
        x["blocks"][1, 2] = bad
        out = first(call()).clone()
        assert _error(c) == "EDEVICE"
        x["blocks"][1, 2] = -1
        assert torch.equal(out, first(call()))
        c.sync()
        assert torch.equal(out[[0, 1, 4, 5]], good[[0, 1, 4, 5]])
    for bad in (1 << 30, -5):
        n = x["args"]["kv_len"].clone()
        n[1] = bad
        out = first(call(kv_len=n))
        assert _error(c) == "EDEVICE"
        assert torch.equal(out[[0, 1, 4, 5]], good[[0, 1, 4, 5]])
    for starts in ([0, 2, 1, 6], [0, 2, 4, 99], [-4, 2, 4, 6]):
        call(q_start=_gpu(np.array(starts, np.int32)))
        assert _error(c) == "EDEVICE"


@pytest.mark.parametrize("form", FORMS)
def test_rows_behind_the_last_sequence_stay(form):
    c, call, want, x = problem(7, kv=[90, 310], nq=[2, 140], heads=2, tail=11, form=form)
    wide = 256 if form == "absorbed" else 64
    out = torch.full((153, 2, wide), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((153, 2), 5.0, device="cuda")
    if form == "absorbed":
        call(out=out, lse=lse)
        assert (lse[142:] == 5).all()
        compare((out[:142], lse[:142]), want)
    else:
        call(out=out)
        compare(out[:142], want)
    assert (out[142:] == 3).all()
    fresh = call()
    fresh = fresh[0] if form == "absorbed" else fresh
    assert (fresh[142:] == 0).all() and torch.equal(fresh[:142], out[:142])


@pytest.mark.parametrize("form", FORMS)
def test_strides_and_alignment(form):
    c, call, want, x = problem(8, kv=[200, 260], nq=[3, 140], heads=3, form=form, R=128, P=32)
    good = call()
    good = good[0] if form == "absorbed" else good
    n, h, w = x["q"].shape
    for off, pad in ((1, 3), (8, 8), (4, 0)):
        big = torch.zeros(n, h, w + pad + off, dtype=torch.bfloat16, device="cuda")
        big[..., off:off + w] = x["q"].cuda()
        turned = torch.zeros(h, n, w + off, dtype=torch.bfloat16, device="cuda")
        turned[..., off:] = x["q"].cuda().transpose(0, 1)
        for q in (big[..., off:off + w], turned[..., off:].transpose(0, 1)):
            args = dict(x["args"])
            if form == "absorbed":
                out = torch.empty(n * h * 128 + 2, dtype=torch.bfloat16, device="cuda")[2:].view(n, h, 128)
                c.attend(q, _gpu(x["blocks"]), x["scale"], out=out, **args)
                assert torch.equal(out, good)
    if form == "expanded":
        rng = np.random.default_rng(8)
        rng.permutation(len(x["rows"]) // 64), rng.standard_normal(x["rows"].shape), rng.standard_normal(x["q"].shape)
        w, _ = _round(rng.standard_normal((3, 128, 128)) * 128 ** -0.5, "bf16")
        wide = torch.zeros(4, 128, 136, dtype=torch.bfloat16, device="cuda")
        wide[:3, :, :128] = w.cuda()
        out = torch.empty(n * h * 64 + 2, dtype=torch.bfloat16, device="cuda")[2:].view(n, h, 64)
        big = torch.zeros(n, h, w.shape[2] + 7, dtype=torch.bfloat16, device="cuda")[..., 3:3 + x["q"].shape[2]]
        big.copy_(x["q"])
        c.attend_expanded(big, wide[:3, :64, :128], wide[:3, 64:, :128], _gpu(x["blocks"]), out=out, **x["args"])
        assert torch.equal(out, good)
        apart = wide[:3, :64, :128].contiguous(), wide[:3, 64:, :128].contiguous()
        assert torch.equal(c.attend_expanded(x["q"].cuda(), *apart, _gpu(x["blocks"]), **x["args"]), good)


@pytest.mark.parametrize("form", FORMS)
def test_same_bits_streams_and_graphs(form):
    """The same bits every time, on other streams, and from two graphs replayed in turn and
    at once."""
    c, call, want, x = problem(9, kv=[1500, 700], nq=[3, 160], heads=5, form=form, tags=2)
    first = (lambda g: g[0]) if form == "absorbed" else (lambda g: g)
    good = first(call()).clone()
    for _ in range(3):
        assert torch.equal(first(call()), good)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    q, blocks = x["q"].cuda(), _gpu(x["blocks"])
    torch.cuda.synchronize()
    both = []
    for s in (s1, s2, s1, s2):
        both.append(first(call(stream=s)))
    torch.cuda.synchronize()
    assert all(torch.equal(b, good) for b in both)
    if form == "absorbed":
        run = lambda: c.attend(q, blocks, x["scale"], **x["args"])[0]           # noqa: E731
    else:
        w = torch.randn(5, 128, 256, device="cuda", dtype=torch.bfloat16) / 16
        run = lambda: c.attend_expanded(q, w[:, :64], w[:, 64:], blocks, **x["args"])    # noqa: E731
    ref = run().clone()
    torch.cuda.synchronize()
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(run())
    for _ in range(2):
        for o in outs:
            o.fill_(7)
        graphs[0].replay(), graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, ref) for o in outs)
        for o in outs:
            o.fill_(7)
        torch.cuda.synchronize()
        for g, s in zip(graphs, (s1, s2)):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, ref) for o in outs)


@pytest.mark.parametrize("form", FORMS)
def test_thousands_of_sequences(form):
    rng = np.random.default_rng(10)
    kv = [int(n) for n in rng.integers(0, 40, 2100)]
    c, call, want, _ = problem(10, kv=kv, nq=[int(n) for n in rng.integers(0, 3, 2100)], heads=2, R=128, P=32, T=16,
                               form=form)
    got = call()
    c.sync()
    compare(got, want)


def test_even_rows_without_starts():
    c, call, want, x = problem(11, kv=[128, 128, 128], nq=[2, 2, 2], heads=3, T=64)
    a, la = call()
    b, lb = c.attend(x["q"].cuda(), _gpu(x["blocks"]), x["scale"])
    assert torch.equal(a, b) and torch.equal(la, lb)
    e = torch.empty(0, 3, 320, dtype=torch.bfloat16, device="cuda")
    out, lse = c.attend(e, torch.empty(0, 4, dtype=torch.int64, device="cuda"), 1.0)
    assert out.shape == (0, 3, 256) and lse.shape == (0, 3)
    # nothing listed: nothing seen
    out, lse = c.attend(x["q"].cuda(), torch.empty(3, 0, dtype=torch.int64, device="cuda"), 1.0)
    assert (out == 0).all() and torch.isneginf(lse).all()
    w = torch.zeros(3, 64, 256, dtype=torch.bfloat16, device="cuda")
    out = c.attend_expanded(x["q"].cuda()[..., :128], w, w, torch.empty(3, 0, dtype=torch.int64, device="cuda"))
    assert (out == 0).all()


def _exact(q, X, R, scale, limit):
    """One sequence, single rows: 64 bits on the GPU."""
    z = (q.double() @ X.double().T) * scale
    z[..., limit:] = -float("inf")
    return torch.softmax(z, -1) @ X[:, :R].double(), torch.logsumexp(z, -1)


@pytest.mark.parametrize("R,heads", [(512, 64), (256, 16), (512, 24)])
def test_long_context_past_32_bits(R, heads):
    """A cache of more than 4 GB, its last blocks and its first."""
    from paper_2607_05708_gb300 import LatentCache
    T, n = 64, 70_001
    n_blocks = (1 << 32) // ((R + 64) * 2 * T) + 600
    c = LatentCache(n_blocks, R, 64, block_tokens=T)
    assert c.data.numel() * 2 > 1 << 32
    g = torch.Generator("cuda").manual_seed(0)
    width = -(-n // T)
    blocks = torch.cat((torch.arange(width // 2), torch.arange(n_blocks - (width - width // 2), n_blocks))).cuda()
    slots = (blocks[:, None] * T + torch.arange(T, device="cuda")).reshape(-1)
    rows = torch.randn(len(slots), R + 64, device="cuda", generator=g).bfloat16()
    c.append(rows[:, :R], rows[:, R:], slots)
    assert torch.equal(c.data[slots], rows)
    q = torch.randn(1, heads, R + 64, device="cuda", generator=g).bfloat16()
    out, lse = c.attend(q, blocks[None], (R + 64) ** -0.5, kv_len=torch.tensor([n], dtype=torch.int32).cuda())
    c.sync()
    o, e = _exact(q[0], rows, R, (R + 64) ** -0.5, n)
    # weights off by 2^-8 and a little more of themselves, the result by 2^-8
    X = rows[:n, :R].double().abs()
    z = (q[0].double() @ rows[:n].double().T) * (R + 64) ** -0.5
    bound = 1.02 * 2.0 ** -8 * (torch.softmax(z, -1) @ X + o.abs()) + 1e-30
    assert ((out[0].double() - o).abs() <= bound).all()
    assert ((lse[0].double() - e).abs() <= 1e-4).all()


def test_both_forms_agree_and_follow_retrieval():
    """Chunks are stored, retrieved in a namespace, their latent rows rotated on the way in, and
    attended over in both forms."""
    from paper_2607_05708_gb300 import LatentCache, MemStore
    rng = np.random.default_rng(12)
    R, P, T, H, N, V, chunks, n_ns = 128, 64, 16, 4, 64, 64, 96, 4
    emb = torch.from_numpy(rng.standard_normal((chunks, 64))).bfloat16().cuda()
    ns = (torch.arange(chunks) % n_ns).int()
    store = MemStore(64, chunks)
    store.append_chunks(emb.view(torch.int16))
    store.set_namespace(0, ns.cuda())
    c = LatentCache(chunks, R, P, block_tokens=T, tagged=True)
    n = chunks * T
    half = P // 2
    freq = 1000.0 ** (-np.arange(half) / half)
    angle = np.arange(n)[:, None] * freq
    cos, sin = np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)
    lat, k = _round(rng.standard_normal((n, R)), "bf16")[0], _round(rng.standard_normal((n, P)), "bf16")[0]
    tags = ns.repeat_interleave(T)
    c.append(lat.cuda(), k.cuda(), torch.arange(n).cuda(), torch.arange(n).cuda(), _gpu(cos), _gpu(sin),
             tags=tags.cuda())
    rows = torch.cat((lat.float(), torch.from_numpy(orc.rotate(k.float().numpy()[:, None], np.arange(n), cos, sin,
                                                               False)[:, 0])), 1).bfloat16()
    assert torch.equal(c.data.cpu(), rows)
    B = 8
    q_ns = (torch.arange(B) % n_ns).int().cuda()
    ids = store.retrieve(emb[:B].contiguous().view(torch.int16), 8, 0.5, 1, q_ns=q_ns)[0]
    q, q64 = _round(rng.standard_normal((B, H, N + P)), "bf16")
    w, w64 = _round(rng.standard_normal((H, N + V, R)) * R ** -0.5, "bf16")
    scale = (N + P) ** -0.5
    lists = ids.cpu().numpy()
    kw = dict(causal=False, tags=tags.numpy(), q_tags=q_ns.cpu().numpy())
    starts = np.arange(B + 1)
    out = c.attend_expanded(q.cuda(), w[:, :N].cuda(), w[:, N:].cuda(), ids, causal=False, q_tags=q_ns)
    want = orc.attend(q64, rows.double().numpy(), lists, T, [8 * T] * B, starts, scale, True, R, w_k=w64[:, :N],
                      w_v=w64[:, N:], **kw)
    compare(out, want)
    absorbed = torch.cat((torch.einsum("bhn,hnr->bhr", q[..., :N].double(), w[:, :N].double()), q[..., N:].double()),
                         -1).bfloat16()
    o, lse = c.attend(absorbed.cuda(), ids, scale, causal=False, q_tags=q_ns)
    c.sync()
    want = orc.attend(absorbed.double().numpy(), rows.double().numpy(), lists, T, [8 * T] * B, starts, scale, True,
                      R, **kw)
    compare((o, lse), want)
    # out of the latent space: the forms differ by the roundings of both
    v = torch.einsum("bhr,hvr->bhv", o.double().cpu(), w[:, N:].double())
    assert float((v - out.double().cpu()).norm() / v.norm()) < 0.03


def test_tensors_that_are_refused():
    from paper_2607_05708_gb300 import AkashicError, LatentCache
    e = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d, device="cuda")    # noqa: E731
    c = LatentCache(4, 128, 32, block_tokens=16)
    blocks = torch.zeros(2, 2, dtype=torch.int64).cuda()
    good = dict(q=e(2, 3, 160), blocks=blocks, scale=1.0)
    c.attend(**good)
    for bad in (dict(q=e(2, 3, 128)), dict(q=e(2, 3, 160, d=torch.float16)), dict(q=e(2, 160)), dict(blocks=blocks[0]),
                dict(blocks=blocks.int()), dict(q_tags=torch.zeros(2, dtype=torch.int32).cuda()),
                dict(kv_len=torch.zeros(3, dtype=torch.int32).cuda()), dict(out=e(2, 3, 64)), dict(lse=e(2, 3))):
        with pytest.raises((ValueError, TypeError)):
            c.attend(**{**good, **bad})
    for bad in (dict(scale=0.0), dict(scale=float("nan")), dict(q=e(3, 3, 160)), dict(q=e(2, 1025, 160))):
        with pytest.raises(AkashicError):
            c.attend(**{**good, **bad})
    good = dict(q=e(2, 3, 96), w_k=e(3, 64, 128), w_v=e(3, 128, 128), blocks=blocks)
    assert c.attend_expanded(**good).shape == (2, 3, 128)
    for bad in (dict(q=e(2, 3, 128)), dict(w_k=e(2, 64, 128)), dict(w_v=e(3, 64, 64)), dict(w_v=e(3, 64, 128).cpu()),
                dict(w_k=e(3, 64, 128, d=torch.float16)), dict(w_k=e(3, 128, 64).transpose(1, 2)), dict(out=e(2, 3, 64))):
        with pytest.raises((ValueError, TypeError)):
            c.attend_expanded(**{**good, **bad})
    for bad in (dict(w_k=e(3, 96, 128), q=e(2, 3, 128)), dict(w_v=e(3, 32, 128)), dict(w_k=e(3, 64, 129)[..., :128]),
                dict(w_k=e(3 * 64 * 128 + 4)[4:].view(3, 64, 128)), dict(w_k=e(3, 65, 136)[:, :64, :128][:, :, :128]),
                dict(scale=0.0)):
        if "w_k" in bad and bad["w_k"].stride(1) == 136:
            c.attend_expanded(**{**good, **bad})               # evenly spaced: taken
            continue
        with pytest.raises(AkashicError):
            c.attend_expanded(**{**good, **bad})
    for bad in (dict(latent_dim=64), dict(rope_dim=48), dict(block_tokens=24), dict(n_blocks=0)):
        with pytest.raises(AkashicError):
            LatentCache(**{**dict(n_blocks=1, latent_dim=128, rope_dim=32), **bad})
    with pytest.raises(TypeError):
        LatentCache(1, 128, 32, dtype=torch.float32)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dt", ["bf16", "fp16"])
def test_values_near_the_types_largest(form, dt):
    """Equal values of the type's largest: their mean is that, however many there are."""
    from paper_2607_05708_gb300 import LatentCache
    n, R, P, H = 600, 128, 32, 3
    c = LatentCache(10, R, P, dtype=DT[dt])
    # the largest of which the expanded form's product with 1/2 and its sums stay in range
    big = torch.finfo(DT[dt]).max if form == "absorbed" else torch.finfo(DT[dt]).max / 4
    rows = torch.zeros(n, R + P, dtype=DT[dt])
    rows[:, 1::2] = big
    rows[:, R:] = torch.randn(n, P, generator=torch.Generator().manual_seed(0)).to(DT[dt])
    c.append(rows[:, :R].cuda(), rows[:, R:].cuda(), torch.arange(n).cuda())
    blocks = torch.arange(10).cuda()[None]
    kv = torch.tensor([n], dtype=torch.int32).cuda()
    if form == "absorbed":
        q = torch.zeros(2, H, R + P, dtype=DT[dt])
        q[..., R:] = 1.0
        out, lse = c.attend(q.cuda(), blocks, 1.0, kv_len=kv)
        assert torch.isfinite(lse).all()
        want = rows[0, :R].double()
    else:
        q = torch.zeros(2, H, 64 + P, dtype=DT[dt])
        q[..., 64:] = 1.0
        w = torch.zeros(H, 128, R, dtype=DT[dt])
        w[:, 64:, 1] = 0.5
        out = c.attend_expanded(q.cuda(), w[:, :64].cuda(), w[:, 64:].cuda(), blocks, kv_len=kv)
        want = torch.full((64,), float(rows[0, 1]) / 2, dtype=torch.float64)
    c.sync()
    # weights and the result are rounded by half a step each
    assert ((out.double().cpu() - want).abs() <= 1.01 * torch.finfo(DT[dt]).eps * want.abs()).all()


@pytest.mark.parametrize("heads,nq", [(3, 4), (16, 1), (40, 2), (64, 2)])
@pytest.mark.parametrize("R", [256, 512])
def test_short_lists_agree_with_long_ones(heads, nq, R):
    """A call whose lists are short takes no scratch; the same sequences in wider lists do."""
    c, call, want, x = problem(21, kv=[300, 1, 250, 64], nq=[nq] * 4, heads=heads, R=R, T=32, tags=2)
    args = {k: v for k, v in x["args"].items() if k != "q_start"}
    q, blocks = x["q"].cuda(), _gpu(x["blocks"])
    compare(c.attend(q, blocks, x["scale"], **args), want)
    wide = torch.full((4, 200), -1, dtype=torch.int64, device="cuda")
    wide[:, :blocks.shape[1]] = blocks
    compare(c.attend(q, wide, x["scale"], **args), want)
    c.sync()


@pytest.mark.parametrize("T", [16, 32, 48, 64, 80, 112, 128, 256, 4096])
@pytest.mark.parametrize("form", FORMS)
def test_block_sizes(T, form):
    c, call, want, _ = problem(22, kv=[500, 70, T + 1 if T < 1000 else 3], nq=[3, 2, 1], heads=5, R=512, T=T, form=form,
                               holes=T < 100)
    got = call()
    c.sync()
    compare(got, want)


@pytest.mark.parametrize("form", FORMS)
def test_infinite_and_nan_query_rows_stay_theirs(form):
    """A row of NaN or infinities makes no other row's result other than it was."""
    c, call, want, x = problem(23, kv=[400, 300], nq=[3, 140], heads=2, R=128, P=32, form=form)
    first = (lambda g: g[0]) if form == "absorbed" else (lambda g: g)
    good = first(call()).clone()
    q = x["q"].clone()
    q[1, 0, 5], q[2, 1, :] = float("nan"), float("inf")
    q[77, 1, 3] = -float("inf")
    if form == "absorbed":
        out = c.attend(q.cuda(), _gpu(x["blocks"]), x["scale"], **x["args"])[0]
    else:
        rng = np.random.default_rng(23)
        rng.permutation(len(x["rows"]) // 64), rng.standard_normal(x["rows"].shape), rng.standard_normal(x["q"].shape)
        w, _ = _round(rng.standard_normal((2, 128, 128)) * 128 ** -0.5, "bf16")
        out = c.attend_expanded(q.cuda(), w[:, :64].cuda(), w[:, 64:].cuda(), _gpu(x["blocks"]), **x["args"])
    keep = torch.ones(143, 2, dtype=torch.bool)
    keep[1, 0] = keep[2, 1] = keep[77, 1] = False
    assert torch.equal(out[keep.cuda()], good[keep.cuda()])
    assert torch.isnan(out[1, 0]).all()


def test_heads_in_several_goes():
    """Keys and values of all heads beyond what the scratch takes at a time."""
    from paper_2607_05708_gb300 import LatentCache
    g = torch.Generator("cuda").manual_seed(5)
    H, T, S, width = 40, 64, 30, 160                     # 30 x 10240 tokens: 79 MB a head
    c = LatentCache(64, 128, 32, block_tokens=T)
    rows = torch.randn(64 * T, 160, device="cuda", generator=g).bfloat16()
    c.append(rows[:, :128], rows[:, 128:], torch.arange(64 * T, device="cuda"))
    blocks = torch.full((S, width), -1, dtype=torch.int64, device="cuda")
    blocks[:, :3] = torch.randint(64, (S, 3), device="cuda", generator=g)
    q = torch.randn(S, H, 96, device="cuda", generator=g).bfloat16()
    w = (torch.randn(H, 128, 128, device="cuda", generator=g) / 11).bfloat16()
    kv = torch.full((S,), 150, dtype=torch.int32, device="cuda")
    out = c.attend_expanded(q, w[:, :64], w[:, 64:], blocks, kv_len=kv)
    narrow = c.attend_expanded(q, w[:, :64], w[:, 64:], blocks[:, :3].contiguous(), kv_len=kv)
    c.sync()
    n_q, _, _ = q.shape
    want = orc.attend(q.double().cpu().numpy(), rows.double().cpu().numpy(), blocks.cpu().numpy(), T, [150] * S,
                      np.arange(S + 1), 96 ** -0.5, True, 128, w_k=w[:, :64].double().cpu().numpy(),
                      w_v=w[:, 64:].double().cpu().numpy())
    compare(out, want)
    compare(narrow, want)


@pytest.mark.parametrize("R,dt,S,width,H", [(512, "bf16", 4, 256, 2), (256, "fp16", 5, 100, 13),
                                            (512, "fp16", 200, 8, 1), (256, "bf16", 1, 900, 3)])
def test_wide_lists(R, dt, S, width, H):
    """Lists far wider than the contexts: where keys and values are made by pairs of CTAs; an odd number
    of tiles, more sequences than threads, sequences without tokens."""
    from paper_2607_05708_gb300 import LatentCache
    rng = np.random.default_rng(S)
    T, P, N, V = 64, 64, 128, 128
    kv = rng.integers(0, 300, S)
    kv[0], kv[S // 2] = 130 if sum(-(-n // 128) for n in kv[1:]) % 2 else 300, 0 if S > 1 else 300
    need = -(-kv // T)
    n_blocks = max(int(need.max()), 6)
    blocks = np.full((S, width), -1, np.int64)
    for i, m in enumerate(need):
        blocks[i, :m] = rng.permutation(n_blocks)[:m]
    rows, rows64 = _round(rng.standard_normal((n_blocks * T, R + P)), dt)
    c = LatentCache(n_blocks, R, P, block_tokens=T, dtype=DT[dt])
    c.append(rows[:, :R].cuda(), rows[:, R:].cuda(), torch.arange(n_blocks * T).cuda())
    q, q64 = _round(rng.standard_normal((S, H, N + P)), dt)
    w, w64 = _round(rng.standard_normal((H, N + V, R)) * R ** -0.5, dt)
    w = w.cuda()
    out = [c.attend_expanded(q.cuda(), w[:, :N], w[:, N:], _gpu(blocks), kv_len=_gpu(kv.astype(np.int32)))
           for _ in range(3)]
    c.sync()
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
    compare(out[0], orc.attend(q64, rows64, blocks, T, kv, np.arange(S + 1), (N + P) ** -0.5, dt == "bf16", R,
                               w_k=w64[:, :N], w_v=w64[:, N:]))


# prompts with rows for pairs of CTAs, of 512 rows an item, which are taken where lists are long: ends in
# either CTA's rows and row tiles
PROMPTS = {
    "causal": dict(kv=[700, 1300], nq=[700, 600]),
    "prefix": dict(kv=[1600, 513], nq=[513, 512], prefix=[1000, 400], dt="fp16"),
    "uneven": dict(kv=[1100, 10, 40, 1500], nq=[1100, 0, 5, 1500], T=48, heads=1, tail=3),
    "bidirectional": dict(kv=[900], nq=[640], causal=False, R=128, P=32),
    "tags": dict(kv=[1000, 1040], nq=[700, 800], tags=3, T=16, holes=True, causal=False),
    "tags_causal": dict(kv=[2000], nq=[1537], tags=2, prefix=[300], dt="fp16", R=512),
    "loud": dict(kv=[800], nq=[650], gain=8.0, R=512),
}


@pytest.mark.parametrize("listed", [0, 8256])
@pytest.mark.parametrize("case", PROMPTS)
def test_long_prompts(case, listed):
    kw = {"heads": 2, **PROMPTS[case]}
    c, call, want, _ = problem(len(case), form="expanded", nope=128, value=128, listed=listed, **kw)
    got = [call() for _ in range(3)]
    c.sync()
    rows = len(want["out"])
    assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
    compare(got[0], want, rows)
    assert (got[0][rows:] == 0).all()


def test_streams_in_turn():
    """Calls on streams of their own that follow each other by events, without the host between."""
    c, call, want, x = problem(24, kv=[900, 130], nq=[1, 2], heads=16, R=256)
    q, blocks = x["q"].cuda(), _gpu(x["blocks"])
    good = c.attend(q, blocks, x["scale"], **x["args"])[0].clone()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    rows = c.data.clone()
    slots = torch.arange(len(rows), device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(a):
            c.data.zero_()
            c.append(rows[:, :256], rows[:, 256:], slots)
        b.wait_stream(a)
        out = c.attend(q, blocks, x["scale"], stream=b, **x["args"])[0]
        a.wait_stream(b)
        b.synchronize()
        assert torch.equal(out, good)

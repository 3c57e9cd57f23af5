"""How the quantised cache's calls behave: bad indices, streams, graphs, strides, rows that
are not theirs, long offsets, retrieval and attention together."""
import ctypes

import numpy as np
import pytest

import _kv_oracle as orc
from test_gpu_kv_cache import DT, _built, _cache, _compare, _gpu, _problem, _values  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _error(c):
    from paper_2607_05708_gb300 import AkashicError
    with pytest.raises(AkashicError) as e:
        c.sync()
    c.sync()                               # cleared
    return e.value.code


def test_slots_out_of_range_are_reported_and_skipped():
    rng = np.random.default_rng(1)
    c = _cache(3, 2, 64, block_tokens=16, tagged=True)
    every = _gpu(np.arange(48))
    k0, k64 = _values(rng, 48, 2, 64, "bf16")
    c.write(k0, k0, every)
    c.sync()
    for bad in (48, 1 << 33, -2, -(1 << 40)):
        slots = np.array([5, bad, 7])
        k, kk = _values(rng, 3, 2, 64, "bf16")
        c.write(k, k, _gpu(slots), tags=_gpu([1, 2, 3], torch.int32))
        assert _error(c) == "EDEVICE"
        rk, _ = c.read(_gpu(slots), dtype=torch.float32)
        assert _error(c) == "EDEVICE"
        want = orc.stored(kk, 4)
        want[1] = 0
        assert torch.equal(rk.cpu(), torch.from_numpy(want).float())
    rest = np.setdiff1d(np.arange(48), [5, 7])
    rk, _ = c.read(_gpu(rest), dtype=torch.float32)
    assert torch.equal(rk.cpu(), torch.from_numpy(orc.stored(k64, 4)[rest]).float())
    c.sync()


@pytest.mark.parametrize("rows", [1, 300])
def test_bad_lists_and_lengths_are_reported_and_bounded(rows):
    """A block ID, a length or row range out of bounds: EDEVICE, the entry counted as not
    listed or clamped, the other sequences as ever."""
    kw = dict(kv=(300, 310, 320), nq=(rows,) * 3, heads=1, group=1, T=64)
    c, q, blocks, args, want = _problem(3, **kw)
    good = [x.clone() for x in c.attend(q, blocks, **args)]
    c.sync()
    b = blocks.clone()
    for bad in (c.n_blocks, 1 << 40, -7):
        b[1, 2] = bad
        out, lse = c.attend(q, b, **args)
        assert _error(c) == "EDEVICE"
        b[1, 2] = -1
        out2, lse2 = c.attend(q, b, **args)
        c.sync()
        assert torch.equal(out, out2) and torch.equal(lse, lse2)
        keep = [r for r in range(3 * rows) if r // rows != 1]
        assert torch.equal(out[keep], good[0][keep]) and torch.equal(lse[keep], good[1][keep])
    n = args["kv_len"].clone()
    for bad in (1 << 30, -5):
        n[1] = bad
        out, lse = c.attend(q, blocks, **{**args, "kv_len": n})
        assert _error(c) == "EDEVICE"
        keep = [r for r in range(3 * rows) if r // rows != 1]
        assert torch.equal(out[keep], good[0][keep])
    for starts in ([0, rows, rows - 1, 3 * rows], [0, rows, 2 * rows, 3 * rows + 9], [-4, rows, 2 * rows, 3 * rows]):
        c.attend(q, blocks, **{**args, "q_start": _gpu(np.array(starts, np.int32))})
        assert _error(c) == "EDEVICE"


@pytest.mark.parametrize("rows", [(1, 2, 1), (40, 300, 7)])
def test_rows_behind_the_last_sequence_stay(rows):
    c, q, blocks, args, want = _problem(5, kv=(90, 310, 44), nq=rows, heads=2, group=2, tail=11)
    out = torch.full_like(q, 3.0)
    lse = torch.full(q.shape[:2], 4.0, device="cuda")
    c.attend(q, blocks, out=out, lse=lse, **args)
    c.sync()
    n = sum(rows)
    assert (out[n:] == 3.0).all() and (lse[n:] == 4.0).all()
    _compare((out, lse), want, 128, "bf16", 4, rows=n)
    out, lse = c.attend(q, blocks, **args)
    assert (out[n:] == 0).all()


@pytest.mark.parametrize("bits,dim,dtype", [(4, 128, "bf16"), (8, 64, "fp16"), (4, 256, "fp16"), (8, 256, "bf16")])
@pytest.mark.parametrize("extra", [{}, dict(docs=2), dict(cap=5.0, slopes=True, causal=False)], ids=["plain", "tags", "cap"])
def test_rows_around_the_switch_of_kernels(bits, dim, dtype, extra):
    """The last number of rows of the kernel for few and the first of the one for many, where
    items are many (ten) and few, and all of them in one call."""
    turns = (32, 129) if dim == 256 else (64, 257)
    for i, rows in enumerate((turns[0], turns[0] + 1)):
        kv = (200, 90, 131, 300, 17)
        c, q, blocks, args, want = _problem(40 + i, kv=kv, nq=(rows,) * 5, heads=2, group=1, bits=bits,
                                            dim=dim, dtype=dtype, T=32, **extra)
        got = c.attend(q, blocks, **args)
        c.sync()
        _compare(got, want, dim, dtype, bits)
    for i, rows in enumerate((turns[1] - 1, turns[1])):
        c, q, blocks, args, want = _problem(50 + i, kv=(500,), nq=(rows,), heads=1, group=1, bits=bits,
                                            dim=dim, dtype=dtype, T=32, **extra)
        got = c.attend(q, blocks, **args)
        c.sync()
        _compare(got, want, dim, dtype, bits)
    nq = (1, turns[0], turns[0] + 1, 0, 150, turns[1])
    c, q, blocks, args, want = _problem(60, kv=(100, 200, 200, 20, 170, 260), nq=nq, heads=2, group=1,
                                        bits=bits, dim=dim, dtype=dtype, T=32, tail=3, **extra)
    got = c.attend(q, blocks, **args)
    c.sync()
    _compare(got, want, dim, dtype, bits, rows=sum(nq))


@pytest.mark.parametrize("docs", [0, 2])
def test_more_sequences_than_threads(docs):
    """3000 sequences, most of them without a row, some without a token, some of many rows."""
    rng = np.random.default_rng(71)
    S = 3000
    nq = np.where(np.arange(S) % 7 == 3, 1, 0)
    nq[[5, 1500, 2999]] = 70, 3, 66
    kv = rng.integers(0, 40, S)
    c, q, blocks, args, want = _problem(72, kv=tuple(kv), nq=tuple(nq), heads=2, group=1, docs=docs)
    got = c.attend(q, blocks, **args)
    c.sync()
    _compare(got, want, 128, "bf16", 4)
    ones = (1,) * S
    c, q, blocks, args, want = _problem(73, kv=tuple(kv), nq=ones, heads=2, group=1, docs=docs, dim=64)
    got = c.attend(q, blocks, **args)
    c.sync()
    _compare(got, want, 64, "bf16", 4)


@pytest.mark.parametrize("causal", [False, True])
def test_tags_over_a_long_context(causal):
    """More steps than the ranges of tags are kept for."""
    c, q, blocks, args, want = _problem(74, kv=(530_000,), nq=(66,), heads=1, group=1, docs=3, dim=64,
                                        T=128, causal=causal, dtype="fp16")
    got = c.attend(q, blocks, **args)
    c.sync()
    _compare(got, want, 64, "fp16", 4)


def test_strided_queries():
    """Queries inside a wider projection, heads first, at odd offsets."""
    for rows in (3, 290):
        c, q, blocks, args, want = _problem(7, kv=(300,), nq=(rows,), heads=2, group=2, T=64)
        wide = torch.zeros(rows, 3 * 4 * 128 + 5, dtype=q.dtype, device="cuda")
        views = [wide[:, 5:5 + 512].unflatten(1, (4, 128)), wide[:, 8:520].unflatten(1, (4, 128)),
                 torch.empty(4, rows, 128, dtype=q.dtype, device="cuda").transpose(0, 1)]
        for v in views:
            v.copy_(q)
            got = c.attend(v, blocks, **args)
            c.sync()
            _compare(got, want, 128, "bf16", 4)


@pytest.mark.parametrize("rows", [2, 300])
def test_a_bad_block_among_tags(rows):
    """Steps without a tag of the row's are left out; a bad block ID is reported all the same."""
    c, q, blocks, args, want = _problem(17, kv=(700,), nq=(rows,), heads=1, group=1, docs=2, T=64)
    c.sync()
    n = args["kv_len"]
    for at in (0, 4, 9):
        b = blocks.clone()
        b[0, at] = c.n_blocks
        c.attend(q, b, **{**args, "causal": False, "kv_len": n})
        assert _error(c) == "EDEVICE"


@pytest.mark.parametrize("cap", [2e-38, 1e-3, 1e4, 1e8, 3e38])
@pytest.mark.parametrize("rows", [3, 290])
def test_caps_of_any_size(rows, cap):
    """A cap far above the scores changes none of them; one far below makes them all
    alike."""
    c, q, blocks, args, want = _problem(19, kv=(400,), nq=(rows,), heads=1, group=1, cap=cap)
    got = c.attend(q, blocks, **args)
    c.sync()
    _compare(got, want, 128, "bf16", 4)


def test_the_same_bits_every_time():
    for kw in (dict(kv=(5000, 40, 900), heads=3), dict(kv=(900, 700), nq=(900, 400), heads=1)):
        c, q, blocks, args, _ = _problem(11, **kw)
        a = [x.clone() for x in c.attend(q, blocks, **args)]
        for _ in range(3):
            b = c.attend(q, blocks, **args)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    c.sync()


def test_values_that_are_not_finite_stay_in_their_row():
    """An infinite or NaN query makes its own row NaN and no other; stored infinities and
    NaN are finite."""
    for rows in (4, 300):
        c, q, blocks, args, want = _problem(13, kv=(200,), nq=(rows,), heads=1, group=2, causal=False)
        q[1, 0, 5] = float("nan")
        q[2, 1, 7] = float("inf")
        out, lse = c.attend(q, blocks, **args)
        c.sync()
        assert torch.isnan(out[1, 0]).all() and torch.isnan(lse[1, 0])
        assert not torch.isfinite(out[2, 1]).all()
        ok = torch.ones(rows, 2, dtype=torch.bool, device="cuda")
        ok[1, 0] = ok[2, 1] = False
        assert torch.isfinite(out[ok]).all() and torch.isfinite(lse[ok]).all()


def test_streams_side_by_side():
    """Two problems' calls on two streams at once, many times, each against its own
    result alone: scratch and outputs are the call's own."""
    kws = (dict(kv=(4000, 777, 90), heads=4), dict(kv=(600, 500), nq=(600, 300), heads=2),
           dict(kv=(30, 900, 2000, 64, 5), heads=2, bits=8, dim=64, dtype="fp16"))
    probs = [_problem(20 + i, **kw) for i, kw in enumerate(kws)]
    alone = [[x.clone() for x in p[0].attend(p[1], p[2], **p[3])] for p in probs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in probs]
    got = [[] for _ in probs]
    for _ in range(12):
        for i, (p, s) in enumerate(zip(probs, streams)):
            got[i].append(p[0].attend(p[1], p[2], stream=s, **p[3]))
    for i, (p, s) in enumerate(zip(probs, streams)):
        p[0].sync(stream=s)
        for out, lse in got[i]:
            assert torch.equal(out, alone[i][0]) and torch.equal(lse, alone[i][1])


def test_graphs_replayed_with_new_contents():
    """A decoding step (write, then attend) captured without a call before it and replayed with
    new tokens, lengths and queries in place; two graphs in flight on two streams."""
    rng = np.random.default_rng(6)
    steps, dim, heads, T = 5, 128, 2, 16
    graphs = []
    for seed in (0, 1):
        c = _cache(8, heads, dim, block_tokens=T)
        k, k64 = _values(rng, 8 * T, heads, dim, "bf16")
        v, v64 = _values(rng, 8 * T, heads, dim, "bf16")
        q = torch.from_numpy(rng.standard_normal((steps, 1, heads * 4, dim))).bfloat16()
        order = rng.permutation(8)
        st = dict(k=k[:1].clone(), v=v[:1].clone(), q=q[0].cuda(), slot=_gpu(np.zeros(1, np.int64)),
                  n=_gpu(np.ones(1, np.int32)), blocks=_gpu(order[None]))
        start = 90
        slots = order[np.arange(8 * T) // T] * T + np.arange(8 * T) % T
        c.write(k[:start], v[:start], _gpu(slots[:start]))
        torch.cuda.synchronize()
        stream, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            c.write(st["k"], st["v"], st["slot"])
            out, lse = c.attend(st["q"], st["blocks"], kv_len=st["n"])
        graphs.append((c, st, g, stream, out, lse, k, v, k64, v64, q, slots, start, order))
    for i in range(steps):
        for c, st, g, stream, out, lse, k, v, k64, v64, q, slots, start, order in graphs:
            with torch.cuda.stream(stream):
                st["k"].copy_(k[start + i:start + i + 1])
                st["v"].copy_(v[start + i:start + i + 1])
                st["q"].copy_(q[i])
                st["slot"].fill_(int(slots[start + i]))
                st["n"].fill_(start + i + 1)
                g.replay()
        for c, st, g, stream, out, lse, k, v, k64, v64, q, slots, start, order in graphs:
            c.sync(stream=stream)
            n = start + i + 1
            keys = np.zeros((8 * T, heads, dim))
            vals = np.zeros((8 * T, heads, dim))
            keys[slots[:n]], vals[slots[:n]] = orc.stored(k64[:n], 4), orc.stored(v64[:n], 4)
            want = orc.attend(q[i].double().numpy(), keys, vals, order[None], T, [n], [0, 1])
            _compare((out, lse), want, dim, "bf16", 4)


def test_offsets_past_32_bits():
    """Blocks beyond 4 GiB of cache, written, read and attended."""
    rng = np.random.default_rng(9)
    nb, heads, dim, T = 64_000, 8, 128, 64
    c = _cache(nb, heads, dim, block_tokens=T)
    assert c.data.numel() > 4 << 30
    ids = np.array([nb - 1, 3, nb - 2, 50_001])
    slots = (ids[:, None] * T + np.arange(T)).reshape(-1)
    k, k64 = _values(rng, len(slots), heads, dim, "bf16")
    v, v64 = _values(rng, len(slots), heads, dim, "bf16")
    c.write(k, v, _gpu(slots))
    rk, rv = c.read(_gpu(slots), dtype=torch.float32)
    assert torch.equal(rk.cpu(), torch.from_numpy(orc.stored(k64, 4)).float())
    for rows in (1, 100):
        q = torch.from_numpy(rng.standard_normal((rows, heads * 4, dim))).bfloat16()
        got = c.attend(q.cuda(), _gpu(ids[None]))
        c.sync()
        local = np.arange(4)[None]
        want = orc.attend(q.double().numpy(), orc.stored(k64, 4), orc.stored(v64, 4), local, T,
                          [4 * T], [0, rows])
        _compare(got, want, dim, "bf16", 4)


def test_empty_calls():
    c = _cache(2, 2, 64, block_tokens=16)
    q = torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = c.attend(q, torch.zeros(0, 3, dtype=torch.int64, device="cuda"))
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    torch.full((1 << 20,), 7.0, device="cuda")              # what the pool may hand out next
    out, lse = c.attend(torch.ones(5, 4, 64, dtype=torch.bfloat16, device="cuda"),
                        torch.zeros(0, 3, dtype=torch.int64, device="cuda"))
    assert (out == 0).all() and (lse == 0).all()            # rows of no sequence
    q = torch.ones(3, 4, 64, dtype=torch.bfloat16, device="cuda")
    for width in (0, 2):            # nothing listed, nothing in the list
        b = torch.full((3, width), -1, dtype=torch.int64, device="cuda")
        out, lse = c.attend(q, b)
        assert (out == 0).all() and torch.isneginf(lse).all()
    q = torch.ones(300, 4, 64, dtype=torch.bfloat16, device="cuda")
    out, lse = c.attend(q, torch.zeros(1, 0, dtype=torch.int64, device="cuda"))
    assert (out == 0).all() and torch.isneginf(lse).all()
    c.sync()


def test_arguments_are_checked():
    c = _cache(2, 2, 64, block_tokens=16)
    t = _cache(2, 2, 64, block_tokens=16, tagged=True)
    k = torch.zeros(3, 2, 64, device="cuda")
    slots = torch.arange(3, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    for bad in (dict(k=k[:, :1]), dict(k=k.double()), dict(k=k[:2]), dict(k=k.cpu()),
                dict(v=k.half()), dict(slots=slots[:2]), dict(slots=slots.int()), dict(slots=slots.cpu()),
                dict(k=torch.zeros(3, 2, 128, device="cuda")[..., ::2]),
                dict(tags=torch.zeros(3, **i32))):
        with pytest.raises((ValueError, TypeError)):
            c.write(**{**dict(k=k, v=k, slots=slots), **bad})
    with pytest.raises((ValueError, TypeError)):
        t.write(k, k, slots, tags=torch.zeros(2, **i32))
    for bad in (dict(dtype=torch.float64), dict(slots=slots.int()), dict(k=k[:2]),
                dict(k=k.half(), v=k)):
        with pytest.raises((ValueError, TypeError)):
            c.read(**{**dict(slots=slots), **bad})
    q = torch.zeros(3, 4, 64, dtype=torch.float16, device="cuda")
    b = torch.zeros(3, 1, dtype=torch.int64, device="cuda")
    for bad in (dict(q=q.float()), dict(q=q[:, :, :32]), dict(q=q.cpu()), dict(blocks=b.int()),
                dict(blocks=b[0]), dict(kv_len=torch.zeros(2, **i32)), dict(kv_len=torch.zeros(3, device="cuda")),
                dict(q_start=torch.zeros(3, **i32)), dict(slopes=torch.zeros(3, device="cuda")),
                dict(q_tags=torch.zeros(3, **i32)), dict(out=q[:2]), dict(out=q.bfloat16()),
                dict(lse=torch.zeros(3, 4, dtype=torch.float16, device="cuda")),
                dict(blocks=torch.zeros(3, 4, dtype=torch.int64, device="cuda")[:, ::2])):
        with pytest.raises((ValueError, TypeError)):
            c.attend(**{**dict(q=q, blocks=b), **bad})
    from paper_2607_05708_gb300 import AkashicError
    for bad in (dict(q=torch.zeros(3, 3, 64, dtype=torch.float16, device="cuda")), dict(cap=-1.0),
                dict(scale=float("inf")), dict(q=torch.zeros(4, 4, 64, dtype=torch.float16, device="cuda"))):
        with pytest.raises(AkashicError) as e:
            c.attend(**{**dict(q=q, blocks=b), **bad})
        assert e.value.code == "EINVAL"
    # scratch that is too small
    from paper_2607_05708_gb300 import _KVAttend, load_library
    starts = torch.arange(4, dtype=torch.int32, device="cuda")          # (without them it needs none)
    a = _KVAttend(q.data_ptr(), 256, 64, 1, 3, 4, 3, starts.data_ptr(), None, b.data_ptr(), 1, 1, None, 0.0, 0.0,
                  None, None, None, q.data_ptr(), None)
    scratch = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    assert load_library().akashic_mem_kv_attend(c._cfg, c.data.data_ptr(), ctypes.byref(a),
                                                scratch.data_ptr(), 64, None, None) == 1


@pytest.mark.parametrize("bits,dim,dtype", [(4, 128, "bf16"), (8, 64, "fp16")])
def test_retrieved_chunks_attended(bits, dim, dtype):
    """A store of chunks with namespaces, its chunks' keys and values in a cache (block ID =
    chunk ID): scoped retrieval in time order, then each query's attention over what
    it retrieved, its lists' padding and all, with the namespaces as tags; and the log-sum-exps
    join it to attention over the request's own tokens."""
    from paper_2607_05708_gb300 import MemStore
    rng = np.random.default_rng(31)
    n, e, k, T, heads, group, B = 96, 64, 8, 16, 2, 2, 6
    emb = rng.standard_normal((n, e))
    emb /= np.linalg.norm(emb, axis=1, keepdims=True)
    bits16 = torch.from_numpy(emb).bfloat16().view(torch.int16)
    store = MemStore(e, n, chunks_per_page=4)
    store.append_chunks(bits16.cuda())
    ns = (np.arange(n) % 16).astype(np.int32)          # six chunks each: lists end early
    store.set_namespace(0, _gpu(ns))
    q_ns = np.arange(B).astype(np.int32)
    ids, _, _, _ = store.retrieve(bits16[10:10 + B].contiguous().cuda(), k, 0.0, 0, q_ns=_gpu(q_ns),
                                  sort_by_time=True)
    store.sync()
    assert int((ids < 0).sum()) == B * (k - 6)

    c = _cache(n, heads, dim, block_tokens=T, bits=bits, tagged=True)
    kk, k64 = _values(rng, n * T, heads, dim, dtype)
    vv, v64 = _values(rng, n * T, heads, dim, dtype)
    short = np.arange(n * T) % T >= np.repeat(rng.integers(3, T + 1, n), T)    # chunks of any length
    tags = np.where(short, -1, np.repeat(ns, T)).astype(np.int32)
    c.write(kk, vv, _gpu(np.where(short, -1, np.arange(n * T))), tags=_gpu(tags))
    q = torch.from_numpy(rng.standard_normal((B, heads * group, dim))).to(DT[dtype])
    got = c.attend(q.cuda(), ids, causal=False, q_tags=_gpu(q_ns))
    c.sync()
    want = orc.attend(q.double().numpy(), orc.stored(k64, bits), orc.stored(v64, bits), ids.cpu().numpy(),
                      T, [k * T] * B, np.arange(B + 1), causal=False, tags=tags, q_tags=q_ns)
    _compare(got, want, dim, dtype, bits)

    # the same chunks and some more tokens in one list: the two parts join by their totals
    own = _gpu((np.arange(B)[:, None] * 3 + np.arange(3)) % n)
    part = c.attend(q.cuda(), own, causal=False, q_tags=_gpu(q_ns))
    both = c.attend(q.cuda(), torch.cat((ids, own), 1), causal=False, q_tags=_gpu(q_ns))
    c.sync()
    lse = torch.logaddexp(got[1], part[1])
    w = [torch.exp(x[1] - lse)[..., None].nan_to_num() for x in (got, part)]
    mix = got[0].float() * w[0] + part[0].float() * w[1]
    # three results rounded to 16 bits, and the weights' roundings twice
    eps = torch.finfo(DT[dtype]).eps
    scale = float(torch.from_numpy(np.abs(v64)).max())
    assert float((mix - both[0].float()).abs().max()) <= 3 * eps * scale
    seen = torch.isfinite(both[1])
    assert torch.allclose(lse[seen], both[1][seen], atol=1e-4, rtol=1e-5)

"""Decode in 4 bits on the GPU: precision, streams, stored bits and sizes beside those of test_gpu_q4.py (same oracle, same tolerances)."""
import math

import numpy as np
import pytest

from oracle import fp4_oracle as fp4
from paper_2601_13155_amd import binding, runtime, synth
from tests import test_gpu_q4 as q4_tests
from tests.test_gpu_q4 import HALF, SUM, append, ctx_for, layer_for, make_pairs, rounded, torch  # noqa: F401  (torch: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grp,Hkv,d", [(1, 4, 32), (4, 2, 128), (7, 2, 64), (8, 1, 128), (9, 1, 128), (16, 2, 64)])
@pytest.mark.parametrize("n", [2, 5, 40, 1100, 5000])
def test_attention_weights_are_not_rounded_to_bf16(torch, dtype, grp, Hkv, d, n):  # noqa: F811
    """Every dimension has one key with a value, so an output is that key's weight by its value and shows the weight's own error.  The bound leaves room for the
    output's rounding once and for a weight that is off by 2^-15 (two bf16 parts: 2^-7 is left behind a truncation, of that 2^-8), not for one that is off by 2^-8.  Scores: SUM(d) of their
    terms and 2^-22 of the largest, twice (a weight and the sum over all); exponential 2^-22 twice; the sum SUM(n); the merge and the division three steps."""
    ctx, shape = ctx_for(dtype, H=grp * Hkv, Hkv=Hkv, d=d)
    rng = np.random.default_rng(grp * 1000 + d + n)
    caches = runtime.KV4Batch(shape, [n, n])
    pairs = []
    for _ in range(2):
        k, v = make_pairs(rng, n, Hkv, d, dtype)
        few = min(n, 8)
        at = np.sort(rng.permutation(n)[:few])
        v[:] = 0
        for i, j in enumerate(at):
            v[j, :, i::few] = 1.0 + 0.5 * (i % 3)
        k[at] *= 2.0                                    # the keys with values reach the largest scores more often
        pairs.append((rounded(k, dtype), v))
    append(torch, ctx, caches, [(k, v, np.arange(n)) for k, v in pairs], dtype)
    q = rounded(rng.standard_normal((2, grp * Hkv, d)), dtype)
    out = torch.empty(q.shape, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    ctx.spts_kv4_attn(runtime.to_device(q, dtype), caches.structs, out)
    torch.cuda.synchronize()
    got = runtime.to_host(out).astype(np.float64)
    weight = 2.0 ** -15 if dtype == "bf16" else 2.0 ** -23
    for b in range(2):
        k, v = (fp4.fp4_round(a) for a in pairs[b])
        ref = fp4.attend(q[b].astype(np.float64), k, v)
        for h in range(grp * Hkv):
            kh, qh = k[:, h // grp], q[b, h].astype(np.float64)
            ds = (SUM(d) * (np.abs(kh) @ np.abs(qh)).max() + 2.0 ** -22 * np.abs(kh @ qh).max()) / math.sqrt(d)
            tol = (2 * (ds + 2.0 ** -22) + SUM(n) + weight + 3 * 2.0 ** -23 + HALF[dtype]) * np.abs(ref[h])
            err = np.abs(got[b, h] - ref[h])
            assert np.all(err <= tol), (b, h, float((err / np.maximum(tol, 1e-300)).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grp,d", [(4, 32), (8, 128), (12, 64)])
@pytest.mark.parametrize("n,low", [(33, [32]), (70, list(range(32))), (700, list(range(0, 64)) + [699]), (1500, list(range(256)) + [1499]),
                                   (9000, list(range(128, 512)) + [8999])])
def test_attention_scores_below_all_of_fp32(torch, dtype, grp, d, n, low):  # noqa: F811
    """Keys whose score is -inf in fp32 (d products of -2^190) weigh nothing, also where a wavefront, a share or the end of the cache has no others; the
    remaining scores are small multiples of 2^-4 over sqrt(d), exact sums in fp32, so the bound is that of the exponentials and the weighted sum alone."""
    ctx, shape = ctx_for(dtype, H=2 * grp, Hkv=2, d=d)
    rng = np.random.default_rng(n)
    k = 2.0 ** -95 * rng.choice([-2.0, -1.0, -0.5, 0.5, 1.0, 2.0], (n, 2, d))
    k[low] = -2.0 ** 95
    v = rounded(rng.standard_normal((n, 2, d)), dtype)
    v[low] = 1000.0
    q = 2.0 ** 95 * rng.choice([0.125, 0.25], (1, 2 * grp, d))
    caches = runtime.KV4Batch(shape, [n])
    append(torch, ctx, caches, [(k.astype(np.float32), v, np.arange(n))], dtype)
    out = torch.empty(q.shape, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    ctx.spts_kv4_attn(runtime.to_device(q.astype(np.float32), dtype), caches.structs, out)
    torch.cuda.synchronize()
    got = runtime.to_host(out).astype(np.float64)[0]
    kq, vq = fp4.fp4_round(k), fp4.fp4_round(v)
    assert np.array_equal(kq, k)
    ref = fp4.attend(q[0], kq, vq)
    keep = np.setdiff1d(np.arange(n), low)
    for h in range(2 * grp):
        s = kq[keep, h // grp] @ q[0, h] / math.sqrt(d)
        p = np.exp(s - s.max())
        mag = p @ np.abs(vq[keep, h // grp]) / p.sum()
        tol = (2 * (2.0 ** -22 * np.abs(s).max() + 2.0 ** -22 + SUM(n)) + 2.0 ** -15 + 3 * 2.0 ** -23) * mag + HALF[dtype] * np.abs(ref[h])
        assert np.all(np.abs(got[h] - ref[h]) <= tol), (h, got[h][:4], ref[h][:4])


# -------------------------------------------------------------------------------------------------------------- streams
_BUSY = {}


def keep_busy(torch, stream):  # noqa: F811
    """Some 20 ms of products on a stream: what it is given next is late."""
    if not _BUSY:
        _BUSY["a"] = torch.ones((4096, 4096), device="cuda")
        _BUSY["c"] = torch.empty_like(_BUSY["a"])
        torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(20):
            torch.matmul(_BUSY["a"], _BUSY["a"], out=_BUSY["c"])


@pytest.fixture
def side(torch):  # noqa: F811
    """A context on a stream of its own, over the shape of ctx_for("bf16"); the tests call from the default stream."""
    _, shape = ctx_for("bf16")
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = binding.Context(shape, 256, 1, 1, shape.Dff, stream=st)
    torch.cuda.synchronize()
    assert torch.cuda.current_stream() != st
    return ctx


@pytest.mark.parametrize("view", ["transposed", "columns", "rows"])
def test_a_copied_matrix_is_packed_after_it_is_copied(torch, side, view):  # noqa: F811
    """The copy of a strided matrix is made behind a busy current stream and packed on an idle one."""
    base = torch.randn((640, 640), device="cuda").to(torch.bfloat16)
    W = {"transposed": base.t(), "columns": base[:, 64:], "rows": base[::2]}[view]
    alone = W.contiguous()
    want = runtime.Q4Matrix(ctx_for("bf16")[0], alone)
    torch.cuda.synchronize()
    del alone
    junk = torch.full(W.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    del junk
    keep_busy(torch, torch.cuda.current_stream())
    got = runtime.Q4Matrix(side, W)
    torch.cuda.synchronize()
    assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales)


def test_a_cache_is_read_back_after_earlier_work(torch, side):  # noqa: F811
    """A prefill's cache converted and read back while the current stream is still writing the pairs, and then what lies where the rows are read to."""
    _, shape = ctx_for("bf16")
    rng = np.random.default_rng(5)
    k, v = make_pairs(rng, 100, shape.Hkv, shape.d, "bf16")
    kd, vd = runtime.to_device(k, "bf16"), runtime.to_device(v, "bf16")
    kept, caches = runtime.KVCache(shape, 100), runtime.KV4Batch(shape, [100])
    torch.cuda.synchronize()
    keep_busy(torch, torch.cuda.current_stream())
    kept.k.copy_(kd)
    kept.v.copy_(vd)
    kept.pos.copy_(torch.arange(100, device="cuda"))
    kept.struct.count = 100
    caches.append_cache(side, 0, kept)
    late = [torch.full((100, shape.Hkv, shape.d), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    del late
    gk, gv, gp = caches.host(side, shape, 0)
    assert np.array_equal(gk, fp4.fp4_round(k)) and np.array_equal(gv, fp4.fp4_round(v)) and np.array_equal(gp, np.arange(100))


def make_runner(torch, ctx, nseq, history):  # noqa: F811
    """A runner over two layers and caches of its own, everything made from fixed seeds; (runner, history tensor)."""
    shape, main = ctx.shape, ctx_for("bf16")[0]
    rng, V = np.random.default_rng(70), 416
    layers = [layer_for(torch, main, shape, 71 + l)[0] for l in range(2)]
    lens = [40, 7, 25][:nseq]
    caches = [runtime.KV4Batch(shape, [n + 16 for n in lens]) for _ in layers]
    for c in caches:
        append(torch, main, c, [make_pairs(rng, n, shape.Hkv, shape.d, "bf16") + (np.arange(n),) for n in lens], "bf16")
    table = runtime.to_device(rounded(rng.standard_normal((V, shape.D)), "bf16"), "bf16")
    gamma = runtime.to_device(rounded(1.0 + 0.1 * rng.standard_normal(shape.D), "bf16"), "bf16")
    hist = torch.from_numpy(rng.integers(0, V, (nseq, 20)).astype(np.int32)).cuda() if history else None
    rules = runtime.LogitsRules(nseq, history=hist, history_len=[5, 3, 9][:nseq], prompt_len=[5, 3, 9][:nseq], repetition=[1.3] * nseq, frequency=[0.8] * nseq) if history else None
    run = runtime.Q4DecodeRunner(ctx, shape, layers, caches, gamma, table, runtime.Q4Matrix(main, table), rules)
    return run, hist, table[3:3 + nseq].clone(), lens


@pytest.mark.parametrize("history", [False, True])
@pytest.mark.parametrize("nseq", [1, 3])
def test_generate_on_a_side_stream(torch, side, nseq, history):  # noqa: F811
    """The first state is written by a busy current stream, the context's stream is busy as well: tokens, history, states and logits of five steps are
    those of a run on one stream; and the same for a step and a token of their own."""
    res = []
    for ctx in (ctx_for("bf16")[0], side):
        run, hist, x0, lens = make_runner(torch, ctx, nseq, history)
        toks = torch.full((nseq, 5), -5, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        if ctx is side:
            keep_busy(torch, torch.cuda.current_stream())
        run.x.copy_(x0)
        if ctx is side:
            keep_busy(torch, ctx.stream)
        run.generate(lens, 5, toks)
        got = [t.clone() for t in [toks, run.x, run.logits, run.tokens] + ([hist] if history else [])]
        if ctx is side:
            keep_busy(torch, torch.cuda.current_stream())
        run.x.copy_(x0)
        if ctx is side:
            keep_busy(torch, ctx.stream)
        run.step([n + 5 for n in lens])
        got.append(run.x.clone())
        run.next_token()
        got += [run.logits.clone(), run.tokens.clone(), run.x_next.clone()]
        torch.cuda.synchronize()
        res.append([t.cpu() for t in got] + [torch.tensor(c.counts) for c in run.caches])
    assert all(torch.equal(a, b) for a, b in zip(*res)), [torch.equal(a, b) for a, b in zip(*res)]
    assert (res[0][0] >= 0).all()


# --------------------------------------------------------------------------------------------- the layer's stored pairs
def pairs_of_every_kind(rng, n, dtype):
    """n values (a multiple of 32) whose blocks have sizes of their own over 2^-20 .. 2^20: random ones, ties between codes, zeros, one value alone, the edges of an
    exponent."""
    out = np.empty((n // 32, 32))
    for i in range(n // 32):
        kind, a = i % 6, rng.standard_normal(32)
        if kind == 1:
            a = np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], 32) * rng.choice([-1.0, 1.0], 32)
        elif kind == 2:
            a = np.where(np.arange(32) == rng.integers(32), 1.0, 0.0)
        elif kind == 3:
            a = a / np.abs(a).max() * (6.0 if i % 4 else 6.03125)      # the largest that an exponent holds, and the next bf16
        elif kind == 4 and i % 12 == 4:
            a = np.zeros(32)
        out[i] = a * 2.0 ** rng.integers(-20, 21)
    return rounded(out.reshape(-1), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,d", [(5, 32), (3, 64), (1, 64), (2, 128), (8, 128)])
@pytest.mark.parametrize("nseq", [1, 3, 16])
def test_the_layer_stores_the_nearest_4_bit_values(torch, dtype, Hkv, d, nseq):  # noqa: F811
    """States of +-1 have a norm of exactly 1 (an epsilon of 2^-100 vanishes beside it), so a projection row with a single 1 gives the gain of its column with the state's sign, exactly;
    at position 0 the rotation is the identity.  Keys and values of the new pair are then known to the bit, and so is what 4 bits make of them."""
    n = Hkv * d
    D = 2 * n
    ctx, shape = ctx_for(dtype, H=Hkv, Hkv=Hkv, d=d, D=D, Dff=1024, rms_eps=2.0 ** -100)
    rng = np.random.default_rng(n + nseq)
    gains = np.concatenate([pairs_of_every_kind(rng, n, dtype), pairs_of_every_kind(rng, n, dtype)])
    eye = np.eye(D, dtype=np.float32)
    w = {"Wq": np.zeros((n, D)), "Wk": eye[:n], "Wv": eye[n:], "Wo": np.zeros((D, n)), "Wgate": np.zeros((1024, D)), "Wup": np.zeros((1024, D)), "Wdown": np.zeros((D, 1024))}
    t = {k: runtime.to_device(np.asarray(a, dtype=np.float32), dtype) for k, a in w.items()}
    t["gamma1"], t["gamma2"] = runtime.to_device(gains.astype(np.float32), dtype), runtime.to_device(np.ones(D, dtype=np.float32), dtype)
    q4 = runtime.pack_layer_q4(ctx, binding.layer_weights(t))
    held = [int(c) for c in rng.integers(0, 40, nseq)]
    caches = runtime.KV4Batch(shape, [c + 2 for c in held])
    append(torch, ctx, caches, [make_pairs(rng, c, Hkv, d, dtype) + (np.arange(c),) for c in held], dtype)
    before = [caches.host(ctx, shape, b) for b in range(nseq)]
    for _ in range(2):
        sign = rng.choice([-1.0, 1.0], (nseq, D)).astype(np.float32)
        x = runtime.to_device(sign.copy(), dtype)
        ctx.spts_decode_layer_q4(x, [0] * nseq, q4, caches.structs)
        torch.cuda.synchronize()
        assert np.array_equal(runtime.to_host(x), sign)                # nothing is added to the state
        for b in range(nseq):
            k, v, p = caches.host(ctx, shape, b)
            assert len(k) == len(before[b][0]) + 1 and p[-1] == 0
            assert np.array_equal(k[:-1], before[b][0]) and np.array_equal(v[:-1], before[b][1])
            new = gains * sign[b].astype(np.float64)
            assert np.array_equal(k[-1], fp4.fp4_round(new[:n].reshape(Hkv, d))), b
            assert np.array_equal(v[-1], fp4.fp4_round(new[n:].reshape(Hkv, d))), b
            before[b] = (k, v, p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nseq,D", [(1, 4096), (2, 2568), (3, 2568), (4, 2568), (3, 4096), (4, 4096), (3, 4616), (4, 4104)])
def test_decode_layer_of_several_slabs(torch, monkeypatch, dtype, nseq, D):  # noqa: F811
    """The layer in lockstep with the oracle where the norm of one to four vectors inside the products goes over several slabs of 512, whole and partial
    last ones, up to the most that LDS is kept for, and just beyond."""
    monkeypatch.setattr(q4_tests, "LAYERS", [(D, 4, 2, 32, 64)])
    q4_tests.test_decode_layer_lockstep(torch, dtype, nseq, 0)


def test_append_and_read_of_more_rows_than_a_launch(torch):  # noqa: F811
    """2^24 + 1000 rows of two sequences: rows on both sides of where the second launch begins, the ends, and some between."""
    Hkv, d, n = 1, 32, (1 << 24) + 1000
    ctx, shape = ctx_for("bf16", H=1, Hkv=Hkv, d=d)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    lens = [n - 700, 700]
    k = torch.randn((n, Hkv, d), generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn((n, Hkv, d), generator=g, device="cuda").to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 3
    caches = runtime.KV4Batch(shape, lens)
    for t in caches.tensors:
        for x in t[:4]:
            x.fill_(0xFF)
        t[4].fill_(-1)
    offs = [0, lens[0], n]
    ctx.spts_kv4_append(k, v, pos, offs, caches.structs)
    torch.cuda.synchronize()
    assert caches.counts == lens
    assert torch.equal(caches.tensors[0][4][:lens[0]], pos[:lens[0]]) and torch.equal(caches.tensors[1][4][:700], pos[lens[0]:])
    kb, vb = torch.empty_like(k), torch.empty_like(v)
    ctx.spts_kv4_read(caches.structs, offs, kb, vb)
    torch.cuda.synchronize()
    rows = np.unique(np.concatenate([np.arange(64), np.arange((1 << 24) - 64, n), np.random.default_rng(3).integers(0, n, 2000)]))
    at = torch.from_numpy(rows).cuda()
    for src, back in ((k, kb), (v, vb)):
        assert np.array_equal(runtime.to_host(back[at]), fp4.fp4_round(runtime.to_host(src[at])))
    # the same bytes as from calls that stay below a launch's rows
    again = runtime.KV4Batch(shape, lens)
    half = 1 << 23
    for lo in range(0, n, half):
        hi = min(lo + half, n)
        cut = [0, max(0, min(hi, lens[0]) - lo), hi - lo]
        ctx.spts_kv4_append(k[lo:hi], v[lo:hi], pos[lo:hi], cut, again.structs)
    torch.cuda.synchronize()
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    for lo in range(0, lens[0], half):
        c = min(half, lens[0] - lo)
        ctx.spts_kv4_read([again.structs[0]], [0, c], k2[lo:lo + c], v2[lo:lo + c], first=[lo])
    ctx.spts_kv4_read([again.structs[1]], [0, 700], k2[lens[0]:], v2[lens[0]:])
    torch.cuda.synchronize()
    assert torch.equal(k2, kb) and torch.equal(v2, vb)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,Hkv,d", [(16, 8, 64), (9, 9, 128)])
def test_decode_layer_with_more_head_dimensions_than_hidden_ones(torch, monkeypatch, dtype, heads, Hkv, d):  # noqa: F811
    """Sixteen sequences' projections are larger than everything that the feed-forward block of this model needs."""
    monkeypatch.setattr(q4_tests, "LAYERS", [(64, heads, Hkv, d, 8)])
    q4_tests.test_decode_layer_lockstep(torch, dtype, 16, 0)


@pytest.mark.parametrize("own_stream", [False, True])
def test_generate_captured_and_replayed(torch, side, own_stream):  # noqa: F811
    """One step of generate with a history under a graph, captured on the context's stream or on another that the context's joins; replayed between eager runs of another
    runner over the same context, after which every buffer is what the eager step leaves."""
    want, (run, hist, x0, lens) = [], make_runner(torch, side, 3, True)
    eager, hist_e, _, _ = make_runner(torch, side, 3, True)
    toks, toks_e = (torch.full((3, 1), -5, dtype=torch.int32, device="cuda") for _ in range(2))
    eager.x.copy_(x0)
    eager.generate(lens, 1, toks_e)                     # the first use of every kernel, and the result
    want = [t.clone() for t in (toks_e, eager.x, eager.logits, hist_e)]
    start = hist.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side.stream if own_stream else torch.cuda.Stream()):
        run.x.copy_(x0)
        run.generate(lens, 1, toks)
    for t in range(4):
        for b in (run.x, run.logits, run.x_next, toks):
            b.zero_()
        hist.copy_(start)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((toks, run.x, run.logits, hist), want)), t
        eager.generate([n + 1 + t for n in lens], 1, toks_e)
        torch.cuda.synchronize()
    assert [c.counts for c in run.caches] == [[n + 1 for n in lens]] * 2
    for a, b in zip(run.caches, eager.caches):
        for s, n in enumerate(lens):
            assert all(np.array_equal(p, q[:n + 1]) for p, q in zip(a.host(side, side.shape, s), b.host(side, side.shape, s)))

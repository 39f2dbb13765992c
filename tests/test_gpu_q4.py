"""Decode in 4 bits on the GPU through the C ABI: packed matrices and their products, 4-bit caches and their attention, rules on
logits, and the layer that uses them, against the fp64 oracle.

Tolerances.  Stored values are exact, so reading back is compared bit for bit.  A product's terms (a 4-bit value times a bf16, or
a third of an fp32) are exact in fp32; what is left is the sum.  Whatever its order, a sum of n terms that is taken in
pieces of 32 has at most n / 32 + 64 additions behind one another (64: within a piece and over the lanes and wavefronts), each off
by a step (2^-23) of a partial sum, which is at most sum|term|: SUM(n) = (n / 32 + 64) 2^-23.  An output in bf16 is off by
another 2^-8 of itself, in fp32 by 2^-24."""
import math

import numpy as np
import pytest

from oracle import fp4_oracle as fp4
from oracle import spts_oracle as orc
from paper_2601_13155_amd import binding, runtime, synth
from tests import helpers as H

pytestmark = pytest.mark.gpu

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def SUM(n):
    return (n / 32 + 64) * 2.0 ** -23


@pytest.fixture(scope="module")
def torch():
    import torch
    assert torch.cuda.is_available()
    return torch


_CTX = {}


def ctx_for(dtype, H=4, Hkv=2, d=64, D=256, Dff=688, rows=256, **kw):
    shape = synth.ModelShape(D=D, H=H, Hkv=Hkv, d=d, Dff=Dff, dtype=dtype, **kw)
    if (shape, rows) not in _CTX:
        _CTX[shape, rows] = runtime.make_context(shape, rows, 1, 1, Dff)
    return _CTX[shape, rows], shape


def rounded(a, dtype):
    a = np.asarray(a, dtype=np.float32)
    return orc.bf16_round(a).astype(np.float32) if dtype == "bf16" else a


# ----------------------------------------------------------------------------------------------------------- matrices
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,nb", [(1, 8, 1), (16, 32, 2), (17, 40, 3), (15, 512, 16), (64, 520, 5), (33, 688, 7), (100, 1032, 4), (48, 2048, 8),
                                       (16, 4096, 1), (1003, 688, 16), (5, 18944, 9),
                                       (4090, 520, 3), (4100, 1032, 1), (8200, 520, 2), (8216, 1544, 3), (4100, 264, 6), (8190, 136, 16), (8216, 648, 8), (8200, 392, 13)])
def test_product_of_whole_numbers_is_exact(torch, dtype, rows, K, nb):
    """Grid values times small whole numbers: every sum is a multiple of 1/2 below 2^23 whatever its order, so each output has one
    right bit pattern, and a missed, doubled or misplaced term shows."""
    ctx, _ = ctx_for(dtype)
    rng = np.random.default_rng(rows * 31 + K)
    W = rng.choice(np.concatenate([fp4.GRID, -fp4.GRID]), (rows, K))
    W[:, ::32] = 6.0                                   # the block's exponent is 0
    x = rng.integers(-8, 9, (nb, K)).astype(np.float64)
    assert np.abs(W).max() * 8 * K < 2 ** 22
    m = runtime.Q4Matrix(ctx, runtime.to_device(W.astype(np.float32), dtype))
    y = torch.full((nb, rows), 7.0, dtype=torch.float32, device="cuda")
    ctx.spts_matvec_q4(m.struct, runtime.to_device(x.astype(np.float32), dtype), nb, y, 1)
    torch.cuda.synchronize()
    assert np.array_equal(y.cpu().numpy().astype(np.float64), x @ W.T)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,K,nb", [(64, 256, 1), (31, 1000, 3), (256, 4096, 16), (70, 14336, 2)])
def test_product_against_the_oracle(torch, dtype, rows, K, nb):
    ctx, _ = ctx_for(dtype)
    rng = np.random.default_rng(K)
    W = rounded(rng.standard_normal((rows, K)) / math.sqrt(K) * np.exp(rng.standard_normal((rows, 1))), dtype)
    x = rounded(rng.standard_normal((nb, K)) * np.exp(rng.standard_normal((1, K))), dtype)
    m = runtime.Q4Matrix(ctx, runtime.to_device(W, dtype))
    xd = runtime.to_device(x, dtype)
    y = torch.empty((nb, rows), dtype=xd.dtype, device="cuda")
    f = torch.empty((nb, rows), dtype=torch.float32, device="cuda")
    ctx.spts_matvec_q4(m.struct, xd, nb, y)
    ctx.spts_matvec_q4(m.struct, xd, nb, f, 1)
    alone = torch.empty((1, rows), dtype=torch.float32, device="cuda")
    torch.cuda.synchronize()
    Wq = fp4.fp4_round(W)
    ref, mag = x.astype(np.float64) @ Wq.T, np.abs(x.astype(np.float64)) @ np.abs(Wq).T
    tol = SUM(K) * mag + 2.0 ** -24 * np.abs(ref)
    assert np.all(np.abs(f.cpu().numpy() - ref) <= tol)
    assert np.all(np.abs(runtime.to_host(y) - ref) <= tol + HALF[dtype] * np.abs(ref))
    for b in range(nb):                                # the same bits alone as in the batch
        ctx.spts_matvec_q4(m.struct, xd[b].contiguous(), 1, alone, 1)
        torch.cuda.synchronize()
        assert torch.equal(alone[0], f[b])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pack_limits(torch, dtype):
    """Values at the ends of the type's range, blocks of zeros, ties, a NaN block: each row of W times the identity."""
    ctx, _ = ctx_for(dtype)
    K = 96
    W = np.zeros((9, K), dtype=np.float32)
    W[0, :32] = np.linspace(-6, 6, 32)
    W[1, :16] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, -6.0]
    W[2, 32:64] = 3.3e38
    W[3, 64:] = 1e-37
    W[4, 5] = 1e-20
    W[5, :] = np.random.default_rng(3).standard_normal(K)
    W[6, 40] = np.nan
    W[6, 64:] = 1.0
    W[7, 3], W[7, 33] = np.inf, -np.inf
    W[8, 0] = 1e-40
    W = rounded(W, dtype)
    W[6, 40] = np.nan
    m = runtime.Q4Matrix(ctx, runtime.to_device(W, dtype))
    got = np.empty((K, 9))
    for k0 in range(0, K, 16):
        x = np.zeros((16, K), dtype=np.float32)
        x[np.arange(16), k0 + np.arange(16)] = 1.0
        y = torch.empty((16, 9), dtype=torch.float32, device="cuda")
        ctx.spts_matvec_q4(m.struct, runtime.to_device(x, dtype), 16, y, 1)
        torch.cuda.synchronize()
        got[k0:k0 + 16] = y.cpu().numpy()
    clean = np.where(np.isinf(W), np.sign(W) * 3e38, np.nan_to_num(W)).astype(np.float64)
    want = fp4.fp4_round(clean).T
    ok = [0, 1, 2, 3, 4, 5, 7, 8]
    assert np.array_equal(got[:, ok], want[:, ok])
    assert np.isnan(got[:, 6]).all()                   # a NaN block poisons the row's sums


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_product_with_infinities_and_the_largest_numbers(torch, dtype):
    """A vector's infinity, NaN or largest number reaches the rows as IEEE arithmetic has it (an infinity times a stored zero is NaN), and no other
    vector of the batch."""
    ctx, _ = ctx_for(dtype)
    rng = np.random.default_rng(8)
    rows, K = 33, 600
    W = rng.choice(np.array([0.0, 0.25, -0.25, 0.5, -0.5]), (rows, K)).astype(np.float32)
    W[:, ::32] = 0.5                                    # exact in 4 bits
    x = rng.integers(-8, 9, (6, K)).astype(np.float32)
    top = np.float32(3.4028234e38) if dtype == "f32" else np.float32(3.3895314e38)
    x[0, 37], x[1, 599], x[3, 0], x[4, 300], x[4, 301] = np.inf, -np.inf, top, top, -top
    x[2, 5] = np.array([0x7f800001], dtype=np.uint32).view(np.float32)[0]               # a NaN whose upper half alone is an infinity
    xd = runtime.to_device(x, dtype)
    if dtype == "bf16":
        xd[2, 5] = float("nan")
    m = runtime.Q4Matrix(ctx, runtime.to_device(W, dtype))
    y = torch.empty((6, rows), dtype=torch.float32, device="cuda")
    ctx.spts_matvec_q4(m.struct, xd, 6, y, 1)
    torch.cuda.synchronize()
    got = y.cpu().numpy().astype(np.float64)
    with np.errstate(invalid="ignore"):
        x64 = x.astype(np.float64)
        ref = np.array([[(W[r].astype(np.float64) * x64[b]).sum() for r in range(rows)] for b in range(6)])
    assert np.isinf(ref[:2]).any() and np.isnan(ref[:2]).any() and np.isnan(ref[2]).all()
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    fin = np.isfinite(ref)
    mag = np.abs(np.where(np.isfinite(x64), x64, 0.0)) @ np.abs(W.astype(np.float64)).T
    assert np.all(np.abs(got[fin] - ref[fin]) <= (SUM(K) * mag + 2.0 ** -24 * np.abs(np.where(fin, ref, 0)))[fin])
    assert np.array_equal(got[5], ref[5])               # whole numbers and quarters


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_product_of_the_longest_rows(torch, dtype):
    """16 vectors of 2^26 values (fp32: 4 GB, byte offsets just below 2^32) that are zero but for a few whole numbers at either end."""
    ctx, _ = ctx_for(dtype)
    K = 1 << 26
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    W = torch.ones((1, K), dtype=tdt, device="cuda")
    W[0, 1::2] = -1.0
    m = runtime.Q4Matrix(ctx, W)
    del W
    x = torch.zeros((16, K), dtype=tdt, device="cuda")
    want = []
    for b in range(16):
        at = [b, K // 2 + 33 * b + 1, K - 1, K - 1 - 7 * b - 2]
        vals = [1.0, 4.0, 16.0, 64.0]
        for i, v in zip(at, vals):
            x[b, i] = v
        want.append(sum(v * (-1.0 if i % 2 else 1.0) for i, v in zip(at, vals)))
    y = torch.empty((16, 1), dtype=torch.float32, device="cuda")
    ctx.spts_matvec_q4(m.struct, x, 16, y, 1)
    torch.cuda.synchronize()
    assert y[:, 0].tolist() == want


# ------------------------------------------------------------------------------------------------------------- caches
def make_pairs(rng, n, Hkv, d, dtype):
    k = rounded(rng.standard_normal((n, Hkv, d)) * np.exp(rng.standard_normal((1, Hkv, d))), dtype)
    return k, rounded(rng.standard_normal((n, Hkv, d)), dtype)


def append(torch, ctx, caches, parts, dtype):
    """parts: (k, v, pos) per sequence, in one call."""
    offs = np.concatenate([[0], np.cumsum([len(p[0]) for p in parts])])
    k, v, pos = (np.concatenate([p[i] for p in parts]) for i in range(3))
    ctx.spts_kv4_append(runtime.to_device(k, dtype), runtime.to_device(v, dtype), torch.from_numpy(pos.astype(np.int32)).cuda(), offs.tolist(), caches.structs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,d", [(1, 32), (2, 64), (3, 128), (8, 128)])
def test_append_and_read_back(torch, dtype, Hkv, d):
    """Ragged appends in several calls, none at all to one sequence in some: values, positions and counts; rows behind the counts
    keep what was there."""
    ctx, shape = ctx_for(dtype, H=Hkv, Hkv=Hkv, d=d)
    rng = np.random.default_rng(Hkv * d)
    caps = [40, 8, 1, 200]
    caches = runtime.KV4Batch(shape, caps)
    for t in caches.tensors:
        for x in t[:4]:
            x.fill_(0xA5)
        t[4].fill_(-7)
    held = [[], [], [], []]
    for sizes in ([3, 8, 0, 65], [1, 0, 1, 1], [0, 0, 0, 0], [36, 0, 0, 77]):
        parts = []
        for b, n in enumerate(sizes):
            k, v = make_pairs(rng, n, Hkv, d, dtype)
            parts.append((k, v, rng.integers(0, 1 << 20, n)))
            held[b].append(parts[-1])
        append(torch, ctx, caches, parts, dtype)
    counts = [40, 8, 1, 143]
    assert caches.counts == counts
    for b in range(4):
        k, v, pos = (np.concatenate([p[i] for p in held[b]]) for i in range(3))
        gk, gv, gp = caches.host(ctx, shape, b)
        assert np.array_equal(gk, fp4.fp4_round(k)) and np.array_equal(gv, fp4.fp4_round(v)) and np.array_equal(gp, pos)
        assert (caches.tensors[b][4][counts[b]:] == -7).all()
    # rows behind the counts: the bytes that a fresh cache with the same rows does not write either
    t = caches.tensors[3]
    row = d // 2
    tail = t[0].view(Hkv, 200, row)[:, 143:]
    assert (tail == 0xA5).all() and (t[2].view(Hkv, 200, d // 32)[:, 143:] == 0xA5).all()
    assert (t[1].view(Hkv, 25, 16, 8, d // 32)[:, 18:] == 0xA5).all() and (t[1].view(Hkv, 25, 16, 8, d // 32)[:, 17, :, 7] == 0xA5).all()
    # a middle part of some sequences in one call
    k = torch.empty((60, Hkv, d), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    v = torch.empty_like(k)
    ctx.spts_kv4_read(caches.structs, [0, 10, 10, 11, 60], k, v, first=[7, 8, 0, 90])
    torch.cuda.synchronize()
    for b, (lo, at, n) in enumerate([(7, 0, 10), (8, 10, 0), (0, 10, 1), (90, 11, 49)]):
        gk, gv, _ = caches.host(ctx, shape, b)
        assert np.array_equal(runtime.to_host(k[at:at + n]), gk[lo:lo + n]) and np.array_equal(runtime.to_host(v[at:at + n]), gv[lo:lo + n])


def attend_tol(q, k, v, dtype):
    """Elementwise bound for one head, q [d], k, v [n, d].  Scores: a sum of d exact terms, two more roundings, 2^-24 of the argument of the
    exponential; each shifts its weight by that much of itself.  Weights: rounded to the type (bf16: 2^-8, fp32: three bf16 parts, 2^-24) and
    the exponential's own 2^-22; sums over n pairs; the merge of shares and the division are three more steps."""
    n, d = k.shape
    s = k @ q / math.sqrt(d)
    ds = SUM(d) * (np.abs(k) @ np.abs(q)).max() / math.sqrt(d) + 2.0 ** -22 * np.abs(s).max()
    p = np.exp(s - s.max())
    p /= p.sum()
    o = p @ v
    return (HALF[dtype] + 2 * (ds + 2.0 ** -22 + SUM(n)) + 2.0 ** -21) * (p @ np.abs(v)) + (HALF[dtype] + 2.0 ** -22) * np.abs(o)


def check_attend(torch, ctx, caches, q, lens, pairs, dtype):
    out = torch.full(q.shape, 9.0, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    ctx.spts_kv4_attn(runtime.to_device(q, dtype), caches.structs, out)
    torch.cuda.synchronize()
    got = runtime.to_host(out).astype(np.float64)
    for b, n in enumerate(lens):
        k, v = (fp4.fp4_round(a[:n]) if n else a[:0].astype(np.float64) for a in pairs[b])
        ref = fp4.attend(q[b].astype(np.float64), k, v)
        if n == 0:
            assert not got[b].any()
            continue
        grp = q.shape[1] // k.shape[1]
        for h in range(q.shape[1]):
            tol = attend_tol(q[b, h].astype(np.float64), k[:, h // grp], v[:, h // grp], dtype)
            err = np.abs(got[b, h] - ref[h])
            assert np.all(err <= tol), (b, n, h, float((err / tol).max()))
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("grp,Hkv,d", [(1, 2, 32), (4, 2, 64), (7, 4, 128), (16, 1, 128), (3, 3, 64), (8, 1, 32)])
def test_attention_lengths(torch, dtype, grp, Hkv, d):
    """Lengths around every step of the kernels (one key, pieces of 8 and 16, steps of 32, splits), an empty cache among them; what lies
    behind the counts is NaN throughout."""
    ctx, shape = ctx_for(dtype, H=grp * Hkv, Hkv=Hkv, d=d)
    rng = np.random.default_rng(grp * d)
    for lens in ([1], [0], [5, 0, 8, 9, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 7, 2], [300, 1, 0, 511, 512, 513, 1025], [4099]):
        caches = runtime.KV4Batch(shape, [n + 3 for n in lens])
        for t in caches.tensors:
            for x in t[:4]:
                x.fill_(0xFF)
        pairs = [make_pairs(rng, n, Hkv, d, dtype) for n in lens]
        append(torch, ctx, caches, [(k, v, np.arange(len(k))) for k, v in pairs], dtype)
        q = rounded(1.5 * rng.standard_normal((len(lens), grp * Hkv, d)), dtype)
        check_attend(torch, ctx, caches, q, lens, pairs, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_attention_finds_each_key(torch, dtype, d):
    """A query that points at one key so sharply that every other weight is 0 in fp32 returns that key's value, bit for bit."""
    ctx, shape = ctx_for(dtype, H=2, Hkv=2, d=d)
    rng = np.random.default_rng(d)
    n = 171
    k = rng.choice([-1.0, 1.0], (n, 2, d)).astype(np.float32)
    v = rounded(rng.standard_normal((n, 2, d)), dtype)
    caches = runtime.KV4Batch(shape, [n])
    append(torch, ctx, caches, [(k, v, np.arange(n))], dtype)
    kq, vq = fp4.fp4_round(k), fp4.fp4_round(v)
    assert np.array_equal(kq, k)
    out = torch.empty((16, 2, d), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    same = (binding.spts_kv4 * 16)(*[caches.structs[0]] * 16)      # one cache, sixteen queries
    for j0 in range(0, n, 16):
        at = [min(j0 + i, n - 1) for i in range(16)]
        q = (512.0 * k[at]).astype(np.float32)
        ctx.spts_kv4_attn(runtime.to_device(q, dtype), same, out)
        torch.cuda.synchronize()
        got = runtime.to_host(out)
        for i, j in enumerate(at):
            for h in range(2):
                s = 512.0 * (k[:, h] @ k[j, h])
                twins = np.flatnonzero(s == s[j])
                if len(twins) == 1:
                    assert np.array_equal(got[i, h], vq[j, h].astype(np.float32)), (j, h)
                assert s[j] - np.max(np.delete(s, twins), initial=-np.inf) > 140 * math.sqrt(d)   # e^-140 < 2^-149


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_rising_scores(torch, dtype):
    """Scores that grow along the cache move the running maximum at every step; a long cache among short ones."""
    ctx, shape = ctx_for(dtype, H=8, Hkv=2, d=64)
    rng = np.random.default_rng(8)
    lens = [2500, 90, 700]
    pairs = []
    for n in lens:
        k, v = make_pairs(rng, n, 2, 64, dtype)
        k[:, :, :32] = np.linspace(0.1, 6.0, n)[:, None, None]
        pairs.append((rounded(k, dtype), v))
    caches = runtime.KV4Batch(shape, lens)
    append(torch, ctx, caches, [(k, v, np.arange(len(k))) for k, v in pairs], dtype)
    q = rounded(np.abs(rng.standard_normal((3, 8, 64))) * 0.5, dtype)
    q[:, 1] *= -1
    q[:, 2] = 0.0                                       # every weight the same
    check_attend(torch, ctx, caches, q, lens, pairs, dtype)


def test_attention_over_a_long_cache(torch):
    """A cache whose byte offsets pass 2^31 (and 2^32 with the second head): uniform weights over rows that differ only at the far end."""
    Hkv, d, n = 2, 128, 40_000_003
    ctx, shape = ctx_for("bf16", H=2, Hkv=Hkv, d=d)
    caches = runtime.KV4Batch(shape, [n])
    t = caches.tensors[0]
    cap = int(caches.structs[0].capacity)
    t[0].zero_(); t[1].zero_()
    t[2].fill_(127); t[3].fill_(127)
    caches.structs[0].count = n - 3
    rng = np.random.default_rng(4)
    k, v = np.zeros((3, Hkv, d), dtype=np.float32), rng.choice([1.0, 2.0, 3.0], (3, Hkv, d)).astype(np.float32)
    k[:, :, 0] = 6.0
    append(torch, ctx, caches, [(k, v, np.array([1, 2, 3]))], "bf16")
    assert caches.counts == [n] and cap * Hkv * 64 > 2 ** 32
    q = np.zeros((1, 2, d), dtype=np.float32)
    q[:, :, 0] = 128.0                                  # 6 * 128 / sqrt(128) = 67.9: e^-67.9 * 4e7 < 2^-70
    out = torch.empty((1, 2, d), dtype=torch.bfloat16, device="cuda")
    ctx.spts_kv4_attn(runtime.to_device(q, "bf16"), caches.structs, out)
    torch.cuda.synchronize()
    want = v.astype(np.float64).mean(0)
    assert np.all(np.abs(runtime.to_host(out)[0] - want) <= 3 * HALF["bf16"] * want)
    back = torch.empty((3, Hkv, d), dtype=torch.bfloat16, device="cuda")
    vb = torch.empty_like(back)
    ctx.spts_kv4_read(caches.structs, [0, 3], back, vb, first=[n - 3])
    torch.cuda.synchronize()
    assert np.array_equal(runtime.to_host(vb), v) and np.array_equal(runtime.to_host(back), k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_in_place_and_on_two_streams(torch, dtype):
    """The output may be the queries' place; two contexts on streams of their own do not touch each other's shares (one launch and two)."""
    rng = np.random.default_rng(77)
    shape = synth.ModelShape(D=256, H=8, Hkv=2, d=64, Dff=688, dtype=dtype)
    made = []
    for lens in ([2100, 70, 4000], [100, 300, 9]):
        for _ in range(2):
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                c = binding.Context(shape, 64, 1, 1, shape.Dff, stream=st)
                caches = runtime.KV4Batch(shape, [n + 1 for n in lens])
                append(torch, c, caches, [make_pairs(rng, n, 2, 64, dtype) + (np.arange(n),) for n in lens], dtype)
                q = runtime.to_device(rounded(rng.standard_normal((3, 8, 64)), dtype), dtype)
                alone = torch.empty_like(q)
                c.spts_kv4_attn(q, caches.structs, alone)
            torch.cuda.synchronize()
            made.append((c, caches, q, alone, st))
    for _ in range(20):
        outs = [torch.full_like(m[2], 9.0) for m in made]
        torch.cuda.synchronize()
        for (c, caches, q, _, st), out in zip(made, outs):
            c.spts_kv4_attn(q, caches.structs, out)
        torch.cuda.synchronize()
        assert all(torch.equal(out, m[3]) for out, m in zip(outs, made))
    for c, caches, q, alone, _ in made:
        c.spts_kv4_attn(q, caches.structs, q)
    torch.cuda.synchronize()
    assert all(torch.equal(m[2], m[3]) for m in made)


@pytest.mark.parametrize("n", [200, 2500])
def test_one_cache_for_several_queries(torch, n):
    """The same buffers given to several queries, with counts of their own; a repeated query's result is the same bits, rows behind the last are left."""
    ctx, shape = ctx_for("bf16", H=8, Hkv=2, d=128)
    rng = np.random.default_rng(n)
    caches = runtime.KV4Batch(shape, [n])
    k, v = make_pairs(rng, n, 2, 128, "bf16")
    append(torch, ctx, caches, [(k, v, np.arange(n))], "bf16")
    counts = [n, n // 2, n, 0, 1]
    many = (binding.spts_kv4 * 5)(*[caches.structs[0]] * 5)
    for s, c in zip(many, counts):
        s.count = c
    q = rounded(rng.standard_normal((5, 8, 128)), "bf16")
    q[2] = q[0]
    qd = runtime.to_device(q, "bf16")
    out = torch.full_like(qd, 9.0)
    behind = torch.full((2, 8, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    both = torch.cat([out, behind])
    ctx.spts_kv4_attn(qd, many, both)
    torch.cuda.synchronize()
    assert torch.equal(both[5:], behind)                # rows behind the last query
    assert torch.equal(both[0], both[2]) and not both[3].any()
    got = runtime.to_host(both).astype(np.float64)
    for b, c in enumerate(counts):
        if c == 0:
            continue
        kq, vq = fp4.fp4_round(k[:c]), fp4.fp4_round(v[:c])
        ref = fp4.attend(q[b].astype(np.float64), kq, vq)
        for h in range(8):
            tol = attend_tol(q[b, h].astype(np.float64), kq[:, h // 4], vq[:, h // 4], "bf16")
            assert np.all(np.abs(got[b, h] - ref[h]) <= tol), (b, h)


# -------------------------------------------------------------------------------------------------------------- rules
def words(allowed):
    """Bit masks [n, ceil(V / 32)] int32 of truth values [n, V]."""
    n, V = allowed.shape
    bits = np.zeros((n, -(-V // 32) * 32), dtype=np.uint64)
    bits[:, :V] = allowed
    w = (bits.reshape(n, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1)
    return w.astype(np.uint32).view(np.int32)


@pytest.mark.parametrize("V,nb,most", [(1, 1, 3), (33, 2, 100), (4095, 3, 64), (4096, 1, 5000), (4097, 16, 300), (10001, 5, 0), (32000, 4, 2048), (128256, 2, 40000)])
@pytest.mark.parametrize("which", ["all", "penalties", "shared", "mask", "none"])
def test_rules_step_by_step(torch, V, nb, most, which):
    """Every rounding is one of fp32 in the documented order: results, token and table row are those of numpy's fp32, bit for bit."""
    ctx, shape = ctx_for("bf16", D=64)
    rng = np.random.default_rng(V + nb)
    x = (3.0 * rng.standard_normal((nb, V))).astype(np.float32)
    x[:, rng.integers(0, V, 5)] = x.max()               # ties on top
    hist = rng.integers(-3, V + 3, (nb, most + 2)).astype(np.int32)
    hist[:, ::3] = rng.integers(0, min(V, 20), hist[:, ::3].shape)
    lens = [max(0, most - 7 * b) for b in range(nb)]
    prompt = [n // 3 for n in lens]
    rep, freq, pres = (np.float32(rng.uniform(lo, hi, nb)) for lo, hi in ((0.7, 1.5), (-0.1, 0.6), (-0.3, 1.0)))
    pens = which in ("all", "penalties", "shared")
    one = 1 if which == "shared" else nb
    bias = (rng.standard_normal((one, V)) * (rng.random((one, V)) < 0.1)).astype(np.float32) if which in ("all", "shared") else None
    allowed = rng.random((one, V)) < 0.1 if which in ("all", "shared", "mask") else None
    if allowed is not None and one > 1:
        allowed[0] = False                              # a mask that leaves nothing
    if allowed is not None:
        x[:, 0] = np.where(np.broadcast_to(allowed, (nb, V))[:, 0], x[:, 0], np.nan)   # NaN and infinity behind the mask
        x[:, -1] = np.where(np.broadcast_to(allowed, (nb, V))[:, -1], x[:, -1], np.inf)
    hd = torch.from_numpy(hist).cuda()
    bd, md = (torch.from_numpy(a).cuda() if a is not None else None for a in (bias, words(allowed) if allowed is not None else None))
    kw = dict(history=hd, history_len=lens, prompt_len=prompt, repetition=rep.tolist(), frequency=freq.tolist(), presence=pres.tolist()) if pens else {}
    rules = runtime.LogitsRules(nb, bias=bd, mask=md, **kw)
    xd = torch.from_numpy(x).cuda()
    out, tok = torch.full_like(xd, 5.0), torch.full((nb,), -9, dtype=torch.int32, device="cuda")
    table = torch.randn((V, 64), device="cuda").to(torch.bfloat16)
    nxt = torch.full((nb, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    ctx.spts_process_logits(xd, V, nb, rules.struct, out, tok, table, nxt)
    torch.cuda.synchronize()
    assert np.array_equal(xd.cpu().numpy(), x, equal_nan=True)
    got = out.cpu().numpy()
    for b in range(nb):
        args = (hist[b, :lens[b]], prompt[b], rep[b], freq[b], pres[b]) if pens else (None,)
        ref, t = fp4.process_logits(x[b], *args, bias=None if bias is None else bias[b % one],
                                    allowed=None if allowed is None else allowed[b % one], num=np.float32)
        bad = np.flatnonzero(~((got[b] == ref) | (np.isnan(got[b]) & np.isnan(ref))))
        assert not len(bad), (b, len(bad), [(int(w), float(x[b, w]), float(got[b, w]), float(ref[w])) for w in bad[:5]])
        assert int(tok[b]) == t and (t >= 0 or (allowed is not None and not allowed[b % one].any()))
        assert torch.equal(nxt[b], table[t] if t >= 0 else torch.zeros_like(nxt[b]))
    ctx.spts_process_logits(xd, V, nb, rules.struct, xd)            # in place, no token asked for
    torch.cuda.synchronize()
    assert np.array_equal(xd.cpu().numpy(), got, equal_nan=True)


def test_rules_leave_nothing_or_nan(torch):
    ctx, _ = ctx_for("f32", D=64)
    x = torch.tensor([[float("nan"), 1.0, float("-inf"), float("-inf")]] * 4, device="cuda")
    allowed = np.array([[1, 0, 0, 0], [1, 0, 1, 1], [0, 0, 0, 0], [1, 1, 1, 1]], dtype=bool)
    tok = torch.full((4,), 9, dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    ctx.spts_process_logits(x, 4, 4, runtime.LogitsRules(4, mask=torch.from_numpy(words(allowed)).cuda()).struct, out, tok)
    torch.cuda.synchronize()
    assert tok.tolist() == [-1, 2, -1, 1]


# -------------------------------------------------------------------------------------------------------- the layer
def layer_for(torch, ctx, shape, seed):
    w = synth.make_layer(seed, 0, shape, 16)
    dw = runtime.pack_layer_q4(ctx, runtime.upload_layer(w, shape, 16, pack=False))
    abi = synth.to_abi_layout({n: w[n] for n in ("Wq", "Wk", "Wv", "Wo", "Wgate", "Wup", "Wdown", "gamma1", "gamma2")})
    back = {n: (fp4.fp4_round(rounded(abi[n], shape.dtype)) if n[0] == "W" else abi[n]) for n in abi}
    # the oracle's orientation: y = x W, except W_down which the method applies transposed
    same = {n: w[n].shape == abi[n].shape and np.array_equal(w[n], abi[n]) for n in abi}
    return dw, {n: back[n] if same[n] else np.ascontiguousarray(back[n].T) for n in back}


# (D, H, Hkv, d, Dff): the rows of each product, in strips of 16, on either side of where the kernels change
LAYERS = [(256, 4, 2, 64, 688), (64, 64, 16, 128, 8704), (4224, 4, 2, 32, 64), (8320, 4, 2, 32, 64), (64, 48, 6, 128, 2104), (16392, 4, 2, 32, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nseq,dims", [(1, 0), (2, 0), (5, 0), (16, 0), (1, 1), (3, 1), (1, 2), (2, 2), (1, 3), (2, 3), (3, 3),
                                       (1, 4), (4, 4), (1, 5), (7, 1), (16, 1)])
def test_decode_layer_lockstep(torch, dtype, nseq, dims):
    """Caches of different lengths filled from random pairs, three steps of the layer: the appended pair against the oracle's (to the
    element type's rounding, then one of 4 bits), the state against the oracle's over the pairs as stored."""
    D, heads, Hkv, d, Dff = LAYERS[dims]
    ctx, shape = ctx_for(dtype, H=heads, Hkv=Hkv, d=d, D=D, Dff=Dff)
    mdl, rnd, tol = H.oracle_model(shape), H.rnd_for(dtype), H.TOL[dtype]["hidden"]
    rng = np.random.default_rng(nseq)
    dw, w = layer_for(torch, ctx, shape, 31)
    lens = [300, 45, 0, 64, 511, 33, 96, 257, 40, 1, 77, 18, 200, 31, 8, 99][:nseq]
    caches = runtime.KV4Batch(shape, [n + 3 for n in lens])
    append(torch, ctx, caches, [make_pairs(rng, n, shape.Hkv, shape.d, dtype) + (np.arange(n),) for n in lens], dtype)
    new = synth.hidden_states(32, 3 * nseq, shape.D, dtype).reshape(3, nseq, shape.D)
    for t in range(3):
        before = [caches.host(ctx, shape, b) for b in range(nseq)]
        xt = runtime.to_device(new[t].copy(), dtype)
        x_in = runtime.to_host(xt).astype(np.float64)
        pos = [2 * n + t for n in lens]
        ctx.spts_decode_layer_q4(xt, pos, dw, caches.structs)
        torch.cuda.synchronize()
        got = runtime.to_host(xt).astype(np.float64)
        assert caches.counts == [n + t + 1 for n in lens]
        for b in range(nseq):
            k, v, p = before[b]
            k2, v2, p2 = caches.host(ctx, shape, b)
            assert np.array_equal(k2[:-1], k) and np.array_equal(v2[:-1], v) and p2[-1] == pos[b]
            ref, k_new, v_new = fp4.decode_layer(x_in[b], pos[b], w, mdl, k, v, rnd, stored=(k2[-1:], v2[-1:]))
            for stored, true in ((k2[-1], k_new[0]), (v2[-1], v_new[0])):
                # half of the widest gap (2 * 2^e, between 4 and 6) where the two exponents agree; e may be one more on the GPU's side
                unit = np.repeat(2.0 ** fp4.exponents(np.maximum(np.abs(stored), np.abs(true))), fp4.BLOCK, axis=-1)[..., :shape.d]
                assert np.all(np.abs(stored - true) <= unit + tol * np.abs(true).max())
            assert H.row_rel_err(got[b][None], ref[None]) <= tol, (t, b, H.row_rel_err(got[b][None], ref[None]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_run_of_all_together(torch, dtype):
    """Prefill, its caches converted, two layers of decode, the head in 4 bits, penalties, bias and mask: every step's logits and tokens
    against the oracle from the GPU's own state, the history growing by the tokens."""
    ctx, shape = ctx_for(dtype, rows=512)
    mdl, rnd, tol = H.oracle_model(shape), H.rnd_for(dtype), H.TOL[dtype]["hidden"]
    rng = np.random.default_rng(40)
    nseq, V, layers, lens = 3, 416, 2, [120, 33, 64]
    raw = [synth.make_layer(41 + l, 0, shape, 16) for l in range(layers)]
    dense = [runtime.upload_layer(w, shape, 16, pack=False) for w in raw]
    q4 = [layer_for(torch, ctx, shape, 41 + l) for l in range(layers)]
    caches = [runtime.KV4Batch(shape, [n + 6 for n in lens]) for _ in range(layers)]
    for b, n in enumerate(lens):
        x = runtime.to_device(synth.hidden_states(50 + b, n, shape.D, dtype), dtype)
        for l in range(layers):
            kc = runtime.KVCache(shape, n)
            ctx.spts_layer_prefill(x, torch.arange(n, dtype=torch.int32, device="cuda"), n, dense[l], binding.spts_layer_cfg(0, 1, n, n, 1, 0), kc.struct)
            caches[l].append_cache(ctx, b, kc)
            k, v, p = kc.host()
            gk, gv, gp = caches[l].host(ctx, shape, b)
            assert np.array_equal(gk, fp4.fp4_round(k)) and np.array_equal(gv, fp4.fp4_round(v)) and np.array_equal(gp, p)
    table = rounded(rng.standard_normal((V, shape.D)), dtype)
    td = runtime.to_device(table, dtype)
    gamma = rounded(1.0 + 0.1 * rng.standard_normal(shape.D), dtype)
    hist = rng.integers(0, V, (nseq, 20)).astype(np.int32)
    allowed = rng.random((nseq, V)) < 0.5
    bias = rng.standard_normal(V).astype(np.float32)
    rep, freq, pres = [1.2, 1.0, 1.3], [0.1, 0.4, 0.0], [0.2, 0.0, 0.3]
    hd = torch.from_numpy(hist).cuda()
    rules = runtime.LogitsRules(nseq, history=hd, history_len=[10, 4, 12], prompt_len=[10, 4, 12], repetition=rep, frequency=freq, presence=pres,
                                bias=torch.from_numpy(bias).cuda(), mask=torch.from_numpy(words(allowed)).cuda())
    head = runtime.Q4Matrix(ctx, td)
    run = runtime.Q4DecodeRunner(ctx, shape, [d for d, _ in q4], caches, runtime.to_device(gamma, dtype), td, head, rules)
    run.x.copy_(td[torch.tensor([3, 1, 4]).cuda()])
    headq, said = fp4.fp4_round(table), [[], [], []]
    for t in range(4):
        x0 = runtime.to_host(run.x).astype(np.float64)
        before = [[caches[l].host(ctx, shape, b) for b in range(nseq)] for l in range(layers)]
        toks = torch.zeros((nseq, 1), dtype=torch.int32, device="cuda")
        run.generate([n + t for n in lens], 1, toks)
        torch.cuda.synchronize()
        for b in range(nseq):
            x = x0[b]
            for l in range(layers):
                k2, v2, _ = caches[l].host(ctx, shape, b)
                x, _, _ = fp4.decode_layer(x, lens[b] + t, q4[l][1], mdl, before[l][b][0], before[l][b][1], rnd, stored=(k2[-1:], v2[-1:]))
            xn = rnd(orc.rmsnorm(x[None], gamma, mdl.rms_eps))[0]
            raw_logits = headq @ xn
            h = hist[b, :[10, 4, 12][b]].tolist() + said[b]
            ref, _ = fp4.process_logits(raw_logits, h, [10, 4, 12][b], rep[b], freq[b], pres[b], bias, allowed[b])
            got = run.logits[b].cpu().numpy().astype(np.float64)
            assert np.array_equal(np.isinf(got), ~allowed[b])
            # the error of the state of two layers (each within tol of its largest) reaches every logit
            slack = 2 * layers * tol * np.abs(raw_logits).max()
            assert np.all(np.abs(got[allowed[b]] - ref[allowed[b]]) <= slack)
            tok = int(toks[b, 0])
            assert got[tok] == got.max() and tok == int(np.argmax(got))
            said[b].append(tok)
            assert hd[b, len(h)].item() == tok and rules.history_len[b] == len(h) + 1
            assert torch.equal(run.x[b], td[tok])


def test_captured_and_replayed(torch):
    """The whole step under a graph, replayed between eager calls of the same kind: the caches' counts are those of the capture, so every replay
    writes the same row, and its results are the eager call's."""
    ctx_e, shape = ctx_for("bf16")
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(shape, 256, 1, 1, shape.Dff, stream=stream)
    dw, _ = layer_for(torch, ctx_e, shape, 61)
    rng = np.random.default_rng(61)
    lens = [700, 41, 0]
    caches, eager = runtime.KV4Batch(shape, [n + 8 for n in lens]), runtime.KV4Batch(shape, [n + 8 for n in lens])
    parts = [make_pairs(rng, n, 2, 64, "bf16") + (np.arange(n),) for n in lens]
    for c in (caches, eager):
        append(torch, ctx_e, c, parts, "bf16")
    V = 5000
    x0 = runtime.to_device(synth.hidden_states(62, 3, shape.D, "bf16"), "bf16")
    head = runtime.Q4Matrix(ctx_e, torch.randn((V, shape.D), device="cuda").to(torch.bfloat16))
    hist = torch.randint(0, V, (3, 50), dtype=torch.int32, device="cuda")
    rules = runtime.LogitsRules(3, history=hist, history_len=[50, 3, 0], repetition=[1.2] * 3)
    bufs = lambda: (x0.clone(), torch.zeros((3, V), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros_like(x0))  # noqa: E731
    xe, le, te, ne = bufs()
    xg, lg, tg, ng = bufs()

    def step(c, cs, x, logits, tok, xn):
        c.spts_decode_layer_q4(x, [800, 50, 0], dw, cs.structs)
        c.spts_rmsnorm(x, dw._keepalive["gamma1"], 3, xn)
        c.spts_matvec_q4(head.struct, xn, 3, logits, 1)
        c.spts_process_logits(logits, V, 3, rules.struct, logits, tok)

    step(ctx_e, eager, xe, le, te, ne)
    torch.cuda.synchronize()
    warm = runtime.KV4Batch(shape, [8, 8, 8])
    with torch.cuda.stream(stream):
        step(ctx, warm, *bufs())                         # first use of every kernel outside the capture
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=stream):
        xg.copy_(x0)
        step(ctx, caches, xg, lg, tg, ng)
    for _ in range(4):
        for t in (xg, lg, tg, ng):
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(xg, xe) and torch.equal(lg, le) and torch.equal(tg, te) and torch.equal(ng, ne)
        other = runtime.KV4Batch(shape, [n + 8 for n in lens])          # eager work in between, over the eager context's workspace
        append(torch, ctx_e, other, parts, "bf16")
        xo, lo, to, no = bufs()
        step(ctx_e, other, xo, lo, to, no)
        torch.cuda.synchronize()
        assert torch.equal(lo, le)
    assert caches.counts == [n + 1 for n in lens]
    for b in range(3):
        for a, e in zip(caches.host(ctx_e, shape, b), eager.host(ctx_e, shape, b)):
            assert np.array_equal(a, e)


def test_phases_are_named(torch):
    ctx, shape = ctx_for("bf16")
    caches = runtime.KV4Batch(shape, [16])
    ctx.spts_profile_begin()
    m = runtime.Q4Matrix(ctx, torch.zeros((16, 64), dtype=torch.bfloat16, device="cuda"))
    y = torch.empty((1, 16), dtype=torch.bfloat16, device="cuda")
    ctx.spts_matvec_q4(m.struct, torch.zeros((1, 64), dtype=torch.bfloat16, device="cuda"), 1, y)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    ctx.spts_kv4_append(k, k, torch.zeros(3, dtype=torch.int32, device="cuda"), [0, 3], caches.structs)
    ctx.spts_kv4_read(caches.structs, [0, 3], torch.empty_like(k), torch.empty_like(k))
    ctx.spts_kv4_attn(torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda"), caches.structs, torch.empty((1, 4, 64), dtype=torch.bfloat16, device="cuda"))
    x = torch.zeros((1, 64), device="cuda")
    ctx.spts_process_logits(x, 64, 1, runtime.LogitsRules(1).struct, x)
    got = ctx.spts_profile_end()
    assert {n: got[n][1] for n in ("q4_pack", "q4_matvec", "kv4_append", "kv4_read", "kv4_attn", "logits_rules")} == dict.fromkeys(
        ("q4_pack", "q4_matvec", "kv4_append", "kv4_read", "kv4_attn", "logits_rules"), 1)

"""Decode in 4 bits on the GPU: precision, streams, stored bits and sizes beside those of test_gpu_q4.py (same oracle, same tolerances)."""
import math

import numpy as np
import pytest

from oracle import fp4_oracle as fp4
from tests.test_gpu_q4 import HALF, SUM, append, ctx_for, make_pairs, rounded, torch  # noqa: F401  (torch: the fixture)
from paper_2601_13155_amd import runtime

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

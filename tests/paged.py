"""Plain forms in 64 bits of the operators over caches in pages, and the inputs of their tests."""
import math

import numpy as np
import torch

from paper_2601_13155_amd import runtime, synth

TD = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # half a step of the type, relative


def shape_of(H, Hkv, d, dtype):
    return synth.ModelShape(D=256, H=H, Hkv=Hkv, d=d, Dff=256, dtype=dtype)


def context(shape, rows=256):
    return runtime.make_context(shape, max(256, rows), 1, 1, 256)


def filled(shape, page, rows, seed, capacity=None, spare=3, weights=True, garbage=math.nan):
    """A PagedKV whose sequence b holds rows[b] random rows on pages in random order; what is behind them is garbage."""
    g = torch.Generator().manual_seed(seed)
    cap = max(1, max(rows)) if capacity is None else capacity
    per = -(-cap // page)
    pages = len(rows) * per + spare
    kv = runtime.PagedKV(shape, pages, page, len(rows), cap, weights=weights, free=torch.randperm(pages, generator=g).tolist())
    for t, scale in ((kv.k, 1.0), (kv.v, 1.0)):
        t.fill_(garbage)
    if weights:
        kv.weight.fill_(garbage)
    host = []
    for b, n in enumerate(rows):
        kv.reserve(b, n)
        k = torch.randn((n, shape.Hkv, shape.d), generator=g).to(kv.k.dtype)
        v = torch.randn((n, shape.Hkv, shape.d), generator=g).to(kv.k.dtype)
        put(kv, b, 0, k, v)
        kv.pos[b, :n] = 3 * torch.arange(n, dtype=torch.int32, device="cuda") + 1
        if weights:
            kv.weight[b, :n] = torch.rand(n, generator=g).cuda()
        kv.structs[b].count = n
        host.append((k, v))
    return kv, host


def put(kv, b, first, k, v):
    """Rows k, v [n, Hkv, d] at sequence b's rows first .. (through the table, not the library)."""
    i = torch.arange(first, first + k.shape[0])
    page, at = kv.table[b].cpu().long()[i // kv.page].cuda(), (i % kv.page).cuda()
    kv.k[page, :, at] = k.cuda()
    kv.v[page, :, at] = v.cuda()


def attend64(q, k, v, H, Hkv):
    """q [m, H, d] of the last m of the rows k, v [n, Hkv, d], in float64: (out, sum of p |v|, largest sum of |q k| / sqrt d, weights)."""
    m, n, d, G = q.shape[0], k.shape[0], q.shape[2], H // Hkv
    q, k, v = (t.double().cpu() for t in (q, k, v))
    out, spread, big, got = torch.zeros_like(q), torch.zeros_like(q), 0.0, torch.zeros(n, dtype=torch.float64)
    for i in range(m):
        seen = n - m + i + 1
        for h in range(H):
            ks, vs = k[:seen, h // G], v[:seen, h // G]
            s = (ks @ q[i, h]) / math.sqrt(d)
            p = torch.softmax(s, 0)
            out[i, h], spread[i, h] = p @ vs, p @ vs.abs()
            big = max(big, float((ks.abs() @ q[i, h].abs()).max()) / math.sqrt(d))
            got[:seen] += p
    return out, spread, big, got


def attend64_wide(q, k, v, H, Hkv):
    """attend64 on the GPU, a head's queries at once."""
    m, n, d, G = q.shape[0], k.shape[0], q.shape[2], H // Hkv
    q, k, v = (t.cuda().double() for t in (q, k, v))
    out, spread, big, got = torch.zeros_like(q), torch.zeros_like(q), 0.0, torch.zeros(n, dtype=torch.float64, device="cuda")
    unseen = torch.ones((m, n), dtype=torch.bool, device="cuda").triu(n - m + 1)
    for h in range(H):
        kh, vh, qh = k[:, h // G].contiguous(), v[:, h // G].contiguous(), q[:, h].contiguous()
        p = torch.softmax(((qh @ kh.t()) / math.sqrt(d)).masked_fill(unseen, -math.inf), 1)
        out[:, h], spread[:, h] = p @ vh, p @ vh.abs()
        big = max(big, float((qh.abs() @ kh.t().abs()).masked_fill(unseen, 0.0).max()) / math.sqrt(d))
        got += p.sum(0)
    return out.cpu(), spread.cpu(), big, got.cpu()


def score_error(big, d):
    """How far a score is off: d products summed in fp32 (each addition and, of fp32 operands, each product half a step), the scaling, the difference to the maximum and the exponential's
    few steps."""
    return (2 * d + 16) * 2.0 ** -24 * max(big, 1.0)


def attend_bound(out, spread, big, n, d, dtype, chunk):
    """Tolerance of an output: the scores' errors on both sides of the quotient, fp32 sums over n rows, the weights' rounding (half a step of the type; 2^-15 where two bf16 parts
    hold them) and the output's own."""
    weights = 0.0 if dtype == "f32" else HALF["bf16"] if chunk else 2.0 ** -15
    return spread * (2 * score_error(big, d) + 2 * (n + 64) * 2.0 ** -24 + weights) + out.abs() * HALF[dtype] + 1e-30


def evict64(weight, pos, keep, below, start):
    """(rows that stay by new row, number of them): the definition, in Python."""
    n = len(weight)
    if keep >= n:
        return list(range(n))
    w = [math.inf if math.isnan(x) else max(float(x), 0.0) for x in weight]
    nan = [math.isnan(x) for x in weight]
    first = [(below is not None and p < below) or (start is not None and p >= start) for p in pos]
    order = sorted(range(n), key=lambda i: (not first[i], not nan[i], -w[i], i))
    kept = sorted(order[:keep])
    stay, late = set(i for i in kept if i < keep), iter([i for i in kept if i >= keep])
    return [i if i in stay else next(late) for i in range(keep)]


def logprobs64(x, tokens, top):
    """x [rows, V] float64 numpy: (logprob, entropy, ids, top log probabilities)."""
    lp, ent, ids, tops = [], [], [], []
    with np.errstate(all="ignore"):
        for row, t in zip(x, tokens):
            m = np.max(row) if not np.isnan(row).any() else np.nan
            allowed = row > -np.inf
            if m == -np.inf:
                e = 0.0
                l = np.full_like(row, -np.inf)
            else:
                l = (row - m) - np.log(np.sum(np.exp(row - m)))      # (m itself may be so large that a sum with it loses the logarithm)
                fine = np.isfinite(m)
                l = l if fine else np.full_like(row, np.nan)
                p = np.exp(l)
                e = -np.sum(np.where(p > 0, p * np.where(p > 0, l, 0.0), 0.0)) if fine else np.nan
            lp.append(l[t] if 0 <= t < len(row) else np.nan)
            ent.append(e)
            order = sorted(np.nonzero(allowed)[0], key=lambda i: (-row[i], i))[:top] if top else []
            ids.append(list(order) + [-1] * (top - len(order)))
            tops.append([l[i] for i in order] + [-np.inf] * (top - len(order)))
    return np.array(lp), np.array(ent), np.array(ids, dtype=np.int64).reshape(len(x), top), np.array(tops).reshape(len(x), top)

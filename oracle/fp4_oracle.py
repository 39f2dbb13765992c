"""CPU oracle of the decode step in 4 bits: numpy fp64, from the definitions in the C header's comments.

Nothing here comes from the library; the decoder layer is composed of the steps of ``spts_oracle``.
"""
from __future__ import annotations

from typing import Dict, Optional

import numpy as np

from . import spts_oracle as orc

Array = np.ndarray

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32
E_MIN, E_MAX = -126, 125


def exponents(a: Array) -> Array:
    """Per block of 32 along the last axis: the smallest e in [-126, 125] with max|v| <= 6 * 2^e."""
    a = np.abs(np.asarray(a, dtype=np.float64))
    a = np.concatenate([a, np.zeros(a.shape[:-1] + (-a.shape[-1] % BLOCK,))], axis=-1)
    top = a.reshape(a.shape[:-1] + (-1, BLOCK)).max(axis=-1)
    e = np.full(top.shape, E_MIN)
    for s in range(E_MIN, E_MAX):      # by the definition: raised while the largest value does not fit
        e = np.where(top > 6.0 * 2.0 ** s, s + 1, e)
    return e


def fp4_round(a: Array) -> Array:
    """The values that `a` stands for in 4 bits: nearest of the grid times 2^e, ties to the even code, saturating."""
    a = np.asarray(a, dtype=np.float64)
    n = a.shape[-1]
    unit = np.repeat(2.0 ** exponents(a), BLOCK, axis=-1)[..., :n]
    mag = np.minimum(np.abs(a) / unit, 6.0)
    code = np.zeros(a.shape, dtype=np.int64)
    for c in range(1, 8):              # mid < mag, or mid == mag and c is the even one of the two
        mid = 0.5 * (GRID[c - 1] + GRID[c])
        code = np.where((mag > mid) | ((mag == mid) & (c % 2 == 0)), c, code)
    return np.where(np.signbit(a), -GRID[code], GRID[code]) * unit


def attend(q: Array, k: Array, v: Array) -> Array:
    """q [H, d] over pairs k, v [n, Hkv, d]; zeros for n = 0."""
    H, d = q.shape
    out = np.zeros((H, d))
    if k.shape[0] == 0:
        return out
    grp = H // k.shape[1]
    for h in range(H):
        p = orc.softmax_rows((k[:, h // grp] @ q[h] / np.sqrt(d))[None, :])[0]
        out[h] = p @ v[:, h // grp]
    return out


def process_logits(logits: Array, history=None, prompt_len: int = 0, repetition: float = 1.0, frequency: float = 0.0, presence: float = 0.0,
                   bias: Optional[Array] = None, allowed: Optional[Array] = None, num=np.float64):
    """One sequence's logits [V] under the rules, one after the other in arithmetic of type `num`; history: the token ids that
    count (ids outside [0, V) are skipped).  Returns (logits, token): the token is the lowest id of the largest allowed value, -1
    where there is none."""
    x = np.array(logits, dtype=num)
    V = len(x)
    if history is not None:
        history = np.asarray(history, dtype=np.int64)
        inside = (history >= 0) & (history < V)
        said = np.bincount(history[prompt_len:][inside[prompt_len:]], minlength=V)
        seen = np.bincount(history[inside], minlength=V) > 0
        x = np.where(seen, np.where(x > 0, x / num(repetition), x * num(repetition)), x)
        x = np.where(said > 0, x - num(frequency) * said.astype(num), x)
        x = np.where(said > 0, x - num(presence), x)
    if bias is not None:
        x = x + np.asarray(bias, dtype=num)
    ok = np.ones(V, dtype=bool) if allowed is None else np.asarray(allowed, dtype=bool)
    x = np.where(ok, x, num(-np.inf))
    choice = np.flatnonzero(ok & ~np.isnan(x))
    return x, int(choice[np.argmax(x[choice])]) if len(choice) else -1


def decode_layer(x_t: Array, pos_t: int, w: Dict[str, Array], mdl: orc.Model, k: Array, v: Array, rnd=orc.identity, stored=None):
    """``spts_oracle.decode_layer`` over weights `w` and pairs k, v [n, Hkv, d] that are already 4-bit values (w: as the layer
    multiplies with them).  The new pair is rounded to the element type and to 4 bits before it is attended to; `stored`
    (k, v of it) takes its place when given.  Returns (x_out [D], new key, new value before the 4-bit rounding)."""
    x = rnd(np.array(x_t, dtype=np.float64)).reshape(1, -1)
    p = np.array([pos_t])
    xn = rnd(orc.rmsnorm(x, w["gamma1"], mdl.rms_eps))
    k_new = orc.project_keys(xn, p, w["Wk"], mdl, rnd)
    v_new = rnd((xn @ np.asarray(w["Wv"], dtype=np.float64)).reshape(1, mdl.Hkv, mdl.d))
    q = orc.project_queries(xn, p, w["Wq"], mdl, rnd)
    ks, vs = stored if stored is not None else (fp4_round(k_new), fp4_round(v_new))
    att = rnd(attend(q[0], np.concatenate([k, ks]), np.concatenate([v, vs]))).reshape(1, -1)
    x = rnd(x + att @ np.asarray(w["Wo"], dtype=np.float64))
    xn2 = rnd(orc.rmsnorm(x, w["gamma2"], mdl.rms_eps))
    return rnd(x + orc.ffn(xn2, w["Wgate"], w["Wup"], w["Wdown"], rnd))[0], k_new, v_new

"""Host-side conveniences around the C-ABI binding: uploads, context creation, layer/stack drivers.

Marshalling and sequencing only: every arithmetic step of the path runs inside libspts kernels.
"""
from __future__ import annotations

import contextlib
import ctypes
from typing import Dict, List, Optional

import numpy as np

from . import binding, synth


def _torch():
    import torch
    return torch


def to_device(a: np.ndarray, dtype: str):
    """fp32 numpy array (already rounded to the storage dtype) -> device tensor of that dtype."""
    torch = _torch()
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to("cuda")
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def to_host(t) -> np.ndarray:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return t.to(torch.float32).cpu().numpy()
    return t.cpu().numpy()


def make_context(shape, max_tokens: int, max_probe: int, max_r: int, max_dlow: int) -> binding.Context:
    return binding.Context(shape, max_tokens, max_probe, max_r, max_dlow)


@contextlib.contextmanager
def _on_stream_of(ctx: binding.Context):
    """The body's work, torch's and the library's, goes to the context's stream: behind what the current stream has been given, and
    ahead of what it is given afterwards (so that what the current stream's pool gets back is no longer in use)."""
    torch = _torch()
    current = torch.cuda.current_stream(ctx.stream.device)
    if current == ctx.stream:
        yield
        return
    ctx.stream.wait_stream(current)
    try:
        with torch.cuda.stream(ctx.stream):
            yield
    finally:
        current.wait_stream(ctx.stream)


SLAB_PACKED = ("Wq", "Wk", "Wv", "Wo", "Wgate", "Wup", "Wdown", "Vg", "Vu", "Vd", "Ug", "Uu")


def pack_slab32(a: np.ndarray) -> np.ndarray:
    """Host-side slab-major copy of a row-major [rows, K] matrix (K % 32 == 0): element (s * rows + r) * 32 + j of the
    result is a[r, 32 * s + j]; same shape and dtype, the layout spts_pack_slab32 writes on the device."""
    rows, K = a.shape
    return np.ascontiguousarray(a.reshape(rows, K // 32, 32).transpose(1, 0, 2)).reshape(rows, K)


def ud_columns_orthonormal(Ud: np.ndarray, Vd: np.ndarray, tol: float = 1e-2) -> bool:
    """True when U_down [D, r] has orthonormal columns up to `tol` (what a truncated SVD with Sigma folded into V gives,
    also after rounding to bf16), all-zero columns of a zero-padded rank allowed if the matching rows of Vd are zero."""
    U = np.asarray(Ud, dtype=np.float64)
    G = U.T @ U
    d = np.diag(G).copy()
    zero = d == 0.0
    if np.any(np.abs(d[~zero] - 1.0) > tol) or np.max(np.abs(G - np.diag(d)), initial=0.0) > tol:
        return False
    return not zero.any() or not np.any(np.asarray(Vd)[zero])


def upload_layer(w: Dict[str, np.ndarray], shape, r: int, pack: bool = True,
                 ud_orthonormal: Optional[bool] = None) -> binding.spts_layer_weights:
    """Weights in the paper's orientation (synth.make_layer) -> device struct in the ABI layout.  pack (bf16 only): the
    projection and FFN matrices also get the slab-major copies that the prefill GEMMs prefer.  ud_orthonormal: whether to
    tell the library that U_down has orthonormal columns (it then takes the proxy's output norm from z alone); None =
    check the matrix here."""
    if ud_orthonormal is None:
        ud_orthonormal = "Ud" in w and "Vd" in w and ud_columns_orthonormal(w["Ud"], w["Vd"])
    abi = synth.to_abi_layout(w)
    dev = {k: to_device(v, shape.dtype) for k, v in abi.items()}
    if pack and shape.dtype == "bf16":
        for name in SLAB_PACKED:
            if name in abi and abi[name].shape[1] % 32 == 0:
                dev[name + "_s"] = to_device(pack_slab32(np.asarray(abi[name])), shape.dtype)
    dlow = int(abi["Vd"].shape[1]) if "Vd" in abi else 0
    return binding.layer_weights(dev, r=r if "Ug" in abi else 0, Dlow=dlow, ud_orthonormal=bool(ud_orthonormal))


def run_layer(ctx: binding.Context, x: np.ndarray, pos: np.ndarray, dw: binding.spts_layer_weights, shape, *, skip: int,
              probe_len: int, m_attn: int, m_ffn: int, protect_last: int = 1, kv_mode: int = 0, want_kv: bool = False):
    """One spts_layer_prefill call on host arrays; returns host arrays (tests and smoke use this)."""
    torch = _torch()
    N = int(x.shape[0])
    xd = to_device(x, shape.dtype)
    posd = torch.from_numpy(np.ascontiguousarray(pos, dtype=np.int32)).cuda()
    Ma = min(N, m_attn) if skip else N
    Mf = min(N, m_ffn) if skip else N
    s = torch.zeros(max(N, 1), dtype=torch.float32, device="cuda")
    ia = torch.full((max(Ma, 1),), -1, dtype=torch.int32, device="cuda")
    iff = torch.full((max(Mf, 1),), -1, dtype=torch.int32, device="cuda")
    cfg = binding.spts_layer_cfg(skip, probe_len, m_attn, m_ffn, protect_last, kv_mode)
    kv = None
    if want_kv:
        cap = N if (not skip or kv_mode == 1) else Ma
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        kk = torch.zeros((max(cap, 1), shape.Hkv, shape.d), dtype=tdt, device="cuda")
        vv = torch.zeros_like(kk)
        pp = torch.zeros(max(cap, 1), dtype=torch.int32, device="cuda")
        kv = binding.spts_kv_out(kk.data_ptr(), vv.data_ptr(), pp.data_ptr(), cap, 0)
    with _on_stream_of(ctx):
        ctx.spts_layer_prefill(xd, posd, N, dw, cfg, kv, s, ia, iff)
    torch.cuda.synchronize()
    out = dict(x=to_host(xd).astype(np.float64), s_mha=s[:N].cpu().numpy(), idx_attn=ia[:Ma].cpu().numpy(),
               idx_ffn=iff[:Mf].cpu().numpy())
    if want_kv:
        cnt = int(kv.count)
        out.update(kv_count=cnt, k_cache=to_host(kk[:cnt]).astype(np.float64), v_cache=to_host(vv[:cnt]).astype(np.float64),
                   pos_cache=pp[:cnt].cpu().numpy())
    return out


def select_proxy_channels(ctx: binding.Context, dw: binding.spts_layer_weights, shape, x_cal: np.ndarray, k: int, dlow: int):
    """The data-driven part of the offline proxy construction (Sec. 3.3) on the GPU: channel scores of Eq.
    (channel_importance) over the calibration rows x_cal [T, D], then C = TopK(I, dlow).  Returns (channel ids
    ascending [dlow] int32, scores [Dff] fp32) as host arrays; the SVD of the sliced matrices stays in the harness
    (synth.proxy_factors).  Sequencing of two library calls only."""
    torch = _torch()
    T = int(x_cal.shape[0])
    imp = torch.zeros(shape.Dff, dtype=torch.float32, device="cuda")
    sel = torch.empty(dlow, dtype=torch.int32, device="cuda")
    xd = to_device(x_cal, shape.dtype)
    with _on_stream_of(ctx):
        ctx.spts_channel_importance(xd, T, dw, int(k), imp)
        ctx.spts_select_topk(imp, shape.Dff, dlow, 0, sel)
    torch.cuda.synchronize()
    return sel.cpu().numpy(), imp.cpu().numpy()


class KVCache:
    """Device buffers of one layer's cache: k, v [capacity, Hkv, d], pos [capacity]; count lives on the host."""

    def __init__(self, shape, capacity: int):
        torch = _torch()
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        self.k = torch.zeros((max(capacity, 1), shape.Hkv, shape.d), dtype=tdt, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.pos = torch.zeros(max(capacity, 1), dtype=torch.int32, device="cuda")
        self.struct = binding.spts_kv_out(self.k.data_ptr(), self.v.data_ptr(), self.pos.data_ptr(), capacity, 0)

    @property
    def count(self) -> int:
        return int(self.struct.count)

    def host(self):
        """(k, v, pos) of the filled rows as host arrays (fp64 / int32)."""
        n = self.count
        return to_host(self.k[:n]).astype(np.float64), to_host(self.v[:n]).astype(np.float64), self.pos[:n].cpu().numpy()


class DecodeRunner:
    """Decode phase on the GPU: per token one spts_decode_layer per layer over that layer's cache, then
    (optionally) spts_greedy_token.  Only enqueues work; token ids stay on the device."""

    def __init__(self, ctx: binding.Context, shape, layers: List[binding.spts_layer_weights], caches: List[KVCache],
                 gamma_f=None, table=None):
        torch = _torch()
        self.ctx, self.shape, self.layers, self.caches = ctx, shape, layers, caches
        self.gamma_f, self.table = gamma_f, table
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        self.x = torch.zeros(shape.D, dtype=tdt, device="cuda")
        self.x_next = torch.zeros(shape.D, dtype=tdt, device="cuda")
        self.token = torch.zeros(4, dtype=torch.int32, device="cuda")
        self.logits = torch.zeros(table.shape[0], dtype=torch.float32, device="cuda") if table is not None else None

    def step(self, pos: int):
        """Runs self.x (in place) through every layer as the token at absolute position pos."""
        with _on_stream_of(self.ctx):
            for w, c in zip(self.layers, self.caches):
                self.ctx.spts_decode_layer(self.x, pos, w, c.struct)

    def greedy(self):
        """token = argmax over the table of the final-normed self.x; self.x_next = table[token]."""
        with _on_stream_of(self.ctx):
            self.ctx.spts_greedy_token(self.x, self.gamma_f, self.table, int(self.table.shape[0]), self.token, self.logits,
                                       self.x_next)

    def generate(self, pos0: int, steps: int, tokens_out=None):
        """steps greedy decode steps starting from self.x at position pos0; tokens_out [steps] int32 device."""
        with _on_stream_of(self.ctx):
            for t in range(steps):
                self.step(pos0 + t)
                self.greedy()
                if tokens_out is not None:
                    tokens_out[t:t + 1].copy_(self.token[:1])
                self.x.copy_(self.x_next)


class BatchedDecodeRunner:
    """Decode phase for a batch of sequences: per step one spts_decode_layer_batched per layer over the sequences'
    caches of that layer (caches[b][l]), then spts_greedy_token_batched.  Only enqueues work."""

    def __init__(self, ctx: binding.Context, shape, layers: List[binding.spts_layer_weights], caches: List[List[KVCache]],
                 gamma_f, table):
        torch = _torch()
        self.ctx, self.shape, self.layers, self.caches = ctx, shape, layers, caches
        self.gamma_f, self.table = gamma_f, table
        self.batch = len(caches)
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        self.x = torch.zeros((self.batch, shape.D), dtype=tdt, device="cuda")
        self.x_next = torch.zeros_like(self.x)
        self.tokens = torch.zeros(max(self.batch, 4), dtype=torch.int32, device="cuda")
        self.logits = torch.zeros((self.batch, table.shape[0]), dtype=torch.float32, device="cuda")

    def step(self, pos: List[int]):
        with _on_stream_of(self.ctx):
            for l, w in enumerate(self.layers):
                self.ctx.spts_decode_layer_batched(self.x, pos, w, [seq[l].struct for seq in self.caches])

    def generate(self, pos0: List[int], steps: int):
        with _on_stream_of(self.ctx):
            for t in range(steps):
                self.step([p + t for p in pos0])
                self.ctx.spts_greedy_token_batched(self.x, self.gamma_f, self.table, int(self.table.shape[0]), self.batch,
                                                   self.tokens, self.logits, self.x_next)
                self.x.copy_(self.x_next)


# ------------------------------------------------------------------------------------------- decode in 4 bits
class Q4Matrix:
    """A matrix [rows, K] packed into 4 bits (spts_q4_pack); W: device tensor of the context's element type (ValueError otherwise)."""

    def __init__(self, ctx: binding.Context, W):
        torch = _torch()
        want = torch.bfloat16 if ctx.shape.dtype == "bf16" else torch.float32
        if W.dim() != 2 or W.dtype != want or not W.is_cuda:
            raise ValueError(f"a device matrix of {want}, not {W.dtype} {list(W.shape)} on {W.device}")
        rows, K = (int(n) for n in W.shape)
        cb, sb = binding.spts_q4_bytes(rows, K)
        self.codes = torch.empty(cb, dtype=torch.uint8, device=W.device)
        self.scales = torch.empty(sb, dtype=torch.uint8, device=W.device)
        self.struct = binding.spts_q4(self.codes.data_ptr(), self.scales.data_ptr(), rows, K)
        self.struct._keepalive = (self.codes, self.scales)
        with _on_stream_of(ctx):
            ctx.spts_q4_pack(W.contiguous(), self.struct)


def pack_layer_q4(ctx: binding.Context, w: binding.spts_layer_weights) -> binding.spts_layer_q4:
    """The 4-bit form of a layer that upload_layer has put on the device (gains are shared with it, not copied)."""
    t, out = w._keepalive, binding.spts_layer_q4()
    out._keepalive = {n: Q4Matrix(ctx, t[n]) for n in ("Wq", "Wk", "Wv", "Wo", "Wgate", "Wup", "Wdown")}
    for n, m in out._keepalive.items():
        setattr(out, n, m.struct)
    out.gamma1, out.gamma2 = t["gamma1"].data_ptr(), t["gamma2"].data_ptr()
    out._keepalive.update(gamma1=t["gamma1"], gamma2=t["gamma2"])
    return out


class KV4Batch:
    """One layer's caches of several sequences in 4 bits; capacities are rounded up to a multiple of 8.  `structs` is what
    the calls take (a ctypes array of spts_kv4, its counts kept up to date by them)."""

    def __init__(self, shape, capacities):
        torch = _torch()
        m = binding.model_desc(shape)
        self.structs = (binding.spts_kv4 * len(capacities))()
        self._parts, at = [], 0               # (offset, bytes) of a sequence's k, v, k_scale, v_scale, pos in one allocation
        for s, cap in zip(self.structs, capacities):
            s.capacity = cap = max(8, (int(cap) + 7) // 8 * 8)
            cb, sb = binding.spts_kv4_bytes(m, cap)
            parts = []
            for n in (cb, cb, sb, sb, 4 * cap):
                parts.append((at, n))
                at += (n + 255) // 256 * 256
            self._parts.append(parts)
        self._buffer = torch.empty(at, dtype=torch.uint8, device="cuda")
        self.structs._keepalive = self._buffer
        base = self._buffer.data_ptr()
        for s, parts in zip(self.structs, self._parts):
            s.k, s.v, s.k_scale, s.v_scale, s.pos = (base + p for p, _ in parts)
        self._empty = bytes(self.structs)

    @property
    def tensors(self):
        """Per sequence the buffers as tensors: codes of k and v and their scales (uint8), positions (int32)."""
        view = [[self._buffer[p:p + n] for p, n in parts] for parts in self._parts]
        return [t[:4] + [t[4].view(_torch().int32)] for t in view]

    @property
    def counts(self) -> List[int]:
        return [int(s.count) for s in self.structs]

    def clear(self):
        ctypes.memmove(self.structs, self._empty, len(self._empty))

    def append_cache(self, ctx: binding.Context, b: int, cache: "KVCache"):
        """Appends every pair of a prefill's cache to sequence b's."""
        one = [self.structs[b]]
        with _on_stream_of(ctx):
            ctx.spts_kv4_append(cache.k, cache.v, cache.pos, [0, cache.count], one)
        self.structs[b].count = one[0].count

    def host(self, ctx: binding.Context, shape, b: int):
        """(k, v, pos) that sequence b's filled rows stand for, as host arrays (fp64 / int32)."""
        torch = _torch()
        n = self.counts[b]
        k = torch.empty((max(n, 1), shape.Hkv, shape.d), dtype=torch.bfloat16 if shape.dtype == "bf16" else torch.float32, device="cuda")
        v = torch.empty_like(k)
        with _on_stream_of(ctx):
            ctx.spts_kv4_read([self.structs[b]], [0, n], k, v)
        return to_host(k[:n]).astype(np.float64), to_host(v[:n]).astype(np.float64), self.tensors[b][4][:n].cpu().numpy()


class LogitsRules:
    """spts_logits_rules for a batch of sequences.  history, bias, mask: device tensors (int32 [batch, n], fp32 and int32 of one
    row or one per sequence); the rest: host sequences of one value per sequence.  history_len and prompt_len may be
    changed between calls through the arrays of the same name."""

    def __init__(self, batch: int, history=None, history_len=None, prompt_len=None, repetition=None, frequency=None, presence=None,
                 bias=None, mask=None):
        self.struct = s = binding.spts_logits_rules()
        self.batch, self._keepalive = batch, (history, bias, mask)

        def host(values, typ):
            if values is None:
                return None
            if len(values) != batch:
                raise ValueError(f"one value per sequence: got {len(values)} for a batch of {batch}")
            return (typ * batch)(*values)

        def rows(t):
            if t.dim() not in (1, 2) or not t.is_contiguous() or (t.dim() == 2 and t.shape[0] not in (1, batch)):
                raise ValueError("bias and mask: one contiguous row, or one per sequence")
            return t.data_ptr(), 0 if t.dim() == 1 or t.shape[0] == 1 else t.shape[1]

        torch = _torch()
        for t, name, dts in ((history, "history", (torch.int32,)), (bias, "bias", (torch.float32,)), (mask, "mask", (torch.int32, torch.uint32))):
            if t is not None and t.dtype not in dts:
                raise ValueError(f"{name}: {dts[0]}, not {t.dtype}")
        if history is not None:
            if history.dim() != 2 or history.shape[0] != batch or not history.is_contiguous() or history_len is None:
                raise ValueError("history: a contiguous [batch, n] tensor, with history_len")
            if any(n > history.shape[1] for n in history_len):
                raise ValueError("history_len exceeds the history's rows")
            s.history, s.history_stride = history.data_ptr(), history.shape[1]
        self.history_len, self.prompt_len = host(history_len, ctypes.c_int64), host(prompt_len, ctypes.c_int64)
        self.repetition, self.frequency, self.presence = (host(v, ctypes.c_float) for v in (repetition, frequency, presence))
        for name in ("history_len", "prompt_len", "repetition", "frequency", "presence"):
            if getattr(self, name) is not None:
                setattr(s, name, getattr(self, name))
        if bias is not None:
            s.bias, s.bias_stride = rows(bias)
        if mask is not None:
            s.mask, s.mask_stride = rows(mask)
        s._keepalive = self._keepalive
        each = history is not None or s.bias_stride or s.mask_stride or any(v is not None for v in (self.repetition, self.frequency, self.presence))
        s._room = (batch if each else None, None if bias is None else bias.shape[-1], None if mask is None else mask.shape[-1])


class Q4DecodeRunner:
    """Decode phase with weights and caches in 4 bits for a batch of sequences: per step one spts_decode_layer_q4 per layer,
    the final norm, the head's 4-bit matrix and spts_process_logits.  Only enqueues work; tokens stay on the device.  All of it goes to the
    context's stream, between what torch's current stream has been given before and is given later.

    caches: one KV4Batch per layer; table [V, D]: the embedding (element type); head: its 4-bit form or another
    output matrix's; rules: LogitsRules, whose history the runner extends by the tokens it decodes (None = plain argmax)."""

    def __init__(self, ctx: binding.Context, shape, layers: List[binding.spts_layer_q4], caches: List[KV4Batch], gamma_f, table,
                 head: Q4Matrix, rules: Optional[LogitsRules] = None):
        torch = _torch()
        self.ctx, self.shape, self.layers, self.caches = ctx, shape, layers, caches
        self.gamma_f, self.table, self.head = gamma_f, table, head
        self.batch = len(caches[0].structs)
        self.rules = rules if rules is not None else LogitsRules(self.batch)
        V = int(table.shape[0])
        if len(layers) != len(caches) or any(len(c.structs) != self.batch for c in caches):
            raise ValueError("one KV4Batch per layer, all of the same number of sequences")
        if head.struct.rows != V or head.struct.K != shape.D or int(table.shape[1]) != shape.D:
            raise ValueError("table and head: [V, D]")
        if self.rules.batch != self.batch:
            raise ValueError("rules for another number of sequences")
        _, bias, mask = self.rules._keepalive
        if (bias is not None and bias.shape[-1] < V) or (mask is not None and mask.shape[-1] < (V + 31) // 32):
            raise ValueError(f"bias and mask: rows of {V} words")
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        if table.dtype != tdt or not table.is_contiguous():
            raise ValueError(f"table: a contiguous tensor of {tdt}")
        if gamma_f is not None and (gamma_f.dtype != tdt or not gamma_f.is_contiguous() or gamma_f.numel() != shape.D):
            raise ValueError(f"gamma_f: {shape.D} values of {tdt}")
        if any(t is not None and t.device != table.device for t in (*self.rules._keepalive, gamma_f)):
            raise ValueError(f"history, bias, mask and gamma_f: on {table.device} as the table is")
        self.x = torch.zeros((self.batch, shape.D), dtype=tdt, device="cuda")
        self.x_next, self.xn = torch.zeros_like(self.x), torch.zeros_like(self.x)
        self.tokens = torch.zeros(self.batch, dtype=torch.int32, device="cuda")
        self.logits = torch.zeros((self.batch, int(table.shape[0])), dtype=torch.float32, device="cuda")

    def step(self, pos):
        """Runs self.x (in place) through every layer as the tokens at the host positions pos."""
        with _on_stream_of(self.ctx):
            for w, c in zip(self.layers, self.caches):
                self.ctx.spts_decode_layer_q4(self.x, pos, w, c.structs)

    def next_token(self):
        """self.tokens and self.x_next from self.x: final norm, logits, rules, argmax, table row."""
        V = int(self.table.shape[0])
        with _on_stream_of(self.ctx):
            self.ctx.spts_rmsnorm(self.x, self.gamma_f, self.batch, self.xn)
            self.ctx.spts_matvec_q4(self.head.struct, self.xn, self.batch, self.logits, 1)
            self.ctx.spts_process_logits(self.logits, V, self.batch, self.rules.struct, self.logits, self.tokens, self.table, self.x_next)

    def generate(self, pos0: List[int], steps: int, tokens_out=None):
        """steps decode steps from self.x at positions pos0; tokens_out [batch, steps] int32 device.  With a history in the
        rules every token joins it: ValueError, before any step, if its rows, the caches or tokens_out have no room for that many, or
        positions are missing."""
        if len(pos0) != self.batch:
            raise ValueError(f"pos0: one position for each of {self.batch} sequences, got {len(pos0)}")
        if tokens_out is not None and (tokens_out.dim() != 2 or tokens_out.shape[0] != self.batch or tokens_out.shape[1] < steps):
            raise ValueError(f"tokens_out: [{self.batch}, {steps}]")
        hist, lens = self.rules._keepalive[0], self.rules.history_len
        if hist is not None and any(n + steps > hist.shape[1] for n in lens):
            raise ValueError(f"the history's rows of {hist.shape[1]} ids have no room for {steps} more")
        if any(s.count + steps > s.capacity for c in self.caches for s in c.structs):
            raise ValueError(f"a cache has no room for {steps} more pairs")
        with _on_stream_of(self.ctx):
            for t in range(steps):
                self.step([p + t for p in pos0])
                self.next_token()
                if hist is not None:
                    for b in range(self.batch):
                        hist[b, lens[b]:lens[b] + 1].copy_(self.tokens[b:b + 1])
                        lens[b] += 1
                if tokens_out is not None:
                    tokens_out[:, t].copy_(self.tokens)
                self.x.copy_(self.x_next)


# ------------------------------------------------------------------------------------------- caches in pages
class PagedKV:
    """One layer's caches of several sequences in pages of a pool that they share.  `pool` and `structs` are what the calls take (structs: a ctypes array of
    spts_kvp, its counts kept up to date by them); k, v [pages, Hkv, page, d], table [sequences, capacity / page], pos and weight
    [sequences, capacity] are the tensors behind them.  The host hands out the pages: reserve before appending, release after an eviction.
    A struct's capacity is what its sequence has pages for, from its first reserve or release on: appending more is refused.

    capacity: rows that a sequence may grow to (rounded up to whole pages); free: the order in which pages are handed out (None = 0, 1, 2, ..)."""

    def __init__(self, shape, pages: int, page: int, sequences: int, capacity: int, weights: bool = True, free=None):
        torch = _torch()
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        per = max(1, -(-int(capacity) // page))
        stride = (per + 3) // 4 * 4                     # rows of the table begin at multiples of 16 bytes
        self.page, self.shape = page, shape
        self.k = torch.empty((pages, shape.Hkv, page, shape.d), dtype=tdt, device="cuda")
        self.v = torch.empty_like(self.k)
        self._table = torch.full((sequences, stride), -1, dtype=torch.int32, device="cuda")
        self.table = self._table[:, :per]
        self.pos = torch.zeros((sequences, per * page), dtype=torch.int32, device="cuda")
        self.weight = torch.zeros((sequences, per * page), dtype=torch.float32, device="cuda") if weights else None
        self.pool = binding.spts_kv_pool(self.k.data_ptr(), self.v.data_ptr(), pages, page)
        self.pool._keepalive = (self.k, self.v)
        self.structs = (binding.spts_kvp * sequences)()
        self.structs._keepalive = (self._table, self.pos, self.weight)
        for b, s in enumerate(self.structs):
            s.table, s.pos = self._table.data_ptr() + 4 * stride * b, self.pos.data_ptr() + 4 * per * page * b
            s.weight = self.weight.data_ptr() + 4 * per * page * b if weights else None
            s.capacity = per * page
        self._most = per * page
        self.structs._unreserved = set(range(sequences))     # sequences that have never had a page
        every = np.arange(pages, dtype=np.int32)
        self._free = (every if free is None else np.array(free, dtype=np.int32).reshape(-1))[::-1].copy()      # the first _left are free, the last of them is the next
        self._left = pages
        if not np.array_equal(np.sort(self._free), every):
            raise ValueError(f"free: each of {pages} pages once")
        self.pages = [[] for _ in range(sequences)]     # the pages of each sequence, as its table has them

    @property
    def counts(self) -> List[int]:
        return [int(s.count) for s in self.structs]

    @property
    def free_pages(self) -> int:
        return self._left

    def reserve(self, b: int, rows: int, ctx: Optional[binding.Context] = None):
        """Pages for the first `rows` rows of sequence b; ValueError where its capacity or the pool has no room.  Writes the table from the
        host, in order with what the current stream is given, and with ctx in order with what its stream is given."""
        torch = _torch()
        have, need = len(self.pages[b]), -(-int(rows) // self.page)
        if need * self.page > self._most:
            raise ValueError(f"sequence {b}: {rows} rows exceed its capacity of {self._most}")
        if need - have > self._left:
            raise ValueError(f"{need - have} pages needed, {self._left} free")
        if need > have:
            left = self._left - (need - have)
            new = self._free[left:self._left][::-1].copy()
            with _on_stream_of(ctx) if ctx is not None else contextlib.nullcontext():
                self.table[b, have:need].copy_(torch.from_numpy(new))
            self._left = left                           # (the pages are free still where the copy was refused, in a capture for instance)
            self.pages[b] += new.tolist()
        self._owns(b)

    def release(self, b: int, ctx: Optional[binding.Context] = None):
        """Hands back the pages behind sequence b's count rows (all of them where it is 0).  Call it when the work on them is in the stream that
        their next owner uses too.  With ctx the table forgets them as well, in order with what its stream is given, so that a captured append that is
        replayed later writes nothing there."""
        have, need = len(self.pages[b]), -(-int(self.structs[b].count) // self.page)
        if ctx is not None and have > need:
            with _on_stream_of(ctx):
                self.table[b, need:have].fill_(-1)
        while len(self.pages[b]) > need:
            self._free[self._left] = self.pages[b].pop()
            self._left += 1
        self._owns(b)

    def _owns(self, b: int):
        self.structs[b].capacity = len(self.pages[b]) * self.page
        self.structs._unreserved.discard(b % len(self.structs))

    def append_cache(self, ctx: binding.Context, b: int, cache: "KVCache"):
        """Takes over every pair of a prefill's cache behind sequence b's rows (their weights 0); ValueError where it has other heads or
        another type, or there is no room."""
        if cache.k.dtype != self.k.dtype or tuple(cache.k.shape[1:]) != (self.shape.Hkv, self.shape.d):
            raise ValueError(f"a cache of {self.k.dtype} [.., {self.shape.Hkv}, {self.shape.d}], not {cache.k.dtype} {list(cache.k.shape)}")
        one = [self.structs[b]]
        with _on_stream_of(ctx):
            self.reserve(b, self.structs[b].count + cache.count)
            ctx.spts_kvp_append(self.pool, cache.k, cache.v, cache.pos, [0, cache.count], one)
        self.structs[b].count = one[0].count

    def host(self, ctx: binding.Context, b: int):
        """(k, v, pos) of sequence b's filled rows, as host arrays (fp64 / int32)."""
        n = self.counts[b]
        with _on_stream_of(ctx):
            k, v = (to_host(t[self.table[b].clamp(min=0).long()].transpose(1, 2).flatten(0, 1)[:n]).astype(np.float64) for t in (self.k, self.v))
            return k, v, self.pos[b, :n].cpu().numpy()


class StackRunner:
    """Runs Alg. 1's outer loop on the GPU: per layer one spts_layer_prefill, at stage ends one
    spts_msdp_compact.  Buffers are allocated once; run() only enqueues work (no host sync)."""

    def __init__(self, ctx: binding.Context, shape, layers: List[binding.spts_layer_weights], plan: List[dict],
                 probe_len: int, protect_last: int = 1, skip: int = 1, keep_trace: bool = False,
                 caches: Optional[List["KVCache"]] = None):
        torch = _torch()
        self.ctx, self.shape, self.layers, self.plan = ctx, shape, layers, plan
        self.caches = caches   # per-layer KV caches filled by the prefill (None = not kept)
        self.probe_len, self.protect_last, self.skip = probe_len, protect_last, skip
        N0 = plan[0]["N"]
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        self.xa = torch.empty((N0, shape.D), dtype=tdt, device="cuda")
        self.xb = torch.empty((N0, shape.D), dtype=tdt, device="cuda")
        self.posa = torch.empty(N0, dtype=torch.int32, device="cuda")
        self.posb = torch.empty(N0, dtype=torch.int32, device="cuda")
        self.s = torch.empty(N0, dtype=torch.float32, device="cuda")
        self.new2old = torch.empty(N0, dtype=torch.int32, device="cuda")
        self.keep_trace = keep_trace
        self.trace = []
        self.cfgs = []
        for item in plan:
            skip_l = 1 if (skip and item.get("skip", 1)) else 0   # a plan item may mark its layer dense
            self.cfgs.append(binding.spts_layer_cfg(skip_l, probe_len, item["m_attn"], item["m_ffn"], protect_last, 0))

    def run(self, x0, pos0):
        """x0 [N0, D] device tensor (copied, not modified), pos0 [N0] int32 device tensor.
        Returns (x, pos, N_final) as views into the runner's buffers."""
        torch = _torch()
        with _on_stream_of(self.ctx):
            xa, xb, pa, pb = self.xa, self.xb, self.posa, self.posb
            N = self.plan[0]["N"]
            xa[:N].copy_(x0)
            pa[:N].copy_(pos0)
            self.trace = []
            for li, (w, item, cfg) in enumerate(zip(self.layers, self.plan, self.cfgs)):
                tr = None
                if self.keep_trace:
                    tr = dict(N=N, x_in=xa[:N].clone(), pos_in=pa[:N].clone(),
                              idx_attn=torch.empty(max(min(N, item["m_attn"]), 1), dtype=torch.int32, device="cuda"),
                              idx_ffn=torch.empty(max(min(N, item["m_ffn"]), 1), dtype=torch.int32, device="cuda"))
                self.ctx.spts_layer_prefill(xa, pa, N, w, cfg, self.caches[li].struct if self.caches else None, self.s,
                                            tr["idx_attn"] if tr else None, tr["idx_ffn"] if tr else None)
                if tr is not None:
                    tr["x_out"] = xa[:N].clone()
                    tr["s_mha"] = self.s[:N].clone()
                if cfg.skip and item.get("N_next") is not None:
                    n_next = min(N, item["N_next"])
                    self.ctx.spts_msdp_compact(xa, pa, self.s, N, n_next, self.protect_last, xb, pb, self.new2old, None)
                    if tr is not None:
                        tr["map_new2old"] = self.new2old[:n_next].clone()
                    xa, xb = xb, xa
                    pa, pb = pb, pa
                    N = n_next
                if tr is not None:
                    self.trace.append(tr)
            return xa[:N], pa[:N], N


class BatchedStackRunner:
    """Alg. 1's outer loop over a batch of sequences laid back to back: per layer one spts_layer_prefill_batched,
    at stage ends one spts_msdp_compact_batched.  `plans` holds one layer plan (Workload.layer_plan()) per sequence;
    all plans have the same layers, stage ends and skip flags."""

    def __init__(self, ctx: binding.Context, shape, layers: List[binding.spts_layer_weights], plans: List[List[dict]],
                 probe_len: int, protect_last: int = 1):
        torch = _torch()
        self.ctx, self.shape, self.layers, self.plans = ctx, shape, layers, plans
        self.probe_len, self.protect_last = probe_len, protect_last
        n0 = sum(p[0]["N"] for p in plans)
        tdt = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
        self.xa = torch.empty((n0, shape.D), dtype=tdt, device="cuda")
        self.xb = torch.empty((n0, shape.D), dtype=tdt, device="cuda")
        self.posa = torch.empty(n0, dtype=torch.int32, device="cuda")
        self.posb = torch.empty(n0, dtype=torch.int32, device="cuda")
        self.s = torch.empty(n0, dtype=torch.float32, device="cuda")
        self.new2old = torch.empty(n0, dtype=torch.int32, device="cuda")

    def run(self, x0, pos0):
        """x0 [sum N0_b, D], pos0 [sum N0_b]: the sequences back to back.  Returns (x, pos, offsets)."""
        with _on_stream_of(self.ctx):
            xa, xb, pa, pb = self.xa, self.xb, self.posa, self.posb
            offs = [0]
            for p in self.plans:
                offs.append(offs[-1] + p[0]["N"])
            xa[:offs[-1]].copy_(x0)
            pa[:offs[-1]].copy_(pos0)
            for li, w in enumerate(self.layers):
                items = [p[li] for p in self.plans]
                skip_l = int(items[0].get("skip", 1))
                assert all(int(it.get("skip", 1)) == skip_l for it in items), "a layer is dense or skipped for the whole batch"
                self.ctx.spts_layer_prefill_batched(xa, pa, offs, w, self.probe_len, [it["m_attn"] for it in items],
                                                    [it["m_ffn"] for it in items], self.protect_last, None, self.s, skip=skip_l)
                if skip_l and items[0].get("N_next") is not None:
                    offs = self.ctx.spts_msdp_compact_batched(xa, pa, self.s, offs, [it["N_next"] for it in items],
                                                              self.protect_last, xb, pb, self.new2old)
                    xa, xb = xb, xa
                    pa, pb = pb, pa
            return xa[:offs[-1]], pa[:offs[-1]], offs


"""What the Python side of the 4-bit decode refuses because the C side could not see it: host arrays that are too short, tensors of another type
(no GPU: nothing is launched)."""
import ctypes as C
import gc
import types
import weakref

import pytest
import torch

from paper_2601_13155_amd import binding, runtime, synth
from tests.test_q4_refusals import A, ctx, i64, kv4, lib, q4  # noqa: F401  (ctx, lib: the fixtures)


def test_short_host_arrays(ctx):  # noqa: F811
    me = types.SimpleNamespace(handle=ctx())
    call = binding.Context
    for off in ([0], [0, 0], i64(0, 0)):
        with pytest.raises(ValueError):
            call.spts_kv4_append(me, A, A, A, off, kv4(2))
        with pytest.raises(ValueError):
            call.spts_kv4_read(me, kv4(2), off, A, A)
    with pytest.raises(ValueError):
        call.spts_kv4_read(me, kv4(2, count=8), [0, 0, 0], A, A, first=[1])
    w = binding.spts_layer_q4()
    for pos in ([], [3], (C.c_int32 * 1)(3)):
        with pytest.raises(ValueError):
            call.spts_decode_layer_q4(me, A, pos, w, kv4(2))
    call.spts_kv4_append(me, A, A, A, i64(0, 0, 0, 9), kv4(2))         # more than is read
    call.spts_kv4_append(me, A, A, A, [0, 0, 0], list(kv4(2)))
    call.spts_kv4_read(me, kv4(2, count=8), [0, 0, 0], A, A, first=[1, 8])


def test_matrices_of_another_type():
    me = types.SimpleNamespace(shape=synth.ModelShape(D=64, H=4, Hkv=2, d=32, Dff=64, dtype="f32"))
    for W in (torch.zeros((16, 64), dtype=torch.bfloat16), torch.zeros((16, 64), dtype=torch.float64), torch.zeros((16, 64)), torch.zeros((2, 16, 64))):
        with pytest.raises(ValueError):
            runtime.Q4Matrix(me, W)


def test_runner_of_another_type(monkeypatch):
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, _zeros=torch.zeros, **kw: _zeros(*a, **kw))
    shape = synth.ModelShape(D=64, H=4, Hkv=2, d=32, Dff=64, dtype="f32")
    table, gamma = torch.zeros((96, 64)), torch.ones(64)
    caches = types.SimpleNamespace(structs=kv4(2, capacity=16))
    make = lambda t=table, g=gamma, rules=None: runtime.Q4DecodeRunner(  # noqa: E731
        None, shape, [None], [caches], g, t, types.SimpleNamespace(struct=q4(96, 64)), rules)
    run = make()
    meta = torch.empty(96, device="meta")
    for bad in (lambda: make(table.bfloat16()), lambda: make(torch.zeros((64, 96)).t()), lambda: make(g=gamma.bfloat16()), lambda: make(g=torch.ones(32)),
                lambda: make(g=torch.ones(128)[::2]), lambda: make(rules=runtime.LogitsRules(2, bias=meta)),
                lambda: run.generate([0], 3), lambda: run.generate([0, 0, 0], 3),
                lambda: run.generate([0, 0], 3, torch.zeros((2, 2), dtype=torch.int32)), lambda: run.generate([0, 0], 3, torch.zeros((1, 3), dtype=torch.int32)),
                lambda: run.generate([0, 0], 3, torch.zeros(6, dtype=torch.int32))):
        with pytest.raises(ValueError):
            bad()


def test_structs_keep_their_tensors():
    """What a call is given is the struct; the tensors that it points into live as long."""
    hist, bias, mask = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(64), torch.zeros(2, dtype=torch.int32)
    s = runtime.LogitsRules(2, history=hist, history_len=[1, 2], bias=bias, mask=mask, repetition=[1.5, 2.5]).struct
    refs = [weakref.ref(t) for t in (hist, bias, mask)]
    del hist, bias, mask
    gc.collect()
    assert all(r() is not None for r in refs) and list(s.repetition[:2]) == [1.5, 2.5] and list(s.history_len[:2]) == [1, 2]


def test_caches_and_matrices_keep_their_buffers(monkeypatch):
    """The same of packed matrices and caches (host tensors in the place of device ones, nothing is launched)."""
    import contextlib
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, _empty=torch.empty, **kw: _empty(*a, **kw))
    monkeypatch.setattr(runtime, "_on_stream_of", lambda ctx: contextlib.nullcontext())
    shape = synth.ModelShape(D=64, H=4, Hkv=2, d=32, Dff=64, dtype="f32")
    structs = runtime.KV4Batch(shape, [9, 1]).structs
    gc.collect()
    buf = structs._keepalive
    assert structs[0].k == buf.data_ptr() and structs[1].pos + 4 * 8 <= buf.data_ptr() + buf.numel()

    class Matrix(torch.Tensor):
        is_cuda = True

    me = types.SimpleNamespace(shape=shape, spts_q4_pack=lambda W, s: None)
    s = runtime.Q4Matrix(me, torch.zeros((16, 64)).as_subclass(Matrix)).struct
    gc.collect()
    assert [t.data_ptr() for t in s._keepalive] == [s.codes, s.scales]


def test_rules_shorter_than_the_call(ctx):  # noqa: F811
    me = types.SimpleNamespace(handle=ctx())
    call = lambda V, n, **kw: binding.Context.spts_process_logits(me, A, V, n, runtime.LogitsRules(2, **kw).struct, None)  # noqa: E731
    for V, n, kw in ((64, 3, dict(repetition=[1.0, 1.0])), (65, 2, dict(bias=torch.zeros(64))), (65, 1, dict(bias=torch.zeros((2, 64)))), (64, 3, dict(bias=torch.zeros((2, 64)))),
                     (64, 3, dict(history=torch.zeros((2, 4), dtype=torch.int32), history_len=[1, 2])),
                     (65, 2, dict(mask=torch.zeros(2, dtype=torch.int32)))):
        with pytest.raises(ValueError):
            call(V, n, **kw)
    for V, n, kw in ((64, 2, dict(bias=torch.zeros(64), mask=torch.zeros(2, dtype=torch.int32))), (64, 1, {}), (64, 16, {}), (64, 5, dict(bias=torch.zeros(64))), (33, 2, dict(bias=torch.zeros((2, 80))))):
        with pytest.raises(binding.SptsError):           # these come to the library, which refuses the missing result
            call(V, n, **kw)

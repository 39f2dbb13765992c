"""What the Python side of the 4-bit decode refuses because the C side could not see it: host arrays that are too short, tensors of another type
(no GPU: nothing is launched)."""
import ctypes as C
import types

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

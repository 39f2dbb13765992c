"""Arguments that the 4-bit decode calls refuse, before anything is launched (no GPU: the pointers are never followed)."""
import ctypes as C
import os

import pytest

from paper_2601_13155_amd import binding, synth

A = 1 << 21      # aligned addresses that nothing lives at
INVAL, SHAPE, ALIGN, WORKSPACE, OK = binding.SPTS_EINVAL, binding.SPTS_ESHAPE, binding.SPTS_EALIGN, binding.SPTS_EWORKSPACE, binding.SPTS_OK


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return binding.load()


@pytest.fixture
def ctx(lib):
    """A context over TINY (D 256, H 4, Hkv 2, d 64, Dff 688, fp32) or another shape."""
    made = []

    def make(**kw):
        base = dict(D=256, H=4, Hkv=2, d=64, Dff=688, dtype="f32")
        base.update(kw)
        m = binding.model_desc(synth.ModelShape(**base))
        h = C.c_void_p()
        nb = binding.spts_workspace_bytes(m, 64, 1, 1, base["Dff"])
        assert lib.spts_create(C.byref(h), C.byref(m), None, C.c_void_p(1 << 20), nb, 64, 1, 1, base["Dff"]) == OK
        made.append(h)
        return h

    yield make
    for h in made:
        lib.spts_destroy(h)


def q4(rows=16, K=64, codes=A, scales=A):
    return binding.spts_q4(codes, scales, rows, K)


def kv4(n=1, capacity=64, count=0, at=A, **kw):
    arr = (binding.spts_kv4 * n)()
    for i, s in enumerate(arr):
        s.k, s.v, s.k_scale, s.v_scale, s.pos = (at + (5 * i + j) * 65536 for j in range(5))
        s.capacity, s.count = capacity, count
        for name, value in kw.items():
            setattr(s, name, value)
    return arr


def i64(*v):
    return (C.c_int64 * len(v))(*v)


def test_sizes(lib):
    c, s = C.c_size_t(), C.c_size_t()
    assert lib.spts_q4_bytes(1, 8, C.byref(c), C.byref(s)) == OK and (c.value, s.value) == (4096, 256)
    assert lib.spts_q4_bytes(4096, 14336, C.byref(c), C.byref(s)) == OK and (c.value, s.value) == (4096 * 14336 // 2, 4096 * 14336 // 32)
    assert lib.spts_q4_bytes(17, 520, C.byref(c), C.byref(s)) == OK and (c.value, s.value) == (4 * 4096, 4 * 256)
    for rows, K, why in ((0, 8, INVAL), (1, 0, INVAL), (-1, 8, INVAL), (1, 12, SHAPE), (1, 1 << 31, SHAPE), (1, (1 << 26) + 8, SHAPE),
                         ((1 << 28) + 1, 8, SHAPE)):
        assert lib.spts_q4_bytes(rows, K, C.byref(c), C.byref(s)) == why, (rows, K)
    assert lib.spts_q4_bytes(1, 8, None, C.byref(s)) == INVAL and lib.spts_q4_bytes(1, 8, C.byref(c), None) == INVAL
    m = binding.model_desc(synth.TINY)
    assert binding.spts_kv4_bytes(m, 24) == (24 * 2 * 32, 24 * 2 * 2)
    assert lib.spts_kv4_bytes(None, 8, C.byref(c), C.byref(s)) == INVAL
    for cap, why in ((0, INVAL), (-8, INVAL), (12, SHAPE), (1 << 31, SHAPE)):
        assert lib.spts_kv4_bytes(C.byref(m), cap, C.byref(c), C.byref(s)) == why
    for d in (16, 96, 256):
        bad = binding.model_desc(synth.TINY)
        bad.d = d
        assert lib.spts_kv4_bytes(C.byref(bad), 8, C.byref(c), C.byref(s)) == SHAPE


def test_pack_and_matvec(lib, ctx):
    h, w = ctx(), q4()
    pack = lambda W, m: lib.spts_q4_pack(h, W, C.byref(m) if m is not None else None)  # noqa: E731
    assert pack(None, w) == INVAL and pack(A, None) == INVAL and pack(A + 8, w) == ALIGN
    assert lib.spts_q4_pack(None, A, C.byref(w)) == INVAL
    mv = lambda m, x, n, y: lib.spts_matvec_q4(h, C.byref(m) if m is not None else None, x, n, y, 0)  # noqa: E731
    for m, why in ((q4(rows=0), INVAL), (q4(K=0), INVAL), (q4(K=-8), INVAL), (q4(K=60), SHAPE), (q4(codes=None), INVAL), (q4(scales=None), INVAL),
                   (q4(codes=A + 4), ALIGN), (q4(scales=A + 4), ALIGN), (q4(rows=(1 << 28) + 1), SHAPE), (q4(K=(1 << 26) + 8), SHAPE)):
        assert pack(A, m) == why and mv(m, A, 1, 2 * A) == why
    assert mv(w, A, 0, None) == OK
    assert mv(w, A, -1, 2 * A) == INVAL and mv(w, A, 17, 2 * A) == INVAL
    assert mv(w, None, 1, A) == INVAL and mv(w, A, 1, None) == INVAL and mv(w, A, 1, A) == INVAL and mv(None, A, 1, 2 * A) == INVAL
    assert mv(w, A + 2, 1, 2 * A) == ALIGN and mv(w, A, 1, 2 * A + 4) == ALIGN
    assert mv(w, A, 2, A + 496) == INVAL and mv(w, A + 112, 2, A) == INVAL            # 512 bytes of vectors, 128 of results: the last and the first overlap


def test_caches(lib, ctx):
    h = ctx()
    app = lambda off, n, c, k=A, v=A, pos=A, at=None: lib.spts_kv4_append(at or h, k, v, pos, off, n, c)  # noqa: E731
    assert app(None, 0, None) == OK
    assert app(i64(0, 1), -1, kv4()) == INVAL and app(i64(*range(18)), 17, kv4(17)) == INVAL
    assert app(i64(0, 1), 1, None) == INVAL and app(None, 1, kv4()) == INVAL
    assert app(i64(0, 1), 1, kv4(), k=None) == INVAL and app(i64(0, 1), 1, kv4(), v=None) == INVAL and app(i64(0, 1), 1, kv4(), pos=None) == INVAL
    assert app(i64(0, 1), 1, kv4(), k=A + 2) == ALIGN and app(i64(0, 1), 1, kv4(), pos=A + 4) == ALIGN
    assert app(i64(1, 2), 1, kv4()) == INVAL and app(i64(0, 3, 2), 2, kv4(2)) == INVAL
    assert app(i64(0, 65), 1, kv4()) == INVAL and app(i64(0, 5), 1, kv4(count=60)) == INVAL     # behind the capacity
    assert app(i64(0, 0), 1, kv4(count=64)) == OK                                                # nothing to append
    for name in ("k", "v", "k_scale", "v_scale", "pos"):
        assert app(i64(0, 1), 1, kv4(**{name: None})) == INVAL
        assert app(i64(0, 1), 1, kv4(**{name: A + 4})) == ALIGN
        assert app(i64(0, 1, 2), 2, kv4(2, **{name: A})) == INVAL                                # the same buffer twice
    for kw, why in ((dict(capacity=0), INVAL), (dict(count=-1), INVAL), (dict(count=65), INVAL), (dict(capacity=60), SHAPE), (dict(capacity=1 << 31), SHAPE)):
        assert app(i64(0, 1), 1, kv4(**kw)) == why
    for d in (16, 256):
        assert app(i64(0, 1), 1, kv4(), at=ctx(d=d)) == SHAPE
    c = kv4(count=3)
    assert app(i64(0, 64), 1, c) == INVAL and c[0].count == 3
    read = lambda first, off, n, c, k=A, v=A: lib.spts_kv4_read(h, c, first, off, n, k, v)  # noqa: E731
    assert read(None, None, 0, None) == OK and read(None, i64(0, 0), 1, kv4(count=8)) == OK
    assert read(None, i64(0, 9), 1, kv4(count=8)) == INVAL and read(i64(1), i64(0, 8), 1, kv4(count=8)) == INVAL
    assert read(i64(-1), i64(0, 1), 1, kv4(count=8)) == INVAL and read(i64(9), i64(0, 0), 1, kv4(count=8)) == INVAL
    assert read(None, i64(0, 1), 1, kv4(count=8), k=None) == INVAL and read(None, i64(0, 1), 1, kv4(count=8), v=A + 8) == ALIGN


def test_attention(lib, ctx):
    h = ctx()
    att = lambda n, c, q=A, out=A, at=None: lib.spts_kv4_attn(at or h, q, n, c, out)  # noqa: E731
    assert att(0, None) == OK and att(-1, kv4(count=8)) == INVAL and att(17, kv4(17, count=8)) == INVAL
    assert att(1, None) == INVAL and att(1, kv4(count=8), q=None) == INVAL and att(1, kv4(count=8), out=None) == INVAL
    assert att(1, kv4(count=8), q=A + 4) == ALIGN and att(1, kv4(count=8), out=A + 4) == ALIGN
    assert att(2, kv4(2, count=8), out=A + 2032) == INVAL and att(2, kv4(2, count=8), q=A + 1024) == INVAL   # out is q or lies apart
    assert att(1, kv4(count=65)) == INVAL and att(1, kv4(capacity=12, count=8)) == SHAPE
    assert att(1, kv4(count=8), at=ctx(H=17, Hkv=1)) == SHAPE and att(1, kv4(count=8), at=ctx(d=16)) == SHAPE


def test_layer(lib, ctx):
    h = ctx()

    def layer(**kw):
        w = binding.spts_layer_q4()
        for name, rows, K in (("Wq", 256, 256), ("Wk", 128, 256), ("Wv", 128, 256), ("Wo", 256, 256), ("Wgate", 688, 256), ("Wup", 688, 256), ("Wdown", 256, 688)):
            setattr(w, name, kw.get(name, q4(rows, K)))
        w.gamma1, w.gamma2 = kw.get("gamma1", A), kw.get("gamma2", A)
        return w

    pos = (C.c_int32 * 2)(5, 7)
    run = lambda w, n, c, x=A, p=pos: lib.spts_decode_layer_q4(h, x, p, n, C.byref(w), c)  # noqa: E731
    assert run(layer(), 0, None) == OK and run(layer(), 17, kv4(17)) == INVAL
    assert run(layer(), 1, kv4(), x=None) == INVAL and run(layer(), 1, kv4(), x=A + 4) == ALIGN and run(layer(), 1, kv4(), p=None) == INVAL
    assert run(layer(gamma1=None), 1, kv4()) == INVAL and run(layer(gamma2=A + 4), 1, kv4()) == ALIGN
    assert run(layer(Wk=q4(256, 256)), 1, kv4()) == SHAPE and run(layer(Wdown=q4(256, 680)), 1, kv4()) == SHAPE
    assert run(layer(Wo=q4(256, 256, codes=None)), 1, kv4()) == INVAL
    assert run(layer(), 1, kv4(count=64)) == INVAL and run(layer(), 2, kv4(2, k=A)) == INVAL
    assert run(layer(), 2, kv4(2), p=(C.c_int32 * 2)(5, -1)) == INVAL
    m = binding.model_desc(synth.TINY)
    assert lib.spts_rmsnorm(h, A, A, 2, A) == INVAL and lib.spts_rmsnorm(h, A, A, 2, A + 2032) == INVAL
    assert lib.spts_rmsnorm(h, A, A, 0, None) == OK and lib.spts_rmsnorm(h, A, A, 17, A) == INVAL
    assert lib.spts_rmsnorm(h, A, None, 1, A) == INVAL and lib.spts_rmsnorm(h, A, A + 4, 1, A) == ALIGN
    assert m.D == 256


def test_rules(lib, ctx):
    h = ctx()

    def rules(**kw):
        r = binding.spts_logits_rules()
        for name, v in kw.items():
            setattr(r, name, v)
        return r

    f = lambda *v: (C.c_float * len(v))(*v)  # noqa: E731
    run = lambda r, V=64, n=1, x=A, y=A, t=A, table=None, nxt=None: lib.spts_process_logits(h, x, V, n, C.byref(r) if r is not None else None, y, t, table, nxt)  # noqa: E731
    assert run(rules(), n=0) == OK and run(rules(), n=17) == INVAL and run(rules(), V=0) == INVAL and run(None) == INVAL
    assert run(rules(), V=(1 << 28) + 1) == SHAPE
    assert run(rules(), x=None) == INVAL and run(rules(), y=None) == INVAL and run(rules(), nxt=A) == INVAL
    assert run(rules(), t=None, table=A, nxt=A) == INVAL
    assert run(rules(), x=A + 4) == ALIGN and run(rules(), y=A + 4) == ALIGN and run(rules(), t=A + 4) == ALIGN and run(rules(), table=A + 4, nxt=A) == ALIGN
    assert run(rules(history=A)) == INVAL                                               # no lengths
    for n in (i64(-1, 0), i64(1 << 31, 0)):
        assert run(rules(history=A, history_stride=4, history_len=n)) == INVAL
    assert run(rules(history=A, history_stride=4, history_len=i64(5, 4)), n=2) == INVAL  # rows overlap
    assert run(rules(history=A, history_stride=4, history_len=i64(5))) == INVAL
    assert run(rules(), n=2, y=A + 496) == INVAL and run(rules(), x=A + 240) == INVAL       # results are the logits' own place or lie apart
    assert run(rules(history=A, history_stride=4, history_len=i64(4), prompt_len=i64(-1))) == INVAL
    assert run(rules(history=A + 4, history_stride=4, history_len=i64(4))) == ALIGN
    for name in ("repetition", "frequency", "presence"):
        for bad in (float("nan"), float("inf")):
            assert run(rules(**{name: f(1.0, bad)}), n=2) == INVAL
    assert run(rules(repetition=f(0.0))) == INVAL and run(rules(repetition=f(-1.0))) == INVAL
    assert run(rules(bias=A, bias_stride=63)) == INVAL and run(rules(mask=A, mask_stride=2), V=65) == INVAL
    assert run(rules(bias=A + 4)) == ALIGN and run(rules(mask=A + 4)) == ALIGN


def test_runtime_checks_its_arguments():
    import torch
    from paper_2601_13155_amd import runtime
    hist = torch.zeros((2, 8), dtype=torch.int32)
    r = runtime.LogitsRules(2, history=hist, history_len=[3, 8], repetition=[1.1, 1.2], bias=torch.zeros(64))
    assert r.struct.history_stride == 8 and r.struct.bias_stride == 0 and list(r.struct.history_len[:2]) == [3, 8]
    for kw in (dict(history=hist), dict(history=hist, history_len=[3]), dict(history=hist, history_len=[3, 9]), dict(repetition=[1.0]),
               dict(history=hist[:1], history_len=[3, 3]), dict(mask=torch.zeros((3, 2), dtype=torch.int32)), dict(bias=torch.zeros((64, 2)).t()),
               dict(history=hist.long(), history_len=[3, 8]), dict(bias=torch.zeros(64, dtype=torch.float64)), dict(mask=torch.zeros(2, dtype=torch.int64))):
        with pytest.raises(ValueError):
            runtime.LogitsRules(2, **kw)


def test_runner_checks_its_arguments(monkeypatch):
    """What would write behind a buffer, or fail in the middle of a run, is refused before anything is done (host tensors: nothing is launched)."""
    import types

    import torch
    from paper_2601_13155_amd import runtime
    monkeypatch.setattr(torch, "zeros", lambda *a, device=None, _zeros=torch.zeros, **kw: _zeros(*a, **kw))
    shape = synth.ModelShape(D=64, H=4, Hkv=2, d=32, Dff=64, dtype="f32")
    caches = lambda n, count=0: types.SimpleNamespace(structs=kv4(n, capacity=16, count=count))  # noqa: E731
    head = lambda rows, K=64: types.SimpleNamespace(struct=q4(rows, K))  # noqa: E731
    table = torch.zeros((96, 64))
    make = lambda cs, hd=head(96), layers=(None,), t=table, rules=None: runtime.Q4DecodeRunner(None, shape, list(layers), cs, None, t, hd, rules)  # noqa: E731
    make([caches(2)])
    hist = torch.zeros((2, 8), dtype=torch.int32)
    for bad in (lambda: make([caches(2)], layers=(None, None)), lambda: make([caches(2), caches(3)], layers=(None, None)),
                lambda: make([caches(2)], head(112)), lambda: make([caches(2)], head(96, 128)), lambda: make([caches(2)], t=torch.zeros((96, 32))),
                lambda: make([caches(2)], rules=runtime.LogitsRules(3)), lambda: make([caches(2)], rules=runtime.LogitsRules(2, bias=torch.zeros(95))),
                lambda: make([caches(2)], rules=runtime.LogitsRules(2, mask=torch.zeros((2, 2), dtype=torch.int32))),
                lambda: make([caches(2)], rules=runtime.LogitsRules(2, history=hist, history_len=[3, 6])).generate([0, 0], 3),
                lambda: make([caches(2, count=14)]).generate([0, 0], 3)):
        with pytest.raises(ValueError):
            bad()

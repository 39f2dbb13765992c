"""Arguments that the calls over caches in pages and the log probabilities refuse, before anything is launched (no GPU: the pointers are never followed)."""
import contextlib
import ctypes as C
import os
import types

import pytest

from paper_2601_13155_amd import binding, synth

A = 1 << 21      # aligned addresses that nothing lives at
INVAL, SHAPE, ALIGN, WORKSPACE, DTYPE, OK = (binding.SPTS_EINVAL, binding.SPTS_ESHAPE, binding.SPTS_EALIGN, binding.SPTS_EWORKSPACE, binding.SPTS_EDTYPE,
                                             binding.SPTS_OK)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__ as g
        g.build()
    return binding.load()


@pytest.fixture
def ctx(lib):
    """A context over 64 tokens of TINY's heads (H 4, Hkv 2, d 64, fp32) or another shape."""
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


def pool(k=A, v=2 * A, pages=10, page=16):
    return C.byref(binding.spts_kv_pool(k, v, pages, page))


def kvp(n=1, capacity=64, count=0, **kw):
    arr = (binding.spts_kvp * n)()
    for i, s in enumerate(arr):
        s.table, s.pos, s.weight = (3 * A + (3 * i + j) * 65536 for j in range(3))
        s.capacity, s.count = capacity, count
        for name, value in kw.items():
            setattr(s, name, value)
    return arr


def i64(*v):
    return (C.c_int64 * len(v))(*v)


def i32(*v):
    return (C.c_int32 * len(v))(*v)


BAD_POOLS = [(dict(k=None), INVAL), (dict(v=None), INVAL), (dict(k=A, v=A), INVAL), (dict(pages=0), INVAL), (dict(pages=1 << 31), SHAPE), (dict(k=A + 8), ALIGN), (dict(v=A + 2), ALIGN),
             (dict(page=8), SHAPE), (dict(page=0), SHAPE), (dict(page=48), SHAPE), (dict(page=512), SHAPE), (dict(page=-16), SHAPE)]
BAD_CACHES = [(dict(table=None), INVAL), (dict(pos=None), INVAL), (dict(capacity=0), INVAL), (dict(count=-1), INVAL), (dict(count=65), INVAL), (dict(table=3 * A + 4), ALIGN),
              (dict(pos=3 * A + 8), ALIGN), (dict(weight=3 * A + 4), ALIGN), (dict(capacity=72), SHAPE), (dict(capacity=1 << 31), SHAPE), (dict(capacity=(1 << 30) + 16), SHAPE)]


def test_every_call_refuses_bad_pools_and_caches(lib, ctx):
    h = ctx()
    append = lambda p, n, c: lib.spts_kvp_append(h, p, A, A, A, i64(*range(n + 1)), n, c)
    attn = lambda p, n, c: lib.spts_kvp_attn(h, p, A, i64(*range(n + 1)), n, c, A, 0, 1.0)
    evict = lambda p, n, c: lib.spts_kvp_evict(h, p, i64(*([1] * n)), None, None, n, c, None)
    for call in (append, attn, evict):
        for kw, why in BAD_POOLS:
            assert call(pool(**kw), 1, kvp(count=3)) == why, kw
        assert call(None, 1, kvp(count=3)) == INVAL and call(pool(), 1, None) == INVAL
        for kw, why in BAD_CACHES:
            assert call(pool(), 1, kvp(**{"count": 3, **kw})) == why, kw
        assert call(pool(), -1, kvp()) == INVAL and call(pool(), 17, kvp(17)) == INVAL and call(pool(), 0, None) == OK
    for d in (16, 96, 256):
        other = ctx(d=d)
        assert lib.spts_kvp_append(other, pool(), A, A, A, i64(0, 1), 1, kvp()) == SHAPE
        assert lib.spts_kvp_attn(other, pool(), A, i64(0, 1), 1, kvp(count=1), A, 0, 1.0) == SHAPE
        assert lib.spts_kvp_evict(other, pool(), i64(1), None, None, 1, kvp(), None) == SHAPE
    assert lib.spts_kvp_append(None, pool(), A, A, A, i64(0, 1), 1, kvp()) == INVAL
    assert lib.spts_kvp_attn(None, pool(), A, i64(0, 1), 1, kvp(count=1), A, 0, 1.0) == INVAL
    assert lib.spts_kvp_evict(None, pool(), i64(1), None, None, 1, kvp(), None) == INVAL


def test_append(lib, ctx):
    h = ctx()
    call = lambda off, caches, k=A, v=A, p=A: lib.spts_kvp_append(h, pool(), k, v, p, off, len(caches), caches)
    assert call(None, kvp()) == INVAL and call(i64(1, 2), kvp()) == INVAL and call(i64(0, 2, 1), kvp(2)) == INVAL
    assert call(i64(0, 1 << 31), kvp(capacity=1 << 30)) == SHAPE
    assert call(i64(0, 65), kvp()) == INVAL and call(i64(0, 2), kvp(count=63)) == INVAL
    for name in ("table", "pos", "weight"):
        two = kvp(2)
        setattr(two[1], name, getattr(two[0], name))
        assert call(i64(0, 1, 2), two) == INVAL, name
    for kw in (dict(k=None), dict(v=None), dict(p=None)):
        assert call(i64(0, 1), kvp(), **kw) == INVAL
    for kw in (dict(k=A + 8), dict(v=A + 8), dict(p=A + 4)):
        assert call(i64(0, 1), kvp(), **kw) == ALIGN
    c = kvp(2, count=5, weight=None)         # no account for either
    assert call(i64(0, 0, 0), c, k=None) == OK and [s.count for s in c] == [5, 5]


def test_attention(lib, ctx):
    h = ctx()
    call = lambda off, caches, q=A, out=4 * A, add=0, decay=1.0: lib.spts_kvp_attn(h, pool(), q, off, len(caches), caches, out, add, decay)
    assert call(None, kvp()) == INVAL and call(i64(1, 2), kvp(count=9)) == INVAL and call(i64(0, 2, 1), kvp(2, count=9)) == INVAL
    assert call(i64(0, 10), kvp(count=9)) == INVAL                         # more queries than rows
    assert call(i64(0, 65), kvp(capacity=128, count=100)) == WORKSPACE     # more than the context's tokens
    for kw in (dict(q=None), dict(out=None)):
        assert call(i64(0, 1), kvp(count=9), **kw) == INVAL
    for kw in (dict(q=A + 8), dict(out=A + 8)):
        assert call(i64(0, 1), kvp(count=9), **kw) == ALIGN
    assert call(i64(0, 2), kvp(count=9), q=A, out=A + 1024) == INVAL       # overlapping
    assert call(i64(0, 2), kvp(count=9), q=A, out=A, add=1) == INVAL       # the queries are read again for the accounts
    for decay in (-0.1, 1.5, float("nan"), float("inf")):
        assert call(i64(0, 1), kvp(count=9), add=1, decay=decay) == INVAL
    assert call(i64(0, 1), kvp(count=9, weight=None), add=1) == INVAL
    two = kvp(2, count=9)
    two[1].weight = two[0].weight
    assert call(i64(0, 1, 2), two, add=1) == INVAL
    assert call(i64(0, 0, 0), two, q=None, add=1) == OK


def test_evict(lib, ctx):
    h = ctx()
    call = lambda keep, caches, below=None, start=None, old=None: lib.spts_kvp_evict(h, pool(), keep, below, start, len(caches), caches, old)
    assert call(None, kvp()) == INVAL and call(i64(-1), kvp(count=9)) == INVAL
    assert call(i64(1), kvp(count=9, weight=None)) == INVAL
    assert call(i64(1), kvp(count=9), old=A + 4) == ALIGN
    for name in ("table", "pos", "weight"):
        two = kvp(2, count=9)
        setattr(two[1], name, getattr(two[0], name))
        assert call(i64(1, 1), two) == INVAL, name
    big = kvp(1, capacity=1 << 30, count=1 << 30)
    assert call(i64(1 << 29), big) == WORKSPACE and big[0].count == 1 << 30
    c = kvp(2, count=9)                      # nothing leaves, or everything: nothing is launched
    assert call(i64(9, 100), c, below=i32(1, 1), start=i32(5, 5)) == OK and [s.count for s in c] == [9, 9]
    assert call(i64(0, 0), c) == OK and [s.count for s in c] == [0, 0]


def test_logprobs(lib, ctx):
    h = ctx()
    base = dict(logits=A, dtype=0, stride=100, V=100, rows=2, tokens=A, logprob=A, entropy=A, n_top=2, ids=A, top=A)
    def call(**kw):
        a = {**base, **kw}
        return lib.spts_token_logprobs(h, a["logits"], a["dtype"], a["stride"], a["V"], a["rows"], a["tokens"], a["logprob"], a["entropy"], a["n_top"], a["ids"], a["top"])
    assert lib.spts_token_logprobs(None, A, 0, 100, 100, 2, A, A, A, 2, A, A) == INVAL
    for kw, why in ((dict(V=0), INVAL), (dict(rows=-1), INVAL), (dict(n_top=-1), INVAL), (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE), (dict(V=(1 << 28) + 1, stride=1 << 30), SHAPE),
                    (dict(n_top=33), SHAPE), (dict(rows=1 << 31), SHAPE), (dict(stride=99), INVAL), (dict(logits=None), INVAL), (dict(tokens=None), INVAL), (dict(logprob=None), INVAL),
                    (dict(n_top=0), INVAL), (dict(ids=None), INVAL), (dict(top=None), INVAL), (dict(ids=None, top=None), INVAL), (dict(rows=0), OK), (dict(rows=0, logits=None), OK)):
        assert call(**kw) == why, kw
    for name in ("logits", "tokens", "logprob", "entropy", "ids", "top"):
        assert call(**{name: A + 4}) == ALIGN, name


def test_logprobs_results_that_overlap(lib, ctx):
    h = ctx()
    rows, stride, V, top = 3, 120, 100, 4
    places = dict(logits=A, logprob=2 * A, entropy=3 * A, ids=4 * A, top=5 * A)
    size = dict(logits=4 * (2 * stride + V), logprob=4 * rows, entropy=4 * rows, ids=4 * rows * top, top=4 * rows * top)

    def call(dtype=0, **kw):
        a = {**places, **kw}
        return lib.spts_token_logprobs(h, a["logits"], dtype, stride, V, rows, 6 * A, a["logprob"], a["entropy"], top, a["ids"], a["top"])

    for one in places:
        for other in places:
            if one == other:
                continue
            assert call(**{one: places[other]}) == INVAL, (one, other)
            assert call(**{one: places[other] + (size[other] - 1) // 16 * 16}) == INVAL, (one, other)
    assert call(dtype=1, entropy=A + 2 * (2 * stride + V) // 16 * 16) == INVAL


def test_pages_are_handed_out_once(monkeypatch):
    """The host's side of runtime.PagedKV, on CPU tensors."""
    import torch
    from paper_2601_13155_amd import runtime

    class OnCpu:
        def __getattr__(self, name):
            f = getattr(torch, name)
            if name not in ("empty", "zeros", "full"):
                return f
            return lambda *a, device=None, **kw: f(*a, **kw)

    monkeypatch.setattr(runtime, "_torch", lambda: OnCpu())
    shape = synth.ModelShape(D=256, H=4, Hkv=2, d=64, Dff=256, dtype="f32")
    kv = runtime.PagedKV(shape, 6, 16, 3, 70, free=[5, 3, 1, 0, 2, 4])
    assert kv.structs[0].capacity == 80 and kv.free_pages == 6 and kv.counts == [0, 0, 0]
    assert all(s.table % 16 == 0 and s.pos % 16 == 0 and s.weight % 16 == 0 for s in kv.structs)
    kv.reserve(0, 17)
    kv.reserve(2, 16)
    kv.reserve(0, 30)
    assert kv.pages == [[5, 3], [], [1]] and kv.table[0, :3].tolist() == [5, 3, -1] and kv.table[2, 0] == 1
    with pytest.raises(ValueError):
        kv.reserve(1, 81)                    # beyond its capacity
    with pytest.raises(ValueError):
        kv.reserve(1, 64)                    # four pages of three
    assert kv.free_pages == 3
    kv.structs[0].count = 16
    kv.release(0)
    kv.release(1)
    assert kv.pages[0] == [5] and kv.free_pages == 4
    kv.reserve(1, 64)
    assert sorted(kv.pages[0] + kv.pages[1] + kv.pages[2]) == [0, 1, 2, 3, 4, 5]
    for free in ([0, 1, 2, 3, 4], [0, 1, 2, 3, 4, 4], list(range(7))):
        with pytest.raises(ValueError):
            runtime.PagedKV(shape, 6, 16, 3, 70, free=free)


@pytest.fixture
def on_cpu(monkeypatch):
    """runtime.PagedKV on CPU tensors."""
    import torch
    from paper_2601_13155_amd import runtime

    class OnCpu:
        def __getattr__(self, name):
            f = getattr(torch, name)
            return (lambda *a, device=None, **kw: f(*a, **kw)) if name in ("empty", "zeros", "full") else f

    monkeypatch.setattr(runtime, "_torch", lambda: OnCpu())
    monkeypatch.setattr(runtime, "_on_stream_of", lambda ctx: contextlib.nullcontext())
    return runtime.PagedKV


def test_rows_without_pages_are_not_appended(ctx, on_cpu):
    """Pages that were handed back may be another sequence's: what is appended has to lie in a sequence's own."""
    import torch
    shape = synth.ModelShape(D=256, H=4, Hkv=2, d=64, Dff=256, dtype="f32")
    me = types.SimpleNamespace(handle=ctx(), shape=shape, elem=torch.float32, i32=torch.int32)
    kv = on_cpu(shape, 6, 16, 3, 70)

    def append(rows, why, caches=None):
        offs = [sum(rows[:b]) for b in range(4)]
        with pytest.raises(binding.SptsError) as e:
            binding.Context.spts_kvp_append(me, kv.pool, A, A, A, offs, kv.structs if caches is None else caches)
        assert e.value.status == why
        assert kv.counts == before

    before = kv.counts
    for rows in ([0, 1, 0, 0], [0, 0, 0, 16]):
        with pytest.raises(ValueError):
            binding.Context.spts_kvp_append(me, kv.pool, A, A, A, [sum(rows[:b + 1]) for b in range(4)], kv.structs)
    binding.Context.spts_kvp_append(me, kv.pool, A, A, A, [0, 0, 0, 0], kv.structs)
    kv.reserve(0, 17)
    kv.reserve(1, 1)
    assert [s.capacity for s in kv.structs][:2] == [32, 16]
    kv.structs[0].count, kv.structs[1].count = 20, 3
    before = kv.counts
    append([13, 0, 0], INVAL)
    append([13, 0, 0], INVAL, list(kv.structs))
    kv.structs[0].count = 10
    kv.release(0)
    kv.reserve(1, 32)                          # takes the page that was handed back
    assert kv.pages[1][1] == kv.table[0, 1] and kv.structs[0].capacity == 16
    before = kv.counts
    append([7, 0, 0], INVAL)
    append([7, 2, 0], INVAL, list(kv.structs))
    kv.reserve(0, 17)
    assert kv.structs[0].capacity == 32 and not set(kv.pages[0]) & set(kv.pages[1])
    # nothing left: no rows, in any call
    kv.structs[0].count = 0
    kv.release(0, ctx=me)
    assert kv.structs[0].capacity == 0 and (kv.table[0] == -1).all() and kv.free_pages == 4
    before = kv.counts
    append([1, 0, 0], INVAL)
    binding.Context.spts_kvp_append(me, kv.pool, A, A, A, [0, 0, 0, 0], kv.structs)
    binding.Context.spts_kvp_attn(me, kv.pool, A, [0, 0, 0, 0], kv.structs, 4 * A)
    binding.Context.spts_kvp_evict(me, kv.pool, [5, 3, 1], kv.structs)
    assert kv.counts == [0, 3, 0]
    kv.reserve(0, 64)
    with pytest.raises(ValueError):
        kv.reserve(0, 81)
    assert kv.structs[0].capacity == 64 and kv.free_pages == 0


def test_a_reservation_that_failed_takes_no_pages(on_cpu, monkeypatch):
    import torch
    kv = on_cpu(synth.ModelShape(D=256, H=4, Hkv=2, d=64, Dff=256, dtype="f32"), 6, 16, 2, 70)
    kv.reserve(0, 20)

    def refused(*a):
        raise RuntimeError("not now")

    with monkeypatch.context() as m:
        m.setattr(torch, "from_numpy", refused)
        with pytest.raises(RuntimeError):
            kv.reserve(0, 64)
        with pytest.raises(RuntimeError):
            kv.reserve(1, 16)
    assert kv.free_pages == 4 and kv.pages == [[0, 1], []] and kv.structs[0].capacity == 32
    kv.reserve(1, 16)
    kv.reserve(0, 64)
    assert kv.pages == [[0, 1, 3, 4], [2]] and kv.table[0, :4].tolist() == [0, 1, 3, 4] and kv.table[1, 0] == 2


def test_sequences_counted_from_the_end(on_cpu):
    kv = on_cpu(synth.ModelShape(D=256, H=4, Hkv=2, d=64, Dff=256, dtype="f32"), 6, 16, 3, 70)
    kv.reserve(-1, 20)
    assert kv.pages == [[], [], [0, 1]] and [s.capacity for s in kv.structs] == [80, 80, 32] and kv.structs._unreserved == {0, 1}

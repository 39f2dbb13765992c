"""Caches in pages on the GPU: appending, attention of chunks and single tokens with its accounts, eviction; each against the plain form in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2601_13155_amd import binding, runtime, synth
from tests.paged import attend64, attend64_wide, attend_bound, context, evict64, filled, put, score_error, shape_of, TD

pytestmark = pytest.mark.gpu


def run_attn(ctx, kv, q, new, add=0, decay=1.0, out=None):
    out = torch.full_like(q, math.nan) if out is None else out
    offs = np.concatenate([[0], np.cumsum(new)]).tolist()
    ctx.spts_kvp_attn(kv.pool, q, offs, kv.structs, out, add, decay)
    return out


def check_attn(shape, kv, host, q, new, out, add=0, decay=1.0, before=None, chunk=None):
    """Outputs and accounts of every sequence against float64."""
    out, at, G = out.cpu(), 0, shape.H // shape.Hkv
    for b, m in enumerate(new):
        k, v = host[b]
        n = k.shape[0]
        if m:
            want, spread, big, got = attend64(q[at:at + m], k, v, shape.H, shape.Hkv)
            tol = attend_bound(want, spread, big, n, shape.d, shape.dtype, m * G > 16 if chunk is None else chunk)
            err = (out[at:at + m].double() - want).abs()
            assert bool((err <= tol).all()), (b, float((err / tol).max()), float(err.max()))
        at += m
        if not add or before is None:
            continue
        w = kv.weight[b].cpu().double()
        if m:
            want = got + (decay * before[b, :n].double() if decay else 0.0)
            # every term within its score's error on both sides of the quotient; sums of positive terms, of the row's and of the column's
            tol = want * (2 * score_error(big, shape.d) + 2 * (n + m * shape.H + 64) * 2.0 ** -24) + 1e-30
            assert bool(((w[:n] - want).abs() <= tol).all()), (b, float(((w[:n] - want).abs() / tol).max()))
        else:
            n = 0
        assert torch.equal(torch.nan_to_num(w[n:], nan=-7.0), torch.nan_to_num(before[b, n:].double(), nan=-7.0)), b


SETS = {   # rows of each sequence, new ones among them
    "one": ([1], [1]),
    "prompt": ([37], [37]),
    "ragged": ([517, 1, 38, 100, 95, 16], [1, 1, 5, 0, 64, 16]),
    "steps": ([300, 17, 1, 1040], [1, 1, 1, 1]),
    "chunk": ([700, 129], [130, 33]),
    "long": ([2500], [3]),
}


@pytest.mark.parametrize("rows,new", SETS.values(), ids=SETS.keys())
@pytest.mark.parametrize("H,Hkv", [(4, 2), (7, 1), (3, 3), (16, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_ragged_batches(dtype, H, Hkv, rows, new):
    d, page = {(4, 2): (64, 16), (7, 1): (128, 64), (3, 3): (32, 32), (16, 1): (128, 16)}[H, Hkv]
    shape = shape_of(H, Hkv, d, dtype)
    ctx = context(shape)
    kv, host = filled(shape, page, rows, seed=H + len(rows))
    q = (1.5 * torch.randn((sum(new), H, d), generator=torch.Generator().manual_seed(5))).to(TD[dtype]).cuda()
    check_attn(shape, kv, host, q, new, run_attn(ctx, kv, q, new))
    for decay in (1.0, 0.0, 0.75):
        before = kv.weight.cpu().clone()
        out = run_attn(ctx, kv, q, new, 1, decay)
        check_attn(shape, kv, host, q, new, out, 1, decay, before)
        if decay == 0.0:
            assert not torch.isnan(kv.weight[0, :rows[0]]).any()


@pytest.mark.parametrize("rows,new", [(600, 600), (700, 570), (1031, 517), (333, 300), (4000, 260)])
@pytest.mark.parametrize("H,Hkv,d", [(2, 2, 128), (3, 3, 64), (2, 2, 32), (3, 1, 128), (64, 1, 64), (5, 1, 32)])
def test_long_chunks(H, Hkv, d, rows, new):
    """Workgroups whose columns end far apart (a head of its own for every key/value head), groups that divide no block of columns, keys in shares."""
    shape = shape_of(H, Hkv, d, "bf16")
    new = new if H < 64 else new // 8
    ctx = context(shape, 1024)
    kv, host = filled(shape, 32, [rows], seed=rows + d)
    q = torch.randn((new, H, d), generator=torch.Generator().manual_seed(d)).bfloat16().cuda()
    before = kv.weight.cpu().clone()
    check_attn(shape, kv, host, q, [new], run_attn(ctx, kv, q, [new], 1, 0.5), 1, 0.5, before, chunk=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sixteen_sequences(dtype):
    shape = shape_of(8, 2, 64, dtype)
    ctx = context(shape, 512)
    rows = [1, 700, 64, 63, 65, 300, 128, 129, 5, 1000, 16, 17, 31, 32, 33, 250]
    new = [1, 1, 64, 1, 3, 40, 0, 129, 5, 2, 16, 1, 31, 4, 5, 1]
    kv, host = filled(shape, 16, rows, seed=16)
    q = torch.randn((sum(new), 8, 64), generator=torch.Generator().manual_seed(1)).to(TD[dtype]).cuda()
    before = kv.weight.cpu().clone()
    check_attn(shape, kv, host, q, new, run_attn(ctx, kv, q, new, 1, 0.25), 1, 0.25, before)


def check_wide(shape, rows, new, page, decay=0.5):
    """Outputs and accounts of a large call, every query of it."""
    ctx = context(shape, sum(new))
    kv, host = filled(shape, page, rows, seed=sum(rows) + shape.d)
    q = torch.randn((sum(new), shape.H, shape.d), generator=torch.Generator().manual_seed(shape.d)).to(TD[shape.dtype]).cuda()
    before = kv.weight.cpu().clone()
    outs, at = (run_attn(ctx, kv, q, new), run_attn(ctx, kv, q, new, 1, decay)), 0
    for b, m in enumerate(new):
        n = rows[b]
        want, spread, big, got = attend64_wide(q[at:at + m], *host[b], shape.H, shape.Hkv)
        tol = attend_bound(want, spread, big, n, shape.d, shape.dtype, m * shape.H // shape.Hkv > 16)
        for out in outs:
            err = (out[at:at + m].cpu().double() - want).abs()
            assert bool((err <= tol).all()), (b, float((err / tol).max()))
        w = got + decay * before[b, :n].double()
        tol = w * (2 * score_error(big, shape.d) + 2 * (n + m * shape.H + 64) * 2.0 ** -24) + 1e-30
        err = (kv.weight[b, :n].cpu().double() - w).abs()
        assert bool((err <= tol).all()), (b, float((err / tol).max()))
        at += m


@pytest.mark.parametrize("rows,new,H,Hkv,d,page", [([3300], [1024], 64, 8, 128, 16), ([2600], [600], 64, 64, 32, 16), ([3300, 2100], [1024, 300], 64, 16, 64, 32), ([12000], [32], 64, 32, 64, 16),
                                                   ([12000], [33], 32, 32, 32, 16), ([9000], [20], 64, 32, 128, 16)])
def test_chunks_over_more_pages_than_a_wavefront_has_at_hand(rows, new, H, Hkv, d, page):
    """Shares of more than 64 pages, from the first row on and from later ones: entries of the table come 64 at a time."""
    check_wide(shape_of(H, Hkv, d, "bf16"), rows, new, page)


UNEVEN = [int(4000 * (1 - 0.92 * b / 15)) for b in range(16)]


@pytest.mark.parametrize("rows,H,Hkv,d", [([60000], 128, 8, 128), ([150000], 64, 4, 32), (UNEVEN, 32, 8, 32), (UNEVEN, 32, 8, 64), (UNEVEN, 16, 8, 128)])
def test_accounts_of_single_tokens_whose_scores_leave_at_once(rows, H, Hkv, d):
    """Scores of shares that are too long for LDS, or of more workgroups than CUs, are stored as they come."""
    check_wide(shape_of(H, Hkv, d, "bf16"), rows, [1] * len(rows), 16)


def test_results_do_not_depend_on_the_batch():
    """A sequence alone and among others: the same accounts and results where its keys are in as many shares, and in any case within the tolerance."""
    shape = shape_of(8, 2, 64, "bf16")
    ctx = context(shape, 512)
    kv, host = filled(shape, 16, [300, 900, 77], seed=13)
    new = [40, 1, 3]
    q = torch.randn((44, 8, 64), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    run_attn(ctx, kv, q, new, 1, 0.0)
    w, at = kv.weight.clone(), 0
    for b, m in enumerate(new):
        one = (binding.spts_kvp * 1)(kv.structs[b])
        out = torch.empty_like(q[at:at + m])
        ctx.spts_kvp_attn(kv.pool, q[at:at + m].contiguous(), [0, m], one, out, 1, 0.0)
        want, spread, big, _ = attend64(q[at:at + m], *host[b], 8, 2)
        assert bool(((out.cpu().double() - want).abs() <= attend_bound(want, spread, big, 900, 64, "bf16", m * 4 > 16)).all())
        assert torch.allclose(kv.weight[b, :kv.counts[b]], w[b, :kv.counts[b]], rtol=1e-5)
        at += m


def test_accounts_without_room_for_scores():
    """300000 rows of 64 columns: their scores exceed a small context's scratch and are computed anew; and few shares of many columns in fp32."""
    shape = shape_of(64, 4, 32, "bf16")
    ctx = context(shape)
    kv, host = filled(shape, 256, [300000], seed=3)
    q = torch.randn((1, 64, 32), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    check_attn(shape, kv, host, q, [1], run_attn(ctx, kv, q, [1], 1, 0.0), 1, 0.0, kv.weight.cpu().clone())
    shape = shape_of(2, 2, 128, "f32")
    ctx = context(shape)
    kv, host = filled(shape, 64, [20000], seed=4)
    q = torch.randn((200, 2, 128), generator=torch.Generator().manual_seed(1)).cuda()
    check_attn(shape, kv, host, q, [200], run_attn(ctx, kv, q, [200], 1, 0.0), 1, 0.0, kv.weight.cpu().clone())


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_every_page_and_head_size(dtype, d, page):
    shape = shape_of(6, 2, d, dtype)
    ctx = context(shape)
    rows, new = [page, page + 1, 2 * page - 1, 3 * page + 7], [1, 15, 11, 2]
    kv, host = filled(shape, page, rows, seed=page + d)
    q = torch.randn((sum(new), 6, d), generator=torch.Generator().manual_seed(d)).to(TD[dtype]).cuda()
    before = kv.weight.cpu().clone()
    check_attn(shape, kv, host, q, new, run_attn(ctx, kv, q, new, 1, 1.0), 1, 1.0, before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,new", [([90], [70]), ([150], [40]), ([64], [4]), ([400], [300])])
def test_rows_that_a_query_does_not_see_do_not_matter(dtype, rows, new):
    """Keys and values of the chunk's later rows are infinities and NaN: the queries before them are as without these rows, the others are not finite."""
    shape = shape_of(8, 2, 64, dtype)
    ctx = context(shape, 512)
    kv, host = filled(shape, 16, rows, seed=3)
    n, m = rows[0], new[0]
    q = torch.randn((m, 8, 64), generator=torch.Generator().manual_seed(9)).to(TD[dtype]).cuda()
    bad = n - m + m // 2                   # the first row that holds something else
    k, v = (t.clone() for t in host[0])
    for i, x in enumerate((math.inf, -math.inf, math.nan)):
        v[bad + i % (n - bad), :, i::5] = x
        k[bad + i % (n - bad), :, i + 1::7] = x
    put(kv, 0, 0, k, v)
    out = run_attn(ctx, kv, q, new)
    good = m // 2
    want, spread, big, _ = attend64(q[:good], host[0][0][:bad], host[0][1][:bad], 8, 2)
    err = (out[:good].cpu().double() - want).abs()
    assert bool((err <= attend_bound(want, spread, big, n, 64, dtype, True)).all())
    assert not torch.isfinite(out[-1]).all()
    # a query that is NaN itself makes the accounts of the rows that it sees NaN, and only those
    put(kv, 0, 0, *host[0])
    q[m // 3, 3] = math.nan
    run_attn(ctx, kv, q, new, 1, 0.0)
    w = kv.weight[0].cpu()
    sees = n - m + m // 3 + 1
    assert torch.isnan(w[:sees]).all() and torch.isfinite(w[sees:n]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_values_reach_the_queries_that_see_them(dtype):
    """Values alone are infinite: exactly the dimensions of the queries that see such a row become that infinity, or NaN where two of them meet."""
    shape = shape_of(4, 1, 64, dtype)
    ctx = context(shape)
    kv, host = filled(shape, 16, [80], seed=4)
    k, v = (t.clone() for t in host[0])
    v[60, 0, 5], v[70, 0, 5], v[65, 0, 9], v[66, 0, 63] = math.inf, -math.inf, -math.inf, math.nan
    put(kv, 0, 0, k, v)
    q = (0.3 * torch.randn((48, 4, 64), generator=torch.Generator().manual_seed(9))).to(TD[dtype]).cuda()
    out = run_attn(ctx, kv, q, [48]).cpu()
    row = torch.arange(32, 80)
    for e in range(64):
        col = out[:, :, e]
        if e == 5:
            assert torch.isfinite(col[row < 60]).all() and (col[(row >= 60) & (row < 70)] == math.inf).all() and torch.isnan(col[row >= 70]).all()
        elif e == 9:
            assert torch.isfinite(col[row < 65]).all() and (col[row >= 65] == -math.inf).all()
        elif e == 63:
            assert torch.isfinite(col[row < 66]).all() and torch.isnan(col[row >= 66]).all()
        else:
            assert torch.isfinite(col).all(), e


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, 0.3])         # 0: all weights alike, probabilities of exactly 1
@pytest.mark.parametrize("rows,m", [(40, 1), (600, 1), (600, 4), (5000, 2), (5000, 40)])
@pytest.mark.parametrize("d", [32, 64, 128])
def test_infinite_values_wherever_their_row_lies(d, rows, m, scale, dtype):
    """Infinite and NaN values in blocks of keys that every query sees, in the last ones, in one share or several: each query gets the infinity of the dimensions that it sees one in (NaN
    where two meet), the other dimensions and the accounts are as without them."""
    shape = shape_of(8, 2, d, dtype)
    ctx = context(shape)
    kv, host = filled(shape, 16, [rows], seed=rows + d)
    k, v = (t.clone() for t in host[0])
    late = rows - 1 - m // 2                # not all queries see it
    for at, e, x in ((0, 1, math.inf), (7, 2, -math.inf), (rows // 2, 3, math.inf), (rows // 2 + 1, 30, -math.inf), (rows // 3, 5, math.nan), (late, 7, math.inf),
                     (3, 9, math.inf), (rows // 2, 9, math.inf), (3, 11, math.inf), (late, 11, -math.inf), (rows - 1, 13, -math.inf), (rows // 4, d - 1, math.inf)):
        v[at, :, e] = x
    put(kv, 0, 0, k, v)
    q = (scale * torch.randn((m, 8, d), generator=torch.Generator().manual_seed(9))).to(TD[dtype]).cuda()
    fine = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    want, spread, big, got = attend64(q, k, fine, 8, 2)
    bound = attend_bound(want, spread, big, rows, d, dtype, m * 4 > 16)
    for add in (0, 1):
        out = run_attn(ctx, kv, q, [m], add, 0.0).cpu().double()
        for i in range(m):
            seen = v[:rows - m + i + 1].double()
            for h in range(8):
                col = seen[:, h // 4]
                nan, up, down = torch.isnan(col).any(0), (col == math.inf).any(0), (col == -math.inf).any(0)
                nan = nan | (up & down)
                assert torch.equal(torch.isnan(out[i, h]), nan), (i, h, add)
                assert bool((out[i, h][up & ~nan] == math.inf).all()) and bool((out[i, h][down & ~nan] == -math.inf).all()), (i, h, add)
                rest = ~(nan | up | down)
                assert bool(((out[i, h] - want[i, h]).abs() <= bound[i, h])[rest].all()), (i, h, add)
    assert bool(((kv.weight[0, :rows].cpu().double() - got).abs() <= got * (2 * score_error(big, d) + 2 * (rows + m * 8 + 64) * 2.0 ** -24) + 1e-30).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m", [1, 40])
def test_scores_of_minus_infinity_weigh_nothing(dtype, m):
    shape = shape_of(4, 2, 32, dtype)
    ctx = context(shape)
    kv, host = filled(shape, 32, [200], seed=6)
    k, v = (t.clone() for t in host[0])
    q = torch.rand((m, 4, 32), generator=torch.Generator().manual_seed(2)).to(TD[dtype]).cuda() + 0.5
    k[:120] = -math.inf
    put(kv, 0, 0, k, v)
    out = run_attn(ctx, kv, q, [m], 1, 0.0)
    at = 200 - m
    for i in (0, m - 1):                    # as if the first 120 rows were not there
        want, spread, big, _ = attend64(q[i:i + 1], k[120:at + i + 1], v[120:at + i + 1], 4, 2)
        assert bool(((out[i:i + 1].cpu().double() - want).abs() <= attend_bound(want, spread, big, 200, 32, dtype, True)).all())
    assert bool((kv.weight[0, :120] == 0).all()) and abs(float(kv.weight[0, :200].sum()) - 4 * m) < 1e-3 * m
    put(kv, 0, 0, torch.full_like(k, -math.inf), v)
    assert bool((run_attn(ctx, kv, q, [m], 1, 0.0) == 0).all()) and bool((kv.weight[0, :200] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_entries_outside_the_pool_read_page_zero_and_are_not_written(dtype):
    shape = shape_of(4, 2, 64, dtype)
    ctx = context(shape)
    kv, host = filled(shape, 16, [70, 40], seed=8, garbage=0.0)
    kv.k[0], kv.v[0] = (torch.randn(kv.k[0].shape, generator=torch.Generator().manual_seed(1)).to(TD[dtype]).cuda() for _ in range(2))
    table = kv.table.cpu()
    for b, n in ((0, 70), (1, 40)):         # what the tables say, read by the test
        i = torch.arange(n)
        host[b] = tuple(t.cpu()[table[b, i // 16].long(), :, i % 16] for t in (kv.k, kv.v))
    for bad in (-1, kv.pool.pages, 2 ** 31 - 1, -2 ** 31):
        kv.table[0, 1] = bad
        want = [tuple(t.clone() for t in h) for h in host]
        i = torch.arange(16)
        want[0][0][16:32], want[0][1][16:32] = (t.cpu()[0].transpose(0, 1)[i] for t in (kv.k, kv.v))
        for new in ([1, 1], [30, 7]):
            q = torch.randn((sum(new), 4, 64), generator=torch.Generator().manual_seed(2)).to(TD[dtype]).cuda()
            check_attn(shape, kv, want, q, new, run_attn(ctx, kv, q, new, 1, 0.0))
    # appended rows on such a page go nowhere, the others to their places
    kv.structs[0].count, kv.structs[1].count = 16, 8
    k, v = (torch.randn((20, 2, 64), generator=torch.Generator().manual_seed(7)).to(TD[dtype]).cuda() for _ in range(2))
    kb, vb = kv.k.clone(), kv.v.clone()
    ctx.spts_kvp_append(kv.pool, k, v, torch.arange(20, dtype=torch.int32, device="cuda"), [0, 18, 20], kv.structs)
    assert kv.counts == [34, 10]
    for t, before, rows in ((kv.k, kb, k), (kv.v, vb, v)):
        before[table[0, 2].item(), :, :2] = rows[16:18].transpose(0, 1)
        before[table[1, 0].item(), :, 8:10] = rows[18:].transpose(0, 1)
        assert torch.equal(t, before)


def test_sequences_may_share_pages_that_are_read():
    shape = shape_of(4, 2, 64, "bf16")
    ctx = context(shape)
    kv, host = filled(shape, 16, [64, 90], seed=11)
    kv.table[1, :3] = kv.table[0, :3]
    shared = tuple(torch.cat([host[0][i][:48], host[1][i][48:]]) for i in (0, 1))
    new = [20, 1]
    q = torch.randn((21, 4, 64), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    check_attn(shape, kv, [host[0], shared], q, new, run_attn(ctx, kv, q, new, 1, 0.0))


@pytest.mark.parametrize("m", [1, 9])
def test_the_queries_may_be_overwritten_by_the_result(m):
    shape = shape_of(8, 2, 128, "bf16")
    ctx = context(shape)
    kv, _ = filled(shape, 64, [3000, 40], seed=12)
    q = torch.randn((2 * m, 8, 128), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    want = run_attn(ctx, kv, q, [m, m])
    run_attn(ctx, kv, q, [m, m], out=q)
    assert torch.equal(q, want)


def test_attention_beyond_32_bit_offsets():
    """A pool of more than 2^31 elements, the rows in use at both of its ends."""
    shape = shape_of(4, 1, 128, "bf16")
    ctx = context(shape)
    page, pages = 256, (1 << 31) // (256 * 128) + 64
    kv = runtime.PagedKV(shape, pages, page, 1, 1024, free=[pages - 1, 0, pages - 2] + list(range(1, pages - 2)))
    kv.reserve(0, 700)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((700, 1, 128), generator=g).bfloat16() for _ in range(2))
    ctx.spts_kvp_append(kv.pool, k.cuda(), v.cuda(), torch.arange(700, dtype=torch.int32, device="cuda"), [0, 700], kv.structs)
    hk, hv, _ = kv.host(ctx, 0)
    assert np.array_equal(hk, k.double().numpy()) and np.array_equal(hv, v.double().numpy())
    for m in (1, 50):
        q = torch.randn((m, 4, 128), generator=g).bfloat16().cuda()
        check_attn(shape, kv, [(k, v)], q, [m], run_attn(ctx, kv, q, [m], 1, 0.0))
    kv.weight[0, :700] = torch.arange(700.0).cuda()
    old = torch.empty(300, dtype=torch.int32, device="cuda")
    ctx.spts_kvp_evict(kv.pool, [300], kv.structs, old_out=old)
    o = old.cpu().long()
    assert np.array_equal(kv.host(ctx, 0)[0], k.double().numpy()[o])
    del kv
    torch.cuda.empty_cache()


def test_results_do_not_depend_on_the_run():
    shape = shape_of(28, 4, 128, "bf16")
    ctx = context(shape, 512)
    kv, _ = filled(shape, 16, [3000, 900, 77], seed=13)
    new = [40, 200, 1]
    q = torch.randn((241, 28, 128), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    first = run_attn(ctx, kv, q, new, 1, 0.0)
    w = kv.weight.clone()
    for _ in range(3):
        again = run_attn(ctx, kv, q, new, 1, 0.0)
        assert torch.equal(first, again) and torch.equal(torch.nan_to_num(w), torch.nan_to_num(kv.weight))


# ------------------------------------------------------------------------------------------------------------ append
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hkv,d,page", [(1, 32, 16), (3, 64, 32), (8, 128, 256)])
def test_append(dtype, Hkv, d, page):
    shape = shape_of(Hkv, Hkv, d, dtype)
    ctx = context(shape)
    had, new = [5, 0, page, 2 * page - 1, 3], [1, 40, 3 * page + 2, 1, 0]
    kv, host = filled(shape, page, had, seed=1, capacity=6 * page)
    for b in range(5):
        kv.reserve(b, had[b] + new[b])
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((sum(new), Hkv, d), generator=g).to(TD[dtype]) for _ in range(2))
    pos = torch.randint(0, 1 << 30, (sum(new),), generator=g, dtype=torch.int32)
    want = [t.clone() for t in (kv.k, kv.v, kv.pos, kv.weight)]
    ctx.spts_kvp_append(kv.pool, k.cuda(), v.cuda(), pos.cuda(), np.concatenate([[0], np.cumsum(new)]).tolist(), kv.structs)
    assert kv.counts == [h + n for h, n in zip(had, new)]
    at = 0
    table = kv.table.cpu().long()
    for b in range(5):
        for i in range(new[b]):
            r = had[b] + i
            want[0][table[b, r // page], :, r % page], want[1][table[b, r // page], :, r % page] = k[at + i].cuda(), v[at + i].cuda()
            want[2][b, r], want[3][b, r] = int(pos[at + i]), 0.0
        at += new[b]
    for got, w in zip((kv.k, kv.v, kv.pos, kv.weight), want):
        assert torch.equal(torch.nan_to_num(got, nan=-7.0), torch.nan_to_num(w, nan=-7.0))


def test_append_without_accounts_and_from_a_prefill():
    shape = shape_of(4, 2, 64, "f32")
    ctx = context(shape)
    kv = runtime.PagedKV(shape, 8, 16, 2, 64, weights=False)
    cache = runtime.KVCache(shape, 40)
    cache.k.normal_()
    cache.v.normal_()
    cache.pos[:] = torch.arange(40, device="cuda", dtype=torch.int32) * 2
    cache.struct.count = 37
    kv.append_cache(ctx, 1, cache)
    assert kv.counts == [0, 37] and kv.free_pages == 5
    for got, want in zip(kv.host(ctx, 1), cache.host()):
        assert np.array_equal(got, want)
    with pytest.raises(ValueError):
        kv.append_cache(ctx, 1, cache)      # 74 rows
    assert kv.counts == [0, 37]
    with pytest.raises(binding.SptsError):
        ctx.spts_kvp_evict(kv.pool, [1, 1], kv.structs)
    kv.structs[1].count = 16
    kv.release(1)
    assert kv.free_pages == 7 and len(kv.pages[1]) == 1


# ------------------------------------------------------------------------------------------------------------ eviction
def run_evict(shape, rows, keep, below=None, start=None, weights="random", page=16, seed=0, want_old=True, tokens=256):
    ctx = context(shape, tokens)
    kv, host = filled(shape, page, rows, seed=seed)
    r = np.random.default_rng(seed)
    w = [np.zeros(n, np.float32) for n in rows]
    for b, n in enumerate(rows):
        kv.pos[b, :n] = torch.from_numpy(r.permutation(n).astype(np.int32) * 2).cuda()
        if weights == "random":
            w[b] = np.exp(2 * r.standard_normal(n)).astype(np.float32)
        elif weights == "few":
            w[b] = r.integers(0, 3, n).astype(np.float32)
        elif weights == "odd":
            w[b] = r.standard_normal(n).astype(np.float32)
            for x in (np.nan, -np.nan, np.inf, -np.inf, -0.0, 0.0, 1e-40, 3.4e38):
                w[b][r.random(n) < 0.05] = x
        kv.weight[b, :n] = torch.from_numpy(w[b]).cuda()
    before = [t.clone() for t in (kv.k, kv.v, kv.pos, kv.weight)]
    kept = [min(n, k) for n, k in zip(rows, keep)]
    old = torch.full((sum(kept) + 4,), -9, dtype=torch.int32, device="cuda") if want_old else None
    ctx.spts_kvp_evict(kv.pool, keep, kv.structs, below, start, old)
    assert kv.counts == kept
    table, at = kv.table.cpu().long(), 0
    for b, n in enumerate(rows):
        want = evict64(w[b].tolist(), before[2][b, :n].tolist(), keep[b], None if below is None else below[b], None if start is None else start[b])
        if want_old:
            assert old[at:at + kept[b]].tolist() == want, b
        for new, o in enumerate(want):
            if new == o:
                continue
            for t in (0, 1):
                src = (kv.k, kv.v)[t]
                before[t][table[b, new // page], :, new % page] = src[table[b, o // page], :, o % page]
            before[2][b, new], before[3][b, new] = before[2][b, o].item(), before[3][b, o].item()
        at += kept[b]
    if want_old:
        assert old[at:].tolist() == [-9] * 4
    for got, want in zip((kv.k, kv.v, kv.pos, kv.weight), before):   # moved rows came, everything else is as it was
        assert torch.equal(torch.nan_to_num(got, nan=-7.0), torch.nan_to_num(want, nan=-7.0))


@pytest.mark.parametrize("weights", ["random", "few", "zero", "odd"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_evict(dtype, weights):
    shape = shape_of(4, 2, 64, dtype)
    rows = [1, 2, 63, 64, 65, 300, 1023, 1024, 1025, 100, 100, 100, 7]
    keep = [1, 1, 1, 63, 64, 150, 1000, 1, 1024, 0, 100, 200, 3]
    run_evict(shape, rows, keep, weights=weights, seed=1)
    run_evict(shape, rows, keep, below=[4] * 13, start=[2 * n - 20 for n in rows], weights=weights, seed=2, page=64)


@pytest.mark.parametrize("weights", ["few", "random", "zero", "odd"])
@pytest.mark.parametrize("rows,keep", [(5000, 4096), (8192, 4000), (8193, 4096), (20000, 311), (16384, 16383), (16384, 1), (16385, 16384), (40000, 20000)])
def test_evict_long_rows(rows, keep, weights):
    run_evict(shape_of(1, 1, 32, "bf16"), [rows], [keep], below=[10], start=[2 * rows - 500], weights=weights, seed=rows, page=128)


def test_evict_long_and_short_rows_together():
    run_evict(shape_of(1, 1, 32, "f32"), [9000, 20, 700, 30000, 12288, 5, 8192], [4097, 30, 0, 4096, 8192, 2, 8191], weights="few", seed=6, tokens=8192)
    run_evict(shape_of(1, 1, 32, "bf16"), [530000], [270001], weights="few", seed=7, page=256, want_old=False)     # chunks of 8192 rows


def test_evict_where_more_rows_move_than_workgroups_do_it():
    """2 x 1049353 rows, the later half of them with the larger weights: all of it moves, in order."""
    shape = shape_of(1, 1, 32, "bf16")
    ctx = context(shape, 32768)
    keep = (1 << 20) + 777
    n = 2 * keep
    kv = runtime.PagedKV(shape, -(-n // 256), 256, 1, n)
    kv.reserve(0, n)
    i = torch.arange(n, device="cuda")
    fill = lambda shift: ((i[:, None] >> shift) & 255).to(torch.bfloat16).expand(-1, 32)     # (numbers that bf16 holds)
    pages, at = i // 256, i % 256
    kv.k[pages, 0, at], kv.v[pages, 0, at] = fill(0), fill(8)
    kv.pos[0, :n] = (i + 7).int()
    kv.weight[0, :n] = i.float()
    kv.structs[0].count = n
    old = torch.full((keep,), -1, dtype=torch.int32, device="cuda")
    ctx.spts_kvp_evict(kv.pool, [keep], kv.structs, old_out=old)
    torch.cuda.synchronize()
    want = torch.arange(keep, n, device="cuda")
    assert kv.counts == [keep] and torch.equal(old.long(), want) and torch.equal(kv.pos[0, :keep].long(), want + 7) and torch.equal(kv.weight[0, :keep], want.float())
    assert torch.equal(kv.k[pages[:keep], 0, at[:keep]], fill(0)[keep:]) and torch.equal(kv.v[pages[:keep], 0, at[:keep]], fill(8)[keep:])


def test_evict_where_more_rows_go_before_others_than_stay():
    run_evict(shape_of(2, 1, 32, "bf16"), [200, 90], [20, 40], below=[100, 0], start=[300, 0], seed=3)
    run_evict(shape_of(2, 1, 32, "bf16"), [200], [20], start=[-2 ** 31], seed=4, want_old=False)
    run_evict(shape_of(2, 1, 32, "bf16"), [200], [20], below=[-2 ** 31], start=[2 ** 31 - 1], seed=5)


# ------------------------------------------------------------------------------------------------------------ together
def test_a_second_turn(tmp_path):
    """A token-skipped prefill's cache taken over into pages; a turn of new tokens with accounts; eviction to the budget; a step; the logits' log probabilities.
    Every part against 64 bits on what the parts before it left."""
    from tests.paged import logprobs64
    shape = synth.ModelShape(D=256, H=4, Hkv=2, d=64, Dff=512, dtype="bf16")
    wl = synth.scaled(synth.WORKLOADS["c0"], N=300)
    ctx = runtime.make_context(shape, 512, 16, 16, 512)
    dw = runtime.upload_layer(synth.make_layer(1, 0, shape, 16), shape, 16)
    x = runtime.to_device(synth.hidden_states(1, 300, shape.D, shape.dtype), "bf16")
    cache = runtime.KVCache(shape, 120)
    cfg = binding.spts_layer_cfg(1, 16, 120, 120, 1, 0)
    ctx.spts_layer_prefill(x, torch.arange(300, dtype=torch.int32, device="cuda"), 300, dw, cfg, cache.struct)
    kv = runtime.PagedKV(shape, 24, 16, 2, 192)
    kv.append_cache(ctx, 1, cache)
    assert kv.counts == [0, 120]
    g = torch.Generator().manual_seed(1)
    host = [[torch.zeros((0, 2, 64))] * 2, list(torch.from_numpy(t) for t in cache.host()[:2])]
    account = [torch.zeros(0, dtype=torch.float64), torch.zeros(120, dtype=torch.float64)]

    def turn(new):
        k, v = (torch.randn((sum(new), 2, 64), generator=g).bfloat16() for _ in range(2))
        q = torch.randn((sum(new), 4, 64), generator=g).bfloat16().cuda()
        for b, m in enumerate(new):
            kv.reserve(b, kv.counts[b] + m)
        offs = [0, new[0], sum(new)]
        ctx.spts_kvp_append(kv.pool, k.cuda(), v.cuda(), 300 + torch.arange(sum(new), dtype=torch.int32, device="cuda"), offs, kv.structs)
        out = torch.empty_like(q)
        ctx.spts_kvp_attn(kv.pool, q, offs, kv.structs, out, 1, 0.5)
        for b in range(2):
            rows = slice(offs[b], offs[b + 1])
            host[b] = [torch.cat([a.double(), f[rows].double()]) for a, f in zip(host[b], (k, v))]
            got = attend64(q[rows], *host[b], 4, 2)[3]
            account[b] = 0.5 * torch.cat([account[b], torch.zeros(new[b], dtype=torch.float64)]) + got
        check_attn(shape, kv, host, q, new, out)
        for b in range(2):
            assert torch.allclose(kv.weight[b, :kv.counts[b]].cpu().double(), account[b], rtol=1e-4, atol=1e-12)
        return out

    turn([30, 50])
    for b in range(2):                       # what the kernels have accumulated decides
        w, pos = kv.weight[b, :kv.counts[b]].tolist(), kv.pos[b, :kv.counts[b]].tolist()
        stay = evict64(w, pos, [24, 96][b], 2, 300 + 70)
        host[b] = [t[stay] for t in host[b]]
        account[b] = account[b][stay]
    ctx.spts_kvp_evict(kv.pool, [24, 96], kv.structs, [2, 2], [370, 370])
    kv.release(0)
    kv.release(1)
    assert kv.counts == [24, 96] and kv.free_pages == 24 - 2 - 6
    for b in range(2):
        assert all(np.array_equal(a, h.numpy()) for a, h in zip(kv.host(ctx, b)[:2], host[b]))
    out = turn([1, 1])
    table = torch.randn((1000, 256), generator=g).bfloat16().cuda()
    logits = torch.empty((2, 1000), device="cuda")
    tokens = torch.empty(4, dtype=torch.int32, device="cuda")
    gamma = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    ctx.spts_greedy_token_batched(out.reshape(2, 256), gamma, table, 1000, 2, tokens, logits)
    lp, ent, ids, tops = (torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty((2, 3), dtype=torch.int32, device="cuda"), torch.empty((2, 3), device="cuda"))
    ctx.spts_token_logprobs(logits, 1000, 2, tokens, lp, ent, 3, ids, tops)
    want = logprobs64(logits.cpu().double().numpy(), tokens[:2].tolist(), 3)
    assert np.array_equal(ids.cpu().numpy(), want[2]) and torch.equal(ids[:, 0], tokens[:2])
    for got, w in ((lp[:2], want[0]), (ent[:2], want[1]), (tops, want[3])):
        assert np.allclose(got.cpu().numpy(), w, rtol=2e-6, atol=2e-6)


def test_a_context_on_its_own_stream():
    """Tensors made on the current stream, calls on the context's: the conveniences order the two, and results are those of one stream."""
    shape = shape_of(4, 2, 64, "bf16")
    ctx = context(shape)
    side = torch.cuda.Stream()
    other = binding.Context(shape, 256, 1, 1, 256, stream=side)
    cache = runtime.KVCache(shape, 300)
    for t in (cache.k, cache.v):
        t.normal_()
    cache.pos[:] = torch.arange(300, device="cuda", dtype=torch.int32)
    cache.struct.count = 300
    q = torch.randn((3, 4, 64), device="cuda").bfloat16()
    outs = []
    for c in (ctx, other):
        kv = runtime.PagedKV(shape, 24, 16, 1, 330)
        torch.cuda._sleep(20_000_000)          # the current stream is busy: an unordered call would read tables and rows that are not there yet
        kv.append_cache(c, 0, cache)
        kv.reserve(0, 320, c)
        with runtime._on_stream_of(c):
            out = torch.empty_like(q)
            c.spts_kvp_attn(kv.pool, q, [0, 3], kv.structs, out, 1, 0.0)
        outs.append((out.clone(), kv.weight.clone(), kv.host(c, 0)))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
    assert all(np.array_equal(a, b) for a, b in zip(outs[0][2], outs[1][2]))


def test_tensors_that_do_not_fit_are_refused():
    shape = shape_of(4, 2, 64, "bf16")
    ctx = context(shape)
    kv, _ = filled(shape, 16, [40], seed=1, capacity=64)
    kv.reserve(0, 64)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    for k, v, p in ((bf(3, 2, 64), bf(4, 2, 64), pos), (bf(4, 2, 64), bf(4, 2, 64).float(), pos), (bf(4, 2, 64), bf(4, 2, 64), pos.long()), (bf(4, 2, 64).cpu(), bf(4, 2, 64), pos),
                    (bf(4, 2, 128)[:, :, ::2], bf(4, 2, 64), pos), (bf(4, 2, 64), bf(4, 2, 64), pos[:3])):
        with pytest.raises(ValueError):
            ctx.spts_kvp_append(kv.pool, k, v, p, [0, 4], kv.structs)
    for q, out in ((bf(1, 4, 64), bf(2, 4, 64)), (bf(2, 4, 64).float(), bf(2, 4, 64)), (bf(2, 4, 64), bf(2, 4, 128)[..., :64])):
        with pytest.raises(ValueError):
            ctx.spts_kvp_attn(kv.pool, q, [0, 2], kv.structs, out)
    with pytest.raises(ValueError):
        ctx.spts_kvp_attn(kv.pool, bf(2, 4, 64), [0], kv.structs, bf(2, 4, 64))
    for old in (torch.zeros(10, dtype=torch.int64, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            ctx.spts_kvp_evict(kv.pool, [10], kv.structs, old_out=old)
    with pytest.raises(ValueError):
        kv.append_cache(ctx, 0, runtime.KVCache(shape_of(4, 2, 64, "f32"), 4))
    assert kv.counts == [40]


@pytest.mark.parametrize("replays", [4])
def test_calls_captured_into_graphs(replays):
    """A step's append, attention with accounts and eviction in one graph; two graphs of one context take turns, with eager work between them."""
    shape = shape_of(8, 2, 64, "bf16")
    ctx = None
    stream = torch.cuda.Stream()
    g = torch.Generator().manual_seed(1)
    with torch.cuda.stream(stream):
        ctx = binding.Context(shape, 256, 1, 1, 256, stream=stream)
        kv, _ = filled(shape, 16, [600, 90], seed=14, capacity=640)
        for b in range(2):
            kv.reserve(b, 640)
        k, v = (torch.randn((6, 2, 64), generator=g).bfloat16().cuda() for _ in range(2))
        q = torch.randn((6, 8, 64), generator=g).bfloat16().cuda()
        pos = torch.arange(6, dtype=torch.int32, device="cuda") + 5000
        start = [t.clone() for t in (kv.k, kv.v, kv.pos, kv.weight)]
        logits = torch.randn((3, 5000), generator=g).cuda()
        tokens = torch.tensor([3, 7, 4999, 0], dtype=torch.int32, device="cuda")

        def restore():
            for t, s in zip((kv.k, kv.v, kv.pos, kv.weight), start):
                t.copy_(s)

        def work(out, old, lp, ids, tops):
            kv.structs[0].count, kv.structs[1].count = 600, 90
            ctx.spts_kvp_append(kv.pool, k, v, pos, [0, 2, 6], kv.structs)
            ctx.spts_kvp_attn(kv.pool, q, [0, 2, 6], kv.structs, out, 1, 1.0)
            ctx.spts_kvp_evict(kv.pool, [500, 80], kv.structs, None, [5000, 5000], old)
            ctx.spts_token_logprobs(logits, 5000, 3, tokens, lp, None, 5, ids, tops)

        def outputs():
            return [torch.zeros_like(q), torch.zeros(580, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda"),
                    torch.zeros((3, 5), dtype=torch.int32, device="cuda"), torch.zeros((3, 5), device="cuda")]

        eager = outputs()
        restore()
        work(*eager)
        state = [t.clone() for t in (kv.k, kv.v, kv.pos, kv.weight)]
        stream.synchronize()
        graphs, outs = [], []
        for _ in range(2):
            outs.append(outputs())
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=stream):
                work(*outs[-1])
            graphs.append(gr)
        for i in range(replays):
            for gr, o in zip(graphs, outs):
                restore()
                for t in o:
                    t.zero_()
                gr.replay()
                stream.synchronize()
                for a, e in zip(o, eager):
                    assert torch.equal(a, e), i
                for a, e in zip((kv.k, kv.v, kv.pos, kv.weight), state):
                    assert torch.equal(torch.nan_to_num(a, nan=-7.0), torch.nan_to_num(e, nan=-7.0)), i
                (torch.randn(512, 512, device="cuda") @ torch.randn(512, 512, device="cuda")).sum().item()
    torch.cuda.synchronize()

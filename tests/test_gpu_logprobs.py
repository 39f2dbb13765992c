"""Log probabilities of given words, entropies and best alternatives, against the plain form in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2601_13155_amd import binding
from tests.paged import context, logprobs64, shape_of, TD

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return context(shape_of(4, 2, 64, "bf16"))


def check(ctx, x, tokens, top, V=None, stride=None, dtype=None):
    """x: device [rows, >= V]; compares everything that the call gives."""
    rows, V = x.shape[0], x.shape[1] if V is None else V
    t = torch.tensor(tokens, dtype=torch.int32, device="cuda")
    lp, ent = torch.full((rows + 1,), -5.0, device="cuda"), torch.full((rows + 1,), -5.0, device="cuda")
    ids = torch.full((rows + 1, top), -5, dtype=torch.int32, device="cuda") if top else None
    tops = torch.full((rows + 1, top), -5.0, device="cuda") if top else None
    ctx.spts_token_logprobs(x, V, rows, t, lp, ent, top, ids, tops, stride=stride)
    h = x[:, :V].double().cpu().numpy()
    want = logprobs64(h, tokens, top)
    # fp32: the exponentials' and the sums' steps (V of them at most, of positive terms, over 1024 threads and then pairwise), the two differences, the logarithm
    steps = (V / 1024 + 64) * 2.0 ** -24
    with np.errstate(all="ignore"):
        size = np.nan_to_num(np.abs(want[0]), nan=0.0, posinf=0.0) + 1.0
        close = lambda a, b, s: np.all(np.isclose(a, b, rtol=0, atol=0, equal_nan=True) | (np.abs(a - b) <= steps * s * 4))
    assert close(lp[:rows].cpu().numpy().astype(np.float64), want[0], size), (lp[:rows].tolist()[:4], want[0][:4])
    assert close(ent[:rows].cpu().numpy().astype(np.float64), want[1], np.nan_to_num(np.abs(want[1]), nan=0.0) + 1.0 + math.log(V + 1))
    assert float(lp[rows]) == -5.0 and float(ent[rows]) == -5.0
    if top:
        assert np.array_equal(ids[:rows].cpu().numpy(), want[2])
        s = np.nan_to_num(np.abs(want[3]), nan=0.0, posinf=0.0) + 1.0
        assert close(tops[:rows].cpu().numpy().astype(np.float64), want[3], s)
        assert (ids[rows] == -5).all() and (tops[rows] == -5.0).all()


@pytest.mark.parametrize("top", [0, 1, 5, 32])
@pytest.mark.parametrize("V", [1, 2, 31, 32, 500, 1023, 4096, 4097, 16385, 50001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_random_rows(ctx, dtype, V, top):
    g = torch.Generator().manual_seed(V + top)
    for rows in (1, 7):
        x = (3.0 * torch.randn((rows, V), generator=g)).to(TD[dtype]).cuda()
        check(ctx, x, torch.randint(0, V, (rows,), generator=g).tolist(), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V", [(300, 1000), (257, 20011), (1, 128256)])
def test_many_rows_and_long_ones(ctx, dtype, rows, V):
    g = torch.Generator().manual_seed(rows)
    x = (3.0 * torch.randn((rows, V), generator=g)).to(TD[dtype]).cuda()
    check(ctx, x, torch.randint(0, V, (rows,), generator=g).tolist(), 20)


@pytest.mark.parametrize("kind", ["ascending", "descending", "constant", "steps", "saw"])
@pytest.mark.parametrize("rows", [1, 260])
def test_rows_in_every_order(ctx, rows, kind):
    """Rows that fill the list of candidates again and again, and rows of equals, of which the lowest words count."""
    V = 40003
    i = torch.arange(V, dtype=torch.float32)
    x = {"ascending": i / 4000, "descending": -i / 4000, "constant": torch.zeros(V), "steps": (i / 5000).floor(), "saw": (i % 977) + (i / 8000).floor()}[kind]
    for dtype in ("f32", "bf16"):
        y = x.to(TD[dtype]).cuda().repeat(rows, 1)
        for top in (1, 32):
            check(ctx, y[:4] if rows == 1 else y, [V - 1] * (4 if rows == 1 else rows), top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_words_that_are_not_allowed(ctx, dtype):
    g = torch.Generator().manual_seed(3)
    V = 9001
    x = torch.randn((6, V), generator=g)
    x[0] = torch.where(torch.rand(V, generator=g) < 0.999, torch.tensor(-math.inf), x[0])
    x[1] = -math.inf
    x[2, :], x[2, 77] = -math.inf, 2.0
    x[3, 5000] = math.nan
    x[4, 8000] = math.inf
    x[5] = x[5] * 1e37
    check(ctx, x.to(TD[dtype]).cuda(), [0, 5, 77, 3, 8000, 9000], 12)
    check(ctx, x.to(TD[dtype]).cuda().repeat(50, 1), [0, 5, 78, 5000, 3, 100] * 50, 12)
    check(ctx, torch.full((2, 40), -3.4028e38, dtype=torch.float32).to(TD[dtype]).cuda(), [1, 39], 3)


def test_tokens_outside_the_words(ctx):
    x = torch.randn((4, 100), generator=torch.Generator().manual_seed(1)).cuda()
    check(ctx, x, [-1, 100, 2 ** 31 - 1, 99], 2)
    x = x.repeat(100, 100)
    check(ctx, x, [-1, 10000, -2 ** 31, 99] * 100, 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_apart_and_part_of_them(ctx, dtype):
    g = torch.Generator().manual_seed(2)
    x = torch.randn((9, 5037), generator=g).to(TD[dtype]).cuda()
    check(ctx, x, torch.randint(0, 3001, (9,), generator=g).tolist(), 4, V=3001)
    wide = torch.full((5, 2 * 5037), 50.0).to(TD[dtype]).cuda()
    wide[:, :5037] = x[:5]
    check(ctx, wide[:, :5037], [1, 2, 3, 4, 5], 4, V=5037)
    flat = x.reshape(-1)
    check(ctx, flat[:5037 * 3].reshape(3, 5037), [5036, 0, 1], 3, V=5037, stride=5037)


def test_only_what_is_wanted(ctx):
    x = torch.randn((3, 7000), generator=torch.Generator().manual_seed(2)).cuda()
    tokens = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda")
    lp, ent, ids, tops = (torch.empty(4, device="cuda"), torch.empty(4, device="cuda"), torch.empty((3, 2), dtype=torch.int32, device="cuda"), torch.empty((3, 2), device="cuda"))
    ctx.spts_token_logprobs(x, 7000, 3, tokens, lp, ent, 2, ids, tops)
    for args in (dict(tokens=tokens, logprob=torch.empty(4, device="cuda")), dict(entropy=torch.empty(4, device="cuda")),
                 dict(n_top=2, top_ids=torch.empty((3, 2), dtype=torch.int32, device="cuda"), top_logprobs=torch.empty((3, 2), device="cuda"))):
        ctx.spts_token_logprobs(x, 7000, 3, **args)
        for name, want in (("logprob", lp), ("entropy", ent), ("top_ids", ids), ("top_logprobs", tops)):
            if name in args:
                assert torch.equal(args[name][:3], want[:3]), name
    with pytest.raises(ValueError):
        ctx.spts_token_logprobs(x.half(), 7000, 3, tokens, lp)
    with pytest.raises(ValueError):
        ctx.spts_token_logprobs(x.t(), 3, 7000, tokens, lp)
    for bad in (dict(tokens=tokens.long(), logprob=lp), dict(tokens=tokens[:2], logprob=lp), dict(entropy=lp.double()), dict(entropy=lp[::2]), dict(tokens=tokens.cpu(), logprob=lp),
                dict(n_top=3, top_ids=ids, top_logprobs=torch.empty((3, 3), device="cuda"))):
        with pytest.raises(ValueError):
            ctx.spts_token_logprobs(x, 7000, 3, **bad)
    for V, rows, stride in ((7001, 3, None), (7000, 4, None), (7000, 3, 7001)):
        with pytest.raises(ValueError):
            ctx.spts_token_logprobs(x, V, rows, entropy=torch.empty(8, device="cuda"), stride=stride)


@pytest.mark.parametrize("rows,V", [(255, 2049), (255, 20011), (129, 5000), (37, 20011), (1, 140000)])
def test_the_smallest_contexts_serve_every_call(rows, V):
    """Rows in parts with the longest lists, whose scratch is independent of the context's heads and tokens."""
    g = torch.Generator().manual_seed(rows + V)
    x = (3.0 * torch.randn((rows, V), generator=g)).cuda()
    for H, Hkv, d in ((1, 1, 32), (2, 1, 64)):
        check(context(shape_of(H, Hkv, d, "f32"), 1), x, torch.randint(0, V, (rows,), generator=g).tolist(), 32)


def test_more_elements_than_32_bits(ctx):
    rows, V = 16400, 131072 + 64
    x = torch.empty((rows, V), dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 1025):
        x[i:i + 1025].normal_()
    t = torch.arange(rows, dtype=torch.int32, device="cuda")
    lp, ids, tops = torch.empty(rows, device="cuda"), torch.empty((rows, 2), dtype=torch.int32, device="cuda"), torch.empty((rows, 2), device="cuda")
    ctx.spts_token_logprobs(x, V, rows, t, lp, None, 2, ids, tops)
    at = [0, 8191, 16383, 16399]
    want = logprobs64(x[at].double().cpu().numpy(), at, 2)
    assert np.allclose(lp[at].cpu().numpy(), want[0], rtol=1e-5) and np.array_equal(ids[at].cpu().numpy(), want[2])
    del x
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_rows_than_a_launch_has(ctx, dtype):
    """2^24 + 300 rows of two words, against torch in 64 bits."""
    rows = (1 << 24) + 300
    x = torch.randn((rows, 2), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(TD[dtype])
    t = (torch.arange(rows, device="cuda") % 2).int()
    lp, ent, tops = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros((rows, 1), device="cuda")
    ids = torch.full((rows, 1), -5, dtype=torch.int32, device="cuda")
    ctx.spts_token_logprobs(x, 2, rows, t, lp, ent, 1, ids, tops)
    z = torch.log_softmax(x.double(), 1)
    bound = (2 / 1024 + 64) * 2.0 ** -24 * 4 * (1 + float(z.abs().max()))     # as in check()
    assert float((lp.double() - z.gather(1, t.long()[:, None])[:, 0]).abs().max()) <= bound
    assert float((ent.double() + (z.exp() * z).sum(1)).abs().max()) <= bound
    assert float((tops[:, 0].double() - z.max(1).values).abs().max()) <= bound
    assert torch.equal(ids[:, 0].long(), (x[:, 1] > x[:, 0]).long())

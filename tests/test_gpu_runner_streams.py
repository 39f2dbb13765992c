"""The runners over a context on a stream of its own, called from another current stream with work before and behind them: results are those of a run on
one stream, bit for bit."""
import numpy as np
import pytest

from paper_2601_13155_amd import binding, runtime, synth
from tests.test_gpu_q4_edges import keep_busy
from tests.test_gpu_decode import torch  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu

SHAPE = synth.ModelShape(D=256, H=4, Hkv=2, d=64, Dff=688, dtype="bf16")


def contexts(torch):  # noqa: F811
    """On the default stream, then on one of its own."""
    yield runtime.make_context(SHAPE, 1024, 16, 16, SHAPE.Dff)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        ctx = binding.Context(SHAPE, 1024, 16, 16, SHAPE.Dff, stream=st)
    torch.cuda.synchronize()
    yield ctx


@pytest.fixture(scope="module")
def parts(torch):  # noqa: F811
    layers = [runtime.upload_layer(synth.make_layer(80, l, SHAPE, 16), SHAPE, 16) for l in range(3)]
    table = runtime.to_device(synth.vocab_table(81, 512, SHAPE.D, "bf16"), "bf16")
    gamma = torch.ones(SHAPE.D, dtype=torch.bfloat16, device="cuda")
    return layers, table, gamma


def filled(n, seed):
    c = runtime.KVCache(SHAPE, n + 8)
    c.k.copy_(runtime.to_device(np.random.default_rng(seed).standard_normal(c.k.shape), "bf16"))
    c.v.copy_(runtime.to_device(np.random.default_rng(seed + 1).standard_normal(c.v.shape), "bf16"))
    c.struct.count = n
    return c


@pytest.mark.parametrize("nseq", [0, 3])
def test_decode_on_a_side_stream(torch, parts, nseq):  # noqa: F811
    """DecodeRunner (nseq 0) and BatchedDecodeRunner."""
    layers, table, gamma = parts
    res = []
    for ctx in contexts(torch):
        caches = [[filled(30 + 9 * b, 90 + 10 * b + l) for l in range(3)] for b in range(max(nseq, 1))]
        run = runtime.BatchedDecodeRunner(ctx, SHAPE, layers, caches, gamma, table) if nseq else runtime.DecodeRunner(ctx, SHAPE, layers, caches[0], gamma, table)
        toks = torch.full((5,), -5, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        keep_busy(torch, torch.cuda.current_stream())
        run.x.copy_(table[7:7 + nseq] if nseq else table[7])
        keep_busy(torch, ctx.stream)
        if nseq:
            run.generate([40, 50, 60], 5)
        else:
            run.generate(40, 5, toks)
        got = [t.clone() for t in (run.x, run.logits, toks)]
        keep_busy(torch, torch.cuda.current_stream())
        run.x.copy_(table[11:11 + nseq] if nseq else table[11])
        run.step([45, 55, 65] if nseq else 45)
        got.append(run.x.clone())
        if not nseq:
            run.greedy()
            got += [run.token[:1].clone(), run.x_next.clone()]
        torch.cuda.synchronize()
        res.append([t.cpu() for t in got])
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_layer_and_channels_of_host_arrays_on_a_side_stream(torch, parts):  # noqa: F811
    """run_layer and select_proxy_channels upload and clear on the current stream."""
    x, res = synth.hidden_states(83, 200, SHAPE.D, "bf16"), []
    for ctx in contexts(torch):
        keep_busy(torch, torch.cuda.current_stream())
        out = runtime.run_layer(ctx, x, synth.positions(200), parts[0][0], SHAPE, skip=1, probe_len=16, m_attn=90, m_ffn=100, want_kv=True)
        keep_busy(torch, torch.cuda.current_stream())
        sel, imp = runtime.select_proxy_channels(ctx, parts[0][0], SHAPE, x, 20, 64)
        res.append([np.asarray(v) for _, v in sorted(out.items())] + [sel, imp])
    assert all(np.array_equal(a, b) for a, b in zip(*res))


@pytest.mark.parametrize("batched", [False, True])
def test_stacks_on_a_side_stream(torch, parts, batched):  # noqa: F811
    """StackRunner and BatchedStackRunner: positions and states are copied in behind a busy current stream."""
    layers, _, _ = parts
    lens = [200, 130] if batched else [300]
    plans = [synth.scaled(synth.WORKLOADS["c2"], shape=SHAPE, N=n, layers=3, stage_end_layers=(1, 2), probe_len=16, r=16, stage_cum_keep=(1.0, 0.7, 0.5)).layer_plan()
             for n in lens]
    src = runtime.to_device(synth.hidden_states(82, sum(lens), SHAPE.D, "bf16"), "bf16")
    pos = torch.from_numpy(np.concatenate([synth.positions(n) for n in lens])).cuda()
    res = []
    for ctx in contexts(torch):
        run = runtime.BatchedStackRunner(ctx, SHAPE, layers, plans, 16) if batched else runtime.StackRunner(ctx, SHAPE, layers, plans[0], 16, keep_trace=True)
        torch.cuda.synchronize()
        for _ in range(2):
            x0, p0 = torch.zeros_like(src), torch.zeros_like(pos)
            keep_busy(torch, torch.cuda.current_stream())
            x0.copy_(src)
            p0.copy_(pos)
            x, p, n = run.run(x0, p0)
            x0.zero_()
            got = [x.clone(), p.clone(), torch.tensor(n)] + ([] if batched else [t["x_out"] for t in run.trace])
        torch.cuda.synchronize()
        res.append([t.cpu() for t in got])
    assert all(torch.equal(a, b) for a, b in zip(*res))

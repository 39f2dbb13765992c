"""A batched decode step stays within its workspace where the heads have far more dimensions than the feed-forward block."""
import ctypes as C

import numpy as np
import pytest

from oracle import spts_oracle as orc
from paper_2601_13155_amd import binding, runtime, synth
from tests import helpers as H
from tests.test_gpu_decode import torch  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("nseq", [3, 16])
def test_batched_decode_of_many_head_dimensions(torch, dtype, nseq):  # noqa: F811
    """The fp32 sums of sixteen sequences' projections are larger than the hidden buffer; what lies behind the workspace is left, states are the oracle's."""
    shape = synth.ModelShape(D=64, H=32, Hkv=32, d=128, Dff=16, dtype=dtype)
    mdl, rnd, tol = H.oracle_model(shape), H.rnd_for(dtype), H.TOL[dtype]["hidden"]
    ctx = binding.Context(shape, 64, 1, 1, shape.Dff)
    ctx.close()
    nbytes, behind = ctx.workspace.numel(), 2 << 20
    ctx.workspace = torch.full((nbytes + behind,), 0xA5, dtype=torch.uint8, device="cuda")
    h = C.c_void_p()
    assert binding.load().spts_create(C.byref(h), C.byref(ctx.model), ctx.stream.cuda_stream, ctx.workspace.data_ptr(), nbytes, 64, 1, 1, shape.Dff) == binding.SPTS_OK
    ctx.handle = h
    w = synth.make_layer(5, 0, shape, 16)
    dw = runtime.upload_layer(w, shape, 16, pack=False)
    rng = np.random.default_rng(nseq)
    caches = []
    for b in range(nseq):
        c = runtime.KVCache(shape, 4 + 3 * b)
        for t in (c.k, c.v):
            t.copy_(runtime.to_device(rng.standard_normal(tuple(t.shape)).astype(np.float32), dtype))
        c.struct.count = 3 * b
        caches.append(c)
    before = [c.host() for c in caches]
    x = runtime.to_device(synth.hidden_states(6, nseq, shape.D, dtype), dtype)
    x_in, pos = runtime.to_host(x).astype(np.float64), [5 * b for b in range(nseq)]
    ctx.spts_decode_layer_batched(x, pos, dw, [c.struct for c in caches])
    torch.cuda.synchronize()
    assert (ctx.workspace[nbytes:] == 0xA5).all()
    got = runtime.to_host(x).astype(np.float64)
    for b in range(nseq):
        ref, _ = orc.decode_layer(x_in[b], pos[b], w, mdl, orc.LayerCache(*before[b]), rnd)
        assert H.row_rel_err(got[b][None], ref[None]) <= tol, b

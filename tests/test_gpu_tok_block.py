"""The operators over tokens one behind the other, as a block of a network uses them: the norms around the residual, the gated
feed-forward block and the norms behind it, forward and backward; and in front of an 8-bit product.

Nothing waits between the calls.  Every operator's outputs are held against its formula in 64 bits on the inputs that it was
given (the outputs of the one before), with the bounds of its own test; a captured graph has to give the same bits."""
import pytest
import torch

import test_gpu_tok_ffn as ffn
import test_gpu_tok_i8 as i8
import test_gpu_tok_norm as norm
from tok_util import DT, E32, U, Rand, ctx, matrix, within

pytestmark = pytest.mark.gpu


def replayed(run, outputs):
    """The calls captured and replayed twice over outputs full of something else: the same bits as before."""
    torch.cuda.synchronize()
    first = [t.clone() for t in outputs]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        run()
    for _ in range(2):
        for t in outputs:
            t.fill_(55)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
    for t, f in zip(outputs, first):
        assert torch.equal(t, f)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,D,F,gates", [(1, 64, 136, 0), (12, 264, 520, 3), (200, 1024, 1304, 5), (777, 520, 264, 0)])
def test_training_step_of_a_block(T, D, F, gates, dt):
    a, m, b = norm.setup(T, D, dt, gates, seed=1), ffn.setup(T, D, F, dt), norm.setup(T, D, dt, gates, seed=2)
    m["x"] = a["n"]                     # norm -> block
    b["r"], b["y"] = a["z"], m["y"]     # the residual stream and the block's output -> norm
    m["dy"] = b["dy"]                   # and back
    a["dz"], a["dn"] = b["dr"], m["dx"]
    spaces = [ctx().rtoss_block_norm_workspace(q["y"][0], gated=bool(gates)) for q in (a, b)]

    def run():
        norm.forward(a, T, "rms", "rms", gates)
        ffn.forward(m, "silu")
        norm.forward(b, T, "rms", "layer", gates)
        norm.backward(b, T, "rms", "layer", gates, ws=spaces[1])
        ffn.backward(m, "silu")
        norm.backward(a, T, "rms", "rms", gates, ws=spaces[0])

    run()
    refs = (norm.reference(a, T, D, "rms", "rms", gates, dt), ffn.reference(m, "silu", dt), norm.reference(b, T, D, "rms", "layer", gates, dt))
    norm.check(a, refs[0], norm.ALL)
    ffn.check(m, refs[1], ffn.BOTH)
    norm.check(b, refs[2], norm.ALL)
    get = lambda q, k: q[k][0] if isinstance(q[k], tuple) else q[k]   # noqa: E731
    replayed(run, [get(q, k) for q in (a, b) for k in norm.ALL if get(q, k) is not None] + [get(m, k) for k in ("gate", "up", "y") + ffn.BWD])


@pytest.mark.parametrize("dt", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("T,D,N", [(1, 256, 512), (16, 1000, 264), (300, 520, 1024)])
def test_norm_in_front_of_an_8_bit_product_with_the_residual(T, D, N, dt):
    a, td = norm.setup(T, D, dt, 0), DT[dt]
    w = Rand("w", T, D, N).normal(N, D, D ** -0.5)
    wq, ws = matrix((N, D), torch.int8)[0], torch.empty(N, device="cuda")
    xq, xs = matrix((T, D), torch.int8)[0], torch.empty(T, device="cuda")
    y, res = matrix((T, N), td)[0], matrix(Rand("r", T, N).normal(T, N).to(td), td)[0]
    ctx().rtoss_quantize_rows(w, wq, ws)

    def run():
        norm.forward(a, T, "rms", "rms", 0)
        ctx().rtoss_quantize_rows(a["n"][0], xq, xs)
        ctx().rtoss_matmul_i8(xq, xs, wq, ws, y, residual=res, residual_after_act=True)

    run()
    norm.check(a, norm.reference(a, T, D, "rms", "rms", 0, dt), ("z", "n"))
    for src, q, s in ((a["n"][0], xq, xs), (w, wq, ws)):
        want_q, want_s = i8.codes_of(src)
        assert torch.equal(q.cpu(), want_q) and torch.equal(s.cpu(), want_s)
    p = (xq.double() @ wq.double().T) * xs.double()[:, None] * ws.double()
    want = p + res.double()
    within(y, want, 8 * E32 * (p.abs() + res.double().abs()) + U[dt] * want.abs() + 2.0 ** -25, "y")     # (2^-25: half of fp16's last subnormal)
    replayed(run, [a["z"][0], a["n"][0], xq, xs, y])

"""Gated feed-forward block against its formulas in 64 bits.

Bounds, all in 64 bits: a sum of K products in fp32 is off by at most K * 2^-23 of the sum of their magnitudes (each addition
rounds, and the tensor cores may truncate: a whole step), the exponential and quotient of SiLU by less than 2^-20 of the
value; what passes through memory is rounded once (U).  |act'| <= 1.1 and |act''| <= 0.5 for SiLU; a ReLU whose argument is
within its error of 0 may fall on either side.
"""
import pytest
import torch

from paper_2303_02191_b200 import binding as rt
from tok_util import DT, E32, TINY, U, Rand, ctx, matrix, untouched, within

pytestmark = pytest.mark.gpu


def act_of(v, act):
    """value, slope, bound of the second derivative"""
    if act == "none":
        return v, torch.ones_like(v), 0.0
    if act == "relu":
        return v.clamp(min=0), (v > 0).double(), 0.0
    s = torch.sigmoid(v)
    return v * s, s * (1 + v * (1 - s)), 0.5


def setup(T, D, F, dt, pad=0, seed=0):
    r, td = Rand("ffn", T, D, F, seed), DT[dt]
    m = dict(x=matrix(r.normal(T, D).to(td), td, pad), wg=matrix(r.normal(F, D, D ** -0.5).to(td), td, pad),
             wu=matrix(r.normal(F, D, D ** -0.5).to(td), td, pad), wd=matrix(r.normal(D, F, F ** -0.5).to(td), td, pad),
             dy=matrix(r.normal(T, D).to(td), td, pad))
    for k, s in dict(h=(T, F), gate=(T, F), up=(T, F), dgate=(T, F), dup=(T, F), y=(T, D), dx=(T, D), dwg=(F, D), dwu=(F, D), dwd=(D, F)).items():
        m[k] = matrix(s, td, pad)
    return m


def forward(m, act, save=True, down=True):
    v = {k: t[0] for k, t in m.items()}
    ctx().rtoss_gated_ffn_forward(v["x"], v["wg"], v["wu"], v["wd"] if down else None, v["h"], v["y"] if down else None,
                                  gate=v["gate"] if save else None, up=v["up"] if save else None, act=rt.ACT_NAMES[act])


def backward(m, act, dgate="dgate", dup="dup", **out):
    v = {k: t[0] for k, t in m.items()}
    out = out or dict(dx=v["dx"], dw_gate=v["dwg"], dw_up=v["dwu"], dw_down=v["dwd"])
    ctx().rtoss_gated_ffn_backward(v["x"], v["wg"], v["wu"], v["wd"], v["gate"], v["up"], v["dy"], v["h"], v[dgate], v[dup],
                                   act=rt.ACT_NAMES[act], **out)


def reference(m, act, dt):
    """name -> (value, bound) in 64 bits"""
    u, tiny = U[dt], TINY[dt]
    x, wg, wu, wd, dy = (m[k][0].double() for k in ("x", "wg", "wu", "wd", "dy"))
    T, D = x.shape
    F = wg.shape[0]
    s32 = lambda k: k * 2 * E32   # noqa: E731
    g, up = x @ wg.T, x @ wu.T
    eg, eu = s32(D) * (x.abs() @ wg.abs().T), s32(D) * (x.abs() @ wu.abs().T)
    a, slope, bend = act_of(g, act)
    h = a * up
    ea = 1.1 * eg + 16 * E32 * a.abs()
    eh = (u + 4 * E32) * h.abs() + ea * up.abs() + a.abs() * eu + ea * eu + tiny
    y = h @ wd.T
    ref = dict(gate=(g, eg + u * g.abs() + tiny), up=(up, eu + u * up.abs() + tiny), h=(h, eh),
               y=(y, u * y.abs() + eh @ wd.abs().T + s32(F) * ((h.abs() + eh) @ wd.abs().T) + tiny))
    # backward, from the kept (rounded) projections
    eg, eu = eg + u * g.abs() + tiny, eu + u * up.abs() + tiny
    dh = dy @ wd
    edh = s32(D) * (dy.abs() @ wd.abs())
    eslope = bend * eg + 64 * E32 * (1 + g.abs()) * (0 if act == "none" else 1)
    if act == "relu":
        eslope = eslope + (g.abs() <= eg).double()
    dg, du = dh * up * slope, dh * a
    m1, m2, m3 = dh.abs() + edh, up.abs() + eu, slope.abs() + eslope
    edg = edh * m2 * m3 + m1 * eu * m3 + m1 * m2 * eslope + (u + 4 * E32) * dg.abs() + tiny
    edu = edh * (a.abs() + ea) + m1 * (1.1 * eg + 16 * E32 * a.abs()) + (u + 4 * E32) * du.abs() + tiny
    eh = (u + 4 * E32) * h.abs() + (1.1 * eg + 16 * E32 * a.abs()) * m2 + a.abs() * eu + tiny
    # h of the backward pass is act(g) * u of the kept g and u, each off by a rounding more: |act'| e_g |u| + |act| e_u and its own rounding
    ref["h_again"] = (h, eh)
    dx = dg @ wg + du @ wu
    edx = edg @ wg.abs() + edu @ wu.abs() + s32(2 * F) * ((dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs())
    ref["dx"] = (dx, u * dx.abs() + edx + tiny)
    for k, p, ep in (("dwg", dg, edg), ("dwu", du, edu)):
        w = p.T @ x
        ref[k] = (w, u * w.abs() + ep.T @ x.abs() + s32(T) * ((p.abs() + ep).T @ x.abs()) + tiny)
    w = dy.T @ h
    ref["dwd"] = (w, u * w.abs() + dy.abs().T @ eh + s32(T) * (dy.abs().T @ (h.abs() + eh)) + tiny)
    return ref


def check(m, ref, names):
    torch.cuda.synchronize()
    assert ctx().rtoss_device_status() == 0
    for k in names:
        at = m["h" if k == "h_again" else k]
        within(at[0], *ref[k], k)
        assert untouched(*at), k


FWD, BWD = ("gate", "up", "h", "y"), ("dx", "dwg", "dwu", "dwd")
BOTH = ("gate", "up", "y", "h_again") + BWD     # after both passes


# (tokens, D, F): one token, the few-token kernels and their border, one tile, several tiles, tiles cut along k, ragged
# everything, one feature
SHAPES = [(1, 64, 64), (1, 2048, 704), (3, 1, 1), (7, 200, 88), (8, 1000, 72), (9, 256, 24), (16, 520, 1304), (17, 520, 1304), (40, 75, 131),
          (128, 64, 64), (129, 512, 2050), (255, 1024, 264), (256, 72, 520), (257, 2056, 136), (600, 136, 1000), (1030, 264, 776)]


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,D,F", SHAPES)
def test_forward_and_backward(T, D, F, dt):
    act = ("silu", "relu", "none")[(T + D) % 3]
    m = setup(T, D, F, dt, pad=(T + F) % 3)
    ref = reference(m, act, dt)
    forward(m, act)
    check(m, ref, FWD)
    m["h"][0].fill_(5.0)     # the backward pass forms it again
    backward(m, act)
    check(m, ref, BWD + ("h_again",))


@pytest.mark.parametrize("act", ["silu", "relu", "none"])
@pytest.mark.parametrize("T", [5, 300])
def test_activations(T, act):
    m = setup(T, 136, 200, "bf16")
    ref = reference(m, act, "bf16")
    forward(m, act)
    backward(m, act)
    check(m, ref, BOTH)


@pytest.mark.parametrize("T", [2, 100])
def test_without_kept_projections_and_without_the_last_product(T):
    m = setup(T, 128, 320, "bf16")
    ref = reference(m, "silu", "bf16")
    forward(m, "silu", save=False)
    check(m, ref, ("h", "y"))
    assert bool((m["gate"][1] == 77.0).all()) and bool((m["up"][1] == 77.0).all())
    m["y"][0].fill_(77.0)
    m["h"][0].zero_()
    forward(m, "silu", down=False)
    check(m, ref, FWD[:3])
    assert bool((m["y"][1] == 77.0).all())


def test_gradients_that_are_not_asked_for_and_spent_projections():
    m = setup(90, 136, 264, "bf16", pad=1)
    ref = reference(m, "silu", "bf16")
    forward(m, "silu")
    backward(m, "silu", dw_up=m["dwu"][0])
    check(m, ref, ("dwu",))
    for k in ("dx", "dwg", "dwd"):
        assert bool((m[k][1] == 77.0).all()), k
    backward(m, "silu", dgate="gate", dup="up")     # the gradients of the projections take their place
    check(m, ref, BWD)


def test_gradients_agree_with_differences():
    """The directional derivative of sum(y * dy) along a random change of each operand, from two forward passes in 64 bits of the
    same formula at +- 1e-4: its own error is below 1e-6 of the magnitudes, far below the gradients' rounding."""
    m = setup(60, 64, 96, "f16")
    forward(m, "silu")
    backward(m, "silu")
    torch.cuda.synchronize()
    base = {k: m[k][0].double() for k in ("x", "wg", "wu", "wd")}
    dy = m["dy"][0].double()

    def loss(v):
        g = v["x"] @ v["wg"].T
        return ((g * torch.sigmoid(g) * (v["x"] @ v["wu"].T)) @ v["wd"].T * dy).sum()

    ref = reference(m, "silu", "f16")
    r = Rand("diff")
    for k, grad in (("x", "dx"), ("wg", "dwg"), ("wu", "dwu"), ("wd", "dwd")):
        step = r.normal(*base[k].shape).double()
        e = 1e-4
        slope = (loss({**base, k: base[k] + e * step}) - loss({**base, k: base[k] - e * step})) / (2 * e)
        got = (m[grad][0].double() * step).sum()
        bound = (ref[grad][1] * step.abs()).sum() + 1e-5 * (ref[grad][0] * step).abs().sum()
        assert abs(float(slope - got)) <= float(bound), k


def test_no_tokens():
    m = setup(0, 64, 96, "bf16")
    forward(m, "silu")
    backward(m, "silu")
    torch.cuda.synchronize()
    for k in ("dwg", "dwu", "dwd"):
        assert bool((m[k][0] == 0).all()) and untouched(*m[k]), k


def test_infinities_and_nan_stay_in_their_rows():
    for T in (4, 200):
        m = setup(T, 64, 128, "bf16")
        m["x"][0][1, 3] = float("nan")
        m["x"][0][2, 5] = float("inf")
        forward(m, "silu")
        torch.cuda.synchronize()
        y = m["y"][0]
        assert bool(torch.isnan(y[1]).all()) and not bool(torch.isfinite(y[2]).any())
        keep = [t for t in range(T) if t not in (1, 2)]
        assert bool(torch.isfinite(y[keep]).all())


@pytest.mark.parametrize("T", [1, 16, 300])
def test_same_bits_every_time_and_in_a_graph_on_another_stream(T):
    m = setup(T, 520, 1304, "bf16")
    forward(m, "silu")
    backward(m, "silu")
    torch.cuda.synchronize()
    names = FWD + BWD
    first = {k: m[k][0].clone() for k in names}
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            forward(m, "silu")
            backward(m, "silu")
        for _ in range(3):
            for k in names:
                m[k][0].fill_(77.0)
            graph.replay()
    side.synchronize()
    for k in names:
        assert torch.equal(m[k][0], first[k]), k
        assert untouched(*m[k])


def test_two_streams_at_once():
    a, b = setup(300, 264, 520, "bf16", seed=1), setup(310, 264, 520, "bf16", seed=2)
    refs = [reference(m, "silu", "bf16") for m in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for m, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                forward(m, "silu")
                backward(m, "silu")
    torch.cuda.synchronize()
    for m, ref in zip((a, b), refs):
        check(m, ref, BOTH)


@pytest.mark.parametrize("dt", ["bf16", "f16"])
@pytest.mark.parametrize("T,D,F", [(200, 1024, 2816), (100, 4096, 512), (300, 2048, 264), (40, 520, 4100)])
def test_products_cut_along_k(T, D, F, dt):
    """Few tiles and a long k: shares of k, exchanged between the CTAs of a cluster."""
    m = setup(T, D, F, dt, pad=T % 3)
    ref = reference(m, "silu", dt)
    forward(m, "silu")
    check(m, ref, FWD)
    backward(m, "silu")
    check(m, ref, BWD + ("h_again",))

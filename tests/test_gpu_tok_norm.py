"""Norms around the residual, forward and backward, against the formulas in 64 bits (autograd).

Bounds: a thread adds at most 16 squares one after the other (more only in rows of over 8192 values: a row's share of 512
threads), then a tree of 10: B = (terms + 48) * 2^-24 covers a sum, the root, the quotient and the products around it.  A
normalised value carries B of itself and, with a mean, of mean|t| / spread; a gradient's row terms carry 4 B of the
magnitudes that enter them; a sum over T tokens adds (T + 8) * 2^-24 of the sum of magnitudes."""
import pytest
import torch

from paper_2303_02191_b200 import binding as rt
from tok_util import DT, E32, TINY, U, Rand, ctx, matrix, untouched, within

pytestmark = pytest.mark.gpu

EPS = 1e-5


def setup(T, D, dt, gates, pad=0, align=16, seed=0):
    r, td = Rand("norm", T, D, gates, seed), DT[dt]
    mk = lambda rows, std=1.0, mean=0.0: matrix((r.normal(rows, D, std) + mean).to(td), td, pad, align)   # noqa: E731
    m = dict(r=mk(T), y=mk(T, 2.0, 0.5), dz=mk(T), dn=mk(T))
    for k in ("z", "n", "dr", "dy"):
        m[k] = matrix((T, D), td, pad, align)
    m["gate"] = mk(gates, 0.7) if gates else (None, None)
    m["dgate"] = matrix((gates, D), td, pad, align) if gates else (None, None)
    m["wpost"], m["wpre"] = 1 + 0.2 * r.normal(1, D)[0], 1 + 0.2 * r.normal(1, D)[0]
    m["dwpost"], m["dwpre"] = torch.full((D,), 77.0, device="cuda"), torch.full((D,), 77.0, device="cuda")
    return m


def call_args(m, T, post, pre, gates, scale):
    return dict(post=rt.NORM_NAMES[post], pre=rt.NORM_NAMES[pre], post_weight=m["wpost"] if post != "none" else None,
                pre_weight=m["wpre"] if pre != "none" else None, gate=m["gate"][0], tokens_per_gate=T // gates if gates else 0,
                residual_scale=scale, eps=EPS)


def forward(m, T, post, pre, gates, scale=0.75):
    ctx().rtoss_block_norm_forward(m["r"][0], m["y"][0], m["z"][0], m["n"][0] if pre != "none" else None, **call_args(m, T, post, pre, gates, scale))


def backward(m, T, post, pre, gates, scale=0.75, dz=True, dn=True, sums=True, ws=None):
    if ws is None:
        ws = ctx().rtoss_block_norm_workspace(m["y"][0], gated=bool(gates))
        ws.fill_(float("nan"))      # nothing in it is read before it is written
    more = dict(dpost_weight=m["dwpost"] if post != "none" else None, dpre_weight=m["dwpre"] if pre != "none" else None,
                dgate=m["dgate"][0], workspace=ws) if sums else {}
    ctx().rtoss_block_norm_backward(m["r"][0], m["y"][0], m["dz"][0] if dz else None, m["dn"][0] if dn and pre != "none" else None, m["dr"][0],
                                    m["dy"][0], **call_args(m, T, post, pre, gates, scale), **more)


def reference(m, T, D, post, pre, gates, dt, scale=0.75, dz=True, dn=True):
    u, tiny = U[dt], TINY[dt]
    B = ((16 if D <= 8192 else D // 512 + 1) + 48) * E32
    f = {k: m[k][0].double() for k in ("r", "y", "dz", "dn")}
    gate = m["gate"][0].double().repeat_interleave(T // gates, 0) if gates else torch.ones(T, D, dtype=torch.float64, device="cuda")
    wpost, wpre = m["wpost"].double(), m["wpre"].double()

    def norm(t, kind):
        """normalised rows, 1 / spread, mean|t| / spread"""
        if kind == "none":
            return t, torch.ones_like(t[:, :1]), torch.zeros_like(t[:, :1])
        c = t - t.mean(1, keepdim=True) if kind == "layer" else t
        rstd = 1 / (c.square().mean(1, keepdim=True) + EPS).sqrt()
        return c * rstd, rstd, (t.abs().mean(1, keepdim=True) * rstd if kind == "layer" else torch.zeros_like(rstd))

    yhat, yr, ya = norm(f["y"], post)
    w1 = wpost if post != "none" else torch.ones_like(wpost)
    v = yhat * w1
    z = scale * f["r"] + gate * v
    ehat = B * (yhat.abs() + ya) if post != "none" else 0 * yhat
    ez = gate.abs() * w1.abs() * ehat + 4 * E32 * ((scale * f["r"]).abs() + (gate * v).abs())
    ref = dict(z=(z, ez + u * z.abs() + tiny))
    zhat, zr, za = norm(z, pre)
    # an error of z goes into the row's spread with at most its mean square
    ezhat = (zr * (ez + ez.square().mean(1, keepdim=True).sqrt() * (1 + zhat.abs())) + B * (zhat.abs() + za)) if pre != "none" else 0 * zhat
    if pre != "none":
        ref["n"] = (zhat * wpre, wpre.abs() * ezhat + (u + 2 * E32) * (zhat * wpre).abs() + tiny)
    total = f["dz"] if dz else torch.zeros_like(z)
    etotal = E32 * total.abs()
    gn = f["dn"] * wpre if dn and pre != "none" else None
    mean = lambda t: t.mean(1, keepdim=True)   # noqa: E731
    if gn is not None:
        m0, m1 = mean(gn * zhat), mean(gn) if pre == "layer" else torch.zeros_like(zr)
        total = total + zr * (gn - zhat * m0 - m1)
        a0 = mean(gn.abs() * (zhat.abs() + ezhat))
        size = gn.abs() + zhat.abs() * a0 + mean(gn.abs())
        # zr is off by what ez and B make of it
        ezr = B + zr * ez.square().mean(1, keepdim=True).sqrt()
        etotal = etotal + zr * (4 * (B + ezr) * size + ezhat * a0 + (zhat.abs() + ezhat) * mean(gn.abs() * ezhat)) + 4 * E32 * total.abs()
    ref["dr"] = (scale * total, scale * etotal + (u + 2 * E32) * (scale * total).abs() + tiny)
    dv = total * gate
    edv = etotal * gate.abs() + 2 * E32 * dv.abs()
    if post != "none":
        gp, egp = dv * w1, edv * w1.abs() + 2 * E32 * (dv * w1).abs()
        p0, p1 = mean(gp * yhat), mean(gp) if post == "layer" else torch.zeros_like(yr)
        dy = yr * (gp - yhat * p0 - p1)
        a0, a1 = mean(gp.abs() * (yhat.abs() + ehat)), mean(gp.abs())
        size = gp.abs() + yhat.abs() * a0 + a1
        edy = yr * (8 * B * size + egp + yhat.abs() * mean(egp * yhat.abs()) + mean(egp) + ehat * a0 + (yhat.abs() + ehat) * mean(gp.abs() * ehat))
        ref["dwpost"] = ((dv * yhat).sum(0), (edv * (yhat.abs() + ehat) + dv.abs() * ehat + (T + 8) * E32 * (dv * yhat).abs()).sum(0))
        if T > 1:
            ref["dwpost"] = (ref["dwpost"][0], ref["dwpost"][1] + T * E32 * (dv * yhat).abs().sum(0))
    else:
        dy, edy = dv, edv
    ref["dy"] = (dy, edy + (u + 2 * E32) * dy.abs() + tiny)
    if pre != "none":
        d = f["dn"] if gn is not None else torch.zeros_like(z)
        ref["dwpre"] = ((d * zhat).sum(0), (d.abs() * ezhat).sum(0) + (2 * T + 8) * E32 * (d * zhat).abs().sum(0))
    if gates:
        S = T // gates
        p = (total * v).reshape(gates, S, D)
        e = (etotal * (v.abs() + w1.abs() * ehat) + total.abs() * w1.abs() * ehat).reshape(gates, S, D)
        ref["dgate"] = (p.sum(1), e.sum(1) + (2 * S + 8) * E32 * p.abs().sum(1) + u * p.sum(1).abs() + tiny)
    return ref


def check(m, ref, names):
    torch.cuda.synchronize()
    for k in names:
        if k not in ref:
            continue
        t = m[k][0] if isinstance(m[k], tuple) else m[k]
        within(t, *ref[k], k)
        if isinstance(m[k], tuple):
            assert untouched(*m[k]), k


ALL = ("z", "n", "dr", "dy", "dwpost", "dwpre", "dgate")

# (tokens, D, gates): every kernel (rows up to 256, 1024, 2048, 4096, 8192 and longer), rows that are no multiple of eight,
# gates of one token, of some, of all; tokens beyond what the units take at once
SHAPES = [(1, 1, 0), (1, 2048, 1), (2, 8, 2), (5, 100, 0), (64, 256, 64), (3000, 64, 0), (9000, 24, 30), (7, 257, 1), (700, 1000, 7), (1500, 1024, 0),
          (3, 1025, 0), (640, 2048, 5), (333, 2040, 0), (4, 4096, 2), (300, 3001, 3), (2, 8192, 0), (310, 8192, 31), (5, 8200, 5), (300, 9001, 3), (151, 20000, 0)]


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,D,gates", SHAPES)
def test_forward_and_backward(T, D, gates, dt):
    kinds = ("rms", "layer", "none")
    post, pre = kinds[(T + D) % 3], kinds[(T + 2 * D) % 3]
    if D == 1:
        post, pre = "rms", "rms"      # (one value less its mean is nothing)
    m = setup(T, D, dt, gates, pad=(T + D) % 2)
    ref = reference(m, T, D, post, pre, gates, dt)
    forward(m, T, post, pre, gates)
    backward(m, T, post, pre, gates)
    check(m, ref, ALL)


@pytest.mark.parametrize("pre", ["none", "rms", "layer"])
@pytest.mark.parametrize("post", ["none", "rms", "layer"])
def test_kinds_of_norm(post, pre):
    for dt, D in (("f32", 96), ("bf16", 1536)):
        m = setup(50, D, dt, 5)
        ref = reference(m, 50, D, post, pre, 5, dt)
        forward(m, 50, post, pre, 5)
        backward(m, 50, post, pre, 5)
        check(m, ref, ALL)


def test_one_of_the_two_gradients_and_no_sums():
    for dz, dn in ((True, False), (False, True)):
        m = setup(40, 512, "bf16", 0)
        ref = reference(m, 40, 512, "rms", "layer", 0, "bf16", dz=dz, dn=dn)
        backward(m, 40, "rms", "layer", 0, dz=dz, dn=dn, sums=False)
        check(m, ref, ("dr", "dy"))
        assert bool((m["dwpost"] == 77.0).all())
        backward(m, 40, "rms", "layer", 0, dz=dz, dn=dn)
        check(m, ref, ("dr", "dy", "dwpost", "dwpre"))


@pytest.mark.parametrize("S", [1, 3, 7, 50, 1000, 3000])
def test_gates_that_run_across_units(S):
    T = 6000 // S * S
    m = setup(T, 40, "f32", T // S)
    ref = reference(m, T, 40, "rms", "rms", T // S, "f32")
    forward(m, T, "rms", "rms", T // S)
    backward(m, T, "rms", "rms", T // S)
    check(m, ref, ALL)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_rows_that_start_anywhere(dt):
    """Odd row strides and a base off every boundary."""
    T, D, td = 30, 120, DT[dt]
    m = setup(T, D, dt, 2)
    for k in ("r", "y", "dz", "dn", "z", "n", "dr", "dy", "gate", "dgate"):
        src = m[k][0]
        buf = torch.full(((src.shape[0] + 2) * (D + 3) + 1,), 77.0, device="cuda").to(td)
        whole = buf[1:].reshape(-1, D + 3)
        whole[:src.shape[0], :D].copy_(src)
        m[k] = (whole[:src.shape[0], :D], whole)
    ref = reference(m, T, D, "layer", "rms", 2, dt)
    forward(m, T, "layer", "rms", 2)
    backward(m, T, "layer", "rms", 2)
    check(m, ref, ALL)


@pytest.mark.parametrize("D", [300, 9000])
def test_in_place(D):
    m = setup(20, D, "bf16", 0)
    ref = reference(m, 20, D, "rms", "rms", 0, "bf16")
    r, y = m["r"][0].clone(), m["y"][0].clone()
    args = call_args(m, 20, "rms", "rms", 0, 0.75)
    ctx().rtoss_block_norm_forward(r, y, r, y, **args)
    check(dict(z=r, n=y), ref, ("z", "n"))
    dz, dn = m["dz"][0].clone(), m["dn"][0].clone()
    ctx().rtoss_block_norm_backward(m["r"][0], m["y"][0], dz, dn, dz, dn, **args)
    check(dict(dr=dz, dy=dn), ref, ("dr", "dy"))


def test_rows_of_zeros_and_rows_with_nan():
    m = setup(6, 64, "f32", 0)
    m["y"][0][2] = 0
    m["r"][0][2] = 0
    m["y"][0][4, 5] = float("nan")
    ref = reference(m, 6, 64, "rms", "rms", 0, "f32")
    forward(m, 6, "rms", "rms", 0)
    torch.cuda.synchronize()
    assert bool((m["z"][0][2] == 0).all()) and bool((m["n"][0][2] == 0).all())
    keep = [0, 1, 2, 3, 5]
    assert bool(torch.isnan(m["z"][0][4]).all())
    for k in ("z", "n"):
        within(m[k][0][keep], ref[k][0][keep], ref[k][1][keep], k)


def test_no_tokens():
    m = setup(0, 64, "bf16", 0)
    forward(m, 0, "rms", "rms", 0)
    backward(m, 0, "rms", "rms", 0)
    torch.cuda.synchronize()
    assert bool((m["dwpost"] == 0).all()) and bool((m["dwpre"] == 0).all())


def test_same_bits_every_time_and_in_graphs_with_their_own_workspaces():
    T, D = 1000, 1000
    m = setup(T, D, "bf16", 4)
    m2 = dict(m, dr=matrix((T, D), DT["bf16"]), dy=matrix((T, D), DT["bf16"]), dwpost=torch.zeros(D, device="cuda"), dwpre=torch.zeros(D, device="cuda"),
              dgate=matrix((4, D), DT["bf16"]))
    backward(m, T, "rms", "layer", 4)
    torch.cuda.synchronize()
    names = ("dr", "dy", "dwpost", "dwpre", "dgate")
    get = lambda q, k: q[k][0] if isinstance(q[k], tuple) else q[k]   # noqa: E731
    first = {k: get(m, k).clone() for k in names}
    graphs, side = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for q, s in zip((m, m2), side):
        ws = ctx().rtoss_block_norm_workspace(q["y"][0], gated=True)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            backward(q, T, "rms", "layer", 4, ws=ws)
        graphs.append((g, s, ws))
    for _ in range(3):
        for g, s, _ws in graphs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for q in (m, m2):
        for k in names:
            assert torch.equal(get(q, k), first[k]), k


# D of every way that rows are dealt out: units of 8, 16 and 32 threads, blocks that are not full, two pieces a thread; rows enough
# for several to a unit, with gates that begin and end inside blocks
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,D,gates", [(9000, 64, 18), (4100, 72, 0), (5000, 128, 10), (9000, 200, 9), (4900, 264, 7), (2000, 648, 0), (1800, 1280, 6), (800, 2056, 2),
                                       (900, 2560, 30), (333, 4104, 0), (400, 5000, 5)])
def test_rows_of_every_length(T, D, gates, dt):
    kinds = ("rms", "layer", "none")
    post, pre = kinds[(T // 100 + D) % 2], kinds[D // 8 % 3]
    m = setup(T, D, dt, gates)
    ref = reference(m, T, D, post, pre, gates, dt)
    forward(m, T, post, pre, gates)
    backward(m, T, post, pre, gates)
    check(m, ref, ALL)
    assert ctx().rtoss_device_status() == 0


def test_weights_that_start_anywhere():
    T, D = 40, 512
    m = setup(T, D, "bf16", 0)
    for k in ("wpost", "wpre"):
        m[k] = torch.cat([torch.zeros(1, device="cuda"), m[k]])[1:]
    ref = reference(m, T, D, "rms", "layer", 0, "bf16")
    forward(m, T, "rms", "layer", 0)
    backward(m, T, "rms", "layer", 0)
    check(m, ref, ALL)

"""Operators of transformer blocks over tokens (or over the positions of a channels-last map), as a user's program calls
them, with their plain forms.

Three kinds of work:
  i8    tokens in 16 or 32 bits are quantised row by row and multiplied with 8-bit weights: a scale for each token and
        for each output channel, bias, activation and a residual operand in the same pass
  ffn   a gated feed-forward block h = act(x Wg^T) * (x Wu^T), y = h Wd^T; with train also its whole backward pass
  norm  z = residual_scale * r + gate * norm(y), n = norm(z): the norms behind one block and in front of the next, with
        the gate and the residual between them; with train also the backward pass

`listed()` holds the fixed cases, `draw()` gives more of the same ranges.  Where `own` is false, `run` computes in plain
fp32 torch operations.
"""
import math

import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def listed():
    i8 = dict(kind="i8", bias=False, residual="none", act="none", dtype="bf16")
    ffn = dict(kind="ffn", act="silu", dtype="bf16", train=False)
    norm = dict(kind="norm", post="rms", pre="rms", gate="none", S=1, dtype="bf16", train=False)
    return [
        # serving one token at a time: 16 MB of weights, latency and bandwidth decide
        dict(i8, name="i8_one_token", T=1, K=4096, N=4096),
        # a 1x1 layer of a detector on eight 80x80 maps: thin channels, many positions
        dict(i8, name="i8_map_positions", T=51200, K=128, N=128, bias=True, act="silu"),
        # sizes that are multiples of nothing, fp16, everything the epilogue does
        dict(i8, name="i8_ragged", T=331, K=1003, N=1001, bias=True, act="relu", residual="before", dtype="f16"),
        # a prompt, or a batch of frames' tokens, through a wide projection
        dict(i8, name="i8_large", T=8192, K=4096, N=8192),
        # one token through the block: three weight matrices are read once
        dict(ffn, name="ffn_one_token", T=1, D=2048, F=5632),
        # a batch of requests decoded together, not a multiple of any tile, fp16
        dict(ffn, name="ffn_200_tokens", T=200, D=1024, F=2816, dtype="f16"),
        # a long prompt: the largest products
        dict(ffn, name="ffn_prompt", T=8192, D=2048, F=8192),
        # one training step's block: all gradients
        dict(ffn, name="ffn_train", T=4096, D=2048, F=5632, train=True),
        # training on what a ragged batch leaves, with ReLU, fp16
        dict(ffn, name="ffn_train_ragged", T=777, D=520, F=1304, act="relu", dtype="f16", train=True),
        # one token between two blocks: launch latency
        dict(norm, name="norm_one_token", T=1, D=2048),
        # a long prompt between two blocks: bandwidth
        dict(norm, name="norm_prompt", T=16384, D=2048),
        # training with a gate per sample (eight samples), norms of both kinds
        dict(norm, name="norm_train", T=8192, D=2048, gate="sample", S=1024, pre="layer", train=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {"i8": max(2.0 * c["T"] * c["K"] * c["N"] for c in listed() if c["kind"] == "i8"),
            "ffn": max(work(c)["flops"] for c in listed() if c["kind"] == "ffn"),
            "norm": max(work(c)["bytes"] for c in listed() if c["kind"] == "norm")}
    kind = rng.choice(["i8", "i8", "ffn", "ffn", "norm", "norm"])
    while True:
        if kind == "i8":
            c = dict(kind=kind, T=_log_int(rng, 1, 51200), K=_log_int(rng, 32, 8192), N=_log_int(rng, 32, 8192),
                     bias=rng.random() < 0.5, act=rng.choice(["none", "silu", "relu"]),
                     residual=rng.choice(["none", "none", "before", "after"]), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]))
            if rng.random() < 0.6:      # most layers are multiples of 16
                c["K"], c["N"] = max(16, c["K"] // 16 * 16), max(16, c["N"] // 16 * 16)
            if work(c)["flops"] <= most[kind] and work(c)["bytes"] <= 4e8:
                return c
        elif kind == "ffn":
            c = dict(kind=kind, T=_log_int(rng, 1, 8192), D=8 * _log_int(rng, 8, 512), F=8 * _log_int(rng, 8, 1408),
                     act=rng.choice(["silu", "silu", "relu", "none"]), dtype=rng.choice(["bf16", "bf16", "f16"]),
                     train=rng.random() < 0.5)
            if work(c)["flops"] <= most[kind]:
                return c
        else:
            c = dict(kind=kind, T=_log_int(rng, 1, 16384), D=_log_int(rng, 64, 8192), post=rng.choice(["rms", "rms", "layer", "none"]),
                     pre=rng.choice(["rms", "rms", "layer", "none"]), gate=rng.choice(["none", "channel", "sample"]), S=1,
                     dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), train=rng.random() < 0.5)
            if rng.random() < 0.6:
                c["D"] = max(64, c["D"] // 64 * 64)
            if c["gate"] == "sample":   # S tokens share a gate
                c["S"] = _log_int(rng, 1, c["T"])
                c["T"] = c["S"] * max(1, c["T"] // c["S"])
            if work(c)["bytes"] <= most[kind]:
                return c


# ---- inputs ---------------------------------------------------------------------------------------------------

class _Rand:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed))

    def normal(self, shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=self.g).to(dtype)


def _padded(rows, cols, dtype, to=16):
    """[rows, cols] whose rows start on 16-byte boundaries."""
    unit = to // torch.empty(0, dtype=dtype).element_size()
    return torch.zeros(rows, (cols + unit - 1) // unit * unit, dtype=dtype, device="cuda")[:, :cols]


def prepare(case, seed):
    rand, td, T = _Rand(seed), DTYPE[case["dtype"]], case["T"]
    if case["kind"] == "i8":
        K, N = case["K"], case["N"]
        x = rand.normal((T, K))
        x[:, ::97] *= 12.0                                  # a few channels stand out, as they do in trained networks
        w = rand.normal((N, K), 1.0 / math.sqrt(K))
        ws = w.abs().amax(dim=1) / 127.0                    # the weights are quantised once, when the model is loaded
        wq = _padded(N, K, torch.int8)
        wq.copy_((w / ws[:, None]).round().clamp(-127, 127))
        y = _padded(T, N, td)
        res = _padded(T, N, td)
        if case["residual"] != "none":
            res.copy_(rand.normal((T, N)))
        return dict(case=case, x=x.to(td), wq=wq, ws=ws, bias=rand.normal((N,), 0.1) if case["bias"] else None,
                    residual=res if case["residual"] != "none" else None, y=y, xq=_padded(T, K, torch.int8),
                    xs=torch.empty(T, dtype=torch.float32, device="cuda"))
    D = case["D"]
    new = lambda *shape, dtype=td: torch.empty(shape, dtype=dtype, device="cuda")   # noqa: E731
    if case["kind"] == "ffn":
        F = case["F"]
        s = dict(case=case, x=rand.normal((T, D), 1.0, td), wg=rand.normal((F, D), 1.0 / math.sqrt(D), td),
                 wu=rand.normal((F, D), 1.0 / math.sqrt(D), td), wd=rand.normal((D, F), 1.0 / math.sqrt(F), td),
                 h=new(T, F), y=new(T, D), gate=None, up=None)
        if case["train"]:
            s.update(dy=rand.normal((T, D), 1.0, td), gate=new(T, F), up=new(T, F), dgate=new(T, F), dup=new(T, F),
                     dx=new(T, D), dwg=new(F, D), dwu=new(F, D), dwd=new(D, F))
        return s
    G = {"none": 0, "channel": 1, "sample": T // case["S"]}[case["gate"]]
    weight = lambda kind: 1.0 + rand.normal((D,), 0.1) if kind != "none" else None   # noqa: E731
    s = dict(case=case, r=rand.normal((T, D), 1.0, td), y=(rand.normal((T, D)) * 2.0 + 0.3).to(td), z=new(T, D),
             n=new(T, D) if case["pre"] != "none" else None, wpost=weight(case["post"]), wpre=weight(case["pre"]),
             gate=rand.normal((G, D), 0.5, td) if G else None, scale=0.8, S=case["S"] if G > 1 else T)
    if case["train"]:
        s.update(dz=rand.normal((T, D), 1.0, td), dn=rand.normal((T, D), 1.0, td) if s["n"] is not None else None,
                 dr=new(T, D), dy=new(T, D), dwpost=new(D, dtype=torch.float32) if s["wpost"] is not None else None,
                 dwpre=new(D, dtype=torch.float32) if s["wpre"] is not None else None, dgate=new(G, D) if G else None, work=None)
    return s


# ---- one pass -------------------------------------------------------------------------------------------------

_CTX = []


def _ctx():
    """The one context a program keeps per device."""
    if not _CTX:
        from paper_2303_02191_b200 import binding as rt
        _CTX.append((rt, rt.Context(0)))
    return _CTX[0]


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"i8": _own_i8, "ffn": _own_ffn, "norm": _own_norm}[kind](state)
    return {"i8": _plain_i8, "ffn": _plain_ffn, "norm": _plain_norm}[kind](state)


def _own_i8(s):
    rt, ctx = _ctx()
    c = s["case"]
    ctx.rtoss_quantize_rows(s["x"], s["xq"], s["xs"])
    return ctx.rtoss_matmul_i8(s["xq"], s["xs"], s["wq"], s["ws"], s["y"], act=rt.ACT_NAMES[c["act"]], bias=s["bias"],
                               residual=s["residual"], residual_after_act=c["residual"] == "after")


def _own_ffn(s):
    rt, ctx = _ctx()
    act = rt.ACT_NAMES[s["case"]["act"]]
    ctx.rtoss_gated_ffn_forward(s["x"], s["wg"], s["wu"], s["wd"], s["h"], s["y"], gate=s["gate"], up=s["up"], act=act)
    if not s["case"]["train"]:
        return s["y"]
    ctx.rtoss_gated_ffn_backward(s["x"], s["wg"], s["wu"], s["wd"], s["gate"], s["up"], s["dy"], s["h"], s["dgate"], s["dup"],
                                 dx=s["dx"], dw_gate=s["dwg"], dw_up=s["dwu"], dw_down=s["dwd"], act=act)
    return s["y"], s["dx"], s["dwg"], s["dwu"], s["dwd"]


def _own_norm(s):
    rt, ctx = _ctx()
    post, pre = rt.NORM_NAMES[s["case"]["post"]], rt.NORM_NAMES[s["case"]["pre"]]
    ctx.rtoss_block_norm_forward(s["r"], s["y"], s["z"], s["n"], post=post, pre=pre, post_weight=s["wpost"], pre_weight=s["wpre"],
                                 gate=s["gate"], tokens_per_gate=s["S"], residual_scale=s["scale"], eps=EPS)
    out = [s["z"]] if s["n"] is None else [s["z"], s["n"]]
    if not s["case"]["train"]:
        return out
    if s["work"] is None:       # a program keeps its workspace
        s["work"] = ctx.rtoss_block_norm_workspace(s["y"], gated=s["gate"] is not None)
    ctx.rtoss_block_norm_backward(s["r"], s["y"], s["dz"], s["dn"], s["dr"], s["dy"], post=post, pre=pre, post_weight=s["wpost"],
                                  pre_weight=s["wpre"], gate=s["gate"], tokens_per_gate=s["S"], residual_scale=s["scale"], eps=EPS,
                                  dpost_weight=s["dwpost"], dpre_weight=s["dwpre"], dgate=s["dgate"], workspace=s["work"])
    return out + [s["dr"], s["dy"]] + [s[k] for k in ("dwpost", "dwpre", "dgate") if s[k] is not None]


def _act(v, act):
    return v if act == "none" else v.clamp(min=0) if act == "relu" else v / (1.0 + torch.exp(-v))


def _act_and_slope(v, act):
    if act == "none":
        return v, torch.ones_like(v)
    if act == "relu":
        return v.clamp(min=0), (v > 0).to(v.dtype)
    sg = 1.0 / (1.0 + torch.exp(-v))
    return v * sg, sg * (1.0 + v * (1.0 - sg))


def _plain_i8(s):
    c, x = s["case"], s["x"].float()
    xs = x.abs().amax(dim=1, keepdim=True) / 127.0
    xq = torch.where(xs > 0, x / xs, 0.0).round().clamp(-127, 127)
    y = (xq @ s["wq"].float().T) * xs * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if c["residual"] == "before":
        y = y + s["residual"].float()
    y = _act(y, c["act"])
    if c["residual"] == "after":
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _plain_ffn(s):
    act, td = s["case"]["act"], s["x"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    g, u = x @ wg.T, x @ wu.T
    a, slope = _act_and_slope(g, act)
    h = a * u
    y = h @ wd.T
    if not s["case"]["train"]:
        return y.to(td)
    dy = s["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    dx = dg @ wg + du @ wu
    return y.to(td), dx.to(td), (dg.T @ x).to(td), (du.T @ x).to(td), (dy.T @ h).to(td)


def _norm(v, kind):
    """(normalised rows, 1 / root of the mean square)"""
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    rstd = 1.0 / torch.sqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    return v * rstd, rstd


def _norm_back(g, hat, rstd, kind):
    if kind == "layer":
        g = g - g.mean(dim=1, keepdim=True)
    return rstd * (g - hat * (g * hat).mean(dim=1, keepdim=True))


def _plain_norm(s):
    c, td = s["case"], s["y"].dtype
    T, D = s["y"].shape
    y, r = s["y"].float(), s["r"].float()
    gate = s["gate"].float().repeat_interleave(s["S"], dim=0) if s["gate"] is not None else None
    yhat, yrstd = _norm(y, c["post"]) if c["post"] != "none" else (y, None)
    v = yhat * s["wpost"] if s["wpost"] is not None else yhat
    z = s["scale"] * r + (v * gate if gate is not None else v)
    out = [z.to(td)]
    if c["pre"] != "none":
        zhat, zrstd = _norm(z, c["pre"])
        out.append((zhat * s["wpre"]).to(td))
    if not c["train"]:
        return out
    total, sums = s["dz"].float(), []
    if c["pre"] != "none":
        dn = s["dn"].float()
        total = total + _norm_back(dn * s["wpre"], zhat, zrstd, c["pre"])
    dv = total * gate if gate is not None else total
    if c["post"] != "none":
        dy = _norm_back(dv * s["wpost"], yhat, yrstd, c["post"])
        sums.append((dv * yhat).sum(dim=0))
    else:
        dy = dv
    if c["pre"] != "none":
        sums.append((dn * zhat).sum(dim=0))
    if gate is not None:
        sums.append((total * v).reshape(-1, s["S"], D).sum(dim=1).to(td))
    return out + [(s["scale"] * total).to(td), dy.to(td)] + sums


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    e, T = 4 if case["dtype"] == "f32" else 2, case["T"]
    if case["kind"] == "i8":
        K, N = case["K"], case["N"]
        reads = T * K * e + N * K + 4 * N + (4 * N if case["bias"] else 0) + (T * N * e if case["residual"] != "none" else 0)
        return {"bytes": reads + T * N * e, "flops": 2.0 * T * K * N}
    D = case["D"]
    if case["kind"] == "ffn":
        F = case["F"]
        if case["train"]:   # x, dy, y, dx once, the weights and their gradients once
            return {"bytes": (4.0 * T * D + 6.0 * D * F) * e, "flops": 18.0 * T * D * F}
        return {"bytes": (2.0 * T * D + 3.0 * D * F) * e, "flops": 6.0 * T * D * F}
    G = {"none": 0, "channel": 1, "sample": T // case["S"]}[case["gate"]]
    pre = case["pre"] != "none"
    bytes_ = (3 + pre) * T * D * e + G * D * e
    if case["train"]:       # r and y are read again: the backward pass is another call
        bytes_ += (5 + pre) * T * D * e + 2 * G * D * e
    return {"bytes": float(bytes_), "flops": (30.0 if case["train"] else 10.0) * T * D}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    f64 = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    sigma = lambda t: torch.special.expit(t)   # noqa: E731
    phi = {"none": lambda t: t, "relu": lambda t: torch.maximum(t, torch.zeros_like(t)), "silu": lambda t: t * sigma(t)}[case["act"]] if "act" in case else None
    if case["kind"] == "i8":
        x = f64["x"]
        top = x.abs().max(dim=1).values
        step = (top / 127.0).float().double()                # a scale is held in 32 bits
        codes = torch.zeros_like(x)
        live = step > 0
        codes[live] = torch.round(x[live] / step[live].unsqueeze(1))
        t = torch.einsum("tk,nk->tn", codes, s["wq"].double()) * torch.outer(step, f64["ws"])
        if case["bias"]:
            t = t + f64["bias"].unsqueeze(0)
        if case["residual"] == "before":
            return phi(t + f64["residual"])
        return phi(t) + f64["residual"] if case["residual"] == "after" else phi(t)
    if case["kind"] == "ffn":
        x, wg, wu, wd = f64["x"], f64["wg"], f64["wu"], f64["wd"]
        if not case["train"]:
            return torch.einsum("tf,df->td", phi(torch.einsum("td,fd->tf", x, wg)) * torch.einsum("td,fd->tf", x, wu), wd)
        x, wg, wu, wd = (t.requires_grad_(True) for t in (x, wg, wu, wd))
        y = torch.matmul(phi(torch.matmul(x, wg.t())) * torch.matmul(x, wu.t()), wd.t())
        grads = torch.autograd.grad(y, (x, wg, wu, wd), f64["dy"])
        return (y.detach(),) + grads
    leaves = {k: f64[k].requires_grad_(True) for k in ("r", "y", "wpost", "wpre", "gate") if k in f64}

    def normed(t, kind, weight):
        if kind == "none":
            return t
        centre = t.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(t[:, :1])
        spread = torch.sqrt(((t - centre) ** 2).sum(1, keepdim=True) / t.shape[1] + EPS)
        return (t - centre) / spread * weight

    v = normed(leaves["y"], case["post"], leaves.get("wpost"))
    if "gate" in leaves:
        v = (v.reshape(leaves["gate"].shape[0], -1, v.shape[1]) * leaves["gate"].unsqueeze(1)).reshape(v.shape)
    z = s["scale"] * leaves["r"] + v
    outs, seeds = [z], [f64.get("dz")]
    if case["pre"] != "none":
        outs.append(normed(z, case["pre"], leaves.get("wpre")))
        seeds.append(f64.get("dn"))
    if not case["train"]:
        return [t.detach() for t in outs]
    order = [k for k in ("r", "y", "wpost", "wpre", "gate") if k in leaves]
    grads = torch.autograd.grad(outs, [leaves[k] for k in order], seeds)
    return [t.detach() for t in outs] + list(grads)

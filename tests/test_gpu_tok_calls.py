"""The Python calls of the operators over tokens: what they refuse, and that the extension module and the checks in Python make the
same call."""
import pytest
import torch

from paper_2303_02191_b200 import binding as rt
from tok_util import Rand, ctx

pytestmark = pytest.mark.gpu
T, D, F = 20, 64, 96


def operands():
    r, b = Rand("calls"), torch.bfloat16
    new = lambda *s, dtype=b: torch.empty(s, dtype=dtype, device="cuda")   # noqa: E731
    q = lambda *s: r.normal(*s, 40).to(torch.int8)   # noqa: E731
    v = lambda n: 1 + 0.1 * r.normal(1, n)[0]   # noqa: E731
    m = dict(x=r.normal(T, D).to(b), wg=r.normal(F, D, 0.1).to(b), wu=r.normal(F, D, 0.1).to(b), wd=r.normal(D, F, 0.1).to(b), dy=r.normal(T, D).to(b))
    c = ctx()
    return {
        "quantize": (c.rtoss_quantize_rows, dict(x=m["x"], q=new(T, D, dtype=torch.int8), scale=new(T, dtype=torch.float32)), ("q", "scale")),
        "matmul": (c.rtoss_matmul_i8, dict(x=q(T, D), x_scale=v(T), w=q(F, D), w_scale=v(F), y=new(T, F), bias=v(F), residual=r.normal(T, F).to(b)), ("y",)),
        "ffn": (c.rtoss_gated_ffn_forward, dict(x=m["x"], w_gate=m["wg"], w_up=m["wu"], w_down=m["wd"], h=new(T, F), y=new(T, D), gate=new(T, F), up=new(T, F)),
                ("h", "y", "gate", "up")),
        "ffn_back": (c.rtoss_gated_ffn_backward, dict(x=m["x"], w_gate=m["wg"], w_up=m["wu"], w_down=m["wd"], gate=r.normal(T, F).to(b), up=r.normal(T, F).to(b), dy=m["dy"],
                                                      h=new(T, F), dgate=new(T, F), dup=new(T, F), dx=new(T, D), dw_gate=new(F, D), dw_up=new(F, D), dw_down=new(D, F)),
                     ("h", "dgate", "dup", "dx", "dw_gate", "dw_up", "dw_down")),
        "norm": (c.rtoss_block_norm_forward, dict(r=m["x"], y=m["dy"], z=new(T, D), n=new(T, D), post_weight=v(D), pre_weight=v(D), gate=r.normal(4, D).to(b),
                                                  tokens_per_gate=5, residual_scale=0.5), ("z", "n")),
        "norm_back": (c.rtoss_block_norm_backward, dict(r=m["x"], y=m["dy"], dz=m["dy"], dn=m["x"], dr=new(T, D), dy=new(T, D), post_weight=v(D), pre_weight=v(D),
                                                        gate=r.normal(4, D).to(b), tokens_per_gate=5, residual_scale=0.5, dpost_weight=new(D, dtype=torch.float32),
                                                        dpre_weight=new(D, dtype=torch.float32), dgate=new(4, D), workspace=c.rtoss_block_norm_workspace(m["x"], gated=True)),
                      ("dr", "dy", "dpost_weight", "dpre_weight", "dgate")),
    }


NAMES = ("quantize", "matmul", "ffn", "ffn_back", "norm", "norm_back")


@pytest.fixture
def in_python(monkeypatch):
    """The checks in Python instead of the extension module."""
    rt._types()
    monkeypatch.setattr(rt, "_calls", None)


def call(name):
    f, args, outs = operands()[name]
    f(**args)
    torch.cuda.synchronize()
    return [args[k] for k in outs]


@pytest.mark.parametrize("name", NAMES)
def test_both_ways_make_the_same_call(name, monkeypatch):
    rt._types()
    assert rt._calls is not None        # built for this interpreter and torch
    native = call(name)
    monkeypatch.setattr(rt, "_calls", None)
    for a, b in zip(native, call(name)):
        assert torch.equal(a, b)


def refuses(name):
    f, args, _ = operands()[name]
    for k, t in args.items():
        if not isinstance(t, torch.Tensor):
            continue
        wrong = [t.cpu(), t.double(), t[:-1], torch.cat([t, t]), t[None], t.unsqueeze(-1).expand(*t.shape, 2)]
        if k == "workspace":
            wrong = [t.cpu(), t.double(), t[:-1], t[None], t[::2]]
        if t.dim() == 2:
            wrong += [t.t().contiguous().t(), t.contiguous()[:1].expand(t.shape), torch.cat([t, t], 1)]
        elif k != "workspace":
            wrong += [torch.stack([t, t], 1)[:, 0]]
        if name == "quantize" and k == "x":     # (any of the three types, as many rows as the codes have)
            wrong = wrong[:1] + wrong[2:]
            wrong[0:0] = [t.to(torch.int32)]
        for w in wrong:
            with pytest.raises((rt.RtossError, KeyError)):
                f(**{**args, k: w})
    torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_operands_that_do_not_fit(name):
    refuses(name)


@pytest.mark.parametrize("name", NAMES)
def test_operands_that_do_not_fit_in_python(name, in_python):
    refuses(name)


def test_a_closed_context_is_refused():
    c = rt.Context(0)
    c.close()
    f = operands()["quantize"][1]
    with pytest.raises(rt.RtossError):
        c.rtoss_quantize_rows(**f)


def test_on_the_current_stream():
    _, args, _ = operands()["quantize"]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)       # what the call has to wait for
        args["x"].fill_(1.0)
        ctx().rtoss_quantize_rows(**args)
    side.synchronize()
    assert bool((args["q"] == 127).all())


def test_threads_on_streams_of_their_own():
    """Four threads, one context: each calls on its own stream with its own operands, over and over."""
    import threading
    sets = [operands() for _ in range(4)]
    for f, args, _ in sets[0].values():
        f(**args)
    torch.cuda.synchronize()
    want = {n: [sets[0][n][1][k].clone() for k in sets[0][n][2]] for n in NAMES}
    errors = []

    def work(mine):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    for n in NAMES:
                        mine[n][0](**mine[n][1])
                torch.cuda.current_stream().synchronize()
        except Exception as e:   # (told below)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(m,)) for m in sets]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for mine in sets:
        for n in NAMES:
            for k, w in zip(mine[n][2], want[n]):
                assert torch.equal(mine[n][1][k], w), (n, k)


FIRST_CALLS = """
import sys, torch
sys.path[:0] = [%r, %r]
import test_gpu_tok_calls as t
sets = t.operands()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    for f, args, _ in sets.values():
        f(**args)
g.replay()
torch.cuda.synchronize()
got = {n: [sets[n][1][k].clone() for k in sets[n][2]] for n in t.NAMES}
for f, args, _ in sets.values():
    f(**args)
torch.cuda.synchronize()
assert all(torch.equal(a, sets[n][1][k]) for n in t.NAMES for a, k in zip(got[n], sets[n][2]))
print("same")
"""


def test_first_calls_of_a_process_inside_a_capture():
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS % (here, os.path.dirname(here))], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]

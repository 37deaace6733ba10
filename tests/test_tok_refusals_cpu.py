"""What the operators over tokens refuse.  Arguments are checked on the host before a device is touched, so no GPU is needed: the
context is a zeroed block of memory (errors write their text into it) and the addresses are never dereferenced."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED, ALIGNMENT = 0, 1, 3, 4
P = 1 << 20            # an aligned address


@pytest.fixture(scope="module")
def rt():
    from paper_2303_02191_b200 import _build
    _build.build()
    from paper_2303_02191_b200 import binding
    return binding


@pytest.fixture(scope="module")
def fake():
    return ctypes.create_string_buffer(1 << 16)


def i8(rt, h, tokens=4, K=64, N=32, x=(P, 0), w=(P, 0), y=(P, 0), res=(0, 0), xs=P, ws=P, bias=0, dtype=1, act=0, after=0):
    return rt.lib.rtoss_matmul_i8(h, rt._I8_PRODUCT.pack(tokens, K, N, *x, *w, *y, *res, xs, ws, bias, dtype, act, after), None)


@pytest.mark.parametrize("want,args", [
    (OK, dict(tokens=0)), (INVALID, dict(tokens=-1)), (INVALID, dict(K=0)), (INVALID, dict(N=0)), (INVALID, dict(tokens=(1 << 30) + 1)),
    (UNSUPPORTED, dict(K=131072)), (INVALID, dict(dtype=3)), (INVALID, dict(act=3)), (INVALID, dict(act=-1)), (INVALID, dict(x=(0, 0))), (INVALID, dict(w=(0, 0))),
    (INVALID, dict(y=(0, 0))), (INVALID, dict(xs=0)), (INVALID, dict(ws=0)), (INVALID, dict(x=(P, 48))), (INVALID, dict(y=(P, 16))),
    (INVALID, dict(x=(P, -64))), (ALIGNMENT, dict(x=(P + 8, 0))), (ALIGNMENT, dict(x=(P, 72))), (ALIGNMENT, dict(K=63)), (ALIGNMENT, dict(w=(P, 65))),
    (ALIGNMENT, dict(N=33)), (ALIGNMENT, dict(y=(P, 36))), (ALIGNMENT, dict(y=(P, 34), dtype=0)), (ALIGNMENT, dict(res=(P + 2, 0))), (ALIGNMENT, dict(res=(P, 33))),
    (ALIGNMENT, dict(xs=P + 4)), (ALIGNMENT, dict(ws=P + 4)), (ALIGNMENT, dict(bias=P + 4))])
def test_matmul_i8(rt, fake, want, args):
    assert i8(rt, fake, **args) == want
    if want:
        assert rt.lib.rtoss_last_error(fake).decode().startswith("matmul i8: ")


def test_quantize_rows(rt, fake):
    q = rt.lib.rtoss_quantize_rows
    assert q(fake, P, 1, 0, 8, 0, P, 0, P, None) == OK
    for bad in ((P, 1, -1, 8, 0, P, 0, P), (P, 1, 4, 0, 0, P, 0, P), (0, 1, 4, 8, 0, P, 0, P), (P, 1, 4, 8, 0, 0, 0, P), (P, 1, 4, 8, 0, P, 0, 0),
                (P, 5, 4, 8, 0, P, 0, P), (P, 1, 4, 8, 7, P, 0, P), (P, 1, 4, 8, 0, P, 7, P)):
        assert q(fake, *bad, None) == INVALID
        assert rt.lib.rtoss_last_error(fake).decode().startswith("quantize rows: ")


NAMES = "x wg wu wd h gate up y dy dgate dup dx dwg dwu dwd".split()


def ffn(rt, handle, backward, tokens=4, D=64, F=32, dtype=1, act=2, **rows):
    flat = [v for k in NAMES for v in rows.get(k, (P, 0))]
    fn = rt.lib.rtoss_gated_ffn_backward if backward else rt.lib.rtoss_gated_ffn_forward
    return fn(handle, rt._FFN.pack(tokens, D, F, dtype, act, *flat), None)


NULL = (0, 0)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("want,args", [
    (INVALID, dict(tokens=-1)), (INVALID, dict(D=0)), (INVALID, dict(F=0)), (UNSUPPORTED, dict(dtype=0)), (INVALID, dict(dtype=3)), (INVALID, dict(act=7)),
    (ALIGNMENT, dict(D=63)), (ALIGNMENT, dict(F=30)), (ALIGNMENT, dict(x=(P + 2, 0))), (ALIGNMENT, dict(wd=(P, 36))), (ALIGNMENT, dict(h=(P, 34))),
    (INVALID, dict(wg=(P, 32))), (INVALID, dict(h=(P, 24))), (INVALID, dict(h=NULL)), (INVALID, dict(gate=NULL)), (INVALID, dict(up=NULL))])
def test_gated_ffn(rt, fake, want, args, backward):
    assert ffn(rt, fake, backward, **args) == want
    assert rt.lib.rtoss_last_error(fake).decode().startswith("gated ffn backward: " if backward else "gated ffn forward: ")


def test_gated_ffn_pairs(rt, fake):
    assert ffn(rt, fake, False, tokens=0) == OK
    assert ffn(rt, fake, False, wd=NULL) == INVALID
    assert ffn(rt, fake, False, y=NULL) == INVALID
    assert ffn(rt, fake, False, x=NULL) == INVALID
    for k in ("dy", "dgate", "dup", "wd"):
        assert ffn(rt, fake, True, **{k: NULL}) == INVALID, k
    assert ffn(rt, fake, True, x=NULL) == INVALID           # dwg needs it
    assert ffn(rt, fake, True, wg=NULL) == INVALID          # dx needs it
    assert ffn(rt, fake, True, tokens=0, dwg=NULL, dwu=NULL, dwd=NULL) == OK


def norm(rt, h, backward, tokens=4, D=64, dtype=1, post=1, pre=1, scale=1.0, eps=1e-6, share=4, wpost=P, wpre=P, dwpost=P, dwpre=P, ws=P, floats=1 << 20, **rows):
    names = "r y gate z n dz dn dr dy dgate".split()
    flat = [v for k in names for v in rows.get(k, (P, 0))]
    fn = rt.lib.rtoss_block_norm_backward if backward else rt.lib.rtoss_block_norm_forward
    return fn(h, rt._BLOCK_NORM.pack(tokens, D, dtype, post, pre, scale, eps, share, wpost, wpre, *flat, dwpost, dwpre, ws, floats), None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("args", [
    dict(tokens=-1), dict(D=0), dict(dtype=3), dict(post=3), dict(pre=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(share=3), dict(share=0), dict(r=NULL), dict(y=NULL),
    dict(post=0), dict(pre=0), dict(r=(P, 63)), dict(gate=(P, 8))])
def test_block_norm(rt, fake, args, backward):
    assert norm(rt, fake, backward, **args) == INVALID
    assert rt.lib.rtoss_last_error(fake).decode().startswith("block norm backward: " if backward else "block norm forward: ")


def test_block_norm_operands(rt, fake):
    assert norm(rt, fake, False, z=NULL) == INVALID
    assert norm(rt, fake, False, n=NULL) == INVALID
    assert norm(rt, fake, True, dr=NULL) == INVALID
    assert norm(rt, fake, True, dy=NULL) == INVALID
    assert norm(rt, fake, True, gate=NULL) == INVALID       # a gradient of no gate
    assert norm(rt, fake, True, ws=0) == INVALID
    assert norm(rt, fake, True, ws=P + 4) == ALIGNMENT
    assert norm(rt, fake, True, floats=4 * 64 * 4 - 1) == INVALID
    assert norm(rt, fake, False, tokens=0) == OK


def test_workspace_grows_with_what_is_asked(rt, fake):
    def floats(tokens, D, gated):
        n = ctypes.c_int64(-1)
        assert rt.lib.rtoss_block_norm_workspace(fake, tokens, D, gated, ctypes.byref(n)) == OK
        return n.value
    assert floats(0, 64, 1) == 0
    for T in (1, 7, 148, 5000, 1 << 20):
        for D in (1, 64, 1000, 2048, 4096, 8192, 30000):
            n, g = floats(T, D, 0), floats(T, D, 1)
            assert n % (2 * D) == 0 and 1 <= n // (2 * D) <= min(T, 148 * 16) and g == 2 * n
    assert rt.lib.rtoss_block_norm_workspace(None, 1, 1, 0, ctypes.byref(ctypes.c_int64())) == INVALID


def test_null_context(rt):
    assert i8(rt, None) == INVALID and ffn(rt, None, False) == INVALID and ffn(rt, None, True) == INVALID
    assert norm(rt, None, False) == INVALID and rt.lib.rtoss_quantize_rows(None, P, 1, 1, 8, 0, P, 0, P, None) == INVALID

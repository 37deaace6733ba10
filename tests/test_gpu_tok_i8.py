"""8-bit product and row quantiser.

Codes and scales are defined in fp32 and are compared bit for bit; the integer sum is exact, so a product is off only by the few
fp32 operations behind it (conversion, two scales, bias, residual: 8 roundings of the magnitudes; SiLU's exponential and
quotient 2^-20) and one rounding to the output's type."""
import numpy as np
import pytest
import torch

from paper_2303_02191_b200 import binding as rt
from tok_util import DT, E32, TINY, U, Rand, ctx, matrix, untouched, within

pytestmark = pytest.mark.gpu


def codes_of(x):
    x = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        s = (np.abs(x).max(axis=1) / np.float32(127)).astype(np.float32)
        s[~np.isfinite(x).all(axis=1)] = np.nan
        q = np.rint((x / s[:, None]).astype(np.float32))
        q = np.where(s[:, None] > 0, q, 0)
    return torch.from_numpy(np.clip(np.nan_to_num(q), -127, 127).astype(np.int8)), torch.from_numpy(s)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 0), (5, 64, 1), (33, 1000, 0), (9, 1024, 0), (4, 1025, 2), (130, 2048, 0), (2, 8192, 0),
                                           (2, 8200, 0), (3, 30011, 1)])
def test_codes_and_scales(rows, cols, pad, dt):
    x = Rand("q", rows, cols).normal(rows, cols, 3.0)
    x[:, ::13] *= 20
    x, _ = matrix(x.to(DT[dt]), DT[dt], pad)
    q, whole = matrix((rows, cols), torch.int8, pad)
    scale = torch.empty(rows, device="cuda")
    ctx().rtoss_quantize_rows(x, q, scale)
    want_q, want_s = codes_of(x)
    assert torch.equal(scale.cpu(), want_s) and torch.equal(q.cpu(), want_q)
    assert untouched(q, whole)


def test_values_on_the_borders_between_codes():
    """Scale exactly 2: every odd number is a tie, and its neighbours are not."""
    odd = torch.arange(-253, 254, 2, dtype=torch.float32)
    x = torch.cat([torch.tensor([254.0]), odd, torch.nextafter(odd, torch.tensor(1e9)), torch.nextafter(odd, torch.tensor(-1e9))])[None].cuda()
    for k in (1.0, 2.0 ** -40, 2.0 ** 60, 1 / 3):
        xs = (x * k).contiguous()
        q, scale = torch.empty_like(xs, dtype=torch.int8), torch.empty(1, device="cuda")
        ctx().rtoss_quantize_rows(xs, q, scale)
        want_q, want_s = codes_of(xs)
        assert torch.equal(scale.cpu(), want_s) and torch.equal(q.cpu(), want_q)


@pytest.mark.parametrize("cols", [40, 3000])
def test_rows_of_zeros_subnormals_infinities_and_nan(cols):
    x = torch.zeros(7, cols, device="cuda")
    x[1, 3] = 1e-45
    x[2, :] = torch.linspace(-1e-38, 1e-38, cols)
    x[3, 5] = float("inf")
    x[4, 6] = float("nan")
    x[5, :] = 3.4e38
    x[6, 0] = -0.0
    q, scale = torch.empty(7, cols, dtype=torch.int8, device="cuda"), torch.empty(7, device="cuda")
    ctx().rtoss_quantize_rows(x, q, scale)
    want_q, want_s = codes_of(x)
    assert np.array_equal(scale.cpu().numpy(), want_s.numpy(), equal_nan=True) and torch.equal(q.cpu(), want_q)


def test_unaligned_rows():
    buf = Rand("un").normal(20, 101)
    for dt in ("f32", "bf16"):
        x = buf.to(DT[dt]).reshape(-1)[1:1 + 19 * 101].reshape(19, 101)[:, :97]
        q = torch.empty(19 * 97 + 3, dtype=torch.int8, device="cuda")[3:].reshape(19, 97)
        scale = torch.empty(19, device="cuda")
        ctx().rtoss_quantize_rows(x, q, scale)
        want_q, want_s = codes_of(x)
        assert torch.equal(scale.cpu(), want_s) and torch.equal(q.cpu(), want_q)


def act64(v, act):
    return v if act == "none" else v.clamp(min=0) if act == "relu" else v * torch.sigmoid(v)


def product(T, K, N, dt, act="none", bias=False, res=None, pad=0, extreme=False):
    r = Rand("i8", T, K, N)
    if extreme:
        xq, wq = torch.full((T, K), -128.0), torch.full((N, K), -128.0)
        wq[::2] = 127
    else:
        xq, wq = (r.normal(T, K, 50.0).round().clamp(-128, 127), r.normal(N, K, 50.0).round().clamp(-128, 127))
    x, _ = matrix(xq.to(torch.int8), torch.int8, pad)
    w, _ = matrix(wq.to(torch.int8), torch.int8, pad)
    xs, ws = (r.normal(1, n)[0].abs() * 0.01 + 1e-4 for n in (T, N))
    b = r.normal(1, N)[0] if bias else None
    y, whole = matrix((T, N), DT[dt], pad)
    rv = matrix(r.normal(T, N).to(DT[dt]), DT[dt], pad + 1)[0] if res else None
    ctx().rtoss_matmul_i8(x, xs, w, ws, y, act=rt.ACT_NAMES[act], bias=b, residual=rv, residual_after_act=res == "after")
    torch.cuda.synchronize()
    assert ctx().rtoss_device_status() == 0
    s = (x.double() @ w.double().T) * xs.double()[:, None] * ws.double()
    size = s.abs()
    if bias:
        s, size = s + b.double(), size + b.double().abs()
    if res == "before":
        s, size = s + rv.double(), size + rv.double().abs()
    v = act64(s, act)
    tol = 1.1 * 8 * E32 * size + 16 * E32 * v.abs()
    if res == "after":
        v = v + rv.double()
        tol = tol + E32 * v.abs()
    within(y, v, tol + (U[dt] + E32) * v.abs() + TINY[dt], "y")
    assert untouched(y, whole)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,K,N", [(1, 1, 1), (1, 4096, 100), (2, 17, 33), (8, 1003, 129), (9, 64, 16), (16, 520, 77), (17, 128, 32), (20, 1, 1), (100, 100, 300),
                                   (128, 2048, 64), (256, 128, 256), (257, 129, 257), (331, 1003, 1001), (1000, 31, 40), (200, 8000, 500), (2500, 136, 2000)])
def test_products(T, K, N, dt):
    i = T + K + N
    product(T, K, N, dt, act=("none", "silu", "relu")[i % 3], bias=i % 2 == 0, res=(None, "before", "after")[i // 2 % 3], pad=i % 3)


@pytest.mark.parametrize("T", [3, 150])
@pytest.mark.parametrize("res", [None, "before", "after"])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_epilogues(T, act, res):
    product(T, 200, 75, "bf16", act, True, res)
    product(T, 200, 75, "f32", act, False, res)


@pytest.mark.parametrize("T", [1, 40])
def test_longest_sums_do_not_overflow(T):
    product(T, 131071, 24, "f32", extreme=True)


def test_residual_in_place():
    for T in (4, 70):
        r = Rand("inplace", T)
        x, w = (matrix(r.normal(n, 96, 40.0).round().clamp(-127, 127).to(torch.int8), torch.int8)[0] for n in (T, 48))
        xs, ws = torch.full((T,), 0.01, device="cuda"), torch.full((48,), 0.02, device="cuda")
        y = r.normal(T, 48).to(torch.bfloat16)
        want = (x.double() @ w.double().T) * xs.double()[:, None] * ws.double() + y.double()
        size = want.abs() + 2 * y.double().abs()
        ctx().rtoss_matmul_i8(x, xs, w, ws, y, residual=y)
        within(y, want, 8 * E32 * size + U["bf16"] * want.abs(), "y")


def test_a_row_that_is_not_finite_gives_nan_in_its_row_alone():
    for T in (3, 50):
        x = Rand("nf", T).normal(T, 64)
        x[1, 7] = float("inf")
        q, s = torch.empty(T, 64, dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        w, ws = torch.ones(32, 64, dtype=torch.int8, device="cuda"), torch.ones(32, device="cuda")
        y = torch.empty(T, 32, device="cuda")
        for act in (rt.ACT_NONE, rt.ACT_RELU, rt.ACT_SILU):
            ctx().rtoss_quantize_rows(x, q, s)
            ctx().rtoss_matmul_i8(q, s, w, ws, y, act=act)
            bad = torch.isnan(y).all(dim=1)
            assert bad.tolist() == [t == 1 for t in range(T)] and bool(torch.isfinite(y[~bad]).all())


def test_pruned_pointwise_layer_in_eight_bits():
    """Select and pack a 1x1 layer, expand it, quantise its rows: the 8-bit product over the positions of a map stays within the
    quantisation's bound of the library's own convolution with the same weights."""
    from paper_2303_02191_b200 import synth
    c, (N, H, W, Cin, Cout) = ctx(), (2, 20, 20, 64, 96)
    masks = rt.rtoss_pattern_preset(4, rt.PRESET_CENTRE8)
    w = torch.from_numpy(synth.kaiming_weights(3, 1, Cout, Cin, 1)).cuda()
    x = torch.from_numpy(synth.activations(3, 1, N, Cin, H, W)).cuda().permute(0, 2, 3, 1).contiguous()
    bias = torch.from_numpy(synth.bias(3, 1, Cout)).cuda()
    packed = c.rtoss_pack(w, 1, masks, 4, c.rtoss_select_patterns(w, 1, masks, 4), rt.F32)
    dense = packed.to_dense().reshape(Cout, Cin)
    want = torch.empty(N, H, W, Cout, device="cuda")
    c.rtoss_conv1x1_pattern(packed, x, want, N, H, W, 1, rt.NHWC, rt.ACT_NONE, bias)
    wq, ws = torch.empty(Cout, Cin, dtype=torch.int8, device="cuda"), torch.empty(Cout, device="cuda")
    xm = x.reshape(-1, Cin)
    xq, xs = torch.empty(xm.shape, dtype=torch.int8, device="cuda"), torch.empty(xm.shape[0], device="cuda")
    y = torch.empty(xm.shape[0], Cout, device="cuda")
    c.rtoss_quantize_rows(dense, wq, ws)
    c.rtoss_quantize_rows(xm, xq, xs)
    c.rtoss_matmul_i8(xq, xs, wq, ws, y, bias=bias)
    xd, wd = xm.double(), dense.double()
    # a code is off by half a scale at most
    hx, hw = 0.5001 * xs.double()[:, None], 0.5001 * ws.double()[:, None]
    tol = xd.abs() @ hw.expand(-1, Cin).T + hx.expand(-1, Cin) @ wd.abs().T + Cin * hx * hw.T
    ref = xd @ wd.T + bias.double()
    rms = ref.square().mean().sqrt()
    within(y, want.reshape(-1, Cout).double(), tol + 2e-4 * torch.maximum(ref.abs(), rms), "y")   # (the convolution's own bound: 1e-4)
    packed.close()


@pytest.mark.parametrize("dt,bits", [("bf16", 7), ("f16", 10)])
def test_codes_of_every_mantissa_against_every_maximum(dt, bits):
    """A code depends on the mantissas of a value and of its row's maximum and on how far their exponents lie apart: all of them, below
    a tenth of a step left out, for maxima of several exponents.  The codes are those of the fp32 quotient, half to even."""
    n = 1 << bits
    m = torch.arange(n, 2 * n, dtype=torch.float64) / n
    x = torch.cat([m * 2.0 ** -e for e in range(0, 11)]).to(DT[dt])
    for scale in (1.0, 2.0 ** -9, 1024.0) + ((2.0 ** 100, 2.0 ** -95, 2.0 ** -110) if dt == "bf16" else ()):
        rows = x.double()[None, :].repeat(n, 1) * scale
        rows = torch.where(rows <= (m * scale)[:, None], rows, 0.0)
        rows[:, 1::2] *= -1
        rows[:, 0] = m * scale
        xd = rows.to(DT[dt]).cuda()
        q, s = torch.empty(n, x.numel(), dtype=torch.int8, device="cuda"), torch.empty(n, device="cuda")
        ctx().rtoss_quantize_rows(xd, q, s)
        want_q, want_s = codes_of(xd)
        assert torch.equal(s.cpu(), want_s) and torch.equal(q.cpu(), want_q), (dt, scale)


@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T,K,N", [(128, 8192, 1000), (331, 1003, 1001), (200, 4096, 4096), (64, 2048, 520), (1000, 1030, 1024)])
def test_products_cut_along_k(T, K, N, dt):
    """Few tiles and a long k: shares of k, exchanged between the CTAs of a cluster."""
    product(T, K, N, dt, act="silu", bias=True, res="before" if T % 2 else "after", pad=1)

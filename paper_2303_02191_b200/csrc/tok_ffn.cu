// Gated feed-forward block over tokens, forward and backward (bf16 / fp16).
//
//   g = x Wg^T, u = x Wu^T, h = act(g) * u     one launch: a tile's accumulators hold 128 columns of g and the same of u
//   y = h Wd^T                                 one launch
//   dh = dy Wd; dg = dh * u * act'(g), du = dh * act(g), h again    one launch
//   dx = dg Wg + du Wu                         one launch, the two products are two segments of k
//   dWg = dg^T x, dWu = du^T x, dWd = dy^T h   one launch over the tiles of all three
//
// h is formed again in the backward pass from the saved g and u (it costs a multiplication; keeping it would cost tokens * F
// values).  g, u, h, dg and du are rounded to the data's 16 bits where they pass through memory, as the next product takes
// 16-bit operands; all sums are fp32.
#include "tok_few.cuh"
#include "tok_launch.cuh"

namespace {

using namespace rtoss_tok;

constexpr const char* kFwd = "gated ffn forward";
constexpr const char* kBwd = "gated ffn backward";

Rows rows_of(const rtoss_rows& r, int64_t dense) { return Rows{r.dev, r.row_stride ? r.row_stride : dense}; }

struct Operand {
    const rtoss_rows* r;
    int cols;
    bool needed;
};

rtoss_status check(rtoss_ctx* ctx, const rtoss_ffn* f, bool backward, const char* where) {
    if (!ctx) return RTOSS_ERR_INVALID_ARG;
    if (!f) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "null argument");
    if (f->tokens < 0 || f->D < 1 || f->F < 1 || f->tokens > kMaxDim || f->D > kMaxDim || f->F > kMaxDim)
        return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "need 0 <= tokens, 1 <= D, F, all at most 2^30");
    if (f->dtype != RTOSS_BF16 && f->dtype != RTOSS_F16)
        return fail(ctx, f->dtype == RTOSS_F32 ? RTOSS_ERR_UNSUPPORTED : RTOSS_ERR_INVALID_ARG, where, "the data types are bf16 and fp16");
    if (!act_ok(f->act)) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "bad activation");
    if (f->tokens && !backward && !f->w_down.dev != !f->y.dev) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "w_down and y come together or not at all");
    if (f->tokens && !f->gate.dev != !f->up.dev) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "gate and up come together or not at all");
    const Operand fwd[] = {{&f->x, f->D, true}, {&f->w_gate, f->D, true}, {&f->w_up, f->D, true}, {&f->w_down, f->F, false}, {&f->h, f->F, true},
                           {&f->gate, f->F, false}, {&f->up, f->F, false}, {&f->y, f->D, false}};
    const bool dwi = f->dw_gate.dev || f->dw_up.dev;
    const Operand bwd[] = {{&f->x, f->D, dwi}, {&f->w_gate, f->D, f->dx.dev != nullptr}, {&f->w_up, f->D, f->dx.dev != nullptr}, {&f->w_down, f->F, true},
                           {&f->h, f->F, true}, {&f->gate, f->F, true}, {&f->up, f->F, true}, {&f->dy, f->D, true}, {&f->dgate, f->F, true},
                           {&f->dup, f->F, true}, {&f->dx, f->D, false}, {&f->dw_gate, f->D, false}, {&f->dw_up, f->D, false}, {&f->dw_down, f->F, false}};
    const Operand* o = backward ? bwd : fwd;
    for (int i = 0, n = backward ? 14 : 8; i < n; ++i) {
        const rtoss_rows& r = *o[i].r;
        if (!r.dev) {
            if (o[i].needed && f->tokens) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "null matrix");
            continue;
        }
        const int64_t ld = r.row_stride ? r.row_stride : o[i].cols;
        if (ld < o[i].cols || ld > (int64_t)1 << 36) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "a row stride is below the row's length");
        if (!aligned16(r.dev) || ld % 8) return fail(ctx, RTOSS_ERR_ALIGNMENT, where, "rows must start on 16-byte boundaries");
    }
    return RTOSS_OK;
}

template <typename T, int MODE, int NP>
int run_gemm(const rtoss_ctx* ctx, GemmArgs<NP>& g, const Product* ps, int np, bool a_mn, bool b_mn, cudaStream_t s) {
    const Shape c = choose_shape<T, MODE, NP>(ctx, ps, np);
    return c.bn == 256 ? launch_gemm<T, MODE, 256, NP>(ctx, g, ps, np, a_mn, b_mn, c.KS, s) : launch_gemm<T, MODE, 128, NP>(ctx, g, ps, np, a_mn, b_mn, c.KS, s);
}

template <typename T>
int forward(const rtoss_ctx* ctx, const rtoss_ffn* f, cudaStream_t s) {
    const int M = (int)f->tokens;
    const Rows x = rows_of(f->x, f->D), wg = rows_of(f->w_gate, f->D), wu = rows_of(f->w_up, f->D), wd = rows_of(f->w_down, f->F), h = rows_of(f->h, f->F),
               gate = rows_of(f->gate, f->F), up = rows_of(f->up, f->F), y = rows_of(f->y, f->D);
    if (M <= kFewTokens) {
        FewArgs a = {};
        a.x = x.p, a.x_ld = x.ld, a.w0 = wg.p, a.w_ld = wg.ld, a.w1 = wu.p, a.w1_ld = wu.ld;
        a.tokens = M, a.rows = f->F, a.K = f->D, a.y = const_cast<void*>(h.p), a.y_ld = h.ld, a.act = f->act;
        a.gate = const_cast<void*>(gate.p), a.gate_ld = gate.ld, a.up = const_cast<void*>(up.p), a.up_ld = up.ld;
        if (const int e = launch_few<T, T, true>(ctx, a, s)) return e;
        if (!y.p) return 0;
        FewArgs b = {};
        b.x = h.p, b.x_ld = h.ld, b.w0 = wd.p, b.w_ld = wd.ld, b.tokens = M, b.rows = f->D, b.K = f->F, b.y = const_cast<void*>(y.p), b.y_ld = y.ld;
        return launch_few<T, T, false>(ctx, b, s);
    }
    GemmArgs<1> g = {};
    g.act = f->act;
    g.save = f->gate.dev != nullptr;
    const Product in = {M, f->F, f->D, 1, {x, x}, {wg, wu}, {h, gate, up}};
    if (const int e = run_gemm<T, kGated, 1>(ctx, g, &in, 1, false, false, s)) return e;
    if (!y.p) return 0;
    GemmArgs<3> d = {};
    const Product out = {M, f->D, f->F, 1, {h, h}, {wd, wd}, {y, {}, {}}};
    return run_gemm<T, kPlain, 3>(ctx, d, &out, 1, false, false, s);
}

template <typename T>
int backward(const rtoss_ctx* ctx, const rtoss_ffn* f, cudaStream_t s) {
    const int M = (int)f->tokens;
    const Rows x = rows_of(f->x, f->D), wg = rows_of(f->w_gate, f->D), wu = rows_of(f->w_up, f->D), wd = rows_of(f->w_down, f->F), h = rows_of(f->h, f->F),
               gate = rows_of(f->gate, f->F), up = rows_of(f->up, f->F), dy = rows_of(f->dy, f->D), dg = rows_of(f->dgate, f->F), du = rows_of(f->dup, f->F),
               dx = rows_of(f->dx, f->D), dwg = rows_of(f->dw_gate, f->D), dwu = rows_of(f->dw_up, f->D), dwd = rows_of(f->dw_down, f->F);
    GemmArgs<1> g = {};
    g.act = f->act;
    const Product grad = {M, f->F, f->D, 1, {dy, dy}, {wd, wd}, {h, dg, du}, {gate, up}};
    if (const int e = run_gemm<T, kGateGrad, 1>(ctx, g, &grad, 1, false, true, s)) return e;
    if (dx.p) {
        GemmArgs<3> d = {};
        const Product p = {M, f->D, f->F, 2, {dg, du}, {wg, wu}, {dx, {}, {}}};
        if (const int e = run_gemm<T, kPlain, 3>(ctx, d, &p, 1, false, true, s)) return e;
    }
    Product w[3];
    int n = 0;
    if (dwg.p) w[n++] = {f->F, f->D, M, 1, {dg, dg}, {x, x}, {dwg, {}, {}}};
    if (dwu.p) w[n++] = {f->F, f->D, M, 1, {du, du}, {x, x}, {dwu, {}, {}}};
    if (dwd.p) w[n++] = {f->D, f->F, M, 1, {dy, dy}, {h, h}, {dwd, {}, {}}};
    if (!n) return 0;
    GemmArgs<3> d = {};
    return run_gemm<T, kPlain, 3>(ctx, d, w, n, true, true, s);
}

// No tokens: the weights' gradients are sums of nothing.
int zero_rows(const rtoss_rows& r, int rows, int cols, cudaStream_t s) {
    if (!r.dev) return 0;
    return (int)cudaMemset2DAsync(r.dev, (size_t)(r.row_stride ? r.row_stride : cols) * 2, 0, (size_t)cols * 2, (size_t)rows, s);
}

}  // namespace

extern "C" {

rtoss_status rtoss_gated_ffn_forward(rtoss_ctx* ctx, const rtoss_ffn* f, void* cuda_stream) {
    const rtoss_status st = check(ctx, f, false, kFwd);
    if (st != RTOSS_OK || f->tokens == 0) return st;
    rtoss_device_guard on_device(ctx->device);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    return launched(ctx, kFwd, f->dtype == RTOSS_BF16 ? forward<__nv_bfloat16>(ctx, f, s) : forward<__half>(ctx, f, s));
}

rtoss_status rtoss_gated_ffn_backward(rtoss_ctx* ctx, const rtoss_ffn* f, void* cuda_stream) {
    const rtoss_status st = check(ctx, f, true, kBwd);
    if (st != RTOSS_OK) return st;
    rtoss_device_guard on_device(ctx->device);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (f->tokens == 0) {
        int e = zero_rows(f->dw_gate, f->F, f->D, s);
        if (!e) e = zero_rows(f->dw_up, f->F, f->D, s);
        if (!e) e = zero_rows(f->dw_down, f->D, f->F, s);
        return launched(ctx, kBwd, e);
    }
    return launched(ctx, kBwd, f->dtype == RTOSS_BF16 ? backward<__nv_bfloat16>(ctx, f, s) : backward<__half>(ctx, f, s));
}

}  // extern "C"


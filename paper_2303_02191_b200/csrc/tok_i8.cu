// Matrix product in 8-bit integers with a scale for each token and each output channel, and the row quantiser in front of it.
#include "tok_few.cuh"
#include "tok_launch.cuh"

namespace {

using namespace rtoss_tok;

constexpr const char* kQuant = "quantize rows";
constexpr const char* kMul = "matmul i8";

// ---- rows to 8 bits -------------------------------------------------------------------------------------------------
// bound: bytes (a row is read once and one byte a value written).  A group of G threads takes a row and holds up to 32 values
// a thread in registers between the maximum and the rounding; longer rows are read again, from the caches.
constexpr int kHold = 4;   // pieces of eight values a thread holds

// Eight values from element i of a row on (zeros behind its end).
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T* row, int i, int cols, float (&v)[8]) {
    if (VEC && i + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            const float4 p = *reinterpret_cast<const float4*>(row + i), q = *reinterpret_cast<const float4*>(row + i + 4);
            v[0] = p.x, v[1] = p.y, v[2] = p.z, v[3] = p.w, v[4] = q.x, v[5] = q.y, v[6] = q.z, v[7] = q.w;
        } else {
            const uint4 p = *reinterpret_cast<const uint4*>(row + i);
            const T* e = reinterpret_cast<const T*>(&p);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = rtoss_dev::to_f32<T>(e[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i + j < cols ? rtoss_dev::to_f32<T>(row[i + j]) : 0.f;
    }
}

// The code of x: the quotient x / s in fp32, rounded half to even.  The product with 1 / s is within 3e-5 of it, so only
// values that close to a border need the division.
__device__ __forceinline__ int code_of(float x, float s, float inv, bool divide) {
    float q = x * inv, r = rintf(q);
    if (divide || fabsf(fabsf(q - r) - 0.5f) < 1e-4f) r = rintf(__fdiv_rn(x, s));
    return (int)fminf(fmaxf(r, -127.f), 127.f);
}

// G: threads of a row, 32 (eight rows a block) or 256.
template <typename T, bool VEC, int G>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const T* __restrict__ x, long long x_ld, signed char* __restrict__ q, long long q_ld,
                                                            float* __restrict__ scale, int rows, int cols) {
    rtoss_dev::pdl_enter();
    __shared__ unsigned s_top[8];
    const int row = G == 32 ? (int)blockIdx.x * 8 + ((int)threadIdx.x >> 5) : (int)blockIdx.x, at = (int)threadIdx.x % G;
    if (row >= rows) return;   // (a whole warp, or nobody)
    const T* xr = x + (long long)row * x_ld;
    float v[kHold][8];
    unsigned top = 0u;
#pragma unroll
    for (int p = 0; p < kHold; ++p) {
        const int i = (p * G + at) * 8;
        if (i < cols) load8<T, VEC>(xr, i, cols, v[p]);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) v[p][j] = 0.f;
    }
    // magnitudes compare as integers, and Inf and NaN lie above every number
#pragma unroll
    for (int p = 0; p < kHold; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[p][j]) & 0x7FFFFFFFu);
    for (int i = (kHold * G + at) * 8; i < cols; i += G * 8) {
        float w[8];
        load8<T, VEC>(xr, i, cols, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(w[j]) & 0x7FFFFFFFu);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if (G > 32) {
        if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 8; ++w) top = max(top, s_top[w]);
    }
    const bool finite = top < 0x7F800000u;
    const float s = finite ? __fdiv_rn(__uint_as_float(top), 127.f) : __int_as_float(0x7FC00000);
    if (at == 0) scale[row] = s;
    const bool live = finite && s > 0.f, divide = !(s > 1e-30f);
    const float inv = live ? __fdiv_rn(1.f, s) : 0.f;
    signed char* qr = q + (long long)row * q_ld;
    const bool vec_out = (reinterpret_cast<unsigned long long>(qr) & 7u) == 0;
    auto put = [&](int i, const float (&w)[8]) {
        unsigned b[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j / 4] |= (unsigned)(unsigned char)(signed char)(live ? code_of(w[j], s, inv, divide) : 0) << (8 * (j & 3));
        if (vec_out && i + 8 <= cols) *reinterpret_cast<uint2*>(qr + i) = make_uint2(b[0], b[1]);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j < cols) qr[i + j] = (signed char)(b[j / 4] >> (8 * (j & 3)));
    };
#pragma unroll
    for (int p = 0; p < kHold; ++p) {
        const int i = (p * G + at) * 8;
        if (i < cols) put(i, v[p]);
    }
    for (int i = (kHold * G + at) * 8; i < cols; i += G * 8) {
        float w[8];
        load8<T, VEC>(xr, i, cols, w);
        put(i, w);
    }
}

template <typename T>
int quantize(const void* x, int64_t x_ld, int8_t* q, int64_t q_ld, float* scale, int rows, int cols, cudaStream_t s) {
    const bool vec = aligned16(x) && (x_ld * (int64_t)sizeof(T)) % 16 == 0;
    const T* xt = (const T*)x;
    if (cols <= 1024) {   // one warp holds a row
        const unsigned grid = (unsigned)((rows + 7) / 8);
        return vec ? (int)rtoss_dev::launch_pdl(quantize_rows_kernel<T, true, 32>, grid, 256, 0, s, xt, (long long)x_ld, (signed char*)q, (long long)q_ld, scale, rows, cols)
                   : (int)rtoss_dev::launch_pdl(quantize_rows_kernel<T, false, 32>, grid, 256, 0, s, xt, (long long)x_ld, (signed char*)q, (long long)q_ld, scale, rows, cols);
    }
    return vec ? (int)rtoss_dev::launch_pdl(quantize_rows_kernel<T, true, 256>, (unsigned)rows, 256, 0, s, xt, (long long)x_ld, (signed char*)q, (long long)q_ld, scale, rows, cols)
               : (int)rtoss_dev::launch_pdl(quantize_rows_kernel<T, false, 256>, (unsigned)rows, 256, 0, s, xt, (long long)x_ld, (signed char*)q, (long long)q_ld, scale, rows, cols);
}

// ---- the product ----------------------------------------------------------------------------------------------------
template <typename T>
int multiply(const rtoss_ctx* ctx, const rtoss_i8_product* p, cudaStream_t s) {
    const int64_t y_ld = p->y.row_stride ? p->y.row_stride : p->N, r_ld = p->residual.row_stride ? p->residual.row_stride : p->N;
    const Rows x = {p->x.dev, p->x.row_stride ? p->x.row_stride : p->K}, w = {p->w.dev, p->w.row_stride ? p->w.row_stride : p->K};
    if (p->tokens <= kFewTokens) {
        FewArgs a = {};
        a.x = x.p, a.x_ld = x.ld, a.w0 = w.p, a.w_ld = w.ld, a.tokens = (int)p->tokens, a.rows = p->N, a.K = p->K;
        a.y = p->y.dev, a.y_ld = y_ld, a.act = p->act, a.row_scale = p->x_scale_dev, a.col_scale = p->w_scale_dev, a.bias = p->bias_dev;
        a.res = p->residual.dev, a.res_ld = r_ld, a.res_after = p->residual_after_act;
        return launch_few<signed char, T, false>(ctx, a, s);
    }
    GemmArgs<1> g = {};
    g.act = p->act;
    g.e0 = p->residual.dev, g.e_ld = r_ld, g.res_after = p->residual_after_act;
    g.row_scale = p->x_scale_dev, g.col_scale = p->w_scale_dev, g.bias = p->bias_dev;
    const Product d = {(int)p->tokens, p->N, p->K, 1, {x, x}, {w, w}, {{p->y.dev, y_ld}, {}, {}}};
    const Shape c = choose_shape(&d, 1, false, true, 128, ctx->sm_count > 0 ? ctx->sm_count : 148);
    return c.bn == 256 ? launch_gemm<T, kInt8, 256, 1>(ctx, g, &d, 1, false, false, c.KS, s) : launch_gemm<T, kInt8, 128, 1>(ctx, g, &d, 1, false, false, c.KS, s);
}

}  // namespace

extern "C" {

rtoss_status rtoss_quantize_rows(rtoss_ctx* ctx, const void* x_dev, rtoss_dtype dtype, int64_t rows, int cols, int64_t x_row_stride, int8_t* q_dev,
                                 int64_t q_row_stride, float* scale_dev, void* cuda_stream) {
    if (!ctx) return RTOSS_ERR_INVALID_ARG;
    if (rows < 0 || cols < 1 || rows > kMaxDim || cols > kMaxDim) return fail(ctx, RTOSS_ERR_INVALID_ARG, kQuant, "need 0 <= rows, 1 <= cols, both at most 2^30");
    if (dtype != RTOSS_F32 && dtype != RTOSS_BF16 && dtype != RTOSS_F16) return fail(ctx, RTOSS_ERR_INVALID_ARG, kQuant, "bad dtype");
    if (rows == 0) return RTOSS_OK;
    if (!x_dev || !q_dev || !scale_dev) return fail(ctx, RTOSS_ERR_INVALID_ARG, kQuant, "null argument");
    const int64_t x_ld = x_row_stride ? x_row_stride : cols, q_ld = q_row_stride ? q_row_stride : cols;
    if (x_ld < cols || q_ld < cols || x_ld > (int64_t)1 << 36 || q_ld > (int64_t)1 << 36) return fail(ctx, RTOSS_ERR_INVALID_ARG, kQuant, "a row stride is below the row's length");
    rtoss_device_guard on_device(ctx->device);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    int e;
    if (dtype == RTOSS_F32) e = quantize<float>(x_dev, x_ld, q_dev, q_ld, scale_dev, (int)rows, cols, s);
    else if (dtype == RTOSS_BF16) e = quantize<__nv_bfloat16>(x_dev, x_ld, q_dev, q_ld, scale_dev, (int)rows, cols, s);
    else e = quantize<__half>(x_dev, x_ld, q_dev, q_ld, scale_dev, (int)rows, cols, s);
    return launched(ctx, kQuant, e);
}

rtoss_status rtoss_matmul_i8(rtoss_ctx* ctx, const rtoss_i8_product* p, void* cuda_stream) {
    if (!ctx) return RTOSS_ERR_INVALID_ARG;
    if (!p) return fail(ctx, RTOSS_ERR_INVALID_ARG, kMul, "null argument");
    if (p->tokens < 0 || p->K < 1 || p->N < 1 || p->tokens > kMaxDim || p->N > kMaxDim)
        return fail(ctx, RTOSS_ERR_INVALID_ARG, kMul, "need 0 <= tokens, 1 <= K, N, at most 2^30");
    if (p->K > 131071) return fail(ctx, RTOSS_ERR_UNSUPPORTED, kMul, "K above 131071: a 32-bit sum could overflow");
    if ((p->y_dtype != RTOSS_F32 && p->y_dtype != RTOSS_BF16 && p->y_dtype != RTOSS_F16) || !act_ok(p->act))
        return fail(ctx, RTOSS_ERR_INVALID_ARG, kMul, "bad dtype or activation");
    if (p->tokens == 0) return RTOSS_OK;
    if (!p->x.dev || !p->w.dev || !p->y.dev || !p->x_scale_dev || !p->w_scale_dev) return fail(ctx, RTOSS_ERR_INVALID_ARG, kMul, "null argument");
    const int64_t es = (int64_t)rtoss_dtype_size(p->y_dtype);
    const rtoss_rows* m[4] = {&p->x, &p->w, &p->y, &p->residual};
    for (int i = 0; i < 4; ++i) {
        if (!m[i]->dev) continue;
        const int64_t cols = i < 2 ? p->K : p->N, ld = m[i]->row_stride ? m[i]->row_stride : cols;
        if (ld < cols || ld > (int64_t)1 << 36) return fail(ctx, RTOSS_ERR_INVALID_ARG, kMul, "a row stride is below the row's length");
        if (!aligned16(m[i]->dev) || (ld * (i < 2 ? 1 : es)) % 16) return fail(ctx, RTOSS_ERR_ALIGNMENT, kMul, "rows must start on 16-byte boundaries");
    }
    if (!aligned16(p->x_scale_dev) || !aligned16(p->w_scale_dev) || (p->bias_dev && !aligned16(p->bias_dev)))
        return fail(ctx, RTOSS_ERR_ALIGNMENT, kMul, "scales and bias must be 16-byte aligned");
    rtoss_device_guard on_device(ctx->device);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    int e;
    if (p->y_dtype == RTOSS_F32) e = multiply<float>(ctx, p, s);
    else if (p->y_dtype == RTOSS_BF16) e = multiply<__nv_bfloat16>(ctx, p, s);
    else e = multiply<__half>(ctx, p, s);
    return launched(ctx, kMul, e);
}

}  // extern "C"

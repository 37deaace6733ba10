// Products of at most sixteen tokens: the weights are read once and everything else is small.
//
//   sum over k of W[row, k] * X[token, k],   fp32 (16-bit operands) or exact 32-bit integer (8-bit operands) sums
//
// bound: the bytes of the weights.  A block takes sixteen rows of weights (kGated: eight of the gate and the same eight of
// the up projection, whose sums then meet in one thread) and its eight warps share k; blocks of a cluster share it further
// where there are few rows.  A lane reads 16 bytes of a row at a time straight into the registers of an m16n8
// instruction: the order of k inside an instruction does not matter as long as both operands use the same one, so four
// lanes' 16 bytes are two instructions' worth of k and nothing passes through shared memory.  (Single-row dot products on the
// FMA pipes would have to widen every weight and could not serve more than about four tokens at this rate.)
#ifndef RTOSS_TOK_FEW_CUH
#define RTOSS_TOK_FEW_CUH

#include "tok_internal.h"
#include "tok_math.cuh"

namespace rtoss_tok {

constexpr int kFewTokens = 16;
constexpr int kFewWarps = 8;

struct FewArgs {
    const void* x;
    const void* w0;     // weights; gated: the gate's
    const void* w1;     // gated: the up projection's
    long long x_ld, w_ld, w1_ld;   // elements
    int tokens, rows, K;
    int share;          // 16-byte pieces of k that one block of a cluster takes (a multiple of 4)
    void* y;
    long long y_ld;
    int act;
    // gated
    void* gate;
    void* up;
    long long gate_ld, up_ld;
    // 8-bit
    const float* row_scale;
    const float* col_scale;
    const float* bias;
    const void* res;
    long long res_ld;
    int res_after;
};

// Sixteen bytes of a row from element k on, zeros behind its end (no byte behind it is read).
template <typename E>
__device__ __forceinline__ uint4 row_piece(const E* row, int k, int K) {
    constexpr int kPer = 16 / (int)sizeof(E);
    if (k + kPer <= K) return *reinterpret_cast<const uint4*>(row + k);
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (k < K) {
        unsigned* w = reinterpret_cast<unsigned*>(&v);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (k + i < K) {
                if constexpr (sizeof(E) == 1) w[i / 4] |= (unsigned)(unsigned char)row[k + i] << (8 * (i & 3));
                else w[i / 2] |= (unsigned)reinterpret_cast<const unsigned short*>(row)[k + i] << (16 * (i & 1));
            }
        }
    }
    return v;
}

template <typename E>
__device__ __forceinline__ void mma_few(unsigned (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    if constexpr (sizeof(E) == 1) {
        int* d = reinterpret_cast<int*>(c);
        asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    } else {
        float* d = reinterpret_cast<float*>(c);
        if constexpr (std::is_same<E, __nv_bfloat16>::value)
            asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                         : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                         : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
        else
            asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                         : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                         : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
}

// E: type of the operands, T: of the outputs, NT: tiles of eight tokens.
template <typename E, typename T, bool GATED, int NT>
__global__ void __launch_bounds__(kFewWarps * 32) tok_few_kernel(const FewArgs a) {
    constexpr int kPer = 16 / (int)sizeof(E), kTok = 8 * NT;
    // Groups of four pieces that a warp loads before it multiplies: two, so that more blocks fit an SM and none waits for long
    // (one token, 2048 -> 5632: 15.0 us, with four 18.0); four for 9 to 16 tokens in 16 bits (1024 -> 2816: 7.9 us, with two 10.1).
    constexpr int kUnroll = NT == 2 && sizeof(E) == 2 ? 4 : 2;
    __shared__ unsigned s_part[kFewWarps][16 * kTok];
    __shared__ unsigned s_sum[8][16 * kTok];   // of the blocks of the cluster (rank 0's copy is the one that counts)
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    unsigned rank, ranks;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const int group = (int)(blockIdx.x / ranks);
    if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // (waited for before anything goes to another block)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int r0 = GATED ? group * 8 : group * 16;
    // (what rows behind the last one and tokens that are not there would add up to is not written: they read the first ones)
    const E* w0 = reinterpret_cast<const E*>(a.w0);
    const E* rowA = w0 + (long long)(r0 + g < a.rows ? r0 + g : r0) * a.w_ld;
    const E* rowB = GATED ? reinterpret_cast<const E*>(a.w1) + (long long)(r0 + g < a.rows ? r0 + g : r0) * a.w1_ld
                          : w0 + (long long)(r0 + g + 8 < a.rows ? r0 + g + 8 : r0) * a.w_ld;
    const E* x[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) x[n] = reinterpret_cast<const E*>(a.x) + (8 * n + g < a.tokens ? (long long)(8 * n + g) * a.x_ld : 0ll);
    unsigned c[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[n][i] = 0u;

    // pieces of 16 bytes: this block takes [first, last), a warp kUnroll groups of four at a time
    const int pieces = (a.K + kPer - 1) / kPer, first = (int)rank * a.share, last = min(pieces, first + a.share);
    // (loads without conditions, all in flight at once, but for the last round and rows whose end cuts a piece: with conditions
    // the block of one token, 2048 -> 5632, took 20.9 us, without them 15.0, 4.6 TB/s)
    const int all = min(last, a.K / kPer);
    for (int p0 = first + warp * 4 * kUnroll; p0 < last; p0 += kFewWarps * 4 * kUnroll) {
        uint4 wa[kUnroll], wb[kUnroll], xb[kUnroll][NT];
        if (p0 + 4 * kUnroll <= all) {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int k = (p0 + 4 * u + t) * kPer;
                wa[u] = *reinterpret_cast<const uint4*>(rowA + k);
                wb[u] = *reinterpret_cast<const uint4*>(rowB + k);
#pragma unroll
                for (int n = 0; n < NT; ++n) xb[u][n] = *reinterpret_cast<const uint4*>(x[n] + k);
            }
        } else {
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int p = p0 + 4 * u + t;
                wa[u] = wb[u] = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int n = 0; n < NT; ++n) xb[u][n] = make_uint4(0u, 0u, 0u, 0u);
                if (p < last) {
                    wa[u] = row_piece(rowA, p * kPer, a.K);
                    wb[u] = row_piece(rowB, p * kPer, a.K);
#pragma unroll
                    for (int n = 0; n < NT; ++n) xb[u][n] = row_piece(x[n], p * kPer, a.K);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mma_few<E>(c[n], wa[u].x, wb[u].x, wa[u].y, wb[u].y, xb[u][n].x, xb[u][n].y);
                mma_few<E>(c[n], wa[u].z, wb[u].z, wa[u].w, wb[u].w, xb[u][n].z, xb[u][n].w);
            }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_part[warp][(g + 8 * (i >> 1)) * kTok + 8 * n + 2 * t + (i & 1)] = c[n][i];
    __syncthreads();
    if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    // sums over the warps, in their order; then over the blocks of the cluster, in theirs
    const int e = (int)threadIdx.x;
    const bool adds = e < 16 * kTok;
    unsigned v = 0u;
    auto plus = [](unsigned p, unsigned q) {
        if constexpr (sizeof(E) == 1) return p + q;
        else return __float_as_uint(__uint_as_float(p) + __uint_as_float(q));
    };
    if (adds) {
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) v = plus(v, s_part[w][e]);
        const unsigned mine = (unsigned)__cvta_generic_to_shared(&s_sum[rank][e]);
        if (ranks > 1) {
            unsigned to;
            asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(to) : "r"(mine));
            asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(v) : "memory");
        } else {
            s_sum[0][e] = v;
        }
    }
    __syncthreads();
    if (ranks > 1) {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (rank) return;
    }
    auto total = [&](int i) {
        unsigned s = s_sum[0][i];
        for (unsigned r = 1; r < ranks; ++r) s = plus(s, s_sum[r][i]);
        return s;
    };
    // row fastest: neighbouring threads write neighbouring outputs of a token
    constexpr int kOutRows = GATED ? 8 : 16;
    if (e < kOutRows * kTok) {
        const int r = e % kOutRows, tok = e / kOutRows, row = r0 + r;
        if (row < a.rows && tok < a.tokens) {
            T* y = reinterpret_cast<T*>(a.y) + (long long)tok * a.y_ld + row;
            const unsigned s = total(r * kTok + tok);
            if constexpr (GATED) {
                const float gv = __uint_as_float(s), uv = __uint_as_float(total((r + 8) * kTok + tok));
                if (a.gate) {
                    reinterpret_cast<T*>(a.gate)[(long long)tok * a.gate_ld + row] = rtoss_dev::from_f32<T>(gv);
                    reinterpret_cast<T*>(a.up)[(long long)tok * a.up_ld + row] = rtoss_dev::from_f32<T>(uv);
                }
                with_act(a.act, [&](auto act) { *y = rtoss_dev::from_f32<T>(act_of<decltype(act)::value>(gv) * uv); });
            } else if constexpr (sizeof(E) == 1) {
                const float res = a.res ? rtoss_dev::to_f32<T>(reinterpret_cast<const T*>(a.res)[(long long)tok * a.res_ld + row]) : 0.f;
                const float bias = a.bias ? a.bias[row] : 0.f;
                with_act(a.act, [&](auto act) {
                    *y = rtoss_dev::from_f32<T>(i8_value<decltype(act)::value>((int)s, a.row_scale[tok], a.col_scale[row], bias, res, a.res_after));
                });
            } else {
                *y = rtoss_dev::from_f32<T>(__uint_as_float(s));
            }
        }
    }
}

template <typename E, typename T, bool GATED>
int launch_few(const rtoss_ctx* ctx, FewArgs& a, cudaStream_t stream) {
    const int per = GATED ? 8 : 16, sms = ctx->sm_count > 0 ? ctx->sm_count : 148;
    const int groups = (a.rows + per - 1) / per, pieces = (a.K + 16 / (int)sizeof(E) - 1) / (16 / (int)sizeof(E));
    // as many blocks to a cluster as it takes to have two blocks an SM, while each still has work for its warps
    int ranks = 1;
    while (ranks < 8 && groups * ranks < 2 * sms && pieces / (2 * ranks) >= kFewWarps * 4) ranks *= 2;
    a.share = ((pieces + ranks - 1) / ranks + 3) / 4 * 4;
    const dim3 grid((unsigned)(groups * ranks));
    auto go = [&](auto kernel) { return (int)rtoss_dev::launch_pdl(kernel, grid, dim3(kFewWarps * 32), 0, stream, ranks, a); };
    return a.tokens <= 8 ? go(tok_few_kernel<E, T, GATED, 1>) : go(tok_few_kernel<E, T, GATED, 2>);
}

}  // namespace rtoss_tok

#endif

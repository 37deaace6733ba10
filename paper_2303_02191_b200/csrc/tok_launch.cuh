// Choosing a tile and launching tok_gemm_kernel.
#ifndef RTOSS_TOK_LAUNCH_CUH
#define RTOSS_TOK_LAUNCH_CUH

#include <atomic>

#include "tok_gemm.cuh"

namespace rtoss_tok {

// A product as its operator states it: D[M, N] = A B^T over one or two segments of k.
struct Rows {
    const void* p;
    int64_t ld;   // elements
};
struct Product {
    int M, N, K;        // K: of each segment
    int segments;
    Rows a[2], b[2];    // kGated: b[0] the gate's weights, b[1] the up projection's (N: columns of h)
    Rows out[3];
    Rows edge[2];       // kGateGrad: the saved projections
};

template <typename T> struct MapType;
template <> struct MapType<float> { static constexpr CUtensorMapDataType v = CU_TENSOR_MAP_DATA_TYPE_FLOAT32; };
template <> struct MapType<__nv_bfloat16> { static constexpr CUtensorMapDataType v = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16; };
template <> struct MapType<__half> { static constexpr CUtensorMapDataType v = CU_TENSOR_MAP_DATA_TYPE_FLOAT16; };

// How many clusters of 2 KS CTAs (one CTA an SM) the device holds at once.
template <typename Kernel>
int resident_clusters(Kernel kernel, int smem, int cluster, int sms) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(sms / cluster * cluster));
    cfg.blockDim = dim3(kGemmThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = sms / cluster;
    }
    return n;
}

// Shape of a launch.  Clocks of a block of 128 bytes of k: 4 instructions of 128 clocks (256 columns) or, bound by what shared
// memory moves, about 4 x 100 (128 columns).  Shares of k cost the exchange: two barriers of the cluster and reading the sums, about
// 4000 clocks, and what a CTA sends at 24 bytes a clock (traced).
struct Shape {
    int bn, KS;
    double clocks;
};
template <int MODE, typename T>
Shape choose_shape(const Product* ps, int np, int sms) {
    constexpr bool gated = MODE == kGated;
    constexpr int kper = MODE == kInt8 ? 128 : 64;
    const int pairs = sms / 2;
    Shape best = {256, 1, 1e300};
    for (int bn = 256; bn >= 128; bn -= 128) {
        const int tn = gated ? bn / 2 : bn, shares = bn / (gated ? 64 : 32);
        int64_t tiles = 0;
        int kb = 0, kb_min = 1 << 30;
        double work = 0;
        for (int i = 0; i < np; ++i) {
            const int64_t t = (int64_t)((ps[i].M + 255) / 256) * ((ps[i].N + tn - 1) / tn);
            const int k = (ps[i].K + kper - 1) / kper * ps[i].segments;
            tiles += t;
            work += (double)t * k;
            kb = k > kb ? k : kb;
            kb_min = k < kb_min ? k : kb_min;
        }
        const double per_kb = bn == 256 ? 512.0 : 400.0;
        for (int ks = 1; ks <= kMaxKS && ks <= shares; ks *= 2) {
            if (ks > 1 && (np > 1 || kb_min < 4 * ks || tiles * ks > pairs)) continue;
            if ((bn == 256 ? GemmShape<MODE, 256, T>::stages_of(ks) : GemmShape<MODE, 128, T>::stages_of(ks)) < 3) continue;
            const double waves = (double)((tiles * ks + pairs - 1) / pairs);
            const double c = ks == 1 ? (waves < 4 ? waves * kb * per_kb : work / pairs * per_kb) + 2000.0
                                     : (double)((kb + ks - 1) / ks) * per_kb + 6000.0 + 512.0 * bn * (ks - 1) / ks / 24.0;
            if (c < best.clocks) best = {bn, ks, c};
        }
    }
    return best;
}

template <typename T, int MODE, int BN, int NP>
int launch_gemm(const rtoss_ctx* ctx, GemmArgs<NP>& g, const Product* ps, int np, bool a_mn, bool b_mn, int KS, cudaStream_t stream) {
    using S = GemmShape<MODE, BN, T>;
    auto kernel = tok_gemm_kernel<T, MODE, BN, NP>;
    constexpr bool i8 = MODE == kInt8;
    const CUtensorMapDataType in_type = i8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : MapType<T>::v;
    const int in_size = i8 ? 1 : 2, kper = 128 / in_size;
    static std::atomic<int> resident[64];   // pairs the device holds at once; 0: not asked yet
    const int sms = ctx->sm_count > 0 ? ctx->sm_count : 148;
    const int dev = ctx->device;
    // (the driver encodes for the thread's current context, and a thread that has made no runtime call yet has none)
    if (const cudaError_t e = cudaSetDevice(dev)) return (int)e;
    int held = dev < 64 ? resident[dev].load(std::memory_order_acquire) : 0;
    if (!held) {
        if (const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem)) return (int)e;
        held = resident_clusters(kernel, S::kSmem, 2, sms);
        if (dev < 64) resident[dev].store(held, std::memory_order_release);
    }
    g.n_problems = np;
    g.KS = KS;
    g.stages = S::stages_of(KS);
    g.a_mn = a_mn;
    g.b_mn = b_mn;
    g.status = ctx->dev_status;
    g.wait = ctx->wait_cycles > 0 ? ctx->wait_cycles : 2000000000ll;
    const unsigned fmt = i8 ? 1u : MapType<T>::v == CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 ? 1u : 0u;   // signed 8-bit; bf16; fp16
    g.idesc = ((i8 ? 2u : 1u) << 4) | (fmt << 7) | (fmt << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((unsigned)(BN >> 3) << 17) |
              ((unsigned)(256 >> 4) << 24);
    int64_t tiles = 0;
    bool ok = true;
    for (int i = 0; i < np; ++i) {
        GemmProblem& q = g.p[i];
        const Product& p = ps[i];
        q.M = p.M;
        q.N = p.N;
        q.tiles_m = (p.M + 255) / 256;
        q.tiles_n = (p.N + S::kTileN - 1) / S::kTileN;
        q.first = (int)tiles;
        q.kb0 = (p.K + kper - 1) / kper;
        q.kb = q.kb0 * p.segments;
        tiles += (int64_t)q.tiles_m * q.tiles_n;
        for (int s = 0; s < 2; ++s) {
            const int sa = s < p.segments ? s : 0, sb = MODE == kGated || s < p.segments ? s : 0;
            ok = ok && (a_mn ? encode_rows(&q.a[s], in_type, p.a[sa].p, p.K, p.M, p.a[sa].ld * in_size, 64, 64, 128)
                             : encode_rows(&q.a[s], in_type, p.a[sa].p, p.M, p.K, p.a[sa].ld * in_size, kper, 128, 128));
            ok = ok && (b_mn ? encode_rows(&q.b[s], in_type, p.b[sb].p, p.K, p.N, p.b[sb].ld * in_size, 64, 64, 128)
                             : encode_rows(&q.b[s], in_type, p.b[sb].p, p.N, p.K, p.b[sb].ld * in_size, kper, BN / 2, 128));
            if (MODE != kGated && p.segments == 1) {
                q.a[1] = q.a[0];
                q.b[1] = q.b[0];
                break;
            }
        }
        for (int o = 0; o < 3; ++o) {
            const Rows& out = p.out[o].p ? p.out[o] : p.out[0];
            q.op[o] = const_cast<void*>(out.p);
            q.o_ld[o] = out.ld;
            if (MODE == kPlain && o == 1) ok = ok && encode_rows(&q.o[1], MapType<T>::v, out.p, p.M, p.N, out.ld * (int64_t)sizeof(T), 32, 32, 64);
            else if (o && !p.out[o].p) q.o[o] = q.o[0];
            else ok = ok && encode_rows(&q.o[o], MapType<T>::v, out.p, p.M, p.N, out.ld * (int64_t)sizeof(T), S::kUnitCols, 32, S::kOutRow);
        }
    }
    if constexpr (MODE == kGateGrad)
        for (int o = 0; o < 2; ++o)
            ok = ok && encode_rows(&g.e[o], MapType<T>::v, ps[0].edge[o].p, ps[0].M, ps[0].N, ps[0].edge[o].ld * (int64_t)sizeof(T), 32, 32, 64);
    if (!ok) return (int)cudaErrorInvalidValue;
    if (tiles > 0x3FFFFFFF) return (int)cudaErrorInvalidConfiguration;
    g.tiles = (int)tiles;
    const int64_t clusters = KS > 1 ? tiles : tiles < held ? tiles : held;
    return (int)rtoss_dev::launch_pdl(kernel, dim3((unsigned)(clusters * 2 * KS)), dim3(kGemmThreads), (size_t)S::kSmem, stream, 2 * KS, g);
}

}  // namespace rtoss_tok

#endif

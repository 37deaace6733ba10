// The norms behind one block of a network and in front of the next, with the gate and the residual between them, forward and
// backward:
//
//   v = norm_post(y),  z = residual_scale * r + gate * v,  n = norm_pre(z)
//   norm(t) = (t - mean) / sqrt(mean((t - mean)^2) + eps) * weight     (root-mean-square norm: mean = 0)
//
// bound: bytes.  A row is read once and every intermediate stays in registers: forward 4 rows of traffic a token, backward 6
// (r, y, dz, dn in, dr, dy out).  The backward pass forms v and z again from r and y in fp32: reading the stored z instead would
// cost the same bytes and bring its rounding into every gradient.  A unit of G threads takes a contiguous run of rows; weights,
// gates and the sums over tokens stay in its registers, and the next row is on its way while this one is reduced.  Sums over
// tokens (the gradients of weights and gates) end as one row per unit in the workspace and are added in the units' order by
// a second launch: no atomics, the same bits every time.  All arithmetic is fp32; squares are summed after the mean is
// subtracted, not as a difference of moments.
#include "tok_internal.h"
#include "tok_math.cuh"

namespace {

using namespace rtoss_tok;
using rtoss_dev::from_f32;
using rtoss_dev::to_f32;

constexpr const char* kFwd = "block norm forward";
constexpr const char* kBwd = "block norm backward";

struct NormArgs {
    const void *r, *y, *dz, *dn, *gate;
    void *z, *n, *dr, *dy;
    long long r_ld, y_ld, z_ld, n_ld, dz_ld, dn_ld, dr_ld, dy_ld, gate_ld, dgate_ld;
    const float *wpost, *wpre;
    int rows, D, post, pre, vec;
    int S;             // tokens that share a gate
    int per_unit;      // rows of a unit
    float scale, eps;
    float *p_post, *p_pre, *p_gate;   // partial sums: [unit][D], [unit][D], [unit][2][D]
    void* dgate;
};

// ---- eight values -----------------------------------------------------------------------------------------------------
// As they lie in memory: a row's loads stay in flight until its values are widened.
template <typename T>
struct __align__(16) Raw {
    T e[8];
};
// (VEC: rows and pieces are multiples of 16 bytes)
template <typename T, bool VEC>
__device__ __forceinline__ void fetch8(const void* base, long long ld, int row, int i, int D, Raw<T>& r) {
    const T* at = reinterpret_cast<const T*>(base) + (long long)row * ld + i;
    if (VEC) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(&r)[j] = reinterpret_cast<const uint4*>(at)[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.e[j] = i + j < D ? at[j] : from_f32<T>(0.f);
    }
}
template <typename T>
__device__ __forceinline__ void zero8(Raw<T>& r) {
#pragma unroll
    for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(&r)[j] = make_uint4(0u, 0u, 0u, 0u);
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw<T>& r, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = to_f32<T>(r.e[j]);
}
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const void* base, long long ld, int row, int i, int D, float (&v)[8]) {
    Raw<T> r;
    fetch8<T, VEC>(base, ld, row, i, D, r);
    widen8<T>(r, v);
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(void* base, long long ld, int row, int i, int D, const float (&v)[8]) {
    T* at = reinterpret_cast<T*>(base) + (long long)row * ld + i;
    if (VEC) {
        Raw<T> r;
#pragma unroll
        for (int j = 0; j < 8; ++j) r.e[j] = from_f32<T>(v[j]);
#pragma unroll
        for (int j = 0; j < (int)sizeof(T) / 2; ++j) reinterpret_cast<uint4*>(at)[j] = reinterpret_cast<const uint4*>(&r)[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (i + j < D) at[j] = from_f32<T>(v[j]);
    }
}

// Sums of N values over the G threads of a unit (G = 32: a warp of its own).  Consecutive calls take alternating halves of the
// buffer, so that one barrier a call is enough.
template <int G>
struct Reduce {
    float* buf;   // [2][2][G / 32]
    int turn, warp, lane;
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
        if (G > 32) {
            constexpr int W = G / 32;
            float* b = buf + turn * 2 * W;
            turn ^= 1;
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) b[k * W + warp] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                float t = lane < W ? b[k * W + lane] : 0.f;
#pragma unroll
                for (int o = W / 2; o; o >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
                v[k] = __shfl_sync(0xFFFFFFFFu, t, 0);
            }
        }
    }
};

// Mean (layer norm) and 1 / root of the mean square of the P pieces a thread holds; `in`: the piece lies inside the row.
template <int P, int G>
__device__ __forceinline__ void stats(Reduce<G>& red, const float (&v)[P][8], const bool (&in)[P], int at, int D, int kind, float eps, float* mean, float* rstd) {
    float m = 0.f;
    if (kind == RTOSS_NORM_LAYER) {
        float s[1] = {0.f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[0] += v[p][j];   // (zeros outside the row)
        red.template sum<1>(s);
        m = s[0] / (float)D;
    }
    float q[1] = {0.f};
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = (p * G + at) * 8 + j < D ? v[p][j] - m : 0.f;
            q[0] += d * d;
        }
    red.template sum<1>(q);
    *mean = m;
    *rstd = 1.f / sqrtf(q[0] / (float)D + eps);
}

// Threads of a unit, units of a block: G = 32 has eight warps to a block, each a unit.
template <int G> constexpr int block_of() { return G == 32 ? 256 : G; }

template <typename T, bool VEC, int G, int P>
__global__ void __launch_bounds__(block_of<G>()) norm_forward_kernel(const NormArgs a) {
    __shared__ float buf[4 * (G / 32)];
    const int at = (int)threadIdx.x % G, unit = G == 32 ? (int)blockIdx.x * 8 + (int)threadIdx.x / 32 : (int)blockIdx.x;
    Reduce<G> red{buf, 0, at / 32, (int)threadIdx.x & 31};
    const int D = a.D;
    rtoss_dev::pdl_enter();
    const int row0 = unit * a.per_unit, row1 = min(a.rows, row0 + a.per_unit);
    if (row0 >= row1) return;   // (a whole unit)
    bool in[P];
    float wpost[P][8], wpre[P][8], gate[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = (p * G + at) * 8;
        in[p] = i < D;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            wpost[p][j] = a.wpost && i + j < D ? a.wpost[i + j] : 1.f;
            wpre[p][j] = a.wpre && i + j < D ? a.wpre[i + j] : 1.f;
            gate[p][j] = 1.f;
        }
    }
    int gate_row = -1;
    float y[P][8], r[P][8];
    Raw<T> yn[P], rn[P];   // of the next row
#pragma unroll
    for (int p = 0; p < P; ++p) {
        zero8(yn[p]);
        zero8(rn[p]);
    }
    auto fetch = [&](int row) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (in[p]) {
                fetch8<T, VEC>(a.y, a.y_ld, row, (p * G + at) * 8, D, yn[p]);
                fetch8<T, VEC>(a.r, a.r_ld, row, (p * G + at) * 8, D, rn[p]);
            }
    };
    fetch(row0);
    for (int row = row0; row < row1; ++row) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            widen8<T>(yn[p], y[p]);
            widen8<T>(rn[p], r[p]);
        }
        if (row + 1 < row1) fetch(row + 1);
        if (a.gate && row / a.S != gate_row) {
            gate_row = row / a.S;
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (in[p]) load8<T, VEC>(a.gate, a.gate_ld, gate_row, (p * G + at) * 8, D, gate[p]);
        }
        float mean = 0.f, rstd = 1.f;
        if (a.post != RTOSS_NORM_NONE) stats<P, G>(red, y, in, at, D, a.post, a.eps, &mean, &rstd);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = (y[p][j] - mean) * rstd * wpost[p][j];
                y[p][j] = (p * G + at) * 8 + j < D ? fmaf(gate[p][j], v, a.scale * r[p][j]) : 0.f;   // z
            }
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (in[p]) store8<T, VEC>(a.z, a.z_ld, row, (p * G + at) * 8, D, y[p]);
        if (a.pre != RTOSS_NORM_NONE) {
            stats<P, G>(red, y, in, at, D, a.pre, a.eps, &mean, &rstd);
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int j = 0; j < 8; ++j) y[p][j] = (y[p][j] - mean) * rstd * wpre[p][j];
                if (in[p]) store8<T, VEC>(a.n, a.n_ld, row, (p * G + at) * 8, D, y[p]);
            }
        }
    }
}

template <typename T, bool VEC, int G, int P>
__global__ void __launch_bounds__(block_of<G>()) norm_backward_kernel(const NormArgs a) {
    __shared__ float buf[4 * (G / 32)];
    const int at = (int)threadIdx.x % G, unit = G == 32 ? (int)blockIdx.x * 8 + (int)threadIdx.x / 32 : (int)blockIdx.x;
    Reduce<G> red{buf, 0, at / 32, (int)threadIdx.x & 31};
    const int D = a.D;
    rtoss_dev::pdl_enter();
    const int row0 = unit * a.per_unit, row1 = min(a.rows, row0 + a.per_unit);
    if (row0 >= row1) return;
    const float inv_d = 1.f / (float)D;
    bool in[P];
    float wpost[P][8], wpre[P][8], gate[P][8], s_post[P][8], s_pre[P][8], s_gate[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = (p * G + at) * 8;
        in[p] = i < D;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            wpost[p][j] = a.wpost && i + j < D ? a.wpost[i + j] : 1.f;
            wpre[p][j] = a.wpre && i + j < D ? a.wpre[i + j] : 1.f;
            gate[p][j] = 1.f;
            s_post[p][j] = s_pre[p][j] = s_gate[p][j] = 0.f;
        }
    }
    int gate_row = -1;
    float y[P][8], r[P][8], dz[P][8], dn[P][8];
    Raw<T> yn[P], rn[P], dzn[P], dnn[P];   // of the next row
#pragma unroll
    for (int p = 0; p < P; ++p) {
        zero8(yn[p]);
        zero8(rn[p]);
        zero8(dzn[p]);
        zero8(dnn[p]);
    }
    auto fetch = [&](int row) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (in[p]) {
                const int i = (p * G + at) * 8;
                fetch8<T, VEC>(a.y, a.y_ld, row, i, D, yn[p]);
                fetch8<T, VEC>(a.r, a.r_ld, row, i, D, rn[p]);
                if (a.dz) fetch8<T, VEC>(a.dz, a.dz_ld, row, i, D, dzn[p]);
                if (a.dn) fetch8<T, VEC>(a.dn, a.dn_ld, row, i, D, dnn[p]);
            }
    };
    fetch(row0);
    for (int row = row0; row < row1; ++row) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            widen8<T>(yn[p], y[p]);
            widen8<T>(rn[p], r[p]);
            widen8<T>(dzn[p], dz[p]);
            widen8<T>(dnn[p], dn[p]);
        }
        if (row + 1 < row1) fetch(row + 1);
        if (a.gate && row / a.S != gate_row) {
            gate_row = row / a.S;
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (in[p]) load8<T, VEC>(a.gate, a.gate_ld, gate_row, (p * G + at) * 8, D, gate[p]);
        }
        // v and z again
        float ymean = 0.f, yrstd = 1.f, zmean = 0.f, zrstd = 1.f;
        if (a.post != RTOSS_NORM_NONE) stats<P, G>(red, y, in, at, D, a.post, a.eps, &ymean, &yrstd);
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool here = (p * G + at) * 8 + j < D;
                y[p][j] = here ? (y[p][j] - ymean) * yrstd : 0.f;   // y normalised
                r[p][j] = here ? fmaf(gate[p][j], y[p][j] * wpost[p][j], a.scale * r[p][j]) : 0.f;   // z
            }
        if (a.pre != RTOSS_NORM_NONE) {
            stats<P, G>(red, r, in, at, D, a.pre, a.eps, &zmean, &zrstd);
            float m[2] = {0.f, 0.f};
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float hat = (p * G + at) * 8 + j < D ? (r[p][j] - zmean) * zrstd : 0.f, gn = dn[p][j] * wpre[p][j];
                    s_pre[p][j] += dn[p][j] * hat;
                    r[p][j] = hat;
                    m[0] += gn * hat;
                    m[1] += gn;
                }
            red.template sum<2>(m);
            const float m0 = m[0] * inv_d, m1 = a.pre == RTOSS_NORM_LAYER ? m[1] * inv_d : 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < 8; ++j) dz[p][j] += zrstd * (dn[p][j] * wpre[p][j] - r[p][j] * m0 - m1);
        }
        // dz holds the whole gradient of z
        float m[2] = {0.f, 0.f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float out[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                out[j] = a.scale * dz[p][j];
                s_gate[p][j] += dz[p][j] * (y[p][j] * wpost[p][j]);
                const float dv = dz[p][j] * gate[p][j];
                s_post[p][j] += dv * y[p][j];
                dz[p][j] = dv * wpost[p][j];
                m[0] += dz[p][j] * y[p][j];
                m[1] += (p * G + at) * 8 + j < D ? dz[p][j] : 0.f;
            }
            if (in[p]) store8<T, VEC>(a.dr, a.dr_ld, row, (p * G + at) * 8, D, out);
        }
        if (a.post != RTOSS_NORM_NONE) {
            red.template sum<2>(m);
            const float m0 = m[0] * inv_d, m1 = a.post == RTOSS_NORM_LAYER ? m[1] * inv_d : 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < 8; ++j) dz[p][j] = yrstd * (dz[p][j] - y[p][j] * m0 - m1);
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (in[p]) store8<T, VEC>(a.dy, a.dy_ld, row, (p * G + at) * 8, D, dz[p]);
        // a gate's last row here: its sum is final when all its rows were this unit's, else one of the unit's two shares
        if (a.dgate && (row + 1 == row1 || (row + 1) / a.S != row / a.S)) {
            const int first = row / a.S * a.S, last = first + a.S;   // (S divides the tokens)
            const bool whole = first >= row0 && last <= row1;
            float* part = a.p_gate + ((long long)unit * 2 + (first > row0 ? 1 : 0)) * D;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int i = (p * G + at) * 8;
                if (in[p]) {
                    if (whole) store8<T, VEC>(a.dgate, a.dgate_ld, row / a.S, i, D, s_gate[p]);
                    else store8<float, VEC>(part, 0, 0, i, D, s_gate[p]);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) s_gate[p][j] = 0.f;
            }
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int i = (p * G + at) * 8;
        if (!in[p]) continue;
        if (a.p_post) store8<float, VEC>(a.p_post, D, unit, i, D, s_post[p]);
        if (a.p_pre) store8<float, VEC>(a.p_pre, D, unit, i, D, s_pre[p]);
    }
}

// ---- rows of more than 8192 values: a block a run of rows, every pass reads them again (from the caches) -----------------
constexpr int kLongThreads = 512;

template <typename T>
__device__ __forceinline__ float at_of(const void* base, long long ld, int row, int i) {
    return base ? to_f32<T>(reinterpret_cast<const T*>(base)[(long long)row * ld + i]) : 0.f;
}

template <typename T, bool BACKWARD>
__global__ void __launch_bounds__(kLongThreads) norm_long_kernel(const NormArgs a) {
    __shared__ float buf[4 * (kLongThreads / 32)];
    Reduce<kLongThreads> red{buf, 0, (int)threadIdx.x / 32, (int)threadIdx.x & 31};
    rtoss_dev::pdl_enter();
    const int unit = (int)blockIdx.x, row0 = unit * a.per_unit, row1 = min(a.rows, row0 + a.per_unit), D = a.D, tid = (int)threadIdx.x;
    const float inv_d = 1.f / (float)D;
    if (row0 >= row1) return;
    if (BACKWARD) {   // the sums over tokens live in this unit's rows of the workspace (a thread only meets its own columns)
        for (int i = tid; i < D; i += kLongThreads) {
            if (a.p_post) a.p_post[(long long)unit * D + i] = 0.f;
            if (a.p_pre) a.p_pre[(long long)unit * D + i] = 0.f;
            if (a.p_gate) a.p_gate[(long long)unit * 2 * D + i] = a.p_gate[((long long)unit * 2 + 1) * D + i] = 0.f;
        }
    }
    for (int row = row0; row < row1; ++row) {
        const int gr = a.gate ? row / a.S : 0;
        auto stat = [&](int kind, auto value, float* mean, float* rstd) {
            float m = 0.f;
            if (kind == RTOSS_NORM_LAYER) {
                float s[1] = {0.f};
                for (int i = tid; i < D; i += kLongThreads) s[0] += value(i);
                red.template sum<1>(s);
                m = s[0] * inv_d;
            }
            float q[1] = {0.f};
            for (int i = tid; i < D; i += kLongThreads) {
                const float d = value(i) - m;
                q[0] += d * d;
            }
            red.template sum<1>(q);
            *mean = m;
            *rstd = 1.f / sqrtf(q[0] * inv_d + a.eps);
        };
        float ymean = 0.f, yrstd = 1.f, zmean = 0.f, zrstd = 1.f;
        auto y_of = [&](int i) { return at_of<T>(a.y, a.y_ld, row, i); };
        if (a.post != RTOSS_NORM_NONE) stat(a.post, y_of, &ymean, &yrstd);
        auto hat_of = [&](int i) { return (y_of(i) - ymean) * yrstd; };
        auto post_w = [&](int i) { return a.wpost ? a.wpost[i] : 1.f; };
        auto pre_w = [&](int i) { return a.wpre ? a.wpre[i] : 1.f; };
        auto gate_of = [&](int i) { return a.gate ? at_of<T>(a.gate, a.gate_ld, gr, i) : 1.f; };
        auto z_of = [&](int i) { return fmaf(gate_of(i), hat_of(i) * post_w(i), a.scale * at_of<T>(a.r, a.r_ld, row, i)); };
        if (a.pre != RTOSS_NORM_NONE) stat(a.pre, z_of, &zmean, &zrstd);
        if (!BACKWARD) {
            // (z may lie where r or y does: a value is read by the thread that then writes it, and not read again)
            for (int i = tid; i < D; i += kLongThreads) {
                const float z = z_of(i);
                reinterpret_cast<T*>(a.z)[(long long)row * a.z_ld + i] = from_f32<T>(z);
                if (a.pre != RTOSS_NORM_NONE) reinterpret_cast<T*>(a.n)[(long long)row * a.n_ld + i] = from_f32<T>((z - zmean) * zrstd * pre_w(i));
            }
            continue;
        }
        float pm[2] = {0.f, 0.f};
        if (a.pre != RTOSS_NORM_NONE) {
            for (int i = tid; i < D; i += kLongThreads) {
                const float dn = at_of<T>(a.dn, a.dn_ld, row, i), hat = (z_of(i) - zmean) * zrstd;
                if (a.p_pre) a.p_pre[(long long)unit * D + i] += dn * hat;
                pm[0] += dn * pre_w(i) * hat;
                pm[1] += dn * pre_w(i);
            }
            red.template sum<2>(pm);
            pm[0] *= inv_d;
            pm[1] = a.pre == RTOSS_NORM_LAYER ? pm[1] * inv_d : 0.f;
        }
        auto total_of = [&](int i) {
            float t = at_of<T>(a.dz, a.dz_ld, row, i);
            if (a.pre != RTOSS_NORM_NONE) t += zrstd * (at_of<T>(a.dn, a.dn_ld, row, i) * pre_w(i) - (z_of(i) - zmean) * zrstd * pm[0] - pm[1]);
            return t;
        };
        float qm[2] = {0.f, 0.f};
        const int first = row / a.S * a.S, last = first + a.S;
        const bool whole = first >= row0 && last <= row1;
        float* part = a.p_gate + ((long long)unit * 2 + (first > row0 ? 1 : 0)) * D;
        for (int i = tid; i < D; i += kLongThreads) {
            const float t = total_of(i), hat = hat_of(i), dv = t * gate_of(i);
            if (a.dgate) {
                const float sum = (row == first || row == row0 ? 0.f : part[i]) + t * (hat * post_w(i));
                part[i] = sum;
                if (whole && row + 1 == last) reinterpret_cast<T*>(a.dgate)[(long long)gr * a.dgate_ld + i] = from_f32<T>(sum);
            }
            if (a.p_post) a.p_post[(long long)unit * D + i] += dv * hat;
            qm[0] += dv * post_w(i) * hat;
            qm[1] += dv * post_w(i);
        }
        if (a.post != RTOSS_NORM_NONE) {
            red.template sum<2>(qm);
            qm[0] *= inv_d;
            qm[1] = a.post == RTOSS_NORM_LAYER ? qm[1] * inv_d : 0.f;
        }
        for (int i = tid; i < D; i += kLongThreads) {
            const float t = total_of(i);
            float dy = t * gate_of(i) * post_w(i);
            if (a.post != RTOSS_NORM_NONE) dy = yrstd * (dy - hat_of(i) * qm[0] - qm[1]);
            reinterpret_cast<T*>(a.dr)[(long long)row * a.dr_ld + i] = from_f32<T>(a.scale * t);
            reinterpret_cast<T*>(a.dy)[(long long)row * a.dy_ld + i] = from_f32<T>(dy);
        }
    }
}

// ---- the sums over tokens ---------------------------------------------------------------------------------------------------
struct JoinArgs {
    const float *p_post, *p_pre, *p_gate;
    float *dpost, *dpre;
    void* dgate;
    long long dgate_ld;
    int D, units, per_unit, S, by_gate;
};

// 32 columns a block, 32 runs of units side by side, joined in their order.
constexpr int kJoinRuns = 32;
template <typename T>
__global__ void __launch_bounds__(kJoinRuns * 32) norm_join_kernel(const JoinArgs a) {
    __shared__ float s[kJoinRuns][32];
    rtoss_dev::pdl_enter();
    const int col = (int)blockIdx.x * 32 + ((int)threadIdx.x & 31), run = (int)threadIdx.x >> 5, what = (int)blockIdx.y;
    const bool in = col < a.D;
    const float* p = what == 0 ? a.p_post : a.p_pre;
    int first = 0, last = a.units;   // units that hold a share
    long long pitch = a.D;
    long long row0 = 0;   // first row of the gate
    if (what >= 2) {
        // gates that run across the end of a unit (the others are written already), counted by gate or, where there are fewer
        // of them, by the unit whose end is a gate's first such end
        const long long end = (long long)(what - 1) * a.per_unit;
        row0 = a.by_gate ? (long long)(what - 2) * a.S : end / a.S * a.S;
        first = (int)(row0 / a.per_unit);
        last = (int)((row0 + a.S - 1) / a.per_unit) + 1;
        if (last - first == 1 || (!a.by_gate && (row0 == end || first != what - 2))) return;
        p = a.p_gate;
        pitch = 2ll * a.D;
    } else if (!p) {
        return;
    }
    const int each = (last - first + kJoinRuns - 1) / kJoinRuns, lo = first + run * each, hi = min(last, lo + each);
    float sum = 0.f;
    if (in)
#pragma unroll 4
        for (int u = lo; u < hi; ++u) {
            // (a gate that begins inside a unit is that unit's second share)
            const long long second = what >= 2 && row0 > (long long)u * a.per_unit ? a.D : 0;
            sum += p[u * pitch + second + col];
        }
    s[run][threadIdx.x & 31] = sum;
    __syncthreads();
    if (run == 0 && in) {
        sum = 0.f;
#pragma unroll
        for (int k = 0; k < kJoinRuns; ++k) sum += s[k][threadIdx.x & 31];
        if (what == 0) a.dpost[col] = sum;
        else if (what == 1) a.dpre[col] = sum;
        else reinterpret_cast<T*>(a.dgate)[row0 / a.S * a.dgate_ld + col] = from_f32<T>(sum);
    }
}

// ---- host -------------------------------------------------------------------------------------------------------------------
// How rows are dealt out: threads of a unit by the row's length, units by what the device holds at once.
struct Plan {
    int G, P, units, per_unit;
};
Plan plan_of(int64_t rows, int D, int sms, bool backward) {
    Plan p;
    if (D <= 256) p.G = 32, p.P = 1;
    else if (D <= 1024) p.G = 128, p.P = 1;
    else if (D <= 2048) p.G = 256, p.P = 1;
    else if (D <= 4096) p.G = 512, p.P = 1;
    else if (D <= 8192) p.G = 512, p.P = 2;
    else p.G = kLongThreads, p.P = 0;
    const int64_t most = (int64_t)sms * (backward ? (p.G == 32 ? 16 : p.G == 128 ? 4 : p.G == 256 ? 2 : 1) : p.G == 32 ? 32 : 1024 / p.G);
    const int64_t units = rows < most ? rows : most;
    p.per_unit = (int)((rows + units - 1) / units);
    p.units = (int)((rows + p.per_unit - 1) / p.per_unit);
    return p;
}

template <typename T, bool VEC, bool BACKWARD>
int launch_as(const Plan& p, const NormArgs& a, cudaStream_t s) {
    const unsigned grid = (unsigned)(p.G == 32 ? (p.units + 7) / 8 : p.units);
    auto go = [&](auto kernel, int threads) { return (int)rtoss_dev::launch_pdl(kernel, grid, (unsigned)threads, 0, s, a); };
    if (p.P == 0) return go(norm_long_kernel<T, BACKWARD>, kLongThreads);
    if (BACKWARD) {
        if (p.G == 32) return go(norm_backward_kernel<T, VEC, 32, 1>, 256);
        if (p.G == 128) return go(norm_backward_kernel<T, VEC, 128, 1>, 128);
        if (p.G == 256) return go(norm_backward_kernel<T, VEC, 256, 1>, 256);
        if (p.P == 1) return go(norm_backward_kernel<T, VEC, 512, 1>, 512);
        return go(norm_backward_kernel<T, VEC, 512, 2>, 512);
    }
    if (p.G == 32) return go(norm_forward_kernel<T, VEC, 32, 1>, 256);
    if (p.G == 128) return go(norm_forward_kernel<T, VEC, 128, 1>, 128);
    if (p.G == 256) return go(norm_forward_kernel<T, VEC, 256, 1>, 256);
    if (p.P == 1) return go(norm_forward_kernel<T, VEC, 512, 1>, 512);
    return go(norm_forward_kernel<T, VEC, 512, 2>, 512);
}

template <typename T, bool BACKWARD>
int launch(const Plan& p, const NormArgs& a, cudaStream_t s) {
    return a.vec ? launch_as<T, true, BACKWARD>(p, a, s) : launch_as<T, false, BACKWARD>(p, a, s);
}

bool norm_ok(int k) { return k == RTOSS_NORM_NONE || k == RTOSS_NORM_RMS || k == RTOSS_NORM_LAYER; }
int64_t ws_floats(const Plan& p, int D, bool gated) { return (int64_t)p.units * D * (gated ? 4 : 2); }

rtoss_status check(rtoss_ctx* ctx, const rtoss_block_norm* b, bool backward, const char* where) {
    if (!ctx) return RTOSS_ERR_INVALID_ARG;
    if (!b) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "null argument");
    if (b->tokens < 0 || b->D < 1 || b->tokens > kMaxDim || b->D > kMaxDim) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "need 0 <= tokens, 1 <= D, at most 2^30");
    if (b->dtype != RTOSS_F32 && b->dtype != RTOSS_BF16 && b->dtype != RTOSS_F16) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "bad dtype");
    if (!norm_ok(b->post) || !norm_ok(b->pre)) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "bad norm");
    if (!(b->eps >= 0.f)) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "eps must not be negative");
    if (b->gate.dev && (b->tokens_per_gate < 1 || b->tokens % b->tokens_per_gate != 0))
        return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "tokens_per_gate must divide the tokens");
    if (b->tokens == 0) return RTOSS_OK;
    if (b->post == RTOSS_NORM_NONE && (b->post_weight_dev || (backward && b->dpost_weight_dev))) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "a weight of no norm (post)");
    if (b->pre == RTOSS_NORM_NONE && (b->pre_weight_dev || (backward && b->dpre_weight_dev) || (!backward && b->n.dev) || (backward && b->dn.dev)))
        return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "an operand of no norm (pre)");
    if (!b->r.dev || !b->y.dev || (!backward && (!b->z.dev || (b->pre != RTOSS_NORM_NONE && !b->n.dev))) || (backward && (!b->dr.dev || !b->dy.dev)))
        return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "null matrix");
    if (backward && b->dgate.dev && !b->gate.dev) return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "a gradient of no gate");
    const rtoss_rows* m[10] = {&b->r, &b->y, &b->z, &b->n, &b->gate, &b->dz, &b->dn, &b->dr, &b->dy, &b->dgate};
    for (const rtoss_rows* r : m)
        if (r->dev && r->row_stride && (r->row_stride < b->D || r->row_stride > (int64_t)1 << 36))
            return fail(ctx, RTOSS_ERR_INVALID_ARG, where, "a row stride is below the row's length");
    return RTOSS_OK;
}

// Rows that can be moved 16 bytes at a time: D, strides and bases are multiples of what eight values (four fp32 ones) take.
NormArgs args_of(const rtoss_block_norm* b, const Plan& p, bool backward) {
    NormArgs a = {};
    const int es = (int)rtoss_dtype_size(b->dtype);
    bool vec = b->D % 8 == 0;
    auto take = [&](const rtoss_rows& r, long long* ld) {
        *ld = r.row_stride ? r.row_stride : b->D;
        if (r.dev && (!aligned16(r.dev) || (*ld * es) % 16)) vec = false;
        return r.dev;
    };
    a.r = take(b->r, &a.r_ld), a.y = take(b->y, &a.y_ld), a.gate = take(b->gate, &a.gate_ld);
    if (backward) {
        a.dz = take(b->dz, &a.dz_ld), a.dn = take(b->dn, &a.dn_ld), a.dr = take(b->dr, &a.dr_ld), a.dy = take(b->dy, &a.dy_ld), a.dgate = take(b->dgate, &a.dgate_ld);
    } else {
        a.z = take(b->z, &a.z_ld), a.n = take(b->n, &a.n_ld);
    }
    a.wpost = b->post_weight_dev, a.wpre = b->pre_weight_dev;
    a.rows = (int)b->tokens, a.D = b->D, a.post = b->post, a.pre = b->pre, a.vec = vec;
    a.S = b->gate.dev ? (int)b->tokens_per_gate : 1;
    a.per_unit = p.per_unit;
    a.scale = b->residual_scale, a.eps = b->eps;
    return a;
}

template <typename T>
int backward(const rtoss_block_norm* b, const Plan& p, cudaStream_t s) {
    NormArgs a = args_of(b, p, true);
    float* ws = b->workspace_dev;
    const int64_t part = (int64_t)p.units * b->D;
    a.p_post = b->dpost_weight_dev ? ws : nullptr;
    a.p_pre = b->dpre_weight_dev ? ws + part : nullptr;
    a.p_gate = b->dgate.dev ? ws + 2 * part : nullptr;
    if (const int e = launch<T, true>(p, a, s)) return e;
    const bool join_gates = a.dgate && p.units > 1 && p.per_unit % a.S != 0;   // (else every gate's rows were one unit's)
    if (!a.p_post && !a.p_pre && !join_gates) return 0;
    const int gates = (int)(b->tokens / a.S), by_gate = gates < p.units;
    JoinArgs j = {a.p_post, a.p_pre, a.p_gate, b->dpost_weight_dev, b->dpre_weight_dev, a.dgate, a.dgate_ld, b->D, p.units, p.per_unit, a.S, by_gate};
    return (int)rtoss_dev::launch_pdl(norm_join_kernel<T>, dim3((unsigned)((b->D + 31) / 32), (unsigned)(2 + (!join_gates ? 0 : by_gate ? gates : p.units - 1))), dim3(kJoinRuns * 32), 0, s, j);
}

}  // namespace

extern "C" {

rtoss_status rtoss_block_norm_forward(rtoss_ctx* ctx, const rtoss_block_norm* b, void* cuda_stream) {
    const rtoss_status st = check(ctx, b, false, kFwd);
    if (st != RTOSS_OK || b->tokens == 0) return st;
    rtoss_device_guard on_device(ctx->device);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const Plan p = plan_of(b->tokens, b->D, ctx->sm_count > 0 ? ctx->sm_count : 148, false);
    const NormArgs a = args_of(b, p, false);
    return launched(ctx, kFwd, b->dtype == RTOSS_F32 ? launch<float, false>(p, a, s) : b->dtype == RTOSS_BF16 ? launch<__nv_bfloat16, false>(p, a, s) : launch<__half, false>(p, a, s));
}

rtoss_status rtoss_block_norm_workspace(const rtoss_ctx* ctx, int64_t tokens, int D, int gated, int64_t* floats) {
    if (!ctx || !floats || tokens < 0 || D < 1 || tokens > kMaxDim || D > kMaxDim) return RTOSS_ERR_INVALID_ARG;
    *floats = tokens ? ws_floats(plan_of(tokens, D, ctx->sm_count > 0 ? ctx->sm_count : 148, true), D, gated != 0) : 0;
    return RTOSS_OK;
}

rtoss_status rtoss_block_norm_backward(rtoss_ctx* ctx, const rtoss_block_norm* b, void* cuda_stream) {
    const rtoss_status st = check(ctx, b, true, kBwd);
    if (st != RTOSS_OK) return st;
    rtoss_device_guard on_device(ctx->device);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    if (b->tokens == 0) {   // sums of nothing
        int e = b->dpost_weight_dev ? (int)cudaMemsetAsync(b->dpost_weight_dev, 0, sizeof(float) * (size_t)b->D, s) : 0;
        if (!e && b->dpre_weight_dev) e = (int)cudaMemsetAsync(b->dpre_weight_dev, 0, sizeof(float) * (size_t)b->D, s);
        return launched(ctx, kBwd, e);
    }
    const Plan p = plan_of(b->tokens, b->D, ctx->sm_count > 0 ? ctx->sm_count : 148, true);
    if (b->dpost_weight_dev || b->dpre_weight_dev || b->dgate.dev) {
        if (!b->workspace_dev) return fail(ctx, RTOSS_ERR_INVALID_ARG, kBwd, "null workspace");
        if (!aligned16(b->workspace_dev)) return fail(ctx, RTOSS_ERR_ALIGNMENT, kBwd, "the workspace must be 16-byte aligned");
        if (b->workspace_floats < ws_floats(p, b->D, b->dgate.dev != nullptr)) return fail(ctx, RTOSS_ERR_INVALID_ARG, kBwd, "workspace too small");
    }
    return launched(ctx, kBwd, b->dtype == RTOSS_F32 ? backward<float>(b, p, s) : b->dtype == RTOSS_BF16 ? backward<__nv_bfloat16>(b, p, s) : backward<__half>(b, p, s));
}

}  // extern "C"

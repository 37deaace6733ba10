// Host side of the operators over tokens: shared declarations.
#ifndef RTOSS_TOK_INTERNAL_H
#define RTOSS_TOK_INTERNAL_H

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstdio>

#include "rtoss_internal.h"

namespace rtoss_tok {

inline rtoss_status fail(rtoss_ctx* ctx, rtoss_status st, const char* where, const char* what) {
    if (ctx) snprintf(ctx->err, sizeof(ctx->err), "%s: %s", where, what);
    return st;
}
inline rtoss_status launched(rtoss_ctx* ctx, const char* where, int e) {
    return e ? fail(ctx, RTOSS_ERR_CUDA, where, cudaGetErrorString((cudaError_t)e)) : RTOSS_OK;
}
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool act_ok(int a) { return a == RTOSS_ACT_NONE || a == RTOSS_ACT_RELU || a == RTOSS_ACT_SILU; }

constexpr int kMaxDim = 1 << 30;   // tokens and features: coordinates stay well inside 32 bits

// A TMA map of a [rows, cols] matrix whose rows are `stride_bytes` apart; boxes of box_cols x box_rows elements, box rows of
// 64 or 128 bytes with the swizzle of that size.  (tok_maps.cu)
bool encode_rows(CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t rows, int64_t cols, int64_t stride_bytes, int box_cols,
                 int box_rows, int swizzle_bytes);

}  // namespace rtoss_tok

#endif

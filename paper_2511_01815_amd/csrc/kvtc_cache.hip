// Tokens into the pages of a live cache, quantised on the way, and out of it, for gfx950.
//
// A wave to a row (token, head, keys or values): a lane has D / 64 neighbouring features, the largest magnitude or the
// extremes of a group come from lane exchanges.
#include <hip/hip_runtime.h>
#include "kvtc_cache.h"
#include "kvtc_numeric.h"

namespace kvtc {

__device__ __forceinline__ float feature(const uint16_t* x) { return bf16_f32(*x); }
__device__ __forceinline__ float feature(const float* x) { return *x; }
__device__ __forceinline__ void put_feature(uint16_t* x, float v) { *x = f32_bf16(v); }
__device__ __forceinline__ void put_feature(float* x, float v) { *x = v; }

// E4M3 codes of two values within +-448 (or NaN)
__device__ __forceinline__ uint32_t e4m3_pair(float a, float b) { return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xffffu; }

// The place of a row: false if there is none.
struct RowAt { int64_t row, scale; };
__device__ __forceinline__ bool row_of(const CacheTokenArgs& a, int64_t token, int head, RowAt& at) {
    const int64_t slot = a.slots[token];
    if (slot < 0) return false;
    const int64_t page = slot / a.c.page_tokens, in = slot - page * a.c.page_tokens;
    if (page >= a.c.n_pages) {
        if (head == 0) report_lowest(a.status, (uint32_t)token);
        return false;
    }
    at.row = page * a.c.page_stride + head * a.c.head_stride + in * a.c.token_stride;
    at.scale = (page * a.c.n_heads + head) * a.c.page_tokens + in;
    return true;
}

template <typename XT, int F, int D>
__global__ void __launch_bounds__(256) cache_write_kernel(const CacheTokenArgs a) {
    constexpr int N = D / 64;                              // features of a lane
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = a.n_tokens * a.c.n_heads * 2;
    for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < rows; r += (int64_t)gridDim.x * 4) {
        const int side = (int)(r & 1);
        const int64_t token = (r >> 1) / a.c.n_heads;
        const int head = (int)((r >> 1) - token * a.c.n_heads);
        RowAt at;
        if (!row_of(a, token, head, at)) continue;
        const XT* x = static_cast<const XT*>(side ? a.v : a.k) + token * a.token_stride + head * a.head_stride + lane * N;
        uint8_t* row = static_cast<uint8_t*>(side ? a.c.v_dev : a.c.k_dev) + at.row;
        uint8_t* scales = static_cast<uint8_t*>(side ? a.c.v_scales_dev : a.c.k_scales_dev);
        float v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = feature(x + i);
        if (F == KVTC_CACHE_BF16) {
#pragma unroll
            for (int i = 0; i < N; ++i) reinterpret_cast<uint16_t*>(row)[lane * N + i] = f32_bf16(v[i]);
        } else if (F == KVTC_CACHE_FP8) {
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float m = __builtin_fabsf(v[i]);
                most = m < __builtin_huge_valf() && m > most ? m : most;
            }
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d, 64));
            float scale = div_rn(most, 448.0f);
            if (scale < 0x1p-126f) scale = 0.0f;
            const float inv = scale > 0.0f ? div_rn(1.0f, scale) : 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float y = v[i] * inv, z = v[i] == v[i] && scale > 0.0f ? fminf(fmaxf(y, -448.0f), 448.0f) : (v[i] == v[i] ? 0.0f : v[i]);
                row[lane * N + i] = (uint8_t)e4m3_pair(z, z);
            }
            if (lane == 0) reinterpret_cast<float*>(scales)[at.scale] = scale;
        } else {
            constexpr int kLanes = kCacheGroup / N;        // of a group
            float lo = v[0], hi = v[0];
#pragma unroll
            for (int i = 1; i < N; ++i) { lo = fminf(lo, v[i]); hi = fmaxf(hi, v[i]); }
#pragma unroll
            for (int d = kLanes / 2; d > 0; d >>= 1) { lo = fminf(lo, __shfl_xor(lo, d, 64)); hi = fmaxf(hi, __shfl_xor(hi, d, 64)); }
            const GroupQ g = group_header(lo, hi, 4);
            uint32_t code[N];
#pragma unroll
            for (int i = 0; i < N; ++i) code[i] = (uint32_t)code_of(v[i], g.shift, g.inv, 15.0f) & 15u;
            if (lane % kLanes == 0) reinterpret_cast<uint32_t*>(scales)[at.scale * (D / kCacheGroup) + lane / kLanes] = (uint32_t)g.shift16 | (uint32_t)g.scale16 << 16;
            if (N == 1) {
                const uint32_t next = (uint32_t)__shfl_down((int)code[0], 1, 64);
                if ((lane & 1) == 0) row[(lane % 32) / 2 * (D / kCacheGroup) + lane / 32] = (uint8_t)(code[0] | next << 4);
            } else {
#pragma unroll
                for (int i = 0; i + 1 < N; i += 2) {
                    const int f = lane * N + i;
                    row[(f % kCacheGroup) / 2 * (D / kCacheGroup) + f / kCacheGroup] = (uint8_t)(code[i] | code[i + 1 < N ? i + 1 : i] << 4);
                }
            }
        }
    }
}

// A value of a row as the cache holds it.
template <int F, int D>
__device__ __forceinline__ float cache_value(const uint8_t* row, const uint8_t* scales, int64_t scale_at, int f) {
    if (F == KVTC_CACHE_BF16) return bf16_f32(reinterpret_cast<const uint16_t*>(row)[f]);
    if (F == KVTC_CACHE_FP8) return __builtin_amdgcn_cvt_f32_fp8((int)row[f], 0) * reinterpret_cast<const float*>(scales)[scale_at];
    const uint32_t header = reinterpret_cast<const uint32_t*>(scales)[scale_at * (D / kCacheGroup) + f / kCacheGroup];
    const uint32_t code = row[(f % kCacheGroup) / 2 * (D / kCacheGroup) + f / kCacheGroup] >> (4 * (f & 1)) & 15u;
    return __builtin_fmaf((float)code, f16_bits_to_f32((uint16_t)(header >> 16)), f16_bits_to_f32((uint16_t)header));
}

template <typename XT, int F, int D>
__global__ void __launch_bounds__(256) cache_read_kernel(const CacheTokenArgs a) {
    constexpr int N = D / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t rows = a.n_tokens * a.c.n_heads * 2;
    for (int64_t r = (int64_t)blockIdx.x * 4 + wave; r < rows; r += (int64_t)gridDim.x * 4) {
        const int side = (int)(r & 1);
        const int64_t token = (r >> 1) / a.c.n_heads;
        const int head = (int)((r >> 1) - token * a.c.n_heads);
        XT* x = static_cast<XT*>(side ? a.v : a.k) + token * a.token_stride + head * a.head_stride + lane * N;
        RowAt at;
        const bool is = row_of(a, token, head, at);
        const uint8_t* row = static_cast<const uint8_t*>(side ? a.c.v_dev : a.c.k_dev) + (is ? at.row : 0);
        const uint8_t* scales = static_cast<const uint8_t*>(side ? a.c.v_scales_dev : a.c.k_scales_dev);
#pragma unroll
        for (int i = 0; i < N; ++i) put_feature(x + i, is ? cache_value<F, D>(row, scales, at.scale, lane * N + i) : 0.0f);
    }
}

template <bool kWrite, typename XT, int F>
hipError_t launch_tokens(const CacheTokenArgs& a, hipStream_t stream) {
    const int64_t rows = a.n_tokens * a.c.n_heads * 2, want = (rows + 3) / 4;
    const dim3 grid((uint32_t)(want < 65536 ? want : 65536)), block(256);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a); };
    if (a.c.d_head == 64) { if constexpr (kWrite) go(cache_write_kernel<XT, F, 64>); else go(cache_read_kernel<XT, F, 64>); }
    else if (a.c.d_head == 128) { if constexpr (kWrite) go(cache_write_kernel<XT, F, 128>); else go(cache_read_kernel<XT, F, 128>); }
    else { if constexpr (kWrite) go(cache_write_kernel<XT, F, 256>); else go(cache_read_kernel<XT, F, 256>); }
    return hipGetLastError();
}
template <bool kWrite, typename XT>
hipError_t launch_format(const CacheTokenArgs& a, hipStream_t stream) {
    if (a.c.format == KVTC_CACHE_BF16) return launch_tokens<kWrite, XT, KVTC_CACHE_BF16>(a, stream);
    if (a.c.format == KVTC_CACHE_FP8) return launch_tokens<kWrite, XT, KVTC_CACHE_FP8>(a, stream);
    return launch_tokens<kWrite, XT, KVTC_CACHE_INT4>(a, stream);
}

hipError_t launch_cache_write(const CacheTokenArgs& a, kvtc_dtype dtype, hipStream_t stream) {
    return dtype == KVTC_BF16 ? launch_format<true, uint16_t>(a, stream) : launch_format<true, float>(a, stream);
}
hipError_t launch_cache_read(const CacheTokenArgs& a, kvtc_dtype dtype, hipStream_t stream) {
    return dtype == KVTC_BF16 ? launch_format<false, uint16_t>(a, stream) : launch_format<false, float>(a, stream);
}

}  // namespace kvtc

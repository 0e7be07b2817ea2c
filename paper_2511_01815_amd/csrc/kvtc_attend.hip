// Attention of one new token of every sequence over the pages of a live cache, for gfx950.
//
// One pass over keys and values with the running maximum m and sum l of a softmax: for a score s,
//     m' = max(m, s),  l' = l e^(m - m') + e^(s - m'),  o' = o e^(m - m') + e^(s - m') v.
// A workgroup has a (sequence, query head), its waves every fourth token each, joined in the LDS at the end; a lane has D / 64
// features of the token in hand.
#include <hip/hip_runtime.h>
#include "kvtc_cache.h"
#include "kvtc_numeric.h"

namespace kvtc {

__device__ __forceinline__ float query(const uint16_t* x) { return bf16_f32(*x); }
__device__ __forceinline__ float query(const float* x) { return *x; }
__device__ __forceinline__ void put_out(uint16_t* x, float v) { *x = f32_bf16(v); }
__device__ __forceinline__ void put_out(float* x, float v) { *x = v; }

template <int F, int D>
__device__ __forceinline__ float cache_value(const uint8_t* row, const uint8_t* scales, int64_t scale_at, int f) {
    if (F == KVTC_CACHE_BF16) return bf16_f32(reinterpret_cast<const uint16_t*>(row)[f]);
    if (F == KVTC_CACHE_FP8) return __builtin_amdgcn_cvt_f32_fp8((int)row[f], 0) * reinterpret_cast<const float*>(scales)[scale_at];
    const uint32_t header = reinterpret_cast<const uint32_t*>(scales)[scale_at * (D / kCacheGroup) + f / kCacheGroup];
    const uint32_t code = row[(f % kCacheGroup) / 2 * (D / kCacheGroup) + f / kCacheGroup] >> (4 * (f & 1)) & 15u;
    return __builtin_fmaf((float)code, f16_bits_to_f32((uint16_t)(header >> 16)), f16_bits_to_f32((uint16_t)header));
}

template <typename XT, int F, int D>
__global__ void __launch_bounds__(256) attend_kernel(const AttendArgs a) {
    constexpr int N = D / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int b = (int)(blockIdx.x / (uint32_t)a.n_q_heads), hq = (int)(blockIdx.x - (uint32_t)b * (uint32_t)a.n_q_heads), h = hq / (a.n_q_heads / a.c.n_heads);
    int64_t length = a.lengths[b];
    if (length < 0 || length > a.max_tokens) {
        if (threadIdx.x == 0) report_lowest(a.status, (uint32_t)b);
        length = 0;
    }
    const int64_t from = a.window ? length - a.window : 0;
    const XT* q = static_cast<const XT*>(a.q) + b * a.q_seq_stride + hq * a.q_head_stride + lane * N;
    float qv[N], o[N], m = -__builtin_huge_valf(), l = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) { qv[i] = query(q + i) * a.scale; o[i] = 0.0f; }
    for (int64_t t = wave; t < length; t += 4) {
        if (t >= a.sinks && t < from) continue;
        const int64_t index = t / a.c.page_tokens, in = t - index * a.c.page_tokens, page = a.pages[b * a.pages_stride + index];
        if (page < 0 || page >= a.c.n_pages) {
            if (lane == 0) report_lowest(a.status, (uint32_t)b);
            continue;
        }
        const int64_t at = page * a.c.page_stride + h * a.c.head_stride + in * a.c.token_stride, scale_at = (page * a.c.n_heads + h) * a.c.page_tokens + in;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) s += qv[i] * cache_value<F, D>(static_cast<const uint8_t*>(a.c.k_dev) + at, static_cast<const uint8_t*>(a.c.k_scales_dev), scale_at, lane * N + i);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d, 64);
        const float top = fmaxf(m, s), base = top == -__builtin_huge_valf() ? 0.0f : top, keep = expf(m - base), p = expf(s - base);
        l = l * keep + p;
#pragma unroll
        for (int i = 0; i < N; ++i)
            o[i] = o[i] * keep + p * cache_value<F, D>(static_cast<const uint8_t*>(a.c.v_dev) + at, static_cast<const uint8_t*>(a.c.v_scales_dev), scale_at, lane * N + i);
        m = top;
    }
    __shared__ float part[4][D + 2];
#pragma unroll
    for (int i = 0; i < N; ++i) part[wave][lane * N + i] = o[i];
    if (lane == 0) { part[wave][D] = m; part[wave][D + 1] = l; }
    __syncthreads();
    if (wave != 0) return;
    float top = part[0][D];
    for (int w = 1; w < 4; ++w) top = fmaxf(top, part[w][D]);
    const float base = top == -__builtin_huge_valf() ? 0.0f : top;
    float total = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = 0.0f;
    for (int w = 0; w < 4; ++w) {
        const float keep = expf(part[w][D] - base);
        total += part[w][D + 1] * keep;
#pragma unroll
        for (int i = 0; i < N; ++i) o[i] += part[w][lane * N + i] * keep;
    }
    const int64_t row = (int64_t)b * a.n_q_heads + hq;
    XT* out = static_cast<XT*>(a.out) + row * D + lane * N;
#pragma unroll
    for (int i = 0; i < N; ++i) put_out(out + i, total == 0.0f ? 0.0f : o[i] / total);
    if (a.lse && lane == 0) a.lse[row] = base + logf(total);
}

size_t attend_work_bytes(const kvtc_cache&, int, int, int64_t) { return 256; }

template <typename XT, int F>
hipError_t launch_d(const AttendArgs& a, hipStream_t stream) {
    const dim3 grid((uint32_t)a.n_seqs * (uint32_t)a.n_q_heads), block(256);
    if (a.c.d_head == 64) hipLaunchKernelGGL((attend_kernel<XT, F, 64>), grid, block, 0, stream, a);
    else if (a.c.d_head == 128) hipLaunchKernelGGL((attend_kernel<XT, F, 128>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((attend_kernel<XT, F, 256>), grid, block, 0, stream, a);
    return hipGetLastError();
}
template <typename XT>
hipError_t launch_format(const AttendArgs& a, hipStream_t stream) {
    if (a.c.format == KVTC_CACHE_BF16) return launch_d<XT, KVTC_CACHE_BF16>(a, stream);
    if (a.c.format == KVTC_CACHE_FP8) return launch_d<XT, KVTC_CACHE_FP8>(a, stream);
    return launch_d<XT, KVTC_CACHE_INT4>(a, stream);
}
hipError_t launch_attend(const AttendArgs& a, kvtc_dtype dtype, hipStream_t stream) {
    return dtype == KVTC_BF16 ? launch_format<uint16_t>(a, stream) : launch_format<float>(a, stream);
}

}  // namespace kvtc

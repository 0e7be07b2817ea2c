// Attention over several sets of tokens, worked out apart, joined to attention over all of them, for gfx950.
//
// Of a row's parts (out_p, lse_p), with m = max lse_p:   out = sum_p e^(lse_p - m) out_p / sum_p e^(lse_p - m),   lse = m + log sum_p e^(lse_p - m).
// A lane has eight neighbouring features of a row in all parts, one part after another: its log-sum, then, unless that is minus infinity (the row may hold anything), the features.  Large calls are bound by memory, with waves
// enough to cover that (3 fp32 parts of 6001 rows of 32 heads of 128 into bf16, 347 MB: 64 us, 5.4 TB/s), small ones by the launch and by two latencies to a part (64 rows of 2 parts 3.5 us in the kernel, of 16 parts 10.6).
#include <hip/hip_runtime.h>
#include <cmath>
#include "kvtc_cache.h"
#include "kvtc_dev.h"

namespace kvtc {
kvtc_status set_error(kvtc_status st, const char* fmt, ...);

constexpr int kJoinParts = 16;

struct JoinArgs {
    const void* outs[kJoinParts];
    const float* lses[kJoinParts];
    void* out;
    float* lse;
    int64_t rows;                                          // rows and heads
    int32_t parts;
};

typedef uint32_t join_u32x4 __attribute__((ext_vector_type(4)));
template <typename XT> struct Eight;
template <> struct Eight<uint16_t> {
    join_u32x4 w;
    __device__ __forceinline__ void load(const uint16_t* p) { w = *reinterpret_cast<const join_u32x4*>(p); }
    __device__ __forceinline__ float at(int i) const { return i % 2 ? __uint_as_float(w[i / 2] & 0xffff0000u) : __uint_as_float(w[i / 2] << 16); }
};
template <> struct Eight<float> {
    join_u32x4 w[2];
    __device__ __forceinline__ void load(const float* p) {
        w[0] = reinterpret_cast<const join_u32x4*>(p)[0];
        w[1] = reinterpret_cast<const join_u32x4*>(p)[1];
    }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i / 4][i % 4]); }
};

template <typename XT, typename OT, int D>
__global__ void __launch_bounds__(256) join_kernel(const JoinArgs a) {
    constexpr int LANES = D / 8;                           // of a row: within a wave, so that all of a row is read before any of it is written over
    const int64_t step = (int64_t)gridDim.x * (256 / LANES);
    const int at = threadIdx.x % LANES * 8;
    for (int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES; row < a.rows; row += step) {
        float top = -__builtin_huge_valf(), sum = 0.0f, o[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        for (int p = 0; p < a.parts; ++p) top = fmaxf(top, a.lses[p][row]);
        const float base = top == -__builtin_huge_valf() ? 0.0f : top;
        for (int p = 0; p < a.parts; ++p) {
            const float lse = a.lses[p][row], share = expf(lse - base);
            if (lse == -__builtin_huge_valf()) continue;   // (a part without a token: its row may hold anything)
            Eight<XT> x;
            x.load(static_cast<const XT*>(a.outs[p]) + row * D + at);
            sum += share;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = __builtin_fmaf(share, x.at(i), o[i]);
        }
        const bool none = sum == 0.0f;
        const float inverse = none ? 0.0f : 1.0f / sum;
        OT* to = static_cast<OT*>(a.out) + row * D + at;
        if constexpr (sizeof(OT) == 2) {
            join_u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_bf16(o[2 * i] * inverse) | (uint32_t)f32_bf16(o[2 * i + 1] * inverse) << 16;
            *reinterpret_cast<join_u32x4*>(to) = w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = o[i] * inverse;
        }
        if (a.lse && at == 0) a.lse[row] = none ? -__builtin_huge_valf() : base + logf(sum);
    }
}

template <typename XT, typename OT>
static hipError_t launch_join(const JoinArgs& a, int d, hipStream_t stream) {
    const int64_t each = 256 / (d / 8), blocks = (a.rows + each - 1) / each, most = (int64_t)1 << 23;
    const dim3 grid((uint32_t)(blocks < most ? blocks : most));
    if (d == 64) hipLaunchKernelGGL((join_kernel<XT, OT, 64>), grid, dim3(256), 0, stream, a);
    else if (d == 128) hipLaunchKernelGGL((join_kernel<XT, OT, 128>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((join_kernel<XT, OT, 256>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvtc

extern "C" kvtc_status kvtc_attend_join(int n_parts, const void* const* part_outs, const float* const* part_lses, kvtc_dtype part_dtype, int64_t n_rows, int n_heads, int d_head, void* out_dev,
                                        kvtc_dtype out_dtype, float* lse_dev, kvtc_stream stream) {
    using namespace kvtc;
    if (n_parts < 1 || n_parts > kJoinParts) return set_error(KVTC_E_ARG, "kvtc_attend_join: n_parts=%d outside 1..%d", n_parts, kJoinParts);
    if ((part_dtype != KVTC_BF16 && part_dtype != KVTC_F32) || (out_dtype != KVTC_BF16 && out_dtype != KVTC_F32)) return set_error(KVTC_E_ARG, "kvtc_attend_join: unknown dtype %d or %d", (int)part_dtype, (int)out_dtype);
    if (n_rows < 0 || n_rows > 0x7fffffffLL) return set_error(KVTC_E_ARG, "kvtc_attend_join: n_rows=%lld", (long long)n_rows);
    if (n_heads < 1 || n_heads > kCacheMaxHeads) return set_error(KVTC_E_ARG, "kvtc_attend_join: n_heads=%d outside 1..%d", n_heads, kCacheMaxHeads);
    if (d_head != 64 && d_head != 128 && d_head != 256) return set_error(KVTC_E_UNSUPPORTED, "kvtc_attend_join: d_head=%d (64, 128 and 256 are served)", d_head);
    if (n_rows == 0) return KVTC_OK;
    if (!part_outs || !part_lses || !out_dev) return set_error(KVTC_E_ARG, "kvtc_attend_join: null buffer");
    JoinArgs a{};
    for (int p = 0; p < n_parts; ++p) {
        if (!part_outs[p] || !part_lses[p]) return set_error(KVTC_E_ARG, "kvtc_attend_join: null part %d", p);
        if ((reinterpret_cast<uintptr_t>(part_outs[p]) & 15u) || (reinterpret_cast<uintptr_t>(part_lses[p]) & 3u)) return set_error(KVTC_E_ARG, "kvtc_attend_join: part %d is not aligned (16 bytes, its lse 4)", p);
        a.outs[p] = part_outs[p];
        a.lses[p] = part_lses[p];
    }
    if ((reinterpret_cast<uintptr_t>(out_dev) & 15u) || (reinterpret_cast<uintptr_t>(lse_dev) & 3u)) return set_error(KVTC_E_ARG, "kvtc_attend_join: the output is not aligned (16 bytes, its lse 4)");
    if (part_dtype != out_dtype)
        for (int p = 0; p < n_parts; ++p)
            if (part_outs[p] == out_dev) return set_error(KVTC_E_ARG, "kvtc_attend_join: the output has part %d's place, but another type", p);
    a.out = out_dev;
    a.lse = lse_dev;
    a.rows = n_rows * n_heads;
    a.parts = n_parts;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (part_dtype == KVTC_BF16) e = out_dtype == KVTC_BF16 ? launch_join<uint16_t, uint16_t>(a, d_head, st) : launch_join<uint16_t, float>(a, d_head, st);
    else e = out_dtype == KVTC_BF16 ? launch_join<float, uint16_t>(a, d_head, st) : launch_join<float, float>(a, d_head, st);
    if (e != hipSuccess) return set_error(KVTC_E_HIP, "kvtc_attend_join: launch failed: %s", hipGetErrorString(e));
    return KVTC_OK;
}

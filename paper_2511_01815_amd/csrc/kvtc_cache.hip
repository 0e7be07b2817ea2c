// Tokens into the pages of a live cache, quantised on the way, and out of it, for gfx950.
//
// Formats (per row = token, head, keys or values; d features):
//   bf16   the features
//   fp8    a = largest finite magnitude, scale = a * (1/448) in fp32, codes = e4m3(x * (1/scale))
//   int4   per 32 features: shift = fp16 downwards of the least, scale = fp16 upwards of (most - shift) * (1/15), codes =
//          clamp(rne((x - shift) * (1/scale)), 0, 15); byte pair * (d/32) + group of the row has the codes of features 2 pair, 2 pair + 1 of the
//          group, so that d/32 neighbouring bytes are of one pair (what the attention's matrix products take in one piece)
// Streaming kernels, bound by memory: a lane has 8 neighbouring features (16 bytes of bf16) of ROWS rows, whose loads are on their way together; a row's d/8 lanes
// find its extremes by lane exchanges.  32768 tokens of 8 heads of 128 bf16 features, 192 MB in all: into 8 bits 45 us, 4.5 TB/s (a copy of as much 43), out of 4 bits 39.5; one token of each
// of 64 caches 2.2, a launch's time (replayed from a graph; 5.4 a call where each is launched by itself).
#include <hip/hip_runtime.h>
#include "kvtc_cache.h"
#include "kvtc_numeric.h"

namespace kvtc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// n / d for n < 2^31, by one product (m = ceil(2^(31 + s) / d), s = ceil(log2 d): its excess over 2^(31 + s) / d is below 2^s / d, so n times it stays below the next quotient)
struct Divisor { uint32_t d, mul, shift; };
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divisor& v) { return (uint32_t)(((uint64_t)n * v.mul) >> v.shift); }
Divisor divisor_of(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return {d, (uint32_t)(((1ull << (31 + s)) + d - 1) / d), 31 + s};
}

struct TokenArgs { CacheTokenArgs t; Divisor heads, page; uint32_t token0; };      // token0: of the launch's first token, in the call

// Place of a token in the pool.
struct Place { uint32_t page, in; bool is; };
__device__ __forceinline__ Place place_of(const TokenArgs& a, uint32_t token, int64_t slot, bool first) {
    Place p{0u, 0u, false};
    if (slot < 0) return p;
    int64_t page, in;
    if (slot < 0x80000000LL) {
        page = divide((uint32_t)slot, a.page);
        in = slot - page * (int64_t)a.page.d;
    } else {
        page = slot / a.page.d;
        in = slot - page * a.page.d;
    }
    if (page >= a.t.c.n_pages) {
        if (first) report_lowest(a.t.status, a.token0 + token);
        return p;
    }
    return {(uint32_t)page, (uint32_t)in, true};
}

__device__ __forceinline__ void load_features(const uint16_t* x, float* v) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(x);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_f32(w[i] & 0xffffu); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void load_features(const float* x, float* v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const u32x4 w = reinterpret_cast<const u32x4*>(x)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * i + j] = __uint_as_float(w[j]);
    }
}
__device__ __forceinline__ u32x4 pack_bf16(const float* v) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_bf16(v[2 * i]) | (uint32_t)f32_bf16(v[2 * i + 1]) << 16;
    return w;
}
__device__ __forceinline__ void store_features(uint16_t* x, const float* v) { *reinterpret_cast<u32x4*>(x) = pack_bf16(v); }
__device__ __forceinline__ void store_features(float* x, const float* v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<u32x4*>(x)[i] = u32x4{__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
}

// A row's codes of 4 bits change hands on their way in and out: lane (group g, quarter j) of the row has the codes of pairs 4j .. 4j + 3 of
// its group, a byte each, and dword g of the 4 G bytes of those pairs holds bytes [pair][group] (G = D/32 groups, as many lanes).  Byte k of that dword: place 4g + k.
template <int G>
__device__ __forceinline__ uint32_t pairs_to_row(uint32_t mine, int lane) {
    const int j = lane & 3, g = lane >> 2 & (G - 1), base = lane & ~(4 * G - 1);
    uint32_t out = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int at = 4 * g + k, pair = at / G, group = at % G;
        out |= ((uint32_t)__shfl((int)mine, base + group * 4 + j, 64) >> (8 * pair) & 0xffu) << (8 * k);
    }
    return out;
}
template <int G>
__device__ __forceinline__ uint32_t row_to_pairs(uint32_t row, int lane) {
    const int j = lane & 3, g = lane >> 2 & (G - 1), base = lane & ~(4 * G - 1);
    uint32_t out = 0;
#pragma unroll
    for (int pair = 0; pair < 4; ++pair) {
        const int at = pair * G + g;
        out |= ((uint32_t)__shfl((int)row, base + (at >> 2) * 4 + j, 64) >> (8 * (at & 3)) & 0xffu) << (8 * pair);
    }
    return out;
}
// the dword of a row (of D/8) that holds what pairs_to_row gives a lane
template <int G> __device__ __forceinline__ int row_dword(int lane) { return (lane & 3) * G + (lane >> 2 & (G - 1)); }

// The largest of a row's lanes (LANES neighbouring ones).
template <int LANES, typename OP>
__device__ __forceinline__ float over_lanes(float v, OP op) {
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) v = op(v, __shfl_xor(v, d, 64));
    return v;
}

template <typename XT, int F, int D, int ROWS>
__global__ void __launch_bounds__(256) cache_write_kernel(const TokenArgs a) {
    constexpr int L = D / 8, G = D / kCacheGroup;          // lanes of a row; groups of a row
    const int lane = threadIdx.x & 63, at = threadIdx.x % L;
    const bool side = blockIdx.y;
    const CacheTokenArgs& t = a.t;
    const uint32_t rows = (uint32_t)t.n_tokens * (uint32_t)t.c.n_heads, row0 = blockIdx.x * (uint32_t)(ROWS * 256 / L) + threadIdx.x / L;
    const XT* x = static_cast<const XT*>(side ? t.v : t.k);
    float v[ROWS][8];
    int64_t slot[ROWS];
    uint32_t token[ROWS], head[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const uint32_t r = row0 + u * (256 / L), rr = r < rows ? r : 0;      // (past the end: the first row, not stored)
        token[u] = divide(rr, a.heads);
        head[u] = rr - token[u] * a.heads.d;
        load_features(x + (int64_t)token[u] * t.token_stride + (int64_t)head[u] * t.head_stride + at * 8, v[u]);
        slot[u] = t.slots[token[u]];
        if (r >= rows) slot[u] = -1;
    }
    uint8_t* rows_out = static_cast<uint8_t*>(side ? t.c.v_dev : t.c.k_dev);
    void* scales_out = side ? t.c.v_scales_dev : t.c.k_scales_dev;
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const Place p = place_of(a, token[u], slot[u], at == 0 && head[u] == 0);
        uint8_t* row = rows_out + (int64_t)p.page * t.c.page_stride + (int64_t)head[u] * t.c.head_stride + (int64_t)p.in * t.c.token_stride;
        const int64_t scale_at = ((int64_t)p.page * t.c.n_heads + head[u]) * t.c.page_tokens + p.in;
        if constexpr (F == KVTC_CACHE_BF16) {
            if (p.is) reinterpret_cast<u32x4*>(row)[at] = pack_bf16(v[u]);
        } else if constexpr (F == KVTC_CACHE_FP8) {
            float most = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, __builtin_fabsf(v[u][i]));
            if (__any(most == __builtin_huge_valf())) {    // an infinity: the largest of the others
                most = 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) { const float m = __builtin_fabsf(v[u][i]); most = m < __builtin_huge_valf() ? fmaxf(most, m) : most; }
            }
            most = over_lanes<L>(most, [](float p, float q) { return fmaxf(p, q); });
            float scale = most * (1.0f / 448.0f);
            if (scale < 0x1p-126f) scale = 0.0f;
            const float inv = scale > 0.0f ? div_rn(1.0f, scale) : 0.0f;
            float z[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float w = v[u][i];
                // (no scale: zero, also for an infinity, whose product with zero is none.  The clamp would make a number of NaN.)
                const float y = __builtin_amdgcn_fmed3f(__builtin_amdgcn_fmed3f(w, -0x1.fffffep127f, 0x1.fffffep127f) * inv, -448.0f, 448.0f);
                z[i] = w == w ? y : w;
            }
            u32x2 c;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int low = __builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i], z[4 * i + 1], 0, false);
                c[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(z[4 * i + 2], z[4 * i + 3], low, true);
            }
            if (p.is) {
                reinterpret_cast<u32x2*>(row)[at] = c;
                if (at == 0) static_cast<float*>(scales_out)[scale_at] = scale;
            }
        } else {
            float lo = v[u][0], hi = v[u][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) { lo = fminf(lo, v[u][i]); hi = fmaxf(hi, v[u][i]); }
            lo = over_lanes<4>(lo, [](float p, float q) { return fminf(p, q); });
            hi = over_lanes<4>(hi, [](float p, float q) { return fmaxf(p, q); });
            float shift, scale;
            const uint32_t shift16 = f16_round_dir_dev(lo, false, shift);
            const uint32_t scale16 = f16_round_dir_dev(__fmul_rn(__fsub_rn(hi, shift), 1.0f / 15.0f), true, scale);
            const float inv = scale > 0.0f ? rcp_rn_dev(scale) : 0.0f;
            uint32_t pairs = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) pairs |= ((uint32_t)code_of(v[u][i], shift, inv, 15.0f) & 15u) << (4 * i);
            const uint32_t mine = pairs_to_row<G>(pairs, lane);
            if (p.is) {
                reinterpret_cast<uint32_t*>(row)[row_dword<G>(lane)] = mine;
                if ((at & 3) == 0) static_cast<uint32_t*>(scales_out)[scale_at * G + at / 4] = (shift16 & 0xffffu) | scale16 << 16;
            }
        }
    }
}

template <typename XT, int F, int D, int ROWS>
__global__ void __launch_bounds__(256) cache_read_kernel(const TokenArgs a) {
    constexpr int L = D / 8, G = D / kCacheGroup;
    const int lane = threadIdx.x & 63, at = threadIdx.x % L;
    const bool side = blockIdx.y;
    const CacheTokenArgs& t = a.t;
    const uint32_t rows = (uint32_t)t.n_tokens * (uint32_t)t.c.n_heads, row0 = blockIdx.x * (uint32_t)(ROWS * 256 / L) + threadIdx.x / L;
    int64_t slot[ROWS];
    uint32_t token[ROWS], head[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const uint32_t r = row0 + u * (256 / L), rr = r < rows ? r : 0;
        token[u] = divide(rr, a.heads);
        head[u] = rr - token[u] * a.heads.d;
        slot[u] = t.slots[token[u]];
    }
    const uint8_t* rows_in = static_cast<const uint8_t*>(side ? t.c.v_dev : t.c.k_dev);
    const void* scales_in = side ? t.c.v_scales_dev : t.c.k_scales_dev;
    u32x4 held[ROWS];
    uint32_t scale[ROWS];
    bool is[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const Place p = place_of(a, token[u], slot[u], at == 0 && head[u] == 0);
        is[u] = p.is;
        // (no place: the pool's first row, not used)
        const uint32_t h = p.is ? head[u] : 0u;
        const uint8_t* row = rows_in + (int64_t)p.page * t.c.page_stride + (int64_t)h * t.c.head_stride + (int64_t)p.in * t.c.token_stride;
        const int64_t scale_at = ((int64_t)p.page * t.c.n_heads + h) * t.c.page_tokens + p.in;
        if constexpr (F == KVTC_CACHE_BF16) {
            held[u] = reinterpret_cast<const u32x4*>(row)[at];
        } else if constexpr (F == KVTC_CACHE_FP8) {
            const u32x2 w = reinterpret_cast<const u32x2*>(row)[at];
            held[u][0] = w[0];
            held[u][1] = w[1];
            scale[u] = static_cast<const uint32_t*>(scales_in)[scale_at];
        } else {
            held[u][0] = reinterpret_cast<const uint32_t*>(row)[row_dword<G>(lane)];
            scale[u] = static_cast<const uint32_t*>(scales_in)[scale_at * G + at / 4];
        }
    }
    XT* x = static_cast<XT*>(side ? t.v : t.k);
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        float v[8];
        if constexpr (F == KVTC_CACHE_BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[2 * i] = bf16_f32(held[u][i] & 0xffffu); v[2 * i + 1] = __uint_as_float(held[u][i] & 0xffff0000u); }
        } else if constexpr (F == KVTC_CACHE_FP8) {
            const float s = __uint_as_float(scale[u]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const auto low = __builtin_amdgcn_cvt_pk_f32_fp8((int)held[u][i], false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)held[u][i], true);
                v[4 * i] = low[0] * s;
                v[4 * i + 1] = low[1] * s;
                v[4 * i + 2] = high[0] * s;
                v[4 * i + 3] = high[1] * s;
            }
        } else {
            const uint32_t pairs = row_to_pairs<G>(held[u][0], lane);
            const float shift = (float)__builtin_bit_cast(_Float16, (uint16_t)scale[u]), s = (float)__builtin_bit_cast(_Float16, (uint16_t)(scale[u] >> 16));
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_fmaf((float)(pairs >> (4 * i) & 15u), s, shift);
        }
        if (!is[u]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.0f;
        }
        if (row0 + u * (256 / L) < rows) store_features(x + (int64_t)token[u] * t.token_stride + (int64_t)head[u] * t.head_stride + at * 8, v);
    }
}

template <bool kWrite, typename XT, int F, int D, int ROWS>
void launch_rows(const TokenArgs& a, hipStream_t stream) {
    constexpr int64_t kEach = ROWS * 256 / (D / 8);        // rows of a workgroup
    const dim3 grid((uint32_t)((a.t.n_tokens * a.t.c.n_heads + kEach - 1) / kEach), 2), block(256);
    if constexpr (kWrite) hipLaunchKernelGGL((cache_write_kernel<XT, F, D, ROWS>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((cache_read_kernel<XT, F, D, ROWS>), grid, block, 0, stream, a);
}

// Four rows to a lane, quantised bf16 only, from where they gain: with more to wait for per lane, and a quarter of the waves, a call that does not fill the chip many times over
// is longer.  (us, one row and four.  Into 8 bits, 8 heads of 128: 64 tokens 2.2 and 3.8, 9001 12.9 and 14.0, 32768 49.6 and 45.3, 60000 81 and 73; out of 4 bits 2000 4.5 and 4.6, 9001 13.0 and
// 11.4, 32768 59 and 40.  bf16 pages, in and out, 32768 49.5 and 50.6, fp32 features, 4 heads of 64, 60000 into 8 bits 30.0 and 31.8, out 37.6 and 43.4: never.)
template <bool kWrite, typename XT, int F, int D>
hipError_t launch_tokens(const CacheTokenArgs& all, int64_t most, hipStream_t stream) {
    for (int64_t from = 0; from < all.n_tokens; from += most) {
        TokenArgs a{all, divisor_of((uint32_t)all.c.n_heads), divisor_of((uint32_t)all.c.page_tokens), (uint32_t)from};
        a.t.n_tokens = all.n_tokens - from < most ? all.n_tokens - from : most;
        a.t.k = static_cast<XT*>(all.k) + from * all.token_stride;
        a.t.v = static_cast<XT*>(all.v) + from * all.token_stride;
        a.t.slots += from;
        const int64_t lanes = a.t.n_tokens * all.c.n_heads * (D / 8);
        if constexpr (sizeof(XT) == 2 && F != KVTC_CACHE_BF16) {
            if (lanes >= (kWrite ? 1 << 21 : 1 << 20)) launch_rows<kWrite, XT, F, D, 4>(a, stream);
            else launch_rows<kWrite, XT, F, D, 1>(a, stream);
        } else {
            launch_rows<kWrite, XT, F, D, 1>(a, stream);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <bool kWrite, typename XT, int F>
hipError_t launch_width(const CacheTokenArgs& a, int64_t most, hipStream_t stream) {
    if (a.c.d_head == 64) return launch_tokens<kWrite, XT, F, 64>(a, most, stream);
    if (a.c.d_head == 128) return launch_tokens<kWrite, XT, F, 128>(a, most, stream);
    return launch_tokens<kWrite, XT, F, 256>(a, most, stream);
}
template <bool kWrite, typename XT>
hipError_t launch_format(const CacheTokenArgs& a, int64_t most, hipStream_t stream) {
    if (a.c.format == KVTC_CACHE_BF16) return launch_width<kWrite, XT, KVTC_CACHE_BF16>(a, most, stream);
    if (a.c.format == KVTC_CACHE_FP8) return launch_width<kWrite, XT, KVTC_CACHE_FP8>(a, most, stream);
    return launch_width<kWrite, XT, KVTC_CACHE_INT4>(a, most, stream);
}

hipError_t launch_cache_write(const CacheTokenArgs& a, kvtc_dtype dtype, int64_t launch_tokens, hipStream_t stream) {
    return dtype == KVTC_BF16 ? launch_format<true, uint16_t>(a, launch_tokens, stream) : launch_format<true, float>(a, launch_tokens, stream);
}
hipError_t launch_cache_read(const CacheTokenArgs& a, kvtc_dtype dtype, int64_t launch_tokens, hipStream_t stream) {
    return dtype == KVTC_BF16 ? launch_format<false, uint16_t>(a, launch_tokens, stream) : launch_format<false, float>(a, launch_tokens, stream);
}

}  // namespace kvtc

// Attention of many new tokens of every sequence over the pages of a live cache, for gfx950: launches, the kernel for fp32 queries, and the join of parts.  (bf16 queries: kvtc_many_mfma.hip.)
//
// For a row (a new token's query head) at position i of its sequence, over the tokens that it sees,
//     s_t = scale q . k_t,   out = sum_t e^(s_t) v_t / sum_t e^(s_t),   lse = log sum_t e^(s_t),
// in one pass over the tokens with the running maximum m and sum l:  m' = max(m, s),  l' = l e^(m - m') + sum e^(s - m'),  o' = o e^(m - m') + sum e^(s - m') v.
// A workgroup has an item: rows of one sequence and KV head, all query heads of a token together, so that keys and values are fetched once for all of them, a tile of tokens at a time, as numbers, through
// the LDS.  Where items are few, their tiles are cut into parts, which are joined by a second launch.
//
// Products: S^T = K Q^T, O^T = V^T P^T with tokens in the rows of the first and in the sum of the second, so that a lane has scores of one row only, and of those tokens that its operand of the second
// product needs: probabilities never leave their registers.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <cmath>
#include "kvtc_dev.h"
#include "kvtc_many.h"
#include "../../include/kvtc_test_hooks.h"

namespace kvtc {
kvtc_status set_error(kvtc_status st, const char* fmt, ...);

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#define KVTC_GLOBAL __attribute__((address_space(1)))

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoScore = -__builtin_huge_valf();
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

// ---- fp32: keys, values, queries and probabilities as they are -----------------------------------------------------------------

constexpr int kPlainRows = 64, kPlainTile = 32;

// N neighbouring bytes in dwords.
template <int N>
__device__ __forceinline__ void load_bytes(ManyBytes p, uint32_t* w) {
    if constexpr (N == 4) w[0] = *reinterpret_cast<const KVTC_GLOBAL uint32_t*>(p);
    else if constexpr (N == 8) { const uint64_t v = *reinterpret_cast<const KVTC_GLOBAL uint64_t*>(p); w[0] = (uint32_t)v; w[1] = (uint32_t)(v >> 32); }
    else {
#pragma unroll
        for (int i = 0; i < N / 16; ++i) {
            const u32x4 v = reinterpret_cast<const KVTC_GLOBAL u32x4*>(p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
        }
    }
}

// An eighth of a row: as the cache has it, and its scales.
template <int F, int D>
struct Eighth {
    static constexpr int kBytes = cache_row_bytes(F, D) / 8, kScale = F == KVTC_CACHE_BF16 ? 0 : F == KVTC_CACHE_FP8 ? 1 : D / 32;
    uint32_t w[kBytes / 4], scale[kScale > 0 ? kScale : 1];
    __device__ __forceinline__ void load(ManyBytes row, ManyBytes scales, int part) {
        load_bytes<kBytes>(row + part * kBytes, w);
        if constexpr (kScale == 1) scale[0] = *reinterpret_cast<const KVTC_GLOBAL uint32_t*>(scales);
        else if constexpr (kScale > 1) load_bytes<4 * kScale>(scales, scale);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kBytes / 4; ++i) w[i] = 0u;
#pragma unroll
        for (int i = 0; i < (kScale > 0 ? kScale : 1); ++i) scale[i] = 0u;
    }
    // f(feature, value) for all of them
    template <typename FN>
    __device__ __forceinline__ void each(int part, FN f) const {
        if constexpr (F == KVTC_CACHE_BF16) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                f(part * (D / 8) + 2 * i, __uint_as_float(w[i] << 16));
                f(part * (D / 8) + 2 * i + 1, __uint_as_float(w[i] & 0xffff0000u));
            }
        } else if constexpr (F == KVTC_CACHE_FP8) {
            const float s = __uint_as_float(scale[0]);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const auto low = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), high = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
                f(part * (D / 8) + 4 * i, low[0] * s);
                f(part * (D / 8) + 4 * i + 1, low[1] * s);
                f(part * (D / 8) + 4 * i + 2, high[0] * s);
                f(part * (D / 8) + 4 * i + 3, high[1] * s);
            }
        } else {
            constexpr int G = D / 32;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const int pair = (part * (D / 16) + i) / G, group = i % G;          // (D / 16 is a multiple of G)
                const uint32_t codes = w[i / 4] >> (8 * (i % 4)), header = scale[group];
                const float shift = (float)__builtin_bit_cast(_Float16, (uint16_t)header), s = (float)__builtin_bit_cast(_Float16, (uint16_t)(header >> 16));
                f(group * 32 + 2 * pair, __builtin_fmaf((float)(codes & 15u), s, shift));
                f(group * 32 + 2 * pair + 1, __builtin_fmaf((float)(codes >> 4 & 15u), s, shift));
            }
        }
    }
};

// Of lanes 16, 32 and 48 apart.  (A swap with itself gives a lane its own and the other's, in either order.)
template <typename FN>
__device__ __forceinline__ float over_quarters(float v, FN both) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = both(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return both(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float max_over_quarters(float v) { return over_quarters(v, [](float x, float y) { return fmaxf(x, y); }); }
__device__ __forceinline__ float sum_over_quarters(float v) { return over_quarters(v, [](float x, float y) { return x + y; }); }
__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// Four waves of 16 rows; a row's scores over lanes 16 apart, four neighbouring tokens of every 16 to each.
template <int F, int D>
__global__ void __launch_bounds__(256) many_plain_kernel(const ManyPlan p) {
    constexpr int LD = D + 4, NS = D / 4, NO = D / 16;     // (rows 4 banks apart)
    __shared__ float keys[kPlainTile][LD], values[kPlainTile][LD];
    __shared__ uint8_t there[4], wild[4];                  // a bit for each token: it has a page; it has values that are not finite
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, quarter = lane >> 4;
    const int head = blockIdx.y, part = blockIdx.z;
    many_report(p, ((uint64_t)part * gridDim.y + head) * gridDim.x * 256 + blockIdx.x * 256ull + tid);
    ManyItem it;
    if (!many_item(p, blockIdx.x, it)) return;
    uint32_t n0 = 0, n1 = it.tiles;
    const bool whole = it.tiles <= p.r.part_tiles;
    if (!whole) {
        n0 = min(it.tiles, part * p.r.part_tiles);
        n1 = min(it.tiles, n0 + p.r.part_tiles);
        if (n0 == n1) return;
    } else if (part > 0) {
        return;
    }

    // the wave's rows
    const int row = wave * 16 + col, r = it.row0 + row;
    const bool is_row = row < it.rows;
    const int token = is_row ? r / p.group : 0, q_head = head * p.group + (is_row ? r - token * p.group : 0);
    const int at = it.length - it.n_new + token;
    const float factor = p.a.scale * kLog2e;
    float q[NS];                                           // features quarter * NS and on
    {
        const float* from = static_cast<const float*>(p.a.q) + (int64_t)(it.first + token) * p.a.q_token_stride + (int64_t)q_head * p.a.q_head_stride + quarter * NS;
#pragma unroll
        for (int i = 0; i < NS; ++i) q[i] = is_row ? from[i] : 0.0f;
    }
    f32x4 o[NO];
#pragma unroll
    for (int c = 0; c < NO; ++c) o[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    float m = kNoScore, l = 0.0f;

    // the work-item's part of the tiles: an eighth of a token
    const int mine = tid >> 3, eighth = tid & 7;
    const int32_t* table = p.a.pages + (int64_t)it.b * p.a.pages_stride;
    const ManyBytes k0 = (ManyBytes)(uintptr_t)p.a.c.k_dev + (int64_t)head * p.a.c.head_stride, v0 = (ManyBytes)(uintptr_t)p.a.c.v_dev + (int64_t)head * p.a.c.head_stride;
    const int64_t scale0 = (int64_t)head * p.a.c.page_tokens * cache_scale_bytes(F, D);
    const ManyBytes ks0 = (ManyBytes)(uintptr_t)p.a.c.k_scales_dev + scale0, vs0 = (ManyBytes)(uintptr_t)p.a.c.v_scales_dev + scale0;
    auto places = [&](uint32_t t, int64_t& in_rows, int64_t& in_scales) {       // whether token t is there, and where
        in_rows = in_scales = 0;
        if (t >= (uint32_t)it.end || (p.window != 0u && t >= p.sinks && (int64_t)t <= (int64_t)it.at0 - (int64_t)p.window)) return false;
        const uint32_t index = many_page(p, t);
        const int page = table[index];
        if ((uint32_t)page >= (uint64_t)p.a.c.n_pages) {
            report_lowest(p.a.status, (uint32_t)it.b);
            return false;
        }
        const uint32_t in = t - index * (uint32_t)p.a.c.page_tokens;
        in_rows = (int64_t)page * p.a.c.page_stride + (int64_t)in * p.a.c.token_stride;
        in_scales = (int64_t)page * p.scale_stride + (int64_t)in * cache_scale_bytes(F, D);
        return true;
    };
    Eighth<F, D> k, v;
    bool is = false;
    auto fetch = [&](uint32_t n) {
        int64_t in_rows, in_scales;
        is = n < n1 && places(many_tile(it, n) * kPlainTile + mine, in_rows, in_scales);
        if (is) {
            k.load(k0 + in_rows, ks0 + in_scales, eighth);
            v.load(v0 + in_rows, vs0 + in_scales, eighth);
        } else {
            k.clear();
            v.clear();
        }
    };
    fetch(n0);
    for (uint32_t n = n0; n < n1; ++n) {
        const int t0 = (int)(many_tile(it, n) * kPlainTile);
        __syncthreads();                                   // (the tile before has been used)
        bool odd = false;
        k.each(eighth, [&](int f, float x) { keys[mine][f] = x; });
        v.each(eighth, [&](int f, float x) {
            const bool w = not_finite(x);
            odd |= w;
            values[mine][f] = w ? 0.0f : x;
        });
        const uint64_t have = __ballot(is && eighth == 0), strange = __ballot(odd);
        if (lane == 0) {
            uint32_t h = 0, s = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                h |= (uint32_t)(have >> (8 * i) & 1u) << i;
                s |= (uint32_t)((strange >> (8 * i) & 0xffu) != 0) << i;
            }
            there[wave] = (uint8_t)h;
            wild[wave] = (uint8_t)s;
        }
        __syncthreads();
        fetch(n + 1);
        const uint32_t is_there = *reinterpret_cast<const uint32_t*>(there);
        uint32_t is_wild = *reinterpret_cast<const uint32_t*>(wild);
        float s[8];                                        // of tokens 16 (i / 4) + 4 quarter + i % 4
        float top = kNoScore;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < NS; i += 4) {
                const f32x4 a = *reinterpret_cast<const f32x4*>(&keys[16 * u + col][quarter * NS + i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc = mfma4(a[j], q[i + j], acc);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = 16 * u + 4 * quarter + i;
                const bool seen = (is_there >> t & 1u) && many_sees(p, at, t0 + t);
                s[4 * u + i] = seen ? acc[i] * factor : kNoScore;
                top = fmaxf(top, s[4 * u + i]);
            }
        }
        top = max_over_quarters(top);
        const float now = fmaxf(m, top), base = now == kNoScore ? 0.0f : now, keep = exp2_fast(m - base);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[i] = exp2_fast(s[i] - base);
            sum += s[i];
        }
        l = l * keep + sum;
        m = now;
#pragma unroll
        for (int c = 0; c < NO; ++c) {
            f32x4 acc = o[c];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] *= keep;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc = mfma4(values[16 * u + 4 * quarter + i][16 * c + col], s[4 * u + i], acc);
            o[c] = acc;
        }
        // Values that are not finite reach the rows that see their tokens, and no other (a product with a probability of zero would be NaN).
        while (is_wild) {
            const int t = __builtin_ctz(is_wild);
            is_wild &= is_wild - 1;
            int64_t in_rows, in_scales;
            if (!places((uint32_t)(t0 + t), in_rows, in_scales)) continue;
            const bool seen = many_sees(p, at, t0 + t);
            for (int e = 0; e < 8; ++e) {
                Eighth<F, D> x;
                x.load(v0 + in_rows, vs0 + in_scales, e);
                x.each(e, [&](int f, float value) {
                    if (seen && not_finite(value) && (f >> 2 & 3) == quarter) {
#pragma unroll
                        for (int c = 0; c < NO; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (f == 16 * c + 4 * quarter + i) o[c][i] += value;
                    }
                });
            }
        }
    }
    l = sum_over_quarters(l);
    if (!is_row) return;
    const int64_t place = (int64_t)(it.first + token) * p.a.n_q_heads + q_head;
    if (!whole) {
        float* out = p.part_out + ((int64_t)part * p.a.n_tokens * p.a.n_q_heads + place) * D;
#pragma unroll
        for (int c = 0; c < NO; ++c) *reinterpret_cast<f32x4*>(out + 16 * c + 4 * quarter) = o[c];
        if (quarter == 0) p.part_sums[(int64_t)part * p.a.n_tokens * p.a.n_q_heads + place] = make_float2(m, l);
        return;
    }
    const bool none = m == kNoScore && l == 0.0f;
    const float inverse = none ? 0.0f : 1.0f / l;
    float* out = static_cast<float*>(p.a.out) + place * D;
#pragma unroll
    for (int c = 0; c < NO; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) out[16 * c + 4 * quarter + i] = none ? 0.0f : o[c][i] * inverse;
    if (p.a.lse && quarter == 0) p.a.lse[place] = none ? kNoScore : (m + __builtin_log2f(l)) * kLn2;
}

// ---- parts of an item's tiles, joined ------------------------------------------------------------------------------------------

// Few rows: a workgroup to a row, its four waves take parts in turn, eight parts' loads of a wave together.  (24 rows of 64 parts, heads of 128: one after another 121 us, so 5.9.)
template <typename XT, int D>
__global__ void __launch_bounds__(256) many_join_few_kernel(const ManyPlan p) {
    constexpr int N = D / 64, WAVES = 4;
    typedef float Features __attribute__((ext_vector_type(N == 1 ? 2 : N)));
    __shared__ float sums[WAVES][D], of_waves[WAVES];
    ManyItem it;
    if (!many_item(p, blockIdx.x, it) || it.tiles <= p.r.part_tiles || (int)blockIdx.z >= it.rows) return;
    const int head = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int parts = (int)((it.tiles + p.r.part_tiles - 1) / p.r.part_tiles);
    const int64_t all = (int64_t)p.a.n_tokens * p.a.n_q_heads;
    const int r = it.row0 + (int)blockIdx.z, token = r / p.group, q_head = head * p.group + r - token * p.group;
    const int64_t place = (int64_t)(it.first + token) * p.a.n_q_heads + q_head;
    float m = kNoScore, l = 0.0f;
    for (int i = lane; i < parts; i += 64) m = fmaxf(m, p.part_sums[i * all + place].x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    const float base = m == kNoScore ? 0.0f : m;
    float o[N];
#pragma unroll
    for (int j = 0; j < N; ++j) o[j] = 0.0f;
    for (int i0 = wave; i0 < parts; i0 += 8 * WAVES) {
        float x[8][N];
        float2 s[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = i0 + k * WAVES < parts ? i0 + k * WAVES : wave;
            s[k] = p.part_sums[i * all + place];
            const float* from = p.part_out + (i * all + place) * D + lane * N;
            if constexpr (N == 1) {
                x[k][0] = from[0];
            } else {
                const Features v = *reinterpret_cast<const Features*>(from);
#pragma unroll
                for (int j = 0; j < N; ++j) x[k][j] = v[j];
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (i0 + k * WAVES < parts) {
                const float share = exp2_fast(s[k].x - base);
                l += s[k].y * share;
#pragma unroll
                for (int j = 0; j < N; ++j) o[j] += x[k][j] * share;
            }
    }
    if (lane == 0) of_waves[wave] = l;
#pragma unroll
    for (int j = 0; j < N; ++j) sums[wave][lane * N + j] = o[j];
    __syncthreads();
    if (wave > 0) return;
    for (int w = 1; w < WAVES; ++w) {
        l += of_waves[w];
#pragma unroll
        for (int j = 0; j < N; ++j) o[j] += sums[w][lane * N + j];
    }
    const bool none = m == kNoScore && l == 0.0f;
    XT* out = static_cast<XT*>(p.a.out) + place * D + lane * N;
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float v = none ? 0.0f : o[j] / l;
        if constexpr (sizeof(XT) == 2) out[j] = f32_bf16(v);
        else out[j] = v;
    }
    if (p.a.lse && lane == 0) p.a.lse[place] = none ? kNoScore : (m + __builtin_log2f(l)) * kLn2;
}

// Many rows: D / 4 lanes to each, several rows to a wave, four parts together, in one pass with a running maximum: what an item's workgroups wait for is its sequence and a part's loads once or twice.
template <typename XT, int D>
__global__ void __launch_bounds__(256) many_join_kernel(const ManyPlan p) {
    constexpr int LANES = D / 4, AT_ONCE = 256 / LANES;
    ManyItem it;
    if (!many_item(p, blockIdx.x, it) || it.tiles <= p.r.part_tiles) return;
    const int head = blockIdx.y, lane = threadIdx.x % LANES;
    const int parts = (int)((it.tiles + p.r.part_tiles - 1) / p.r.part_tiles);
    const int64_t all = (int64_t)p.a.n_tokens * p.a.n_q_heads;
    for (int row = blockIdx.z * AT_ONCE + threadIdx.x / LANES; row < it.rows; row += gridDim.z * AT_ONCE) {
        const int r = it.row0 + row, token = r / p.group, q_head = head * p.group + r - token * p.group;
        const int64_t place = (int64_t)(it.first + token) * p.a.n_q_heads + q_head;
        float m = kNoScore, l = 0.0f;
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int i0 = 0; i0 < parts; i0 += 4) {
            f32x4 x[4];
            float2 s[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t at = (i0 + k < parts ? i0 + k : i0) * all + place;
                s[k] = p.part_sums[at];
                x[k] = *reinterpret_cast<const f32x4*>(p.part_out + at * D + 4 * lane);
            }
            float now = m;
#pragma unroll
            for (int k = 0; k < 4; ++k) now = fmaxf(now, s[k].x);
            const float base = now == kNoScore ? 0.0f : now, keep = exp2_fast(m - base);
            m = now;
            l *= keep;
            o *= keep;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (i0 + k < parts) {
                    const float share = exp2_fast(s[k].x - base);
                    l += s[k].y * share;
                    o += x[k] * share;
                }
        }
        const bool none = m == kNoScore && l == 0.0f;
        XT* out = static_cast<XT*>(p.a.out) + place * D + 4 * lane;
        f32x4 v;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = none ? 0.0f : o[j] / l;
        if constexpr (sizeof(XT) == 2) {
            u32x2 w;
#pragma unroll
            for (int j = 0; j < 2; ++j) w[j] = (uint32_t)f32_bf16(v[2 * j]) | (uint32_t)f32_bf16(v[2 * j + 1]) << 16;
            *reinterpret_cast<u32x2*>(out) = w;
        } else {
            *reinterpret_cast<f32x4*>(out) = v;
        }
        if (p.a.lse && lane == 0) p.a.lse[place] = none ? kNoScore : (m + __builtin_log2f(l)) * kLn2;
    }
}
template <typename XT, int D>
static void launch_join_width(const ManyPlan& p, hipStream_t stream) {
    constexpr int each = 2 * 256 / (D / 4);                // rows of a workgroup
    if ((int64_t)p.a.n_tokens * p.a.n_q_heads <= 8 * compute_units()) {
        hipLaunchKernelGGL((many_join_few_kernel<XT, D>), dim3(p.r.items, p.a.c.n_heads, p.r.rows), dim3(256), 0, stream, p);
    } else {
        hipLaunchKernelGGL((many_join_kernel<XT, D>), dim3(p.r.items, p.a.c.n_heads, (p.r.rows + each - 1) / each), dim3(256), 0, stream, p);
    }
}
template <typename XT>
static hipError_t launch_join(const ManyPlan& p, hipStream_t stream) {
    if (p.a.c.d_head == 64) launch_join_width<XT, 64>(p, stream);
    else if (p.a.c.d_head == 128) launch_join_width<XT, 128>(p, stream);
    else launch_join_width<XT, 256>(p, stream);
    return hipGetLastError();
}

// ---- many sequences: the largest start so far ----------------------------------------------------------------------------------

// A workgroup writes 1024 of them, and looks at all starts before for itself.
__global__ void __launch_bounds__(1024) many_order_kernel(const ManyPlan p) {
    __shared__ int of_waves[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, first = (int)blockIdx.x * 1024, b = first + tid;
    int before = 0;
    for (int i = tid; i < first; i += 1024) before = max(before, many_start_or_zero(p, p.a.starts[i]));
    before = __builtin_amdgcn_readlane(many_running_max(before), 63);
    int v = many_running_max(many_start_or_zero(p, b < p.a.n_seqs ? p.a.starts[b] : 0));
    if (lane == 63) {
        of_waves[0][wave] = before;
        of_waves[1][wave] = v;
    }
    __syncthreads();
    for (int w = 0; w < 16; ++w) v = max(v, max(of_waves[0][w], w < wave ? of_waves[1][w] : 0));
    if (b < p.a.n_seqs) p.order[b] = v;
}

// ---- host ----------------------------------------------------------------------------------------------------------------------

// A kernel's rows, tokens of a tile and workgroups to a compute unit, and the time of a tile (us) where a compute unit has one workgroup and where it has all of them.
struct ManyCost { int rows, tile, each; float alone, among; };
// (Measured: heads of 128 features; one sequence of 8000 tokens with 64 new ones, and of 32768 with 2048, 32 query heads to 8; those of 64 and of 256 by their share of the work.)
static ManyCost many_cost(int kind, int format, int d) {
    static constexpr ManyCost of_128[3][4] = {
        {{64, 32, 3, 4.0f, 8.2f}, {128, 64, 2, 1.36f, 2.15f}, {64, 64, 2, 1.0f, 1.33f}, {32, 128, 1, 1.2f, 1.55f}},
        {{64, 32, 3, 4.0f, 8.2f}, {128, 64, 2, 2.02f, 2.73f}, {64, 64, 2, 1.74f, 2.3f}, {32, 128, 2, 2.07f, 2.65f}},
        {{64, 32, 3, 4.0f, 8.2f}, {128, 64, 2, 2.45f, 3.8f}, {64, 64, 2, 2.1f, 3.1f}, {32, 128, 2, 2.7f, 4.2f}}};
    ManyCost c = of_128[format][kind];
    if (d == 64) {
        c.alone *= 0.6f;
        c.among *= kind == kManyPlain ? 0.5f : 0.6f;
        if (kind == kManyOne) c.each = 2;
    } else if (d == 256) {
        c.alone *= 2.0f;
        c.among *= kind == kManyPlain ? 2.0f : 1.2f;       // (one workgroup where there were two)
        c.each = kind == kManyPlain ? 2 : 1;
        if (kind == kManyOne && format == KVTC_CACHE_BF16) c.tile = 64;
    }
    return c;
}

// The kernel, and into how many parts an item's tiles are cut, by an estimate of the call's time: the tiles of the longest item one after another, those of all items by all compute units, and their bytes; and what parts have to
// write and join.  The lengths stand on the device: a lone sequence's is max_tokens, of more of them the mean is taken for a third of it (0.35), and for more of what a window leaves (0.7).
//
// In us: 8 for a call's start and end, 2 more for a kernel of 32 rows (its waves' results are joined through the LDS); parts: a fiftieth of the time for what they repeat, 6 for the launch that joins them, 16 where sequences
// differ (as many parts are started for short ones, which have nothing in them), their fp32 outputs written and read at 6 TB/s, and a twelfth for the kernel of 64 rows, which in parts was slower than its tiles.  Pages are read
// at 5 TB/s.  Of a lone sequence the longer of path and work counts; of several the root of both's squares, since the long ones' path ends among others' work.  All of it is fitted, with many_cost(), to calls with the kernel and
// parts forced: one sequence of 16 to 2048 new tokens behind 0 to 30720, batches of 4 to 33.  The choice is within 5 % of the fastest there, but 12 % off for 16 sequences of up to 200 tokens, 20 for 33 of up to 600, 27 for
// windows of 1024 in a batch of 4: whoever changes a kernel measures many_cost() again, then those.  By a bound far above the lengths more parts are taken than pay: with max_tokens of 131072, 8 tokens of each of 32 caches of
// up to 16384 take 203 us for 158 in bf16, 338 for 262 in 4 bits, 12 ragged prompts of up to 1200 behind up to 2000 in 4 bits 67 for 50.
static ManyRoute many_estimate(const kvtc_cache& c, kvtc_dtype dtype, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens, int64_t sinks, int64_t window) {
    const int64_t group = n_q_heads / c.n_heads, mean = n_tokens * group / n_seqs, cus = compute_units();
    const bool lone = n_seqs == 1;
    if (sinks > max_tokens) sinks = max_tokens;
    if (window > max_tokens) window = max_tokens;
    const int64_t seen = window && sinks + window < max_tokens ? sinks + window : max_tokens;      // tokens that a row sees, at most
    const float length = lone ? (float)seen - 0.5f * (float)(n_tokens < seen ? n_tokens : seen) : (window ? 0.7f : 0.35f) * (float)seen;
    const float bytes = (float)n_seqs * (float)c.n_heads * length * 2.0f * (float)(cache_row_bytes(c.format, c.d_head) + cache_scale_bytes(c.format, c.d_head)) / 5.0e6f;
    ManyRoute best{};
    float least = 0.0f;
    for (int kind = dtype == KVTC_F32 ? kManyPlain : kManyWide; kind <= (dtype == KVTC_F32 ? kManyPlain : kManyOne); ++kind) {
        if (kind == kManyOne && !lone && mean > 32) continue;
        const ManyCost k = many_cost(kind, c.format, c.d_head);
        const int64_t items = n_tokens * group / k.rows + n_seqs, blocks = ((mean > 0 ? mean : 1) + k.rows - 1) / k.rows * n_seqs * c.n_heads;
        int64_t tiles = (max_tokens + k.tile - 1) / k.tile;    // of an item, at most
        if (window) {
            const int64_t some = sinks / k.tile + window / k.tile + (k.rows + k.tile - 1) / k.tile + 3;
            tiles = some < tiles ? some : tiles;
        }
        const float among = kind == kManyWide && mean < k.rows ? k.alone + (k.among - k.alone) * (float)mean / (float)k.rows : k.among;      // (its waves without rows leave the others their time)
        for (int64_t parts = 1; parts <= tiles && parts <= 512; parts += parts < 4 ? 1 : parts < 8 ? 2 : parts / 2) {
            if (parts > 1 && blocks * parts > 32 * cus * k.each) break;
            const int64_t part_tiles = (tiles + parts - 1) / parts, rounds = (blocks * parts + cus * k.each - 1) / (cus * k.each);
            const float path = (float)part_tiles * (blocks * parts <= cus ? k.alone : among);
            float all = (float)blocks * length / (float)k.tile * among / (float)(cus * k.each);
            if (lone && rounds < 3 && blocks * parts > cus && all < (float)rounds * (float)part_tiles * among) all = (float)rounds * (float)part_tiles * among;
            if (all < bytes) all = bytes;
            float time = 8.0f + (lone ? (path > all ? path : all) : sqrtf(path * path + all * all)) + (kind == kManyOne ? 2.0f : 0.0f);
            if (parts > 1) time = 1.02f * time + (lone ? 6.0f : 16.0f) + (float)n_tokens * (float)n_q_heads * (float)parts * (float)c.d_head * 8.0f / 6.0e6f;
            if (kind == kManyTwo && parts > 1) time *= 1.08f;
            if (best.parts == 0 || time < least) {
                least = time;
                best = {kind, k.rows, k.tile, (int)items, (int)((tiles + part_tiles - 1) / part_tiles), (uint32_t)part_tiles};
            }
        }
    }
    return best;
}

ManyRoute many_route(const kvtc_cache& c, kvtc_dtype dtype, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens, int64_t sinks, int64_t window) {
    ManyRoute r = many_estimate(c, dtype, n_seqs, n_tokens, n_q_heads, max_tokens, sinks, window);
    if (window) {                                          // no more parts than the workspace has room for, which is sized without one
        const int most = many_estimate(c, dtype, n_seqs, n_tokens, n_q_heads, max_tokens, 0, 0).parts;
        if (r.parts > most) {
            const uint32_t tiles = r.part_tiles * (uint32_t)r.parts;
            r.part_tiles = (tiles + most - 1) / most;
            r.parts = most;
        }
    }
    if (r.parts == 1) r.part_tiles = 0xffffffffu;
    return r;
}

size_t many_work_bytes(const kvtc_cache& c, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens) {
    size_t most = 0;
    for (int type = 0; type < 2; ++type) {
        const int parts = many_route(c, (kvtc_dtype)type, n_seqs < 1 ? 1 : n_seqs, n_tokens < 1 ? 1 : n_tokens, n_q_heads, max_tokens, 0, 0).parts;
        const size_t need = parts > 1 ? (size_t)parts * (size_t)n_tokens * n_q_heads * (c.d_head + 2) * sizeof(float) : 0;
        most = need > most ? need : most;
    }
    return most + kAttendMaxShares * 4 + (n_seqs > kManyScanned ? (size_t)n_seqs * 4 : 0);
}

hipError_t launch_many_mfma_0(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_1(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_2(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_3(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_4(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_5(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_6(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_7(const ManyPlan& p, hipStream_t stream);
hipError_t launch_many_mfma_8(const ManyPlan& p, hipStream_t stream);

template <int F, int D>
static void launch_plain(const ManyPlan& p, hipStream_t stream) {
    hipLaunchKernelGGL((many_plain_kernel<F, D>), dim3(p.r.items, p.a.c.n_heads, p.r.parts), dim3(256), 0, stream, p);
}
template <int F>
static void launch_plain_width(const ManyPlan& p, hipStream_t stream) {
    if (p.a.c.d_head == 64) launch_plain<F, 64>(p, stream);
    else if (p.a.c.d_head == 128) launch_plain<F, 128>(p, stream);
    else launch_plain<F, 256>(p, stream);
}
static void launch_plain_format(const ManyPlan& p, hipStream_t stream) {
    if (p.a.c.format == KVTC_CACHE_BF16) launch_plain_width<KVTC_CACHE_BF16>(p, stream);
    else if (p.a.c.format == KVTC_CACHE_FP8) launch_plain_width<KVTC_CACHE_FP8>(p, stream);
    else launch_plain_width<KVTC_CACHE_INT4>(p, stream);
}

hipError_t launch_many(const ManyArgs& a, kvtc_dtype dtype, hipStream_t stream) {
    ManyPlan p;
    p.a = a;
    p.r = many_route(a.c, dtype, a.n_seqs, a.n_tokens, a.n_q_heads, a.max_tokens, a.sinks, a.window);
    p.group = a.n_q_heads / a.c.n_heads;
    auto in_31 = [](int64_t v) { return (uint32_t)(v < 0x7fffffffLL ? v : 0x7fffffffLL); };
    p.sinks = in_31(a.sinks);
    p.window = in_31(a.window);
    p.scale_stride = (int64_t)a.c.n_heads * a.c.page_tokens * cache_scale_bytes(a.c.format, a.c.d_head);
    uint32_t s = 0;                                        // (n < 2^31: m = ceil(2^(31 + s) / d) is near enough)
    while ((1ull << s) < (uint64_t)a.c.page_tokens) ++s;
    p.page_mul = (uint32_t)(((1ull << (31 + s)) + a.c.page_tokens - 1) / a.c.page_tokens);
    p.page_shift = 31 + s;
    const int64_t rows = (int64_t)a.n_tokens * a.n_q_heads;
    p.part_out = static_cast<float*>(a.work) + kAttendMaxShares;           // (behind kvtc_attend's counters)
    p.part_sums = reinterpret_cast<float2*>(p.part_out + (p.r.parts > 1 ? p.r.parts * rows * a.c.d_head : 0));
    p.order = reinterpret_cast<int32_t*>(p.part_sums + (p.r.parts > 1 ? p.r.parts * rows : 0));
    if (a.n_seqs > kManyScanned) hipLaunchKernelGGL(many_order_kernel, dim3((a.n_seqs + 1023) / 1024), dim3(1024), 0, stream, p);
    hipError_t e;
    if (p.r.kind == kManyPlain) {
        launch_plain_format(p, stream);
        e = hipGetLastError();
    } else {
        static hipError_t (*const launch[9])(const ManyPlan&, hipStream_t) = {launch_many_mfma_0, launch_many_mfma_1, launch_many_mfma_2, launch_many_mfma_3, launch_many_mfma_4,
                                                                              launch_many_mfma_5, launch_many_mfma_6, launch_many_mfma_7, launch_many_mfma_8};
        e = launch[3 * a.c.format + (a.c.d_head == 64 ? 0 : a.c.d_head == 128 ? 1 : 2)](p, stream);
    }
    if (e != hipSuccess || p.r.parts == 1) return e;
    return dtype == KVTC_BF16 ? launch_join<uint16_t>(p, stream) : launch_join<float>(p, stream);
}

}  // namespace kvtc

extern "C" {

static kvtc_status check_many(const char* who, const kvtc_cache* c, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens) {
    using namespace kvtc;
    const kvtc_status st = cache_check(who, c);
    if (st != KVTC_OK) return st;
    if (n_seqs < 0 || n_seqs > kAttendMaxSeqs) return set_error(KVTC_E_ARG, "%s: n_seqs=%d outside 0..%d", who, n_seqs, kAttendMaxSeqs);
    if (n_q_heads < 1 || n_q_heads > kCacheMaxHeads || n_q_heads % c->n_heads != 0)
        return set_error(KVTC_E_ARG, "%s: n_q_heads=%d must be a multiple of the cache's %d heads, at most %d", who, n_q_heads, c->n_heads, kCacheMaxHeads);
    if (max_tokens < 1 || max_tokens > 0x7fffffffLL) return set_error(KVTC_E_ARG, "%s: max_tokens=%lld outside 1..2^31-1", who, (long long)max_tokens);
    if (n_tokens < 0 || n_tokens > 0x7fffffffLL) return set_error(KVTC_E_ARG, "%s: n_tokens=%lld", who, (long long)n_tokens);
    if (n_tokens * n_q_heads > kManyMaxRows) return set_error(KVTC_E_UNSUPPORTED, "%s: %lld tokens of %d query heads are more than 2^29 rows", who, (long long)n_tokens, n_q_heads);
    return KVTC_OK;
}

kvtc_status kvtc_host_attend_many_route(const kvtc_cache* cache, kvtc_dtype dtype, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens, int64_t sinks, int64_t window, int32_t* route) {
    using namespace kvtc;
    const kvtc_status st = check_many("kvtc_host_attend_many_route", cache, n_seqs, n_tokens, n_q_heads, max_tokens);
    if (st != KVTC_OK) return st;
    if ((dtype != KVTC_BF16 && dtype != KVTC_F32) || n_seqs < 1 || n_tokens < 1 || sinks < 0 || window < 0 || !route) return set_error(KVTC_E_ARG, "kvtc_host_attend_many_route: bad argument");
    const ManyRoute r = many_route(*cache, dtype, n_seqs, n_tokens, n_q_heads, max_tokens, sinks, window);
    const int32_t all[6] = {r.kind, r.rows, r.tile, r.items, r.parts, r.parts == 1 ? 0 : (int32_t)r.part_tiles};
    std::copy(all, all + 6, route);
    return KVTC_OK;
}

size_t kvtc_attend_many_work_bytes(const kvtc_cache* cache, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens) {
    return check_many("kvtc_attend_many_work_bytes", cache, n_seqs, n_tokens, n_q_heads, max_tokens) == KVTC_OK ? kvtc::many_work_bytes(*cache, n_seqs, n_tokens, n_q_heads, max_tokens) : 0;
}

kvtc_status kvtc_attend_many(const kvtc_cache* cache, const void* q_dev, kvtc_dtype dtype, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t q_token_stride, int64_t q_head_stride,
                             const int32_t* starts_dev, const int32_t* pages_dev, int64_t pages_stride, const int32_t* lengths_dev, int64_t max_tokens, float scale, int causal, int64_t sinks,
                             int64_t window, void* out_dev, float* lse_dev, void* work_dev, size_t work_bytes, uint32_t* status_dev, kvtc_stream stream) {
    using namespace kvtc;
    const kvtc_status st = check_many("kvtc_attend_many", cache, n_seqs, n_tokens, n_q_heads, max_tokens);
    if (st != KVTC_OK) return st;
    if (dtype != KVTC_BF16 && dtype != KVTC_F32) return set_error(KVTC_E_ARG, "kvtc_attend_many: unknown dtype %d", (int)dtype);
    if (!std::isfinite(scale)) return set_error(KVTC_E_ARG, "kvtc_attend_many: scale must be finite");
    if (causal != 0 && causal != 1) return set_error(KVTC_E_ARG, "kvtc_attend_many: causal must be 0 or 1");
    if (sinks < 0 || window < 0 || (!causal && window != 0)) return set_error(KVTC_E_ARG, "kvtc_attend_many: sinks=%lld window=%lld (a window needs causal)", (long long)sinks, (long long)window);
    if (n_seqs == 0 || n_tokens == 0) return KVTC_OK;
    if (!q_dev || !starts_dev || !pages_dev || !lengths_dev || !out_dev || !work_dev) return set_error(KVTC_E_ARG, "kvtc_attend_many: null buffer");
    const int64_t e = dtype == KVTC_BF16 ? 2 : 4, far = (int64_t)1 << 40;
    if (q_token_stride < 0 || q_token_stride > far || q_head_stride < 0 || q_head_stride > far)
        return set_error(KVTC_E_ARG, "kvtc_attend_many: query strides (token %lld, head %lld)", (long long)q_token_stride, (long long)q_head_stride);
    if (((reinterpret_cast<uintptr_t>(q_dev) | reinterpret_cast<uintptr_t>(out_dev)) & 15u) || (q_token_stride * e) % 16 != 0 || (q_head_stride * e) % 16 != 0)
        return set_error(KVTC_E_ARG, "kvtc_attend_many: queries, their strides and the output must be 16-byte aligned");
    if (((reinterpret_cast<uintptr_t>(starts_dev) | reinterpret_cast<uintptr_t>(pages_dev) | reinterpret_cast<uintptr_t>(lengths_dev) | reinterpret_cast<uintptr_t>(lse_dev) |
          reinterpret_cast<uintptr_t>(status_dev)) & 3u) || (reinterpret_cast<uintptr_t>(work_dev) & 255u))
        return set_error(KVTC_E_ARG, "kvtc_attend_many: misaligned starts, table, lengths, lse, status (4 bytes) or workspace (256)");
    if (pages_stride < (max_tokens + cache->page_tokens - 1) / cache->page_tokens)
        return set_error(KVTC_E_ARG, "kvtc_attend_many: pages_stride=%lld holds less than max_tokens=%lld", (long long)pages_stride, (long long)max_tokens);
    const size_t need = many_work_bytes(*cache, n_seqs, n_tokens, n_q_heads, max_tokens);
    if (work_bytes < need) return set_error(KVTC_E_SMALL, "kvtc_attend_many: work_bytes=%zu < %zu", work_bytes, need);
    const ManyArgs a{*cache, q_dev, q_token_stride, q_head_stride, starts_dev, pages_dev, pages_stride, lengths_dev, max_tokens, sinks, window, scale, causal, n_seqs, (int32_t)n_tokens,
                     n_q_heads, out_dev, lse_dev, work_dev, status_dev};
    const hipError_t err = launch_many(a, dtype, static_cast<hipStream_t>(stream));
    if (err != hipSuccess) return set_error(KVTC_E_HIP, "kvtc_attend_many: launch failed: %s", hipGetErrorString(err));
    return KVTC_OK;
}

}  // extern "C"

// Attention of many new tokens over the pages of a live cache, bf16 queries: 16-bit matrix products, for gfx950.
//
// The mathematics and the division into items and parts: kvtc_many.hip.  A workgroup has RW x TW waves: RW blocks of 32 rows, and for each TW waves that share the tokens of a tile
// (64, or 32 to a wave), whose results are joined through the LDS in the end.
//
// Operands.  bf16 pages: keys, values and queries as they are, probabilities rounded to bf16 (off by 2^-8 of themselves at most, as much as the rounding of the output; sums of probabilities are of those before it).
// Outputs are 0.00168 to 0.00173 of themselves off, of which 0.00166 are their own rounding; in two parts, 16 bits, probabilities make that 0.00166, for half as many products again: a prompt of 8192 tokens 770 us for 578, of
// 1000 33 for 29, 8 tokens of each of 32 caches 168 for 154.  (kvtc_attend, which memory bounds, keeps 24 bits: the same token's result differs in its last place.)
// 8 and 4 bits: fp16.  Queries times a power of two, a row's largest below 2^15 (4 bits: 2^10); codes of keys as they are.  8 bits: a token's scales go into its scores and probabilities.  4 bits: a score is the sum over groups of
// 32 features of scale * (codes . queries), scaled in fp32, and of shift * (sum of queries), one product more with that sum in three parts: no key is rounded (rounded once to fp16 they were 20 % faster, and lse, which is fp32,
// 1e-5 off and more); values are shift + code * scale, rounded once to fp16 (2^-11, as the probabilities; a number of the format below 2^-14 is one of fp16; 16 tokens of which one passes 2^15 are all divided by a power of two),
// which the output's rounding to bf16 covers.  Probabilities, of 8 bits times the values' scale, are rounded to fp16.  The scales of 16 tokens' values have an exponent in common, which goes into the probabilities' exponential.
// Queries more than 2^28 (over 4 bits: 2^23) below a row's largest lose bits.  Probabilities stand 2^kBias = 2^6 times as high as they are of the largest so far (of 8 bits, times the largest scale so far): they keep 11 bits
// down to 2^-20 of it, and are off by 2^-31 of it at most below.
//
// Products.  32 x 32 x 16 instructions, S^T = K Q^T and O^T = V^T P^T.  A lane has the scores of one row, of tokens 8 (i / 4) + 4 (lane / 32) + i % 4, i = 0..15, of every 32.  The second product sums over
// tokens in that order: its operand of probabilities is what the lane has, and that of values comes out of the LDS by transposing loads of four tokens of a feature.  Maxima and sums need one exchange of halves.
// The maximum that is taken off the scores follows the true one when that has grown by more than slack(): outputs are rarely rescaled.
//
// Tiles.  Two buffers in the LDS: while one is used, the next tile is on its way, bf16 rows directly from memory to the LDS, others by registers, where they become numbers.  16-byte pieces of a row lie in an order that differs
// from row to row, so that neither the loads of keys (32 rows at a column) nor those of values (8 rows at two columns) meet in a bank.
//
// Tiles of which some row does not see all (or that have no page) are masked, row by row, as 32 bits to 32 tokens.  Their values that are not finite are zeros in the LDS, lest a probability of zero make NaN of them, and are added
// afterwards to the rows that see them.
//
// What bounds it.  Large calls: matrix products and, by the same waves in between, the softmax; two workgroups to a compute unit work at both at once.  A prompt of 8192 tokens, 32 query heads of 128 to 8: 570 to 580 us,
// 960 TFLOP/s of products that count, 77 % of what a large product alone reaches here (both at the clock that power leaves).  2048 tokens behind 30720: 1405 us in 8 bits, 2100 in 4: the vector unit, with scales, codes to
// numbers and the softmax.
// Few items: a tile's chain of instructions, 1.0 to 2.3 us with one workgroup to a compute unit, hence parts; 6 tokens behind 131066 in 8 bits 66 us, 4.2 TB/s.
#include <hip/hip_runtime.h>
#include <type_traits>
#include "kvtc_dev.h"
#include "kvtc_many.h"

namespace kvtc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
#define KVTC_GLOBAL __attribute__((address_space(1)))
#define KVTC_LDS __attribute__((address_space(3)))

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoScore = -__builtin_huge_valf();
constexpr float kLeastFactor = 0x1p-126f, kMostFactor = 0x1p127f;

template <int F> constexpr bool is_bf16() { return F == KVTC_CACHE_BF16; }
// By how much, in powers of two, scores may pass the maximum that is taken off; fp16: and the values' exponents theirs, with probabilities times 2^kBias: below 2^15 together.
template <int F> constexpr float slack() { return is_bf16<F>() ? 8.0f : 4.0f; }
constexpr int kProducts = 0x8, kLdsReads = 0x100;           // of instructions whose order is asked for
constexpr int kBias = 6, kExponentSlack = 4, kLeastExponent = -100;

template <int F> __device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (is_bf16<F>()) return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <int F> __device__ __forceinline__ uint32_t round_pair(float first, float second) {
    if constexpr (is_bf16<F>()) {
        bf16x2 v;
        v[0] = (__bf16)first;
        v[1] = (__bf16)second;
        return __builtin_bit_cast(uint32_t, v);
    } else {
        f16x2 v;
        v[0] = (_Float16)first;
        v[1] = (_Float16)second;
        return __builtin_bit_cast(uint32_t, v);
    }
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23 & 255u) - 127; }
// The other half's value of a lane 32 apart, joined with its own.
__device__ __forceinline__ float max_of_halves(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
// The largest of lanes whose numbers differ by a multiple of four.  (By the LDS, a step after another, this was 0.1 us of a tile's 2 for each of keys and values.)
__device__ __forceinline__ float max_of_quarters(float v) {
    auto turned = [&](auto by) { return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x120 + decltype(by)::value, 0xf, 0xf, false)); };      // within 16 lanes
    v = fmaxf(v, turned(std::integral_constant<int, 4>{}));
    v = fmaxf(v, turned(std::integral_constant<int, 8>{}));
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return max_of_halves(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
}
__device__ __forceinline__ float sum_of_halves(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}
__device__ __forceinline__ uint32_t same(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ int64_t lane_value64(int64_t v, int lane) { return (int64_t)((uint64_t)lane_value((uint32_t)((uint64_t)v >> 32), lane) << 32 | lane_value((uint32_t)v, lane)); }
__device__ __forceinline__ int64_t shfl64(int64_t v, int from) {
    const int lo = __shfl((int)(uint32_t)v, from, 64), hi = __shfl((int)(v >> 32), from, 64);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

template <int F, int D, int RW, int TW, int TOKENS>
struct Shape {
    static constexpr int NW = RW * TW;
    static constexpr int NT = TOKENS;                      // of a wave, to a tile
    static constexpr int TILE = NT * TW, ROWS = 32 * RW;
    static constexpr int RPW = TILE / NW;                  // tokens that a wave brings in
    static constexpr int ROW = 2 * D;                      // bytes of a token in the LDS
    static constexpr int BUFFER = TILE * ROW;
    static constexpr int NS = D / 16, NF = D / 32, NB = NT / 32, NG = RPW / 16;
    // Where a wave's tokens are those that it brings in, it waits for no other, and numbers that it makes itself need one buffer.
    static constexpr bool ALONE = RW == 1;
    static constexpr int BUFFERS = ALONE && !is_bf16<F>() ? 1 : 2;
    // behind the buffers of keys and values: exponents of 16 tokens' values; 8 bits: every token's scales, 4 bits: its keys' scales and shifts; tokens with values that are not finite, by waves
    static constexpr int G = F == KVTC_CACHE_INT4 ? D / 32 : 0;              // groups of a row with a header each
    static constexpr int kExponents = 2 * BUFFERS * BUFFER, kScales = kExponents + BUFFERS * (TILE / 16) * 4, kWild = kScales + (F == KVTC_CACHE_FP8 ? BUFFERS * 2 * TILE * 4 : BUFFERS * TILE * G * 6),
                         kLds = kWild + BUFFERS * NW * 4;
    static_assert(RPW % 16 == 0, "");
};

// The order of a row's 16-byte pieces of keys, and of its 32-byte pieces of values.
template <int D> __device__ __forceinline__ uint32_t key_turn(uint32_t t) { return D == 64 ? t >> 1 & 7u : t & 15u; }
template <int D> __device__ __forceinline__ uint32_t value_turn(uint32_t t) { return D == 64 ? t >> 1 & 3u : t & 7u; }

// One value of a row as the cache has it.
template <int F, int D>
__device__ __forceinline__ float value_at(ManyBytes row, ManyBytes scales, int f) {
    if constexpr (is_bf16<F>()) {
        return __uint_as_float((uint32_t)reinterpret_cast<const KVTC_GLOBAL uint16_t*>(row)[f] << 16);
    } else if constexpr (F == KVTC_CACHE_FP8) {
        return __builtin_amdgcn_cvt_f32_fp8((int)row[f], 0) * *reinterpret_cast<const KVTC_GLOBAL float*>(scales);
    } else {
        constexpr int G = D / 32;
        const uint32_t codes = row[(f % 32) / 2 * G + f / 32], header = reinterpret_cast<const KVTC_GLOBAL uint32_t*>(scales)[f / 32];
        return __builtin_fmaf((float)(codes >> (f % 2 * 4) & 15u), (float)__builtin_bit_cast(_Float16, (uint16_t)(header >> 16)), (float)__builtin_bit_cast(_Float16, (uint16_t)header));
    }
}

// 8 and 4 bits: a quarter of a row, on its way.  Lane: row lane / 4, quarter lane % 4.
template <int F, int D>
struct Quarter {
    static constexpr int kBytes = cache_row_bytes(F, D) / 4, kScales = F == KVTC_CACHE_FP8 ? 1 : D / 32;
    uint32_t w[kBytes / 4], scale[kScales];
    __device__ __forceinline__ void load(ManyBytes row, ManyBytes scales) {
        if constexpr (kBytes == 8) {
            const u32x2 v = *reinterpret_cast<const KVTC_GLOBAL u32x2*>(row);
            w[0] = v[0];
            w[1] = v[1];
        } else {
#pragma unroll
            for (int i = 0; i < kBytes / 16; ++i) {
                const u32x4 v = reinterpret_cast<const KVTC_GLOBAL u32x4*>(row)[i];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
            }
        }
#pragma unroll
        for (int i = 0; i < kScales; ++i) scale[i] = reinterpret_cast<const KVTC_GLOBAL uint32_t*>(scales)[i];
    }
    // 8 bits: the scale, 4 bits: a bound of the magnitudes of the row; zero if it is not finite
    __device__ __forceinline__ float most() const {
        if constexpr (F == KVTC_CACHE_FP8) {
            const float s = __builtin_fabsf(__uint_as_float(scale[0]));
            return not_finite(s) ? 0.0f : s;
        } else {
            float m = 0.0f;
#pragma unroll
            for (int i = 0; i < kScales; ++i) {
                const float shift = (float)__builtin_bit_cast(_Float16, (uint16_t)scale[i]), s = (float)__builtin_bit_cast(_Float16, (uint16_t)(scale[i] >> 16));
                const float b = fmaxf(__builtin_fabsf(shift), __builtin_fabsf(__builtin_fmaf(15.0f, s, shift)));
                m = not_finite(b) ? m : fmaxf(m, b);
            }
            return m;
        }
    }
    // A byte's codes in fp16: the low one behind 1024, the high one behind 64, where they stand.
    __device__ __forceinline__ f16x2 codes(int byte) const {
        const uint32_t twice = __builtin_amdgcn_perm(w[byte / 4], w[byte / 4], 0x0c000c00u | (uint32_t)(byte % 4) | (uint32_t)(byte % 4) << 16);
        return __builtin_bit_cast(f16x2, (twice & 0x00f0000fu) | 0x54006400u) - f16x2{(_Float16)1024.0f, (_Float16)64.0f};
    }
    // 4 bits: each(), of the codes.
    template <typename FN>
    __device__ __forceinline__ void each_code(int quarter, FN f) const {
#pragma unroll
        for (int g = 0; g < D / 32; ++g) {
            u32x4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(uint32_t, codes(j * (D / 32) + g));
            f(4 * g + quarter, v);
        }
    }
    // f(piece, its eight features in fp16) for the quarter's pieces.  8 bits: the codes; 4 bits: values times 2^-e.
    template <typename FN>
    __device__ __forceinline__ void each(int quarter, int e, FN f) const {
        u32x4 v;
        if constexpr (F == KVTC_CACHE_FP8) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    v[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i + j], 1.0f, false));
                    v[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[2 * i + j], 1.0f, true));
                }
                f(quarter * (D / 32) + i, v);
            }
        } else {
            constexpr int G = D / 32;                      // pairs 4 quarter .. + 3 of every group: byte pair * G + group
#pragma unroll
            for (int g = 0; g < G; ++g) {
                uint32_t header = scale[g];
                if (e != 0) {                              // (the same for 16 rows)
                    const f16x2 h = __builtin_bit_cast(f16x2, header);
                    header = round_pair<F>(__builtin_amdgcn_ldexpf((float)h[0], -e), __builtin_amdgcn_ldexpf((float)h[1], -e));
                }
                const f16x2 shift = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(header, header, 0x01000100u)), size = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(header, header, 0x03020302u));
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(codes(j * G + g), size, shift));
                f(4 * g + quarter, v);
            }
        }
    }
};

template <int F, int D, int RW, int TW, int TOKENS, bool IN_PAGE>
__global__ void __launch_bounds__(64 * RW * TW, D == 256 ? 1 : 2) many_mfma_kernel(const ManyPlan p) {
    using S = Shape<F, D, RW, TW, TOKENS>;
    constexpr bool BF = is_bf16<F>();
    constexpr int NW = S::NW, NT = S::NT, TILE = S::TILE, RPW = S::RPW, NS = S::NS, NF = S::NF, NB = S::NB, NG = S::NG;
    constexpr int UNITS = IN_PAGE ? 1 : (TILE + 63) / 64;  // what a lane looks up: 16 tokens in a page, or tokens of a tile
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = (int)same(tid >> 6), rw = wave / TW, tw = wave % TW, col = lane & 31, half = lane >> 5;
    const int head = blockIdx.x, part = blockIdx.z;
    many_report(p, (((uint64_t)part * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x) * (64 * NW) + tid);
    ManyItem it;
    if (!many_item(p, gridDim.y - 1 - blockIdx.y, it)) return;       // (the last rows of a causal sequence, which see the most, first)
    uint32_t n0 = 0, n1 = it.tiles;
    const bool whole = it.tiles <= p.r.part_tiles;
    if (!whole) {
        n0 = min(it.tiles, (uint32_t)part * p.r.part_tiles);
        n1 = min(it.tiles, n0 + p.r.part_tiles);
        if (n0 == n1) return;
    } else if (part > 0) {
        return;
    }

    // ---- the wave's rows ----
    const int row = rw * 32 + col, r = it.row0 + row;
    const bool is_row = row < it.rows, any_row = rw * 32 < it.rows;
    const int behind = it.length - it.n_new;
    const int token = is_row ? r / p.group : 0, q_head = head * p.group + (is_row ? r - token * p.group : 0);
    const int at = is_row ? behind + token : it.at1;
    const int from = p.window != 0u && at - (int64_t)p.window + 1 > 0 ? at - (int)p.window + 1 : 0;
    const int first_at = (int)same((uint32_t)at), last_at = (int)lane_value((uint32_t)at, 31);           // (positions rise with the rows)
    const int last_from = (int)lane_value((uint32_t)from, 31);
    const float size = __builtin_fabsf(p.a.scale);
    float factor = size == 0.0f ? 1.0f : size * kLog2e;    // of a score
    u32x4 q[NS];
    {
        const uint16_t* src = static_cast<const uint16_t*>(p.a.q) + (int64_t)(it.first + token) * p.a.q_token_stride + (int64_t)q_head * p.a.q_head_stride + 8 * half;
        const uint32_t keep = is_row && size != 0.0f ? 0xffffffffu : 0u, flip = p.a.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            q[s] = *reinterpret_cast<const KVTC_GLOBAL u32x4*>((uintptr_t)(src + 16 * s));
#pragma unroll
            for (int j = 0; j < 4; ++j) q[s][j] = (q[s][j] ^ flip) & keep;
        }
        if constexpr (!BF) {
            float most = 0.0f;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float a = __builtin_fabsf(__uint_as_float(q[s][j] << 16)), b = __builtin_fabsf(__uint_as_float(q[s][j] & 0xffff0000u));
                    most = fmaxf(most, fmaxf(not_finite(a) ? 0.0f : a, not_finite(b) ? 0.0f : b));
                }
            most = max_of_halves(most);
            const int e = most == 0.0f ? 0 : exponent_of(most) - (F == KVTC_CACHE_INT4 ? 9 : 14);      // (4 bits: and sums of 32 below 2^15)
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    q[s][j] = round_pair<F>(__builtin_amdgcn_ldexpf(__uint_as_float(q[s][j] << 16), -e), __builtin_amdgcn_ldexpf(__uint_as_float(q[s][j] & 0xffff0000u), -e));
            factor = __builtin_amdgcn_ldexpf(factor, e);
        }
        factor = __builtin_amdgcn_fmed3f(factor, kLeastFactor, kMostFactor);
    }
    // 4 bits: a row's queries summed over each group, in three parts of fp16 (33 bits): part c of group g is number c * G + g of the operand that goes with the tokens' shifts
    constexpr int G = S::G, NSHIFT = (3 * G + 15) / 16;
    u32x4 q_sums[F == KVTC_CACHE_INT4 ? NSHIFT : 1];
    if constexpr (F == KVTC_CACHE_INT4) {
        float part[3][G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float sum = 0.0f;
#pragma unroll
            for (int s = 2 * g; s < 2 * g + 2; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f16x2 v = __builtin_bit_cast(f16x2, (uint32_t)q[s][j]);
                    sum += (float)v[0] + (float)v[1];
                }
            sum = sum_of_halves(sum);
#pragma unroll
            for (int c = 0; c < 3; ++c) {
                part[c][g] = (float)(_Float16)sum;
                sum -= part[c][g];
            }
        }
#pragma unroll
        for (int n = 0; n < NSHIFT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float v[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int low = 16 * n + 2 * j + i, high = low + 8;
                    const float of_low = low < 3 * G ? part[low / G % 3][low % G] : 0.0f, of_high = high < 3 * G ? part[high / G % 3][high % G] : 0.0f;
                    v[i] = half ? of_high : of_low;
                }
                q_sums[n][j] = round_pair<F>(v[0], v[1]);
            }
    }
    f32x16 o[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[f][i] = 0.0f;
    float m = kNoScore, base = 0.0f, l = 0.0f;             // the maximum that is taken off, or zero where there is none yet
    int exponent = -200;                                   // fp16: of the values so far; o is in units of 2^(exponent - kBias)

    // ---- the tokens ----
    const int32_t* table = p.a.pages + (int64_t)it.b * p.a.pages_stride;
    const int64_t head_at = (int64_t)head * p.a.c.head_stride, scale_at = (int64_t)head * p.a.c.page_tokens * cache_scale_bytes(F, D);
    const ManyBytes k0 = (ManyBytes)(uintptr_t)p.a.c.k_dev + head_at, v0 = (ManyBytes)(uintptr_t)p.a.c.v_dev + head_at;
    const ManyBytes ks0 = (ManyBytes)(uintptr_t)p.a.c.k_scales_dev + scale_at, vs0 = (ManyBytes)(uintptr_t)p.a.c.v_scales_dev + scale_at;
    const uint32_t ts = (uint32_t)p.a.c.token_stride;
    const int gap = p.window == 0u ? 0 : (int)max((int64_t)0, (int64_t)it.at0 - (int64_t)p.window + 1);      // tokens from p.sinks to before it are seen by no row
    auto there = [&](uint32_t t) { return t < (uint32_t)it.end && (p.window == 0u || t < p.sinks || (int)t >= gap); };

    // Where tokens are: bytes from the pools' (and the scales') bases.  IN_PAGE: of every 16 tokens, a lane each, for PER tiles at a time, the next ones' page numbers on their way; what a tile needs of that is read out of
    // the lanes.  Else of the next tile, a token to a lane.  (Worked out for every tile, by the scalar unit, this was up to 0.4 us a tile where a wave is alone; page numbers through the scalar cache make every wait for the
    // LDS one for them, and a load of the vector unit for every tile one for all keys and values before it: loads come back in their order.)
    constexpr int GROUPS = TILE / 16, PER = 64 / GROUPS;
    int32_t pages[UNITS];
    int64_t rows_of[UNITS], scales_of[BF ? 1 : UNITS];
    uint64_t valid[UNITS];
    auto look = [&](uint32_t n) {                          // page numbers from tile n on
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const uint32_t t = IN_PAGE ? many_tile(it, n + lane / GROUPS) * TILE + (lane % GROUPS) * 16 : many_tile(it, n) * TILE + lane + 64 * u;
            pages[u] = -1;
            if (IN_PAGE ? n + lane / GROUPS < n1 && t < (uint32_t)it.end : n < n1 && there(t)) pages[u] = table[many_page(p, t)];
        }
    };
    auto find = [&](uint32_t n) {                          // ... and places
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const uint32_t t = IN_PAGE ? many_tile(it, n + lane / GROUPS) * TILE + (lane % GROUPS) * 16 : many_tile(it, n) * TILE + lane + 64 * u;
            const bool is = (uint32_t)pages[u] < (uint64_t)p.a.c.n_pages;
            const uint32_t in = t - many_page(p, t) * (uint32_t)p.a.c.page_tokens;
            rows_of[u] = is ? (int64_t)pages[u] * p.a.c.page_stride + (int64_t)((uint64_t)in * ts) : 0;
            if constexpr (!BF) scales_of[u] = is ? (int64_t)pages[u] * p.scale_stride + (int64_t)in * cache_scale_bytes(F, D) : 0;
            valid[u] = __ballot(is);
        }
    };
    int64_t rows_at[IN_PAGE ? NG : 1], scales_at[IN_PAGE ? NG : 1];          // IN_PAGE: of the wave's own 16 tokens, the same in all lanes
    uint64_t have[(TILE + 63) / 64];                       // tokens that are there, a bit each
    auto place = [&](uint32_t n) {
        const uint32_t t0 = many_tile(it, n) * TILE;
        if constexpr (IN_PAGE) {
            const int first = (int)((n - n0) % PER) * GROUPS;
            if (first == 0) {
                find(n);
                look(n + PER);
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                rows_at[g] = lane_value64(rows_of[0], first + wave * NG + g);
                if constexpr (!BF) scales_at[g] = lane_value64(scales_of[0], first + wave * NG + g);
            }
            const uint32_t is = (uint32_t)(valid[0] >> first) & ((1u << GROUPS) - 1u);
            if (is == (1u << GROUPS) - 1u && t0 + TILE <= (uint32_t)it.end && (p.window == 0u || t0 + TILE <= p.sinks || (int)t0 >= gap)) {
#pragma unroll
                for (int w = 0; w < (TILE + 63) / 64; ++w) have[w] = ~0ull;
                return;
            }
#pragma unroll
            for (int w = 0; w < (TILE + 63) / 64; ++w) {
                const bool wanted = there(t0 + 64 * w + lane), page = (is >> ((64 * w + lane) / 16) & 1u) != 0;
                have[w] = __ballot(wanted && page);
                if (__ballot(wanted && !page) && lane == 0) report_lowest(p.a.status, (uint32_t)it.b);
            }
        } else {
            find(n);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                const bool wanted = there(t0 + lane + 64 * u);
                have[u] = __ballot(wanted) & valid[u];
                if (have[u] != __ballot(wanted) && wanted && !(valid[u] >> lane & 1u)) report_lowest(p.a.status, (uint32_t)it.b);
            }
        }
    };
    // Whether the tile's tokens are all there and seen by all rows.
    auto is_full = [&](uint32_t n) {
        const uint32_t t0 = many_tile(it, n) * TILE, t1 = t0 + TILE - 1;
        bool full = true;
#pragma unroll
        for (int w = 0; w < (TILE + 63) / 64; ++w) full &= have[w] == ~0ull;
        return full && (!p.a.causal || (int)t1 <= it.at0) && (p.window == 0u || t1 < p.sinks || (int64_t)t0 > (int64_t)it.at1 - (int64_t)p.window);
    };

    // Bringing a tile in.  bf16: piece j of the wave's rows, lane after lane, by the order that the LDS has them in.
    constexpr int NJ = RPW * S::ROW / 1024;
    uint32_t k_off[BF ? NJ : 1], v_off[BF ? NJ : 1];
    Quarter<BF ? KVTC_CACHE_FP8 : F, D> kq[BF ? 1 : NG], vq[BF ? 1 : NG];
    if constexpr (BF) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const uint32_t byte = j * 1024 + lane * 16, in_wave = byte / S::ROW, slot = byte % S::ROW / 16, t = wave * RPW + in_wave;
            k_off[j] = (IN_PAGE ? (in_wave & 15) * ts : 0u) + ((slot ^ key_turn<D>(t)) << 4);
            v_off[j] = (IN_PAGE ? (in_wave & 15) * ts : 0u) + ((((slot >> 1) ^ value_turn<D>(t)) << 5) | (slot & 1) << 4);
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(KVTC_LDS uint8_t*)lds;
    // bf16: keys (side 0) or values (1) of the tile that was placed last, NJ loads
    auto bring_side = [&](int side, int buffer) {
        if constexpr (BF) {
            const uint32_t to = lds0 + (buffer * 2 + side) * S::BUFFER + wave * RPW * S::ROW;
            const ManyBytes from = side ? v0 : k0;
            const uint32_t* off_of = side ? v_off : k_off;
            if constexpr (IN_PAGE) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const int64_t off = rows_at[g];
                    constexpr int each = NJ / NG;
#pragma unroll
                    for (int j = 0; j < each; ++j) {
                        dma16_async((const void*)(uintptr_t)(from + off), off_of[g * each + j], to + (g * each + j) * 1024);
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const uint32_t t = wave * RPW + (j * 1024 + lane * 16) / S::ROW;
                    const int64_t off = shfl64(rows_of[TILE > 64 ? (wave * RPW) / 64 : 0], t & 63);
                    dma16_async((const void*)(uintptr_t)(from + off + off_of[j]), to + j * 1024);
                }
            }
        }
    };
    // 8 and 4 bits: both, into registers
    auto bring = [&]() {
        if constexpr (!BF) {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const int in_group = lane >> 2, quarter = lane & 3;
                int64_t off, scale_off;
                if constexpr (IN_PAGE) {
                    off = rows_at[g] + (uint32_t)(in_group * ts);
                    scale_off = scales_at[g] + in_group * cache_scale_bytes(F, D);
                } else {
                    const int t = wave * RPW + 16 * g + in_group;
                    off = shfl64(rows_of[TILE > 64 ? (wave * RPW) / 64 : 0], t & 63);
                    scale_off = shfl64(scales_of[TILE > 64 ? (wave * RPW) / 64 : 0], t & 63);
                }
                kq[g].load(k0 + off + quarter * Quarter<F, D>::kBytes, ks0 + scale_off);
                vq[g].load(v0 + off + quarter * Quarter<F, D>::kBytes, vs0 + scale_off);
            }
        }
    };
    float* exponents = reinterpret_cast<float*>(lds + S::kExponents);        // [buffer][16 tokens]: of values
    float* scales = reinterpret_cast<float*>(lds + S::kScales);              // 8 bits: [buffer][keys, values][token], values' without the 16 tokens' exponent; 4 bits: [buffer][group][token], of keys
    uint16_t* shifts = reinterpret_cast<uint16_t*>(lds + S::kScales + S::BUFFERS * TILE * G * 4);      // 4 bits: [buffer][token][group], of keys
    uint32_t* wild = reinterpret_cast<uint32_t*>(lds + S::kWild);            // [buffer][wave]: of its tokens, a bit each, those with values that are not finite
    // 8 and 4 bits: into the LDS, as numbers.
    auto settle = [&](int buffer, bool masked) {
        if constexpr (!BF) {
            uint32_t strange = 0;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const int in_group = lane >> 2, quarter = lane & 3, t = wave * RPW + 16 * g + in_group;
                const bool is = (have[TILE > 64 ? (wave * RPW) / 64 : 0] >> (t & 63) & 1u) != 0;
                auto over_rows = [&](float v) { return __uint_as_float(same(__float_as_uint(max_of_quarters(v)))); };
                int ve;
                float value_scale = 0.0f;
                bool odd = false;
                const float v_most = over_rows(is ? vq[g].most() : 0.0f);
                if constexpr (F == KVTC_CACHE_FP8) {
                    ve = v_most == 0.0f ? kLeastExponent : max(kLeastExponent, exponent_of(v_most));
                    value_scale = __uint_as_float(vq[g].scale[0]);
                    if (masked) {
                        odd = not_finite(value_scale);
                        value_scale = odd || !is ? 0.0f : value_scale;
                    }
                    if (quarter == 0) {
                        scales[(buffer * 2 + 0) * TILE + t] = __uint_as_float(kq[g].scale[0]);
                        scales[(buffer * 2 + 1) * TILE + t] = __builtin_amdgcn_ldexpf(value_scale, -ve);
                    }
                } else {
                    ve = max(0, exponent_of(v_most) - 14);
                    if (quarter == 0) {
#pragma unroll
                        for (int i = 0; i < G; ++i) {
                            scales[(buffer * G + i) * TILE + t] = (float)__builtin_bit_cast(_Float16, (uint16_t)(kq[g].scale[i] >> 16));
                            shifts[(buffer * TILE + t) * G + i] = (uint16_t)kq[g].scale[i];
                        }
                    }
                }
                if (lane == 0) exponents[buffer * (TILE / 16) + wave * NG + g] = (float)ve;
                uint8_t* to_k = lds + buffer * 2 * S::BUFFER + t * S::ROW;
                uint8_t* to_v = to_k + S::BUFFER;
                auto put_key = [&](int piece, u32x4 w) { *reinterpret_cast<u32x4*>(to_k + ((piece ^ key_turn<D>(t)) << 4)) = w; };
                if constexpr (F == KVTC_CACHE_FP8) kq[g].each(quarter, 0, put_key);
                else kq[g].each_code(quarter, put_key);
                vq[g].each(quarter, F == KVTC_CACHE_FP8 ? 0 : ve, [&](int piece, u32x4 w) {
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const bool high = (w[i] & 0x7c000000u) == 0x7c000000u, low = (w[i] & 0x7c00u) == 0x7c00u;
                            odd |= high || low;
                            w[i] &= is ? (high ? 0x0000ffffu : 0xffffffffu) & (low ? 0xffff0000u : 0xffffffffu) : 0u;
                        }
                    }
                    *reinterpret_cast<u32x4*>(to_v + ((((piece >> 1) ^ value_turn<D>(t)) << 5) | (piece & 1) << 4)) = w;
                });
                if (masked) {
                    const uint64_t b = __ballot(odd && is);
#pragma unroll
                    for (int i = 0; i < 16; ++i) strange |= (uint32_t)((b >> (4 * i) & 15u) != 0) << (16 * g + i);
                }
            }
            if (lane == 0) wild[buffer * NW + wave] = strange;
        }
    };
    // bf16, a masked tile: the wave's own tokens' values, in the LDS.
    auto clean = [&](int buffer, const uint64_t (&there_bits)[(TILE + 63) / 64]) {
        if constexpr (BF) {
            uint32_t strange = 0;
            constexpr int in_piece = 1024 / S::ROW, lanes = S::ROW / 16;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int in_wave = (j * 1024 + lane * 16) / S::ROW, t = wave * RPW + in_wave;
                const bool is = (there_bits[TILE > 64 ? (wave * RPW) / 64 : 0] >> (t & 63) & 1u) != 0;
                u32x4* at_lds = reinterpret_cast<u32x4*>(lds + (buffer * 2 + 1) * S::BUFFER + wave * RPW * S::ROW + j * 1024 + lane * 16);
                u32x4 w = *at_lds;
                bool odd = false;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const bool high = (w[i] & 0x7f800000u) == 0x7f800000u, low = (w[i] & 0x7f80u) == 0x7f80u;
                    odd |= high || low;
                    w[i] &= is ? (high ? 0x0000ffffu : 0xffffffffu) & (low ? 0xffff0000u : 0xffffffffu) : 0u;
                }
                if (odd || !is) *at_lds = w;
                const uint64_t b = __ballot(odd && is);
#pragma unroll
                for (int i = 0; i < in_piece; ++i)
                    strange |= (uint32_t)((b >> (lanes * i) & (lanes == 64 ? ~0ull : (1ull << lanes) - 1ull)) != 0) << (j * in_piece + i);
            }
            if (lane == 0) wild[buffer * NW + wave] = strange;
        }
    };

    // ---- a tile's products ----
    // LDS places of the operands, in buffer 0: keys of token `col` of every 32, and values of four tokens of a lane's feature
    uint32_t k_at[NS > 8 ? 8 : NS], v_at[NF > 4 ? 4 : NF];
    {
        const uint32_t slice = tw * NT, in = lane & 15, group = lane >> 4, t = 4 * (group >> 1) + (in >> 2);
#pragma unroll
        for (int s = 0; s < (NS > 8 ? 8 : NS); ++s) k_at[s] = lds0 + (slice + col) * S::ROW + (((2 * s + half) ^ key_turn<D>(col)) << 4);
#pragma unroll
        for (int f = 0; f < (NF > 4 ? 4 : NF); ++f)
            v_at[f] = lds0 + S::BUFFER + (slice + t) * S::ROW + (((2 * f + (group & 1)) ^ value_turn<D>(t)) << 5) + (in & 3) * 8;
    }
    // (masked tiles by the same code, with a step more where it is needed: with code of their own for them outputs were moved from registers to registers)
    u32x4 pr[2 * NB];                                      // probabilities
    auto scores = [&](bool masked, uint32_t n, int buffer, const uint64_t (&mine)[(TILE + 63) / 64]) {
        const uint32_t shift_of_buffer = buffer * 2 * S::BUFFER;
        const int t0 = (int)(many_tile(it, n) * TILE + tw * NT);
        f32x16 s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
        if constexpr (F == KVTC_CACHE_INT4) {
            // sum over groups of scale * (codes . queries) + shift * (sum of queries)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int t = tw * NT + 32 * b;
                u32x4 shift;
                if constexpr (G == 2) {
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(shifts + (buffer * TILE + t + col) * G);
                    shift = u32x4{w, w, w, w};
                } else if constexpr (G == 4) {
                    const u32x2 w = *reinterpret_cast<const u32x2*>(shifts + (buffer * TILE + t + col) * G);
                    shift = u32x4{w[0], w[1], w[0], w[1]};
                } else {
                    shift = *reinterpret_cast<const u32x4*>(shifts + (buffer * TILE + t + col) * G);
                }
#pragma unroll
                for (int n = 0; n < NSHIFT; ++n) s[b] = mfma<F>(shift, q_sums[n], s[b]);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    f32x16 dot;
#pragma unroll
                    for (int i = 0; i < 16; ++i) dot[i] = 0.0f;
#pragma unroll
                    for (int k = 2 * g; k < 2 * g + 2; ++k) {
                        const u32x4 a = *reinterpret_cast<const KVTC_LDS u32x4*>((uintptr_t)(k_at[k & 7] + shift_of_buffer + b * 32 * S::ROW + (k >> 3) * 256));
                        dot = mfma<F>(a, q[k], dot);
                    }
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f32x4 w = *reinterpret_cast<const f32x4*>(scales + (buffer * G + g) * TILE + t + 2 * i + 4 * half);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[b][i + j] = __builtin_fmaf(dot[i + j], w[j], s[b][i + j]);
                    }
                }
            }
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 6, 0);
#pragma unroll
            for (int n = 0; n < NB * (NSHIFT + NS); ++n) {
                __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsReads, 3, 0);
            }
        } else {
#pragma unroll
            for (int k = 0; k < NS; ++k)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const u32x4 a = *reinterpret_cast<const KVTC_LDS u32x4*>((uintptr_t)(k_at[k & 7] + shift_of_buffer + b * 32 * S::ROW + (k >> 3) * 256));
                    s[b] = mfma<F>(a, q[k], s[b]);
                }
            // (a few loads ahead of the products, no more: the compiler left to itself puts them all first, and what they load does not fit the registers)
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 8, 0);
#pragma unroll
            for (int k = 0; k < NS * NB; ++k) {
                __builtin_amdgcn_sched_group_barrier(kProducts, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kLdsReads, 1, 0);
            }
        }
        if constexpr (F == KVTC_CACHE_FP8) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4 w = *reinterpret_cast<const f32x4*>(scales + (buffer * 2 + 0) * TILE + tw * NT + 32 * b + 2 * i + 4 * half);
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[b][i + j] *= w[j];
                }
        }
        if (masked) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int t = t0 + 32 * b, in_tile = tw * NT + 32 * b;
                uint32_t seen = (uint32_t)(mine[in_tile / 64] >> (in_tile % 64));
                if (p.a.causal) {
                    seen &= low_bits(at - t + 1);
                    if (p.window != 0u) seen &= low_bits((int)p.sinks - t) | ~low_bits(from - t);
                }
                seen >>= 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = seen >> (8 * (i / 4) + i % 4) & 1u ? s[b][i] : kNoScore;
            }
        }
        // the values' exponents, of every 16 tokens
        int ve[2 * NB], ve_most = kLeastExponent;
        if constexpr (!BF) {
#pragma unroll
            for (int g = 0; g < 2 * NB; ++g) {
                ve[g] = (int)same((uint32_t)(int)exponents[buffer * (TILE / 16) + tw * (NT / 16) + g]);
                ve_most = max(ve_most, ve[g]);
            }
        }
        float top = kNoScore;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            float g0 = s[b][0], g1 = s[b][8];
#pragma unroll
            for (int i = 1; i < 8; ++i) {
                g0 = fmaxf(g0, s[b][i]);
                g1 = fmaxf(g1, s[b][8 + i]);
            }
            top = fmaxf(top, fmaxf(g0, g1));
        }
        top = max_of_halves(top * factor);
        if (__any(top > m + slack<F>()) || (!BF && ve_most > exponent + kExponentSlack)) {
            const float now = fmaxf(m, top);
            base = now == kNoScore ? 0.0f : now;
            float keep = exp2_fast(m - base);
            l *= keep;
            m = now;
            if constexpr (!BF) {
                const int e = max(exponent, ve_most);
                keep = __builtin_amdgcn_ldexpf(keep, exponent - e);
                exponent = e;
            }
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[f][i] *= keep;
        }
#pragma unroll
        for (int g = 0; g < 2 * NB; ++g) {
            int dv = 0;
            if constexpr (!BF) dv = max(ve[g] - exponent, -60) + kBias;
            const float off = BF ? base : base - (float)dv;
            float sum = 0.0f, e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = exp2_fast(__builtin_fmaf(s[g / 2][8 * (g & 1) + i], factor, -off));
                sum += e[i];
            }
            l += BF ? sum : __builtin_amdgcn_ldexpf(sum, -dv);
            if constexpr (F == KVTC_CACHE_FP8) {
#pragma unroll
                for (int i = 0; i < 8; i += 4) {
                    const f32x4 w = *reinterpret_cast<const f32x4*>(scales + (buffer * 2 + 1) * TILE + tw * NT + 16 * g + 2 * i + 4 * half);
#pragma unroll
                    for (int j = 0; j < 4; ++j) e[i + j] *= w[j];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) pr[g][i] = round_pair<F>(e[2 * i], e[2 * i + 1]);
        }
    };
    auto sums = [&](bool masked, uint32_t n, int buffer) {
        const uint32_t shift = buffer * 2 * S::BUFFER;
#pragma unroll
        for (int g = 0; g < 2 * NB; ++g)
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const uint32_t place_v = v_at[f & 3] + shift + 16 * g * S::ROW + (f >> 2) * 256;
                const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((KVTC_LDS s16x4*)(uintptr_t)place_v));
                const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((KVTC_LDS s16x4*)(uintptr_t)(place_v + 8 * S::ROW)));
                o[f] = mfma<F>(u32x4{a[0], a[1], b[0], b[1]}, pr[g], o[f]);
            }
        __builtin_amdgcn_sched_group_barrier(kLdsReads, F == KVTC_CACHE_INT4 ? 4 : 12, 1);
#pragma unroll
        for (int k = 0; k < 2 * NB * NF; ++k) {
            __builtin_amdgcn_sched_group_barrier(kProducts, 1, 1);
            __builtin_amdgcn_sched_group_barrier(kLdsReads, 2, 1);
        }
        if (masked) {
            for (int w = S::ALONE ? wave : 0; w < (S::ALONE ? wave + 1 : NW); ++w) {      // values that are not finite, to the rows that see them
                uint32_t bits = same(wild[buffer * NW + w]);
                while (bits) {
                    const int in_tile = w * RPW + __builtin_ctz(bits), t = (int)(many_tile(it, n) * TILE) + in_tile;
                    bits &= bits - 1;
                    if (in_tile / NT != tw) continue;
                    const uint32_t index = many_page(p, (uint32_t)t), in = (uint32_t)t - index * (uint32_t)p.a.c.page_tokens;
                    const int64_t page = table[index];
                    const ManyBytes at_row = v0 + page * p.a.c.page_stride + (int64_t)((uint64_t)in * ts), at_scales = vs0 + page * p.scale_stride + (int64_t)in * cache_scale_bytes(F, D);
                    const bool seen = many_sees(p, at, t);
#pragma unroll
                    for (int f = 0; f < NF; ++f)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float x = value_at<F, D>(at_row, at_scales, 32 * f + 8 * (i / 4) + 4 * half + i % 4);
                            if (seen && not_finite(x)) o[f][i] += x;
                            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);      // (a rare path: not all of its loads at once, in registers that the others need)
                        }
                }
            }
        }
    };

    // Whether the wave has rows that see anything of tile n, and whether it has to mask them.
    auto is_seen = [&](uint32_t n, bool full) { return any_row && (full || !p.a.causal || (int)(many_tile(it, n) * TILE + tw * NT) <= last_at); };
    auto is_masked = [&](uint32_t n, bool full, const uint64_t (&mine)[(TILE + 63) / 64]) {
        if (full) return false;
        const uint32_t t0 = many_tile(it, n) * TILE + tw * NT;
        const uint64_t bits = mine[tw * NT / 64] >> (tw * NT % 64);
        return !((!p.a.causal || (int)(t0 + NT - 1) <= first_at) && (p.window == 0u || t0 + NT - 1 < p.sinks || (int)t0 >= last_from) && (NT == 64 ? bits == ~0ull : (uint32_t)bits == 0xffffffffu));
    };
    constexpr int WORDS = (TILE + 63) / 64;
    uint64_t now_have[WORDS], next_have[WORDS];
    bool now_full, next_full = true;
    if (n0 == n1) {                                        // (rows that see nothing)
    } else if constexpr (BF) {
        // A tile's keys are asked for when the scores of the tile two before it are done, its values a barrier later; each has a tile and a half to arrive.  Loads come back in their order: what may be on its way
        // still, when keys or values are waited for, is what was asked for after them.  What a wave reads out of the LDS it has before others write there.
        auto arrive = [&](bool two, bool keys) {           // two: the next tile's keys and values are on their way as well
            if (two) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * NJ) : "memory");
            else if (keys) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(NJ) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            if constexpr (!S::ALONE) asm volatile("s_barrier" ::: "memory");
        };
        look(n0);
        place(n0);
        now_full = is_full(n0);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) now_have[w] = have[w];
        bring_side(0, 0);
        bring_side(1, 0);
        if constexpr (!IN_PAGE) look(n0 + 1);
        if (n0 + 1 < n1) {
            place(n0 + 1);
            next_full = is_full(n0 + 1);
            bring_side(0, 1);
            if constexpr (!IN_PAGE) look(n0 + 2);
        }
#pragma unroll
        for (int w = 0; w < WORDS; ++w) next_have[w] = have[w];
        for (uint32_t n = n0; n < n1; ++n) {
            const int buffer = (int)(n - n0) & 1;
            arrive(n + 1 < n1, true);
            if (n + 1 < n1) bring_side(1, buffer ^ 1);     // (all waves are through with the values before)
            const bool seen = is_seen(n, now_full), masked = is_masked(n, now_full, now_have);
            if (seen) scores(masked, n, buffer, now_have);
            arrive(n + 1 < n1, false);
            bool then_full = true;
            if (n + 2 < n1) {                              // (all waves are through with the keys)
                place(n + 2);
                then_full = is_full(n + 2);
                bring_side(0, buffer);
                if constexpr (!IN_PAGE) look(n + 3);
            }
            if (!now_full) {
                clean(buffer, now_have);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                if constexpr (!S::ALONE) asm volatile("s_barrier" ::: "memory");
            }
            if (seen) sums(!now_full, n, buffer);
            now_full = next_full;
            next_full = then_full;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                now_have[w] = next_have[w];
                next_have[w] = have[w];
            }
        }
    } else {
        look(n0);
        place(n0);
        bring();
        now_full = is_full(n0);
#pragma unroll
        for (int w = 0; w < WORDS; ++w) now_have[w] = have[w];
        if constexpr (!IN_PAGE) look(n0 + 1);
        settle(0, !now_full);
        for (uint32_t n = n0; n < n1; ++n) {
            const int buffer = S::BUFFERS == 1 ? 0 : (int)(n - n0) & 1, next = S::BUFFERS - 1 - buffer;
            if constexpr (S::ALONE) asm volatile("" ::: "memory");   // (a wave's accesses to the LDS are done in their order, which the compiler is to keep)
            else __syncthreads();
            next_full = true;
            if (n + 1 < n1) {
                place(n + 1);
                next_full = is_full(n + 1);
                bring();
                if constexpr (!IN_PAGE) look(n + 2);
            }
            if (is_seen(n, now_full)) {
                scores(is_masked(n, now_full, now_have), n, buffer, now_have);
                sums(!now_full, n, buffer);
            }
            if constexpr (S::ALONE) asm volatile("" ::: "memory");
            if (n + 1 < n1) settle(next, !next_full);
            now_full = next_full;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) now_have[w] = have[w];
        }
    }

    // ---- results ----
    l = sum_of_halves(l);
    if constexpr (!BF) {
        if (exponent == -200) exponent = 0;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[f][i] = __builtin_amdgcn_ldexpf(o[f][i], exponent - kBias);
    }
    if constexpr (TW > 1) {                                // the waves that have the same rows
        float* parts = reinterpret_cast<float*>(lds) + rw * (TW / 2) * (NF * 16 + 2) * 64;
#pragma unroll
        for (int step = 1; step < TW; step *= 2) {
            __syncthreads();
            if (tw % (2 * step) == step) {
                float* to = parts + (tw / (2 * step)) * (NF * 16 + 2) * 64 + lane;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int i = 0; i < 16; ++i) to[(16 * f + i) * 64] = o[f][i];
                to[NF * 16 * 64] = m;
                to[(NF * 16 + 1) * 64] = l;
            }
            __syncthreads();
            if (tw % (2 * step) == 0) {
                const float* of = parts + (tw / (2 * step)) * (NF * 16 + 2) * 64 + lane;
                const float other = of[NF * 16 * 64], now = fmaxf(m, other), zero = now == kNoScore ? 0.0f : now, a = exp2_fast(m - zero), b = exp2_fast(other - zero);
                l = l * a + of[(NF * 16 + 1) * 64] * b;
                m = now;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[f][i] = o[f][i] * a + of[(16 * f + i) * 64] * b;
            }
        }
        if (tw != 0) return;
    }
    if (!is_row) return;
    const int64_t at_out = (int64_t)(it.first + token) * p.a.n_q_heads + q_head;
    if (!whole) {
        float* out = p.part_out + ((int64_t)part * p.a.n_tokens * p.a.n_q_heads + at_out) * D;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<f32x4*>(out + 32 * f + 8 * (i / 4) + 4 * half) = f32x4{o[f][i], o[f][i + 1], o[f][i + 2], o[f][i + 3]};
        if (half == 0) p.part_sums[(int64_t)part * p.a.n_tokens * p.a.n_q_heads + at_out] = make_float2(m, l);
        return;
    }
    const bool none = m == kNoScore && l == 0.0f;
    const float inverse = none ? 0.0f : 1.0f / l;
    uint16_t* out = static_cast<uint16_t*>(p.a.out) + at_out * D;
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            u32x2 w;
#pragma unroll
            for (int j = 0; j < 2; ++j) w[j] = none ? 0u : (uint32_t)f32_bf16(o[f][i + 2 * j] * inverse) | (uint32_t)f32_bf16(o[f][i + 2 * j + 1] * inverse) << 16;
            *reinterpret_cast<u32x2*>(out + 32 * f + 8 * (i / 4) + 4 * half) = w;
        }
    if (p.a.lse && half == 0) p.a.lse[at_out] = none ? kNoScore : (m + __builtin_log2f(l)) * kLn2;
}

template <int F, int D, int RW, int TW, int TOKENS>
static hipError_t launch_shape(const ManyPlan& p, hipStream_t stream) {
    using S = Shape<F, D, RW, TW, TOKENS>;
    const dim3 grid(p.a.c.n_heads, p.r.items, p.r.parts), block(64 * S::NW);
    constexpr int lds = S::kLds > (TW > 1 ? RW * (TW / 2) * (S::NF * 16 + 2) * 256 : 0) ? S::kLds : RW * (TW / 2) * (S::NF * 16 + 2) * 256;
    if (p.a.c.page_tokens % 16 == 0) {
        const hipError_t e = allow_full_lds(reinterpret_cast<const void*>(&many_mfma_kernel<F, D, RW, TW, TOKENS, true>));
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((many_mfma_kernel<F, D, RW, TW, TOKENS, true>), grid, block, lds, stream, p);
    } else {
        const hipError_t e = allow_full_lds(reinterpret_cast<const void*>(&many_mfma_kernel<F, D, RW, TW, TOKENS, false>));
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((many_mfma_kernel<F, D, RW, TW, TOKENS, false>), grid, block, lds, stream, p);
    }
    return hipGetLastError();
}
template <int F, int D>
static hipError_t launch_kind(const ManyPlan& p, hipStream_t stream) {
    if (p.r.kind == kManyWide) return launch_shape<F, D, 4, 1, 64>(p, stream);
    if (p.r.kind == kManyTwo) return launch_shape<F, D, 2, 2, 32>(p, stream);
    return launch_shape<F, D, 1, D == 256 && F == KVTC_CACHE_BF16 ? 2 : 4, 32>(p, stream);
}

#define KVTC_MANY_NAME2(n) launch_many_mfma_##n
#define KVTC_MANY_NAME(n) KVTC_MANY_NAME2(n)
hipError_t KVTC_MANY_NAME(KVTC_MANY_PART)(const ManyPlan& p, hipStream_t stream) { return launch_kind<KVTC_MANY_PART / 3, 64 << (KVTC_MANY_PART % 3)>(p, stream); }

}  // namespace kvtc

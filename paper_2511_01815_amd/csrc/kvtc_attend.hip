// Attention of one new token of every sequence over the pages of a live cache, for gfx950.
//
// One pass over keys and values with the running maximum m and sum l of a softmax: for the scores s of some more tokens,
//     m' = max(m, s),  l' = l e^(m - m') + sum e^(s - m'),  o' = o e^(m - m') + sum e^(s - m') v.
// Bytes bound it: every key and value is used for the few query heads of its group only.  (64 ragged rows of 512 to 16384 tokens, 8 heads of 128 features, bf16:
// 207 us for 1146 MB, 5.5 TB/s, the rate at which this card reads at all.  One row of 131072 tokens in 8 bits: 61.5 us, 4.5 TB/s.  4 bits: 16 rows of 32768 tokens 154 us, 4.2 TB/s, where the
// vector unit's unpacking and scaling is in the way as well.)
//
// Work.  An item is (sequence, KV head, up to 16 of its query heads); its tokens come in tiles of four pieces of 32, one to a wave.  The tiles of all
// items, one after another, are cut into as many equal shares as there are workgroups: whatever the lengths, all workgroups have
// the same amount to read, and a share begins and ends inside an item where it happens to.  Parts of an item are left in the
// workspace as (m, l, o); the last of its workgroups to arrive joins them, in their order.  Many short rows are a wave's each instead, whole.
// (A tile has eight pieces where a step has two; and of an item made of several KV heads, whose rows share cache lines, a wave or two to each.)
//
// Products.  Matrix instructions of 16 x 16 x 32, tokens in the rows and query heads in the columns: S^T = K Q^T, O^T = V^T P^T.  Both sum over an
// index whose order is free, so long as both operands have the same one, and so
//   keys    a lane has 16 bytes of one token (lane % 16): the operand as it lies in memory; the queries are laid out to match
//   scores  a lane has those of one query head (lane % 16) and four tokens, 4 (lane / 16) + 0..3, of each of two products: the
//           8 tokens that its part of the next operand needs -- probabilities never leave their registers
//   values  a lane has d / 16 neighbouring features of those 8 tokens (a row over 16 lanes), and turns 8 tokens x d / 16 features into d / 16
//           operands by byte permutations: a matrix product for every d / 16-th feature
// Nothing goes through the LDS before the four waves' results are joined.
//
// 8 bits: E4M3 codes are bf16 values; scores and probabilities take the token's scale.  4 bits: byte pair * G + group of a row
// (G = d / 32 groups) holds two neighbouring features, so that a lane's bytes are of one pair or four and of every group.  A code as it stands is the bf16
// pattern of a number below the normal ones, code * 2^-133, and the matrix unit takes such numbers for what they are: a code needs no conversion, but a mask; and the
// high code of a byte, where it stands, is 16 of them.  Scores: per group a product of its own, times the token's scale, plus the query's sum times its shift.  Values:
// per group the probabilities times the tokens' scales; low codes, and whole bytes, low + 16 high, from which the low ones' sums are taken in the end; shifts by
// sums apart.  (With 128 + code from an or, and the 128s taken off by products of their own: 16 rows of 32768 tokens 164 us for 153, with fp32 queries 245 for 199.)
// Probabilities have 24 bits and their operand 8: they enter as a sum of three operands.  In 4 bits with bf16 outputs, where the vector unit has no time to spare, of two, both to nearest, 18 bits: the error
// is one of code * scale, larger than the value where a group lies around zero, but 32 times below the output's rounding.  (16 rows of 32768 tokens 154 us with two and 161 with three, head-major pages 144 and 154;
// in bf16 64 ragged rows 206.4 and 207.0, in 8 bits 212 and 210.)  With bf16 values, which may be infinite, all parts have one sign and none is zero, so that an infinite value stays one; where its
// probability is zero, e^-88 and less in fp32, it makes NaN, as zero times infinity does.
#include <hip/hip_runtime.h>
#include "kvtc_cache.h"
#include "kvtc_dev.h"
#include "kvtc_numeric.h"

namespace kvtc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kAttendCols = 16;                            // query heads of an item, at most
constexpr int kAttendMaxShares = 1024;                     // shares of a launch, at most: a counter each in the workspace
// Rows of at most so many pieces may be a wave's each, whole: no shares to find, nothing to join, and a workgroup takes the next row as it ends; but the last rows run alone, and in 4 bits
// a step is of one piece.  (256 rows of 8 heads of 128 features, us, shares and so.  bf16: 40 tokens 20.4 and 13.5, 300 65.6 and 61.4, 100 to 1000 102 and 94, 200 to 2000 166 and 178; 8 bits: 300
// 45.2 and 36.9, 100 to 1000 77.5 and 67.8, 200 to 2000 110 and 126; 4 bits: 300 49.6 and 38.8, 512 61.8 and 58.6, 1 to 600 41.9 and 53.9, 100 to 1000 76 and 92.)
constexpr int short_pieces(int format) { return format == KVTC_CACHE_INT4 ? 16 : 32; }
// Workgroups to a compute unit, by their registers.  (Three of 64 features, unless there are less than two tiles for each: 16 heads, 8 rows of 32768 tokens in bf16 219 us with two and 199 with three, 16
// rows in 8 bits 251 and 216, in 4 bits 200 and 209, with fp32 queries 258 and 220; 24 rows of 0 to 4001 tokens of 12 heads in 8 bits, with two tiles for each of two workgroups, 15.3 and 18.0.  Two of 128 features: three have registers
// enough in 8 bits, and 64 rows of 4096 tokens took 111 us for 101.)
__host__ __device__ constexpr int groups_each(int format, int d, bool bf16) { return d == 256 ? 1 : d == 64 && !(bf16 && format == KVTC_CACHE_INT4) ? 3 : 2; }
constexpr float kNoScore = -__builtin_huge_valf();

struct AttendPlan {                                        // what the host works out
    AttendArgs a;
    int32_t group, parts, cols;                            // query heads of a KV head; items that share them; of each, at most
    int32_t in_page;                                       // 16 tokens from a multiple of 16 on lie in one page
    int32_t seqs_each;                                     // sequences whose lengths a lane adds up
    uint32_t max_tokens, sinks, window;                    // those of `a`, at most 2^31 - 1
    int32_t in_turn;                                       // shares go to the XCDs in turn
    uint32_t few;                                          // shares of less than two tiles: so many at most
    int64_t scale_stride;                                  // bytes of a page's scales
    uint32_t page_mul, page_shift;                         // token / page_tokens = token * page_mul >> page_shift
};

// The call's arguments once more, from memory: where they are used outside the loop over the tokens, that they need not be kept in scalar registers, nor, where these do not do, in lanes of
// vector registers, through it.  (The kernels' first and only argument.)
typedef const __attribute__((address_space(4))) AttendPlan& ScalarPlan;
__device__ __forceinline__ ScalarPlan plan_again() {
    uint64_t at = reinterpret_cast<uint64_t>(__builtin_amdgcn_kernarg_segment_ptr());
    asm volatile("" : "+s"(at));
    return *reinterpret_cast<const __attribute__((address_space(4))) AttendPlan*>(at);
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ bf16x8 operand(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf16x8, u32x4{a, b, c, d}); }
__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// The larger of what lanes 16 and 32 apart hold, in all lanes.
__device__ __forceinline__ float max_over_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_quarters(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// the high halves of two words (bf16 by cutting), first one low
__device__ __forceinline__ uint32_t high_halves(uint32_t first, uint32_t second) { return __builtin_amdgcn_perm(second, first, 0x07060302u); }
__device__ __forceinline__ uint32_t low_halves(uint32_t first, uint32_t second) { return __builtin_amdgcn_perm(second, first, 0x05040100u); }
__device__ __forceinline__ float cut(float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); }
__device__ __forceinline__ uint32_t round_pair(float first, float second) {
    bf16x2 v;
    v[0] = (__bf16)first;
    v[1] = (__bf16)second;
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float half_of(uint32_t w, int high) { return (float)__builtin_bit_cast(_Float16, (uint16_t)(high ? w >> 16 : w)); }

// Eight values as a sum of PARTS operands.  (Two parts, each to nearest: within 2^-18; three: all 24 bits, of values of at least 2^-109.)
// One sign, for what goes with bf16 features, which may be infinite: all parts have the value's sign, and none is zero where the value is not, lest an infinity times zero make NaN of another part's
// infinity.  The least part that there is, 2^-133, is below what a probability may be off by in fp32 (2^-126), whatever feature it meets; a value of zero has parts of zero.
enum class Signs { kAny, kOne, kPositive };                // (kPositive: kOne of values that are not negative)
template <int PARTS, Signs SIGNS>
__device__ __forceinline__ void split(const float (&v)[8], bf16x8 (&out)[PARTS]) {
    static_assert(PARTS != 2 || SIGNS == Signs::kAny, "the second of two may have another sign");
    constexpr bool kNearest = PARTS == 2;
    float rest[8];
    uint32_t w[4];
    auto first = [&](int i) { return !kNearest ? cut(v[i]) : __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16); };
    auto least = [](float r, float of) {
        if constexpr (SIGNS == Signs::kAny) return r;
        else if constexpr (SIGNS == Signs::kPositive) return fmaxf(r, fminf(of, 0x1p-133f));
        else return __builtin_copysignf(fmaxf(__builtin_fabsf(r), fminf(__builtin_fabsf(of), 0x1p-133f)), of);
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = PARTS == 1 || kNearest ? round_pair(v[2 * i], v[2 * i + 1]) : high_halves(__float_as_uint(v[2 * i]), __float_as_uint(v[2 * i + 1]));
    out[0] = operand(w[0], w[1], w[2], w[3]);
    if constexpr (PARTS > 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) rest[i] = least(v[i] - first(i), v[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = PARTS > 2 ? high_halves(__float_as_uint(rest[2 * i]), __float_as_uint(rest[2 * i + 1])) : round_pair(rest[2 * i], rest[2 * i + 1]);
        out[1] = operand(w[0], w[1], w[2], w[3]);
    }
    if constexpr (PARTS > 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = round_pair(least(rest[2 * i] - cut(rest[2 * i]), v[2 * i]), least(rest[2 * i + 1] - cut(rest[2 * i + 1]), v[2 * i + 1]));
        out[2] = operand(w[0], w[1], w[2], w[3]);
    }
}

// A constant whose value the compiler is not told, so that v * half + zero is one instruction.
struct Constants { float zero; };
__device__ __forceinline__ Constants constants() {
    Constants c{0.0f};
    asm volatile("" : "+s"(c.zero));
    return c;
}

// ---- the tokens in hand --------------------------------------------------------------------------------------------------------

#define KVTC_GLOBAL __attribute__((address_space(1)))
typedef const KVTC_GLOBAL uint8_t* Bytes;                  // (said to be global memory, so that a place kept in scalar registers stays known as that)
__device__ __forceinline__ Bytes bytes_at(const void* p) { return reinterpret_cast<Bytes>(reinterpret_cast<uintptr_t>(p)); }
// BYTES of a row, in dwords (or half of one).
template <int BYTES>
__device__ __forceinline__ void load(Bytes p, uint32_t* w) {
    if constexpr (BYTES == 2) w[0] = *reinterpret_cast<const KVTC_GLOBAL uint16_t*>(p);
    else if constexpr (BYTES == 4) w[0] = *reinterpret_cast<const KVTC_GLOBAL uint32_t*>(p);
    else if constexpr (BYTES == 8) { const u32x2 v = *reinterpret_cast<const KVTC_GLOBAL u32x2*>(p); w[0] = v[0]; w[1] = v[1]; }
    else {
#pragma unroll
        for (int i = 0; i < BYTES / 16; ++i) {
            const u32x4 v = reinterpret_cast<const KVTC_GLOBAL u32x4*>(p)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
        }
    }
}
// Values that are the same in all lanes, back in scalar registers.
__device__ __forceinline__ uint32_t same(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ uint64_t same64(uint64_t v) { return (uint64_t)same((uint32_t)(v >> 32)) << 32 | same((uint32_t)v); }
// Of such values (divisions are the vector unit's; one of 64 bits costs several times one of 32).
__device__ __forceinline__ uint64_t quotient(uint64_t n, uint64_t d) {
    if ((n | d) >> 32) return same64(n / d);
    return same((uint32_t)n / (uint32_t)d);
}
__device__ __forceinline__ int64_t shfl64(int64_t v, int from) {
    const int lo = __shfl((int)(uint32_t)v, from, 64), hi = __shfl((int)(v >> 32), from, 64);
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}

// What the tokens of an item (a sequence, a KV head) have in common; the same in all lanes.  (Few words: with the call's arguments at hand instead, the scalar registers did not
// do, and half of the vector unit's work in 8 bits was to keep and fetch theirs.)
struct Item {
    const int32_t* table;
    Bytes k, v, k_scales, v_scales;                        // the head's, in page 0
    uint32_t length, from, sinks, b;
};
// A place that is the same in all lanes, in scalar registers, and 32 bits of the lane's own.  (The compiler left to itself keeps these as 64 bits, and adds them up for every load.)
__device__ __forceinline__ Bytes lane_at(Bytes base, int64_t offset, uint32_t lane) {
    const uint64_t p = reinterpret_cast<uint64_t>(base + offset);
    const uint64_t q = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p);
    asm volatile("" : "+v"(lane));
    return reinterpret_cast<Bytes>(q) + lane;
}
// Where a wave's 32 tokens are, and which of them are seen.
template <bool IN_PAGE>
struct Where {
    uint32_t seen;             // a bit each, the same in all lanes; none: nothing is loaded
    int64_t row[IN_PAGE ? 2 : 1], scale[IN_PAGE ? 2 : 1];      // bytes from the item's bases.  IN_PAGE: of the first token of each half, the same in all lanes; else of token lane % 32
};
// The same before the pages are known: their numbers are on their way, and are not waited for until the places are worked out, a step later.  (The vector
// unit's loads come back in order: a look that is waited for at once waits for the keys and values before it.)  IN_PAGE: 16 tokens lie in one
// page, and the numbers come through the scalar cache.
template <bool IN_PAGE>
struct Look {
    uint32_t seen, token;
    int32_t page[IN_PAGE ? 2 : 1];
};
typedef const __attribute__((address_space(4))) int32_t* ScalarInts;
__device__ __forceinline__ int32_t scalar_at(const int32_t* p, int64_t i) { return reinterpret_cast<ScalarInts>(reinterpret_cast<uintptr_t>(p))[i]; }

__device__ __forceinline__ uint32_t page_index(const AttendPlan& p, uint32_t token) { return (uint32_t)(((uint64_t)token * p.page_mul) >> p.page_shift); }

// t: the first of the 32 tokens, below 2^31
template <bool IN_PAGE>
__device__ __forceinline__ Look<IN_PAGE> look_at(const AttendPlan& p, const Item& item, uint32_t t) {
    auto below = [&](uint32_t end) {                       // of the 32 tokens, those before `end`
        const int32_t n = (int32_t)(end - t);
        return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
    };
    Look<IN_PAGE> w;
    w.seen = below(item.length) & (below(item.sinks) | ~below(item.from));
    if constexpr (IN_PAGE) {
        w.token = t;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            w.page[n] = 0;
            if (w.seen >> (16 * n) & 0xffffu) w.page[n] = scalar_at(item.table, page_index(p, w.token + 16 * n));
        }
    } else {
        const int mine = (int)(threadIdx.x & 31);
        w.token = t + mine;
        w.page[0] = 0;
        if (w.seen >> mine & 1u) w.page[0] = item.table[page_index(p, w.token)];
    }
    return w;
}

template <int SW, bool IN_PAGE>
__device__ __forceinline__ Where<IN_PAGE> where(const AttendPlan& p, const Item& item, const Look<IN_PAGE>& l) {
    Where<IN_PAGE> w;
    w.seen = l.seen;
    auto place = [&](uint32_t token, int32_t page, int64_t& row, int64_t& scale) {
        const uint32_t in = token - page_index(p, token) * (uint32_t)p.a.c.page_tokens;
        row = (int64_t)page * p.a.c.page_stride + (uint32_t)(in * (uint32_t)p.a.c.token_stride);
        scale = (int64_t)page * p.scale_stride + (int64_t)((uint64_t)in * (4 * SW));
    };
    if constexpr (IN_PAGE) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const uint32_t mine = 0xffffu << (16 * n);
            w.row[n] = w.scale[n] = 0;
            if ((l.seen & mine) == 0u) continue;
            if ((uint32_t)l.page[n] < (uint32_t)p.a.c.n_pages) {
                place(l.token + 16 * n, l.page[n], w.row[n], w.scale[n]);
            } else {
                if ((threadIdx.x & 63) == 0) report_lowest(plan_again().a.status, item.b);
                w.seen &= ~mine;
            }
        }
    } else {
        w.row[0] = w.scale[0] = 0;
        const bool mine = l.seen >> (threadIdx.x & 31) & 1u, is = mine && (uint32_t)l.page[0] < (uint32_t)p.a.c.n_pages;
        if (is) place(l.token, l.page[0], w.row[0], w.scale[0]);
        else if (mine) report_lowest(plan_again().a.status, item.b);
        w.seen = (uint32_t)__ballot(is);
    }
    return w;
}

template <int F, int D>
struct Shape {
    static constexpr int NK = D / 32;                                          // products over a row of keys; groups of the 4-bit format
    static constexpr int KW = F == KVTC_CACHE_BF16 ? 4 * NK : F == KVTC_CACHE_FP8 ? 2 * NK : NK;      // dwords of a lane's part of a row of keys
    static constexpr int VB = F == KVTC_CACHE_BF16 ? 4 * NK : F == KVTC_CACHE_FP8 ? 2 * NK : NK;      // bytes of a lane's part of a row of values
    static constexpr int VW = (VB + 3) / 4;
    static constexpr int SW = F == KVTC_CACHE_BF16 ? 0 : F == KVTC_CACHE_FP8 ? 1 : NK;                // dwords of a row's scales
    static constexpr int NO = D / 16;                                          // products for the features
};

// A lane's parts of J pieces of 32 tokens.  Of a row's 16 columns a group of few query heads fills few, and what the vector unit does to scores and probabilities it does to
// all: with J > 1 the columns come in J sets of 16 / J, each with all the heads, and a set keeps the scores of its own piece only.  Then a lane has its 8 tokens' scales of
// one piece, the softmax is worked out once for 32 J tokens, and each set has its own maximum and sums, joined at the end like those of waves.
// Keys: of tokens lane % 16 and 16 + lane % 16 of each piece, and the scales of the lane's 8 tokens.
template <int F, int D, int J>
struct Keys {
    using S = Shape<F, D>;
    uint32_t w[J][2][S::KW], scale[8][S::SW > 0 ? S::SW : 1];
};
template <int F, int D, int J>
struct Values {
    using S = Shape<F, D>;
    uint32_t w[J][8][S::VW], scale[8][S::SW > 0 ? S::SW : 1];
};
// the set of a column
template <int J> __device__ __forceinline__ int set_of(int col) { return col / (kAttendCols / J); }
template <int J, bool IN_PAGE>
__device__ __forceinline__ uint32_t any_seen(const Where<IN_PAGE> (&at)[J]) {
    uint32_t seen = 0u;
#pragma unroll
    for (int j = 0; j < J; ++j) seen |= at[j].seen;
    return seen;
}

// the k-th of the lane's 8 tokens, among the wave's 32
__device__ __forceinline__ int token_of(int k, int quarter) { return (k < 4 ? k : 12 + k) + 4 * quarter; }

template <int F, int D, bool IN_PAGE, int J>
__device__ __forceinline__ void load_scales(Bytes scales, const Where<IN_PAGE> (&at)[J], int lane, uint32_t (&out)[8][Shape<F, D>::SW > 0 ? Shape<F, D>::SW : 1]) {
    constexpr int SW = Shape<F, D>::SW;
    const int quarter = lane >> 4;
    if constexpr (SW > 0) {
        if constexpr (IN_PAGE) {                           // the four tokens' scales lie side by side
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                uint32_t w[4 * SW];
                if constexpr (J == 1) {
                    load<16 * SW>(lane_at(scales, at[0].scale[n], quarter * 16 * SW), w);
                } else {
                    int64_t mine = at[0].scale[n];
#pragma unroll
                    for (int j = 1; j < J; ++j) mine = set_of<J>(lane & 15) == j ? at[j].scale[n] : mine;
                    load<16 * SW>(scales + mine + quarter * 16 * SW, w);
                }
#pragma unroll
                for (int i = 0; i < 4 * SW; ++i) out[4 * n + i / SW][i % SW] = w[i];
            }
        } else {
            static_assert(IN_PAGE || J == 1, "");
#pragma unroll
            for (int k = 0; k < 8; ++k) load<4 * SW>(scales + shfl64(at[0].scale[0], token_of(k, quarter)), out[k]);
        }
    }
}

// (Tokens that are not seen: IN_PAGE, rows of the same page or, of halves without a seen token, the first rows of page 0, which exist; else the first row of page 0.)
template <int F, int D, bool IN_PAGE, int J>
__device__ __forceinline__ void load_keys(const Item& item, uint32_t ts, const Where<IN_PAGE> (&at)[J], Keys<F, D, J>& k) {
    using S = Shape<F, D>;
    if (any_seen(at) == 0u) return;
    const int lane = threadIdx.x & 63, row = lane & 15, quarter = lane >> 4;
    constexpr int kPiece = F == KVTC_CACHE_INT4 ? 4 * S::KW : 16, kPieces = 4 * S::KW / kPiece, kStep = F == KVTC_CACHE_INT4 ? 0 : 64;
    const uint32_t mine = quarter * kPiece;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            Bytes p;
            if constexpr (IN_PAGE) p = lane_at(item.k, at[j].row[n], (uint32_t)row * ts + mine);
            else p = item.k + shfl64(at[j].row[0], 16 * n + row) + mine;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) load<kPiece>(p + i * kStep, &k.w[j][n][i * kPiece / 4]);
        }
    load_scales<F, D, IN_PAGE, J>(item.k_scales, at, lane, k.scale);
}

template <int F, int D, bool IN_PAGE, int J>
__device__ __forceinline__ void load_values(const Item& item, uint32_t ts, const Where<IN_PAGE> (&at)[J], Values<F, D, J>& v) {
    using S = Shape<F, D>;
    if (any_seen(at) == 0u) return;
    const int lane = threadIdx.x & 63, mine = (lane & 15) * S::VB, quarter = lane >> 4;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            Bytes p;
            if constexpr (IN_PAGE) p = lane_at(item.v, at[j].row[k / 4], (uint32_t)(4 * quarter + k % 4) * ts + mine);
            else p = item.v + shfl64(at[j].row[0], token_of(k, quarter)) + mine;
            load<S::VB>(p, v.w[j][k]);
        }
    load_scales<F, D, IN_PAGE, J>(item.v_scales, at, lane, v.scale);
}

// ---- queries and scores --------------------------------------------------------------------------------------------------------

// Operands of a query, and of a probability.
template <typename XT> constexpr int query_parts() { return sizeof(XT) == 2 ? 1 : 3; }
template <typename XT, int F> constexpr int probability_parts() { return sizeof(XT) == 2 && F == KVTC_CACHE_INT4 ? 2 : 3; }

template <typename XT, int F, int D>
struct Query {
    static constexpr int NK = D / 32;
    bf16x8 w[NK][query_parts<XT>()];
    float factor;                                          // of a score
    float sum[F == KVTC_CACHE_INT4 ? NK : 1];              // 4 bits: of the query over a group
};

// Of one query head (or none: zeros) the features that go with the lane's part of the keys: on their way, and as operands.
template <typename XT, int D>
struct RawQuery { uint32_t w[D / 32][8 * sizeof(XT) / 4]; };
template <typename XT, int F, int D>
__device__ __forceinline__ void load_query(const XT* q, RawQuery<XT, D>& out) {
    const int quarter = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int s = 0; s < D / 32; ++s) {
        // (8 bits: 16 bytes of keys are two products' worth)
        const int first = F == KVTC_CACHE_FP8 ? s / 2 * 64 + quarter * 16 + s % 2 * 8 : s * 32 + quarter * 8;
        load<8 * sizeof(XT)>(bytes_at(q + first), out.w[s]);
    }
}
// 4 bits: a code as it stands is the bf16 pattern of code * 2^-133, a number below the normal ones, which the matrix unit takes for what it is; so is the whole byte of two codes, of low + 16 high.
// The query is multiplied by 2^up, its largest magnitude to 2^120, so that sums of a group stay finite, and odd features by 1 / 16.  The factor of a score makes that good, and has to stay finite itself:
// 2^up is no less than it needs, which is too much only for queries whose product with the factor passes 2^114.
constexpr int kCodeUnit = -133;
// Low codes as operands of the values' products: where they stand, or, for fp32 outputs, 16 of them.  (The matrix unit aligns products by their exponents as they are written, and cuts below; a number that begins
// lower down in its pattern has fewer bits.  16 rows of 32768 tokens, fp32: 2.0e-6 off, relative, and 1.2e-6, 208 us and 212; of bf16 outputs that is far below the rounding.)
template <typename XT> constexpr float low_code_up() { return sizeof(XT) == 2 ? 1.0f : 16.0f; }
constexpr float kUp = 0x1p60f;                             // of probabilities times scales
template <typename XT, int F, int D>
__device__ __forceinline__ void to_operands(const RawQuery<XT, D>& raw, bool is, float factor, Query<XT, F, D>& out) {
    constexpr int NK = D / 32;
    out.factor = factor;
    if constexpr (F != KVTC_CACHE_INT4 && sizeof(XT) == 2) {
#pragma unroll
        for (int s = 0; s < NK; ++s) out.w[s][0] = operand(is ? raw.w[s][0] : 0u, is ? raw.w[s][1] : 0u, is ? raw.w[s][2] : 0u, is ? raw.w[s][3] : 0u);
    } else {
        float v[NK][8];
#pragma unroll
        for (int s = 0; s < NK; ++s)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t w;
                if constexpr (sizeof(XT) == 2) w = i % 2 ? raw.w[s][i / 2] & 0xffff0000u : raw.w[s][i / 2] << 16;
                else w = raw.w[s][i];
                v[s][i] = __uint_as_float(is ? w : 0u);
            }
        if constexpr (F == KVTC_CACHE_INT4) {
            float top = 0.0f;
#pragma unroll
            for (int s = 0; s < NK; ++s)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, __builtin_fabsf(v[s][i]));
            top = max_over_quarters(top);
            auto exponent = [](float x) { return (int)(__float_as_uint(x) >> 23 & 255u) - 127; };
            const int up = max(exponent(factor) + 6, 119 - exponent(top));
            out.factor = __builtin_amdgcn_ldexpf(factor, -kCodeUnit - up);
#pragma unroll
            for (int s = 0; s < NK; ++s) {
                float o[8];                                // the order in which codes come out of their bytes
#pragma unroll
                for (int i = 0; i < 8; ++i) v[s][i] = __builtin_amdgcn_ldexpf(v[s][i], up);
                const float sum = ((v[s][0] + v[s][1]) + (v[s][2] + v[s][3])) + ((v[s][4] + v[s][5]) + (v[s][6] + v[s][7]));
                out.sum[s] = __builtin_amdgcn_ldexpf(sum_over_quarters(sum), kCodeUnit);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = v[s][(i & 4) + (i & 1) * 2 + (i >> 1 & 1)] * (i & 2 ? 0.0625f : 1.0f);
                split<query_parts<XT>(), Signs::kAny>(o, out.w[s]);
            }
        } else {
#pragma unroll
            for (int s = 0; s < NK; ++s) split<query_parts<XT>(), F == KVTC_CACHE_BF16 ? Signs::kOne : Signs::kAny>(v[s], out.w[s]);
        }
    }
}

// byte `at` of one and of another run of dwords, each in 16 bits
__device__ __forceinline__ uint32_t bytes_of(uint32_t first, uint32_t second, int at_first, int at_second) {
    return __builtin_amdgcn_perm(second, first, (uint32_t)at_first | 0x0c00u | (uint32_t)(at_second + 4) << 16 | 0x0c000000u);
}
// two E4M3 codes (the low or the high ones of a dword) as bf16
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_to_bf16(uint32_t w) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH)); }

// Scores (without the query's factor) of the lane's query head and 8 tokens of its set's piece.
template <typename XT, int F, int D, int J>
__device__ __forceinline__ void scores(const Query<XT, F, D>& q, const Keys<F, D, J>& k, float (&s)[8]) {
    constexpr int NK = D / 32, QP = query_parts<XT>();
    const int set = set_of<J>(threadIdx.x & 15);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (F == KVTC_CACHE_INT4) {
#pragma unroll
            for (int g = 0; g < NK; ++g) {
                f32x4 codes;
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    auto at = [&](int pair) { return pair * NK + g; };                    // byte of the lane's run
                    auto pairs = [&](int a, int b) { return bytes_of(k.w[j][n][at(a) / 4], k.w[j][n][at(b) / 4], at(a) % 4, at(b) % 4); };
                    f32x4 now = {0.0f, 0.0f, 0.0f, 0.0f};
                    const uint32_t u = pairs(0, 1), v = pairs(2, 3);
                    const bf16x8 w = operand(u & 0x000f000fu, u & 0x00f000f0u, v & 0x000f000fu, v & 0x00f000f0u);
#pragma unroll
                    for (int i = QP - 1; i >= 0; --i) now = mfma(w, q.w[g][i], now);
#pragma unroll
                    for (int i = 0; i < 4; ++i) codes[i] = j == 0 || set == j ? now[i] : codes[i];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t header = k.scale[4 * n + i][g];
                    sum[i] = __builtin_fmaf(half_of(header, 1), codes[i], __builtin_fmaf(half_of(header, 0), q.sum[g], sum[i]));
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < NK; ++t) {
                const uint32_t* w = k.w[0][n];
                bf16x8 a;
                if constexpr (F == KVTC_CACHE_BF16) a = operand(w[4 * t], w[4 * t + 1], w[4 * t + 2], w[4 * t + 3]);
                else a = operand(e4m3_to_bf16<false>(w[2 * t]), e4m3_to_bf16<true>(w[2 * t]), e4m3_to_bf16<false>(w[2 * t + 1]), e4m3_to_bf16<true>(w[2 * t + 1]));
#pragma unroll
                for (int i = QP - 1; i >= 0; --i) sum = mfma(a, q.w[t][i], sum);
            }
            if constexpr (F == KVTC_CACHE_FP8) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] *= __uint_as_float(k.scale[4 * n + i][0]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * n + i] = sum[i];
    }
}

// ---- running sums --------------------------------------------------------------------------------------------------------------

// Of the lane's query head: the maximum (of all lanes of the head), and this lane's parts of the sums.
template <typename XT, int F, int D>
struct Running {
    static constexpr int NO = D / 16, G = D / 32;
    f32x4 o[NO];
    float m, l;
    float low[F == KVTC_CACHE_INT4 ? G : 1];               // 4 bits: of p * shift, per group
};

// the feature of o[i][r]
template <int F, int D>
__device__ __forceinline__ int feature_of(int i, int r, int quarter) {
    const int c = 4 * quarter + r;
    return F == KVTC_CACHE_INT4 ? i / 2 * 32 + 2 * c + i % 2 : c * (D / 16) + i;
}

// What a step's products begin with.  They are added to the running sums by the vector unit, which rounds to nearest: the matrix unit cuts, product by product, what lies below the last bit of the largest it adds, so
// that sums over many steps that grow in there come out too small.  (Relative, fp32, 16 rows of 32768 tokens: 4 bits 2.4e-5 so, 1.9e-6 with sums of its own for every step; positive values in bf16 and 8 bits 1.1e-6
// and 0.7e-7.  64 ragged rows in bf16 207.4 us both, 16 of 32768 tokens in 8 bits 210.5 and 209.5, in 4 bits 153.6 and 154.3, fp32 201 and 208.)
constexpr f32x4 kNothing = {0.0f, 0.0f, 0.0f, 0.0f};
template <typename XT, int F, int D, bool IN_PAGE, int J>
__device__ __forceinline__ void add_tokens(Running<XT, F, D>& run, Values<F, D, J>& v, float (&s)[8], const Where<IN_PAGE> (&at)[J], float factor, const Constants& known) {
    constexpr int NO = D / 16, G = D / 32, P = probability_parts<XT, F>();
    const int quarter = (threadIdx.x & 63) >> 4, set = set_of<J>(threadIdx.x & 15);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] *= factor;
    uint32_t all = 0xffffffffu;
#pragma unroll
    for (int j = 0; j < J; ++j) all &= at[j].seen;
    if (all != 0xffffffffu) {                              // what is not seen counts for nothing, whatever it holds
        uint32_t mine = at[0].seen;
#pragma unroll
        for (int j = 1; j < J; ++j) mine = set == j ? at[j].seen : mine;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bool is = mine >> token_of(k, quarter) & 1u;
            s[k] = is ? s[k] : kNoScore;
#pragma unroll
            for (int i = 0; i < Shape<F, D>::SW; ++i) v.scale[k][i] = is ? v.scale[k][i] : 0u;
            if constexpr (F != KVTC_CACHE_INT4) {          // (4 bits are finite whatever they are)
#pragma unroll
                for (int i = 0; i < Shape<F, D>::VW; ++i) v.w[0][k][i] = is ? v.w[0][k][i] : 0u;
            }
        }
    }
    float top = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    top = max_over_quarters(top);
    if (__any(top > run.m)) {
        const float now = fmaxf(top, run.m), keep = exp2_fast(run.m - (now == kNoScore ? 0.0f : now));
        run.l *= keep;
        run.m = now;
#pragma unroll
        for (int i = 0; i < NO; ++i) run.o[i] *= keep;
        if constexpr (F == KVTC_CACHE_INT4) {
#pragma unroll
            for (int g = 0; g < G; ++g) run.low[g] *= keep;
        }
    }
    const float base = run.m == kNoScore ? 0.0f : run.m;
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = exp2_fast(s[i] - base);
    run.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    if constexpr (F == KVTC_CACHE_INT4) {
        float up[8];                                       // (codes are small numbers)
#pragma unroll
        for (int i = 0; i < 8; ++i) up[i] = p[i] * kUp;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            __builtin_amdgcn_sched_barrier(0);             // (one group after the other: all at once, the unpacked codes do not fit the registers, 330 us for 153)
            float ps[8], shifts = known.zero;                // (of the step: one rounding less for the running sums in eight.  fp32, as above, 1.2e-6 off, and 0.8e-6)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t header = v.scale[i][g];
                ps[i] = __builtin_fmaf(half_of(header, 1), up[i], known.zero);
                shifts = __builtin_fmaf(half_of(header, 0), p[i], shifts);
            }
            run.low[g] += shifts;
            bf16x8 b[P];
            split<P, Signs::kAny>(ps, b);
            constexpr float kLowUp = low_code_up<XT>();
            f32x4 low_now = kNothing, both_now = kNothing;
#pragma unroll
            for (int j = 0; j < J; ++j) {
                uint32_t low[4], both[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    both[i] = bytes_of(v.w[j][2 * i][g / 4], v.w[j][2 * i + 1][g / 4], g % 4, g % 4);
                    low[i] = kLowUp == 16.0f ? both[i] << 4 & 0x00f000f0u : both[i] & 0x000f000fu;
                }
#pragma unroll
                for (int i = P - 1; i >= 0; --i) {
                    u32x4 own = __builtin_bit_cast(u32x4, b[i]);               // (a set's probabilities go with its own piece's values only)
                    if constexpr (J > 1) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) own[k] = set == j ? own[k] : 0u;
                    }
                    low_now = mfma(operand(low[0], low[1], low[2], low[3]), __builtin_bit_cast(bf16x8, own), low_now);
                    both_now = mfma(operand(both[0], both[1], both[2], both[3]), __builtin_bit_cast(bf16x8, own), both_now);
                }
            }
            run.o[2 * g] += low_now;
            run.o[2 * g + 1] += both_now;
        }
    } else {
        if constexpr (F == KVTC_CACHE_FP8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] *= __uint_as_float(v.scale[i][0]);
        }
        bf16x8 b[P];
        split<P, F == KVTC_CACHE_BF16 ? Signs::kPositive : Signs::kAny>(p, b);
        if constexpr (F == KVTC_CACHE_BF16) {
#pragma unroll
            for (int i = 0; i < NO; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = i % 2 ? high_halves(v.w[0][2 * k][i / 2], v.w[0][2 * k + 1][i / 2]) : low_halves(v.w[0][2 * k][i / 2], v.w[0][2 * k + 1][i / 2]);
                f32x4 now = kNothing;
#pragma unroll
                for (int k = P - 1; k >= 0; --k) now = mfma(operand(w[0], w[1], w[2], w[3]), b[k], now);
                run.o[i] += now;
            }
        } else {
#pragma unroll
            for (int i = 0; i < NO; i += 2) {
                uint32_t w[4], x[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {                                 // features i and i + 1 of two tokens: [i, i, i + 1, i + 1]
                    const uint32_t from = (uint32_t)(i % 4), u = __builtin_amdgcn_perm(v.w[0][2 * k + 1][i / 4], v.w[0][2 * k][i / 4], from | (from + 4) << 8 | (from + 1) << 16 | (from + 5) << 24);
                    w[k] = e4m3_to_bf16<false>(u);
                    x[k] = e4m3_to_bf16<true>(u);
                }
                f32x4 now = kNothing, next = kNothing;
#pragma unroll
                for (int k = P - 1; k >= 0; --k) {
                    now = mfma(operand(w[0], w[1], w[2], w[3]), b[k], now);
                    next = mfma(operand(x[0], x[1], x[2], x[3]), b[k], next);
                }
                run.o[i] += now;
                run.o[i + 1] += next;
            }
        }
    }
}

// The sums as they are: 4 bits, of single codes, with their unit and shifts.
template <typename XT, int F, int D>
__device__ __forceinline__ void settle(Running<XT, F, D>& run) {
    run.l = sum_over_quarters(run.l);
    if constexpr (F == KVTC_CACHE_INT4) {
        constexpr float kUnit = 0x1p73f;
        static_assert((double)kUnit * kUp == 0x1p133, "2^-kCodeUnit");
#pragma unroll
        for (int g = 0; g < D / 32; ++g) {
            const float shift = sum_over_quarters(run.low[g]);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float low = run.o[2 * g][r] * (1.0f / low_code_up<XT>()), high = (run.o[2 * g + 1][r] - low) * 0.0625f;
                run.o[2 * g][r] = __builtin_fmaf(low, kUnit, shift);
                run.o[2 * g + 1][r] = __builtin_fmaf(high, kUnit, shift);
            }
        }
    }
}

// ---- the shares ----------------------------------------------------------------------------------------------------------------

// The 32-token pieces of a sequence that hold a seen token -- those of the sinks, then those of the window -- and its tiles of PIECES of them.  (At least one: every
// row has a result.)
struct Tiles { uint32_t n, pieces, sinks, window0, length, from; };
template <int PIECES, typename PLAN>
__device__ __forceinline__ Tiles tiles_of(PLAN& p, int32_t length) {
    Tiles t;
    t.length = (uint32_t)length <= p.max_tokens ? (uint32_t)length : 0u;
    t.from = p.window && t.length > p.window ? t.length - p.window : 0u;
    const uint32_t all = (t.length + 31) / 32;
    t.sinks = p.window ? (min(p.sinks, t.length) + 31) / 32 : 0u;
    t.window0 = max(t.sinks, t.from / 32);
    t.pieces = t.sinks + (all > t.window0 ? all - t.window0 : 0u);
    t.n = max(1u, (t.pieces + PIECES - 1) / PIECES);
    return t;
}

template <typename XT> __device__ __forceinline__ void put_out(XT* x, float v);
template <> __device__ __forceinline__ void put_out<uint16_t>(uint16_t* x, float v) { *x = f32_bf16(v); }
template <> __device__ __forceinline__ void put_out<float>(float* x, float v) { *x = v; }

// floats of a part of an item in the workspace
__host__ __device__ constexpr int part_floats(int cols, int d) { return (cols * (d + 2) + 3) / 4 * 4; }

// Parts go from one workgroup to another whose L2 is another one.  They are stored and loaded at agent scope, past the L2: no cache needs to be written back or
// emptied for them, which, at the end of every workgroup, cost more than all else there.  A workgroup is counted as come when its stores have been acknowledged.
union Pair { uint64_t u; float f[2]; };
__device__ __forceinline__ void put_pair(float* p, float first, float second) {
    Pair v;
    v.f[0] = first;
    v.f[1] = second;
    __hip_atomic_store(reinterpret_cast<uint64_t*>(p), v.u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Pair get_pair(const float* p) {
    Pair v;
    v.u = __hip_atomic_load(reinterpret_cast<const uint64_t*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return v;
}

// The parts g0 .. g1 of an item, joined by a workgroup in their order: (m, l) of every row, then the outputs, two to a thread; where the rows have fewer than
// 512 outputs, several threads share the parts of one.  kAhead parts are on their way together, the first of them while the maxima are found (one after another
// 64 parts took 17 us).  weight: [16][kJoinStep]; sum: [512]; stats: [32].
constexpr int kJoinStep = 64, kAhead = 16;
// An item's rows and their places in the output: the `cols` query heads of a KV head, and those of the next one.
struct OutRows {
    int64_t row0;
    int n, cols, group;
    __device__ __forceinline__ int64_t at(int c) const { return row0 + (c >= cols ? c / cols * (group - cols) : 0) + c; }
};
template <typename XT, int D>
__device__ __forceinline__ void join_parts(ScalarPlan plan, int tid, const float* slots, int slot_floats, uint32_t g0, uint32_t g1, int rows_all, const OutRows& rows, float* weight, float* sum,
                                           float* stats) {
    const int cols = rows.n;
    const int lane = tid & 63, wave = tid >> 6;
    const int n = (int)(g1 - g0) + 1;
    auto part_at = [&](int k) { return slots + (int64_t)(2 * (g0 + k) + (k == 0 ? 1 : 0)) * slot_floats; };
    const int pairs = cols * D / 2, teams = pairs < 256 ? 256 / pairs : 1;
    for (int j0 = 0; j0 < pairs; j0 += 256) {
        const int team = teams > 1 ? tid / pairs : 0, j = min(teams > 1 ? tid - team * pairs : j0 + tid, pairs - 1), c = 2 * j / D;
        const bool is = team < teams && (teams > 1 || j0 + tid < pairs);
        // parts team, team + teams, ...; those past the last are the last again, and count for nothing
        auto get = [&](int k) { return get_pair(part_at(min(k, n - 1)) + 2 * rows_all + 2 * j); };
        float o0 = 0.0f, o1 = 0.0f;
        for (int from = 0; from < n; from += kJoinStep) {
            Pair v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                v[i].u = 0;
                if (from + i * teams < n) v[i] = get(from + team + i * teams);      // (the same in all threads)
            }
            if (from > 0 || j0 > 0) __syncthreads();       // (the weights before these have been used)
            if (j0 == 0 && from == 0) {
                for (int cc = wave; cc < cols; cc += 4) {  // maximum and sum of a row, and the weights of its first parts
                    float m = kNoScore, l = 0.0f, m0 = kNoScore;
                    for (int k = lane; k < n; k += 64) {
                        const Pair w = get_pair(part_at(k) + 2 * cc);
                        const float top = fmaxf(m, w.f[0]), base = top == kNoScore ? 0.0f : top;
                        l = l * exp2_fast(m - base) + w.f[1] * exp2_fast(w.f[0] - base);
                        m = top;
                        if (k < 64) m0 = w.f[0];
                    }
                    float top = m;
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
                    const float base = top == kNoScore ? 0.0f : top;
                    l *= exp2_fast(m - base);
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d, 64);
                    if (lane == 0) { stats[cc] = base; stats[16 + cc] = l; }
                    weight[cc * kJoinStep + lane] = exp2_fast(m0 - base);
                }
            } else if (n > kJoinStep) {
                for (int k = tid; k < cols * kJoinStep; k += 256) {
                    const int cc = k / kJoinStep, g = from + k % kJoinStep;
                    weight[k] = g < n ? exp2_fast(get_pair(part_at(g) + 2 * cc).f[0] - stats[cc]) : 0.0f;
                }
            }
            __syncthreads();
            const int here = min(kJoinStep, n - from);
            for (int k0 = team; k0 < here; k0 += kAhead * teams) {
                if (k0 != team) {
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) v[i] = get(from + k0 + i * teams);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int k = k0 + i * teams;
                    const bool one = k < here;
                    const float w = one ? weight[c * kJoinStep + k] : 0.0f;
                    o0 = __builtin_fmaf(one ? v[i].f[0] : 0.0f, w, o0);
                    o1 = __builtin_fmaf(one ? v[i].f[1] : 0.0f, w, o1);
                }
            }
        }
        if (teams > 1) {
            sum[2 * tid] = o0;
            sum[2 * tid + 1] = o1;
            __syncthreads();
            if (is && team == 0)
                for (int k = 1; k < teams; ++k) {
                    o0 += sum[2 * (k * pairs + j)];
                    o1 += sum[2 * (k * pairs + j) + 1];
                }
        }
        if (is && team == 0) {
            const int f = 2 * j - c * D;
            const float l = stats[16 + c];
            XT* out = static_cast<XT*>(plan.a.out) + rows.at(c) * D + f;
            put_out(out, l == 0.0f ? 0.0f : o0 / l);
            put_out(out + 1, l == 0.0f ? 0.0f : o1 / l);
            if (plan.a.lse && f == 0) plan.a.lse[rows.at(c)] = l == 0.0f ? kNoScore : (stats[c] + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
        }
    }
}

// A lane's results in runs of neighbouring features: put(first feature, values).
template <typename XT, int F, int D, typename PUT>
__device__ __forceinline__ void in_runs(const Running<XT, F, D>& run, int quarter, PUT put) {
    if constexpr (F == KVTC_CACHE_INT4) {
#pragma unroll
        for (int g = 0; g < D / 32; ++g) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = run.o[2 * g + i % 2][i / 2];
            put(g * 32 + 8 * quarter, v);
        }
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float v[D / 16];
#pragma unroll
            for (int i = 0; i < D / 16; ++i) v[i] = run.o[i][r];
            put((4 * quarter + r) * (D / 16), v);
        }
    }
}
template <int N>
__device__ __forceinline__ void put_run(uint16_t* x, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<u32x2*>(x + i) = u32x2{round_pair(v[i], v[i + 1]), round_pair(v[i + 2], v[i + 3])};
}
template <int N>
__device__ __forceinline__ void put_run(float* x, const float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4*>(x + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
}

// The query heads of an item: of KV head `next` of the NEXT neighbouring ones that it is made of.
struct Heads { int h, col0, cols; };
template <int NEXT>
__device__ __forceinline__ Heads heads_of_item(ScalarPlan p, uint32_t item, int next) {
    const uint32_t of = p.parts == 1 ? item : (uint32_t)quotient(item, (uint32_t)p.parts);
    const int h = (int)of * NEXT + next, part = (int)(item - of * (uint32_t)p.parts);
    return {h, h * p.group + part * p.cols, min(p.cols, p.group - part * p.cols)};
}

// What wave `wave` of WAVES has to do with the tiles tile0 .. tile1 of an item, J pieces to a step.
template <typename XT, int F, int D, bool IN_PAGE, int WAVES, int J>
__device__ __forceinline__ void attend_tiles(const AttendPlan& p, int b, const Heads& part, const Tiles& t, uint32_t tile0, uint32_t tile1, uint32_t wave, const Constants& known, Running<XT, F, D>& run) {
    static_assert(J == 1 || F == KVTC_CACHE_INT4, "sets are made for 4 bits");
    ScalarPlan again = plan_again();
    const int col = threadIdx.x & 15;
    const float factor = again.a.scale * 1.44269504088896340736f;
    constexpr int kSet = kAttendCols / J;
    const int mine = col % kSet;                       // the head of the lane's column
    RawQuery<XT, D> raw;
    load_query<XT, F, D>(static_cast<const XT*>(again.a.q) + (int64_t)b * again.a.q_seq_stride + (int64_t)(part.col0 + (mine < part.cols ? mine : 0)) * again.a.q_head_stride, raw);
    const int64_t scale_head = (int64_t)part.h * again.a.c.page_tokens * (4 * Shape<F, D>::SW);
    const int64_t row_head = (int64_t)part.h * again.a.c.head_stride;
    const Item of{again.a.pages + (int64_t)b * again.a.pages_stride, bytes_at(again.a.c.k_dev) + row_head, bytes_at(again.a.c.v_dev) + row_head, bytes_at(again.a.c.k_scales_dev) + scale_head, bytes_at(again.a.c.v_scales_dev) + scale_head,
                  t.length, t.from, again.window ? again.sinks : 0u, (uint32_t)b};
    const uint32_t ts = (uint32_t)p.a.c.token_stride;
    auto look = [&](uint32_t i, Look<IN_PAGE> (&l)[J]) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const uint32_t k = (WAVES * i + wave) * J + j, piece = k < t.sinks ? k : t.window0 + (k - t.sinks);
            l[j] = look_at<IN_PAGE>(p, of, i < tile1 && k < t.pieces ? piece * 32 : t.length);
        }
    };
    auto places = [&](const Look<IN_PAGE> (&l)[J], Where<IN_PAGE> (&w)[J]) {
#pragma unroll
        for (int j = 0; j < J; ++j) w[j] = where<Shape<F, D>::SW, IN_PAGE>(p, of, l[j]);
    };
#pragma unroll
    for (int i = 0; i < D / 16; ++i) run.o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    run.m = kNoScore;
    run.l = 0.0f;
#pragma unroll
    for (int g = 0; g < (F == KVTC_CACHE_INT4 ? D / 32 : 1); ++g) run.low[g] = 0.0f;

    Keys<F, D, J> keys;
    Values<F, D, J> values;
    Look<IN_PAGE> ahead[J];
    Where<IN_PAGE> now[J], next[J];
    look(tile0, ahead);
    places(ahead, now);
    look(tile0 + 1, ahead);
    load_keys<F, D, IN_PAGE, J>(of, ts, now, keys);
    load_values<F, D, IN_PAGE, J>(of, ts, now, values);
    Query<XT, F, D> q;
    to_operands<XT, F, D>(raw, mine < part.cols, factor, q);       // (the keys are on their way meanwhile)
    for (uint32_t i = tile0; i < tile1; ++i) {
        places(ahead, next);
        look(i + 2, ahead);
        float s[8];
        const bool some = any_seen(now) != 0u;
        if (some) scores<XT, F, D, J>(q, keys, s);
        load_keys<F, D, IN_PAGE, J>(of, ts, next, keys);
        if (some) add_tokens<XT, F, D, IN_PAGE, J>(run, values, s, now, q.factor, known);
        load_values<F, D, IN_PAGE, J>(of, ts, next, values);
#pragma unroll
        for (int j = 0; j < J; ++j) now[j] = next[j];
    }

    settle<XT, F, D>(run);
}

// Workgroups go to the eight XCDs in turn.  Each XCD takes neighbouring shares of n, the heads of a sequence one after another, so that where several heads' rows or scales are in one cache line its
// L2 has it for all of them (24 rows of 12 heads of 64 features, 8 bits, token-major, 15.6 us, with the shares in turn 16.9; 64 ragged rows in bf16 206.6 and 208.7).  Of few long items the shares that read
// the same tokens lie far apart; where an item's shares are a multiple of eight, they go in turn, which has them meet in an L2.
__device__ __forceinline__ uint32_t neighbours_to_an_xcd(uint32_t block, uint32_t n) { return (block & 7u) * (n / 8) + min(block & 7u, n % 8) + block / 8; }

// Long rows: shares of equal numbers of tiles, four waves to each.
template <typename XT, int F, int D, bool IN_PAGE, int J, int NEXT>
__global__ void __launch_bounds__(256, groups_each(F, D, sizeof(XT) == 2)) attend_kernel(const AttendPlan p) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int kSet = kAttendCols / J;
    __shared__ float s_o[4][kAttendCols][D + 4], s_m[4][kAttendCols], s_l[4][kAttendCols];
    __shared__ uint32_t s_last;
    // what is not needed among the tokens: tiles of all items; the sequence's first tile, the share's next and end, counted over all items; ...
    __shared__ struct { uint64_t all, seq0, at, end; uint32_t me, groups; } s_share;

    uint32_t b, item, tile0, tile1;
    Tiles t;
    {
        // where the workgroup's share begins: a prefix sum over the sequences' tiles, in every wave
        const AttendArgs& a = p.a;
        const int tid = threadIdx.x, lane = tid & 63;
        const uint32_t heads = (uint32_t)a.c.n_heads / NEXT * (uint32_t)p.parts;
        uint32_t mine = 0;
        const int first = lane * p.seqs_each, last = min(first + p.seqs_each, a.n_seqs);
        for (int b = first; b < last; ++b) {
            const int32_t length = a.lengths[b];
            if (blockIdx.x == 0 && (uint32_t)length > p.max_tokens) report_lowest(a.status, (uint32_t)b);
            mine += tiles_of<4 / NEXT * J>(p, length).n;
        }
        const uint32_t upto = wave_inclusive_scan(mine);
        const uint64_t all = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)upto, 63) * heads;
        // no share is empty: each of an item's workgroups is waited for
        const uint32_t most = groups_each(F, D, sizeof(XT) == 2) > 2 && all < 2 * (uint64_t)gridDim.x ? min(p.few, gridDim.x) : gridDim.x, groups = all < most ? (uint32_t)all : most;
        if (blockIdx.x >= groups) return;
        const uint32_t me = p.in_turn ? blockIdx.x : neighbours_to_an_xcd(blockIdx.x, groups);
        // me * all / groups, by the quotient and the remainder of all / groups
        uint64_t share0 = me, share1 = me + 1;
        if (all != groups) {
            const uint64_t each = quotient(all, groups);
            const uint32_t odd = (uint32_t)(all - each * groups);
            share0 = me * each + quotient(me * odd, groups);
            share1 = (me + 1) * each + quotient((me + 1) * odd, groups);
        }
        // the lane whose sequences it falls among, and the sequence
        const int holder = __popcll(__ballot((uint64_t)upto * heads <= share0));
        b = (uint32_t)__builtin_amdgcn_readfirstlane(holder * p.seqs_each);
        uint64_t seq0 = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(upto - mine), holder) * heads;
        t = tiles_of<4 / NEXT * J>(p, scalar_at(a.lengths, b));
        while (share0 >= seq0 + (uint64_t)t.n * heads) {
            seq0 += (uint64_t)t.n * heads;
            t = tiles_of<4 / NEXT * J>(p, scalar_at(a.lengths, ++b));
        }
        item = (uint32_t)quotient(share0 - seq0, t.n);
        tile0 = (uint32_t)(share0 - seq0 - (uint64_t)item * t.n);
        tile1 = (uint32_t)min((uint64_t)t.n, tile0 + (share1 - share0));
        if (tid == 0) {
            s_share.all = all;
            s_share.seq0 = seq0;
            s_share.at = share0;
            s_share.end = share1;
            s_share.me = me;
            s_share.groups = groups;
        }
    }
    const Constants known = constants();

    for (;;) {
        // (the compiler does not see that these are)
        b = same(b), item = same(item), tile0 = same(tile0), tile1 = same(tile1);
        t = {same(t.n), same(t.pieces), same(t.sinks), same(t.window0), same(t.length), same(t.from)};
        Running<XT, F, D> run;
        const Heads part = heads_of_item<NEXT>(plan_again(), item, 0);
        attend_tiles<XT, F, D, IN_PAGE, 4 / NEXT, J>(p, (int)b, {part.h + wave % NEXT, part.col0 + wave % NEXT * p.group, part.cols}, t, tile0, tile1, wave / NEXT, known, run);

        // (from here on the thread's number is said to be another one, lest what follows from it be worked out before the loop over the tokens and kept through it)
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        const int lane = tid & 63, col = lane & 15, quarter = lane >> 4;
        ScalarPlan plan = plan_again();
        const uint32_t tiles = t.n;
        const int cols = part.cols, rows_all = NEXT * plan.cols;
        const OutRows rows{(int64_t)b * plan.a.n_q_heads + part.col0, NEXT * cols, cols, plan.group};
        const bool whole = tile0 == 0 && tile1 == tiles;
        // the waves' and the sets' results, joined
        if (col % kSet < cols) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) s_o[wave][col][feature_of<F, D>(i, r, quarter)] = run.o[i][r];
            if (quarter == 0) { s_m[wave][col] = run.m; s_l[wave][col] = run.l; }
        }
        __syncthreads();
        const uint32_t me = same(s_share.me);
        float* slots = reinterpret_cast<float*>(static_cast<uint8_t*>(plan.a.work) + kAttendMaxShares * 4);
        const int slot_floats = part_floats(rows_all, D);
        float* slot = slots + (int64_t)(2 * me + (tile0 == 0 ? 1 : 0)) * slot_floats;
        for (int j = tid; j < rows.n * D / 2; j += 256) {
            const int c = 2 * j / D, f = 2 * j % D;
            const int next = NEXT > 1 ? c / cols : 0, head = c - next * cols;
            auto wave_of = [&](int i) { return i / J * NEXT + next; };        // the waves of this KV head, and their sets
            auto col_of = [&](int i) { return i % J * kSet + head; };
            constexpr int kOf = 4 / NEXT * J;
            float top = s_m[next][head];
#pragma unroll
            for (int i = 1; i < kOf; ++i) top = fmaxf(top, s_m[wave_of(i)][col_of(i)]);
            const float base = top == kNoScore ? 0.0f : top;
            float l = 0.0f, o0 = 0.0f, o1 = 0.0f;
#pragma unroll
            for (int i = 0; i < kOf; ++i) {
                const int w = wave_of(i), from = col_of(i);
                const float keep = exp2_fast(s_m[w][from] - base);
                l = __builtin_fmaf(s_l[w][from], keep, l);
                o0 = __builtin_fmaf(s_o[w][from][f], keep, o0);
                o1 = __builtin_fmaf(s_o[w][from][f + 1], keep, o1);
            }
            if (whole) {
                XT* out = static_cast<XT*>(plan.a.out) + rows.at(c) * D + f;
                put_out(out, l == 0.0f ? 0.0f : o0 / l);
                put_out(out + 1, l == 0.0f ? 0.0f : o1 / l);
                if (plan.a.lse && f == 0) plan.a.lse[rows.at(c)] = l == 0.0f ? kNoScore : (base + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
            } else {
                put_pair(slot + 2 * rows_all + c * D + f, o0, o1);
                if (f == 0) put_pair(slot + 2 * c, top, l);
            }
        }
        if (!whole) {
            // the workgroups that the item's first and last tile fall to; the last of them to come here joins the parts
            const uint64_t item0 = same64(s_share.seq0) + (uint64_t)item * tiles, all = same64(s_share.all);
            const uint32_t groups = same(s_share.groups);
            const uint32_t g0 = tile0 == 0 ? me : (uint32_t)quotient((item0 + 1) * groups - 1, all);
            const uint32_t g1 = tile1 == tiles ? me : (uint32_t)quotient((item0 + tiles) * groups - 1, all);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            uint32_t* counter = static_cast<uint32_t*>(plan.a.work) + g0;
            if (tid == 0) {
                const uint32_t came = __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                s_last = came == g1 - g0;
                if (came == g1 - g0) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            __syncthreads();
            if (s_last) join_parts<XT, D>(plan, tid, slots, slot_floats, g0, g1, rows_all, rows, &s_o[0][0][0], &s_o[1][0][0], &s_m[0][0]);
        }
        const uint64_t at = same64(s_share.at) + (tile1 - tile0), end = same64(s_share.end);
        if (at >= end) return;
        const uint32_t heads = (uint32_t)plan.a.c.n_heads / NEXT * (uint32_t)plan.parts;
        tile0 = 0;
        __syncthreads();
        if (tid == 0) {
            s_share.at = at;
            if (item + 1 == heads) s_share.seq0 += (uint64_t)tiles * heads;
        }
        if (++item == heads) {                             // the sequence's last item: the next one's first
            item = 0;
            t = tiles_of<4 / NEXT * J>(plan, scalar_at(plan.a.lengths, ++b));
        }
        tile1 = (uint32_t)min((uint64_t)t.n, end - at);
    }
}

// Many short rows: a wave, which is a workgroup, to an item, and nothing to be joined.
template <typename XT, int F, int D, bool IN_PAGE>
__global__ void __launch_bounds__(64, D == 256 ? 1 : 2) attend_rows_kernel(const AttendPlan p) {
    const AttendArgs& a = p.a;
    const int lane = threadIdx.x, col = lane & 15, quarter = lane >> 4;
    const uint32_t heads = (uint32_t)a.c.n_heads * (uint32_t)p.parts, me = neighbours_to_an_xcd(blockIdx.x, gridDim.x);
    const int b = (int)quotient(me, heads);
    const uint32_t item = me - (uint32_t)b * heads;
    const int32_t length = scalar_at(a.lengths, b);
    if (item == 0 && lane == 0 && (uint32_t)length > p.max_tokens) report_lowest(a.status, (uint32_t)b);
    const Tiles t = tiles_of<1>(p, length);
    const Heads part = heads_of_item<1>(plan_again(), item, 0);
    const Constants known = constants();
    Running<XT, F, D> run;
    attend_tiles<XT, F, D, IN_PAGE, 1, 1>(p, b, part, t, 0, t.n, 0, known, run);
    if (col < part.cols) {
        const int64_t row = (int64_t)b * a.n_q_heads + part.col0 + col;
        const float l = run.l;
        XT* out = static_cast<XT*>(a.out) + row * D;
        in_runs<XT, F, D>(run, quarter, [&](int f, auto& v) {
#pragma unroll
            for (float& x : v) x = l == 0.0f ? 0.0f : x / l;
            put_run(out + f, v);
        });
        if (a.lse && quarter == 0) a.lse[row] = l == 0.0f ? kNoScore : (run.m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------------------

// What runs: a wave to every item (rows), or shares of tiles; pieces to a wave's step; KV heads of an item; workgroups.
struct Shares { bool rows, in_turn; int pieces, next, n; };
// KV heads whose rows of a token can lie in one cache line of 128 bytes.
constexpr int heads_to_a_line(int format, int d, bool in_page) { return !in_page ? 1 : 128 / cache_row_bytes(format, d) < 1 ? 1 : 128 / cache_row_bytes(format, d); }
// Whether there is a kernel of two pieces to a wave's step: of 4 bits, which is bound by the vector unit (64 rows of 4096 tokens, us, one piece and two: 90.6 and 77.5; in 8 bits
// 102 and 105; four pieces do not fit the registers: 243).
constexpr bool two_pieces(int format, bool bf16, int d, bool in_page) { return format == KVTC_CACHE_INT4 && bf16 && d <= 128 && in_page; }

template <typename XT, int F, int D, bool IN_PAGE, int J, int NEXT>
static void launch_kernel(const AttendPlan& p, const Shares& s, hipStream_t stream) {
    hipLaunchKernelGGL((attend_kernel<XT, F, D, IN_PAGE, J, NEXT>), dim3(s.n), dim3(256), 0, stream, p);
}
template <typename XT, int F, int D, bool IN_PAGE, int J>
static void launch_shares(const AttendPlan& p, const Shares& s, hipStream_t stream) {
    constexpr int most = J == 1 && two_pieces(F, sizeof(XT) == 2, D, IN_PAGE) ? 1 : heads_to_a_line(F, D, IN_PAGE);
    if constexpr (most >= 4) { if (s.next == 4) return launch_kernel<XT, F, D, IN_PAGE, J, 4>(p, s, stream); }
    if constexpr (most >= 2) { if (s.next == 2) return launch_kernel<XT, F, D, IN_PAGE, J, 2>(p, s, stream); }
    launch_kernel<XT, F, D, IN_PAGE, J, 1>(p, s, stream);
}
template <typename XT, int F, int D, bool IN_PAGE>
static void launch_pieces(const AttendPlan& p, const Shares& s, hipStream_t stream) {
    if (s.rows) { hipLaunchKernelGGL((attend_rows_kernel<XT, F, D, IN_PAGE>), dim3(s.n), dim3(64), 0, stream, p); return; }
    if constexpr (two_pieces(F, sizeof(XT) == 2, D, IN_PAGE)) { if (s.pieces == 2) return launch_shares<XT, F, D, IN_PAGE, 2>(p, s, stream); }
    launch_shares<XT, F, D, IN_PAGE, 1>(p, s, stream);
}
template <typename XT, int F, int D>
static void launch_pages(const AttendPlan& p, const Shares& s, hipStream_t stream) {
    if (p.in_page) launch_pieces<XT, F, D, true>(p, s, stream);
    else launch_pieces<XT, F, D, false>(p, s, stream);
}
template <typename XT, int F>
static void launch_width(const AttendPlan& p, const Shares& s, hipStream_t stream) {
    if (p.a.c.d_head == 64) launch_pages<XT, F, 64>(p, s, stream);
    else if (p.a.c.d_head == 128) launch_pages<XT, F, 128>(p, s, stream);
    else launch_pages<XT, F, 256>(p, s, stream);
}
// The kernels of one type and format (the file is compiled once for each, side by side), and with the first of them the host's part.
#if KVTC_ATTEND_PART < 3
typedef uint16_t PartType;
#else
typedef float PartType;
#endif
#define KVTC_ATTEND_NAME_(k) launch_attend_##k
#define KVTC_ATTEND_NAME(k) KVTC_ATTEND_NAME_(k)
void KVTC_ATTEND_NAME(KVTC_ATTEND_PART)(const AttendPlan& p, const Shares& s, hipStream_t stream) { launch_width<PartType, KVTC_ATTEND_PART % 3>(p, s, stream); }

#if KVTC_ATTEND_PART == 0
void launch_attend_1(const AttendPlan&, const Shares&, hipStream_t);
void launch_attend_2(const AttendPlan&, const Shares&, hipStream_t);
void launch_attend_3(const AttendPlan&, const Shares&, hipStream_t);
void launch_attend_4(const AttendPlan&, const Shares&, hipStream_t);
void launch_attend_5(const AttendPlan&, const Shares&, hipStream_t);

// Items that share a KV head's query heads, and how many of these each has.
static void heads_of(const kvtc_cache& c, int n_q_heads, int& parts, int& cols) {
    const int group = n_q_heads / c.n_heads;
    parts = (group + kAttendCols - 1) / kAttendCols;
    cols = (group + parts - 1) / parts;
}

// Shares: as many as run at once, no more than there can be tiles.
static Shares shares_at_once(const kvtc_cache& c, bool bf16, int n_seqs, int parts, int cols, int64_t max_tokens, int64_t sinks, int64_t window) {
    int64_t pieces = (max_tokens + 31) / 32;
    if (window) {
        const int64_t some = (sinks < max_tokens ? sinks : max_tokens) / 32 + (window < max_tokens ? window : max_tokens) / 32 + 3;
        pieces = some < pieces ? some : pieces;
    }
    const int64_t places = (int64_t)compute_units() * groups_each(c.format, c.d_head, bf16), rows = (int64_t)n_seqs * c.n_heads * parts;
    Shares s;
    s.rows = pieces <= short_pieces(c.format) && rows >= (int64_t)compute_units() * (c.d_head == 256 ? 4 : 8) && rows < (1 << 25);
    // Several KV heads to an item, the waves of a workgroup among them, where their rows of a token share a cache line, which they each fetch if apart; for caches that may be larger than the
    // Infinity Cache, which has the line for the second as well, and of many items: fewer items are of more parts, and larger ones, to join.  (Token-major, 16 rows of 32768 tokens, us, apart and
    // so: 4 bits, 8 heads of 128 175 and 167, 16 of 64 298 and 213; 8 bits, 16 of 64 292 and 252; 4 bits with fp32 queries, 8 of 128 199 and 199, 16 of 64 302 and 220.  32 rows of
    // 2000, 4 bits, 8 of 128, 30 and 33; one of 32768 28 and 46.)
    s.next = 1;
    // (The sequences' tiles are added up in 32 bits.  Tiles of four pieces, of which there are at most 2^31 by the checks of the call, always fit.)
    auto counted = [&](int n) { return (pieces + 4 / n - 1) / (4 / n) * n_seqs <= 0xffffffffLL; };
    const bool large = (__int128)pieces * 32 * rows * 2 * cache_row_bytes(c.format, c.d_head) >= 1 << 28;
    const int to_a_line = c.head_stride < c.token_stride && c.head_stride == cache_row_bytes(c.format, c.d_head) ? heads_to_a_line(c.format, c.d_head, c.page_tokens % 16 == 0) : 1;
    if (!s.rows && large)
        for (int n = to_a_line; n > 1 && s.next == 1; n /= 2)
            if (c.n_heads % n == 0 && n * cols <= kAttendCols && rows / n >= places / 8 && counted(n)) s.next = n;
    const int64_t items = rows / s.next;
    // two pieces to a step: two sets of the heads have to fit the columns, and a wave should have as much to do (us, one and two pieces: one row of 700 tokens of 8 heads 9.5 and 12.5, of 4096
    // 12.6 and 11.3; 16 of 32768 178 and 153)
    // (several KV heads to an item, of a large call, always have: for these there is no kernel of one)
    s.pieces = !s.rows && two_pieces(c.format, bf16, c.d_head, c.page_tokens % 16 == 0) && cols <= kAttendCols / 2 && (s.next > 1 || pieces * rows >= 2 * places) ? 2 : 1;
    const int64_t tile = 4 / s.next * s.pieces, tiles = (pieces + tile - 1) / tile, most = places < kAttendMaxShares ? places : kAttendMaxShares;
    const __int128 all = (__int128)tiles * items;
    s.n = (int)(s.rows ? rows : all < most ? (int64_t)all : most);
    // Few items whose rows share cache lines, each of a multiple of eight shares: in turn, the shares that read the same tokens are an XCD's.  (One row of 131072 tokens, us, neighbours to an XCD and in turn.  4 bits,
    // heads of 128, two workgroups to a compute unit: 8 heads 62.3 and 55.8, 16 101 and 87, 2 45.8 and 46.5; 5, 10 and 12, no such multiples, 50.1 and 50.7, 73 and 75, 84 and 85.  8 bits, heads of 64, three: 3 heads 35.9 and
    // 33.4, 8 55 and 42, 12 66 and 55, 16 84 and 67; 5, 7 and 10 43.1 and 43.1, 50.1 and 50.8, 61.3 and 61.8.  3 rows of 32768 of 4 heads 25.0 and 20.7; 3 of 20000 of 5 21.4 and 24.2, 5 of 30000 of 2 23.1 and 24.7.)
    s.in_turn = s.next == 1 && to_a_line > 1 && rows <= 16 && s.n % (8 * rows) == 0;
    return s;
}

AttendRoute attend_route(const kvtc_cache& c, kvtc_dtype dtype, int n_seqs, int n_q_heads, int64_t max_tokens, int64_t sinks, int64_t window) {
    int parts, cols;
    heads_of(c, n_q_heads, parts, cols);
    const Shares s = shares_at_once(c, dtype == KVTC_BF16, n_seqs, parts, cols, max_tokens, sinks, window);
    return {s.rows, s.in_turn, s.pieces, s.next, s.n};
}

size_t attend_work_bytes(const kvtc_cache& c, int n_seqs, int n_q_heads, int64_t max_tokens) {
    int parts, cols;
    heads_of(c, n_q_heads, parts, cols);
    // (types, windows and short rows make for other tiles and fewer workgroups, and none for more shares that are joined than this; an item of several KV heads has up to 16 rows)
    const int64_t places = (int64_t)compute_units() * groups_each(c.format, c.d_head, false), tiles = (max_tokens + 127) / 128;
    const __int128 all = (__int128)tiles * (n_seqs < 1 ? 1 : n_seqs) * c.n_heads * parts;
    const int64_t most = places < kAttendMaxShares ? places : kAttendMaxShares, n = all < most ? (int64_t)all : most;
    const int rows = heads_to_a_line(c.format, c.d_head, true) > 1 ? kAttendCols : cols;
    return (size_t)kAttendMaxShares * 4 + (size_t)n * 2 * part_floats(rows, c.d_head) * sizeof(float);
}

hipError_t launch_attend(const AttendArgs& a, kvtc_dtype dtype, hipStream_t stream) {
    AttendPlan p;
    p.a = a;
    int parts, cols;
    heads_of(a.c, a.n_q_heads, parts, cols);
    p.group = a.n_q_heads / a.c.n_heads;
    p.parts = parts;
    p.cols = cols;
    p.in_page = a.c.page_tokens % 16 == 0;
    p.few = 2 * (uint32_t)compute_units();
    p.seqs_each = (a.n_seqs + 63) / 64;
    auto in_31 = [](int64_t v) { return (uint32_t)(v < 0x7fffffffLL ? v : 0x7fffffffLL); };
    p.max_tokens = in_31(a.max_tokens);
    p.sinks = in_31(a.sinks);
    p.window = in_31(a.window);
    p.scale_stride = (int64_t)a.c.n_heads * a.c.page_tokens * cache_scale_bytes(a.c.format, a.c.d_head);
    uint32_t s = 0;                                        // (n < 2^31: m = ceil(2^(31 + s) / d) is near enough)
    while ((1ull << s) < (uint64_t)a.c.page_tokens) ++s;
    p.page_mul = (uint32_t)(((1ull << (31 + s)) + a.c.page_tokens - 1) / a.c.page_tokens);
    p.page_shift = 31 + s;
    const Shares shares = shares_at_once(a.c, dtype == KVTC_BF16, a.n_seqs, parts, cols, a.max_tokens, a.sinks, a.window);
    static void (*const launch[6])(const AttendPlan&, const Shares&, hipStream_t) = {launch_attend_0, launch_attend_1, launch_attend_2, launch_attend_3, launch_attend_4, launch_attend_5};
    p.in_turn = shares.in_turn;
    launch[(dtype == KVTC_BF16 ? 0 : 3) + a.c.format](p, shares, stream);
    return hipGetLastError();
}

#endif

}  // namespace kvtc

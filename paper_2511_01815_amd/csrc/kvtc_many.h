// Attention of many new tokens over the pages of a live cache: what its kernels share.  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "kvtc_cache.h"

namespace kvtc {

constexpr int64_t kManyMaxRows = 1LL << 29;                // tokens times query heads of a call: items of 64 rows and 256 threads are fewer than 2^32 threads

struct ManyArgs {
    kvtc_cache c;
    const void* q;
    int64_t q_token_stride, q_head_stride;                 // elements
    const int32_t* starts;
    const int32_t* pages;
    int64_t pages_stride;
    const int32_t* lengths;
    int64_t max_tokens;
    int64_t sinks, window;                                 // window 0: every token up to the row's own
    float scale;
    int32_t causal, n_seqs, n_tokens, n_q_heads;
    void* out;
    float* lse;
    void* work;
    uint32_t* status;
};

// Kinds of kernel: all in fp32; blocks of 128, of 64 and of 32 rows in 16 bits.
enum ManyKind { kManyPlain = 0, kManyWide = 1, kManyTwo = 2, kManyOne = 3 };
// How a call runs: rows (token, query head of the group) of an item and tokens of a tile by the kernel's kind, items that there can be, parts that an item's tiles are cut into, tiles of a part.
struct ManyRoute { int kind, rows, tile, items, parts; uint32_t part_tiles; };

struct ManyPlan {                                          // what the host works out
    ManyArgs a;
    ManyRoute r;
    int32_t group;                                         // query heads of a KV head
    uint32_t sinks, window;                                // those of `a`, at most 2^31 - 1
    int64_t scale_stride;                                  // bytes of a page's scales
    uint32_t page_mul, page_shift;                         // token / page_tokens = token * page_mul >> page_shift
    float* part_out;                                       // [parts][n_tokens * n_q_heads][d_head]
    float2* part_sums;                                     // [parts][n_tokens * n_q_heads]: the largest score, in powers of two, and the sum
    int32_t* order;                                        // [n_seqs] where they are more than kManyScanned: the largest start so far
};

// An item: up to r.rows rows of one sequence and KV head, row = new token * group + query head of the group, and the tokens that any of them sees.
struct ManyItem {
    int b, n_new, length, row0, rows;                      // the sequence, its new tokens, its tokens; the item's first row, in the sequence, and their number
    int first;                                             // the sequence's first token, in the batch
    int at0, at1;                                          // positions of the first and the last row's tokens
    uint32_t tiles, sink_tiles, from_tile;                 // tiles: the first sink_tiles, then those from from_tile on
    int end;                                               // tokens from here on are not seen by any row
};

typedef const __attribute__((address_space(1))) uint8_t* ManyBytes;
__device__ __forceinline__ uint32_t many_tile(const ManyItem& it, uint32_t n) { return n < it.sink_tiles ? n : it.from_tile + (n - it.sink_tiles); }
__device__ __forceinline__ uint32_t many_page(const ManyPlan& p, uint32_t token) { return (uint32_t)(((uint64_t)token * p.page_mul) >> p.page_shift); }
// Whether the row at position `at` sees token t (below the sequence's length).
__device__ __forceinline__ bool many_sees(const ManyPlan& p, int at, int t) {
    return !p.a.causal || (t <= at && (p.window == 0u || (uint32_t)t < p.sinks || (uint32_t)(at - t) < p.window));
}

// Items are numbered so that the first of sequence b is m[b] * group / rows + b, where m[b] is the largest of starts[0] .. starts[b] that are in 0..n_tokens: numbers rise with b, whatever starts holds, and a sequence that
// begins at m[b] and has n tokens has no more items than there are numbers to the next one's.  (No prefix sum is needed; some numbers have no item.)  A sequence that begins below m[b] has none: its rows may be another's.
//
// Few sequences: every wave looks at all starts, 256 at a time, and works m out.  More: many_order_kernel has, in a launch before.  (By halving over starts as they are, one that does not ascend hides items of sequences before
// and behind it.  Both ways, sequences of 1 to 4 new tokens behind 50 to 400, 32 query heads of 128 to 8, bf16, us: 256 of them 61.6 and 64.1, 500 113.3 and 113.0, 1000 222.6 and 207.5, 4000 1150 and 804.)
constexpr int kManyScanned = 512;

// The running maximum of numbers that are not negative over the lanes.
__device__ __forceinline__ int many_running_max(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));              // from 1, 2, 4 and 8 lanes before, of 16
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));              // lanes 15 and 47 to the 16 behind them
    return max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));           // lane 31 to the 32 behind it
}
__device__ __forceinline__ int many_start_or_zero(const ManyPlan& p, int start) { return (uint32_t)start <= (uint32_t)p.a.n_tokens ? start : 0; }

// The same in all lanes of a wave; all of them take part.
__device__ inline bool many_item(const ManyPlan& p, uint32_t number, ManyItem& it) {
    const int lane = threadIdx.x & 63, shift = __builtin_ctz((uint32_t)p.r.rows);
    auto number_of = [&](int m, int b) { return ((uint32_t)m * (uint32_t)p.group >> shift) + (uint32_t)b; };        // (below 2^29 / 32 + 2^16)
    int lo = -1, m = 0;                                    // the last sequence whose first item's number is not above the wanted one, and its m
    if (p.a.n_seqs <= kManyScanned) {
        for (int first = 0, before = 0; first < p.a.n_seqs; first += 256) {
            int v[4];
            bool all = true;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = first + 64 * c + lane < p.a.n_seqs ? p.a.starts[first + 64 * c + lane] : 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (first + 64 * c >= p.a.n_seqs || !all) break;
                const int b = first + 64 * c + lane, mine = max(many_running_max(many_start_or_zero(p, v[c])), before);
                const uint64_t below = __ballot(b < p.a.n_seqs && number_of(mine, b) <= number);
                if (below != 0) {
                    const int last = 63 - __builtin_clzll(below);
                    lo = first + 64 * c + last;
                    m = __builtin_amdgcn_readlane(mine, last);
                }
                all = below == ~0ull;
                before = __builtin_amdgcn_readlane(mine, 63);
            }
            if (!all) break;
        }
    } else {
        lo = 0;
        for (int hi = p.a.n_seqs; hi - lo > 1;) {
            const int step = (hi - lo + 63) / 64, b = lo + lane * step;
            const uint64_t below = __ballot(b < hi && number_of(p.order[b < hi ? b : lo], b) <= number);
            if (below == 0) break;
            lo += (63 - __builtin_clzll(below)) * step;
            hi = lo + step < hi ? lo + step : hi;
        }
        lo = __builtin_amdgcn_readfirstlane(lo);
        m = __builtin_amdgcn_readfirstlane(p.order[lo]);
    }
    if (lo < 0 || number < number_of(m, lo)) return false;
    const int s0 = __builtin_amdgcn_readfirstlane(p.a.starts[lo]), s1 = __builtin_amdgcn_readfirstlane(p.a.starts[lo + 1]);
    if (s0 != m || s1 < s0 || s1 > p.a.n_tokens) return false;
    const int64_t block = number - number_of(m, lo);
    const int64_t all = (int64_t)(s1 - s0) * p.group, row0 = block * p.r.rows;
    if (row0 >= all) return false;
    it.b = lo;
    it.first = s0;
    it.n_new = s1 - s0;
    it.length = __builtin_amdgcn_readfirstlane(p.a.lengths[lo]);
    if (it.length < 0 || it.length > p.a.max_tokens) it.length = 0;         // (reported elsewhere)
    it.rows = (int)(all - row0 < p.r.rows ? all - row0 : p.r.rows);
    // row0 and rows count from the sequence's first row; both fit 31 bits, as all rows of a call do
    it.row0 = (int)row0;
    const int behind = it.length - it.n_new;
    it.at0 = behind + it.row0 / p.group;
    it.at1 = behind + (it.row0 + it.rows - 1) / p.group;
    it.end = p.a.causal ? (it.at1 + 1 < 0 ? 0 : it.at1 + 1) : it.length;
    if (it.length == 0) it.end = 0;
    const uint32_t size = (uint32_t)p.r.tile, last = ((uint32_t)it.end + size - 1) / size;
    it.sink_tiles = 0;
    it.from_tile = 0;
    if (p.window != 0u) {
        const int64_t from = (int64_t)it.at0 - (int64_t)p.window + 1;
        const uint32_t sinks = p.sinks < (uint32_t)it.end ? p.sinks : (uint32_t)it.end;
        it.sink_tiles = (sinks + size - 1) / size;
        it.from_tile = from > 0 ? (uint32_t)from / size : 0u;
        if (it.from_tile < it.sink_tiles) it.from_tile = it.sink_tiles;
        if (it.from_tile > last) it.from_tile = last;
    }
    it.tiles = it.sink_tiles + (last - it.from_tile);
    return true;
}

// Sequences that cannot be: each work-item of the launch looks at one.
__device__ __forceinline__ void many_report(const ManyPlan& p, uint64_t item) {
    if (item >= (uint64_t)p.a.n_seqs) return;
    const int s0 = p.a.starts[item], s1 = p.a.starts[item + 1], length = p.a.lengths[item];
    if (s0 < 0 || s1 < s0 || s1 > p.a.n_tokens || length < 0 || length > p.a.max_tokens) report_lowest(p.a.status, (uint32_t)item);
}

ManyRoute many_route(const kvtc_cache& c, kvtc_dtype dtype, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens, int64_t sinks, int64_t window);
size_t many_work_bytes(const kvtc_cache& c, int n_seqs, int64_t n_tokens, int n_q_heads, int64_t max_tokens);
hipError_t launch_many(const ManyArgs& a, kvtc_dtype dtype, hipStream_t stream);

}  // namespace kvtc

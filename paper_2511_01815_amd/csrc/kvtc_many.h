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

// Items are numbered so that the first of sequence b is starts[b] * group / rows + b: a sequence of n tokens has no more than there are to the next one's.  (No prefix sum is needed; some numbers have no item.)
// The same in all lanes of a wave; all of them take part.
__device__ inline bool many_item(const ManyPlan& p, uint32_t number, ManyItem& it) {
    const int lane = threadIdx.x & 63;
    const int64_t want = number;
    auto number_of = [&](int b) { return (int64_t)p.a.starts[b] * p.group / p.r.rows + b; };
    int lo = 0, hi = p.a.n_seqs;                           // the last sequence whose first item's number is not above the wanted one
    while (hi - lo > 1) {
        const int step = (hi - lo + 63) / 64, b = lo + lane * step;
        const uint64_t below = __ballot(b < hi && number_of(b < hi ? b : lo) <= want);
        if (below == 0) break;
        lo += (63 - __builtin_clzll(below)) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int s0 = __builtin_amdgcn_readfirstlane(p.a.starts[lo]), s1 = __builtin_amdgcn_readfirstlane(p.a.starts[lo + 1]);
    const int64_t block = want - ((int64_t)s0 * p.group / p.r.rows + lo);
    if (s0 < 0 || s1 < s0 || s1 > p.a.n_tokens || block < 0) return false;
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

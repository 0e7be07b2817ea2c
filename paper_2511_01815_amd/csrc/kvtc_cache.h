// The live cache as the kernels see it: rows in pages, in 16, 8 or 4 bits.  Internal to the library.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "../../include/kvtc.h"

namespace kvtc {

constexpr int kCacheMaxHeads = 1024;
constexpr int kAttendMaxSeqs = 65536;
constexpr int kAttendMaxShares = 1024;                     // shares of a kvtc_attend, at most: a counter each at the workspace's begin, which calls leave zero and kvtc_attend_many keeps clear of
constexpr int kCacheGroup = 32;                            // features that share a shift and a scale in the 4-bit format

__host__ __device__ constexpr int cache_row_bytes(int format, int d) { return format == KVTC_CACHE_BF16 ? 2 * d : format == KVTC_CACHE_FP8 ? d : d / 2; }
__host__ __device__ constexpr int cache_scale_bytes(int format, int d) { return format == KVTC_CACHE_BF16 ? 0 : format == KVTC_CACHE_FP8 ? 4 : 4 * d / kCacheGroup; }

struct CacheTokenArgs {                                    // tokens into the cache or out of it
    kvtc_cache c;
    void *k, *v;                                           // features (write: read only)
    int64_t token_stride, head_stride;                     // of the features, in elements
    const int64_t* slots;
    int64_t n_tokens;
    uint32_t* status;
};

struct AttendArgs {
    kvtc_cache c;
    const void* q;
    int64_t q_seq_stride, q_head_stride;                   // elements
    const int32_t* pages;
    int64_t pages_stride;
    const int32_t* lengths;
    int64_t max_tokens;
    int64_t sinks, window;                                 // window 0: every token is seen
    float scale;
    int32_t n_seqs, n_q_heads;
    void* out;
    float* lse;
    void* work;
    uint32_t* status;
};

// The checks of a cache that every call makes; `who` is the call.
kvtc_status cache_check(const char* who, const kvtc_cache* c);

// *status = 1 + the lowest index reported, 0 as long as there is none.
__device__ __forceinline__ void report_lowest(uint32_t* status, uint32_t index) {
    if (!status) return;
    uint32_t seen = __hip_atomic_load(status, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    while (seen == 0u || seen > index + 1u)
        if (__hip_atomic_compare_exchange_strong(status, &seen, index + 1u, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) break;
}

__device__ __forceinline__ float bf16_f32(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint16_t f32_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }

// Tokens of one launch, at most: a row is up to d / 8 work-items, in whole workgroups of 256, and a launch of 2^32 of them is refused.  (So rows fit 31 bits.)
constexpr int64_t cache_launch_tokens(int n_heads, int d) { return ((1LL << 32) - 256) / (d / 8) / n_heads; }
hipError_t launch_cache_write(const CacheTokenArgs& a, kvtc_dtype dtype, int64_t launch_tokens, hipStream_t stream);
hipError_t launch_cache_read(const CacheTokenArgs& a, kvtc_dtype dtype, int64_t launch_tokens, hipStream_t stream);
hipError_t launch_attend(const AttendArgs& a, kvtc_dtype dtype, hipStream_t stream);
// How a call runs: a wave to a row (1) or shares (0), shares to the XCDs in turn, pieces of 32 tokens to a wave's step, KV heads to a workgroup, workgroups.
struct AttendRoute { int rows, in_turn, pieces, next, workgroups; };
AttendRoute attend_route(const kvtc_cache& c, kvtc_dtype dtype, int n_seqs, int n_q_heads, int64_t max_tokens, int64_t sinks, int64_t window);
size_t attend_work_bytes(const kvtc_cache& c, int n_seqs, int n_q_heads, int64_t max_tokens);

}  // namespace kvtc

// Places of new tokens in a paged cache, worked out on the GPU from the sequences' lengths: rows of a ragged batch, slots, positions, and the page tables grown from a list of free pages, for gfx950.
//
// Sequence b has had[b] tokens in ceil(had / page_tokens) pages and gets new[b] more.  With the running sums over the sequences, in their order,
//     starts[b] = sum of new,   dealt[b] = sum of ceil((had + new) / page_tokens) - ceil(had / page_tokens),
// its i-th new token is row starts[b] + i of the batch, at position had[b] + i, and its j-th new page the free list's entry dealt[b] + j from the end.
//
// A workgroup works both sums out for itself, a thread to a sequence, a block of sequences after another, finds the sequence of each of its rows among those in the LDS by halving, and writes the
// rows' slots; whoever has a page's first token writes the page into the table.  One workgroup, where that has rows few enough, writes the sequences' results as well: one launch, of which latencies in a row
// are the time (64 sequences of one token each, 5.1 us a call: loads, six steps of a sum, a search, stores).  Of more rows a workgroup of its own does (27578 rows of 256 sequences: 5.7 us a call), or, where the
// results may be written over what other workgroups read, a second launch (27648 rows of 256 sequences with lengths and the number of free pages in place 12.5 us a call, in buffers of their own 6.3).
#include <hip/hip_runtime.h>
#include "kvtc_cache.h"
#include "kvtc_dev.h"

namespace kvtc {
kvtc_status set_error(kvtc_status st, const char* fmt, ...);

struct PlaceArgs {
    const int32_t *had, *fresh;
    int32_t* pages;
    int64_t pages_stride, most;                            // most: tokens that a row of the table holds
    const int32_t *free_list, *n_free;
    int32_t *starts, *lengths, *left;
    int64_t* slots;
    int32_t* positions;
    uint32_t* status;
    int32_t n_seqs, n_tokens, page_tokens, rows_each;      // rows_each: of a workgroup
    uint32_t page_mul, page_shift;
};

constexpr uint32_t kSumsEnd = 0x80000000u;                 // sums stop here, beyond every number of rows or pages
__device__ __forceinline__ uint32_t sum_to_end(uint32_t a, uint32_t b) {
    const uint64_t s = (uint64_t)a + b;
    return s < kSumsEnd ? (uint32_t)s : kSumsEnd;
}

// ROWS: slots and positions of workgroup `group` of those that have rows are written; SEQS: the sequences' results.
template <int THREADS, bool ROWS, bool SEQS>
__device__ __forceinline__ void place_group(const PlaceArgs& a, uint32_t group) {
    constexpr int WAVES = THREADS / 64;
    __shared__ uint32_t end_of[THREADS], dealt_of[THREADS], sums[2][WAVES];
    __shared__ int32_t had_of[THREADS], start_of[THREADS];
    __shared__ uint32_t most_dealt;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t n_free = a.n_free[0];
    const uint32_t row0 = ROWS ? group * (uint32_t)a.rows_each : 0u, row1 = ROWS ? min((uint32_t)a.n_tokens, row0 + (uint32_t)a.rows_each) : 0u;
    auto pages_of = [&](uint32_t n) { return n == 0u ? 0u : (uint32_t)(((uint64_t)(n - 1u) * a.page_mul) >> a.page_shift) + 1u; };
    if (tid == 0) most_dealt = 0u;
    uint32_t rows_before = 0, dealt_before = 0;
    for (int first = 0; first < a.n_seqs; first += THREADS) {
        const int b = first + tid;
        const bool is = b < a.n_seqs;
        const int32_t had = is ? a.had[b] : 0, fresh = is ? a.fresh[b] : 0;
        // the sum of v up to and with this sequence; `start`: without it
        auto over_block = [&](uint32_t v, uint32_t (&of_waves)[WAVES], uint32_t before, uint32_t& start) {
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t w = (uint32_t)__shfl_up((int)v, d, 64);
                if (lane >= d) v = sum_to_end(v, w);
            }
            if (lane == 63) of_waves[wave] = v;
            __syncthreads();
            uint32_t base = before;
            for (int w = 0; w < wave; ++w) base = sum_to_end(base, of_waves[w]);
            const uint32_t last = (uint32_t)__shfl_up((int)v, 1, 64);
            start = lane > 0 ? sum_to_end(base, last) : base;
            return sum_to_end(base, v);
        };
        uint32_t start, dealt_start;
        const uint32_t end = over_block(fresh > 0 ? (uint32_t)fresh : 0u, sums[0], rows_before, start);
        start = min(start, (uint32_t)a.n_tokens);
        const int64_t length = (int64_t)had + fresh;
        bool fine = is && had >= 0 && fresh >= 0 && end <= (uint32_t)a.n_tokens && length <= a.most;
        const uint32_t held = had > 0 ? pages_of((uint32_t)had) : 0u, need = fine ? pages_of((uint32_t)length) - held : 0u;
        const uint32_t dealt = over_block(need, sums[1], dealt_before, dealt_start);
        fine = fine && (need == 0u || (int64_t)dealt <= n_free);
        if constexpr (SEQS) {
            if (is) {
                a.starts[b] = (int32_t)start;
                a.lengths[b] = fine ? (int32_t)length : had;
                if (!fine) report_lowest(a.status, (uint32_t)b);
                if (b == a.n_seqs - 1) a.starts[a.n_seqs] = (int32_t)min(end, (uint32_t)a.n_tokens);
                if (fine && need > 0u) atomicMax(&most_dealt, dealt);
            }
        }
        end_of[tid] = end;
        if constexpr (ROWS) {
            dealt_of[tid] = dealt_start;
            had_of[tid] = fine ? had : -1;
            start_of[tid] = (int32_t)start;
        }
        __syncthreads();
        const int n = min(THREADS, a.n_seqs - first);
        const uint32_t from = rows_before, to = min(end_of[n - 1], (uint32_t)a.n_tokens);
        if constexpr (ROWS) {
            for (uint32_t i = max(row0, from) + tid; i < min(row1, to); i += THREADS) {
                int lo = 0, hi = n - 1;                    // the first sequence that ends behind row i
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (end_of[mid] > i) hi = mid;
                    else lo = mid + 1;
                }
                const int32_t has = had_of[lo];
                int64_t slot = -1;
                uint32_t position = 0;
                if (has >= 0) {
                    position = (uint32_t)has + (i - (uint32_t)start_of[lo]);
                    const uint32_t index = (uint32_t)(((uint64_t)position * a.page_mul) >> a.page_shift), in = position - index * (uint32_t)a.page_tokens, kept = pages_of((uint32_t)has);
                    int32_t* entry = a.pages + (int64_t)(first + lo) * a.pages_stride + index;
                    int32_t page;
                    if (index < kept) {
                        page = *entry;
                    } else {
                        page = a.free_list[n_free - 1 - (int64_t)(dealt_of[lo] + (index - kept))];
                        if (in == 0u) *entry = page;
                    }
                    if (page >= 0) slot = (int64_t)page * a.page_tokens + in;
                }
                a.slots[i] = slot;
                if (a.positions) a.positions[i] = (int32_t)position;
            }
        }
        // (the block's last sequence has the block's sums; a copy, before the next block's are written)
        rows_before = end_of[n - 1];
        __shared__ uint32_t dealt_end;
        if (tid == n - 1) dealt_end = dealt;
        __syncthreads();
        dealt_before = dealt_end;
        if (ROWS && !SEQS && rows_before >= row1) break;
    }
    if constexpr (ROWS) {
        for (uint32_t i = max(row0, min(rows_before, (uint32_t)a.n_tokens)) + tid; i < row1; i += THREADS) {
            a.slots[i] = -1;
            if (a.positions) a.positions[i] = 0;
        }
    }
    if constexpr (SEQS) {
        __syncthreads();
        if (tid == 0) {
            a.left[0] = (int32_t)(n_free - most_dealt);
            if (a.n_seqs == 0) a.starts[0] = 0;
        }
    }
}

template <int THREADS, bool ROWS, bool SEQS>
__global__ void __launch_bounds__(THREADS) place_kernel(const PlaceArgs a) {
    place_group<THREADS, ROWS, SEQS>(a, blockIdx.x);
}
// The first workgroup writes the sequences' results.
__global__ void __launch_bounds__(1024) place_all_kernel(const PlaceArgs a) {
    if (blockIdx.x == 0) place_group<1024, false, true>(a, 0u);
    else place_group<1024, true, false>(a, blockIdx.x - 1u);
}

constexpr int kPlaceRows = 4096, kPlaceRowsEach = 1024;    // rows of a workgroup that is alone, and of one among others

// Whether nothing that a workgroup reads is written by another: results in buffers of their own.
static bool place_apart(const PlaceArgs& a) {
    struct Range { uintptr_t at, bytes; };
    const size_t seqs = (size_t)a.n_seqs * 4;
    const Range in[3] = {{reinterpret_cast<uintptr_t>(a.had), seqs}, {reinterpret_cast<uintptr_t>(a.fresh), seqs}, {reinterpret_cast<uintptr_t>(a.n_free), 4}};
    const Range out[3] = {{reinterpret_cast<uintptr_t>(a.lengths), seqs}, {reinterpret_cast<uintptr_t>(a.starts), seqs + 4}, {reinterpret_cast<uintptr_t>(a.left), 4}};
    for (const Range& i : in)
        for (const Range& o : out)
            if (i.at < o.at + o.bytes && o.at < i.at + i.bytes) return false;
    return true;
}

hipError_t launch_place(PlaceArgs a, hipStream_t stream) {
    if (a.n_tokens <= kPlaceRows) {
        a.rows_each = kPlaceRows;
        if (a.n_seqs <= 256 && a.n_tokens <= 1024) hipLaunchKernelGGL((place_kernel<256, true, true>), dim3(1), dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((place_kernel<1024, true, true>), dim3(1), dim3(1024), 0, stream, a);
        return hipGetLastError();
    }
    a.rows_each = kPlaceRowsEach;
    const int groups = (int)(((int64_t)a.n_tokens + kPlaceRowsEach - 1) / kPlaceRowsEach);
    if (place_apart(a)) {
        hipLaunchKernelGGL(place_all_kernel, dim3(groups + 1), dim3(1024), 0, stream, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((place_kernel<1024, true, false>), dim3(groups), dim3(1024), 0, stream, a);
    hipLaunchKernelGGL((place_kernel<1024, false, true>), dim3(1), dim3(1024), 0, stream, a);
    return hipGetLastError();
}

}  // namespace kvtc

extern "C" kvtc_status kvtc_cache_place(int n_seqs, const int32_t* lengths_dev, const int32_t* new_dev, int page_tokens, int32_t* pages_dev, int64_t pages_stride, const int32_t* free_dev,
                                        const int32_t* n_free_dev, int64_t n_tokens, int32_t* starts_dev, int32_t* lengths_out_dev, int32_t* n_free_out_dev, int64_t* slots_dev,
                                        int32_t* positions_dev, uint32_t* status_dev, kvtc_stream stream) {
    using namespace kvtc;
    if (n_seqs < 0 || n_seqs > kAttendMaxSeqs) return set_error(KVTC_E_ARG, "kvtc_cache_place: n_seqs=%d outside 0..%d", n_seqs, kAttendMaxSeqs);
    if (n_tokens < 0 || n_tokens > 0x7fffffffLL) return set_error(KVTC_E_ARG, "kvtc_cache_place: n_tokens=%lld", (long long)n_tokens);
    if (page_tokens < 1) return set_error(KVTC_E_ARG, "kvtc_cache_place: page_tokens=%d", page_tokens);
    if (pages_stride < 1 || pages_stride > 0x7fffffffLL) return set_error(KVTC_E_ARG, "kvtc_cache_place: pages_stride=%lld outside 1..2^31-1", (long long)pages_stride);
    if (!starts_dev || !n_free_dev || !n_free_out_dev || !free_dev || (n_tokens > 0 && !slots_dev)) return set_error(KVTC_E_ARG, "kvtc_cache_place: null buffer");
    if (n_seqs > 0 && (!lengths_dev || !new_dev || !pages_dev || !lengths_out_dev)) return set_error(KVTC_E_ARG, "kvtc_cache_place: null buffer");
    auto off = [](const void* p, uintptr_t by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) != 0; };
    if (off(lengths_dev, 4) || off(new_dev, 4) || off(pages_dev, 4) || off(free_dev, 4) || off(n_free_dev, 4) || off(starts_dev, 4) || off(lengths_out_dev, 4) || off(n_free_out_dev, 4) ||
        off(positions_dev, 4) || off(status_dev, 4) || off(slots_dev, 8))
        return set_error(KVTC_E_ARG, "kvtc_cache_place: misaligned buffer (slots: 8 bytes, others 4)");
    PlaceArgs a{};
    a.had = lengths_dev;
    a.fresh = new_dev;
    a.pages = pages_dev;
    a.pages_stride = pages_stride;
    const __int128 holds = (__int128)pages_stride * page_tokens;
    a.most = holds < 0x7fffffffLL ? (int64_t)holds : 0x7fffffffLL;
    a.free_list = free_dev;
    a.n_free = n_free_dev;
    a.starts = starts_dev;
    a.lengths = lengths_out_dev;
    a.left = n_free_out_dev;
    a.slots = slots_dev;
    a.positions = positions_dev;
    a.status = status_dev;
    a.n_seqs = n_seqs;
    a.n_tokens = (int32_t)n_tokens;
    a.page_tokens = page_tokens;
    uint32_t s = 0;                                        // (n < 2^31: m = ceil(2^(31 + s) / d) is near enough)
    while ((1ull << s) < (uint64_t)page_tokens) ++s;
    a.page_mul = (uint32_t)(((1ull << (31 + s)) + page_tokens - 1) / page_tokens);
    a.page_shift = 31 + s;
    const hipError_t e = launch_place(a, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(KVTC_E_HIP, "kvtc_cache_place: launch failed: %s", hipGetErrorString(e));
    return KVTC_OK;
}

// The pages of the compressed KV cache (include/ecco_paged.h): which pages a step's new tokens get, where each token goes, and the way
// back of pages that are no longer needed.
//
// Everything is running sums over the sequences (rows, pages) and then one item per page or per row, found again by a search in the
// running sums.  What it costs is latency: a workgroup loads the lengths, sums, reads the stack and writes, each step waiting
// for the one before.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ecco_launch.h"
#include "ecco_paged.h"
#include "ecco_plan.h"

using namespace ecco;

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr uint32_t kFull = 0x7FFFFFFFu;  // where sums stop: lengths are the caller's, and their sum may be anything

__device__ __forceinline__ uint32_t add_full(uint32_t a, uint32_t b) { return min(a + b, kFull); }  // both at most kFull

// Sum, up to kFull, over the workgroup's threads up to and including this one.  at: kWaves words of LDS; total: of all threads.
__device__ __forceinline__ uint32_t scan(uint32_t v, uint32_t* at, uint32_t& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(v, d);
        v = lane >= d ? add_full(v, o) : v;
    }
    __syncthreads();  // the words' last readers are done
    if (lane == 63) at[wave] = v;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before = w == wave ? total : before;
        total = add_full(total, at[w]);
    }
    return add_full(before, v);
}
// how many of the n ascending numbers are at most v: the sequence that item v belongs to, given the sums up to and including each
__device__ __forceinline__ int upper(const uint32_t* sums, int n, uint32_t v) {
    int lo = 0;
    for (int step = 1 << (31 - __builtin_clz(n)); step > 0; step >>= 1)
        if (lo + step <= n && sums[lo + step - 1] <= v) lo += step;
    return lo;
}
__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, int shift) { return (tokens >> shift) + ((tokens & ((1u << shift) - 1u)) != 0u); }

struct TakeArgs {
    const int32_t* seq_len;
    const int32_t* new_len;
    int32_t* table;
    const int32_t* free_pages;
    const int32_t* free_count;
    int32_t* free_left;
    int32_t* q_start;
    int32_t* kv_len;
    int32_t* slots;
    int B, shift, max_pages, n_pages, n_tokens;
};
// the slot of token `pos` of sequence b, which is served: its table has an entry for the token
__device__ __forceinline__ int32_t slot_of(const TakeArgs& a, int b, uint32_t pos) {
    const int32_t page = a.table[(size_t)b * a.max_pages + (pos >> a.shift)];
    return (uint32_t)page < (uint32_t)a.n_pages ? (int32_t)(((uint32_t)page << a.shift) | (pos & ((1u << a.shift) - 1u))) : -1;
}

// One workgroup, 1024 sequences at a time.  kSlots: the rows' slots as well; otherwise slots_kernel writes them, with as many
// workgroups as there is work for.
template <bool kSlots>
__global__ __launch_bounds__(kThreads) void take_kernel(TakeArgs a) {
    __shared__ uint32_t at[kWaves], row_end[kThreads], page_end[kThreads], held_of[kThreads], given;
    __shared__ bool served_of[kThreads];
    const int tid = threadIdx.x;
    const uint32_t count = (uint32_t)min(max(*a.free_count, 0), a.n_pages), n_tokens = (uint32_t)a.n_tokens;
    uint32_t rows = 0, pages = 0;  // of the sequences before these
    if (tid == 0) {
        a.q_start[0] = 0;
        given = 0u;
    }
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid, n_seq = min(kThreads, a.B - b0);
        const uint32_t held = b < a.B ? (uint32_t)max(a.seq_len[b], 0) : 0u, fresh = b < a.B ? (uint32_t)max(a.new_len[b], 0) : 0u;
        uint32_t new_rows, new_pages;
        const uint32_t end = add_full(rows, scan(fresh, at, new_rows));
        const uint32_t first = pages_of(held, a.shift), last = pages_of(held + fresh, a.shift);  // (the sum is below 2^32)
        const bool fits = end <= n_tokens && end < kFull && last <= (uint32_t)a.max_pages;
        const uint32_t need = fits ? last - first : 0u, asked = add_full(pages, scan(need, at, new_pages));
        const bool served = fits && (need == 0u || asked <= count);
        if (b < a.B) {
            a.q_start[b + 1] = (int32_t)min(end, n_tokens);
            a.kv_len[b] = served ? (int32_t)(held + fresh) : 0;
        }
        row_end[tid] = min(end, n_tokens);
        page_end[tid] = asked;
        held_of[tid] = held;
        served_of[tid] = served;
        if (served && need != 0u) atomicMax(&given, asked);
        __syncthreads();
        // The i-th page from the top of the stack is for the sequence in whose sum it lies.  Of those that need pages the first ones are served,
        // so a page that is not given has none behind it that is.
        const uint32_t pages_after = add_full(pages, new_pages), rows_after = add_full(rows, new_rows), row0 = min(rows, n_tokens);
        for (uint32_t i = min(pages, count) + tid; i < min(pages_after, count); i += kThreads) {
            const int s = upper(page_end, n_seq, i);
            const uint32_t before = s > 0 ? page_end[s - 1] : pages;
            if (served_of[s]) a.table[(size_t)(b0 + s) * a.max_pages + pages_of(held_of[s], a.shift) + (i - before)] = a.free_pages[count - 1u - i];
        }
        if (kSlots) {
            __threadfence_block();
            __syncthreads();
            for (uint32_t t = row0 + tid; t < min(rows_after, n_tokens); t += kThreads) {
                const int s = upper(row_end, n_seq, t);
                const uint32_t before = s > 0 ? row_end[s - 1] : row0;
                a.slots[t] = served_of[s] ? slot_of(a, b0 + s, held_of[s] + (t - before)) : -1;
            }
        }
        rows = rows_after;
        pages = pages_after;
        __syncthreads();  // the sums have been read
    }
    if (kSlots)
        for (uint32_t t = min(rows, n_tokens) + tid; t < n_tokens; t += kThreads) a.slots[t] = -1;
    if (tid == 0) *a.free_left = (int32_t)(count - given);
}

// The slots of the rows, behind take_kernel<false>: a row finds its sequence in q_start.
constexpr int kSlotThreads = 256;
__global__ __launch_bounds__(kSlotThreads) void slots_kernel(TakeArgs a) {
    for (uint32_t t = blockIdx.x * kSlotThreads + threadIdx.x; t < (uint32_t)a.n_tokens; t += gridDim.x * kSlotThreads) {
        const int s = upper(reinterpret_cast<const uint32_t*>(a.q_start + 1), a.B, t);
        int32_t slot = -1;
        if (s < a.B && a.kv_len[s] > 0) slot = slot_of(a, s, (uint32_t)max(a.seq_len[s], 0) + (t - (uint32_t)a.q_start[s]));
        a.slots[t] = slot;
    }
}

struct ReleaseArgs {
    const int32_t* seq_len;
    const int32_t* keep_len;
    const int32_t* table;
    int32_t* free_pages;
    const int32_t* free_count;
    int32_t* free_left;
    int B, shift, max_pages, n_pages;
};
// One workgroup, 1024 sequences at a time, their entries in rounds of eight per thread: entry 1024 j + i of a round is the j-th one of thread i.
// Entries that are pages keep their order on the stack: each is counted in by ballots.
constexpr int kEach = 8;
__global__ __launch_bounds__(kThreads) void release_kernel(ReleaseArgs a) {
    __shared__ uint32_t at[kWaves], end_of[kThreads], first_of[kThreads], found[kEach * kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t count = (uint32_t)min(max(*a.free_count, 0), a.n_pages);
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid, n_seq = min(kThreads, a.B - b0);
        const int held = b < a.B ? max(a.seq_len[b], 0) : 0, keep = b < a.B ? min(max(a.keep_len[b], 0), held) : 0;
        const uint32_t first = pages_of((uint32_t)keep, a.shift), last = min(pages_of((uint32_t)held, a.shift), (uint32_t)a.max_pages);
        uint32_t total;
        end_of[tid] = scan(last > first ? last - first : 0u, at, total);
        first_of[tid] = first;
        __syncthreads();
        for (uint32_t i0 = 0; i0 < total; i0 += kThreads * kEach) {
            int32_t page[kEach];
            uint32_t before[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint32_t i = i0 + j * kThreads + tid;
                page[j] = -1;
                if (i < total) {
                    const int s = upper(end_of, n_seq, i);
                    page[j] = a.table[(size_t)(b0 + s) * a.max_pages + first_of[s] + (i - (s > 0 ? end_of[s - 1] : 0u))];
                }
            }
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint64_t pages = __ballot((uint32_t)page[j] < (uint32_t)a.n_pages);
                before[j] = __builtin_amdgcn_mbcnt_hi((uint32_t)(pages >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)pages, 0u));
                if (lane == 0) found[j * kWaves + wave] = (uint32_t)__builtin_popcountll(pages);
            }
            __syncthreads();
            if (wave == 0) {  // running sums of the counts, two per lane
                static_assert(kEach * kWaves == 128, "two counts per lane");
                const uint32_t x = found[2 * lane], y = found[2 * lane + 1];
                uint32_t sum = x + y;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const uint32_t o = __shfl_up(sum, d);
                    sum += lane >= d ? o : 0u;
                }
                found[2 * lane] = sum - y;
                found[2 * lane + 1] = sum;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int w = j * kWaves + wave;
                const uint32_t to = count + (w > 0 ? found[w - 1] : 0u) + before[j];
                if ((uint32_t)page[j] < (uint32_t)a.n_pages && to < (uint32_t)a.n_pages) a.free_pages[to] = page[j];
            }
            count = min(count + found[kEach * kWaves - 1], (uint32_t)a.n_pages);
            __syncthreads();  // the counts have been read
        }
        __syncthreads();
    }
    if (tid == 0) *a.free_left = (int32_t)count;
}

int shift_of(int page_tokens) { return __builtin_ctz((unsigned)page_tokens); }

}  // namespace

extern "C" {

int ecco_kv_pages_take(const int32_t* seq_len, const int32_t* new_len, int B, int page_tokens, int max_pages, int32_t* page_table,
                       const int32_t* free_pages, const int32_t* free_count, int32_t* free_left, int n_pages,
                       int n_tokens, int32_t* q_start, int32_t* kv_len, int32_t* slots, void* stream) {
    if (!seq_len || !new_len || !page_table || !free_pages || !free_count || !free_left || !q_start || !kv_len || (!slots && n_tokens > 0)) return ECCO_EINVAL;
    if (B <= 0 || n_tokens < 0 || !pool_fits(page_tokens, max_pages) || !pool_fits(page_tokens, n_pages)) return ECCO_ESHAPE;
    for (const void* p : {(const void*)seq_len, (const void*)new_len, (const void*)page_table, (const void*)free_pages, (const void*)free_count, (const void*)free_left,
                          (const void*)q_start, (const void*)kv_len, (const void*)slots})
        if (!aligned(p, 4)) return ECCO_EALIGN;
    const TakeArgs a{seq_len, new_len, page_table, free_pages, free_count, free_left, q_start, kv_len, slots, B, shift_of(page_tokens), max_pages, n_pages, n_tokens};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (n_tokens <= kThreads) {
        hipLaunchKernelGGL(take_kernel<true>, dim3(1), dim3(kThreads), 0, st, a);
    } else {
        hipLaunchKernelGGL(take_kernel<false>, dim3(1), dim3(kThreads), 0, st, a);
        ECCO_HIP_CHECK(hipGetLastError());
        hipLaunchKernelGGL(slots_kernel, dim3(std::min(1024, (n_tokens - 1) / kSlotThreads + 1)), dim3(kSlotThreads), 0, st, a);
    }
    ECCO_HIP_CHECK(hipGetLastError());
    return ECCO_OK;
}

int ecco_kv_pages_release(const int32_t* seq_len, const int32_t* keep_len, int B, int page_tokens, int max_pages, const int32_t* page_table,
                          int32_t* free_pages, const int32_t* free_count, int32_t* free_left, int n_pages, void* stream) {
    if (!seq_len || !keep_len || !page_table || !free_pages || !free_count || !free_left) return ECCO_EINVAL;
    if (B <= 0 || !pool_fits(page_tokens, max_pages) || !pool_fits(page_tokens, n_pages)) return ECCO_ESHAPE;
    for (const void* p : {(const void*)seq_len, (const void*)keep_len, (const void*)page_table, (const void*)free_pages, (const void*)free_count, (const void*)free_left})
        if (!aligned(p, 4)) return ECCO_EALIGN;
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kThreads), 0, static_cast<hipStream_t>(stream),
                       ReleaseArgs{seq_len, keep_len, page_table, free_pages, free_count, free_left, B, shift_of(page_tokens), max_pages, n_pages});
    ECCO_HIP_CHECK(hipGetLastError());
    return ECCO_OK;
}

}  // extern "C"

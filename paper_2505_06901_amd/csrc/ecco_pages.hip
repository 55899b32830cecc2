// The pages of the compressed KV cache (include/ecco_paged.h): which pages a step's new tokens get, where each token goes, and the way
// back of pages that are no longer needed.
//
// Everything is running sums over the sequences (rows, pages) and then one item per row or per page, whose sequence is found again: by a search in the
// running sums when pages are taken, by marks at the sequences' first entries when they are given back.  What it costs is latency: a workgroup loads the lengths, sums, reads the stack and writes, each step waiting
// for the one before.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ecco_launch.h"
#include "ecco_paged.h"
#include "ecco_plan.h"

using namespace ecco;

namespace {

constexpr uint32_t kFull = 0x7FFFFFFFu;  // where sums stop: lengths are the caller's, and their sum may be anything

__device__ __forceinline__ uint32_t add_full(uint32_t a, uint32_t b) { return min(a + b, kFull); }  // both at most kFull

// Sums, up to kFull, over the workgroup's threads up to and including this one, of two numbers at once.  at: two words of LDS per wavefront; total: of all threads.
struct Two {
    uint32_t x, y;
};
template <int kThreads>
__device__ __forceinline__ Two scan(Two v, uint32_t* at, Two& total) {
    constexpr int kWaves = kThreads / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t x = __shfl_up(v.x, d), y = __shfl_up(v.y, d);
        v.x = lane >= d ? add_full(v.x, x) : v.x;
        v.y = lane >= d ? add_full(v.y, y) : v.y;
    }
    __syncthreads();  // the words' last readers are done
    if (lane == 63) {
        at[wave] = v.x;
        at[kWaves + wave] = v.y;
    }
    __syncthreads();
    Two before = {0u, 0u};
    total = {0u, 0u};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        before.x = w == wave ? total.x : before.x;
        before.y = w == wave ? total.y : before.y;
        total.x = add_full(total.x, at[w]);
        total.y = add_full(total.y, at[kWaves + w]);
    }
    return {add_full(before.x, v.x), add_full(before.y, v.y)};
}
// The largest v of the threads in front of this one
template <int kThreads>
__device__ __forceinline__ uint32_t largest_before(uint32_t v, uint32_t* at) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(v, d);
        v = lane >= d ? max(v, o) : v;
    }
    const uint32_t mine = __shfl_up(v, 1);
    __syncthreads();
    if (lane == 63) at[wave] = v;
    __syncthreads();
    uint32_t before = lane > 0 ? mine : 0u;
    for (int w = 0; w < wave; ++w) before = max(before, at[w]);
    return before;
}
// For each of kEach items v: how many of the n ascending sums are at most v, which is the sequence that the item belongs to, given the sums up to
// and including each.  The searches go on side by side, so that one does not wait for another's reads.
template <int kEach>
__device__ __forceinline__ void find(const uint32_t* sums, int n, const uint32_t (&v)[kEach], int (&lo)[kEach]) {
#pragma unroll
    for (int j = 0; j < kEach; ++j) lo[j] = 0;
    for (int step = 1 << (31 - __builtin_clz(n)); step > 0; step >>= 1) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int to = lo[j] + step;
            const uint32_t sum = sums[min(to, n) - 1];
            lo[j] = (to <= n ? sum : ~0u) <= v[j] ? to : lo[j];  // (items are below kFull)
        }
    }
}
__device__ __forceinline__ uint32_t pages_of(uint32_t tokens, int shift) { return (tokens >> shift) + ((tokens & ((1u << shift) - 1u)) != 0u); }

struct TakeArgs {
    const int32_t* seq_len;
    const int32_t* new_len;
    int32_t* table;
    const int32_t* free_pages;
    const int32_t* free_count;
    int32_t* free_left;  // null: not yet
    int32_t* q_start;
    int32_t* kv_len;
    int32_t* slots;
    int B, shift, max_pages, n_pages, n_tokens;
};

// Every workgroup sums over all sequences, kThreads at a time, and writes the slots of its share of the rows; the first one also what there is one of per
// sequence.  A new page's first token is one of the new ones: the thread that has it writes the table's entry.  What a row needs is either an
// entry that was there before or a page of the stack, so that no thread reads what another writes, and only free_left may be an
// input as well: then it is written by a launch of its own behind this one.
constexpr int kRows = 2;  // per thread and round
template <int kThreads, bool kOnlyLeft>
__global__ __launch_bounds__(kThreads) void take_kernel(TakeArgs a) {
    __shared__ uint32_t at[kThreads / 32], row_end[kThreads], held_of[kThreads], page_of[kThreads], given;
    const int tid = threadIdx.x;
    const bool chief = blockIdx.x == 0;
    const uint32_t count = (uint32_t)min(max(*a.free_count, 0), a.n_pages), n_tokens = (uint32_t)a.n_tokens, mask = (1u << a.shift) - 1u;
    uint32_t rows = 0, pages = 0;  // of the sequences before these
    if (tid == 0) {
        given = 0u;
        if (chief && !kOnlyLeft) a.q_start[0] = 0;
    }
    constexpr uint32_t kNot = ~0u;  // page_of: not served
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid, n_seq = min(kThreads, a.B - b0);
        const uint32_t held = b < a.B ? (uint32_t)max(a.seq_len[b], 0) : 0u, fresh = b < a.B ? (uint32_t)max(a.new_len[b], 0) : 0u;
        const uint32_t first = pages_of(held, a.shift), last = pages_of(held + fresh, a.shift);  // (the sum is below 2^32)
        uint32_t need = last <= (uint32_t)a.max_pages ? last - first : 0u;
        Two total;
        Two sum = scan<kThreads>({fresh, need}, at, total);
        const uint32_t end = add_full(rows, sum.x), rows_after = add_full(rows, total.x);
        const bool fits = end <= n_tokens && end < kFull && last <= (uint32_t)a.max_pages;
        if (rows_after > n_tokens) {  // uniform: sequences whose rows have no place ask for no pages
            need = fits ? need : 0u;
            Two again;
            sum.y = scan<kThreads>({0u, need}, at, again).y;
            total.y = again.y;
        }
        const uint32_t asked = add_full(pages, sum.y), pages_after = add_full(pages, total.y);
        const bool served = fits && (need == 0u || asked <= count);
        if (b < a.B && chief && !kOnlyLeft) {
            a.q_start[b + 1] = (int32_t)min(end, n_tokens);
            a.kv_len[b] = served ? (int32_t)(held + fresh) : 0;
        }
        row_end[tid] = min(end, n_tokens);
        held_of[tid] = held;
        page_of[tid] = served ? asked - need : kNot;  // its first page, counted from the top of the stack
        if (chief && served && need != 0u) atomicMax(&given, asked);  // those that need pages and get them are the first ones of those that need any
        __syncthreads();
        const uint32_t row0 = min(rows, n_tokens), row1 = min(rows_after, n_tokens), step = gridDim.x * kThreads * kRows;
        for (uint32_t t0 = kOnlyLeft ? row1 : row0 + blockIdx.x * kThreads * kRows; t0 < row1; t0 += step) {
            uint32_t t[kRows];
            int s[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) t[j] = t0 + j * kThreads + tid;
            find(row_end, n_seq, t, s);
            int32_t page[kRows];
            uint32_t pos[kRows];
            bool top[kRows];
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                page[j] = -1;
                top[j] = false;
                if (t[j] < row1) {
                    const uint32_t h = held_of[s[j]], from = page_of[s[j]];
                    pos[j] = h + (t[j] - (s[j] > 0 ? row_end[s[j] - 1] : row0));
                    if (from != kNot) {
                        const uint32_t col = pos[j] >> a.shift, had = pages_of(h, a.shift);
                        top[j] = col >= had && (pos[j] & mask) == 0u;
                        page[j] = col >= had ? a.free_pages[count - 1u - (from + (col - had))] : a.table[(size_t)(b0 + s[j]) * a.max_pages + col];
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < kRows; ++j) {
                if (t[j] >= row1) continue;
                if (top[j]) a.table[(size_t)(b0 + s[j]) * a.max_pages + (pos[j] >> a.shift)] = page[j];
                a.slots[t[j]] = (uint32_t)page[j] < (uint32_t)a.n_pages ? (int32_t)(((uint32_t)page[j] << a.shift) | (pos[j] & mask)) : -1;
            }
        }
        rows = rows_after;
        pages = pages_after;
        __syncthreads();  // the sums have been read
    }
    if (!kOnlyLeft)
        for (uint32_t t = min(rows, n_tokens) + blockIdx.x * kThreads + tid; t < n_tokens; t += gridDim.x * kThreads) a.slots[t] = -1;
    if (tid == 0 && chief && a.free_left) *a.free_left = (int32_t)(count - given);
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
// One workgroup, 1024 sequences at a time, their entries in rounds of sixteen per thread, one behind the other.  Which sequence an entry belongs to:
// each sequence marks its first entry of the round, and an entry is of the last one that is marked at it or before it.  Entries that are pages keep
// their order on the stack.  (A search per entry, or one per thread that goes on from there, is a chain of dependent reads: 256 sequences of one to
// two pages 7.9 us, of 256 pages each in two rounds 13.7 us.)
constexpr int kReleaseThreads = 1024, kEach = 16;
__global__ __launch_bounds__(kReleaseThreads) void release_kernel(ReleaseArgs a) {
    constexpr int kThreads = kReleaseThreads, kRound = kThreads * kEach;
    __shared__ uint32_t at[kThreads / 32], first_of[kThreads + 1];
    __shared__ __align__(16) uint16_t marks[kRound];
    const int tid = threadIdx.x;
    uint32_t count = (uint32_t)min(max(*a.free_count, 0), a.n_pages);
    for (int b0 = 0; b0 < a.B; b0 += kThreads) {
        const int b = b0 + tid;
        const int held = b < a.B ? max(a.seq_len[b], 0) : 0, keep = b < a.B ? min(max(a.keep_len[b], 0), held) : 0;
        const uint32_t first = pages_of((uint32_t)keep, a.shift), last = min(pages_of((uint32_t)held, a.shift), (uint32_t)a.max_pages);
        const uint32_t n = last > first ? last - first : 0u;
        Two total;
        const uint32_t end = scan<kThreads>({n, 0u}, at, total).x, begin = end - n;
        first_of[tid + 1] = first - begin;  // what an entry's place among all has to be added to
        for (uint32_t i0 = 0; i0 < total.x; i0 += kRound) {
            uint4* own = reinterpret_cast<uint4*>(marks) + tid * 2;
            own[0] = own[1] = make_uint4(0u, 0u, 0u, 0u);
            __syncthreads();
            if (n != 0u && begin < i0 + kRound && end > i0) marks[max(begin, i0) - i0] = (uint16_t)(tid + 1);
            __syncthreads();
            const uint4 lo = own[0], hi = own[1];
            const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            uint32_t s[kEach], most = 0;  // (marks ascend: the last one is the largest)
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                most = max(most, (w[j / 2] >> (16 * (j % 2))) & 0xFFFFu);
                s[j] = most;
            }
            const uint32_t before = largest_before<kThreads>(most, at);
            int32_t page[kEach];
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const uint32_t item = i0 + tid * kEach + j, of = max(s[j], before);
                page[j] = -1;
                if (item < total.x) page[j] = a.table[(size_t)(b0 + (int)of - 1) * a.max_pages + (first_of[of] + item)];
            }
            uint32_t mine = 0;
#pragma unroll
            for (int j = 0; j < kEach; ++j) mine += (uint32_t)page[j] < (uint32_t)a.n_pages ? 1u : 0u;
            Two found;
            uint32_t to = count + scan<kThreads>({mine, 0u}, at, found).x - mine;
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                if ((uint32_t)page[j] >= (uint32_t)a.n_pages) continue;
                if (to < (uint32_t)a.n_pages) a.free_pages[to] = page[j];
                ++to;
            }
            count = min(count + found.x, (uint32_t)a.n_pages);
        }
        __syncthreads();  // the places have been read
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
    if (kv_len == seq_len || kv_len == new_len) return ECCO_EINVAL;  // one workgroup writes what others may yet have to read
    TakeArgs a{seq_len, new_len, page_table, free_pages, free_count, free_left, q_start, kv_len, slots, B, shift_of(page_tokens), max_pages, n_pages, n_tokens};
    hipStream_t st = static_cast<hipStream_t>(stream);
    // Few sequences and rows: a workgroup whose barriers meet four wavefronts and not sixteen.  Sequences / rows, four and sixteen wavefronts, us: 1 / 1 2.9 and 4.0,
    // 64 / 64 3.7 and 4.5, 256 / 512 4.6 and 4.9; but 8 / 1024 5.2 and 4.6, 256 / 1024 6.5 and 5.4, 300 / 300 5.8 and 4.8, 512 / 512 6.2 and 5.0.
    if (B <= 256 && n_tokens <= 256 * kRows) {
        hipLaunchKernelGGL((take_kernel<256, false>), dim3(1), dim3(256), 0, st, a);
        ECCO_HIP_CHECK(hipGetLastError());
        return ECCO_OK;
    }
    const int grid = std::min(std::max((n_tokens + 1024 * kRows - 1) / (1024 * kRows), 1), 256);
    const bool late = grid > 1 && free_left == free_count;  // other workgroups may yet have to read it
    if (late) a.free_left = nullptr;
    hipLaunchKernelGGL((take_kernel<1024, false>), dim3(grid), dim3(1024), 0, st, a);
    ECCO_HIP_CHECK(hipGetLastError());
    if (!late) return ECCO_OK;
    a.free_left = free_left;
    hipLaunchKernelGGL((take_kernel<1024, true>), dim3(1), dim3(1024), 0, st, a);
    ECCO_HIP_CHECK(hipGetLastError());
    return ECCO_OK;
}

int ecco_kv_pages_release(const int32_t* seq_len, const int32_t* keep_len, int B, int page_tokens, int max_pages, const int32_t* page_table,
                          int32_t* free_pages, const int32_t* free_count, int32_t* free_left, int n_pages, void* stream) {
    if (!seq_len || !keep_len || !page_table || !free_pages || !free_count || !free_left) return ECCO_EINVAL;
    if (B <= 0 || !pool_fits(page_tokens, max_pages) || !pool_fits(page_tokens, n_pages)) return ECCO_ESHAPE;
    for (const void* p : {(const void*)seq_len, (const void*)keep_len, (const void*)page_table, (const void*)free_pages, (const void*)free_count, (const void*)free_left})
        if (!aligned(p, 4)) return ECCO_EALIGN;
    hipLaunchKernelGGL(release_kernel, dim3(1), dim3(kReleaseThreads), 0, static_cast<hipStream_t>(stream),
                       ReleaseArgs{seq_len, keep_len, page_table, free_pages, free_count, free_left, B, shift_of(page_tokens), max_pages, n_pages});
    ECCO_HIP_CHECK(hipGetLastError());
    return ECCO_OK;
}

}  // extern "C"

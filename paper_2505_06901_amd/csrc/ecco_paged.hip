// Attention of a step's new tokens over the paged compressed cache (include/ecco_paged.h).
//
// What bounds it.  With few rows (new tokens times query heads that share a key/value head) a block's 128 values are decoded for a handful of products:
// the decoders' table reads from LDS are the limit, about 22 blocks per ns on the whole chip, and a chain of 64 values, 4 us, where there are few
// blocks.  They are decoded on the way into the products then (attend_rows_kernel).  With many rows it is the matrix cores: sequences are decoded once,
// into operands in the workspace (attend_expand_kernel, 9 blocks per ns with the writing), and the products run from there (attend_tiles_kernel).
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <algorithm>
#include <type_traits>

#include "ecco_decode.h"
#include "ecco_launch.h"
#include "ecco_paged.h"
#include "ecco_plan.h"

using namespace ecco;
using namespace ecco_chain;

namespace {

typedef float float16_t __attribute__((ext_vector_type(16)));

struct PagedArgs {
    const uint32_t* dev_k;
    const uint32_t* dev_v;
    const uint16_t* q;
    const uint4* k_blocks;
    const uint32_t* k_meta;
    const uint4* v_blocks;
    const uint32_t* v_meta;
    const int32_t* table;
    const int32_t* q_start;
    const int32_t* kv_len;
    void* out;
    float* ws;        // partial results of ranges
    int32_t* ranges;  // [B] (first, count) of the sequences' ranges
    int64_t q_stride;
    int Sk, Sv, B, Hq, Hkv, n_tokens, n_pages, shift, max_pages, max_kv;
    int table_words, both, span, step, half;
    int few;       // rows of a sequence and key/value head up to which it is decoded on the way
    int cut, cus;  // whether sequences are cut into ranges, and for how many workgroups at once
};

// The arguments of the running kernel, read again: what the loops need of them once per unit would otherwise take scalar registers
// throughout, and those are short beside the decoders.
typedef const __attribute__((address_space(4))) PagedArgs args_t;
__device__ __forceinline__ args_t* fresh_args() {
    args_t* a = (args_t*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(a));
    return a;
}
template <class T>
__device__ __forceinline__ const __attribute__((address_space(1))) T* in_global(const T* p) { return (const __attribute__((address_space(1))) T*)p; }

__device__ __forceinline__ void store_out(args_t* a, size_t at, float v) {
    if (a->half) ((__attribute__((address_space(1))) _Float16*)a->out)[at] = (_Float16)v;
    else ((__attribute__((address_space(1))) float*)a->out)[at] = v;
}
// A row that sees nothing has no weights and gives zeros; one whose scores are no numbers has a denominator that is none, and gives NaN.
__device__ __forceinline__ float normalised(float num, float den) { return den == 0.0f ? 0.0f : num / den; }
// (a pointer that is read back is known to be global memory only by a cast there and back)
__device__ __forceinline__ const uint32_t* global_words(const uint32_t* p) { return (const uint32_t*)in_global(p); }

// What the lengths of the device say of sequence b, within what the host has sized the launch for (no rows if they are none of q's)
struct Sequence {
    int row0, n_new, kv;  // first row, rows, tokens to read
    __device__ __forceinline__ Sequence() : row0(0), n_new(0), kv(0) {}
    __device__ __forceinline__ Sequence(args_t* a, int b) {
        const auto* start = in_global(a->q_start);
        row0 = start[b];
        const int end = start[b + 1];
        n_new = row0 >= 0 && end <= a->n_tokens ? max(0, end - row0) : 0;
        kv = max(0, min(in_global(a->kv_len)[b], a->max_kv));
    }
};

// The pages that hold the two halves of a unit of 32 tokens (a page has 16 tokens at least).  The same for all lanes, but in vector
// registers.
struct UnitPages {
    int page[2];
};
__device__ __forceinline__ bool in_pool(int page, int n_pages) { return (uint32_t)page < (uint32_t)n_pages; }
// of the unit that begins at token t0 of sequence b; `last`: the last token that is read of it
__device__ __forceinline__ UnitPages unit_pages(int b, int t0, int last) {
    args_t* a = fresh_args();
    int zero = 0;
    asm volatile("" : "+v"(zero));
    const auto* row = in_global(a->table) + (size_t)b * a->max_pages;
    UnitPages p;
    p.page[0] = row[(min(t0, last) >> a->shift) + zero];
    p.page[1] = row[(min(t0 + kUnitBlocks / 2, last) >> a->shift) + zero];
    return p;
}
// As load_unit of the contiguous caches: the payload pieces of this lane and the meta word of the unit's block `tok`, which it decodes.  Slots of a
// page are all readable, whether they hold a token or not; of a page that is none the first one's are read.  ok: whether the page of token `tok` is one
template <bool kValues>
__device__ __forceinline__ UnitLoad load_unit(const UnitPages& p, int hkv, int t0, int lane, int tok, bool& ok) {
    args_t* a = fresh_args();
    const uint32_t mask = (1u << a->shift) - 1u;
    size_t at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
        at[h] = (((size_t)(uint32_t)(in_pool(p.page[h], a->n_pages) ? p.page[h] : 0) * (uint32_t)a->Hkv + (uint32_t)hkv) << a->shift) + (((uint32_t)t0 + 16u * h) & mask);
    const global_u4* blocks = (const global_u4*)(kValues ? a->v_blocks : a->k_blocks);
    const auto* meta = in_global(kValues ? a->v_meta : a->k_meta);
    const u32x4 v0 = blocks[at[0] * 4 + lane], v1 = blocks[at[1] * 4 + lane];
    UnitLoad u;
    u.v0 = make_uint4(v0.x, v0.y, v0.z, v0.w);
    u.v1 = make_uint4(v1.x, v1.y, v1.z, v1.w);
    u.meta = meta[(tok < 16 ? at[0] : at[1]) + (tok & 15)];
    ok = in_pool(tok < 16 ? p.page[0] : p.page[1], a->n_pages);
    return u;
}

// ---- few rows per key/value head ---------------------------------------------------------------------------------------
// The rows of a sequence and a key/value head are its new tokens times the grp = Hq / Hkv query heads that share it, row r being head r % grp of
// new token r / grp.  A workgroup takes up to kRows of them (8, 16 or 32) over a range of the sequence's tokens, and decodes every K and V block of
// the range on the way into the products, as the grouped-query kernel over contiguous caches does (kv_attend_gqa_kernel says how tiles, halves
// and rests lie; the columns here are rows in this sense, each with an end of its own: what a token sees ends with itself).  From 9 rows on the
// scores come from v_mfma_f32_32x32x16_f16 instead: one product per eight values and chain for 32 tokens and up to 32 rows, no half of its operand
// zeroed, eight query values of one row per lane (lane l decodes chain l / 32 of token l % 32).  With 32 rows the second product runs over two tiles
// of 16.
//
// grid: ranges of the tokens (Range) that there may be, times Hkv.  Where a sequence has several, the workspace takes 128 outputs of each range
// and row, then (maximum, denominator) pairs, and a second kernel merges them.
// Five new tokens each of eight sequences of 570 to 2880 tokens, 32/8 heads: 48.6 us with 16 rows at a time, every block decoded twice; 30.7 us so.

constexpr float kLog2E = 1.4426950408889634f;
constexpr float kWeightTop = 15.0f;  // the largest weight's power of two: FP16 holds up to 2^16; numerators and denominators share it

// Which range of which sequence a workgroup takes.  Ranges are of one length for all sequences, so that one long sequence beside short ones
// gets many of them: the least length, kRangeLeast units or more, with which all workgroups find a place at once, looked for among 64 (one per
// lane).  Every wavefront works it out for itself from all the sequences' lengths, a load for up to 64 of them.  (Eight sequences of 690 to
// 3398 tokens, 8 x 4 heads: 29.3 us with four ranges each, 27.0 us with a workgroup per compute unit, 24.8 us with two; 16 sequences up to 4096 tokens
// 56.8 us and 50.6 us.)  A merge costs 3 to 4 us, as much as six units more per range: ranges of 4 and 12 units at the least, one sequence of 1000
// tokens 15.7 and 21.2 us, of 8 units 16.5 us; four of 2000 20.0, 21.6 and 17.1 us.
struct Range {
    int b, hkv;          // sequence, key/value head; b < 0: nothing to do
    int first, n, index; // ranges of the sequences before this one, of this one, and which of its it is
    int begin, end;      // tokens
    Sequence seq;
};
template <int kCtrl>
__device__ __forceinline__ int dpp_int(int v) { return __builtin_amdgcn_mov_dpp(v, kCtrl, 0xF, 0xF, true); }
// sum over the lanes up to and including this one
__device__ __forceinline__ int wave_scan(int v, int lane) {
    v += dpp_int<0x111>(v);  // row_shr 1, 2, 4, 8; zeros come in
    v += dpp_int<0x112>(v);
    v += dpp_int<0x114>(v);
    v += dpp_int<0x118>(v);
    const int a = __builtin_amdgcn_readlane(v, 15), b = a + __builtin_amdgcn_readlane(v, 31), c = b + __builtin_amdgcn_readlane(v, 47);
    return v + (lane < 16 ? 0 : lane < 32 ? a : lane < 48 ? b : c);
}
__device__ __forceinline__ Range find_range(args_t* a, int lane) {
    const int Hkv = a->Hkv, hkv = blockIdx.x % Hkv, j = blockIdx.x / Hkv;
    Range r{-1, hkv, 0, 1, 0, 0, 0, Sequence()};
    if (!a->cut) {  // a workgroup per sequence and head
        r.b = r.first = j;
        r.seq = Sequence(a, j);
        r.end = r.seq.kv;
        return r;
    }
    const int grp = a->Hq / Hkv, B = a->B;
    constexpr int kChunks = kRangeSequences / 64;
    int units[kChunks], total = 0;  // of sequence 64 c + l, -1 if it is not one of this kernel's
    Sequence of[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        units[c] = -1;
        if (c * 64 >= B) continue;
        of[c] = Sequence(a, min(c * 64 + lane, B - 1));
        const int rows = of[c].n_new * grp;
        if (c * 64 + lane < B && rows > 0 && rows <= a->few) units[c] = of[c].kv > 0 ? units_of(of[c].kv) : 0;
        total += max(units[c], 0);
    }
    const int least = range_least(wave_sum((float)total), Hkv, a->cus), step = max(1, least / 16);
    int length = least + least / 4;
    if (B <= 32) {
        const int mine = least + lane * step;
        const float per = __builtin_amdgcn_rcpf((float)mine);
        int n = 0;
        for (int b = 0; b < B; ++b) {
            const int u = __builtin_amdgcn_readlane(units[0], b);
            if (u >= 0) n += max(1, (int)((float)(u + mine - 1) * per));
        }
        const uint64_t good = __ballot(n * Hkv <= a->cus);
        if (good != 0ull) length = least + (int)__builtin_ctzll(good) * step;
    }
    int before = 0;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (c * 64 >= B || r.b >= 0) continue;
        const int n = units[c] < 0 ? 0 : max(1, (units[c] + length - 1) / length), end = wave_scan(n, lane);
        const uint64_t behind = __ballot(before + end > j);
        if (behind != 0ull) {
            const int l = __builtin_ctzll(behind);
            const auto lane_of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
            r.b = c * 64 + l;
            r.n = lane_of(n);
            r.first = before + lane_of(end) - r.n;
            r.index = j - r.first;
            r.seq.row0 = lane_of(of[c].row0);
            r.seq.n_new = lane_of(of[c].n_new);
            r.seq.kv = lane_of(of[c].kv);
            const int u = lane_of(units[c]), own = (u + r.n - 1) / r.n;  // the sequence's ranges, alike: at most `length`
            const auto tokens = [](int n) { return (int)min((int64_t)n * kUnitBlocks, (int64_t)0x7FFFFFFF); };
            r.begin = tokens(min(r.index * own, u));
            r.end = tokens(min((r.index + 1) * own, u));
        }
        before += __builtin_amdgcn_readlane(end, 63);
    }
    return r;
}

template <bool kLongK, bool kLongV, int kRows, int kWaves>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(kWaves == 12 ? 3 : kRows > 8 ? 2 : 4))) void attend_rows_kernel(PagedArgs) {
    constexpr int kThreads = kWaves * 64;
    static_assert(2 * kThreads >= kMaxS * kK, "load_table_items: two table items per thread cover every model");
    constexpr bool kWide = kRows > 8;
    constexpr int kTiles = kRows == 32 ? 2 : 1, kTileRows = kRows / kTiles;  // of the second product
    constexpr int kOutputs = (kTileRows * kGroup + kThreads - 1) / kThreads;  // output elements per thread and tile
    // (one more register than the allocation that bodies of up to 16 rows end in: none of its 64-bit shifts may have its amount in the last one, see build.py)
    if constexpr (kWide) asm volatile("" ::: "v136");
    args_t* const first = fresh_args();
    const int both = first->both, table_words = first->table_words;
    extern __shared__ __align__(16) uint32_t smem[];
    const int grp = first->Hq / first->Hkv, sstride = gqa_score_stride(first->span);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Range range = find_range(first, lane);
    const int b = range.b, hkv = range.hkv;
    if (b < 0) return;  // uniform, ahead of every barrier
    const Sequence seq = range.seq;
    const int rows = seq.n_new * grp;
    if (rows <= 0 || rows > first->few) return;
    uint32_t* k_tables = smem;
    uint32_t* wbuf = k_tables + table_words + wave * kUnitWords;
    uint32_t* tile = k_tables + table_words + kWaves * kUnitWords + wave * kTileWords;
    float* scores = reinterpret_cast<float*>(k_tables + table_words + kWaves * (kUnitWords + kTileWords));  // [rows][sstride]
    uint32_t* v_tables = k_tables + (both ? decode_table_words(first->Sk, kLongK) : 0);
    if (lane < kUnitBlocks) wbuf[lane * kStride + kBlockWords] = 0u;

    const int last = seq.kv - 1, t_begin = min(range.begin, max(seq.kv, 0)), t_end = min(range.end, max(seq.kv, 0)), n_splits = range.n;
    const int span_max = t_end - t_begin <= first->span ? first->span : first->step;  // a range that one span holds is not cut
    struct Place {
        int lane, n, slice, half, tok;  // n: matrix-core row or column; slice: k slice; half: chain of the lane's token `tok` of the unit
        __device__ Place() : lane(fresh_thread() & 63), n(lane & 15), slice(lane >> 4), half(slice & 1), tok(n + 16 * (lane >> 5)) {}
    };
    const float inv_sqrt_d = 0.08838834764831845f;  // 1 / sqrt(128)
    float4_t o[kTiles][8];  // tile j: row r is dimension 64 (r / 8) + 8 j + r % 8, column the row
    float run_max[kTiles], run_den[kTiles];  // of this wavefront and of row l % 16 of the tile; the denominator of the lane's tokens
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
#pragma unroll
        for (int j = 0; j < 8; ++j) o[t][j] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        run_max[t] = -INFINITY;
        run_den[t] = 0.0f;
    }

    for (int s0 = t_begin; s0 < t_end; s0 += span_max) {
        const int span = min(span_max, t_end - s0);
        const int units = (span + kUnitBlocks - 1) / kUnitBlocks;  // s0 is a multiple of 32
        UnitLoad pre;
        bool pre_ok;
        UnitPages now, next;  // of the unit that `pre` holds, and of the one behind it
        const auto pages_at = [&](int u) { return unit_pages(b, s0 + min(u, units - 1) * kUnitBlocks, last); };
        // ---- scores of the span, all rows
        float mx = -INFINITY;
        {
        const Place P;
        const int lane = P.lane, n = kWide ? lane & 31 : P.n, slice = P.slice, half = kWide ? lane >> 5 : P.half, tok = kWide ? n : P.tok;
        const int row = kWide ? n : n & 7;                              // row of this lane's column
        const bool row_ok = row < rows, b_ok = row_ok && (kWide || (n >> 3) == (lane >> 5));
        const int r = min(row, rows - 1), token = r / grp;
        const int sees = min(span, seq.kv - seq.n_new + token + 1 - s0);  // tokens of the span
        int u = wave;
        const auto load_k = [&](int at) { pre = load_unit<false>(now, hkv, s0 + min(at, units - 1) * kUnitBlocks, lane, tok, pre_ok); };
        uint4 bq[kHalf / 8];  // B operands: the query of this lane's row, dimensions 64 * half + 8j .. + 7
        const auto load_q = [&] {
            args_t* a = fresh_args();
            const global_u4* qsrc = (const global_u4*)(a->q + (int64_t)(seq.row0 + token) * a->q_stride + (hkv * grp + r - token * grp) * kGroup + half * kHalf);
#pragma unroll
            for (int j = 0; j < kHalf / 8; ++j) {
                const u32x4 v = qsrc[j];
                bq[j] = make_uint4(v.x, v.y, v.z, v.w);
            }
        };
        now = pages_at(u);
        next = pages_at(u + kWaves);
        if (!both) {
            args_t* a = fresh_args();
            const TableItems items = load_table_items(global_words(a->dev_k), a->Sk);
            load_k(u);
            load_q();
            __syncthreads();  // the V tables of the span before have been read
            a = fresh_args();
            build_tables<kLongK>(k_tables, global_words(a->dev_k), a->Sk, items);
            __syncthreads();
        } else if (s0 == t_begin) {  // both models' items, then the payload, then both builds
            args_t* a = fresh_args();
            const TableItems k_items = load_table_items(global_words(a->dev_k), a->Sk), v_items = load_table_items(global_words(a->dev_v), a->Sv);
            load_k(u);
            load_q();
            a = fresh_args();
            build_tables<kLongK>(k_tables, global_words(a->dev_k), a->Sk, k_items);
            build_tables<kLongV>(v_tables, global_words(a->dev_v), a->Sv, v_items);
            __syncthreads();
        } else {
            load_k(u);
            load_q();
        }
        const int Sk = fresh_args()->Sk;
        const Tables TK = table_pointers(k_tables, Sk);
#pragma unroll
        for (int j = 0; j < kHalf / 8; ++j) bq[j] = b_ok ? bq[j] : make_uint4(0u, 0u, 0u, 0u);
        for (; u < units; u += kWaves) {
            store_unit(wbuf, pre, lane);
            // a slot past the range, or of no page, may hold anything: scale 0, so that its values are zeros (up to 8 rows, tokens m and 16 + m share
            // a row of the product, and NaN * 0 would poison it)
            const uint32_t mw = u * kUnitBlocks + tok < span && pre_ok ? pre.meta : (pre.meta & 0xFFFF0000u);
            const uint64_t pool = __ballot(pre_ok);
            const bool ok0 = (pool & 1u) != 0u, ok1 = ((pool >> (kWide ? 16 : 32)) & 1u) != 0u;  // of the unit's two halves
            if (u + kWaves < units) {
                now = next;
                load_k(u + kWaves);
                next = pages_at(u + 2 * kWaves);
            }
            const Lane L = lane_setup(TK, mw, Sk);
            const _Float16 sh16 = __builtin_bit_cast(_Float16, (unsigned short)(mw & 0xFFFFu));
            const half2_t s2 = {sh16, sh16};
            uint32_t pk[4];
            std::conditional_t<kWide, float16_t, float4_t> acc = {};
            decode_chain<kLongK, kHalf>(wbuf + tok * kStride, half ? L.second_start : 0u, L, [&](int i, uint32_t e) {
                if ((i & 1) == 0) {
                    pk[(i >> 1) & 3] = e >> 16;
                    return;
                }
                pk[(i >> 1) & 3] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, pk[(i >> 1) & 3] | (e & 0xFFFF0000u)) * s2);
                if ((i & 7) != 7) return;
                const half8_t bv = __builtin_bit_cast(half8_t, bq[i >> 3]);
                const half8_t av = __builtin_bit_cast(half8_t, make_uint4(pk[0], pk[1], pk[2], pk[3]));
                if constexpr (kWide) acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(av, bv, acc, 0, 0, 0);
                else acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(av, bv, acc, 0, 0, 0);
            });
            // accumulator layouts: register i of lane l of a 16 x 16 tile is row 4 * (l / 16) + i, column l % 16; of a 32 x 32 one row
            // 8 (i / 4) + 4 (l / 32) + i % 4, column l % 32
#pragma unroll
            for (int w = 0; w < (kWide ? 4 : 1); ++w) {
                const bool upper = kWide ? w >= 2 : n >= 8, ok = upper ? ok1 : ok0;  // of the unit's tokens
                const int t0 = u * kUnitBlocks + (kWide ? 8 * w + 4 * half : 4 * slice + (upper ? 16 : 0));
                float4_t v;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = ok && t0 + i < sees ? acc[4 * w + i] * inv_sqrt_d : -INFINITY;
                    mx = fmaxf(mx, v[i]);
                }
                if (row_ok) *reinterpret_cast<float4_t*>(scores + row * sstride + t0) = v;  // for this wavefront alone
            }
        }
        // the wavefront's maximum per row: over the lanes of the column
        if (!kWide) {
            mx = fmaxf(mx, __shfl_xor(mx, 8));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
        }
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        }
        // ---- weighted sum of V over the span
        const Place P;
        const int lane = P.lane, n = P.n, slice = P.slice, half = P.half, tok = P.tok;
        const uint32_t swap_sel = (lane & 1) ? 0x03020706u : 0x05040100u;  // odd lanes keep the high halves, even lanes the low halves
        int u = wave;
        const auto load_v = [&](int at) { pre = load_unit<true>(now, hkv, s0 + min(at, units - 1) * kUnitBlocks, lane, tok, pre_ok); };
        now = pages_at(u);
        next = pages_at(u + kWaves);
        if (both) {
            load_v(u);
        } else {
            args_t* a = fresh_args();
            const TableItems items = load_table_items(global_words(a->dev_v), a->Sv);
            load_v(u);
            __syncthreads();
            a = fresh_args();
            build_tables<kLongV>(v_tables, global_words(a->dev_v), a->Sv, items);
            __syncthreads();
        }
        const int Sv = fresh_args()->Sv;
        const Tables TV = table_pointers(v_tables, Sv);
        float base[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const float before = run_max[t];
            run_max[t] = fmaxf(before, kWide ? __shfl(mx, 16 * t + n) : mx);
            base[t] = run_max[t] == -INFINITY ? 0.0f : run_max[t];  // (a wavefront without units, or without a score above -inf)
            if (s0 != t_begin) {  // every accumulator of a lane belongs to row l % 16
                const float alpha = before == -INFINITY ? 0.0f : __expf(before - base[t]);
                run_den[t] *= alpha;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[t][j] *= alpha;
            }
        }
        const int row = kWide ? n : n & 7;
        for (; u < units; u += kWaves) {
            store_unit(wbuf, pre, lane);
            const uint32_t mw = u * kUnitBlocks + tok < span && pre_ok ? pre.meta : (pre.meta & 0xFFFF0000u);
            if (u + kWaves < units) {
                now = next;
                load_v(u + kWaves);
                next = pages_at(u + 2 * kWaves);
            }
            const Lane L = lane_setup(TV, mw, Sv);
            const _Float16 sh16 = __builtin_bit_cast(_Float16, (unsigned short)(mw & 0xFFFFu));
            const half2_t s2 = {sh16, sh16};
            // B operand: weights of row l % 16 of the tile for tokens 8 * (l / 16) .. + 7 of the unit, 0 for what is not seen.  What an FP16 weight
            // leaves of the FP32 one is the operand of a product of its own, or with up to eight rows of columns 8..15.  The largest weight is
            // 2^kWeightTop, so that the pair keeps 22 bits down to 2^-18 of it and is off by 2^-40 of it at the most below (2^-25 with weights up to 1:
            // the many tokens far behind a leading one vanished from the sum, but not from the denominator).
            const float taken = !kWide && n < 8 ? 0.0f : 1.0f;
            half8_t pb[kTiles], rest[kTiles];
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const float* score = scores + min(16 * t + row, rows - 1) * sstride + 8 * slice + u * kUnitBlocks;
                const float4_t s[2] = {reinterpret_cast<const float4_t*>(score)[0], reinterpret_cast<const float4_t*>(score)[1]};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = 16 * t + row < rows ? __builtin_amdgcn_exp2f(fmaf(s[i >> 2][i & 3] - base[t], kLog2E, kWeightTop)) : 0.0f;
                    pb[t][i] = (_Float16)p;
                    rest[t][i] = (_Float16)fmaf(-taken, (float)pb[t][i], p);
                    run_den[t] += p;
                }
                if (!kWide) pb[t] = rest[t];
            }
            uint32_t pk[4];
            decode_chain<kLongV, kHalf>(wbuf + tok * kStride, half ? L.second_start : 0u, L, [&](int i, uint32_t e) {
                if ((i & 1) == 0) {
                    pk[(i >> 1) & 3] = e >> 16;
                    return;
                }
                pk[(i >> 1) & 3] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, pk[(i >> 1) & 3] | (e & 0xFFFF0000u)) * s2);
                if ((i & 7) != 7) return;
                // 8 values of this lane's token -> rows 8 * half + r of the tile (dimension 64 * half + 8 * (i / 8) + r);
                // an even lane takes dimension 2 r2 of its own and its neighbour's token, the odd neighbour dimension 2 r2 + 1
                wave_lds_fence();
#pragma unroll
                for (int r2 = 0; r2 < 4; ++r2) {
                    const uint32_t other = (uint32_t)__builtin_amdgcn_mov_dpp((int)pk[r2], 0xB1, 0xF, 0xF, true);  // quad_perm [1,0,3,2]
                    tile[(8 * half + 2 * r2 + (lane & 1)) * kTileStride + (tok >> 1)] = __builtin_amdgcn_perm(other, pk[r2], swap_sel);
                }
                wave_lds_fence();
                const uint4 a0 = *reinterpret_cast<const uint4*>(tile + n * kTileStride + 4 * slice);
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    o[t][i >> 3] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a0), pb[t], o[t][i >> 3], 0, 0, 0);
                    if (kWide) o[t][i >> 3] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a0), rest[t], o[t][i >> 3], 0, 0, 0);
                }
            });
        }
    }
    // ---- sum over the wavefronts, a tile of rows after the other; everything in LDS is dead behind the first barrier
    const Place P;
    const int n = P.n, slice = P.slice;
    args_t* const a = fresh_args();
    float* const ws = a->ws;
    // of the first row; the sequence's and head's rows lie one behind the other, each with its ranges
    const size_t part = ((size_t)range.first * a->Hkv + (size_t)hkv * n_splits) * kRows + range.index;
    const size_t total = (size_t)gridDim.x * kRows;
    if (a->cut && range.index == 0 && hkv == 0 && tid == 0) reinterpret_cast<int2*>(a->ranges)[b] = make_int2(range.first, n_splits);
    float* red = reinterpret_cast<float*>(smem);  // [wavefront][8 tiles][4 slices][16 lanes][4]
    float* state = red + kWaves * 8 * kRedTile;   // [wavefront][16] maxima, [wavefront][16] denominators
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        run_den[t] += __shfl_xor(run_den[t], 16);
        run_den[t] += __shfl_xor(run_den[t], 32);
        __syncthreads();
        if (lane < 16) state[wave * kGqaMaxGroup + lane] = run_max[t];
        __syncthreads();
        float most = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, state[w * kGqaMaxGroup + n]);
        const float mine = run_max[t] == -INFINITY ? 0.0f : __expf(run_max[t] - most);
        if (lane < 16) state[(kWaves + wave) * kGqaMaxGroup + lane] = run_den[t] * mine;
        if (!kWide) {  // what the rests contributed
#pragma unroll
            for (int j = 0; j < 8; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float here = o[t][j][i];
                    o[t][j][i] = here + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, here), 0x128, 0xF, 0xF, true));  // row_ror:8
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) *reinterpret_cast<float4_t*>(red + (wave * 8 + j) * kRedTile + slice * kRedRow + n * 4) = o[t][j] * mine;
        __syncthreads();
        const auto denominator = [&](int g) {
            float den = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) den += state[(kWaves + w) * kGqaMaxGroup + g];
            return den;
        };
        const int here = min(rows - 16 * t, kTileRows);  // rows of the tile
        if (n_splits > 1 && tid < here) {  // (the first wavefront's lane of row `tid` holds that row's maximum)
            const size_t at = total * kGroup + (part + (size_t)(16 * t + tid) * n_splits) * 2;
            ws[at] = most;
            ws[at + 1] = denominator(tid);
        }
#pragma unroll
        for (int k = 0; k < kOutputs; ++k) {
            const int e = tid + k * kThreads, g = e / kGroup, dim = e % kGroup;
            if (g < here) {
                const int at_row = 8 * (dim >> 6) + (dim & 7);
                const float* at = red + ((dim & 63) >> 3) * kRedTile + (at_row >> 2) * kRedRow + g * 4 + (at_row & 3);
                float sum = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) sum += at[w * 8 * kRedTile];
                const int r = 16 * t + g;
                if (n_splits == 1) {
                    const float den = denominator(g);
                    const int token = r / grp;
                    store_out(a, ((size_t)(seq.row0 + token) * a->Hq + hkv * grp + r - token * grp) * kGroup + dim, normalised(sum, den));
                } else {
                    ws[(part + (size_t)r * n_splits) * kGroup + dim] = sum;
                }
            }
        }
    }
}

// merges the token ranges of a row: grid (B * Hkv, rows that there may be), 128 threads
__global__ __launch_bounds__(kGroup) void attend_rows_merge_kernel(PagedArgs args, int kernel_rows, int n_wgs) {
    args_t* const a = fresh_args();
    const int b = blockIdx.x / args.Hkv, hkv = blockIdx.x - b * args.Hkv, grp = args.Hq / args.Hkv;
    const int2 ranges = reinterpret_cast<const int2*>(args.ranges)[b];  // (of a sequence that has none, anything: not looked at)
    const Sequence seq(a, b);
    const int r = blockIdx.y, token = r / grp;
    if (r >= seq.n_new * grp || seq.n_new * grp > args.few || ranges.y == 1) return;
    if (ranges.x < 0 || ranges.y < 1 || ((int64_t)ranges.x + ranges.y) * args.Hkv > n_wgs) return;  // not in the workspace
    const size_t at = ((size_t)ranges.x * args.Hkv + (size_t)hkv * ranges.y) * kernel_rows + (size_t)r * ranges.y, total = (size_t)n_wgs * kernel_rows;
    const Merged v = merge_splits(args.ws + total * kGroup + at * 2, args.ws + at * kGroup + threadIdx.x, ranges.y);
    store_out(a, ((size_t)(seq.row0 + token) * a->Hq + hkv * grp + r - token * grp) * kGroup + threadIdx.x, normalised(v.num, v.den));
}

// ---- many rows per key/value head ----------------------------------------------------------------------------------------
// Decoding a block costs as much as the products of its 128 values with a few hundred rows, so a sequence with more than kFewRows rows per
// key/value head (beside such ones, with more rows than a token has) is decoded once, into the workspace, and then read by all its rows.  What is
// written are the operands of
// v_mfma_f32_32x32x16_f16 in the order in which its lanes take them, a unit of 32 tokens at a time (16 KB):
//   K   A operands of S[token][row] = sum_dim K[token][dim] q[row][dim]: eight of 1 KB, the s-th for dimensions 16 s .. + 15; lane l takes token
//       l % 32 and the eight dimensions from 16 s + 8 (l / 32) on
//   V   A operands of O[dim][row] = sum_token V[token][dim] P[token][row]: the (2 d + s)-th for dimensions 32 d .. + 31 and tokens 16 s .. + 15; lane
//       l takes dimension 32 d + l % 32 and the tokens 16 s + 4 (l / 32) + (0 1 2 3 8 9 10 11): those whose scores the lane holds after the
//       first product, so that probabilities become B operands where they are
// so a unit is copied to LDS as it is, and read from there without bank conflicts.

// Where sequences lie in the workspace and in the launch: running sums over the sequences
struct Layout {
    int32_t* unit_start;  // [B + 1] units of 32 tokens of the sequences with many rows
    int32_t* tile_start;  // [B + 1] tiles of rows
    uint32_t* seen;       // [units] a bit per token: whether there is one, on a page of the pool
    uint4* operands;      // unit u of sequence b and head h at ((unit_start[b] * Hkv + h * units of b) + u) * kUnitBytes
    float* partial;       // of the splits
    int units, tiles;     // how many the workspace and the launch hold
};
struct TileArgs : PagedArgs {
    Layout lay;
    int tile_rows, splits;
    int layout;  // whether attend_expand_kernel finds the layout by itself
};

// What sequence 64 c + l of a batch takes, for lane l: units of 32 tokens in the workspace, tiles of rows.  Nothing if it has few rows.
struct Takes {
    int units, tiles;
    Sequence seq;
    __device__ __forceinline__ Takes(const TileArgs& a, int c, int lane) : units(0), tiles(0) {
        const int b = 64 * c + lane;
        seq = Sequence((args_t*)__builtin_amdgcn_kernarg_segment_ptr(), min(b, a.B - 1));
        const int rows = seq.n_new * (a.Hq / a.Hkv);
        if (b >= a.B || rows <= a.few) return;
        units = seq.kv > 0 ? units_of(seq.kv) : 0;
        tiles = (rows - 1) / a.tile_rows + 1;
    }
};
// One wavefront, 64 sequences at a time.  What does not fit the workspace or the launch, by lengths that the host did not announce, gets no tiles,
// nor does anything behind it.
__global__ __launch_bounds__(64) void attend_layout_kernel(TileArgs a) {
    const int lane = threadIdx.x;
    int units = 0, tiles = 0;
    if (lane == 0) a.lay.unit_start[0] = a.lay.tile_start[0] = 0;
    for (int c = 0; c * 64 < a.B; ++c) {
        const Takes takes(a, c, lane);
        int64_t end_u = takes.units, end_t = takes.tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t ou = __shfl_up(end_u, d), ot = __shfl_up(end_t, d);
            end_u += lane >= d ? ou : 0;
            end_t += lane >= d ? ot : 0;
        }
        const bool fits = units + end_u <= a.lay.units && tiles + end_t <= a.lay.tiles;
        // those that fit are the first ones: sums do not fall
        const uint64_t good = __ballot(fits);
        const int last = good == ~0ull ? 63 : __builtin_ctzll(~good) - 1;
        const int64_t cap_u = last < 0 ? 0 : __shfl(end_u, max(last, 0)), cap_t = last < 0 ? 0 : __shfl(end_t, max(last, 0));
        if (64 * c + lane < a.B) {
            a.lay.unit_start[64 * c + lane + 1] = units + (int)(fits ? end_u : cap_u);
            a.lay.tile_start[64 * c + lane + 1] = tiles + (int)(fits ? end_t : cap_t);
        }
        units += (int)cap_u;
        tiles += (int)cap_t;
        if (last < 63) a.lay.units = a.lay.tiles = -1;
    }
}
// The same for up to 64 sequences and sums that an int holds, by any wavefront for itself: the kernel that decodes needs no launch before it then.
constexpr int kLayoutMost = 1 << 24;  // units, and tiles
struct Layout64 {
    int units, end;  // of lane's sequence, and up to and including it
    Sequence seq;
    __device__ __forceinline__ Layout64(const TileArgs& a, int lane, bool write) {
        const Takes takes(a, 0, lane);
        seq = takes.seq;
        const int end_u = wave_scan(min(takes.units, kLayoutMost), lane), end_t = wave_scan(min(takes.tiles, kLayoutMost), lane);
        const uint64_t good = __ballot(end_u <= a.lay.units && end_t <= a.lay.tiles);
        const int last = good == ~0ull ? 63 : __builtin_ctzll(~good) - 1;
        const int cap_u = last < 0 ? 0 : __builtin_amdgcn_readlane(end_u, max(last, 0)), cap_t = last < 0 ? 0 : __builtin_amdgcn_readlane(end_t, max(last, 0));
        units = lane <= last ? takes.units : 0;
        end = lane <= last ? end_u : cap_u;
        if (!write) return;
        if (lane == 0) a.lay.unit_start[0] = a.lay.tile_start[0] = 0;
        if (lane < a.B) {
            a.lay.unit_start[lane + 1] = end;
            a.lay.tile_start[lane + 1] = lane <= last ? end_t : cap_t;
        }
    }
};
// the sequence that place v of the running sums lies in: the last one that starts at v or before it (and is not empty)
__device__ __forceinline__ int place_of(const int32_t* start, int B, int v) {
    int lo = 0;
    for (int step = 1 << (31 - __builtin_clz(B)); step > 0; step >>= 1)
        if (lo + step <= B && start[lo + step] <= v) lo += step;
    return lo;
}

// Decodes units into operands: grid (workgroups, 2), keys and values.  Lane l decodes chain l / 32 of token l % 32; eight decoded key values are sixteen
// bytes of an operand as they are, values pass through a tile of 16 dimensions in LDS, where tokens become neighbours.  8192 tokens, 8 heads, 64
// patterns: 14.7 to 15.6 us, 8.4 to 8.9 blocks per ns; 33.5 MB are written.
constexpr int kExpandWaves = 16;
constexpr int kTurnStride = 20;  // words per dimension of the tile in which values are turned
constexpr size_t expand_lds_bytes(int S) { return (table_words(S) + (size_t)kExpandWaves * (kUnitWords + 16 * kTurnStride)) * 4; }

template <bool kLong, bool kValues>
__device__ __forceinline__ void expand(const TileArgs& a) {
    extern __shared__ __align__(16) uint32_t smem[];
    const int S = kValues ? a.Sv : a.Sk;
    const uint32_t* dev = kValues ? a.dev_v : a.dev_k;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tok = lane & 31, half = lane >> 5;
    uint32_t* wbuf = smem + table_words(S) + wave * (kUnitWords + 16 * kTurnStride);
    uint32_t* tile = wbuf + kUnitWords;
    if (lane < kUnitBlocks) wbuf[lane * kStride + kBlockWords] = 0u;
    const TableItems items = load_table_items(dev, S);
    const Layout64 own(a, lane, a.layout && !kValues && blockIdx.x == 0 && wave == 0);
    build_tables<kLong>(smem, dev, S, items);
    const Tables T = table_pointers(smem, S);
    __syncthreads();
    const int64_t total = (int64_t)(a.layout ? __builtin_amdgcn_readlane(own.end, 63) : a.lay.unit_start[a.B]) * a.Hkv, waves = (int64_t)gridDim.x * kExpandWaves;
    for (int64_t item = (int64_t)blockIdx.x * kExpandWaves + wave; item < total; item += waves) {
        const int place = (int)(item / a.Hkv);
        int b, first, units, kv;
        if (a.layout) {
            b = (int)__builtin_ctzll(__ballot(own.end > place));  // (place is below the last sum)
            units = __builtin_amdgcn_readlane(own.units, b);
            first = __builtin_amdgcn_readlane(own.end, b) - units;
            kv = __builtin_amdgcn_readlane(own.seq.kv, b);
        } else {
            b = __builtin_amdgcn_readfirstlane(place_of(a.lay.unit_start, a.B, place));
            first = a.lay.unit_start[b];
            units = a.lay.unit_start[b + 1] - first;
            kv = Sequence((args_t*)__builtin_amdgcn_kernarg_segment_ptr(), b).kv;
        }
        const int at = (int)(item - (int64_t)first * a.Hkv), hkv = at / units, u = at - hkv * units, t0 = u * kUnitBlocks;
        const UnitPages pages = unit_pages(b, t0, kv - 1);
        bool ok;
        const UnitLoad pre = load_unit<kValues>(pages, hkv, t0, lane, tok, ok);
        const bool there = ok && t0 + tok < kv;
        const uint32_t mw = there ? pre.meta : 0u;
        if (!kValues && hkv == 0) {
            const uint64_t m = __ballot(there);
            if (lane == 0) a.lay.seen[first + u] = (uint32_t)m;
        }
        store_unit(wbuf, pre, lane);
        const Lane L = lane_setup(T, mw, S);
        const _Float16 sh16 = __builtin_bit_cast(_Float16, (unsigned short)(mw & 0xFFFFu));
        const half2_t s2 = {sh16, sh16};
        uint4* out = a.lay.operands + item * (kUnitBytes / 16) + (kValues ? kUnitBytes / 32 : 0);
        uint32_t pk[4];
        const uint32_t swap_sel = (lane & 1) ? 0x03020706u : 0x05040100u;
        const int pair = tok >> 1, word = (pair & 8) | ((pair >> 1) & 1) << 2 | ((pair >> 2) & 1) << 1 | (pair & 1);  // tokens in the operand's order
        decode_chain<kLong, kHalf>(wbuf + tok * kStride, half ? L.second_start : 0u, L, [&](int i, uint32_t e) {
            if ((i & 1) == 0) {
                pk[(i >> 1) & 3] = e >> 16;
                return;
            }
            pk[(i >> 1) & 3] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2_t, pk[(i >> 1) & 3] | (e & 0xFFFF0000u)) * s2);
            if ((i & 7) != 7) return;
            const int j = i >> 3;  // dimensions 64 half + 8 j .. + 7
            if (!kValues) {
                out[(half * 4 + (j >> 1)) * 64 + (j & 1) * 32 + tok] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
            } else {
                wave_lds_fence();
#pragma unroll
                for (int r2 = 0; r2 < 4; ++r2) {
                    const uint32_t mate = (uint32_t)__builtin_amdgcn_mov_dpp((int)pk[r2], 0xB1, 0xF, 0xF, true);  // quad_perm [1,0,3,2]
                    tile[(8 * half + 2 * r2 + (lane & 1)) * kTurnStride + word] = __builtin_amdgcn_perm(mate, pk[r2], swap_sel);
                }
                wave_lds_fence();
                const int r = lane & 15, part = lane >> 4;  // dimension 64 (r / 8) + 8 j + r % 8, tokens of step part / 2 and lane half part % 2
                const uint4 v = *reinterpret_cast<const uint4*>(tile + r * kTurnStride + 4 * part);
                const int d = 64 * (r >> 3) + 8 * j + (r & 7);
                out[((d >> 5) * 2 + (part >> 1)) * 64 + (part & 1) * 32 + (d & 31)] = v;
            }
        });
    }
}
template <bool kLongK, bool kLongV>
__global__ __launch_bounds__(kExpandWaves * 64) void attend_expand_kernel(TileArgs a) {
    if (blockIdx.y == 0) expand<kLongK, false>(a);
    else expand<kLongV, true>(a);
}

// The products: a workgroup takes a tile of rows of one sequence and key/value head, a wavefront 32 of them, over a range of the sequence's tokens, two
// units at a time.  The scores of a pair of units, 32 per lane and all of one row, become probabilities and the next product's operand where they are;
// they are relative to `most`, which follows a row's largest score only when that is ahead by more than 2^kAhead, so that the sums are rescaled a
// few times per row instead of once per pair, and the score `most` has the weight 2^(kWeightTop - kAhead), so that weights reach FP16's top and the
// smallest ones keep their bits: the second number of a pair, or the first one alone, is whole down to 2^-25 of that weight and off by 2^-36 of it at
// the most below.  (kAhead 8, 4, 2, 0: a 4096-token chunk over 8192 416.9, 421.4, 425.2, 431.7 us; 414.8 with 8 and the weight 1, which lost
// the tokens far behind a leading one.)  For FP32 outputs what an FP16 probability leaves of the
// FP32 one goes through a product of its own (the error against 64 bits 1.1e-6 in a step of two 450-token chunks over 4096); for FP16 outputs it is left out: half a step of a
// weight, at random, adds 19 % to the error that the outputs' own rounding makes (2.5e-4 for 2.1e-4), and without it the chunk above takes 441 us
// instead of 572.
// What bounds it: a 4096-token chunk over 8192, 32/8 heads, FP16 outputs, 408 to 411 us for 412 GFLOP; in a run of 434 us the matrix cores were busy 53 % of
// the time at 1.85 GHz.  Power holds the clock there: with zeros for queries and values the whole call took 347 us beside 439, and the library's
// product of 8192^3 reaches 1.16 PFLOP/s with random values and 1.72 with zeros.  Two wavefronts of a SIMD held in opposite phases by barriers:
// 501 us beside 422; exponentials left out, for the measurement alone: the call 401 us beside 433.
constexpr float kScoreToExp2 = 0.08838834764831845f * 1.4426950408889634f;  // log2(e) / sqrt(128)

// the larger of the two lanes' values that hold a row's scores, l and l + 32
__device__ __forceinline__ float halves_max(float v) {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// Eight wavefronts, 32 rows each, in kGroups groups that each take every kGroups-th pair of units for the tile's rows and add up at the end: what one
// wavefront of a SIMD waits for, the other one covers, and a workgroup of two groups has half the rows to find work for.
constexpr int kTileWaves = 8;
// two pairs of units per group; at the end 66 words per lane of the second group, and 32 x 68 words per wavefront with rows
constexpr size_t tiles_lds_bytes(int groups) { return groups == 1 ? 8 * 32 * 68 * 4 : (size_t)groups * 4 * kUnitBytes; }
static_assert(tiles_lds_bytes(1) >= 4 * kUnitBytes && tiles_lds_bytes(2) >= 4 * (66 * 64 + 32 * 68) * 4, "room for either");
template <int kGroups, bool kRest>
__global__ __launch_bounds__(kTileWaves * 64) __attribute__((amdgpu_waves_per_eu(2, 2))) void attend_tiles_kernel(TileArgs a) {
    constexpr int kPair = 2 * kUnitBytes / 16;            // sixteen-byte pieces of two units
    constexpr int kThreads = kTileWaves * 64 / kGroups;   // of a group
    constexpr int kPieces = kPair / kThreads;             // per thread
    extern __shared__ __align__(16) uint32_t smem[];
    const int tid = threadIdx.x % kThreads, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), group = kGroups == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads);
    u32x4* const lds = reinterpret_cast<u32x4*>(smem) + group * 2 * kPair;
    const int grp = a.Hq / a.Hkv, hkv = blockIdx.x % a.Hkv, split = blockIdx.y;
    const int tiles = a.lay.tile_start[a.B], at = tiles - 1 - (int)(blockIdx.x / a.Hkv);  // the last tiles have the most tokens: first
    if (at < 0) return;
    const int b = __builtin_amdgcn_readfirstlane(place_of(a.lay.tile_start, a.B, at));
    const Sequence seq((args_t*)__builtin_amdgcn_kernarg_segment_ptr(), b);
    const int row_begin = (at - a.lay.tile_start[b]) * a.tile_rows, rows = min(a.tile_rows, seq.n_new * grp - row_begin);
    const int unit0 = a.lay.unit_start[b], units_b = a.lay.unit_start[b + 1] - unit0;
    const int T = max(0, seq.kv - seq.n_new + (row_begin + rows - 1) / grp + 1);  // what the last row sees
    const int units = T > 0 ? units_of(T) : 0, per = ((units + 1) / 2 + a.splits - 1) / a.splits * 2;
    const int u_begin = min(units, split * per), u_end = min(units, u_begin + per);
    const u32x4* src = reinterpret_cast<const u32x4*>(a.lay.operands) + ((int64_t)unit0 * a.Hkv + (int64_t)hkv * units_b) * (kUnitBytes / 16);
    const uint32_t* seen = a.lay.seen + unit0;

    const int r = row_begin + min(wave * 32 + n, rows - 1), token = r / grp, head = hkv * grp + r - token * grp;
    const int sees = min(seq.kv - seq.n_new + token + 1, u_end * kUnitBlocks);
    half8_t q[8];
    {
        const uint4* from = reinterpret_cast<const uint4*>(a.q + (int64_t)(seq.row0 + token) * a.q_stride + head * kGroup) + h;
#pragma unroll
        for (int s = 0; s < 8; ++s) q[s] = __builtin_bit_cast(half8_t, from[2 * s]);
    }
    // units in front of which every row of the wavefront sees every token (rows are in the order of their tokens: the first sees the least)
    const int whole = __builtin_amdgcn_readfirstlane(max(sees, 0)) / kUnitBlocks;
    float16_t o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] = float16_t{};
    float most = -INFINITY, den = 0.0f;
    u32x4 piece[kPieces];
    uint32_t seen0, seen1;
    const auto load = [&](int u) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int unit = u + i * kThreads / (kPair / 2);
            piece[i] = src[(int64_t)min(unit, units - 1) * (kUnitBytes / 16) + i * kThreads % (kPair / 2) + tid];
        }
        seen0 = seen[min(u, units - 1)];
        seen1 = seen[min(u + 1, units - 1)];
    };
    const auto keep = [&](int which) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) lds[which * kPair + i * kThreads + tid] = piece[i];
    };
    static_assert(kThreads <= kPair / 2, "a round of the threads stays inside a unit");
    if (u_begin < u_end) {
        load(u_begin + 2 * group);
        keep(0);
    }
    constexpr float kAhead = 4.0f;
    float minus = -1.0f;
    if constexpr (kRest) asm volatile("" : "+v"(minus));
    int which = 0;
    for (int u0 = u_begin; u0 < u_end; u0 += 2 * kGroups, which ^= 1) {
        const int u = u0 + 2 * group;  // (a group may have nothing left in the last round)
        const uint32_t there0 = seen0, there1 = seen1;
        __syncthreads();
        const half8_t* op = reinterpret_cast<const half8_t*>(lds + which * kPair) + lane;
        float16_t s[2];
#pragma unroll
        for (int k = 0; k < 8; ++k)
#pragma unroll
            for (int w = 0; w < 2; ++w) s[w] = __builtin_amdgcn_mfma_f32_32x32x16_f16(op[w * (kPair / 2) + k * 64], q[k], k == 0 ? float16_t{} : s[w], 0, 0, 0);
        // six operands ahead of the products
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int k = 0; k < 10; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
        load(u + 2 * kGroups);
        if (u + 2 > whole || (__builtin_amdgcn_readfirstlane(there0) & __builtin_amdgcn_readfirstlane(there1)) != ~0u) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const int left = sees - (u + w) * kUnitBlocks;
                const uint32_t there = w ? there1 : there0;
                const uint32_t bits = (left >= 32 ? there : left <= 0 ? 0u : there & ((1u << left) - 1u)) >> (4 * h);
#pragma unroll
                for (int i = 0; i < 16; ++i) s[w][i] = (bits >> (8 * (i / 4) + i % 4)) & 1u ? s[w][i] : -INFINITY;
            }
        }
        float mx = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) mx = fmaxf(fmaxf(mx, s[0][i]), s[1][i]);
        mx = halves_max(mx);
        if (__ballot(mx > most + kAhead / kScoreToExp2) != 0ull) {
            const float now = fmaxf(most, mx), alpha = most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((most - now) * kScoreToExp2);
            most = now;
            den *= alpha;
#pragma unroll
            for (int d = 0; d < 4; ++d) o[d] *= alpha;
        }
        const float base = most == -INFINITY ? 0.0f : fmaf(most, kScoreToExp2, kAhead - kWeightTop);
        half8_t p[4], rest[4];
        const auto weight = [&](int i) { return __builtin_amdgcn_exp2f(fmaf(s[i / 16][i % 16], kScoreToExp2, -base)); };
        if constexpr (kRest) {
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                typedef float float2_t __attribute__((ext_vector_type(2)));
                const float2_t e = {weight(i), weight(i + 1)};
                den += e[0];
                den += e[1];
                const half2_t rounded = __builtin_convertvector(e, half2_t);
                // (the factor in a register: a product with a constant -1 becomes two conversions and a subtraction)
                const half2_t left = __builtin_convertvector(float2_t{fmaf((float)rounded[0], minus, e[0]), fmaf((float)rounded[1], minus, e[1])}, half2_t);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    p[i / 8][i % 8 + j] = rounded[j];
                    rest[i / 8][i % 8 + j] = left[j];
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float e = weight(i);
                den += e;
                p[i / 8][i % 8] = (_Float16)e;
            }
        }
        keep(which ^ 1);  // (here, and requested behind the first product: between the products they pass unnoticed)
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const half8_t v = op[(k / 2) * (kPair / 2) + kPair / 4 + (2 * d + k % 2) * 64];
                o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[k], o[d], 0, 0, 0);
                if (kRest) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, rest[k], o[d], 0, 0, 0);
            }
    }
    if constexpr (kGroups == 2) {  // the second group's sums to the first
        float* const to = reinterpret_cast<float*>(smem) + wave * 66 * 64 + lane;
        __syncthreads();
        if (group == 1) {
            to[0] = most;
            to[64] = den;
#pragma unroll
            for (int i = 0; i < 64; ++i) to[(2 + i) * 64] = o[i / 16][i % 16];
        }
        __syncthreads();
        if (group == 1) return;
        const float other = to[0], now = fmaxf(most, other);
        const float mine = most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((most - now) * kScoreToExp2);
        const float theirs = other == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((other - now) * kScoreToExp2);
        most = now;
        den = den * mine + to[64] * theirs;
#pragma unroll
        for (int i = 0; i < 64; ++i) o[i / 16][i % 16] = o[i / 16][i % 16] * mine + to[(2 + i) * 64] * theirs;
    }
    // The lane holds dimensions 32 d + 8 (i / 4) + 4 h + i % 4 of its row: 64 dimensions at a time the wavefront's rows pass through LDS, so that sixteen
    // lanes store 64 neighbouring values.
    den += __shfl_xor(den, 32);
    const float scale = a.splits > 1 ? 1.0f : den > 0.0f ? 1.0f / den : 0.0f;
    const size_t part = (((size_t)at * a.Hkv + hkv) * a.tile_rows + wave * 32) * a.splits + split, all = (size_t)tiles * a.Hkv * a.tile_rows * a.splits;
    if (a.splits > 1 && h == 0 && wave * 32 + n < rows) {
        float* ml = a.lay.partial + all * kGroup + (part + (size_t)n * a.splits) * 2;
        ml[0] = most * 0.08838834764831845f;
        ml[1] = den;
    }
    constexpr int kTurnRow = 68;  // words of a row's 64 values
    if constexpr (kGroups == 1) __syncthreads();  // the last units have been read
    float* const turn = reinterpret_cast<float*>(smem) + (kGroups == 2 ? kTileWaves / 2 * 66 * 64 : 0) + wave * 32 * kTurnRow;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        wave_lds_fence();
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float16_t& v = o[2 * half + d];
                *reinterpret_cast<float4_t*>(turn + n * kTurnRow + 32 * d + 8 * i + 4 * h) = float4_t{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]} * scale;
            }
        wave_lds_fence();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = 4 * i + (lane >> 4), dim = 4 * (lane & 15);
            const float4_t v = *reinterpret_cast<const float4_t*>(turn + row * kTurnRow + dim);
            const int r = row_begin + wave * 32 + row, token = r / grp;
            if (wave * 32 + row >= rows) continue;
            const size_t to = ((size_t)(seq.row0 + token) * a.Hq + hkv * grp + r - token * grp) * kGroup + 64 * half + dim;
            if (a.splits > 1) {
                *reinterpret_cast<float4_t*>(a.lay.partial + (part + (size_t)row * a.splits) * kGroup + 64 * half + dim) = v;
            } else if (kRest) {
                *reinterpret_cast<float4_t*>(static_cast<float*>(a.out) + to) = v;
            } else {
                typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
                *reinterpret_cast<half4_t*>(static_cast<_Float16*>(a.out) + to) = half4_t{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
            }
        }
    }
}

// merges the token ranges of rows: grid (tiles that there may be * Hkv, sets of 32 rows), 32 threads a row
constexpr int kMergeThreads = 256, kMergeRows = 32;
__global__ __launch_bounds__(kMergeThreads) void attend_tiles_merge_kernel(TileArgs a) {
    const int tiles = a.lay.tile_start[a.B], at = blockIdx.x / a.Hkv, hkv = blockIdx.x - at * a.Hkv, grp = a.Hq / a.Hkv, n = a.splits;
    if (at >= tiles) return;
    const int b = place_of(a.lay.tile_start, a.B, at);
    const Sequence seq((args_t*)__builtin_amdgcn_kernarg_segment_ptr(), b);
    const size_t first = ((size_t)at * a.Hkv + hkv) * a.tile_rows, all = (size_t)tiles * a.Hkv * a.tile_rows * n;
    const int row_begin = (at - a.lay.tile_start[b]) * a.tile_rows, rows = min(a.tile_rows, seq.n_new * grp - row_begin), dim = 4 * (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < kMergeRows * 32 / kMergeThreads; ++i) {
        const int row = blockIdx.y * kMergeRows + i * (kMergeThreads / 32) + (threadIdx.x >> 5);
        if (row >= rows) continue;
        const float* ml = a.lay.partial + (all * kGroup) + (first + row) * n * 2;
        const float* part = a.lay.partial + (first + row) * n * kGroup + dim;
        float mx = -INFINITY, den = 0.0f;
        for (int s = 0; s < n; ++s) mx = fmaxf(mx, ml[2 * s]);
        float4_t num = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
        for (int s = 0; s < n; ++s) {
            const float w = ml[2 * s] == -INFINITY ? 0.0f : __expf(ml[2 * s] - mx);
            num += w * *reinterpret_cast<const float4_t*>(part + (size_t)s * kGroup);
            den += w * ml[2 * s + 1];
        }
        num *= den > 0.0f ? 1.0f / den : 0.0f;
        const int r = row_begin + row, token = r / grp;
        const size_t to = ((size_t)(seq.row0 + token) * a.Hq + hkv * grp + r - token * grp) * kGroup + dim;
        if (a.half) {
            typedef _Float16 half4_t __attribute__((ext_vector_type(4)));
            *reinterpret_cast<half4_t*>(static_cast<_Float16*>(a.out) + to) = half4_t{(_Float16)num[0], (_Float16)num[1], (_Float16)num[2], (_Float16)num[3]};
        } else {
            *reinterpret_cast<float4_t*>(static_cast<float*>(a.out) + to) = num;
        }
    }
}

// ---- host side -----------------------------------------------------------------------------------------------------------
// (a step without rows may have nothing else either)
bool sizes_fit(int n_tokens, int B, int Hq, int Hkv, int max_new, int max_kv, int64_t total_kv) {
    const int least = n_tokens == 0 ? 0 : 1;
    return n_tokens >= 0 && B >= least && Hq > 0 && Hkv > 0 && Hq % Hkv == 0 && Hq / Hkv <= kGqaMaxGroup && max_new >= least && max_kv >= least && total_kv >= least &&
           (long long)B * Hkv <= 0x7FFFFFFF && (long long)n_tokens * Hq <= 0x7FFFFFFF;
}

}  // namespace

extern "C" {

size_t ecco_kv_attend_paged_workspace(int device, int n_tokens, int B, int Hq, int Hkv, int max_new, int max_kv, int64_t total_kv) {
    if (n_tokens == 0 || !sizes_fit(n_tokens, B, Hq, Hkv, max_new, max_kv, total_kv)) return 0;
    return paged_workspace(n_tokens, B, Hq, Hkv, max_new, max_kv, total_kv, cu_count(device));
}

int ecco_kv_attend_paged(const ecco_model* mk, const ecco_model* mv, const uint16_t* q, int64_t q_stride,
                         const void* k_blocks, const uint32_t* k_meta, const void* v_blocks, const uint32_t* v_meta,
                         const int32_t* page_table, const int32_t* q_start, const int32_t* kv_len,
                         int n_tokens, int B, int Hq, int Hkv, int n_pages, int page_tokens, int max_pages,
                         int max_new, int max_kv, int64_t total_kv, void* workspace, size_t workspace_bytes,
                         void* out, int out_half, void* stream) {
    if (!mk || !mv) return ECCO_EINVAL;
    if (n_tokens != 0 && (!q || !k_blocks || !k_meta || !v_blocks || !v_meta || !page_table || !q_start || !kv_len || !out)) return ECCO_EINVAL;
    if (out_half != 0 && out_half != 1) return ECCO_EINVAL;
    if (!sizes_fit(n_tokens, B, Hq, Hkv, max_new, max_kv, total_kv) || !pool_fits(page_tokens, n_pages) || !pool_fits(page_tokens, max_pages)) return ECCO_ESHAPE;
    if (q_stride < (int64_t)Hq * kGroup || q_stride % 8 != 0 || q_stride > ((int64_t)1 << 40)) return ECCO_ESHAPE;
    if (!aligned(k_blocks, 64) || !aligned(v_blocks, 64) || !aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 256)) return ECCO_EALIGN;
    for (const void* p : {(const void*)k_meta, (const void*)v_meta, (const void*)page_table, (const void*)q_start, (const void*)kv_len})
        if (!aligned(p, 4)) return ECCO_EALIGN;
    if (model_ready(mk) != ECCO_OK || model_ready(mv) != ECCO_OK || mk->device != mv->device) return ECCO_EINVAL;
    if (n_tokens == 0) return ECCO_OK;
    const int dev_id = mk->device, cus = cu_count(dev_id), shift = __builtin_ctz((unsigned)page_tokens);
    const PagedPlan plan = paged_plan(n_tokens, B, Hq, Hkv, max_new, max_kv, total_kv, cus);
    const size_t bytes = paged_workspace(n_tokens, B, Hq, Hkv, max_new, max_kv, total_kv, cus);
    if (bytes > 0 && (!workspace || workspace_bytes < bytes)) return ECCO_EINVAL;
    const bool lk = mk->max_len > kPeekBits, lv = mv->max_len > kPeekBits;
    max_kv = std::min(max_kv, max_pages << shift);
    hipStream_t st = static_cast<hipStream_t>(stream);
    PagedArgs args{mk->dev, mv->dev, q, static_cast<const uint4*>(k_blocks), k_meta, static_cast<const uint4*>(v_blocks), v_meta, page_table, q_start, kv_len,
                   out, reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up((size_t)B * 8)), static_cast<int32_t*>(workspace), q_stride, mk->S, mv->S, B, Hq, Hkv, n_tokens, n_pages, shift, max_pages, max_kv,
                   0, 0, 0, 0, out_half, plan.few, plan.cut, 0};
    if (plan.wide_tiles > 0) {
        char* at = static_cast<char*>(workspace) + plan.few_bytes;
        const auto part = [&](size_t bytes) {
            char* p = at;
            at += round_up(bytes);
            return p;
        };
        TileArgs t{args, {}, plan.tile_rows, plan.wide_splits, B <= 64 && plan.wide_units < kLayoutMost && plan.wide_tiles < kLayoutMost};
        t.lay.unit_start = reinterpret_cast<int32_t*>(part(((size_t)B + 1) * 4));
        t.lay.tile_start = reinterpret_cast<int32_t*>(part(((size_t)B + 1) * 4));
        t.lay.seen = reinterpret_cast<uint32_t*>(part((size_t)plan.wide_units * 4));
        t.lay.operands = reinterpret_cast<uint4*>(part((size_t)plan.wide_units * Hkv * kUnitBytes));
        t.lay.partial = reinterpret_cast<float*>(at);
        t.lay.units = plan.wide_units;
        t.lay.tiles = plan.wide_tiles;
        if (!t.layout) {
            hipLaunchKernelGGL(attend_layout_kernel, dim3(1), dim3(64), 0, st, t);
            ECCO_HIP_CHECK(hipGetLastError());
        }
        const auto expand = [&](auto kernel) -> int {
            const size_t lds = expand_lds_bytes(std::max(mk->S, mv->S));
            const int rc = allow_lds(kernel, dev_id, lds);
            if (rc != ECCO_OK) return rc;
            const long long wgs = ((long long)plan.wide_units * Hkv + kExpandWaves - 1) / kExpandWaves;
            hipLaunchKernelGGL(kernel, dim3((unsigned)std::max<long long>(1, std::min<long long>(wgs, cus / 2)), 2), dim3(kExpandWaves * 64), lds, st, t);
            ECCO_HIP_CHECK(hipGetLastError());
            return ECCO_OK;
        };
        int rc = lk ? (lv ? expand(attend_expand_kernel<true, true>) : expand(attend_expand_kernel<true, false>))
                    : (lv ? expand(attend_expand_kernel<false, true>) : expand(attend_expand_kernel<false, false>));
        if (rc != ECCO_OK) return rc;
        const dim3 grid((unsigned)plan.wide_tiles * Hkv, plan.wide_splits);
        const auto products = [&](auto kernel, int groups) -> int {
            const int rc = allow_lds(kernel, dev_id, tiles_lds_bytes(groups));
            if (rc != ECCO_OK) return rc;
            hipLaunchKernelGGL(kernel, grid, dim3(kTileWaves * 64), tiles_lds_bytes(groups), st, t);
            return ECCO_OK;
        };
        if (plan.tile_rows == 256) rc = out_half ? products(attend_tiles_kernel<1, false>, 1) : products(attend_tiles_kernel<1, true>, 1);
        else rc = out_half ? products(attend_tiles_kernel<2, false>, 2) : products(attend_tiles_kernel<2, true>, 2);
        if (rc != ECCO_OK) return rc;
        ECCO_HIP_CHECK(hipGetLastError());
        if (plan.wide_splits > 1) {
            hipLaunchKernelGGL(attend_tiles_merge_kernel, dim3((unsigned)plan.wide_tiles * Hkv, plan.tile_rows / kMergeRows), dim3(kMergeThreads), 0, st, t);
            ECCO_HIP_CHECK(hipGetLastError());
        }
    }
    if (plan.few == 0) return ECCO_OK;
    // ranges for as many workgroups as find a place at once
    args.cus = rows_can_share(mk->S, lk, mv->S, lv, plan.few) ? 2 * cus : cus;
    const int wgs = B * Hkv + (plan.cut ? args.cus : 0);
    const int units = plan.cut ? (int)std::min<long long>(plan.units, std::max<long long>(kRangeLeast, ((long long)plan.units * B * Hkv + args.cus - 1) / args.cus)) : plan.units;
    const GqaPlan g = rows_plan(mk->S, lk, mv->S, lv, plan.few, (size_t)wgs, units, cus, plan.cut);
    args.table_words = g.table_words;
    args.both = g.both;
    args.span = g.span;
    args.step = g.step;
    const auto launch = [&](auto kernel) -> int {
        const int rc = allow_lds(kernel, dev_id, g.lds);
        if (rc != ECCO_OK) return rc;
        hipLaunchKernelGGL(kernel, dim3(wgs), dim3(g.waves * 64), g.lds, st, args);
        ECCO_HIP_CHECK(hipGetLastError());
        return ECCO_OK;
    };
    const auto pick = [&](auto row_tag) -> int {
        constexpr int kRows = decltype(row_tag)::value;
        constexpr int kLongWaves = kRows == kFewRows ? 8 : 12;
        if (lk) return lv ? launch(attend_rows_kernel<true, true, kRows, kLongWaves>) : launch(attend_rows_kernel<true, false, kRows, kLongWaves>);
        if (lv) return launch(attend_rows_kernel<false, true, kRows, kLongWaves>);
        if constexpr (kRows <= 16)
            if (g.waves == 8) return launch(attend_rows_kernel<false, false, kRows, 8>);
        return launch(attend_rows_kernel<false, false, kRows, 12>);
    };
    const int rc = plan.few_rows == 8 ? pick(std::integral_constant<int, 8>{}) : plan.few_rows == 16 ? pick(std::integral_constant<int, 16>{}) : pick(std::integral_constant<int, kFewRows>{});
    if (rc != ECCO_OK || !plan.cut) return rc;
    hipLaunchKernelGGL(attend_rows_merge_kernel, dim3(B * Hkv, plan.few), dim3(kGroup), 0, st, args, plan.few_rows, wgs);
    ECCO_HIP_CHECK(hipGetLastError());
    return ECCO_OK;
}

}  // extern "C"

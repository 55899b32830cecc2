// Decoding a chain of the two-chain block format on the device: the tables in LDS, the chain decoder, the staging of payloads.
// Shared by the kernels that read contiguous blocks (ecco_kernels.hip) and pages (ecco_paged.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "ecco_internal.h"
#include "ecco_plan.h"

namespace ecco_chain {

using namespace ecco;

constexpr int kHalf = kGroup / 2;         // values per chain

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float half_bits_f(uint32_t bits) { return __half2float(__ushort_as_half((unsigned short)bits)); }

// orders the LDS accesses of one wavefront (private buffers need no workgroup barrier)
__device__ inline void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---- LDS tables -------------------------------------------------------------------------------------
struct Tables {
    const uint32_t* lut;      // [S][256]
    const uint32_t* rawlut;   // [S][16]
    const uint32_t* longtab;  // [S][16]
    const __half* cent;       // [S][16]
};
__host__ __device__ constexpr size_t table_words(int S) { return (size_t)S * (kPeekEntries + kK + kK + kK / 2); }  // LDS words of a model's decode tables

// copies `words` (a multiple of 4; both sides 16-byte aligned) from global memory to LDS with all
// threads of the workgroup, four 16-byte loads in flight per thread
__device__ inline void stage_vec(uint32_t* dst, const uint32_t* __restrict__ src, int words) {
    const uint4* s = reinterpret_cast<const uint4*>(src);
    uint4* d = reinterpret_cast<uint4*>(dst);
    const int n = words >> 2, step = blockDim.x;
    for (int i = threadIdx.x; i < n; i += 4 * step) {
        uint4 v0, v1, v2, v3;
        const int i1 = i + step, i2 = i + 2 * step, i3 = i + 3 * step;
        v0 = s[i];
        if (i1 < n) v1 = s[i1];
        if (i2 < n) v2 = s[i2];
        if (i3 < n) v3 = s[i3];
        d[i] = v0;
        if (i1 < n) d[i1] = v1;
        if (i2 < n) d[i2] = v2;
        if (i3 < n) d[i3] = v3;
    }
}

// The thread's index, taken afresh: in a kernel that stages tables in every span, what is derived from it is then formed there and
// does not take registers through the decode loops.
__device__ __forceinline__ int fresh_thread() {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    return tid;
}
// A model's size, likewise: what the staging of a model with long codes derives from it (masks, addresses) would otherwise be formed
// once for all spans and take scalar registers throughout
__device__ __forceinline__ int fresh_size(int S) {
    asm volatile("" : "+s"(S));
    return S;
}

// Building the decode tables of a model in LDS from the compact tables in global memory.  Item
// (p, k) is index k of pattern p: its code of length l <= 8 is the prefix of 2^(8-l) consecutive
// 8-bit peeks, which all get the entry (centroid, index, length); a longer code marks its single
// 8-bit prefix with 0.  The two global loads of an item are split from the LDS writes so that a
// kernel can issue them first, put its payload loads behind them, and build the tables while the
// payload is still on its way.
struct TableItem {
    uint32_t enc, cent;
};
__device__ __forceinline__ TableItem load_table_item(const uint32_t* __restrict__ dev, int S, int t) {
    const DevLayout D{S};
    TableItem it;
    it.enc = dev[D.enc() + t];
    it.cent = reinterpret_cast<const uint16_t*>(dev + D.cent())[t];
    return it;
}
__device__ __forceinline__ void build_table_item(uint32_t* base, int S, int t, TableItem it) {
    uint32_t* lut = base;
    uint32_t* rawlut = lut + S * kPeekEntries;
    const uint32_t code = it.enc & 0xFFFFu, len = it.enc >> 16, k = (uint32_t)t & (kK - 1);
    const uint32_t value = (it.cent << 16) | (k << 8);
    rawlut[t] = value | 4u;
    uint32_t* row = lut + (t / kK) * kPeekEntries;
    if (len > (uint32_t)kPeekBits) {
        row[code >> (len - kPeekBits)] = 0u;  // several long codes may share this prefix: same value
    } else {
        const uint32_t entry = value | len, n = 1u << (kPeekBits - len);
        uint32_t* dst = row + (code << (kPeekBits - len));
        if (n >= 4) {
            // neighbouring items start their runs at different offsets: all rows begin on the same LDS
            // bank and equal-length codes are a multiple of the run length apart, so without the
            // rotation the 64 items of a wavefront would write to a handful of banks at a time
            const uint4 v = make_uint4(entry, entry, entry, entry);
            const uint32_t rot = ((uint32_t)t + ((uint32_t)t >> 4) + (code >> 2)) * 4u;
            for (uint32_t j = 0; j < n; j += 4) *reinterpret_cast<uint4*>(dst + ((j + rot) & (n - 1))) = v;
        } else {
            for (uint32_t j = 0; j < n; ++j) dst[j] = entry;
        }
    }
}
__device__ __forceinline__ Tables table_pointers(uint32_t* base, int S) {
    Tables tb;
    tb.lut = base;
    tb.rawlut = base + S * kPeekEntries;
    tb.longtab = base + S * (kPeekEntries + kK);
    tb.cent = reinterpret_cast<const __half*>(base + S * (kPeekEntries + 2 * kK));
    return tb;
}
// The whole job for a workgroup of at least S * 16 / 2 threads, with a payload prefetch in its shadow: every
// thread first requests its (up to) two table items, then the loads of its first unit, then
// builds the tables.  Loads return in issue order and a wait names how many may still be outstanding, so with
// the items requested first -- the same loads on one straight path in every thread, indices clamped, threads
// beyond the items repeating the last one -- the build does not wait for the payload.  The lists of the long
// codes and the centroids are copied only for a model that needs them (behind the payload, then).  The caller
// synchronises afterwards.
struct TableItems {
    TableItem item[2];
};
__device__ __forceinline__ TableItems load_table_items(const uint32_t* __restrict__ dev, int S) {
    const int n = S * kK, tid = fresh_thread();
    TableItems t;
    t.item[0] = load_table_item(dev, S, min(tid, n - 1));
    t.item[1] = load_table_item(dev, S, min(tid + (int)blockDim.x, n - 1));
    __builtin_amdgcn_sched_barrier(0);
    return t;
}
template <bool kLong>
__device__ __forceinline__ void build_tables(uint32_t* base, const uint32_t* __restrict__ dev, int S, const TableItems& t) {
    __builtin_amdgcn_sched_barrier(0);
    const int n = S * kK, tid = fresh_thread();
    build_table_item(base, S, min(tid, n - 1), t.item[0]);
    build_table_item(base, S, min(tid + (int)blockDim.x, n - 1), t.item[1]);
    if (kLong) {
        const DevLayout D{S};
        stage_vec(base + S * (kPeekEntries + kK), dev + D.longtab(), S * kK);
        stage_vec(base + S * (kPeekEntries + 2 * kK), dev + D.cent(), S * kK / 2);
    }
}

// what one lane needs to decode one chain
struct Lane {
    const uint32_t* lut;      // this lane's table (Huffman: 256 entries, raw: 16)
    uint32_t shift;           // 32 - peek width
    const uint32_t* longtab;  // pattern's canonical list (codes longer than the peek)
    const __half* cent;       // pattern's centroids
    float scale;
    uint32_t second_start;    // stream bit where value 64 begins
};
__device__ __forceinline__ Lane lane_setup(const Tables& T, uint32_t meta, int S) {
    Lane L;
    uint32_t p = (meta >> 16) & 0x3Fu;
    p = p < (uint32_t)S ? p : (uint32_t)(S - 1);
    const bool raw = (meta >> 22) & 1u;
    L.lut = raw ? T.rawlut + p * kK : T.lut + p * kPeekEntries;
    L.shift = raw ? 28u : (uint32_t)(32 - kPeekBits);
    L.longtab = T.longtab + p * kK;
    L.cent = T.cent + p * kK;
    L.scale = half_bits_f(meta & 0xFFFFu);
    L.second_start = raw ? 4u * kHalf : (meta >> 23);
    return L;
}

typedef __attribute__((address_space(3))) uint32_t lds_u32;  // a 32-bit word in LDS, addressed as such
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) u32x4 global_u4;   // sixteen bytes in global memory

// Priority of a wavefront's instructions on its SIMD while it decodes (0 otherwise), in the batch-1 product and the plain attention:
// wavefronts that store and request units, add up or meet at barriers then do so in the gaps of the others' table reads.  8192 x 28672
// 64.9 -> 63.5 us, attention over 16 x 32 sequences and heads of 1000 tokens 66.3 -> 64.4 us (64 patterns), 48.1 -> 46.3 us (16).  The batched
// product (11008 x 4096, batch 8: 18.0 -> 18.5 us), the standalone decoder (131072 groups 12.65 -> 12.87 us) and the grouped-query
// attention (1024 tokens 20.6 -> 20.9 us) lose by it and go without.
constexpr int kPriorityDecode = 1;

// ---- the chain decoder ----------------------------------------------------------------------------------
// Decodes kCount values starting at stream bit `start` of the staged block `w` (16 words and a zero word), calling sink(i, entry)
// with the table entry of each (length, index, centroid).  Values are taken in runs of 4 (2 when the model has codes longer than
// 8 bits: kLong) out of a left-aligned 64-bit window, so there is no refill test and no branch inside a run.  A run consumes at
// most 32 bits: its upper half is whole again when the run ends, and only the lower half is filled anew, from the words that
// follow.  The next run's first table read and shift need the upper half alone, so the refill passes in the shadow of that read and the
// dependent chain holds the table reads, a shift and two address instructions each.  (With the whole window rebuilt at the end of a
// run, seven more dependent instructions per run: 8192 x 28672 64.1 -> 63.2 us, 4096 x 4096 7.55 -> 7.50 us, batch 8 over 11008 x 4096 18.4 -> 18.3 us,
// append and attention over 8 x 32 sequences and heads of 4096 tokens 92.1 -> 91.0 us.  A shift of either half by v_alignbit, with 32 - length
// in the table, costs an instruction per value: 65.0, 7.65, 19.5 and 94.1 us.)  The word after next is requested a run ahead: a run
// moves by one word at most.  From the block's end on every word is the zero word: arbitrary bytes decode without touching other memory.
// kWhole: the whole window is rebuilt with every run, the position clamped to 512, where its upper half is the zero word and its lower half
// is never looked at (two words behind the zero word have to be readable).  An instruction less where there is a run for every two values: the batched
// product of long codes, bound by its vector instructions and not by the chain (8192 x 28672, batch 8 107.2 -> 104.0 us, 1000 x 28672 56.8 -> 55.3 us).
template <bool kLong, int kCount, bool kWhole = false, class Sink>
__device__ __forceinline__ void decode_chain(const uint32_t* w, uint32_t start, const Lane& L, Sink&& sink) {
    constexpr int kRun = kLong ? 2 : 4;
    static_assert(kCount % kRun == 0, "chain length");
    static_assert(kRun * (kLong ? kMaxLen : kPeekBits) <= 32, "a run stays inside two words");
    // Otherwise the lower half of the window comes from the words w1 and w2, w1 being the first that begins at the position or behind it: with
    // the position counted down from 0, the position itself is the shift count, also on a word's border.
    int32_t down = -(int32_t)start;  // start <= 511
    int32_t next = down >> 5;        // index of w1, negated
    const auto word = [&](int32_t i) { return w[min((uint32_t)i, (uint32_t)kBlockWords)]; };
    [[maybe_unused]] uint32_t pos = start, w0, w1, w2, w3;
    uint32_t wi = start >> 5;
    uint64_t win;
    if constexpr (kWhole) {
        w0 = w[wi], w1 = w[wi + 1], w2 = w[wi + 2];
        win = (((uint64_t)w0 << 32) | (uint64_t)w1) << (start & 31u);
    } else {
        w1 = word(-next), w2 = word(1 - next), w3 = word(2 - next);
        win = ((((uint64_t)w[wi] << 32) | (uint64_t)w[wi + 1]) << (start & 31u)) & 0xFFFFFFFF00000000ull;
        win |= __builtin_amdgcn_alignbit(w1, w2, (uint32_t)down);
    }
#pragma unroll
    for (int i0 = 0; i0 < kCount; i0 += kRun) {
        uint32_t used = 0;  // sum of the run's entries; its low byte is the number of bits consumed (at most 4 x 8 or 2 x 12)
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            uint32_t e = L.lut[(uint32_t)(win >> 32) >> L.shift];
            if (kLong) {
                if ((e & 0xFFu) == 0u) {
                    // code longer than the peek: rank of the next 12 bits among the left-aligned canonical codes
                    const uint32_t v = (uint32_t)(win >> 32) >> (32 - kMaxLen);
                    // the list is read here, on the rare path, not held in 16 registers throughout: its LDS byte address
                    // passes through an empty asm statement (a pointer passed through one would come back without its
                    // address space, and the reads below would become flat loads instead of LDS reads)
                    uint32_t lt_at = (uint32_t)(size_t)(const lds_u32*)L.longtab;
                    asm volatile("" : "+v"(lt_at));
                    const lds_u32* lt = (const lds_u32*)(size_t)lt_at;
                    int rank = 0;
                    for (int q = 1; q < kK; ++q) rank += ((lt[q] & 0xFFFu) <= v) ? 1 : 0;
                    const uint32_t t = lt[rank];
                    const uint32_t idx = (t >> 12) & 15u;
                    e = ((uint32_t)__half_as_ushort(L.cent[idx]) << 16) | (idx << 8) | (t >> 16);
                }
            }
            sink(i0 + j, e);
            used += e;
            win <<= (e & 0xFFu);
        }
        if constexpr (kWhole) {
            if (i0 + kRun == kCount) break;
            pos = min(pos + (used & 0xFFu), (uint32_t)(kBlockWords * 32));
            const uint32_t now = pos >> 5;  // wi or wi + 1
            const bool adv = now != wi;
            w0 = adv ? w1 : w0;
            w1 = adv ? w2 : w1;
            w2 = w[now + 2];  // used one run later at the earliest
            win = (((uint64_t)w0 << 32) | (uint64_t)w1) << (pos & 31u);
            wi = now;
        } else if (i0 + kRun < kCount) {
            down -= (int32_t)(used & 0xFFu);
            const int32_t now = down >> 5;  // next or next - 1
            const bool adv = now != next;
            w1 = adv ? w2 : w1;
            w2 = adv ? w3 : w2;
            w3 = word(2 - now);  // used one run later at the earliest
            win = (win & 0xFFFFFFFF00000000ull) | (uint64_t)__builtin_amdgcn_alignbit(w1, w2, (uint32_t)down);
            next = now;
        }
    }
}

// ---- sums and payload staging of a wavefront ---------------------------------------------------------------
template <int kCtrl>
__device__ __forceinline__ float dpp_mov(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), kCtrl, 0xF, 0xF, true));
}
__device__ __forceinline__ float read_lane(float v, int l) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l));
}
// sum over the 64 lanes of a wavefront in a fixed order, on the VALU (cross-lane moves inside rows of
// 16 lanes, then the four row sums through scalar registers); every lane returns the total
__device__ __forceinline__ float wave_sum(float t) {
    t += dpp_mov<0xB1>(t);   // quad_perm [1,0,3,2]
    t += dpp_mov<0x4E>(t);   // quad_perm [2,3,0,1]
    t += dpp_mov<0x141>(t);  // row_half_mirror
    t += dpp_mov<0x140>(t);  // row_mirror
    return (read_lane(t, 0) + read_lane(t, 16)) + (read_lane(t, 32) + read_lane(t, 48));
}

// the same walk for any associative, commutative, exact operation (minimum, maximum): the order does not matter
template <class T, class Op>
__device__ __forceinline__ T wave_all(T v, Op op) {
    float t = __builtin_bit_cast(float, v);
    const auto f = [&](float a, float b) { return __builtin_bit_cast(float, op(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b))); };
    t = f(t, dpp_mov<0xB1>(t));
    t = f(t, dpp_mov<0x4E>(t));
    t = f(t, dpp_mov<0x141>(t));
    t = f(t, dpp_mov<0x140>(t));
    return __builtin_bit_cast(T, f(f(read_lane(t, 0), read_lane(t, 16)), f(read_lane(t, 32), read_lane(t, 48))));
}

struct UnitLoad {
    uint4 v0, v1;
    uint32_t meta;
};
// the payload pieces of this lane for unit (row, ct) and the meta word of the unit's block `slot` (the one it decodes).
// Block indices are clamped into the row, so every lane issues the same loads and a slot past the row end holds a copy of
// the row's last block: it decodes to finite values, which the caller drops.  Nothing here uses the loaded
// data, so the loads stay in flight while the previous unit is decoded.
__device__ __forceinline__ UnitLoad load_unit(const uint4* __restrict__ blocks, const uint32_t* __restrict__ meta,
                                              int row, int gpr, int ct, int lane, int slot) {
    UnitLoad u;
    const size_t row_base = (size_t)row * gpr;
    const int g0 = ct * kUnitBlocks + (lane >> 2), g1 = g0 + 16;
    u.v0 = blocks[(row_base + min(g0, gpr - 1)) * 4 + (lane & 3)];
    u.v1 = blocks[(row_base + min(g1, gpr - 1)) * 4 + (lane & 3)];
    u.meta = meta[row_base + min(ct * kUnitBlocks + slot, gpr - 1)];
    return u;
}
__device__ __forceinline__ UnitLoad load_unit(const uint4* __restrict__ blocks, const uint32_t* __restrict__ meta,
                                              int row, int gpr, int ct, int lane) {
    return load_unit(blocks, meta, row, gpr, ct, lane, lane & (kUnitBlocks - 1));
}
// Lane l writes pieces of blocks l / 4 and l / 4 + 16; the chains are then read by other lanes (lane b and b + 32
// read block b).  The exchange goes through the wavefront's private buffer without a workgroup barrier, so it is
// fenced on both sides at wavefront scope: the reads of the previous unit come before these writes, and these
// writes before the reads that follow.
__device__ __forceinline__ void store_unit(uint32_t* wbuf, const UnitLoad& u, int lane) {
    wave_lds_fence();
    uint32_t* d = wbuf + (lane >> 2) * kStride + (lane & 3) * 4;
    d[0] = u.v0.x; d[1] = u.v0.y; d[2] = u.v0.z; d[3] = u.v0.w;
    d += 16 * kStride;
    d[0] = u.v1.x; d[1] = u.v1.y; d[2] = u.v1.z; d[3] = u.v1.w;
    wave_lds_fence();
}


// The merge of n_splits partial results of one query head, a dimension per thread: ml holds their (maximum, denominator) pairs, part this
// dimension's unnormalised outputs, kGroup apart.
struct Merged {
    float num, den;
};
__device__ __forceinline__ Merged merge_splits(const float* __restrict__ ml, const float* __restrict__ part, int n_splits) {
    // Sixteen splits at a time (four or eight where there are no more) with all their loads in flight together, indices
    // clamped; the additions run in split order.  An empty split (maximum -inf, zeros) gets weight 0, also when every
    // split is empty (mx = -inf).  The kernel is bound by the latency of the partial results, which come from memory: up to
    // sixteen splits the maximum is formed from the values in hand and not in a round trip of its own.
    float num = 0.0f, den = 0.0f;
    const auto batch = [&](auto count, int s0, float mx) {
        constexpr int kCount = decltype(count)::value;
        float m[kCount], d[kCount], v[kCount];
#pragma unroll
        for (int j = 0; j < kCount; ++j) {
            const int sj = min(s0 + j, n_splits - 1);
            m[j] = ml[2 * sj];
            d[j] = ml[2 * sj + 1];
            v[j] = part[(size_t)sj * kGroup];
        }
        if (s0 == 0 && n_splits <= kCount) {
            mx = m[0];
#pragma unroll
            for (int j = 1; j < kCount; ++j) mx = fmaxf(mx, m[j]);
        }
#pragma unroll
        for (int j = 0; j < kCount; ++j) {
            if (s0 + j < n_splits) {  // uniform
                const float w = m[j] == -INFINITY ? 0.0f : __expf(m[j] - mx);
                num += w * v[j];
                den += w * d[j];
            }
        }
    };
    if (n_splits <= 4) batch(std::integral_constant<int, 4>{}, 0, 0.0f);
    else if (n_splits <= 8) batch(std::integral_constant<int, 8>{}, 0, 0.0f);
    else if (n_splits <= 16) batch(std::integral_constant<int, 16>{}, 0, 0.0f);
    else {
        // the largest of the splits' maxima: a few splits per lane and a wavefront maximum (exact whatever the order),
        // instead of a chain of n_splits dependent loads
        float mx = -INFINITY;
        for (int s = threadIdx.x & 63; s < n_splits; s += 64) mx = fmaxf(mx, ml[2 * s]);
        mx = wave_all(mx, [](float a, float b) { return fmaxf(a, b); });
        for (int s0 = 0; s0 < n_splits; s0 += 16) batch(std::integral_constant<int, 16>{}, s0, mx);
    }
    return {num, den};
}

}  // namespace ecco_chain

// How the attention kernels of the two-chain format are launched: wavefronts, tables, spans and workspaces by sizes alone.  Host code without a
// runtime call, so that every size can be looked at without a GPU; the constants are shared with the kernels (ecco_kernels.hip).
#pragma once

#include <algorithm>
#include <cstddef>

#include "ecco_internal.h"

namespace ecco {

constexpr int kStride = kBlockWords + 1;  // LDS words per staged block (last one is a zero pad)
constexpr int kUnitBlocks = 32;
// private payload buffer of a wavefront, and behind it two words that a chain of whole windows reads, though it does not use them
constexpr int kUnitWords = kUnitBlocks * kStride + 4;
constexpr int kLdsWords = 160 * 1024 / 4;              // of a compute unit
// LDS words of the decode tables: the long-code lists and the centroids are only copied for models that need them
constexpr int decode_table_words(int S, bool lng) { return S * (kPeekEntries + kK + (lng ? kK + kK / 2 : 0)); }
// Units of 32 tokens in a capacity of `tokens`, which may be any positive number up to 2^31 - 1: of that many units, the tokens no longer
// fit an int.
constexpr int units_of(int tokens) { return (tokens - 1) / kUnitBlocks + 1; }
// Ranges of a step over pages: sequences are cut into ranges of one length, so that those of all heads find a place at once among `places`
// workgroups.  The least length for `total` units of all sequences.  The total is FP32, since it may exceed an int; ranges of this length or
// more, and at least one per sequence, are at most places / Hkv and one per sequence.
constexpr int kRangeLeast = 8;        // units: one for each wavefront
constexpr int kRangeSequences = 256;  // sequences up to which ranges are cut
constexpr int range_least(float total, int Hkv, int places) {
    const float share = total * (float)Hkv / (float)places * 0.9999f;
    if (share >= 134217728.0f) return 134217728;  // longer than any sequence
    const int whole = (int)share;
    return std::max(kRangeLeast, whole + ((float)whole < share ? 1 : 0));
}
// Tokens of `units` units, or more than a span ever holds
constexpr int kSpanMax = 8192, kSpanLeast = 2048;
constexpr int span_tokens(int units) { return std::min(units, kSpanMax / kUnitBlocks + 1) * kUnitBlocks; }

// Whether two workgroups are to share a compute unit, each with half of the wavefronts that one alone would have: the other's decoding
// then covers what is fixed per workgroup, but a sequence by itself takes longer.  `units`: of the longest sequence (or range) that may come.
// It is taken where that one, if it is the only long one, is no more than the work of a compute unit otherwise: 16 units per workgroup there.
// 16 patterns, alone -> shared, in us, at full capacity / lengths drawn evenly / one sequence of full length beside others of an eighth of it:
//    288 workgroups of 500 tokens   32.0 -> 25.0     26.3 -> 20.3     23.8 -> 18.9     shared
//    512 of 1024                    50.7 -> 43.2     36.6 -> 33.7     34.7 -> 30.7     shared
//   1024 of 1024                    96.2 -> 79.9     76.8 -> 63.3     55.9 -> 32.2     shared
//    288 of 4096                   149.9 -> 140.8    87.5 -> 126.5    75.9 -> 102.6
//    384 of 2048                    82.4 -> 75.4     55.9 -> 58.0     41.8 -> 53.9
//    512 of 4096                   153.6 -> 145.0   133.6 -> 133.4    76.0 -> 103.6
//    768 of 2048                   123.6 -> 118.3   104.1 -> 96.3     49.6 -> 55.6
// Grouped queries, ranges of as many tokens: 320 of 3000 133.8 -> 125.2, 85.2 -> 102.0, 67.5 -> 82.8; 512 of 500 36.7 -> 29.3, 35.1 -> 28.0,
// 30.5 -> 20.1; 512 of 2000 97.5 -> 87.7, 79.7 -> 74.0, 49.0 -> 57.9; 1024 of 1000 108.6 -> 88.9, 97.0 -> 75.2, 60.3 -> 34.8.
inline bool share_units(size_t wgs, int units, int cus) { return wgs > (size_t)cus && (size_t)units * (size_t)cus <= 16 * wgs; }

// ---- pages (include/ecco_paged.h)
// whether `pages` pages of `page_tokens` tokens are a pool, or a row of a page table, whose tokens an int32 counts
constexpr int kPageLeast = kUnitBlocks / 2, kPageMost = 1024;
constexpr bool pool_fits(int page_tokens, int pages) {
    return page_tokens >= kPageLeast && page_tokens <= kPageMost && (page_tokens & (page_tokens - 1)) == 0 && pages > 0 && (long long)page_tokens * pages <= 0x7FFFFFFF;
}

// ---- kv_attend_kernel
// Two workgroups of eight wavefronts share a compute unit where there are workgroups for it and both models' tables fit half its
// LDS: each decodes while the other builds or sums.  Otherwise one workgroup takes it, of as few wavefronts as take the fewest rounds over the units
// of the capacity: a table read costs less the more wavefronts wait for theirs (one workgroup, 8192 tokens: 166.7 us with sixteen,
// 177.9 us with twelve), barriers and sums the more the more meet (64 patterns, ten units: 21.5 us with twelve, 22.2 us with sixteen;
// two units: 15.8 us with eight, 16.5 us with twelve).  The decoders of long codes need the registers of twelve.
struct AttnPlan {
    int waves;
    int table_words;  // LDS words of the tables: both models', or the larger one's
    int both;         // the V tables have their own place, behind those of K
    int span;         // tokens per span, a multiple of 32
    size_t lds;
};
inline AttnPlan attn_plan(int Sk, bool lk, int Sv, bool lv, size_t wgs, int T_max, int cus) {
    const int wk = decode_table_words(Sk, lk), wv = decode_table_words(Sv, lv), units = units_of(T_max), tokens = span_tokens(units);
    const auto plan = [&](int waves, int lds_words) {
        AttnPlan p;
        const int fixed = waves * (kUnitWords + 2);
        p.waves = waves;
        p.both = wk + wv + fixed + std::min(kSpanLeast, tokens) <= lds_words;
        p.table_words = p.both ? wk + wv : std::max(wk, wv);
        p.span = std::min({kSpanMax, tokens, (lds_words - p.table_words - fixed) / kUnitBlocks * kUnitBlocks});
        p.lds = (size_t)(p.table_words + fixed + p.span) * 4;
        return p;
    };
    if (lk || lv) return plan(12, kLdsWords);
    const AttnPlan two = plan(8, kLdsWords / 2);
    if (two.both && share_units(wgs, units, cus)) return two;
    const auto rounds = [&](int waves) { return (units + waves - 1) / waves; };
    const int waves = rounds(8) == rounds(16) ? 8 : rounds(12) == rounds(16) ? 12 : 16;
    return plan(waves, kLdsWords);
}

// ---- kv_attend_gqa_kernel
constexpr int kGqaMaxGroup = 16;
constexpr int kTileStride = 20;                 // words per row of the transposition tile: 32 tokens (16 words) + 4 of padding
constexpr int kTileWords = 16 * kTileStride;
constexpr int kGqaScoreWords = 7936;            // query heads x tokens of a span kept in LDS, at most
constexpr int kRedTile = 276, kRedRow = 68;     // words of a tile, and of 16 lanes of it, in the sum over wavefronts (skewed over the banks)
constexpr int gqa_state_words(int waves) { return 2 * waves * kGqaMaxGroup; }  // per wavefront and head: maximum, denominator

constexpr int gqa_score_stride(int span) { return span + 4; }   // words: 16-byte aligned, and 4 modulo 32 so that heads fall on different banks
// As AttnPlan, but eight wavefronts up to 8 units of a range (17.9 us, 19.3 us with twelve) and twelve beyond.  (Sixteen, in us for a quarter of the
// capacity / all of it: 16 units, 16 patterns, groups of 4 15.4 -> 16.5 / 21.6 -> 21.2, groups of 8 16.5 -> 18.2 / 22.7 -> 22.7, 64 patterns 17.6 -> 19.1
// / 24.1 -> 24.2; 32 units at all of it 31.7 -> 32.7, 64 patterns 33.1 -> 34.6, groups of 8 38.6 -> 40.6.)
struct GqaPlan {
    int waves;
    int table_words;  // LDS words of the tables: both models', or the larger one's
    int both;         // the V tables have their own place, behind those of K
    int span;         // tokens of a span that the LDS holds, a multiple of 32
    int step;         // tokens per span of a range that takes several: whole rounds of the wavefronts, where a span holds one
    size_t lds;
};
inline GqaPlan gqa_plan(int Sk, bool lk, int Sv, bool lv, int grp, size_t wgs, int units, int cus) {
    const int wk = decode_table_words(Sk, lk), wv = decode_table_words(Sv, lv), tokens = span_tokens(units);
    const auto plan = [&](int waves, int lds_words) {
        const int fixed = waves * (kUnitWords + kTileWords) + gqa_state_words(waves);
        GqaPlan p;
        p.waves = waves;
        const int round = std::min(units, waves) * kUnitBlocks;  // tokens that the wavefronts take at a time
        p.both = wk + wv + fixed + grp * gqa_score_stride(round) <= lds_words;
        p.table_words = p.both ? wk + wv : std::max(wk, wv);
        const int scores = std::min(kGqaScoreWords, lds_words - p.table_words - fixed);
        p.span = std::min((scores / grp - 4) & ~(kUnitBlocks - 1), tokens);
        p.step = p.span < tokens && p.span > round ? p.span - p.span % round : p.span;
        p.lds = (size_t)std::max(p.table_words + fixed + grp * gqa_score_stride(p.span), gqa_state_words(waves) + waves * 8 * kRedTile) * 4;
        return p;
    };
    if (lk || lv) return plan(12, kLdsWords);
    const GqaPlan two = plan(8, kLdsWords / 2);
    if (two.both && share_units(wgs, units, cus)) return two;
    return plan(units <= 8 ? 8 : 12, kLdsWords);
}

// ---- attend_rows_kernel (pages)
// As GqaPlan for up to `rows` rows (1 to 32), without LDS of its own for the state.  More than 8 rows take more than the 128 registers with which
// two workgroups share a compute unit; 32 with long codes more than those of twelve wavefronts.
constexpr int kFewRows = 2 * kGqaMaxGroup;
inline GqaPlan rows_plan_of(int waves, int lds_words, int wk, int wv, int rows, int units) {
    const int fixed = waves * (kUnitWords + kTileWords), tokens = span_tokens(units);
    GqaPlan p;
    p.waves = waves;
    const int round = std::min(units, waves) * kUnitBlocks;  // tokens that the wavefronts take at a time
    p.both = wk + wv + fixed + rows * gqa_score_stride(round) <= lds_words;
    p.table_words = p.both ? wk + wv : std::max(wk, wv);
    const int scores = lds_words - p.table_words - fixed;
    p.span = std::min((scores / rows - 4) & ~(kUnitBlocks - 1), tokens);
    p.step = p.span < tokens && p.span > round ? p.span - p.span % round : p.span;
    p.lds = (size_t)std::max(p.table_words + fixed + rows * gqa_score_stride(p.span), gqa_state_words(waves) + waves * 8 * kRedTile) * 4;
    return p;
}
// whether two workgroups of eight wavefronts can share a compute unit
inline bool rows_can_share(int Sk, bool lk, int Sv, bool lv, int rows) {
    return !lk && !lv && rows <= kGqaMaxGroup / 2 && rows_plan_of(8, kLdsWords / 2, decode_table_words(Sk, lk), decode_table_words(Sv, lv), rows, 8).both;
}
// cut: ranges of one length, of which none outlasts the others where workgroups share.  Otherwise as the contiguous cache's
inline GqaPlan rows_plan(int Sk, bool lk, int Sv, bool lv, int rows, size_t wgs, int units, int cus, bool cut) {
    const int wk = decode_table_words(Sk, lk), wv = decode_table_words(Sv, lv);
    if (lk || lv) return rows_plan_of(rows > kGqaMaxGroup ? 8 : 12, kLdsWords, wk, wv, rows, units);
    if (rows_can_share(Sk, lk, Sv, lv, rows) && (cut || share_units(wgs, units, cus))) return rows_plan_of(8, kLdsWords / 2, wk, wv, rows, units);
    return rows_plan_of(units <= 8 && rows <= kGqaMaxGroup ? 8 : 12, kLdsWords, wk, wv, rows, units);
}

// ---- attention over pages: what is decoded on the way and what into the workspace, and how much of that there may be
constexpr int kUnitBytes = 2 * kUnitBlocks * kGroup * 2;  // a unit's K and V as operands in the workspace
struct PagedPlan {
    int few, few_rows, cut, units;               // sequences with up to `few` rows are decoded on the way: the kernel's rows, whether in ranges, units of the longest
    int wide_tiles, tile_rows, wide_splits, wide_units;  // the others: tiles that there may be, their rows, ranges of the tokens, units in the workspace
    size_t few_bytes, bytes;                     // of the workspace
};
constexpr size_t round_up(size_t n) { return (n + 255) & ~(size_t)255; }
constexpr size_t kBytesMost = (size_t)1 << 60;  // where products of sizes stop: more than any memory
constexpr size_t bytes_of(size_t a, size_t b) { return b != 0 && a > kBytesMost / b ? kBytesMost : a * b; }
constexpr size_t kPartBytes = (kGroup + 2) * sizeof(float);  // of a row and a range: outputs, maximum, denominator
constexpr int rows_bucket(int rows) { return rows <= 8 ? 8 : rows <= 16 ? 16 : kFewRows; }
// of the ranges: (first, count) per sequence, and the parts of all that there may be
inline size_t range_bytes(int B, int Hkv, int cus, int rows) { return round_up((size_t)B * 8) + round_up(((size_t)B * Hkv + 2 * (size_t)cus) * rows * kPartBytes); }
// of the operands and the running sums beside them
inline size_t operand_bytes(int B, int Hkv, int units) { return 2 * round_up(((size_t)B + 1) * 4) + round_up((size_t)units * 4) + bytes_of((size_t)units * kUnitBytes, Hkv); }
// units of `many` sequences of up to max_kv tokens, and total_kv together
inline int units_of_all(long long many, int max_kv, long long total_kv) { return (int)std::min<long long>(std::min(total_kv, many * max_kv) / kUnitBlocks + many, 0x7FFFFFFF); }
constexpr int splits_most(int max_kv) { return (int)std::min<long long>(((long long)max_kv + 511) / 512, 64); }

inline PagedPlan paged_plan(int n_tokens, int B, int Hq, int Hkv, int max_new, int max_kv, long long total_kv, int cus) {
    PagedPlan p{};
    max_new = std::min(max_new, n_tokens);
    const int grp = Hq / Hkv;
    const long long rows = (long long)max_new * grp;
    const bool wide = rows > kFewRows, all = wide && (long long)max_new * B == n_tokens;  // every sequence has as many rows
    // Beside chunks, what is taken on the way is sequences with a token each, in the kernel that suits those.
    const long long few = wide ? grp : rows;
    p.few_rows = rows_bucket((int)few);
    p.few = all ? 0 : (int)few;
    if (!all) {
        // Into ranges where there are fewer sequences and heads than compute units, and sequences that one round of the wavefronts does not take.  (256
        // compute units, 8 heads; 31 sequences in ranges, 32 whole, us: all of 2304 tokens 60.9 and 55.8; 512 to 4096 67.3 and 87.8; one of 32768 beside
        // 2048 94.5 and 656: what this leaves behind is uneven lengths in steps of many sequences.)
        p.units = units_of(max_kv);
        p.cut = B * (long long)Hkv < cus && B <= kRangeSequences && p.units > kRangeLeast;
        if (p.cut) p.few_bytes = range_bytes(B, Hkv, cus, p.few_rows);
    }
    p.bytes = p.few_bytes;
    if (wide) {
        // rows that the sequences have at the most, and sequences that have more than `few` of them: two tokens each, then
        const long long tokens = std::min<long long>(n_tokens, (long long)max_new * B), many = all ? B : std::min<long long>(B, tokens / 2);
        // A tile of 256 rows reads what it needs once for twice the rows, but there have to be enough of them: a 2048-token prompt, 32/8 heads, 69.3 us
        // with 512 tiles of 128 rows, 78.1 us with 256 of 256; four chunks of up to 1024 tokens over 8192, 684 us with 980, 625 us with 490.
        p.tile_rows = tokens * grp / 256 * Hkv * 2 >= 3ll * cus ? 256 : 128;
        const long long each = (rows + p.tile_rows - 1) / p.tile_rows;
        p.wide_tiles = (int)(all ? each * B : std::min(each * many, tokens * grp / p.tile_rows + many));
        p.wide_units = units_of_all(many, max_kv, total_kv);
        // Split over the tokens where that makes a workgroup for every compute unit, and a range is worth its share of the merge: a chunk of 512 tokens
        // over 4096, 128 tiles, 87.4 us whole, 71.7 us in two, 75.3 us in four; 64 tokens over 4096, 16 tiles, 99.1 us, in four 52.2 us, in eight
        // 46.2 us; 1000 tokens over themselves, 128 tiles, 38.2 us, in two 40.1 us.
        const long long wgs = (long long)p.wide_tiles * Hkv;
        p.wide_splits = (int)std::min<long long>(std::max<long long>(1, cus / wgs), splits_most(max_kv));
        p.bytes += operand_bytes(B, Hkv, p.wide_units);
        if (p.wide_splits > 1) p.bytes += round_up((size_t)wgs * p.tile_rows * p.wide_splits * kPartBytes);
    }
    return p;
}
// Bytes that the workspace is asked to have: what any step within these sizes takes, so that one that is allocated for a program's largest step
// serves all of them.  (A plan by itself can take more for less: fewer sequences and heads than compute units are cut into ranges, fewer tiles
// are split.)  Each part is the most of its own: of the ranges with as many sequences as are ever cut and the widest kernel, of the
// operands with all sequences that may have many rows, of the splits with as many tiles of 128 rows as there are compute units.  (256-row tiles are at
// least three for two compute units, so that they are not split.)
inline size_t paged_workspace(int n_tokens, int B, int Hq, int Hkv, int max_new, int max_kv, long long total_kv, int cus) {
    max_new = std::min(max_new, n_tokens);
    const int grp = Hq / Hkv, cut = std::min({B, kRangeSequences, (cus - 1) / Hkv});
    const long long rows = (long long)max_new * grp;
    size_t bytes = 0;
    if (cut > 0 && units_of(max_kv) > kRangeLeast) bytes += range_bytes(cut, Hkv, cus, rows_bucket((int)std::min<long long>(rows, kFewRows / grp * grp)));
    if (rows > kFewRows) {
        const long long tokens = std::min<long long>(n_tokens, (long long)max_new * B), many = std::min<long long>(B, tokens / 2);
        const long long tiles = std::min((rows + 127) / 128 * many, tokens * grp / 128 + many);
        bytes += operand_bytes(B, Hkv, units_of_all(many, max_kv, total_kv));
        if (splits_most(max_kv) > 1) bytes += round_up((size_t)std::min<long long>(cus, tiles * Hkv * splits_most(max_kv)) * 128 * kPartBytes);
    }
    return bytes;
}

}  // namespace ecco

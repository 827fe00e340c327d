// Where tokens lie in the paged 8-bit cache and how the launches of its operators are cut: functions of
// sizes and of the sequences' offsets alone, used by host code and kernels alike.
#pragma once
#include <algorithm>

#include "dv_internal.h"

namespace dv {

// ---- pages ---------------------------------------------------------------------------------------
// A page holds `pt` tokens (16, 32, 64 or 128) of every key/value head.  Keys lie token by token
// [page, head, token, channel], values channel by channel [page, head, channel, token]: a lane of a
// score product reads channels of one key, a lane of the value product tokens of one channel, both
// 8 or 16 bytes at once and with no transposition.
inline bool page_tokens_ok(int pt) { return pt == 16 || pt == 32 || pt == 64 || pt == 128; }
__host__ __device__ inline int page_shift(int pt) { return pt == 16 ? 4 : pt == 32 ? 5 : pt == 64 ? 6 : 7; }

// Page of a sequence's j-th stretch of pt tokens, or -1: past the table, or no page of the cache.
__host__ __device__ inline int page_of(const int* table, int table_pages, int pages, int s, int j) {
    if (j < 0 || j >= table_pages) return -1;
    const long long at = (long long)s * table_pages + j;
    const long long p = table ? (long long)table[at] : at;
    return p >= 0 && p < pages ? (int)p : -1;
}

// The same in two steps, for kernels that ask for a page well before they need it: a table entry (of the
// table's last stretch, past it; without a table any int), and the page or -1.  The load takes no branch,
// so that the wait for it need not be for all loads.
__host__ __device__ inline int entry_of(const SeqArgs& q, int s, int j) {
    const long long at = (long long)s * q.table_pages + (j < q.table_pages ? j : q.table_pages - 1);
    const int* p = q.table ? q.table + at : q.at;
    return *p;
}
__host__ __device__ inline int page_from(const SeqArgs& q, int pages, int entry, int s, int j) {
    const int e = q.table ? entry : (int)((long long)s * q.table_pages + j);
    return j < q.table_pages && (unsigned)e < (unsigned)pages ? e : -1;
}

// ---- rows of a call ------------------------------------------------------------------------------
// Rows of sequence s: offsets[s] .. offsets[s + 1] - 1, cut to the rows there are; without offsets
// sequence s has row s (or the call's one sequence has them all).
struct Seq {
    int s;          // -1: none
    int row0, n;    // its rows
    int at;         // q.at[s]
    int slot0;      // its first slot (with offsets)
};
__host__ __device__ inline Seq seq_from(const SeqArgs& q, int s, int off, int next, int at) {
    const int a = off < 0 ? 0 : off, b = next < q.rows ? next : q.rows;
    return {s, a, b > a ? b - a : 0, at, 0};
}
// ... without offsets
__host__ __device__ inline Seq seq_of(const SeqArgs& q, int s) {
    if (s < 0 || s >= q.n_seqs) return {-1, 0, 0, 0, 0};
    if (q.one) return {s, 0, q.rows, q.at[s], 0};
    return {s, s, s < q.rows ? 1 : 0, q.at[s], 0};
}

// Kernels deal blocks to slots.  With offsets a sequence owns as many as it has pages or tiles, one sequence after the
// other; a block finds the sequence of its slot by summing those numbers (find_seq), so that a ragged batch needs
// no list made on the host.  The host, which does not know the offsets, launches as many slots as there can be:
//   pages that n rows touch, from any start: at most n / pt + 2 (floor)
//   tiles of R packed rows (rows x query heads of a key head): at most n group / R + 1 (floor)
// The slots that nobody owns are the last ones.  (Between the sequences instead, every second one empty, one query
// of 16 heads a key head over 64 sequences of up to 12,000 keys takes 224 us, so 177: presumably blocks are dealt to
// the chip's engines in rotation, and the empty ones all went to the same.)
__host__ __device__ inline int part_count(const Seq& s, int shift) {
    return s.n == 0 || s.at < 0 ? 0 : (int)(((long long)s.at + s.n - 1) >> shift) - (s.at >> shift) + 1;
}
__host__ __device__ inline int tile_count(const Seq& s, int group, int shift) {
    return (int)(((long long)s.n * group + (1 << shift) - 1) >> shift);
}
__host__ __device__ inline long long page_slots(bool offsets, int n_seqs, int rows, int shift) {
    return offsets ? ((long long)rows >> shift) + 2ll * n_seqs : n_seqs;
}

// One page of one sequence that a call's rows touch.
struct PagePart {
    int page;       // -1: the cache does not have it
    int row0;       // row of its first token
    int slot0, n;   // its places slot0 .. slot0 + n - 1; n = 0: nothing
};
// ... slot u, of sequence s
__host__ __device__ inline PagePart part_at(const SeqArgs& q, int pt, int pages, const Seq& sp, long long u) {
    PagePart p = {-1, 0, 0, 0};
    const int shift = page_shift(pt), s = sp.s, start = sp.at;
    if (s < 0 || sp.n == 0 || start < 0) return p;
    const long long j = q.one ? u : q.offsets ? u - sp.slot0 : 0;
    if (j < 0) return p;
    const long long page = ((long long)start >> shift) + j;     // of the sequence
    const long long end = (long long)start + sp.n, next = (page + 1) << shift;
    const long long a = start > page << shift ? start : page << shift, b = end < next ? end : next;
    if (a >= b) return p;
    p.page = page < q.table_pages ? page_of(q.table, q.table_pages, pages, s, (int)page) : -1;
    p.row0 = sp.row0 + (int)(a - start);
    p.slot0 = (int)(a - (page << shift));
    p.n = (int)(b - a);
    return p;
}

// A tile of at most R = 2^shift packed rows of one sequence.
struct Tile {
    int seq;     // -1: none
    int row0;    // the sequence's first row
    int n;       // its rows
    int first;   // the tile's first packed row
    int rows;    // packed rows of the tile
    int len;     // keys of the sequence
    int end;     // keys that the tile's last row sees
    int skip0, left_out;   // keys skip0 .. skip0 + left_out - 1, whole steps of 64, which no row of it sees
    int group, front_len;  // behind a prefix: its group (-1: none) and the prefix's keys, in places 0 .. skip0 - 1 (left_out is -skip0)
};
__host__ __device__ inline long long tile_slots(bool offsets, int n_seqs, int rows, int group, int shift) {
    return offsets ? ((long long)rows * group >> shift) + n_seqs
                   : (long long)n_seqs * ((group + (1 << shift) - 1) >> shift);
}
// ... slot u, of sequence s (without offsets: of sequence u / tiles of a row, unless the sequences are groups)
__host__ __device__ inline Tile tile_of(const SeqArgs& q, int pt, int group, int shift, bool causal, const Seq& sp,
                                        long long u, bool groups = false) {
    Tile t = {-1, 0, 0, 0, 0, 0, 0, 0, 0, -1, 0};
    const int s = sp.s;
    if (s < 0) return t;
    const long long j = q.offsets || groups ? u - sp.slot0 : u - (long long)s * ((group + (1 << shift) - 1) >> shift);
    const long long first = j << shift, left = (long long)sp.n * group - first;
    if (j < 0 || left <= 0) return t;
    t.seq = s;
    t.row0 = sp.row0;
    t.n = sp.n;
    t.first = (int)first;
    t.rows = (int)(left < (1 << shift) ? left : 1 << shift);
    const int most = q.table_pages * pt, len = sp.at < most ? sp.at : most;
    t.len = len > 0 ? len : 0;
    t.end = t.len;
    if (causal) {
        const long long e = (long long)t.len - sp.n + (t.first + t.rows - 1) / group + 1;
        t.end = e > 0 ? (int)e : 0;
    }
    return t;
}

// With a window: a row that sees the keys below e without one sees those from e - window on, and the first `sinks`.
__host__ __device__ inline void leave_out(Tile& t, int group, bool causal, int window, int sinks) {
    const int first = causal ? t.len - t.n + t.first / group + 1 : t.len;   // what the tile's first row sees without a window
    const int low = (first > window ? first - window : 0) & ~63, high = ((sinks < t.end ? sinks : t.end) + 63) & ~63;
    if (t.seq < 0 || high >= low) return;
    t.skip0 = high;
    t.left_out = low - high;
}

// ---- launches of rotary positions and of a write --------------------------------------------------
constexpr int ROT_ROWS = 16;   // rows a block turns at most
// Rows a block turns: about four items of 2 `vec` channels a thread.
inline int rows_a_block(int heads, int dh, int vec) {
    return std::max(1, std::min(ROT_ROWS, 1024 / std::max(1, heads * (dh / (2 * vec)))));
}
// A block of a write has 512 threads where a page and head have more than 512 items of 16 channels (more than
// 64 tokens of 128 channels), else 256.
inline int write_threads(int pt, int dh) { return pt * (dh / 16) <= 512 ? 256 : 512; }
constexpr int WRITE_HEADS = 16;   // heads a block of a write quantises at most
// Heads of such a block: as many as leave two blocks a compute unit, which share the angles of their tokens and the
// search for their page (us on 256 units, with the heads that fill the block's threads once / as many as that: 9232
// tokens of 16 heads of 64 28.5 / 22.7, 100,000 of 8 heads of 128 607 / 425; 9232 with one block a unit 30).
inline int write_heads(long long slots, int kv_heads, int cus) {
    const long long least = 2ll * (cus > 0 ? cus : 256);
    int heads = std::min(WRITE_HEADS, kv_heads);
    while (heads > 1 && slots * 2 * ((kv_heads + heads - 1) / heads) < least) heads = (heads + 1) / 2;
    return heads;
}
// Whether a block of about the mean of the sequences' tokens takes its heads in one pass of two items a thread.
inline bool write_in_one_pass(int pt, int dh, int heads, int n_seqs, int rows) {
    const long long tokens = std::min<long long>(pt, ((long long)rows + n_seqs - 1) / std::max(1, n_seqs));
    return tokens * (dh / 16) * heads <= 2 * write_threads(pt, dh);
}
// Threads that a write launches at most: a block per page, head and keys or values, and those of the queries.
inline long long cache_write_threads(int pt, int dh, int kv_heads, int n_seqs, int rows, bool offsets, int q_heads) {
    const int per = q_heads ? rows_a_block(q_heads, dh, 1) : 1;
    return (page_slots(offsets, n_seqs, rows, page_shift(pt)) * 2 * kv_heads + (q_heads ? ((long long)rows + per - 1) / per : 0)) *
           write_threads(pt, dh);
}

// ---- how an attention call is cut ----------------------------------------------------------------
constexpr int TS = 4, LS = 7;      // small tiles of 16 packed rows, large ones of 128
// Blocks of small bf16 tiles that a compute unit holds at least (their registers grow with the head; at 96 and 112 channels
// it holds three, counted as two), and packed rows of a sequence up to which they take it where both kernels run.
__host__ __device__ inline int small_resident(int head_dim) { return head_dim > 85 ? 2 : head_dim > 64 ? 3 : 4; }
__host__ __device__ inline int few_rows(int head_dim) { return small_resident(head_dim) << TS; }
constexpr int MAX_SPLITS = 512;

// partial results: per tile of R rows, head and split R rows of dh fp32, R maxima, R sums
__host__ __device__ inline size_t part_floats(int R, int dh) { return (size_t)R * (dh + 2); }

// window > 0: rows see at most that many keys before their own place and `sinks` first ones.
inline CacheAttnPlan cache_attn_plan(bool bf, int n_seqs, int rows, bool offsets, int max_rows, int table_pages,
                                     int page_tokens, int kv_heads, int q_heads, int head_dim, int cus, int window = 0,
                                     int sinks = 0) {
    CacheAttnPlan p{};
    const int G = q_heads / kv_heads;
    const long long unit = cus > 0 ? cus : 256;
    const long long held = (long long)table_pages * page_tokens;   // at most 2^30
    if (window >= held) window = 0;
    // keys that a tile takes at most (leave_out): the rows of a tile, which lie side by side, move its window's end
    auto keys_of = [&](int shift) {
        const long long more = std::min<long long>(rows, (1 << shift) / G + 1);
        return window ? std::min(held, (std::min<long long>(held, sinks) + 63) / 64 * 64 + window + more + 63) : held;
    };
    const long long most_rows = std::min<long long>(rows, !offsets ? 1 : max_rows > 0 ? max_rows : rows);
    // Large tiles (bf16) decode a key once for 128 rows and give the matrix units long products; small ones read
    // keys at the memory's rate and have eight times the blocks.  Large ones take sequences of more than few_rows
    // packed rows of batches whose small tiles would be more than twice as many as are resident at once.  us, small /
    // large: 8 heads of 128 with 4 queries each, 32 sequences of 2048 keys: 32 packed rows 29 / 50, 64 50 / 51, 96 73 /
    // 54, 512 364 / 159; 64 of 8192: 16 rows 214 / 208, 32 261 / 210, 64 426 / 270, 512 2763 / 1177; 4 of 4096: 128
    // rows 33 / 36, 256 58 / 53, 512 106 / 75; one of 4096: 512 rows 27 / 33; 16 heads of 64, 32 of 2048: 64 rows 41 /
    // 55, 128 80 / 60; 16 of 80, 4 of 700: 128 rows 10 / 27.
    // Where some sequences may have fewer, both kernels run, each on its own: they need not if there is one
    // sequence, or if all have as many rows as the longest.
    const long long small_blocks = tile_slots(offsets, n_seqs, rows, G, TS) * kv_heads;
    const bool alike = n_seqs == 1 || (max_rows > 0 && (long long)n_seqs * max_rows == rows);
    p.route = !bf || most_rows * G <= few_rows(head_dim) || small_blocks <= 2 * small_resident(head_dim) * unit ? ATTN_FEW : alike ? ATTN_MANY : ATTN_BOTH;

    // Splits of equal length.  One sequence: as many as are resident at once, two blocks a compute unit (one
    // query over 200,001 keys of 8 heads of 128, us with 32 / 64 / 98 / 126 splits: 85 / 77 / 87 / 82).
    // Several may have any lengths up to the table's: splits of 2048 keys at most, so that the long ones
    // spread over the chip (64 sequences of 1 to 12,000 keys, us with splits of 1024 / 2048 / 3136 /
    // 6272 / 12,032 keys: 171 / 161 / 167 / 180 / 182) unless there are many tiles anyway -- but not into more
    // than 64 blocks a compute unit, most of them empty where tables are far longer than sequences (the same
    // 64 with tables of 131,072 / 524,288 places: 169 / 179 with that bound, 212 / 411 without).  What takes no
    // longer than the join's launch is not split (`whole` keys and fewer, and into no less than 512; us of one call, whole /
    // split, one query: 1000 / 2000 keys of 128 channels 9.4 / 12.4, 14.6 / 12.4; 2000 of 64 9.0 / 12.5; a large tile of
    // 700 keys takes 27).
    auto cut = [&](CacheAttnCut& c, int shift, long long cap, long long whole) {
        const long long keys = keys_of(shift);
        c.slots = tile_slots(offsets, n_seqs, rows, G, shift);
        const long long units = std::max(1ll, c.slots * kv_heads);
        // Windows shorter than most sequences leave all of them as many keys: resident blocks (two a unit) are counted to the nearest split
        // of a tile and head, and the cap does not hold.  Streams of 1 to 12,000 places of 8 heads of 128, us one split / in splits of
        // 2048 / without a window: 64 with windows of 1024 31.7 / 32.2 / 138, 2048 48.6 / 55.6, 4096 87 / 94; 70 with 2048 60.5 / 62.3
        // / 180, 100 92 / 96 / 251, 128 122 / 130 / 344.  Windows that hold most of the sequences leave them uneven, and lose by it: 64
        // with 8192 140 / 130 / 138, 11,900 158 / 139 / 139.
        const long long most = std::min<long long>(MAX_SPLITS, std::max(1ll, (2 * unit + (window ? units / 2 : 0)) / units));
        long long chunk = (keys + most - 1) / most;
        if (n_seqs > 1 && units < 16 * unit && !window) chunk = std::min(chunk, cap);
        const long long splits = std::min<long long>(MAX_SPLITS, std::max(1ll, 64 * unit / units));
        chunk = std::max({chunk, 512ll, (keys + splits - 1) / splits});
        if (keys <= whole) chunk = std::max(chunk, keys);
        c.chunk = (int)((chunk + 255) / 256 * 256);
        c.splits = (int)std::max(1ll, (keys + c.chunk - 1) / c.chunk);
        c.tile_rows = (int)std::min<long long>(1 << shift, std::max(1ll, most_rows * G));
        return c.splits > 1 ? (size_t)c.slots * kv_heads * c.splits * part_floats(1 << shift, head_dim) : 0;
    };
    if (p.route != ATTN_MANY) p.few_floats = cut(p.few, TS, 2048, (bf ? 1 << 17 : 1 << 16) / head_dim);
    size_t many = 0;
    if (p.route != ATTN_FEW) many = cut(p.many, LS, held, 512);
    p.bytes = (p.few_floats + many) * sizeof(float);
    return p;
}

// Two plans of a call with shared prefixes: its sequences' own keys, taken as without prefixes, and the prefixes', whose
// sequences are the groups (rows: all of the call's).  Every result is left as a partial one for the join, so that more
// splits cost no launch.
struct CacheSharedPlan {
    CacheAttnPlan own, prefix;
    size_t bytes;
    long long blocks;   // of the launch that takes both
    bool behind;        // one plan, `own`: tiles of the sequences take the prefix's keys and then their own
};
inline CacheSharedPlan cache_shared_plan(bool bf, int n_seqs, int rows, bool offsets, int max_rows, int table_pages,
                                         int n_groups, int prefix_table_pages, int page_tokens, int kv_heads, int q_heads,
                                         int head_dim, int cus) {
    CacheSharedPlan p{};
    const int G = q_heads / kv_heads;
    const long long unit = cus > 0 ? cus : 256;
    p.own = cache_attn_plan(bf, n_seqs, rows, offsets, max_rows, table_pages, page_tokens, kv_heads, q_heads, head_dim, cus);
    // Large tiles take prefixes of many rows and keys: us of a call, small / large, one group of 64, 96, 128, 256, 1024 packed rows; 8
    // heads of 128, 65,536 keys 59 / 52, 84 / 56, 99 / 61, 186 / 99, 709 / 305, 16,384 28 / 31, 33 / 34, 37 / 37, 60 / 49, 202 /
    // 112, 4096 19 / 18, 20 / 20, 21 / 22, 29 / 31, 81 / 63; 8 of 80, 65,536 42 / 50, 60 / 55, 69 / 60, 123 / 98, 427 / 259, 16,384
    // 22 / 29, 28 / 34, 33 / 39, 53 / 58, 126 / 98.  Where groups differ each goes to its kernel (few_rows).
    const long long packed = (long long)rows * G, keys = (long long)prefix_table_pages * page_tokens;
    const bool large = bf && packed >= 64ll * n_groups && (double)packed * keys * kv_heads * head_dim >= 3e9;
    p.prefix.route = !large ? ATTN_FEW : n_groups == 1 ? ATTN_MANY : ATTN_BOTH;
    // Tiles of the sequences take the prefix themselves where that is less than a pass of its own costs.  Estimates in us: a
    // large tile takes its keys at 0.95 PFLOP/s; a small one 2 head_dim + 96 bytes a key at 13.7 TB/s, most of them from the
    // caches, and in a pass of its own, whose blocks are cut to fill the chip, 2 head_dim at 14; a pass no faster than the memory
    // has them once, tiles that repeat it no faster than that and the caches (12.8 TB/s) the rest.  Two parts are 4 us and 1.2 ns
    // a row and head of 128 channels more (partial results and their join).  us of a call, two parts / behind, 8 heads of 128
    // with 4 queries each, prefixes of 128, 512, 2048, 8192: 64 sequences of a row 14 / 11, 15 / 14, 21 / 35, 37 / 105; 12 of 33
    // 29 / 16, 33 / 24, 44 / 62, 90 / 178; 64 of 40 141 / 37, 125 / 60, 191 / 158, 511 / 539; 16 heads of 64 in fp32, 12 of 33 16
    // / 11, 18 / 12, 26 / 34, 68 / 82; 8 heads of 128 again, prefixes of 10,000, 40,000, 100,000: one sequence of a row 15.8 /
    // 13.1, 26.4 / 24.8, 43.7 / 41.8, two 16.1 / 16.8, 26.6 / 27.1, 44.0 / 58.1, four of a row behind 100,000 45.4 / 92.
    const double places = (double)keys * kv_heads, once = n_groups * places * 2 * head_dim / 4.5e6;
    auto big_cost = [&](long long tiles) { return tiles * places * 128 * 4 * head_dim / 0.95e9; };
    const long long per = ((long long)rows + n_seqs - 1) / n_seqs * G;   // packed rows of a sequence, were all alike
    const bool big = p.own.route != ATTN_FEW && per > few_rows(head_dim);
    const long long tiles = n_seqs * (big ? (per + 127) / 128 : (per + 15) / 16);
    const double behind = std::max(big ? big_cost(tiles) : tiles * places * (2 * head_dim + 96) / 13.7e6,
                                   once + std::max(0ll, tiles - n_groups) * places * 2 * head_dim / 12.8e6);
    const double pass = large ? big_cost((packed + 127) / 128 + n_groups - 1) : ((packed + 15) / 16 + n_groups - 1) * places * 2 * head_dim / 14e6;
    const double apart = std::max(once, pass) + 4 + 1.2e-3 * rows * q_heads * head_dim / 128;
    const long long places_of_both = (keys + 63) / 64 * 64 + (long long)table_pages * page_tokens;
    if (places_of_both <= 1 << 30 && behind < apart) {   // (counted in ints)
        p.behind = true;
        p.own = cache_attn_plan(bf, n_seqs, rows, offsets, max_rows, table_pages + (int)((keys + 63) / 64 * 64 / page_tokens),
                                page_tokens, kv_heads, q_heads, head_dim, cus);
        p.bytes = p.own.bytes;
        return p;
    }
    // `most` blocks fill the chip; splits end with a step of 64 keys and hold four of them at least
    auto cut = [&](CacheAttnCut& c, int shift, int n, long long held, bool ragged, long long row_most, long long most) {
        c.slots = tile_slots(ragged, n, rows, G, shift);
        if (ragged && n == 1) c.slots = std::max(1ll, (packed + (1 << shift) - 1) >> shift);   // rows lie side by side
        const long long units = std::max(1ll, c.slots * kv_heads), splits = std::min<long long>(MAX_SPLITS, std::max(1ll, most / units));
        c.chunk = (int)((std::max((held + splits - 1) / splits, 256ll) + 63) / 64 * 64);
        c.splits = (int)std::max(1ll, (held + c.chunk - 1) / c.chunk);
        c.tile_rows = (int)std::min<long long>(1 << shift, std::max(1ll, row_most * G));
        p.blocks += units * c.splits;
        return (size_t)units * c.splits * part_floats(1 << shift, head_dim);
    };
    auto both = [&](CacheAttnPlan& x, int n, long long held, bool ragged, long long row_most) {
        // groups or sequences of different lengths leave some of their splits empty (12 questions about three clips of up to
        // 2056 keys in fp32: 16.7 us with two blocks a unit, 13.4 with four; one group of 32 packed rows over 100,003 keys 52, 57)
        x.few_floats = x.route == ATTN_MANY ? 0 : cut(x.few, TS, n, held, ragged, row_most, (n > 1 ? 4 : 2) * unit);
        const size_t many = x.route == ATTN_FEW ? 0 : cut(x.many, LS, n, held, ragged, row_most, 2 * unit);
        x.bytes = (x.few_floats + many) * sizeof(float);
        p.bytes += x.bytes;
    };
    both(p.own, n_seqs, (long long)table_pages * page_tokens, offsets, !offsets ? 1 : max_rows > 0 ? std::min(max_rows, rows) : rows);
    both(p.prefix, n_groups, keys, true, rows);
    return p;
}

#ifdef __HIPCC__
// x of the lanes up to this one, summed (each step adds what lies 1, 2, 4, 8 lanes of 16 below, then the row below's last,
// then the lower half's)
__device__ __forceinline__ int sum_up(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}
// The sequence that owns slot u (every lane of a wavefront calls, with the same u); count: the slots of one.  N times 64
// sequences are looked at together: a chain of loads is what small calls wait for.
// from(s): sequence s.
template <int N, class From, class Count>
__device__ __forceinline__ Seq find_among(const SeqArgs& q, const From& from, const Count& count, int u) {
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b = 0; b < q.n_seqs; b += 64 * N) {
        Seq sp[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int s = b + i * 64 + lane, c = s < q.n_seqs ? s : q.n_seqs - 1;
            sp[i] = from(c);
            sp[i].s = s;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int n = sp[i].s < q.n_seqs ? count(sp[i]) : 0, upto = base + sum_up(n);
            const int k = __popcll(__ballot(upto <= u));
            if (k < 64)
                return {b + i * 64 + k, __builtin_amdgcn_readlane(sp[i].row0, k), __builtin_amdgcn_readlane(sp[i].n, k),
                        __builtin_amdgcn_readlane(sp[i].at, k), __builtin_amdgcn_readlane(upto - n, k)};
            base = __builtin_amdgcn_readlane(upto, 63);
        }
    }
    return {-1, 0, 0, 0, 0};
}
// Group g as a sequence: its sequences' rows lie together.
__device__ __forceinline__ Seq group_from(const SeqArgs& q, const GroupArgs& by, int g) {
    auto first = [&](int i) {   // row of its first sequence
        const int s = by.first ? max(0, min(by.first[i], by.n)) : i ? by.n : 0;
        return q.offsets ? q.offsets[s] : s;
    };
    return seq_from(q, g, first(g), first(g + 1), q.at[g]);
}
// The group of sequence `seq` (-1: none; every lane of a wavefront calls, with the same one).
__device__ __forceinline__ int group_of(const SeqArgs& q, const GroupArgs& by, int seq) {
    if (!by.first) return 0;
    const int lane = threadIdx.x & 63;
    for (int b = 0; b < q.n_seqs; b += 64) {
        const int g = b + lane, c = g < q.n_seqs ? g : q.n_seqs - 1;
        const uint64_t here = __ballot(g < q.n_seqs && by.first[c] <= seq && seq < by.first[c + 1]);
        if (here) return b + __ffsll((unsigned long long)here) - 1;
    }
    return -1;
}
// The tile takes its group's prefix first, in whole steps.
__device__ __forceinline__ void put_behind(Tile& t, const SeqArgs& q, const GroupArgs& by, int pt) {
    if (t.seq < 0) return;
    t.group = group_of(q, by, t.seq);
    if (t.group < 0) return;
    t.front_len = max(0, min(q.at[t.group], q.table_pages * pt));
    t.skip0 = (t.front_len + 63) & ~63;
    t.left_out = -t.skip0;
}
template <class Count>
__device__ __forceinline__ Seq find_seq(const SeqArgs& q, const Count& count, int u) {
    auto from = [&](int s) { return seq_from(q, s, q.offsets[s], q.offsets[s + 1], q.at[s]); };
    return q.n_seqs <= 64 ? find_among<1>(q, from, count, u) : find_among<4>(q, from, count, u);
}
template <class Count>
__device__ __forceinline__ Seq find_group(const SeqArgs& q, const GroupArgs& by, const Count& count, int u) {
    auto from = [&](int g) { return group_from(q, by, g); };
    return q.n_seqs <= 64 ? find_among<1>(q, from, count, u) : find_among<4>(q, from, count, u);
}
#endif

}  // namespace dv

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
};
__host__ __device__ inline long long tile_slots(bool offsets, int n_seqs, int rows, int group, int shift) {
    return offsets ? ((long long)rows * group >> shift) + n_seqs
                   : (long long)n_seqs * ((group + (1 << shift) - 1) >> shift);
}
// ... slot u, of sequence s (without offsets: of sequence u / tiles of a row)
__host__ __device__ inline Tile tile_of(const SeqArgs& q, int pt, int group, int shift, bool causal, const Seq& sp,
                                        long long u) {
    Tile t = {-1, 0, 0, 0, 0, 0, 0};
    const int s = sp.s;
    if (s < 0) return t;
    const long long j = q.offsets ? u - sp.slot0 : u - (long long)s * ((group + (1 << shift) - 1) >> shift);
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

inline CacheAttnPlan cache_attn_plan(bool bf, int n_seqs, int rows, bool offsets, int max_rows, int table_pages,
                                     int page_tokens, int kv_heads, int q_heads, int head_dim, int cus) {
    CacheAttnPlan p{};
    const int G = q_heads / kv_heads;
    const long long unit = cus > 0 ? cus : 256;
    const long long keys = (long long)table_pages * page_tokens;   // at most 2^30
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
        c.slots = tile_slots(offsets, n_seqs, rows, G, shift);
        const long long units = std::max(1ll, c.slots * kv_heads);
        const long long most = std::min<long long>(MAX_SPLITS, std::max(1ll, 2 * unit / units));
        long long chunk = (keys + most - 1) / most;
        if (n_seqs > 1 && units < 16 * unit) chunk = std::min(chunk, cap);
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
    if (p.route != ATTN_FEW) many = cut(p.many, LS, keys, 512);
    p.bytes = (p.few_floats + many) * sizeof(float);
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
template <int N, class Count>
__device__ __forceinline__ Seq find_among(const SeqArgs& q, const Count& count, int u) {
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b = 0; b < q.n_seqs; b += 64 * N) {
        Seq sp[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int s = b + i * 64 + lane, c = s < q.n_seqs ? s : q.n_seqs - 1;
            sp[i] = seq_from(q, s, q.offsets[c], q.offsets[c + 1], q.at[c]);
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
template <class Count>
__device__ __forceinline__ Seq find_seq(const SeqArgs& q, const Count& count, int u) {
    return q.n_seqs <= 64 ? find_among<1>(q, count, u) : find_among<4>(q, count, u);
}
#endif

}  // namespace dv

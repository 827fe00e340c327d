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
    int off;        // its first row as the call says
    int row0, n;    // its rows
    int at;         // q.at[s]
};
__host__ __device__ inline Seq seq_from(const SeqArgs& q, int s, int off, int next, int at) {
    const int a = off < 0 ? 0 : off, b = next < q.rows ? next : q.rows;
    return {s, off, a, b > a ? b - a : 0, at};
}
__host__ __device__ inline Seq seq_of(const SeqArgs& q, int s) {
    if (s < 0 || s >= q.n_seqs) return {-1, 0, 0, 0, 0};
    if (q.one) return {s, 0, 0, q.rows, q.at[s]};
    if (!q.offsets) return {s, s, s, s < q.rows ? 1 : 0, q.at[s]};
    return seq_from(q, s, q.offsets[s], q.offsets[s + 1], q.at[s]);
}

// Kernels deal blocks to slots: sequence s owns the slots from slot_base(s), and a slot finds its
// sequence by comparing bases, so that a ragged batch needs no list made on the host.
//   pages that n rows touch, from any start: at most n / pt + 2 (floor), so base = offset / pt + 2 s
//   tiles of R packed rows (row x query heads of a key head, `mul`): at most n mul / R + 1 (floor)
__host__ __device__ inline long long slot_base(int offset, int mul, int shift, int add, int s) {
    return ((long long)offset * mul >> shift) + (long long)add * s;
}
__host__ __device__ inline long long page_slots(bool offsets, int n_seqs, int rows, int shift) {
    return offsets ? slot_base(rows, 1, shift, 2, n_seqs) : n_seqs;
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
    const long long j = q.one ? u : q.offsets ? u - slot_base(sp.off, 1, shift, 2, s) : 0;
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
    return offsets ? slot_base(rows, group, shift, 1, n_seqs)
                   : (long long)n_seqs * ((group + (1 << shift) - 1) >> shift);
}
// ... slot u, of sequence s (without offsets: of sequence u / tiles of a row)
__host__ __device__ inline Tile tile_of(const SeqArgs& q, int pt, int group, int shift, bool causal, const Seq& sp,
                                        long long u) {
    Tile t = {-1, 0, 0, 0, 0, 0, 0};
    const int s = sp.s;
    if (s < 0) return t;
    const long long j = q.offsets ? u - slot_base(sp.off, group, shift, 1, s)
                                  : u - (long long)s * ((group + (1 << shift) - 1) >> shift);
    const long long first = j << shift, left = (long long)sp.n * group - first;
    if (left <= 0) return t;
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

#ifdef __HIPCC__
// The sequence whose slots hold slot u (every lane of a wavefront calls, with the same u).  Its offsets and
// place are loaded along with the search: a chain of loads is what small calls wait for.
__device__ __forceinline__ Seq find_seq(const SeqArgs& q, int mul, int shift, int add, long long u) {
    Seq r = {-1, 0, 0, 0, 0};
    for (int b = 0; b < q.n_seqs; b += 64) {
        const int s = b + (threadIdx.x & 63), c = s < q.n_seqs ? s : q.n_seqs - 1;
        const int off = q.offsets[c], next = q.offsets[c + 1], at = q.at[c];
        const unsigned long long before = __ballot(s < q.n_seqs && slot_base(off, mul, shift, add, s) <= u);
        if (!before) break;
        const int k = __popcll(before) - 1;
        r = seq_from(q, b + k, __builtin_amdgcn_readlane(off, k), __builtin_amdgcn_readlane(next, k),
                     __builtin_amdgcn_readlane(at, k));
        if (k < 63) break;
    }
    return r;
}
#endif

}  // namespace dv

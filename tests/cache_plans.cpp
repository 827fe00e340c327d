// Where rows of the 8-bit cache's operators go (host code of their header) under C names, for
// test_cache.py.
#include "cache_plan.h"

using namespace dv;

// The sequence that owns slot u: the first whose slots reach past it (count: the slots of one).
template <class Count>
static Seq owner(const SeqArgs& q, const Count& count, int u) {
    int base = 0;
    for (int s = 0; s < q.n_seqs; ++s) {
        Seq sp = seq_from(q, s, q.offsets[s], q.offsets[s + 1], q.at[s]);
        sp.slot0 = base;
        base += count(sp);
        if (u < base) return sp;
    }
    return {-1, 0, 0, 0, 0};
}

extern "C" {

// For every slot of a write or read: sequence, page, first row, first place, places (5 ints a slot).
// Returns the slots.
int t_page_parts(const int* table, int table_pages, int pages, const int* offsets, int n_seqs, int rows,
                 const int* starts, int pt, int* out) {
    const SeqArgs q = {n_seqs, table_pages, rows, table, offsets, starts};
    const int slots = (int)page_slots(offsets != nullptr, n_seqs, rows, page_shift(pt));
    for (int u = 0; u < slots; ++u) {
        const Seq s = offsets ? owner(q, [&](const Seq& x) { return part_count(x, page_shift(pt)); }, u) : seq_of(q, u);
        const PagePart p = part_at(q, pt, pages, s, u);
        const int v[] = {s.s, p.page, p.row0, p.slot0, p.n};
        for (int i = 0; i < 5; ++i) out[5 * u + i] = v[i];
    }
    return slots;
}

// For every tile slot of an attention call: sequence, first row, first packed row, packed rows, keys
// of the sequence, keys the tile sees (6 ints a slot).
int t_tiles(int table_pages, const int* offsets, int n_seqs, int rows, const int* lengths, int pt, int group,
            int shift, int causal, int* out) {
    const SeqArgs q = {n_seqs, table_pages, rows, nullptr, offsets, lengths};
    const int slots = (int)tile_slots(offsets != nullptr, n_seqs, rows, group, shift);
    for (int u = 0; u < slots; ++u) {
        const Seq s = offsets ? owner(q, [&](const Seq& x) { return tile_count(x, group, shift); }, u)
                              : seq_of(q, u / ((group + (1 << shift) - 1) >> shift));
        const Tile t = tile_of(q, pt, group, shift, causal != 0, s, u);
        const int v[] = {t.seq, t.row0, t.first, t.rows, t.len, t.end};
        for (int i = 0; i < 6; ++i) out[6 * u + i] = v[i];
    }
    return slots;
}

// An attention call's plan: route; out: small tiles' chunk, splits, slots, then large ones', workspace bytes.
int t_attn_plan(int bf16, int n_seqs, int rows, int offsets, int max_rows, int table_pages, int page_tokens,
                int kv_heads, int q_heads, int head_dim, int cus, long long* out) {
    const CacheAttnPlan p = cache_attn_plan(bf16 != 0, n_seqs, rows, offsets != 0, max_rows, table_pages,
                                            page_tokens, kv_heads, q_heads, head_dim, cus);
    const long long v[] = {p.few.chunk, p.few.splits, p.few.slots, p.many.chunk, p.many.splits, p.many.slots,
                           (long long)p.bytes};
    for (int i = 0; i < 7; ++i) out[i] = v[i];
    return p.route;
}

}  // extern "C"

// Where rows of the 8-bit cache's operators go (host code of their header) under C names, for
// test_cache.py.
#include "cache_plan.h"

using namespace dv;

extern "C" {

// For every slot of a write or read: sequence, page, first row, first place, places (5 ints a slot).
// Returns the slots; the sequence of a slot is the last whose base is not above it.
int t_page_parts(const int* table, int table_pages, int pages, const int* offsets, int n_seqs, int rows,
                 const int* starts, int pt, int* out) {
    const SeqArgs q = {n_seqs, table_pages, rows, table, offsets, starts};
    const int slots = (int)page_slots(offsets != nullptr, n_seqs, rows, page_shift(pt));
    for (int u = 0; u < slots; ++u) {
        int s = offsets ? -1 : u;
        if (offsets)
            while (s + 1 < n_seqs && slot_base(offsets[s + 1], 1, page_shift(pt), 2, s + 1) <= u) ++s;
        const PagePart p = part_at(q, pt, pages, seq_of(q, s), u);
        const int v[] = {s, p.page, p.row0, p.slot0, p.n};
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
        int s = offsets ? -1 : u / ((group + (1 << shift) - 1) >> shift);
        if (offsets)
            while (s + 1 < n_seqs && slot_base(offsets[s + 1], group, shift, 1, s + 1) <= u) ++s;
        const Tile t = tile_of(q, pt, group, shift, causal != 0, seq_of(q, s), u);
        const int v[] = {t.seq, t.row0, t.first, t.rows, t.len, t.end};
        for (int i = 0; i < 6; ++i) out[6 * u + i] = v[i];
    }
    return slots;
}

}  // extern "C"

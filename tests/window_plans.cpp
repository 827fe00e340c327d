// Which keys tiles of attention with a window take, and how such calls and those of shared prefixes are cut, under C names
// (host code of the header), for test_window.py.
#include "cache_plan.h"

using namespace dv;

extern "C" {

// Sequence of n rows and `length` keys: for every tile first packed row, packed rows, keys it sees, first key left out, keys
// left out (5 ints a tile).  Returns the tiles.
int t_window_tiles(int n, int length, int table_pages, int pt, int group, int shift, int causal, int window, int sinks, int* out) {
    const int offsets[2] = {0, n}, at[1] = {length};
    const SeqArgs q = {1, table_pages, n, nullptr, offsets, at};
    const Seq s = seq_from(q, 0, 0, n, length);
    const int tiles = tile_count(s, group, shift);
    for (int u = 0; u < tiles; ++u) {
        Tile t = tile_of(q, pt, group, shift, causal != 0, s, u);
        leave_out(t, group, causal != 0, window, sinks);
        const int v[] = {t.first, t.rows, t.end, t.skip0, t.left_out};
        for (int i = 0; i < 5; ++i) out[5 * u + i] = v[i];
    }
    return tiles;
}

// route; out: small tiles' chunk, splits, slots, large ones', workspace bytes
int t_window_plan(int bf16, int n_seqs, int rows, int offsets, int max_rows, int table_pages, int page_tokens, int kv_heads,
                  int q_heads, int head_dim, int cus, int window, int sinks, long long* out) {
    const CacheAttnPlan p = cache_attn_plan(bf16 != 0, n_seqs, rows, offsets != 0, max_rows, table_pages, page_tokens, kv_heads,
                                            q_heads, head_dim, cus, window, sinks);
    const long long v[] = {p.few.chunk, p.few.splits, p.few.slots, p.many.chunk, p.many.splits, p.many.slots, (long long)p.bytes};
    for (int i = 0; i < 7; ++i) out[i] = v[i];
    return p.route;
}

// The plans of a call with shared prefixes, one after the other; then the bytes and blocks of both,
// and whether the first takes the prefixes too.
void t_shared_plan(int bf16, int n_seqs, int rows, int offsets, int max_rows, int table_pages, int n_groups, int prefix_table_pages,
                   int page_tokens, int kv_heads, int q_heads, int head_dim, int cus, long long* out) {
    const CacheSharedPlan p = cache_shared_plan(bf16 != 0, n_seqs, rows, offsets != 0, max_rows, table_pages, n_groups,
                                                prefix_table_pages, page_tokens, kv_heads, q_heads, head_dim, cus);
    for (const CacheAttnPlan* x : {&p.own, &p.prefix}) {
        const long long v[] = {x->route, x->few.chunk, x->few.splits, x->few.slots, x->many.chunk, x->many.splits, x->many.slots,
                               (long long)x->bytes};
        for (long long y : v) *out++ = y;
    }
    out[0] = (long long)p.bytes;
    out[1] = p.blocks;
    out[2] = p.behind;
}

}  // extern "C"

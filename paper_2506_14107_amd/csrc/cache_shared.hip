// Attention over the paged 8-bit cache for sequences behind a prefix that a group of them shares.  The rows of a group lie together,
// so that tiles of them take the prefix's keys as one sequence's, read once for all; each sequence's own keys are taken by tiles of its
// rows; a row's outputs are joined from the splits of both.
#include "cache_attn.h"

namespace dv {

namespace {

template <int DH, bool BF>
__global__ __launch_bounds__(256, 2) void cache_part_k(CacheAttnArgs a) {
    attend_small<DH, BF, PART>(a);
}
template <int DH, bool ONE>
__global__ __launch_bounds__(256, 2) void cache_part_tile_k(CacheAttnArgs a) {
    attend_large<DH, ONE, PART>(a);
}
struct PartKeys {
    template <int DH, bool BF>
    static constexpr auto small() { return cache_part_k<DH, BF>; }
    template <int DH, bool ONE>
    static constexpr auto large() { return cache_part_tile_k<DH, ONE>; }
};

// A tile's partial results in the splits of its cut.
struct Splits {
    const float* part;   // of the first split, this head's
    size_t per;
    int n, row, rows;    // splits, the row in the tile, the tile's rows
};
// Where a row's partial results over its prefix lie: group g has the row's sequence.
struct Prefix {
    int g, row0, n, len, few0, many0;   // (its first slots of small and large tiles)
};
__device__ __forceinline__ Prefix prefix_of(const SeqArgs& q, int seq, int G, int few_rows_, int route) {
    const int lane = threadIdx.x & 63;
    int few = 0, many = 0;
    for (int b = 0; b < q.n_seqs; b += 64) {
        const int g = b + lane, c = min(g, q.n_seqs - 1);
        const Seq s = group_from(q, c);
        const int from = q.groups ? q.groups[c] : 0, to = q.groups ? q.groups[c + 1] : q.grouped;
        const bool small = route == ATTN_FEW || (route == ATTN_BOTH && (long long)s.n * G <= few_rows_);
        const int nf = g < q.n_seqs && small ? tile_count(s, G, TS) : 0, nm = g < q.n_seqs && !small ? tile_count(s, G, LS) : 0;
        const int uf = sum_up(nf), um = sum_up(nm);
        const uint64_t here = __ballot(g < q.n_seqs && from <= seq && seq < to);
        if (here) {
            const int k = __ffsll((unsigned long long)here) - 1;
            return {b + k, __builtin_amdgcn_readlane(s.row0, k), __builtin_amdgcn_readlane(s.n, k), __builtin_amdgcn_readlane(s.at, k),
                    few + __builtin_amdgcn_readlane(uf - nf, k), many + __builtin_amdgcn_readlane(um - nm, k)};
        }
        few += __builtin_amdgcn_readlane(uf, 63), many += __builtin_amdgcn_readlane(um, 63);
    }
    return {-1, 0, 0, 0, 0, 0};
}

// Joins a tile's rows: the splits of their own keys (a) and of their group's prefix (pre).  A wavefront takes a row.
template <bool BF, int SHIFT>
__global__ __launch_bounds__(256) void cache_shared_join_k(CacheAttnArgs a, CacheAttnArgs pre) {
    constexpr int R = 1 << SHIFT;
    __shared__ f32x4 s_x[256];
    const CacheAttnCut& cut = SHIFT == TS ? a.few : a.many;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int H = a.c.kv_heads, DH = a.c.head_dim, G = a.q_heads / H;
    const int h = blockIdx.x % H;
    const long long u = blockIdx.x / H;
    const Tile t = tile_at<SHIFT, PART>(a, u);
    if (t.seq < 0) return;
    const float sl2 = exponent_factor(a.scale);
    const int limit = few_rows(DH);
    const Prefix p = prefix_of(pre.seq, t.seq, G, limit, pre.route);
    const bool small = pre.route == ATTN_FEW || (pre.route == ATTN_BOTH && (long long)p.n * G <= limit);
    const int lanes = DH / 4, groups = 64 / lanes;        // of a wavefront
    const int ch = lane % lanes * 4, grp = lane / lanes;
    for (int row0 = blockIdx.y * 4; row0 < t.rows; row0 += gridDim.y * 4) {
        const int row = min(row0 + wave, t.rows - 1), pr = t.first + row;
        Splits list[2];
        list[0] = {cut.part + ((size_t)u * H + h) * cut.splits * part_floats(R, DH), part_floats(R, DH),
                   max(1, (t.end + cut.chunk - 1) / cut.chunk), row, R};
        list[1] = {nullptr, 0, 0, 0, 0};
        if (p.g >= 0) {
            const CacheAttnCut& pc = small ? pre.few : pre.many;
            const int shift = small ? TS : LS;
            const long long at = ((long long)t.row0 + pr / G - p.row0) * G + pr % G, slot = (small ? p.few0 : p.many0) + (at >> shift);
            const int len = (int)min((long long)max(p.len, 0), (long long)pre.seq.table_pages * a.c.page_tokens);
            const size_t per = part_floats(1 << shift, DH);
            if (at >= 0 && slot < pc.slots)
                list[1] = {pc.part + ((size_t)slot * H + h) * pc.splits * per, per, max(1, (len + pc.chunk - 1) / pc.chunk),
                           (int)(at & ((1 << shift) - 1)), 1 << shift};
        }
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 2; ++w)
            for (int s = lane; s < list[w].n; s += 64)
                top = fmaxf(top, list[w].part[s * list[w].per + list[w].rows * DH + list[w].row]);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            const Splits& l = list[v];
            for (int s0 = 0; s0 < l.n; s0 += 64) {
                const int s = s0 + lane, n = min(64, l.n - s0);
                float w = 0.f;
                if (s < l.n) {
                    const float* ml = l.part + s * l.per + l.rows * DH + l.row;
                    w = __builtin_amdgcn_exp2f((ml[0] - ref) * sl2);
                    sum += ml[l.rows] * w;
                }
                const float* from = l.part + s0 * l.per + l.row * DH + ch;
                for (int i = 0; i < n; i += groups) {
                    const int j = i + grp;
                    const float wj = __shfl(w, j & 63, 64);
                    if (grp < groups && j < n) x += *(const f32x4*)(from + j * l.per) * wj;
                }
            }
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
        s_x[tid] = x;
        __syncthreads();
        if (grp == 0 && row0 + wave < t.rows) {
            for (int k = 1; k < groups; ++k) x += s_x[wave * 64 + k * lanes + lane];
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            store4<BF>(a.out, (size_t)(t.row0 + pr / G) * a.o_stride + (size_t)(h * G + pr % G) * DH + ch, x * inv);
        }
        __syncthreads();
    }
}

template <bool BF, int SHIFT>
void launch_shared_join(const CacheAttnArgs& a, const CacheAttnArgs& pre, const CacheAttnCut& c, hipStream_t s) {
    const dim3 grid((unsigned)(c.slots * a.c.kv_heads), (unsigned)((c.tile_rows + 3) / 4));
    cache_shared_join_k<BF, SHIFT><<<grid, 256, 0, s>>>(a, pre);
}

}  // namespace

void launch_cache_shared(bool bf, CacheAttnArgs a, const SeqArgs& prefix, const CacheAttnPlan& p, const CacheAttnPlan& pre,
                         float* workspace, hipStream_t s) {
    CacheAttnArgs b = a;
    b.seq = prefix;
    b.causal = 0;
    set_plan(a, p, workspace);
    set_plan(b, pre, workspace + p.bytes / sizeof(float));
    launch_parts<PartKeys>(bf, b, s);
    launch_parts<PartKeys>(bf, a, s);
    if (a.route != ATTN_MANY) bf ? launch_shared_join<true, TS>(a, b, a.few, s) : launch_shared_join<false, TS>(a, b, a.few, s);
    if (a.route != ATTN_FEW) launch_shared_join<true, LS>(a, b, a.many, s);
}

}  // namespace dv

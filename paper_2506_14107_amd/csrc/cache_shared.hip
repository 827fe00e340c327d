// Attention over the paged 8-bit cache for sequences behind a prefix that a group of them shares.  The rows of a group lie together,
// so that tiles of them take the prefix's keys as one sequence's, read once for all; each sequence's own keys are taken by tiles of its
// rows; a row's outputs are joined from the splits of both.  One launch takes both parts (two, one behind the other: 208 us of a call
// with small tiles, 64 answers of up to 700 own keys behind 50,001, 8 heads of 128 with 4 queries each); with large tiles 91: the
// matrix work on the prefix 51, starting, own keys and 34 MB of partial results the rest of 85, the join 11.  8 answers behind
// 100,003 keys read the prefix at 4 TB/s (51 us and 8), two small tiles of 16 rows sharing it in a cache; one sequence's tiles read at 5.7.
#include "cache_attn.h"

namespace dv {

namespace {

// Both parts of a call in one launch: blocks of the prefixes' tiles, then of the sequences' own, large ones first.
struct SharedArgs {
    CacheAttnArgs part[2];   // the sequences' own keys, the prefixes'
    unsigned first[4];       // first block behind the prefixes' large tiles, their small ones, the sequences' large ones, all
};
struct Block {
    int part;
    bool large;
    unsigned bx, by;
};
__device__ __forceinline__ Block block_of(const SharedArgs& a) {
    const unsigned b = blockIdx.x;
    const int i = (b >= a.first[0]) + (b >= a.first[1]) + (b >= a.first[2]);
    const bool large = i % 2 == 0;
    const CacheAttnArgs& x = a.part[i < 2];
    const unsigned r = i ? b - a.first[i - 1] : b, wide = (unsigned)((large ? x.many.slots : x.few.slots) * x.c.kv_heads);
    return {i < 2, large, r % wide, r / wide};
}
template <int DH, bool ONE>
__global__ __launch_bounds__(256, 2) void cache_shared_k(SharedArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    const Block b = block_of(a);
    const CacheAttnArgs& x = a.part[b.part];
    if (b.large) attend_large<DH, ONE, PART>(x, *(Lds<DH>*)smem, b.bx, b.by);
    else attend_small<DH, true, PART>(x, *(Small<DH>*)smem, b.bx, b.by);
}
template <int DH, bool BF>
__global__ __launch_bounds__(256, 2) void cache_shared_small_k(SharedArgs a) {
    __shared__ Small<DH> lds;
    const Block b = block_of(a);
    const CacheAttnArgs& x = a.part[b.part];
    attend_small<DH, BF, PART>(x, lds, b.bx, b.by);
}

// Where a row's partial results over its prefix lie: group g has the row's sequence.
struct Prefix {
    int g, row0, n, len, few0, many0;   // (its first slots of small and large tiles)
};
__device__ __forceinline__ Prefix prefix_of(const SeqArgs& q, const GroupArgs& by, int seq, int G, int few_rows_, int route) {
    const int lane = threadIdx.x & 63;
    int few = 0, many = 0;
    for (int b = 0; b < q.n_seqs; b += 64) {
        const int g = b + lane, c = min(g, q.n_seqs - 1);
        const Seq s = group_from(q, by, c);
        const int from = by.first ? by.first[c] : 0, to = by.first ? by.first[c + 1] : by.n;
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

// The partial results of a tile's rows over their own keys and over their group's prefix, one list of splits.
struct Parts {
    const float *own, *pre;      // of the tile and head; of the head in the prefix's tiles
    size_t per0, per1, tiles1;   // floats of a split, of a prefix's tile of all heads
    int n0, n1, R, shift;
    long long at0, slots;        // the tile's first packed row in its group (below 0: none), tiles of prefixes
    int slot0, dh;
    // of packed row `row` of the tile: where split s has its output and its maximum, how many splits there are
    __device__ __forceinline__ bool behind(int row) const { return at0 >= 0 && slot0 + ((at0 + row) >> shift) < slots; }
    __device__ __forceinline__ int splits(int row) const { return n0 + (behind(row) ? n1 : 0); }
    __device__ __forceinline__ const float* split(int s, int row) const {
        return s < n0 ? own + s * per0 : pre + (slot0 + ((at0 + row) >> shift)) * tiles1 + (s - n0) * per1;
    }
    __device__ __forceinline__ const float* output(int s, int row) const {
        return split(s, row) + (s < n0 ? row : (int)((at0 + row) & ((1 << shift) - 1))) * dh;
    }
    __device__ __forceinline__ const float* maximum(int s, int row) const {   // the sum lies `rows(s)` floats behind
        return split(s, row) + (s < n0 ? R * dh + row : (dh << shift) + (int)((at0 + row) & ((1 << shift) - 1)));
    }
    __device__ __forceinline__ int rows(int s) const { return s < n0 ? R : 1 << shift; }
};
template <int SHIFT>
__device__ __forceinline__ Parts parts_of(const CacheAttnArgs& a, const CacheAttnArgs& pre, const Tile& t, long long u, int h) {
    const int H = a.c.kv_heads, DH = a.c.head_dim, G = a.q_heads / H, limit = few_rows(DH);
    const CacheAttnCut& cut = SHIFT == TS ? a.few : a.many;
    const Prefix p = prefix_of(pre.seq, pre.groups, t.seq, G, limit, pre.route);
    const bool small = pre.route == ATTN_FEW || (pre.route == ATTN_BOTH && (long long)p.n * G <= limit);
    const CacheAttnCut& pc = small ? pre.few : pre.many;
    const int len = (int)min((long long)max(p.len, 0), (long long)pre.seq.table_pages * a.c.page_tokens);
    Parts x;
    x.shift = small ? TS : LS;
    x.R = 1 << SHIFT;
    x.dh = DH;
    x.per0 = part_floats(x.R, DH), x.per1 = part_floats(1 << x.shift, DH);
    x.own = cut.part + ((size_t)u * H + h) * cut.splits * x.per0;
    x.tiles1 = (size_t)H * pc.splits * x.per1;
    x.pre = pc.part + (size_t)h * pc.splits * x.per1;
    x.n0 = max(1, (t.end + cut.chunk - 1) / cut.chunk);
    x.n1 = max(1, (len + pc.chunk - 1) / pc.chunk);
    x.at0 = p.g < 0 ? -1 : ((long long)t.row0 - p.row0) * G + t.first;
    x.slots = pc.slots;
    x.slot0 = small ? p.few0 : p.many0;
    return x;
}
template <bool BF>
__device__ __forceinline__ void store_row(const CacheAttnArgs& a, const Tile& t, int h, int row, int ch, f32x4 x, float sum) {
    const int pr = t.first + row, G = a.q_heads / a.c.kv_heads;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    store4<BF>(a.out, (size_t)(t.row0 + pr / G) * a.o_stride + (size_t)(h * G + pr % G) * a.c.head_dim + ch, x * inv);
}

// Joins a tile's rows where no row has more than FEW splits: dh / 4 lanes take a row and hold all of it (401 fp32 rows of 16 heads of 64 in 3
// splits: 5 us; a wavefront a row 12).
constexpr int FEW = 8;
template <bool BF, int SHIFT>
__global__ __launch_bounds__(256) void cache_shared_join_few_k(SharedArgs args) {
    const CacheAttnArgs &a = args.part[0], &pre = args.part[1];
    const int tid = threadIdx.x, lane = tid & 63, H = a.c.kv_heads, h = blockIdx.x % H;
    const long long u = blockIdx.x / H;
    const Tile t = tile_at<SHIFT, PART>(a, u);
    if (t.seq < 0) return;
    const float sl2 = exponent_factor(a.scale);
    const Parts p = parts_of<SHIFT>(a, pre, t, u, h);
    const int lanes = a.c.head_dim / 4, groups = 64 / lanes, ch = lane % lanes * 4, rows = 4 * groups;   // of a block
    if (lane / lanes >= groups) return;
    for (int row = blockIdx.y * rows + (tid >> 6) * groups + lane / lanes; row < t.rows; row += gridDim.y * rows) {
        const int total = min(p.splits(row), FEW);
        f32x4 y[FEW];
        float m[FEW], l[FEW], top = -INFINITY;
#pragma unroll
        for (int s = 0; s < FEW; ++s) {
            if (s >= total) continue;
            const float* at = p.maximum(s, row);
            m[s] = at[0], l[s] = at[p.rows(s)];
            y[s] = *(const f32x4*)(p.output(s, row) + ch);
        }
#pragma unroll
        for (int s = 0; s < FEW; ++s) top = s < total ? fmaxf(top, m[s]) : top;
        const float ref = top == -INFINITY ? 0.f : top;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < FEW; ++s) {
            if (s >= total) continue;
            const float w = __builtin_amdgcn_exp2f((m[s] - ref) * sl2);
            sum += l[s] * w;
            x += y[s] * w;
        }
        store_row<BF>(a, t, h, row, ch, x, sum);
    }
}

// ... any number of splits: a row takes W wavefronts of a block; every lane weighs one split in 64, then lanes go over the channels
// and groups of lanes over the splits.
template <bool BF, int SHIFT, int W>
__global__ __launch_bounds__(256) void cache_shared_join_k(SharedArgs args) {
    constexpr int ROWS = 4 / W, AHEAD = 8;   // loads asked for together
    __shared__ f32x4 s_x[256];
    const CacheAttnArgs &a = args.part[0], &pre = args.part[1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, H = a.c.kv_heads, h = blockIdx.x % H;
    const long long u = blockIdx.x / H;
    const Tile t = tile_at<SHIFT, PART>(a, u);
    if (t.seq < 0) return;
    const float sl2 = exponent_factor(a.scale);
    const Parts p = parts_of<SHIFT>(a, pre, t, u, h);
    const int lanes = a.c.head_dim / 4, groups = 64 / lanes;        // of a wavefront
    const int ch = lane % lanes * 4, grp = lane / lanes;
    // one round, unless a sequence has more rows than it was said to have
    for (int row0 = blockIdx.y * ROWS; row0 < t.rows; row0 += gridDim.y * ROWS) {
        const int row = min(row0 + wave / W, t.rows - 1), total = p.splits(row);
        // the first splits' results are asked for before their weights are known
        const int s1 = min(lane, total - 1), step = W * groups;
        const float *m1 = p.maximum(s1, row), m = lane < total ? m1[0] : -INFINITY, l = m1[p.rows(s1)];
        f32x4 y[AHEAD];
        auto ask = [&](int i) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) y[k] = *(const f32x4*)(p.output(min(i + k * step, total - 1), row) + ch);
        };
        const int mine = wave % W * groups + grp;   // the lane's first split
        ask(mine);
        float top = m;
        for (int s = lane + 64; s < total; s += 64) top = fmaxf(top, *p.maximum(s, row));
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
        const float ref = top == -INFINITY ? 0.f : top;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f, w = lane < total ? __builtin_amdgcn_exp2f((m - ref) * sl2) : 0.f;
        if (lane < total) sum = l * w;
        for (int s0 = 0;;) {
            const int n = min(64, total - s0);
            for (int i = wave % W * groups; i < n; i += step * AHEAD) {
                if (s0 + i > wave % W * groups) ask(s0 + i + grp);
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int j = i + k * step + grp;
                    const float wj = __shfl(w, j & 63, 64);
                    if (grp < groups && j < n) x += y[k] * wj;
                }
            }
            if ((s0 += 64) >= total) break;
            const int s = min(s0 + lane, total - 1);
            const float* at = p.maximum(s, row);
            w = s0 + lane < total ? __builtin_amdgcn_exp2f((at[0] - ref) * sl2) : 0.f;
            if (s0 + lane < total) sum += at[p.rows(s)] * w;
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
        s_x[tid] = x;
        __syncthreads();
        if (wave % W == 0 && grp == 0 && row0 + wave / W < t.rows) {
            for (int v = 0; v < W; ++v)
                for (int k = v == 0; k < groups; ++k) x += s_x[(wave + v) * 64 + k * lanes + lane];
            store_row<BF>(a, t, h, row, ch, x, sum);
        }
        __syncthreads();
    }
}

template <bool BF, int SHIFT>
void launch_shared_join(const SharedArgs& a, const CacheAttnCut& c, hipStream_t s) {
    const CacheAttnArgs& pre = a.part[1];
    const int splits = c.splits + std::max(pre.route == ATTN_MANY ? 1 : pre.few.splits, pre.route == ATTN_FEW ? 1 : pre.many.splits);
    const unsigned tiles = (unsigned)(c.slots * a.part[0].c.kv_heads);
    const int rows = 4 * (64 / (a.part[0].c.head_dim / 4));
    if (splits <= FEW) cache_shared_join_few_k<BF, SHIFT><<<dim3(tiles, (c.tile_rows + rows - 1) / rows), 256, 0, s>>>(a);
    // us of 640 tiles of 4 rows in 33 splits: 11 with one wavefront a row, 17 with four; of 80 in 33: 8, 7
    else if (splits <= 64) cache_shared_join_k<BF, SHIFT, 1><<<dim3(tiles, (c.tile_rows + 3) / 4), 256, 0, s>>>(a);
    else cache_shared_join_k<BF, SHIFT, 4><<<dim3(tiles, c.tile_rows), 256, 0, s>>>(a);
}

template <int DH>
void launch_shared(bool bf, const SharedArgs& a, hipStream_t s) {
    const dim3 grid(a.first[3]);
    if (a.part[0].route == ATTN_FEW && a.part[1].route == ATTN_FEW) {
        bf ? cache_shared_small_k<DH, true><<<grid, 256, 0, s>>>(a) : cache_shared_small_k<DH, false><<<grid, 256, 0, s>>>(a);
        return;
    }
    constexpr size_t lds = sizeof(Lds<DH>) > sizeof(Small<DH>) ? sizeof(Lds<DH>) : sizeof(Small<DH>);
    auto go = [&](auto one) {
        constexpr auto k = cache_shared_k<DH, decltype(one)::value>;
        static const bool ok = allow_lds((const void*)k, lds);
        (void)ok;
        k<<<grid, 256, lds, s>>>(a);
    };
    if (a.part[0].c.page_tokens >= STEP) go(std::true_type());
    else go(std::false_type());
}

}  // namespace

void launch_cache_shared(bool bf, CacheAttnArgs a, const CacheAttnPlan& p, const CacheAttnPlan& pre, float* workspace,
                         hipStream_t s) {
    SharedArgs x{{a, a}, {}};
    x.part[1].seq = a.front;
    x.part[1].groups.on = 1;
    x.part[1].causal = 0;
    set_plan(x.part[0], p, workspace);
    set_plan(x.part[1], pre, workspace + p.bytes / sizeof(float));
    unsigned first = 0;
    for (int i = 0; i < 4; ++i) {
        const CacheAttnArgs& y = x.part[i < 2];
        const CacheAttnCut& c = i % 2 ? y.few : y.many;
        if (y.route != (i % 2 ? ATTN_MANY : ATTN_FEW)) first += (unsigned)(c.slots * y.c.kv_heads * c.splits);
        x.first[i] = first;
    }
    switch (a.c.head_dim) {
        case 16: launch_shared<16>(bf, x, s); break;
        case 32: launch_shared<32>(bf, x, s); break;
        case 48: launch_shared<48>(bf, x, s); break;
        case 64: launch_shared<64>(bf, x, s); break;
        case 80: launch_shared<80>(bf, x, s); break;
        case 96: launch_shared<96>(bf, x, s); break;
        case 112: launch_shared<112>(bf, x, s); break;
        default: launch_shared<128>(bf, x, s); break;
    }
    if (p.route != ATTN_MANY) bf ? launch_shared_join<true, TS>(x, p.few, s) : launch_shared_join<false, TS>(x, p.few, s);
    if (p.route != ATTN_FEW) launch_shared_join<true, LS>(x, p.many, s);
}

}  // namespace dv

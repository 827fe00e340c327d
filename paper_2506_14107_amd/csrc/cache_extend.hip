// A batch's next rows: where they go, and the pages that hold them.
//
// Sums over the sequences give each its first row and its place in the ring of free pages; rows and pages then find their
// sequence by bisection of those sums.  Everything is whole numbers, so that the order of the sums does not matter.  A
// call moves little (20 bytes a row, 8 a page, 20 a sequence) and is bound by its chain of dependent loads, so it
// is one launch: every block sums over all sequences by itself (1024 at once, one a thread) instead of waiting for a block that
// does, and then takes its share of the rows and of the new pages, or of the pages that go back.  A step of 256
// sequences 5.4 us, 100,003 rows of 1000 prompts in pages of 16, a hundred of which end, 11 (blocks of 256 threads, with rows, pages and
// entries that go back found one by one: 7.1 and 20.6).
#include "cache_plan.h"

namespace dv {

namespace {

constexpr int XT = 1024, WAVES = XT / 64;   // threads of a block, and sequences that it sums at once

struct Next {
    int len, count;    // places, new rows (below 0: the sequence ends)
    int held, want;    // pages it has in its table, pages it needs
    bool fits;         // the table holds its new places
};
__device__ __forceinline__ Next next_of(const ExtendArgs& a, int s) {
    Next x = {0, 0, 0, 0, true};
    if (s >= a.n_seqs) return x;
    x.len = max(a.lengths[s], 0);
    x.count = a.counts[s];
    const int round = (1 << a.shift) - 1;
    const long long held = ((long long)x.len + round) >> a.shift;
    const long long after = ((long long)x.len + max(x.count, 0) + round) >> a.shift;
    x.fits = x.count <= 0 || after <= a.table_pages;
    x.held = (int)min(held, (long long)a.table_pages);
    x.want = x.fits && x.count > 0 ? (int)(after - held) : 0;
    return x;
}

// x of the threads up to this one, summed, and of all.  s: WAVES numbers of LDS, free again after the next barrier.
__device__ __forceinline__ int block_sum_up(int x, int* s, int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int up = sum_up(x);
    if (lane == 63) s[wave] = up;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? s[w] : 0;
        all += s[w];
    }
    return before + up;
}

// The i with from[i] <= x < from[i + 1], of n ranges that rise.
__device__ __forceinline__ int range_of(const int* from, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (from[mid + 1] > x) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

struct Ring {
    int room, get, put;   // free pages; the places of the next one to take and to give
};
__device__ __forceinline__ Ring ring_of(const ExtendArgs& a) {
    const long long taken = a.cursor[0], given = a.cursor[1], room = min(max(given - taken, 0ll), (long long)a.pages);
    auto at = [&](long long x) { const long long r = x % a.pages; return (int)(r < 0 ? r + a.pages : r); };
    return {(int)room, at(taken), at(given)};
}

// Rows and new pages, and with the first block what is written of each sequence.
__device__ __forceinline__ void rows_and_pages(const ExtendArgs& a, const Ring& ring, int* s_off, int* s_base, int* s_len,
                                               int* s_sum) {
    const int tid = threadIdx.x, mask = (1 << a.shift) - 1;
    const long long stride = (long long)a.row_blocks * XT;
    __shared__ int s_got;
    if (tid == 0) s_got = 0;
    int rows0 = 0, pages0 = 0;
    for (int s0 = 0; s0 < a.n_seqs; s0 += XT) {
        const int s = s0 + tid;
        const Next x = next_of(a, s);
        const int fresh = max(x.count, 0);
        int all_rows, all_pages;
        const int off = rows0 + block_sum_up(fresh, s_sum, all_rows) - fresh;
        const int base = pages0 + block_sum_up(x.want, s_sum + WAVES, all_pages) - x.want;
        const bool served = x.fits && (x.want == 0 || base + x.want <= ring.room);
        s_off[tid] = off, s_base[tid] = base, s_len[tid] = served ? x.len : ~x.len;
        rows0 += all_rows, pages0 += all_pages;
        if (tid == XT - 1) s_off[XT] = rows0, s_base[XT] = pages0;
        if (blockIdx.x == 0 && s < a.n_seqs) {
            a.offsets[s] = off;
            a.starts[s] = served && x.count >= 0 ? x.len : -1;
            a.lengths_out[s] = x.count < 0 ? 0 : served ? x.len + fresh : x.len;
            if (s == a.n_seqs - 1) a.offsets[a.n_seqs] = off + fresh;
            if (served && x.want) atomicMax(&s_got, base + x.want);   // (of LDS; the order does not matter)
        }
        __syncthreads();
        // the first of the thread's rows (r + k stride) that is not before the chunk
        auto first = [&](long long from) {
            const long long r = (long long)blockIdx.x * XT + tid;
            return r >= from ? r : r + (from - r + stride - 1) / stride * stride;
        };
        if (a.positions || a.slots)
            for (long long r = first(s_off[0]); r < min(rows0, a.rows); r += stride) {
                const int i = range_of(s_off, XT, (int)r), l = s_len[i], len = l < 0 ? ~l : l, p = len + (int)r - s_off[i];
                if (a.positions) {
                    int* to = a.positions + 3 * r;
                    to[0] = p, to[1] = p, to[2] = p;
                }
                if (a.slots) {
                    const int j = p >> a.shift, fresh = j - ((len + mask) >> a.shift), nth = s_base[i] + fresh;
                    int page = -1;   // (the bounds hold unless the sum of counts passes an int)
                    if (l >= 0 && fresh >= 0 && (unsigned)nth < (unsigned)ring.room)
                        page = a.ring[ring.get + nth < a.pages ? ring.get + nth : ring.get + nth - a.pages];
                    else if (l >= 0 && fresh < 0 && (unsigned)j < (unsigned)a.table_pages && s0 + i < a.n_seqs)
                        page = a.table[(long long)(s0 + i) * a.table_pages + j];
                    a.slots[r] = (unsigned)page < (unsigned)a.pages ? ((long long)page << a.shift) + (p & mask) : -1;
                }
            }
        for (long long u = first(s_base[0]); u < min(pages0, ring.room); u += stride) {
            const int i = range_of(s_base, XT, (int)u), at = ring.get + (int)u;
            if (s_len[i] < 0) continue;
            const int j = ((s_len[i] + mask) >> a.shift) + (int)u - s_base[i];
            a.table[(long long)(s0 + i) * a.table_pages + j] = a.ring[at < a.pages ? at : at - a.pages];
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) {
        a.cursor_out[0] = a.cursor[0] + s_got;
        a.cursor_out[2] = pages0 - s_got;
    }
}

// Pages of the sequences that end (entries that are pages of the cache), of the b-th part of these sequences in each chunk, behind
// those of the sequences before.  A wavefront takes four sequences at once, 64 entries of each.
__device__ __forceinline__ void pages_back(const ExtendArgs& a, const Ring& ring, int b, int* s_first, int* s_id, int* s_held,
                                           int* s_sum) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, free = a.pages - ring.room;
    long long place = 0;   // pages that went back so far
    for (int s0 = 0; s0 < a.n_seqs; s0 += XT) {
        const Next x = next_of(a, s0 + tid);
        const bool ends = x.count < 0;
        int n;
        const int nth = block_sum_up(ends, s_sum, n) - 1;
        if (ends) s_id[nth] = s0 + tid, s_held[nth] = x.held;
        __syncthreads();
        const int lo = (int)((long long)n * b / a.back_blocks), hi = (int)((long long)n * (b + 1) / a.back_blocks);
        // f(e, page, done) for every 64 entries of the e-th sequence that ends: the lane's page or -1, the pages so far; end(e, done)
        auto over = [&](int from, auto f, auto end) {
            for (int e0 = from + wave * 4; e0 < hi; e0 += WAVES * 4) {
                auto entry = [&](int e, int j) {
                    const int page = j < s_held[e] ? a.table[(long long)s_id[e] * a.table_pages + j] : -1;
                    return (unsigned)page < (unsigned)a.pages ? page : -1;
                };
                int page[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) page[k] = e0 + k < hi ? entry(e0 + k, lane) : -1;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int e = e0 + k;
                    if (e >= hi) continue;
                    int done = 0;
                    auto take = [&](int x) {
                        f(e, x, done);
                        done += __popcll(__ballot(x >= 0));
                    };
                    take(page[k]);
                    for (int j0 = 64; j0 < s_held[e]; j0 += 256) {
                        int more[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) more[i] = entry(e, j0 + i * 64 + lane);
#pragma unroll
                        for (int i = 0; i < 4; ++i) take(more[i]);
                    }
                    end(e, done);
                }
            }
        };
        over(0, [](int, int, int) {}, [&](int e, int done) {
            if (lane == 0) s_first[e] = done;
        });
        __syncthreads();
        int all;
        const int mine = tid < hi ? s_first[tid] : 0, upto = block_sum_up(mine, s_sum + WAVES, all);
        if (tid < hi) s_first[tid] = upto - mine;
        __syncthreads();
        over(lo, [&](int e, int page, int done) {
            const long long to = place + s_first[e] + done + __popcll(__ballot(page >= 0) & ((1ull << lane) - 1));
            if (page >= 0 && to < free) {
                const long long at = ring.put + to;
                a.ring[at < a.pages ? at : at - a.pages] = page;
            }
        }, [](int, int) {});
        // the sequences behind the part count for the chunks that follow
        if (hi < n && s0 + XT < a.n_seqs) {
            int rest = 0, total;
            for (int e = hi + wave; e < n; e += WAVES)
                for (int j = lane; j < s_held[e]; j += 64) {
                    const int page = a.table[(long long)s_id[e] * a.table_pages + j];
                    rest += (unsigned)page < (unsigned)a.pages;
                }
            __syncthreads();
            block_sum_up(rest, s_sum, total);
            all += total;
        }
        place += all;
        __syncthreads();
    }
    if (b == a.back_blocks - 1 && tid == 0) a.cursor_out[1] = a.cursor[1] + min(place, (long long)free);
}

__global__ __launch_bounds__(XT) void cache_extend_k(ExtendArgs a) {
    __shared__ int s_off[XT + 1], s_base[XT + 1], s_len[XT], s_sum[2 * WAVES];
    const Ring ring = ring_of(a);
    if ((int)blockIdx.x < a.row_blocks) rows_and_pages(a, ring, s_off, s_base, s_len, s_sum);
    else pages_back(a, ring, blockIdx.x - a.row_blocks, s_off, s_base, s_len, s_sum);
}

}  // namespace

void launch_cache_extend(ExtendArgs a, hipStream_t s) {
    a.row_blocks = (int)std::min<long long>(512, std::max(1ll, ((long long)a.rows + XT - 1) / XT));
    a.back_blocks = (int)std::min<long long>(16, ((long long)a.n_seqs * a.table_pages + 32767) / 32768);
    cache_extend_k<<<dim3((unsigned)(a.row_blocks + a.back_blocks)), XT, 0, s>>>(a);
}

}  // namespace dv

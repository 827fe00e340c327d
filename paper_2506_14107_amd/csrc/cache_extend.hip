// A batch's next rows: where they go, and the pages that hold them.
//
// Sums over the sequences give each its first row and its place in the ring of free pages; rows and pages then find their
// sequence by bisection of those sums.  Everything is whole numbers, so that the order of the sums does not matter.  A
// call moves little (20 bytes a row, 8 a page, 20 a sequence) and is bound by its chain of dependent loads, so it
// is one launch: every block sums over all sequences by itself (1024 at once, four a thread) instead of waiting for a block that
// does, and then takes its share of the rows and of the new pages, or of the pages that go back.
#include "cache_plan.h"

namespace dv {

namespace {

constexpr int XT = 256, PER = 4, CHUNK = XT * PER;   // threads; sequences of a thread and of a block at once

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

// x of the threads up to this one, summed, and of all.  s: XT / 64 numbers of LDS, free again after the next barrier.
__device__ __forceinline__ int block_sum_up(int x, int* s, int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int up = sum_up(x);
    if (lane == 63) s[wave] = up;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < XT / 64; ++w) {
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
    for (int s0 = 0; s0 < a.n_seqs; s0 += CHUNK) {
        Next x[PER];
        int rows = 0, pages = 0, all_rows, all_pages;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            x[k] = next_of(a, s0 + tid * PER + k);
            rows += max(x[k].count, 0), pages += x[k].want;
        }
        const int upto_rows = block_sum_up(rows, s_sum, all_rows), upto_pages = block_sum_up(pages, s_sum + XT / 64, all_pages);
        int off = rows0 + upto_rows - rows, base = pages0 + upto_pages - pages, got = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = tid * PER + k, s = s0 + i, fresh = max(x[k].count, 0);
            const bool served = x[k].fits && (x[k].want == 0 || base + x[k].want <= ring.room);
            s_off[i] = off, s_base[i] = base, s_len[i] = served ? x[k].len : ~x[k].len;
            if (blockIdx.x == 0 && s < a.n_seqs) {
                a.offsets[s] = off;
                a.starts[s] = served && x[k].count >= 0 ? x[k].len : -1;
                a.lengths_out[s] = x[k].count < 0 ? 0 : served ? x[k].len + fresh : x[k].len;
                if (s == a.n_seqs - 1) a.offsets[a.n_seqs] = off + fresh;
            }
            off += fresh, base += x[k].want;
            if (served && x[k].want) got = base;
        }
        rows0 += all_rows, pages0 += all_pages;
        if (tid == XT - 1) s_off[CHUNK] = rows0, s_base[CHUNK] = pages0;
        if (blockIdx.x == 0 && got) atomicMax(&s_got, got);
        __syncthreads();
        // the first of the thread's rows (r + k stride) that is not before the chunk
        auto first = [&](long long from) {
            const long long r = (long long)blockIdx.x * XT + tid;
            return r >= from ? r : r + (from - r + stride - 1) / stride * stride;
        };
        if (a.positions || a.slots)
            for (long long r = first(s_off[0]); r < min(rows0, a.rows); r += stride) {
                const int i = range_of(s_off, CHUNK, (int)r), l = s_len[i], len = l < 0 ? ~l : l, p = len + (int)r - s_off[i];
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
            const int i = range_of(s_base, CHUNK, (int)u), at = ring.get + (int)u;
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

// Pages of the sequences that end, the b-th part of them: those that are pages of the cache, behind those of the parts before.
__device__ __forceinline__ void pages_back(const ExtendArgs& a, const Ring& ring, int b, int* s_from, int* s_sum) {
    const int tid = threadIdx.x;
    auto ended = [&](int s) {
        const Next x = next_of(a, s);
        return x.count < 0 ? x.held : 0;
    };
    long long total = 0;
    {
        long long mine = 0;
        for (int s = tid; s < a.n_seqs; s += XT) mine += ended(s);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) mine += __shfl_xor(mine, o, 64);
        __shared__ long long s_total[XT / 64];
        if ((tid & 63) == 0) s_total[tid >> 6] = mine;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < XT / 64; ++w) total += s_total[w];
    }
    const long long lo = total * b / a.back_blocks, hi = total * (b + 1) / a.back_blocks;
    if (lo == hi && b != a.back_blocks - 1) return;
    const int free = a.pages - ring.room;
    long long place = 0, from = 0;   // pages that went back so far, entries of the chunks so far
    for (int s0 = 0; s0 < a.n_seqs && from < hi; s0 += CHUNK) {
        int own[PER], sum = 0, all;
#pragma unroll
        for (int k = 0; k < PER; ++k) sum += own[k] = ended(s0 + tid * PER + k);
        const int upto = block_sum_up(sum, s_sum, all);
        int at = upto - sum;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            s_from[tid * PER + k] = at;
            at += own[k];
        }
        if (tid == XT - 1) s_from[CHUNK] = all;
        __syncthreads();
        auto page_at = [&](int e) {   // entry e of the chunk: its page, or -1
            const int i = range_of(s_from, CHUNK, e);
            const int page = a.table[(long long)(s0 + i) * a.table_pages + e - s_from[i]];
            return (unsigned)page < (unsigned)a.pages ? page : -1;
        };
        const int before = (int)min((long long)all, max(lo - from, 0ll)), end = (int)min((long long)all, hi - from);
        int mine = 0, there;   // entries of the parts before are only counted
        for (int e = tid; e < before; e += XT) mine += page_at(e) >= 0;
        block_sum_up(mine, s_sum + XT / 64, there);
        place += there;
        for (int e0 = before; e0 < end; e0 += XT) {
            const int page = e0 + tid < end ? page_at(e0 + tid) : -1;
            __syncthreads();   // s_sum
            const int up = block_sum_up(page >= 0, s_sum, there);
            const long long to = place + up - 1;
            if (page >= 0 && to < free) {
                const long long slot = ring.put + to;
                a.ring[slot < a.pages ? slot : slot - a.pages] = page;
            }
            place += there;
        }
        from += all;
        __syncthreads();
    }
    if (b == a.back_blocks - 1 && tid == 0) a.cursor_out[1] = a.cursor[1] + min(place, (long long)free);
}

__global__ __launch_bounds__(XT) void cache_extend_k(ExtendArgs a) {
    __shared__ int s_off[CHUNK + 1], s_base[CHUNK + 1], s_len[CHUNK], s_sum[2 * XT / 64];
    const Ring ring = ring_of(a);
    if ((int)blockIdx.x < a.row_blocks) rows_and_pages(a, ring, s_off, s_base, s_len, s_sum);
    else pages_back(a, ring, blockIdx.x - a.row_blocks, s_off, s_sum);
}

}  // namespace

void launch_cache_extend(ExtendArgs a, hipStream_t s) {
    a.row_blocks = (int)std::min<long long>(1024, std::max(1, (a.rows + 4 * XT - 1) / (4 * XT)));
    a.back_blocks = (int)std::min<long long>(64, ((long long)a.n_seqs * a.table_pages + 8191) / 8192);
    cache_extend_k<<<dim3((unsigned)(a.row_blocks + a.back_blocks)), XT, 0, s>>>(a);
}

}  // namespace dv

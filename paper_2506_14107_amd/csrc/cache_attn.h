// Attention of query rows over the paged 8-bit cache: what a block does.
//
// A tile is R packed rows of one sequence and key/value head: packed row r is query row r / G, head
// h G + r % G, so that the G query heads that share keys share their loads.  As in the encoder's
// attention every quantity is kept with one query per lane:
//   S^T = K . Q^T     A = 16 keys, B = 16 queries (MFMA 16x16x32, fp32 accumulate): lane l gets the scores of
//                     query l % 16 against 4 keys of each 16
//   O^T += V^T . P^T  the probabilities stay in the lanes that computed them
// A step takes 64 keys.  Row m of score tile t is key (m / 4) 16 + 4 t + m % 4 of the step, so that lane group
// g = l / 16 ends up with the scores of the 16 keys 16 g .. 16 g + 15: the order in which the value
// product contracts them, and 16 bytes of one channel's row of a page.
// Codes become bf16 exactly (3 fraction bits, power-of-two scales) by v_cvt_scalef32_pk_bf16_fp8, which
// applies the scale.  The softmax is one pass with a running maximum and sum in fp32; probabilities
// are rounded to bf16 for the value product of large tiles, at most a relative 2^-8 each, as in the encoder; small ones,
// whose time the memory sets, take them as two bf16 terms (16 bits, the same times: outputs of bf16 0.0016 off, which
// is their own rounding, where one term gives 0.0019).  fp32 queries are three bf16 terms (24 bits), and so are
// their probabilities: K and V being exact in bf16, three products give fp32 results at the bf16 matrix rate.
// Single tokens are bound by the cache's bytes: one query over 200,001 keys of 8 heads of 128 72 us (5.7 TB/s of
// the 6.2 that plain reads reach), one of each of 64 sequences of 1 to 12,000 keys 144 (5.3; the longest end last);
// joining the splits adds 6 to 8.  Questions of some rows over short caches are bound by the latency of a
// tile's steps (fp32, 333 rows of 16 heads of 80 over up to 1801 keys: 21 us; matrix units 8 % busy, 0.6 wavefronts a
// SIMD).
#pragma once
#include <type_traits>

#include "cache_plan.h"

namespace dv {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// What the keys of a call are: all up to a row's own; those of a window and the first ones (the steps between the two are
// left out: Tile::skip0); a part of what the rows see, whose result is joined with another part's; or those of a prefix in
// another table and then the sequence's own.
enum Keys : int { ALL = 0, WINDOW = 1, PART = 2, BEHIND = 3 };

constexpr int TR = 1 << TS, LR = 1 << LS;   // packed rows of a tile
constexpr int STEP = 64;                    // keys of a step
constexpr int WAVES = 4;

// f of the two values that lanes whose numbers differ in one bit (4 or 5) hold, in both: the swap gives
// one lane's value in its first result and the other's in its second.  (The elements are copied before
// the bit cast, which takes element 0 of a vector for any.)
template <int BIT, class F>
__device__ __forceinline__ float across(float x, F f) {
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = BIT == 4 ? __builtin_amdgcn_permlane16_swap(u, u, false, false)
                            : __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const unsigned a = r[0], b = r[1];
    return f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
// maximum and sum over the four 16-lane groups, in every lane
__device__ __forceinline__ float group_max(float x) {
    const auto f = [](float a, float b) { return fmaxf(a, b); };
    return across<5>(across<4>(x, f), f);
}
__device__ __forceinline__ float group_sum(float x) {
    const auto f = [](float a, float b) { return a + b; };
    return across<5>(across<4>(x, f), f);
}

// eight codes to bf16, times a power of two
__device__ __forceinline__ bf16x8 decode8(uint32_t lo, uint32_t hi, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
    const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return (bf16x8){a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The largest of three (v_maximum3_f32, a NaN if one is: fmaxf would quiet every operand first).  Left to the
// compiler because the operands are products of the matrix units: it keeps the 8 or 12 wait states behind those, and
// would not for inline assembly.
__device__ __forceinline__ float max3(float a, float b, float c) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}
// Scores are kept as products; exponents of 2 are (score - maximum) times this.  (Where the factor itself passes fp32, the
// largest number stands for it: a difference of one unit is past any exponent long before.)
__device__ __forceinline__ float exponent_factor(float scale) {
    return fminf(scale * 1.4426950408889634f, 3.4028235e38f);
}
// An exponent is one fma, score * factor + off with off = -maximum * factor, whose rounding a row's probabilities share.
// At 2^31 that rounding would be as large as exponents get, so rows whose |off| passes FAR have their maximum taken off
// the scores first (take_off).  Up to FAR it is at most 2^-15, and the largest probability a 1 in bf16.
constexpr float FAR = 1024.f;
template <class TakeOff>
__device__ __forceinline__ float offset_of(float m, float factor, TakeOff take_off) {
    const float off = m == -INFINITY ? 0.f : -m * factor;      // no key seen yet: all probabilities 0
    const bool far = fabsf(off) > FAR;
    if (!__any(far)) return off;
    take_off(far ? m : 0.f);
    return far ? 0.f : off;
}
// x as T bf16 terms: the first its rounding, each next the rounding of what is left
template <int T>
__device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&t)[T]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float rest = x[e];
#pragma unroll
        for (int k = 0; k < T; ++k) {
            t[k][e] = (__bf16)rest;
            if (k + 1 < T) rest -= (float)t[k][e];
        }
    }
}
// Waits for the queries here: left to their first use, the wait would stand in the loop of steps, where
// it waits for the loads of the next step at every turn.
template <int K, int T>
__device__ __forceinline__ void settle(bf16x8 (&q)[K][T]) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int n = 0; n < T; ++n) asm volatile("" : "+v"(q[k][n]));
}
template <int K>
__device__ __forceinline__ void settle(bf16x8 (&q)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) asm volatile("" : "+v"(q[k]));
}
// Codes that decode to NaN (magnitude 0x7F) or, where the scale is 2^120 and more, to infinity: 256 times 2^120 is 2^128,
// and each doubling of the scale takes in another exponent (8 codes).  odd_codes: what, added to the magnitude, carries
// into the sign's bit for these codes, in every byte; odd_bytes: the bytes of w that hold one, as 0xFF.
__device__ __forceinline__ uint32_t odd_codes(float scale) {
    const int over = (int)(__builtin_bit_cast(uint32_t, scale) >> 23 & 255) - (127 + 119);
    return 0x01010101u * (uint32_t)max(1, 8 * over);
}
__device__ __forceinline__ uint32_t odd_bytes(uint32_t w, uint32_t odd) {
    return (((w & 0x7F7F7F7Fu) + odd & 0x80808080u) >> 7) * 255u;
}
constexpr uint32_t HUGE_SCALE = (127 + 120) << 23;   // bits of the scale from which on a page may hold infinities

// A NaN or infinity among values that only some rows of a tile see: its products with the other rows' zero
// probabilities would be NaN too.  Steps that not all rows see in full take such codes as 0 and say so; if there was one,
// each lane looks through the values that its row sees in those steps and adds what it finds to its sums.  (Products of
// indicators on the matrix units instead, within the step, cost every step registers.)  Small tiles do the same with all
// pages that may hold infinities: a probability's second term can be 0, its product with an infinity NaN.
// Keys first .. last - 1 of sequence s, key/value head h: bit i tells of the lane's i-th channel, base +
// stride (i / 4) + i % 4 (those below DH).
struct Odd {
    uint64_t nan, up, down;
    __device__ __forceinline__ float add_to(float x, int i) const {
        if (nan >> i & 1) return __builtin_nanf("");
        if (up >> i & 1) x += INFINITY;
        if (down >> i & 1) x -= INFINITY;
        return x;
    }
};
__device__ __forceinline__ void find_odd(Odd& f, const CacheAttnArgs& a, const SeqArgs& q, int s, int h, int first, int last,
                                         int stride, int base) {
    const int pt = a.c.page_tokens, shift = page_shift(pt), DH = a.c.head_dim;
#pragma unroll 1
    for (int key = first; key < last; ++key) {
        const int page = page_of(q.table, q.table_pages, a.c.pages, s, key >> shift);
        if (page < 0) continue;
        const size_t at = (size_t)page * a.c.kv_heads + h;
        const uint8_t* v = a.c.v + at * DH * pt + (key & (pt - 1));
        const uint32_t odd = odd_codes(a.c.v_scale[at]) & 255;
#pragma unroll 1
        for (int i = 0; i < 64; ++i) {
            const int ch = base + stride * (i >> 2) + (i & 3);
            if (ch >= DH) continue;
            const uint32_t w = v[(size_t)ch * pt];
            if ((w & 0x7F) == 0x7F) f.nan |= 1ull << i;
            else if ((w & 0x7F) + odd >= 0x80) (w & 0x80 ? f.down : f.up) |= 1ull << i;
        }
    }
}

template <int SHIFT, int KEYS>
__device__ __forceinline__ Tile tile_at(const CacheAttnArgs& a, long long u) {
    const int G = a.q_heads / a.c.kv_heads;
    // a mixed batch: short sequences go to the kernel of single tokens, the others to that of tiles
    auto other = [&](const Seq& s) { return a.route == ATTN_BOTH && ((long long)s.n * G > few_rows(a.c.head_dim)) != (SHIFT == LS); };
    auto count = [&](const Seq& x) { return other(x) ? 0 : tile_count(x, G, SHIFT); };
    Seq s;
    const bool groups = KEYS == PART && a.groups.on;
    if (groups) s = find_group(a.seq, a.groups, count, (int)u);
    else s = a.seq.offsets ? find_seq(a.seq, count, (int)u) : seq_of(a.seq, (int)(u / ((G + (1 << SHIFT) - 1) >> SHIFT)));
    Tile t = tile_of(a.seq, a.c.page_tokens, G, SHIFT, a.causal != 0, s, u, groups);
    if (other(s)) t.seq = -1;
    if constexpr (KEYS == WINDOW) leave_out(t, G, a.causal != 0, a.window, a.sinks);
    if constexpr (KEYS == BEHIND) put_behind(t, a.front, a.groups, a.c.page_tokens);
    return t;
}
// The key at place v of those that a tile takes (steps of 64 lie together).
template <int KEYS>
__device__ __forceinline__ int key_at(const Tile& t, int v) {
    return (KEYS == WINDOW || KEYS == BEHIND) && v >= t.skip0 ? v + t.left_out : v;
}
// Whether that is the prefix's.
template <int KEYS>
__device__ __forceinline__ bool in_front(const Tile& t, int v) {
    return KEYS == BEHIND && v < t.skip0;
}
// Table entry and page of the key `off` places behind place v, both of one step (entry_of, page_from).
template <int KEYS>
__device__ __forceinline__ int entry_at(const CacheAttnArgs& a, const Tile& t, int shift, int v, int off) {
    const int j = (key_at<KEYS>(t, v) + off) >> shift;
    if constexpr (KEYS == BEHIND) {
        const SeqArgs& q = a.front;
        const int* own = a.seq.table ? a.seq.table + (long long)t.seq * a.seq.table_pages + min(j, a.seq.table_pages - 1) : a.seq.at;
        return *(in_front<KEYS>(t, v) ? q.table + (long long)t.group * q.table_pages + min(j, q.table_pages - 1) : own);
    }
    return entry_of(a.seq, t.seq, j);
}
template <int KEYS>
__device__ __forceinline__ int page_at(const CacheAttnArgs& a, const Tile& t, int shift, int v, int off, int entry) {
    const int j = (key_at<KEYS>(t, v) + off) >> shift;
    if (in_front<KEYS>(t, v)) return j < a.front.table_pages && (unsigned)entry < (unsigned)a.c.pages ? entry : -1;
    return page_from(a.seq, a.c.pages, entry, t.seq, j);
}
// Where the window of a tile's first row starts, and whether that leaves the 16 keys from `key` on to no row of the tile: the
// steps at either end of what is left out (leave_out) hold such keys, whole pages of them where those are of 16 or 32.
__device__ __forceinline__ int window_start(const CacheAttnArgs& a, const Tile& t, int G) {
    return max(a.causal ? t.len - t.n + t.first / G + 1 : t.len, 0) - a.window;
}
__device__ __forceinline__ bool hidden(const CacheAttnArgs& a, int tlow, int key) { return key >= a.sinks && key + 16 <= tlow; }
// What the row that sees keys below `sees` sees of the step at place v, of keys before `last` (find_odd).
template <int KEYS>
__device__ __forceinline__ void find_odd_seen(Odd& f, const CacheAttnArgs& a, const Tile& t, int h, int v, int last, int sees,
                                              int stride, int base) {
    int first = key_at<KEYS>(t, v);
    const bool front = in_front<KEYS>(t, v);
    last = min(min(last, first + STEP), front ? t.front_len : sees);
    if constexpr (KEYS == WINDOW) {
        find_odd(f, a, a.seq, t.seq, h, first, min(last, a.sinks), stride, base);
        first = max(first, max(sees - a.window, a.sinks));
    }
    find_odd(f, a, front ? a.front : a.seq, front ? t.group : t.seq, h, first, last, stride, base);
}

template <bool BF>
__device__ __forceinline__ void store4(void* out, size_t at, f32x4 x) {
    if constexpr (BF) {
        const bf16x4 r = {(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
        *(bf16x4*)((uint16_t*)out + at) = r;
    } else {
        *(f32x4*)((float*)out + at) = x;
    }
}


// One tile, head and split of the keys per block; its wavefronts take the steps of the split in turn and
// join their results through LDS.
template <int DH>
struct __attribute__((aligned(16))) Small {   // (rows of o go in and out 16 bytes at once: by fours, as of a struct of floats,
    float o[WAVES][TR][DH + 4], m[WAVES][TR], l[WAVES][TR];   // 333 fp32 rows of 128 channels took 33.1 us, 32.4 so)
    static_assert((DH + 4) % 4 == 0, "rows of o start on 16 bytes");
};
// Block bx of a split's, by: the split.
template <int DH, bool BF, int KEYS>
__device__ __forceinline__ void attend_small(const CacheAttnArgs& a, Small<DH>& lds, unsigned bx, unsigned by) {
    constexpr int NT = BF ? 1 : 3;             // bf16 terms of queries
    constexpr int PT = BF ? 2 : 3;             // ... of probabilities
    constexpr int KS = (DH + 31) / 32;         // 32-channel steps of S^T
    constexpr int CT = DH / 16;                // 16-channel tiles of O^T
    constexpr bool WIDE = DH % 64 == 0;        // 16-byte key loads
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int H = a.c.kv_heads, pt = a.c.page_tokens, shift = page_shift(pt);
    const int h = bx % H;
    const long long u = bx / H;
    const Tile t = tile_at<TS, KEYS>(a, u);
    if (t.seq < 0) return;
    const int k0 = by * a.few.chunk, k1 = min(t.end - t.left_out, k0 + a.few.chunk);
    if (by > 0 && k0 >= k1) return;    // the first split also writes rows that see no key
    const int kend = KEYS == WINDOW || KEYS == BEHIND ? t.end : k1;   // (splits end with a step)
    const int G = a.q_heads / H;
    const int g = lane >> 4, c16 = lane & 15;
    const float sl2 = exponent_factor(a.scale);

    // the lane's query: packed row first + c16 (rows past the tile repeat its last one)
    const int r = t.first + min(c16, t.rows - 1), qi = r / G;
    const int sees = a.causal ? t.len - t.n + qi + 1 : t.len;
    const int low = max(sees, 0) - a.window;   // WINDOW: keys from here on, and the first `sinks`
    const int tlow = window_start(a, t, G);    // ... of the tile's first row: no row sees keys from the first ones up to here
    const size_t qat = (size_t)(t.row0 + qi) * a.q_stride + (size_t)(h * G + r % G) * DH;
    bf16x8 qf[KS][NT];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int ch = WIDE ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (ch < DH) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = BF ? bf16_to_f32(((const uint16_t*)a.q)[qat + ch + e]) : ((const float*)a.q)[qat + ch + e];
        }
        split8<NT>(x, qf[s]);
    }
    settle(qf);

    f32x4 o[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) o[c] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    // pages of the step at kb: of the key rows that the lane loads (group c16 / 4), and of the group it owns
    struct Pages {
        int k, v;
    };
    auto pages = [&](int v) {
        return Pages{entry_at<KEYS>(a, t, shift, v, (c16 >> 2) * 16), entry_at<KEYS>(a, t, shift, v, g * 16)};
    };
    uint32_t kw[4][KS][2];
    u32x4 vw[CT];
    float ks, vs;
    bool present = false;   // the lane's group of the step has a page
    auto load_keys = [&](int v, const Pages& pg) {
        const int kk = key_at<KEYS>(t, v) + (c16 >> 2) * 16;
        const size_t page = (size_t)max(page_at<KEYS>(a, t, shift, v, (c16 >> 2) * 16, pg.k), 0) * H + h;
        const uint8_t* base = a.c.k + (page * pt + (kk & (pt - 1)) + (c16 & 3)) * DH;
        ks = a.c.k_scale[page];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint8_t* row = base + q * 4 * DH;
            if constexpr (WIDE) {
#pragma unroll
                for (int s = 0; s < KS; s += 2) {
                    const u32x4 w = *(const u32x4*)(row + s * 32 + g * 16);
                    kw[q][s][0] = w[0], kw[q][s][1] = w[1], kw[q][s + 1][0] = w[2], kw[q][s + 1][1] = w[3];
                }
            } else {
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const int ch = s * 32 + g * 8;
                    u32x2 w = {0, 0};
                    if (ch < DH) w = *(const u32x2*)(row + ch);
                    kw[q][s][0] = w[0], kw[q][s][1] = w[1];
                }
            }
        }
    };
    auto load_values = [&](int v, const Pages& pg) {
        const int kv = key_at<KEYS>(t, v) + g * 16;
        const int p = page_at<KEYS>(a, t, shift, v, g * 16, pg.v);
        present = p >= 0;
        const size_t page = (size_t)max(p, 0) * H + h;
        const uint8_t* base = a.c.v + (page * DH + c16) * pt + (kv & (pt - 1));
        vs = a.c.v_scale[page];
#pragma unroll
        for (int c = 0; c < CT; ++c) vw[c] = *(const u32x4*)(base + (size_t)c * 16 * pt);
    };

    // The wavefront's steps.  The registers of a step's keys take the next step's codes as soon as its scores
    // are computed, those of its values when their product is; the pages of the step after that are
    // asked for between the two, because loads are waited for in order.
    constexpr int NEXT = WAVES * STEP;
    uint32_t odds = 0;
    int kb = k0 + wave * STEP;
    Pages next = pages(kb);
    if (kb < k1) {   // in the order of the loop, whose waits count on it
        load_keys(kb, next);
        __builtin_amdgcn_sched_barrier(0);
        const Pages after = pages(kb + NEXT);
        __builtin_amdgcn_sched_barrier(0);
        load_values(kb, next);
        next = after;
    }
    auto step = [&](auto last) {   // the last one loads nothing: no wait in the others stands behind a branch
        constexpr bool more = !decltype(last)::value;
        const int kv = key_at<KEYS>(t, kb) + g * 16;
        float sc[16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const bf16x8 kf = decode8(kw[q][s][0], kw[q][s][1], ks);
#pragma unroll
                for (int n = NT - 1; n >= 0; --n)
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[s][n], acc, 0, 0, 0);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[q * 4 + e] = acc[e];
        }
        __builtin_amdgcn_sched_barrier(0);
        Pages after = next;
        if constexpr (more) {
            load_keys(kb + NEXT, next);
            after = pages(kb + 2 * NEXT);
        }
        __builtin_amdgcn_sched_barrier(0);
        // keys kv .. kv + 15 belong to the lane; those it does not see, and those of pages that are
        // not there, get -inf
        const bool front = in_front<KEYS>(t, kb);
        const int until = front ? t.front_len : kend;
        const int live = present ? min(front ? until : sees, until) - kv : 0;
        bool part = live < 16 || __builtin_bit_cast(uint32_t, vs) >= HUGE_SCALE;
        if constexpr (KEYS == WINDOW) part |= kv < low && kv + 16 > a.sinks;
        const bool some = __any(part);
        if (some) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                bool in = e < live;
                if constexpr (KEYS == WINDOW) in = in && (kv + e >= low || kv + e < a.sinks);
                sc[e] = in ? sc[e] : -INFINITY;
            }
            // values that no row of the tile sees may hold anything, and so may the scale of a page
            // that has none else: 0
            int there = present ? until - kv : 0;
            if constexpr (KEYS == WINDOW) there = hidden(a, tlow, kv) ? 0 : there;
            if (there <= 0) vs = 1.f;
            const uint32_t odd = odd_codes(vs);
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int b = there - 4 * w;
                    vw[c][w] &= b >= 4 ? 0xFFFFFFFFu : b <= 0 ? 0u : (1u << 8 * b) - 1;
                    const uint32_t bad = odd_bytes(vw[c][w], odd);
                    odds |= bad;
                    vw[c][w] &= ~bad;
                }
        }
        float top = max3(sc[0], sc[1], sc[2]), top2 = max3(sc[3], sc[4], sc[5]);
#pragma unroll
        for (int e = 6; e < 14; e += 4) top = max3(top, sc[e], sc[e + 1]), top2 = max3(top2, sc[e + 2], sc[e + 3]);
        top = group_max(max3(max3(top, sc[14], sc[15]), top2, top2));
        // Rescale when some row's maximum has grown.  (Only when it has by more than 2^8 would be safe, and in the
        // large tiles 1.5 % faster, but the largest probability is then not 1, which bf16 holds exactly: outputs
        // over keys of uneven sizes 0.0022 off, relative, instead of 0.0019; their own rounding is 0.0016.)
        if (__any(top > m)) {
            const float mn = fmaxf(m, top);
            const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * sl2);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < CT; ++c) o[c] *= alpha;
        }
        const float off = offset_of(m, sl2, [&](float top) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] -= top;
        });
        float p[2][8];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            p[e >> 3][e & 7] = __builtin_amdgcn_exp2f(fmaf(sc[e], sl2, off));
            l += p[e >> 3][e & 7];
        }
        bf16x8 pf[2][PT];
        split8<PT>(p[0], pf[0]);
        split8<PT>(p[1], pf[1]);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bf16x8 vf = decode8(vw[c][2 * k], vw[c][2 * k + 1], vs);
#pragma unroll
                for (int n = PT - 1; n >= 0; --n)
                    o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[k][n], o[c], 0, 0, 0);
            }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (more) load_values(kb + NEXT, next);
        __builtin_amdgcn_sched_barrier(0);
        next = after;
    };
    if (kb < k1) {
        for (; kb + NEXT < k1; kb += NEXT) step(std::false_type());
        step(std::true_type());
    }

    if (__any(odds != 0)) {
        Odd found{};
        for (kb = k0 + wave * STEP; kb < k1; kb += NEXT) find_odd_seen<KEYS>(found, a, t, h, kb, in_front<KEYS>(t, kb) ? t.front_len : kend, sees, 16, g * 4);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][e] = found.add_to(o[c][e], c * 4 + e);
    }

    // join the wavefronts
    l = group_sum(l);
    if (g == 0) lds.m[wave][c16] = m, lds.l[wave][c16] = l;
#pragma unroll
    for (int c = 0; c < CT; ++c) *(f32x4*)&lds.o[wave][c16][c * 16 + g * 4] = o[c];
    __syncthreads();
    const bool whole = KEYS != PART && t.end - t.left_out <= a.few.chunk;      // no other split has keys
    float* part = a.few.part + (((size_t)u * H + h) * a.few.splits + by) * part_floats(TR, DH);
    for (int i = tid; i < TR * (DH / 4); i += 256) {
        const int row = i / (DH / 4), ch = i % (DH / 4) * 4;
        if (row >= t.rows) break;
        float top = lds.m[0][row];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, lds.m[w][row]);
        const float ref = top == -INFINITY ? 0.f : top;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f((lds.m[w][row] - ref) * sl2);
            sum += lds.l[w][row] * f;
            x += *(const f32x4*)&lds.o[w][row][ch] * f;
        }
        if (whole) {
            const int pr = t.first + row;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            store4<BF>(a.out, (size_t)(t.row0 + pr / G) * a.o_stride + (size_t)(h * G + pr % G) * DH + ch, x * inv);
        } else {
            *(f32x4*)(part + row * DH + ch) = x;
            if (ch == 0) part[TR * DH + row] = top, part[TR * DH + TR + row] = sum;
        }
    }
}

// ---- large tiles -----------------------------------------------------------------------------------
// 128 packed rows per block, 32 per wavefront (MFMA 32x32x16, queries in registers); the 64 keys of a step are
// decoded to bf16 once per block into one of two LDS buffers, while the other is read: a
// wavefront's matrix work on a step (1024 clocks of a SIMD at 128 channels) needs 32 KB of it.
// 4096 rows of two sequences of 5000 to 6144 keys, 32 heads of 128 on 8: 348 us, 968 TFLOP/s (a large library
// product: 1210 to 1360, by the card).  By the counters matrix units are busy 42 % of the time, vector units 49 (59 with exponentials at a
// quarter of the rate), LDS 37 (fragments read by four wavefronts each, decoded codes written), at 1.75 wavefronts a
// SIMD: they overlap in part.
// Row m of a 32-key score block is key m with bits 2 and 3 exchanged, so that lane half hl ends up with
// keys 16 j + 8 hl .. + 7 of each 16: the order in which the value product takes them.  Keys
// lie in LDS at the exchanged rows.
template <int DH>
struct Lds {
    static constexpr int KLD = DH * 2 + 16, VLD = STEP * 2 + 16;   // row strides: 8 rows on distinct banks
    uint8_t k[2][STEP * KLD];
    uint8_t v[2][DH * VLD];
    uint8_t there[2][4];   // whether a step's four 16-key groups have a page
    int odd;               // first key of the first step that held a value taken as 0 (find_odd), or more
};

// ONE: a step lies in one page (64 or 128 tokens), whose address is scalar then.
template <int DH, bool ONE, int KEYS>
__device__ __forceinline__ void attend_large(const CacheAttnArgs& a, Lds<DH>& lds, unsigned bx, unsigned by) {
    constexpr int KS = DH / 16;                      // 16-channel steps of S^T
    constexpr int CB = (DH + 31) / 32;               // 32-channel blocks of O^T
    constexpr int PARTS = DH / 16;                   // 16-byte parts of a key
    constexpr int NL = (STEP * PARTS + 255) / 256;   // parts a thread copies of each of keys and values
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hl = lane >> 5, lr = lane & 31;
    const int H = a.c.kv_heads, pt = a.c.page_tokens, shift = page_shift(pt);
    const int h = bx % H;
    const long long u = a.many.slots - 1 - bx / H;   // a sequence's last rows, with the most keys, first
    const Tile t = tile_at<LS, KEYS>(a, u);
    if (t.seq < 0) return;
    const int k0 = by * a.many.chunk, k1 = min(t.end - t.left_out, k0 + a.many.chunk);
    if (by > 0 && k0 >= k1) return;
    const int kend = KEYS == WINDOW || KEYS == BEHIND ? t.end : k1;
    const int G = a.q_heads / H;
    const float sl2 = exponent_factor(a.scale);

    const int mine = t.first + wave * 32;                    // the wavefront's first packed row
    const int r = min(mine + lr, t.first + t.rows - 1), qi = r / G;
    const int sees = a.causal ? t.len - t.n + qi + 1 : t.len;
    // keys that the wavefront's last row sees, and that all its rows see
    const int wlast = min(mine + 31, t.first + t.rows - 1) / G, wfirst = min(mine, t.first + t.rows - 1) / G;
    const int wend = mine < t.first + t.rows ? min(kend, a.causal ? t.len - t.n + wlast + 1 : t.len) : 0;
    const int wall = a.causal ? t.len - t.n + wfirst + 1 : t.len;
    const int ball = a.causal ? t.len - t.n + t.first / G + 1 : t.len;   // ... all of the block's
    // WINDOW: where the windows of the lane's row and of the last rows of the wavefront and the block start, and of the
    // wavefront's first
    const int low = max(sees, 0) - a.window, blow = t.end - a.window, wfrom = max(wall, 0) - a.window;
    const int tlow = window_start(a, t, G);   // ... of the block's first row
    const int wlow = max(a.causal ? t.len - t.n + wlast + 1 : t.len, 0) - a.window;
    bf16x8 qf[KS];
    {
        const uint16_t* q = (const uint16_t*)a.q + (size_t)(t.row0 + qi) * a.q_stride + (size_t)(h * G + r % G) * DH;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            uint16_t x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = q[s * 16 + hl * 8 + e];
            qf[s] = __builtin_bit_cast(bf16x8, x);
        }
        settle(qf);
    }

    // Codes of a step: part i of the keys is 16 channels of key i / PARTS, of the values 16 keys (group
    // i % 4) of channel i / 4.  The pages of a step are asked for a step before its codes.
    struct Pages {
        int k[NL], v;
    };
    auto pages = [&](int v) {
        Pages p;
        if constexpr (ONE) {
            p.v = entry_at<KEYS>(a, t, shift, v, 0);
            return p;
        }
#pragma unroll
        for (int n = 0; n < NL; ++n) p.k[n] = entry_at<KEYS>(a, t, shift, v, (tid + n * 256) / PARTS);
        p.v = entry_at<KEYS>(a, t, shift, v, tid % 4 * 16);
        return p;
    };
    u32x4 kc[NL], vc[NL];
    float ksc[NL], vsc;
    bool vin;
    const uint32_t kat = tid * 16, vat = tid / 4 * pt + tid % 4 * 16;   // ONE: of part tid, in the page
    auto load = [&](int v, const Pages& p) {
        const int kb = key_at<KEYS>(t, v);
        if constexpr (ONE) {
            const int page = page_at<KEYS>(a, t, shift, v, 0, __builtin_amdgcn_readfirstlane(p.v));
            const size_t at = (size_t)max(page, 0) * H + h;
            const uint8_t* kbase = a.c.k + (at * pt + (kb & (pt - 1))) * DH;
            const uint8_t* vbase = a.c.v + at * DH * pt + (kb & (pt - 1));
            vin = page >= 0;
#pragma unroll
            for (int n = 0; n < NL; ++n) {
                if (STEP * PARTS % 256 && tid + n * 256 >= STEP * PARTS) break;
                kc[n] = *(const u32x4*)(kbase + kat + n * 4096u);
                vc[n] = *(const u32x4*)(vbase + vat + n * 64u * pt);
                ksc[n] = a.c.k_scale[at];
            }
            vsc = a.c.v_scale[at];
            return;
        }
        const int tok = kb + tid % 4 * 16;
        const int vp = page_at<KEYS>(a, t, shift, v, tid % 4 * 16, p.v);
        vin = vp >= 0;
        const size_t vpage = (size_t)max(vp, 0) * H + h;
        const uint8_t* vbase = a.c.v + vpage * DH * pt + (tok & (pt - 1));
        vsc = a.c.v_scale[vpage];
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            const int i = tid + n * 256;
            if (STEP * PARTS % 256 && i >= STEP * PARTS) break;
            const size_t kpage = (size_t)max(page_at<KEYS>(a, t, shift, v, i / PARTS, p.k[n]), 0) * H + h;
            kc[n] = *(const u32x4*)(a.c.k + (kpage * pt + ((kb + i / PARTS) & (pt - 1))) * DH + i % PARTS * 16);
            ksc[n] = a.c.k_scale[kpage];
            vc[n] = *(const u32x4*)(vbase + i / 4 * pt);
        }
    };
    auto store = [&](int v, int buf) {
        const int kb = key_at<KEYS>(t, v);
        if (tid < 4) lds.there[buf][tid] = vin;   // the four groups of the first channel
        // values past the keys that anyone sees, and of pages that are not there, are 0
        const bool front = in_front<KEYS>(t, v);
        const int until = front ? t.front_len : kend;
        int there = vin ? until - kb - tid % 4 * 16 : 0;
        if constexpr (KEYS == WINDOW && !ONE) there = hidden(a, tlow, kb + tid % 4 * 16) ? 0 : there;   // (a row sees some key of every step)
        bool part = kb + STEP > min(front ? until : ball, until) || !vin;   // not all rows see all of it
        if constexpr (KEYS == WINDOW) part |= kb < blow && kb + STEP > a.sinks;
        if (there <= 0) vsc = 1.f;
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            const int i = tid + n * 256;
            if (STEP * PARTS % 256 && i >= STEP * PARTS) break;
            const int key = i / PARTS, row = (key & ~12) | (key & 4) << 1 | (key & 8) >> 1;
            u32x4* k = (u32x4*)(lds.k[buf] + row * Lds<DH>::KLD + i % PARTS * 32);
            k[0] = __builtin_bit_cast(u32x4, decode8(kc[n][0], kc[n][1], ksc[n]));
            k[1] = __builtin_bit_cast(u32x4, decode8(kc[n][2], kc[n][3], ksc[n]));
            if (part) {
                const uint32_t odd = odd_codes(vsc);
                uint32_t bad = 0;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int b = there - 4 * w;
                    vc[n][w] &= b >= 4 ? 0xFFFFFFFFu : b <= 0 ? 0u : (1u << 8 * b) - 1;
                    const uint32_t x = odd_bytes(vc[n][w], odd);
                    bad |= x;
                    vc[n][w] &= ~x;
                }
                if (bad) atomicMin(&lds.odd, v);   // (the order does not matter)
            }
            u32x4* to = (u32x4*)(lds.v[buf] + i / 4 * Lds<DH>::VLD + i % 4 * 32);
            to[0] = __builtin_bit_cast(u32x4, decode8(vc[n][0], vc[n][1], vsc));
            to[1] = __builtin_bit_cast(u32x4, decode8(vc[n][2], vc[n][3], vsc));
        }
    };

    f32x16 o[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[c][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    auto step = [&](int v, int buf) {
        const int kb = key_at<KEYS>(t, v);
        f32x16 sc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[b][e] = 0.f;
        const uint8_t* krow = lds.k[buf] + lr * Lds<DH>::KLD + hl * 16;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < KS; ++s)   // two chains
#pragma unroll
            for (int b = 0; b < 2; ++b)
                sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8*)(krow + b * 32 * Lds<DH>::KLD + s * 32),
                                                                qf[s], sc[b], 0, 0, 0);
        // the LDS reads run AHEAD matrix instructions ahead
        constexpr int AHEAD = KS < 3 ? 2 * KS : 6;
        __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
        for (int s = 0; s < 2 * KS - AHEAD; ++s) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, AHEAD, 0);
        __builtin_amdgcn_sched_barrier(0);
        // element e of block b is key kb + 32 b + 16 (e / 8) + 8 hl + e % 8
        const uint32_t there = *(const uint32_t*)lds.there[buf];
        const bool front = in_front<KEYS>(t, v);
        const int until = front ? t.front_len : kend;
        bool some = kb + STEP > min(front ? until : wall, until) || there != 0x01010101u;
        if constexpr (KEYS == WINDOW) some |= kb < wlow && kb + STEP > a.sinks;
        if (some) {
            const int live = min(front ? until : sees, until) - kb - 8 * hl;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = 2 * b + (e >> 3), i = 16 * j + (e & 7);
                    if constexpr (KEYS == WINDOW) {
                        const bool in = i < live && (there >> 8 * j & 1) && (i >= low - kb - 8 * hl || i < a.sinks - kb - 8 * hl);
                        sc[b][e] = in ? sc[b][e] : -INFINITY;
                    } else {
                        sc[b][e] = i < live && (there >> 8 * j & 1) ? sc[b][e] : -INFINITY;
                    }
                }
        }
        float mx[5];   // five chains
#pragma unroll
        for (int e = 0; e < 5; ++e) mx[e] = max3(sc[0][3 * e], sc[0][3 * e + 1], sc[0][3 * e + 2]);
#pragma unroll
        for (int e = 0; e < 5; ++e) mx[e] = max3(mx[e], sc[1][3 * e], sc[1][3 * e + 1]);
#pragma unroll
        for (int e = 0; e < 5; ++e) mx[e] = e < 4 ? max3(mx[e], sc[1][3 * e + 2], mx[e]) : max3(mx[e], sc[0][15], sc[1][15]);
        mx[0] = max3(mx[0], mx[1], sc[1][14]);
        mx[0] = max3(mx[0], mx[2], max3(mx[3], mx[4], mx[4]));
        const float top = across<5>(mx[0], [](float x, float y) { return fmaxf(x, y); });
        if (__any(top > m)) {
            const float mn = fmaxf(m, top);
            const float alpha = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * sl2);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int c = 0; c < CB; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[c][e] *= alpha;
        }
        const float off = offset_of(m, sl2, [&](float top) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[b][e] -= top;
        });
        bf16x8 pf[4];
        // (sums of the rounded probabilities, two a v_dot2_f32_bf16, take as long)
        float sum[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[0][e], sl2, off));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[1][e], sl2, off));
            sum[e] = p0 + p1;
            pf[e >> 3][e & 7] = (__bf16)p0;
            pf[2 + (e >> 3)][e & 7] = (__bf16)p1;
        }
#pragma unroll
        for (int w = 8; w >= 1; w >>= 1)
#pragma unroll
            for (int e = 0; e < w; ++e) sum[e] += sum[e + w];
        l += sum[0];
        const uint8_t* vrow = lds.v[buf] + lr * Lds<DH>::VLD + hl * 16;
        // (channels past DH take those 16 before: they are not stored)
        auto at = [&](int c, int j) {
            const int back = DH % 32 && c == CB - 1 ? (lr & 16) * Lds<DH>::VLD : 0;
            return *(const bf16x8*)(vrow + c * 32 * Lds<DH>::VLD - back + j * 32);
        };
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < CB; ++c)
                o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at(c, j), pf[j], o[c], 0, 0, 0);
    };

    auto turn = [&](int v, int buf) {   // a wavefront takes the steps that some row of it sees
        const int kb = key_at<KEYS>(t, v);
        bool any = in_front<KEYS>(t, v) ? mine < t.first + t.rows : kb < wend;
        if constexpr (KEYS == WINDOW) any = any && (kb + STEP > wfrom || kb < a.sinks);
        if (any) step(v, buf);
    };

    if (tid == 0) lds.odd = k1;
    Pages next = pages(k0);
    if (k0 < k1) load(k0, next);
    next = pages(k0 + STEP);
    __syncthreads();
    if (k0 < k1) store(k0, 0);
    __syncthreads();
    int buf = 0;
    int kb = k0;
    for (; kb + STEP < k1; kb += STEP, buf ^= 1) {
        const Pages after = pages(kb + 2 * STEP);   // first: loads are waited for in order
        load(kb + STEP, next);
        next = after;
        __builtin_amdgcn_sched_barrier(0);
        turn(kb, buf);
        store(kb + STEP, buf ^ 1);
        __syncthreads();
    }
    turn(kb, buf);

    if (lds.odd < k1) {
        Odd found{};
        if constexpr (KEYS == WINDOW || KEYS == BEHIND) {
            for (int v = lds.odd; v < k1; v += STEP)
                find_odd_seen<KEYS>(found, a, t, h, v, in_front<KEYS>(t, v) ? t.front_len : kend, sees, 8, hl * 4);
        } else {
            find_odd(found, a, a.seq, t.seq, h, lds.odd, min(sees, k1), 8, hl * 4);
        }
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[c][e] = found.add_to(o[c][e], c * 16 + e);
    }
    l = across<5>(l, [](float x, float y) { return x + y; });
    const int row = mine + lr - t.first;
    if (row >= t.rows) return;
    const bool whole = KEYS != PART && t.end - t.left_out <= a.many.chunk;
    float* part = a.many.part + (((size_t)u * H + h) * a.many.splits + by) * part_floats(LR, DH);
    const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int ch = c * 32 + e * 8 + hl * 4;
            if (ch >= DH) break;
            const f32x4 x = (f32x4){o[c][e * 4], o[c][e * 4 + 1], o[c][e * 4 + 2], o[c][e * 4 + 3]} * inv;
            if (whole)
                store4<true>(a.out, (size_t)(t.row0 + qi) * a.o_stride + (size_t)(h * G + r % G) * DH + ch, x);
            else
                *(f32x4*)(part + row * DH + ch) = x;
        }
    if (!whole && hl == 0) part[LR * DH + row] = m, part[LR * DH + LR + row] = l;
}

// Joins the splits of a tile's rows.  A row takes W wavefronts of a block (1, or 4 where it has many
// splits); every lane weighs one split in 64, then lanes go over the channels and groups of lanes over the
// splits.
template <bool BF, int SHIFT, int W, int KEYS>
__device__ __forceinline__ void join(const CacheAttnArgs& a) {
    constexpr int R = 1 << SHIFT, ROWS = 4 / W;
    __shared__ f32x4 s_x[256];
    const CacheAttnCut& cut = SHIFT == TS ? a.few : a.many;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int H = a.c.kv_heads, DH = a.c.head_dim, G = a.q_heads / H;
    const int h = blockIdx.x % H;
    const long long u = blockIdx.x / H;
    const Tile t = tile_at<SHIFT, KEYS>(a, u);
    const int keys = t.end - t.left_out;
    if (t.seq < 0 || keys <= cut.chunk) return;
    const int splits = (keys + cut.chunk - 1) / cut.chunk;
    const float sl2 = exponent_factor(a.scale);
    const size_t per = part_floats(R, DH);
    const float* part = cut.part + (((size_t)u * H + h) * cut.splits) * per;
    const int lanes = DH / 4, groups = 64 / lanes;        // of a wavefront
    const int ch = lane % lanes * 4, grp = lane / lanes;
    // one round, unless a sequence has more rows than it was said to have
    for (int row0 = blockIdx.y * ROWS; row0 < t.rows; row0 += gridDim.y * ROWS) {
        const int row = min(row0 + wave / W, t.rows - 1);
        float mx[MAX_SPLITS / 64], top = -INFINITY;
#pragma unroll
        for (int k = 0; k < (W == 1 ? 1 : MAX_SPLITS / 64); ++k) {
            const int s = lane + k * 64;
            mx[k] = s < splits ? part[s * per + R * DH + row] : -INFINITY;
            top = fmaxf(top, mx[k]);
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
        const float ref = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < (W == 1 ? 1 : MAX_SPLITS / 64); ++k) {
            const int s = lane + k * 64, n = min(64, splits - k * 64);
            float w = 0.f;
            if (s < splits) {
                w = __builtin_amdgcn_exp2f((mx[k] - ref) * sl2);
                sum += part[s * per + R * DH + R + row] * w;
            }
            const float* p = part + (size_t)k * 64 * per + row * DH + ch;
            for (int i = wave % W * groups; i < n; i += W * groups) {
                const int j = i + grp;
                const float wj = __shfl(w, j & 63, 64);
                if (grp < groups && j < n) x += *(const f32x4*)(p + (size_t)j * per) * wj;
            }
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
        s_x[tid] = x;
        __syncthreads();
        if (wave % W == 0 && grp == 0 && row0 + wave / W < t.rows) {
            for (int v = 0; v < W; ++v)
                for (int k = v == 0; k < groups; ++k) x += s_x[(wave + v) * 64 + k * lanes + lane];
            const int pr = t.first + row;
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            store4<BF>(a.out, (size_t)(t.row0 + pr / G) * a.o_stride + (size_t)(h * G + pr % G) * DH + ch, x * inv);
        }
        __syncthreads();
    }
}

// ---- launches ------------------------------------------------------------------------------------------
// K: a call's kernels: small<DH, BF>(), large<DH, ONE>(), join<BF, SHIFT, W>().
template <class K, bool BF, int SHIFT>
void launch_join(const CacheAttnArgs& a, const CacheAttnCut& c, hipStream_t s) {
    const bool few = c.splits <= 16;   // us of 8 tiles of 4 rows in 61 splits: 15 with one wavefront a row, 6 with four; of 640 in 6: 6, 10
    const dim3 grid((unsigned)(c.slots * a.c.kv_heads), (unsigned)(few ? (c.tile_rows + 3) / 4 : c.tile_rows));
    if (few) K::template join<BF, SHIFT, 1>()<<<grid, 256, 0, s>>>(a);
    else K::template join<BF, SHIFT, 4>()<<<grid, 256, 0, s>>>(a);
}

template <class K, int DH>
void launch_dh(bool bf, const CacheAttnArgs& a, hipStream_t s) {
    if (a.route != ATTN_MANY) {
        const dim3 grid((unsigned)(a.few.slots * a.c.kv_heads), (unsigned)a.few.splits);
        if (bf) K::template small<DH, true>()<<<grid, 256, 0, s>>>(a);
        else K::template small<DH, false>()<<<grid, 256, 0, s>>>(a);
    }
    if (a.route != ATTN_FEW) {
        const dim3 grid((unsigned)(a.many.slots * a.c.kv_heads), (unsigned)a.many.splits);
        auto go = [&](auto one) {
            constexpr auto k = K::template large<DH, decltype(one)::value>();
            static const bool ok = allow_lds((const void*)k, sizeof(Lds<DH>));
            (void)ok;
            k<<<grid, 256, sizeof(Lds<DH>), s>>>(a);
        };
        if (a.c.page_tokens >= STEP) go(std::true_type());
        else go(std::false_type());
    }
}
template <class K>
void launch_parts(bool bf, const CacheAttnArgs& a, hipStream_t s) {
    switch (a.c.head_dim) {
        case 16: launch_dh<K, 16>(bf, a, s); break;
        case 32: launch_dh<K, 32>(bf, a, s); break;
        case 48: launch_dh<K, 48>(bf, a, s); break;
        case 64: launch_dh<K, 64>(bf, a, s); break;
        case 80: launch_dh<K, 80>(bf, a, s); break;
        case 96: launch_dh<K, 96>(bf, a, s); break;
        case 112: launch_dh<K, 112>(bf, a, s); break;
        default: launch_dh<K, 128>(bf, a, s); break;
    }
}
inline void set_plan(CacheAttnArgs& a, const CacheAttnPlan& p, float* workspace) {
    a.route = p.route;
    a.few = p.few;
    a.many = p.many;
    a.few.part = workspace;
    a.many.part = workspace + p.few_floats;
}
template <class K>
void launch_all(bool bf, CacheAttnArgs a, const CacheAttnPlan& p, float* workspace, hipStream_t s) {
    set_plan(a, p, workspace);
    launch_parts<K>(bf, a, s);
    if (a.route != ATTN_MANY && a.few.splits > 1) bf ? launch_join<K, true, TS>(a, a.few, s) : launch_join<K, false, TS>(a, a.few, s);
    if (a.route != ATTN_FEW && a.many.splits > 1) launch_join<K, true, LS>(a, a.many, s);
}

}  // namespace

}  // namespace dv

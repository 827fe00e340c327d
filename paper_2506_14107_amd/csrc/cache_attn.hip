// Attention of query rows over the paged 8-bit cache.
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
__device__ __forceinline__ void find_odd(Odd& f, const CacheAttnArgs& a, int s, int h, int first, int last, int stride,
                                         int base) {
    const int pt = a.c.page_tokens, shift = page_shift(pt), DH = a.c.head_dim;
#pragma unroll 1
    for (int key = first; key < last; ++key) {
        const int page = page_of(a.seq.table, a.seq.table_pages, a.c.pages, s, key >> shift);
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

template <int SHIFT>
__device__ __forceinline__ Tile tile_at(const CacheAttnArgs& a, long long u) {
    const int G = a.q_heads / a.c.kv_heads;
    // a mixed batch: short sequences go to the kernel of single tokens, the others to that of tiles
    auto other = [&](const Seq& s) { return a.route == ATTN_BOTH && ((long long)s.n * G > few_rows(a.c.head_dim)) != (SHIFT == LS); };
    const Seq s = a.seq.offsets ? find_seq(a.seq, [&](const Seq& x) { return other(x) ? 0 : tile_count(x, G, SHIFT); }, (int)u)
                                : seq_of(a.seq, (int)(u / ((G + (1 << SHIFT) - 1) >> SHIFT)));
    Tile t = tile_of(a.seq, a.c.page_tokens, G, SHIFT, a.causal != 0, s, u);
    if (other(s)) t.seq = -1;
    return t;
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
template <int DH, bool BF>
__global__ __launch_bounds__(256, 2) void cache_attn_k(CacheAttnArgs a) {
    constexpr int NT = BF ? 1 : 3;             // bf16 terms of queries
    constexpr int PT = BF ? 2 : 3;             // ... of probabilities
    constexpr int KS = (DH + 31) / 32;         // 32-channel steps of S^T
    constexpr int CT = DH / 16;                // 16-channel tiles of O^T
    constexpr bool WIDE = DH % 64 == 0;        // 16-byte key loads
    __shared__ float s_o[WAVES][TR][DH + 4];
    __shared__ float s_m[WAVES][TR], s_l[WAVES][TR];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int H = a.c.kv_heads, pt = a.c.page_tokens, shift = page_shift(pt);
    const int h = blockIdx.x % H;
    const long long u = blockIdx.x / H;
    const Tile t = tile_at<TS>(a, u);
    if (t.seq < 0) return;
    const int k0 = blockIdx.y * a.few.chunk, k1 = min(t.end, k0 + a.few.chunk);
    if (blockIdx.y > 0 && k0 >= k1) return;    // the first split also writes rows that see no key
    const int G = a.q_heads / H;
    const int g = lane >> 4, c16 = lane & 15;
    const float sl2 = exponent_factor(a.scale);

    // the lane's query: packed row first + c16 (rows past the tile repeat its last one)
    const int r = t.first + min(c16, t.rows - 1), qi = r / G;
    const int sees = a.causal ? t.len - t.n + qi + 1 : t.len;
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
    auto pages = [&](int kb) {
        return Pages{entry_of(a.seq, t.seq, (kb + (c16 >> 2) * 16) >> shift),
                     entry_of(a.seq, t.seq, (kb + g * 16) >> shift)};
    };
    uint32_t kw[4][KS][2];
    u32x4 vw[CT];
    float ks, vs;
    bool present = false;   // the lane's group of the step has a page
    auto load_keys = [&](int kb, const Pages& pg) {
        const int kk = kb + (c16 >> 2) * 16;
        const size_t page = (size_t)max(page_from(a.seq, a.c.pages, pg.k, t.seq, kk >> shift), 0) * H + h;
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
    auto load_values = [&](int kb, const Pages& pg) {
        const int kv = kb + g * 16;
        const int p = page_from(a.seq, a.c.pages, pg.v, t.seq, kv >> shift);
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
        const int kv = kb + g * 16;
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
        const int live = present ? min(sees, k1) - kv : 0;
        const bool some = __any(live < 16 || __builtin_bit_cast(uint32_t, vs) >= HUGE_SCALE);
        if (some) {
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[e] = e < live ? sc[e] : -INFINITY;
            // values that no row of the tile sees may hold anything, and so may the scale of a page
            // that has none else: 0
            const int there = present ? k1 - kv : 0;
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
        for (kb = k0 + wave * STEP; kb < k1; kb += NEXT)
            find_odd(found, a, t.seq, h, kb, min(min(kb + STEP, k1), sees), 16, g * 4);
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[c][e] = found.add_to(o[c][e], c * 4 + e);
    }

    // join the wavefronts
    l = group_sum(l);
    if (g == 0) s_m[wave][c16] = m, s_l[wave][c16] = l;
#pragma unroll
    for (int c = 0; c < CT; ++c) *(f32x4*)&s_o[wave][c16][c * 16 + g * 4] = o[c];
    __syncthreads();
    const bool whole = t.end <= a.few.chunk;      // no other split has keys
    float* part = a.few.part + (((size_t)u * H + h) * a.few.splits + blockIdx.y) * part_floats(TR, DH);
    for (int i = tid; i < TR * (DH / 4); i += 256) {
        const int row = i / (DH / 4), ch = i % (DH / 4) * 4;
        if (row >= t.rows) break;
        float top = s_m[0][row];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_m[w][row]);
        const float ref = top == -INFINITY ? 0.f : top;
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f((s_m[w][row] - ref) * sl2);
            sum += s_l[w][row] * f;
            x += *(const f32x4*)&s_o[w][row][ch] * f;
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
// product: 1210).  By the counters matrix units are busy 42 % of the time, vector units 49 (59 with exponentials at a
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
template <int DH, bool ONE>
__global__ __launch_bounds__(256, 2) void cache_attn_tile_k(CacheAttnArgs a) {
    constexpr int KS = DH / 16;                      // 16-channel steps of S^T
    constexpr int CB = (DH + 31) / 32;               // 32-channel blocks of O^T
    constexpr int PARTS = DH / 16;                   // 16-byte parts of a key
    constexpr int NL = (STEP * PARTS + 255) / 256;   // parts a thread copies of each of keys and values
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    Lds<DH>& lds = *(Lds<DH>*)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, hl = lane >> 5, lr = lane & 31;
    const int H = a.c.kv_heads, pt = a.c.page_tokens, shift = page_shift(pt);
    const int h = blockIdx.x % H;
    const long long u = a.many.slots - 1 - blockIdx.x / H;   // a sequence's last rows, with the most keys, first
    const Tile t = tile_at<LS>(a, u);
    if (t.seq < 0) return;
    const int k0 = blockIdx.y * a.many.chunk, k1 = min(t.end, k0 + a.many.chunk);
    if (blockIdx.y > 0 && k0 >= k1) return;
    const int G = a.q_heads / H;
    const float sl2 = exponent_factor(a.scale);

    const int mine = t.first + wave * 32;                    // the wavefront's first packed row
    const int r = min(mine + lr, t.first + t.rows - 1), qi = r / G;
    const int sees = a.causal ? t.len - t.n + qi + 1 : t.len;
    // keys that the wavefront's last row sees, and that all its rows see
    const int wlast = min(mine + 31, t.first + t.rows - 1) / G, wfirst = min(mine, t.first + t.rows - 1) / G;
    const int wend = mine < t.first + t.rows ? min(k1, a.causal ? t.len - t.n + wlast + 1 : t.len) : 0;
    const int wall = a.causal ? t.len - t.n + wfirst + 1 : t.len;
    const int ball = a.causal ? t.len - t.n + t.first / G + 1 : t.len;   // ... all of the block's
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
    auto pages = [&](int kb) {
        Pages p;
        if constexpr (ONE) {
            p.v = entry_of(a.seq, t.seq, kb >> shift);
            return p;
        }
#pragma unroll
        for (int n = 0; n < NL; ++n)
            p.k[n] = entry_of(a.seq, t.seq, (kb + (tid + n * 256) / PARTS) >> shift);
        p.v = entry_of(a.seq, t.seq, (kb + tid % 4 * 16) >> shift);
        return p;
    };
    u32x4 kc[NL], vc[NL];
    float ksc[NL], vsc;
    bool vin;
    const uint32_t kat = tid * 16, vat = tid / 4 * pt + tid % 4 * 16;   // ONE: of part tid, in the page
    auto load = [&](int kb, const Pages& p) {
        if constexpr (ONE) {
            const int page = page_from(a.seq, a.c.pages, __builtin_amdgcn_readfirstlane(p.v), t.seq, kb >> shift);
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
        const int vp = page_from(a.seq, a.c.pages, p.v, t.seq, tok >> shift);
        vin = vp >= 0;
        const size_t vpage = (size_t)max(vp, 0) * H + h;
        const uint8_t* vbase = a.c.v + vpage * DH * pt + (tok & (pt - 1));
        vsc = a.c.v_scale[vpage];
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            const int i = tid + n * 256;
            if (STEP * PARTS % 256 && i >= STEP * PARTS) break;
            const size_t kpage = (size_t)max(page_from(a.seq, a.c.pages, p.k[n], t.seq, (kb + i / PARTS) >> shift), 0) * H + h;
            kc[n] = *(const u32x4*)(a.c.k + (kpage * pt + ((kb + i / PARTS) & (pt - 1))) * DH + i % PARTS * 16);
            ksc[n] = a.c.k_scale[kpage];
            vc[n] = *(const u32x4*)(vbase + i / 4 * pt);
        }
    };
    auto store = [&](int kb, int buf) {
        if (tid < 4) lds.there[buf][tid] = vin;   // the four groups of the first channel
        // values past the keys that anyone sees, and of pages that are not there, are 0
        const int there = vin ? k1 - kb - tid % 4 * 16 : 0;
        if (there <= 0) vsc = 1.f;
#pragma unroll
        for (int n = 0; n < NL; ++n) {
            const int i = tid + n * 256;
            if (STEP * PARTS % 256 && i >= STEP * PARTS) break;
            const int key = i / PARTS, row = (key & ~12) | (key & 4) << 1 | (key & 8) >> 1;
            u32x4* k = (u32x4*)(lds.k[buf] + row * Lds<DH>::KLD + i % PARTS * 32);
            k[0] = __builtin_bit_cast(u32x4, decode8(kc[n][0], kc[n][1], ksc[n]));
            k[1] = __builtin_bit_cast(u32x4, decode8(kc[n][2], kc[n][3], ksc[n]));
            if (kb + STEP > min(ball, k1) || !vin) {
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
                if (bad) atomicMin(&lds.odd, kb);   // (the order does not matter)
            }
            u32x4* v = (u32x4*)(lds.v[buf] + i / 4 * Lds<DH>::VLD + i % 4 * 32);
            v[0] = __builtin_bit_cast(u32x4, decode8(vc[n][0], vc[n][1], vsc));
            v[1] = __builtin_bit_cast(u32x4, decode8(vc[n][2], vc[n][3], vsc));
        }
    };

    f32x16 o[CB];
#pragma unroll
    for (int c = 0; c < CB; ++c)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[c][e] = 0.f;
    float m = -INFINITY, l = 0.f;

    auto step = [&](int kb, int buf) {
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
        const bool some = kb + STEP > min(wall, k1) || there != 0x01010101u;
        if (some) {
            const int live = min(sees, k1) - kb - 8 * hl;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int j = 2 * b + (e >> 3);
                    sc[b][e] = 16 * j + (e & 7) < live && (there >> 8 * j & 1) ? sc[b][e] : -INFINITY;
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
        if (kb < wend) step(kb, buf);
        store(kb + STEP, buf ^ 1);
        __syncthreads();
    }
    if (kb < wend) step(kb, buf);

    if (lds.odd < k1) {
        Odd found{};
        find_odd(found, a, t.seq, h, lds.odd, min(sees, k1), 8, hl * 4);
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[c][e] = found.add_to(o[c][e], c * 16 + e);
    }
    l = across<5>(l, [](float x, float y) { return x + y; });
    const int row = mine + lr - t.first;
    if (row >= t.rows) return;
    const bool whole = t.end <= a.many.chunk;
    float* part = a.many.part + (((size_t)u * H + h) * a.many.splits + blockIdx.y) * part_floats(LR, DH);
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
template <bool BF, int SHIFT, int W>
__global__ __launch_bounds__(256) void cache_join_k(CacheAttnArgs a) {
    constexpr int R = 1 << SHIFT, ROWS = 4 / W;
    __shared__ f32x4 s_x[256];
    const CacheAttnCut& cut = SHIFT == TS ? a.few : a.many;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int H = a.c.kv_heads, DH = a.c.head_dim, G = a.q_heads / H;
    const int h = blockIdx.x % H;
    const long long u = blockIdx.x / H;
    const Tile t = tile_at<SHIFT>(a, u);
    if (t.seq < 0 || t.end <= cut.chunk) return;
    const int splits = (t.end + cut.chunk - 1) / cut.chunk;
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

template <bool BF, int SHIFT>
void launch_join(const CacheAttnArgs& a, const CacheAttnCut& c, hipStream_t s) {
    const bool few = c.splits <= 16;   // us of 8 tiles of 4 rows in 61 splits: 15 with one wavefront a row, 6 with four; of 640 in 6: 6, 10
    const dim3 grid((unsigned)(c.slots * a.c.kv_heads), (unsigned)(few ? (c.tile_rows + 3) / 4 : c.tile_rows));
    if (few) cache_join_k<BF, SHIFT, 1><<<grid, 256, 0, s>>>(a);
    else cache_join_k<BF, SHIFT, 4><<<grid, 256, 0, s>>>(a);
}

template <int DH>
void launch_dh(bool bf, const CacheAttnArgs& a, hipStream_t s) {
    if (a.route != ATTN_MANY) {
        const dim3 grid((unsigned)(a.few.slots * a.c.kv_heads), (unsigned)a.few.splits);
        if (bf) cache_attn_k<DH, true><<<grid, 256, 0, s>>>(a);
        else cache_attn_k<DH, false><<<grid, 256, 0, s>>>(a);
    }
    if (a.route != ATTN_FEW) {
        const dim3 grid((unsigned)(a.many.slots * a.c.kv_heads), (unsigned)a.many.splits);
        auto go = [&](auto one) {
            constexpr auto k = cache_attn_tile_k<DH, decltype(one)::value>;
            static const bool ok = allow_lds((const void*)k, sizeof(Lds<DH>));
            (void)ok;
            k<<<grid, 256, sizeof(Lds<DH>), s>>>(a);
        };
        if (a.c.page_tokens >= STEP) go(std::true_type());
        else go(std::false_type());
    }
}

}  // namespace

void launch_cache_attention(bool bf, CacheAttnArgs a, const CacheAttnPlan& p, float* workspace, hipStream_t s) {
    a.route = p.route;
    a.few = p.few;
    a.many = p.many;
    a.few.part = workspace;
    a.many.part = workspace + p.few_floats;
    switch (a.c.head_dim) {
        case 16: launch_dh<16>(bf, a, s); break;
        case 32: launch_dh<32>(bf, a, s); break;
        case 48: launch_dh<48>(bf, a, s); break;
        case 64: launch_dh<64>(bf, a, s); break;
        case 80: launch_dh<80>(bf, a, s); break;
        case 96: launch_dh<96>(bf, a, s); break;
        case 112: launch_dh<112>(bf, a, s); break;
        default: launch_dh<128>(bf, a, s); break;
    }
    if (a.route != ATTN_MANY && a.few.splits > 1) bf ? launch_join<true, TS>(a, a.few, s) : launch_join<false, TS>(a, a.few, s);
    if (a.route != ATTN_FEW && a.many.splits > 1) launch_join<true, LS>(a, a.many, s);
}

}  // namespace dv

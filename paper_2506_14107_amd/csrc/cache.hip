// Rotary positions of token rows, and the paged 8-bit cache of keys and values: quantised as it is
// written, read back.  All three move bytes: rotary positions and reads at the rate of a device copy (169 MB in
// 36 us, 614 MB in 128: 4.7 and 4.8 TB/s), writes of long batches at 4 to 5.3 TB/s (95 MB in 23 us, 2.2 GB in 425),
// and calls of a few rows take their chain of dependent loads (3 to 8 us).
//
// Rotary positions: pair i of a row is turned by pos[axis(i)] * f_i radians.  The angle is kept in turns:
// f_i / 2 pi as a 64-bit fraction (RotaryPlan::turn), so that the product with a 32-bit position, taken
// modulo 2^64, is the turn's fraction to 2^-33 at any position; fp32 angles are off by 2^-24 of the whole
// angle, 64 radians at position 2^30.
//
// Codes are e4m3 (1 sign, 4 exponent, 3 fraction bits; largest 448), rounded to nearest even by
// v_cvt_pk_fp8_f32.  Scales are powers of two, the least with every |x| <= 448 scale: a floating code
// gains nothing from a finer scale, and a power of two can grow with a page that fills over several
// calls while codes away from the format's underflow (2^-6 of a scale) stay exact.  Scales and sums are
// fp32.
#include <algorithm>
#include <type_traits>

#include "cache_plan.h"

namespace dv {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- rows ------------------------------------------------------------------------------------------
template <bool BF>
struct Elem {
    using T = float;
};
template <>
struct Elem<true> {
    using T = uint16_t;
};

// V consecutive channels as fp32 (V = 8: 16 or 32 bytes at once; V = 1: one element)
template <bool BF, int V>
__device__ __forceinline__ void load_ch(const void* base, size_t at, float (&x)[V]) {
    if constexpr (V == 8 && BF) {
        const bf16x8 r = *(const bf16x8*)((const uint16_t*)base + at);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)r[i];
    } else if constexpr (V == 8) {
        const f32x4* p = (const f32x4*)((const float*)base + at);
        const f32x4 a = p[0], b = p[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else if constexpr (BF) {
        x[0] = bf16_to_f32(((const uint16_t*)base)[at]);
    } else {
        x[0] = ((const float*)base)[at];
    }
}
template <bool BF, int V>
__device__ __forceinline__ void store_ch(void* base, size_t at, const float (&x)[V]) {
    if constexpr (V == 8 && BF) {
        bf16x8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (__bf16)x[i];
        *(bf16x8*)((uint16_t*)base + at) = r;
    } else if constexpr (V == 8) {
        f32x4* p = (f32x4*)((float*)base + at);
        p[0] = (f32x4){x[0], x[1], x[2], x[3]};
        p[1] = (f32x4){x[4], x[5], x[6], x[7]};
    } else if constexpr (BF) {
        ((__bf16*)base)[at] = (__bf16)x[0];
    } else {
        ((float*)base)[at] = x[0];
    }
}

// ---- rotary positions ------------------------------------------------------------------------------
// cos and sin of 2 pi pos turn / 2^64, rounded to fp32 from fp64: keys are quantised from turned values, and
// every error there moves values across a code's border.  The low 64 bits of the product hold the fraction of
// a turn.  The nearest quarter is taken off (|r| <= pi/4), then the Taylor polynomials of degree 11 and
// 10: remainders (pi/4)^13 / 13! = 7e-12 and (pi/4)^12 / 12! = 1.2e-10, far below half a step of fp32.
__device__ __forceinline__ void turn_cos_sin(int pos, uint64_t turn, float& c, float& s) {
    const uint64_t p = (uint64_t)(int64_t)pos * turn;
    const uint32_t q = (uint32_t)((p + (1ull << 61)) >> 62);    // nearest quarter, modulo 4
    const int64_t f = (int64_t)(p - ((uint64_t)q << 62));
    const double r = fma((double)(int32_t)(f >> 32), 4294967296.0, (double)(uint32_t)f) * 3.4061215800865545e-19;   // 2 pi / 2^64
    const double r2 = r * r;
    double u = fma(-2.505210838544172e-08, r2, 2.7557319223985893e-06);
    u = fma(u, r2, -1.984126984126984e-04);
    u = fma(u, r2, 8.333333333333333e-03);
    u = fma(u, r2, -1.6666666666666666e-01);
    const float sn = (float)fma(u * r2, r, r);
    double v = fma(-2.755731922398589e-07, r2, 2.48015873015873e-05);
    v = fma(v, r2, -1.388888888888889e-03);
    v = fma(v, r2, 4.1666666666666664e-02);
    v = fma(v, r2, -0.5);
    const float cs = (float)fma(v, r2, 1.0);
    c = q & 1 ? sn : cs;
    s = q & 1 ? cs : sn;
    if (q == 1 || q == 2) c = -c;
    if (q >= 2) s = -s;
}

// An item is two groups of V channels of one row and head that the rotation mixes (or, past the turned
// channels, leaves): items of the `dim` turned channels first.
//   halves: channels o .. o + V - 1 with o + dim/2 ..; pairs (V = 8): 16 channels in a row, (V = 1): 2
// Either way the i-th item turns the V pairs from V i on.
struct Item {
    int o0, o1;
    bool turned;
};
template <int V>
__device__ __forceinline__ Item item_at(int dim, bool pairs, int i) {
    const int turned = dim / (2 * V);
    if (i >= turned || pairs) return {i * 2 * V, i * 2 * V + V, i < turned};
    return {i * V, i * V + dim / 2, true};
}
template <int V>
__device__ __forceinline__ void turn_item(bool pairs, const float* cos, const float* sin, float (&a)[V], float (&b)[V]) {
    float c[V], s[V];
    if constexpr (V == 8) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 x = *(const f32x4*)(cos + 4 * i), y = *(const f32x4*)(sin + 4 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) c[4 * i + e] = x[e], s[4 * i + e] = y[e];
        }
    } else {
        c[0] = *cos, s[0] = *sin;
    }
    auto rotate = [&](int i, float& x, float& y) {   // the same roundings however rows are aligned
        const float u = fmaf(x, c[i], -(y * s[i]));
        y = fmaf(x, s[i], y * c[i]);
        x = u;
    };
    if (V == 1 || !pairs) {
#pragma unroll
        for (int i = 0; i < V; ++i) rotate(i, a[i], b[i]);
    } else if constexpr (V > 1) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            rotate(i / 2, a[i], a[i + 1]);
            rotate(V / 2 + i / 2, b[i], b[i + 1]);
        }
    }
}

// The cosines and sines of n rows' angles (row(r): the positions of the r-th), into cos and sin [n][ld]: a lane
// keeps its pair.  NT threads.
template <int NT, class Row>
__device__ __forceinline__ void angles_of(const RotaryPlan& rot, int n, float* cos, float* sin, int ld, Row row) {
    const int lane = threadIdx.x & 63, half = rot.dim / 2, rows = 64 / half;   // of a wavefront at once
    const int pair = lane % half, sub = lane / half;
    if (sub >= rows) return;
    const uint64_t turn = rot.turn[pair];
    const int axis = pair < rot.end0 ? 0 : pair < rot.end1 ? 1 : 2;
    for (int r = (threadIdx.x >> 6) * rows + sub; r < n; r += NT / 64 * rows) {
        float c, s;
        turn_cos_sin(row(r)[axis], turn, c, s);
        cos[r * ld + pair] = c;
        sin[r * ld + pair] = s;
    }
}

// Rows row0 .. row0 + n - 1 of x, heads turned, to out (a block; n at most ROT_ROWS).  Each angle is computed
// once, into LDS, and used by all heads (16,448 rows of 32 heads of 80 channels, bf16: 36 us, with every head
// computing its own 51).
constexpr int ROT_LDS = ROT_ROWS * 64 * 2;
template <bool BF, int V, int NT>
__device__ __forceinline__ void turn_rows(const RowsArgs& a, const RotaryPlan& rot, int row0, int n, float* lds) {
    const int tid = threadIdx.x, half = rot.dim / 2, ld = (half + 3) & ~3;
    float *cos = lds, *sin = lds + ROT_ROWS * 64;
    angles_of<NT>(rot, n, cos, sin, ld, [&](int r) {
        return a.pos + (size_t)(a.pos_idx ? a.pos_idx[row0 + r] % a.pos_mod : row0 + r) * 3;
    });
    __syncthreads();
    const int per_head = a.dh / (2 * V), per_row = per_head * a.heads;
    for (int i = tid; i < n * per_row; i += NT) {
        const int r = i / per_row, rest = i % per_row, h = rest / per_head, c = rest % per_head;
        const Item it = item_at<V>(rot.dim, rot.pairs, c);
        float x[V], y[V];
        const size_t at = (size_t)(row0 + r) * a.x_stride + (size_t)h * a.dh;
        load_ch<BF, V>(a.x, at + it.o0, x);
        load_ch<BF, V>(a.x, at + it.o1, y);
        if (it.turned) turn_item<V>(rot.pairs, cos + r * ld + c * V, sin + r * ld + c * V, x, y);
        const size_t to = (size_t)(row0 + r) * a.out_stride + (size_t)h * a.dh;
        store_ch<BF, V>(a.out, to + it.o0, x);
        store_ch<BF, V>(a.out, to + it.o1, y);
    }
}

template <bool BF, int V>
__global__ __launch_bounds__(256) void rotary_k(RotaryArgs a) {
    __shared__ __attribute__((aligned(16))) float lds[ROT_LDS];
    const int row0 = blockIdx.x * a.per_block;
    const int n = min(a.rows_dev ? *a.rows_dev : a.rows, a.rows) - row0;
    if (n > 0) turn_rows<BF, V, 256>(a, a.rot, row0, min(n, a.per_block), lds);
}

// ---- codes -----------------------------------------------------------------------------------------
// e4m3 codes of four floats already divided by the scale
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
__device__ __forceinline__ void decode4(uint32_t w, float s, float (&x)[4]) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a[0] * s, x[1] = a[1] * s, x[2] = b[0] * s, x[3] = b[1] * s;
}
// four dwords of bytes, transposed
__device__ __forceinline__ void transpose4(uint32_t (&w)[4]) {
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400), b = __builtin_amdgcn_perm(w[3], w[2], 0x05010400);
    const uint32_t c = __builtin_amdgcn_perm(w[1], w[0], 0x07030602), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
    w[0] = __builtin_amdgcn_perm(b, a, 0x05040100), w[1] = __builtin_amdgcn_perm(b, a, 0x07060302);
    w[2] = __builtin_amdgcn_perm(d, c, 0x05040100), w[3] = __builtin_amdgcn_perm(d, c, 0x07060302);
}
// The least power of two >= 2^-126 with most <= 448 of it: 448 = 1.75 * 2^8, so the exponent of `most` goes up
// by one where its fraction passes 0.75.
__device__ __forceinline__ float scale_for(float most) {
    const int e = (int)((__builtin_bit_cast(uint32_t, most) + 0x1FFFFFu) >> 23) - 8;
    return __builtin_bit_cast(float, (uint32_t)max(e, 1) << 23);
}
// 1 / s of a power of two in [2^-126, 2^120]
__device__ __forceinline__ float inverse(float s) {
    return __builtin_bit_cast(float, 0x7F000000u - __builtin_bit_cast(uint32_t, s));
}
// The part of a page that slot u stands for.
__device__ __forceinline__ PagePart page_part(const SeqArgs& q, int pt, int pages, int u) {
    const int shift = page_shift(pt);
    const Seq s = q.offsets ? find_seq(q, [&](const Seq& x) { return part_count(x, shift); }, u) : seq_of(q, q.one ? 0 : u);
    return part_at(q, pt, pages, s, u);
}

// ---- write -----------------------------------------------------------------------------------------
// A block quantises the new tokens of one page, keys or values, of a few heads, and owns those: it alone reads and
// writes their codes and scales.  A pass asks for all its loads together, 32 bytes or more a thread (one item a
// thread, at five or six wavefronts a SIMD instead of four, is 20 % slower: more passes, each a chain of the page's
// table entry, rows, scale and codes).  Further blocks turn the query rows.
constexpr int MAX_ITEMS = 2;                    // items of 16 channels a thread and pass
// WT threads a block (write_threads).
template <bool BF, int V, int WT>
__global__ __launch_bounds__(WT, 4) void cache_write_k(WriteArgs a) {
    constexpr int PASS = MAX_ITEMS * WT;      // items of a pass: one head's, or more heads'
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ uint32_t s_most[WRITE_HEADS];
    __shared__ float s_scale[WRITE_HEADS], s_old[WRITE_HEADS];
    const int tid = threadIdx.x;
    const int dh = a.c.head_dim, pt = a.c.page_tokens, H = a.c.kv_heads;
    if (blockIdx.x >= (unsigned)a.kv_blocks) {   // queries
        const RowsArgs q = {a.q, a.q_out, a.q_stride, a.qo_stride, a.q_heads, dh, a.pos, nullptr, 0};
        const int b = (blockIdx.x - a.kv_blocks) * a.q_rows;
        const int row0 = a.seq.offsets ? max(a.seq.offsets[0], b) : b;   // rows before it are no sequence's
        const int live = a.seq.offsets ? min(a.seq.offsets[a.seq.n_seqs], a.seq.rows) : min(a.seq.n_seqs, a.seq.rows);
        const int n = min(live, b + a.q_rows) - row0;
        if (n > 0) turn_rows<BF, V, WT>(q, a.rot, row0, n, (float*)lds);
        return;
    }
    const int groups = (H + a.heads - 1) / a.heads, hg = blockIdx.x % groups;
    const bool values = blockIdx.x / groups & 1;
    const PagePart p = page_part(a.seq, pt, a.c.pages, blockIdx.x / (2 * groups));
    if (p.page < 0 || p.n == 0) return;
    const void* src = values ? a.v : a.k;
    const size_t stride = values ? a.v_stride : a.k_stride;
    const int dim = values ? 0 : a.rot.dim;   // channels that are turned
    const int per_tok = dh / 16, per_head = p.n * per_tok, keep = p.slot0;
    const int end = min(H, (hg + 1) * a.heads);
    // keys: cosines and sines [token][pair], once for all heads; values: codes [head][token][channel + 4]
    const int ald = (dim / 2 + 3) & ~3, ld = dh + 4;
    float *cos = (float*)lds, *sin = cos + p.n * ald;
    uint8_t* tile = lds;
    if (dim) angles_of<WT>(a.rot, p.n, cos, sin, ald, [&](int r) { return a.pos + (size_t)(p.row0 + r) * 3; });
    // i / per_head for i < 2^10, per_head <= 2^10 (the error of the factor, below per_head, times i is below 2^20)
    const uint32_t by_head = ((1u << 20) + per_head - 1) / per_head;

    for (int h0 = hg * a.heads, hn; h0 < end; h0 += hn) {
        hn = max(1, min(end - h0, PASS / per_head));
        float* scales = (values ? a.c.v_scale : a.c.k_scale) + (size_t)p.page * H + h0;
        uint8_t* codes = (values ? a.c.v : a.c.k) + ((size_t)p.page * H + h0) * pt * dh;
        float old = 0.f;
        if (tid < hn) {
            s_most[tid] = 0;
            if (keep > 0) old = scales[tid];
        }
        // the pass's new values in registers
        float x[MAX_ITEMS][16];
        int hh[MAX_ITEMS], tt[MAX_ITEMS], cc[MAX_ITEMS];
#pragma unroll
        for (int k = 0; k < MAX_ITEMS; ++k) {
            const int i = tid + k * WT;
            hh[k] = (int)(i * by_head >> 20);
            const int rest = i - hh[k] * per_head;
            tt[k] = div_by(rest, a.by_tok), cc[k] = rest - tt[k] * per_tok;
            if (hh[k] >= hn) continue;
            const int row = p.row0 + tt[k];
            const size_t at = (size_t)(a.row_idx ? a.row_idx[row] : row) * stride + (size_t)(h0 + hh[k]) * dh;
#pragma unroll
            for (int e = 0; e < 8 / V; ++e) {
                const Item it = item_at<V>(dim, a.rot.pairs, cc[k] * (8 / V) + e);
                float u[V], w[V];
                load_ch<BF, V>(src, at + it.o0, u);
                load_ch<BF, V>(src, at + it.o1, w);
#pragma unroll
                for (int f = 0; f < V; ++f) x[k][e * V + f] = u[f], x[k][8 + e * V + f] = w[f];
            }
        }
        __syncthreads();   // s_most is cleared, the angles are there
#pragma unroll
        for (int k = 0; k < MAX_ITEMS; ++k) {
            if (hh[k] >= hn) continue;
#pragma unroll
            for (int e = 0; e < 8 / V; ++e) {
                const int c = cc[k] * (8 / V) + e, at = tt[k] * ald + c * V;
                if (c * 2 * V >= dim) continue;
                float u[V], w[V];
#pragma unroll
                for (int f = 0; f < V; ++f) u[f] = x[k][e * V + f], w[f] = x[k][8 + e * V + f];
                turn_item<V>(a.rot.pairs, cos + at, sin + at, u, w);
#pragma unroll
                for (int f = 0; f < V; ++f) x[k][e * V + f] = u[f], x[k][8 + e * V + f] = w[f];
            }
            float most = 0.f;   // a NaN does not count
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, fabsf(x[k][e]));
            if (most > 3.4028235e38f) {   // infinities become NaN: the format has none, and 448 would hide them
                most = 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    x[k][e] = fabsf(x[k][e]) <= 3.4028235e38f ? x[k][e] : __builtin_nanf("");
                    most = fmaxf(most, fabsf(x[k][e]));
                }
            }
            atomicMax(&s_most[hh[k]], __builtin_bit_cast(uint32_t, most));   // (of LDS; the order does not matter)
        }
        __syncthreads();
        if (tid < hn) {
            const float scale = fmaxf(old, scale_for(__builtin_bit_cast(float, s_most[tid])));
            s_old[tid] = keep > 0 ? old : scale;
            s_scale[tid] = scale;
            scales[tid] = scale;
        }
        __syncthreads();
        for (int j = 0; keep > 0 && j < hn; ++j) {   // the tokens that the page held, where the scale has grown
            if (!(s_old[j] < s_scale[j])) continue;
            const float f = s_old[j] * inverse(s_scale[j]);
            uint8_t* base = codes + (size_t)j * pt * dh;
            auto again = [&](uint32_t w) {
                float v[4];
                decode4(w, f, v);
                return code4(v[0], v[1], v[2], v[3]);
            };
            if (!values) {
                for (int i = tid; i < keep * dh / 4; i += WT) ((uint32_t*)base)[i] = again(((uint32_t*)base)[i]);
            } else {
                const int words = (keep + 3) / 4;   // of each channel; the last may hold places that stay as they are
                for (int i = tid; i < words * dh; i += WT) {
                    uint32_t* at = (uint32_t*)(base + (size_t)(i / words) * pt) + i % words;
                    const int live = min(4, keep - i % words * 4);
                    const uint32_t mask = live == 4 ? 0xFFFFFFFFu : (1u << 8 * live) - 1, w = *at;
                    *at = (again(w) & mask) | (w & ~mask);
                }
            }
        }
        // codes: keys go to their place; values into LDS, token by token
#pragma unroll
        for (int k = 0; k < MAX_ITEMS; ++k) {
            if (hh[k] >= hn) continue;
            const float inv = inverse(s_scale[hh[k]]);
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                w[e] = code4(x[k][4 * e] * inv, x[k][4 * e + 1] * inv, x[k][4 * e + 2] * inv, x[k][4 * e + 3] * inv);
            if constexpr (V == 8) {
                const Item it = item_at<8>(dim, a.rot.pairs, cc[k]);
                if (values) {
                    uint32_t* to = (uint32_t*)(tile + (hh[k] * p.n + tt[k]) * ld + it.o0);   // (o1 = o0 + 8)
                    to[0] = w[0], to[1] = w[1], to[2] = w[2], to[3] = w[3];
                } else {
                    uint8_t* to = codes + ((size_t)hh[k] * pt + p.slot0 + tt[k]) * dh;
                    *(u32x2*)(to + it.o0) = (u32x2){w[0], w[1]};
                    *(u32x2*)(to + it.o1) = (u32x2){w[2], w[3]};
                }
            } else {
                uint8_t* to = values ? tile + (hh[k] * p.n + tt[k]) * ld
                                     : codes + ((size_t)hh[k] * pt + p.slot0 + tt[k]) * dh;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const Item it = item_at<1>(dim, a.rot.pairs, cc[k] * 8 + e);
                    to[it.o0] = (uint8_t)(w[e >> 2] >> 8 * (e & 3));
                    to[it.o1] = (uint8_t)(w[2 + (e >> 2)] >> 8 * (e & 3));
                }
            }
        }
        if (values) {
            __syncthreads();   // the rescaled words and the tile are complete
            // four channels of 16 tokens at once, neighbouring lanes on a channel's neighbouring tokens; where
            // the new tokens fill fewer, by fours and byte by byte (300 sequences of 30 tokens of 16 heads of 64: 57
            // us with bytes alone, 38 so)
            const int first = keep >> 4, chunks = ((keep + p.n + 15) >> 4) - first, quads = dh / 4;
            for (int i = tid; i < hn * quads * chunks; i += WT) {
                const int row = i / chunks, j = first + i - row * chunks;           // row: head and four channels
                const int hd = row / quads, c4 = row - hd * quads, t0 = j * 16 - keep;   // t0: token of the first byte
                const uint8_t* from = tile + (hd * p.n + t0) * ld + c4 * 4;
                uint8_t* to = codes + ((size_t)hd * dh + c4 * 4) * pt + j * 16;
                if (t0 >= 0 && t0 + 16 <= p.n) {
                    u32x4 w[4];
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        uint32_t q[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) q[e] = *(const uint32_t*)(from + (4 * g + e) * ld);
                        transpose4(q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e][g] = q[e];
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) *(u32x4*)(to + (size_t)e * pt) = w[e];
                    continue;
                }
                for (int t = max(0, -t0); t < min(16, p.n - t0);) {
                    if ((t & 3) == 0 && t0 + t + 4 <= p.n) {
                        uint32_t q[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) q[e] = *(const uint32_t*)(from + (t + e) * ld);
                        transpose4(q);
#pragma unroll
                        for (int e = 0; e < 4; ++e) *(uint32_t*)(to + e * pt + t) = q[e];
                        t += 4;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[e * pt + t] = from[t * ld + e];
                        ++t;
                    }
                }
            }
        }
        __syncthreads();   // the next pass takes the tile and the scales' places again
    }
}

// ---- read ------------------------------------------------------------------------------------------
// four codes to bf16 (v_cvt_scalef32_pk_bf16_fp8 applies the scale, exactly)
__device__ __forceinline__ u32x2 decode_bf16(uint32_t w, float scale) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
    return (u32x2){__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
}
// Eight codes of one row to its channels `to` ..
template <bool BF, bool WIDE>
__device__ __forceinline__ void store_codes(void* dst, size_t to, uint32_t lo, uint32_t hi, float scale) {
    if constexpr (BF) {
        const u32x2 a = decode_bf16(lo, scale), b = decode_bf16(hi, scale);
        const u32x4 r = {a[0], a[1], b[0], b[1]};
        uint16_t* p = (uint16_t*)dst + to;
        if constexpr (WIDE) {
            *(u32x4*)p = r;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = (uint16_t)(r[e >> 1] >> 16 * (e & 1));
        }
    } else {
        float x[4], y[4];
        decode4(lo, scale, x);
        decode4(hi, scale, y);
        float* p = (float*)dst + to;
        if constexpr (WIDE) {
            *(f32x4*)p = (f32x4){x[0], x[1], x[2], x[3]};
            *(f32x4*)(p + 4) = (f32x4){y[0], y[1], y[2], y[3]};
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] = x[e], p[4 + e] = y[e];
        }
    }
}

// One block per page part, head, and keys or values.  A page that the cache does not have reads as zeros.  A
// lane stores eight channels of a token, neighbouring lanes neighbouring channels; values pass through
// LDS, where a lane takes eight channels of four tokens (100,003 tokens of 8 heads of 128, us: 155 with those
// dwords from memory, 173 byte by byte from LDS).
template <bool BF, bool WIDE>
__global__ __launch_bounds__(256) void cache_read_k(ReadArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t tile[];   // values: codes [channel][token + 4]
    const int tid = threadIdx.x;
    const int dh = a.c.head_dim, pt = a.c.page_tokens, H = a.c.kv_heads;
    const int h = blockIdx.x % H;
    const bool values = blockIdx.x / H & 1;
    const PagePart p = page_part(a.seq, pt, a.c.pages, blockIdx.x / (2 * H));
    if (p.n == 0) return;
    const bool there = p.page >= 0;
    const size_t at = (size_t)max(p.page, 0) * H + h;
    const uint8_t* codes = (values ? a.c.v : a.c.k) + at * pt * dh;
    const float scale = there ? (values ? a.c.v_scale : a.c.k_scale)[at] : 1.f;
    const uint32_t keep = there ? 0xFFFFFFFFu : 0u;
    const int oct = dh / 8;
    if (!values) {
        for (int i = tid; i < p.n * oct; i += 256) {
            const int t = div_by(i, a.by_oct), c = (i - t * oct) * 8;
            const u32x2 w = *(const u32x2*)(codes + (size_t)(p.slot0 + t) * dh + c);
            store_codes<BF, WIDE>(a.k, (size_t)(p.row0 + t) * a.k_stride + (size_t)h * dh + c, w[0] & keep, w[1] & keep,
                                  scale);
        }
        return;
    }
    const int ld = pt + 4, shift = page_shift(pt) - 4;
    for (int i = tid; i < dh << shift; i += 256) {   // 16 tokens of a channel
        const u32x4 w = ((const u32x4*)codes)[i];
        uint32_t* to = (uint32_t*)(tile + (i >> shift) * ld + (i & ((1 << shift) - 1)) * 16);
        to[0] = w[0], to[1] = w[1], to[2] = w[2], to[3] = w[3];
    }
    __syncthreads();
    const int first = p.slot0 >> 2, groups = ((p.slot0 + p.n + 3) >> 2) - first;
    for (int i = tid; i < groups * oct; i += 256) {
        const int j = div_by(i, a.by_oct), c = (i - j * oct) * 8, tok = (first + j) * 4;
        uint32_t w[2][4];
#pragma unroll
        for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int e = 0; e < 4; ++e) w[g][e] = *(const uint32_t*)(tile + (c + 4 * g + e) * ld + tok) & keep;
            transpose4(w[g]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = tok + e - p.slot0;
            if (t >= 0 && t < p.n)
                store_codes<BF, WIDE>(a.v, (size_t)(p.row0 + t) * a.v_stride + (size_t)h * dh + c, w[0][e], w[1][e], scale);
        }
    }
}

bool aligned16(const void* p, size_t stride, size_t el) { return (uintptr_t)p % 16 == 0 && stride * el % 16 == 0; }

}  // namespace

void launch_rotary(bool bf, RotaryArgs a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    // eight channels at once where rows and heads start on 16 bytes and both halves of a turned pair do
    const bool wide = a.dh % 16 == 0 && a.rot.dim % 16 == 0 && aligned16(a.x, a.x_stride, el) &&
                      aligned16(a.out, a.out_stride, el);
    a.per_block = rows_a_block(a.heads, a.dh, wide ? 8 : 1);
    const dim3 grid((unsigned)(((long long)a.rows + a.per_block - 1) / a.per_block));
    if (bf && wide) rotary_k<true, 8><<<grid, 256, 0, s>>>(a);
    else if (bf) rotary_k<true, 1><<<grid, 256, 0, s>>>(a);
    else if (wide) rotary_k<false, 8><<<grid, 256, 0, s>>>(a);
    else rotary_k<false, 1><<<grid, 256, 0, s>>>(a);
}

void launch_cache_write(bool bf, WriteArgs a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    const CacheView& c = a.c;
    bool wide = a.rot.dim % 16 == 0 && aligned16(a.k, a.k_stride, el) && aligned16(a.v, a.v_stride, el);
    if (a.q) wide = wide && aligned16(a.q, a.q_stride, el) && aligned16(a.q_out, a.qo_stride, el);
    const int threads = write_threads(c.page_tokens, c.head_dim), pass = MAX_ITEMS * threads;
    const bool ragged = a.seq.offsets || a.seq.one;
    const long long slots = page_slots(ragged, a.seq.n_seqs, a.seq.rows, page_shift(c.page_tokens));
    a.heads = write_heads(slots, c.kv_heads, a.cus);
    a.kv_blocks = (int)(slots * 2 * ((c.kv_heads + a.heads - 1) / a.heads));
    a.q_rows = rows_a_block(std::max(1, a.q_heads), c.head_dim, wide ? 8 : 1);
    const dim3 grid((unsigned)(a.kv_blocks + (a.q ? ((long long)a.seq.rows + a.q_rows - 1) / a.q_rows : 0)));
    a.by_tok = div_magic(c.head_dim / 16);
    // a pass's codes, rows padded by 4 bytes (16 channels: a row an item); the angles of a page, or of q_rows rows
    const size_t lds = std::max({(size_t)pass * 20, (size_t)c.page_tokens * ((a.rot.dim / 2 + 3) & ~3) * 2 * sizeof(float),
                                 ROT_LDS * sizeof(float)});   // 64 KB at most
    auto go = [&](auto f, auto v) {
        constexpr bool B = decltype(f)::value;
        constexpr int V = decltype(v)::value;
        if (threads == 256) {
            cache_write_k<B, V, 256><<<grid, 256, lds, s>>>(a);
        } else {   // 64 KB beside the kernel's own
            static const bool ok = allow_lds((const void*)cache_write_k<B, V, 512>, 64 << 10);
            (void)ok;
            cache_write_k<B, V, 512><<<grid, 512, lds, s>>>(a);
        }
    };
    using W8 = std::integral_constant<int, 8>;
    using W1 = std::integral_constant<int, 1>;
    if (bf && wide) go(std::true_type(), W8());
    else if (bf) go(std::true_type(), W1());
    else if (wide) go(std::false_type(), W8());
    else go(std::false_type(), W1());
}

void launch_cache_read(bool bf, ReadArgs a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    const bool wide = aligned16(a.k, a.k_stride, el) && aligned16(a.v, a.v_stride, el);
    const long long slots = page_slots(a.seq.offsets || a.seq.one, a.seq.n_seqs, a.seq.rows,
                                       page_shift(a.c.page_tokens));
    a.by_oct = div_magic(a.c.head_dim / 8);
    const size_t lds = (size_t)a.c.head_dim * (a.c.page_tokens + 4);
    const dim3 grid((unsigned)(slots * 2 * a.c.kv_heads));
    if (bf && wide) cache_read_k<true, true><<<grid, 256, lds, s>>>(a);
    else if (bf) cache_read_k<true, false><<<grid, 256, lds, s>>>(a);
    else if (wide) cache_read_k<false, true><<<grid, 256, lds, s>>>(a);
    else cache_read_k<false, false><<<grid, 256, lds, s>>>(a);
}

}  // namespace dv

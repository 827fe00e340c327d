// Rotary positions of token rows, and the paged 8-bit cache of keys and values: quantised as it is
// written, read back.  All three are bound by the bytes they move.
//
// Rotary positions: pair i of a row is turned by pos[axis(i)] * f_i radians.  The angle is kept in turns:
// f_i / 2 pi as a 64-bit fraction (RotaryPlan::turn), so that the product with a 32-bit position, taken
// modulo 2^64, is the turn's fraction to 2^-33 at any position; fp32 angles are off by 2^-24 of the whole
// angle, 64 radians at position 2^30.  Sine and cosine are polynomials on an eighth of a turn, in fp32.
//
// Codes are e4m3 (1 sign, 4 exponent, 3 fraction bits; largest 448), rounded to nearest even by
// v_cvt_pk_fp8_f32.  Scales are powers of two, the least with every |x| <= 448 scale: a floating code
// gains nothing from a finer scale, and a power of two can grow with a page that fills over several
// calls while codes away from the format's underflow (2^-6 of a scale) stay exact.  Scales and sums are
// fp32.
#include "cache_plan.h"

namespace dv {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
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
// cos and sin of 2 pi pos turn / 2^64.  The low 64 bits of the product hold the fraction of a turn; its
// high half, rounded by the half of its low half, is a signed 32-bit fraction f.  The nearest eighth of a turn
// is taken off (|r| <= pi/4 after the nearest quarter), then the Taylor polynomials of degree 9 and 8:
// remainders (pi/4)^11 / 11! = 1.8e-9 and (pi/4)^10 / 10! = 2.5e-8, below half a step of fp32.
__device__ __forceinline__ void turn_cos_sin(int pos, uint64_t turn, float& c, float& s) {
    const uint64_t p = (uint64_t)(int64_t)pos * turn;
    const uint32_t f = (uint32_t)((p + 0x80000000ull) >> 32);
    const uint32_t q = (f + 0x20000000u) >> 30;                 // nearest quarter, modulo 4
    const float r = (float)(int32_t)(f - (q << 30)) * 1.4629180792671596e-09f;   // 2 pi / 2^32
    const float r2 = r * r;
    const float sn = fmaf(fmaf(fmaf(fmaf(2.7557319e-6f, r2, -1.9841270e-4f), r2, 8.3333333e-3f), r2, -1.6666667e-1f),
                          r2 * r, r);
    const float cs = fmaf(fmaf(fmaf(fmaf(2.4801587e-5f, r2, -1.3888889e-3f), r2, 4.1666667e-2f), r2, -0.5f), r2, 1.0f);
    c = q & 1 ? sn : cs;
    s = q & 1 ? cs : sn;
    if (q == 1 || q == 2) c = -c;
    if (q >= 2) s = -s;
}
__device__ __forceinline__ int axis_of(const RotaryPlan& r, int pair) {
    return pair < r.end0 ? 0 : pair < r.end1 ? 1 : 2;
}

// An item is two groups of V channels of one row and head that the rotation mixes (or, past the turned
// channels, leaves): items of the `dim` turned channels first.
//   halves: channels o .. o + V - 1 with o + dim/2 ..; pairs (V = 8): 16 channels in a row, (V = 1): 2
struct Item {
    int o0, o1;
    bool turned;
};
template <int V>
__device__ __forceinline__ Item item_at(int dim, bool pairs, int i) {
    const int turned = dim / (2 * V);
    if (i >= turned) return {i * 2 * V, i * 2 * V + V, false};
    if (pairs) return {i * 2 * V, i * 2 * V + V, true};
    return {i * V, i * V + dim / 2, true};
}
template <int V>
__device__ __forceinline__ void turn_item(const RotaryPlan& r, const Item& it, const int* pos, float (&a)[V],
                                          float (&b)[V]) {
    if (!it.turned) return;
    int p3[3];
#pragma unroll
    for (int x = 0; x < 3; ++x) p3[x] = pos[x];
    auto rotate = [&](int pair, float& x, float& y) {
        const int ax = axis_of(r, pair);
        float c, s;
        turn_cos_sin(ax == 0 ? p3[0] : ax == 1 ? p3[1] : p3[2], r.turn[pair], c, s);
        const float u = x * c - y * s;
        y = fmaf(x, s, y * c);
        x = u;
    };
    if (V == 1 || !r.pairs) {
        const int first = r.pairs ? it.o0 / 2 : it.o0;
#pragma unroll
        for (int i = 0; i < V; ++i) rotate(first + i, a[i], b[i]);
    } else if constexpr (V > 1) {
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            rotate((it.o0 + i) / 2, a[i], a[i + 1]);
            rotate((it.o1 + i) / 2, b[i], b[i + 1]);
        }
    }
}

// out row = the row with its heads turned.  One item per thread.
template <bool BF, int V>
__global__ __launch_bounds__(256) void rotary_k(RotaryArgs a) {
    const int per_head = a.dh / (2 * V), per_row = per_head * a.heads;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(i / per_row);
    const int rows = a.rows_dev ? *a.rows_dev : a.rows;
    if (row >= rows) return;
    const int rest = (int)(i % per_row), h = rest / per_head;
    const Item it = item_at<V>(a.rot.dim, a.rot.pairs, rest % per_head);
    const int* pos = a.pos + (size_t)(a.pos_idx ? a.pos_idx[row] % a.pos_mod : row) * 3;
    float x[V], y[V];
    const size_t at = (size_t)row * a.x_stride + (size_t)h * a.dh;
    load_ch<BF, V>(a.x, at + it.o0, x);
    load_ch<BF, V>(a.x, at + it.o1, y);
    turn_item<V>(a.rot, it, pos, x, y);
    const size_t to = (size_t)row * a.out_stride + (size_t)h * a.dh;
    store_ch<BF, V>(a.out, to + it.o0, x);
    store_ch<BF, V>(a.out, to + it.o1, y);
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
// Infinities are stored as NaN: the format has none, and a largest finite value would hide them.
__device__ __forceinline__ float storable(float x) {
    return fabsf(x) <= 3.4028235e38f ? x : __builtin_nanf("");
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
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// The part of a page that slot u stands for.
__device__ __forceinline__ PagePart page_part(const SeqArgs& q, int pt, int pages, int u) {
    const int s = q.one ? 0 : q.offsets ? find_seq(q.offsets, q.n_seqs, 1, page_shift(pt), 2, u) : u;
    return part_at(q, pt, pages, s, u);
}

// ---- write -----------------------------------------------------------------------------------------
// A block quantises the new tokens of one page and key/value head, keys or values, and owns that page: it
// alone reads and writes its codes and its scale.  Further blocks turn the query rows.
constexpr int MAX_ITEMS = 4;   // items of 16 channels per thread: 128 tokens of 128 channels over 256 threads

template <bool BF, int V>
__device__ __forceinline__ void load_item(const void* src, size_t at, const Item& it, const RotaryPlan& r,
                                          const int* pos, float (&x)[V], float (&y)[V]) {
    load_ch<BF, V>(src, at + it.o0, x);
    load_ch<BF, V>(src, at + it.o1, y);
    turn_item<V>(r, it, pos, x, y);
}

template <bool BF>
__global__ __launch_bounds__(256) void cache_write_k(WriteArgs a) {
    __shared__ float s_most[4];
    extern __shared__ __attribute__((aligned(16))) uint8_t tile[];   // values: codes [token][channel + 4]
    const int tid = threadIdx.x;
    const int dh = a.c.head_dim, pt = a.c.page_tokens, H = a.c.kv_heads;
    const long long kv_blocks = (long long)a.slots * 2 * H;
    if (blockIdx.x >= kv_blocks) {   // queries: one item of 2 x 8 (or 2 x 1) channels per thread
        const int V = a.vec;
        const int per_head = dh / (2 * V), per_row = per_head * a.q_heads;
        const long long i = ((long long)blockIdx.x - kv_blocks) * 256 + tid;
        const int row = (int)(i / per_row);
        const int live = a.seq.offsets ? min(a.seq.offsets[a.seq.n_seqs], a.seq.rows) : min(a.seq.n_seqs, a.seq.rows);
        if (row >= live) return;
        const int rest = (int)(i % per_row), h = rest / per_head;
        const size_t at = (size_t)row * a.q_stride + (size_t)h * dh, to = (size_t)row * a.qo_stride + (size_t)h * dh;
        auto go = [&](auto v) {
            constexpr int W = decltype(v)::value;
            const Item it = item_at<W>(a.rot.dim, a.rot.pairs, rest % per_head);
            float x[W], y[W];
            load_item<BF, W>(a.q, at, it, a.rot, a.pos + (size_t)row * 3, x, y);
            store_ch<BF, W>(a.q_out, to + it.o0, x);
            store_ch<BF, W>(a.q_out, to + it.o1, y);
        };
        if (V == 8) go(std::integral_constant<int, 8>());
        else go(std::integral_constant<int, 1>());
        return;
    }
    const int h = blockIdx.x % H;
    const bool values = blockIdx.x / H & 1;
    const PagePart p = page_part(a.seq, pt, a.c.pages, blockIdx.x / (2 * H));
    if (p.page < 0 || p.n == 0) return;
    const void* src = values ? a.v : a.k;
    const size_t stride = values ? a.v_stride : a.k_stride;
    float* scales = (values ? a.c.v_scale : a.c.k_scale) + (size_t)p.page * H + h;
    uint8_t* codes = (values ? a.c.v : a.c.k) + ((size_t)p.page * H + h) * pt * dh;
    const int dim = values ? 0 : a.rot.dim;   // channels that are turned

    // all new values of the page and head in registers: 16 (or 2) channels an item
    const int per_tok = dh / 16, items = p.n * per_tok;
    float x[MAX_ITEMS][16];
    float most = 0.f;
#pragma unroll
    for (int k = 0; k < MAX_ITEMS; ++k) {
        const int i = tid + k * 256;
        if (i >= items) break;
        const int t = i / per_tok, c = i % per_tok, row = p.row0 + t;
        const size_t at = (size_t)(a.row_idx ? a.row_idx[row] : row) * stride + (size_t)h * dh;
        const int* pos = a.pos + (size_t)row * 3;
        if (a.vec == 8) {
            float u[8], w[8];
            load_item<BF, 8>(src, at, item_at<8>(dim, a.rot.pairs, c), a.rot, pos, u, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[k][e] = u[e], x[k][8 + e] = w[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float u[1], w[1];
                load_item<BF, 1>(src, at, item_at<1>(dim, a.rot.pairs, c * 8 + e), a.rot, pos, u, w);
                x[k][e] = u[0], x[k][8 + e] = w[0];
            }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            x[k][e] = storable(x[k][e]);
            most = fmaxf(most, fabsf(x[k][e]));   // a NaN does not count
        }
    }
    most = wave_max(most);
    if ((tid & 63) == 0) s_most[tid >> 6] = most;
    __syncthreads();
    most = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3]));
    const int keep = p.slot0;
    const float old = keep > 0 ? *scales : 0.f;
    const float scale = fmaxf(old, scale_for(most)), inv = inverse(scale);
    if (keep > 0 && old < scale) {   // the tokens that the page held
        const float f = old * inv;
        auto again = [&](uint32_t w) {
            float v[4];
            decode4(w, f, v);
            return code4(v[0], v[1], v[2], v[3]);
        };
        if (!values) {
            for (int i = tid; i < keep * dh / 4; i += 256) ((uint32_t*)codes)[i] = again(((uint32_t*)codes)[i]);
        } else {
            const int words = (keep + 3) / 4;   // of each channel; the last may hold places that stay as they are
            for (int i = tid; i < words * dh; i += 256) {
                uint32_t* at = (uint32_t*)(codes + (size_t)(i / words) * pt) + i % words;
                const int live = min(4, keep - i % words * 4);
                const uint32_t mask = live == 4 ? 0xFFFFFFFFu : (1u << 8 * live) - 1;
                *at = (again(*at) & mask) | (*at & ~mask);
            }
        }
    }
    // codes: keys go to their place; values into LDS, token by token
    const int ld = dh + 4;
#pragma unroll
    for (int k = 0; k < MAX_ITEMS; ++k) {
        const int i = tid + k * 256;
        if (i >= items) break;
        const int t = i / per_tok, c = i % per_tok;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            w[e] = code4(x[k][4 * e] * inv, x[k][4 * e + 1] * inv, x[k][4 * e + 2] * inv, x[k][4 * e + 3] * inv);
        uint8_t* to = values ? tile + t * ld : codes + (size_t)(p.slot0 + t) * dh;
        if (a.vec == 8) {
            const Item it = item_at<8>(dim, a.rot.pairs, c);
            ((uint32_t*)(to + it.o0))[0] = w[0];
            ((uint32_t*)(to + it.o0))[1] = w[1];
            ((uint32_t*)(to + it.o1))[0] = w[2];
            ((uint32_t*)(to + it.o1))[1] = w[3];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const Item it = item_at<1>(dim, a.rot.pairs, c * 8 + e);
                to[it.o0] = (uint8_t)(w[e >> 2] >> 8 * (e & 3));
                to[it.o1] = (uint8_t)(w[2 + (e >> 2)] >> 8 * (e & 3));
            }
        }
    }
    __syncthreads();   // the rescaled words and the tile are complete
    if (values) {
        for (int i = tid; i < p.n * dh; i += 256) {
            const int ch = i / p.n, t = i % p.n;
            codes[(size_t)ch * pt + p.slot0 + t] = tile[t * ld + ch];
        }
    }
    if (tid == 0) *scales = scale;
}

// ---- read ------------------------------------------------------------------------------------------
// One block per page part, head, and keys or values.  A page that the cache does not have reads as zeros.
template <bool BF>
__global__ __launch_bounds__(256) void cache_read_k(ReadArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t tile[];   // values: codes [channel][token + 4]
    const int tid = threadIdx.x;
    const int dh = a.c.head_dim, pt = a.c.page_tokens, H = a.c.kv_heads;
    const int h = blockIdx.x % H;
    const bool values = blockIdx.x / H & 1;
    const PagePart p = page_part(a.seq, pt, a.c.pages, blockIdx.x / (2 * H));
    if (p.n == 0) return;
    void* dst = values ? a.v : a.k;
    const size_t stride = values ? a.v_stride : a.k_stride;
    const int per_tok = dh / 16, items = p.n * per_tok;
    const bool there = p.page >= 0;
    const size_t at = ((size_t)max(p.page, 0) * H + h);
    const uint8_t* codes = (values ? a.c.v : a.c.k) + at * pt * dh;
    const float scale = there ? (values ? a.c.v_scale : a.c.k_scale)[at] : 0.f;
    const int ld = pt + 4;
    if (values) {
        const int words = pt / 4;
        for (int i = tid; i < words * dh; i += 256)
            *(uint32_t*)(tile + i / words * ld + i % words * 4) = ((const uint32_t*)codes)[i];
        __syncthreads();
    }
    for (int i = tid; i < items; i += 256) {
        const int t = i / per_tok, c = i % per_tok * 16;
        uint32_t w[4];
        if (values) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = 0;
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    w[e] |= (uint32_t)tile[(c + 4 * e + b) * ld + p.slot0 + t] << 8 * b;
            }
        } else {
            const u32x4 r = *(const u32x4*)(codes + (size_t)(p.slot0 + t) * dh + c);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = r[e];
        }
        float x[16];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float v[4];
            decode4(w[e], scale, v);
#pragma unroll
            for (int b = 0; b < 4; ++b) x[4 * e + b] = there ? v[b] : 0.f;
        }
        const size_t to = (size_t)(p.row0 + t) * stride + (size_t)h * dh + c;
        if (a.vec == 8) {
            float u[8], v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = x[e], v[e] = x[8 + e];
            store_ch<BF, 8>(dst, to, u);
            store_ch<BF, 8>(dst, to + 8, v);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float u[1] = {x[e]};
                store_ch<BF, 1>(dst, to + e, u);
            }
        }
    }
}

bool aligned16(const void* p, size_t stride, size_t el) { return (uintptr_t)p % 16 == 0 && stride * el % 16 == 0; }

}  // namespace

void launch_rotary(bool bf, const RotaryArgs& a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    // eight channels at once where rows and heads start on 16 bytes and both halves of a turned pair do
    const bool wide = a.dh % 16 == 0 && a.rot.dim % 16 == 0 && aligned16(a.x, a.x_stride, el) &&
                      aligned16(a.out, a.out_stride, el);
    const long long items = (long long)a.rows * a.heads * (a.dh / (wide ? 16 : 2));
    const dim3 grid((unsigned)((items + 255) / 256));
    if (bf && wide) rotary_k<true, 8><<<grid, 256, 0, s>>>(a);
    else if (bf) rotary_k<true, 1><<<grid, 256, 0, s>>>(a);
    else if (wide) rotary_k<false, 8><<<grid, 256, 0, s>>>(a);
    else rotary_k<false, 1><<<grid, 256, 0, s>>>(a);
}

void launch_cache_write(bool bf, WriteArgs a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    bool wide = a.rot.dim % 16 == 0 && aligned16(a.k, a.k_stride, el) && aligned16(a.v, a.v_stride, el);
    if (a.q) wide = wide && aligned16(a.q, a.q_stride, el) && aligned16(a.q_out, a.qo_stride, el);
    a.vec = wide ? 8 : 1;
    a.slots = (int)page_slots(a.seq.offsets || a.seq.one, a.seq.n_seqs, a.seq.rows, page_shift(a.c.page_tokens));
    const long long q_items = a.q ? (long long)a.seq.rows * a.q_heads * (a.c.head_dim / (2 * a.vec)) : 0;
    const dim3 grid((unsigned)((long long)a.slots * 2 * a.c.kv_heads + (q_items + 255) / 256));
    const size_t lds = (size_t)a.c.page_tokens * (a.c.head_dim + 4);
    if (bf) cache_write_k<true><<<grid, 256, lds, s>>>(a);
    else cache_write_k<false><<<grid, 256, lds, s>>>(a);
}

void launch_cache_read(bool bf, ReadArgs a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    a.vec = aligned16(a.k, a.k_stride, el) && aligned16(a.v, a.v_stride, el) ? 8 : 1;
    const long long slots = page_slots(a.seq.offsets || a.seq.one, a.seq.n_seqs, a.seq.rows,
                                       page_shift(a.c.page_tokens));
    const dim3 grid((unsigned)(slots * 2 * a.c.kv_heads));
    const size_t lds = (size_t)a.c.head_dim * (a.c.page_tokens + 4);
    if (bf) cache_read_k<true><<<grid, 256, lds, s>>>(a);
    else cache_read_k<false><<<grid, 256, lds, s>>>(a);
}

}  // namespace dv

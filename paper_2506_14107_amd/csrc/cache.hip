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
typedef float f32x8 __attribute__((ext_vector_type(8), aligned(16)));   // (rows start on 16 bytes, not on 32)
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
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

// V consecutive channels as fp32 (V = 8 and 4: 16 or 8 bytes at once, or 16; V = 1: one element)
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
    } else if constexpr (V == 4 && BF) {
        const bf16x4 r = *(const bf16x4*)((const uint16_t*)base + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)r[i];
    } else if constexpr (V == 4) {
        const f32x4 r = *(const f32x4*)((const float*)base + at);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = r[i];
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
    } else if constexpr (V == 4 && BF) {
        *(bf16x4*)((uint16_t*)base + at) = (bf16x4){(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
    } else if constexpr (V == 4) {
        *(f32x4*)((float*)base + at) = (f32x4){x[0], x[1], x[2], x[3]};
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
//   halves: channels o .. o + V - 1 with o + dim/2 ..; pairs: 2 V channels in a row
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
    if constexpr (V > 1) {
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
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

// ---- norms of heads --------------------------------------------------------------------------------
// A head x of dh channels becomes x w / sqrt(mean x^2 + eps), and is then turned: the sum of squares, the factor
// and the products are fp32, rounded once with the turned value.  A thread holds 16 channels of a head, of which the
// rotation mixes only those (item_at); the head's threads leave their sums of squares in LDS, side by side, and
// each adds them in the same order.  The rows' bytes bind: 16,448 rows of 32 heads of 80, bf16, 169 MB in 38 us (4.4 TB/s; a
// copy 4.96), where the turn alone takes 36; two chunks a thread, four 40.  Rows aligned to four channels but not to eight, or a
// quarter of a head turned, take loads of four (9232 rows of 16 heads of 80: 15 us, element by element 55).

// Channels of chunk c of a head (16 of them): x[e V + f] is channel o0 + f of item e, x[8 + e V + f] channel o1 + f.
template <bool BF, int V>
__device__ __forceinline__ void load_chunk(const void* base, size_t at, int dim, bool pairs, int c, float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 8 / V; ++e) {
        const Item it = item_at<V>(dim, pairs, c * (8 / V) + e);
        float u[V], w[V];
        load_ch<BF, V>(base, at + it.o0, u);
        load_ch<BF, V>(base, at + it.o1, w);
#pragma unroll
        for (int f = 0; f < V; ++f) x[e * V + f] = u[f], x[8 + e * V + f] = w[f];
    }
}
template <bool BF, int V>
__device__ __forceinline__ void store_chunk(void* base, size_t at, int dim, bool pairs, int c, const float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 8 / V; ++e) {
        const Item it = item_at<V>(dim, pairs, c * (8 / V) + e);
        float u[V], w[V];
#pragma unroll
        for (int f = 0; f < V; ++f) u[f] = x[e * V + f], w[f] = x[8 + e * V + f];
        store_ch<BF, V>(base, at + it.o0, u);
        store_ch<BF, V>(base, at + it.o1, w);
    }
}
// The same in two steps, for loads that are asked for well before they are needed: the chunk as it lies in memory, and x.
template <bool BF, int V>
struct Group;   // V channels; (a type passed as a template's argument would lose its alignment)
template <>
struct Group<true, 8> { using T = bf16x8; };
template <>
struct Group<true, 4> { using T = bf16x4; };
template <>
struct Group<true, 1> { using T = __bf16; };
template <>
struct Group<false, 8> { using T = f32x8; };
template <>
struct Group<false, 4> { using T = f32x4; };
template <>
struct Group<false, 1> { using T = float; };
template <bool BF, int V>
struct Raw {
    using T = typename Group<BF, V>::T;
    T v[16 / V];   // item e's two groups at 2 e and 2 e + 1
    static_assert(alignof(T) <= 16, "rows start on 16 bytes at best");
};
template <bool BF, int V>
__device__ __forceinline__ void load_raw(const void* base, size_t at, int dim, bool pairs, int c, Raw<BF, V>& r) {
    using T = typename Raw<BF, V>::T;
    const typename Elem<BF>::T* p = (const typename Elem<BF>::T*)base + at;
#pragma unroll
    for (int e = 0; e < 8 / V; ++e) {
        const Item it = item_at<V>(dim, pairs, c * (8 / V) + e);
        r.v[2 * e] = *(const T*)(p + it.o0);
        r.v[2 * e + 1] = *(const T*)(p + it.o1);
    }
}
template <bool BF, int V>
__device__ __forceinline__ void unpack(const Raw<BF, V>& r, float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 16 / V; ++e)
#pragma unroll
        for (int f = 0; f < V; ++f) {
            float y;
            if constexpr (V > 1) y = (float)r.v[e][f];
            else y = (float)r.v[e];
            x[e % 2 * 8 + e / 2 * V + f] = y;
        }
}
// ... turned where it is; cos and sin of its row
template <int V>
__device__ __forceinline__ void turn_chunk(int dim, bool pairs, int c, const float* cos, const float* sin, float (&x)[16]) {
#pragma unroll
    for (int e = 0; e < 8 / V; ++e) {
        const int i = c * (8 / V) + e;
        if (i * 2 * V >= dim) continue;
        float u[V], w[V];
#pragma unroll
        for (int f = 0; f < V; ++f) u[f] = x[e * V + f], w[f] = x[8 + e * V + f];
        turn_item<V>(pairs, cos + i * V, sin + i * V, u, w);
#pragma unroll
        for (int f = 0; f < V; ++f) x[e * V + f] = u[f], x[8 + e * V + f] = w[f];
    }
}
__device__ __forceinline__ float sum_squares(const float (&x)[16]) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) s = fmaf(x[e], x[e], s);
    return s;
}
// A head's squares are summed as this times their size, a power of two: channels of 2^60 each then sum to 2^127 at most, whatever
// the head (1 up to 128 channels).  Scaled exactly, sums round as they would without.
__device__ __forceinline__ float sum_scale(int dh) {
    const int over = 25 - __builtin_clz(dh - 1);   // of the least 2^n >= dh over 2^7
    return __builtin_bit_cast(float, (uint32_t)(127 - max(over, 0)) << 23);
}
// The weight's chunk, where there is a weight.
template <bool BF, int V>
__device__ __forceinline__ void load_weight(const NormArgs& nm, int dh, int h, int dim, bool pairs, int c, Raw<BF, V>& w) {
    if (nm.weight) load_raw<BF, V>(nm.weight, nm.per_head ? (size_t)h * dh : 0, dim, pairs, c, w);
}
// The mean square of a head; part: the sums of squares of its dh / 16 chunks.  WIDE: heads of more than 128 channels, in kernels of
// their own (the scale in all heads' sums, 1 up to 128 channels, cost 0.3 us of a call, a branch a register too many in fp32).
template <bool WIDE>
__device__ __forceinline__ float mean_square(const float* part, int dh) {
    const int n = dh / 16;
    float sum = 0.f, size = (float)dh;
    if (!WIDE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += i < n ? part[i] : 0.f;
    } else {
        const float down = sum_scale(dh);
        for (int i = 0; i < n; ++i) sum += part[i] * down;
        size *= down;
    }
    return sum / size;
}
// The chunk normed.
template <bool BF, int V, bool WIDE>
__device__ __forceinline__ void norm_chunk(const NormArgs& nm, const float* part, int dh, const Raw<BF, V>& w, float (&x)[16]) {
    const float f = rsqrtf(mean_square<WIDE>(part, dh) + nm.eps);
    if (nm.weight) {
        float y[16];
        unpack(w, y);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = x[e] * f * y[e];
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = x[e] * f;
    }
}

// Rows row0 .. row0 + n - 1 of x (n at most ROT_ROWS), heads of a multiple of 16 channels normed and turned, to out (a block
// of NT threads).  lds: ROT_LDS floats and NORM_ITEMS NT more.
constexpr int NORM_ITEMS = 2;   // chunks of a thread at once
template <bool BF, int V, int NT, bool WIDE>
__device__ __forceinline__ void norm_rows(const RowsArgs& a, const RotaryPlan& rot, const NormArgs& nm, int row0, int n,
                                          float* lds) {
    const int tid = threadIdx.x, ld = (rot.dim / 2 + 3) & ~3;
    float *cos = lds, *sin = lds + ROT_ROWS * 64, *part = lds + ROT_LDS;
    if (rot.dim) angles_of<NT>(rot, n, cos, sin, ld, [&](int r) { return a.pos + (size_t)(row0 + r) * 3; });
    const int per_head = a.dh / 16, per_row = per_head * a.heads, total = n * per_row;
    const int batch = NORM_ITEMS * NT / per_head * per_head;   // whole heads
    for (int first = 0; first < total; first += batch) {
        const int end = min(batch, total - first);
        float x[NORM_ITEMS][16];
        Raw<BF, V> r[NORM_ITEMS];
        int rr[NORM_ITEMS], hh[NORM_ITEMS], cc[NORM_ITEMS];
#pragma unroll
        for (int k = 0; k < NORM_ITEMS; ++k) {
            const int i = tid + k * NT;
            if (i >= end) continue;
            const int rest = (first + i) % per_row;
            rr[k] = (first + i) / per_row, hh[k] = rest / per_head, cc[k] = rest % per_head;
            load_raw<BF, V>(a.x, (size_t)(row0 + rr[k]) * a.x_stride + (size_t)hh[k] * a.dh, rot.dim, rot.pairs, cc[k], r[k]);
        }
#pragma unroll
        for (int k = 0; k < NORM_ITEMS; ++k) {
            if (tid + k * NT >= end) continue;
            unpack(r[k], x[k]);
            part[tid + k * NT] = sum_squares(x[k]);
        }
        __syncthreads();   // (the angles are there too)
#pragma unroll
        for (int k = 0; k < NORM_ITEMS; ++k) {
            const int i = tid + k * NT;
            if (i >= end) continue;
            Raw<BF, V> w;
            load_weight<BF, V>(nm, a.dh, hh[k], rot.dim, rot.pairs, cc[k], w);
            norm_chunk<BF, V, WIDE>(nm, part + i - cc[k], a.dh, w, x[k]);
            turn_chunk<V>(rot.dim, rot.pairs, cc[k], cos + rr[k] * ld, sin + rr[k] * ld, x[k]);
            store_chunk<BF, V>(a.out, (size_t)(row0 + rr[k]) * a.out_stride + (size_t)hh[k] * a.dh, rot.dim, rot.pairs, cc[k],
                               x[k]);
        }
        __syncthreads();   // the next batch takes the sums' places
    }
}
// The same for heads of any even number of channels: a wavefront goes over a head twice.
template <bool BF, int NT>
__device__ __forceinline__ void norm_rows_any(const RowsArgs& a, const RotaryPlan& rot, const NormArgs& nm, int row0, int n,
                                              float* lds) {
    const int lane = threadIdx.x & 63, ld = (rot.dim / 2 + 3) & ~3;
    const float down = sum_scale(a.dh);
    float *cos = lds, *sin = lds + ROT_ROWS * 64;
    if (rot.dim) angles_of<NT>(rot, n, cos, sin, ld, [&](int r) { return a.pos + (size_t)(row0 + r) * 3; });
    __syncthreads();
    for (int i = threadIdx.x >> 6; i < n * a.heads; i += NT / 64) {
        const int r = i / a.heads, h = i % a.heads;
        const size_t at = (size_t)(row0 + r) * a.x_stride + (size_t)h * a.dh;
        const size_t to = (size_t)(row0 + r) * a.out_stride + (size_t)h * a.dh, wat = nm.per_head ? (size_t)h * a.dh : 0;
        float sum = 0.f;
        for (int c = lane; c < a.dh; c += 64) {
            float x[1];
            load_ch<BF, 1>(a.x, at + c, x);
            sum = fmaf(x[0] * down, x[0], sum);
        }
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
        const float f = rsqrtf(sum / ((float)a.dh * down) + nm.eps);
        for (int p = lane; p < a.dh / 2; p += 64) {
            const Item it = item_at<1>(rot.dim, rot.pairs, p);
            float x[1], y[1], u[1] = {1.f}, w[1] = {1.f};
            load_ch<BF, 1>(a.x, at + it.o0, x);
            load_ch<BF, 1>(a.x, at + it.o1, y);
            if (nm.weight) {
                load_ch<BF, 1>(nm.weight, wat + it.o0, u);
                load_ch<BF, 1>(nm.weight, wat + it.o1, w);
            }
            x[0] = x[0] * f * u[0], y[0] = y[0] * f * w[0];
            if (it.turned) turn_item<1>(rot.pairs, cos + r * ld + p, sin + r * ld + p, x, y);
            store_ch<BF, 1>(a.out, to + it.o0, x);
            store_ch<BF, 1>(a.out, to + it.o1, y);
        }
    }
}

// V = 0: heads of any even number of channels.
template <bool BF, int V, bool WIDE>
__global__ __launch_bounds__(256) void norm_rotary_k(NormRotaryArgs a) {
    __shared__ __attribute__((aligned(16))) float lds[ROT_LDS + (V ? NORM_ITEMS * 256 : 0)];
    const int row0 = blockIdx.x * a.per_block, n = min(a.rows - row0, a.per_block);
    if constexpr (V > 0) norm_rows<BF, V, 256, WIDE>(a, a.rot, a.norm, row0, n, lds);
    else norm_rows_any<BF, 256>(a, a.rot, a.norm, row0, n, lds);
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
// table entry, rows, scale and codes).  Further blocks turn the query rows.  In bf16 the rows of the next pass are asked for while
// one is computed (60,000 tokens of 8 heads of 128 94 us without, 80 so; fp32 would spill: 26 us, 36), and the kernels with norms
// take three wavefronts a SIMD, whose registers hold that (9232 tokens of 16 heads of 80 with as many query heads, normed: 59 us with
// four and no rows ahead, 74 with four and spills, 52 with three and none ahead, 48 so; 118 MB).  Without norms the rows ahead spill four
// registers, which a call of one pass would only pay for (one token a sequence of 16 heads of 80, kernels one behind the other, us with / without
// them: 1 sequence 4.98 / 4.83, 48 6.41 / 6.25; 48 without a rotation 6.38 / 6.15): such calls take an instance without (write_in_one_pass).
constexpr int MAX_ITEMS = 2;                    // items of 16 channels a thread and pass
// WT threads a block (write_threads).  NORM: keys, queries or both are normed first.  MORE: blocks may take several passes.
template <bool BF, int V, int WT, bool NORM, bool MORE>
__global__ __launch_bounds__(WT, NORM ? 3 : 4) void cache_write_k(WriteArgs a) {
    constexpr int PASS = MAX_ITEMS * WT;      // items of a pass: one head's, or more heads'
    constexpr bool AHEAD = V > 1 && BF && MORE;   // (the others have no registers for it)
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
        if (n <= 0) return;
        if (NORM && a.q_norm.on) norm_rows<BF, V, WT, false>(q, a.rot, a.q_norm, row0, n, (float*)lds);
        else turn_rows<BF, V, WT>(q, a.rot, row0, n, (float*)lds);
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
    // keys: cosines and sines [token][pair], once for all heads, and sums of squares of the pass's items; values: codes
    // [head][token][channel + 4]
    const int ald = (dim / 2 + 3) & ~3, ld = dh + 4;
    float *cos = (float*)lds, *sin = cos + p.n * ald, *part = sin + p.n * ald;
    uint8_t* tile = lds;
    if (dim) angles_of<WT>(a.rot, p.n, cos, sin, ald, [&](int r) { return a.pos + (size_t)(p.row0 + r) * 3; });
    // i / per_head for i < 2^10, per_head <= 2^10 (the error of the factor, below per_head, times i is below 2^20)
    const uint32_t by_head = ((1u << 20) + per_head - 1) / per_head;

    // the thread's items of a pass: head, token, chunk
    int hh[MAX_ITEMS], tt[MAX_ITEMS], cc[MAX_ITEMS];
    auto place = [&](int k) {
        const int i = tid + k * WT;
        hh[k] = (int)(i * by_head >> 20);
        const int rest = i - hh[k] * per_head;
        tt[k] = div_by(rest, a.by_tok), cc[k] = rest - tt[k] * per_tok;
    };
    auto row_at = [&](int k, int h0) {
        const int row = p.row0 + tt[k];
        return (size_t)(a.row_idx ? a.row_idx[row] : row) * stride + (size_t)(h0 + hh[k]) * dh;
    };
    auto heads_from = [&](int h0) { return max(1, min(end - h0, PASS / per_head)); };
    auto scale_of = [&](int h0, int hn) {
        return keep > 0 && tid < hn ? (values ? a.c.v_scale : a.c.k_scale)[(size_t)p.page * H + h0 + tid] : 0.f;
    };
    // AHEAD: the rows and scales of a pass are asked for while the one before is computed
    Raw<BF, V> raw[AHEAD ? MAX_ITEMS : 1];
    float next = 0.f;
    auto ask = [&](int h0) {
        const int hn = heads_from(h0);
        next = scale_of(h0, hn);
#pragma unroll
        for (int k = 0; k < MAX_ITEMS; ++k)
            if (hh[k] < hn) load_raw<BF, V>(src, row_at(k, h0), dim, a.rot.pairs, cc[k], raw[k]);
    };
    if constexpr (AHEAD) {
#pragma unroll
        for (int k = 0; k < MAX_ITEMS; ++k) place(k);
        ask(hg * a.heads);
    }
    for (int h0 = hg * a.heads, hn; h0 < end; h0 += hn) {
        hn = heads_from(h0);
        float* scales = (values ? a.c.v_scale : a.c.k_scale) + (size_t)p.page * H + h0;
        uint8_t* codes = (values ? a.c.v : a.c.k) + ((size_t)p.page * H + h0) * pt * dh;
        if (tid < hn) s_most[tid] = 0;
        // the pass's new values in registers
        const float old = AHEAD ? next : scale_of(h0, hn);
        float x[MAX_ITEMS][16];
#pragma unroll
        for (int k = 0; k < MAX_ITEMS; ++k) {
            if constexpr (AHEAD) {
                if (hh[k] < hn) unpack(raw[k], x[k]);
            } else {
                place(k);
                if (hh[k] < hn) load_chunk<BF, V>(src, row_at(k, h0), dim, a.rot.pairs, cc[k], x[k]);
            }
        }
        if constexpr (AHEAD)
            if (h0 + hn < end) ask(h0 + hn);
        const bool normed = NORM && !values && a.k_norm.on;
        if (normed) {
#pragma unroll
            for (int k = 0; k < MAX_ITEMS; ++k) {
                if (hh[k] >= hn) continue;
                part[tid + k * WT] = sum_squares(x[k]);
            }
        }
        __syncthreads();   // s_most is cleared, the angles and the sums are there
#pragma unroll
        for (int k = 0; k < MAX_ITEMS; ++k) {
            if (hh[k] >= hn) continue;
            if (normed) {
                Raw<BF, V> w;
                load_weight<BF, V>(a.k_norm, dh, h0 + hh[k], dim, a.rot.pairs, cc[k], w);
                norm_chunk<BF, V, false>(a.k_norm, part + tid + k * WT - cc[k], dh, w, x[k]);
            }
            turn_chunk<V>(dim, a.rot.pairs, cc[k], cos + tt[k] * ald, sin + tt[k] * ald, x[k]);
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
            if constexpr (V == 4) {   // w[e] is group e / 2 of item e % 2
                uint8_t* to = values ? tile + (hh[k] * p.n + tt[k]) * ld
                                     : codes + ((size_t)hh[k] * pt + p.slot0 + tt[k]) * dh;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const Item it = item_at<4>(dim, a.rot.pairs, cc[k] * 2 + e);
                    *(uint32_t*)(to + it.o0) = w[e];
                    *(uint32_t*)(to + it.o1) = w[2 + e];
                }
            } else if constexpr (V == 8) {
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

bool aligned(size_t to, const void* p, size_t stride, size_t el) { return (uintptr_t)p % to == 0 && stride * el % to == 0; }
bool aligned16(const void* p, size_t stride, size_t el) { return aligned(16, p, stride, el); }

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

void launch_norm_rotary(bool bf, NormRotaryArgs a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    const bool chunks = a.dh % 16 == 0 && a.dh <= 16 * NORM_ITEMS * 256;
    auto fits = [&](int v, size_t to) {   // v channels at once, loads of `to` bytes
        return chunks && a.rot.dim % (2 * v) == 0 && aligned(to, a.x, a.x_stride, el) && aligned(to, a.out, a.out_stride, el) &&
               (uintptr_t)a.norm.weight % to == 0;
    };
    a.per_block = rows_a_block(a.heads, a.dh, chunks ? 8 : 1);
    const dim3 grid((unsigned)(((long long)a.rows + a.per_block - 1) / a.per_block));
    auto launch = [&](auto v, auto wide) {
        constexpr int V = decltype(v)::value;
        constexpr bool W = decltype(wide)::value;
        bf ? norm_rotary_k<true, V, W><<<grid, 256, 0, s>>>(a) : norm_rotary_k<false, V, W><<<grid, 256, 0, s>>>(a);
    };
    auto go = [&](auto v) { a.dh > 128 ? launch(v, std::true_type()) : launch(v, std::false_type()); };
    if (fits(8, 16)) go(std::integral_constant<int, 8>());
    else if (fits(4, 4 * el)) go(std::integral_constant<int, 4>());
    else if (chunks) go(std::integral_constant<int, 1>());
    else launch(std::integral_constant<int, 0>(), std::true_type());
}

void launch_cache_write(bool bf, WriteArgs a, hipStream_t s) {
    const size_t el = bf ? 2 : 4;
    const CacheView& c = a.c;
    const bool norm = a.k_norm.on || a.q_norm.on;
    auto fits = [&](int v, size_t to) {   // v channels at once, loads of `to` bytes
        return a.rot.dim % (2 * v) == 0 && aligned(to, a.k, a.k_stride, el) && aligned(to, a.v, a.v_stride, el) &&
               (!a.q || (aligned(to, a.q, a.q_stride, el) && aligned(to, a.q_out, a.qo_stride, el))) &&
               (uintptr_t)a.k_norm.weight % to == 0 && (uintptr_t)a.q_norm.weight % to == 0;
    };
    const bool wide = fits(8, 16);
    const int threads = write_threads(c.page_tokens, c.head_dim), pass = MAX_ITEMS * threads;
    const bool ragged = a.seq.offsets || a.seq.one;
    const long long slots = page_slots(ragged, a.seq.n_seqs, a.seq.rows, page_shift(c.page_tokens));
    a.heads = write_heads(slots, c.kv_heads, a.cus);
    a.kv_blocks = (int)(slots * 2 * ((c.kv_heads + a.heads - 1) / a.heads));
    a.q_rows = rows_a_block(std::max(1, a.q_heads), c.head_dim, wide || a.q_norm.on ? 8 : 1);
    const dim3 grid((unsigned)(a.kv_blocks + (a.q ? ((long long)a.seq.rows + a.q_rows - 1) / a.q_rows : 0)));
    a.by_tok = div_magic(c.head_dim / 16);
    // a pass's codes, rows padded by 4 bytes (16 channels: a row an item); the angles of a page, or of q_rows rows, and
    // sums of squares
    const size_t lds = std::max({(size_t)pass * 20,
                                 ((size_t)c.page_tokens * ((a.rot.dim / 2 + 3) & ~3) * 2 + (norm ? pass : 0)) * sizeof(float),
                                 (ROT_LDS + (norm ? NORM_ITEMS * threads : 0)) * sizeof(float)});   // 64 KB, 68 at most
    auto launch = [&](auto f, auto v, auto normed, auto several) {
        constexpr bool B = decltype(f)::value, N = decltype(normed)::value, M = decltype(several)::value;
        constexpr int V = decltype(v)::value;
        if (threads == 256) {
            cache_write_k<B, V, 256, N, M><<<grid, 256, lds, s>>>(a);
        } else {   // 64 KB beside the kernel's own
            static const bool ok = allow_lds((const void*)cache_write_k<B, V, 512, N, M>, N ? 68 << 10 : 64 << 10);
            (void)ok;
            cache_write_k<B, V, 512, N, M><<<grid, 512, lds, s>>>(a);
        }
    };
    using W8 = std::integral_constant<int, 8>;
    using W4 = std::integral_constant<int, 4>;
    using W1 = std::integral_constant<int, 1>;
    auto go = [&](auto v, auto normed) {
        bf ? launch(std::true_type(), v, normed, std::true_type()) : launch(std::false_type(), v, normed, std::true_type());
    };
    if (norm) {
        if (wide) go(W8(), std::true_type());
        else if (fits(4, 4 * el)) go(W4(), std::true_type());
        else go(W1(), std::true_type());
    } else if (wide && bf && write_in_one_pass(c.page_tokens, c.head_dim, a.heads, a.seq.n_seqs, a.seq.rows)) {
        launch(std::true_type(), W8(), std::false_type(), std::false_type());
    } else if (wide) {
        go(W8(), std::false_type());
    } else {
        go(W1(), std::false_type());
    }
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

"""Plain 64-bit versions of the operators on token rows and their 8-bit cache (numpy), and how far
the kernels may be from them.

Rounding is off by at most half a step: bf16 2^-8, e4m3 2^-4 (below 2^-6 of the scale half of 2^-9
of it), fp32 2^-24, relative to the value."""
import numpy as np

HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def angles(pos, sections, per_axis, base):
    dim = 2 * sum(sections)
    out, i = [], 0
    for axis, s in enumerate(sections):
        for j in range(s):
            rate = base ** (-j / s) if per_axis else base ** (-2 * i / dim)
            out.append(pos[:, axis].astype(np.float64) * rate)
            i += 1
    return np.stack(out, 1)                                    # [rows, dim / 2]


def turn(x, pos, sections, layout="halves", per_axis=False, base=1e4):
    """(turned rows, |x| + |y| of each channel's pair) of x [rows, heads, dh]."""
    x = np.asarray(x, np.float64)
    dim = 2 * sum(sections)
    w = angles(np.asarray(pos), sections, per_axis, base)[:, None]
    a = np.arange(dim // 2) if layout == "halves" else np.arange(0, dim, 2)
    b = a + (dim // 2 if layout == "halves" else 1)
    y, size = x.copy(), np.abs(x)
    y[..., a] = x[..., a] * np.cos(w) - x[..., b] * np.sin(w)
    y[..., b] = x[..., b] * np.cos(w) + x[..., a] * np.sin(w)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    return y, size


# One turned channel, relative to |x| + |y|, in halves of a step of fp32: sine and cosine are fp64 (off by
# 1.3e-10, 0.002) rounded to fp32 (1), two products (1, the second perhaps fused) and their sum (1): 3, and
# 2^-23 of that for errors of errors; angles of 2^31 units are off by 2^31 * 2^-64 turns (0.02).  The fp64
# reference's own are off by 2^-53 of the angle, which turn_tolerance adds.
TURN = 3.03 * 2.0 ** -24


def turn_tolerance(y, size, dtype, far=0):
    own = far * 2.0 ** -52                     # the reference's angle: a rounded rate, a rounded product
    t = (TURN + own) * size
    return t if dtype == "f32" else t + HALF["bf16"] * (np.abs(y) + t)


def e4m3(x):
    """Nearest e4m3 value, ties to even, of |x| <= 448 (NaN stays)."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        _, e = np.frexp(np.abs(x))
        step = np.exp2(np.maximum(e - 1, -6) - 3.0)
        return np.where(np.isnan(x), np.nan, np.round(np.where(np.isnan(x), 0, x) / step) * step)


def codes_table():
    """Values of the 256 codes."""
    c = np.arange(256)
    e, f, s = c >> 3 & 15, c & 7, np.where(c & 128, -1.0, 1.0)
    v = np.where(e == 0, f * 2.0 ** -9, (8 + f) * np.exp2(e - 10.0))
    return np.where((c & 127) == 127, np.nan, s * v)


def scale_of(most):
    """Least power of two >= 2^-126 whose 448-fold is at least `most`."""
    m, e = np.frexp(np.asarray(most, np.float64) / 448)
    s = np.where(m == 0.5, e - 1, e)
    return np.exp2(np.maximum(np.where(np.asarray(most) > 0, s, -126), -126).astype(np.float64))


class Cache:
    """Pages as values (codes times scale), token first for keys and values alike."""

    def __init__(self, pages, heads, pt, dh):
        self.pt, self.pages = pt, pages
        self.x = [np.zeros((pages, heads, pt, dh)) for _ in range(2)]
        self.scale = [np.zeros((pages, heads)) for _ in range(2)]

    def page(self, table, s, p):
        j = p // self.pt
        if j >= len(table[s]):
            return -1
        return table[s][j] if 0 <= table[s][j] < self.pages else -1

    def write(self, table, offsets, starts, k, v):
        """Rows in 64 bits (already turned), sequence by sequence."""
        for s, start in enumerate(starts):
            n, row = offsets[s + 1] - offsets[s], offsets[s]
            done = 0
            while start >= 0 and done < n:
                p = start + done
                page, slot = self.page(table, s, p), p % self.pt
                part = min(n - done, self.pt - slot)
                for which, rows in enumerate((k, v)):
                    if page < 0:
                        continue
                    new = rows[row + done:row + done + part].transpose(1, 0, 2)
                    new = np.where(np.isfinite(new), new, np.nan)
                    most = np.nan_to_num(np.abs(new)).max((1, 2))
                    size = scale_of(most)
                    if slot:
                        old = self.scale[which][page]
                        size = np.maximum(size, old)
                        held = self.x[which][page, :, :slot]
                        z = size[:, None, None]
                        self.x[which][page, :, :slot] = e4m3(held / z) * z
                    self.x[which][page, :, slot:slot + part] = \
                        e4m3(new / size[:, None, None]) * size[:, None, None]
                    self.scale[which][page] = size
                done += part

    def history(self, table, s, length):
        """Keys, values [length, heads, dh] and which of them are there."""
        heads, dh = self.x[0].shape[1], self.x[0].shape[3]
        out = [np.zeros((length, heads, dh)) for _ in range(2)]
        there = np.zeros(length, bool)
        for p in range(length):
            page = self.page(table, s, p)
            if page >= 0:
                there[p] = True
                for w in range(2):
                    out[w][p] = self.x[w][page, :, p % self.pt]
        return out[0], out[1], there


def attention(q, k, v, sees, scale):
    """q [rows, heads, dh] over k, v [keys, kv_heads, dh]; sees [rows, keys].  Returns the output, and what its
    tolerance is made of: sum p |v| and the largest sum |q| |k| scale of each row and head."""
    G = q.shape[1] // k.shape[1]
    out, mass, size = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
    for i in range(len(q)):
        j = np.flatnonzero(sees[i])
        if not len(j):
            continue
        for h in range(q.shape[1]):
            kk, vv = k[j, h // G], v[j, h // G]
            s = kk @ q[i, h] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h], mass[i, h] = p @ vv, p @ np.abs(vv)
            size[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, mass, size


def attention_tolerance(out, mass, size, dtype, dh, keys):
    """A score is a sum of dh products of exact factors (fp32 queries: their three terms leave 2^-24), each
    sum rounded or cut by at most 2^-23: off by dh 2^-23 size.  Its exponential: the argument (up to 40
    where it matters; below that a probability is 2^-57) is rounded three times with the maximum and
    factor, the exponential itself twice: (3 * 40 + 4) 2^-24.  A probability is rounded to bf16 (fp32: 2^-24),
    its products are summed in fp32 over the keys, and so are the sums that divide them, joined over
    wavefronts and splits: (2 keys + 20) 2^-23 at worst, 2 sqrt(keys) of these in any real sum but not
    here.  The score's error counts twice, in the probability and in the sum.
    A probability below 2^-126 of the largest is 0 in fp32 (a score 88 below the maximum), which takes away
    at most that times its value (below 2^6 in these tests) for each key: 64-bit results of 1e-62 come out 0."""
    e = 2 * (dh * 2.0 ** -23 * size[..., None] + 124 * 2.0 ** -24) + (2 * keys + 20) * 2.0 ** -23
    t = mass * (e + HALF[dtype]) + keys * 2.0 ** -120
    return t + HALF[dtype] * (np.abs(out) + t)

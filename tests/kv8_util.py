"""A plain model of the 8-bit KV cache, in numpy: e4m3 by its definition, pages as [16, dh] arrays of
codes, the tables of a batch, the write of a batch's rows and attention in float64."""
import numpy as np

import synth

PAGE = 16


def _e4m3_table():
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = np.nan if (c & 127) == 127 else x
        if c & 128:
            v[c] = -v[c]
    return v


VALUES = _e4m3_table()


def encode(x):
    """Codes of the nearest e4m3 values (ties to even; |x| <= 448 where finite, otherwise NaN)."""
    x = np.asarray(x, np.float64)
    pos = VALUES[:127]                                   # ascending: codes 0 .. 126
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    hi = np.clip(np.searchsorted(pos, a), 0, 126)        # first value >= a
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    code = np.where(np.isfinite(x), code, 127).astype(np.uint8)
    return np.where(np.signbit(x) & np.isfinite(x), code | 128, code)


def same_codes(a, b):
    """Equal codes, any NaN being as good as another."""
    a, b = np.asarray(a), np.asarray(b)
    return bool(np.all((a == b) | (((a & 127) == 127) & ((b & 127) == 127))))


def scale_for(amax):
    """Least power of two s with amax <= 448 s, no less than 2^-100."""
    s = 2.0 ** -100
    if amax > 448 * s:
        m, e = np.frexp(amax / 448.0)
        s = 2.0 ** (e if m > 0.5 else e - 1)
    return s


def pack(pages, kind):
    """Pages [.., 16, dh] -> their bytes in the pool's layout [.., 16 * dh]."""
    *lead, _, dh = pages.shape
    if kind == "k":
        x = pages.reshape(*lead, PAGE, dh // 16, 16)
        return np.ascontiguousarray(np.swapaxes(x, -3, -2)).reshape(*lead, PAGE * dh)
    x = pages.reshape(*lead, 4, 4, dh)
    return np.ascontiguousarray(np.swapaxes(x, -2, -1)).reshape(*lead, PAGE * dh)


def unpack(raw, kind, dh):
    *lead, _ = raw.shape
    if kind == "k":
        return np.swapaxes(raw.reshape(*lead, dh // 16, PAGE, 16), -3, -2).reshape(*lead, PAGE, dh)
    return np.swapaxes(raw.reshape(*lead, 4, dh, 4), -2, -1).reshape(*lead, PAGE, dh)


class Cache:
    """Codes [Hkv, nb, 16, dh] and scales [Hkv, nb] of both pools; everything unwritten is NaN."""

    def __init__(self, hkv, nb, dh):
        self.hkv, self.nb, self.dh = hkv, nb, dh
        self.codes = {k: np.full((hkv, nb, PAGE, dh), 0x7F, np.uint8) for k in "kv"}
        self.scale = {k: np.full((hkv, nb), np.nan, np.float32) for k in "kv"}

    def fill(self, rng, blocks, spread=3):
        """Random finite pages, of sizes 2^-spread .. 2^spread."""
        for k in "kv":
            shape = (self.hkv, len(blocks), PAGE, self.dh)
            x = rng.standard_normal(shape) * 60
            self.codes[k][:, blocks] = encode(np.clip(x, -448, 448))
            self.scale[k][:, blocks] = 2.0 ** (rng.integers(-spread, spread + 1, shape[:2]) - 6)

    def poison(self, block, from_token):
        """NaN in a page's places from from_token on."""
        for k in "kv":
            self.codes[k][:, block, from_token:] = 0x7F

    def values(self, kind, h, blocks):
        return (VALUES[self.codes[kind][h, blocks]] *
                self.scale[kind][h, blocks].astype(np.float64)[:, None, None]).reshape(-1, self.dh)

    def write_run(self, kind, block, first, x):
        """x float32 [n, Hkv, dh] to places first .. of one page."""
        with np.errstate(invalid="ignore"):                # (casts of NaN)
            x = x.astype(np.float64)
        for h in range(self.hkv):
            a = np.abs(x[:, h])
            s = scale_for(np.max(a[np.isfinite(a)], initial=0.0))
            page = self.codes[kind][h, block]
            if first:
                old = float(self.scale[kind][h, block])
                s = max(s, old)
                if s != old:
                    page[:first] = encode(VALUES[page[:first]] * (old / s))
            page[first:first + len(x)] = encode(x[:, h] / s)
            self.scale[kind][h, block] = s

    def write(self, k, v, slot):
        """Rows k, v float32 [T, Hkv, dh] to their slots (None or negative: skipped), run by run."""
        t = 0
        while t < len(slot):
            n = 1
            if slot[t] >= 0:
                while t + n < len(slot) and slot[t + n] == slot[t] + n and slot[t + n] % PAGE:
                    n += 1
                for kind, x in (("k", k), ("v", v)):
                    self.write_run(kind, slot[t] // PAGE, slot[t] % PAGE, x[t:t + n])
            t += n


def rope_table(max_pos, dh, base=10000.0):
    """float32 [max_pos, dh/2, 2]: cos and sin of p * base^(-2i/dh)."""
    a = np.arange(max_pos)[:, None] * base ** (-2.0 * np.arange(dh // 2) / dh)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def rotate(x, cs):
    """Rotate-half RoPE of x float32 [T, H, dh] by cs [T, dh/2, 2], each operation rounded to float32."""
    half = x.shape[-1] // 2
    a, b, c, s = x[..., :half], x[..., half:], cs[:, None, :, 0], cs[:, None, :, 1]
    with np.errstate(all="ignore"):
        return np.concatenate([a * c - b * s, b * c + a * s], -1)


def slot_map(start, n_new, free, bt, T):
    """The tables of a batch: (bt, row0, pos, slot, ctx, status), one sequence after the other."""
    S, stride = bt.shape
    bt, free = bt.copy(), list(free)
    ctx, row0 = np.maximum(start, 0), np.zeros(S + 1, np.int64)
    pos, slot = np.zeros(T, np.int64), np.full(T, -1)
    need = [-(-(a + n) // PAGE) - -(-a // PAGE) for a, n in zip(start, n_new)]
    if (np.any(start < 0) or np.any(n_new < 0) or sum(need) > len(free) or n_new.sum() > T or
            any(-(-(a + n) // PAGE) > stride for a, n in zip(start, n_new))):
        return bt, row0, pos, slot, ctx, np.array([-1, 0])
    r = taken = 0
    for s in range(S):
        row0[s] = r
        have = -(-start[s] // PAGE)
        for j in range(need[s]):
            bt[s, have + j] = free[taken]
            taken += 1
        for i in range(n_new[s]):
            p = start[s] + i
            pos[r], slot[r] = p, bt[s, p // PAGE] * PAGE + p % PAGE
            r += 1
        ctx[s] = start[s] + n_new[s]
    row0[S] = r
    return bt, row0, pos, slot, ctx, np.array([taken, r])


def attend(q, cache, blocks, n, hq, first=None):
    """softmax(q k / sqrt(dh)) v over the first n places of `blocks`: q float64 [m, Hq, dh]; query i sees the
    positions up to first + i (None: all).  Places of an entry that is no page have no weight.  Returns the
    outputs, and the error that assert_attention allows apart from the output's own rounding."""
    m, G = len(q), hq // cache.hkv
    out, size = np.zeros_like(q), np.zeros_like(q)
    if n == 0:
        return out, size
    at = np.asarray(blocks[:-(-n // PAGE)])
    ok = (at >= 0) & (at < cache.nb)
    there = np.repeat(ok, PAGE)[:n]
    if not there.any():
        return out, size
    at = np.where(ok, at, at[ok][0])
    for h in range(cache.hkv):
        k, v = cache.values("k", h, at)[:n], cache.values("v", h, at)[:n]
        x = q[:, h * G:(h + 1) * G] @ np.where(there[:, None], k, 0).T / np.sqrt(cache.dh)
        seen = np.broadcast_to(there, (m, n)).copy()
        if first is not None:
            seen &= np.arange(n) <= (first + np.arange(m))[:, None]
        x = np.where(seen[:, None], x, -np.inf)
        w = np.exp(x - x.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        v = np.where(there[:, None], v, 0)
        out[:, h * G:(h + 1) * G] = w @ v
        # Weights in fp16: off by 2^-11 of each, or, under 2^-14, by 2^-25, where the largest weight is 2^7 or more; so
        # the second kind by 2^-32 p_j of the normalised ones, p_j the largest: 2^-32 p_j sum |v| in all.
        # V in fp16, in units of the largest page scale 2^E: exact for scales from 2^-15 of it on (codes are
        # multiples of 2^-9, fp16's subnormals of 2^-24), otherwise off by 2^-25 2^E, which the weights average.
        floor = 2.0 ** -32 * w.max(-1, keepdims=True) * (seen[:, None].astype(np.float64) @ np.abs(v))
        scales = cache.scale["v"][h, at].astype(np.float64)
        if scales.min() < 2.0 ** -15 * scales.max():
            floor += 2.0 ** -25 * scales.max()
        size[:, h * G:(h + 1) * G] = (2.0 ** -11 + 2.0 ** -11) * (w @ np.abs(v)) + floor
    return out, size


def assert_attention(got, ref, size, what):
    """The kernels take q, K and V exactly, sum in float32, and round twice: the weights of the product with V to fp16
    (see attend) and the output to bf16 (2^-8).  The float32 scores (sums of dh products, times a constant,
    exponentials) are off by under 2^-12 for the scores of these tests (|x| < 64: 64 * 2^-24 * a few
    roundings, and 128 * 2^-24 of the products' sum), and the float32 sums by less: 2^-11 of the weights in all."""
    assert np.all(np.isfinite(got)), what
    over = np.abs(got - ref) - (2.0 ** -8 * np.abs(ref) + size + 1e-30)
    assert over.max(initial=-1) <= 0, f"{what}: over by {over.max():.3e} at {np.unravel_index(over.argmax(), over.shape)}"


def f32_of(bits):
    return synth.bf16_bits_to_f32(bits).reshape(bits.shape)

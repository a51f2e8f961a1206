"""float64 oracle of the paged 8-bit cache (one scale per block of 128 tokens and KV head), written from the definitions in
include/bitdecode.h: appending with the position rotation, and attention of a step's queries with a cap, a bias by distance, a
window and a prefix.  Plain numpy; half types are numpy float16, or float32 holding bf16 values."""
import numpy as np

BLOCK = 128
MOST = {"int8": 127.0, "e4m3": 448.0}


def round_half(x64, dtype):
    """float64 rounded to fp32 and then to the half type (as float64 values)."""
    with np.errstate(over="ignore"):
        x32 = np.asarray(x64, np.float64).astype(np.float32)
        if dtype == "fp16":
            return x32.astype(np.float16).astype(np.float64)
    u = x32.view(np.uint32)
    return ((u + np.uint32(0x7FFF) + ((u >> np.uint32(16)) & np.uint32(1))) & np.uint32(0xFFFF0000)).view(np.float32).astype(np.float64)


def round_e4m3(y):
    """Nearest e4m3 number (ties to even), saturating at 448; y float64."""
    mag = np.minimum(np.abs(y), 448.0)
    exp = np.floor(np.log2(np.maximum(mag, 2.0 ** -6)))
    step = np.exp2(exp - 3)
    return np.copysign(np.minimum(np.rint(mag / step) * step, 448.0), y)


def rotate(x, cos, sin, interleaved, dtype):
    """x [rows][heads][D]; cos, sin [rows][pairs] (fp32 values)."""
    x = np.asarray(x, np.float64).copy()
    r = 2 * cos.shape[1]
    first = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., first[0]].copy(), x[..., first[1]].copy()
    c, s = cos[:, None].astype(np.float64), sin[:, None].astype(np.float64)
    x[..., first[0]] = round_half(a * c - b * s, dtype)
    x[..., first[1]] = round_half(a * s + b * c, dtype)
    return x


def quantize(x, code):
    """A block's values -> (codes as the numbers they are, fp32 scale)."""
    scale = np.float32(np.abs(x).max()) / np.float32(MOST[code])
    if not scale > 0:
        return np.zeros_like(x), np.float32(0)
    y = (x / np.float64(scale)).astype(np.float32).astype(np.float64)
    y = np.rint(y) if code == "int8" else round_e4m3(y)
    return np.clip(y, -MOST[code], MOST[code]), scale


class Cache:
    """One cache: pages and residuals as float64 values (codes as numbers), lengths as ints; NaN where nothing was written."""

    def __init__(self, batch, heads, dim, code, dtype, pages, table):
        self.code, self.dtype, self.table, self.pages = code, dtype, np.asarray(table), pages
        self.k_codes, self.v_codes = (np.full((pages, heads, BLOCK, dim), np.nan) for _ in range(2))   # both token by token
        self.k_scales, self.v_scales = (np.full((pages, heads), np.nan) for _ in range(2))
        self.k_res, self.v_res = (np.full((batch, heads, BLOCK, dim), np.nan) for _ in range(2))
        self.lens = [0] * batch

    def page(self, b, block):
        p = int(self.table[b, block]) if block < self.table.shape[1] else -1
        return p if 0 <= p < self.pages else None

    def append(self, b, k, v):
        """k (rotated), v [rows][heads][D] behind the tokens of sequence b; the length stays (as the library's does)."""
        n, length = k.shape[0], self.lens[b]
        for x, codes, scales, res in ((k, self.k_codes, self.k_scales, self.k_res), (v, self.v_codes, self.v_scales, self.v_res)):
            kept = length % BLOCK
            whole = np.concatenate([res[b, :, :kept], np.asarray(x, np.float64).transpose(1, 0, 2)], 1)
            blocks = whole.shape[1] // BLOCK
            for i in range(blocks):
                p = self.page(b, length // BLOCK + i)
                if p is not None:
                    for h in range(whole.shape[0]):
                        codes[p, h], scales[p, h] = quantize(whole[h, i * BLOCK:(i + 1) * BLOCK], self.code)
            left = whole.shape[1] % BLOCK
            start = 0 if blocks else kept
            res[b, :, start:left] = whole[:, blocks * BLOCK + start:]
        return n

    def values(self, b, length):
        """K, V [heads][length][D] and which of the tokens are there."""
        there = np.ones(length, bool)
        out = []
        for codes, scales, res in ((self.k_codes, self.k_scales, self.k_res), (self.v_codes, self.v_scales, self.v_res)):
            x = np.zeros((codes.shape[1], length, codes.shape[3]))
            for i in range(length // BLOCK):
                p = self.page(b, i)
                at = slice(i * BLOCK, (i + 1) * BLOCK)
                if p is None:
                    there[at] = False
                else:
                    x[:, at] = codes[p] * scales[p][:, None, None]
            x[:, length // BLOCK * BLOCK:] = res[b, :, :length % BLOCK]
            out.append(x)
        return out[0], out[1], there


def attention(cache, b, q, before, scale, cap=0.0, slopes=None, window=0, prefix=0):
    """q [rows][query heads][D], the tokens before .. before + rows - 1 of sequence b.  Returns the outputs, and for the bars of a
    comparison sum w |v| / sum w, and the largest magnitudes that scores are made of (products, then whole)."""
    rows, hq, dim = q.shape
    length = before + rows
    k, v, there = cache.values(b, length)
    g = hq // k.shape[0]
    p, j = np.arange(before, length)[:, None], np.arange(length)[None]
    seen = (j < prefix) | ((j <= p) & ((p - j < window) if window else True))
    seen = seen & there[None]
    out, spread = np.zeros((rows, hq, dim)), np.zeros((rows, hq, dim))
    products = whole = 0.0
    for h in range(hq):
        qh = np.asarray(q[:, h], np.float64)
        s = scale * (qh @ k[h // g].T)
        part = abs(scale) * (np.abs(qh) @ np.abs(k[h // g]).T)
        if cap:
            s = cap * np.tanh(s / cap)
        if slopes is not None:
            s = s - float(slopes[h]) * np.abs(p - j)
            whole = max(whole, abs(float(slopes[h])) * length)
        products, whole = max(products, part[seen].max(initial=0.0)), max(whole, np.abs(s[seen]).max(initial=0.0), cap)
        s = np.where(seen, s, -np.inf)
        top = s.max(1, keepdims=True)
        w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
        norm = w.sum(1, keepdims=True)
        norm[norm == 0] = 1.0
        out[:, h] = w @ v[h // g] / norm
        spread[:, h] = w @ np.abs(v[h // g]) / norm
    return out, spread, products, whole


def bar(out, spread, products, whole, dim, length, dtype):
    """How far the library's outputs may be from `out`.  The result's rounding is half a step of the half type.  Weights go to
    the product with 11 bits (half a step is 2^-11 of one).  A score's products are summed in fp32 in any order (dim + 8 roundings of at most their sum's
    size), the operations on the score itself are fewer than eight of its size; a weight is off by what its score is, twice that where the sum of weights
    is off as well.  Sums over the tokens in fp32: 128 terms and one for each of the blocks, in numerator and denominator.  2^-24 of the
    largest: weights below fp16's subnormals."""
    half = 2.0 ** -11 if dtype == "fp16" else 2.0 ** -8
    score = (dim + 8) * 2.0 ** -24 * products + 8 * 2.0 ** -24 * whole
    sums = 2 * (128 + length / BLOCK) * 2.0 ** -24
    return half * np.abs(out) + spread * (2.0 ** -11 + 2 * np.expm1(score) + sums) + 2.0 ** -24 * np.abs(spread).max(initial=0.0)

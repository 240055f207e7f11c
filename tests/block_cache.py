"""Plain implementations, in 64 bits on the CPU, of what the FP8_BLOCK format, the rotary positions and the block tables are
defined to do, and a pool whose blocks a test fills byte by byte.  Shares no code with the library."""
import math

import numpy as np

LOW, HIGH = -15, 7  # exponents of a block's scale


# ------------------------------------------------------------------------------------------------ E4M3 and its scales
def e4m3_value(codes):
    """Values of E4M3 codes (NaN for 0x7F and 0xFF)."""
    c = np.asarray(codes, np.int64)
    exp, man = c >> 3 & 15, c & 7
    mag = np.where(exp > 0, (1 + man / 8.0) * 2.0 ** (exp - 7), man * 2.0 ** -9)
    mag = np.where((c & 0x7F) == 0x7F, np.nan, mag)
    return np.where(c & 0x80, -mag, mag)


def e4m3_round(x):
    """Nearest E4M3 value, ties to even, saturating at 448."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    _, e = np.frexp(a)
    step = 2.0 ** (np.maximum(e - 1, -6) - 3.0)
    return np.copysign(np.rint(a / step) * step, x)


def scale_exponent(amax):
    """Least e in LOW .. HIGH with amax <= 448 * 2^e."""
    m, e = np.frexp(np.asarray(amax, np.float64))
    return np.where(np.asarray(amax) > 0, np.clip(np.where(m <= 0.875, e - 9, e - 8), LOW, HIGH), LOW)


class BlockCache:
    """K (or V) rows of one layer: value / scale of every slot, and the scales' exponents."""

    def __init__(self, n_blocks, heads, tokens, d):
        self.codes = np.zeros((n_blocks, heads, tokens, d))
        self.e = np.zeros((n_blocks, heads), np.int64)
        self.used = np.zeros(n_blocks, np.int64)  # slots that a test may look at

    def append(self, x, blk, slot):
        """x [n][heads][d]: the rows of one call, whose blocks and slots are given."""
        for b in np.unique(blk):
            of = np.flatnonzero(blk == b)
            low = slot[of].min()
            for h in range(x.shape[1]):
                e_old = self.e[b, h] if low else LOW
                e = max(e_old, int(scale_exponent(np.abs(x[of, h]).max())))
                if low:  # what is stored follows the scale
                    self.codes[b, h] = e4m3_round(self.codes[b, h] * 2.0 ** (e_old - e))
                self.e[b, h] = e
                self.codes[b, h, slot[of]] = e4m3_round(x[of, h] * 2.0 ** -e)
            self.used[b] = max(self.used[b] if low else 0, slot[of].max() + 1)


# ------------------------------------------------------------------------------------------------------------- layout
def layout(heads, d, tokens, layers):
    """Offsets of an FP8_BLOCK block."""
    tile = -(-tokens * d // 16) * 16
    layer = -(-heads * (2 * tile + 8) // 256) * 256
    return dict(tile=tile, chunk=2 * tile, scales=heads * 2 * tile, layer=layer, block=layers * layer)


def views(mem, heads, d, tokens, layers, layer):
    """K codes, V codes [block][head][token][d] (bytes) and scales [block][head][K, V] of a pool's memory (a torch uint8 tensor)."""
    import torch
    p = layout(heads, d, tokens, layers)
    n, at = mem.numel() // p["block"], layer * p["layer"]
    k, v = (mem.as_strided((n, heads, tokens, d), (p["block"], p["chunk"], d, 1), at + w * p["tile"]) for w in (0, 1))
    return k, v, mem.view(torch.float32).as_strided((n, heads, 2), (p["block"] // 4, 2, 1), (at + p["scales"]) // 4)


def fill_random(mem, shape, layer, rng, spread=3):
    """Random codes (never NaN) and scales; returns the values K, V [block][head][token][d] in 64 bits."""
    import torch
    heads, d, tokens, layers = shape
    k, v, scales = views(mem, heads, d, tokens, layers, layer)
    values = []
    for which, rows in enumerate((k, v)):
        x = rng.standard_normal(rows.shape) * 100
        x = e4m3_round(x)
        codes = torch.from_numpy(x.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8)
        e = rng.integers(-7 - spread, -7 + spread + 1, rows.shape[:2])
        rows.copy_(codes.to(mem.device))
        scales[:, :, which] = torch.from_numpy((2.0 ** e).astype(np.float32)).to(mem.device)
        values.append(x * 2.0 ** e[:, :, None, None])
    return values


# ---------------------------------------------------------------------------------------------------------- attention
def attention(q, k, v, scale):
    """q [G][d], k, v [n][d] -> out [G][d], lse [G], sum p |v| [G][d]."""
    s = q @ k.T * scale
    top = s.max(1, keepdims=True)
    p = np.exp(s - top)
    l = p.sum(1, keepdims=True)
    p /= l
    return p @ v, (top + np.log(l))[:, 0], p @ np.abs(v)


def out_tolerance(out, sum_abs, n, v_max):
    """fp16 weights (half a step, 2^-11 of each; below 2^-14 2^-25 of the largest) and fp16 results (2^-11, 2^-25 at least), fp32
    logits (5e-5 of a weight)."""
    return 2.0 ** -11 * (sum_abs + np.abs(out)) * 1.02 + 5e-5 * sum_abs + n * 2.0 ** -25 * v_max + 2.0 ** -25


# ------------------------------------------------------------------------------------------------------ rotary positions
def frequencies(r, base, scaling, factor=1.0, low=0.0, high=0.0, original=0):
    i = np.arange(r // 2, dtype=np.float64)
    if scaling == "base":
        base = base * factor ** (r / (r - 2))
    f = base ** (-2 * i / r)
    stretch = np.zeros(r // 2)
    if scaling == "linear":
        stretch[:] = 1
    if scaling == "wavelength":
        stretch = 1 - np.clip((original * f / (2 * math.pi) - low) / (high - low), 0, 1)
    if scaling == "dimension":
        at = [r * math.log(original / (2 * math.pi * n)) / (2 * math.log(base)) for n in (high, low)]
        first, last = max(math.floor(at[0]), 0), min(math.ceil(at[1]), r - 1)
        stretch = np.clip((i - first) / max(last - first, 0.001), 0, 1)
    return f * (1 - stretch) + f / factor * stretch


def rotate(x, pos, f, halves, amplitude=1.0, inverse=False):
    """x [n][heads][d], pos [n] -> (rotated, sum of the magnitudes that make an element)."""
    x = np.asarray(x, np.float64)
    r = 2 * len(f)
    angle = np.asarray(pos, np.float64)[:, None] * f * (-1 if inverse else 1)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    a, b = (slice(0, r // 2), slice(r // 2, r)) if halves else (slice(0, r, 2), slice(1, r, 2))
    y, m = x.copy(), np.abs(x)
    y[..., a], y[..., b] = amplitude * (x[..., a] * c - x[..., b] * s), amplitude * (x[..., b] * c + x[..., a] * s)
    m[..., a] = m[..., b] = amplitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, m


# --------------------------------------------------------------------------------------------------------------- tables
def tables(held, new, ids, table, t, n_tokens, n_blocks, held_given=True):
    """One request after the other; returns a dict of what fs_batch_tables writes."""
    table = table.copy()
    cap = min(table.shape[1] * t, 2 ** 31 - 1)
    flags, taken = 0, 0
    seq, pos, slots, lens, offsets = [], [], [], [], [0]
    for b in range(len(new)):
        h0, n0 = (int(held[b]) if held_given else 0), int(new[b])
        h = min(max(h0, 0), cap)
        n = min(max(n0, 0), cap - h)
        flags |= h != h0 or n != n0
        if len(seq) + n > n_tokens:
            flags |= 2
            n = n_tokens - len(seq)
        for j in range(-(-h // t), -(-(h + n) // t)):
            if taken >= len(ids):
                flags |= 2
            table[b, j] = ids[taken] if taken < len(ids) else -1
            taken += 1
        for p in range(h, h + n):
            blk = int(table[b, p // t])
            seq.append(b)
            pos.append(p)
            slots.append(blk * t + p % t if 0 <= blk < n_blocks else -1)
        lens.append(h + n)
        offsets.append(len(seq))
    pad = [-1] * (n_tokens - len(seq))
    return dict(table=table, seq_lens=np.array(lens), q_offsets=np.array(offsets), seq_idx=np.array(seq + pad), pos=np.array(pos + pad),
                slots=np.array(slots + pad, np.int64), status=flags)

"""Plain references, in 64 bits, of rotary positions and of the 8-bit cache; and what the GPU tests of them make their inputs with."""
from __future__ import annotations

import numpy as np
import torch

BF16, FP32 = 0, 1
HALF_STEP = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}     # of a rounding, relative to the value


def torch_dtype(dtype):
    return torch.bfloat16 if dtype == BF16 else torch.float32


def f64(t):
    return t.detach().cpu().double().numpy()


# --- rotary positions -------------------------------------------------------------------------------------------
def rope_frequencies(d, base, scaling="none", factor=1.0, alpha=1.0, beta=32.0, original_len=0):
    out = []
    for j in range(d // 2):
        b = base * factor ** (d / (d - 2)) if scaling == "base" else base
        f = b ** (-2.0 * j / d)
        if scaling == "linear":
            f = f / factor
        if scaling == "parts":
            turns = original_len * f / (2 * np.pi)
            keep = min(1.0, max(0.0, (turns - alpha) / (beta - alpha)))
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out)


def rope(x, positions, freq, pairs, magnitude, backward):
    """x [..., rows, heads, hs] in float64, positions [rows]; the angle in extended precision.  Returns the result and, per element, the
    sum of the magnitudes of what is added up for it."""
    d = 2 * len(freq)
    angle = np.asarray(positions, dtype=np.longdouble)[:, None] * np.asarray(freq, dtype=np.longdouble)
    if backward:
        angle = -angle
    c, s = np.cos(angle).astype(np.float64)[:, None] * magnitude, np.sin(angle).astype(np.float64)[:, None] * magnitude
    y, size = x.copy(), np.abs(x)
    at = (slice(0, d, 2), slice(1, d, 2)) if pairs else (slice(0, d // 2), slice(d // 2, d))
    a, b = x[..., at[0]], x[..., at[1]]
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    size[..., at[0]] = size[..., at[1]] = (np.abs(a) + np.abs(b)) * abs(magnitude)
    return y, size


def rope_tolerance(y, size, dtype, positions, freq):
    """One rounding of the result; and in 32 bits: half a step each of the sine (and cosine), its multiple by the magnitude, the
    product and the sum, one more for what the polynomial's own steps and its argument are off by, so 5 * 2^-24 < 2^-21 of the
    addends; and the angle's two roundings in 64 bits (the frequency in turns, the product), in radians."""
    far = np.max(np.abs(np.asarray(positions, dtype=np.float64))) * np.max(np.abs(freq)) if len(freq) else 0.0
    return HALF_STEP[dtype] * np.abs(y) + (2.0 ** -21 + far * 2.0 ** -52) * size + 1e-40


# --- e4m3 -------------------------------------------------------------------------------------------------------
def e4m3_values():
    """What each of the 256 codes stands for: sign, 4 exponent bits (bias 7), 3 of mantissa; 0x7f and 0xff are NaN."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where(code & 0x7f == 0x7f, np.nan, v)
    return np.where(code & 0x80, -v, v)


VALUES = e4m3_values()


def e4m3_codes(x):
    """The nearest codes of values within +-448, ties to even; NaN gives 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    grid = VALUES[:0x7f]                                   # 0 .. 448, ascending, even codes at even places
    a = np.minimum(np.abs(x), 448.0)
    hi = np.searchsorted(grid, a).clip(0, 0x7e)
    lo = (hi - 1).clip(0)
    dl, dh = a - grid[lo], grid[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(x), 0x7f, code | np.where(np.signbit(x), 0x80, 0))
    return code.astype(np.uint8)


def same_codes(a, b):
    """Equal, any NaN being like any other."""
    a, b = np.asarray(a), np.asarray(b)
    return bool(np.all((a == b) | ((a & 0x7f == 0x7f) & (b & 0x7f == 0x7f))))


def exponent(most):
    """Smallest e with most <= 448 * 2^e, within [-117, 88]."""
    if most == 0:
        return -117
    e = int(np.ceil(np.log2(most / 448.0)))
    while most <= 448.0 * 2.0 ** (e - 1):
        e -= 1
    while most > 448.0 * 2.0 ** e:
        e += 1
    return max(-117, min(88, e))


def v_rows(v):
    """V codes [pages][hk][page/16][hs][16] as [pages][hk][page][hs]."""
    p, hk, t, hs, _ = v.shape
    return np.ascontiguousarray(np.swapaxes(v, 3, 4)).reshape(p, hk, t * 16, hs)


def v_tiles(rows):
    p, hk, page, hs = rows.shape
    return np.ascontiguousarray(np.swapaxes(rows.reshape(p, hk, page // 16, 16, hs), 3, 4))


def append(codes, scale, x, slots, page):
    """codes [pages][hk][page][hs] and scale [pages][hk] (uint8 arrays, changed in place): rows x [rows][hk][hs] to their slots."""
    pages, hk = scale.shape
    t = 0
    while t < len(slots):
        if not 0 <= slots[t] < pages * page:
            t += 1
            continue
        n = 1
        while t + n < len(slots) and slots[t + n] == slots[t] + n and slots[t + n] // page == slots[t] // page:
            n += 1
        number, old = slots[t] // page, slots[t] % page
        for h in range(hk):
            y = x[t:t + n, h]
            finite = np.abs(y[np.isfinite(y)])
            e = exponent(float(finite.max()) if finite.size else 0.0)
            if old:
                was = int(scale[number, h]) - 127
                e = max(e, was)
                if e > was:
                    codes[number, h, :old] = e4m3_codes(VALUES[codes[number, h, :old]] * 2.0 ** (was - e))
            codes[number, h, old:old + n] = e4m3_codes(np.where(np.isfinite(y), y, np.nan) * 2.0 ** -e)
            scale[number, h] = e + 127
        t += n


def extend(cu, before, total, table, page, pages, free):
    """(table, len_after, slots, positions, taken) after usp_cache_extend."""
    table, n, max_pages = [list(r) for r in table], len(before), len(table[0]) if len(table) else 1
    slots, positions, after, used, asked = [-1] * total, [0] * total, list(before), 0, 0
    for i in range(n):
        m, h = max(0, cu[i + 1] - cu[i]), before[i]
        fits = h >= 0 and h + m <= max_pages * page
        need = -(-(h + m) // page) - -(-h // page) if fits else 0
        served = fits and (need == 0 or asked + need <= len(free))
        if served:
            for j in range(need):
                table[i][-(-h // page) + j] = free[asked + j]
            if need:
                used = asked + need
            after[i] = h + m
        for t in range(cu[i], cu[i] + m):
            pos = h + t - cu[i]
            positions[t] = pos
            if served:
                number = table[i][pos // page]
                slots[t] = number * page + pos % page if 0 <= number < pages else -1
        asked += need
    return table, after, slots, positions, [used, asked]


# --- attention over the cache -----------------------------------------------------------------------------------
def attention(q, k, v, cu, lens, table, page, pages, causal, scale=None, total=None):
    """q [total][hq][hs] float64; k, v: values [pages][hk][page][hs].  Returns o, lse [hq][total], what A = sum P |v| / sum P is
    per element of o, and which rows belong to a request.  Softmax in 64 bits; rows that see nothing: 0 and -inf."""
    total, hq, hs = q.shape
    hk = k.shape[1]
    group = hq // hk
    scale = hs ** -0.5 if scale is None else scale
    o, size, lse, owned = np.zeros(q.shape), np.zeros(q.shape), np.full((hq, total), -np.inf), np.zeros(total, bool)
    for i in range(len(lens)):
        nq = cu[i + 1] - cu[i]
        if nq <= 0:
            continue
        owned[cu[i]:cu[i + 1]] = True
        length = max(0, min(lens[i], table.shape[1] * page))
        pos = np.arange(length)
        number = table[i][pos // page]
        held = (number >= 0) & (number < pages)
        pos, number = pos[held], number[held]
        if not len(pos):
            continue
        kk, vv = k[number, :, pos % page], v[number, :, pos % page]           # [keys][hk][hs]
        last = length - nq + np.arange(nq) if causal else np.full(nq, length - 1)
        sees = pos[None, :] <= last[:, None]                                  # [nq][keys]
        for h in range(hq):
            with np.errstate(all="ignore"):
                s = q[cu[i]:cu[i + 1], h] @ kk[:, h // group].T * scale
                s = np.where(sees, s, -np.inf)
                top = s.max(1)
                top = np.where(np.isneginf(top), 0.0, top)
                p = np.where(sees, np.exp(s - top[:, None]), 0.0)
                tot = p.sum(1)
                w = np.divide(p, tot[:, None], out=np.zeros_like(p), where=(tot[:, None] != 0))
                for a, out in ((vv[:, h // group], o), (np.abs(vv[:, h // group]), size)):
                    if np.isnan(a).any():          # an unseen key's value is not part of the sum, whatever it is
                        out[cu[i]:cu[i + 1], h] = np.stack([w[r, sees[r]] @ a[sees[r]] for r in range(nq)])
                    else:
                        out[cu[i]:cu[i + 1], h] = w @ a
                lse[h, cu[i]:cu[i + 1]] = np.where(tot == 0, -np.inf, np.log(tot) + top)
    return o, lse, size, owned


def check_attention(o, lse, ref, o_dtype, score_size=16.0):
    """Tolerances: P is rounded to bf16 once (half a step 2^-8 of each P, so of A = sum P |v|), the result once to its type; the
    scores are sums of up to 128 products in 32 bits, off by at most 128 * 2^-24 of the sum of their magnitudes (`score_size`
    with the scale: at most 16 for entries about N(0, 1)), and so is the logarithm of their sum; another 2^-20 for exponentials
    and sums."""
    ro, rl, size, owned = ref
    in_score = 128 * 2.0 ** -24 * score_size + 2.0 ** -20
    tol = (2.0 ** -8 + 2 * in_score) * size + HALF_STEP[o_dtype] * np.abs(ro) + 1e-30
    nan = np.isnan(ro)
    assert np.array_equal(nan[owned], np.isnan(o)[owned])
    far = np.abs(o - ro)
    bad = owned[:, None, None] & ~nan & ~(far <= tol)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, at {np.argwhere(bad)[0]}: {o[bad][0]} for {ro[bad][0]} +- {tol[bad][0]}"
    rl, lse = rl[:, owned], lse[:, owned]
    assert np.array_equal(np.isneginf(rl), np.isneginf(lse))
    assert np.array_equal(np.isnan(rl), np.isnan(lse))
    fin = np.isfinite(rl)
    assert np.all(np.abs(lse[fin] - rl[fin]) <= in_score + 2.0 ** -21 * np.abs(rl[fin])), np.abs(lse[fin] - rl[fin]).max()


class Cache:
    """A cache on the device whose codes and exponents are random; `k`, `v`: the values that it holds, [pages][hk][page][hs]."""

    def __init__(self, usp, rng, pages, page, hk, hs):
        self.usp, self.pages, self.page, self.hk, self.hs = usp, pages, page, hk, hs
        self.k_codes = e4m3_codes(rng.standard_normal((pages, hk, page, hs)) * 60)
        rows = e4m3_codes(rng.standard_normal((pages, hk, page, hs)) * 60)
        self.v_codes = v_tiles(rows)
        self.k_scale = rng.integers(119, 123, (pages, hk)).astype(np.uint8)
        self.v_scale = rng.integers(119, 123, (pages, hk)).astype(np.uint8)
        self.to_device()

    def to_device(self):
        self.dev = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (self.k_codes, self.v_codes, self.k_scale, self.v_scale)]
        self.c = self.usp.cache(*self.dev, self.pages, self.page, self.hk, self.hs)

    def values(self):
        k = VALUES[self.k_codes] * 2.0 ** (self.k_scale.astype(float) - 127)[:, :, None, None]
        v = VALUES[v_rows(self.v_codes)] * 2.0 ** (self.v_scale.astype(float) - 127)[:, :, None, None]
        return k, v


def ragged_table(rng, lens, page, pages, max_pages):
    """A block table with distinct random pages for the tokens of each request; what stands behind them is no page."""
    order = rng.permutation(pages)
    table, at = np.full((len(lens), max_pages), 0x7fffff01, dtype=np.int32), 0
    for i, n in enumerate(lens):
        need = -(-n // page)
        table[i, :need] = order[at:at + need]
        at += need
    return table


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")

"""The optimiser step in float64 from its definition (include/gs_optim.h),
in numpy, for the tests: values, what float32 arithmetic may leave between
them and the kernels', and the rounding of 8-bit moments and bfloat16
parameters with the random bits of the definition.

A rounding with given random numbers is monotone, so the kernel's value has
to lie between the roundings of the ends of what float32 may have left: the
definition's own value but for the few elements whose comparison (share of
the way + random number against 1) float32's error could turn."""
import numpy as np

U = 2.0 ** -24       # unit roundoff of float32
TINY = 2.0 ** -149   # smallest float32 denormal
M32 = 0xFFFFFFFF


def mix(x):
    x = np.asarray(x, dtype=np.uint64)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x7FEB352D)) & np.uint64(M32)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x846CA68B)) & np.uint64(M32)
    return x ^ (x >> np.uint64(16))


def random_bits(index, place, step, seed):
    """The 32 random bits of elements `index` (an array) of a tensor."""
    index = np.asarray(index, dtype=np.uint64)
    key = mix((place + 0x9E3779B9) & M32)
    for w in (step & M32, step >> 32, seed & M32, seed >> 32):
        key = mix(key ^ np.uint64(w))
    key = mix(key ^ (index >> np.uint64(32)))
    return mix((index & np.uint64(M32)) ^ key)


def e4m3(code):
    """The number of an E4M3 code (sign, 4 bits of exponent, bias 7, 3 of
    mantissa; 0x7F is NaN)."""
    code = np.asarray(code, dtype=np.int64)
    e, f = (code >> 3) & 15, code & 7
    x = np.where(e == 0, f * 2.0 ** -9, (8 + f) * np.exp2(e - 10.0))
    x = np.where((code & 0x7F) == 0x7F, np.nan, x)
    return np.where(code & 0x80, -x, x)


def scale_value(byte):
    return np.exp2(np.asarray(byte, dtype=np.float64) - 127.0)


def values(codes, scales):
    """The numbers of MXFP8 codes [n] with scales [(n + 31) // 32]."""
    return e4m3(codes) * np.repeat(scale_value(scales), 32)[:len(codes)]


def magnitude_code(y):
    """E4M3 code of a number >= 0 of the grid."""
    y = np.asarray(y, dtype=np.float64)
    e = np.maximum(np.frexp(np.where(y > 0, y, 1.0))[1] - 1, -6)
    q = np.round(y / np.exp2(e - 3.0)).astype(np.int64)  # 8..15, or 0..7 for the lowest exponent
    return np.where(y > 0, (e + 6) * 8 + q, 0)


def blocks(x, fill=0.0):
    n = len(x)
    out = np.full(((n + 31) // 32) * 32, fill, dtype=np.float64)
    out[:n] = x
    return out.reshape(-1, 32)


def exponents(top):
    """Smallest e >= -126 with top <= 448 2^e."""
    f, e = np.frexp(np.where(top > 0, top, 1.0) / 448.0)
    e = np.where(f == 0.5, e - 1, e)
    return np.maximum(np.where(top > 0, e, -126), -126)


def to_grid(y, rnd, lowest, bits):
    """Numbers >= 0 to a grid of `bits` bits below the leading one, spaced as
    at 2^lowest below that: up where share + rnd >= 1, to the nearest (ties
    to even) when rnd is None. Monotone in y."""
    place = np.exp2(np.maximum(np.frexp(np.where(y > 0, y, 1.0))[1] - 1, lowest) - float(bits))
    lower = np.floor(y / place)
    share = y / place - lower
    up = (share > 0.5) | ((share == 0.5) & (lower % 2 == 1)) if rnd is None else share + rnd >= 1.0
    return (lower + up) * place


def check_mxfp8(codes, scales, x, dx, rnd=None, positive=False, sharp=True, label=""):
    """Codes and scales of a tensor against x (float64), known up to dx:
    rounded with the numbers rnd in (0, 1), or to the nearest when None.
    positive: a positive number may not become 0. sharp: the inputs are such
    that few comparisons are left open (not so where squares underflow)."""
    codes, scales = np.asarray(codes, dtype=np.int64), np.asarray(scales, dtype=np.int64)
    finite = np.isfinite(x)
    assert np.all((codes & 0x7F == 0x7F) == ~finite), label
    a, d = np.where(finite, np.abs(x), 0.0), np.where(finite, dx, 0.0)
    lo, hi = blocks(np.maximum(a - d, 0)).max(1), blocks(a + d).max(1)
    elo, ehi = exponents(lo) + 127, exponents(hi) + 127
    assert np.all((scales == elo) | (scales == ehi)), f"{label}: scales"
    e = np.repeat(scales - 127, 32)[:len(x)].astype(np.float64)
    got = np.abs(e4m3(codes))
    low = to_grid(np.maximum(a - d, 0) * np.exp2(-e), rnd, -6, 3)
    high = to_grid((a + d) * np.exp2(-e), rnd, -6, 3)
    if positive:
        low = np.where((a - d > 0) & (low == 0), 2.0 ** -9, low)
        high = np.where((a + d > 0) & (high == 0), 2.0 ** -9, high)
    bad = finite & ~((low <= got) & (got <= high))
    assert not bad.any(), (f"{label}: {bad.sum()} codes, first {np.argmax(bad)}: {got[bad][:3]}, "
                           f"not from {low[bad][:3]} to {high[bad][:3]}")
    assert not sharp or (low != high).mean() < 0.02 or len(x) < 200, f"{label}: the comparison decides too little"
    neg = finite & (got > 0) & (np.abs(x) > dx)
    assert np.all(((codes & 0x80) != 0)[neg] == (x[neg] < 0)), f"{label}: signs"
    if positive:
        assert np.all((got > 0) | (a - d <= 0) | ~finite), f"{label}: a positive value became 0"


def check_bf16(got, x, dx, r16, label=""):
    """bfloat16 values against x, rounded up with the odds of 16 random bits."""
    got = np.asarray(got, dtype=np.float64)
    signed = got
    assert np.array_equal(np.isnan(got), np.isnan(x)), label
    f = np.isfinite(x)
    got, a, d = np.abs(got[f]), np.abs(x[f]), np.broadcast_to(dx, x.shape)[f]
    low, high = (to_grid(y, r16[f] / 65536.0, -126, 7) for y in (np.maximum(a - d, 0), a + d))
    bad = ~((low <= got) & (got <= high))
    assert not bad.any(), f"{label}: {bad.sum()} of {len(bad)}: {got[bad][:3]}, not {low[bad][:3]} to {high[bad][:3]}"
    assert (low != high).mean() < 0.02 or len(got) < 200, f"{label}: the comparison decides too little"
    sure = a > d
    assert np.array_equal(np.sign(_where_sure(x[f], sure)), np.sign(_where_sure(signed[f], sure))), f"{label}: signs"


def _where_sure(x, sure):
    return np.where(sure, x, 0.0)


def f32(x):
    return float(np.float32(x))


def step(p, g, m, v, *, lr, wd, beta1, beta2, eps, t, clip=1.0, lr_scale=1.0):
    """The update in float64 (v itself, not its root) and bounds on what
    float32 arithmetic, every operation rounded, adds: (p, m, v, s, dp, dm,
    ds). A product or sum adds U of its size, the constants (rounded betas,
    rates) U each; TINY for results among the denormals."""
    p, g, m, v = (np.asarray(a, dtype=np.float64) for a in (p, g, m, v))
    lr, wd = f32(lr), f32(wd)
    with np.errstate(all="ignore"):
        x = g * clip
        m1, m2 = beta1 * m, (1 - beta1) * x
        mn = m1 + m2
        dm = 5 * U * (np.abs(m1) + np.abs(m2)) + 3 * TINY * ((m1 != 0) | (m2 != 0))  # sums of zeros are exact
        vn = beta2 * v + (1 - beta2) * x * x
        dv = 7 * U * vn + 3 * TINY * (vn != 0)
        s = np.sqrt(vn)
        ds = np.sqrt(vn + dv) - np.sqrt(np.maximum(vn - dv, 0)) + U * s
        second, rate = 1 / np.sqrt(1 - beta2 ** t), lr * lr_scale / (1 - beta1 ** t)
        den = s * second + eps
        dden = ds * second + 4 * U * den + TINY
        term = rate * mn / den
        dterm = rate * dm / np.maximum(den - dden, TINY) + np.abs(term) * (dden / np.maximum(den - dden, TINY) + 6 * U)
        decay = lr * lr_scale * wd * p
        c = term + decay
        pn = p - c
        dp = dterm + 4 * U * np.abs(decay) + 2 * U * np.abs(c) + U * np.abs(pn) + 3 * TINY
    return pn, mn, vn, s, dp, dm, ds

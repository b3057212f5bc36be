"""The AdamW step by its formulas in 64 bits (numpy, CPU), element by element,
and how far a call may be off it.  Shares no code with the package."""
import numpy as np
import torch

BLOCK = 256
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step, relative
M64 = (1 << 64) - 1


# ---- random numbers ---------------------------------------------------------

def mix(z):
    z = (z & M64) ^ ((z & M64) >> 32)
    z = z * 0x6A09E667F3BCC909 & M64
    z = (z ^ (z >> 29)) * 0xBB67AE8584CAA73B & M64
    return z ^ (z >> 32)


def words(seed, t, tensor, element):
    """(first, second) 32 random bits of each element (an int64 array)."""
    k = mix(mix(mix(seed) + t) + tensor)
    e = np.asarray(element, dtype=np.uint64)
    k0 = np.uint32(k & 0xFFFFFFFF)
    k1 = np.uint32(k >> 32) ^ ((e >> np.uint64(32)).astype(np.uint32) * np.uint32(0xBB67AE85))
    x = ((e & np.uint64(0xFFFFFFFF)).astype(np.uint32) ^ k0) * np.uint32(0xBB67AE85)
    x = (x ^ (x >> np.uint32(17)) ^ k1) * np.uint32(0x6A09E667)
    w = x ^ (x >> np.uint32(15))
    y = (w + k0) * np.uint32(0x9E3779B1)
    return w, y ^ (y >> np.uint32(15))


def turned(w):
    return (w << np.uint32(16)) | (w >> np.uint32(16))


# ---- 8-bit states -------------------------------------------------------------

def exponents(x):
    """E of every block of the fp32 x: floor(log2) of its largest finite |x|, at least -119."""
    a = np.abs(x.astype(np.float64))
    a[~np.isfinite(a)] = 0.0
    full = np.zeros(-(-len(a) // BLOCK) * BLOCK)
    full[:len(a)] = a
    top = full.reshape(-1, BLOCK).max(axis=1)
    return np.maximum(np.frexp(np.maximum(top, 2.0 ** -140))[1] - 1, -119)


def held(x, w, second, exponent=None):
    """(values over their scale, scales) of the fp32 x, w: random words."""
    e = exponents(x) if exponent is None else exponent
    scale = np.ldexp(1.0, e - 7)
    y = x.astype(np.float64) / np.repeat(scale, BLOCK)[:len(x)]
    if second:
        a, u = np.maximum(np.abs(y), 2.0 ** -9), turned(w)
    else:
        a, u = np.abs(y), w
    a[np.isinf(a)] = np.nan
    u = (u >> np.uint32(12)).astype(np.float64) / 2.0 ** 20
    q = np.ldexp(1.0, np.maximum(np.frexp(np.where(a > 0, a, 1.0))[1] - 1, -6) - 3)
    return np.copysign(np.floor(a / q + u) * q, y), scale


def assert_held(codes, scale, x, w, second, what):
    """codes and scales are x's, or those of a neighbour of x: 64 bits rounded to 32
    in another order of operations may differ in the last place."""
    got, s = codes.float().cpu().double().numpy(), scale.cpu().double().numpy()
    near = [x, np.nextafter(x, np.float32(np.inf)), np.nextafter(x, np.float32(-np.inf))]
    fine_scale = np.zeros(len(s), dtype=bool)
    for z in near:
        fine_scale |= s == np.ldexp(1.0, exponents(z) - 7)
    assert fine_scale.all(), f"{what}: {(~fine_scale).sum()} scales"
    fine = np.zeros(len(x), dtype=bool)
    e = (np.frexp(s)[1] - 1 + 7)
    for z in near:
        value = held(z, w, second, e)[0]
        fine |= (got == value) | (np.isnan(got) & np.isnan(value))
    assert fine.all(), f"{what}: {(~fine).sum()} of {len(x)} codes, first at {np.argmin(fine)}"
    exact = held(x, w, second, e)[0]
    differ = ((got != exact) & ~(np.isnan(got) & np.isnan(exact))).mean()
    # a neighbour has another code with probability of about 2^-20, and is rare itself
    assert differ <= 4 / len(x), f"{what}: {differ}"


def values(codes, scale):
    n = codes.numel()
    return (codes.float().cpu().double().numpy() * np.repeat(scale.cpu().double().numpy(), BLOCK)[:n])


# ---- the step -------------------------------------------------------------------

def step64(p, g, m, v, t, lr, betas, eps, decay, clip):
    """p, m, v behind step t, in 64 bits, the size of p's step and of m's two terms;
    `decay`: lambda d_k; `clip`: c in fp32."""
    b1, b2 = betas
    c = np.float64(np.float32(clip))
    with np.errstate(over="ignore", invalid="ignore"):
        g = (np.float32(c) * g.astype(np.float32)).astype(np.float64)
        terms = np.abs(b1 * m) + np.abs((1.0 - b1) * g)
        m = b1 * m + (1.0 - b1) * g
        v = b2 * v + (1.0 - b2) * g * g
        d = np.sqrt(v / (1.0 - b2 ** t)) + eps
        update = lr / (1.0 - b1 ** t) * m / d
        drop = lr * decay * p
        return p - (drop + update), m, v, np.abs(drop) + np.abs(update), terms


def assert_states(got, want, what, terms=0.0):
    """fp32 states: one rounding, of a 64-bit value.  m's terms may cancel: each of them
    and their sum is rounded once in 64 bits on either side, 2^-53 of `terms` each, so
    the two sides' values before the rounding are 6 * 2^-53 of it apart at most."""
    off = np.abs(got.cpu().double().numpy() - want)
    tol = HALF[torch.float32] * np.abs(want) * (1 + 2.0 ** -20) + 6 * 2.0 ** -53 * terms + 2.0 ** -149
    bad = ~(off <= tol) & ~(np.isnan(want) & torch.isnan(got).cpu().numpy()) & ~(np.abs(want) >= 3.4028235e38)
    assert not bad.any(), f"{what}: {bad.sum()} off, first at {np.argmax(bad)}"


# Roundings of p's step, in halves of fp32's step: the factors lr lambda d_k and
# lr / (1 - b1^t) 1 each; m 1; product 1; reciprocal 2; product 1; beneath it the
# root 2, half of v's 1, its factor 1, eps 1, the sum 1; the last sum 1: 14 at most.
STEP = 14 * 2.0 ** -24


def tolerance(want, step):
    """Of p in fp32 before any rounding to its own type."""
    return HALF[torch.float32] * np.abs(want) + STEP * step


def assert_params(got, want, step, what, word=None):
    """`word`: the second random word, where p is rounded stochastically."""
    x = got.cpu().double().numpy()
    tol = tolerance(want, step)
    if word is None:
        if got.dtype == torch.bfloat16:
            tol = tol * (1 + 2.0 ** -8) + HALF[torch.bfloat16] * np.abs(want)
        bad = ~(np.abs(x - want) <= tol + 2.0 ** -133)
        assert not bad.any(), f"{what}: {bad.sum()} off, first at {np.argmax(bad)}"
        return
    u = (word >> np.uint32(16)).astype(np.float64) / 2.0 ** 16
    a = np.abs(want)
    q = np.ldexp(1.0, np.frexp(np.maximum(a, 2.0 ** -126))[1] - 8)
    # what lies within the tolerance of p may be rounded
    low, high = (np.floor(np.maximum(a + d * (tol + q * 2.0 ** -16), 0.0) / q + u) * q for d in (-1, 1))
    bad = ~((np.abs(x) >= low) & (np.abs(x) <= high)) | ((np.sign(x) != np.sign(want)) & (low > 0))
    assert not bad.any(), f"{what}: {bad.sum()} off, first at {np.argmax(bad)}"
    # and most are decided by u alone
    assert (low == high).mean() > 0.98 or len(x) < 200, what

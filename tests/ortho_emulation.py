"""The library's arithmetic of orthogonalised updates on the CPU, in fp16
operands and fp32 sums, and a bound on its error for one given matrix.

`emulate` follows the kernels' formulas (X in two fp16 halves, A = sI + R, F =
(b + 2cs) R + c R^2), not their tiles or their order of summation.  `low=False`
plants the mistake of losing X's low half in a FAST iteration.

The bound has two parts, as relative 2-norms of O.

Within X's own directions a step's roundings of R, F and X act through F, |F| <=
2.8 for the default coefficients:  steps * 2.8 * u,  u = 2^-11 (FAST, half a
step of fp16's 11 bits) or 2^-22 + sqrt(3 k / 32) * 2^-24 (FULL: two such
values, and the fp32 sums' random walk over 3 k / 32 matrix instructions).  It
takes the roundings of different elements for independent.  Where all elements
are alike they are not: F and X are each off by u, R by u and A by 2 u at once,
which changes the step from sigma to sigma p(sigma^2) by
    u (2 |f| + 3 x |b + 2 c x|) / p(x),   x = sigma^2,  f = p(x) - p(s),
of itself (`alike`), and every later step passes a relative error on times
|1 + 2 x p'(x) / p(x)|.

A rank of one, sigma v w^T with |v| = |w| = 1 and elements that differ
(`rank_one`), averages the same roundings: v^T E v of a symmetric E with
|E_ij| <= u m |v_i v_j| apart from its diagonal, |E_ii| <= u d, has a standard
deviation of at most u / sqrt(3) (sqrt(2) m sum v^4 + d sqrt(sum v^4)), and v^T E w
of |E_ij| <= u |v_i w_j| one of u / sqrt(3) sqrt(sum v^4 sum w^4).  F and R are of
the first kind, X of the second.  Five standard deviations of sigma's relative
error, passed on by the later steps as above, are added: polynomials that are
steep where sigma lies pass on a hundred times what they get.

In directions that X lacks, a step multiplies what it finds by a.  It finds the
rounding of X's elements (2^-23 of them: two fp16 halves), and what the step
itself puts there: with FAST the product F (X - X_high) is missing, and F is
-(b s + c s^2) I in those directions, so |b s + c s^2| * 2^-11 of X's norm, s
= ||X||^2 / r; with FULL the products that are left out and the halves' own
rounding, |a| * 2^-22; with both the fp32 sums over r values, |a| sqrt(3 r /
32) * 2^-24.  The steps' shares are independent: they add up in squares.
"""
import math

import torch

from ortho_reference import DEFAULT

X_SCALE, A_SCALE = 8192.0, 2048.0  # powers of two that the halves are stored at


def _split(v):
    hi = v.half().float()
    return hi, (v - hi).half().float()


def _product(p, q, full):
    if full:
        return p[0] @ q[0].t() + p[0] @ q[1].t() + p[1] @ q[0].t()
    return p[0] @ q[0].t()


def emulate(u, precision, steps=5, coefficients=None, low=True):
    """O(u) of one matrix on the CPU, as the library computes it."""
    full = precision == "full"
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    r = x.shape[0]
    halves = _split((x / x.norm() * X_SCALE).float())
    for k in range(steps):
        a, b, c = DEFAULT if coefficients is None else coefficients[k]
        if not low:
            halves = (halves[0], torch.zeros_like(halves[1]))
        s = 1.0 / r if k == 0 else float(((halves[0] + halves[1]).double() / X_SCALE).square().sum()) / r
        keep = a + b * s + c * s * s
        eye = torch.eye(r)
        big_r = _split(_product(halves, halves, full) * (A_SCALE / X_SCALE ** 2) - float(s * A_SCALE) * eye)
        if not full:
            big_r = (big_r[0], torch.zeros_like(big_r[1]))
        f = float(b + 2 * c * s) * (big_r[0] + big_r[1]) + float(c) / A_SCALE * _product(big_r, big_r, full)
        f = _split(f + float(keep * A_SCALE) * eye if full else f)
        x = _product(f, (halves[0].t().contiguous(), halves[1].t().contiguous()), full) / A_SCALE
        if not full:  # the last step leaves the low half out
            x = x + float(keep) * (halves[0] + halves[1] if k + 1 < steps else halves[0])
        halves = _split(x)
    o = x / X_SCALE
    return o.t() if tall else o


def reference_and_bound(u, precision, steps=5, coefficients=None, deficient=False, alike=False, rank_one=False,
                        counted=None):
    """O(u) in fp64 and the relative 2-norm that the library's O may be off by.
    `deficient`: u lacks directions; `rank_one`: all but one; `alike`: all but one,
    and its elements round alike; `counted`: the number of steps to count, where a polynomial is larger
    than the default's."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = (x.t() if tall else x).contiguous()
    r, c_side = x.shape
    x = x / x.norm()
    triples = [DEFAULT if coefficients is None else coefficients[k] for k in range(steps)]
    rest = [math.prod(abs(t[0]) for t in triples[k + 1:]) for k in range(steps)]  # growth behind step k
    fast = precision == "fast"
    half = 2.0 ** -11 if fast else 2.0 ** -22
    noise = (2.0 ** -23 * abs(triples[0][0]) * rest[0]) ** 2
    together = spread = 0.0
    # sums of the fourth powers of the unit vectors' elements, which each carry a part of X
    v4 = float((x.square().sum(1) ** 2).sum())
    w4 = float((x.square().sum(0) ** 2).sum())
    for k, (a, b, c) in enumerate(triples):
        size = float(x.norm())
        s = size * size / r
        share = (abs(b * s + c * s * s) if fast else abs(a)) * half
        stored = 2.0 ** -23 + abs(a) * math.sqrt(3 * r / 32) * 2.0 ** -24
        noise += ((share + stored) * size * rest[k]) ** 2
        if alike or rank_one:
            z = size * size
            p = a + b * z + c * z * z
            f, slope = abs(p - (a + b * s + c * s * s)), abs(z * (b + 2 * c * z))
            passed = abs(1 + 2 * z * (b + 2 * c * z) / p)
            together = together * passed + half * (2 * f + 3 * slope) / abs(p)
            first = [m * math.sqrt(2) * v4 + d * math.sqrt(v4) for m, d in (
                (f, abs(b * s + c * s * s)), (slope, slope / z * s))]
            second = [m * math.sqrt(v4 * w4) for m in (f, 2 * slope)]
            deviation = half / math.sqrt(3) * math.sqrt(sum(t * t for t in first + second)) / abs(p)
            spread = math.hypot(spread * passed, deviation)
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    out = float(x.norm())
    sums = 0.0 if fast else math.sqrt(3 * c_side / 32) * 2.0 ** -24
    bound = (counted or steps) * 2.8 * (half + sums)
    if alike:
        bound = max(bound, together + steps * 2.8 * sums)
    if rank_one:
        bound += 5 * spread
    if deficient:
        bound += math.sqrt(noise) / out
    return (x.t() if tall else x).contiguous(), bound

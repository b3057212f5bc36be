"""A plain 64-bit implementation of the orthogonalised updates, and how far
the library's results may be from it.

Tolerances, for relative 2-norms of a matrix's O.  One iteration rounds three
kinds of operands (R, the polynomial Q, X) to u = 2^-11 (FAST, half a step of
fp16's 11 bits) or about 2^-22 (FULL, two such values), independently, with a
root mean square of u / sqrt(3) each; they act through Q, whose norm the
quintic keeps below 2.8 (|a + b x + c x^2 - (a + bs + cs^2)| for x in
[0, 1.2]).  With the three added in squares and the iterations added up:

    FAST  steps * 2.8 * 2^-11
    FULL  steps * 2.8 * (2^-22 + sqrt(3 k / 32) * 2^-24)

the last term being the fp32 sums' random walk over 3 k / 32 matrix
instructions for a sum of k terms.  Noise in directions that X lacks grows by
a = 3.4445 a step: X's own 22 bits (2^-23) by a^steps against ||O||, added to
both.  An element may be off by ten times that, of its own size or of the
matrix's root mean square where that is more: a rounding is relative to the
value rounded, so where X has rows and columns of very different size (a
product of two Gaussian vectors has elements fourteen times the root mean
square), an element's error grows with the element.
An output of type t adds half a step, finfo(t).eps / 2.
"""
import math

import torch

DEFAULT = (3.4445, -4.7750, 2.0315)


def ortho64(u, steps=5, coefficients=None):
    """O(u) of one matrix in fp64."""
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    x = x.contiguous()
    size = x.norm()
    if float(size) == 0.0:
        return torch.zeros_like(u, dtype=torch.float64)
    x = x / size
    for k in range(steps):
        a, b, c = DEFAULT if coefficients is None else coefficients[k]
        g = x @ x.t().contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return (x.t() if tall else x).contiguous()


def o_tolerance(rows, cols, precision, size, steps=5):
    """Relative 2-norm tolerance of O, whose 2-norm is `size`."""
    k = max(rows, cols)
    u = 2.0 ** -11 if precision == "fast" else 2.0 ** -22 + math.sqrt(3 * k / 32) * 2.0 ** -24
    return steps * 2.8 * u + 2.0 ** -23 * 3.4445 ** steps / max(size, 1e-30)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_o_close(got, ref, precision, what, steps=5):
    """`got` (any type) against O in fp64."""
    rows, cols = ref.shape
    size = float(ref.norm())
    d = got.double() - ref
    if size == 0.0:
        assert float(d.abs().max()) == 0.0, what
        return
    tol = o_tolerance(rows, cols, precision, size, steps)
    half = half_step(got.dtype)
    rel = float(d.norm()) / size
    assert rel <= tol + half, f"{what}: relative error {rel:.3g}, tolerance {tol + half:.3g}"
    rms = size / math.sqrt(rows * cols)
    over = float((d.abs() / ref.abs().clamp(min=rms)).max())
    assert over <= 10 * (tol + half), f"{what}: an element is off by {over:.3g} of itself or of the rms"


def layout(shapes, gaps=None, tail=0):
    """(numel, [(offset, rows, cols)]) of matrices behind gaps of the given lengths."""
    gaps = gaps or [0] * len(shapes)
    at, out = 0, []
    for (r, c), gap in zip(shapes, gaps):
        at += gap
        out.append((at, r, c))
        at += r * c
    return at + tail, out


def mask_of(numel, matrices, device):
    """True where an element belongs to a matrix."""
    m = torch.zeros(numel, dtype=torch.bool, device=device)
    for at, r, c in matrices:
        m[at:at + r * c] = True
    return m


def matrix(t, spec):
    at, r, c = spec
    return t[at:at + r * c].view(r, c)

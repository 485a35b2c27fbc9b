"""Plain 64-bit forms of what stands beside the projections, and how far fp32 kernels may be from them.

u = 2^-24 is half a step of fp32 (relative), eps / 2 that of the output type."""
import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def adapters(x, A, B, parts, rows, base, scale=None, ranks=None):
    """(y, bound on |y - kernel's|).  h is a sum of K fp32 products in any order, tensor cores included, which may cut instead of round:
    off by at most 2 u (K + 8) sum |x a|; kept to 16 bits of significand: 2^-16 |h|; the second sum likewise, (R + 8) of its steps; one
    rounding to y's type, and one of the fp32 sum in front of it."""
    S, P, R, K = A.shape
    y, off = base.double().clone(), torch.zeros(base.shape, dtype=torch.float64, device=base.device)
    for m, a in enumerate(rows.tolist()):
        if not 0 <= a < S:
            continue
        rank = R if ranks is None else min(max(int(ranks[a]), 0), R)
        s = 1.0 if scale is None else float(scale[a])
        begin = 0
        for p, n in enumerate(parts):
            xa = x[m].double() * A[a, p, :rank].double()
            h, hs = xa.sum(1), xa.abs().sum(1)
            b = B[a, begin:begin + n, :rank].double()
            y[m, begin:begin + n] += s * (b @ h)
            e = 2 * U * (K + 8) * hs + 2.0 ** -16 * h.abs() + 2 * U * (R + 8) * h.abs()
            off[m, begin:begin + n] = abs(s) * (b.abs() @ e) * (1 + 2.0 ** -10)
            begin += n
    bound = off + (half_step(base.dtype) + 2 * U) * (y.abs() + off)
    return y, bound


def frequencies(rot, layout="half", scaling="none", base=10000.0, factor=1.0, original_positions=0, beta_fast=32.0, beta_slow=1.0, low_factor=1.0,
                high_factor=4.0, **_):
    """Radians per position of every pair, and the factor of rotated elements."""
    if scaling == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [v / factor for v in f], 1.0
    if scaling == "yarn":
        edge = lambda turns: rot * math.log(original_positions / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(edge(beta_fast)), 0), min(math.ceil(edge(beta_slow)), rot - 1)
        share = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(rot // 2)]
        return [v * (1 - t) + v / factor * t for v, t in zip(f, share)], 0.1 * math.log(factor) + 1
    if scaling == "bands":
        out = []
        for v in f:
            turns = original_positions * v / (2 * math.pi)
            t = min(max((turns - low_factor) / (high_factor - low_factor), 0.0), 1.0)
            out.append(v * t + v / factor * (1 - t))
        return out, 1.0
    return f, 1.0


def heads(t, positions, f, factor, rot, layout, norm=False, weight=None, eps=1e-6):
    """(result, bound) of one tensor (M, heads, D).  The norm: a sum of D squares (off by (D + 2) u of itself, half that in the root), a
    reciprocal root good to 4 u, two products; cosine and sine to 8 u: an angle of at most pi / 4 through one conversion and one product by a
    rounded constant, a polynomial of a few terms; two products and a sum; one rounding to the type."""
    D = t.shape[-1]
    z = t.double()
    rel = 0.0
    if norm:
        z = z / (z.square().mean(-1, keepdim=True) + eps).sqrt()
        if weight is not None:
            z = z * weight.double()
        rel = (D / 2 + 8) * U
    angle = positions.double()[:, None] * torch.tensor(f, dtype=torch.float64, device=t.device)
    # (the product of a far position and a frequency in 64 bits is itself off by 2^-53 of the angle)
    loose = angle.abs().max().item() * 2.0 ** -52 if angle.numel() else 0.0
    c, s = (v[:, None] * factor for v in (angle.cos(), angle.sin()))
    first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    a, b = z[..., first], z[..., second]
    r, off = z.clone(), z.abs() * rel
    r[..., first], r[..., second] = a * c - b * s, b * c + a * s
    both = (a.abs() + b.abs()) * factor * (rel + 12 * U + loose)
    off[..., first] = both
    off[..., second] = both
    return r, off + half_step(t.dtype) * (r.abs() + off) + 1e-37


def adapters_of_many(x, A, B, parts, rows, base, scale=None, ranks=None):
    """The same for many rows: a matrix product in 64 bits per adapter."""
    S, P, R, K = A.shape
    y, off = base.double().clone(), torch.zeros(base.shape, dtype=torch.float64, device=base.device)
    for a in rows.unique().tolist():
        if not 0 <= a < S:
            continue
        at = torch.nonzero(rows == a).flatten()
        rank = R if ranks is None else min(max(int(ranks[a]), 0), R)
        s = 1.0 if scale is None else float(scale[a])
        begin = 0
        for p, n in enumerate(parts):
            xd, w = x[at].double(), A[a, p, :rank].double().T
            h, hs = xd @ w, xd.abs() @ w.abs()
            b = B[a, begin:begin + n, :rank].double().T
            e = 2 * U * (K + 8) * hs + 2.0 ** -16 * h.abs() + 2 * U * (R + 8) * h.abs()
            y[at, begin:begin + n] += s * (h @ b)
            off[at, begin:begin + n] = abs(s) * (e @ b.abs()) * (1 + 2.0 ** -10)
            begin += n
    return y, off + (half_step(base.dtype) + 2 * U) * (y.abs() + off)

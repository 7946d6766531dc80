"""The row operators (dropout, position bias, residual join) from their definitions, in 64 bits and whole numbers, with
bounds on what fp32 arithmetic in any order may differ by.  Torch on the CPU; shares nothing with the library."""
from __future__ import annotations

import math

import numpy as np
import torch

U = 2.0 ** -24  # a rounding to fp32 is off by at most this, relative


def half_step(dtype):
    """Largest relative error of one rounding to dtype."""
    return torch.finfo(dtype).eps / 2


# ---------------------------------------------------------------- dropout


def philox(c0, c1, c2, c3, key):
    """Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw 2011) on numpy arrays of whole numbers below 2^32."""
    c = [np.asarray(v, dtype=np.uint64) for v in (c0, c1, c2, c3)]
    k = [key & 0xFFFFFFFF, key >> 32]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) % 2**32, (k[1] + 0xBB67AE85) % 2**32]
    return c


def threshold(p):
    return math.floor(float(np.float32(p)) * 65536 + 0.5)


def kept(rows, cols, p, seed, offset):
    """Truth [rows, cols]; offset with the step already added."""
    r, g = np.meshgrid(np.arange(rows), np.arange(-(-cols // 8)), indexing="ij")
    n = offset % 2**64
    words = np.stack(philox(g, r, n & 0xFFFFFFFF, n >> 32, seed % 2**64), -1)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], -1).reshape(rows, -1)
    return torch.from_numpy(halves[:, :cols] >= threshold(p))


def drop_scale(p):
    t = threshold(p)
    return 65536.0 / (65536 - t) if t < 65536 else 0.0


# ---------------------------------------------------------------- position bias


def bucket(r, num_buckets, max_distance, two_sided):
    """Bucket of key position minus query position, by comparing whole-number powers."""
    side = num_buckets // 2 if two_sided else num_buckets
    n = abs(r) if two_sided else max(-r, 0)
    E = side // 2
    L = side - E
    if n < E:
        b = n
    else:
        b = E
        while b + 1 < side and n ** L >= E ** (L - (b + 1 - E)) * max_distance ** (b + 1 - E):
            b += 1
    return b + (side if two_sided and r > 0 else 0)


def bias_index(q_len, k_len, start, num_buckets, max_distance, two_sided, causal):
    """Bucket of every place of one sequence, -1 where masked: [q_len, k_len]."""
    of = {}
    out = np.empty((q_len, k_len), dtype=np.int64)
    for d in range(-(q_len - 1), k_len):
        r = d - start
        of[d] = -1 if causal and r > 0 else bucket(r, num_buckets, max_distance, two_sided)
    diagonals = np.array([of[d] for d in range(-(q_len - 1), k_len)], dtype=np.int64)
    for i in range(q_len):
        out[i] = diagonals[q_len - 1 - i:q_len - 1 - i + k_len]
    return torch.from_numpy(out)


# ---------------------------------------------------------------- residual join.  Every function takes 64-bit tensors
# [rows, d] and gives (value, bound): the bound is on the error of fp32 arithmetic in sums of `chain(d)` roundings


def chain(n):
    """Roundings that a term of a sum of n goes through: strided over at least 256 lanes or kept to 32 terms a lane, then
    joined over lanes and warps."""
    return n / 256 + 48


def norm(v, e, layer, eps):
    """Norm of rows known to within e: (n, bound of n, rstd, relative bound of rstd)."""
    d = v.shape[1]
    D = chain(d) * U
    mean = v.mean(1, keepdim=True) if layer else torch.zeros_like(v[:, :1])
    e_mean = (e.mean(1, keepdim=True) + D * v.abs().mean(1, keepdim=True)) if layer else torch.zeros_like(mean)
    c = v - mean
    e_c = e + e_mean + U * c.abs()
    s = (c * c).mean(1, keepdim=True) + eps
    rstd = s.rsqrt()
    # the sum of squares: roundings relative to itself, and what the elements are off by
    rel = ((D + 6 * U) * s + (2 * c.abs() * e_c + e_c * e_c).mean(1, keepdim=True)) / s / 2
    n = c * rstd
    return n, 1.05 * (e_c * rstd + n.abs() * (rel + 3 * U)), rstd, 1.05 * rel + 4 * U


def norm_grad(n, e_n, rstd, rel, g, e_g, layer):
    """Gradient through a norm: rstd (g - [mean g] - n mean(g n))."""
    D = chain(n.shape[1]) * U
    dot = (g * n).mean(1, keepdim=True)
    mass = (g * n).abs().mean(1, keepdim=True)
    e_dot = (e_g * n.abs() + g.abs() * e_n).mean(1, keepdim=True) + (D + 4 * U) * mass
    t = g - n * dot
    size = g.abs() + n.abs() * dot.abs()
    e = e_g + n.abs() * e_dot + e_n * dot.abs()
    if layer:
        mean = g.mean(1, keepdim=True)
        t = t - mean
        size = size + mean.abs()
        e = e + e_g.mean(1, keepdim=True) + (D + 2 * U) * g.abs().mean(1, keepdim=True)
    return rstd * t, 1.05 * rstd * (e + size * (rel + 6 * U))


def spread(gate, rows):
    """Gate [rows / k, d or 1] over all rows."""
    if gate is None:
        return torch.ones(1, 1, dtype=torch.float64)
    return gate.repeat_interleave(rows // max(1, gate.shape[0]), 0)


def join(x, residual, w_post, w_pre, gate, scale, layer, eps, factor):
    """[(out, bound), (normed, bound) or None], before the rounding to the stored type.  factor: what dropout multiplies by."""
    zero = torch.zeros_like(x)
    y, e = x, zero
    if w_post is not None:
        n, e_n, _, _ = norm(x, zero, layer, eps)
        y = n * w_post
        e = e_n * w_post.abs() + U * y.abs()
    m = (factor * scale * spread(gate, x.shape[0])).abs()
    y = y * factor * scale * spread(gate, x.shape[0])
    e = e * m + 5 * U * y.abs()
    out = y if residual is None else residual + y
    e = e + U * out.abs()
    if w_pre is None:
        return [(out, e), None]
    n, e_n, _, _ = norm(out, e, layer, eps)
    return [(out, e), (n * w_pre, e_n * w_pre.abs() + 2 * U * (n * w_pre).abs())]


def join_grad(grad_out, grad_normed, x, out, w_post, w_pre, gate, scale, layer, eps, factor):
    """Dict of (gradient, bound) of x, residual, gate, w_post, w_pre."""
    rows = x.shape[0]
    zero = torch.zeros_like(x)
    t, e_t = (grad_out, zero) if grad_out is not None else (zero, zero)
    got = {}
    R = (rows + 16) * U

    def columns(terms, e, groups=1):
        shape = (groups, rows // groups, -1) if groups else None
        return terms.reshape(shape).sum(1), (e + R * terms.abs()).reshape(shape).sum(1)

    if w_pre is not None:
        n, e_n, rstd, rel = norm(out, zero, layer, eps)
        g = grad_normed * w_pre
        v, e_v = norm_grad(n, e_n, rstd, rel, g, U * g.abs(), layer)
        t, e_t = t + v, e_t + e_v + U * (t + v).abs()
        w, e = columns(grad_normed * n, grad_normed.abs() * e_n + U * (grad_normed * n).abs())
        got["w_pre"] = (w[0], e[0])
    got["residual"] = (t, e_t)
    y, e_y = x, zero
    if w_post is not None:
        n, e_n, rstd, rel = norm(x, zero, layer, eps)
        y, e_y = n * w_post, e_n * w_post.abs() + U * (n * w_post).abs()
    if gate is not None:
        terms = scale * factor * y * t
        e = abs(scale) * factor * (e_y * t.abs() + y.abs() * e_t) + 5 * U * terms.abs()
        if gate.shape[1] == 1 and gate.shape != x.shape:
            got["gate"] = (terms.sum(1, keepdim=True), (e + (chain(x.shape[1]) * U) * terms.abs()).sum(1, keepdim=True))
        elif gate.shape[0] == rows:
            got["gate"] = (terms, e)
        else:
            got["gate"] = columns(terms, e, gate.shape[0])
    m = factor * scale * spread(gate, rows)
    u = m * t
    e_u = m.abs() * e_t + 5 * U * u.abs()
    if w_post is not None:
        w, e = columns(u * n, e_u * n.abs() + u.abs() * e_n + U * (u * n).abs())
        got["w_post"] = (w[0], e[0])
        g = u * w_post
        u, e_u = norm_grad(n, e_n, rstd, rel, g, e_u * w_post.abs() + U * g.abs(), layer)
    got["x"] = (u, e_u)
    return got


def assert_within(got, want, bound, what):
    """got (a tensor of its stored type) against the 64-bit value: the bound, and one rounding to the stored type."""
    g = got.detach().cpu().double().reshape(want.shape)
    tol = bound + half_step(got.dtype) * (want.abs() + bound) + 1e-40
    bad = ~((g - want).abs() <= tol)
    if bool(bad.any()):
        k = int(torch.where(bad, (g - want).abs() / tol, torch.zeros_like(tol)).nan_to_num(math.inf).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} out of tolerance; at {k}: {g.reshape(-1)[k]!r} for "
                             f"{want.reshape(-1)[k]!r}, tolerance {tol.reshape(-1)[k]:.3e}")

"""64-bit definitions of the operators that stand around the attention block (rotary positions, norms between blocks, linear
layers and mixtures of experts on 4-bit weights) in numpy, written apart from the kernels, with the error bounds that the
tests hold the kernels to."""
import numpy as np
import torch

from _decoder import TINY, TYPES, U  # noqa: F401  (types, roundings, subnormal steps)

u = 2.0 ** -24  # fp32


def rng_tensor(rng, shape, dtype, scale=1.0):
    """(a tensor of the type on the CPU, its values in 64 bits)."""
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(TYPES[dtype])
    return t, t.double().numpy()


def check(got, want, bound, what):
    got = np.asarray(got, np.float64)
    assert got.shape == want.shape, f"{what}: shape {got.shape}, not {want.shape}"
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places"
    skip = nan | np.isinf(want)
    d = np.abs(np.where(skip, 0, np.where(skip, 0, got) - np.where(skip, 0, want)))
    bad = np.where(np.isinf(want), got != want, ~(d <= np.where(skip, 0, bound)))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} outside; first at {i}: {got[i]!r}, not {want[i]!r} +- "
                             f"{np.broadcast_to(bound, d.shape)[i]!r}")


# ------------------------------------------------------------------ rotary positions

def freqs(rot, base=10000.0, scaling="none", factor=1.0, length=0.0, low=1.0, high=32.0):
    """Radians a position of each pair."""
    if scaling == "base" and rot > 2:
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-2.0 * np.arange(rot // 2) / rot)
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        k = np.clip((length * f / (2 * np.pi) - low) / (high - low), 0, 1)
        f = k * f + (1 - k) * f / factor
    return f


def rope(x, f, starts, lens, layout, magnitude, inverse, dtype):
    """(y, bound) of x fp64 [B][T][heads][D].  The bound: the output's rounding, and (|a| + |b|) magnitude times 2^-21: an angle
    rounded to 2^-25 half turns (pi 2^-25), sine and cosine within an ulp (2 2^-24), their product with the magnitude, two
    products and a sum (4 2^-24)."""
    B, T, _, _ = x.shape
    rot = 2 * len(f)
    y, mag = x.copy(), np.zeros_like(x)
    a_at, b_at = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    for b in range(B):
        n = T if lens is None else min(T, max(0, int(lens[b])))
        angle = ((int(starts[b]) + np.arange(n, dtype=np.float64))[:, None] * f)[:, None, :]
        c, s = np.cos(angle) * magnitude, np.sin(angle) * magnitude * (-1 if inverse else 1)
        p, q = x[b, :n, :, a_at], x[b, :n, :, b_at]
        y[b, :n, :, a_at], y[b, :n, :, b_at] = p * c - q * s, q * c + p * s
        mag[b, :n, :, a_at] = mag[b, :n, :, b_at] = abs(magnitude) * (np.abs(p) + np.abs(q))
    return y, U[dtype] * np.abs(y) + TINY[dtype] + 2.0 ** -21 * mag


# ------------------------------------------------------------------ norms

def norm(z, e, w, b, kind, eps):
    """(norm of z, its error) given an error e of z, element by element.

    Sums of a row: at most 16 values a thread one after another, then two trees of five; rows past 16384 values 64 at a time
    and their sums; with the products, the mean's factor and rsqrt's 2 ulp that is below 32 u of a sum of magnitudes there and
    100 u here."""
    K = z.shape[-1]
    n = 32 if K <= 16384 else 100 + K / 65536
    mean = lambda a: a.mean(-1, keepdims=True)  # noqa: E731
    if kind == "layer":
        e = e + mean(e) + n * u * (mean(np.abs(z)) + np.abs(z))
        z = z - mean(z)
    ms = mean(z * z) + eps
    inv = 1 / np.sqrt(ms)
    rel = np.sqrt(mean(z * z) * mean(e * e)) / ms + n * u
    y, d = z * inv, 1.01 * (e * inv + np.abs(z) * inv * rel)
    if w is not None:
        y, d = y * w, d * np.abs(w)
    if b is not None:
        y, d = y + b, d + 2 * u * np.abs(b)
    return y, d + 4 * u * np.abs(y)


def add_norm(x, r, pre, post, gate, per, scale, dtype, rtype):
    """((s, bound), (y, bound)); pre, post: (w, b, kind, eps) or None; gate [rows][K] or None."""
    v, e = x, np.zeros_like(x)
    if post is not None:
        v, e = norm(v, e, *post)
    f = np.full_like(x, float(np.float32(scale)))
    if gate is not None:
        f = f * gate[np.arange(x.shape[0]) // per]
    s = f * v
    e = np.abs(f) * e + 3 * u * np.abs(s)
    if r is not None:
        s, e = s + r, e + u * np.abs(s + r)
    out = [(s, e + U[rtype] * np.abs(s) + TINY[rtype])]
    if pre is not None:
        y, d = norm(s, e, *pre)
        out.append((y, d + U[dtype] * np.abs(y) + TINY[dtype]))
    return out


# ------------------------------------------------------------------ 4-bit weights

NIBBLE = (0, 4, 1, 5, 2, 6, 3, 7)


def bf16_up(x):
    """Positive fp32 to the next bf16 value at or above it, as fp32."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((b + np.uint32(0xFFFF)) & np.uint32(0xFFFF0000)).view(np.float32)


def quantize_w4(w, G):
    """fp32 [..., M, K] -> (codes int8 [..., M, K], scales fp32 [..., M, ceil(K / G)])."""
    K = w.shape[-1]
    n = -(-K // G)
    g = np.zeros(w.shape[:-1] + (n * G,), np.float32)
    g[..., :K] = w
    g = g.reshape(w.shape[:-1] + (n, G))
    s = bf16_up(np.abs(g).max(-1) / np.float32(7))
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s[..., None] > 0, np.clip(np.rint(g / s[..., None]), -7, 7), 0)
    return c.reshape(w.shape[:-1] + (n * G,))[..., :K].astype(np.int8), s


def pack_w4(c, s, G, fill=0):
    """(codes uint8 [..][RT][CT][1024], scales uint16 [..][RT][CT][16][128 / G]); what stands past the matrix: code `fill`, scale 0
    (2^90 for other fills)."""
    lead, (M, K) = c.shape[:-2], c.shape[-2:]
    RT, CT, per = -(-M // 16), -(-K // 128), 128 // G
    n = np.full(lead + (RT * 16, CT * 128), fill + 8, np.uint8)
    n[..., :M, :K] = c + 8
    sc = np.full(lead + (RT * 16, CT * per), 2.0 ** 90 if fill else 0.0, np.float32)
    sc[..., :M, :s.shape[-1]] = s
    codes = np.zeros(lead + (RT, CT, 1024), np.uint8)
    for m in range(16):
        r, g = divmod(m, 8)
        for k in range(128):
            j, t, i = k // 32, k % 32 // 8, k % 8
            at = (((8 * r + g) * 4 + t) * 4 + j) * 4 + NIBBLE[i] // 2
            codes[..., at] |= n[..., m::16, k::128] << (4 * (NIBBLE[i] % 2))
    sc = sc.view(np.uint32) >> 16
    sc = np.moveaxis(sc.reshape(lead + (RT, 16, CT, per)), -2, -3).astype(np.uint16)
    return codes, np.ascontiguousarray(sc)


def unpack_w4(codes, M, K):
    out = np.zeros(codes.shape[:-3] + (codes.shape[-3] * 16, codes.shape[-2] * 128), np.int8)
    for m in range(16):
        r, g = divmod(m, 8)
        for k in range(128):
            j, t, i = k // 32, k % 32 // 8, k % 8
            at = (((8 * r + g) * 4 + t) * 4 + j) * 4 + NIBBLE[i] // 2
            out[..., m::16, k::128] = (codes[..., at] >> (4 * (NIBBLE[i] % 2)) & 15).astype(np.int8) - 8
    return out[..., :M, :K]


def random_w4(rng, shape, G, spread=0.3):
    """(codes, scales) of random weights, -8 among the codes, scales of bf16 values; rows of K weights with sums of squares of about 1."""
    M, K = shape[-2:]
    c = np.clip(np.rint(rng.standard_normal(shape) * 3), -8, 7).astype(np.int8)
    s = bf16_up(np.exp(rng.standard_normal(shape[:-1] + (-(-K // G),)) * spread).astype(np.float32) / np.float32(3 * K ** 0.5))
    return c, s


def dequantize_w4(c, s, G):
    return c * np.repeat(s.astype(np.float64), G, -1)[..., :c.shape[-1]]


def weights(c, s, G, dev, fill=0):
    from paper_1705_01462_gb300 import fgq
    codes, sc = pack_w4(c, s, G, fill)
    return fgq.W4Weights(torch.from_numpy(codes).to(dev), torch.from_numpy(sc.view(np.int16)).view(torch.bfloat16).to(dev),
                         *c.shape[-2:])


def beta(K, G, many=False, dtype=None):
    """Error of sums of K exact products, of the sum of their magnitudes.  A matrix instruction adds 16 products to a sum with
    each term cut off at 2^-24 of the largest at worst: 17 2^-24 an instruction and G / 16 a group; groups, warps, parts and a
    cluster's blocks are added in fp32 (many: one sum over K, cut off once in 16 products by at most 2^-23, and up to 16 splits; fp32: runs of 256
    columns of two parts, 17 2^-24 in 16 products as above, the runs added in fp32, and 2^-22 = 4 u that the parts leave out)."""
    if many and dtype == "f32":
        return (17 * 16 + K / 256 + 24) * u
    if many:
        return K * 2.0 ** -27 + 20 * u
    return (17 * G / 16 + K / G + 40) * u


def in_range(y, dtype):
    """y, infinite where the type has no value near it: fp16 rounds from 65520 on, halfway past its largest, to infinity."""
    return np.where(np.abs(y) >= 65520, np.copysign(np.inf, y), y) if dtype == "f16" else y


def linear(x, w, G, bias, dtype, many=False):
    y = x @ w.T
    e = beta(x.shape[1], G, many, dtype) * (np.abs(x) @ np.abs(w).T)
    if many:  # bf16 tokens below 2^-28 of their largest and weights below 2^-28 of their row's lose bits
        e = e + 2.0 ** -36 * np.abs(x).max(1, keepdims=True) * np.abs(w).sum(1) + 2.0 ** -36 * np.abs(w).max(1) * np.abs(x).sum(1, keepdims=True)
    if bias is not None:
        y = y + bias
        e = e + 2 * u * np.abs(y)
    return in_range(y, dtype), e + U[dtype] * np.abs(y) + TINY[dtype]


# ------------------------------------------------------------------ mixture of experts

def route(x, router, top, score, renormalize, scale):
    """(ids, weights, relative error of the weights)."""
    logits = x @ router.T
    ids = np.argsort(-logits, axis=1, kind="stable")[:, :top]
    best = np.take_along_axis(logits, ids, 1)
    # a logit: chains of 8 products in fp32, 8 u of their magnitudes, and its rounding to fp32
    e = 10 * u * (np.abs(x) @ np.abs(router).T).max(1) + u * np.abs(logits - logits.max(1, keepdims=True)).max(1)
    if score == "softmax":
        g = np.exp(best - logits.max(1, keepdims=True))
        g = g / (g if renormalize else np.exp(logits - logits.max(1, keepdims=True))).sum(1, keepdims=True)
    else:
        g = 1 / (1 + np.exp(-best))
        if renormalize:
            g = g / g.sum(1, keepdims=True)
    # exp's 2 ulp, the sum over experts, the division, and what errors of two logits do
    return ids, g * scale, 2 * e[:, None] + 64 * u


def experts(x, ids, g, e_g, wg, wu, wd, G, Gd, dtype):
    """(y, bound); ids outside the experts are left out."""
    P, K = x.shape
    E, F, _ = wg.shape
    y, e = np.zeros((P, K)), np.zeros((P, K))
    # more than two units of 8 tokens an expert, or where long rows make units smaller, may run on the products of many tokens
    many = ids.size > (8 if dtype == "f32" else 16) * E or max(K, F) > 4096
    # between the layers: bf16 tokens' values in 11 bits at least, half a step of them; fp16 ones' in two parts of 8 bits; fp32's exact
    # (many: in two fp16 parts, within 2^-22)
    held = {"f32": 4 * u if many else u, "bf16": 2.0 ** -12, "f16": 2.0 ** -17}[dtype]

    def sums(w, v, n, G, dt):
        """What the sums of w times v, of n products each, are off by."""
        e = beta(n, G, many, dt) * (np.abs(w) @ np.abs(v))
        if many:  # as for a linear layer
            e = e + 2.0 ** -36 * np.abs(v).max() * np.abs(w).sum(1) + 2.0 ** -36 * np.abs(w).max(1) * np.abs(v).sum()
        return e

    for p in range(P):
        for j in range(ids.shape[1]):
            n = ids[p, j]
            if n < 0 or n >= E:
                continue
            a, b = wg[n] @ x[p], wu[n] @ x[p]
            ea, eb = sums(wg[n], x[p], K, G, dtype), sums(wu[n], x[p], K, G, dtype)
            sig = 1 / (1 + np.exp(-a))
            h = a * sig * b
            eh = 1.1 * ea * (np.abs(b) + eb) + np.abs(a * sig) * eb + (held + 8 * u) * np.abs(h)
            if dtype != "f32" or many:  # values that fp16, scaled to a largest of 2^14, holds as subnormals: half their step
                eh = eh + 2.0 ** -39 * np.abs(h).max()
            v = wd[n] @ h
            ev = np.abs(wd[n]) @ eh + sums(wd[n], h, F, Gd, "bf16" if dtype == "bf16" else "f32")
            y[p] += g[p, j] * v
            e[p] += np.abs(g[p, j]) * (ev + e_g[p, 0] * np.abs(v))
            # sums of choices, warps and blocks
            e[p] += 40 * u * np.abs(g[p, j]) * (np.abs(wd[n]) @ np.abs(h))
    return y, e + U[dtype] * np.abs(y) + TINY[dtype]

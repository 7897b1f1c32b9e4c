"""64-bit definitions of the decoder operators (4-bit cache, its attention, 8-bit linear layers) in
numpy, written apart from the kernels, with the error bounds that the tests hold the kernels to."""
import math

import numpy as np
import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# unit roundoffs of the output types
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
# half the spacing of the types' subnormals: what rounding a smaller output may move it by
TINY = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


def bf16_round(x, up):
    """fp32 array to the next bf16 value at or above (up) or at or below it, as fp32."""
    x = np.asarray(x, np.float32)
    with np.errstate(over="ignore"):
        t = (x.view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)  # towards zero
        away = ((x.view(np.uint32) & np.uint32(0xFFFF0000)) + np.uint32(0x10000)).view(np.float32)
    return np.where((t != x) & ((x > 0) == up), away, t)


def quantize4(x, G):
    """fp32 [..., D] -> (codes uint8 [..., D], lo fp32 [..., D / G], s fp32 [..., D / G])."""
    g = np.asarray(x, np.float32).reshape(x.shape[:-1] + (-1, G))
    lo = bf16_round(g.min(-1), up=False)
    s = bf16_round((g.max(-1) - lo) / np.float32(15), up=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        q = np.where(s[..., None] > 0, np.rint((g - lo[..., None]) / s[..., None]), 0)
    return np.clip(q, 0, 15).astype(np.uint8).reshape(x.shape), lo, s


def dequantize4(codes, lo, s):
    """The values that codes stand for, 64 bits."""
    G = codes.shape[-1] // lo.shape[-1]
    rep = lambda a: np.repeat(a.astype(np.float64), G, axis=-1)  # noqa: E731
    return rep(lo) + rep(s) * codes


def pack_params(lo, s):
    return (lo.view(np.uint32) & np.uint32(0xFFFF0000)) | (s.view(np.uint32) >> np.uint32(16))


def nibble_of(d, D, keys):
    """Nibble of a cache row that holds value d."""
    j, r = divmod(d, 32)
    if keys:
        t, i = divmod(r, 8)
        return 8 * (t * (D // 32) + j) + (0, 4, 1, 5, 2, 6, 3, 7)[i]
    g, i = divmod(r, 4)
    return 4 * (g * (D // 32) + j) + i


def unpack_codes(packed, keys):
    D = 2 * packed.shape[-1]
    out = np.empty(packed.shape[:-1] + (D,), np.uint8)
    for d in range(D):
        n = nibble_of(d, D, keys)
        out[..., d] = packed[..., n // 2] >> (4 * (n % 2)) & 15
    return out


def pack_codes(codes, keys):
    D = codes.shape[-1]
    out = np.zeros(codes.shape[:-1] + (D // 2,), np.uint8)
    for d in range(D):
        n = nibble_of(d, D, keys)
        out[..., n // 2] |= codes[..., d] << (4 * (n % 2))
    return out


class Cache:
    """A cache on the host: rows of codes and parameters, scattered over pages."""

    def __init__(self, rng, B, lens, Hkv, D, G, page, garbage=False, scale_v=1.0):
        self.B, self.Hkv, self.D, self.G, self.page = B, Hkv, D, G, page
        per = [max(1, -(-int(n) // page)) for n in lens]
        pages = sum(per) + 2
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((B, max(per)), -1, np.int32)
        at = 0
        for b, n in enumerate(per):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (pages, Hkv, page, D)
        off = rng.standard_normal((Hkv, 1, D)) * np.where(rng.random((Hkv, 1, D)) < 1 / 16, 6, 0.3)
        self.k = quantize4((rng.standard_normal(shape) + off).astype(np.float32), G)
        self.v = quantize4((rng.standard_normal(shape) * scale_v).astype(np.float32), G)
        self.packed = [pack_codes(self.k[0], True), pack_params(*self.k[1:]), pack_codes(self.v[0], False),
                       pack_params(*self.v[1:])]
        if garbage:  # slots past each sequence's end: NaN parameters, as in memory never written
            for b, n in enumerate(lens):
                last = self.table[b, per[b] - 1]
                used = int(n) - (per[b] - 1) * page
                for i in (1, 3):
                    self.packed[i][last, :, max(used, 0):] = 0x7FC07FC0

    def tensors(self, dev):
        c = [torch.from_numpy(a.view(np.int32) if a.dtype == np.uint32 else a).to(dev) for a in self.packed]
        return c, torch.from_numpy(self.table).to(dev)

    def rows(self, b, n):
        """Keys and values of sequence b's first n positions, 64 bits, [kv heads][n][D], and the value scales."""
        pages = self.table[b, :-(-n // self.page)] if n else self.table[b, :0]
        get = lambda a: np.swapaxes(a[pages], 0, 1).reshape(self.Hkv, -1, a.shape[-1])[:, :n]  # noqa: E731
        k, v = (dequantize4(*(get(a) for a in x)) for x in (self.k, self.v))
        return k, v, (get(self.k[1]), get(self.k[2])), (get(self.v[1]), get(self.v[2]))


def attention(cache, q, seq_lens, q_lens, causal, window, scale, dtype, fp16_rows=False):
    """(output, bound) of q fp64 [B][T][Hq][D] (the values the kernel gets).

    The bound, element by element, with p the softmax weights: the output's own rounding; probability times
    value scale rounded to fp16 (fp32: to two parts), 2^-11 (2^-21) of sum p |s c|; its underflow below 2^-24
    at a scale of 2^6 / max s, with sum p >= 1 before the division; and scores off by delta, at most 2^-20 of
    scale sum |q| (|lo| + 15 s), fp32 sums of the matrix instructions and of the groups, which moves the output
    by 2 delta sum p |v|.  fp16_rows (the kernel for long runs of queries): keys, values and probabilities
    rounded to fp16 too.
    """
    B, T, Hq, D = q.shape
    group = Hq // cache.Hkv
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    part = 2.0 ** -21 if dtype == "f32" else 2.0 ** -11
    for b in range(B):
        n = int(seq_lens[b])
        nq = min(int(q_lens[b]), T) if q_lens is not None else T
        k, v, (klo, ks), (vlo, vs) = cache.rows(b, n)
        G = cache.G
        kmag = np.repeat(np.abs(klo) + 15 * ks, G, -1).astype(np.float64)
        vmag = np.abs(v)
        scmag = np.abs(v - np.repeat(vlo.astype(np.float64), G, -1))
        smax = float(vs.max()) if n else 0.0
        for i in range(max(nq, 0)):
            pos = n - nq + i
            lo, hi = 0, n
            if causal:
                hi = min(n, pos + 1)
                lo = max(0, pos - window + 1) if window else 0
            if hi <= lo:
                continue
            for h in range(Hq):
                kv = h // group
                z = scale * (k[kv, lo:hi] @ q[b, i, h])
                delta = float(np.max(np.abs(q[b, i, h]) @ kmag[kv, lo:hi].T)) * scale * (
                    2.0 ** -20 + (2.0 ** -11 if fp16_rows else 0)) + 2.0 ** -20
                p = np.exp(z - z.max())
                p /= p.sum()
                o = p @ v[kv, lo:hi]
                a, m = p @ scmag[kv, lo:hi], p @ vmag[kv, lo:hi]
                out[b, i, h] = o
                bound[b, i, h] = (U[dtype] * np.abs(o) + part * a + 2 * delta * m + (hi - lo) * 15 * smax * 2.0 ** -29
                                  + TINY[dtype] + 2.0 ** -20 * m + (2.0 ** -10 * m if fp16_rows else 0))
    return out, bound


def quantize8(x):
    """fp32-exact per-token codes (int8) and scales (fp32) of fp32 [P][K]."""
    x = np.asarray(x, np.float32)
    amax = np.abs(x).max(1, initial=0).astype(np.float32)
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(amax[:, None] > 0, np.rint((x * np.float32(127)) / amax[:, None]), 0)
    return np.clip(c, -127, 127).astype(np.int8), amax / np.float32(127)


def linear(q, scale, wq, wscale, bias, dtype):
    """(y, bound): the integer sums are exact below 2^24; scales, their product, the sum with the bias and the
    output are rounded."""
    sums = q.astype(np.float64) @ wq.astype(np.float64).T
    y = sums * scale.astype(np.float64)[:, None] * wscale.astype(np.float64)
    b = np.zeros(wq.shape[0]) if bias is None else bias.astype(np.float64)
    total = y + b
    bound = 4 * 2.0 ** -24 * (np.abs(y) + np.abs(b)) + U[dtype] * np.abs(total) + TINY[dtype] + 1e-37
    # past 2^24 the accumulator rounds (or truncates) once per 16 products
    big = np.abs(q.astype(np.float64)) @ np.abs(wq.astype(np.float64)).T >= 2 ** 24
    grow = q.shape[1] / 16 * 2.0 ** -23 * (np.abs(q.astype(np.float64)) @ np.abs(wq.astype(np.float64)).T)
    if dtype == "f16":  # beyond fp16's largest value (and half a step)
        total = np.where(np.abs(total) >= 65520, np.copysign(np.inf, total), total)
    return total, bound + np.where(big, grow * scale.astype(np.float64)[:, None] * wscale.astype(np.float64), 0)


def check(got, want, bound, what):
    got = got.astype(np.float64)
    with np.errstate(invalid="ignore"):
        bad = ~((got == want) | (np.abs(got - want) <= bound))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{what}: {bad.sum()} of {bad.size} outside; first at {i}: got {got[i]!r} want {want[i]!r} "
                             f"bound {bound[i]!r}; worst ratio {np.nanmax(np.abs(got - want) / np.maximum(bound, 1e-300)):.3g}")


def to_type(x, dtype, dev):
    """(tensor of the type, the fp64 values it holds)."""
    t = torch.from_numpy(np.asarray(x, np.float32)).to(TYPES[dtype])
    return t.to(dev), t.double().numpy()

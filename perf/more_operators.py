"""The operators that make a whole decoder layer of the attention block, as cases that can be timed and compared.

Four operators, as a decoder served from quantized state uses them:

* rope   -- queries and keys are turned by angles that grow with their position, before keys go into the cache;
* norm   -- a block's output is normalised, gated, scaled and added to the residual stream, whose norm the next
            block reads: s = r + scale gate post(x), y = pre(s);
* linear -- y = x W^T + bias with W held in 4 bits, a scale for each group of G weights of a row;
* moe    -- a router picks `top` of E experts for each token, and their gated feed-forward layers, held in 4 bits,
            are summed by the router's weights.

Rotation.  Pair j of a head's first `rot` values (j, j + rot / 2: "half"; 2 j, 2 j + 1: "interleaved") turns by
position * freq_j, freq_j = base^(-2 j / rot), for long contexts divided by a factor where a turn takes longer than the
context that the model was trained with.  The table holds freq_j / (2 pi) in units of 2^-64, so that a position's
fraction of a turn is a product of integers.

4-bit weights [M][K] in tiles of 16 rows and 128 columns, rows and columns padded with zeros: row g + 8 r (g < 8, r < 2),
column 32 j + 8 t + i (t, j < 4, i < 8) is nibble (0 4 1 5 2 6 3 7)[i] of 32-bit word ((r 8 + g) 4 + t) 4 + j of the
tile.  Nibble n stands for n - 8; scales are bf16 [tiles of rows][tiles of columns][16][128 / G].

Inputs are what such layers meet: residual streams of unit variance with a few channels of large mean, positions up to
a long context's end, weights whose codes are normal and whose scales differ from group to group, routers whose
logits have a spread of about one.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _rope(name, B, T, Hq, Hkv, D, rot, dtype, layout="half", far=4096, factor=1.0, ragged=False, inverse=False):
    """T new tokens of B sequences that hold up to `far` tokens before them."""
    return {"name": name, "kind": "rope", "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "rot": rot, "dtype": dtype,
            "layout": layout, "far": far, "factor": factor, "ragged": ragged, "inverse": inverse}


def _norm(name, P, K, dtype, norm="rms", residual="same", post=False, gate=0, scale=1.0):
    """gate: tokens that share a row of the gate, 0 for none."""
    return {"name": name, "kind": "norm", "P": P, "K": K, "dtype": dtype, "norm": norm, "residual": residual,
            "post": post, "gate": gate, "scale": scale}


def _linear(name, P, K, M, G, dtype, bias=False):
    return {"name": name, "kind": "linear", "P": P, "K": K, "M": M, "G": G, "dtype": dtype, "bias": bias}


def _moe(name, P, K, F, E, top, G, dtype, score="softmax", renormalize=True):
    return {"name": name, "kind": "moe", "P": P, "K": K, "F": F, "E": E, "top": top, "G": G, "dtype": dtype,
            "score": score, "renormalize": renormalize}


def listed():
    return [
        # a decoding step of 32 sequences far into a long context: latency
        _rope("rope_step_b32", 32, 1, 32, 8, 128, 128, "bf16", far=131071, factor=8.0),
        # prompts of different lengths, interleaved pairs of part of an odd head size, turned back (the gradient's direction)
        _rope("rope_ragged_f32", 5, 701, 9, 3, 80, 20, "f32", layout="interleaved", far=1000, ragged=True, inverse=True),
        # long prompts, the largest rotation
        _rope("rope_prompt_8k", 4, 8192, 32, 8, 128, 128, "bf16", far=100000, factor=4.0),
        # one token between two blocks: latency
        _norm("norm_p1", 1, 4096, "bf16", post=True),
        # a ragged batch of layer norms with a gate of its own for each token, fp32 residuals, odd sizes
        _norm("norm_layer_odd_f16", 333, 1001, "f16", norm="layer", residual="f32", gate=1, scale=0.5),
        # a prompt between two blocks, a gate for each sequence: bytes
        _norm("norm_p8192", 8192, 4096, "bf16", post=True, gate=2048, scale=0.25),
        # one token through a layer
        _linear("linear_p1", 1, 4096, 4096, 64, "bf16"),
        # a few tokens, odd sizes, fp32
        _linear("linear_p19_odd_f32", 19, 1111, 999, 32, "f32", bias=True),
        # eight sequences' tokens to logits over a large vocabulary: the weights' bytes
        _linear("linear_head_p8", 8, 4096, 131072, 128, "bf16"),
        # a prompt through a layer: arithmetic bound
        _linear("linear_p2048", 2048, 4096, 4096, 64, "f16"),
        # one token, eight small experts of 64
        _moe("moe_p1", 1, 2048, 1024, 64, 8, 64, "bf16"),
        # a serving batch that reaches nearly every expert
        _moe("moe_p64", 64, 4096, 1536, 64, 6, 64, "bf16", score="sigmoid"),
    ]


def _log(rng, low, high):
    """A whole number from low to high, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["rope", "norm", "linear", "linear", "moe", "moe"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    G = rng.choice([32, 64, 64, 128])
    if kind == "rope":
        while True:
            D = rng.choice([64, 80, 96, 128, 128, 256])
            Hkv = rng.choice([1, 2, 4, 8])
            c = {"kind": "rope", "B": _log(rng, 1, 64), "T": 1 if rng.random() < 0.4 else _log(rng, 2, 8192),
                 "Hq": Hkv * rng.choice([1, 2, 3, 4, 8]), "Hkv": Hkv, "D": D, "rot": rng.choice([D, D, D // 2, 2 * (D // 5)]),
                 "dtype": dtype, "layout": rng.choice(["half", "interleaved"]), "far": _log(rng, 1, 131071),
                 "factor": rng.choice([1.0, 1.0, 2.0, 8.0]), "ragged": rng.random() < 0.5, "inverse": rng.random() < 0.25}
            if work(c)["bytes"] <= work(listed()[2])["bytes"]:
                return c
    if kind == "norm":
        while True:
            P, K = _log(rng, 1, 8192), _log(rng, 64, 16384)
            if rng.random() < 0.6:  # the usual sizes are multiples of 64
                K = -(-K // 64) * 64
            c = {"kind": "norm", "P": P, "K": K, "dtype": dtype, "norm": rng.choice(["rms", "rms", "layer"]),
                 "residual": rng.choice(["same", "same", "f32", "none"]), "post": rng.random() < 0.5,
                 "gate": rng.choice([0, 0, 1, P, rng.randint(1, P)]), "scale": rng.choice([1.0, 0.5, 0.22])}
            if work(c)["bytes"] <= work(listed()[5])["bytes"]:
                return c
    if kind == "linear":
        while True:
            c = {"kind": "linear", "P": 1 if rng.random() < 0.25 else _log(rng, 2, 2048), "K": _log(rng, 64, 16384),
                 "M": _log(rng, 64, 131072), "G": G, "dtype": dtype, "bias": rng.random() < 0.5}
            if rng.random() < 0.5:
                c["K"], c["M"] = -(-c["K"] // 64) * 64, -(-c["M"] // 64) * 64
            if c["K"] * c["M"] <= 4096 * 131072 and c["P"] * c["K"] * c["M"] <= 2048 * 4096 * 4096:
                return c
    while True:
        E = _log(rng, 2, 128)
        c = {"kind": "moe", "P": 1 if rng.random() < 0.25 else _log(rng, 2, 128), "K": _log(rng, 128, 4096),
             "F": _log(rng, 64, 4096), "E": E, "top": rng.randint(1, min(8, E)), "G": G, "dtype": dtype,
             "score": rng.choice(["softmax", "sigmoid"]), "renormalize": rng.random() < 0.5}
        if rng.random() < 0.6:
            c["K"], c["F"] = -(-c["K"] // 64) * 64, -(-c["F"] // 64) * 64
        big = listed()[-1]
        if E * c["K"] * c["F"] <= big["E"] * big["K"] * big["F"] and \
                c["P"] * c["top"] * c["K"] * c["F"] <= big["P"] * big["top"] * big["K"] * big["F"]:
            return c


# ---------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _stream(shape, g):
    """A residual stream: unit variance, one channel in 100 with a large mean."""
    mean = torch.where(torch.rand(shape[-1], generator=g, device="cuda") < 0.01, 20.0, 0.0)
    return torch.randn(shape, generator=g, device="cuda").add_(mean * torch.randn(shape[-1], generator=g, device="cuda"))


def _freqs(case, device="cuda"):
    """Radians a position of each pair, 64 bits."""
    j = torch.arange(case["rot"] // 2, dtype=torch.float64, device=device)
    f = 1e4 ** (-2 * j / case["rot"])
    if case["factor"] == 1.0:
        return f
    # turns over the trained length (4096): slow pairs are divided by the factor, fast ones stay
    keep = ((4096 * f / (2 * math.pi) - 1) / (32 - 1)).clamp(0, 1)
    return f * keep + f / case["factor"] * (1 - keep)


def _pack(n):
    """Nibbles uint8 [..., rows, columns] (whole tiles) to tiles."""
    v = n.unflatten(-1, (-1, 4, 4, 8)).unflatten(-5, (-1, 2, 8))  # [.., row tile, r, g, column tile, j, t, i]
    b = torch.stack([v[..., 0] | v[..., 2] << 4, v[..., 4] | v[..., 6] << 4, v[..., 1] | v[..., 3] << 4,
                     v[..., 5] | v[..., 7] << 4], -1)
    b = b.movedim(-4, -6)  # [.., row tile, column tile, r, g, j, t, byte]
    return b.transpose(-3, -2).flatten(-5).contiguous()  # [.., row tile, column tile, 1024]


def _unpack(p, M, K):
    """Codes of tiles [..., row tiles, column tiles, 1024] as fp32 [..., M, K]."""
    b = p.unflatten(-1, (2, 8, 4, 4, 4)).transpose(-3, -2)  # [.., row tile, column tile, r, g, j, t, byte]
    lo, hi = b & 15, b >> 4
    v = torch.stack([lo[..., 0], lo[..., 2], hi[..., 0], hi[..., 2], lo[..., 1], lo[..., 3], hi[..., 1], hi[..., 3]], -1)
    v = v.movedim(-6, -4).flatten(-4).flatten(-4, -2)  # [.., row tile, r, g, column tile, j, t, i] -> [.., rows, columns]
    return v[..., :M, :K].float() - 8


def _weights(E, M, K, G, g):
    """(codes, scales) of E matrices [M][K]; each row of K weights has a sum of squares of about one."""
    Mp, Kp = -(-M // 16) * 16, -(-K // 128) * 128
    codes = torch.full((E, Mp, Kp), 8, dtype=torch.uint8, device="cuda")
    codes[:, :M, :K] = torch.randn((E, M, K), generator=g, device="cuda").mul_(2.6).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
    s = torch.zeros((E, Mp, Kp // G), device="cuda")
    n = -(-K // G)
    s[:, :M, :n] = torch.exp(0.2 * torch.randn((E, M, n), generator=g, device="cuda")) / (2.6 * math.sqrt(K))
    s = s.to(torch.bfloat16).unflatten(1, (Mp // 16, 16)).unflatten(3, (Kp // 128, 128 // G)).transpose(2, 3).contiguous()
    return _pack(codes), s


def _dequantized(codes, scales, M, K):
    """fp32 [..., M, K]."""
    s = scales.float().transpose(-3, -2).flatten(-2).flatten(-3, -2)  # [.., rows, groups]
    G = 128 // scales.shape[-1]
    return _unpack(codes, M, K) * s[..., :M, :].repeat_interleave(G, -1)[..., :K]


def prepare(case, seed):
    g = _gen(seed)
    dt = DTYPES[case["dtype"]]
    st = {"case": case}
    if case["kind"] == "rope":
        B, T, D = case["B"], case["T"], case["D"]
        # the projections' output, as attention gets it: queries, keys, values of a token beside one another
        heads = case["Hq"] + case["Hkv"]
        st["x"] = torch.randn((B, T, heads + case["Hkv"], D), generator=g, device="cuda").to(dt)[:, :, :heads]
        r = torch.Generator()
        r.manual_seed(seed)
        st["starts"] = torch.randint(0, case["far"] + 1, (B,), generator=r).to(torch.int32).cuda()
        st["lens"] = None
        if case["ragged"]:
            st["lens"] = torch.randint(0, T + 1, (B,), generator=r).to(torch.int32).cuda()
        st["table"] = torch.round(_freqs(case) / (2 * math.pi) * 2.0 ** 64).to(torch.int64)
        return st
    if case["kind"] == "norm":
        P, K = case["P"], case["K"]
        st["x"] = _stream((P, K), g).to(dt)
        st["r"] = None if case["residual"] == "none" else \
            (3 * _stream((P, K), g)).to(dt if case["residual"] == "same" else torch.float32)
        st["gate"] = None
        if case["gate"]:
            rows = -(-P // case["gate"])
            st["gate"] = torch.sigmoid(torch.randn((rows, K), generator=g, device="cuda")).to(dt)
        for w in ("post", "pre"):
            st[w + "_w"] = 1 + 0.2 * torch.randn(K, generator=g, device="cuda")
            st[w + "_b"] = 0.1 * torch.randn(K, generator=g, device="cuda") if case["norm"] == "layer" else None
        return st
    if case["kind"] == "linear":
        st["x"] = torch.randn((case["P"], case["K"]), generator=g, device="cuda").to(dt)
        codes, scales = _weights(1, case["M"], case["K"], case["G"], g)
        st["codes"], st["scales"] = codes[0], scales[0]
        st["bias"] = torch.randn(case["M"], generator=g, device="cuda") if case["bias"] else None
        return st
    P, K, F, E, G = (case[n] for n in ("P", "K", "F", "E", "G"))
    st["x"] = torch.randn((P, K), generator=g, device="cuda").to(dt)
    st["router"] = (torch.randn((E, K), generator=g, device="cuda") / math.sqrt(K)).to(dt)
    for name, M, N in (("gate", F, K), ("up", F, K), ("down", K, F)):
        st[name + "_codes"], st[name + "_scales"] = _weights(E, M, N, G, g)
    return st


# ---------------------------------------------------------------------------- one pass

def _plain_rope(st):
    case = st["case"]
    x, rot, T = st["x"].float(), case["rot"], case["T"]
    i = torch.arange(T, device="cuda")
    pos = st["starts"].double()[:, None] + i  # [B, T]
    angle = (2 * math.pi) * pos[..., None] * (st["table"].double() * 2.0 ** -64)
    if case["inverse"]:
        angle = -angle
    if st["lens"] is not None:
        angle = torch.where((i < st["lens"][:, None])[..., None], angle, 0.0)
    c, s = torch.cos(angle).float()[:, :, None], torch.sin(angle).float()[:, :, None]
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    return torch.cat([turned, x[..., rot:]], -1).to(st["x"].dtype)


def _plain_normed(z, w, b, layer):
    if layer:
        z = z - z.mean(-1, keepdim=True)
    y = z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-5) * w
    return y if b is None else y + b


def _plain_norm(st):
    case = st["case"]
    layer = case["norm"] == "layer"
    u = st["x"].float()
    if case["post"]:
        u = _plain_normed(u, st["post_w"], st["post_b"], layer)
    if st["gate"] is not None:
        u = u * st["gate"].float().repeat_interleave(case["gate"], 0)[:case["P"]]
    s = u * case["scale"]
    if st["r"] is not None:
        s = s + st["r"].float()
    y = _plain_normed(s, st["pre_w"], st["pre_b"], layer)
    return {"residual": s.to(st["x"].dtype if st["r"] is None else st["r"].dtype), "y": y.to(st["x"].dtype)}


def _plain_linear(st):
    case = st["case"]
    y = torch.matmul(st["x"].float(), _dequantized(st["codes"], st["scales"], case["M"], case["K"]).t())
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(st["x"].dtype)


def _plain_route(st):
    """(experts, weights) [P, top]; equal logits: the lowest index first."""
    case = st["case"]
    logits = torch.matmul(st["x"].double(), st["router"].double().t())  # 64 bits: experts next to the border
    best, ids = torch.sort(logits, dim=1, descending=True, stable=True)
    best, ids = best[:, :case["top"]], ids[:, :case["top"]]
    if case["score"] == "softmax":
        top = logits.amax(1, keepdim=True)
        g = torch.exp(best - top)
        total = g.sum(1, keepdim=True) if case["renormalize"] else torch.exp(logits - top).sum(1, keepdim=True)
        g = g / total
    else:
        g = 1 / (1 + torch.exp(-best))
        if case["renormalize"]:
            g = g / g.sum(1, keepdim=True)
    return ids, g.float()


def _plain_moe(st):
    case = st["case"]
    P, K, F, E, top = (case[n] for n in ("P", "K", "F", "E", "top"))
    ids, g = _plain_route(st)
    x = st["x"].float()
    if P * top < E:  # the chosen experts' weights, one set for each token and place
        pick = lambda n, M, N: _dequantized(st[n + "_codes"][ids.flatten()], st[n + "_scales"][ids.flatten()], M, N)  # noqa: E731
        xs = x.repeat_interleave(top, 0)[:, :, None]
        a, b = torch.matmul(pick("gate", F, K), xs), torch.matmul(pick("up", F, K), xs)
        h = a / (1 + torch.exp(-a)) * b
        y = torch.matmul(pick("down", K, F), h)[..., 0].view(P, top, K)
        return (y * g[..., None]).sum(1).to(st["x"].dtype)
    all_of = lambda n, M, N: _dequantized(st[n + "_codes"], st[n + "_scales"], M, N).transpose(1, 2)  # noqa: E731
    weight = torch.zeros((P, E), device="cuda").scatter_(1, ids, g)
    a, b = torch.matmul(x, all_of("gate", F, K)), torch.matmul(x, all_of("up", F, K))  # [E, P, F]
    h = a / (1 + torch.exp(-a)) * b
    y = torch.matmul(h, all_of("down", K, F)) * weight.t()[..., None]
    return y.sum(0).to(st["x"].dtype)


def run(st):
    case = st["case"]
    if not own:
        return {"rope": _plain_rope, "norm": _plain_norm, "linear": _plain_linear, "moe": _plain_moe}[case["kind"]](st)
    from paper_1705_01462_gb300 import fgq
    if case["kind"] == "rope":
        return fgq.fgq_rope(st["x"], st["table"], st["starts"], lens=st["lens"], layout=case["layout"],
                            inverse=case["inverse"])
    if case["kind"] == "norm":
        pre = fgq.Norm(st["pre_w"], st["pre_b"], kind=case["norm"], eps=1e-5)
        post = fgq.Norm(st["post_w"], st["post_b"], kind=case["norm"], eps=1e-5) if case["post"] else None
        s, y = fgq.fgq_add_norm(st["x"], st["r"], pre, post=post, gate=st["gate"], tokens_per_gate=case["gate"],
                                scale=case["scale"])
        return {"residual": s, "y": y}
    if case["kind"] == "linear":
        return fgq.fgq_linear_w4(st["x"], fgq.W4Weights(st["codes"], st["scales"], case["M"], case["K"]),
                                 bias=st["bias"])
    K, F = case["K"], case["F"]
    w = [fgq.W4Weights(st[n + "_codes"], st[n + "_scales"], M, N)
         for n, M, N in (("gate", F, K), ("up", F, K), ("down", K, F))]
    return fgq.fgq_moe_w4(st["x"], st["router"], case["top"], *w, score=case["score"], renormalize=case["renormalize"])


# ---------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = BYTES[case["dtype"]]
    if case["kind"] == "rope":
        n = case["B"] * case["T"] * (case["Hq"] + case["Hkv"])
        return {"bytes": 2 * n * case["D"] * e + 4 * case["rot"] + 4 * case["B"], "flops": 3 * n * case["rot"]}
    if case["kind"] == "norm":
        n = case["P"] * case["K"]
        r = 4 if case["residual"] == "f32" else e
        rows = -(-case["P"] // case["gate"]) if case["gate"] else 0
        return {"bytes": n * 2 * e + n * r * (1 if case["residual"] == "none" else 2) + rows * case["K"] * e +
                4 * case["K"] * (2 if case["post"] else 1), "flops": 8 * n}
    P, K, G = case["P"], case["K"], case["G"]

    def weights(M, N):
        return M * N / 2 + 2 * M * -(-N // G)

    if case["kind"] == "linear":
        M = case["M"]
        return {"bytes": P * (K + M) * e + weights(M, K) + (4 * M if case["bias"] else 0), "flops": 2 * P * K * M}
    F, E, top = case["F"], case["E"], case["top"]
    reached = E * (1 - (1 - top / E) ** P)  # experts that some token picks, on average
    return {"bytes": P * 2 * K * e + E * K * e + reached * (2 * weights(F, K) + weights(K, F)),
            "flops": 2 * P * E * K + 6 * P * top * K * F}


# ---------------------------------------------------------------------------- the definitions in 64 bits

def _exact_weights(codes, scales, M, K):
    """fp64 [M][K] of one matrix, column by column of the layout's definition."""
    rows = torch.arange(M, device="cuda")
    cols = torch.arange(K, device="cuda")
    r, g = rows % 16 // 8, rows % 8
    j, t, i = cols % 128 // 32, cols % 32 // 8, cols % 8
    nibble = torch.tensor([0, 4, 1, 5, 2, 6, 3, 7], device="cuda")[i]
    byte = (((r * 8 + g)[:, None] * 4 + t) * 4 + j) * 4 + nibble // 2
    at = ((rows // 16)[:, None] * codes.shape[1] + cols // 128) * 1024 + byte
    n = codes.reshape(-1)[at] >> (4 * (nibble % 2)).to(torch.uint8) & 15
    per = scales.shape[-1]
    sat = (((rows // 16)[:, None] * codes.shape[1] + cols // 128) * 16 + (rows % 16)[:, None]) * per + cols % 128 * per // 128
    return (n.double() - 8) * scales.reshape(-1)[sat].double()


def _exact_normed(z, w, b, kind):
    if kind == "layer":
        z = z - z.mean(1, keepdim=True)
    y = z * torch.rsqrt(z.square().mean(1, keepdim=True) + 1e-5) * w.double()
    return y if b is None else y + b.double()


def exact(case, seed):
    st = prepare(case, seed)
    x = st["x"].double()
    if case["kind"] == "rope":
        out = x.clone()
        rot = case["rot"]
        f = _freqs(case)
        for b in range(case["B"]):
            n = case["T"] if st["lens"] is None else int(st["lens"][b])
            turn = (int(st["starts"][b]) + torch.arange(n, device="cuda", dtype=torch.float64))[:, None, None] * f
            z = torch.polar(torch.ones_like(turn), -turn if case["inverse"] else turn)
            first = slice(0, rot // 2) if case["layout"] == "half" else slice(0, rot, 2)
            second = slice(rot // 2, rot) if case["layout"] == "half" else slice(1, rot, 2)
            v = torch.complex(x[b, :n, :, first].contiguous(), x[b, :n, :, second].contiguous()) * z
            out[b, :n, :, first], out[b, :n, :, second] = v.real, v.imag
        return out
    if case["kind"] == "norm":
        u = _exact_normed(x, st["post_w"], st["post_b"], case["norm"]) if case["post"] else x
        if st["gate"] is not None:
            u = u * st["gate"].double()[torch.arange(case["P"], device="cuda") // case["gate"]]
        s = case["scale"] * u + (0 if st["r"] is None else st["r"].double())
        return {"residual": s, "y": _exact_normed(s, st["pre_w"], st["pre_b"], case["norm"])}
    if case["kind"] == "linear":
        M, step = case["M"], 4096
        y = torch.empty((case["P"], M), dtype=torch.float64, device="cuda")
        for m in range(0, M, step):  # whole tiles of rows
            n = min(step, M - m)
            w = _exact_weights(st["codes"][m // 16:(m + step) // 16].contiguous(),
                               st["scales"][m // 16:(m + step) // 16].contiguous(), n, case["K"])
            y[:, m:m + n] = torch.einsum("pk,mk->pm", x, w)
        return y if st["bias"] is None else y + st["bias"].double()
    K, F = case["K"], case["F"]
    logits = torch.einsum("pk,ek->pe", x, st["router"].double())
    score = torch.softmax(logits, 1) if case["score"] == "softmax" else torch.sigmoid(logits)
    y = torch.zeros_like(x)
    chosen = [sorted(range(case["E"]), key=lambda e: (-row[e], e))[:case["top"]] for row in logits.tolist()]
    picked = torch.zeros_like(score, dtype=torch.bool)
    for p, es in enumerate(chosen):
        picked[p, es] = True
    weight = torch.where(picked, score, 0.0)
    if case["renormalize"]:
        weight = weight / weight.sum(1, keepdim=True)
    for e in range(case["E"]):
        p = torch.nonzero(picked[:, e])[:, 0]
        if not p.numel():
            continue
        wg, wu, wd = (_exact_weights(st[n + "_codes"][e], st[n + "_scales"][e], M, N)
                      for n, M, N in (("gate", F, K), ("up", F, K), ("down", K, F)))
        a = x[p] @ wg.t()
        y[p] += weight[p, e, None] * ((a * torch.sigmoid(a) * (x[p] @ wu.t())) @ wd.t())
    return y

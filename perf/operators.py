"""The language-model operators of this library as cases that can be timed and compared.

Three operators, as a decoder served from quantized state uses them:

* append    -- new keys and values are quantized to 4 bits as they are written into a paged cache, and read
               back as the values that they now stand for;
* attention -- queries attend to a paged cache held in 4 bits: one new token per sequence (decoding), a few
               (verifying a draft), or a long run of them (the prompt, or a chunk of it);
* linear    -- y = x W^T + bias with 8-bit integers: x quantized with a scale for each token, W held with a
               scale for each output channel.

The cache.  Keys and values are uint8 [pages][kv heads][page size][D / 2] (two codes a byte) with int32
parameters [pages][kv heads][page size][D / G]: a group of G consecutive values of one token and head holds
lo (bf16, high 16 bits) and s (bf16, low 16 bits), and code c stands for lo + s c.  lo is the group's
minimum rounded down, s = (max - lo) / 15 rounded up, c = (x - lo) / s rounded half to even, so that the
sixteen values span the group.  Within a row the codes of 32-value blocks j interleave: word (t, j) of a key
row (t = 0..3) holds values 32 j + 8 t + 0..7 in nibbles 0 4 1 5 2 6 3 7; 16-bit unit (g, j) of a value row
(g = 0..7) holds values 32 j + 4 g + 0..3 in nibble order.
Position p of sequence b lies in page page_table[b][p / page size]; unused table entries are -1.

Inputs follow what projections of normalised states give: values of unit variance, keys with a few channels
of large mean, queries so scaled that the softmax neither flattens nor picks a single token.  Weights are
normal, quantized to 8 bits with a power-of-two scale per channel.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _append(name, B, T, Hkv, D, G, page, dtype, ragged=False, before=0):
    return {"name": name, "kind": "append", "B": B, "T": T, "Hkv": Hkv, "D": D, "G": G, "page": page, "dtype": dtype,
            "ragged": ragged, "before": before}


def _attention(name, B, T, Hq, Hkv, D, G, page, dtype, low, high, window=0):
    """T new tokens per sequence (already in the cache), lengths from low to high, the longest being high."""
    return {"name": name, "kind": "attention", "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "G": G, "page": page,
            "dtype": dtype, "low": low, "high": high, "window": window}


def _linear(name, P, K, M, dtype, bias=False):
    return {"name": name, "kind": "linear", "P": P, "K": K, "M": M, "dtype": dtype, "bias": bias}


def listed():
    return [
        # a decoding step of 32 sequences: one token each, where the call itself costs most
        _append("append_step_b32", 32, 1, 8, 128, 64, 64, "bf16", before=700),
        # prompts of different lengths in one call, small pages and groups
        _append("append_ragged_f16", 6, 1531, 4, 64, 32, 16, "f16", ragged=True, before=37),
        # long prompts, the largest write
        _append("append_prompt_8k", 4, 8192, 8, 128, 64, 64, "bf16"),
        # one interactive user, a short context: latency
        _attention("decode_b1_short", 1, 1, 32, 8, 128, 64, 64, "bf16", 700, 700),
        # a full serving batch, contexts of very different lengths: the cache is read once
        _attention("decode_b64_ragged", 64, 1, 32, 8, 128, 64, 64, "bf16", 2048, 16384),
        # one very long context: few rows, all of the work along the cache
        _attention("decode_b1_128k", 1, 1, 64, 8, 128, 128, 128, "bf16", 131071, 131071),
        # a few drafted tokens verified at once, sliding window, large heads
        _attention("verify_window_d256", 8, 6, 24, 4, 256, 64, 32, "f16", 900, 9001, window=4096),
        # fp32 inputs and outputs, every query head with keys of its own, small heads
        _attention("decode_f32_mha", 3, 2, 12, 12, 64, 32, 16, "f32", 33, 3001),
        # a chunk of each of two prompts over what the cache already holds: arithmetic bound
        _attention("prompt_chunk_1k", 2, 1024, 32, 8, 128, 64, 64, "bf16", 4096, 6144),
        # one token through a fully connected layer: the weights are read once
        _linear("linear_p1", 1, 4096, 4096, "bf16"),
        # a small batch, odd sizes, fp32
        _linear("linear_p77_odd_f32", 77, 2751, 1003, "f32", bias=True),
        # a prompt through a fully connected layer: arithmetic bound
        _linear("linear_p4096", 4096, 4096, 8192, "bf16"),
    ]


def _log(rng, low, high):
    """A whole number from low to high, spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["append", "attention", "attention", "linear"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if kind == "linear":
        while True:
            c = {"kind": "linear", "P": _log(rng, 1, 4096), "K": _log(rng, 64, 9216), "M": _log(rng, 64, 9216),
                 "dtype": dtype, "bias": rng.random() < 0.5}
            if rng.random() < 0.5:  # the usual sizes are multiples of 64
                c["K"], c["M"] = -(-c["K"] // 64) * 64, -(-c["M"] // 64) * 64
            if c["P"] * c["K"] * c["M"] <= 4096 * 4096 * 8192 and 3072 not in c.values():
                return c
    D = rng.choice([64, 128, 128, 256])
    G = rng.choice([g for g in (32, 64, 128) if g <= D])
    page = rng.choice([16, 32, 48, 64, 128, 256])
    Hkv = rng.choice([1, 2, 4, 8, 8])
    if kind == "append":
        while True:
            c = {"kind": "append", "B": _log(rng, 1, 64), "T": _log(rng, 1, 8192), "Hkv": Hkv, "D": D, "G": G,
                 "page": page, "dtype": dtype, "ragged": rng.random() < 0.5, "before": rng.choice([0, rng.randint(1, 4000)])}
            if c["B"] * c["T"] * Hkv * D * BYTES[dtype] <= 4 * 8192 * 8 * 128 * 2 and 3072 not in c.values():
                return c
    while True:
        high = _log(rng, 64, 131071)
        T = 1 if rng.random() < 0.5 else _log(rng, 2, 1024)
        c = {"kind": "attention", "B": _log(rng, 1, 64), "T": min(T, high), "Hq": Hkv * rng.choice([1, 2, 4, 6, 8]),
             "Hkv": Hkv, "D": D, "G": G, "page": page, "dtype": dtype, "low": max(1, int(high * rng.uniform(0.05, 1))),
             "high": high, "window": rng.choice([0, 0, 0, _log(rng, 16, 8192)])}
        rows = c["B"] * c["T"] * c["Hq"]
        if (c["B"] * high * Hkv * D <= 64 * 16384 * 8 * 128 and rows * high * D <= 2 * 1024 * 32 * 6144 * 128
                and 3072 not in c.values()):
            return c


# ---------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _lens(case, seed):
    """The sequences' lengths, on the host as a scheduler has them; the longest is the case's."""
    r = torch.Generator()
    r.manual_seed(seed)
    B = case["B"]
    if case["kind"] == "append":
        n = torch.randint(1, case["T"] + 1, (B,), generator=r) if case["ragged"] else torch.full((B,), case["T"])
        n[B // 2] = case["T"]
    else:
        n = torch.randint(case["low"], case["high"] + 1, (B,), generator=r)
        n[B // 2] = case["high"]
    return n.to(torch.int32)


def _table(case, longest, seed):
    """A page table whose pages are scattered over the pool, entries past each sequence's last page -1."""
    per = [-(-int(n) // case["page"]) for n in longest]
    pages = sum(per) + 3
    r = torch.Generator()
    r.manual_seed(seed + 1)
    order = torch.randperm(pages, generator=r).to(torch.int32)
    table = torch.full((len(per), max(per)), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    return table, pages


def _keys(shape, g, offsets):
    return torch.randn(shape, generator=g, device="cuda").add_(offsets)


def _offsets(case, g):
    """Means of the key channels: one in 32 is large, as in trained models."""
    D = case["D"]
    o = torch.randn((case["Hkv"], D), generator=g, device="cuda") * 0.3
    big = torch.rand((case["Hkv"], D), generator=g, device="cuda") < 1 / 32
    return torch.where(big, o * 12, o)


def _quantize4(x, G):
    """Codes (uint8) and parameters (int32) of fp32 values [..., D]."""
    D = x.shape[-1]
    x = x.unflatten(-1, (D // G, G))
    lo = x.amin(-1)
    bits = lo.view(torch.int32)
    down = torch.where(bits < 0, (bits + 0xFFFF) & -65536, bits & -65536)
    lo = down.view(torch.float32)
    d = x.amax(-1) - lo
    s = d / torch.full_like(d, 15)  # by a tensor: a division by a number is a product with its rounded reciprocal
    s = ((s.view(torch.int32) + 0xFFFF) & -65536).view(torch.float32)
    c = torch.where(s[..., None] > 0, torch.round((x - lo[..., None]) / s[..., None]), 0.0).clamp_(0, 15)
    par = (lo.view(torch.int32) & -65536) | ((s.view(torch.int32) >> 16) & 0xFFFF)
    return c.flatten(-2).to(torch.uint8), par


def _pack_k(c):
    n = c.unflatten(-1, (c.shape[-1] // 32, 4, 8))  # [.., j, t, i]
    b = torch.stack([n[..., 0] | n[..., 2] << 4, n[..., 4] | n[..., 6] << 4, n[..., 1] | n[..., 3] << 4,
                     n[..., 5] | n[..., 7] << 4], -1)
    return b.transpose(-3, -2).flatten(-3).contiguous()


def _pack_v(c):
    n = c.unflatten(-1, (c.shape[-1] // 32, 8, 4))  # [.., j, g, i]
    b = torch.stack([n[..., 0] | n[..., 1] << 4, n[..., 2] | n[..., 3] << 4], -1)
    return b.transpose(-3, -2).flatten(-3).contiguous()


def _unpack_k(b):
    n = b.unflatten(-1, (4, b.shape[-1] // 16, 4)).transpose(-3, -2)  # [.., j, t, byte]
    l, h = n & 15, n >> 4
    return torch.stack([l[..., 0], l[..., 2], h[..., 0], h[..., 2], l[..., 1], l[..., 3], h[..., 1], h[..., 3]],
                       -1).flatten(-3)


def _unpack_v(b):
    n = b.unflatten(-1, (8, b.shape[-1] // 16, 2)).transpose(-3, -2)  # [.., j, g, byte]
    return torch.stack([n & 15, n >> 4], -1).flatten(-4)


def _values(codes, par):
    """fp32 values of unpacked codes [..., D] with parameters [..., D / G]."""
    D, n = codes.shape[-1], par.shape[-1]
    c = codes.float().unflatten(-1, (n, D // n))
    lo, s = (par & -65536).view(torch.float32), (par << 16).view(torch.float32)
    return (lo[..., None] + s[..., None] * c).flatten(-2)


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] == "linear":
        P, K, M = case["P"], case["K"], case["M"]
        x = torch.randn((P, K), generator=g, device="cuda").to(DTYPES[case["dtype"]])
        w = torch.randn((M, K), generator=g, device="cuda") / math.sqrt(K)
        # int8 codes with a power-of-two scale per channel that covers its largest weight
        e = torch.ceil(torch.log2(w.abs().amax(1) / 127))
        ws = torch.exp2(e)
        wq = torch.round(w / ws[:, None]).clamp_(-127, 127).to(torch.int8)
        bias = torch.randn(M, generator=g, device="cuda") if case["bias"] else None
        return {"case": case, "x": x, "wq": wq, "wscale": ws, "bias": bias}
    B, Hkv, D, G, ps = case["B"], case["Hkv"], case["D"], case["G"], case["page"]
    n = _lens(case, seed)
    off = _offsets(case, g)
    if case["kind"] == "append":
        starts = torch.full((B,), case["before"], dtype=torch.int32)
        table, pages = _table(case, (starts + n).tolist(), seed)
        shape = (pages, Hkv, ps)
        st = {"case": case, "table": table.cuda(), "starts": starts.cuda(), "lens": n.cuda() if case["ragged"] else None}
        dt = DTYPES[case["dtype"]]
        st["k"] = _keys((B, case["T"], Hkv, D), g, off).to(dt)
        st["v"] = torch.randn((B, case["T"], Hkv, D), generator=g, device="cuda").to(dt)
        for w in "kv":
            st[w + "_codes"] = torch.zeros(shape + (D // 2,), dtype=torch.uint8, device="cuda")
            st[w + "_params"] = torch.zeros(shape + (D // G,), dtype=torch.int32, device="cuda")
        return st
    table, pages = _table(case, n.tolist(), seed)
    st = {"case": case, "table": table.cuda(), "lens": n.cuda()}
    for w, pack in (("k", _pack_k), ("v", _pack_v)):
        x = torch.randn((pages, Hkv, ps, D), generator=g, device="cuda")
        if w == "k":
            x += off[:, None, :]
        c, st[w + "_params"] = _quantize4(x, G)
        del x
        st[w + "_codes"] = pack(c)
        del c
    q = torch.randn((B, case["T"], case["Hq"], D), generator=g, device="cuda") * 1.5
    st["q"] = q.to(DTYPES[case["dtype"]])
    return st


# ---------------------------------------------------------------------------- one pass

def _rows(st, positions):
    """Row of every position [B, n] in the cache's [pages * kv heads * page size] rows: [B, kv heads, n]."""
    case = st["case"]
    ps, Hkv = case["page"], case["Hkv"]
    page = torch.gather(st["table"].long(), 1, (positions // ps).clamp_(0, st["table"].shape[1] - 1)).clamp_(min=0)
    heads = torch.arange(Hkv, device="cuda")
    return (page[:, None, :] * Hkv + heads[None, :, None]) * ps + (positions % ps)[:, None, :]


def _plain_append(st):
    case = st["case"]
    B, T, D, G = case["B"], case["T"], case["D"], case["G"]
    i = torch.arange(T, device="cuda")[None, :].expand(B, T)
    rows = _rows(st, st["starts"].long()[:, None] + i)  # [B, Hkv, T]
    live = torch.ones_like(rows, dtype=torch.bool) if st["lens"] is None else \
        (i < st["lens"][:, None])[:, None, :].expand_as(rows)
    out = {}
    for w, pack, unpack in (("k", _pack_k, _unpack_k), ("v", _pack_v, _unpack_v)):
        codes, par = _quantize4(st[w].float().transpose(1, 2).contiguous(), G)  # [B, Hkv, T, .]
        st[w + "_codes"].view(-1, D // 2)[rows[live]] = pack(codes)[live]
        st[w + "_params"].view(-1, D // G)[rows[live]] = par[live]
        back = _values(unpack(st[w + "_codes"].view(-1, D // 2)[rows]), st[w + "_params"].view(-1, D // G)[rows])
        out[w] = torch.where(live[..., None], back, 0.0).transpose(1, 2).to(st[w].dtype).contiguous()
    return out


def _plain_attention(st):
    case = st["case"]
    B, T, Hq, Hkv, D, G = (case[x] for x in ("B", "T", "Hq", "Hkv", "D", "G"))
    S, group = case["high"], Hq // Hkv
    at = torch.arange(S, device="cuda")
    rows = _rows(st, at[None, :].expand(B, S))
    k = _values(_unpack_k(st["k_codes"].view(-1, D // 2)[rows]), st["k_params"].view(-1, D // G)[rows])
    q = st["q"].float().view(B, T, Hkv, group, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, group * T, D)
    s = torch.matmul(q, k.transpose(-1, -2)).view(B, Hkv, group, T, S) / math.sqrt(D)
    del k
    qpos = st["lens"].long()[:, None] - T + torch.arange(T, device="cuda")  # [B, T]
    seen = (at[None, None, :] <= qpos[..., None]) & (qpos[..., None] >= 0)
    if case["window"]:
        seen &= at[None, None, :] > qpos[..., None] - case["window"]
    s = s.masked_fill_(~seen[:, None, None], float("-inf"))
    m = s.amax(-1, keepdim=True).clamp_(min=-1e30)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    v = _values(_unpack_v(st["v_codes"].view(-1, D // 2)[rows]), st["v_params"].view(-1, D // G)[rows])
    o = torch.matmul(p.view(B, Hkv, group * T, S), v).view(B, Hkv, group, T, D)
    o = torch.where(total > 0, o / total, 0.0)
    return o.permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D).to(st["q"].dtype)


def _plain_linear(st):
    x = st["x"].float()
    amax = x.abs().amax(1, keepdim=True)
    q = torch.round(x * 127 / amax)
    y = torch.matmul(q, st["wq"].float().t()) * (amax / torch.full_like(amax, 127)) * st["wscale"]
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(st["x"].dtype)


def run(st):
    case = st["case"]
    if not own:
        return {"append": _plain_append, "attention": _plain_attention, "linear": _plain_linear}[case["kind"]](st)
    from paper_1705_01462_gb300 import fgq
    if case["kind"] == "linear":
        return fgq.fgq_linear_w8a8(st["x"], st["wq"], st["wscale"], bias=st["bias"])
    cache = fgq.KVCache(st["k_codes"], st["k_params"], st["v_codes"], st["v_params"])
    if case["kind"] == "append":
        fgq.fgq_kv_append(cache, st["k"], st["v"], st["table"], st["starts"], lens=st["lens"])
        k, v = fgq.fgq_kv_read(cache, st["table"], st["starts"], case["T"], lens=st["lens"], dtype=st["k"].dtype)
        return {"k": k, "v": v}
    return fgq.fgq_kv_attention(st["q"], cache, st["table"], st["lens"], causal=True, window=case["window"],
                                max_len=case["high"])


# ---------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e = BYTES[case["dtype"]]
    if case["kind"] == "linear":
        P, K, M = case["P"], case["K"], case["M"]
        return {"bytes": P * K * e + M * K + 4 * M * (2 if case["bias"] else 1) + P * M * e, "flops": 2 * P * K * M}
    B, Hkv, D, G = case["B"], case["Hkv"], case["D"], case["G"]
    row = 2 * (D // 2 + 4 * (D // G))  # a token of one head in the cache: codes and parameters, keys and values
    # lengths are spread evenly, and the longest is given: what the cases' seeds give on average
    if case["kind"] == "append":
        tokens = B * case["T"] if not case["ragged"] else case["T"] + (B - 1) * (case["T"] + 1) / 2
        return {"bytes": Hkv * (tokens * (2 * D * e + row) + B * case["T"] * 2 * D * e), "flops": 0}
    T, Hq = case["T"], case["Hq"]
    read = pairs = 0
    for n, share in ((case["high"], 1), ((case["high"] + case["low"]) / 2, B - 1)):
        first = n - T  # position of the first query
        w = case["window"] or n
        read += share * min(n, T + w - 1)
        pairs += share * sum(min(max(first + (i + 0.5) * T / 8 + 0.5, 0), w) for i in range(8)) * T / 8
    return {"bytes": B * T * Hq * D * 2 * e + Hkv * read * row, "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------- the definitions in 64 bits

def _exact_codes(packed, of_keys):
    """Unpacked codes, value by value of the layout's definition."""
    D = 2 * packed.shape[-1]
    out = torch.empty(packed.shape[:-1] + (D,), dtype=torch.float64, device=packed.device)
    for d in range(D):
        j, r = divmod(d, 32)
        if of_keys:
            t, i = divmod(r, 8)
            nibble = 8 * (t * (D // 32) + j) + (0, 4, 1, 5, 2, 6, 3, 7)[i]
        else:
            t, i = divmod(r, 4)
            nibble = 4 * (t * (D // 32) + j) + i
        out[..., d] = ((packed[..., nibble // 2] >> (4 * (nibble % 2))) & 15).double()
    return out


def _exact_values(codes, par, G):
    lo = (par >> 16 << 16).view(torch.float32).double().repeat_interleave(G, -1)
    s = (par << 16).view(torch.float32).double().repeat_interleave(G, -1)
    return lo + s * codes


def _round_bf16(x, up):
    """64-bit x to the next value of 8 significant bits at or above it (up) or at or below it."""
    whole = x.view(torch.int64) & -(1 << 45)  # the low 45 of 52 fraction bits away: towards zero
    near = whole.view(torch.float64)
    far = (whole + (1 << 45)).view(torch.float64)
    return torch.where(near == x, x, torch.where((x > 0) == up, far, near))


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "linear":
        x = st["x"].double()
        amax = x.abs().amax(1)
        q = torch.round(127 * x / amax[:, None])
        y = torch.einsum("pk,mk->pm", q, st["wq"].double()) * amax[:, None] * st["wscale"].double() / 127
        return y if st["bias"] is None else y + st["bias"].double()
    if case["kind"] == "append":
        out = {}
        for w in "kv":
            x = st[w].double()
            groups = x.reshape(x.shape[:-1] + (-1, case["G"]))
            lo = _round_bf16(groups.min(-1, keepdim=True).values.contiguous(), up=False)
            s = _round_bf16((groups.max(-1, keepdim=True).values - lo) / 15, up=True)
            back = (lo + s * torch.round((groups - lo) / s).clamp(0, 15)).reshape(x.shape)
            if st["lens"] is not None:
                for b, n in enumerate(st["lens"].tolist()):
                    back[b, n:] = 0
            out[w] = back
        return out
    T, D, G, ps, W = case["T"], case["D"], case["G"], case["page"], case["window"]
    if case["B"] * T * case["Hq"] * case["high"] * D > 2e12:
        return None
    group = case["Hq"] // case["Hkv"]
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(st["lens"].tolist()):
        pages = st["table"][b, :-(-n // ps)].long()
        kb, vb = (_exact_values(_exact_codes(st[w + "_codes"][pages], w == "k"), st[w + "_params"][pages], G)
                  for w in "kv")
        for i0 in range(0, T, 256):
            i1 = min(T, i0 + 256)
            at = n - T + torch.arange(i0, i1, device="cuda")
            pos = torch.arange(n, device="cuda")
            seen = pos[None, :] <= at[:, None]
            if W:
                seen &= pos[None, :] > at[:, None] - W
            for h in range(case["Hkv"]):
                k, v = (x[:, h].reshape(-1, D)[:n] for x in (kb, vb))
                qh = st["q"][b, i0:i1, h * group:(h + 1) * group].double()
                z = torch.einsum("thd,sd->ths", qh, k) / math.sqrt(D)
                z = z.masked_fill(~seen[:, None, :], -math.inf)
                p = torch.nan_to_num(torch.softmax(z, -1))
                o[b, i0:i1, h * group:(h + 1) * group] = torch.einsum("ths,sd->thd", p, v)
    return o

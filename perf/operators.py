"""Serving operators in 4 bits and with grouped heads: what they compute in plain torch, and the library's calls for the same.

The kinds of case (`op`):
  quantize      rows to microscaled 4 bits and back to the values they stand for
  linear        rows and weights in 4 bits: y = act(x W^T + b) with a residual or a gate (prompts)
  linear_few    bfloat16 rows of a decode step, weights in 4 bits
  cache_store   keys and values of prompts (or of single tokens) into a paged cache in 4 bits, and the values it then holds
  cache_decode  one decode step over such a cache with grouped heads and the conditional append
  prefill       causal attention of packed prompts with grouped heads
"""
import math

import torch

own = False
DEV = "cuda"
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # the magnitudes of a 4-bit element (sign, 2 exponent bits, 1 mantissa bit)


# ---- cases ------------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # a feed-forward matrix of the 7B decoder, laid out once when a model is loaded
        {"name": "quantize 11008x4096", "op": "quantize", "M": 11008, "K": 4096, "dtype": "bf16"},
        # a short float32 batch of odd sizes: latency
        {"name": "quantize 77x1376 f32", "op": "quantize", "M": 77, "K": 1376, "dtype": "f32"},
        # the gated feed-forward product of 16 reduced prompts through a 7B layer (odd number of rows)
        {"name": "linear 5003x4096x11008", "op": "linear", "M": 5003, "K": 4096, "N": 11008, "act": 2, "bias": False},
        # one short prompt through a narrow layer with bias and GELU, K not a multiple of the kernel's step
        {"name": "linear 203x1376x520", "op": "linear", "M": 203, "K": 1376, "N": 520, "act": 1, "bias": True},
        # an output projection for one sequence's next token
        {"name": "linear_few 1x4096x4096", "op": "linear_few", "M": 1, "K": 4096, "N": 4096, "act": 0, "residual": True, "bias": False},
        # the feed-forward's second product for a batch of 37 sequences
        {"name": "linear_few 37x11008x4096", "op": "linear_few", "M": 37, "K": 11008, "N": 4096, "act": 0, "residual": True, "bias": False},
        # reduced prompts of 16 pictures: half of the rows are kept, heads of the 7B decoder
        {"name": "cache_store 16 prompts", "op": "cache_store", "B": 16, "low": 158, "high": 355, "H": 32, "Dh": 128, "dtype": "bf16", "gather": True,
         "start": 0},
        # one more token for each of 64 sequences, in the middle of their pages
        {"name": "cache_store 64 tokens", "op": "cache_store", "B": 64, "low": 1, "high": 1, "H": 8, "Dh": 64, "dtype": "bf16", "gather": False,
         "start": 900},
        # the next token of one short conversation, a K/V head for each query head: latency
        {"name": "cache_decode 1x300", "op": "cache_decode", "B": 1, "low": 300, "high": 300, "Hq": 32, "H": 32, "Dh": 128},
        # a full batch of long conversations, four query heads to a K/V head
        {"name": "cache_decode 32x8000", "op": "cache_decode", "B": 32, "low": 2000, "high": 8000, "Hq": 32, "H": 8, "Dh": 128},
        # four long documents at once
        {"name": "prefill 4x3000", "op": "prefill", "B": 4, "low": 2800, "high": 3050, "Hq": 32, "H": 8, "Dh": 128, "dtype": "bf16"},
        # a ragged handful, an empty sequence and one of a single token among them
        {"name": "prefill 9 ragged", "op": "prefill", "B": 9, "low": 0, "high": 260, "Hq": 14, "H": 2, "Dh": 64, "dtype": "bf16"},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear_few", "cache_store", "cache_decode", "prefill"])
    if op == "quantize":
        return {"op": op, "M": _spread(rng, 1, 11008), "K": 32 * _spread(rng, 1, 128), "dtype": rng.choice(["bf16", "bf16", "f32"])}
    if op == "linear":
        K = 32 * _spread(rng, 8, 160)
        return {"op": op, "M": _spread(rng, 65, 5000), "K": K, "N": 8 * _spread(rng, 16, 1000), "act": rng.choice([0, 1, 2]), "bias": rng.random() < 0.5}
    if op == "linear_few":
        return {"op": op, "M": _spread(rng, 1, 64), "K": 32 * _spread(rng, 8, 344), "N": 8 * _spread(rng, 16, 1376), "act": rng.choice([0, 1, 2]),
                "residual": rng.random() < 0.5, "bias": rng.random() < 0.5}
    if op == "cache_store":
        high = _spread(rng, 1, 700)
        return {"op": op, "B": _spread(rng, 1, 32), "low": rng.randint(0, high), "high": high, "H": rng.choice([2, 8, 32, 40]), "Dh": rng.choice([64, 128]),
                "dtype": rng.choice(["bf16", "bf16", "f32"]), "gather": rng.random() < 0.5, "start": rng.choice([0, 0, _spread(rng, 1, 500)])}
    if op == "cache_decode":
        H, G = rng.choice([1, 2, 4, 8, 32]), rng.choice([1, 2, 4, 7, 8, 16])
        B = _spread(rng, 1, 32)
        high = _spread(rng, 1, max(1, min(50000, 1300000 // (B * H))))
        return {"op": op, "B": B, "low": rng.randint(0, high), "high": high, "Hq": H * G, "H": H, "Dh": rng.choice([64, 128])}
    f32 = rng.random() < 0.25
    high = _spread(rng, 1, 400 if f32 else 1500)
    H, G = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7])
    return {"op": op, "B": _spread(rng, 1, 6), "low": rng.randint(0, high), "high": high, "Hq": H * G, "H": H, "Dh": rng.choice([64, 128]),
            "dtype": "f32" if f32 else "bf16"}


# ---- inputs -----------------------------------------------------------------------------------------------------------------------
def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _normal(gen, *shape, std=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=gen, device=DEV) * std).to(dtype)


def _hidden(gen, M, K, dtype):
    """Rows of a decoder: normal, with a few channels far larger than the others."""
    loud = torch.ones(K, device=DEV)
    loud[torch.randint(0, K, (max(1, K // 256),), generator=gen, device=DEV)] = 12.0
    return (torch.randn((M, K), generator=gen, device=DEV) * loud).to(dtype)


def _lengths(case):
    """The lengths of a case's sequences: part of the case, whatever its seed."""
    low, high = case["low"], case["high"]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000 * case["B"] + high)
    n = torch.randint(low, high + 1, (case["B"],), generator=gen, device=DEV)
    n[0] = high  # (the longest is there, and where there are several the shortest)
    if case["B"] > 1:
        n[1] = low
    if case["B"] > 2 and low == 0 < high:
        n[2] = 1
    return n


def _offsets(n):
    return torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), n.cumsum(0)]).to(torch.int32)


def _pool(gen, B, tokens, H, Dh, fill):
    """Pages of a cache in 4 bits, in no order, with room for `tokens` tokens a sequence; fill: they hold keys and values."""
    mp = tokens // 16 + 1
    table = torch.randperm(B * mp, generator=gen, device=DEV).to(torch.int32).reshape(B, mp)
    if not fill:
        return torch.zeros((B * mp, H, 17 * Dh), dtype=torch.uint8, device=DEV), table
    kv = torch.randn((2, B * mp, H, 16, Dh), generator=gen, device=DEV)
    codes, scales = _codes(kv)
    return _page(codes[0], scales[0], codes[1], scales[1]), table


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    op, s = case["op"], {"case": case}
    if op == "quantize":
        s["x"] = _hidden(gen, case["M"], case["K"], _dtype(case["dtype"]))
    elif op in ("linear", "linear_few"):
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = _hidden(gen, M, K, torch.bfloat16)
        s["W"] = _pack(*_codes(torch.randn((N, K), generator=gen, device=DEV) * K ** -0.5))
        s["bias"] = _normal(gen, N, dtype=torch.float32) if case["bias"] else None
        s["residual"] = _normal(gen, M, N) if case["act"] == 2 or case.get("residual") else None
    elif op == "cache_store":
        n = _lengths(case)
        B, H, Dh, dt = case["B"], case["H"], case["Dh"], _dtype(case["dtype"])
        s["rows"] = int(n.sum())
        s["off"] = _offsets(n)
        s["start"] = torch.randint(case["start"] // 2, case["start"] + 1, (B,), generator=gen, device=DEV).to(torch.int32) if case["start"] else None
        s["src_off"] = s["src_idx"] = None
        total = s["rows"]
        if case["gather"]:  # every second row of the prompt, as a selection leaves them
            s["src_off"] = _offsets(2 * n)
            at = torch.arange(total, device=DEV) - torch.repeat_interleave(s["off"][:-1].long(), n)
            s["src_idx"] = (2 * at + torch.randint(0, 2, (total,), generator=gen, device=DEV)).to(torch.int32)
            total *= 2
        s["K"], s["V"] = _normal(gen, max(1, total), H, Dh, dtype=dt), _normal(gen, max(1, total), H, Dh, dtype=dt)
        s["pages"], s["table"] = _pool(gen, B, case["start"] + case["high"], H, Dh, False)
        s["len"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    elif op == "cache_decode":
        B, Hq, H, Dh = case["B"], case["Hq"], case["H"], case["Dh"]
        s["len0"] = _lengths(case).to(torch.int32)
        s["pages"], s["table"] = _pool(gen, B, case["high"] + 1, H, Dh, True)
        s["len"] = s["len0"].clone()
        s["q"], s["k"], s["v"] = _normal(gen, B, Hq, Dh), _normal(gen, B, H, Dh), _normal(gen, B, H, Dh)
        s["logits"] = _normal(gen, B, 2, dtype=torch.float32)
        s["one"] = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    else:
        n = _lengths(case)
        s["rows"], s["off"] = int(n.sum()), _offsets(n)
        rows, dt = max(1, s["rows"]), _dtype(case["dtype"])
        s["Q"] = _normal(gen, rows, case["Hq"], case["Dh"], dtype=dt)
        s["K"], s["V"] = (_normal(gen, rows, case["H"], case["Dh"], dtype=dt) for _ in range(2))
        s["longest"] = case["high"]
    return s


# ---- the 4-bit formats, in torch ---------------------------------------------------------------------------------------------------
def _codes(x):
    """Element codes (0..15) [..., K] and scale bytes [..., K/32] of float32 values: blocks of 32 along the last axis."""
    b = x.float().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    amax = b.abs().amax(-1)
    byte = ((amax.view(torch.int32) + 0x1FFFFF) >> 23) - 2  # the exponent of amax, one more above 1.75 times a power of two
    byte = torch.where(amax.isfinite(), byte.clamp(1, 252), 255)
    a = torch.ldexp(b.abs(), (127 - byte)[..., None])
    # to the nearest element, ties to the one with an even code
    code = (a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int()
    code = code + 8 * b.signbit().int()
    return code.to(torch.uint8).reshape(x.shape), byte.to(torch.uint8)


def _values(codes, scales):
    """The float32 values that codes [..., K] and scale bytes [..., K/32] stand for."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), device=codes.device)
    v = grid[codes.int()].reshape(*codes.shape[:-1], codes.shape[-1] // 32, 32)
    return torch.ldexp(v, scales.int()[..., None] - 127).reshape(codes.shape)


def _pack(codes, scales):
    """A packed matrix: rows of codes (two a byte, K rounded up to 512), then the scale bytes by tiles of 16 rows x 512 columns."""
    M, K = codes.shape
    Kp, Mp = -(-K // 512) * 512, -(-M // 16) * 16
    c = torch.zeros((M, Kp), dtype=torch.uint8, device=codes.device)
    c[:, :K] = codes
    c = c[:, 0::2] | (c[:, 1::2] << 4)
    z = torch.full((Mp, Kp // 32), 127, dtype=torch.uint8, device=codes.device)
    z[:M, : K // 32] = scales
    z = z.reshape(Mp // 16, 16, Kp // 512, 4, 4).permute(0, 2, 4, 1, 3)  # [tile, window, block % 4, row, block / 4]
    return torch.cat([c.reshape(-1), z.reshape(-1)])


def _unpack(packed, M, K):
    Kp, Mp = -(-K // 512) * 512, -(-M // 16) * 16
    c = packed[: M * Kp // 2].reshape(M, Kp // 2)
    z = packed[M * Kp // 2 :].reshape(Mp // 16, Kp // 512, 4, 16, 4).permute(0, 3, 1, 4, 2).reshape(Mp, Kp // 32)
    c = torch.stack([c & 15, c >> 4], -1).reshape(M, Kp)
    return c[:, :K], z[:M, : K // 32]


def _page(kc, kz, vc, vz):
    """Pages [n, H, 17 Dh] of codes [n, H, 16, Dh] and scale bytes [n, H, 16, Dh/32]."""
    n, H, _, Dh = kc.shape
    k = (kc[..., 0::2] | (kc[..., 1::2] << 4)).reshape(n, H, 8 * Dh)
    v = vc.reshape(n, H, 4, 4, Dh // 32, 2, 16).permute(0, 1, 2, 6, 3, 4, 5)  # [token / 4, column % 16, token % 4, block, half of the block]
    v = (v[..., 0] | (v[..., 1] << 4)).reshape(n, H, 8 * Dh)
    return torch.cat([k, v, kz.reshape(n, H, Dh // 2), vz.reshape(n, H, Dh // 2)], -1)


def _held(pages):
    """Values [n, H, 16, Dh] of the keys and of the values that pages [n, H, 17 Dh] hold."""
    n, H, Dh = pages.shape[0], pages.shape[1], pages.shape[2] // 17
    k = pages[..., : 8 * Dh].reshape(n, H, 16, Dh // 2)
    k = torch.stack([k & 15, k >> 4], -1).reshape(n, H, 16, Dh)
    v = pages[..., 8 * Dh : 16 * Dh].reshape(n, H, 4, 16, 4, Dh // 32)
    v = torch.stack([v & 15, v >> 4], -1).permute(0, 1, 2, 4, 5, 6, 3).reshape(n, H, 16, Dh)
    z = pages[..., 16 * Dh :].reshape(n, H, 2, 16, Dh // 32)
    return _values(k, z[:, :, 0]), _values(v, z[:, :, 1])


# ---- the operators in plain form ---------------------------------------------------------------------------------------------------
def _act(y, case, residual):
    if case["act"] == 1:
        y = 0.5 * y * (1 + torch.erf(y * 0.5 ** 0.5))
    if residual is not None:
        r = residual.float()
        y = y * (r / (1 + torch.exp(-r))) if case["act"] == 2 else y + r
    return y.to(torch.bfloat16)


def _plain_linear(s):
    c = s["case"]
    x = s["x"].float()
    if c["op"] == "linear":
        x = _values(*_codes(x))
    y = x @ _values(*_unpack(s["W"], c["N"], c["K"])).t().contiguous()
    return _act(y if s["bias"] is None else y + s["bias"], c, s["residual"])


def _plain_store(s):
    c = s["case"]
    B, H, Dh = c["B"], c["H"], c["Dh"]
    n = (s["off"][1:] - s["off"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(B, device=DEV), n, output_size=s["rows"])
    at = torch.arange(s["rows"], device=DEV) - s["off"].long()[seq]
    src = torch.arange(s["rows"], device=DEV) if s["src_idx"] is None else s["src_off"].long()[seq] + s["src_idx"].long()
    pos = at if s["start"] is None else at + s["start"].long()[seq]
    kc, kz = _codes(s["K"][src])
    vc, vz = _codes(s["V"][src])
    page, slot = s["table"].long()[seq, pos // 16], pos % 16
    Dh2, blocks = Dh // 2, Dh // 32
    k = kc[..., 0::2] | (kc[..., 1::2] << 4)
    r = torch.arange(Dh2, device=DEV)
    h = torch.arange(H, device=DEV)[None, :, None]
    page, slot = page[:, None, None], slot[:, None, None]
    s["pages"][page, h, slot * Dh2 + r] = k
    v = vc.reshape(-1, H, blocks, 2, 16)
    v = (v[:, :, :, 0] | (v[:, :, :, 1] << 4)).reshape(-1, H, Dh2)  # [block, column % 16]
    s["pages"][page, h, 8 * Dh + ((slot // 4 * 16 + r % 16) * 4 + slot % 4) * blocks + r // 16] = v
    z = torch.arange(blocks, device=DEV)
    s["pages"][page, h, 16 * Dh + slot * blocks + z] = kz
    s["pages"][page, h, 16 * Dh + Dh2 + slot * blocks + z] = vz
    s["len"].copy_(n if s["start"] is None else n + s["start"])
    page, h, slot = page[:, 0, 0], h[0, :, 0], slot[:, 0, 0]
    K, V = _held(s["pages"])
    dt = _dtype(c["dtype"])
    return {"K": K[page, :, slot].to(dt), "V": V[page, :, slot].to(dt), "len": s["len"]}


def _plain_decode(s):
    c = s["case"]
    B, Hq, H, Dh = c["B"], c["Hq"], c["H"], c["Dh"]
    K, V = _held(s["pages"][s["table"].long()].reshape(-1, H, 17 * Dh))
    T = s["table"].shape[1] * 16
    K, V = (t.reshape(B, T // 16, H, 16, Dh).transpose(1, 2).reshape(B, H, T, Dh) for t in (K, V))
    there = torch.arange(T, device=DEV)[None] < s["len0"][:, None]
    K = torch.cat([K, s["k"].float()[:, :, None]], 2)
    V = torch.cat([V * there[:, None, :, None], s["v"].float()[:, :, None]], 2)
    there = torch.cat([there, torch.ones_like(there[:, :1])], 1)
    q = s["q"].float().reshape(B, H, Hq // H, Dh)
    w = torch.matmul(q, K.transpose(2, 3).contiguous()) * Dh ** -0.5
    w = w.masked_fill(~there[:, None, None], float("-inf"))
    w = torch.exp(w - w.amax(-1, keepdim=True))
    o = (torch.matmul(w, V) / w.sum(-1, keepdim=True)).reshape(B, Hq, Dh).to(torch.bfloat16)
    keep = s["logits"][:, 1] - s["logits"][:, 0] > 0
    held = [(_values(*_codes(t)) * keep[:, None, None]).to(torch.bfloat16) for t in (s["k"], s["v"])]
    return {"o": o, "keep": keep.to(torch.uint8), "len": s["len0"] + keep.int(), "K": held[0], "V": held[1]}


def _plain_prefill(s):
    c = s["case"]
    B, Hq, H, Dh = c["B"], c["Hq"], c["H"], c["Dh"]
    n, L = (s["off"][1:] - s["off"][:-1]).long(), s["longest"]
    i = torch.arange(L, device=DEV)
    rows = (s["off"][:-1].long()[:, None] + torch.minimum(i[None], (n - 1).clamp(min=0)[:, None])).clamp(max=s["Q"].shape[0] - 1)  # [B, L]
    Q = s["Q"].float()[rows].reshape(B, L, H, Hq // H, Dh).permute(0, 2, 3, 1, 4)
    K, V = (s[t].float()[rows].permute(0, 2, 1, 3)[:, :, None] for t in ("K", "V"))
    w = torch.matmul(Q, K.transpose(3, 4).contiguous()) * Dh ** -0.5
    w = w.masked_fill(i[None] > i[:, None], float("-inf"))
    w = torch.exp(w - w.amax(-1, keepdim=True))
    w = torch.matmul(w, V) / w.sum(-1, keepdim=True)
    o = w.permute(0, 3, 1, 2, 4).reshape(B, L, Hq, Dh)
    return o[i[None] < n[:, None]].to(s["Q"].dtype)


# ---- the library's calls ------------------------------------------------------------------------------------------------------------
def _ours(s):
    import paper_2412_00876_amd as P
    c = s["case"]
    op = c["op"]
    if op == "quantize":
        x, M, K = s["x"], c["M"], c["K"]
        code = P.F32 if c["dtype"] == "f32" else P.BF16
        packed = torch.empty(P.dllava_mx_bytes(M, K), dtype=torch.uint8, device=DEV)
        P.dllava_mx_quantize(x, K, M, K, packed, code)
        y = torch.empty_like(x)
        P.dllava_mx_dequantize(packed, M, K, y, K, code)
        return y
    if op in ("linear", "linear_few"):
        M, K, N = c["M"], c["K"], c["N"]
        y = torch.empty((M, N), dtype=torch.bfloat16, device=DEV)
        if op == "linear_few":
            P.dllava_mx_linear_few(s["x"], K, M, K, s["W"], s["bias"], N, c["act"], s["residual"], y, N, P.BF16)
            return y
        xq = torch.empty(P.dllava_mx_bytes(M, K), dtype=torch.uint8, device=DEV)
        P.dllava_mx_quantize(s["x"], K, M, K, xq, P.BF16)
        P.dllava_mx_linear(xq, M, K, s["W"], s["bias"], N, c["act"], s["residual"], y, N, P.BF16)
        return y
    if op == "prefill":
        Hq, H, Dh = c["Hq"], c["H"], c["Dh"]
        code = P.F32 if c["dtype"] == "f32" else P.BF16
        O = torch.empty_like(s["Q"])
        P.dllava_group_prefill_attn(s["Q"], Hq * Dh, s["K"], s["V"], H * Dh, c["B"], s["off"], s["rows"], Hq, H, Dh, Dh ** -0.5, O, code)
        return O[: s["rows"]]
    B, H, Dh = c["B"], c["H"], c["Dh"]
    if "cache" not in s:  # the cache's descriptor and the workspace, as a program keeps them
        s["cache"] = P.KVCache(s["pages"], s["table"], s["len"])
        if op == "cache_decode":
            s["ws"] = torch.zeros(P.dllava_mx_decode_workspace(B, c["Hq"], H, Dh, s["table"].shape[1]), dtype=torch.uint8, device=DEV)
    if op == "cache_store":
        code = P.F32 if c["dtype"] == "f32" else P.BF16
        P.dllava_mx_cache_store(s["K"], s["V"], H * Dh, B, s["off"], s["start"], s["rows"], s["src_off"], s["src_idx"], s["cache"], None, code)
        K = torch.empty((s["rows"], H, Dh), dtype=s["K"].dtype, device=DEV)
        V = torch.empty_like(K)
        P.dllava_mx_cache_load(s["cache"], B, s["off"], s["start"], s["rows"], K, V, H * Dh, code)
        return {"K": K, "V": V, "len": s["len"]}
    s["len"].copy_(s["len0"])  # the step's lengths come from the program that schedules it
    o = torch.empty_like(s["q"])
    keep = torch.empty(B, dtype=torch.uint8, device=DEV)
    P.dllava_mx_decode_attn_append(s["q"], s["k"], s["v"], B, c["Hq"], s["logits"], 0.0, None, s["cache"], Dh ** -0.5, o, keep, None, s["ws"])
    K, V = torch.empty_like(s["k"]), torch.empty_like(s["v"])
    P.dllava_mx_cache_load(s["cache"], B, s["one"], s["len0"], B, K, V, H * Dh, P.BF16)  # the token as the cache now holds it
    return {"o": o, "keep": keep, "len": s["len"], "K": K, "V": V}


def run(state):
    if own:
        return _ours(state)
    op = state["case"]["op"]
    if op == "quantize":
        return _values(*_codes(state["x"])).to(state["x"].dtype)
    return {"linear": _plain_linear, "linear_few": _plain_linear, "cache_store": _plain_store, "cache_decode": _plain_decode,
            "prefill": _plain_prefill}[op](state)


# ---- what a pass cannot do without --------------------------------------------------------------------------------------------------
def work(case):
    op, e = case["op"], 4 if case.get("dtype") == "f32" else 2
    if op == "quantize":  # there and back
        n = case["M"] * case["K"]
        return {"bytes": n * (2 * e + 2 * 17 / 32), "flops": 0}
    if op in ("linear", "linear_few"):
        M, K, N = case["M"], case["K"], case["N"]
        more = 2 if case["act"] == 2 or case.get("residual") else 0
        x = 2 * M * K + (2 * M * K * 17 / 32 if op == "linear" else 0)
        return {"bytes": x + N * K * 17 / 32 + M * N * (2 + more) + 4 * N * case["bias"], "flops": 2 * M * N * K}
    mean = (case["low"] + case["high"]) / 2
    rows = case["B"] * mean
    if op == "cache_store":  # there and back
        return {"bytes": 2 * rows * case["H"] * case["Dh"] * (2 * e + 2 * 17 / 32) + 4 * case["B"], "flops": 0}
    if op == "cache_decode":
        kv = 2 * case["H"] * case["Dh"]
        return {"bytes": rows * kv * 17 / 32 + case["B"] * (4 * case["Hq"] * case["Dh"] + 2 * kv + kv * 17 / 32 + 2 * kv), "flops": 4 * rows * case["Hq"] * case["Dh"]}
    return {"bytes": rows * case["Dh"] * e * (2 * case["Hq"] + 2 * case["H"]), "flops": 2 * case["B"] * mean * (mean + 1) * case["Hq"] * case["Dh"]}


# ---- the same from the definitions, in 64 bits --------------------------------------------------------------------------------------
def _nearest(x):
    """The 4-bit values of x, blocks of 32 along the last axis, in float64."""
    x = x.double()
    b = x.reshape(-1, 32)
    amax = b.abs().max(1).values
    m, e = torch.frexp(amax)  # amax = m 2^e, m in [0.5, 1)
    step = torch.pow(2.0, ((e - 3) + (m > 0.875).int()).clamp(-126, 125).double())[:, None]
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    a = b.abs() / step
    lower = (torch.searchsorted(grid, a.contiguous(), right=True) - 1).clamp(max=6)
    upper = lower + 1
    dl, du = a - grid[lower], grid[upper] - a
    pick = torch.where((du < dl) | ((du == dl) & (upper % 2 == 0)), upper, lower)
    return (torch.sign(b) * grid[pick] * step).reshape(x.shape)


def _decoded(byte_pairs, scale_bytes):
    """float64 values of interleaved code bytes [..., n] with one scale byte per 16 of them."""
    both = torch.stack([byte_pairs % 16, byte_pairs // 16], -1).flatten(-2).long()
    mag, sign = both % 8, 1 - 2 * (both // 8).double()
    value = torch.tensor(GRID, dtype=torch.float64, device=both.device)[mag] * sign
    return value * torch.pow(2.0, scale_bytes.double() - 127).repeat_interleave(32, -1)


def _weights(packed, N, K):
    Kp = (K + 511) // 512 * 512
    codes = packed[: N * Kp // 2].view(N, Kp // 2)
    n, blk = torch.arange(N, device=DEV)[:, None], torch.arange(Kp // 32, device=DEV)[None]
    at = ((n // 16 * (Kp // 512) + blk // 16) * 64 + blk % 4 * 16 + n % 16) * 4 + blk % 16 // 4
    return _decoded(codes, packed[N * Kp // 2 :][at])[:, :K]


def _softmax_rows(q, k, v, scale, causal):
    """q [h, m, d], k, v [h, n, d]"""
    w = torch.matmul(q, k.transpose(1, 2).contiguous()) * scale
    if causal:
        w = w + torch.full(w.shape[1:], -math.inf, dtype=w.dtype, device=w.device).triu(1)
    return torch.matmul(torch.softmax(w, -1), v)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "quantize":
        return _nearest(s["x"])
    if op in ("linear", "linear_few"):
        x = _nearest(s["x"]) if op == "linear" else s["x"].double()
        y = torch.matmul(x, _weights(s["W"], case["N"], case["K"]).t())
        if s["bias"] is not None:
            y = y + s["bias"].double()
        if case["act"] == 1:
            y = torch.special.ndtr(y) * y
        if s["residual"] is not None:
            r = s["residual"].double()
            y = y * r * torch.sigmoid(r) if case["act"] == 2 else y + r
        return y
    off = s["off"].tolist() if "off" in s else None
    if op == "cache_store":
        rows, lens = [], []
        for b in range(case["B"]):
            n = off[b + 1] - off[b]
            at = torch.arange(off[b], off[b + 1], device=DEV)
            rows.append(at if s["src_idx"] is None else int(s["src_off"][b]) + s["src_idx"][at].long())
            lens.append(n + (0 if s["start"] is None else int(s["start"][b])))
        rows = torch.cat(rows)
        return {"K": _nearest(s["K"][rows]), "V": _nearest(s["V"][rows]), "len": torch.tensor(lens, dtype=torch.int32)}
    if op == "cache_decode":
        Hq, H, Dh = case["Hq"], case["H"], case["Dh"]
        c = torch.arange(Dh, device=DEV)
        out = []
        for b in range(case["B"]):
            n = int(s["len0"][b])
            p = s["pages"][s["table"][b, : (n + 15) // 16].long()]
            k = _decoded(p[..., : 8 * Dh], p[..., 16 * Dh : 16 * Dh + Dh // 2]).reshape(-1, H, 16, Dh)
            t = torch.arange(16, device=DEV)[:, None]
            byte = p[..., 8 * Dh + ((t // 4 * 16 + c % 16) * 4 + t % 4) * (Dh // 32) + c // 32].long()  # [page, head, token, column]
            code = torch.where(c % 32 < 16, byte % 16, byte // 16)
            v = torch.tensor(GRID, dtype=torch.float64, device=DEV)[code % 8] * (1 - 2 * (code // 8))
            v = v * torch.pow(2.0, p[..., 16 * Dh + Dh // 2 + t * (Dh // 32) + c // 32].double() - 127)
            k, v = (x.transpose(0, 1).reshape(H, -1, Dh)[:, :n] for x in (k, v))
            k, v = (torch.cat([x, s[y][b].double()[:, None]], 1) for x, y in ((k, "k"), (v, "v")))
            out.append(_softmax_rows(s["q"][b].double().reshape(H, Hq // H, Dh), k, v, 1 / math.sqrt(Dh), False).reshape(Hq, Dh))
        keep = (s["logits"][:, 1] > s["logits"][:, 0]).int()
        held = [_nearest(s[x]) * keep[:, None, None] for x in ("k", "v")]
        return {"o": torch.stack(out), "keep": keep.to(torch.uint8), "len": s["len0"] + keep, "K": held[0], "V": held[1]}
    G, out = case["Hq"] // case["H"], []
    for b in range(case["B"]):
        q, k, v = (s[x][off[b] : off[b + 1]].double().transpose(0, 1) for x in ("Q", "K", "V"))
        if q.shape[1]:
            o = torch.cat([_softmax_rows(q[h * G : h * G + G], k[h : h + 1].expand(G, -1, -1).contiguous(), v[h : h + 1].expand(G, -1, -1).contiguous(),
                                         1 / math.sqrt(case["Dh"]), True) for h in range(case["H"])])
            out.append(o.transpose(0, 1))
    return torch.cat(out)

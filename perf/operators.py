"""The operators around a decoder layer's W4A8 linears as measured work: the norm that quantizes, the 4-bit cache of Keys and
Values, and attention over it.

Every case is a plain dict; ``prepare`` makes its inputs on the GPU from a seed, ``run`` is one pass through the operator, either in
elementary torch operations (``own`` false) or by the library's calls, ``work`` says what the pass cannot do without, and ``exact``
evaluates the definition in 64 bits.

The cache.  A row is one (token, head) of Keys or of Values: ``D`` channels as dINT4 codes under one step and zero-point,

    lo = min(0, min x), hi = max(0, max x), step = (hi - lo) / 13 to 20 mantissa bits, z = clamp(rne(-lo / step), 0, 13),
    u = x / step:  1/4 < u <= 3/4 -> +step/2;  -3/4 <= u < -1/4 -> -step/2;  else step * (clamp(rne(u) + z, 0, 13) - z),

kept as D/2 bytes and one 32-bit word, the step's bits with the zero-point in the last four.  Rows lie in pages
``[pages, heads, page_size, D/2]``; ``table[b, j]`` is the page of tokens ``j * page_size ..`` of sequence ``b``.
"""
import math

import torch

own = False

F32_MIN = 1.1754943508222875e-38
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # the norm in front of a linear of a 4096-wide model's decode step, one sequence: latency alone
        dict(name="norm 1x4096", op="norm", M=1, K=4096, dtype="bf16", residual=True, scaled=True),
        # a ragged batch of prompt tokens on a 5120-wide model, first layer (nothing to add)
        dict(name="norm 333x5120", op="norm", M=333, K=5120, dtype="f16", residual=False, scaled=True),
        # a long prompt on a 9216-wide model
        dict(name="norm 4096x9216", op="norm", M=4096, K=9216, dtype="bf16", residual=True, scaled=True),
        # one new token for each of 16 sequences, 32 heads of 128, small pages
        dict(name="cache 16x1x32x128", op="cache", B=16, S=1, H=32, D=128, T=2048, page=16, dtype="bf16", ragged=True),
        # short prompts of unequal lengths on a 12-head model, padded to the longest
        dict(name="cache 5x77x12x64", op="cache", B=5, S=77, H=12, D=64, T=200, page=16, dtype="f16", ragged=True),
        # two long prompts, 40 heads
        dict(name="cache 2x4096x40x128", op="cache", B=2, S=4096, H=40, D=128, T=4096, page=64, dtype="f16", ragged=False),
        # decode, one sequence and a short cache: latency
        dict(name="attn 1x1 of 600", op="attn", B=1, S=1, Hq=32, Hkv=32, D=128, T=600, page=16, dtype="f16", ragged=False),
        # decode, a serving batch of unequal lengths on a 40-head model
        dict(name="attn 32x1 of 4096", op="attn", B=32, S=1, Hq=40, Hkv=40, D=128, T=4096, page=64, dtype="bf16", ragged=True),
        # decode, one very long context, eight query heads to a kv head, a cache in one piece
        dict(name="attn 1x1 of 131073", op="attn", B=1, S=1, Hq=64, Hkv=8, D=128, T=131073, page=0, dtype="bf16", ragged=False),
        # a few drafted tokens to verify for each sequence, heads of 64
        dict(name="attn 7x5 of 3001", op="attn", B=7, S=5, Hq=24, Hkv=12, D=64, T=3001, page=16, dtype="f16", ragged=True),
        # a chunk of a long prompt behind what is cached
        dict(name="attn 1x512 of 8000", op="attn", B=1, S=512, Hq=32, Hkv=32, D=128, T=8000, page=64, dtype="bf16", ragged=False),
        # two whole prompts of unequal lengths, shared heads
        dict(name="attn 2x3000 of 3000", op="attn", B=2, S=3000, Hq=32, Hkv=8, D=128, T=3000, page=64, dtype="f16", ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "cache", "attn", "attn"])
    dtype = rng.choice(["f16", "bf16"])
    if op == "norm":
        K = _log_int(rng, 512, 12288)
        if rng.random() < 0.7:
            K = K // 64 * 64
        M = _log_int(rng, 1, min(8192, 4096 * 9216 // K))
        return dict(op=op, M=M, K=K, dtype=dtype, residual=rng.random() < 0.7, scaled=rng.random() < 0.7)
    D, page, ragged = rng.choice([64, 96, 128, 128, 256]), rng.choice([0, 16, 16, 64, 128]), rng.random() < 0.6
    if op == "cache":
        B, H = _log_int(rng, 1, 32), rng.choice([1, 2, 8, 12, 32, 40])
        S = _log_int(rng, 1, max(1, min(4096, 2 * 4096 * 40 * 128 // (B * H * D))))
        T = S + _log_int(rng, 1, 2000)
        return dict(op=op, B=B, S=S, H=H, D=D, T=T, page=page, dtype=dtype, ragged=ragged)
    Hkv, G = rng.choice([1, 2, 8, 12, 32]), rng.choice([1, 1, 2, 4, 8])
    while Hkv * G > 64:
        G //= 2
    if rng.random() < 0.6:      # decode and drafts
        S, B = rng.choice([1, 1, 1, 2, 5, 8]), _log_int(rng, 1, 32)
        T = max(S, _log_int(rng, 1, min(100000, 32 * 4096 * 40 * 128 // (2 * B * Hkv * D))))
    else:                       # prompts and chunks of them
        S, B = _log_int(rng, 16, 2048), rng.choice([1, 1, 2, 3])
        T = S + (0 if rng.random() < 0.4 else _log_int(rng, 1, 8000))
        while B * Hkv * G * S * T * D > 32 * 3000 * 3000 * 128 or B * Hkv * T * D > 200000000:
            S, T = max(16, S // 2), max(16, T // 2)
    return dict(op=op, B=B, S=S, Hq=Hkv * G, Hkv=Hkv, D=D, T=max(S, T), page=page, dtype=dtype, ragged=ragged)


def _lengths(case):
    """(start, count) of every sequence: cached tokens before this step, and new ones."""
    B, S, T = case["B"], case["S"], case["T"]
    start, count = [], []
    for b in range(B):
        n, c = T, S
        if case["ragged"] and b:
            n = max(1, T - (T * 3 // 4) * b // (B - 1) - (b * 7) % 13)
            c = S if S <= 8 else max(1, S - (S // 2) * b // (B - 1))
        c = min(c, n)
        start.append(n - c)
        count.append(c)
    return start, count


def _page_size(case):
    return case["page"] or (case["T"] + 15) // 16 * 16


# ---------------------------------------------------------------------------------------------------------- the 4-bit rows
def _quantize(x):
    """Codes 0..15 (uint8), step and zero-point (float32) of the rows of x, in 64 bits: 16-bit values often lie on a border."""
    x = x.double()
    lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
    step = (((hi - lo) / 13.0).view(torch.int64) + (1 << 32)) & -(1 << 33)
    step = step.view(torch.float64)
    live = step >= F32_MIN
    step = torch.where(live, step, math.inf)
    zero = torch.round(-lo / step).clamp(0.0, 13.0)
    u = x / step[..., None]
    code = (torch.round(u) + zero[..., None]).clamp(0.0, 13.0).to(torch.uint8)
    code = torch.where((u > 0.25) & (u <= 0.75), 14, code)
    code = torch.where((u < -0.25) & (u >= -0.75), 15, code)
    return code.to(torch.uint8), torch.where(live, step, 0.0).float(), zero.float()


def _pack(code):
    """Codes [..., D] -> bytes [..., D/2]: eight channels to four bytes, the first four in the low nibbles."""
    e = torch.where(code == 14, 15, torch.where(code == 15, 7, (code >> 1) | ((code & 1) << 3))).to(torch.uint8)
    e = e.reshape(*code.shape[:-1], code.shape[-1] // 8, 2, 4)
    return (e[..., 0, :] | (e[..., 1, :] << 4)).reshape(*code.shape[:-1], code.shape[-1] // 2)


def _unpack(packed, words):
    """Values (float32) of rows of bytes [..., D/2] under their words [...]."""
    p = packed.reshape(*packed.shape[:-1], packed.shape[-1] // 4, 1, 4)
    e = torch.cat([p & 15, p >> 4], dim=-2).reshape(*packed.shape[:-1], packed.shape[-1] * 2)
    half = (words & -16).view(torch.float32) * 0.5
    two_z = ((words & 15) * 2).to(torch.int8)
    low = (e & 7).to(torch.int8)
    d = torch.where(low == 7, ((e >> 3) * 2).to(torch.int8) - 1, low * 4 + ((e >> 3) * 2).to(torch.int8) - two_z[..., None])
    return half[..., None] * d


def _words(step, zero):
    return step.view(torch.int32) | zero.to(torch.int32)


def _slots(start, S, table, page):
    """Page and place in it of tokens start .. start + S - 1 of every sequence: int64 [B, S] each."""
    pos = start.to(torch.int64)[:, None] + torch.arange(S, device=start.device)
    pos = pos.clamp(max=table.shape[1] * page - 1)
    return torch.gather(table.to(torch.int64), 1, pos // page), pos % page


# ---------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _cached(g, B, H, T, D, gain):
    """Rows [B, H, T, D] as a model caches them: unequal channels, two of them far out, an offset to each."""
    x = _normal(g, B, H, T, D)
    x *= torch.exp2(0.5 * _normal(g, H, 1, D)) * gain
    x += 0.3 * gain * _normal(g, H, 1, D)
    x[..., :2] *= 3.0
    return x


def prepare(case, seed):
    g, dt = _generator(seed), DTYPES[case["dtype"]]
    if case["op"] == "norm":
        M, K = case["M"], case["K"]
        x = _normal(g, M, K)
        x[:, torch.randperm(K, generator=g, device="cuda")[: max(1, K // 128)]] *= 20.0
        st = dict(case=case, x=x.to(dt), w=(1.0 + 0.2 * _normal(g, K)).to(dt), eps=1e-5)
        st["r"] = _normal(g, M, K).to(dt) if case["residual"] else None
        st["s"] = (0.5 + 1.5 * torch.rand(K, generator=g, device="cuda")) if case["scaled"] else None
        return st
    B, S, T, D, P = case["B"], case["S"], case["T"], case["D"], _page_size(case)
    H = case["H"] if case["op"] == "cache" else case["Hkv"]
    each = (T + P - 1) // P
    start, count = _lengths(case)
    st = dict(case=case, P=P, start=torch.tensor(start, dtype=torch.int32, device="cuda"),
              count=torch.tensor(count, dtype=torch.int32, device="cuda"))
    pages = B * each
    order = torch.randperm(pages, generator=g, device="cuda") if case["page"] else torch.arange(pages, device="cuda")
    st["table"] = order.reshape(B, each).to(torch.int32)
    if case["op"] == "cache":
        st["k"] = _cached(g, B, H, S, D, 1.0).transpose(1, 2).contiguous().to(dt)
        st["v"] = _cached(g, B, H, S, D, 0.5).transpose(1, 2).contiguous().to(dt)
        st["cache"] = [torch.zeros((pages, H, P, D // 2), dtype=torch.uint8, device="cuda") if i % 2 == 0 else
                       torch.zeros((pages, H, P), dtype=torch.int32, device="cuda") for i in range(4)]
        return st
    cache = []
    for gain in (1.0, 0.5):
        code, step, zero = _quantize(_cached(g, B, H, each * P, D, gain).to(dt))
        packed, words = _pack(code), _words(step, zero)
        for x in (packed, words):
            x = x.reshape(B, H, each, P, -1).transpose(1, 2).reshape(pages, H, P, -1)
            paged = torch.empty_like(x)
            paged[order] = x
            cache.append(paged)
        cache[-1] = cache[-1].reshape(pages, H, P)
    st["cache"] = cache
    st["q"] = (1.5 * _normal(g, B, S, case["Hq"], D)).to(dt)
    st["scale"] = 1.0 / math.sqrt(D)
    return st


# ---------------------------------------------------------------------------------------------------------- one pass
def run(st):
    return {"norm": _run_norm, "cache": _run_cache, "attn": _run_attn}[st["case"]["op"]](st)


def _run_norm(st):
    """The int8 activations as the values they stand for (in the activations' type), their scales, and the sum that the next layer adds to."""
    x, r, w, s = st["x"], st["r"], st["w"], st["s"]
    if own:
        import paper_2311_05161_amd as lib
        q, sx, *h = lib.rms_norm_act_int8(x, w, eps=st["eps"], residual=r, s=s)
        return (torch.mul(q, sx[:, None], out=torch.empty_like(x)), sx, *h)
    h = x if r is None else (x.float() + r.float()).to(x.dtype)
    f = h.float()
    gain = w.float() if s is None else w.float() * (1.0 / s)
    u = f * gain
    a = u.abs().amax(-1)
    norm = torch.rsqrt(f.double().square().mean(-1) + st["eps"])
    inv = 127.0 / a
    live = torch.isfinite(inv)
    sx = torch.where(live, (a * norm / 127.0).float(), 1.0)
    q = torch.round(u * torch.where(live, inv, 0.0)[:, None]).clamp(-127.0, 127.0)
    y = (q * sx[:, None]).to(x.dtype)
    return (y, sx, h) if r is not None else (y, sx)


def _run_cache(st):
    """What the cache holds of the new tokens behind the write, zeros where a sequence has no such token."""
    k, v, P, S = st["k"], st["v"], st["P"], st["case"]["S"]
    if own:
        import paper_2311_05161_amd as lib
        cache = lib.KVCacheDint4(*st["cache"])
        lib.kv_cache_write_dint4(k, v, cache, st["start"], st["count"], st["table"])
        return lib.kv_cache_read_dint4(cache, st["start"], S, st["count"], st["table"], dtype=k.dtype)
    page, place = _slots(st["start"], S, st["table"], P)
    there = torch.arange(S, device=k.device) < st["count"][:, None]
    to, at = page[there], place[there]
    for x, packed, words in ((k, *st["cache"][:2]), (v, *st["cache"][2:])):
        code, step, zero = _quantize(x)
        packed[to, :, at] = _pack(code)[there]
        words[to, :, at] = _words(step, zero)[there]
    return tuple((_unpack(packed[page, :, place], words[page, :, place]) * there[:, :, None, None]).to(k.dtype)
                 for packed, words in (st["cache"][:2], st["cache"][2:]))


def _run_attn(st):
    """Attention of the S newest tokens of every sequence: zeros where a sequence has fewer."""
    c, q = st["case"], st["q"]
    if own:
        import paper_2311_05161_amd as lib
        return lib.attention_kv_dint4(q, lib.KVCacheDint4(*st["cache"]), st["start"], st["count"], st["table"],
                                      scale=st["scale"], max_len=c["T"])
    B, S, H, G, D = c["B"], c["S"], c["Hkv"], c["Hq"] // c["Hkv"], c["D"]
    pages = st["table"].to(torch.int64)
    k, v = (_unpack(packed[pages], words[pages]).transpose(1, 2).reshape(B, H, -1, D)
            for packed, words in (st["cache"][:2], st["cache"][2:]))
    rows = q.float().reshape(B, S, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * S, D) * st["scale"]
    score = torch.matmul(rows, k.transpose(-1, -2)).reshape(B, H, G, S, -1)
    at = torch.arange(S, device=q.device)
    last = torch.where(at < st["count"][:, None], st["start"][:, None] + at, -1)          # [B, S]: the last token seen
    score = score.masked_fill_(torch.arange(score.shape[-1], device=q.device) > last[:, None, None, :, None], -math.inf)
    p = torch.softmax(score, -1).reshape(B, H, G * S, -1)
    o = torch.matmul(p, v).reshape(B, H, G, S, D).permute(0, 3, 1, 2, 4).reshape(B, S, H * G, D)
    return torch.where((last >= 0)[:, :, None, None], o, 0.0).to(q.dtype)


# ---------------------------------------------------------------------------------------------------------- what it takes
def work(case):
    if case["op"] == "norm":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (2 + 1 + (4 if case["residual"] else 0)) + 4 * M + K * (2 + (4 if case["scaled"] else 0)), "flops": 8 * M * K}
    start, count = _lengths(case)
    if case["op"] == "cache":   # written, and read back: zeros go to what a sequence has no token for
        rows = sum(count) * case["H"] * 2
        return {"bytes": rows * (2 * case["D"] + 2 * (case["D"] // 2 + 4)) + case["B"] * case["S"] * case["H"] * 2 * 2 * case["D"], "flops": 12 * rows * case["D"]}
    cached = sum(s + c for s, c in zip(start, count)) * case["Hkv"] * 2 * (case["D"] // 2 + 4)
    pairs = sum(c * s + c * (c + 1) // 2 for s, c in zip(start, count)) * case["Hq"]
    return {"bytes": cached + case["B"] * case["S"] * case["Hq"] * case["D"] * 2 * 2, "flops": 4 * case["D"] * pairs}


# ---------------------------------------------------------------------------------------------------------- in 64 bits
LEVELS = [2 * c for c in range(0, 14, 2)] + [None] + [2 * c for c in range(1, 14, 2)] + [None]     # of nibbles 0..15, in half steps


def _pow2(e):
    """2 ** e exactly (a library's power may be off in its last bit), normal range."""
    return (e.to(torch.int64) + 1023 << 52).view(torch.float64)


def _values64(packed, words):
    """The rows' values in float64, from the nibbles' levels."""
    lut = torch.tensor([x or 0 for x in LEVELS], dtype=torch.float64, device=packed.device)
    out = torch.empty((*packed.shape[:-1], 2 * packed.shape[-1]), dtype=torch.float64, device=packed.device)
    w = words.to(torch.int64) & 0xFFFFFFFF
    zero, bits = w % 16, w // 16 * 16
    step = torch.where(bits > 0, (1.0 + (bits % 8388608).double() / 8388608) * _pow2(bits // 8388608 - 127), 0.0)
    for byte in range(packed.shape[-1]):
        for shift, channel in ((1, byte // 4 * 8 + byte % 4), (16, byte // 4 * 8 + byte % 4 + 4)):
            e = packed[..., byte].to(torch.int64) // shift % 16
            level = torch.where(e == 7, -1.0, torch.where(e == 15, 1.0, lut[e] - 2.0 * zero))
            out[..., channel] = level * step / 2
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        x = st["x"].double()
        h = x if st["r"] is None else (x + st["r"].double()).to(st["x"].dtype).double()
        y = h * st["w"].double() / (1.0 if st["s"] is None else st["s"].double())
        y = y / torch.sqrt((h * h).sum(-1, keepdim=True) / h.shape[-1] + st["eps"])
        sx = y.abs().max(-1).values / 127
        got = torch.round(y / sx[:, None]) * sx[:, None]
        return (got, sx) if st["r"] is None else (got, sx, h)
    if case["op"] == "cache":
        got = []
        for x in (st["k"].double(), st["v"].double()):
            low, high = x.min(-1, keepdim=True).values.clamp(max=0), x.max(-1, keepdim=True).values.clamp(min=0)
            frac, power = torch.frexp((high - low) / 13)
            step = torch.floor(frac * 2.0 ** 20 + 0.5) * _pow2(power - 20)      # 20 bits, halves up
            z = torch.round(-low / step)
            u = x / step
            level = torch.minimum(torch.maximum(torch.round(u), -z), 13 - z)
            near = (u.abs() > 0.25) & (u.abs() <= 0.75)
            got.append(torch.where(near, 0.5 * torch.sign(u), level) * step)
        start, count = _lengths(case)
        for b, c in enumerate(count):
            for x in got:
                x[b, c:] = 0
        return tuple(got)
    B, S, G, H, D = case["B"], case["S"], case["Hq"] // case["Hkv"], case["Hkv"], case["D"]
    out = torch.zeros((B, S, case["Hq"], D), dtype=torch.float64, device="cuda")
    start, count = _lengths(case)
    for b in range(B):
        n = start[b] + count[b]
        k, v = (_values64(packed[st["table"][b].long()], words[st["table"][b].long()]).transpose(0, 1).reshape(H, -1, D)[:, :n]
                for packed, words in (st["cache"][:2], st["cache"][2:]))
        behind = torch.arange(n, device="cuda")[None] > start[b] + torch.arange(count[b], device="cuda")[:, None]
        for g in range(G):
            rows = st["q"][b, : count[b], g::G].double().transpose(0, 1).contiguous()
            e = torch.matmul(rows, k.transpose(1, 2).contiguous()) * st["scale"]
            e[:, behind] = -math.inf
            e = torch.exp(e - e.max(-1, keepdim=True).values)
            out[b, : count[b], g::G] = (torch.matmul(e, v) / e.sum(-1, keepdim=True)).transpose(0, 1)
    return out

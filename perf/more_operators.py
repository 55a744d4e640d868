"""Attention and the paged key-value cache that it reads, as a list of measurable cases.

A case is a dict of plain values; `prepare` makes what a program holds before the call, `run` is one pass through the
public entry points (`own`) or through the operators' plain form, `exact` the same result in 64-bit arithmetic.

  rotary   rows of heads turned by their positions: halves or neighbours as pairs, all of a head or its first part
  write    a step's keys, turned, and values into their slots of the cache, in the cache's type; its queries turned
  read     slots of the cache as rows again
  decode   one new token of each sequence over its pages: softmax(scale q K^T) V, a head of the cache for a group of q's
  prompt   packed sequences of different lengths over packed keys and values, causal, earlier context or a window

A cache of 16-bit floats is one array [pages, 2 (keys, values), heads, tokens of a page, dim].  mx8 and mx4 caches hold
codes (e4m3, or e2m1 two a byte, the even one low) of that layout, and behind them the scale bytes of 32 values each,
[pages, 2, heads, dim / 32, tokens of a page]: a value is its code's times 2^(byte - 127).

Queries, keys and values are N(0, 1), 1 % of the keys' channels times 8.  Pages of a sequence lie anywhere in the cache."""
import math
import zlib

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)   # of the e2m1 codes 0..7; 8..15 are their negatives
BITS = {"f16": 16, "bf16": 16, "mx8": 8.25, "mx4": 4.25}

# the largest listed cases, which bound what draw() may give
MOST_TURNED = 8192 * 40 * 128
MOST_WRITTEN = 8192 * 8 * 128
MOST_READ = 65536 * 8 * 128
MOST_CACHED = 64 * 8192 * 8 * 128
MOST_SCORES = 8192 * 8192 * 32


def listed():
    return [
        # queries and keys of a decoded batch, an 8B-shaped layer's 32 + 8 heads: what a call costs
        dict(name="rotary_tokens", kind="rotary", T=32, heads=40, dim=128, turned=128, pairs="halves", far=131072, factor=1.0, dtype="bf16"),
        # queries and keys of a long prompt, neighbours as pairs, half of each head turned, positions stretched eightfold
        dict(name="rotary_prompt", kind="rotary", T=8192, heads=40, dim=128, turned=64, pairs="neighbours", far=65536, factor=8.0, dtype="f16"),
        # a decoded batch's step into a 16-bit cache
        dict(name="write_tokens", kind="write", T=32, q_heads=32, heads=8, dim=128, page=16, cache="bf16", turned=128, pairs="halves", far=131072, factor=1.0, dtype="bf16"),
        # a long prompt into a 4-bit cache, and back
        dict(name="write_prompt", kind="write", T=8192, q_heads=32, heads=8, dim=128, page=64, cache="mx4", turned=128, pairs="halves", far=8192, factor=1.0, dtype="bf16"),
        # a short cached prefix of odd length from an 8-bit cache
        dict(name="read_short", kind="read", T=77, heads=8, dim=96, page=16, cache="mx8", dtype="f16"),
        # a long cached prefix from a 4-bit cache
        dict(name="read_long", kind="read", T=65536, heads=8, dim=128, page=64, cache="mx4", dtype="bf16"),
        # one request's next token: an 8B-shaped layer after a thousand tokens
        dict(name="decode_one", kind="decode", B=1, shortest=1000, longest=1000, q_heads=32, heads=8, dim=128, page=16, cache="bf16", window=0, dtype="bf16"),
        # a batch of requests of all lengths, a 70B-shaped layer; one place of the batch is empty
        dict(name="decode_batch", kind="decode", B=64, shortest=0, longest=8191, q_heads=64, heads=8, dim=128, page=64, cache="bf16", window=0, dtype="bf16"),
        # two requests over very long documents, 4-bit cache
        dict(name="decode_long", kind="decode", B=2, shortest=98304, longest=131072, q_heads=32, heads=8, dim=128, page=64, cache="mx4", window=0, dtype="bf16"),
        # prompts of sixteen requests packed together, heads of 64
        dict(name="prompt_packed", kind="prompt", B=16, shortest=17, longest=500, context=0, q_heads=32, heads=8, dim=64, causal=True, window=0, dtype="f16"),
        # the next piece of a prompt after what is cached
        dict(name="prompt_chunk", kind="prompt", B=1, shortest=512, longest=512, context=7680, q_heads=32, heads=8, dim=128, causal=True, window=0, dtype="bf16"),
        # a long prompt, an 8B-shaped layer
        dict(name="prompt_long", kind="prompt", B=1, shortest=8192, longest=8192, context=0, q_heads=32, heads=8, dim=128, causal=True, window=0, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "write", "read", "decode", "decode", "decode", "prompt", "prompt", "prompt"])
    cache = rng.choice(["f16", "bf16", "bf16", "mx8", "mx4"])
    dtype = cache if kind == "decode" and cache in TYPES else rng.choice(["f16", "bf16"])
    dim = rng.choice([32, 64, 64, 96, 128, 128, 128, 128, 160, 192, 256] + ([] if cache in ("mx8", "mx4") else [40, 72, 80, 120]))
    heads, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 8, 12, 16])
    page = rng.choice([16, 32, 64, 64, 128])
    window = _log(rng, 16, 4096) if rng.random() < 0.2 else 0
    turn = dict(turned=dim if rng.random() < 0.6 else max(1, dim // 4) * 2, pairs=rng.choice(["halves", "neighbours"]),
                far=_log(rng, 16, 1 << 20), factor=rng.choice([1.0, 1.0, 4.0, 32.0]))
    if kind == "rotary":
        heads = rng.randint(1, 80)
        return dict(kind=kind, T=_log(rng, 1, MOST_TURNED // (heads * dim)), heads=heads, dim=dim, dtype=rng.choice(["f16", "bf16", "f32"]), **turn)
    if kind == "write":
        return dict(kind=kind, T=max(1, min(_log(rng, 1, 8192), MOST_WRITTEN // (heads * dim), MOST_TURNED // 2 // (heads * group * dim))), q_heads=heads * group,
                    heads=heads, dim=dim, page=page, cache=cache, dtype=dtype, **turn)
    if kind == "read":
        return dict(kind=kind, T=_log(rng, 1, MOST_READ // 2 // (heads * dim)), heads=heads, dim=dim, page=page, cache=cache, dtype=dtype)
    if kind == "decode":
        B = _log(rng, 1, 128)
        longest = _log(rng, 1, min(131072, MOST_CACHED // 4 // (B * heads * dim)))
        return dict(kind=kind, B=B, shortest=rng.choice([longest, longest // 2, longest // 16, 0]) if B > 1 else longest, longest=longest,
                    q_heads=heads * group, heads=heads, dim=dim, page=page, cache=cache, window=window, dtype=dtype)
    B, heads, group = _log(rng, 1, 32), rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 4, 8])
    context = _log(rng, 1, 8192) if rng.random() < 0.3 else 0
    # the scores of the sequences as one padded batch, and a head of any size at no more than the largest case's work
    most = MOST_SCORES // 3 // (B * heads * group) * 128 // max(128, dim)
    longest = _log(rng, 1, max(1, int((math.sqrt(context * context + 4 * most) - context) / 2)))
    return dict(kind=kind, B=B, shortest=rng.choice([longest, longest // 2, longest // 16, 0]) if B > 1 else longest, longest=longest, context=context,
                q_heads=heads * group, heads=heads, dim=dim, causal=rng.random() < 0.85, window=window, dtype=dtype)


# ---- inputs --------------------------------------------------------------------------------------------------------

def _generator(seed, *key):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) % (1 << 30) << 32) ^ zlib.crc32(repr(key).encode()))
    return g


def _rows(seed, what, T, heads, dim, dtype):
    """[T, heads, dim]; keys have channels larger than the others."""
    g = _generator(seed, what)
    x = torch.randn((T, heads, dim), device="cuda", generator=g)
    if what == "k":
        at = torch.randperm(heads * dim, device="cuda", generator=g)[:max(1, round(0.01 * heads * dim))]
        x.flatten(1)[:, at] *= 8.0
    return x.to(TYPES[dtype])


def _lengths(case, seed):
    """Evenly from the shortest to the longest, in the seed's order; a host list."""
    B = case["B"]
    n = [case["longest"] - (case["longest"] - case["shortest"]) * i // max(1, B - 1) for i in range(B)]
    order = torch.randperm(B, generator=torch.Generator().manual_seed(int(seed) % (1 << 30))).tolist()
    return [n[i] for i in order]


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _frequencies(case):
    """Radians a position of each pair, 10000^(-2 i / turned); with a factor, those of less than one turn over 8192 positions divided by it, those of
    more than four as they are, a ramp between."""
    n = case["turned"] // 2
    out = [10000.0 ** (-i / n) for i in range(n)]
    if case["factor"] != 1.0:
        keep = [min(1.0, max(0.0, (8192 * f / (2 * math.pi) - 1) / 3)) for f in out]
        out = [f * (r + (1 - r) / case["factor"]) for f, r in zip(out, keep)]
    return out


def _magnitude(case):
    """What the turned part is multiplied by where positions are stretched."""
    return 1.0 + 0.1 * math.log(case["factor"])


def prepare(case, seed):
    s = dict(case=case)
    kind = case["kind"]
    if kind in ("rotary", "write"):
        T = case["T"]
        # decoded tokens stand anywhere, a prompt's one after the other
        at = torch.randint(0, case["far"], (T,), generator=_generator(seed, "positions"), device="cuda")
        s["positions"] = (at if T <= 512 else int(at[0]) + torch.arange(T, device="cuda")).int()
        s["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    if kind == "rotary":
        s["x"] = _rows(seed, "k", case["T"], case["heads"], case["dim"], case["dtype"])
        s["out"] = torch.empty_like(s["x"])
    elif kind in ("write", "read"):
        T, page, heads, dim = case["T"], case["page"], case["heads"], case["dim"]
        pages = (T + page - 1) // page + 2
        # whole pages one after the other, as a prompt's, or a place in any page, as a decoded batch's
        order = torch.randperm(pages, device="cuda", generator=_generator(seed, "pages"))
        at = torch.arange(T, device="cuda")
        s["slots"] = torch.randperm(pages * page, device="cuda", generator=_generator(seed, "slots"))[:T] if T <= 512 else order[at // page] * page + at % page
        s["pool"] = _pool(case, seed, pages)
        if kind == "write":
            rows = _rows(seed, "k", T, case["q_heads"] + 2 * heads, dim, case["dtype"])   # q | k | v, as a projection leaves them
            s["q"], s["k"], s["v"] = rows.split([case["q_heads"], heads, heads], 1)
            s["q_out"] = torch.empty((T, case["q_heads"], dim), dtype=rows.dtype, device="cuda")
        if kind == "read" or case["cache"] not in TYPES:
            s["k_out"], s["v_out"] = (torch.empty((T, heads, dim), dtype=TYPES[case["dtype"]], device="cuda") for _ in range(2))
    elif kind == "decode":
        B, page = case["B"], case["page"]
        lengths = _lengths(case, seed)
        wide = max(1, (case["longest"] + page - 1) // page)
        s["table"] = torch.randperm(B * wide, device="cuda", generator=_generator(seed, "table")).int().view(B, wide)
        s["lengths"] = _int32(lengths)
        s["pool"] = _pool(case, seed, B * wide)
        s["q"] = _rows(seed, "q", B, case["q_heads"], case["dim"], case["dtype"])
        s["out"] = torch.empty_like(s["q"])
    else:
        lengths = _lengths(case, seed)
        q_at, k_at = [0], [0]
        for n in lengths:
            q_at.append(q_at[-1] + n)
            k_at.append(k_at[-1] + n + (case["context"] if n else 0))
        s["q_offsets"], s["k_offsets"], s["most"] = _int32(q_at), _int32(k_at), (case["longest"], case["longest"] + case["context"])
        s["q"] = _rows(seed, "q", q_at[-1], case["q_heads"], case["dim"], case["dtype"])
        s["k"], s["v"] = (_rows(seed, what, k_at[-1], case["heads"], case["dim"], case["dtype"]) for what in ("k", "v"))
        s["out"] = torch.empty_like(s["q"])
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program makes once: the rotation, the view of its cache's memory, a workspace."""
    from paper_2510_19482_amd import binding as hlq

    case = s["case"]
    kind = case["kind"]
    if "frequencies" in s:
        s["rotary"] = hlq.Rotary(_frequencies(case), interleaved=case["pairs"] == "neighbours", magnitude=_magnitude(case), device="cuda")
    if "pool" in s:
        kept = TYPES.get(case["cache"]) or {"mx8": hlq.HLQ_MX8, "mx4": hlq.HLQ_MX4}[case["cache"]]
        row = int(BITS[case["cache"]] * case["dim"] / 8)
        s["kv"] = hlq.KvCache(s["pool"], s["pool"].numel() // (2 * case["heads"] * case["page"] * row), case["page"], case["heads"], case["dim"], kept)
    if kind == "decode":
        s["ws"] = hlq.alloc_decode_workspace(s["kv"], case["q_heads"], case["B"], s["table"].shape[1])
    elif kind == "prompt":
        s["ws"] = hlq.alloc_prompt_workspace(s["q"].shape[0], s["k"].shape[0], case["B"], case["q_heads"], case["heads"], case["dim"])


def _pool(case, seed, pages):
    """The bytes of a cache that holds random keys and values."""
    page, heads, dim = case["page"], case["heads"], case["dim"]
    if case["cache"] in TYPES:
        x = torch.empty((pages, 2, heads, page, dim), dtype=TYPES[case["cache"]], device="cuda")
        for i, what in enumerate("kv"):
            x[:, i] = _rows(seed, what, pages * page, heads, dim, case["cache"]).view(pages, page, heads, dim).transpose(1, 2)
        return x.flatten().view(torch.uint8)
    codes, scales = [], []
    for what in "kv":
        c, e = _to_mx(_rows(seed, what, pages * page, heads, dim, "f32").view(pages, page, heads, dim).transpose(1, 2), case["cache"])
        codes.append(_packed(c, case["cache"]))
        scales.append((e.squeeze(-1) + 127).to(torch.uint8).transpose(2, 3))
    return torch.cat((torch.stack(codes, 1).flatten(), torch.stack(scales, 1).flatten()))


# ---- a pass --------------------------------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2510_19482_amd import binding as hlq

    case = s["case"]
    kind = case["kind"]
    if kind == "rotary":
        return hlq.hlq_rotary(s["x"], s["positions"], s["rotary"], s["out"])
    if kind == "write":
        hlq.hlq_kv_write(s["kv"], s["k"], s["v"], s["slots"], rotary=s["rotary"], positions=s["positions"], q=s["q"], q_out=s["q_out"])
        if case["cache"] in TYPES:
            return [s["q_out"], s["kv"].rows]
        return [s["q_out"], *hlq.hlq_kv_read(s["kv"], s["slots"], s["k_out"], s["v_out"])]
    if kind == "read":
        return list(hlq.hlq_kv_read(s["kv"], s["slots"], s["k_out"], s["v_out"]))
    if kind == "decode":
        return hlq.hlq_attn_decode(s["kv"], s["q"], s["table"], s["lengths"], s["out"], window=case["window"], ws=s["ws"])
    return hlq.hlq_attn_prompt(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], s["out"], causal=case["causal"], window=case["window"], ws=s["ws"])


def _turned(s, x):
    """Pairs of the first values of each head turned by position times frequency, in 64 bits: positions are far."""
    case = s["case"]
    n = case["turned"]
    angle = (s["positions"].double()[:, None] * s["frequencies"])[:, None, :]
    c, d = torch.cos(angle) * _magnitude(case), torch.sin(angle) * _magnitude(case)
    x = x.double()
    if case["pairs"] == "halves":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        y = torch.cat((a * c - b * d, b * c + a * d), -1)
    else:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y = torch.stack((a * c - b * d, b * c + a * d), -1).flatten(-2)
    return torch.cat((y, x[..., n:]), -1).to(TYPES[case["dtype"]])


def _to_mx(x, kind):
    """Codes [..., dim / 32, 32] (e2m1: 0..15, e4m3: its values) and the exponents [..., dim / 32, 1] of the scales."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    # the largest value gets the largest exponent that the codes have, 8 or 2: floor(log2(top)) less that, not below -127
    e = torch.where(top > 0, torch.frexp(top).exponent - (9 if kind == "mx8" else 3), -127).clamp(min=-127)
    v = torch.ldexp(x, -e)
    if kind == "mx8":
        return v.clamp(-448, 448).to(torch.float8_e4m3fn), e
    a = v.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    return code + 8 * torch.signbit(v), e


def _packed(codes, kind):
    """Bytes of codes."""
    c = codes.flatten(-2)
    if kind == "mx8":
        return c.view(torch.uint8)
    c = c.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _mx_values(codes, e, kind):
    if kind == "mx8":
        return torch.ldexp(codes.float(), e).flatten(-2)
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device=codes.device)
    return torch.ldexp(table[codes.int()], e).flatten(-2)


def _kept(s, i):
    """The cache's keys (i = 0) or values (1) as 32-bit floats [pages, heads, tokens of a page, dim]."""
    case = s["case"]
    page, heads, dim = case["page"], case["heads"], case["dim"]
    if case["cache"] in TYPES:
        return s["pool"].view(TYPES[case["cache"]]).view(-1, 2, heads, page, dim)[:, i].float()
    row = dim if case["cache"] == "mx8" else dim // 2
    pages = s["pool"].numel() // (2 * heads * page * (row + dim // BLOCK))
    split = pages * 2 * heads * page * row
    c = s["pool"][:split].view(pages, 2, heads, page, row)[:, i]
    e = s["pool"][split:].view(pages, 2, heads, dim // BLOCK, page)[:, i].transpose(2, 3).int().unsqueeze(-1) - 127
    c = c.contiguous().view(torch.float8_e4m3fn) if case["cache"] == "mx8" else torch.stack((c & 15, c >> 4), -1).flatten(-2)
    return _mx_values(c.unflatten(-1, (-1, BLOCK)), e, case["cache"])


def _attended(q, k, v, seen, scale):
    """softmax(scale q k^T over what is seen) v, [batch, heads, rows, ...]; a row that sees nothing is 0."""
    scores = torch.matmul(q, k.transpose(-1, -2)).mul_(scale).masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top > -math.inf, top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total > 0, total, 1.0)


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "rotary":
        return _turned(s, s["x"])
    if kind in ("write", "read"):
        page, heads, dim = case["page"], case["heads"], case["dim"]
        if kind == "write":
            q, k, v = _turned(s, s["q"]), _turned(s, s["k"]), s["v"]
            if case["cache"] in TYPES:
                rows = s["pool"].view(TYPES[case["cache"]]).view(-1, 2, heads, page, dim)
                rows[s["slots"] // page, :, :, s["slots"] % page] = torch.stack((k, v), 1).to(rows.dtype)
                return [q, rows]
            return [q, *(_mx_values(*_to_mx(x, case["cache"]), case["cache"]).to(q.dtype) for x in (k, v))]
        return [_kept(s, i)[s["slots"] // page, :, s["slots"] % page].to(TYPES[case["dtype"]]) for i in (0, 1)]
    if kind == "decode":
        B, heads, dim, page = case["B"], case["heads"], case["dim"], case["page"]
        # a sequence's pages side by side, [B, heads, tokens, dim]
        k, v = (_kept(s, i)[s["table"].long()].transpose(1, 2).flatten(2, 3) for i in (0, 1))
        at, n = torch.arange(k.shape[2], device="cuda"), s["lengths"][:, None, None, None]
        seen = (at < n) & (at >= n - case["window"] if case["window"] else at >= 0)
        out = _attended(s["q"].float().view(B, heads, -1, dim), k, v, seen, dim ** -0.5)
        return out.reshape(B, -1, dim).to(TYPES[case["dtype"]])
    B, heads, dim = case["B"], case["heads"], case["dim"]
    (most_q, most_k), q_at, k_at = s["most"], s["q_offsets"], s["k_offsets"]
    # the sequences as a padded batch
    i, j = torch.arange(most_q, device="cuda"), torch.arange(most_k, device="cuda")
    n_q, n_k = (q_at[1:] - q_at[:-1])[:, None], (k_at[1:] - k_at[:-1])[:, None]
    q_rows = (q_at[:-1, None] + i).clamp(max=len(s["q"]) - 1)
    k_rows = (k_at[:-1, None] + j).clamp(max=len(s["k"]) - 1)
    q = s["q"][q_rows].float().unflatten(2, (heads, -1)).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [B, heads, group x rows, dim]
    k, v = (s[x][k_rows].float().transpose(1, 2) for x in "kv")
    seen = (j < n_k)[:, None, :] & (i < n_q)[:, :, None]
    place = (n_k - n_q + i)[:, :, None]                # of a query among the keys
    if case["causal"]:
        seen = seen & (j <= place)
    if case["window"]:
        seen = seen & (j > place - case["window"])
    seen = seen[:, None, None].expand(-1, 1, q.shape[2] // most_q, -1, -1).flatten(2, 3)
    out = _attended(q, k, v, seen, dim ** -0.5).unflatten(2, (-1, most_q)).permute(0, 3, 1, 2, 4).flatten(2, 3)
    return out[i < n_q].to(TYPES[case["dtype"]])


def work(case):
    kind, dim = case["kind"], case["dim"]
    b = 4 if case["dtype"] == "f32" else 2
    if kind == "rotary":
        return {"bytes": case["T"] * (case["heads"] * dim * 2 * b + 4), "flops": 3 * case["T"] * case["heads"] * case["turned"]}
    row = 2 * case["heads"] * dim * BITS.get(case.get("cache"), 16) / 8   # a token's keys and values in the cache
    if kind == "write":
        T, rows = case["T"], 2 * case["heads"] * dim * b
        read_back = 0 if case["cache"] in TYPES else row + rows
        return {"bytes": T * (case["q_heads"] * dim * 2 * b + rows + row + read_back + 12), "flops": 3 * T * (case["q_heads"] + case["heads"]) * case["turned"]}
    if kind == "read":
        return {"bytes": case["T"] * (row + 2 * case["heads"] * dim * b + 8), "flops": 0}
    lengths = _lengths(case, 0)
    if kind == "decode":
        seen = sum(min(n, case["window"]) if case["window"] else n for n in lengths)
        return {"bytes": seen * row + 2 * case["B"] * case["q_heads"] * dim * b, "flops": 4 * seen * case["q_heads"] * dim}
    pairs = sum(_pairs(n, n + case["context"], case["causal"], case["window"]) for n in lengths if n)
    keys = sum(n + case["context"] for n in lengths if n)
    return {"bytes": (sum(lengths) * 2 * case["q_heads"] + keys * 2 * case["heads"]) * dim * b, "flops": 4 * pairs * case["q_heads"] * dim}


def _pairs(n_q, n_k, causal, window):
    """How many keys the queries of a sequence see together."""
    below = lambda n: n * (n + 1) // 2   # noqa: E731
    first = n_k - n_q                    # place of the first query
    # keys up to a query's place, or all; and of those the ones before its window
    all_ = below(n_k) - below(first) if causal else n_q * n_k
    gone = below(max(0, n_k - window)) - below(max(0, first - window)) if window else 0
    return all_ - gone


# ---- in 64 bits ----------------------------------------------------------------------------------------------------

def _turned_64(case, positions, x):
    """Each pair as a complex number times magnitude e^(i angle)."""
    n = case["turned"]
    f = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    w = torch.polar(torch.full_like(f, _magnitude(case)).expand(len(positions), -1).contiguous(), positions.double()[:, None] * f)
    y = x.double().clone()
    even, odd = (slice(0, n // 2), slice(n // 2, n)) if case["pairs"] == "halves" else (slice(0, n, 2), slice(1, n, 2))
    z = torch.complex(y[..., even].contiguous(), y[..., odd].contiguous()) * w[:, None, :]
    y[..., even], y[..., odd] = z.real, z.imag
    return y


def _mx_64(x, kind):
    """The values that the 8- or 4-bit form of x stands for: a grid whose step doubles with each power of two, rounded half to even."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    largest, bits, most = (8, 3, 448.0) if kind == "mx8" else (2, 1, 6.0)
    unit = torch.exp2(torch.clamp(torch.floor(torch.log2(x.abs().max(-1, keepdim=True).values)) - largest, min=-127.0))
    v = x / unit
    low = -6 if kind == "mx8" else 0                 # exponent of the smallest normal code
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(v.abs())), min=low) - bits)
    return ((torch.round(v / step) * step).clamp(-most, most) * unit).flatten(-2)


def _cached_64(case, pool, i):
    page, heads, dim = case["page"], case["heads"], case["dim"]
    if case["cache"] in TYPES:
        return pool.view(TYPES[case["cache"]]).reshape(-1, 2, heads, page, dim)[:, i]
    per = 1 if case["cache"] == "mx8" else 2
    pages = pool.numel() * 32 // (2 * heads * page * dim * (32 // per + 1))
    cut = pages * 2 * heads * page * dim // per
    codes = pool[:cut].reshape(pages, 2, heads, page, dim // per)[:, i].int()
    scales = pool[cut:].reshape(pages, 2, heads, dim // 32, page)[:, i].transpose(-1, -2).int()
    if per == 2:
        codes = torch.stack((codes % 16, codes // 16), -1).flatten(-2)
    width, bias, top = (3, 7, 7) if per == 1 else (1, 1, 3)   # bits of the fraction, the exponent's bias, the sign's place
    sign, body = 1 - 2 * (codes >> top), codes % (1 << top)
    field, frac = (body >> width).double(), (body % (1 << width)).double() / (1 << width)
    value = torch.where(field > 0, (1 + frac) * torch.exp2(field - bias), frac * 2.0 ** (1 - bias)) * sign
    return value * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def exact(case, seed):
    s = prepare(dict(case), seed)
    kind, dim = case["kind"], case["dim"]
    if kind == "rotary":
        return _turned_64(case, s["positions"], s["x"])
    if kind in ("write", "read"):
        page, slots = case["page"], s["slots"]
        if kind == "read":
            return [_cached_64(case, s["pool"], i).double()[slots // page, :, slots % page] for i in (0, 1)]
        q, k, v = _turned_64(case, s["positions"], s["q"]), _turned_64(case, s["positions"], s["k"]), s["v"].double()
        if case["cache"] in TYPES:
            rows = torch.stack([_cached_64(case, s["pool"], i).double() for i in (0, 1)], 1)
            rows[slots // page, 0, :, slots % page], rows[slots // page, 1, :, slots % page] = k, v
            return [q, rows]
        # a key is rounded to its type once when it is turned; its 8 or 4 bits are of that
        return [q, _mx_64(k.to(TYPES[case["dtype"]]), case["cache"]), _mx_64(v, case["cache"])]
    heads, group = case["heads"], case["q_heads"] // case["heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    if kind == "decode":
        keys, values = (_cached_64(case, s["pool"], i) for i in (0, 1))
        for b, n in enumerate(_lengths(case, seed)):
            first = max(0, n - case["window"]) if case["window"] else 0
            if n == 0:
                continue
            k, v = (x[s["table"][b].long()].transpose(0, 1).flatten(1, 2)[:, first:n].double() for x in (keys, values))
            w = torch.softmax(s["q"][b].double().view(heads, group, dim) @ k.transpose(1, 2).contiguous() / math.sqrt(dim), -1)
            out[b] = (w @ v.contiguous()).flatten(0, 1)
        return out
    q_at = k_at = 0
    for n in _lengths(case, seed):
        m = n + case["context"] if n else 0
        if n == 0:
            continue
        i, j = torch.arange(m - n, m, device="cuda")[:, None], torch.arange(m, device="cuda")[None]
        hidden = (j > i if case["causal"] else j < 0) | (j <= i - case["window"] if case["window"] else j < 0)
        for h in range(case["q_heads"]):
            k, v = (s[x][k_at:k_at + m, h // group].double() for x in "kv")
            w = (s["q"][q_at:q_at + n, h].double() @ k.T / math.sqrt(dim)).masked_fill_(hidden, -math.inf)
            out[q_at:q_at + n, h] = torch.softmax(w, -1) @ v
        q_at, k_at = q_at + n, k_at + m
    return out

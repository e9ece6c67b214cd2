"""Performance cases: prompts and 8-bit caches beside the decode step of a transformer's decoder block.

A case is a dict of plain values.  `op` names the operator:

  write   norm of each head's queries and keys, rotation, keys and values into a paged cache of 16 bits     npas.kv_write
  store   the same into a cache of 8-bit floats (blocks of 32 share a power of two), and its values back    npas.kv_write, npas.kv_read
  decode  attention of one new token a sequence over a cache of 8-bit floats                                npas.paged_attention8
  chunk   causal attention of runs of new tokens over a paged cache of 16 or 8 bits                         npas.chunk_attention

With `own` false `run` computes each in its plain form: elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
BLOCK = 32           # elements of a head that share a scale
RANGE = {"bf16": (-110, 120), "f16": (-15, 8)}   # exponents of a scale: every 8-bit float up to 240 times it is a number of the type


def listed():
    return [
        # A decode step of 24 sequences of a small model, pairwise rotation of half a head: launch and latency.
        dict(name="write_step", op="write", dtype="f16", S=24, T=24, heads=12, kv_heads=4, D=64, rot=32, pairs=True, norm=True, page=16,
             context=1500),
        # Prompts of five sequences at once (ragged), grouped heads.
        dict(name="write_prompt", op="write", dtype="bf16", S=5, T=8191, heads=32, kv_heads=8, D=128, rot=128, pairs=False, norm=True, page=16,
             context=4096),
        # A decode step into the 8-bit cache.
        dict(name="store_step", op="store", dtype="bf16", S=16, T=16, heads=32, kv_heads=8, D=128, rot=128, pairs=False, norm=True, page=16,
             context=4000),
        # Prompts into the 8-bit cache, heads that end inside a block, no norm.
        dict(name="store_prompt", op="store", dtype="f16", S=3, T=5003, heads=20, kv_heads=5, D=80, rot=80, pairs=True, norm=False, page=24,
             context=4000),
        # One sequence in interactive use, every head with keys of its own.
        dict(name="decode_one", op="decode", dtype="f16", S=1, heads=16, kv_heads=16, D=64, page=16, length=777, window=0),
        # A serving batch of ragged lengths, an empty sequence among them.
        dict(name="decode_batch", op="decode", dtype="bf16", S=64, heads=32, kv_heads=8, D=128, page=16, length=8192, window=0),
        # One long document: few rows, a long axis to split.
        dict(name="decode_long", op="decode", dtype="bf16", S=1, heads=32, kv_heads=4, D=128, page=64, length=131071, window=0),
        # A few drafted tokens of one sequence, to be checked at once: latency.
        dict(name="chunk_draft_one", op="chunk", dtype="f16", bits=16, S=1, T=5, heads=16, kv_heads=16, D=64, page=16, context=800, window=0),
        # Drafted tokens of a serving batch over an 8-bit cache.
        dict(name="chunk_draft", op="chunk", dtype="bf16", bits=8, S=32, T=163, heads=32, kv_heads=8, D=128, page=16, context=4096, window=0),
        # Whole prompts of five sequences at once (ragged): nothing cached before them.
        dict(name="chunk_prompt", op="chunk", dtype="bf16", bits=16, S=5, T=8191, heads=32, kv_heads=8, D=128, page=16, context=0, window=0),
        # Prompts in a sliding window, odd tiles.
        dict(name="chunk_window", op="chunk", dtype="f16", bits=16, S=3, T=6001, heads=20, kv_heads=5, D=80, page=24, context=2000, window=1000),
        # The last piece of a long document over an 8-bit cache.
        dict(name="chunk_long", op="chunk", dtype="bf16", bits=8, S=1, T=2048, heads=32, kv_heads=8, D=128, page=64, context=63000, window=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "store", "decode", "decode", "chunk", "chunk", "chunk"])
    kv = rng.choice([1, 2, 4, 5, 8] if op != "decode" else [1, 2, 4, 5, 8, 16])
    D = rng.choice([64, 64, 80, 96, 128, 128, 256])
    heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "f16"]), heads=heads, kv_heads=kv, D=D, page=rng.choice([8, 16, 16, 32, 64, 24]))
    if op in ("write", "store"):
        S = _log_int(rng, 1, 200)
        T = S if rng.random() < 0.5 else max(S, _log_int(rng, 1, max(2, 8191 * 4096 // (D * max(heads, 8)))))
        return dict(c, S=S, T=T, rot=rng.choice([D, D, D // 2, 0]), pairs=rng.random() < 0.5, norm=rng.random() < 0.7,
                    context=min(4000, 160000 // S))
    window = rng.choice([0, 0, 0, 500])
    if op == "decode":
        S = _log_int(rng, 1, 128)
        top = min(131071, 2 ** 28 // (S * kv * D))   # tokens of the longest sequence
        return dict(c, S=S, length=_log_int(rng, 1, max(2, top)), window=window)
    S = _log_int(rng, 1, 64)
    T = max(S, _log_int(rng, 1, 8191))
    context = rng.choice([0, 0, 1]) and _log_int(rng, 1, min(60000, 2 ** 27 // (S * kv * D)))
    while T > S and T * (context + T) * heads * D > 2 ** 39:
        T = max(S, T // 2)
    return dict(c, bits=rng.choice([16, 8]), S=S, T=T, context=context, window=window)


# ---- inputs ------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _quantised(x, limits):
    """Rows of x (32 bits, last axis) in 8-bit floats: (x / 2^e rounded to sign, four exponent and three mantissa bits; e), e the least within
    `limits` with magnitudes of a block of 32 up to 448 * 2^e; at the upper limit magnitudes stop at 240 * 2^e."""
    D = x.shape[-1]
    least, most = limits
    x = torch.nn.functional.pad(x, (0, -D % BLOCK)).unflatten(-1, (-1, BLOCK))
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = (e - torch.where(m <= 0.875, 9, 8)).clamp(min=least, max=most)
    e = torch.where(m == 0, torch.full_like(e, least), e)
    a = torch.ldexp(torch.ldexp(x.abs(), -(e // 2)), -(e - e // 2))
    a = torch.minimum(a, torch.where(e == most, 240.0, 448.0))
    step = torch.ldexp(torch.ones_like(a), (torch.frexp(a).exponent - 1).clamp(min=-6) - 3)
    return torch.copysign(torch.round(a / step) * step, x), e


def _cache(case, g, td, tokens):
    """Keys, values [pages][kv heads][page][D] and a page table of `tokens` tokens a sequence in random pages; codes and scales where the cache
    holds 8-bit floats."""
    per = -(-tokens // case["page"])
    pages = case["S"] * per + 1
    shape = (pages, case["kv_heads"], case["page"], case["D"])
    t = {"table": torch.randperm(pages, generator=g, device="cuda")[:case["S"] * per].reshape(case["S"], per).int()}
    for name in ("k", "v"):
        if case["op"] in ("write", "chunk") and case.get("bits", 16) == 16:
            t[name + "_cache"] = torch.empty(shape, dtype=td, device="cuda").normal_(generator=g)
            continue
        t[name + "_cache"] = torch.empty(shape, dtype=torch.uint8, device="cuda")
        t[name + "_scale"] = torch.empty(shape[:3] + (-(-case["D"] // BLOCK),), dtype=torch.uint8, device="cuda")
        if case["op"] == "store":      # written by the pass
            t[name + "_cache"].zero_()
            t[name + "_scale"].zero_()
            continue
        step = max(1, 2 ** 26 // (shape[1] * shape[2] * shape[3]))
        for lo in range(0, pages, step):
            v, e = _quantised(torch.empty((min(step, pages - lo),) + shape[1:], device="cuda").normal_(generator=g), RANGE[case["dtype"]])
            t[name + "_cache"][lo:lo + step] = v.flatten(-2)[..., :case["D"]].to(torch.float8_e4m3fn).view(torch.uint8)
            t[name + "_scale"][lo:lo + step] = (e[..., 0] + 127).to(torch.uint8)
    return t


def _parts(total, S, g):
    """`total` tokens over S sequences, at least one each; none for the fourth of eight and more, whose tokens the fifth has."""
    n = torch.rand(S, generator=g, device="cuda").add(0.3)
    n = (n / n.sum() * (total - S)).long() + 1
    n[0] += total - n.sum()
    if S >= 8:
        n[4] += n[3]
        n[3] = 0
    return n


def _make(case, seed):
    """The tensors of a case, on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    td, op, S, D, H, KV = DTYPES[case["dtype"]], case["op"], case["S"], case["D"], case["heads"], case["kv_heads"]
    if op == "decode":
        n = ((torch.rand(S, generator=g, device="cuda") * case["length"]).long() + 1).clamp_(max=case["length"])
        n[0] = case["length"]
        if S >= 8:
            n[3] = 0
        t = _cache(case, g, td, case["length"])
        return dict(t, q=(_randn(g, S, H, D) * 1.5).to(td), n=n.int())
    T = case["T"]
    if op == "chunk":
        new = _parts(T, S, g)
        cached = (torch.rand(S, generator=g, device="cuda") * case["context"]).long()
        cached[0] = case["context"]
        n = new + cached
        longest, starts = int(n.max()), torch.zeros(S + 1, dtype=torch.int32, device="cuda")
        starts[1:] = new.cumsum(0)
        t = _cache(case, g, td, longest)
        return dict(t, q=(_randn(g, T, H, D) * 1.5).to(td), n=n.int(), starts=starts, longest=longest, most_new=int(new.max()))
    if T == S:       # a decode step: a token for every sequence
        seq = torch.arange(S, device="cuda")
        pos = (torch.rand(S, generator=g, device="cuda") * case["context"]).long()
    else:            # runs of tokens: every sequence starts somewhere
        seq = torch.randint(0, S, (T,), generator=g, device="cuda").sort().values
        first = torch.searchsorted(seq, torch.arange(S, device="cuda"))
        start = (torch.rand(S, generator=g, device="cuda") * 100).long()
        pos = torch.arange(T, device="cuda") - first[seq] + start[seq]
    longest = max(case["context"], int(pos.max()) + 1)
    t = _cache(case, g, td, longest)
    # channels of unlike sizes, as projections give them
    t |= {"qkv": (_randn(g, T, (H + 2 * KV) * D) * torch.exp(0.5 * _randn(g, 1, (H + 2 * KV) * D))).to(td), "seq": seq.int(), "pos": pos.int(),
          "cos_sin": None, "q_weight": None, "k_weight": None}
    if case["norm"]:
        t["q_weight"], t["k_weight"] = 1.0 + 0.2 * _randn(g, D), 1.0 + 0.2 * _randn(g, D)
    if case["rot"]:
        half = case["rot"] // 2
        freq = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * freq
        t["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
    return t


def prepare(case, seed):
    t = _make(case, seed)
    t["case"] = case
    td, op = DTYPES[case["dtype"]], case["op"]
    if op in ("decode", "chunk"):
        t["y"] = torch.empty_like(t["q"])
    else:
        t["q_out"] = torch.empty((case["T"], case["heads"], case["D"]), dtype=td, device="cuda")
    if op == "store":
        t["k_back"], t["v_back"] = (torch.empty((case["T"], case["kv_heads"], case["D"]), dtype=td, device="cuda") for _ in range(2))
    if not own:
        return t
    import paper_2012_00596_amd as npas
    t["npas"], dt = npas, {"bf16": npas.BF16, "f16": npas.F16}[case["dtype"]]
    if "k_scale" in t:
        t["cache"] = npas.KvCache8(t["k_cache"], t["v_cache"], t["k_scale"], t["v_scale"], t["table"], dt)
    else:
        t["cache"] = npas.KvCache(t["k_cache"], t["v_cache"], t["table"], dt)
    if op == "decode":
        t["bytes"] = npas.paged_attention8_workspace_bytes(t["cache"], case["heads"], case["length"])
    elif op == "chunk":
        t["bytes"] = npas.chunk_attention_workspace_bytes(t["cache"], case["T"], case["heads"], t["longest"])
    if "bytes" in t:
        t["workspace"] = torch.empty(max(t["bytes"], 256), dtype=torch.uint8, device="cuda")
    return t


# ---- the measured call -------------------------------------------------------

def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state, state["case"])


def _split(t, c):
    """Queries, keys and values of the joined projection: views [T][heads][D]."""
    H, KV, D = c["heads"], c["kv_heads"], c["D"]
    return t["qkv"].split([H * D, KV * D, KV * D], 1)


def _own(t):
    npas, c, s = t["npas"], t["case"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "decode":
        npas.paged_attention8(t["cache"], t["q"], t["y"], c["heads"], t["n"], c["length"], c["D"] ** -0.5, window=c["window"],
                              workspace=t["workspace"], workspace_bytes=t["bytes"], stream=s)
        return t["y"]
    if c["op"] == "chunk":
        npas.chunk_attention(t["cache"], t["q"], t["y"], c["T"], c["heads"], t["starts"], t["n"], t["longest"], c["D"] ** -0.5,
                             window=c["window"], workspace=t["workspace"], workspace_bytes=t["bytes"], stream=s)
        return t["y"]
    q, k, v = _split(t, c)
    npas.kv_write(t["cache"], q, k, v, t["q_out"], c["T"], c["heads"], t["pos"], sequences=t["seq"], q_weight=t["q_weight"],
                  k_weight=t["k_weight"], eps=EPS, cos_sin=t["cos_sin"], rot_dim=c["rot"],
                  kind=npas.ROTATE_PAIRS if c["pairs"] else npas.ROTATE_HALVES, stream=s)
    if c["op"] == "write":
        return t["q_out"], t["k_cache"], t["v_cache"]
    npas.kv_read(t["cache"], t["k_back"], t["v_back"], c["T"], t["pos"], sequences=t["seq"], stream=s)
    return t["q_out"], t["k_back"], t["v_back"]


# ---- plain forms: elementary operations in 32 bits, one rounding at the end ---

def _plain_heads(t, c):
    """Normed and rotated queries and keys, values: [T][heads][D] in 32 bits."""
    T, D, rot = c["T"], c["D"], c["rot"]
    q, k, v = (x.reshape(T, -1, D).float() for x in _split(t, c))
    if c["norm"]:
        q = q * torch.rsqrt((q * q).mean(-1, keepdim=True) + EPS) * t["q_weight"]
        k = k * torch.rsqrt((k * k).mean(-1, keepdim=True) + EPS) * t["k_weight"]
    if rot:
        cos, sin = t["cos_sin"][t["pos"].long()][:, None].chunk(2, -1)
        q, k = (_plain_rotate(x, cos, sin, rot, c["pairs"]) for x in (q, k))
    return q, k, v


def _plain_rotate(x, cos, sin, rot, pairs):
    half = rot // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :half], x[..., half:rot])
    u, w = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([u, w], -1).flatten(-2) if pairs else torch.cat([u, w], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _plain_write(t, c):
    td = t["qkv"].dtype
    q, k, v = _plain_heads(t, c)
    pos = t["pos"].long()
    page, slot = t["table"][t["seq"].long(), pos // c["page"]].long(), pos % c["page"]
    t["k_cache"][page, :, slot] = k.to(td)
    t["v_cache"][page, :, slot] = v.to(td)
    return q.to(td), t["k_cache"], t["v_cache"]


def _plain_store(t, c):
    """Codes and scales into the cache, and the values that they stand for out of it."""
    td, pos = t["qkv"].dtype, t["pos"].long()
    q, k, v = _plain_heads(t, c)
    page, slot = t["table"][t["seq"].long(), pos // c["page"]].long(), pos % c["page"]
    back = []
    for name, x in (("k", k), ("v", v)):
        code, e = _quantised(x, RANGE[c["dtype"]])
        t[name + "_cache"][page, :, slot] = code.flatten(-2)[..., :c["D"]].to(torch.float8_e4m3fn).view(torch.uint8)
        t[name + "_scale"][page, :, slot] = (e[..., 0] + 127).to(torch.uint8)
        back.append(_plain_from8(t[name + "_cache"][page, :, slot], t[name + "_scale"][page, :, slot]).to(td))
    return q.to(td), back[0], back[1]


def _plain_from8(codes, scales):
    unit = (scales.int() << 23).view(torch.float32)[..., None].expand(*scales.shape, BLOCK).flatten(-2)
    return codes.view(torch.float8_e4m3fn).float() * unit[..., :codes.shape[-1]]


def _plain_cached(t, table, c, heads=slice(None)):
    """Keys and values of the pages of `table` [sequences][pages], in 32 bits: [sequences][kv heads][tokens][D]."""
    for name in ("k", "v"):
        x = t[name + "_cache"][:, heads][table]
        x = x.float() if c.get("bits") == 16 else _plain_from8(x, t[name + "_scale"][:, heads][table])
        yield x.transpose(1, 2).flatten(2, 3).contiguous()


def _plain_softmax(score, seen, v):
    score = score.masked_fill(~seen, -math.inf)
    p = torch.exp(score - score.amax(-1, keepdim=True).clamp(min=-1e30))
    total = p.sum(-1, keepdim=True)
    return p @ v / total.masked_fill(total == 0, 1.0)


def _plain_decode(t, c):
    S, KV, D, G = c["S"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"]
    L = t["table"].shape[1] * c["page"]
    q = t["q"].float().reshape(S, KV, G, D) * D ** -0.5
    y = torch.zeros_like(q)
    j = torch.arange(L, device=q.device)
    step = max(1, 2 ** 29 // (L * KV * D))     # sequences whose keys are held in 32 bits at once
    for s in range(0, S, step):
        e = min(S, s + step)
        k, v = _plain_cached(t, t["table"][s:e].long(), c)
        n = t["n"][s:e, None]
        seen = j < n
        if c["window"]:
            seen = seen & (j >= n - c["window"])
        y[s:e] = _plain_softmax(q[s:e] @ k.transpose(2, 3).contiguous(), seen[:, None, None], v)
    return y.reshape(S, -1, D).to(t["q"].dtype)


def _plain_chunk(t, c):
    S, KV, D, G, N, T = c["S"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"], t["most_new"], c["T"]
    L = t["table"].shape[1] * c["page"]
    starts, n = t["starts"].long(), t["n"].long()
    i, j = torch.arange(N, device=n.device), torch.arange(L, device=n.device)
    rows = (starts[:-1, None] + i).clamp(max=T - 1)
    at = (n - (starts[1:] - starts[:-1]))[:, None] + i                 # positions of the new tokens
    seen = j <= at[..., None]
    if c["window"]:
        seen = seen & (j > at[..., None] - c["window"])
    y = torch.empty((S, KV, N, G, D), device=n.device)
    step = max(1, 2 ** 30 // (L * N * G * KV))  # sequences, or heads of one, whose scores are held at once
    wide = max(1, min(KV, 2 ** 30 // (L * N * G)))
    for s in range(0, S, step):
        e = min(S, s + step)
        for h in range(0, KV, wide):
            heads = slice(h, min(KV, h + wide))
            k, v = _plain_cached(t, t["table"][s:e].long(), c, heads)
            q = t["q"][rows[s:e]].reshape(e - s, N, KV, G, D)[:, :, heads].float().transpose(1, 2).flatten(2, 3) * D ** -0.5
            mask = seen[s:e, None, :, None].expand(e - s, 1, N, G, L).flatten(2, 3)
            y[s:e, heads] = _plain_softmax(q @ k.transpose(2, 3).contiguous(), mask, v).unflatten(2, (N, G))
    token = torch.arange(T, device=n.device)
    seq = torch.searchsorted(starts, token, right=True) - 1
    return y[seq, :, token - starts[seq]].reshape(T, -1, D).to(t["q"].dtype)


_PLAIN = {"write": _plain_write, "store": _plain_store, "decode": _plain_decode, "chunk": _plain_chunk}


# ---- what a pass cannot do without -------------------------------------------

def _row_bytes(case):
    """Bytes of a token's key or value of one head in the cache."""
    D = case["D"]
    return 2 * D if case.get("bits", 16) == 16 and case["op"] in ("write", "chunk") else D + -(-D // BLOCK)


def work(case):
    op, S, D, H, KV, w = case["op"], case["S"], case["D"], case["heads"], case["kv_heads"], case.get("window", 0)
    row = _row_bytes(case)
    if op in ("write", "store"):
        T, rot = case["T"], case["rot"]
        outside = T * (2 * H + 2 * KV) * D * 2 + T * (12 + 4 * rot) + (8 * D if case["norm"] else 0)
        back = T * KV * 2 * (row + 2 * D) if op == "store" else 0
        return {"bytes": outside + T * KV * 2 * row + back, "flops": T * (H + KV) * (3 * rot + (4 * D if case["norm"] else 0)) + (back and 12 * T * KV * D)}
    if op == "decode":       # lengths uniform in 1 .. n, of min(length, window)
        n = case["length"]
        w = min(w or n, n)
        tokens = w + (S - 1 - (S >= 8)) * (w * (n - w) / n + w * (w + 1) / (2 * n))
        return {"bytes": int(2 * tokens * KV * row + 4 * S * H * D + tokens / case["page"] * 4), "flops": int(4 * tokens * H * D)}
    T, context = case["T"], case["context"]
    new, cached = T / S, context if S == 1 else context / 2 + context / (2 * S)
    tokens = S * (cached + new)
    pairs = T * (cached + new / 2)       # of a new token and one that it sees
    if w:
        pairs = min(pairs, T * w)
        tokens = min(tokens, S * (w + new))
    return {"bytes": int(2 * tokens * KV * row + 4 * T * H * D + tokens / case["page"] * 4), "flops": int(4 * pairs * H * D)}


# ---- 64-bit results ----------------------------------------------------------

def _from8_64(codes, scales):
    """Values of 8-bit codes from the definition: sign, exponent with bias 7, three bits of mantissa; no infinities."""
    c = codes.to(torch.int64)
    exponent, mantissa = c >> 3 & 15, (c & 7).double()
    v = torch.where(exponent == 0, mantissa * 2.0 ** -9, (8 + mantissa) * torch.exp2((exponent - 10).double()))
    unit = torch.exp2(scales.double() - 127)
    return torch.where(c >= 128, -v, v) * unit.repeat_interleave(BLOCK, -1)[..., :c.shape[-1]]


def _values64(x, limits):
    """The values that x stands for in blocks of 8-bit floats: the nearest number of the list, ties to the even code."""
    grid = torch.cat([torch.arange(8, device=x.device).double() * 2.0 ** -9] +
                     [(8 + torch.arange(8, device=x.device)).double() * 2.0 ** (e - 10) for e in range(1, 16)])[:127]
    mids = (grid[1:] + grid[:-1]) / 2
    least, most = limits
    out = torch.empty_like(x)
    for lo in range(0, x.shape[-1], BLOCK):
        b = x[..., lo:lo + BLOCK]
        top = b.abs().amax(-1, keepdim=True).clamp(min=448 * 2.0 ** least)
        e = torch.ceil(torch.log2(top / 448)).clamp(max=most)
        unit = torch.exp2(e)
        r = torch.minimum(b.abs() / unit, torch.where(e == most, 240.0, 448.0).double())
        code = torch.searchsorted(mids, r)
        tie = r == mids[code.clamp(max=125)]
        code = code + (tie & (code % 2 == 1) & (code < 126))
        out[..., lo:lo + BLOCK] = torch.sign(b) * grid[code] * unit
    return out


def exact(case, seed):
    t, op = _make(case, seed), case["op"]
    D, H, KV, G = case["D"], case["heads"], case["kv_heads"], case["heads"] // case["kv_heads"]
    if op in ("write", "store"):
        T, rot = case["T"], case["rot"]
        x = t["qkv"].double().reshape(T, H + 2 * KV, D)
        r = x[:, :H + KV].clone()
        if case["norm"]:
            r = r / torch.sqrt(r.square().sum(-1, keepdim=True) / D + EPS)
            r[:, :H] *= t["q_weight"].double()
            r[:, H:] *= t["k_weight"].double()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + rot // 2)
            row = t["cos_sin"].double()[t["pos"].long()]
            z = torch.complex(r[..., a], r[..., b]) * torch.complex(row[:, i], row[:, i + rot // 2])[:, None]
            r[..., a], r[..., b] = z.real, z.imag
        if op == "store":
            return r[:, :H], _values64(r[:, H:], RANGE[case["dtype"]]), _values64(x[:, H + KV:], RANGE[case["dtype"]])
        k, v = t["k_cache"].double(), t["v_cache"].double()
        at = t["table"].long()[t["seq"].long(), t["pos"].long() // case["page"]] * case["page"] + t["pos"].long() % case["page"]
        for cache, new in ((k, r[:, H:]), (v, x[:, H + KV:])):
            for h in range(KV):
                flat = cache[:, h].reshape(-1, D)
                flat[at] = new[:, h]
                cache[:, h] = flat.reshape(cache[:, h].shape)
        return r[:, :H], k, v
    y = torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda")
    starts = list(range(case["S"] + 1)) if op == "decode" else t["starts"].tolist()
    for s, n in enumerate(t["n"].tolist()):
        lo, hi = starts[s:s + 2]
        if n == 0 or hi == lo:
            continue
        pages = t["table"][s, :-(-n // case["page"])].long()
        for h in range(KV):
            k, v = (t[x + "_cache"][pages, h] for x in "kv")
            if "k_scale" in t:
                k, v = (_from8_64(c, t[x + "_scale"][pages, h]) for c, x in ((k, "k"), (v, "v")))
            k, v = k.double().reshape(-1, D)[:n], v.double().reshape(-1, D)[:n]
            for a in range(lo, hi, 512):         # new tokens at a time
                b = min(hi, a + 512)
                q = t["q"][a:b, h * G:(h + 1) * G].double()
                score = q.flatten(0, 1).matmul(k.t().contiguous()).reshape(b - a, G, n) / math.sqrt(D)
                behind = torch.arange(n - hi + a, n - hi + b, device="cuda")[:, None] - torch.arange(n, device="cuda")
                hidden = behind < 0
                if case["window"]:
                    hidden = hidden | (behind >= case["window"])
                p = torch.softmax(score.masked_fill(hidden[:, None], -math.inf), -1)
                y[a:b, h * G:(h + 1) * G] = p.flatten(0, 1).matmul(v).reshape(b - a, G, D)
    return y

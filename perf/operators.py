"""Performance cases: the operators of a transformer's decoder block around its (pruned or quantised) linear layers.

A case is a dict of plain values.  `op` names the operator:

  norm      norm after a block, its gate, the scaled residual and the norm before the next block   npas.gated_residual_norm
  append    rotation of queries and keys, keys and values written into a paged cache               npas.kv_append
  attention attention of one new token a sequence over the paged cache                             npas.paged_attention
  quantize  rows to microscaled 4-bit floats and back to the values these stand for                npas.mxfp4_quantize, _dequantize
  fc        product of activations and weights in microscaled 4-bit floats                         npas.fc_mxfp4

With `own` false `run` computes each in its plain form: elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6
SCALE = 0.875        # of the residual stream
BLOCK = 32           # elements that share a scale


def listed():
    return [
        # One token between two layers of a small model: launch and latency.
        dict(name="norm_step", op="norm", dtype="bf16", T=1, D=1280, gate="channel", post=True),
        # A prompt's tokens in a wide model, the gate a tensor of its own.
        dict(name="norm_prompt", op="norm", dtype="bf16", T=4096, D=4096, gate="token", post=True),
        # A decode step of 24 sequences, small heads, pairwise rotation, slices of one joined projection.
        dict(name="append_step", op="append", dtype="f16", S=24, T=24, heads=12, kv_heads=4, D=64, rot=32, pairs=True, page=16,
             context=1500),
        # Prompts of five sequences at once (ragged), grouped heads.
        dict(name="append_prompt", op="append", dtype="bf16", S=5, T=8191, heads=32, kv_heads=8, D=128, rot=128, pairs=False, page=16,
             context=4096),
        # One sequence in interactive use, every head with keys of its own.
        dict(name="attention_one", op="attention", dtype="f16", S=1, heads=16, kv_heads=16, D=64, page=16, length=777, window=0),
        # A serving batch of ragged lengths, an empty sequence among them.
        dict(name="attention_batch", op="attention", dtype="bf16", S=64, heads=32, kv_heads=8, D=128, page=16, length=8192, window=0),
        # One long document: few rows, a long axis to split.
        dict(name="attention_long", op="attention", dtype="bf16", S=1, heads=32, kv_heads=4, D=128, page=64, length=131071, window=0),
        # Activations of a small batch.
        dict(name="quantize_step", op="quantize", dtype="f16", M=32, K=1280),
        # Activations of a prompt, rows that end inside a block.
        dict(name="quantize_prompt", op="quantize", dtype="bf16", M=8192, K=4100),
        # One token through a square projection: the weights' bytes.
        dict(name="fc_step", op="fc", dtype="bf16", B=1, IN=4096, OUT=4096, bias=False, act="none"),
        # A classifier on a middling batch, odd tiles.
        dict(name="fc_batch", op="fc", dtype="f16", B=256, IN=1280, OUT=1000, bias=True, act="relu"),
        # A prompt through an up-projection: matrix cores.
        dict(name="fc_prompt", op="fc", dtype="bf16", B=4096, IN=4096, OUT=8192, bias=False, act="none"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:                # no size of 3072, joined ones included
        c = _draw(rng)
        widths = [n * c["D"] for n in (c["heads"], c["kv_heads"], c["heads"] + 2 * c["kv_heads"])] if "heads" in c else []
        if 3072 not in widths + list(c.values()):
            return c


def _draw(rng):
    op = rng.choice(["norm", "append", "attention", "attention", "quantize", "fc", "fc"])
    dt = rng.choice(["bf16", "bf16", "f16"])
    if op == "norm":
        D = rng.choice([8 * _log_int(rng, 8, 1000), 8 * _log_int(rng, 8, 1000), _log_int(rng, 50, 8000)])
        return dict(op=op, dtype=rng.choice([dt, dt, "f32"]), T=_log_int(rng, 1, min(8192, 4096 * 4096 // D // 2)), D=D,
                    gate=rng.choice(["none", "channel", "token"]), post=rng.random() < 0.7)
    if op == "append":
        kv = rng.choice([1, 2, 4, 5, 8])
        D = rng.choice([64, 64, 80, 96, 128, 128, 256])
        heads = kv * rng.choice([1, 2, 3, 4, 7, 8])
        S = _log_int(rng, 1, 200)
        T = S if rng.random() < 0.5 else max(S, _log_int(rng, 1, max(2, 8191 * 4096 // (D * max(heads, 8)))))
        return dict(op=op, dtype=dt, S=S, T=T, heads=heads, kv_heads=kv, D=D, rot=rng.choice([D, D, D // 2, 0]),
                    pairs=rng.random() < 0.5, page=rng.choice([8, 16, 16, 32, 64, 24]), context=min(4000, 160000 // S))
    if op == "attention":
        kv = rng.choice([1, 2, 4, 5, 8, 16])
        D = rng.choice([64, 64, 80, 96, 128, 128, 256])
        S = _log_int(rng, 1, 128)
        top = min(131071, 2 ** 28 // (S * kv * D))   # tokens of the longest sequence
        return dict(op=op, dtype=dt, S=S, heads=kv * rng.choice([1, 2, 3, 4, 7, 8, 16]), kv_heads=kv, D=D,
                    page=rng.choice([8, 16, 16, 32, 64, 24]), length=_log_int(rng, 1, max(2, top)), window=rng.choice([0, 0, 0, 500]))
    if op == "quantize":
        K = rng.choice([8 * _log_int(rng, 4, 1000), _log_int(rng, 20, 8000)])
        return dict(op=op, dtype=rng.choice([dt, dt, "f32"]), M=_log_int(rng, 1, min(8192, 2 ** 24 // K)), K=K)
    IN = rng.choice([8 * _log_int(rng, 8, 1000), 64 * _log_int(rng, 2, 120), _log_int(rng, 50, 8000)])
    OUT = rng.choice([8 * _log_int(rng, 8, 1000), _log_int(rng, 50, 8000)])
    B = rng.choice([_log_int(rng, 1, 64), _log_int(rng, 1, 4096)])
    while B > 1 and B * IN * OUT > 4096 * 4096 * 4096:
        B //= 2
    return dict(op=op, dtype=dt, B=B, IN=IN, OUT=OUT, bias=rng.random() < 0.5,
                act=rng.choice(["none", "none", "relu", "hswish"]))


# ---- inputs ------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _lengths(case, g):
    """Ragged lengths up to case["length"]: the first the longest, one empty sequence in a batch of eight and more."""
    n = (torch.rand(case["S"], generator=g, device="cuda") * case["length"]).long() + 1
    n.clamp_(max=case["length"])
    n[0] = case["length"]
    if case["S"] >= 8:
        n[3] = 0
    return n


def _cache(case, g, td, tokens):
    """Keys, values [pages][kv heads][page][D] and a page table of `tokens` tokens a sequence in random pages."""
    per = -(-tokens // case["page"])
    pages = case["S"] * per + 1
    shape = (pages, case["kv_heads"], case["page"], case["D"])
    table = torch.randperm(pages, generator=g, device="cuda")[:case["S"] * per].reshape(case["S"], per).int()
    k = torch.empty(shape, dtype=td, device="cuda")
    v = torch.empty(shape, dtype=td, device="cuda")
    k.normal_(generator=g)
    v.normal_(generator=g)
    return k, v, table


def _make(case, seed):
    """The tensors of a case, on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    td, op = DTYPES[case["dtype"]], case["op"]
    if op == "norm":
        T, D = case["T"], case["D"]
        t = {"branch": (_randn(g, T, D) * 0.5).to(td), "h": (_randn(g, T, D) * 2.0).to(td),
             "post": 1.0 + 0.2 * _randn(g, D) if case["post"] else None, "pre": 1.0 + 0.2 * _randn(g, D)}
        t["gate"] = None if case["gate"] == "none" else (0.5 + 0.3 * _randn(g, T if case["gate"] == "token" else 1, D)).to(td)
        return t
    if op == "append":
        S, T, D, H, KV = case["S"], case["T"], case["D"], case["heads"], case["kv_heads"]
        if T == S:       # a decode step: a token for every sequence
            seq = torch.arange(S, device="cuda")
            pos = (torch.rand(S, generator=g, device="cuda") * case["context"]).long()
        else:            # runs of tokens: every sequence starts somewhere
            seq = torch.randint(0, S, (T,), generator=g, device="cuda").sort().values
            first = torch.searchsorted(seq, torch.arange(S, device="cuda"))
            start = (torch.rand(S, generator=g, device="cuda") * 100).long()
            pos = torch.arange(T, device="cuda") - first[seq] + start[seq]
        longest = max(case["context"], int(pos.max()) + 1)
        k_cache, v_cache, table = _cache(case, g, td, longest)
        t = {"qkv": _randn(g, T, (H + 2 * KV) * D).to(td), "k_cache": k_cache, "v_cache": v_cache, "table": table,
             "seq": seq.int(), "pos": pos.int(), "cos_sin": None}
        if case["rot"]:
            half = case["rot"] // 2
            freq = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
            angle = torch.arange(longest, device="cuda", dtype=torch.float64)[:, None] * freq
            t["cos_sin"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        return t
    if op == "attention":
        n = _lengths(case, g)
        k, v, table = _cache(case, g, td, case["length"])
        q = (_randn(g, case["S"], case["heads"], case["D"]) * 1.5).to(td)
        return {"q": q, "k_cache": k, "v_cache": v, "table": table, "n": n.int()}
    if op == "quantize":
        x = _randn(g, case["M"], case["K"]) * torch.exp(_randn(g, 1, case["K"]))   # channels of unlike sizes
        return {"x": x.to(td)}
    x = (_randn(g, case["B"], case["IN"]) * torch.exp(0.5 * _randn(g, 1, case["IN"]))).to(td)
    w = (_randn(g, case["OUT"], case["IN"]) * math.sqrt(2.0 / case["IN"])).to(td)
    return {"x": x, "w": w, "bias": 0.5 * _randn(g, case["OUT"]) if case["bias"] else None}


def prepare(case, seed):
    t = _make(case, seed)
    t["case"] = case
    td, op = DTYPES[case["dtype"]], case["op"]
    if not own:
        if op == "fc":       # a program in plain form keeps the quantised weights' values
            t["wq"] = _plain_mx(t.pop("w").float())
        return t
    import paper_2012_00596_amd as npas
    t["npas"], t["dt"] = npas, {"f32": npas.F32, "bf16": npas.BF16, "f16": npas.F16}[case["dtype"]]
    if op == "norm":
        t["h_out"], t["n_out"] = torch.empty_like(t["h"]), torch.empty_like(t["h"])
    elif op in ("append", "attention"):
        t["cache"] = npas.KvCache(t["k_cache"], t["v_cache"], t["table"], t["dt"])
        if op == "append":
            t["q_out"] = torch.empty((case["T"], case["heads"], case["D"]), dtype=td, device="cuda")
        else:
            t["y"] = torch.empty_like(t["q"])
            t["bytes"] = npas.paged_attention_workspace_bytes(t["cache"], case["heads"], case["length"])
            t["workspace"] = torch.empty(max(t["bytes"], 256), dtype=torch.uint8, device="cuda")
    elif op == "quantize":
        blocks = -(-case["K"] // BLOCK)
        t["codes"] = torch.empty((case["M"], blocks * BLOCK // 2), dtype=torch.uint8, device="cuda")
        t["scales"] = torch.empty((case["M"], blocks), dtype=torch.uint8, device="cuda")
        t["y"] = torch.empty_like(t["x"])
    else:
        w = t.pop("w").cpu()
        w = w.numpy() if td == torch.float32 else w.view(torch.int16).numpy().view("uint16")
        t["packed"] = npas.pack_fc_mxfp4(w, t["dt"])
        t["y"] = torch.empty((case["B"], case["OUT"]), dtype=td, device="cuda")
        t["bytes"] = t["packed"].workspace_bytes(case["B"])
        t["workspace"] = torch.empty(max(t["bytes"], 256), dtype=torch.uint8, device="cuda")
        t["act"] = {"none": npas.ACT_NONE, "relu": npas.ACT_RELU, "hswish": npas.ACT_HARDSWISH}[case["act"]]
    return t


# ---- the measured call -------------------------------------------------------

def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state, state["case"])


def _split(t, c):
    """Queries, keys and values of the joined projection: views [T][heads][D]."""
    H, KV, D = c["heads"], c["kv_heads"], c["D"]
    q, k, v = t["qkv"].split([H * D, KV * D, KV * D], 1)
    return q, k, v


def _own(t):
    npas, c, s = t["npas"], t["case"], torch.cuda.current_stream().cuda_stream
    if c["op"] == "norm":
        npas.gated_residual_norm(t["branch"], t["h"], t["h_out"], t["n_out"], c["T"], c["D"], t["dt"], gate=t["gate"],
                                 post_weight=t["post"], pre_weight=t["pre"], residual_scale=SCALE, eps=EPS, stream=s)
        return t["h_out"], t["n_out"]
    if c["op"] == "append":
        q, k, v = _split(t, c)
        npas.kv_append(t["cache"], q, k, v, t["q_out"], c["T"], c["heads"], t["pos"], sequences=t["seq"], cos_sin=t["cos_sin"],
                       rot_dim=c["rot"], kind=npas.ROTATE_PAIRS if c["pairs"] else npas.ROTATE_HALVES, stream=s)
        return t["q_out"], t["k_cache"], t["v_cache"]
    if c["op"] == "attention":
        npas.paged_attention(t["cache"], t["q"], t["y"], c["heads"], t["n"], c["length"], c["D"] ** -0.5, window=c["window"],
                             workspace=t["workspace"], workspace_bytes=t["bytes"], stream=s)
        return t["y"]
    if c["op"] == "quantize":
        npas.mxfp4_quantize(t["x"], t["codes"], t["scales"], c["M"], c["K"], t["dt"], stream=s)
        npas.mxfp4_dequantize(t["codes"], t["scales"], t["y"], c["M"], c["K"], t["dt"], stream=s)
        return t["y"]
    npas.fc_mxfp4(t["packed"], t["x"], t["y"], c["B"], t["bias"], t["act"], t["workspace"], t["bytes"], s)
    return t["y"]


# ---- plain forms: elementary operations in 32 bits, one rounding at the end ---

def _plain_norm(t, c):
    td, p = t["h"].dtype, t["branch"].float()
    if t["post"] is not None:
        p = p * torch.rsqrt((p * p).mean(1, keepdim=True) + EPS) * t["post"]
    if t["gate"] is not None:
        p = p * t["gate"].float()
    h = SCALE * t["h"].float() + p
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * t["pre"]
    return h.to(td), n.to(td)


def _plain_rotate(x, cos, sin, rot, pairs):
    """x [T][heads][D] in 32 bits, cos and sin [T][1][rot / 2]."""
    if not rot:
        return x
    half = rot // 2
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :half], x[..., half:rot])
    c, d = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([c, d], -1).flatten(-2) if pairs else torch.cat([c, d], -1)
    return torch.cat([r, x[..., rot:]], -1)


def _plain_append(t, c):
    td, T, D = t["qkv"].dtype, c["T"], c["D"]
    q, k, v = (x.reshape(T, -1, D) for x in _split(t, c))
    pos, cos, sin = t["pos"].long(), None, None
    if c["rot"]:
        cos, sin = t["cos_sin"][pos][:, None].chunk(2, -1)
    q = _plain_rotate(q.float(), cos, sin, c["rot"], c["pairs"]).to(td)
    k = _plain_rotate(k.float(), cos, sin, c["rot"], c["pairs"]).to(td)
    page, slot = t["table"][t["seq"].long(), pos // c["page"]].long(), pos % c["page"]
    t["k_cache"][page, :, slot] = k
    t["v_cache"][page, :, slot] = v
    return q, t["k_cache"], t["v_cache"]


def _plain_attention(t, c):
    S, KV, D, G = c["S"], c["kv_heads"], c["D"], c["heads"] // c["kv_heads"]
    L = t["table"].shape[1] * c["page"]
    q = t["q"].float().reshape(S, KV, G, D)
    y = torch.zeros_like(q)
    j = torch.arange(L, device=q.device)
    step = max(1, 2 ** 29 // (L * KV * D))     # sequences whose keys are held in 32 bits at once
    for s in range(0, S, step):
        e = min(S, s + step)
        table = t["table"][s:e].long()
        k, v = (x[table].float().transpose(2, 3).reshape(e - s, L, KV, D).transpose(1, 2).contiguous() for x in (t["k_cache"], t["v_cache"]))
        n = t["n"][s:e, None]
        seen = j < n
        if c["window"]:
            seen = seen & (j >= n - c["window"])
        score = (q[s:e] * D ** -0.5) @ k.transpose(2, 3).contiguous()
        score = score.masked_fill(~seen[:, None, None], -math.inf)
        top = score.amax(-1, keepdim=True).clamp(min=-1e30)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        y[s:e] = p @ v / total.masked_fill(total == 0, 1.0)
    return y.reshape(S, -1, D).to(t["q"].dtype)


def _plain_mx(x):
    """The values that rows of x (32 bits) stand for in microscaled 4-bit floats: blocks of 32 with one power of two."""
    M, K = x.shape
    x = torch.nn.functional.pad(x, (0, -K % BLOCK)).reshape(M, -1, BLOCK)
    top = x.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top).exponent - 3).clamp(min=-127)          # floor(log2 top) - 2
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    v = torch.ldexp(torch.ldexp(x, -(e // 2)), -(e - e // 2))
    a = v.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    v = torch.copysign(torch.clamp(torch.round(a / step) * step, max=6.0), v)
    return torch.ldexp(torch.ldexp(v, e // 2), e - e // 2).reshape(M, -1)[:, :K]


def _plain_quantize(t, c):
    return _plain_mx(t["x"].float()).to(t["x"].dtype)


def _plain_fc(t, c):
    y = _plain_mx(t["x"].float()) @ t["wq"].t()
    if t["bias"] is not None:
        y = y + t["bias"]
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "hswish":
        y = y * (y + 3).clamp(0, 6) / 6
    return y.to(t["x"].dtype)


_PLAIN = {"norm": _plain_norm, "append": _plain_append, "attention": _plain_attention, "quantize": _plain_quantize, "fc": _plain_fc}


# ---- what a pass cannot do without -------------------------------------------

def _tokens(case):
    """Mean number of cached tokens a pass of attention reads over all its sequences."""
    S, n, w = case["S"], case["length"], case["window"] or case["length"]
    w = min(w, n)
    mean = w * (n - w) / n + w * (w + 1) / (2 * n)               # of min(length, window), lengths uniform in 1 .. n
    return w + (S - 1 - (S >= 8)) * mean


def work(case):
    size, op = 4 if case["dtype"] == "f32" else 2, case["op"]
    if op == "norm":
        T, D = case["T"], case["D"]
        gate = {"none": 0, "channel": D, "token": T * D}[case["gate"]]
        return {"bytes": (4 * T * D + gate) * size + 4 * D * (1 + case["post"]), "flops": T * D * (7 + 4 * case["post"])}
    if op == "append":
        T, D, H, KV = case["T"], case["D"], case["heads"], case["kv_heads"]
        return {"bytes": 2 * T * (H + 2 * KV) * D * size + T * (12 + 4 * case["rot"]), "flops": 3 * T * (H + KV) * case["rot"]}
    if op == "attention":
        n = _tokens(case)
        rows = case["S"] * case["heads"] * case["D"]
        return {"bytes": int(2 * n * case["kv_heads"] * case["D"] * size + 2 * rows * size + n / case["page"] * 4),
                "flops": int(4 * n * case["heads"] * case["D"])}
    if op == "quantize":
        M, K = case["M"], case["K"]
        # in and out once each, and between them the form itself: written and read
        return {"bytes": int(M * K * (2 * size + 2 * 17 / 32)), "flops": 8 * M * K}
    B, IN, OUT = case["B"], case["IN"], case["OUT"]
    return {"bytes": int(OUT * IN * 17 / 32 + B * (IN + OUT) * size + (4 * OUT if case["bias"] else 0)), "flops": 2 * B * IN * OUT}


# ---- 64-bit results ----------------------------------------------------------

def _mx64(x):
    """Microscaled 4-bit values of x from the definition: the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code."""
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=x.device)
    out = torch.empty_like(x)
    for lo in range(0, x.shape[1], BLOCK):
        b = x[:, lo:lo + BLOCK]
        top = b.abs().amax(1, keepdim=True)
        unit = torch.where(top > 0, torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 2), 1.0).clamp(min=2.0 ** -127)
        r = b.abs() / unit
        code = torch.zeros_like(r, dtype=torch.int64)
        for i in range(7):
            mid = (grid[i] + grid[i + 1]) / 2
            code += (r >= mid) if i % 2 else (r > mid)
        out[:, lo:lo + BLOCK] = torch.sign(b) * grid[code] * unit
    return out


def exact(case, seed):
    t, op = _make(case, seed), case["op"]
    if op == "norm":
        p, h = t["branch"].double(), t["h"].double() * SCALE
        if t["post"] is not None:
            p = t["post"].double() * p / torch.sqrt(p.square().sum(1, keepdim=True) / case["D"] + EPS)
        h = h + (p if t["gate"] is None else t["gate"].double() * p)
        return h, t["pre"].double() * h / torch.sqrt(h.square().sum(1, keepdim=True) / case["D"] + EPS)
    if op == "append":
        T, D, H, KV, rot = case["T"], case["D"], case["heads"], case["kv_heads"], case["rot"]
        x = t["qkv"].double().reshape(T, H + 2 * KV, D)
        r = x[:, :H + KV].clone()
        for i in range(rot // 2):
            a, b = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + rot // 2)
            row = t["cos_sin"].double()[t["pos"].long()]
            z = torch.complex(r[..., a], r[..., b]) * torch.complex(row[:, i], row[:, i + rot // 2])[:, None]
            r[..., a], r[..., b] = z.real, z.imag
        k, v = t["k_cache"].double(), t["v_cache"].double()
        at = t["table"].long()[t["seq"].long(), t["pos"].long() // case["page"]] * case["page"] + t["pos"].long() % case["page"]
        for cache, new in ((k, r[:, H:]), (v, x[:, H + KV:])):
            for h in range(KV):
                flat = cache[:, h].reshape(-1, D)
                flat[at] = new[:, h]
                cache[:, h] = flat.reshape(cache[:, h].shape)
        return r[:, :H], k, v
    if op == "attention":
        y = torch.zeros(t["q"].shape, dtype=torch.float64, device="cuda")
        G, D = case["heads"] // case["kv_heads"], case["D"]
        for s, n in enumerate(t["n"].tolist()):
            first = max(0, n - case["window"]) if case["window"] else 0
            if n == 0:
                continue
            pages = t["table"][s, :-(-n // case["page"])].long()
            for h in range(case["kv_heads"]):
                k, v = (c[pages, h].reshape(-1, D)[first:n].double() for c in (t["k_cache"], t["v_cache"]))
                q = t["q"][s, h * G:(h + 1) * G].double()
                y[s, h * G:(h + 1) * G] = torch.softmax(k.matmul(q.t().contiguous()) / math.sqrt(D), 0).t().contiguous().matmul(v)
        return y
    if op == "quantize":
        return _mx64(t["x"].double())
    y = _mx64(t["x"].double()).matmul(_mx64(t["w"].double()).t().contiguous())
    if t["bias"] is not None:
        y = y + t["bias"].double()
    if case["act"] == "relu":
        return torch.relu(y)
    return y * (y + 3).clamp(0, 6) / 6 if case["act"] == "hswish" else y

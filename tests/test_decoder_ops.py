"""The decoder-block operators through the C ABI: norm with gate and residual, append to the paged cache, attention of one token,
against their formulas in 64 bits; and what they refuse.

Tolerances.  Unit roundoffs: 2^-8 (bf16), 2^-11 (fp16), 2^-24 (fp32).  A result is computed in fp32 and rounded once, so it may be off by
its storage type's roundoff of itself plus the fp32 error of its terms: `STEPS` roundoffs of fp32 per unit of the sum of the terms'
magnitudes (64: no sum here adds more than 64 numbers one after another before a tree takes over; a rotation has four roundings)."""
import ctypes

import numpy as np
import pytest

import paper_2012_00596_amd as npas

U = {npas.F32: 2.0 ** -24, npas.BF16: 2.0 ** -8, npas.F16: 2.0 ** -11}
TINY = {npas.F32: 2.0 ** -149, npas.BF16: 2.0 ** -133, npas.F16: 2.0 ** -25}
STEPS = 64 * 2.0 ** -24
gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


def _td(torch, dt):
    return {npas.F32: torch.float32, npas.BF16: torch.bfloat16, npas.F16: torch.float16}[dt]


def _rand(torch, seed, shape, dt, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(_td(torch, dt))


def _close(got, ref, mag, dt, steps=STEPS):
    """|got - ref| within the storage type's rounding of ref plus `steps` of the magnitude of the terms; NaN where ref is NaN."""
    got, ref = got.double().cpu(), ref.double()
    assert got.shape == ref.shape
    nan = ref != ref
    assert bool(((got != got) == nan).all()), "NaN in other places than the formula's"
    bad = ((got - ref).abs() > U[dt] * ref.abs() + TINY[dt] + steps * mag) & ~nan
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((got - ref).abs()[~nan].max())}"


# ---- norm with gate and residual ----------------------------------------------

def _norm64(branch, h, gate, post, pre, scale, eps):
    h = h.double() * scale
    mag = h.abs()
    if branch is not None:
        p = branch.double()
        if post is not None:
            p = p / (p.square().mean(1, keepdim=True) + eps).sqrt() * post.double()
        if gate is not None:
            p = p * gate.double()
        h, mag = h + p, mag + p.abs()
    if pre is None:
        return h, mag, None, None
    r = pre.double() / (h.square().mean(1, keepdim=True) + eps).sqrt()
    n = h * r
    # the mean square is off by the terms' magnitudes too, where they cancel
    spread = (h.abs() * mag).mean(1, keepdim=True) / (h.square().mean(1, keepdim=True) + eps)
    return h, mag, n, mag * r.abs() + n.abs() * (1 + 2 * spread)


NORM = [(1, 1), (3, 7), (5, 64), (2, 511), (4, 512), (7, 1000), (9, 1024), (3, 1280), (2, 2048), (3, 2049), (2, 4096), (3, 5000),
        (1, 8192), (2, 8193), (2, 16384), (2, 16385), (1, 40001)]


@gpu
@pytest.mark.parametrize("T,D", NORM)
@pytest.mark.parametrize("dt", [npas.F32, npas.BF16, npas.F16])
def test_norm_sizes(torch, T, D, dt):
    print(f"norm T={T} D={D} dtype={dt}", flush=True)
    b, h, g = (_rand(torch, 10 + i, (T, D), dt, s) for i, s in enumerate((0.5, 2.0, 0.7)))
    post, pre = _rand(torch, 20, (D,), npas.F32) + 1, _rand(torch, 21, (D,), npas.F32) + 1
    ho = torch.full((T, D), float("nan"), dtype=h.dtype, device="cuda")
    no = torch.full_like(ho, float("nan"))
    npas.gated_residual_norm(b.cuda(), h.cuda(), ho, no, T, D, dt, gate=g.cuda(), post_weight=post.cuda(), pre_weight=pre.cuda(),
                             residual_scale=0.75, eps=1e-5)
    h64, hmag, n64, nmag = _norm64(b, h, g, post, pre, 0.75, 1e-5)
    _close(ho, h64, hmag, dt)
    _close(no, n64, nmag, dt)


@gpu
@pytest.mark.parametrize("D", [72, 1001, 20000])
@pytest.mark.parametrize("branch,post,gate,pre", [(False, False, None, True), (True, False, None, True), (True, True, None, False),
                                                  (True, False, "row", False), (True, True, "row", True), (True, True, "slice", True)])
def test_norm_parts_in_place(torch, D, branch, post, gate, pre):
    """Every part on its own; h_out over h, n_out over branch; a gate that is one row, or rows of a wider tensor."""
    T, dt = 5, npas.BF16
    b = _rand(torch, 1, (T, D), dt) if branch else None
    h = _rand(torch, 2, (T, D), dt)
    wide = _rand(torch, 3, (T, 2 * D + 1), dt)
    g = {None: None, "row": wide[:1, :D].contiguous(), "slice": wide[:, D + 1:]}[gate]
    gd = None if g is None else (wide.cuda()[:, D + 1:] if gate == "slice" else g.cuda())
    w = _rand(torch, 4, (D,), npas.F32) if post else None
    v = _rand(torch, 5, (D,), npas.F32) if pre else None
    bd, hd = (b.cuda() if branch else None), h.cuda()
    no = None if not pre else (bd if branch else torch.empty_like(hd))
    npas.gated_residual_norm(bd, hd, hd, no, T, D, dt, gate=gd, post_weight=None if w is None else w.cuda(),
                             pre_weight=None if v is None else v.cuda(), residual_scale=-1.5, eps=0.0)
    h64, hmag, n64, nmag = _norm64(b, h, g, w, v, -1.5, 0.0)
    _close(hd, h64, hmag, dt)
    if pre:
        _close(no, n64, nmag, dt)


@gpu
def test_norm_zero_rows_infinities_and_unaligned_rows(torch):
    """A row of zeros stays zero (eps keeps the root from zero); an infinity makes its row NaN or infinite as the formula says and no other;
    tensors at the alignment of one element."""
    T, D, dt = 4, 1003, npas.F16
    base = [torch.zeros(T * D + 1, dtype=torch.float16, device="cuda") for _ in range(4)]
    b, h, ho, no = (x[1:].reshape(T, D) for x in base)
    b.copy_(_rand(torch, 6, (T, D), dt))
    h.copy_(_rand(torch, 7, (T, D), dt))
    b[1] = 0
    h[1] = 0
    b[2, 5] = float("inf")
    pre, post = torch.ones(D, device="cuda"), torch.ones(D, device="cuda")
    npas.gated_residual_norm(b, h, ho, no, T, D, dt, post_weight=post, pre_weight=pre, eps=1e-6)
    h64, hmag, n64, nmag = _norm64(b.cpu(), h.cpu(), None, post.cpu(), pre.cpu(), 1.0, 1e-6)
    assert bool((ho[1] == 0).all()) and bool((no[1] == 0).all())
    rows = [0, 1, 3]
    _close(ho[rows], h64[rows], hmag[rows], dt)
    _close(no[rows], n64[rows], nmag[rows], dt)
    assert bool(torch.isnan(ho[2, 5])) and bool(torch.isnan(no[2]).all())
    assert float(base[2][0]) == 0 and float(base[3][0]) == 0


# ---- paged cache ---------------------------------------------------------------

def _rotate64(x, row, rot, pairs):
    x = x.double().clone()
    mag = x.abs()
    half = rot // 2
    a = torch_index(range(0, rot, 2) if pairs else range(half))
    b = torch_index(range(1, rot, 2) if pairs else range(half, rot))
    c, s = row[:, None, :half].double(), row[:, None, half:].double()
    u, v = x[..., a], x[..., b]
    x[..., a], x[..., b] = u * c - v * s, v * c + u * s
    mag[..., a], mag[..., b] = (u * c).abs() + (v * s).abs(), (v * c).abs() + (u * s).abs()
    return x, mag


def torch_index(r):
    import torch
    return torch.tensor(list(r), dtype=torch.long)


APPEND = [  # T, sequences, heads, kv heads, D, rot, pairs, page, dtype
    (1, 1, 1, 1, 8, 8, True, 1, npas.BF16), (1, 1, 4, 2, 64, 64, False, 16, npas.F16), (9, 9, 12, 3, 64, 32, False, 16, npas.BF16),
    (40, 3, 8, 8, 128, 128, False, 16, npas.BF16), (33, 2, 7, 1, 80, 20, False, 7, npas.F16), (50, 4, 6, 2, 96, 48, True, 5, npas.BF16),
    (21, 2, 16, 4, 256, 64, True, 32, npas.F16), (17, 5, 4, 4, 40, 6, True, 3, npas.BF16), (30, 2, 5, 5, 72, 0, False, 24, npas.F16),
    (300, 2, 32, 8, 128, 128, True, 64, npas.BF16), (64, 1, 3, 1, 24, 2, False, 2, npas.BF16)]


@gpu
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append(torch, case):
    """Ragged runs of tokens from a joined projection at odd alignment, padding tokens among them, holes in the page table."""
    T, S, H, KV, D, rot, pairs, page, dt = case
    print(f"append {case}", flush=True)
    rng = np.random.default_rng(T + D)
    columns = -(-(T + 4) // page) + 1
    pages = S * columns + 2
    table = rng.permutation(pages)[:S * columns].reshape(S, columns).astype(np.int32)
    table[0, -1] = -1
    if columns > 2:
        table[S - 1, 1] = pages            # holes: tokens there are not stored
    seq, pos = np.zeros(T, np.int32), np.zeros(T, np.int32)
    fill = [int(x) for x in rng.integers(0, 4, S)]
    for t in range(T):
        seq[t] = s = int(rng.integers(S))
        pos[t] = fill[s]
        fill[s] += 1
    if T > 8:
        pos[2], seq[4], seq[5], pos[7] = -1, -1, S, columns * page + 3      # three padding tokens; one past the table
    positions = columns * page + 8
    joined = _rand(torch, 30 + D, (T, (H + 2 * KV) * D + 3), dt)
    angle = np.arange(positions)[:, None] / 50.0 ** (np.arange(rot // 2) / max(rot, 1))
    cs = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)) if rot else None
    cache0 = [_rand(torch, 40 + i, (pages, KV, page, D), dt) for i in range(2)]
    k, v = cache0[0].cuda(), cache0[1].cuda()
    cache = npas.KvCache(k, v, torch.from_numpy(table).cuda(), dt)
    jd = joined.cuda()
    q_out = torch.full((T, H, D), float("nan"), dtype=jd.dtype, device="cuda")
    cut = lambda x: (x[:, 3:3 + H * D], x[:, 3 + H * D:3 + (H + KV) * D], x[:, 3 + (H + KV) * D:])   # noqa: E731
    qd, kd, vd = cut(jd)
    npas.kv_append(cache, qd, kd, vd, q_out, T, H, torch.from_numpy(pos).cuda(), sequences=torch.from_numpy(seq).cuda(),
                   cos_sin=None if cs is None else cs.cuda(), rot_dim=rot, kind=npas.ROTATE_PAIRS if pairs else npas.ROTATE_HALVES)
    q, kk, vv = (x.reshape(T, -1, D) for x in cut(joined))
    real = (pos >= 0) & (seq >= 0) & (seq < S) & ((pos < positions) | (rot == 0))
    row = cs[torch.from_numpy(np.clip(pos, 0, positions - 1)).long()] if rot else torch.zeros((T, 0))
    q64, qmag = _rotate64(q, row, rot, pairs)
    k64, kmag = _rotate64(kk, row, rot, pairs)
    q64[torch.from_numpy(~real)] = 0
    _close(q_out, q64, qmag, dt)
    want_k, want_v, mag = cache0[0].double(), cache0[1].clone(), torch.zeros_like(cache0[0], dtype=torch.float64)
    old = torch.ones((pages, page), dtype=torch.bool)
    for t in range(T):
        col = int(pos[t]) // page
        if not real[t] or col >= columns or not 0 <= table[seq[t], col] < pages:
            continue
        p, r = int(table[seq[t], col]), int(pos[t]) % page
        want_k[p, :, r], mag[p, :, r], want_v[p, :, r], old[p, r] = k64[t], kmag[t], vv[t], False
    _close(k, want_k, mag, dt)
    assert torch.equal(v.cpu(), want_v)
    keep = old[:, None, :, None].expand_as(want_v)
    assert torch.equal(k.cpu()[keep], cache0[0][keep]), "a row that no token names has changed"


@gpu
def test_append_without_queries_and_in_place(torch):
    T = S = 6
    KV, D, page, dt = 2, 64, 4, npas.F16
    kx, vx, q = (_rand(torch, 50 + i, (T, n, D), dt) for i, n in enumerate((KV, KV, 4)))
    cs = torch.cat([torch.full((9, 16), 0.6), torch.full((9, 16), 0.8)], 1)
    pos = torch.tensor([0, 3, 4, 8, 9, 1], dtype=torch.int32)             # 9 is past the table of angles
    table = torch.arange(S * 3, dtype=torch.int32).reshape(S, 3)
    results = []
    for with_q in (False, True):
        k, v = (torch.zeros((S * 3, KV, page, D), dtype=torch.float16, device="cuda") for _ in range(2))
        cache = npas.KvCache(k, v, table.cuda(), dt)
        qd = q.cuda() if with_q else None
        npas.kv_append(cache, qd, kx.cuda(), vx.cuda(), qd, T, 4, pos.cuda(), cos_sin=cs.cuda(), rot_dim=32)
        results.append((k.cpu(), v.cpu()))
        if with_q:
            want, mag = _rotate64(q, cs[pos.long().clamp(max=8)], 32, False)
            want[4] = 0
            _close(qd, want, mag, dt)
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert bool((results[0][0][4 * 3 + 2] == 0).all())


# ---- attention of one token ------------------------------------------------------

def _attention64(torch, q, k, v, table, lengths, scale, window, max_length):
    """(y, lse, sum p |v|, largest error bound of a score) per row, tokens of missing pages left out."""
    S, H, D = q.shape
    pages, KV, page, _ = k.shape
    y, w = torch.zeros((S, H, D), dtype=torch.float64), torch.zeros((S, H, D), dtype=torch.float64)
    lse, ds = torch.full((S, H), -float("inf"), dtype=torch.float64), torch.zeros((S, H), dtype=torch.float64)
    for s in range(S):
        n = max(0, min(int(lengths[s]), max_length, table.shape[1] * page))
        j = torch.arange(max(0, n - window) if window else 0, n)
        p = table[s].long()[j // page]
        ok = (p >= 0) & (p < pages)
        j, p = j[ok], p[ok]
        if len(j) == 0:
            continue
        kk, vv = k[p, :, j % page].double(), v[p, :, j % page].double()      # [n][KV][D]
        for h in range(H):
            g = h // (H // KV)
            x = kk[:, g] @ q[s, h].double() * scale
            ds[s, h] = float((kk[:, g].abs() @ q[s, h].double().abs()).max() * abs(scale)) * D * 2.0 ** -24
            pr = torch.softmax(x, 0)
            y[s, h], w[s, h] = pr @ vv[:, g], pr @ vv[:, g].abs()
            lse[s, h] = torch.logsumexp(x, 0)
    return y, lse, w, ds


def _check_attention(torch, q, k, v, table, lengths, scale, window, max_length, dt, y, lse):
    ref, lref, w, ds = _attention64(torch, q, k, v, table, lengths, scale, window, max_length)
    # a weight is off by twice its score's error (its own and the sum's), by the exponential's and the sums' fp32 steps and by its
    # rounding to the storage type for the matrix cores; fp16 weights below 2^-14 by 2^-25 of the largest
    few = U[dt] * 1.0 + (lengths.max().item() * 2.0 ** -25 if dt == npas.F16 else 0.0)
    steps = 2 * ds[..., None] + STEPS + few
    got = y.double().cpu()
    assert bool((got[w.sum(-1) == 0] == 0).all()), "a row without tokens is not zero"
    bad = (got - ref).abs() > U[dt] * ref.abs() + TINY[dt] + steps * w
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((got - ref).abs().max())}, NaN {int((got != got).sum())}"
    assert not bool((got != got).any())
    if lse is not None:
        le = lse.double().cpu()
        none = lref == -float("inf")
        assert bool((le[none] == -float("inf")).all())
        # the sum may be formed of rounded weights
        assert bool(((le - lref).abs()[~none] <= ds[~none] + few + STEPS * (1 + lref[~none].abs())).all())


ATTENTION = [  # heads, kv heads, D, page, lengths, window, dtype, holes
    (1, 1, 8, 1, [0, 1, 2, 3], 0, npas.BF16, False),
    (4, 4, 64, 16, [1, 15, 16, 17, 31, 32, 33, 0, 127, 128, 129], 0, npas.F16, False),
    (8, 2, 128, 16, [500, 1, 0, 64, 1000], 0, npas.BF16, False),
    (32, 8, 128, 16, [2047], 0, npas.BF16, False),
    (6, 2, 80, 7, [100, 13, 700, 14], 0, npas.F16, True),
    (20, 1, 128, 24, [333, 48], 0, npas.BF16, False),
    (48, 3, 64, 32, [257, 95], 0, npas.F16, True),
    (40, 1, 96, 5, [77, 301], 0, npas.BF16, True),
    (16, 16, 256, 64, [130, 4, 640], 0, npas.BF16, False),
    (3, 3, 40, 256, [300, 1, 513], 0, npas.F16, False),
    (7, 1, 24, 3, [50, 0, 200], 0, npas.BF16, True),
    (8, 4, 64, 16, [5, 40, 41, 600, 1300, 0], 37, npas.BF16, False),
    (8, 8, 128, 8, [2500, 3, 1031], 512, npas.F16, True),
    (4, 1, 128, 16, [9000], 0, npas.BF16, True),
    (14, 2, 64, 1, [1500, 1499], 1, npas.BF16, False),
]


@gpu
@pytest.mark.parametrize("case", ATTENTION, ids=str)
def test_attention(torch, case):
    _run_attention(torch, case)


def _run_attention(torch, case):
    """Ragged lengths over random pages; everything that no token names is NaN, in the cache and in the workspace; queries are slices of a
    joined projection at odd alignment."""
    H, KV, D, page, lengths, window, dt, holes = case
    print(f"attention {case}", flush=True)
    S, top = len(lengths), max(lengths)
    rng = np.random.default_rng(H + D + page)
    columns = -(-top // page)
    pages = S * columns + 3
    table = torch.from_numpy(rng.permutation(pages)[:S * columns].reshape(S, columns).astype(np.int32))
    n = torch.tensor(lengths, dtype=torch.int32)
    k, v = (torch.full((pages, KV, page, D), float("nan"), dtype=_td(torch, dt)) for _ in range(2))
    for s in range(S):
        for j in range(lengths[s]):
            if not window or j >= lengths[s] - window:
                k[table[s, j // page], :, j % page] = 0
    used = k == 0
    k = torch.where(used, _rand(torch, 60, k.shape, dt, 1.3), k)
    v = torch.where(used, _rand(torch, 61, v.shape, dt), v)
    if holes:
        table[0, columns // 2], table[S - 1, 0] = -1, pages + 7
        table[0, columns - 1] = 2 ** 31 - 1
    wide = _rand(torch, 62, (S, H * D + 5), dt, 1.5)
    q = wide[:, 5:].reshape(S, H, D)
    cache = npas.KvCache(k.cuda(), v.cuda(), table.cuda(), dt)
    need = npas.paged_attention_workspace_bytes(cache, H, top)
    ws = torch.full((max(need, 16) // 4 + 1,), float("nan"), device="cuda")
    outs = []
    for again in range(2):
        y = torch.full((S, H, D), float("nan"), dtype=q.dtype, device="cuda")
        lse = torch.full((S, H), float("nan"), device="cuda")
        npas.paged_attention(cache, wide.cuda()[:, 5:], y, H, n.cuda(), top, D ** -0.5, window=window, lse=lse, workspace=ws,
                             workspace_bytes=need)
        outs.append(y)
    assert torch.equal(outs[0], outs[1]), "two calls differ"
    _check_attention(torch, q, k, v, table, n, D ** -0.5, window, top, dt, y, lse)


CUTS = [  # many cuts and few, every width of a head's rows; one cut of more tokens than are looked up at once
    (8, 8, 64, 16, [6000, 70], 0, npas.F16, False), (4, 2, 256, 16, [5000, 100], 0, npas.BF16, True),
    (16, 8, 64, 16, [2000, 1, 128, 0], 0, npas.BF16, False), (2, 2, 200, 32, [1100, 500, 257], 0, npas.F16, False),
    (2, 1, 8, 16, [5000], 0, npas.F16, True), (12, 4, 96, 16, [3000, 2900], 1000, npas.BF16, False),
    (17, 1, 128, 16, [700, 640], 0, npas.BF16, False), (64, 1, 64, 16, [3000], 0, npas.F16, False)]


@gpu
@pytest.mark.parametrize("case", CUTS, ids=str)
def test_attention_cuts(torch, case):
    _run_attention(torch, case)


@gpu
@pytest.mark.parametrize("H,KV,D,length", [(4, 2, 64, 40), (8, 2, 128, 3000)])
def test_attention_nan_and_infinities_stay_in_their_heads(torch, H, KV, D, length):
    """A NaN key or an infinite value reaches the heads of its group and no other; a sequence whose pages are all missing is zero."""
    dt, S, page = npas.BF16, 3, 16
    columns = -(-length // page)
    k, v = (_rand(torch, 110 + i, (S * columns, KV, page, D), dt) for i in range(2))
    q = _rand(torch, 112, (S, H, D), dt)
    table = torch.arange(S * columns, dtype=torch.int32).reshape(S, columns)
    n = torch.full((S,), length, dtype=torch.int32)
    gone = table.clone()
    gone[1] = -1
    need = npas.paged_attention_workspace_bytes(npas.KvCache(k.cuda(), v.cuda(), table.cuda(), dt), H, length)
    ws = torch.full((max(need, 16) // 4 + 1,), float("nan"), device="cuda")

    def run(k, v, table):
        y, lse = torch.empty((S, H, D), dtype=q.dtype, device="cuda"), torch.empty((S, H), device="cuda")
        npas.paged_attention(npas.KvCache(k.cuda(), v.cuda(), table.cuda(), dt), q.cuda(), y, H, n.cuda(), length, D ** -0.5, lse=lse,
                             workspace=ws, workspace_bytes=need)
        return y.cpu(), lse.cpu()
    clean, _ = run(k, v, table)
    kb, vb = k.clone(), v.clone()
    kb[table[0, columns - 1], 0, 0, 3] = float("nan")
    vb[table[2, 0], 1, 5, 7] = float("inf")
    y, lse = run(kb, vb, gone)
    G = H // KV
    assert bool(torch.isnan(y[0, :G]).all()) and torch.equal(y[0, G:], clean[0, G:])
    assert bool((y[1] == 0).all()) and bool((lse[1] == -float("inf")).all())
    assert bool((~torch.isfinite(y[2, G:2 * G, 7])).all())
    others = [d for d in range(D) if d != 7]
    assert torch.equal(y[2, G:2 * G][:, others], clean[2, G:2 * G][:, others]) and torch.equal(y[2, :G], clean[2, :G])


@gpu
def test_calls_by_address_and_through_ctypes(torch):
    """The same results from tensors, from addresses of contiguous rows, and where an argument goes through ctypes."""
    S, H, KV, D, page, dt, T = 3, 4, 2, 64, 16, npas.F16, 3
    table = torch.arange(S * 2, dtype=torch.int32).reshape(S, 2).cuda()
    q, kx, vx = (_rand(torch, 120 + i, (T, n, D), dt).cuda() for i, n in enumerate((H, KV, KV)))
    pos, n = torch.tensor([0, 5, 20], dtype=torch.int32, device="cuda"), torch.tensor([1, 6, 21], dtype=torch.int32, device="cuda")
    cs = torch.rand((32, D), device="cuda")
    w = torch.rand(H * D, device="cuda")
    g = _rand(torch, 125, (H * D,), dt).cuda()
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    results = []
    for how in ("tensors", "addresses", "ctypes"):
        k, v = (torch.zeros((S * 2, KV, page, D), dtype=torch.float16, device="cuda") for _ in range(2))
        cache = npas.KvCache(k, v, table, dt)
        qo, y, ho, no = (torch.zeros((T, H, D), dtype=torch.float16, device="cuda") for _ in range(4))
        p = (lambda t: t.data_ptr()) if how == "addresses" else (lambda t: t)
        stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream) if how == "ctypes" else torch.cuda.current_stream().cuda_stream
        npas.kv_append(cache, p(q), p(kx), p(vx), p(qo), T, H, p(pos), cos_sin=cs, rot_dim=D, stream=stream)
        npas.paged_attention(cache, p(qo), p(y), H, p(n), 32, 0.125, workspace=p(ws), workspace_bytes=1 << 16, stream=stream)
        npas.gated_residual_norm(p(y), p(q), p(ho), p(no), T, H * D, dt, gate=g, post_weight=p(w), pre_weight=p(w), stream=stream)
        codes, scales, back = torch.zeros((T, H * D // 2), dtype=torch.uint8, device="cuda"), torch.zeros((T, H * D // 32), dtype=torch.uint8, device="cuda"), torch.zeros_like(no)
        npas.mxfp4_quantize(p(no), p(codes), p(scales), T, H * D, dt, stream)
        npas.mxfp4_dequantize(p(codes), p(scales), p(back), T, H * D, dt, stream)
        packed = npas.pack_fc_mxfp4(np.ones((7, H * D), np.float16).view(np.uint16), dt)
        out = torch.zeros((T, 7), dtype=torch.float16, device="cuda")
        npas.fc_mxfp4(packed, p(no), p(out), T, None, npas.ACT_NONE, p(ws), 1 << 16, stream)
        torch.cuda.synchronize()
        results.append([t.cpu() for t in (qo, k, v, y, ho, no, codes, scales, back, out)])
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))
    with pytest.raises(AssertionError):
        npas.kv_append(cache, q[:, :, ::2], kx, vx, qo, T, H, pos)
    with pytest.raises(npas.NpasError) as e:
        npas.paged_attention(cache, q, y, H, n, 0, 1.0)
    assert e.value.code == npas.E_SHAPE


@gpu
def test_attention_lengths_are_cut_and_large_scores(torch):
    """Lengths below zero and beyond max_length or the table; scores of several hundred, where exp of a score itself would overflow."""
    S, H, KV, D, page, dt = 4, 4, 2, 64, 16, npas.BF16
    k, v = (_rand(torch, 70 + i, (S * 6, KV, page, D), dt, 4.0) for i in range(2))
    table = torch.arange(S * 6, dtype=torch.int32).reshape(S, 6)
    q = _rand(torch, 72, (S, H, D), dt, 4.0)
    n = torch.tensor([-5, 1000, 96, 50], dtype=torch.int32)
    cache = npas.KvCache(k.cuda(), v.cuda(), table.cuda(), dt)
    for max_length in (80, 2000):
        y = torch.full((S, H, D), float("nan"), dtype=q.dtype, device="cuda")
        lse = torch.empty((S, H), device="cuda")
        need = npas.paged_attention_workspace_bytes(cache, H, max_length)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        npas.paged_attention(cache, q.cuda(), y, H, n.cuda(), max_length, 1.0, lse=lse, workspace=ws, workspace_bytes=need)
        _check_attention(torch, q, k, v, table, n, 1.0, 0, max_length, dt, y, lse)


@gpu
def test_append_and_attention_beyond_32_bit_offsets(torch):
    """A cache of more than 2^32 elements a tensor, its last pages in use."""
    KV, D, page, H, dt = 8, 128, 16, 8, npas.BF16
    pages = 2 ** 32 // (KV * D * page) + 40
    k, v = (torch.empty((pages, KV, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    last = pages - 20
    table = torch.arange(last, last + 20, dtype=torch.int32).reshape(2, 10).flip(1).contiguous()
    cache = npas.KvCache(k, v, table.cuda(), dt)
    L = 150
    kx, vx = (_rand(torch, 80 + i, (2 * L, KV, D), dt) for i in range(2))
    pos, seq = torch.arange(L, dtype=torch.int32).repeat(2), torch.arange(2, dtype=torch.int32).repeat_interleave(L)
    npas.kv_append(cache, None, kx.cuda(), vx.cuda(), None, 2 * L, H, pos.cuda(), sequences=seq.cuda())
    q, n = _rand(torch, 82, (2, H, D), dt), torch.tensor([L, L - 7], dtype=torch.int32)
    y = torch.empty((2, H, D), dtype=q.dtype, device="cuda")
    need = npas.paged_attention_workspace_bytes(cache, H, L)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    npas.paged_attention(cache, q.cuda(), y, H, n.cuda(), L, D ** -0.5, workspace=ws, workspace_bytes=need)
    ks, vs = (torch.zeros((20, KV, page, D), dtype=torch.bfloat16) for _ in range(2))
    for t in range(2 * L):
        p = int(table[seq[t], pos[t] // page]) - last
        ks[p, :, pos[t] % page], vs[p, :, pos[t] % page] = kx[t], vx[t]
    _check_attention(torch, q, ks, vs, table - last, n, D ** -0.5, 0, L, dt, y, None)


@gpu
def test_attention_of_the_longest_length(torch):
    """2^31 - 1 tokens: one page stands in every place of the table, so that each of its rows counts 2^16 times, the last once less."""
    D, page, places, dt = 8, 2 ** 15, 2 ** 16, npas.F16
    k, v = _rand(torch, 90, (1, 1, page, D), dt), (_rand(torch, 91, (1, 1, page, D), dt) + 1).half()
    q, n = _rand(torch, 92, (1, 1, D), dt), 2 ** 31 - 1
    cache = npas.KvCache(k.cuda(), v.cuda(), torch.zeros((1, places), dtype=torch.int32, device="cuda"), dt)
    need = npas.paged_attention_workspace_bytes(cache, 1, n)
    y, lse = torch.empty((1, 1, D), dtype=torch.float16, device="cuda"), torch.empty((1, 1), device="cuda")
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    npas.paged_attention(cache, q.cuda(), y, 1, torch.tensor([n], dtype=torch.int32).cuda(), n, 0.25, lse=lse, workspace=ws, workspace_bytes=need)
    times = torch.full((page,), float(places), dtype=torch.float64)
    times[-1] -= 1
    p = times * torch.exp(0.25 * k[0, 0].double() @ q[0, 0].double())
    want = p @ v[0, 0].double() / p.sum()
    # a lane adds up to 2^18 weights in turn, a result register 2^16 products: each addition 2^-24 of what is there; then one rounding
    bound = (2 ** 18 + 2 ** 16) * 2.0 ** -24 * (p @ v[0, 0].double().abs() / p.sum()) + 2.0 ** -11 * want.abs()
    assert bool(((y.cpu()[0, 0].double() - want).abs() <= bound).all()), (y, want)
    assert abs(float(lse) - float(torch.log(p.sum()))) <= 2 ** 18 * 2.0 ** -24 + 2.0 ** -20 * 24


@gpu
def test_step_on_a_side_stream_and_in_a_graph(torch):
    """Append, attention and norm on a stream of the caller's, captured once and replayed as positions and lengths move on; every replay
    equals the eager calls."""
    S, H, KV, D, page, dt, top = 3, 8, 2, 64, 16, npas.BF16, 400
    columns = -(-top // page)
    table = torch.randperm(S * columns, generator=torch.Generator().manual_seed(5)).int().reshape(S, columns).cuda()
    k, v = (_rand(torch, 90 + i, (S * columns, KV, page, D), dt).cuda() for i in range(2))
    cache = npas.KvCache(k, v, table, dt)
    joined = torch.zeros((S, (H + 2 * KV) * D), dtype=torch.bfloat16, device="cuda")
    h = _rand(torch, 92, (S, H * D), dt).cuda()
    pos, n = (torch.zeros(S, dtype=torch.int32, device="cuda") for _ in range(2))
    cs = torch.rand((top, D), device="cuda")
    w = torch.rand(H * D, device="cuda")
    q_out, y, ho, no = (torch.empty((S, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(4))
    need = npas.paged_attention_workspace_bytes(cache, H, top)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()

    def step(stream):
        npas.kv_append(cache, joined[:, :H * D], joined[:, H * D:(H + KV) * D], joined[:, (H + KV) * D:], q_out, S, H, pos, cos_sin=cs,
                       rot_dim=D, stream=stream)
        npas.paged_attention(cache, q_out, y, H, n, top, D ** -0.5, workspace=ws, workspace_bytes=need, stream=stream)
        npas.gated_residual_norm(y, h, ho, no, S, H * D, dt, post_weight=w, pre_weight=w, stream=stream)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side.cuda_stream)
    for i in range(4):
        at = torch.tensor([3 + i, 150 + i, 398 - i], dtype=torch.int32)
        joined.copy_(_rand(torch, 100 + i, tuple(joined.shape), dt))
        pos.copy_(at)
        n.copy_(at + 1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (q_out, y, ho, no, k, v)]
        for t in (q_out, y, ho, no):
            t.zero_()
        torch.cuda.synchronize()
        step(side.cuda_stream)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, (q_out, y, ho, no, k, v))), f"replay {i}"


# ---- refusals (no GPU needed: nothing is launched) --------------------------------

def _desc(**kw):
    d = dict(k_dev=4096, v_dev=8192, page_table_dev=256, dtype=npas.BF16, pages=4, page_size=16, kv_heads=2, head_dim=64, sequences=2,
             table_stride=2)
    d.update(kw)
    return npas.KvCacheDesc(**d)


@pytest.mark.parametrize("change,code", [
    (dict(k_dev=None), npas.E_NULL), (dict(v_dev=None), npas.E_NULL), (dict(page_table_dev=None), npas.E_NULL),
    (dict(dtype=npas.F32), npas.E_DTYPE), (dict(dtype=9), npas.E_DTYPE), (dict(pages=0), npas.E_SHAPE), (dict(page_size=0), npas.E_SHAPE),
    (dict(kv_heads=0), npas.E_SHAPE), (dict(kv_heads=3), npas.E_SHAPE), (dict(head_dim=0), npas.E_SHAPE), (dict(head_dim=12), npas.E_SHAPE),
    (dict(head_dim=264), npas.E_SHAPE), (dict(sequences=0), npas.E_SHAPE), (dict(table_stride=0), npas.E_SHAPE),
    (dict(pages=2 ** 30), npas.E_SHAPE), (dict(k_dev=4098), npas.E_SHAPE), (dict(page_table_dev=257), npas.E_SHAPE)])
def test_bad_caches_are_refused(change, code):
    L, c = npas.lib(), _desc(**change)
    assert L.npas_kv_append(c, 64, 256, 64, 128, 64, 128, 64, 1, 4, None, 64, 64, 8, 64, 0, None) == code
    assert L.npas_paged_attention(c, 64, 256, 64, None, 4, 64, 32, 0, 1.0, None, 0, None) == code
    assert L.npas_paged_attention_workspace_bytes(c, 4, 32) == 0


def test_append_refuses():
    L, good = npas.lib(), [_desc(), 64, 256, 64, 128, 64, 128, 64, 1, 4, None, 64, 64, 8, 64, 0, None]
    for at, value, code in [(1, None, npas.E_NULL), (3, None, npas.E_NULL), (5, None, npas.E_NULL), (7, None, npas.E_NULL),
                            (11, None, npas.E_NULL), (12, None, npas.E_NULL), (0, None, npas.E_NULL), (2, 255, npas.E_SHAPE),
                            (4, 127, npas.E_SHAPE), (6, 0, npas.E_SHAPE), (8, 0, npas.E_SHAPE), (8, -3, npas.E_SHAPE), (9, 0, npas.E_SHAPE),
                            (9, 3, npas.E_SHAPE), (13, 0, npas.E_SHAPE), (14, 63, npas.E_SHAPE), (14, 66, npas.E_SHAPE),
                            (14, -2, npas.E_SHAPE), (15, 2, npas.E_SHAPE), (1, 65, npas.E_SHAPE), (10, 66, npas.E_SHAPE)]:
        args = list(good)
        args[at] = value
        assert L.npas_kv_append(*args) == code, (at, value)
        assert npas.last_error()


def test_attention_refuses():
    L, good = npas.lib(), [_desc(), 64, 256, 64, None, 4, 64, 32, 0, 1.0, None, 0, None]
    for at, value, code in [(1, None, npas.E_NULL), (3, None, npas.E_NULL), (6, None, npas.E_NULL), (2, 100, npas.E_SHAPE),
                            (5, 0, npas.E_SHAPE), (5, 5, npas.E_SHAPE), (7, 0, npas.E_SHAPE), (8, -1, npas.E_SHAPE),
                            (9, float("nan"), npas.E_SHAPE), (1, 63, npas.E_SHAPE), (4, 66, npas.E_SHAPE)]:
        args = list(good)
        args[at] = value
        assert L.npas_paged_attention(*args) == code, (at, value)
    long = _desc(pages=70000, table_stride=70000, sequences=1)
    need = L.npas_paged_attention_workspace_bytes(long, 4, 10 ** 6)
    if need:
        for ws, size in ((None, need), (4096, need - 1), (4100, need)):
            assert L.npas_paged_attention(long, 64, 256, 64, None, 4, 64, 10 ** 6, 0, 1.0, ws, size, None) == npas.E_WORKSPACE


def test_norm_refuses():
    L, good = npas.lib(), [64, 64, 64, 16, 64, 64, 1.0, 1e-6, 128, 256, 2, 16, npas.BF16, None]
    for at, value, code in [(1, None, npas.E_NULL), (8, None, npas.E_NULL), (9, None, npas.E_NULL), (5, None, npas.E_NULL),
                            (0, None, npas.E_NULL), (3, 15, npas.E_SHAPE), (7, -1.0, npas.E_SHAPE), (7, float("nan"), npas.E_SHAPE),
                            (10, 0, npas.E_SHAPE), (11, 0, npas.E_SHAPE), (11, 2 ** 25, npas.E_SHAPE), (12, 3, npas.E_DTYPE),
                            (0, 65, npas.E_SHAPE), (4, 66, npas.E_SHAPE)]:
        args = list(good)
        args[at] = value
        assert L.npas_gated_residual_norm(*args) == code, (at, value)


def test_more_threads_than_a_launch_can_have_are_refused():
    L, big = npas.lib(), 2 ** 31 - 1
    for D in (8, 1024, 1280, 4096, 8192, 20000):
        assert L.npas_gated_residual_norm(64, 64, None, 0, None, 64, 1.0, 1e-6, 128, 256, big, D, npas.BF16, None) == npas.E_SHAPE, D
        assert b"threads" in L.npas_last_error()
    assert L.npas_kv_append(_desc(), None, 0, 64, 128, 64, 128, None, big, 2, None, 64, None, 0, 0, 0, None) == npas.E_SHAPE
    assert b"threads" in L.npas_last_error()
    many = _desc(sequences=2 ** 22, table_stride=2 ** 12)           # 2^23 pairs of 2^16 tokens, 32 cuts each
    need = L.npas_paged_attention_workspace_bytes(many, 4, 2 ** 16)
    assert L.npas_paged_attention(many, 64, 256, 64, None, 4, 64, 2 ** 16, 0, 1.0, 4096, need, None) == npas.E_SHAPE
    assert b"threads" in L.npas_last_error()


def test_binding_refuses_tensors_that_do_not_fit():
    import torch
    k = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16)
    table = torch.zeros((2, 2), dtype=torch.int32)
    with pytest.raises(AssertionError):
        npas.KvCache(k, k[:, :1], table, npas.BF16)
    with pytest.raises(AssertionError):
        npas.KvCache(k, k, table.long(), npas.BF16)
    with pytest.raises(AssertionError):
        npas.KvCache(k.transpose(1, 2), k.transpose(1, 2), table, npas.BF16)
    cache = npas.KvCache(k, k, table, npas.BF16)
    pos = torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros((2, 256), dtype=torch.bfloat16)
    with pytest.raises(AssertionError):
        npas.kv_append(cache, rows[:, ::2], rows[:, :128], rows[:, :128], rows, 2, 4, pos)
    with pytest.raises(AssertionError):
        npas.paged_attention(cache, rows[:, :100], rows, 4, pos, 32, 1.0)
    with pytest.raises(AssertionError):
        npas.gated_residual_norm(rows, rows, rows, rows, 2, 256, npas.BF16, gate=torch.zeros((3, 256)))

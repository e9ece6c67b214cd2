"""Causal attention of runs of new tokens over paged caches of 16-bit and 8-bit numbers, against its formula in 64 bits; a prompt in pieces, drafts
and single tokens one after another, as a server makes the calls; refusals.

Tolerances: a score is off by D fp32 roundoffs of its terms' magnitudes, so a weight by twice that of the largest score; it is rounded once to the
storage type (U; fp16 weights are held from 2^11 down, or up to 2^15 until the maximum in use follows, and numbers below 2^-14
are off by up to 2^-25: by 2^-36 of the largest weight, which is 2^11 or more); sums and exponentials STEPS; the result is rounded once."""
import numpy as np
import pytest

import paper_2012_00596_amd as npas
from tests.test_decoder_ops import STEPS, TINY, U, _rand, _td, torch  # noqa: F401

from . import cache8_reference as c8

gpu = pytest.mark.gpu


def _chunk64(torch, q, k, v, table, starts, lengths, scale, window, max_length):
    """(y, lse, sum p |v|, largest error bound of a score) per row of q; NaN in rows of no sequence."""
    T, H, D = q.shape
    pages, KV, page, _ = k.shape
    G = H // KV
    y, w = torch.full((T, H, D), float("nan"), dtype=torch.float64), torch.zeros((T, H, D), dtype=torch.float64)
    lse, ds = torch.full((T, H), float("nan"), dtype=torch.float64), torch.zeros((T, H), dtype=torch.float64)
    for s in range(len(lengths)):
        lo, hi = int(starts[s]), int(starts[s + 1])
        n = max(0, min(int(lengths[s]), max_length, table.shape[1] * page))
        if hi == lo:
            continue
        y[lo:hi], lse[lo:hi] = 0, -float("inf")
        j = torch.arange(n)
        p = table[s].long()[j // page]
        ok = (p >= 0) & (p < pages)
        j, p = j[ok], p[ok]
        at = n - (hi - lo) + torch.arange(hi - lo)
        seen = j <= at[:, None]
        if window:
            seen &= j > at[:, None] - window
        some = seen.any(1)
        if not bool(some.any()):
            continue
        kk, vv = k[p, :, j % page].double(), v[p, :, j % page].double()          # [n][KV][D]
        used = seen.any(0)[:, None, None]                                        # what nobody sees may be NaN
        kk, vv = torch.where(used, kk, 0.0), torch.where(used, vv, 0.0)
        for h in range(H):
            g = h // G
            qq = q[lo:hi, h].double()
            x = (qq @ kk[:, g].t() * scale).masked_fill(~seen, -float("inf"))
            ds[lo:hi, h] = torch.where(seen, qq.abs() @ kk[:, g].abs().t(), 0.0).amax(1) * abs(scale) * D * 2.0 ** -24
            pr = torch.where(some[:, None], torch.softmax(torch.where(some[:, None], x, 0.0), 1), 0.0)
            # (a product with zero weights would spread infinities)
            fin = torch.nan_to_num(vv[:, g], posinf=0.0, neginf=0.0, nan=0.0)
            yy = pr @ fin
            for jj, d in torch.nonzero(~torch.isfinite(vv[:, g])).tolist():
                yy[:, d] += torch.where(seen[:, jj], vv[jj, g, d], 0.0)
            y[lo:hi, h] = yy
            w[lo:hi, h] = pr @ fin.abs()
            lse[lo:hi, h] = torch.logsumexp(x, 1)
    return y, lse, w, ds


def _check(torch, ref, y, lse, dt, most, untouched=None):
    ry, rl, w, ds = ref
    rows = ~torch.isnan(rl[:, 0])                       # of some sequence (a row without tokens has -inf)
    got, le = y.double().cpu(), lse.double().cpu()
    if untouched is not None:
        assert bool((got[~rows] == untouched).all()) and bool((le[~rows] == untouched).all()), "rows of no sequence were written"
    got, le, ry, rl, w, ds = (t[rows] for t in (got, le, ry, rl, w, ds))
    none = rl == -float("inf")
    assert bool((got[none] == 0).all()) and bool((le[none] == -float("inf")).all()), "a row without tokens is not zero"
    odd = ~torch.isfinite(ry)
    assert bool((~torch.isfinite(got[odd])).all()) and bool((got[odd] == ry[odd])[~torch.isnan(ry[odd]) & ~torch.isnan(got[odd])].all())
    steps = 2 * ds[..., None] + STEPS + U[dt] + (most * 2.0 ** -36 if dt == npas.F16 else 0.0)
    bad = ~((got - ry).abs() <= U[dt] * ry.abs() + TINY[dt] + steps * w) & ~odd
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((got - ry).abs()[~odd].nan_to_num(9e9).max())}, first {torch.nonzero(bad)[0].tolist()}"
    fine = ~none
    assert bool(((le - rl).abs()[fine] <= ds[fine] + STEPS * (1 + rl[fine].abs())).all()), "lse"


def _make(torch, case, seed=0):
    """(q rows of a wider tensor, cache, values of k and v, table, starts, lengths): NaN wherever no token lies."""
    H, KV, D, page, runs, window, dt, e8, holes = case
    S, top = len(runs), max(max(n for _, n in runs), 1)
    rng = np.random.default_rng(H + D + page + seed)
    columns = -(-top // page)
    pages = S * columns + 3
    table = torch.from_numpy(rng.permutation(pages)[:S * columns].reshape(S, columns).astype(np.int32))
    used = torch.zeros((pages, page), dtype=torch.bool)
    for s, (new, n) in enumerate(runs):
        j = torch.arange(max(0, n - new - window + 1) if window else 0, n)
        used[table[s].long()[j // page], j % page] = True
    used = used[:, None, :, None].expand(pages, KV, page, 1)
    x = [_rand(torch, seed + 60 + i, (pages, KV, page, D), npas.F32, 1.3 - 0.3 * i) for i in range(2)]
    if e8:
        (k, ks), (v, vs) = (c8.quantise(t.to(_td(torch, dt)).double(), dt) for t in x)
        k, v = (torch.where(used, t, torch.full_like(t, 0x7f)) for t in (k, v))
        ks, vs = (torch.where(used, t, torch.full_like(t, 255)) for t in (ks, vs))
        values = c8.dequantise(k, ks), c8.dequantise(v, vs)
    else:
        k, v = (torch.where(used, t, float("nan")).to(_td(torch, dt)) for t in x)
        values = k, v
    if holes:
        table[0, columns // 2], table[S - 1, 0] = -1, pages + 7
        table[0, columns - 1] = 2 ** 31 - 1
    cache = npas.KvCache8(k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), table.cuda(), dt) if e8 else npas.KvCache(k.cuda(), v.cuda(), table.cuda(), dt)
    starts = torch.tensor([0] + [n for n, _ in runs], dtype=torch.int32).cumsum(0).int()
    return cache, values, table, starts, torch.tensor([n for _, n in runs], dtype=torch.int32), top


def _run(torch, case, before=0, after=0, scale=None):
    H, KV, D, page, runs, window, dt, e8, holes = case
    cache, (k, v), table, starts, n, top = _make(torch, case)
    starts = starts + before
    T = int(starts[-1]) + after
    wide = _rand(torch, 62, (T, H * D + 5), dt, 1.5)
    q = wide[:, 5:].reshape(T, H, D)
    scale = D ** -0.5 if scale is None else scale
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.full((max(need, 16) // 4 + 1,), float("nan"), device="cuda")
    outs = []
    for again in range(2):
        y, lse = torch.full((T, H, D), 7.0, dtype=q.dtype, device="cuda"), torch.full((T, H), 7.0, device="cuda")
        npas.chunk_attention(cache, wide.cuda()[:, 5:], y, T, H, starts.cuda(), n.cuda(), top, scale, window=window, lse=lse, workspace=ws,
                             workspace_bytes=need)
        outs.append((y, lse))
    assert all(torch.equal(a, b) for a, b in zip(*outs)), "two calls differ"
    _check(torch, _chunk64(torch, q, k, v, table, starts, n, scale, window, top), y, lse, dt, top, 7.0)


RUNS = [  # heads, kv heads, D, page, (new tokens, cached with them) a sequence, window, dtype, 8 bits, holes
    (1, 1, 16, 4, [(1, 1)], 0, npas.BF16, False, False),
    (1, 1, 8, 1, [(2, 5), (0, 3), (1, 0), (4, 2)], 0, npas.F16, False, False),
    (4, 4, 64, 16, [(5, 800)], 0, npas.F16, False, False),
    (16, 2, 64, 16, [(3, 130), (1, 129), (0, 40), (4, 4), (2, 700)], 0, npas.BF16, True, False),
    (32, 8, 128, 16, [(5, 500), (1, 1), (7, 64), (4, 1000)], 0, npas.BF16, True, False),
    (32, 8, 128, 16, [(5, 500), (1, 1), (7, 64), (4, 1000)], 0, npas.BF16, False, True),
    (8, 2, 128, 16, [(300, 300), (17, 17), (64, 128), (129, 400)], 0, npas.BF16, False, False),
    (8, 2, 128, 16, [(300, 300), (17, 17), (64, 128), (129, 400)], 0, npas.F16, True, True),
    (7, 1, 80, 24, [(100, 250), (33, 33), (0, 0), (1, 90)], 0, npas.F16, False, True),
    (6, 3, 96, 7, [(70, 70), (65, 129)], 0, npas.BF16, True, False),
    (6, 3, 96, 7, [(70, 70), (65, 129)], 0, npas.BF16, False, False),
    (20, 5, 80, 24, [(200, 500), (90, 91)], 100, npas.F16, True, False),
    (4, 1, 256, 64, [(70, 200), (3, 300)], 0, npas.BF16, False, False),
    (4, 1, 256, 64, [(70, 200), (3, 300)], 0, npas.F16, True, True),
    (2, 2, 256, 16, [(2, 400), (5, 33), (1, 1)], 0, npas.BF16, True, False),
    (3, 3, 200, 5, [(40, 90), (1, 7)], 20, npas.BF16, False, True),
    (2, 1, 72, 3, [(150, 150)], 1, npas.F16, False, False),
    (40, 1, 64, 32, [(9, 100), (30, 30)], 33, npas.BF16, False, False),
    (1, 1, 32, 16, [(257, 257), (128, 1000), (1, 64)], 64, npas.F16, True, False),
    (8, 8, 64, 8, [(128, 128)], 0, npas.BF16, False, False),
    (8, 8, 112, 16, [(65, 700)], 600, npas.F16, False, True),
    (4, 2, 64, 16, [(1, i) for i in range(70)], 0, npas.BF16, False, False),
    (4, 2, 64, 16, [(i % 3, 40) for i in range(200)], 0, npas.F16, True, False),
    (8, 1, 128, 16, [(6, 9000)], 0, npas.BF16, True, False),
    (8, 1, 128, 16, [(6, 9000)], 0, npas.F16, False, True),
    (4, 4, 64, 16, [(130, 5000), (2, 600)], 0, npas.BF16, False, False),
    (4, 4, 64, 16, [(130, 5000), (2, 600)], 1500, npas.F16, True, False),
]


@gpu
@pytest.mark.parametrize("case", RUNS, ids=str)
def test_runs(torch, case):
    """Ragged runs over random pages, NaN wherever no token lies, queries that are slices of a joined projection at odd alignment."""
    print(f"runs {case}", flush=True)
    _run(torch, case)


@gpu
@pytest.mark.parametrize("e8", [False, True])
def test_rows_of_no_sequence_stay(torch, e8):
    for runs in ([(3, 20), (60, 80)], [(1, 2000)], [(0, 5)], [(130, 130), (0, 0)]):
        _run(torch, (8, 2, 64, 16, runs, 0, npas.BF16, e8, False), before=4, after=37)


@gpu
@pytest.mark.parametrize("case", [
    (8, 1, 128, 16, [(6, 9000), (0, 0), (7, 130), (5, 1)], 0, npas.BF16, False, False),
    (8, 1, 64, 16, [(9, 8000), (1, 30)], 5000, npas.F16, True, True),
    (2, 1, 256, 64, [(40, 7000)], 0, npas.BF16, True, False),
    (4, 1, 80, 16, [(4, 9000), (2, 50), (0, 7)], 0, npas.F16, False, True),
    (4, 1, 128, 16, [(3, 9000), (2, 50)], 6000, npas.BF16, True, False)], ids=str)
def test_many_cuts(torch, case):
    """More than 16 cuts, most of them empty for the short sequences; rows of no sequence on both sides."""
    print(f"cuts {case}", flush=True)
    _run(torch, case, before=3, after=5)


@gpu
@pytest.mark.parametrize("scale", [0.0, -0.3, 40.0])
def test_scales_of_every_sign_and_large_scores(torch, scale):
    _run(torch, (4, 2, 64, 16, [(40, 90), (2, 300)], 0, npas.BF16, False, False), scale=scale)


@gpu
@pytest.mark.parametrize("H,KV,D,runs", [(4, 2, 64, [(3, 40), (2, 300)]), (8, 2, 128, [(100, 150), (64, 64)]), (2, 1, 256, [(70, 70), (4, 20)])])
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
def test_infinities_and_nan_reach_the_rows_that_see_them(torch, H, KV, D, runs, dt):
    """An infinite value or a NaN among the new tokens: rows before it do not see it, others of other heads neither; a NaN key likewise."""
    case = (H, KV, D, 16, runs, 0, dt, False, False)
    cache, (k, v), table, starts, n, top = _make(torch, case)
    T = int(starts[-1])
    q = _rand(torch, 5, (T, H, D), dt)
    for s, (new, length) in enumerate(runs):
        for back, what, d in ((new - 1, float("inf"), 3), (new // 2, -float("inf"), D - 1), (1, float("nan"), D // 2)):
            j = length - 1 - back
            v[table[s, j // 16], KV - 1, j % 16, d] = what
    cache = npas.KvCache(k.cuda(), v.cuda(), table.cuda(), dt)
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")

    def call(cache):
        y, lse = torch.empty_like(q, device="cuda"), torch.empty((T, H), device="cuda")
        npas.chunk_attention(cache, q.cuda(), y, T, H, starts.cuda(), n.cuda(), top, D ** -0.5, lse=lse, workspace=ws, workspace_bytes=need)
        return y.cpu(), lse.cpu()
    y, lse = call(cache)
    _check(torch, _chunk64(torch, q, k, v, table, starts, n, D ** -0.5, 0, top), y, lse, dt, top)
    s, j = 0, runs[0][1] - 1                             # the last token's key: the last row of sequence 0 alone sees it
    kb = k.clone()
    kb[table[s, j // 16], 0, j % 16, 7] = float("nan")
    z, _ = call(npas.KvCache(kb.cuda(), v.cuda(), table.cuda(), dt))
    last, G = int(starts[1]) - 1, H // KV
    assert bool(torch.isnan(z[last, :G]).all())
    others = torch.ones(T, H, dtype=torch.bool)
    others[last, :G] = False
    assert torch.equal(torch.nan_to_num(z[others], 5.0), torch.nan_to_num(y[others], 5.0))


@gpu
@pytest.mark.parametrize("e8", [False, True])
@pytest.mark.parametrize("T,n", [(40, 200), (40, 1000), (40, 6000), (3, 200), (3, 1200), (3, 3000)])
def test_nan_scores_make_their_rows_nan(torch, T, n, e8):
    """One cut, some and many: a NaN in a query makes that head's row NaN alone, one in a key every row that sees it, also where a cut has no other score."""
    H, KV, D, page = 8, 1, 64, 16
    case = (H, KV, D, page, [(T, n)], 0, npas.BF16, e8, False)
    cache, _, _, starts, length, top = _make(torch, case)
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.full((max(need, 16) // 4 + 1,), float("nan"), device="cuda")
    q = _rand(torch, 79, (T, H, D), npas.BF16)

    def run(q):
        y, lse = torch.full((T, H, D), 7.0, dtype=q.dtype, device="cuda"), torch.full((T, H), 7.0, device="cuda")
        npas.chunk_attention(cache, q.cuda(), y, T, H, starts.cuda(), length.cuda(), top, 0.125, lse=lse, workspace=ws, workspace_bytes=need)
        return y.cpu(), lse.cpu()

    clean = run(q)
    bad = q.clone()
    bad[1, 5, 7] = float("nan")
    y, lse = run(bad)
    assert bool(torch.isnan(y[1, 5]).all()) and bool(torch.isnan(lse[1, 5]))
    y[1, 5], lse[1, 5] = clean[0][1, 5], clean[1][1, 5]
    assert torch.equal(y, clean[0]) and torch.equal(lse, clean[1])
    # every key up to the middle (whole cuts of them): all later tokens see one
    pages = cache.page_table[0, :n // 2 // page].long()
    if e8:
        cache.k[pages], cache.k_scale[pages] = 0x7f, 255
    else:
        cache.k[pages] = float("nan")
    y, lse = run(q)
    assert bool(torch.isnan(y).all()) and bool(torch.isnan(lse).all())


@gpu
def test_infinite_scores(torch):
    """As for one token: a score of plus infinity makes the row NaN and its lse infinite, minus infinity has no weight, all of them give zero."""
    H = KV = 1
    D, page, dt = 16, 16, npas.BF16
    k, v = torch.zeros((1, 1, page, D), dtype=torch.bfloat16), torch.ones((1, 1, page, D), dtype=torch.bfloat16)
    k[0, 0, :, 0] = torch.tensor([-1e38] * 2 + [0.0] * 2 + [1e38] + [0.0] * 11)
    q = torch.zeros((5, 1, D), dtype=torch.bfloat16)
    q[:, 0, 0] = 1e30
    cache = npas.KvCache(k.cuda(), v.cuda(), torch.zeros((1, 1), dtype=torch.int32).cuda(), dt)
    y, lse = torch.full((5, 1, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((5, 1), 7.0, device="cuda")
    npas.chunk_attention(cache, q.cuda(), y, 5, 1, torch.tensor([0, 5], dtype=torch.int32).cuda(), torch.tensor([5], dtype=torch.int32).cuda(), 5,
                         1.0, lse=lse)
    y, lse = y.cpu(), lse.cpu().flatten()
    assert bool((y[:2] == 0).all()) and lse[:2].tolist() == [-float("inf")] * 2
    assert bool((y[2:4] == 1).all()) and abs(float(lse[3]) - np.log(2)) < 1e-6
    assert bool(torch.isnan(y[4]).all()) and float(lse[4]) == float("inf")


@gpu
def test_lengths_are_cut(torch):
    """Lengths below zero, beyond max_length and beyond the table: runs end where the cut length ends."""
    H, KV, D, page, dt, S = 4, 2, 64, 16, npas.BF16, 4
    k, v = (_rand(torch, 70 + i, (S * 6, KV, page, D), dt, 2.0) for i in range(2))
    table = torch.arange(S * 6, dtype=torch.int32).reshape(S, 6)
    starts, n = torch.tensor([0, 2, 40, 45, 50], dtype=torch.int32), torch.tensor([-5, 1000, 96, 50], dtype=torch.int32)
    q = _rand(torch, 72, (50, H, D), dt, 2.0)
    cache = npas.KvCache(k.cuda(), v.cuda(), table.cuda(), dt)
    for most in (80, 2000):
        y, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full((50, H), 7.0, device="cuda")
        need = npas.chunk_attention_workspace_bytes(cache, 50, H, most)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        npas.chunk_attention(cache, q.cuda(), y, 50, H, starts.cuda(), n.cuda(), most, 1.0, lse=lse, workspace=ws, workspace_bytes=need)
        _check(torch, _chunk64(torch, q, k, v, table, starts, n, 1.0, 0, most), y, lse, dt, most, 7.0)


@gpu
@pytest.mark.parametrize("H", [2, 16])
def test_starts_that_fall_write_no_other_rows(torch, H):
    """No call has such starts; what they give is undefined, but nothing outside y's rows is written."""
    KV, D, page, dt, T = 1, 64, 16, npas.BF16, 40
    k, v = (_rand(torch, 76 + i, (20, KV, page, D), dt) for i in range(2))
    cache = npas.KvCache(k.cuda(), v.cuda(), torch.arange(20, dtype=torch.int32).reshape(4, 5).cuda(), dt)
    q = _rand(torch, 78, (T, H, D), dt).cuda()
    for starts in ([30, 0, 10, 10, 5], [40, 40, 0, 40, 0], [7, -9, 90, 3, 40]):
        y, lse = torch.full((T + 200, H, D), 7.0, dtype=q.dtype, device="cuda"), torch.full((T + 200, H), 7.0, device="cuda")
        npas.chunk_attention(cache, q, y[100:100 + T], T, H, torch.tensor(starts, dtype=torch.int32).cuda(), torch.full((4,), 60, dtype=torch.int32).cuda(),
                             80, 0.1, lse=lse[100:100 + T])
        for x in (y, lse):
            assert bool((x[:100] == 7.0).all()) and bool((x[100 + T:] == 7.0).all())


@gpu
def test_chunk_beyond_32_bit_offsets(torch):
    KV, D, page, H, dt = 8, 128, 16, 8, npas.BF16
    pages = 2 ** 32 // (KV * D * page) + 40
    k, v = (torch.empty((pages, KV, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    last = pages - 20
    table = torch.arange(last, last + 20, dtype=torch.int32).reshape(2, 10).flip(1).contiguous()
    small = [_rand(torch, 80 + i, (20, KV, page, D), dt) for i in range(2)]
    k[last:last + 20], v[last:last + 20] = small[0].cuda(), small[1].cuda()
    cache = npas.KvCache(k, v, table.cuda(), dt)
    starts, n = torch.tensor([0, 90, 93], dtype=torch.int32), torch.tensor([150, 143], dtype=torch.int32)
    q = _rand(torch, 82, (93, H, D), dt)
    y, lse = torch.empty(q.shape, dtype=q.dtype, device="cuda"), torch.empty((93, H), device="cuda")
    need = npas.chunk_attention_workspace_bytes(cache, 93, H, 150)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    npas.chunk_attention(cache, q.cuda(), y, 93, H, starts.cuda(), n.cuda(), 150, D ** -0.5, lse=lse, workspace=ws, workspace_bytes=need)
    _check(torch, _chunk64(torch, q, *small, table - last, starts, n, D ** -0.5, 0, 150), y, lse, dt, 150)


@gpu
@pytest.mark.parametrize("H,KV,D,runs", [(4, 2, 64, [(3, 40), (2, 300)]), (8, 2, 128, [(100, 150), (64, 64)]), (2, 1, 256, [(70, 70), (4, 20)])])
def test_nan_blocks_of_8_bit_values_reach_the_rows_that_see_them(torch, H, KV, D, runs):
    dt = npas.BF16
    cache, _, table, starts, n, top = _make(torch, (H, KV, D, 16, runs, 0, dt, True, False))
    for s, (new, length) in enumerate(runs):
        for back, block in ((new - 1, 0), (1, D // 32 - 1)):
            j = length - 1 - back
            at = (int(table[s, j // 16]), KV - 1, j % 16)
            cache.v[at][32 * block:32 * block + 32] = 0x7f
            cache.v_scale[at][block] = 255
    k, v = c8.dequantise(cache.k.cpu(), cache.k_scale.cpu()), c8.dequantise(cache.v.cpu(), cache.v_scale.cpu())
    T = int(starts[-1])
    q = _rand(torch, 5, (T, H, D), dt)
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    y, lse = torch.empty_like(q, device="cuda"), torch.empty((T, H), device="cuda")
    npas.chunk_attention(cache, q.cuda(), y, T, H, starts.cuda(), n.cuda(), top, D ** -0.5, lse=lse, workspace=ws, workspace_bytes=need)
    ref = _chunk64(torch, q, k, v, table, starts, n, D ** -0.5, 0, top)
    assert bool(torch.isnan(ref[0]).any()) and bool(torch.isfinite(ref[0]).any())
    _check(torch, ref, y, lse, dt, top)


@gpu
@pytest.mark.parametrize("e8", [False, True])
@pytest.mark.parametrize("runs,D", [([(3, 200), (2, 90)], 64), ([(90, 200), (64, 64)], 128), ([(90, 200), (64, 64)], 80), ([(40, 90)], 256)])
def test_missing_pages_bring_nothing_in(torch, runs, D, e8):
    """The first page of the cache, which stands in for what is missing, holds NaN and infinities and is no sequence's."""
    H, KV, page, dt = 4, 2, 16, npas.BF16
    cache, (k, v), table, starts, n, top = _make(torch, (H, KV, D, page, runs, 0, dt, e8, False))
    table = table.clone()
    table[table == 0] = int(max(set(range(k.shape[0])) - set(table.flatten().tolist())))      # (page 0 out of use; its place in another, NaN)
    table[:, 1] = -1
    table[0, 3 % table.shape[1]] = k.shape[0]
    if e8:
        cache.k[0], cache.v[0], cache.k_scale[0], cache.v_scale[0] = 0x7f, 0x7f, 255, 255
        cache = npas.KvCache8(cache.k, cache.v, cache.k_scale, cache.v_scale, table.cuda(), dt)
    else:
        cache.k[0], cache.v[0] = float("nan"), float("inf")
        cache = npas.KvCache(cache.k, cache.v, table.cuda(), dt)
    lost = set((table[s, j]).item() for s in range(len(runs)) for j in range(table.shape[1]))
    for p in lost & set(range(k.shape[0])):                  # pages that nobody wrote in this table's use of them become zeros
        for parts in ((cache.k, cache.v),):
            for t in parts:
                x = t[p].float() if not e8 else None
                if e8:
                    t[p][t[p] == 0x7f] = 0
                else:
                    t[p] = torch.nan_to_num(x, 0.0).to(t.dtype)
        if e8:
            for t in (cache.k_scale, cache.v_scale):
                t[p][t[p] == 255] = 127
    k, v = (c8.dequantise(cache.k.cpu(), cache.k_scale.cpu()), c8.dequantise(cache.v.cpu(), cache.v_scale.cpu())) if e8 else (cache.k.cpu(), cache.v.cpu())
    T = int(starts[-1])
    q = _rand(torch, 5, (T, H, D), dt)
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    y, lse = torch.empty_like(q, device="cuda"), torch.empty((T, H), device="cuda")
    npas.chunk_attention(cache, q.cuda(), y, T, H, starts.cuda(), n.cuda(), top, D ** -0.5, lse=lse, workspace=ws, workspace_bytes=need)
    _check(torch, _chunk64(torch, q, k, v, table, starts, n, D ** -0.5, 0, top), y, lse, dt, top)
    assert bool(torch.isfinite(y).all())


@gpu
@pytest.mark.parametrize("runs", [[(5, 3), (40, 20), (1, 0)], [(3, 400), (200, 260)]])
def test_the_largest_windows_and_runs_longer_than_their_sequence(torch, runs):
    H, KV, D, dt = 4, 2, 64, npas.F16
    cache, (k, v), table, starts, n, top = _make(torch, (H, KV, D, 16, runs, 0, dt, False, False))
    T = int(starts[-1])
    q = _rand(torch, 5, (T, H, D), dt)
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    for window in (1, 2 ** 31 - 1):
        y, lse = torch.empty_like(q, device="cuda"), torch.empty((T, H), device="cuda")
        npas.chunk_attention(cache, q.cuda(), y, T, H, starts.cuda(), n.cuda(), top, 0.1, window=window, lse=lse, workspace=ws, workspace_bytes=need)
        _check(torch, _chunk64(torch, q, k, v, table, starts, n, 0.1, window, top), y, lse, dt, top)


@gpu
@pytest.mark.parametrize("T", [2, 40])
@pytest.mark.parametrize("window", [0, 1000])
def test_runs_at_the_longest_length(torch, T, window):
    """2^31 - 1 tokens, by both forms: one page stands in every place of the table.  A lane adds up to 2^23 weights in turn, each addition 2^-24 of what
    is there: half of the sum at most."""
    D, page, places, dt = 16, 2 ** 15, 2 ** 16, npas.F16
    k, v = _rand(torch, 90, (1, 1, page, D), dt), (_rand(torch, 91, (1, 1, page, D), dt) + 1).half()
    q, n = _rand(torch, 92, (T, 1, D), dt), 2 ** 31 - 1
    cache = npas.KvCache(k.cuda(), v.cuda(), torch.zeros((1, places), dtype=torch.int32, device="cuda"), dt)
    need = npas.chunk_attention_workspace_bytes(cache, T, 1, n)
    y, lse = torch.empty((T, 1, D), dtype=torch.float16, device="cuda"), torch.empty((T, 1), device="cuda")
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    npas.chunk_attention(cache, q.cuda(), y, T, 1, torch.tensor([0, T], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda(), n, 0.25,
                         window=window, lse=lse, workspace=ws, workspace_bytes=need)
    x = torch.exp(0.25 * q[:, 0].double() @ k[0, 0].double().t())             # [T][page]
    for t in range(T):
        at = n - T + t
        if window:
            times = torch.bincount(torch.arange(at - window + 1, at + 1) % page, minlength=page).double()
        else:
            times = torch.full((page,), float((at + 1) // page), dtype=torch.float64)
            times[:(at + 1) % page] += 1
        p = times * x[t]
        want, mag = p @ v[0, 0].double() / p.sum(), p @ v[0, 0].double().abs() / p.sum()
        assert bool(((y[t, 0].double().cpu() - want).abs() <= (2 ** -10 if window else 0.5) * mag).all()), (t, y[t, 0], want)
        assert abs(float(lse[t]) - float(torch.log(p.sum()))) <= (1e-4 if window else 0.5)


@gpu
def test_two_streams_at_once(torch):
    """Prompts and drafts on two streams, a workspace each, many times over: what one stream alone gives."""
    cases = [(8, 2, 128, 16, [(200, 600), (30, 30)], 0, npas.BF16, False, False), (8, 2, 128, 16, [(3, 3000), (2, 900)], 0, npas.BF16, True, False)]
    made = []
    for case in cases:
        cache, _, _, starts, n, top = _make(torch, case)
        T, H, D = int(starts[-1]), case[0], case[2]
        need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
        made.append((cache, _rand(torch, 5, (T, H, D), case[6]).cuda(), torch.empty((T, H, D), dtype=torch.bfloat16, device="cuda"), T, H, starts.cuda(), n.cuda(),
                     top, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), need, torch.cuda.Stream()))

    def call(cache, q, y, T, H, starts, n, top, ws, need, stream):
        npas.chunk_attention(cache, q, y, T, H, starts, n, top, 0.09, workspace=ws, workspace_bytes=need, stream=stream.cuda_stream)
    torch.cuda.synchronize()
    alone = []
    for m in made:
        call(*m)
        torch.cuda.synchronize()
        alone.append(m[2].clone())
        m[2].zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for m in made:
            call(*m)
    torch.cuda.synchronize()
    assert all(torch.equal(a, m[2]) for a, m in zip(alone, made))


# ---- together ----------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("e8", [False, True])
def test_a_server_s_calls_in_a_graph(torch, e8):
    """Prompts in pieces, then drafts, then single tokens: each step writes keys and values with norms and rotation, then attends; once on a side stream,
    once captured and replayed with other tokens, positions, partings and lengths, and against the formulas over what the cache holds."""
    S, H, KV, D, page, dt, top, T = 3, 8, 2, 64, 16, npas.BF16, 400, 96
    columns = -(-top // page)
    table = torch.randperm(S * columns, generator=torch.Generator().manual_seed(5)).int().reshape(S, columns)
    shape = (S * columns, KV, page, D)
    if e8:
        parts = [torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2)] + \
            [torch.full(shape[:3] + (2,), 127, dtype=torch.uint8, device="cuda") for _ in range(2)]
        cache = npas.KvCache8(*parts, table.cuda(), dt)
    else:
        parts = [torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        cache = npas.KvCache(*parts, table.cuda(), dt)
    joined = torch.zeros((T, (H + 2 * KV) * D), dtype=torch.bfloat16, device="cuda")
    seq, pos = (torch.full((T,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    starts, n = torch.zeros(S + 1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    cs, w = torch.rand((top, D), device="cuda"), torch.rand(D, device="cuda") + 0.5
    q_out, y = (torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.zeros((T, H), device="cuda")
    one_q, one_y = (torch.zeros((S, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    attend = npas.paged_attention8 if e8 else npas.paged_attention
    one_need = (npas.paged_attention8_workspace_bytes if e8 else npas.paged_attention_workspace_bytes)(cache, H, top)
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.empty(max(need, one_need, 16), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()

    def step(stream):
        npas.kv_write(cache, joined[:, :H * D], joined[:, H * D:(H + KV) * D], joined[:, (H + KV) * D:], q_out, T, H, pos, sequences=seq,
                      q_weight=w, k_weight=w, cos_sin=cs, rot_dim=D, stream=stream)
        npas.chunk_attention(cache, q_out, y, T, H, starts, n, top, D ** -0.5, lse=lse, workspace=ws, workspace_bytes=need, stream=stream)
        attend(cache, one_q, one_y, H, n, top, D ** -0.5, workspace=ws, workspace_bytes=one_need, stream=stream)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(side.cuda_stream)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(side.cuda_stream)
    filled = [0] * S
    for i, new in enumerate([(60, 10, 26), (1, 80, 15), (4, 5, 3), (0, 1, 7), (1, 1, 1), (90, 0, 2)]):
        places = [(s, filled[s] + j) for s in range(S) for j in range(new[s])]
        filled = [f + c for f, c in zip(filled, new)]
        joined.copy_(_rand(torch, 100 + i, tuple(joined.shape), dt))
        pad = T - len(places)
        seq.copy_(torch.tensor([p[0] for p in places] + [-1] * pad, dtype=torch.int32))
        pos.copy_(torch.tensor([p[1] for p in places] + [0] * pad, dtype=torch.int32))
        starts.copy_(torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32))
        n.copy_(torch.tensor(filled, dtype=torch.int32))
        one_q.copy_(_rand(torch, 200 + i, tuple(one_q.shape), dt))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [t.clone() for t in (q_out, y, lse, one_y, *parts)]
        for t in (q_out, y, lse, one_y):
            t.zero_()
        torch.cuda.synchronize()
        step(side.cuda_stream)
        side.synchronize()
        live = len(places)
        for a, b in zip(replayed[:3], (q_out, y, lse)):
            assert torch.equal(a[:live], b[:live]), f"replay {i}"
        assert all(torch.equal(a, b) for a, b in zip(replayed[3:], (one_y, *parts))), f"replay {i}"
        assert bool((y[live:] == 0).all()) and bool((q_out[live:] == 0).all())
        held = [p.cpu() for p in parts]
        k, v = (c8.dequantise(held[0], held[2]), c8.dequantise(held[1], held[3])) if e8 else held
        ref = _chunk64(torch, q_out.cpu(), k, v, table, starts.cpu(), n.cpu(), D ** -0.5, 0, top)
        _check(torch, ref, y, lse, dt, top, 0.0)


@gpu
def test_one_token_as_a_run_is_the_decode_step(torch):
    """A run of one token and the call for one token: the same formula, within both tolerances; calls by address and through ctypes."""
    import ctypes
    for e8 in (False, True):
        case = (8, 2, 128, 16, [(1, 300), (1, 1), (1, 77)], 0, npas.BF16, e8, False)
        cache, (k, v), table, starts, n, top = _make(torch, case)
        q = _rand(torch, 3, (3, 8, 128), npas.BF16)
        qd, nd, sd = q.cuda(), n.cuda(), starts.cuda()
        need = npas.chunk_attention_workspace_bytes(cache, 3, 8, top)
        ws = torch.empty(max(need, 1 << 20), dtype=torch.uint8, device="cuda")
        outs = []
        stream = torch.cuda.current_stream().cuda_stream
        for how in ("tensors", "addresses", "ctypes"):
            p = (lambda t: t.data_ptr()) if how == "addresses" else (lambda t: t)
            y, one = (torch.empty((3, 8, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            st = ctypes.c_void_p(stream) if how == "ctypes" else stream
            npas.chunk_attention(cache, p(qd), p(y), 3, 8, p(sd), p(nd), top, 0.09, workspace=p(ws), workspace_bytes=1 << 20, stream=st)
            (npas.paged_attention8 if e8 else npas.paged_attention)(cache, p(qd), p(one), 8, p(nd), top, 0.09, workspace=p(ws),
                                                                    workspace_bytes=1 << 20, stream=st)
            outs.append((y.cpu(), one.cpu()))
        assert all(torch.equal(a, b) for o in outs[1:] for a, b in zip(outs[0], o))
        ry, _, w, ds = _chunk64(torch, q, k, v, table, starts, n, 0.09, 0, top)
        bound = U[npas.BF16] * ry.abs() + (2 * ds[..., None] + STEPS + U[npas.BF16]) * w
        for y in outs[0]:
            assert bool(((y.double() - ry).abs() <= bound).all())


# ---- refusals (no GPU needed: nothing is launched) --------------------------------

def _desc(**kw):
    d = dict(k_dev=4096, v_dev=8192, page_table_dev=256, dtype=npas.BF16, pages=4, page_size=16, kv_heads=2, head_dim=64, sequences=2, table_stride=2)
    d.update(kw)
    return npas.KvCacheDesc(**d)


def test_chunk_refuses():
    L, good = npas.lib(), [_desc(), None, 64, 256, 64, None, 3, 4, 64, 64, 32, 0, 1.0, None, 0, None]
    for at, value, code in [(0, None, npas.E_NULL), (2, None, npas.E_NULL), (4, None, npas.E_NULL), (8, None, npas.E_NULL), (9, None, npas.E_NULL),
                            (3, 100, npas.E_SHAPE), (6, 0, npas.E_SHAPE), (6, -1, npas.E_SHAPE), (7, 0, npas.E_SHAPE), (7, 5, npas.E_SHAPE),
                            (10, 0, npas.E_SHAPE), (11, -1, npas.E_SHAPE), (12, float("nan"), npas.E_SHAPE), (2, 63, npas.E_SHAPE),
                            (4, 65, npas.E_SHAPE), (5, 66, npas.E_SHAPE), (8, 66, npas.E_SHAPE), (9, 66, npas.E_SHAPE), (6, 2 ** 31 - 1, npas.E_SHAPE)]:
        args = list(good)
        args[at] = value
        assert L.npas_chunk_attention(*args) == code, (at, value)
        assert npas.last_error()
    long = _desc(pages=70000, table_stride=70000, sequences=1)
    need = L.npas_chunk_attention_workspace_bytes(long, None, 3, 4, 10 ** 6)
    assert need
    for ws, size in ((None, need), (4096, 15), (4100, need)):
        assert L.npas_chunk_attention(long, None, 64, 256, 64, None, 3, 4, 64, 64, 10 ** 6, 0, 1.0, ws, size, None) == npas.E_WORKSPACE
    assert L.npas_chunk_attention_workspace_bytes(long, None, 0, 4, 10 ** 6) == 0
    assert L.npas_chunk_attention_workspace_bytes(long, None, 3, 4, 0) == 0


def test_the_workspace_is_enough_for_every_window_and_parting():
    """bytes of a call without its workspace (its refusal names them) never pass what is asked for."""
    L = npas.lib()
    for S, T, kv, heads, D, top in [(1, 1, 1, 1, 64, 10 ** 6), (1, 5, 1, 8, 128, 9000), (3, 500, 8, 32, 128, 70000), (64, 64, 8, 32, 256, 4000),
                                    (2, 2048, 2, 4, 80, 30000), (200, 300, 1, 1, 64, 500)]:
        c = _desc(pages=70000, table_stride=70000, sequences=S, kv_heads=kv, head_dim=D)
        have = L.npas_chunk_attention_workspace_bytes(c, None, T, heads, top)
        for window in (0, 1, 100, 255, 256, 257, 300, 1000, 4096, 20000, 10 ** 6):
            rc = L.npas_chunk_attention(c, None, 64, heads * D, 64, None, T, heads, 64, 64, top, window, 1.0, None, 0, None)
            if rc == npas.E_WORKSPACE:
                assert int(L.npas_last_error().split(b"needs ")[1].split()[0]) <= have, (S, T, window)


def _fit(torch):
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t)     # noqa: E731
    T, H, KV, D, S, I32, F32, U8 = 5, 4, 2, 64, 3, torch.int32, torch.float32, torch.uint8
    c8_ = npas.KvCache8(z(9, KV, 16, D, t=U8), z(9, KV, 16, D, t=U8), z(9, KV, 16, 2, t=U8), z(9, KV, 16, 2, t=U8), z(S, 3, t=I32), npas.BF16)
    write = dict(cache=c8_, q=z(T, H, D), k=z(T, KV, D), v=z(T, KV, D), q_out=z(T, H, D), T=T, heads=H, positions=z(T, t=I32), sequences=z(T, t=I32),
                 q_weight=z(D, t=F32), k_weight=z(D, t=F32), eps=1e-6, cos_sin=z(9, D, t=F32), rot_dim=D, kind=npas.ROTATE_HALVES, stream=None)
    read = dict(cache=c8_, k=z(T, KV, D), v=z(T, KV, D), T=T, positions=z(T, t=I32), sequences=z(T, t=I32), stream=None)
    decode = dict(cache=c8_, q=z(S, H * D), y=z(S, H, D), heads=H, lengths=z(S, t=I32), max_length=32, scale=1.0, window=0, lse=z(S, H, t=F32),
                  workspace=z(64, t=U8), workspace_bytes=64, stream=None)
    chunk = dict(cache=c8_, q=z(T, H * D), y=z(T, H, D), T=T, heads=H, starts=z(S + 1, t=I32), lengths=z(S, t=I32), max_length=32, scale=1.0, window=0,
                 lse=z(T, H, t=F32), workspace=z(64, t=U8), workspace_bytes=64, stream=None)
    b = npas.binding
    calls = {"write": (npas.kv_write, b._kv_write, write, dict(kind=2)), "read": (npas.kv_read, b._kv_read, read, dict(T=0)),
             "decode": (npas.paged_attention8, b._paged_attention8, decode, dict(max_length=0)),
             "chunk": (npas.chunk_attention, b._chunk_attention, chunk, dict(max_length=0))}
    short, size, rows, index, fp32 = "shorter", "element size", "fewer rows", "32-bit integers", "not fp32"
    bad = {"write": [("q", z(T - 1, H, D), rows), ("k", z(1, KV, D), rows), ("v", z(T, KV, D, t=F32), size), ("q_out", z(T - 1, H, D), short),
                     ("positions", z(T, t=torch.int64), size), ("sequences", z(T, t=F32), index), ("q_weight", z(D - 1, t=F32), short),
                     ("k_weight", z(D), size), ("k_weight", z(D, t=I32), fp32), ("cos_sin", z(9, D), size), ("cos_sin", z(9, D, t=I32), fp32)],
           "read": [("k", z(T - 1, KV, D), short), ("v", z(T, KV, D, t=F32), size), ("positions", z(T - 1, t=I32), short),
                    ("sequences", z(T, t=F32), index)],
           "decode": [("q", z(S - 1, H * D), rows), ("y", z(S, H, D, t=F32), size), ("lengths", z(1, t=I32), short), ("lse", z(S, t=F32), short),
                      ("workspace", z(63, t=U8), short)],
           "chunk": [("q", z(T - 1, H * D), rows), ("y", z(T - 1, H, D), short), ("starts", z(S, t=I32), short), ("starts", z(S + 1, t=F32), index),
                     ("lengths", z(S, t=torch.int64), size), ("lse", z(T, H), size), ("workspace", z(63, t=U8), short)]}
    return calls, bad


@pytest.mark.parametrize("through_ctypes", [False, True])
@pytest.mark.parametrize("name", ["write", "read", "decode", "chunk"])
def test_tensors_that_do_not_fit_are_refused(name, through_ctypes):
    import torch
    calls, bad = _fit(torch)
    call, direct, args, refused = calls[name]
    run = (lambda a: direct(*a.values())) if through_ctypes else (lambda a: call(**a))
    for key, value, why in bad[name]:
        with pytest.raises(AssertionError, match=why):
            run({**args, key: value})
    with pytest.raises(npas.NpasError) as e:              # as they are they reach the library, whose own refusal tells
        run({**args, **refused})
    assert e.value.code == npas.E_SHAPE

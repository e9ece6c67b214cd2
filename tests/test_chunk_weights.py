"""Attention of runs where a weight's last bits, an infinite value or a single token decide: as test_attention_weights has it for one token.  By the mean
run (of heads that share none) 2 rows go through the kernel of short runs with one group of rows, 20 with two, 40 and 150 through tiles.

Bounds: those of test_attention_weights.  Parts of a bf16 weight are taken so that it counts as larger by up to u (2^-24) of itself: 10.4 u + u, still within 12.
A fp16 weight is two parts, the first below it by up to 2^-10, the second off by 2^-12 of that: 4 u more."""
import numpy as np
import pytest

import paper_2012_00596_amd as npas
from tests import test_chunk_attention as runs
from tests.test_attention_weights import TINY, U, _cancelling, _counts, _counts_hold, _outside, _round, _td, torch, u  # noqa: F401

from . import cache8_reference as c8

gpu = pytest.mark.gpu
MORE = {npas.BF16: 0, npas.F16: 4}


def _runs(torch, dt, q, k, v, page, lengths, scale, window=0, e8=False):
    """q [S][T][H][D]: the last T tokens of each sequence; k, v [S][tokens][KV][D] laid into pages in random order -> y, lse [S][T][..] on the CPU."""
    S, T, H, D = q.shape
    tokens, KV = k.shape[1:3]
    columns = -(-tokens // page)
    order = torch.from_numpy(np.random.default_rng(tokens).permutation(S * columns))
    pages = []
    for x in (k, v):
        full = torch.zeros((S, columns * page, KV, D), dtype=torch.float64)
        full[:, :tokens] = x
        full = full.reshape(S * columns, page, KV, D).transpose(1, 2)
        out = torch.empty_like(full)
        out[order] = full
        pages.append(out.contiguous())
    table = order.int().reshape(S, columns).cuda()
    if e8:
        (kc, ks), (vc, vs) = (c8.quantise(x, dt) for x in pages)
        cache = npas.KvCache8(kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda(), table, dt)
    else:
        cache = npas.KvCache(*(x.to(_td(torch, dt)).cuda() for x in pages), table, dt)
    starts, n = torch.arange(S + 1, dtype=torch.int32, device="cuda") * T, torch.tensor(lengths, dtype=torch.int32, device="cuda")
    need = npas.chunk_attention_workspace_bytes(cache, S * T, H, max(lengths))
    ws = torch.full((max(need, 16) // 4 + 1,), float("nan"), device="cuda")
    y = torch.full((S * T, H, D), float("nan"), dtype=_td(torch, dt), device="cuda")
    lse = torch.full((S * T, H), float("nan"), device="cuda")
    npas.chunk_attention(cache, q.to(_td(torch, dt)).reshape(S * T, H, D).cuda(), y, S * T, H, starts, n, max(lengths), scale, window=window, lse=lse,
                         workspace=ws, workspace_bytes=need)
    return y.double().cpu().reshape(S, T, H, D), lse.double().cpu().reshape(S, T, H)


def _weights(torch, dt, T, D, where, steps):
    S, H = 4, 8
    x, v3, ref, w = _cancelling(torch, dt, S, H, D, 1)
    n = where[-1] + 1 + T
    k, v = torch.zeros((S, n, H, D), dtype=torch.float64), torch.zeros((S, n, H, D), dtype=torch.float64)
    k[..., 0] = -200.0                                   # the other tokens: exp(-200) is zero in fp32
    for i, j in enumerate(where):
        k[:, j, :, 0], v[:, j] = x[:, i], v3[:, i]
    q = torch.zeros((S, T, H, D), dtype=torch.float64)
    q[..., 0] = 1
    y, _ = _runs(torch, dt, q, k, v, 16, [n] * S, 1.0)
    bad = _outside(y, ref[:, None], w[:, None], dt, steps + MORE[dt])
    assert int(bad.sum()) == 0, f"{int(bad.sum())} of {bad.numel()} off, worst {float(((y - ref[:, None]).abs() / w[:, None]).max() / u)} steps"


WHERE = [(64, (0, 1, 2), 12), (96, (0, 1, 2), 12), (128, (0, 1, 2), 12), (256, (0, 1, 2), 12), (80, (5, 40, 90), 12), (64, (3, 2500, 5990), 24),
         (128, (100, 1000, 4999), 24), (256, (100, 1000, 4999), 24)]


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
@pytest.mark.parametrize("D,where,steps", WHERE)
@pytest.mark.parametrize("T", [40, 150])
def test_weights_keep_the_bits_of_fp32_in_tiles(torch, dt, T, D, where, steps):
    _weights(torch, dt, T, D, where, steps)


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
@pytest.mark.parametrize("D,where,steps", WHERE)
@pytest.mark.parametrize("T", [2, 20])
def test_weights_keep_the_bits_of_fp32_in_short_runs(torch, dt, T, D, where, steps):
    _weights(torch, dt, T if D <= 128 else T // 2, D, where, steps)


def _strict(torch, ref, y, lse, dt, most, untouched=None):
    """_check without an allowance for a weight's rounding to the storage type: 320 u for sums as in test_attention_weights (a lane's sums in turn, of up to some
    2500 weights here, are off by the root of their number), the fp16 parts' 4 u, and what is lost below 2^-36 of the largest weight."""
    ry, rl, w, ds = ref
    rows = ~torch.isnan(rl[:, 0])
    got, le = y.double().cpu(), lse.double().cpu()
    if untouched is not None:
        assert bool((got[~rows] == untouched).all()) and bool((le[~rows] == untouched).all()), "rows of no sequence were written"
    got, le, ry, rl, w, ds = (t[rows] for t in (got, le, ry, rl, w, ds))
    none = rl == -float("inf")
    assert bool((got[none] == 0).all()) and bool((le[none] == -float("inf")).all())
    assert bool(torch.isfinite(ry).all())
    steps = 2 * ds[..., None] + (320 + MORE[dt]) * u + (most * 2.0 ** -36 if dt == npas.F16 else 0.0)
    bad = ~((got - ry).abs() <= U[dt] * ry.abs() + TINY[dt] + steps * w)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((got - ry).abs().max())}"
    assert bool(((le - rl).abs()[~none] <= ds[~none] + 320 * u + 4 * u * rl[~none].abs()).all())


def _is_short(case):
    """Whether a case of runs.RUNS goes through the kernel of short runs."""
    H, KV, _, _, new = case[:5]
    mean = -(-sum(n for n, _ in new) * (H // KV) // len(new))
    return mean <= 32


@gpu
@pytest.mark.parametrize("case", [c for c in runs.RUNS if not _is_short(c)], ids=str)
def test_runs_in_tiles_without_an_allowance_for_rounded_weights(torch, monkeypatch, case):
    monkeypatch.setattr(runs, "_check", _strict)
    runs._run(torch, case)


@gpu
@pytest.mark.parametrize("case", [c for c in runs.RUNS if _is_short(c)], ids=str)
def test_short_runs_without_an_allowance_for_rounded_weights(torch, monkeypatch, case):
    monkeypatch.setattr(runs, "_check", _strict)
    runs._run(torch, case)


@gpu
@pytest.mark.parametrize("T,D", [(2, 64), (20, 128), (2, 256), (40, 64), (150, 128), (30, 256)])
@pytest.mark.parametrize("n,e8", [(600, False), (600, True), (6000, False)])
def test_large_bf16_values_beside_scores_that_grow(torch, T, D, n, e8):
    """Values of 2^114 to 2^115 whose weights sum to their number at most: 2^13 2^115 is a number of fp32.  Scores grow by 5.5 halfway, a factor of 245 that a maximum
    need not follow.  An exponent is off by 2.44 u and u 8, a sum's roundings are as many as test_attention_weights' 320 u has."""
    S, H = 2, 2
    g = torch.Generator().manual_seed(4)
    k, v = torch.zeros((S, n, H, D), dtype=torch.float64), 2.0 ** 114 * (1 + _round(torch, torch.rand((S, n, H, D), generator=g, dtype=torch.float64), npas.BF16))
    v = _round(torch, v, npas.BF16)
    if e8:
        v = c8.dequantise(*c8.quantise(v, npas.BF16))
    k[:, n // 2:, :, 0] = 5.5
    q = torch.zeros((S, T, H, D), dtype=torch.float64)
    q[..., 0] = 1
    y, lse = _runs(torch, npas.BF16, q, k, v, 16, [n] * S, 1.0, e8=e8)
    for t in range(T):
        seen = n - T + t + 1
        p = torch.softmax(k[:, :seen, :, 0], 1)[..., None]
        ref = (p * v[:, :seen]).sum(1)
        assert not bool(_outside(y[:, t], ref, ref, npas.BF16, 320).any()), t
        assert float((lse[:, t] - torch.logsumexp(k[:, :seen, :, 0], 1)).abs().max()) <= 320 * u


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
@pytest.mark.parametrize("H,KV,D,T,n,window", [
    (4, 2, 64, 2, 40, 0), (8, 2, 128, 3, 300, 0), (2, 1, 96, 10, 3000, 0), (4, 2, 64, 14, 2500, 700), (4, 2, 256, 3, 300, 0), (2, 1, 256, 7, 2500, 0),
    (4, 4, 64, 60, 60, 0), (8, 2, 128, 40, 300, 0), (2, 1, 96, 70, 3000, 0), (4, 2, 256, 33, 500, 0), (2, 1, 80, 90, 600, 100), (1, 1, 128, 130, 2500, 0)])
@pytest.mark.parametrize("scores", ["spread", "same", "low"])
def test_infinite_values_come_out_as_they_are_where_they_are_seen(torch, scores, dt, H, KV, D, T, n, window):
    """Two of three elements of a head have an infinite value of one token, of the prefix or the run; the last two have one of each sign or a NaN.  Rows that see it
    have it, of its sign; all else is what it is without.  Weights of every size down to where the library promises it: by scores within 7; all the same, exact
    16-bit numbers; and all but the first 2^-11.7 of it (bf16: 2^-69.3) or some more."""
    S = 3
    g = torch.Generator().manual_seed(H + D + T)
    q, k, v = (torch.randn(shape, generator=g, dtype=torch.float64) for shape in ((S, T, H, D), (S, n, KV, D), (S, n, KV, D)))
    q[..., 1:] = 0
    if scores == "low":
        q[..., 0] = 1
        k[..., 0] = 0.2 * torch.rand((S, n, KV), generator=g)
        k[:, 0, :, 0] = 8.1 if dt == npas.F16 else 48
    else:
        q, k = (q * (scores == "spread")).clamp(-1, 1), k.clamp(-3.5, 3.5)
    clean, lse = _runs(torch, dt, q, k, v, 16, [n] * S, 1.0, window)
    bad, token = v.clone(), torch.randint(max(0, n - T - 40), n, (S, KV, D), generator=g)
    far = torch.rand((S, KV, D), generator=g) < 0.3
    token = torch.where(far, torch.randint(0, n, (S, KV, D), generator=g), token)
    sign = torch.where(torch.rand((S, KV, D), generator=g) < 0.5, -1.0, 1.0).double()
    at = torch.arange(n - T, n)
    want = clean.clone()
    for s in range(S):
        for h in range(KV):
            for d in range(D):
                if d % 3 == 2 and d < D - 2:
                    continue
                odd = [(int(token[s, h, d]), float(sign[s, h, d]) * float("inf"))]
                if d >= D - 2:
                    odd.append(((odd[0][0] + 1) % n, -odd[0][1] if s % 2 else float("nan")))
                for j, value in odd:
                    bad[s, j, h, d] = value
                    see = (j <= at) & ((j > at - window) if window else True)
                    before = want[s, see, h * (H // KV):(h + 1) * (H // KV), d]
                    want[s, see, h * (H // KV):(h + 1) * (H // KV), d] = torch.where(torch.isfinite(before), value, before + value)
    y, again = _runs(torch, dt, q, k, bad, 16, [n] * S, 1.0, window)
    assert torch.equal(again, lse)
    same = (y == want) | ((y != y) & (want != want))
    assert int((~same).sum()) == 0, f"{int((~same).sum())} of {y.numel()}, first {torch.nonzero(~same)[0].tolist()}"


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
@pytest.mark.parametrize("H,KV,D,T,n", [(4, 2, 64, 3, 300), (8, 2, 128, 2, 3000), (4, 2, 64, 40, 90), (8, 2, 128, 40, 3000), (2, 1, 96, 130, 500), (2, 1, 256, 30, 300)])
def test_infinite_and_nan_scores_of_runs(torch, dt, H, KV, D, T, n):
    """By sequence: a score of inf; one of -inf; only -inf; one of inf and one NaN; none of these.  The odd keys stand among the run, so that some rows do not see them."""
    S, a = 5, n - T // 2 - 1
    g = torch.Generator().manual_seed(H + D + 1)
    k, v, q = (torch.randn(shape, generator=g, dtype=torch.float64) for shape in ((S, n, KV, D), (S, n, KV, D), (S, T, H, D)))
    q[..., 0] = 1
    q, k, v = (_round(torch, x, dt) for x in (q, k, v))
    k[0, a, :, 0] = k[3, a, :, 0] = float("inf")
    k[1, a, :, 0] = k[2, :, :, 0] = -float("inf")
    k[3, n - 1, :, 0] = float("nan")
    y, lse = _runs(torch, dt, q, k, v, 16, [n] * S, 0.125)
    sees = torch.arange(n - T, n) >= a
    assert bool(sees.any())
    assert bool((y[0, sees] != y[0, sees]).all()) and bool((lse[0, sees] == float("inf")).all())
    assert bool((y[3, sees] != y[3, sees]).all()) and bool((lse[3, sees][:-1] == float("inf")).all()) and bool((lse[3, -1] != lse[3, -1]).all())
    assert bool((y[2] == 0).all()) and bool((lse[2] == -float("inf")).all())
    for s in (0, 1, 3, 4):
        for t in range(T):
            if s in (0, 3) and bool(sees[t]):
                continue
            j = [i for i in range(n - T + t + 1) if not (s == 1 and i == a)]
            for h in range(H):
                keys = k[s, j, h // (H // KV)]
                x = keys @ q[s, t, h] * 0.125
                off = D * u * float((keys.abs() @ q[s, t, h].abs()).max()) * 0.125
                p, value = torch.softmax(x, 0), v[s, j, h // (H // KV)]
                lost = n * 2.0 ** -36 / u if dt == npas.F16 else 0
                assert not bool(_outside(y[s, t, h], p @ value, p @ value.abs(), dt, 2 * off / u + 320 + MORE[dt] + lost).any()), (s, t, h)
                assert abs(float(lse[s, t, h] - torch.logsumexp(x, 0))) <= off + 320 * u


@gpu
@pytest.mark.parametrize("case", [
    (8, 2, 64, 16, [(300, 300)] + [(1, 50 + 7 * i) for i in range(40)] + [(0, 9)] * 5, 0, npas.BF16, False, False),     # by the mean in tiles of 32 rows
    (4, 4, 128, 16, [(1, 90)] * 20 + [(0, 0)] * 11 + [(260, 700), (2, 2)], 0, npas.BF16, True, False),                    # of 16
    (4, 2, 256, 16, [(0, 5)] * 9 + [(100, 140), (1, 33)], 0, npas.F16, False, False),
    (8, 1, 64, 16, [(1, 40)] * 30 + [(500, 800)], 100, npas.F16, True, False),                                            # of 128
    (16, 2, 96, 24, [(700, 700), (0, 3), (1, 2000), (1, 1), (3, 64)], 0, npas.BF16, False, False)], ids=lambda c: str(c[:4]))
def test_a_long_run_among_single_tokens_and_idle_sequences(torch, monkeypatch, case):
    """The mean run decides how all of them go; results are those of each by itself."""
    monkeypatch.setattr(runs, "_check", _strict)
    runs._run(torch, case)


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
@pytest.mark.parametrize("H,KV,D,page,T,lengths,window", [
    (4, 1, 128, 16, 3, [9000], 0), (8, 8, 64, 16, 7, [6000, 70, 2047, 7], 0), (2, 2, 256, 64, 5, [5000, 129], 0), (16, 2, 80, 7, 4, [2600, 2049, 33], 1000),
    (4, 1, 128, 16, 40, [9000], 0), (8, 8, 64, 16, 50, [6000, 70, 2047, 50], 0), (2, 2, 256, 64, 65, [5000, 129], 0), (16, 2, 80, 7, 33, [2600, 2049, 33], 1000),
    (1, 1, 24, 3, 130, [1400, 131], 0), (32, 8, 128, 16, 64, [2047, 4097], 63)])
def test_every_token_of_a_run_counts_once(torch, dt, H, KV, D, page, T, lengths, window):
    S, top = len(lengths), max(lengths)
    v = torch.zeros((S, top, KV, D), dtype=torch.float64)
    for s, n in enumerate(lengths):
        v[s, :n] = _counts(torch, n, 0, D)[0][:, None]
        v[s, n:] = 100                                    # must not come in
    y, lse = _runs(torch, dt, torch.zeros((S, T, H, D), dtype=torch.float64), torch.ones_like(v), v, page, lengths, 0.125, window)
    for s, n in enumerate(lengths):
        for t in range(T):
            seen = n - T + t + 1
            first = max(0, seen - window) if window else 0
            assert _counts_hold(y[s, t], lse[s, t], _counts(torch, seen, first, D)[1], seen - first, dt), (s, t)

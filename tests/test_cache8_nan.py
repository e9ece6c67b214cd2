"""Caches of 8-bit floats that somebody else filled: NaN codes (0x7f, 0xff) under any byte, byte 255 over any codes.  Both stand for NaN, as the
definition in cache8_reference has it, and reach what sees them and nothing else."""
import pytest

import paper_2012_00596_amd as npas
from tests import test_cache8 as one
from tests import test_chunk_attention as runs
from tests.test_decoder_ops import U, STEPS, _attention64, _rand, _td, torch  # noqa: F401

from . import cache8_reference as c8

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
def test_byte_255_is_nan_over_every_code(torch, dt):
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).reshape(1, 1, 1, 256).cuda()
    byte = torch.full((1, 1, 1, 8), 255, dtype=torch.uint8).cuda()
    cache = npas.KvCache8(codes, codes.clone(), byte, byte.clone(), torch.zeros((1, 1), dtype=torch.int32).cuda(), dt)
    k, v = (torch.zeros((1, 1, 256), dtype=_td(torch, dt), device="cuda") for _ in range(2))
    npas.kv_read(cache, k, v, 1, torch.zeros(1, dtype=torch.int32).cuda())
    assert bool(torch.isnan(k).all()) and bool(torch.isnan(v).all()), (int((~torch.isnan(k)).sum()), k[~torch.isnan(k)])


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
@pytest.mark.parametrize("H,KV,D,n", [(4, 2, 64, 300), (8, 2, 128, 3000), (2, 1, 80, 90), (2, 2, 256, 400)])
def test_one_token_sees_nan_codes_and_bytes(torch, dt, H, KV, D, n):
    S, page = 2, 16
    k, v, ks, vs, table = one._cache8(torch, [n, n - 3], 0, KV, D, page, dt, D)
    v[table[0, 1], 0, 3, 5] = 0xff
    vs[table[0, 2], KV - 1, 2, D // 32 - 1] = 255                      # over ordinary codes
    ks[table[1, 0], 0, 0, 0] = 255                                      # sequence 1: no score of key head 0 is a number
    q = _rand(torch, 1, (S, H, D), dt)
    cache = npas.KvCache8(k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), table.cuda(), dt)
    need = npas.paged_attention8_workspace_bytes(cache, H, n)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    y = torch.zeros((S, H, D), dtype=q.dtype, device="cuda")
    lengths = torch.tensor([n, n - 3], dtype=torch.int32)
    npas.paged_attention8(cache, q.cuda(), y, H, lengths.cuda(), n, D ** -0.5, workspace=ws, workspace_bytes=need)
    got, G = y.cpu().double(), H // KV
    nan = torch.zeros(S, H, D, dtype=torch.bool)
    nan[0, :G, 5] = nan[1, :G] = True
    nan[0, H - G:, 32 * (D // 32 - 1):32 * (D // 32)] = True
    assert torch.equal(torch.isnan(got), nan)
    vv = torch.nan_to_num(c8.dequantise(v, vs))
    kk = torch.nan_to_num(c8.dequantise(k, ks))
    ref, _, w, ds = _attention64(torch, q, kk, vv, table, lengths, D ** -0.5, 0, n)
    assert bool((((got - ref).abs() <= U[dt] * ref.abs() + (2 * ds[..., None] + STEPS + n * 2.0 ** -36) * w) | nan).all())


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
@pytest.mark.parametrize("H,KV,D,new,window", [(4, 2, 64, [(3, 40), (2, 300)], 0), (2, 2, 64, [(14, 140), (20, 20)], 9), (8, 2, 128, [(3, 70), (5, 64)], 0),
                                               (2, 1, 128, [(16, 90), (9, 9)], 4), (2, 1, 256, [(4, 70), (3, 20)], 0), (2, 1, 80, [(4, 70), (3, 20)], 2),
                                               (8, 2, 128, [(100, 150), (64, 64)], 0), (4, 2, 64, [(70, 300), (33, 40)], 20), (2, 1, 256, [(70, 70), (40, 90)], 0),
                                               (2, 1, 80, [(130, 130), (65, 400)], 50), (1, 1, 96, [(65, 65)], 0)])
def test_runs_see_nan_codes_and_bytes_that_they_see(torch, dt, H, KV, D, new, window):
    """In values: a NaN code among ordinary ones, byte 255 over ordinary codes, in the run and before it; in a key, of the last token."""
    case = (H, KV, D, 16, new, window, dt, True, False)
    cache, _, table, starts, n, top = runs._make(torch, case)
    k, v, ks, vs = (t.cpu() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale))
    place = lambda s, j: (int(table[s, j // 16]), j % 16)              # noqa: E731
    for s, (m, length) in enumerate(new):
        for back, d, code in ((m - 1, 3, 0x7f), (m // 2, D - 1, 0xff), (1, D // 2, 0x7f)):
            p, i = place(s, length - 1 - back)
            v[p, KV - 1, i, d] = code
        p, i = place(s, length - 1 - m // 3)
        vs[p, 0, i, (D - 1) // 32] = 255
    T = int(starts[-1])
    q = _rand(torch, 5, (T, H, D), dt)
    need = npas.chunk_attention_workspace_bytes(cache, T, H, top)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    for in_keys in (False, True):
        if in_keys:
            for s, (m, length) in enumerate(new):
                p, i = place(s, length - 1)
                if s:
                    ks[p, 0, i, 0] = 255
                else:
                    k[p, 0, i, 1] = 0x7f
        y, lse = torch.zeros((T, H, D), dtype=q.dtype, device="cuda"), torch.zeros((T, H), device="cuda")
        npas.chunk_attention(npas.KvCache8(k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), table.cuda(), dt), q.cuda(), y, T, H, starts.cuda(), n.cuda(), top,
                             D ** -0.5, window=window, lse=lse, workspace=ws, workspace_bytes=need)
        kk, vv = torch.nan_to_num(c8.dequantise(k, ks)), c8.dequantise(v, vs)
        ref = list(runs._chunk64(torch, q, kk, vv, table, starts, n, D ** -0.5, window, top))
        if in_keys:                                                     # the last row of a run alone sees that key
            for s in range(len(new)):
                ref[0][int(starts[s + 1]) - 1, :H // KV] = float("nan")
        got, odd = y.double().cpu(), torch.isnan(ref[0])
        assert bool(odd.any()) and not bool(odd.all())
        assert torch.equal(torch.isnan(got), odd), f"{int((torch.isnan(got) != odd).sum())} of {odd.numel()}"
        steps = 2 * ref[3][..., None] + STEPS + (top * 2.0 ** -36 if dt == npas.F16 else 0.0)
        assert bool((((got - ref[0]).abs() <= U[dt] * ref[0].abs() + 2.0 ** -25 + steps * ref[2]) | odd).all())

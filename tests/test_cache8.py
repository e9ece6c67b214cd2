"""Keys and values written with per-head norms into paged caches of 16-bit and 8-bit numbers, read back, and the attention of one new token over
8-bit ones, against the definitions in 64 bits.

Tolerances are those of test_decoder_ops: a result is computed in fp32 (STEPS of the terms' magnitudes) and rounded once; an 8-bit number
may be off by half the spacing of its numbers there."""
import numpy as np
import pytest

import paper_2012_00596_amd as npas
from tests.test_decoder_ops import STEPS, TINY, U, _attention64, _rand, _rotate64, _td, torch  # noqa: F401

from . import cache8_reference as c8

gpu = pytest.mark.gpu


def _empty8(torch, pages, KV, page, D, fill=0x7f, scale=255):
    shape = (pages, KV, page, D)
    return [torch.full(shape, fill, dtype=torch.uint8, device="cuda") for _ in range(2)] + \
        [torch.full(shape[:3] + (-(-D // 32),), scale, dtype=torch.uint8, device="cuda") for _ in range(2)]


def _normed64(x, w, eps):
    """(x w / sqrt(mean x^2 + eps), the sum of the terms' magnitudes an element)"""
    if w is None:
        return x.double(), x.double().abs()
    y = x.double() / (x.double().square().mean(-1, keepdim=True) + eps).sqrt() * w.double()
    return y, y.abs()


def _heads64(torch, x, w, eps, cs, pos, rot, pairs):
    y, mag = _normed64(x, w, eps)
    if not rot:
        return y, mag
    return _rotate64(y, cs[pos], rot, pairs)


WRITE = [  # heads, kv heads, D, page, tokens, rot, pairs, norms, 8 bits, dtype
    (1, 1, 16, 4, 1, 16, False, "qk", True, npas.BF16),
    (12, 4, 64, 16, 24, 32, True, "qk", False, npas.F16),
    (32, 8, 128, 16, 37, 128, False, "qk", True, npas.BF16),
    (32, 8, 128, 16, 37, 128, False, "qk", False, npas.BF16),
    (20, 5, 80, 24, 33, 80, True, "", True, npas.F16),
    (20, 5, 80, 24, 33, 40, False, "k", True, npas.F16),
    (6, 3, 96, 7, 19, 96, False, "q", True, npas.BF16),
    (7, 1, 256, 1, 21, 256, False, "qk", True, npas.BF16),
    (2, 2, 256, 64, 5, 128, True, "qk", True, npas.F16),
    (3, 1, 8, 3, 11, 6, False, "qk", False, npas.F16),
    (5, 5, 24, 5, 13, 10, True, "qk", False, npas.BF16),
    (4, 2, 200, 16, 9, 36, False, "qk", False, npas.BF16),
    (4, 4, 48, 16, 9, 20, False, "qk", True, npas.F16),
    (0, 3, 64, 16, 17, 64, False, "k", True, npas.BF16),
    (8, 2, 112, 16, 6, 0, False, "qk", True, npas.BF16),
]


@gpu
@pytest.mark.parametrize("case", WRITE, ids=str)
def test_write(torch, case):
    """Slices of a joined projection at odd alignment; padding tokens and missing pages among them; the rest of the cache as it was."""
    H, KV, D, page, T, rot, pairs, norms, e8, dt = case
    print(f"write {case}", flush=True)
    S, top, eps = 3, 50, 1e-3
    rng = np.random.default_rng(T + D)
    columns = -(-top // page)
    pages = S * columns + 2
    table = torch.from_numpy(rng.permutation(pages)[:S * columns].reshape(S, columns).astype(np.int32))
    table[1, columns // 2] = -1
    places = rng.permutation(S * top)[:T]
    seq, pos = torch.from_numpy((places // top).astype(np.int32)), torch.from_numpy((places % top).astype(np.int32))
    if T > 4:
        pos[1], seq[2], seq[3] = -1, -1, S
        if rot:
            pos[4] = top                            # past the angles
    wide = _rand(torch, 3, (T, (H + 2 * KV) * D + 3), dt, 2.0)
    wide *= torch.exp(_rand(torch, 4, (1, wide.shape[1]), npas.F32)).to(wide.dtype)
    wide[:, 3 + H * D] = 0
    heads = [x.reshape(T, -1, D) for x in wide[:, 3:].split([H * D, KV * D, KV * D], 1)]
    cs = torch.rand((top, rot), generator=torch.Generator().manual_seed(9)) * 2 - 1 if rot else None
    qw, kw = (_rand(torch, 5 + i, (D,), npas.F32) if n in norms else None for i, n in enumerate("qk"))
    if e8:
        k, v, ks, vs = _empty8(torch, pages, KV, page, D, 0x15, 99)
        cache = npas.KvCache8(k, v, ks, vs, table.cuda(), dt)
    else:
        k, v = (torch.full((pages, KV, page, D), 7.0, dtype=_td(torch, dt), device="cuda") for _ in range(2))
        cache = npas.KvCache(k, v, table.cuda(), dt)
    q_out = torch.full((T, max(H, 1), D), float("nan"), dtype=wide.dtype, device="cuda") if H else None
    dev = wide.cuda()[:, 3:].split([H * D, KV * D, KV * D], 1)
    npas.kv_write(cache, dev[0] if H else None, dev[1], dev[2], q_out, T, max(H, KV), pos.cuda(), sequences=seq.cuda(),
                  q_weight=None if qw is None else qw.cuda(), k_weight=None if kw is None else kw.cuda(), eps=eps,
                  cos_sin=None if cs is None else cs.cuda(), rot_dim=rot, kind=npas.ROTATE_PAIRS if pairs else npas.ROTATE_HALVES)
    token = (seq >= 0) & (seq < S) & (pos >= 0) & ((pos < top) if rot else True)
    safe = torch.where(token, pos, 0).long()
    if H:
        ref, mag = _heads64(torch, heads[0], qw, eps, cs, safe, rot, pairs)
        got = q_out.double().cpu()
        assert bool((got[~token] == 0).all())
        bad = (got - ref).abs() > U[dt] * ref.abs() + TINY[dt] + STEPS * mag
        assert not bool(bad[token].any()), f"queries: {int(bad[token].sum())}"
    column = safe // page
    there = token & (column < columns)
    p = table[torch.where(there, seq, 0).long(), column.clamp(max=columns - 1)].long()
    there &= (p >= 0) & (p < pages)
    untouched = torch.ones((pages, page), dtype=torch.bool)
    untouched[p[there], (safe % page)[there]] = False
    for name, x, w, got, scales in (("k", heads[1], kw, k, ks if e8 else None), ("v", heads[2], None, v, vs if e8 else None)):
        got = got.cpu()
        assert bool((got.transpose(1, 2)[untouched] == (0x15 if e8 else 7)).all())
        ref, mag = _heads64(torch, x, w, eps, cs, safe, rot, pairs) if name == "k" else (x.double(), x.double().abs())
        ref, mag, new = ref[there], mag[there], got[p[there], :, (safe % page)[there]]
        if not e8:
            bad = (new.double() - ref).abs() > U[dt] * ref.abs() + TINY[dt] + STEPS * mag
            assert not bool(bad.any()), f"{name}: {int(bad.sum())}"
            continue
        scales = scales.cpu()
        assert bool((scales.transpose(1, 2)[untouched] == 99).all())
        byte = scales[p[there], :, (safe % page)[there]]
        if name == "v":
            codes, want = c8.quantise(ref, dt)
            assert torch.equal(byte, want) and torch.equal(new, codes)
            continue
        # the largest magnitude may lie on either side of 448 2^e by its error in fp32
        near = STEPS * torch.nn.functional.pad(mag, (0, -D % 32)).unflatten(-1, (-1, 32)).amax(-1)
        low, high = ((c8.exponents(ref, dt)[1] * f + n * g) for f, n, g in ((1, near, -1), (1, near, 1)))
        bytes_of = lambda t: (torch.where(t <= 0, -200, torch.frexp(t)[1] - 9 + (torch.frexp(t)[0] > 0.875).int())  # noqa: E731
                              ).clamp(*c8.LIMITS[dt]) + 127
        assert bool(((byte >= bytes_of(low)) & (byte <= bytes_of(high))).all())
        unit = torch.exp2(byte.double() - 127).repeat_interleave(32, -1)[..., :D]
        far = ref.abs() + STEPS * mag
        spacing = unit * torch.exp2(torch.floor(torch.log2((far / unit).clamp(min=2.0 ** -6))) - 3)
        cap = torch.where(byte == c8.LIMITS[dt][1] + 127, 240.0, 448.0).repeat_interleave(32, -1)[..., :D] * unit
        bad = (c8.dequantise(new, byte) - ref.clamp(-cap, cap)).abs() > spacing / 2 + STEPS * mag
        assert not bool(bad.any()), f"keys in 8 bits: {int(bad.sum())}"


@gpu
@pytest.mark.parametrize("dt", [npas.BF16, npas.F16])
def test_every_16_bit_value_to_8_bits_and_back(torch, dt):
    """Codes and scales of every 16-bit pattern beside largest magnitudes from the least to the greatest, bit for bit; what is read are the same values."""
    D, KV, page = 64, 1, 64
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    rows = bits.view(_td(torch, dt)).reshape(-1, 31)[:2114] if 65536 % 31 == 0 else torch.cat([bits, bits[:31 - 65536 % 31]]).view(_td(torch, dt)).reshape(-1, 31)
    tops = [0.0, 2.0 ** -24, 2.0 ** -14, 0.874, 0.875, 0.876, 1.0, 447.0, 448.0, 449.0, 6e4] + ([] if dt == npas.F16 else [2.0 ** -126, 2.0 ** -100, 3e38, 1e30])
    top = torch.tensor(tops).to(rows.dtype)
    x = torch.cat([torch.cat([rows, t.expand(rows.shape[0], 1)], 1) for t in top])     # blocks of 32
    x = torch.cat([x, x.new_zeros((-x.shape[0]) % 2, 32)]).reshape(-1, 64)
    T = x.shape[0]
    pages = -(-T // page)
    table = torch.arange(pages, dtype=torch.int32).reshape(1, pages).cuda()
    cache = npas.KvCache8(*_empty8(torch, pages, KV, page, D), table, dt)
    pos, seq = torch.arange(T, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    xd = x.cuda()
    npas.kv_write(cache, None, xd, xd, None, T, 1, pos, sequences=seq)
    codes, bytes_ = c8.quantise(x.double(), dt)
    for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        assert torch.equal(s.cpu().reshape(-1, 2)[:T], bytes_)
        got = c.cpu().reshape(-1, D)[:T]
        assert torch.equal(got, codes), int((got != codes).sum())
    back = [torch.empty((T, KV, D), dtype=x.dtype, device="cuda") for _ in range(2)]
    npas.kv_read(cache, *back, T, pos, sequences=seq)
    want = c8.dequantise(codes, bytes_)
    for b in back:
        b = b.cpu().double().reshape(T, D)
        assert bool(((b == want) | (torch.isnan(b) & torch.isnan(want))).all())
        assert bool(torch.isfinite(b[torch.isfinite(want)]).all())


@gpu
def test_every_code_under_every_scale_is_read_exactly(torch):
    for dt in (npas.BF16, npas.F16):
        least, most = c8.LIMITS[dt]
        T = most - least + 1
        codes = torch.arange(256, dtype=torch.int32).to(torch.uint8).expand(T, 256).contiguous()
        codes[-1][(codes[-1] & 127) > 0x77] = 0x77            # at the largest exponent 240 is the last
        byte = (torch.arange(least, most + 1) + 127).to(torch.uint8)[:, None].expand(T, 8).contiguous()
        table = torch.zeros((1, 1), dtype=torch.int32).cuda()
        cache = npas.KvCache8(codes.reshape(1, 1, T, 256).cuda(), codes.reshape(1, 1, T, 256).cuda(), byte.reshape(1, 1, T, 8).cuda(),
                              byte.reshape(1, 1, T, 8).cuda(), table, dt)
        out = torch.empty((T, 1, 256), dtype=_td(torch, dt), device="cuda")
        npas.kv_read(cache, None, out, T, torch.arange(T, dtype=torch.int32).cuda(), sequences=torch.zeros(T, dtype=torch.int32).cuda())
        got, want = out.cpu().double().reshape(T, 256), c8.dequantise(codes, byte)
        assert bool(((got == want) | (torch.isnan(got) & torch.isnan(want))).all())


@gpu
def test_read_of_missing_tokens_is_zero(torch):
    KV, D, page, dt = 2, 48, 4, npas.F16
    table = torch.tensor([[1, -1], [0, 7]], dtype=torch.int32).cuda()          # 2 pages: 7 is none of them
    k, v, ks, vs = _empty8(torch, 2, KV, page, D, 0x38, 127)                     # ones
    cache = npas.KvCache8(k, v, ks, vs, table, dt)
    seq, pos = torch.tensor([0, 0, 1, 1, 2, -1, 0, 1]), torch.tensor([3, 4, 0, 5, 0, 1, -1, 2 ** 31 - 1])
    ko, vo = (torch.full((8, KV, D), float("nan"), dtype=torch.float16, device="cuda") for _ in range(2))
    npas.kv_read(cache, ko, vo, 8, pos.int().cuda(), sequences=seq.int().cuda())
    want = torch.tensor([1.0, 0, 1, 0, 0, 0, 0, 0])[:, None, None].expand(8, KV, D)
    assert bool((ko.cpu() == want).all()) and bool((vo.cpu() == want).all())
    only = torch.full_like(ko, float("nan"))
    npas.kv_read(cache, only, None, 2, pos.int().cuda(), sequences=seq.int().cuda())
    assert bool((only[:2].cpu() == want[:2]).all()) and bool(torch.isnan(only[2:]).all())


@gpu
def test_write_of_infinities_and_nan(torch):
    """A block with one is NaN throughout, the others of the row are not; in 16 bits they are stored as they are; finite values past fp16 stop at 61440."""
    KV, D, page = 1, 96, 8
    table = torch.zeros((1, 1), dtype=torch.int32).cuda()
    x = _rand(torch, 1, (4, KV, D), npas.F16)
    x[0, 0, 5], x[1, 0, 40], x[2, 0, 95] = float("inf"), float("nan"), -float("inf")
    pos, seq = torch.arange(4, dtype=torch.int32).cuda(), torch.zeros(4, dtype=torch.int32).cuda()
    cache = npas.KvCache8(*_empty8(torch, 1, KV, page, D), table, npas.F16)
    npas.kv_write(cache, None, x.cuda(), x.cuda(), None, 4, 1, pos, sequences=seq)
    codes, byte = c8.quantise(x.double(), npas.F16)
    assert torch.equal(cache.k[0, 0, :4].cpu(), codes[:, 0]) and torch.equal(cache.k_scale[0, 0, :4].cpu(), byte[:, 0])
    assert int((byte == 255).sum()) == 3
    big = torch.full((1, 1, D), 60000.0, dtype=torch.float16)
    w = torch.full((D,), 1e7)
    npas.kv_write(cache, None, big.cuda(), big.cuda(), None, 1, 1, pos, sequences=seq, k_weight=w.cuda())
    ko, vo = (torch.empty((1, 1, D), dtype=torch.float16, device="cuda") for _ in range(2))
    npas.kv_read(cache, ko, vo, 1, pos, sequences=seq)
    assert bool((ko == 61440).all()) and bool((vo == 61440).all())


@gpu
@pytest.mark.parametrize("e8", [False, True])
@pytest.mark.parametrize("D,rot,pairs", [(64, 64, False), (96, 20, False), (256, 256, True)])
def test_write_over_the_queries(torch, D, rot, pairs, e8):
    """q_out may be q; without norms a 16-bit write is kv_append's, bit for bit."""
    S, H, KV, page, dt = 7, 6, 2, 16, npas.BF16
    table = torch.arange(S * 2, dtype=torch.int32).reshape(S, 2).cuda()
    q, kx, vx = (_rand(torch, 30 + i, (S, n, D), dt).cuda() for i, n in enumerate((H, KV, KV)))
    pos, cs = torch.arange(S, dtype=torch.int32).cuda() * 3, torch.rand((32, rot)).cuda()
    w = _rand(torch, 40, (D,), npas.F32).cuda()
    outs = []
    for inplace in (False, True):
        k, v = (torch.zeros((S * 2, KV, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        cache = npas.KvCache8(*_empty8(torch, S * 2, KV, page, D), table, dt) if e8 else npas.KvCache(k, v, table, dt)
        qi = q.clone()
        qo = qi if inplace else torch.empty_like(q)
        npas.kv_write(cache, qi, kx, vx, qo, S, H, pos, q_weight=w, k_weight=w, cos_sin=cs, rot_dim=rot,
                      kind=npas.ROTATE_PAIRS if pairs else npas.ROTATE_HALVES)
        outs.append([qo, cache.k, cache.v])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    if e8:
        return
    caches = []
    for call in (npas.kv_append, npas.kv_write):
        k, v = (torch.zeros((S * 2, KV, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        qo = torch.empty_like(q)
        call(npas.KvCache(k, v, table, dt), q, kx, vx, qo, S, H, pos, cos_sin=cs, rot_dim=rot, kind=npas.ROTATE_PAIRS if pairs else npas.ROTATE_HALVES)
        caches.append([qo, k, v])
    assert torch.equal(caches[0][2], caches[1][2])
    for a, b in zip(caches[0][:2], caches[1][:2]):          # products and sums may be contracted in another way: a step of the result apart
        assert bool(((a.double() - b.double()).abs() <= 2 * U[dt] * a.double().abs() + STEPS * 4).all())


# ---- attention of one token over 8-bit floats -------------------------------------

def _cache8(torch, lengths, window, KV, D, page, dt, seed, scale_of=1.0):
    """Codes of random keys and values where a sequence's tokens lie, NaN everywhere else; (k, v, k_scale, v_scale, table) on the CPU."""
    S, top = len(lengths), max(max(lengths), 1)
    columns = -(-top // page)
    pages = S * columns + 3
    rng = np.random.default_rng(seed)
    table = torch.from_numpy(rng.permutation(pages)[:S * columns].reshape(S, columns).astype(np.int32))
    used = torch.zeros((pages, page), dtype=torch.bool)
    for s in range(S):
        j = torch.arange(max(0, lengths[s] - window) if window else 0, lengths[s])
        used[table[s].long()[j // page], j % page] = True
    used = used[:, None, :, None].expand(pages, KV, page, 1)
    out = []
    for i in range(2):
        x = _rand(torch, seed + i, (pages, KV, page, D), npas.F32, 1.3 * scale_of) * torch.exp(0.5 * _rand(torch, seed + 9, (1, 1, 1, D), npas.F32))
        out.append(c8.quantise(x.double(), dt))
    k, v = (torch.where(used, c, torch.full_like(c, 0x7f)) for c, _ in out)
    ks, vs = (torch.where(used, s, torch.full_like(s, 255)) for _, s in out)
    return k, v, ks, vs, table


ATTENTION8 = [  # heads, kv heads, D, page, lengths, window, dtype, holes
    (1, 1, 16, 16, [0, 1, 2, 3], 0, npas.BF16, False),
    (4, 4, 64, 16, [1, 15, 16, 17, 31, 32, 33, 0, 127, 128, 129], 0, npas.F16, False),
    (8, 2, 128, 16, [500, 1, 0, 64, 1000], 0, npas.BF16, False),
    (32, 8, 128, 16, [2047], 0, npas.F16, False),
    (6, 2, 80, 7, [100, 13, 700, 14], 0, npas.F16, True),
    (20, 1, 128, 24, [333, 48], 0, npas.BF16, True),
    (48, 3, 64, 32, [257, 95], 0, npas.F16, True),
    (40, 1, 96, 5, [77, 301], 0, npas.BF16, True),
    (16, 16, 256, 64, [130, 4, 640], 0, npas.BF16, True),
    (3, 3, 48, 256, [300, 1, 513], 0, npas.F16, False),
    (7, 1, 32, 3, [50, 0, 200], 0, npas.BF16, True),
    (8, 4, 64, 16, [5, 40, 41, 600, 1300, 0], 37, npas.BF16, False),
    (8, 8, 128, 8, [2500, 3, 1031], 512, npas.F16, True),
    (4, 1, 128, 16, [9000], 0, npas.BF16, True),
    (2, 2, 208, 32, [1100, 500, 257], 0, npas.F16, False),
    (4, 2, 256, 16, [5000, 100], 0, npas.F16, True),
    (8, 8, 64, 16, [6000, 70], 0, npas.BF16, False),
    (14, 2, 64, 1, [1500, 1499], 1, npas.BF16, False),
]


@gpu
@pytest.mark.parametrize("case", ATTENTION8, ids=str)
def test_attention8(torch, case):
    """Ragged lengths over random pages; every place that no token names holds NaN; a workspace of NaN; twice the same bits."""
    H, KV, D, page, lengths, window, dt, holes = case
    print(f"attention8 {case}", flush=True)
    S, top = len(lengths), max(lengths)
    k, v, ks, vs, table = _cache8(torch, lengths, window, KV, D, page, dt, H + D)
    if holes:
        table[0, table.shape[1] // 2], table[S - 1, 0] = -1, k.shape[0] + 7
        table[0, -1] = 2 ** 31 - 1
    n = torch.tensor(lengths, dtype=torch.int32)
    wide = _rand(torch, 62, (S, H * D + 5), dt, 1.5)
    q = wide[:, 5:].reshape(S, H, D)
    cache = npas.KvCache8(k.cuda(), v.cuda(), ks.cuda(), vs.cuda(), table.cuda(), dt)
    need = npas.paged_attention8_workspace_bytes(cache, H, top)
    ws = torch.full((max(need, 16) // 4 + 1,), float("nan"), device="cuda")
    outs = []
    for again in range(2):
        y = torch.full((S, H, D), float("nan"), dtype=q.dtype, device="cuda")
        lse = torch.full((S, H), float("nan"), device="cuda")
        npas.paged_attention8(cache, wide.cuda()[:, 5:], y, H, n.cuda(), top, D ** -0.5, window=window, lse=lse, workspace=ws, workspace_bytes=need)
        outs.append(y)
    assert torch.equal(outs[0], outs[1]), "two calls differ"
    ref, lref, w, ds = _attention64(torch, q, c8.dequantise(k, ks), c8.dequantise(v, vs), table, n, D ** -0.5, window, top)
    # weights keep their fp32 bits, but for those of fp16 below 2^-39 of the largest
    steps = 2 * ds[..., None] + STEPS + (top * 2.0 ** -39 if dt == npas.F16 else 0.0)
    got = y.double().cpu()
    assert bool((got[w.sum(-1) == 0] == 0).all()), "a row without tokens is not zero"
    bad = ~((got - ref).abs() <= U[dt] * ref.abs() + TINY[dt] + steps * w)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, worst {float((got - ref).abs().max())}, NaN {int((got != got).sum())}"
    none = lref == -float("inf")
    le = lse.double().cpu()
    assert bool((le[none] == -float("inf")).all())
    assert bool(((le - lref).abs()[~none] <= ds[~none] + STEPS * (1 + lref[~none].abs())).all())


@gpu
def test_write_read_and_attention8_beyond_32_bit_offsets(torch):
    """A cache of more than 2^32 bytes a tensor, its last pages in use."""
    KV, D, page, H, dt = 8, 128, 16, 8, npas.BF16
    pages = 2 ** 32 // (KV * D * page) + 40
    codes = [torch.empty((pages, KV, page, D), dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty((pages, KV, page, D // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
    last = pages - 20
    table = torch.arange(last, last + 20, dtype=torch.int32).reshape(2, 10).flip(1).contiguous()
    cache = npas.KvCache8(*codes, *scales, table.cuda(), dt)
    L = 150
    kx, vx = (_rand(torch, 80 + i, (2 * L, KV, D), dt) for i in range(2))
    pos, seq = torch.arange(L, dtype=torch.int32).repeat(2), torch.arange(2, dtype=torch.int32).repeat_interleave(L)
    npas.kv_write(cache, None, kx.cuda(), vx.cuda(), None, 2 * L, H, pos.cuda(), sequences=seq.cuda())
    ko, vo = (torch.empty((2 * L, KV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    npas.kv_read(cache, ko, vo, 2 * L, pos.cuda(), sequences=seq.cuda())
    k64, v64 = (c8.dequantise(*c8.quantise(x.double(), dt)) for x in (kx, vx))
    assert torch.equal(ko.cpu().double(), k64) and torch.equal(vo.cpu().double(), v64)
    q, n = _rand(torch, 82, (2, H, D), dt), torch.tensor([L, L - 7], dtype=torch.int32)
    y = torch.empty((2, H, D), dtype=q.dtype, device="cuda")
    need = npas.paged_attention8_workspace_bytes(cache, H, L)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    npas.paged_attention8(cache, q.cuda(), y, H, n.cuda(), L, D ** -0.5, workspace=ws, workspace_bytes=need)
    ks, vs = (torch.zeros((20, KV, page, D), dtype=torch.float64) for _ in range(2))
    for t in range(2 * L):
        p = int(table[seq[t], pos[t] // page]) - last
        ks[p, :, pos[t] % page], vs[p, :, pos[t] % page] = k64[t], v64[t]
    ref, _, w, ds = _attention64(torch, q, ks, vs, table - last, n, D ** -0.5, 0, L)
    assert bool(((y.double().cpu() - ref).abs() <= U[dt] * ref.abs() + (2 * ds[..., None] + STEPS) * w).all())


# ---- refusals (no GPU needed: nothing is launched) --------------------------------

def _desc(**kw):
    d = dict(k_dev=4096, v_dev=8192, page_table_dev=256, dtype=npas.E4M3, pages=4, page_size=16, kv_heads=2, head_dim=64, sequences=2, table_stride=2)
    d.update(kw)
    return npas.KvCacheDesc(**d)


def _scales(**kw):
    return npas.KvScalesDesc(**{**dict(k_scale_dev=16384, v_scale_dev=32768, dtype=npas.BF16), **kw})


def _every(L, c, s):
    """The codes that the calls give on this cache."""
    return [L.npas_kv_write(c, s, 64, 256, 64, 128, 64, 128, 64, 1, 4, None, 64, None, None, 1e-6, 64, 8, 64, 0, None),
            L.npas_chunk_attention(c, s, 64, 256, 64, None, 1, 4, 64, 64, 32, 0, 1.0, None, 0, None)] + \
        ([L.npas_kv_read(c, s, 64, 64, 1, None, 64, None), L.npas_paged_attention8(c, s, 64, 256, 64, None, 4, 64, 32, 0, 1.0, None, 0, None)] if s else [])


@pytest.mark.parametrize("change,scales,code", [
    (dict(k_dev=None), {}, npas.E_NULL), (dict(v_dev=None), {}, npas.E_NULL), (dict(page_table_dev=None), {}, npas.E_NULL),
    ({}, dict(k_scale_dev=None), npas.E_NULL), ({}, dict(v_scale_dev=None), npas.E_NULL), (dict(dtype=npas.BF16), {}, npas.E_DTYPE),
    ({}, dict(dtype=npas.E4M3), npas.E_DTYPE), ({}, dict(dtype=npas.F32), npas.E_DTYPE), ({}, None, npas.E_DTYPE),
    (dict(pages=0), {}, npas.E_SHAPE), (dict(head_dim=72), {}, npas.E_SHAPE), (dict(head_dim=272), {}, npas.E_SHAPE),
    (dict(k_dev=4104), {}, npas.E_SHAPE), ({}, dict(v_scale_dev=32772), npas.E_SHAPE), (dict(pages=2 ** 30), {}, npas.E_SHAPE)])
def test_bad_8_bit_caches_are_refused(change, scales, code):
    L, c = npas.lib(), _desc(**change)
    s = None if scales is None else _scales(**scales)
    assert set(_every(L, c, s)) == {code}, npas.last_error()
    assert L.npas_paged_attention8_workspace_bytes(c, s, 4, 32) == 0
    assert L.npas_chunk_attention_workspace_bytes(c, s, 1, 4, 32) == 0


def test_16_bit_calls_refuse_8_bit_caches():
    L, c = npas.lib(), _desc()
    assert L.npas_kv_append(c, 64, 256, 64, 128, 64, 128, 64, 1, 4, None, 64, 64, 8, 64, 0, None) == npas.E_DTYPE
    assert L.npas_paged_attention(c, 64, 256, 64, None, 4, 64, 32, 0, 1.0, None, 0, None) == npas.E_DTYPE
    assert L.npas_paged_attention_workspace_bytes(c, 4, 32) == 0
    assert L.npas_kv_read(_desc(dtype=npas.BF16), None, 64, 64, 1, None, 64, None) == npas.E_NULL
    assert L.npas_paged_attention8(_desc(dtype=npas.BF16), None, 64, 256, 64, None, 4, 64, 32, 0, 1.0, None, 0, None) == npas.E_NULL
    assert L.npas_paged_attention8_workspace_bytes(_desc(dtype=npas.BF16), None, 4, 32) == 0


def test_write_refuses():
    L, good = npas.lib(), [_desc(), _scales(), 64, 256, 64, 128, 64, 128, 64, 1, 4, None, 64, 64, 64, 1e-6, 64, 8, 64, 0, None]
    for at, value, code in [(2, None, npas.E_NULL), (4, None, npas.E_NULL), (6, None, npas.E_NULL), (8, None, npas.E_NULL),
                            (12, None, npas.E_NULL), (16, None, npas.E_NULL), (0, None, npas.E_NULL), (3, 255, npas.E_SHAPE),
                            (5, 127, npas.E_SHAPE), (7, 0, npas.E_SHAPE), (9, 0, npas.E_SHAPE), (9, -3, npas.E_SHAPE), (10, 0, npas.E_SHAPE),
                            (10, 3, npas.E_SHAPE), (17, 0, npas.E_SHAPE), (18, 63, npas.E_SHAPE), (18, 66, npas.E_SHAPE),
                            (18, -2, npas.E_SHAPE), (19, 2, npas.E_SHAPE), (2, 65, npas.E_SHAPE), (11, 66, npas.E_SHAPE),
                            (13, 66, npas.E_SHAPE), (14, 65, npas.E_SHAPE), (15, -1.0, npas.E_SHAPE), (15, float("nan"), npas.E_SHAPE),
                            (9, 2 ** 31 - 1, npas.E_SHAPE)]:
        args = list(good)
        args[at] = value
        assert L.npas_kv_write(*args) == code, (at, value)
        assert npas.last_error()
    args = list(good)
    args[2] = args[8] = None
    assert L.npas_kv_write(*args) == npas.E_NULL             # a norm of queries that are not there


def test_read_refuses():
    L, good = npas.lib(), [_desc(), _scales(), 64, 64, 1, None, 64, None]
    for at, value, code in [(0, None, npas.E_NULL), (1, None, npas.E_NULL), (6, None, npas.E_NULL), (4, 0, npas.E_SHAPE), (4, -1, npas.E_SHAPE),
                            (2, 65, npas.E_SHAPE), (3, 65, npas.E_SHAPE), (5, 66, npas.E_SHAPE), (6, 66, npas.E_SHAPE), (4, 2 ** 31 - 1, npas.E_SHAPE)]:
        args = list(good)
        args[at] = value
        assert L.npas_kv_read(*args) == code, (at, value)
    assert L.npas_kv_read(_desc(), _scales(), None, None, 1, None, 64, None) == npas.E_NULL


def test_attention8_refuses():
    L, good = npas.lib(), [_desc(), _scales(), 64, 256, 64, None, 4, 64, 32, 0, 1.0, None, 0, None]
    for at, value, code in [(2, None, npas.E_NULL), (4, None, npas.E_NULL), (7, None, npas.E_NULL), (3, 100, npas.E_SHAPE),
                            (6, 0, npas.E_SHAPE), (6, 5, npas.E_SHAPE), (8, 0, npas.E_SHAPE), (9, -1, npas.E_SHAPE),
                            (10, float("nan"), npas.E_SHAPE), (2, 63, npas.E_SHAPE), (5, 66, npas.E_SHAPE)]:
        args = list(good)
        args[at] = value
        assert L.npas_paged_attention8(*args) == code, (at, value)
    long = _desc(pages=70000, table_stride=70000, sequences=1)
    need = L.npas_paged_attention8_workspace_bytes(long, _scales(), 4, 10 ** 6)
    assert need
    for ws, size in ((None, need), (4096, 15), (4100, need)):
        assert L.npas_paged_attention8(long, _scales(), 64, 256, 64, None, 4, 64, 10 ** 6, 0, 1.0, ws, size, None) == npas.E_WORKSPACE


def test_binding_refuses_8_bit_caches_that_do_not_fit():
    import torch
    U8 = torch.uint8
    k, s, table = torch.zeros((4, 2, 16, 80), dtype=U8), torch.zeros((4, 2, 16, 3), dtype=U8), torch.zeros((2, 2), dtype=torch.int32)
    npas.KvCache8(k, k, s, s, table, npas.BF16)
    for bad in ((k, k[:, :1], s, s, table), (k.bfloat16(), k.bfloat16(), s, s, table), (k, k, s[..., :2], s[..., :2], table),
                (k, k, s, s.int(), table), (k, k, s.transpose(1, 2), s, table), (k, k, s, s, table.long())):
        with pytest.raises(AssertionError):
            npas.KvCache8(*bad, npas.BF16)
    with pytest.raises(npas.NpasError) as e:                 # an 8-bit cache where one of 16 bits is expected
        npas.kv_append(npas.KvCache8(k, k, s, s, table, npas.BF16), None, torch.zeros(1, 160).bfloat16(), torch.zeros(1, 160).bfloat16(), None, 1, 2,
                       torch.zeros(1, dtype=torch.int32))
    assert e.value.code == npas.E_DTYPE

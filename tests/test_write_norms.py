"""kv_write's norms where the mean square is a subnormal number of fp32."""
import pytest

import paper_2012_00596_amd as npas
from tests.test_decoder_ops import STEPS, TINY, U, _rand, torch  # noqa: F401

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("scale", [2.0 ** -62, 2.0 ** -64, 2.0 ** -66, 2.0 ** -68])
def test_norms_of_small_rows_without_eps(torch, D, scale):
    """Squares are off by 2^-150 each where they are subnormal, of 2^-136 and more on average here: 2^-14 of the mean, half of that of the root."""
    T, H, KV, page, dt = 3, 2, 2, 4, npas.BF16
    q, k, v = (((_rand(torch, 20 + i, (T, n, D), npas.F32).abs() + 0.5) * scale).to(torch.bfloat16) for i, n in enumerate((H, KV, KV)))
    kc, vc = (torch.zeros((1, KV, page, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache = npas.KvCache(kc, vc, torch.zeros((1, 1), dtype=torch.int32).cuda(), dt)
    out, w = torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda"), torch.ones(D, device="cuda")
    npas.kv_write(cache, q.cuda(), k.cuda(), v.cuda(), out, T, H, torch.arange(T, dtype=torch.int32).cuda(), sequences=torch.zeros(T, dtype=torch.int32).cuda(),
                  q_weight=w, k_weight=w, eps=0.0)
    for x, got in ((q, out), (k, kc[0, :, :T].transpose(0, 1))):
        ref = x.double() / x.double().square().mean(-1, keepdim=True).sqrt()
        assert bool(((got.double().cpu() - ref).abs() <= (U[dt] + STEPS + 2.0 ** -15) * ref.abs() + TINY[dt]).all()), got

"""The example's decode steps: a graph's replays against the eager calls (bit for bit), and every call against its definition in 64 bits,
fed what the library stored before it.  (Whole steps cannot be compared: a block of 4-bit codes changes its exponent where its largest
value crosses a power of two, so two 64-bit walks that differ by 1e-7 before each rounding to bfloat16 end 4 to 8 % apart.)"""
import numpy as np
import pytest

import paper_2012_00596_amd as npas
from tests.test_mxfp4 import reference, values

pytestmark = pytest.mark.gpu
U = 2.0 ** -8          # of bfloat16


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


class Recorder:
    """The binding, keeping a copy of what each call of a step has written."""

    def __init__(self, torch):
        self.torch, self.outputs = torch, []

    def __getattr__(self, name):
        written = {"fc_sparse": (2,), "kv_append": (4,), "paged_attention": (2,), "gated_residual_norm": (2, 3), "fc_mxfp4": (2,)}.get(name)
        if written is None:
            return getattr(npas, name)

        def call(*args, **kw):
            getattr(npas, name)(*args, **kw)
            self.torch.cuda.synchronize()
            self.outputs.append((name, [args[i].double().cpu().numpy() for i in written]))
        return call


class Reference:
    """The blocks' definition in 64 bits, call by call; `stored` gives what the library made of the call before."""

    def __init__(self, d):
        from examples import decoder_block as ex
        self.d, self.scale, self.eps = d, ex.SCALE, ex.EPS
        f64 = lambda t: t.double().cpu().numpy()                                      # noqa: E731
        self.w4 = [(values(*reference(b.w_up), d.width), values(*reference(b.w_down), b.w_down.shape[1])) for b in d.blocks]
        self.par = [[(f64(b.gate[i]), f64(b.post[i]), f64(b.pre[i])) for i in range(2)] for b in d.blocks]
        self.cos_sin, self.f64, self.table = f64(d.cos_sin), f64, d.table.cpu().numpy()

    def check(self, name, want, mag, terms):
        """One recorded output against `want`: the rounding of the result, and `terms` fp32 steps of the terms' magnitudes."""
        got_name, got = self.recorded.pop(0)
        assert got_name == name, f"{got_name} called where {name} belongs"
        for g, w, m in zip(got, want, mag):
            w = w.reshape(g.shape)
            bad = np.abs(g - w) > U * np.abs(w) + 2.0 ** -133 + terms * 2.0 ** -24 * m.reshape(g.shape)
            assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.abs(g - w).max()}"
        return got

    def norm(self, x, w):
        return x / np.sqrt((x * x).mean(1, keepdims=True) + self.eps) * w

    def product(self, name, x, w, act=lambda v: v, slope=1.0):
        return self.check(name, [act(x @ w.T)], [slope * np.abs(x) @ np.abs(w).T], x.shape[1] + 128)[0]

    def step(self, x, i, recorded):
        d, D, H, KV = self.d, self.d.D, self.d.H, self.d.KV
        self.recorded = recorded
        n64 = self.norm(x, np.ones(d.width))
        h, n = self.check("gated_residual_norm", [x, n64], [np.abs(x), np.abs(n64)], 128)
        for b, blk in enumerate(d.blocks):
            qkv = self.product("fc_sparse", n, blk.w_qkv).reshape(d.S, H + 2 * KV, D)
            c, s = self.cos_sin[i][:D // 2], self.cos_sin[i][D // 2:]
            u, v = qkv[:, :H + KV, :D // 2], qkv[:, :H + KV, D // 2:]
            rot = np.concatenate([u * c - v * s, v * c + u * s], 2)
            mag = np.concatenate([np.abs(u * c) + np.abs(v * s), np.abs(v * c) + np.abs(u * s)], 2)
            q = self.check("kv_append", [rot[:, :H]], [mag[:, :H]], 8)[0].reshape(d.S, H, D)
            k_cache, v_cache = self.f64(d.caches[b].k), self.f64(d.caches[b].v)
            page = d.caches[b].page_size
            y, ym = np.zeros((d.S, H, D)), np.zeros((d.S, H, D))
            for t in range(d.S):
                at = [(self.table[t, j // page], j % page) for j in range(i + 1)]
                k, w = (np.stack([cache[p, :, r] for p, r in at]) for cache in (k_cache, v_cache))
                assert (np.abs(k[i] - rot[t, H:]) <= U * np.abs(rot[t, H:]) + 8 * 2.0 ** -24 * mag[t, H:]).all(), "the new token's keys"
                assert (w[i] == qkv[t, H + KV:]).all(), "the new token's values"
                for j in range(H):
                    p = k[:, j // (H // KV)] @ q[t, j] * D ** -0.5
                    p = np.exp(p - p.max())
                    p /= p.sum()
                    y[t, j], ym[t, j] = p @ w[:, j // (H // KV)], p @ np.abs(w[:, j // (H // KV)])
            # scores are sums of D terms (below 2^7 here), weights may be rounded to bfloat16
            ctx = self.check("paged_attention", [y], [ym], 2 * D * 2 ** 7 + 2 ** 16)[0].reshape(d.S, H * D)
            branch = self.product("fc_sparse", ctx, blk.w_out)
            for half in range(2):
                gate, post, pre = self.par[b][half]
                if half:
                    hswish = lambda v: v * np.clip(v + 3, 0, 6) / 6                       # noqa: E731
                    mid = self.product("fc_mxfp4", values(*reference(n), d.width), self.w4[b][0], hswish, 3.0)
                    branch = self.product("fc_mxfp4", values(*reference(mid), mid.shape[1]), self.w4[b][1])
                part = gate * self.norm(branch, post)
                full = self.scale * h + part
                mag = np.abs(self.scale * h) + np.abs(part)
                n64 = self.norm(full, pre)
                r = np.abs(pre) / np.sqrt((full * full).mean(1, keepdims=True) + self.eps)
                spread = (np.abs(full) * mag).mean(1, keepdims=True) / (full * full).mean(1, keepdims=True)
                h, n = self.check("gated_residual_norm", [full, n64], [mag, mag * r + np.abs(n64) * (1 + 2 * spread)], 64)
        assert not recorded


def test_decode_steps(torch, monkeypatch):
    from examples import decoder_block as ex
    S, steps = 3, 20
    d = ex.Decoder(S, 48, keep=True)
    x = [torch.randn((S, d.width), generator=torch.Generator().manual_seed(i)).bfloat16() for i in range(steps)]

    def feed(i):
        d.x.copy_(x[i])
        d.position.fill_(i)
        d.length.fill_(i + 1)

    recorder, ref, eager = Recorder(torch), Reference(d), []
    monkeypatch.setattr(ex, "npas", recorder)
    for i in range(steps):
        print(f"step {i}", flush=True)
        feed(i)
        recorder.outputs.clear()
        eager.append(d.step().cpu())
        ref.step(x[i].double().numpy(), i, recorder.outputs)
    monkeypatch.undo()
    graph = d.capture()
    for i in range(steps):
        feed(i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(d.n.cpu(), eager[i]), f"step {i}: a replay differs from the eager calls"

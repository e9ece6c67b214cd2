#!/usr/bin/env python3
"""A transformer's decoder blocks at their decode step, every call of the library where such a program makes it.

A block is norm -> attention -> norm, gate, residual, norm -> feed-forward -> norm, gate, residual, norm of the next block:

    joined q, k, v projection   fc_sparse            block-based pruned weights (16 x 32 blocks)
    rotation, cache             kv_append            keys and values go into the paged cache
    attention                   paged_attention      one new token a sequence
    output projection           fc_sparse            block-based pruned
    h, n                        gated_residual_norm  norm of the branch, gate, scaled residual, norm before the feed-forward
    feed-forward                fc_mxfp4 (hard-swish), fc_mxfp4   weights in microscaled 4-bit floats
    h, n                        gated_residual_norm  ... and before the next block's attention

The weights are random, of a small model's shape.  A step allocates nothing: `Decoder.capture` records one as a HIP graph, which is replayed
with new tokens, positions and lengths.

    python examples/decoder_block.py [--sequences 16] [--steps 200]
"""
import argparse
import math
import os
import sys
import time

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2012_00596_amd as npas          # noqa: E402
from workloads import masks                  # noqa: E402

SCALE = math.sqrt(0.5)   # of the residual stream
EPS = 1e-6


def _bits(x):
    """A float32 NumPy array rounded to bfloat16, as uint16 bit patterns."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).bfloat16().view(torch.int16).numpy().view(np.uint16)


def _exact(bits):
    return (bits.astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


class Block:
    """One block's weights: packed handles, and the values they stand for where `keep` asks for them (tests)."""

    def __init__(self, rng, width, heads, kv_heads, head_dim, inner, rate, seed, keep):
        def pruned(out, into):
            mask = masks.fc_block_mask(out, into, 16, 32, rate, seed + out + into)
            w = _bits(rng.standard_normal((out, into)) * math.sqrt(rate / into))
            return npas.pack_fc_block(w, mask, 16, 32, npas.BF16), _exact(w) * mask if keep else None

        def four_bit(out, into):
            w = _bits(rng.standard_normal((out, into)) * math.sqrt(2.0 / into))
            return npas.pack_fc_mxfp4(w, npas.BF16), _exact(w) if keep else None

        self.qkv, self.w_qkv = pruned((heads + 2 * kv_heads) * head_dim, width)
        self.out, self.w_out = pruned(width, heads * head_dim)
        self.up, self.w_up = four_bit(inner, width)
        self.down, self.w_down = four_bit(width, inner)
        cuda = lambda x, t=torch.float32: torch.from_numpy(x.astype(np.float32)).to(t).cuda()        # noqa: E731
        self.post = [cuda(1 + 0.1 * rng.standard_normal(width)) for _ in range(2)]
        self.pre = [cuda(1 + 0.1 * rng.standard_normal(width)) for _ in range(2)]
        self.gate = [cuda(0.7 + 0.1 * rng.standard_normal(width), torch.bfloat16) for _ in range(2)]


class Decoder:
    def __init__(self, sequences, max_length, blocks=2, width=512, heads=8, kv_heads=2, head_dim=64, inner=2048, page_size=16, rate=3,
                 seed=7, keep=False):
        rng = np.random.default_rng(seed)
        self.S, self.H, self.KV, self.D, self.width, self.max_length = sequences, heads, kv_heads, head_dim, width, max_length
        self.blocks = [Block(rng, width, heads, kv_heads, head_dim, inner, rate, seed + 100 * i, keep) for i in range(blocks)]
        self.first_norm = torch.ones(width, device="cuda")
        # one page table for all blocks, a cache each; pages in any order
        per = -(-max_length // page_size)
        self.table = torch.from_numpy(rng.permutation(sequences * per).astype(np.int32).reshape(sequences, per)).cuda()
        shape = (sequences * per, kv_heads, page_size, head_dim)
        self.caches = [npas.KvCache(*(torch.zeros(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2)), self.table, npas.BF16)
                       for _ in range(blocks)]
        freq = 10000.0 ** (-np.arange(head_dim // 2) / (head_dim // 2))
        angle = np.arange(max_length)[:, None] * freq
        self.cos_sin = torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)).cuda()
        # what a step reads and writes
        self.position = torch.zeros(sequences, dtype=torch.int32, device="cuda")   # of the new token
        self.length = torch.ones(sequences, dtype=torch.int32, device="cuda")      # with it
        new = lambda n: torch.empty((sequences, n), dtype=torch.bfloat16, device="cuda")              # noqa: E731
        self.x, self.h, self.n, self.branch = new(width), new(width), new(width), new(width)
        self.qkv, self.q, self.ctx, self.mid = new((heads + 2 * kv_heads) * head_dim), new(heads * head_dim), new(heads * head_dim), new(inner)
        self.att_bytes = npas.paged_attention_workspace_bytes(self.caches[0], heads, max_length)
        self.fc_bytes = max(b.workspace_bytes(sequences) for blk in self.blocks for b in (blk.up, blk.down))
        self.work = torch.empty(max(self.att_bytes, self.fc_bytes, 256), dtype=torch.uint8, device="cuda")   # calls of one stream share it

    def step(self, stream=None):
        """One token of every sequence: self.x [sequences][width] in, self.n out (the normed residual stream that the logits would read)."""
        S, W, H, KV, D, dt = self.S, self.width, self.H, self.KV, self.D, npas.BF16
        npas.gated_residual_norm(None, self.x, self.h, self.n, S, W, dt, pre_weight=self.first_norm, eps=EPS, stream=stream)
        for i, (b, cache) in enumerate(zip(self.blocks, self.caches)):
            npas.fc_sparse(b.qkv, self.n, self.qkv, S, None, npas.ACT_NONE, stream)
            npas.kv_append(cache, self.qkv[:, :H * D], self.qkv[:, H * D:(H + KV) * D], self.qkv[:, (H + KV) * D:], self.q, S, H, self.position,
                           cos_sin=self.cos_sin, rot_dim=D, stream=stream)
            npas.paged_attention(cache, self.q, self.ctx, H, self.length, self.max_length, D ** -0.5, workspace=self.work,
                                 workspace_bytes=self.att_bytes, stream=stream)
            npas.fc_sparse(b.out, self.ctx, self.branch, S, None, npas.ACT_NONE, stream)
            npas.gated_residual_norm(self.branch, self.h, self.h, self.n, S, W, dt, gate=b.gate[0], post_weight=b.post[0], pre_weight=b.pre[0],
                                     residual_scale=SCALE, eps=EPS, stream=stream)
            npas.fc_mxfp4(b.up, self.n, self.mid, S, None, npas.ACT_HARDSWISH, self.work, self.fc_bytes, stream)
            npas.fc_mxfp4(b.down, self.mid, self.branch, S, None, npas.ACT_NONE, self.work, self.fc_bytes, stream)
            npas.gated_residual_norm(self.branch, self.h, self.h, self.n, S, W, dt, gate=b.gate[1], post_weight=b.post[1], pre_weight=b.pre[1],
                                     residual_scale=SCALE, eps=EPS, stream=stream)
        return self.n

    def capture(self):
        """A HIP graph of one step (run one eagerly first: the first call on a handle sets kernel attributes)."""
        graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            self.step(stream.cuda_stream)
        return graph


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--sequences", type=int, default=16)
    ap.add_argument("--steps", type=int, default=200)
    args = ap.parse_args()
    d = Decoder(args.sequences, args.steps + 1)
    g = torch.Generator(device="cuda").manual_seed(0)
    tokens = torch.randn((args.steps, args.sequences, d.width), generator=g, device="cuda").bfloat16()
    d.x.copy_(tokens[0])
    d.step()
    graph = d.capture()
    for name, run in (("eager", d.step), ("graph", graph.replay)):
        torch.cuda.synchronize()
        t = time.perf_counter()
        for i in range(args.steps):
            d.x.copy_(tokens[i])
            d.position.fill_(i)
            d.length.fill_(i + 1)
            run()
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        print(f"{name}: {args.steps} steps of {args.sequences} sequences through {len(d.blocks)} blocks, {1e6 * t / args.steps:.1f} us a step, "
              f"{args.steps * args.sequences / t:.0f} tokens/s", flush=True)
    assert bool(torch.isfinite(d.n).all())


if __name__ == "__main__":
    main()

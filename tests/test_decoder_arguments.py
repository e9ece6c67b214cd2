"""Tensors that do not fit a decoder-block or 4-bit call are refused before anything is launched, by the CPython entry points and by the calls
through ctypes alike: too short, elements of another size, indices that are not 32-bit integers.  No GPU needed."""
import numpy as np
import pytest
import torch

import paper_2012_00596_amd as npas
from paper_2012_00596_amd import binding

T, H, KV, D, S, B, IN, OUT = 5, 4, 2, 64, 3, 4, 40, 7
BF, I32, I64, F64, U8 = torch.bfloat16, torch.int32, torch.int64, torch.float64, torch.uint8


def z(*shape, t=BF):
    return torch.zeros(shape, dtype=t)


def _cache():
    return npas.KvCache(z(9, KV, 16, D), z(9, KV, 16, D), z(S, 3, t=I32), npas.BF16)


def _calls():
    """By call: the function, the one through ctypes, the arguments in that one's order, and a change that the library refuses (so that
    the tensors as they are must have passed)."""
    cache, packed = _cache(), npas.pack_fc_mxfp4(np.ones((OUT, IN), np.uint16), npas.BF16)
    norm = dict(branch=z(T, IN), h=z(T, IN), h_out=z(T, IN), n_out=z(T, IN), T=T, D=IN, dtype=npas.BF16, gate=z(T, IN),
                post_weight=z(IN, t=torch.float32), pre_weight=z(IN, t=torch.float32), residual_scale=1.0, eps=1e-6, stream=None)
    append = dict(cache=cache, q=z(T, H, D), k=z(T, KV, D), v=z(T, KV, D), q_out=z(T, H, D), T=T, heads=H, positions=z(T, t=I32),
                  sequences=z(T, t=I32), cos_sin=z(9, D, t=torch.float32), rot_dim=D, kind=npas.ROTATE_HALVES, stream=None)
    attention = dict(cache=cache, q=z(S, H * D), y=z(S, H, D), heads=H, lengths=z(S, t=I32), max_length=32, scale=1.0, window=0,
                     lse=z(S, H, t=torch.float32), workspace=z(64, t=U8), workspace_bytes=64, stream=None)
    quantize = dict(x=z(B, IN), codes=z(B, 32, t=U8), scales=z(B, 2, t=U8), M=B, K=IN, dtype=npas.BF16, stream=None)
    dequantize = dict(codes=z(B, 32, t=U8), scales=z(B, 2, t=U8), y=z(B, IN), M=B, K=IN, dtype=npas.BF16, stream=None)
    fc = dict(packed=packed, x=z(B, IN), y=z(B, OUT), B=B, bias=z(OUT, t=torch.float32), act=npas.ACT_NONE, workspace=z(64, t=U8),
              workspace_bytes=64, stream=None)
    odd = z(200, t=U8)[1:]                    # codes at an address that is no multiple of 4
    return {"norm": (npas.gated_residual_norm, binding._gated_residual_norm, norm, dict(eps=-1.0)),
            "append": (npas.kv_append, binding._kv_append, append, dict(kind=2)),
            "attention": (npas.paged_attention, binding._paged_attention, attention, dict(max_length=0)),
            "quantize": (npas.mxfp4_quantize, binding._mxfp4_quantize, quantize, dict(codes=odd)),
            "dequantize": (npas.mxfp4_dequantize, binding._mxfp4_dequantize, dequantize, dict(codes=odd)),
            "fc": (npas.fc_mxfp4, binding._fc_mxfp4, fc, dict(act=9))}


def _run(name, change, through_ctypes):
    call, direct, args, _ = _calls()[name]
    args = {**args, **change}
    if not through_ctypes:
        call(**args)
    elif name == "fc":
        p = args["packed"]
        direct(*args.values(), p.IN, p.OUT, p.dtype)
    else:
        direct(*args.values())


SHORT, SIZE, ROWS, INDEX, FP32 = "shorter", "element size", "fewer rows", "32-bit integers", "not fp32"
BAD = [
    ("norm", dict(branch=z(T - 1, IN)), SHORT), ("norm", dict(h=z(T, IN - 1)), SHORT), ("norm", dict(h_out=z(IN)), SHORT),
    ("norm", dict(n_out=z(0, IN)), SHORT), ("norm", dict(h=z(T, IN, t=torch.float32)), SIZE), ("norm", dict(branch=z(T, IN, t=U8)), SIZE),
    ("norm", dict(gate=z(T, IN, t=torch.float32)), SIZE), ("norm", dict(gate=z(IN, t=F64)), SIZE), ("norm", dict(gate=z(T - 1, IN)), "gate is"),
    ("norm", dict(post_weight=z(IN - 1, t=torch.float32)), SHORT), ("norm", dict(pre_weight=z(IN)), SIZE),
    ("norm", dict(pre_weight=z(IN, t=I32)), FP32),
    ("append", dict(q=z(T - 1, H, D)), ROWS), ("append", dict(k=z(1, KV, D)), ROWS), ("append", dict(v=z(T - 1, KV * D)), ROWS),
    ("append", dict(q=z(T, H, D, t=torch.float32)), SIZE), ("append", dict(k=z(T, KV, D, t=F64)), SIZE),
    ("append", dict(q_out=z(T - 1, H, D)), SHORT), ("append", dict(q_out=z(T, H, D, t=torch.float32)), SIZE),
    ("append", dict(positions=z(T, t=I64)), SIZE), ("append", dict(positions=z(T, t=torch.float32)), INDEX),
    ("append", dict(positions=z(T - 1, t=I32)), SHORT), ("append", dict(sequences=z(T, t=I64)), SIZE),
    ("append", dict(sequences=z(1, t=I32)), SHORT), ("append", dict(sequences=z(T, t=torch.float32)), INDEX),
    ("append", dict(cos_sin=z(9, D, t=F64)), SIZE), ("append", dict(cos_sin=z(9, D, t=I32)), FP32), ("append", dict(cos_sin=z(9, D)), SIZE),
    ("attention", dict(q=z(S - 1, H * D)), ROWS), ("attention", dict(q=z(S, H, D, t=torch.float32)), SIZE),
    ("attention", dict(y=z(S - 1, H, D)), SHORT), ("attention", dict(y=z(S, H, D, t=torch.float32)), SIZE),
    ("attention", dict(lengths=z(S, t=I64)), SIZE), ("attention", dict(lengths=z(1, t=I32)), SHORT),
    ("attention", dict(lengths=z(S, t=torch.float32)), INDEX), ("attention", dict(lse=z(S, t=torch.float32)), SHORT),
    ("attention", dict(lse=z(S, H)), SIZE), ("attention", dict(workspace=z(63, t=U8)), SHORT),
    ("quantize", dict(x=z(B - 1, IN)), ROWS), ("quantize", dict(x=z(B, IN, t=torch.float32)), SIZE),
    ("quantize", dict(codes=z(B, 31, t=U8)), SHORT), ("quantize", dict(scales=z(B, 1, t=U8)), SHORT),
    ("quantize", dict(scales=z(B, 2, t=I32)), SIZE),
    ("dequantize", dict(codes=z(B - 1, 32, t=U8)), SHORT), ("dequantize", dict(scales=z(1, t=U8)), SHORT),
    ("dequantize", dict(y=z(B, IN - 1)), SHORT), ("dequantize", dict(y=z(B, IN, t=torch.float32)), SIZE),
    ("fc", dict(x=z(B - 1, IN)), ROWS), ("fc", dict(x=z(B, IN, t=torch.float32)), SIZE), ("fc", dict(y=z(B, OUT - 1)), SHORT),
    ("fc", dict(y=z(B, OUT, t=torch.float32)), SIZE), ("fc", dict(bias=z(OUT - 1, t=torch.float32)), SHORT), ("fc", dict(bias=z(OUT)), SIZE),
    ("fc", dict(bias=z(OUT, t=I32)), FP32), ("fc", dict(workspace=z(63, t=U8)), SHORT)]


@pytest.mark.parametrize("through_ctypes", [False, True])
@pytest.mark.parametrize("name,change,why", BAD, ids=lambda v: None if not isinstance(v, dict) else "-".join(v))
def test_tensors_that_do_not_fit_are_refused(name, change, why, through_ctypes):
    with pytest.raises(AssertionError, match=why):
        _run(name, change, through_ctypes)


@pytest.mark.parametrize("through_ctypes", [False, True])
@pytest.mark.parametrize("name", ["norm", "append", "attention", "quantize", "dequantize", "fc"])
def test_tensors_that_fit_reach_the_library(name, through_ctypes):
    """As they are, and where they are larger than the call needs or hold bit patterns of their size; the library's own refusal tells."""
    refused = _calls()[name][3]
    larger = {"norm": dict(branch=z(T + 1, IN), h=z(T, IN, t=torch.int16), gate=z(1, IN)),
              "append": dict(q=z(T + 2, H * D), k=z(T, KV, D, t=torch.int16), sequences=None, positions=z(T + 9, t=I32)),
              "attention": dict(q=z(S + 1, H, D), y=z(S + 1, H, D), lse=None, lengths=z(S + 1, t=I32), workspace=z(99, t=U8)),
              "quantize": dict(x=z(B, 2 * IN)[:, IN:]), "dequantize": dict(y=z(B + 1, IN, t=torch.int16)),
              "fc": dict(x=z(B + 1, IN, t=torch.int16), y=z(B + 1, OUT), bias=None, workspace=None, workspace_bytes=0)}[name]
    for change in ({}, larger):
        with pytest.raises(npas.NpasError) as e:
            _run(name, {**change, **refused}, through_ctypes)
        assert e.value.code == npas.E_SHAPE


def test_caches_of_another_type_are_refused():
    table = z(S, 3, t=I32)
    for k, v in ((z(9, KV, 16, D, t=torch.float32), z(9, KV, 16, D, t=torch.float32)), (z(9, KV, 16, D), z(9, KV, 16, D, t=torch.float32))):
        with pytest.raises(AssertionError):
            npas.KvCache(k, v, table, npas.BF16)

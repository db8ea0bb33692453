"""Inputs and checks of the tests of attention over sequences."""
import numpy as np
import torch

from oracle import seq_oracle

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# Half a step of the type, and what is held in fp32 on the way: a score of D products and its exponential.  The sums are at most 512 terms here
# (2^-24 each, in any order below 2^-15); scores reach a few tens, so a weight is off by their 2^-24 times that.
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
FP32 = 2.0 ** -15
# fp16: a weight below 2^-14 of the largest is rounded to a multiple of 2^-24; it counts from 2^-8 of the maximum on at worst
TINY = {"f32": 0.0, "f16": 2.0 ** -24, "bf16": 0.0}


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def normal(g, shape, dtype, std=1.0):
    return torch.from_numpy((std * g.standard_normal(shape)).astype(np.float32)).to(TYPES[dtype]).cuda()


def check(name, got, want, bound):
    got = f64(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    with np.errstate(invalid="ignore"):
        off = np.where((got == want) | (np.isnan(got) & np.isnan(want)), 0.0, np.abs(got - want))
    bad = ~(off <= bound + 1e-30)
    assert not bad.any(), f"{name}: {bad.sum()} of {bad.size} off, worst {np.nanmax(off / (bound + 1e-30)):.3g} times the bound, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


def expect(q, k, v, dout=None, dtype="f32", **mask):
    """The oracle's results and bounds for tensors of `dtype`."""
    host = {n: (f64(x) if n == "slopes" else None if x is None else x.cpu().numpy()) if isinstance(x, torch.Tensor) else x for n, x in mask.items()}
    return seq_oracle.attention(f64(q), f64(k), f64(v), f64(dout), u=HALF[dtype], e=FP32, tiny=TINY[dtype], **host)

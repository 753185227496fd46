"""What the tests of the operators around the FP8 layers share: plain 64-bit
references on the CPU, and the checks of codes and scales against them."""
import ctypes

import numpy as np
import torch

import paper_2609_22870_amd as fp8q

from _par import bf16_half_ulp

DEV = "cuda:0"
F64 = torch.float64
E4M3_MAX, E5M2_MAX = 448.0, 57344.0


def values(codes, e5m2=False):
    """The values of FP8 codes, in 64 bits."""
    return codes.cpu().contiguous().view(torch.float8_e5m2 if e5m2 else torch.float8_e4m3fn).float().to(F64)


def block_scales(scales, rows, cols):
    """1x128 scales [cols / 128][rows] as [rows, cols]."""
    return scales.cpu().to(F64).view(cols // 128, rows).t().repeat_interleave(128, dim=1)


def _cast(v, e5m2):
    top = E5M2_MAX if e5m2 else E4M3_MAX
    f8 = torch.float8_e5m2 if e5m2 else torch.float8_e4m3fn
    return v.clamp(-top, top).float().to(f8).float().to(F64)


def check_units(codes, scales, v, rel, e5m2=False, pow2=False, tiny=0.0):
    """codes [R, C] in units of 128 along a row with scales [R, C] (one value a
    unit, repeated), against the 64-bit values v: every scale is amax / F_max
    (or the power of two) to the relative error `rel` that v itself may have, 1
    for a unit of zeros; every code is the nearest to v / S for some v within
    `rel` (and S as it is, with a further 2^-22 for the quotient)."""
    top = E5M2_MAX if e5m2 else E4M3_MAX
    amax = v.abs().view(v.shape[0], -1, 128).amax(dim=2)
    s = scales[:, ::128]
    if pow2:
        want = torch.exp2(torch.ceil(torch.log2(amax / top)))
        near = torch.exp2(torch.ceil(torch.log2(amax * (1 + rel) / top)))
        far = torch.exp2(torch.ceil(torch.log2(amax * (1 - rel) / top)))
        ok = (s == want) | (s == near) | (s == far)
        ok = torch.where(amax == 0, s == 1, ok)
    else:
        ok = (s - amax / top).abs() <= (rel + 2.0 ** -23) * amax / top + 2.0 ** -149
        ok = torch.where(amax <= tiny, (s == 1) | ok, ok)
    assert bool(ok.all()), ("scales", s[~ok][:5], amax[~ok][:5] / top)
    q = v / scales
    d = rel + 2.0 ** -22
    lo, hi = torch.minimum(_cast(q * (1 - d), e5m2), _cast(q * (1 + d), e5m2)), torch.maximum(
        _cast(q * (1 - d), e5m2), _cast(q * (1 + d), e5m2))
    got = values(codes, e5m2)
    bad = ~((got >= lo) & (got <= hi))
    assert not bool(bad.any()), ("codes", got[bad][:5], q[bad][:5], int(bad.sum()))


def bf16_half(x):
    """Half a bf16 unit at magnitude x: the largest error of rounding to bf16 a
    value of at most that magnitude."""
    return torch.from_numpy(bf16_half_ulp(x.abs().numpy()))


def within(got, ref, bound, what):
    got, bad = got.cpu().to(F64), None
    d = (got - ref).abs()
    bad = ~(d <= bound)
    print("  %s: worst %.3g of its bound" % (what, float((d / torch.as_tensor(bound).clamp(min=1e-300)).max())),
          flush=True)
    assert not bool(bad.any()), (what, got[bad][:5], ref[bad][:5], int(bad.sum()))


def gated_route(M, F, K):
    """(kernel, whether quantized output goes through bf16) of a gated product."""
    fn = fp8q.lib().fp8q_gated_route
    fn.argtypes, fn.restype = [ctypes.c_int64] * 3, ctypes.c_int
    r = fn(M, F, K)
    names = ("large", "mid", "eight waves", "small", "two K groups", "thin", "split-K", "half")
    thin = ("16 x 16", "16 x 32", "32 x 32", "32 x 64", "64 x 64")
    name = names[r % 10]
    return name + (" " + thin[r % 100 // 10] if name == "thin" else ""), r >= 100


def strided(t, extra):
    """t in a wider buffer: the same values, rows `extra` elements further apart."""
    wide = torch.zeros(t.shape[0], t.shape[1] + extra, dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def bits(t):
    return t.detach().cpu().contiguous().view(torch.uint8).numpy()


def same(a, b, what):
    assert np.array_equal(bits(a), bits(b)), what

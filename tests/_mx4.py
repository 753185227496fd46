"""MXFP4 in 64 bits on the CPU, from its definition: what the tests of the 4-bit
operators share."""
import torch

from _ops import F64

LEVELS = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=F64)


def padded(cols):
    return -(-cols // 256) * 256


def quantize(x):
    """(codes 0 .. 15 [rows, P] uint8, scale bytes [rows, P / 32] int64) of a bf16 x: per unit
    of 32 S = 2^(floor(log2 amax) - 2), at least 2^-127; the level nearest to |x| / S, in the
    middle between two the one of even index, 6 above."""
    rows, cols = x.shape
    v = torch.zeros(rows, padded(cols), dtype=F64)
    v[:, :cols] = x.to(F64)
    sign = torch.zeros(rows, padded(cols), dtype=torch.bool)
    sign[:, :cols] = torch.signbit(x)
    u = v.abs().view(rows, -1, 32)
    amax = u.amax(dim=2)
    bad = ~torch.isfinite(amax)
    _, e = torch.frexp(torch.where(bad, torch.ones_like(amax), amax))  # (amax = m 2^e, m in [0.5, 1))
    k = (e.long() - 3).clamp(min=-127)
    k = torch.where(amax == 0, torch.zeros_like(k), k)
    a = u / torch.exp2(k.to(F64))[:, :, None]
    middle = (LEVELS[1:] + LEVELS[:-1]) / 2
    i = (a[..., None] > middle).sum(dim=-1)  # (a middle itself stays below)
    i = i + ((i < 7) & (a == middle[i.clamp(max=6)]) & (i % 2 == 1)).long()
    codes = i.view(rows, -1) + 8 * sign.long()
    return codes.to(torch.uint8), torch.where(bad, torch.full_like(k, 255), k + 127)


def values(codes, scales):
    """The values of codes [rows, P] with scale bytes [rows, P / 32], in 64 bits."""
    v = LEVELS[(codes & 7).long()] * torch.where(codes >= 8, -1.0, 1.0)
    s = torch.exp2(scales.to(F64) - 127.0)
    s = torch.where(scales == 255, torch.full_like(s, float("nan")), s)
    return v * s.repeat_interleave(32, dim=1)


def packed(codes, scales):
    """The library's layout: two codes a byte, the first in the low half; scale bytes [P /
    256][rows][8]."""
    rows = codes.shape[0]
    return (codes[:, 0::2] | codes[:, 1::2] << 4).contiguous(), scales.to(torch.uint8).view(rows, -1, 8).permute(
        1, 0, 2).reshape(-1).contiguous()


def unpacked(codes, scales):
    """The reverse, from tensors on any device."""
    codes, scales = codes.cpu(), scales.cpu()
    rows = codes.shape[0]
    c = torch.stack((codes & 15, codes >> 4), dim=2).reshape(rows, -1)
    return c, scales.view(-1, rows, 8).permute(1, 0, 2).reshape(rows, -1).long()


def random_operand(rows, K, seed, spread=6):
    """Codes and scale bytes at random: every code, scales over 2^-spread .. 2^spread."""
    g = torch.Generator().manual_seed(seed)
    codes = torch.randint(0, 16, (rows, K), generator=g).to(torch.uint8)
    return codes, torch.randint(127 - spread, 128 + spread, (rows, K // 32), generator=g)

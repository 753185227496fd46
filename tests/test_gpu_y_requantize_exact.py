"""The requantizer bit for bit: v = RN32(S code), S' = RN32(amax / 448), codes of
RN32(v / S'), each a single IEEE operation on the host."""
import numpy as np
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, same, values

pytestmark = pytest.mark.gpu


def check(codes, scales):
    """codes uint8 [rows, cols] and scales fp32 [cols / 128, rows] on the host, rows a multiple of 128."""
    rows, cols = codes.shape
    ct, st = fp8q.requantize_transposed(torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).view(-1).to(DEV))
    v = values(torch.from_numpy(codes)).float().numpy() * np.repeat(scales, 128, axis=0).T
    s = np.abs(v).reshape(rows // 128, 128, cols).max(axis=1) / np.float32(448)
    s[s == 0] = 1
    q = np.clip(v / np.repeat(s, 128, axis=0), -448, 448).astype(np.float32)
    same(st, torch.from_numpy(s).view(-1), "scales")
    same(ct, torch.from_numpy(q).to(torch.float8_e4m3fn).view(torch.uint8).t(), "codes")


def test_random():
    rng = np.random.default_rng(91)
    rows, cols = 2048, 1024
    codes = rng.integers(0, 256, (rows, cols), dtype=np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x3A
    check(codes, np.exp2(rng.uniform(-12, 4, (cols // 128, rows))).astype(np.float32))


def test_middles_between_codes():
    """One row of 448 k in every unit makes S' = k, of 19 bits; the others, m k with m the
    middle between two codes, have quotients of m exactly."""
    rng = np.random.default_rng(92)
    rows, cols = 1024, 1024
    k = rng.integers(1 << 17, 1 << 18, (cols // 128, rows // 128)) * 2 + 1
    m = np.concatenate([(1 + np.arange(1, 16, 2) / 16) * 2.0 ** e for e in range(-4, 8)])
    m = rng.choice(m, (cols // 128, rows))
    m[:, ::128] = 448
    codes = rng.choice(np.array([0x38, 0xB8], np.uint8), (rows, cols))  # +-1
    scales = m * np.repeat(k, 128, axis=1) * 2.0 ** -22
    assert (scales.astype(np.float32) == scales).all()
    check(codes, scales.astype(np.float32))

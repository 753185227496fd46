"""Units whose scale is an fp32 subnormal of a few bits, in every operator that
forms its own codes.  There S = RN32(amax / F_max) may be up to a third below
amax / F_max, so that x / S passes F_max: such magnitudes clamp to F_max, and a
finite input never gives NaN or an infinity.

Every value here is a whole number n of 2^-149, made without a rounding, so scales
and codes are known bit for bit: S = RN32(n_max 2^-149 / F_max), 1 where that is
0, and the code of RN32(x / S) clamped."""
import numpy as np
import pytest
import torch

import paper_2609_22870_amd as fp8q

from _ops import DEV, same

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -149
# Largest magnitudes, in 2^-149: where S is 0, 1, the largest that rounds down to S = 1, 2 and 14, exact multiples of
# F_max and the last that overflows the rounding to F_max (464; 61440), and larger ones
E4M3_TOPS = (200, 300, 448, 463, 464, 600, 671, 672, 1119, 1120, 6272, 6493, 6494, 20000)
# (products of two numbers below 256 and a power of two: the gated gradient's operands are bf16)
E5M2_TOPS = (57344, 65025, 130050, 195 * 5 * 64, 253 * 255 * 2, 251 * 16, 255 * 255 * 16)


def expected(n, top, e5m2=False):
    """Scales and code bytes of units (rows of whole numbers n of 2^-149)."""
    x = (n.astype(np.float64) * TINY).astype(np.float32)
    s = np.abs(x).max(axis=1) / np.float32(top)
    s = np.where(s == 0, np.float32(1), s).astype(np.float32)
    q = np.clip(x / s[:, None], -top, top)
    f8 = torch.float8_e5m2 if e5m2 else torch.float8_e4m3fn
    return torch.from_numpy(s), torch.from_numpy(q.astype(np.float32)).to(f8).view(torch.uint8)


def test_the_numbers_reach_the_overflow():
    """(of the cases: quotients past the last value that rounds to F_max)"""
    for tops, top, last in ((E4M3_TOPS, 448, 464), (E5M2_TOPS, 57344, 61440)):
        x = (np.array(tops) * TINY).astype(np.float32)
        s = x / np.float32(top)
        q = x[s > 0] / s[s > 0]
        assert (q >= last).sum() >= 2 and (q <= top).any()


def units(tops, length=128, seed=61):
    """One unit a top: whole numbers up to it, the top itself with both signs, zeros."""
    rng = np.random.default_rng(seed)
    n = np.stack([rng.integers(-t, t + 1, length) for t in tops])
    n[:, 3], n[:, 77], n[:, 5] = tops, [-t for t in tops], 0
    return n


@pytest.mark.parametrize("what", ["block", "row"])
def test_norm(what):
    """x of +-1 with eps 0 has rstd 1: y is the weight, in fp32."""
    n = units(E4M3_TOPS)
    x = torch.ones(3, 128 * len(E4M3_TOPS), dtype=torch.bfloat16)
    x[1] = -1
    x[2, ::2] = -1
    w = torch.from_numpy((n.reshape(-1) * TINY).astype(np.float32))
    if what == "block":
        codes, scales, _, rstd = fp8q.rmsnorm_quantize(x.to(DEV), w.to(DEV), 0.0)
        y = (x.double().numpy() * n.reshape(-1)).reshape(-1, 128)
        s, c = expected(y, 448)
        s = s.view(3, -1).t().reshape(-1)
        assert bool((rstd == 1).all())
        same(scales, s, "scales")
        same(codes, c.view(3, -1), "codes")
        return
    for i in range(len(E4M3_TOPS)):
        part = slice(128 * i, 128 * (i + 1))
        codes, scales, _, _ = fp8q.rmsnorm_quantize(x[:, part].contiguous().to(DEV), w[part].to(DEV), 0.0, fp8q.ROW)
        s, c = expected(x[:, part].double().numpy() * n[i], 448)
        same(scales, s, ("scales", E4M3_TOPS[i]))
        same(codes, c, ("codes", E4M3_TOPS[i]))


def test_requantize():
    """Codes of 0, +-1/2 and +-1 under subnormal scales: a column's unit holds scale n of
    every row, whole numbers again."""
    cols = 128 * 2
    tops = [t for t in E4M3_TOPS if t % 2 == 0]
    rows = 128 * len(tops)
    rng = np.random.default_rng(62)
    scale = np.concatenate([np.r_[t, rng.integers(0, t // 2 + 1, 127) * 2] for t in tops])  # (even: halves are whole)
    lut = np.array([0x00, 0x38, 0xb8, 0x30, 0xb0], np.uint8)
    value = np.array([0.0, 1.0, -1.0, 0.5, -0.5])
    pick = rng.integers(0, 5, (rows, cols))
    pick[::128] = rng.integers(1, 3, (len(tops), cols))  # the top itself in every column
    scales = torch.from_numpy((scale * TINY).astype(np.float32)).repeat(cols // 128).to(DEV)
    ct, st = fp8q.requantize_transposed(torch.from_numpy(lut[pick]).to(DEV), scales)
    n = value[pick] * scale[:, None]
    s, c = expected(n.T.reshape(-1, 128), 448)  # unit (column, rows / 128)
    same(ct, c.view(cols, rows), "codes")
    same(st, s.view(cols, -1).t().reshape(-1), "scales")


@pytest.mark.parametrize("along", ["rows", "columns"])
@pytest.mark.parametrize("e5m2", [False, True])
def test_gated_backward(e5m2, along):
    """dH of a 2^-99, G and U of b 2^-49, whole a and b below 256: s is 1/2, and dU = dH G s
    and dG = dH U s are a b 2^-149 exactly.  along: a, and with it the unit's top,
    goes by row or by column."""
    top = 57344.0 if e5m2 else 448.0
    M = F = 256
    rng = np.random.default_rng(63)
    # rows of tops that S rounds down for, among others
    if e5m2:
        a = rng.choice([255, 254, 253, 16, 240], M)
        # (255 x 255 = 65025: S = 1; 510 x 255 and 240 x 510 = 122400: S = 2)
        b = np.stack([rng.integers(-255, 256, M) for _ in range(2 * F)]) * rng.choice([1, 2, 4], 2 * F)[:, None]
        b[::16] = rng.choice([255, 510, -255, -510], b[::16].shape)
    else:
        a = rng.choice([1, 2, 5, 11, 9, 27], M)
        b = np.stack([rng.integers(-61, 62, M) for _ in range(2 * F)])
        b[::16] = rng.choice([61, -61, 241, -241], b[::16].shape)
    if along == "rows":
        dh, pre = np.repeat(a[:, None], F, axis=1), b.T  # [M, F], [M, 2 F]
    else:
        dh, pre = np.repeat(a[None, :], M, axis=0), np.concatenate((b[:F], b[F:]), axis=0).T
    bf = lambda v, e: torch.from_numpy(np.ascontiguousarray(v * 2.0 ** e, np.float32)).bfloat16()  # noqa: E731
    d, p = bf(dh, -99), bf(pre, -49)
    assert bool((d.double().numpy() == dh * 2.0 ** -99).all() and (p.double().numpy() == pre * 2.0 ** -49).all())
    cr, sr, ct, st = fp8q.gated_backward(d.to(DEV), p.to(DEV), e5m2=e5m2)
    # D = [dG | dU]: dG from U, dU from G
    D = np.concatenate((dh * pre[:, F:], dh * pre[:, :F]), axis=1)
    s, c = expected(D.reshape(-1, 128), top, e5m2)
    same(sr, s.view(M, -1).t().reshape(-1), "scales")
    assert np.array_equal(cr.cpu().numpy() & 0x7f, c.view(M, -1).numpy() & 0x7f), "codes"
    s, c = expected(np.ascontiguousarray(D.T).reshape(-1, 128), top, e5m2)
    same(st, s.view(2 * F, -1).t().reshape(-1), "transposed scales")
    assert np.array_equal(ct.cpu().numpy() & 0x7f, c.view(2 * F, -1).numpy() & 0x7f), "transposed codes"
    nonzero = D != 0
    assert np.array_equal((cr.cpu().numpy() >> 7)[nonzero], (D < 0)[nonzero]), "signs"

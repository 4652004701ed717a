"""How exact a rotation is before its rounding to 32 bits and to the type: results bit for bit, but where the exact value lies beside a border.

With A = |a cos|, B = |b sin| (times the amplitude), as csd_rotate.cuh adds them: products of the first 12 bits of cosine and sine and their difference
with its error are exact.  The rests, below 2^-11 of them, are rounded to 24 bits, 2^-35 (A + B); the second product of the rests is added to the error,
2^-35 B, and the first to that, 2^-35 (A + B): 3 * 2^-35 (A + B) in all."""
import numpy as np
import pytest
import torch

from paper_2503_05330_amd import verify

BF, F16 = torch.bfloat16, torch.float16
CASES = [  # dim, head dim, interleaved, amplitude, furthest position
    (128, 128, False, 1.0, 1 << 12), (128, 128, True, 1.25, 1 << 24), (64, 128, False, 0.7, 1 << 24), (96, 96, True, 1.0, 1 << 12)]


def inputs(dim, D, far):
    gen = torch.Generator()
    gen.manual_seed(dim + far)
    T, H = 4096, 2
    return torch.randn((T, H, D), generator=gen), torch.randint(-far, far + 1, (T,), generator=gen, dtype=torch.int32)


def halves(x, dim, interleaved):
    return (x[..., 0:dim:2], x[..., 1:dim:2]) if interleaved else (x[..., :dim // 2], x[..., dim // 2:dim])


def between(x, positions, turns, dim, interleaved, amplitude, dtype):
    """The least and the largest that the pairs' first and second results may be, from 64 bits of mantissa."""
    wide = np.longdouble
    assert np.finfo(wide).nmant >= 63
    t = positions.numpy().astype(wide)[:, None] * turns.cpu().numpy().astype(wide)
    angle = (t - np.rint(t)) * (2 * wide("3.14159265358979323846264338327950288"))
    cos, sin = (amplitude * f(angle)[:, None] for f in (np.cos, np.sin))
    a, b = (y.double().numpy().astype(wide) for y in halves(x, dim, interleaved))
    out = []
    for u, v, s in ((a, b, -sin), (b, a, sin)):
        want = u * cos + v * s
        # t is below 2^22 turns and rounded to 64 bits, 2^-43; and again 2^-53 where 64-bit arithmetic makes and multiplies sine and cosine
        off = 3 * wide(2) ** -35 * (abs(u * cos) + abs(v * s)) + wide(2) ** -39 * amplitude * (abs(u) + abs(v)) + wide(2) ** -149
        out.append([torch.from_numpy((want + sign * off).astype(np.float32)).to(dtype).float() for sign in (-1, 1)])
    return out


def outside(got, bounds, dim, interleaved):
    """How many of the pairs' results are out of their bounds."""
    return sum(int(((y < low) | (y > high)).sum()) for y, (low, high) in zip(halves(got.float(), dim, interleaved), bounds))


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("dim,D,interleaved,amplitude,far", CASES)
def test_products_in_32_bits_would_be_told(dim, D, interleaved, amplitude, far, dtype):
    x, positions = inputs(dim, D, far)
    x, turns = x.to(dtype), verify.Rotary(dim, device="cpu").turns
    bounds = between(x, positions, turns, dim, interleaved, amplitude, dtype)
    # the bounds are of one value for all but one of some 10^4 (a border of the type within 2^-33 of 2^-8 or 2^-11; where terms cancel, more)
    assert all((low != high).double().mean() < 1e-4 for low, high in bounds)
    t = positions.double()[:, None] * turns
    angle = 2 * torch.pi * (t - t.round())
    cos, sin = ((amplitude * f(angle)).float()[:, None] for f in (torch.cos, torch.sin))
    a, b = (y.float() for y in halves(x, dim, interleaved))
    plain = x.clone()
    for y, z in zip(halves(plain, dim, interleaved), (a * cos - b * sin, b * cos + a * sin)):
        y.copy_(z)
    assert outside(plain, bounds, dim, interleaved) > 0
    # and what is right is not
    exact = x.clone()
    for y, (low, high) in zip(halves(exact, dim, interleaved), bounds):
        y.copy_(high)
    assert outside(exact, bounds, dim, interleaved) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("dim,D,interleaved,amplitude,far", CASES)
def test_rotation_bit_for_bit(dim, D, interleaved, amplitude, far, dtype):
    x, positions = inputs(dim, D, far)
    x, rotary = x.to(dtype), verify.Rotary(dim, interleaved=interleaved, amplitude=amplitude)
    got = verify.rotate(x.cuda(), positions.cuda(), rotary).cpu()
    assert outside(got, between(x, positions, rotary.turns, dim, interleaved, rotary._cfg.amplitude, dtype), dim, interleaved) == 0

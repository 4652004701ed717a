"""Rotary positions against a plain implementation in 64 bits, alone and with the write to the cache."""
import math

import pytest
import torch

from paper_2503_05330_amd import binding, verify
from test_verify import BF, F16, ROUND, gen, held, ints, normal, same  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu


def plain(x, positions, frequencies, dim, interleaved, amplitude=1.0):
    """Pairs turned as complex numbers."""
    y = x.double().clone()
    angle = (positions.double()[..., None] * frequencies.to(x.device))[..., None, :]
    turn = torch.complex(angle.cos(), angle.sin()) * amplitude
    if interleaved:
        z = torch.complex(y[..., 0:dim:2], y[..., 1:dim:2]) * turn
        y[..., 0:dim:2], y[..., 1:dim:2] = z.real, z.imag
    else:
        z = torch.complex(y[..., :dim // 2], y[..., dim // 2:dim]) * turn
        y[..., :dim // 2], y[..., dim // 2:dim] = z.real, z.imag
    return y


def near(got, want, x, dtype, dim, interleaved, amplitude=1.0):
    """One rounding to the type, and in 32 bits: the angle and its sine and cosine 2^-22, two products and a sum, of |a| + |b|."""
    size = torch.zeros_like(want)
    y = x.double().abs()
    if interleaved:
        size[..., 0:dim:2] = size[..., 1:dim:2] = y[..., 0:dim:2] + y[..., 1:dim:2]
    else:
        size[..., :dim // 2] = size[..., dim // 2:dim] = y[..., :dim // 2] + y[..., dim // 2:dim]
    error = (got.double() - want).abs() - ROUND[dtype] * want.abs() - 2.0 ** -20 * abs(amplitude) * size - (2.0 ** -25 if dtype == F16 else 0)
    assert error.max().item() <= 0, error.max().item()
    assert torch.equal(got[..., dim:], x[..., dim:])


def frequencies(dim, base=10000.0):
    return base ** (torch.arange(0, dim, 2, dtype=torch.float64) / -dim)


SHAPES = [  # leading axes, heads, head dim, rotated
    ((1,), 1, 64, 64), ((3,), 5, 128, 128), ((4, 9), 8, 96, 48), ((2, 3, 7), 10, 128, 64), ((70,), 3, 256, 256), ((129,), 40, 64, 16),
    ((8,), 7, 80, 32), ((33,), 2, 512, 512), ((1000,), 36, 128, 128), ((5,), 1024, 64, 64), ((9,), 3, 24, 16), ((11,), 6, 512, 256)]


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rotation(gen, shape, interleaved, dtype):
    lead, H, D, dim = SHAPES[shape]
    print(SHAPES[shape], interleaved, dtype, flush=True)
    x = normal(gen, (*lead, H + 3, D), dtype)[..., :H, :] if shape % 2 else normal(gen, (*lead, H, D), dtype)
    positions = torch.randint(-10, 10000, lead, generator=gen, device="cuda", dtype=torch.int32)
    rotary = verify.Rotary(dim, interleaved=interleaved)
    got = verify.rotate(x, positions, rotary)
    assert got.shape == x.shape and got.is_contiguous()
    near(got, plain(x, positions, frequencies(dim), dim, interleaved), x, dtype, dim, interleaved)
    other = torch.full((*lead, 2 * H, D), 3.0, dtype=dtype, device="cuda")
    assert verify.rotate(x, positions, rotary, out=other[..., H:, :]).data_ptr() == other[..., H:, :].data_ptr()
    assert torch.equal(other[..., H:, :], got) and (other[..., :H, :] == 3).all()
    mine = x.clone() if shape % 2 == 0 else normal(gen, (*lead, H + 3, D), dtype)[..., :H, :].copy_(x)
    verify.rotate(mine, positions, rotary, out=mine)
    assert torch.equal(mine, got)


def test_far_positions(gen):
    positions = torch.tensor([0, 1, -1, 1 << 20, (1 << 24) - 1, 1 << 30, (1 << 31) - 1, -(1 << 31)], dtype=torch.int32, device="cuda")
    x = normal(gen, (8, 4, 128), F16)
    near(verify.rotate(x, positions, verify.Rotary(128)), plain(x, positions, frequencies(128), 128, False), x, F16, 128, False)
    assert torch.equal(verify.rotate(x, torch.zeros_like(positions), verify.Rotary(128)), x)


@pytest.mark.parametrize("factor,original,low,high,base", [(4.0, 0, 1.0, 4.0, 10000.0), (8.0, 8192, 1.0, 4.0, 500000.0), (32.0, 4096, 1.0, 32.0, 10000.0)])
def test_scaled_for_longer_contexts(gen, factor, original, low, high, base):
    dim = 128
    f = frequencies(dim, base)
    want = f / factor
    if original:
        want = torch.tensor([y if original * y / (2 * math.pi) >= high else z if original * y / (2 * math.pi) <= low else
                             z + (y - z) * (original * y / (2 * math.pi) - low) / (high - low) for y, z in zip(f.tolist(), want.tolist())], dtype=torch.float64)
        assert (want == f).any() and (want == f / factor).any()
    rotary = verify.Rotary(dim, base=base, factor=factor, original=original, low=low, high=high, amplitude=1.25)
    assert ((rotary.turns.cpu() * 2 * math.pi - want).abs() <= 1e-14 * want).all()
    x = normal(gen, (50, 3, dim), BF)
    positions = torch.arange(50, dtype=torch.int32, device="cuda") * 2621
    near(verify.rotate(x, positions, rotary), plain(x, positions, want, dim, False, 1.25), x, BF, dim, False, 1.25)
    given = verify.Rotary(dim, frequencies=want, amplitude=1.25)
    near(verify.rotate(x, positions, given), plain(x, positions, want, dim, False, 1.25), x, BF, dim, False, 1.25)


def test_infinities_and_nan_stay_in_their_pairs(gen):
    x = normal(gen, (4, 2, 64), BF)
    x[1, 0, 5], x[2, 1, 40] = torch.inf, torch.nan
    got = verify.rotate(x, ints([3, 4, 5, 6]), verify.Rotary(64))
    odd = ~got.isfinite()
    assert odd[1, 0, 5] and odd[1, 0, 37] and odd[2, 1, 8] and odd[2, 1, 40] and int(odd.sum()) == 4


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("P,N,n,H,Hk,D,dim,interleaved", [(1, 1, 1, 1, 1, 64, 64, False), (2, 3, 5, 8, 2, 128, 128, False), (1, 7, 9, 28, 4, 128, 64, True),
                                                         (3, 2, 2, 6, 3, 96, 96, True), (2, 2, 17, 4, 2, 96, 48, False), (1, 5, 3, 16, 8, 256, 128, False),
                                                         (2, 1, 33, 12, 12, 64, 32, True), (64, 16, 9, 8, 2, 64, 64, False)])
def test_written_as_rotated_and_then_written(gen, P, N, n, H, Hk, D, dim, interleaved, fp8, dtype):
    print(P, N, n, H, Hk, D, dim, interleaved, fp8, dtype, flush=True)
    cap = n + 30
    one, two = (verify.PathCache(P, N, 4, cap, H, Hk, D, n, n_layers=2, dtype=dtype, fp8=fp8) for _ in range(2))
    old = normal(gen, (P, N, cap, Hk, D), dtype)
    for c in (one, two):
        c.write(0, old, old)
        c.write(1, old, old)
    rotary = verify.Rotary(dim, interleaved=interleaved)
    for turn in range(3):
        if turn == 0:
            q, k, v = normal(gen, (P, N, n, H, D), dtype), normal(gen, (P, N, n, Hk, D), dtype), normal(gen, (P, N, n, Hk, D), dtype)
        else:
            qkv = normal(gen, (P, N, n, H + 2 * Hk, D), dtype)
            q, k, v = qkv[..., :H, :], qkv[..., H:H + Hk, :], qkv[..., H + Hk:, :]
        start = None if turn == 0 else torch.randint(0, cap - n + 1, (P, N), generator=gen, device="cuda", dtype=torch.int32)
        counts = None if turn == 1 else torch.randint(0, n + 1, (P, N), generator=gen, device="cuda", dtype=torch.int32)
        positions = torch.randint(0, 5000, (P, N, n), generator=gen, device="cuda", dtype=torch.int32)
        got = one.write_rotated(1, q, k, v, rotary, positions, start, counts)
        assert torch.equal(got, verify.rotate(q, positions, rotary))
        two.write(1, verify.rotate(k, positions, rotary), v, start, counts)
        for layer in range(2):
            for a, b in zip(one.read(layer, cap), two.read(layer, cap)):
                assert torch.equal(a, b)
    assert one.status() == 0


def test_positions_outside_of_the_cache_are_dropped_and_reported(gen):
    c = verify.PathCache(1, 3, 0, 20, 4, 2, 64, 4)
    zero = torch.zeros((1, 3, 20, 2, 64), dtype=BF, device="cuda")
    c.write(0, zero, zero)
    qkv = normal(gen, (1, 3, 4, 8, 64), BF)
    q, k, v = qkv[..., :4, :], qkv[..., 4:6, :], qkv[..., 6:, :]
    at = torch.zeros((1, 3, 4), dtype=torch.int32, device="cuda")
    rotary = verify.Rotary(64)
    assert torch.equal(c.write_rotated(0, q, k, v, rotary, at, ints([[0, 16, 30]]), ints([[-3, 4, 0]])), q)
    assert c.status() == 0
    c.write_rotated(0, q, k, v, rotary, at, ints([[-2, 18, 16]]))
    assert c.status() == binding.STATUS_CAPACITY
    got = c.read(0, 20)[1]
    assert same(got[0, 0, :2], v[0, 0, 2:]) and same(got[0, 1, 18:], v[0, 1, :2]) and same(got[0, 2, 16:], v[0, 2])
    assert not got[0, 0, 2:].any() and not got[0, 2, :16].any()


def test_another_stream_and_graph_replays(gen):
    P, N, n, H, Hk, D = 2, 3, 4, 8, 2, 64
    c = verify.PathCache(P, N, 0, 40, H, Hk, D, n, fp8=True)
    qkv, rotary = normal(gen, (P, N, n, H + 2 * Hk, D), BF), verify.Rotary(D)
    at, start = torch.zeros((P, N, n), dtype=torch.int32, device="cuda"), ints([[0] * N] * P)

    def call():
        turned = verify.rotate(qkv[..., :H + Hk, :], at, rotary)
        q = c.write_rotated(0, qkv[..., :H, :], qkv[..., H:H + Hk, :], qkv[..., H + Hk:, :], rotary, at, start)
        return (turned, q, *c.read(0, n, start))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = call()
    torch.cuda.current_stream().wait_stream(side)
    assert all(map(torch.equal, there, call()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(4):
        qkv.copy_(normal(gen, qkv.shape, BF))
        at.copy_(torch.randint(0, 9999, at.shape, generator=gen, device="cuda", dtype=torch.int32))
        start += i
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert torch.equal(got[1], got[0][..., :H, :])
        assert all(map(torch.equal, got, call()))


def test_arguments_that_are_refused(gen):
    x, at, rotary = normal(gen, (6, 4, 64), BF), torch.zeros(6, dtype=torch.int32, device="cuda"), verify.Rotary(64)
    assert verify.rotate(x[:0], at[:0], rotary).shape == (0, 4, 64)
    wants = lambda t: t.clone().requires_grad_()
    for call, error in [
        (lambda: verify.rotate(x.float(), at, rotary), TypeError), (lambda: verify.rotate(x, at.long(), rotary), TypeError),
        (lambda: verify.rotate(x, at[:5], rotary), ValueError), (lambda: verify.rotate(x, at.cpu(), rotary), TypeError),
        (lambda: verify.rotate(x.cpu(), at, rotary), TypeError), (lambda: verify.rotate(x[..., :32], at, rotary), binding.CsdError),
        (lambda: verify.rotate(x[..., ::2], at, verify.Rotary(32)), TypeError), (lambda: verify.rotate(x[:, 0], at, rotary), TypeError),
        (lambda: verify.rotate(x, at, rotary, out=x[:, :3]), ValueError), (lambda: verify.rotate(x, at, rotary, out=x.flip(0)[:, :2]), ValueError),
        (lambda: verify.rotate(x[:5], at[:5], rotary, out=x[1:]), ValueError), (lambda: verify.rotate(wants(x), at, rotary), TypeError),
        (lambda: verify.rotate(x, at, rotary, out=wants(x)), TypeError), (lambda: verify.rotate(x[..., 1:57], at, verify.Rotary(16)), ValueError),
        (lambda: verify.rotate(x, at, verify.Rotary(64, device="cpu")), TypeError),
    ]:
        with pytest.raises(error):
            call()
    c = verify.PathCache(2, 3, 0, 8, 4, 2, 64, 4)
    q, k, at = normal(gen, (2, 3, 4, 4, 64), BF), normal(gen, (2, 3, 4, 2, 64), BF), torch.zeros((2, 3, 4), dtype=torch.int32, device="cuda")
    for call, error in [
        (lambda: c.write_rotated(0, q, k, k[:, :, :2], rotary, at), ValueError), (lambda: c.write_rotated(0, q[:, :, :2], k, k, rotary, at), ValueError),
        (lambda: c.write_rotated(0, q, k, k, rotary, at[:1]), ValueError), (lambda: c.write_rotated(0, q, k, k, rotary, at.long()), TypeError),
        (lambda: c.write_rotated(1, q, k, k, rotary, at), binding.CsdError), (lambda: c.write_rotated(0, q, k, k, verify.Rotary(128), at), binding.CsdError),
        (lambda: c.write_rotated(0, q.half(), k, k, rotary, at), TypeError), (lambda: c.write_rotated(0, q, wants(k), k, rotary, at), TypeError),
        (lambda: c.write_rotated(0, q, k, k, rotary, at, ints([1])), ValueError),
        (lambda: c.write_rotated(0, q, k, k, verify.Rotary(64, device="cpu"), at), TypeError),
    ]:
        with pytest.raises(error):
            call()


def test_results_at_one_place_are_refused(gen):
    x, at, rotary = normal(gen, (6, 4, 64), BF), torch.zeros(6, dtype=torch.int32, device="cuda"), verify.Rotary(64)
    same_for_all = x[:1].expand(6, 4, 64)
    assert same(verify.rotate(same_for_all, at, rotary), same_for_all)                                  # read from one place
    for out in (same_for_all, x[:, :1].expand(6, 4, 64), torch.empty(10000, dtype=BF, device="cuda").as_strided((6, 4, 64), (128, 64, 1))):
        with pytest.raises(binding.CsdError):
            verify.rotate(same_for_all if out is same_for_all else x[:, :1].expand(6, 4, 64) if out.stride(1) == 0 else x, at, rotary, out=out)
    heads_first = torch.zeros((4, 6, 64), dtype=BF, device="cuda").transpose(0, 1)
    assert same(verify.rotate(x, at, rotary, out=heads_first).contiguous(), x)

"""Attention in half precision where the weights of what a row's result is made of are small beside that of a token without
values: half has no numbers below 2^-24, and the weights' sum, which is in 32 bits, has them all."""
import pytest
import torch

from paper_2503_05330_amd import verify
from test_verify import F16, ROUND, gen, held, ints, normal, plain_attend  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu


def check(gen, fp8, size, gap, T, U, at, n=2, H=4, spread=0.3, one=False):
    """Values of one sign and about `size`; the keys of token `at` (of the prompt, then the path) raise its score by `gap` for
    all rows, its values are zero (`one`: but the first, and the others' are between 1 and 1.25 times `size`)."""
    P, N, Hk, D = 1, 2, 2, 64
    c = verify.PathCache(P, N, T, U, H, Hk, D, n, dtype=F16, fp8=fp8)
    c._buf.fill_(255)
    prompt = [normal(gen, (P, T, Hk, D), F16) for _ in range(2)]
    path = [normal(gen, (P, N, U, Hk, D), F16) for _ in range(2)]
    for k, v in (prompt, path):
        k *= spread
        k[..., 0] = 0
        v.abs_()
        if one:
            v.clamp_(max=2).div_(8).add_(1)
        v *= size
    k, v = prompt if at < T else path
    x = at if at < T else at - T
    k[..., x, :, :], v[..., x, :, :] = 0, 0
    k[..., x, :, 0] = gap                                # times 8, over sqrt(64)
    if one:
        v[..., x, :, 0] = size
    q = normal(gen, (P, N, n, H, D), F16)
    q[..., 0] = 8
    if T:
        c.write_prompt(0, *prompt)
    c.write(0, *path)
    lse = torch.empty((P, N, n, H), device="cuda")
    got = c.attend(0, q, ints([T]), ints([[U, U - 1]]), None, None, None, lse).double().cpu()
    prompt, path = [tuple(held(x, fp8) for x in pair) for pair in (prompt, path)]
    want, want_lse, sizes = plain_attend(q.cpu(), prompt, path, [T], [[U, U - 1]], [[n] * N] * P, D ** -0.5)
    tokens = T + U
    length = max(x[0].norm(dim=-1).max().item() for x in (prompt, path) if x[0].numel())
    score = D ** -0.5 * q.double().norm(dim=-1).max().item() * length
    loose = 2 * ((D + 4) * 2.0 ** -24 * score + (tokens + 8) * 2.0 ** -24)
    high = max(x[1].max().item() for x in (prompt, path) if x[1].numel())
    # a weight (8 bits: weight times scale) is rounded to 11 bits, or, where it is a subnormal number of half, to 2^-25 beside a
    # largest one of 2^7 at least (8 bits: of a token whose codes go beyond 224); the result to 11 bits or 2^-25
    error = ROUND[F16] * (want.abs() + sizes) + loose * sizes + 2 * tokens * 2.0 ** -32 * high + 2.0 ** -25
    over = ((got - want).abs() / error).max().item()
    assert over <= 1, over
    assert ((lse.double().cpu() - want_lse).abs() <= loose + 2.0 ** -22 * (1 + want_lse.abs())).all()


@pytest.mark.parametrize("size,gap,T,U", [(0.02, 7, 900, 124), (0.02, 8, 3000, 1096), (1e-4, 4, 700, 300), (1e-5, 0, 200, 60)])
@pytest.mark.parametrize("of_path", [False, True])
def test_a_token_without_values_in_an_8_bit_cache(gen, size, gap, T, U, of_path):
    check(gen, True, size, gap, T, U, T + 11 if of_path else 5)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,U,at,n,H", [(40, 30, 3, 2, 4), (40, 30, 60, 2, 4), (300, 100, 130, 17, 8), (0, 64, 40, 2, 8)])
def test_weights_below_the_range_of_half(gen, fp8, T, U, at, n, H):
    """All weights but one are 2^-26 of that one."""
    check(gen, fp8, 1000.0, 18, T, U, at, n, H, spread=0.1, one=True)


@pytest.mark.parametrize("value", [63456.0, 63488.0, 65504.0, -65504.0, float("inf")])
def test_the_largest_numbers_of_half_in_an_8_bit_cache(gen, value):
    """63488 and more are held as 65536, an infinity as 448 times the scale of 256: attention works with what is held, reading
    back rounds it to half."""
    c = verify.PathCache(1, 1, 0, 4, 2, 1, 64, 1, dtype=F16, fp8=True)
    k, v = torch.zeros((1, 1, 4, 1, 64), dtype=F16, device="cuda"), torch.zeros((1, 1, 4, 1, 64), dtype=F16, device="cuda")
    v[0, 0, 1, 0, :2] = torch.tensor([value, 60000.0])
    c.write(0, k, v)
    stands_for = held(v, True)
    assert stands_for[0, 0, 1, 0, 0].abs() == {63456.0: 61440, float("inf"): 448 * 256}.get(value, 65536)
    assert torch.equal(c.read(0, 4)[1].cpu(), stands_for.to(F16))
    out = c.attend(0, normal(gen, (1, 1, 1, 2, 64), F16), None, ints([[4]])).double().cpu()
    want = stands_for[0, 0].sum(0) / 4                   # four equal weights
    assert ((out[0, 0, 0] - want).abs() <= ROUND[F16] * want.abs()).all()

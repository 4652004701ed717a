"""Tokens and heads at any distance: what rotates and writes gives the bits that it gives for contiguous copies."""
import pytest
import torch

from paper_2503_05330_amd import verify
from test_verify import BF, F16, gen, ints, normal, same  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu


def spread(x, more, between):
    """x [.., heads, D] with `between` more elements from a head to the next and `more` from a token to the next, NaN there and nothing behind the last value."""
    lead, H, D = x.shape[:-2], x.shape[-2], x.shape[-1]
    head, token = D + between, (H - 1) * (D + between) + D + more
    strides = [token]
    for n in reversed(lead[1:]):
        strides.insert(0, strides[0] * n)
    flat = torch.full((lead.numel() * token - more,), torch.nan, dtype=x.dtype, device=x.device)
    return flat.as_strided(x.shape, (*strides, head, 1)).copy_(x)


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D,dim,interleaved", [(64, 64, True), (96, 48, False), (128, 128, False), (256, 256, True)])
@pytest.mark.parametrize("more,between", [(8, 0), (0, 8), (24, 40)])
def test_tokens_at_any_distance(gen, more, between, D, dim, interleaved, fp8, dtype):
    P, N, n, H, Hk, cap = 2, 3, 5, 6, 3, 20
    rotary, offsets = verify.Rotary(dim, interleaved=interleaved), ints([0, 13, 30])
    q, k, v = normal(gen, (P, N, n, H, D), dtype), normal(gen, (P, N, n, Hk, D), dtype), normal(gen, (P, N, n, Hk, D), dtype)
    at = torch.randint(0, 5000, (P, N, n), generator=gen, device="cuda", dtype=torch.int32)
    apart = [spread(x, more, between) for x in (q, k, v)]
    packed = normal(gen, (30, 2, Hk, D), dtype)
    got = []
    for x, y, z, a, b in ((q, k, v, packed[:, 0].contiguous(), packed[:, 1].contiguous()), (*apart, *(spread(packed[:, i], more, between) for i in range(2)))):
        c = verify.PathCache(P, N, cap, cap, H, Hk, D, n, dtype=dtype, fp8=fp8)
        turned = c.write_rotated(0, x, y, z, rotary, at, ints([[3, 0, 7]] * P))
        c.write_packed(0, a, b, offsets)
        to = spread(torch.zeros_like(q), more, between)
        verify.rotate(x, at, rotary, out=to)
        got.append((turned, verify.rotate(x, at, rotary), verify.rotate(y, at, rotary), to.contiguous(), *c.read(0, n, ints([[3, 0, 7]] * P)),
                    *c.read_prompt(0, cap, None, ints([13, 17]))))
    for a, b in zip(*got):
        assert a.isfinite().all() and same(a, b)

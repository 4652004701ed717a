"""A cache of another device than the current one: the launches are the current device's, which may not reach its memory."""
import pytest
import torch

from paper_2503_05330_amd import verify
from test_verify import BF, gen, ints, normal, same  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu


class Elsewhere:
    """What a buffer of another device says of itself."""
    is_cuda = True

    def __init__(self, device):
        self.get_device = lambda: device


def test_writes_to_a_cache_of_another_device_are_refused(gen):
    P, N, n, H, Hk, D = 1, 2, 3, 4, 2, 64
    c, rotary = verify.PathCache(P, N, 8, 8, H, Hk, D, n), verify.Rotary(D)
    q, k, at = normal(gen, (P, N, n, H, D), BF), normal(gen, (P, N, n, Hk, D), BF), torch.zeros((P, N, n), dtype=torch.int32, device="cuda")
    packed, offsets, zero = normal(gen, (5, Hk, D), BF), ints([0, 5]), torch.zeros((P, N, 8, Hk, D), dtype=BF, device="cuda")
    c.write(0, zero, zero)
    c.write_prompt(0, zero[:, 0], zero[:, 0])
    buf, place = c._buf, c._place
    assert place == buf.get_device() == torch.cuda.current_device()
    c._buf, c._place = Elsewhere(place + 1), place + 1
    for call in (lambda: c.write_rotated(0, q, k, k, rotary, at), lambda: c.write_packed(0, packed, packed, offsets)):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert not c.read(0, 8)[0].any() and not c.read_prompt(0, 8)[0].any()
    c._buf, c._place = buf, place
    assert same(c.write_rotated(0, q, k, k, rotary, at), q)
    c.write_packed(0, packed, packed, offsets)
    assert same(c.read(0, n)[1], k) and same(c.read_prompt(0, 5)[0][0], packed)

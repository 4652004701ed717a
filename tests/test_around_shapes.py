"""Tensors of other shapes than the operators around the cache take: with numbers enough, they were read as if they were of the right one."""
import pytest
import torch

from paper_2503_05330_amd import verify
from test_around_calls import Declines
from test_verify import BF, F32, gen, ints, normal, same  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "python"])
def way(request, monkeypatch):
    """Both ways that a call is marshalled."""
    verify.load()
    if request.param == "python":
        monkeypatch.setattr(verify, "_native", Declines())


def test_positions_of_another_shape_are_refused(gen, way):
    P, N, n, H, Hk, D = 2, 3, 4, 4, 2, 64
    c, rotary = verify.PathCache(P, N, 0, 16, H, Hk, D, 8), verify.Rotary(D)
    q, k, v = normal(gen, (P, N, n, H, D), BF), normal(gen, (P, N, n, Hk, D), BF), normal(gen, (P, N, n, Hk, D), BF)
    zero = torch.zeros((P, N, 16, Hk, D), dtype=BF, device="cuda")
    c.write(0, zero, zero)
    at = torch.arange(P * N * 8, dtype=torch.int32, device="cuda")
    for wrong in (at.view(P, N, 8), at.view(N, P, 8), at[:24].view(N, P, n), at[:24].view(P, n, N), at[:24], at[:24].view(P * N, n), at[:24].view(1, P, N, n)):
        with pytest.raises(ValueError):
            c.write_rotated(0, q, k, v, rotary, wrong)
    assert not c.read(0, 16)[0].any()                        # nothing was enqueued
    right = at.view(P, N, 8)[..., :n].contiguous()
    assert same(c.write_rotated(0, q, k, v, rotary, right), verify.rotate(q, right, rotary))


def test_penalties_of_another_shape_are_refused(gen, way):
    P, N, n, V = 4, 2, 3, 100
    logits, tokens, length = normal(gen, (P, N, n, V), F32), torch.zeros((P, N, 5), dtype=torch.int32, device="cuda"), ints([[5] * N] * P)
    penalties = torch.tensor([[1.5, 0.5, 0.25]] * P, device="cuda")
    for wrong in (penalties.T.contiguous(), penalties.flatten(), penalties.repeat(1, 2), penalties.repeat(2, 1), penalties[None], penalties[:, :2].contiguous()):
        with pytest.raises(ValueError):
            verify.adjust(logits, tokens, length, penalties=wrong)
    got = verify.adjust(logits, tokens, length, penalties=penalties)
    assert torch.equal(got[..., 1:], logits[..., 1:]) and not torch.equal(got, logits)


def test_results_of_attention_of_another_shape_are_refused(gen):
    T, H, Hk, D = 10, 4, 2, 64
    q, k, v, offsets = normal(gen, (T, H, D), BF), normal(gen, (T, Hk, D), BF), normal(gen, (T, Hk, D), BF), ints([0, 3, 10])
    out, lse = torch.zeros((T + 1, H, D), dtype=BF, device="cuda"), torch.zeros((T + 1, H), device="cuda")
    for wrong in (out, out[:T].view(H, T, D), out[:T].view(T, H * D), out[:T].flatten()):
        with pytest.raises(ValueError):
            verify.prompt_attend(q, k, v, offsets, out=wrong)
    for wrong in (lse, lse[:T].view(H, T), lse[:T].flatten(), lse[None, :T]):
        with pytest.raises(ValueError):
            verify.prompt_attend(q, k, v, offsets, lse=wrong)
    assert not out.any() and not lse.any()
    assert verify.prompt_attend(q, k, v, offsets, out=out[:T], lse=lse[:T]).data_ptr() == out.data_ptr()
    assert same(out[:T], verify.prompt_attend(q, k, v, offsets)) and lse[:T].any(0).all()


def test_offsets_of_another_number_of_prompts_are_refused(gen):
    P, T, Hk, D = 2, 10, 2, 64
    c, k = verify.PathCache(P, 1, 16, 1, Hk, Hk, D, 1), normal(gen, (T, Hk, D), BF)
    zero = torch.zeros((P, 16, Hk, D), dtype=BF, device="cuda")
    c.write_prompt(0, zero, zero)
    for wrong in (ints([0, 4, 7, 10]), ints([0, 10]), ints([[0, 4, 10]]), ints([0, 4, 10, 10])):       # (a third prompt would be lost)
        with pytest.raises(ValueError):
            c.write_packed(0, k, k, wrong)
    assert not c.read_prompt(0, 16)[0].any()
    c.write_packed(0, k, k, ints([0, 4, 10]))
    got = c.read_prompt(0, 16)[0]
    assert same(got[0, :4], k[:4]) and same(got[1, :6], k[4:]) and not got[0, 4:].any() and not got[1, 6:].any()

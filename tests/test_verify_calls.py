"""Calls of the verifying pass's operators: what they are given, what they refuse, what they say of a launch."""
import pytest
import torch

from paper_2503_05330_amd import verify
from test_verify import BF, gen, ints, normal  # noqa: F401 (gen: a fixture)


@pytest.mark.gpu
def test_tensors_that_want_gradients_are_refused(gen):
    c = verify.PathCache(2, 3, 16, 16, 8, 2, 64, 4)
    q, length = normal(gen, (2, 3, 4, 8, 64), BF), ints([[4] * 3] * 2)
    k, prompt = normal(gen, (2, 3, 4, 2, 64), BF), normal(gen, (2, 4, 2, 64), BF)
    logits, noise = normal(gen, (3, 100), BF), normal(gen, (3, 100), torch.float32)
    lse = torch.zeros((2, 3, 4, 8), device="cuda")
    wants = lambda t: t.clone().requires_grad_()
    calls = [lambda: c.write(0, wants(k), k), lambda: c.write(0, k, wants(k)), lambda: c.write_prompt(0, prompt, wants(prompt)),
             lambda: c.attend(0, wants(q), None, length), lambda: c.attend(0, wants(q) * 2, None, length),
             lambda: c.attend(0, q, None, length, out=wants(q)), lambda: c.attend(0, q, None, length, lse=wants(lse)),
             lambda: verify.targets(wants(logits)), lambda: verify.targets(logits, wants(noise))]
    for call in calls:
        with pytest.raises(TypeError, match="gradient"):
            call()
    c.write(0, k, k)
    c.write_prompt(0, prompt, prompt)
    with torch.no_grad():
        for call in calls:
            call()
    out = c.attend(0, wants(q).detach(), ints([4, 4]), length)
    with torch.inference_mode():
        assert torch.equal(c.attend(0, wants(q), ints([4, 4]), length), out)
    assert torch.equal(verify.targets(wants(logits).detach())[0], verify.targets(logits)[0])

"""The operators around the cache: calls marshalled in native code and in Python, and a run of all of them as a model makes it."""
import pytest
import torch

from paper_2503_05330_amd import verify
from test_verify import BF, F16, F32, gen, ints, normal, same  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu


class Declines:
    """Native code that serves no call."""

    def __getattr__(self, name):
        return lambda *args: None


@pytest.mark.parametrize("dtype", [BF, F16])
def test_calls_in_native_code_and_in_python_do_the_same(gen, monkeypatch, dtype):
    P, N, n, H, Hk, D, V = 2, 3, 4, 8, 2, 64, 5000
    verify.load()
    native = verify._native
    served = []

    class Counts:
        def __getattr__(self, name):
            def call(*args):
                got = getattr(native, name)(*args)
                served.append((name, got is not None))
                return got
            return call
    cache = verify.PathCache(P, N, 40, 40, H, Hk, D, n, dtype=dtype)
    qkv, rotary = normal(gen, (P, N, n, H + 2 * Hk, D), dtype), verify.Rotary(D)
    q, k, v = qkv[..., :H, :], qkv[..., H:H + Hk, :], qkv[..., H + Hk:, :]
    at = torch.randint(0, 99, (P, N, n), generator=gen, device="cuda", dtype=torch.int32)
    start, counts = ints([[3, 0, 30]] * P), ints([[4, 0, 2]] * P)
    packed = normal(gen, (70, H + 2 * Hk, D), dtype)
    offsets = ints([0, 40, 70])
    logits = normal(gen, (P, N, n, V), dtype)
    said, prompt = torch.randint(0, V, (P, N, 30), generator=gen, device="cuda", dtype=torch.int32), torch.randint(0, V, (P, 9), generator=gen, device="cuda", dtype=torch.int32)
    length, penalties = ints([[30, 4, 9]] * P), torch.tensor([[1.5, 0.25, 0.5]] * P, device="cuda")
    bias, mask = normal(gen, (V,), F32), torch.randint(-1 << 31, 1 << 31, (P, N, n, 157), generator=gen, device="cuda", dtype=torch.int64).int()

    def calls():
        yield verify.rotate(qkv[..., :H + Hk, :], at, rotary)
        yield verify.rotate(packed, at.flatten().repeat(3)[:70], verify.Rotary(32, interleaved=True, amplitude=1.5))
        yield cache.write_rotated(0, q, k, v, rotary, at, start, counts)
        yield cache.write_rotated(0, q, k, v, rotary, at)
        yield torch.cat(cache.read(0, 40))
        yield verify.prompt_attend(packed[:, :H], packed[:, H:H + Hk], packed[:, H + Hk:], offsets)
        yield verify.prompt_attend(packed[:, :H], packed[:, H:H + Hk], packed[:, H + Hk:], offsets, 0.5)
        yield verify.adjust(logits, said, length, counts, prompt, None, penalties, bias, mask)
        yield verify.adjust(logits, penalties=penalties, prompt=prompt, prompt_len=ints([9, 2]))
        mine = logits.clone()
        yield verify.adjust(mine, bias=bias, out=mine)
    zero = torch.zeros((P, N, 40, Hk, D), dtype=dtype, device="cuda")
    cache.write(0, zero, zero)
    monkeypatch.setattr(verify, "_native", Counts())
    here = list(calls())
    names = ("rotate", "cache_write_rotated", "prompt_attend", "adjust")
    assert all(done for _, done in served) and {name for name, _ in served} >= set(names)
    monkeypatch.setattr(verify, "_native", Declines())
    cache.write(0, zero, zero)
    there = list(calls())
    assert all(map(same, here, there))


def plain_pass(tokens, at, w, rotary, H, Hk, D):
    """One layer of attention of a sequence in 64 bits: q, k, v turned, keys and values, and the result."""
    qkv = (w["x"][tokens].double() @ w["qkv"].double()).unflatten(-1, (H + 2 * Hk, D)).to(BF).double()
    angle = at.double()[:, None] * (rotary.turns * 6.283185307179586)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    z = torch.complex(qkv[:, :H + Hk, :D // 2], qkv[:, :H + Hk, D // 2:]) * turn
    qk = torch.cat([z.real, z.imag], -1).to(BF).double()
    q, k, v = qk[:, :H], qk[:, H:], qkv[:, H + Hk:]
    s = torch.einsum("thd,xhd->htx", q, k.repeat_interleave(H // Hk, 1)) * D ** -0.5
    s = s.masked_fill(torch.ones(s.shape[1:], dtype=torch.bool, device=s.device).triu(1), -torch.inf)
    return k, v, torch.einsum("htx,xhd->thd", torch.softmax(s, -1), v.repeat_interleave(H // Hk, 1))


def test_prompts_paths_and_logits_one_after_the_other(gen):
    """Packed prompts through rotate, prompt_attend and write_packed; paths through write_rotated and attend; adjust and targets on what
    comes out: as one sequence each in 64 bits."""
    P, N, n, H, Hk, D, V, E = 3, 2, 4, 8, 2, 64, 300, 32
    lengths = [33, 1, 70]
    w = dict(x=normal(gen, (V, E), BF), qkv=normal(gen, (E, (H + 2 * Hk) * D), BF) * E ** -0.5, out=normal(gen, (H * D, V), BF) * (H * D) ** -0.5)
    rotary = verify.Rotary(D, base=500.0)
    prompts = [torch.randint(0, V, (x,), generator=gen, device="cuda") for x in lengths]
    new = torch.randint(0, V, (P, N, n), generator=gen, device="cuda")
    project = lambda tokens: (w["x"][tokens].double() @ w["qkv"].double()).to(BF).unflatten(-1, (H + 2 * Hk, D))
    cache = verify.PathCache(P, N, 80, n, H, Hk, D, n)
    offsets = ints([0, 33, 34, 104])
    at = torch.cat([torch.arange(x) for x in lengths]).int().cuda()
    qkv = project(torch.cat(prompts))
    verify.rotate(qkv[:, :H + Hk], at, rotary, out=qkv[:, :H + Hk])
    of_prompts = verify.prompt_attend(qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], offsets)
    cache.write_packed(0, qkv[:, H:H + Hk], qkv[:, H + Hk:], offsets)
    qkv = project(new)
    prompt_len = ints(lengths)
    positions = (prompt_len[:, None, None] + torch.arange(n, device="cuda", dtype=torch.int32)).expand(P, N, n).contiguous()
    q = cache.write_rotated(0, qkv[..., :H, :], qkv[..., H:H + Hk, :], qkv[..., H + Hk:, :], rotary, positions)
    of_paths = cache.attend(0, q, prompt_len, ints([[n] * N] * P))
    logits = (of_paths.flatten(-2).double() @ w["out"].double()).float() * 10
    penalties = torch.tensor([[1.5, 0.5, 0.25]] * P, device="cuda")
    asked = torch.nn.utils.rnn.pad_sequence(prompts, batch_first=True).int()
    adjusted = verify.adjust(logits, new.int(), ints([[n] * N] * P), None, asked, prompt_len, penalties)
    picked, probs = verify.targets(adjusted)
    keys = cache.read_prompt(0, 80)
    for p in range(P):
        for i in range(N):
            tokens = torch.cat([prompts[p], new[p, i]])
            k, v, out = plain_pass(tokens, torch.arange(len(tokens), device="cuda"), w, rotary, H, Hk, D)
            T = lengths[p]
            for got, want in zip(keys, (k, v)):
                # (a rounding of the turned value that 32 bits put on the other side)
                assert ((got[p, :T].double() - want[:T]).abs() <= 2.0 ** -7 * want[:T].abs() + 2.0 ** -18).all()
            a, b = (of_prompts[int(offsets[p]):int(offsets[p + 1])].double() - out[:T]).abs(), (of_paths[p, i].double() - out[T:]).abs()
            # weights and results are rounded to 8 bits, and a few keys and queries to the other side: 2^-8 of a score of up to 4 or so
            high = v.abs().max()
            assert a.max() <= 2.0 ** -8 * 4 * high and b.max() <= 2.0 ** -8 * 4 * high
            for t in range(n):
                x = logits[p, i, t].double()
                said = torch.bincount(new[p, i, :t + 1], minlength=V)
                seen = (torch.bincount(prompts[p], minlength=V) > 0) | (said > 0)
                x = torch.where(seen, torch.where(x > 0, x / 1.5, x * 1.5), x) - 0.25 * said - 0.5 * (said > 0)
                assert ((adjusted[p, i, t].double() - x).abs() <= 2.0 ** -21 * (x.abs() + 4)).all()
                best = int(picked[p, i, t])
                assert x[best] >= x.max() - 2.0 ** -20 * (x.abs().max() + 4)
                assert abs(probs[p, i, t].item() - torch.softmax(x, -1)[best].item()) <= 1e-5

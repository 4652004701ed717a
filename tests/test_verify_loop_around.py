"""The decode loop with packed prompts of different lengths, rotary positions and penalties: its logits, caches and tokens against the
model in 64 bits without drafts."""
import pytest
import torch

from paper_2503_05330_amd import verify, verify_loop
from test_verify import held
from test_verify_loop_tokens import rms

pytestmark = pytest.mark.gpu


def plain(model, sequence, cache, rounded, before, fp8):
    """Logits of a sequence [T], all attention at once over the keys and values that `cache` holds for it, and each layer's keys
    and values, in 64 bits; rounded: with every result rounded as the model's type does.  The first `before` tokens, the packed prompt, attend to
    each other in the model's type, before their keys and values become 8 bits."""
    kept = (lambda t: t.to(model.dtype).double()) if rounded else (lambda t: t)
    norm = lambda t: kept(t * kept(torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)))
    H, Hk, D = model.heads, model.kv_heads, model.head_dim
    x = model.tokens[sequence].double()
    at = torch.arange(len(sequence), device=x.device)
    if model.rotary is None:
        x = kept(x + model.positions[at].double())
    else:
        angle = at.double()[:, None] * model.rotary.turns * 6.283185307179586
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    hidden = torch.ones((len(sequence), len(sequence)), dtype=torch.bool, device=x.device).triu(1)
    made = []
    for w, (k, v) in zip(model.layers, cache):
        qkv = kept(norm(x) @ w["qkv"].double()).unflatten(-1, (H + 2 * Hk, D))
        if model.rotary is not None:
            z = torch.complex(qkv[:, :H + Hk, :D // 2], qkv[:, :H + Hk, D // 2:]) * turn
            qkv = torch.cat([kept(torch.cat([z.real, z.imag], -1)), qkv[:, H + Hk:]], 1)
        made.append((qkv[:, H:H + Hk], qkv[:, H + Hk:]))
        own = [t.to(model.dtype).double() for t in made[-1]] if fp8 else (k, v)

        def attend(q, k, v, hidden):
            q, k, v = (t.transpose(0, 1) for t in (q, k.repeat_interleave(H // Hk, 1), v.repeat_interleave(H // Hk, 1)))
            s = (q @ k.transpose(1, 2)) * D ** -0.5
            return kept(torch.softmax(s.masked_fill(hidden, -torch.inf), -1) @ v)
        a = torch.cat([attend(qkv[:before, :H], own[0][:before], own[1][:before], hidden[:before, :before]),
                       attend(qkv[before:, :H], k, v, hidden[before:])], 1)
        x = kept(x + kept(a.transpose(0, 1).flatten(-2) @ w["o"].double()))
        gate, up = kept(norm(x) @ w["up"].double()).chunk(2, -1)
        x = kept(x + kept(kept(kept(torch.nn.functional.silu(gate)) * up) @ w["down"].double()))
    return kept(norm(x) @ model.out.double()), made


def adjusted(x, prompt, said, penalties, bias):
    """Logits x [T][V] behind a prompt, row t of which has said the first t + 1 tokens."""
    x = x.clone()
    for t in range(len(x)):
        if penalties is not None:
            rep, pres, freq = penalties
            times = torch.bincount(said[:t + 1], minlength=x.shape[1]).double()
            seen = (torch.bincount(prompt, minlength=x.shape[1]) > 0) | (times > 0)
            x[t] = torch.where(seen, torch.where(x[t] > 0, x[t] / rep, x[t] * rep), x[t]) - freq * times - pres * (times > 0)
        if bias is not None:
            x[t] += bias
    return x


@pytest.mark.parametrize("greedy,fp8,rotary,lengths,penalties,bias", [
    (True, False, True, (70, 1, 33), None, False), (True, False, False, (5, 66, 2), (1.2, 0.1, 0.05), False), (False, True, True, (33, 40, 65), (1.1, 0.0, 0.1), True),
    (False, False, True, (1, 1, 1), (0.9, 0.3, 0.0), False), (True, True, True, (64, 64, 64), None, True)])
def test_loop_around(monkeypatch, greedy, fp8, rotary, lengths, penalties, bias):
    torch.manual_seed(5)
    calls, real = [], verify.targets

    def targets(logits, noise=None, inv_temperature=1.0):
        calls.append((logits.clone(), None if noise is None else noise.clone()))
        return real(logits, noise, inv_temperature)
    monkeypatch.setattr(verify, "targets", targets)
    model = verify_loop.Model(vocab=300, dim=128, heads=4, kv_heads=2, head_dim=64, layers=2, max_position=1024,
                              rotary=verify.Rotary(64, base=1000.0) if rotary else None)
    P, N, steps, L, inv_temperature = 3, 4, 30, 4, 4.0
    prompts = [torch.randint(0, model.vocab, (x,), device="cuda") for x in lengths]
    given = None if penalties is None else torch.tensor([penalties] * P, device="cuda")
    biases = torch.randn(300, device="cuda") if bias else None
    loop = verify_loop.Loop(model, prompts, N, steps * (L + 1), query_len=2, draft_len=L, inv_temperature=inv_temperature, greedy=greedy, fp8=fp8,
                            penalties=given, bias=biases)
    tokens, logits = ([[[] for _ in range(N)] for _ in range(P)] for _ in range(2))
    for _ in range(steps):
        picked, taken = loop.step()
        said, noise = calls[-1]
        z = said.float() if noise is None else said.float() * inv_temperature + noise
        assert (noise is None) == greedy
        assert torch.equal(picked.long(), (z == z.amax(-1, keepdim=True)).int().argmax(-1))
        for p in range(P):
            for i in range(N):
                n = int(taken[p, i])
                tokens[p][i] += picked[p, i, :n].tolist()
                logits[p][i].append(said[p, i, :n].double())
    assert len(calls) == steps and loop.cache.status() == 0 and loop.index.status() == 0
    most, longest = int(loop.length.max()), max(lengths) - 1
    layers = range(len(model.layers))
    of_prompts = [loop.cache.read_prompt(x, longest) if longest else None for x in layers]
    of_paths = [loop.cache.read(x, most) for x in layers]
    for p in range(P):
        before = lengths[p] - 1
        for i in range(N):
            path = torch.tensor([int(prompts[p][-1])] + tokens[p][i][:-1], device="cuda", dtype=torch.long)
            sequence = torch.cat([prompts[p][:-1], path])
            n = int(loop.length[p, i])
            cache = [[torch.cat(([of_prompts[x][y][p, :before]] if longest else []) + [of_paths[x][y][p, i, :n]]).double() for y in range(2)] for x in layers]
            assert len(sequence) == len(cache[0][0])
            want, want_kv = plain(model, sequence, cache, False, before, fp8)
            near, near_kv = plain(model, sequence, cache, True, before, fp8)
            want, near = (adjusted(x[before:], prompts[p], path, penalties, None if biases is None else biases.double()) for x in (want, near))
            if penalties is not None or bias:             # the adjusted ones are rounded again
                near = near.to(model.dtype).double()
            got = torch.cat(logits[p][i])
            # The loop rounds where the rounded form does, sums in another order: both are as far from the exact values, thousands of
            # them, in the mean; 4 times leaves room for what the rounding of a few early values does to all.
            assert rms(got - want) <= 4 * rms(near - want), (p, i)
            for layer in layers:
                for x in range(2):
                    exact, held_now = want_kv[layer][x], cache[layer][x]
                    # of 10^5 values none is off by more than 8 times the mean, and 8 bits round to 4, or to 2^-10 of a scale that is
                    # less than 2 / 448 of the largest
                    off = 8 * rms(near_kv[layer][x] - exact) + 2.0 ** -8 * exact.abs()
                    if fp8:
                        off = off + 2.0 ** -4 * (exact.abs() + off) + 2.0 ** -10 * 2 / 448 * (exact.abs() + off).amax(-1, keepdim=True)
                    assert ((held_now - exact).abs() <= off).all(), (p, i, layer, x)
                    if fp8:
                        assert torch.equal(held(held_now, True), held_now.cpu())


def test_packed_prompts_of_one_length_are_as_those_taken_in_steps():
    """The caches of both ways are as far from each other as roundings are."""
    torch.manual_seed(2)
    model = verify_loop.Model(vocab=300, dim=128, heads=4, kv_heads=2, head_dim=64, layers=2, max_position=1024)
    prompts = torch.randint(0, 300, (2, 77), device="cuda")
    loops = [verify_loop.Loop(model, x, 2, 20, query_len=2, draft_len=4, greedy=True) for x in (prompts, list(prompts))]
    for layer in range(2):
        for a, b in zip(*(loop.cache.read_prompt(layer, 76) for loop in loops)):
            # The first layer's are the same product, whose sums may be taken in another order: a rounding to the other side.  The second's have 8 roundings
            # to 8 bits before them, which add up by squares; none is off by more than 24 times the mean.
            a, b = a.double(), b.double()
            assert ((a - b).abs() <= 2.0 ** -7 * a.abs() + (2.0 ** -14 if layer == 0 else 24 * 8 ** 0.5 * 2.0 ** -8) * rms(a)).all()


@pytest.mark.parametrize("argv", [["--rotary", "--shortest", "20", "--repetition", "1.1", "--frequency", "0.1"], ["--shortest", "1", "--fp8", "--greedy"]])
def test_command(argv, capsys):
    verify_loop.main(["--problems", "2", "--paths", "3", "--prompt", "50", "--tokens", "8", "--draft", "4", *argv])
    assert "status 0 0" in capsys.readouterr().out

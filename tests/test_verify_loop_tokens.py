"""The decode loop, greedy and sampled, with caches of 16 and of 8 bits: its logits and what its cache holds are the model's, its
tokens those that the logits and the noise pick."""
import pytest
import torch

from paper_2503_05330_amd import verify, verify_loop
from test_verify import held

pytestmark = pytest.mark.gpu


def plain(model, sequence, cache, rounded):
    """Logits of a sequence [T], all attention at once over the keys and values that `cache` holds for it, and each layer's keys
    and values of its tokens [T][Hk][D], in 64 bits; rounded: with every result rounded as the model's type does."""
    kept = (lambda t: t.to(model.dtype).double()) if rounded else (lambda t: t)
    norm = lambda t: kept(t * kept(torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)))
    H, Hk, D = model.heads, model.kv_heads, model.head_dim
    x = kept(model.tokens[sequence].double() + model.positions[:len(sequence)].double())
    hidden = torch.ones((len(sequence), len(sequence)), dtype=torch.bool, device=x.device).triu(1)
    made = []
    for w, (k, v) in zip(model.layers, cache):
        qkv = kept(norm(x) @ w["qkv"].double()).unflatten(-1, (H + 2 * Hk, D))
        made.append((qkv[:, H:H + Hk], qkv[:, H + Hk:]))
        q, k, v = (t.transpose(0, 1) for t in (qkv[:, :H], k.repeat_interleave(H // Hk, 1), v.repeat_interleave(H // Hk, 1)))
        s = (q @ k.transpose(1, 2)) * D ** -0.5
        a = kept(torch.softmax(s.masked_fill(hidden, -torch.inf), -1) @ v)
        x = kept(x + kept(a.transpose(0, 1).flatten(-2) @ w["o"].double()))
        gate, up = kept(norm(x) @ w["up"].double()).chunk(2, -1)
        x = kept(x + kept(kept(kept(torch.nn.functional.silu(gate)) * up) @ w["down"].double()))
    return kept(norm(x) @ model.out.double()), made


def rms(t):
    return t.square().mean().sqrt().item()


@pytest.mark.parametrize("greedy,fp8,prompt", [(True, False, 70), (True, True, 40), (True, True, 1), (False, False, 33), (False, True, 65)])
def test_logits_cache_and_tokens(monkeypatch, greedy, fp8, prompt):
    torch.manual_seed(3)
    calls, real = [], verify.targets

    def targets(logits, noise=None, inv_temperature=1.0):
        calls.append((logits.clone(), None if noise is None else noise.clone()))
        return real(logits, noise, inv_temperature)
    monkeypatch.setattr(verify, "targets", targets)
    model = verify_loop.Model(vocab=300, dim=128, heads=4, kv_heads=2, head_dim=64, layers=2, max_position=1024)
    P, N, steps, L, inv_temperature = 2, 5, 40, 4, 4.0
    prompts = torch.randint(0, model.vocab, (P, prompt), device="cuda")
    loop = verify_loop.Loop(model, prompts, N, steps * (L + 1), query_len=2, draft_len=L, inv_temperature=inv_temperature, greedy=greedy, fp8=fp8)
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
    assert len(calls) == steps and loop.cache.status() == 0 and int(loop.accepted) > 0
    most = int(loop.length.max())
    layers = range(len(model.layers))
    of_prompts = [loop.cache.read_prompt(x, prompt - 1) if prompt > 1 else None for x in layers]
    of_paths = [loop.cache.read(x, most) for x in layers]
    for p in range(P):
        for i in range(N):
            sequence = torch.cat([prompts[p], torch.tensor(tokens[p][i][:-1], device="cuda", dtype=torch.long)])
            n = int(loop.length[p, i])
            cache = [[torch.cat(([before[x][p]] if before else []) + [path[x][p, i, :n]]).double() for x in range(2)]
                     for before, path in zip(of_prompts, of_paths)]
            assert len(sequence) == len(cache[0][0])
            want, want_kv = plain(model, sequence, cache, False)
            near, near_kv = plain(model, sequence, cache, True)
            want, near, got = want[prompt - 1:], near[prompt - 1:], torch.cat(logits[p][i])
            # The loop rounds where the rounded form does, sums in another order: both are as far from the exact values, thousands
            # of them, in the mean; 4 times leaves room for what the rounding of a few early values does to all.
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
                    if fp8:                              # and it is numbers of 8 bits that are held
                        assert torch.equal(held(held_now, True), held_now.cpu())

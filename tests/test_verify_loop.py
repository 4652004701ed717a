"""The decode loop with a target model: its tokens are what the model, computed without cache and drafts, picks."""
import pytest
import torch

from paper_2503_05330_amd import verify_loop

pytestmark = pytest.mark.gpu


def plain_logits(model, sequence):
    """Logits of a sequence [T] in 64 bits, all attention at once."""
    double = lambda t: t.double()
    x = double(model.tokens[sequence]) + double(model.positions[:len(sequence)])
    H, Hk, D = model.heads, model.kv_heads, model.head_dim
    norm = lambda t: t * torch.rsqrt(t.square().mean(-1, keepdim=True) + 1e-6)
    hidden = torch.ones((len(sequence), len(sequence)), dtype=torch.bool, device=x.device).triu(1)
    for w in model.layers:
        qkv = (norm(x) @ double(w["qkv"])).unflatten(-1, (H + 2 * Hk, D))
        q, k, v = (t.transpose(0, 1) for t in (qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]))
        k, v = k.repeat_interleave(H // Hk, 0), v.repeat_interleave(H // Hk, 0)
        s = (q @ k.transpose(1, 2)) * D ** -0.5
        a = torch.softmax(s.masked_fill(hidden, -torch.inf), -1) @ v
        x = x + a.transpose(0, 1).flatten(-2) @ double(w["o"])
        gate, up = (norm(x) @ double(w["up"])).chunk(2, -1)
        x = x + (torch.nn.functional.silu(gate) * up) @ double(w["down"])
    return norm(x) @ double(model.out)


@pytest.mark.parametrize("greedy,fp8,prompt", [(True, False, 70), (True, False, 1), (False, False, 33), (True, True, 40), (False, True, 65)])
def test_loop(greedy, fp8, prompt):
    torch.manual_seed(3)
    model = verify_loop.Model(vocab=300, dim=128, heads=4, kv_heads=2, head_dim=64, layers=2, max_position=1024)
    P, N, steps, L = 2, 5, 40, 4
    prompts = torch.randint(0, model.vocab, (P, prompt), device="cuda")
    loop = verify_loop.Loop(model, prompts, N, steps * (L + 1), query_len=2, draft_len=L, inv_temperature=4.0, greedy=greedy, fp8=fp8)
    paths = [[[] for _ in range(N)] for _ in range(P)]
    for _ in range(steps):
        picked, taken = (t.tolist() for t in loop.step())
        for p in range(P):
            for i in range(N):
                assert 1 <= taken[p][i] <= len(picked[p][i])
                paths[p][i] += picked[p][i][:taken[p][i]]
    length = loop.length.tolist()
    assert loop.cache.status() == 0 and loop.index.status() == 0
    assert [[len(x) for x in row] for row in paths] == length and all(steps <= x for row in length for x in row)
    assert int(loop.accepted) == sum(x - steps for row in length for x in row)
    if greedy:                                           # a model that repeats itself: its drafts are confirmed
        assert int(loop.accepted) > 0
    for p in range(P):
        for i in range(N):
            sequence = torch.cat([prompts[p], torch.tensor(paths[p][i][:-1], device="cuda", dtype=torch.long)])
            tokens = torch.tensor(paths[p][i], device="cuda")
            logits = plain_logits(model, sequence)[prompt - 1:]
            if greedy and not fp8:
                # every layer rounds six times to 8 bits, the last product once more: 2^-8 of the largest logit each
                behind = logits.amax(-1) - logits.gather(-1, tokens[:, None])[:, 0]
                assert (behind <= 13 * 2.0 ** -8 * logits.abs().amax(-1)).all(), behind.max()
    if not fp8:                                          # what the cache holds for the paths' tokens
        p, i = P - 1, N - 1
        k, v = loop.cache.read(0, length[p][i])
        x = model.tokens[torch.tensor([int(prompts[p, -1])] + paths[p][i][:-1], device="cuda")].double()
        x = x + model.positions[prompt - 1:prompt - 1 + len(x)].double()
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        qkv = (x @ model.layers[0]["qkv"].double()).unflatten(-1, (8, 64))
        for got, want in ((k, qkv[:, 4:6]), (v, qkv[:, 6:])):
            # input, its norm and the product are rounded to 8 bits: 3 * 2^-8 of sums of 128 terms, which add up by squares
            error = (got[p, i].double() - want).abs()
            assert (error <= 4 * 3 * 2.0 ** -8 * want.square().mean().sqrt() + 2.0 ** -8 * want.abs()).all(), error.max()

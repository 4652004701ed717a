"""A decode loop with a target model: drafts, the verifying pass over them, acceptance.

  python -m paper_2503_05330_amd.verify_loop [--fp8] [--greedy] [--problems P] [--paths N] [--tokens T] ...

The model is a small transformer with random weights, whose matrix products are torch's; what is special to many samples
of one prompt is this package's: the prompts' keys and values are held once (PathCache.write_prompt), every step writes those
of each path's newest token and of the draft behind it (write), attends to prompt and path (attend), picks the model's token
at every position with its probability (targets), counts the confirmed draft tokens (Index.accept), and appends them and
drafts again (Index.step).  Nothing of a step waits for the host.

Prompts of different lengths are packed behind each other for one pass of the model (prompt_attend, PathCache.write_packed).  A model
with rotary positions (--rotary) turns queries and keys as they come (rotate, PathCache.write_rotated), and penalties for repeated
tokens or biases (--repetition, --presence, --frequency) are applied to the logits before the tokens are picked (adjust).
"""
from __future__ import annotations

import argparse
import time

import torch

from . import binding, verify


class Model:
    """Layers of attention with grouped heads and a gated product, token and position embeddings.  It says the
    first 32 tokens more often than others, and 5 v + 1 (mod 32) after v of these as a rule: drafts are made of what samples share."""

    def __init__(self, vocab=4096, dim=512, heads=8, kv_heads=2, head_dim=64, layers=2, max_position=8192, dtype=torch.bfloat16,
                 device="cuda", seed=0, rotary=None):
        """rotary: a verify.Rotary, which queries and keys are turned by instead of the positions' embeddings; whoever attends does it."""
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)

        def weight(rows, cols, size):
            return (torch.randn((rows, cols), generator=gen, device=device) * size * rows ** -0.5).to(dtype)
        self.vocab, self.heads, self.kv_heads, self.head_dim, self.dtype = vocab, heads, kv_heads, head_dim, dtype
        self.rotary = rotary
        self.tokens = weight(vocab, dim, vocab ** 0.5)
        self.positions = weight(max_position, dim, 0.3 * max_position ** 0.5)
        common = torch.arange(32, device=device)
        out = weight(dim, vocab, 0.5).float()
        out[:, common] += weight(dim, 32, 1.0).float()
        out[:, (5 * common + 1) % 32] += 20 / dim * self.tokens[common].float().T
        self.out = out.to(dtype)
        self.layers = [dict(qkv=weight(dim, (heads + 2 * kv_heads) * head_dim, 1.5), o=weight(heads * head_dim, dim, 1.0),
                            up=weight(dim, 4 * dim, 1.0), down=weight(2 * dim, dim, 2.0)) for _ in range(layers)]

    @staticmethod
    def norm(x):
        return x * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6).to(x.dtype)

    def __call__(self, tokens, first, attention, at=None):
        """Logits [..., n, vocab] of tokens [..., n] at positions first [...] and on, or at [..., n]; attention(layer, q, k, v)."""
        x = self.tokens[tokens.long().clamp(min=0)]
        if self.rotary is None:
            if at is None:
                at = first[..., None] + torch.arange(tokens.shape[-1], device=tokens.device)
            x = x + self.positions[at.clamp(max=len(self.positions) - 1)]
        H, Hk = self.heads, self.kv_heads
        for i, w in enumerate(self.layers):
            qkv = (self.norm(x) @ w["qkv"]).unflatten(-1, (H + 2 * Hk, self.head_dim))
            a = attention(i, qkv[..., :H, :], qkv[..., H:H + Hk, :], qkv[..., H + Hk:, :])
            x = x + a.flatten(-2) @ w["o"]
            gate, up = (self.norm(x) @ w["up"]).chunk(2, -1)
            x = x + (torch.nn.functional.silu(gate) * up) @ w["down"]
        return self.norm(x) @ self.out


class Loop:
    """P x N paths that continue P prompts by up to path_cap tokens each.

    prompts: a tensor [P][T], or a list of tensors of different lengths.  penalties [P][3] (repetition, presence, frequency) and bias
    [P][vocab] or [vocab], float32: see verify.adjust; a path has said what was sampled for it, and the drafted tokens before a position."""

    def __init__(self, model, prompts, paths, path_cap, query_len=3, draft_len=8, inv_temperature=1.0, greedy=False, fp8=False, seed=1,
                 penalties=None, bias=None):
        packed = not torch.is_tensor(prompts)
        P, T = (len(prompts), max(map(len, prompts))) if packed else prompts.shape
        dev = prompts[0].device
        self.model, self.P, self.N, self.L, self.k = model, P, paths, draft_len, query_len
        self.inv_temperature, self.greedy = inv_temperature, greedy
        self.shape = shape = dict(n_heads=model.heads, n_kv_heads=model.kv_heads, head_dim=model.head_dim, n_layers=len(model.layers),
                                  dtype=model.dtype, fp8=fp8)
        self.cache = verify.PathCache(P, paths, T - 1, path_cap, max_step=draft_len + 1, **shape)
        self.index = binding.Index(P, paths, path_cap, model.vocab, query_len, draft_len, flags=binding.INCLUDE_SELF)
        self.gen = torch.Generator(device=dev)
        self.gen.manual_seed(seed)
        if packed or model.rotary is not None:
            self.prompt_tokens = self._packed([x for x in prompts])
            self.last = torch.stack([x[-1] for x in prompts])[:, None, None].expand(P, paths, 1).to(torch.int32)
        else:
            self._in_steps(prompts)
            self.prompt_tokens = T - 1
            self.last = prompts[:, -1:, None].expand(P, paths, 1).to(torch.int32)
        self.length = torch.zeros((P, paths), dtype=torch.int32, device=dev)       # of each path in the cache
        self.draft = None
        self.accepted = torch.zeros((), dtype=torch.int64, device=dev)
        self.penalties, self.bias = penalties, bias
        if penalties is not None:                        # the paths' tokens, behind their prompts' last, and the prompts
            self.said = torch.zeros((P, paths, path_cap + draft_len + 1), dtype=torch.int32, device=dev)
            self.asked = torch.nn.utils.rnn.pad_sequence([x for x in prompts], batch_first=True).to(torch.int32)
            self.asked_len = torch.tensor([len(x) for x in prompts], dtype=torch.int32).to(dev)

    def _in_steps(self, prompts):
        # the prompt but for its last token, which is every path's first: a few tokens at a time through the path part of another
        # cache, whose contents become the prompt of this one
        model, (P, T), dev = self.model, prompts.shape, prompts.device
        first = verify.PathCache(P, 1, 0, max(T - 1, 1), max_step=32, **self.shape)
        for t in range(0, T - 1, 32):
            part = prompts[:, None, t:min(t + 32, T - 1)]
            start = torch.full((P, 1), t, dtype=torch.int32, device=dev)
            model(part, start, lambda i, q, k, v: self._attend(first, i, q, k, v, start, None, None))
        for i in range(len(model.layers) if T > 1 else 0):
            k, v = first.read(i, T - 1)
            self.cache.write_prompt(i, k[:, 0], v[:, 0])

    def _packed(self, prompts):
        # the same, all prompts behind each other in one pass; returns their lengths [P][1]
        model, dev = self.model, prompts[0].device
        length = torch.tensor([len(x) - 1 for x in prompts])
        offsets = torch.nn.functional.pad(length.cumsum(0), (1, 0)).to(torch.int32).to(dev)
        if int(length.sum()):
            at = torch.cat([torch.arange(n, dtype=torch.int32) for n in length]).to(dev)

            def attention(i, q, k, v):
                if model.rotary is not None:
                    verify.rotate(q, at, model.rotary, out=q)
                    verify.rotate(k, at, model.rotary, out=k)
                self.cache.write_packed(i, k, v, offsets)
                return verify.prompt_attend(q, k, v, offsets)
            model(torch.cat([x[:-1] for x in prompts]), None, attention, at)
        return length.to(torch.int32).to(dev)[:, None]

    @staticmethod
    def _attend(cache, layer, q, k, v, start, prompt_len, counts, rotary=None, at=None):
        if rotary is None:
            cache.write(layer, k, v, start, counts)
        else:
            q = cache.write_rotated(layer, q, k, v, rotary, at, start, counts)
        n = q.shape[-3] if counts is None else counts
        return cache.attend(layer, q, prompt_len, start + n, counts)

    def _adjust(self, logits, tokens, counts):
        n = tokens.shape[-1]
        if self.penalties is None:
            return logits if self.bias is None else verify.adjust(logits, counts=counts, bias=self.bias, out=logits)
        at = self.length.long()[..., None] + torch.arange(n, device=tokens.device)
        self.said.scatter_(-1, at.clamp(max=self.said.shape[-1] - 1), tokens)
        return verify.adjust(logits, self.said[..., 1:], self.length + counts - 1, counts, self.asked, self.asked_len, self.penalties, self.bias, out=logits)

    def step(self):
        """One verifying pass: returns the model's tokens [P][N][n] and how many of them each path takes [P][N]."""
        P, N, L = self.P, self.N, self.L
        if self.draft is None:
            tokens, counts = self.last, torch.ones((P, N), dtype=torch.int32, device=self.last.device)
        else:
            tokens, counts = torch.cat([self.last, self.draft["tokens"]], -1), self.draft["length"] + 1
        first, prompt_len, at = self.length + self.prompt_tokens, None, None
        if torch.is_tensor(self.prompt_tokens):
            prompt_len = self.prompt_tokens
            at = first[..., None] + torch.arange(tokens.shape[-1], device=tokens.device, dtype=torch.int32)
        logits = self.model(tokens, first, lambda i, q, k, v: self._attend(self.cache, i, q, k, v, self.length, prompt_len, counts,
                                                                           self.model.rotary, at), at)
        logits = self._adjust(logits, tokens, counts)
        noise = None
        if not self.greedy:
            u = torch.rand(logits.shape, generator=self.gen, device=logits.device).clamp_(min=1e-30)
            noise = u.log_().neg_().log_().neg_()
        picked, probs = verify.targets(logits, noise, self.inv_temperature)
        if self.draft is None:
            taken = counts
        else:
            taken = self.index.accept(self.draft["tokens"], self.draft["length"], picked[..., :L].contiguous(), L) + 1
        self.length = self.length + taken
        self.accepted = self.accepted + (taken - 1).sum()
        self.last = picked.gather(-1, (taken - 1)[..., None].long())
        self.draft = self.index.step(picked, probs, taken, picked.shape[-1], self.k, L)
        return picked, taken


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    parser.add_argument("--problems", type=int, default=4)
    parser.add_argument("--paths", type=int, default=16)
    parser.add_argument("--prompt", type=int, default=512)
    parser.add_argument("--shortest", type=int, default=0, help="prompts of different lengths, from this to --prompt")
    parser.add_argument("--tokens", type=int, default=128, help="steps are run until every path must have so many")
    parser.add_argument("--draft", type=int, default=8)
    parser.add_argument("--temperature", type=float, default=0.25)
    parser.add_argument("--greedy", action="store_true")
    parser.add_argument("--fp8", action="store_true", help="an 8-bit cache")
    parser.add_argument("--rotary", action="store_true", help="rotary positions")
    parser.add_argument("--repetition", type=float, default=1.0)
    parser.add_argument("--presence", type=float, default=0.0)
    parser.add_argument("--frequency", type=float, default=0.0)
    a = parser.parse_args(argv)
    model = Model(rotary=verify.Rotary(64) if a.rotary else None)
    prompts = torch.randint(0, model.vocab, (a.problems, a.prompt), device="cuda")
    if a.shortest:
        prompts = [x[:a.shortest + (a.prompt - a.shortest) * i // max(1, a.problems - 1)] for i, x in enumerate(prompts)]
    penalties = None
    if (a.repetition, a.presence, a.frequency) != (1.0, 0.0, 0.0):
        penalties = torch.tensor([[a.repetition, a.presence, a.frequency]], device="cuda").expand(a.problems, 3).contiguous()
    loop = Loop(model, prompts, a.paths, a.tokens * (a.draft + 1), draft_len=a.draft, inv_temperature=1 / a.temperature,
                greedy=a.greedy, fp8=a.fp8, penalties=penalties)
    loop.step()
    torch.cuda.synchronize()
    begin = time.perf_counter()
    for _ in range(a.tokens - 1):
        loop.step()
    torch.cuda.synchronize()
    seconds = time.perf_counter() - begin
    rows = a.problems * a.paths
    print("%d paths, %d steps: %.2f draft tokens accepted per path and step, %.0f tokens/s, status %d %d"
          % (rows, a.tokens, loop.accepted.item() / rows / (a.tokens - 1), (loop.length.sum().item() - rows) / seconds,
             loop.cache.status(), loop.index.status()))


if __name__ == "__main__":
    main()

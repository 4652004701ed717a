"""The operators of a target model's verifying pass over the drafts of many samples, as cases to be timed.

Between a draft and its acceptance the target model sees, for every path (sample) of every problem (prompt), the token
that the path ends with and the drafted ones behind it.  What is special to many samples of one prompt there:

  attend    attention of these tokens to the problem's prompt, which all its paths share, and to the path's own tokens,
            from a cache of 16-bit values or of e4m3 values with a power-of-two scale per token and head
  turn      the new tokens' keys and values written to that cache (quantised as they are written), and read back
  targets   the model's own token at every position (noise, if any, is given) and the probability it gave it

The plain forms compute in 32 bits by elementary operations.  Rows of `counts` tokens out of `step` are ragged as drafts are;
outputs of positions beyond a row's count are zero (tokens: not masked, every position has logits).
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_DEVICE = "cuda"


def _attend(name, problems, paths, step, prompt, path, heads=32, kv_heads=8, dim=128, type="bf16", fp8=False, ragged=True):
    c = dict(op="attend", problems=problems, paths=paths, step=step, prompt=prompt, path=path, heads=heads, kv_heads=kv_heads,
             dim=dim, type=type, fp8=fp8, ragged=ragged)
    return dict(c, name=name) if name else c


def _turn(name, problems, paths, step, path, kv_heads=8, dim=128, type="bf16", fp8=False, ragged=True):
    """paths 0: the prompts' part of the cache, `step` tokens from the start of each."""
    c = dict(op="turn", problems=problems, paths=paths, step=step, path=path, kv_heads=kv_heads, dim=dim, type=type, fp8=fp8,
             ragged=ragged)
    return dict(c, name=name) if name else c


def _targets(name, rows, vocab, type="bf16", noise=False):
    c = dict(op="targets", rows=rows, vocab=vocab, type=type, noise=noise)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest request: four short samples, a token each.  Launches and latency are all there is to it.
        _attend("attend_4x1", 1, 4, 1, 256, 64),
        # sixteen samples without drafts: plain decoding, bound by the paths' own caches
        _attend("attend_16x1", 1, 16, 1, 1024, 1024),
        # the same samples verify drafts of up to eight tokens
        _attend("attend_16x9", 1, 16, 9, 1024, 1024),
        # the longest histories of one problem, drafts of sixteen, seven query heads to a kv head: matrix products
        _attend("attend_64x17_long", 1, 64, 17, 4096, 4096, heads=28, kv_heads=4),
        # a server's batch of 64 problems, verifying drafts out of an 8-bit cache
        _attend("attend_64_problems", 64, 16, 9, 1024, 1024, fp8=True),
        # the batch without drafts on long prompts: the 8-bit cache is read once
        _attend("attend_64_problems_x1", 64, 16, 1, 4096, 512, fp8=True),
        # odd sizes, heads of 64 without groups, half precision
        _attend("attend_3x13_odd", 3, 13, 8, 777, 333, heads=12, kv_heads=12, dim=64, type="f16"),
        # the smallest write: one new token of four samples
        _turn("turn_4x1", 1, 4, 1, 256),
        # a batch's verified tokens, quantised
        _turn("turn_64_problems", 64, 16, 9, 1024, fp8=True),
        # eight whole prompts, quantised: what a prefill leaves, read back to be handed to another server
        _turn("turn_prompts", 8, 0, 4096, 4096, fp8=True),
        # greedy tokens of four samples
        _targets("targets_4", 4, 32000),
        # sampled tokens of 64 paths' verified positions, the largest vocabulary
        _targets("targets_64x17", 64 * 17, 152064, noise=True),
    ]


def _spread(rng, lo, hi):
    """A whole number in lo .. hi, evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Sizes over the ranges that the listed cases span; a case that costs more than the largest listed one of its operator
    is drawn again."""
    op = rng.choice(("attend", "attend", "turn", "targets"))
    most = {"bytes": 0, "flops": 0}
    for c in listed():
        if c["op"] == op:
            most = {k: max(x, work(c)[k]) for k, x in most.items()}
    while True:
        heads, kv_heads, dim = rng.choice(((32, 8, 128), (28, 4, 128), (12, 12, 64), (16, 2, 128), (14, 2, 64), (8, 8, 128)))
        problems = _spread(rng, 1, 64) if rng.random() < 0.6 else 1
        paths, step = _spread(rng, 1, 64), rng.choice((1, 1, rng.randint(2, 17)))
        more = dict(kv_heads=kv_heads, dim=dim, type=rng.choice(("bf16", "bf16", "f16")), fp8=rng.random() < 0.5,
                    ragged=rng.random() < 0.8)
        if op == "attend":
            c = _attend("", problems, paths, step, _spread(rng, 1, 8192), step + _spread(rng, 1, 4096), heads=heads, **more)
        elif op == "turn":
            if rng.random() < 0.3:
                n = _spread(rng, 1, 4096)
                c = _turn("", problems, 0, n, n + rng.randint(0, 64), **more)
            else:
                c = _turn("", problems, paths, step, step + _spread(rng, 1, 1024), **more)
        else:
            c = _targets("", _spread(rng, 1, 64 * 17), _spread(rng, 1000, 152064), type=rng.choice(("bf16", "f16", "f32")),
                         noise=rng.random() < 0.5)
        cost = work(c)
        if all(cost[k] <= most[k] for k in cost):
            return c


# ---------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device=_DEVICE)
    gen.manual_seed(seed)
    return gen


def _keys_values(gen, lead, case):
    """Keys with a few channels that are larger than the others, as trained models have them, values of one size."""
    kw = dict(generator=gen, device=_DEVICE, dtype=_TYPES[case["type"]])
    H, D = case["kv_heads"], case["dim"]
    k = torch.randn((*lead, H, D), **kw)
    k[..., 3::29] *= 2.5
    return k, torch.randn((*lead, H, D), **kw)


def _ragged(gen, shape, lo, hi):
    return torch.randint(lo, hi + 1, shape, generator=gen, device=_DEVICE, dtype=torch.int32)


def _inputs(case, seed):
    gen = _generator(seed)
    s = {"case": case}
    if case["op"] == "targets":
        R, V = case["rows"], case["vocab"]
        x = torch.randn((R, V), generator=gen, device=_DEVICE)
        x *= 2.5
        # a few tokens that the model thinks of, and some that it may not use
        likely = torch.randint(0, V, (R, 8), generator=gen, device=_DEVICE)
        x.scatter_add_(1, likely, 12 * torch.rand((R, 8), generator=gen, device=_DEVICE))
        banned = torch.randint(0, V, (max(1, V // 100),), generator=gen, device=_DEVICE)
        x[:, banned] = -math.inf
        s["logits"] = x.to(_TYPES[case["type"]])
        s["noise"] = None
        if case["noise"]:
            u = torch.rand((R, V), generator=gen, device=_DEVICE).clamp_(min=1e-30)
            s["noise"] = u.log_().neg_().clamp_(min=1e-30).log_().neg_()
        s["inv_temperature"] = 1.25 if case["noise"] else 1.0
        return s
    P, N, n = case["problems"], case["paths"], case["step"]
    if case["op"] == "turn":
        lead = (P, N, n) if N else (P, n)
        # keys and values as a projection leaves them, beside each other
        kv = torch.empty((*lead, 2 * case["kv_heads"], case["dim"]), device=_DEVICE, dtype=_TYPES[case["type"]])
        k, v = _keys_values(gen, lead, case)
        kv[..., :case["kv_heads"], :], kv[..., case["kv_heads"]:, :] = k, v
        s["k"], s["v"] = kv[..., :case["kv_heads"], :], kv[..., case["kv_heads"]:, :]
        rows = (P, N) if N else (P,)
        s["start"] = _ragged(gen, rows, 0, case["path"] - n)
        s["counts"] = _ragged(gen, rows, 0, n) if case["ragged"] and n > 1 else None
        return s
    s["prompt_k"], s["prompt_v"] = _keys_values(gen, (P, case["prompt"]), case)
    s["path_k"], s["path_v"] = _keys_values(gen, (P, N, case["path"]), case)
    H, D = case["heads"], case["dim"]
    qkv = torch.randn((P, N, n, H + 2 * case["kv_heads"], D), generator=gen, device=_DEVICE, dtype=_TYPES[case["type"]])
    s["q"] = qkv[..., :H, :]
    if case["ragged"]:
        s["prompt_len"] = _ragged(gen, (P,), (case["prompt"] + 1) // 2, case["prompt"])
        s["path_len"] = _ragged(gen, (P, N), max(n, case["path"] // 4), case["path"])
        s["counts"] = _ragged(gen, (P, N), 1, n)
        # a path that has ended offers no token
        s["counts"] *= (torch.rand((P, N), generator=gen, device=_DEVICE) > 1 / 16).int()
    else:
        s["prompt_len"] = torch.full((P,), case["prompt"], device=_DEVICE, dtype=torch.int32)
        s["path_len"] = torch.full((P, N), case["path"], device=_DEVICE, dtype=torch.int32)
        s["counts"] = None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "targets":
        return s
    P, N, n = case["problems"], case["paths"], case["step"]
    if own:
        from paper_2503_05330_amd import verify
        attend = case["op"] == "attend"
        prompt = case["prompt"] if attend else 0 if N else case["path"]
        s["cache"] = cache = verify.PathCache(P, max(N, 1), prompt, case["path"] if N else 1, case.get("heads", case["kv_heads"]),
                                              case["kv_heads"], case["dim"], n if N else 1, dtype=_TYPES[case["type"]],
                                              fp8=case["fp8"])
        if attend:
            cache.write_prompt(0, s.pop("prompt_k"), s.pop("prompt_v"))
            cache.write(0, s.pop("path_k"), s.pop("path_v"))
    elif case["op"] == "attend":
        for name in ("prompt_k", "prompt_v", "path_k", "path_v"):
            s[name] = _store(s[name], case["fp8"])
    else:
        cap = (P, N, case["path"]) if N else (P, case["path"])
        empty = torch.zeros((*cap, case["kv_heads"], case["dim"]), device=_DEVICE, dtype=_TYPES[case["type"]])
        s["k_cache"], s["v_cache"] = _store(empty, case["fp8"]), _store(empty, case["fp8"])
    return s


# ----------------------------------------------------------------------------------------------------- plain forms

def _store(x, fp8):
    """What a cache holds of x: (values,), or (codes, scales) with the least power of two that takes the largest value of
    a token's head to at most 448, the largest e4m3 number."""
    if not fp8:
        return (x,)
    x = x.float()
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))      # amax = m * 2^e, m in [0.5, 1)
    e = torch.where(m > 0.875, e - 8, e - 9)
    scale = torch.where(m > 0, torch.exp2(e.float().clamp(min=-126)), 1.0)
    return ((x / scale).to(torch.float8_e4m3fn), scale)


def _load(held):
    return held[0].float() if len(held) == 1 else held[0].float() * held[1]


def _plain_attend(s):
    case, q = s["case"], s["q"].float()
    P, N, n, H, D = q.shape
    Hk, T, U = case["kv_heads"], case["prompt"], case["path"]
    G = H // Hk
    q = q.reshape(P, N, n, Hk, G, D).permute(0, 3, 1, 2, 4, 5) * D ** -0.5               # [P][Hk][N][n][G][D]
    q = q.reshape(P, Hk, N * n * G, D)
    keys = _load(s["prompt_k"]).permute(0, 2, 3, 1).contiguous()                         # [P][Hk][D][T]
    to_prompt = torch.matmul(q, keys).reshape(P, Hk, N, n * G, T)
    seen = torch.arange(T, device=_DEVICE) < s["prompt_len"][:, None]
    to_prompt.masked_fill_(~seen[:, None, None, None, :], -math.inf)
    own_q = q.reshape(P, Hk, N, n * G, D).transpose(1, 2).contiguous()                   # [P][N][Hk][n G][D]
    keys = _load(s["path_k"]).permute(0, 1, 3, 4, 2).contiguous()                        # [P][N][Hk][D][U]
    to_path = torch.matmul(own_q, keys)
    counts = s["counts"] if s["counts"] is not None else torch.full((P, N), n, device=_DEVICE, dtype=torch.int32)
    t = torch.arange(n, device=_DEVICE)
    end = s["path_len"][..., None] - counts[..., None] + t + 1                           # [P][N][n]
    seen = torch.arange(U, device=_DEVICE) < end[..., None]                              # [P][N][n][U]
    seen = seen[:, :, None, :, None, :].expand(P, N, 1, n, G, U).reshape(P, N, 1, n * G, U)
    to_path.masked_fill_(~seen, -math.inf)
    to_path = to_path.transpose(1, 2)                                                    # [P][Hk][N][n G][U]
    top = torch.maximum(to_prompt.amax(-1), to_path.amax(-1))
    top = torch.where(top == -math.inf, 0.0, top)[..., None]
    to_prompt, to_path = to_prompt.sub_(top).exp_(), (to_path - top).exp_()
    total = to_prompt.sum(-1) + to_path.sum(-1)
    values = _load(s["prompt_v"]).permute(0, 2, 1, 3).contiguous()                       # [P][Hk][T][D]
    out = torch.matmul(to_prompt.reshape(P, Hk, N * n * G, T), values).reshape(P, Hk, N, n * G, D)
    values = _load(s["path_v"]).permute(0, 1, 3, 2, 4).contiguous()                      # [P][N][Hk][U][D]
    out = out + torch.matmul(to_path.transpose(1, 2).contiguous(), values).transpose(1, 2)
    out = torch.where(total[..., None] > 0, out / total[..., None], 0.0)
    out = out.reshape(P, Hk, N, n, G, D).permute(0, 2, 3, 1, 4, 5).reshape(P, N, n, H, D)
    return torch.where((t < counts[..., None])[..., None, None], out, 0.0).to(_TYPES[case["type"]])


def _plain_turn(s):
    case = s["case"]
    n, start, counts = case["step"], s["start"].long(), s["counts"]
    t = torch.arange(n, device=_DEVICE)
    at = start[..., None] + t
    live = (t < counts[..., None]) if counts is not None else torch.ones_like(at, dtype=torch.bool)
    if case["paths"]:
        row = torch.arange(start.numel(), device=_DEVICE).reshape(start.shape)[..., None].expand_as(at)
    else:
        row = torch.arange(start.shape[0], device=_DEVICE)[:, None].expand_as(at)
    outs = []
    for new, cache in ((s["k"], s["k_cache"]), (s["v"], s["v_cache"])):
        parts = []
        for held, part in zip(cache, _store(new, case["fp8"])):
            flat = held.view(-1, *held.shape[-3:])                                       # rows of tokens
            if part.dtype == torch.float8_e4m3fn:                                        # bytes are what is moved
                flat, part = flat.view(torch.uint8), part.view(torch.uint8)
            flat[row[live], at[live]] = part[live]
            got = flat[row, at]
            parts.append(got.view(torch.float8_e4m3fn) if held.dtype == torch.float8_e4m3fn else got)
        outs.append(torch.where(live[..., None, None], _load(parts), 0.0).to(_TYPES[case["type"]]))
    return tuple(outs)


def _plain_targets(s):
    x = s["logits"].float()
    y = x * s["inv_temperature"]
    z = x if s["noise"] is None else y + s["noise"]
    best = z.amax(-1, keepdim=True)
    place = torch.arange(z.shape[1], device=_DEVICE)
    token = torch.where(z == best, place, z.shape[1]).amin(-1)                           # the lowest of equals
    y = (y - y.amax(-1, keepdim=True)).exp_()
    return token.int(), y.gather(1, token[:, None])[:, 0] / y.sum(-1)


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"attend": _plain_attend, "turn": _plain_turn, "targets": _plain_targets}[op](state)
    if op == "targets":
        from paper_2503_05330_amd import verify
        return verify.targets(state["logits"], state["noise"], state["inv_temperature"])
    cache = state["cache"]
    if op == "attend":
        return cache.attend(0, state["q"], state["prompt_len"], state["path_len"], state["counts"])
    start, counts, n = state["start"], state["counts"], state["case"]["step"]
    if state["case"]["paths"]:
        cache.write(0, state["k"], state["v"], start, counts)
        return cache.read(0, n, start, counts)
    cache.write_prompt(0, state["k"], state["v"], start, counts)
    return cache.read_prompt(0, n, start, counts)


# ----------------------------------------------------------------------------------------------------------- exact

def _held64(x, fp8):
    """The values that a cache holds of x, from the format's definition: three bits behind the leading one, exponents down
    to -6, below which the spacing stays 2^-9."""
    x = x.double()
    if not fp8:
        return x
    high = x.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(torch.where(high > 0, high, 448.0) / 448))
    # the logarithm is rounded: the least power that holds 448 * 2^power >= high
    power = torch.where(448 * torch.exp2(power - 1) >= high, power - 1, power)
    power = torch.where(448 * torch.exp2(power) < high, power + 1, power)
    power = torch.where(high > 0, power.clamp(min=-126), 0.0)
    y = x * torch.exp2(-power)
    lead = torch.frexp(y)[1].double() - 1
    grain = torch.exp2(lead.clamp(min=-6) - 3)
    return torch.round(y / grain) * grain * torch.exp2(power)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "targets":
        tokens, probs = [], []
        for r in range(0, case["rows"], 128):
            x = s["logits"][r:r + 128].double()
            y = x * s["inv_temperature"]
            z = x if s["noise"] is None else y + s["noise"][r:r + 128].double()
            first = (z == z.max(-1, keepdim=True).values).int().argmax(-1)
            tokens.append(first.int())
            probs.append((y.gather(1, first[:, None])[:, 0] - torch.logsumexp(y, -1)).exp())
        return torch.cat(tokens), torch.cat(probs)
    P, N, n = case["problems"], case["paths"], case["step"]
    if case["op"] == "turn":
        t = torch.arange(n, device=_DEVICE)
        live = t < (s["counts"][..., None] if s["counts"] is not None else n)
        return tuple(torch.where(live[..., None, None], _held64(x, case["fp8"]), 0.0) for x in (s["k"], s["v"]))
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    out = torch.zeros((P, N, n, H, D), device=_DEVICE, dtype=torch.float64)
    prompt_len, path_len = s["prompt_len"].tolist(), s["path_len"].tolist()
    counts = s["counts"].tolist() if s["counts"] is not None else [[n] * N] * P
    for p in range(P):
        T = prompt_len[p]
        prompt_k = _held64(s["prompt_k"][p, :T], case["fp8"]).transpose(0, 1)            # [Hk][T][D]
        prompt_v = _held64(s["prompt_v"][p, :T], case["fp8"]).transpose(0, 1)
        for i in range(N):
            c, U = counts[p][i], path_len[p][i]
            if c == 0:
                continue
            k = torch.cat([prompt_k, _held64(s["path_k"][p, i, :U], case["fp8"]).transpose(0, 1)], 1)
            v = torch.cat([prompt_v, _held64(s["path_v"][p, i, :U], case["fp8"]).transpose(0, 1)], 1)
            q = s["q"][p, i, :c].double().reshape(c, Hk, H // Hk, D).permute(1, 0, 2, 3).reshape(Hk, -1, D)
            score = torch.matmul(q, k.transpose(1, 2)) / math.sqrt(D)                    # [Hk][c G][T + U]
            end = T + U - c + 1 + torch.arange(c, device=_DEVICE).repeat_interleave(H // Hk)
            hidden = torch.arange(T + U, device=_DEVICE) >= end[:, None]
            weight = torch.softmax(score.masked_fill(hidden, -math.inf), -1)
            o = torch.matmul(weight, v).reshape(Hk, c, H // Hk, D)
            out[p, i, :c] = o.permute(1, 0, 2, 3).reshape(c, H, D)
    return out


# ------------------------------------------------------------------------------------------------------------ work

def work(case):
    """attend: each prompt's and each path's keys and values once, queries and outputs; two products.  turn: keys and values
    read, what the cache holds of them written and read again, the values written.  targets: logits and noise once."""
    if case["op"] == "targets":
        cells = case["rows"] * case["vocab"]
        size = _TYPES[case["type"]].itemsize + (4 if case["noise"] else 0)
        return {"bytes": cells * size + 8 * case["rows"], "flops": cells * (5 if case["noise"] else 3)}
    D, Hk, n = case["dim"], case["kv_heads"], case["step"]
    held = 2 * Hk * (D + 1 if case["fp8"] else 2 * D)                                    # bytes of a token, K and V
    if case["op"] == "turn":
        rows = case["problems"] * max(case["paths"], 1)
        tokens = rows * (n / 2 if case["ragged"] and n > 1 else n)
        return {"bytes": tokens * (2 * held + 4 * Hk * D) + rows * n * 4 * Hk * D, "flops": tokens * 4 * Hk * D}
    P, N, H = case["problems"], case["paths"], case["heads"]
    prompt, path, queries = case["prompt"], case["path"], n
    if case["ragged"]:
        prompt, path = 0.75 * prompt, (max(n, path // 4) + path) / 2
        queries = 15 / 16 * (1 + n) / 2
    rows = P * N * queries * H
    return {"bytes": P * (prompt + N * path) * held + rows * D * 2 + P * N * n * H * D * 2,
            "flops": rows * (prompt + path) * 4 * D}

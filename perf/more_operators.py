"""What a target model does around its attention over the cache, as cases to be timed.

  prompt   attention of whole prompts to themselves: causal, grouped heads, sequences of different lengths packed behind each other
  rotate   rotary positions on queries and keys where a projection left them
  place    a verifying pass's new tokens: queries and keys rotated, keys and values written to the cache (quantised where it
           holds 8 bits), and read back
  adjust   logits of every position of a verifying pass: penalties for tokens that the prompt or the path has, biases, a
           grammar's mask.  The drafted tokens before a position count as said.

The plain forms compute in 32 bits by elementary operations, angles in 64.  Rows of `counts` tokens out of `step` are ragged as
drafts are; what lies beyond a row's count is zero (place: queries are all rotated).
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_DEVICE = "cuda"
_HEADS = ((32, 8, 128), (28, 4, 128), (12, 12, 64), (16, 2, 128), (14, 2, 64), (8, 8, 128), (8, 2, 64), (32, 8, 96), (16, 8, 256))


def _prompt(name, sequences, longest, shortest, heads=32, kv_heads=8, dim=128, type="bf16"):
    """Lengths are spread evenly over shortest .. longest, in an order of the seed's."""
    c = dict(op="prompt", sequences=sequences, longest=longest, shortest=shortest, heads=heads, kv_heads=kv_heads, dim=dim, type=type)
    return dict(c, name=name) if name else c


def _positions(rotated, interleaved, factor=1.0, original=0, base=10000.0):
    return dict(rotated=rotated, interleaved=interleaved, factor=factor, original=original, base=base)


def _rotate(name, tokens, first, how, heads=32, kv_heads=8, dim=128, type="bf16"):
    """Eight sequences' tokens (fewer: each its own), at positions first and on."""
    c = dict(op="rotate", tokens=tokens, first=first, heads=heads, kv_heads=kv_heads, dim=dim, type=type, **how)
    return dict(c, name=name) if name else c


def _place(name, problems, paths, step, path, how, heads=32, kv_heads=8, dim=128, type="bf16", fp8=False, ragged=True):
    c = dict(op="place", problems=problems, paths=paths, step=step, path=path, heads=heads, kv_heads=kv_heads, dim=dim, type=type,
             fp8=fp8, ragged=ragged, **how)
    return dict(c, name=name) if name else c


def _adjust(name, problems, paths, step, vocab, prompt, path, type="bf16", mask=False, bias=False, ragged=True):
    c = dict(op="adjust", problems=problems, paths=paths, step=step, vocab=vocab, prompt=prompt, path=path, type=type, mask=mask,
             bias=bias, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one short question, a small model: launches and latency
        _prompt("prompt_40", 1, 40, 40, heads=8, kv_heads=2, dim=64),
        # a server's batch of new requests, from a few words to a page
        _prompt("prompt_16_ragged", 16, 1024, 1),
        # odd lengths, heads of 64 without groups, half precision
        _prompt("prompt_5x777_odd", 5, 777, 331, heads=12, kv_heads=12, dim=64, type="f16"),
        # eight whole prompts, as a prefill takes them
        _prompt("prompt_8x4096", 8, 4096, 4096),
        # one long document, seven query heads to a kv head
        _prompt("prompt_16384", 1, 16384, 16384, heads=28, kv_heads=4),
        # plain decoding of sixteen paths: a token each
        _rotate("rotate_16", 16, 1500, _positions(128, False)),
        # eight whole prompts, positions scaled for a longer context than the model was trained on
        _rotate("rotate_8x4096", 8 * 4096, 0, _positions(128, False, 8.0, 8192, 500000.0)),
        # sixteen paths' tokens and drafts, neighbours as pairs, half of the head
        _place("place_16x9", 1, 16, 9, 1024, _positions(64, True)),
        # a server's batch, into an 8-bit cache
        _place("place_64_problems", 64, 16, 9, 1024, _positions(128, False, 4.0, 4096, 500000.0), fp8=True),
        # four samples' next tokens, penalties alone
        _adjust("adjust_4", 1, 4, 1, 32000, 256, 64),
        # 32 bits, an odd vocabulary, a bias for every token
        _adjust("adjust_3x13_odd", 3, 13, 5, 50257, 777, 333, type="f32", bias=True),
        # 64 paths' verified positions, the largest vocabulary, a grammar for every position
        _adjust("adjust_64x17", 1, 64, 17, 152064, 4096, 4096, mask=True),
    ]


def _spread(rng, lo, hi):
    """A whole number in lo .. hi, evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Sizes over the ranges that the listed cases span; a case that costs more than the largest listed one of its operator
    is drawn again."""
    op = rng.choice(("prompt", "prompt", "prompt", "rotate", "place", "adjust", "adjust"))
    most = {"bytes": 0, "flops": 0}
    for c in listed():
        if c["op"] == op:
            most = {k: max(x, work(c)[k]) for k, x in most.items()}
    while True:
        heads, kv_heads, dim = rng.choice(_HEADS)
        more = dict(heads=heads, kv_heads=kv_heads, dim=dim, type=rng.choice(("bf16", "bf16", "f16")))
        how = _positions(rng.choice((dim, dim, dim // 2)) // 16 * 16, rng.random() < 0.4,
                         *rng.choice(((1.0, 0, 10000.0), (8.0, 8192, 500000.0), (4.0, 0, 10000.0), (32.0, 4096, 1000000.0))))
        problems = _spread(rng, 1, 64) if rng.random() < 0.6 else 1
        paths, step = _spread(rng, 1, 64), rng.choice((1, 1, rng.randint(2, 17)))
        if op == "prompt":
            longest = _spread(rng, 1, 16384)
            c = _prompt("", _spread(rng, 1, 64), longest, rng.choice((1, longest, _spread(rng, 1, longest))), **more)
            if c["sequences"] * heads * longest ** 2 > 28 * 16384 ** 2:                  # (what the plain form holds at once)
                continue
        elif op == "rotate":
            c = _rotate("", _spread(rng, 1, 8 * 4096), rng.choice((0, _spread(rng, 1, 1 << 20))), how, **more)
        elif op == "place":
            c = _place("", problems, paths, step, step + _spread(rng, 1, 1024), how, fp8=rng.random() < 0.5, ragged=rng.random() < 0.8,
                       **more)
        else:
            c = _adjust("", problems, paths, step, _spread(rng, 1000, 152064), _spread(rng, 1, 8192), step + _spread(rng, 1, 4096),
                        type=rng.choice(("bf16", "f16", "f32")), mask=rng.random() < 0.5, bias=rng.random() < 0.3,
                        ragged=rng.random() < 0.8)
        cost = work(c)
        if all(cost[k] <= most[k] for k in cost):
            return c


# ---------------------------------------------------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device=_DEVICE)
    gen.manual_seed(seed)
    return gen


def _ragged(gen, shape, lo, hi):
    return torch.randint(lo, hi + 1, shape, generator=gen, device=_DEVICE, dtype=torch.int32)


def _projection(gen, lead, case):
    """Queries, keys and values beside each other, as a projection leaves them; a few channels of the keys are larger."""
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    x = torch.randn((*lead, H + 2 * Hk, D), generator=gen, device=_DEVICE, dtype=_TYPES[case["type"]])
    x[..., H:H + Hk, 3::29] *= 2.5
    return x


def _lengths(case):
    a, b, n = case["shortest"], case["longest"], case["sequences"]
    return [b - (b - a) * i // max(1, n - 1) for i in range(n)]


def _said(gen, shape, vocab):
    """Tokens as texts have them: a few of them often."""
    u = torch.rand(shape, generator=gen, device=_DEVICE, dtype=torch.float64)
    return (torch.exp(u * math.log(vocab)) - 1).int().clamp_(0, vocab - 1)


def _inputs(case, seed):
    gen = _generator(seed)
    s = {"case": case}
    if case["op"] == "prompt":
        order = torch.randperm(case["sequences"], generator=gen, device=_DEVICE)
        length = torch.tensor(_lengths(case), device=_DEVICE)[order]
        s["offsets"] = torch.nn.functional.pad(length.cumsum(0), (1, 0)).int()
        s["qkv"] = _projection(gen, (sum(_lengths(case)),), case)
        return s
    if case["op"] == "rotate":
        t = torch.arange(case["tokens"], device=_DEVICE, dtype=torch.int32)
        s["positions"] = case["first"] + (t % -(-case["tokens"] // 8) if case["tokens"] >= 64 else 0 * t)
        s["qkv"] = _projection(gen, (case["tokens"],), case)
        return s
    P, N, n = case["problems"], case["paths"], case["step"]
    s["counts"] = None
    if case["ragged"]:
        s["counts"] = _ragged(gen, (P, N), 1, n)
        # a path that has ended offers no token
        s["counts"] *= (torch.rand((P, N), generator=gen, device=_DEVICE) > 1 / 16).int()
    if case["op"] == "place":
        s["qkv"] = _projection(gen, (P, N, n), case)
        s["start"] = _ragged(gen, (P, N), 0, case["path"] - n)
        before = _ragged(gen, (P, 1), 0, 4096)           # the prompts' tokens
        s["positions"] = (before + s["start"])[..., None] + torch.arange(n, device=_DEVICE, dtype=torch.int32)
        return s
    V = case["vocab"]
    x = torch.randn((P, N, n, V), generator=gen, device=_DEVICE)
    s["logits"] = (x * 2.5).to(_TYPES[case["type"]])
    s["prompt"], s["tokens"] = _said(gen, (P, case["prompt"]), V), _said(gen, (P, N, case["path"]), V)
    s["prompt_len"] = _ragged(gen, (P,), (case["prompt"] + 1) // 2, case["prompt"])
    s["path_len"] = _ragged(gen, (P, N), max(n, case["path"] // 4), case["path"])
    # repetition, presence, frequency; one request in a few asks for none of it
    s["penalties"] = torch.tensor([1.05, 0.1, 0.05], device=_DEVICE) + torch.rand((P, 3), generator=gen, device=_DEVICE) * 0.25
    s["penalties"][3::4] = torch.tensor([1.0, 0.0, 0.0], device=_DEVICE)
    s["bias"] = s["mask"] = None
    if case["bias"]:
        s["bias"] = torch.randn((P, V), generator=gen, device=_DEVICE)
    if case["mask"]:
        # inside a string all but a few tokens go on, elsewhere a few only
        words = (P, N, n, -(-V // 32))
        bits = torch.randint(-1 << 31, 1 << 31, (3, *words), generator=gen, device=_DEVICE, dtype=torch.int64).int()
        few = torch.rand((P, N, n, 1), generator=gen, device=_DEVICE) < 0.5
        s["mask"] = torch.where(few, bits[0] & bits[1] & bits[2], bits[0] | bits[1] | bits[2])
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2503_05330_amd import verify
        if case["op"] in ("rotate", "place"):
            s["rotary"] = verify.Rotary(case["rotated"], base=case["base"], interleaved=case["interleaved"], factor=case["factor"],
                                        original=case["original"])
        if case["op"] == "place":
            s["cache"] = verify.PathCache(case["problems"], case["paths"], 0, case["path"], case["heads"], case["kv_heads"], case["dim"],
                                          case["step"], dtype=_TYPES[case["type"]], fp8=case["fp8"])
    elif case["op"] == "place":
        cap = (case["problems"], case["paths"], case["path"], case["kv_heads"], case["dim"])
        empty = torch.zeros(cap, device=_DEVICE, dtype=_TYPES[case["type"]])
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


def _turned(x, positions, case):
    """x [..., heads, D] at positions [...], in 32 bits."""
    R, original = case["rotated"], case["original"]
    turns = case["base"] ** (torch.arange(0, R, 2, device=_DEVICE, dtype=torch.float64) / -R)
    if original:
        keep = ((original * turns / (2 * math.pi) - 1.0) / 3.0).clamp(0, 1)             # from one turn to four over the original length
        turns = turns * (keep + (1 - keep) / case["factor"])
    else:
        turns = turns / case["factor"]
    angle = positions[..., None].double() * turns
    cos, sin = angle.cos().float()[..., None, :], angle.sin().float()[..., None, :]
    x = x.float()
    y, rest = x[..., :R], x[..., R:]
    if case["interleaved"]:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :R // 2], y[..., R // 2:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, rest], -1).to(_TYPES[case["type"]])


def _plain_prompt(s):
    case, x = s["case"], s["qkv"]
    H, Hk, D, L, S = case["heads"], case["kv_heads"], case["dim"], case["longest"], case["sequences"]
    first, end = s["offsets"][:-1].long(), s["offsets"][1:].long()
    t = torch.arange(L, device=_DEVICE)
    at = first[:, None] + t
    live = at < end[:, None]                                                             # [S][L]
    x = x[at.clamp(max=len(x) - 1)].float().masked_fill_(~live[..., None, None], 0.0)    # [S][L][H + 2 Hk][D]
    q = x[:, :, :H].reshape(S, L, Hk, H // Hk, D).permute(0, 2, 3, 1, 4).reshape(S, Hk, H // Hk * L, D) * D ** -0.5
    k = x[:, :, H:H + Hk].permute(0, 2, 3, 1).contiguous()                               # [S][Hk][D][L]
    v = x[:, :, H + Hk:].permute(0, 2, 1, 3).contiguous()
    score = torch.matmul(q, k).reshape(S, H, L, L)
    score.masked_fill_(t > t[:, None], -math.inf)
    score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = score.sum(-1, keepdim=True)                                                  # [S][H][L][1]
    out = torch.matmul(score.reshape(S, Hk, H // Hk * L, L), v).reshape(S, H, L, D) / total
    return out.transpose(1, 2)[live].to(_TYPES[case["type"]])


def _plain_place(s):
    case, x = s["case"], s["qkv"]
    H, Hk, n, start, counts = case["heads"], case["kv_heads"], case["step"], s["start"].long(), s["counts"]
    turned = _turned(x[..., :H + Hk, :], s["positions"], case)
    t = torch.arange(n, device=_DEVICE)
    at = start[..., None] + t
    live = (t < counts[..., None]) if counts is not None else torch.ones_like(at, dtype=torch.bool)
    row = torch.arange(start.numel(), device=_DEVICE).reshape(start.shape)[..., None].expand_as(at)

    def through(new, cache):
        def part(held, y):
            flat = held.view(-1, *held.shape[-3:])                                       # rows of tokens
            if y.dtype == torch.float8_e4m3fn:                                           # bytes are what is moved
                flat, y = flat.view(torch.uint8), y.view(torch.uint8)
            flat[row[live], at[live]] = y[live]
            got = flat[row, at]
            return got.view(torch.float8_e4m3fn) if held.dtype == torch.float8_e4m3fn else got
        parts = tuple(map(part, cache, _store(new, case["fp8"])))
        return torch.where(live[..., None, None], _load(parts), 0.0).to(_TYPES[case["type"]])
    return turned[..., :H, :].contiguous(), through(turned[..., H:, :], s["k_cache"]), through(x[..., H + Hk:, :], s["v_cache"])


def _plain_adjust(s):
    case, x = s["case"], s["logits"].float()
    P, N, n, V = x.shape
    counts = s["counts"] if s["counts"] is not None else torch.full((P, N), n, device=_DEVICE, dtype=torch.int32)
    t = torch.arange(n, device=_DEVICE)
    end = (s["path_len"] - counts)[..., None] + t + 1                                    # [P][N][n]
    seen = torch.arange(case["path"], device=_DEVICE) < end[..., None]                   # [P][N][n][path]
    tokens = s["tokens"].long()[:, :, None].expand(P, N, n, case["path"])
    times = torch.zeros_like(x).scatter_add_(-1, tokens, seen.float())
    asked = torch.arange(case["prompt"], device=_DEVICE) < s["prompt_len"][:, None]
    in_prompt = torch.zeros((P, V), device=_DEVICE).scatter_add_(-1, s["prompt"].long(), asked.float()) > 0
    repetition, presence, frequency = (y[:, None, None, None] for y in s["penalties"].unbind(-1))
    said = in_prompt[:, None, None] | (times > 0)
    x = torch.where(said, torch.where(x > 0, x / repetition, x * repetition), x)
    x = torch.where(times > 0, x - (frequency * times + presence), x)
    if s["bias"] is not None:
        x = x + s["bias"][:, None, None]
    if s["mask"] is not None:
        v = torch.arange(V, device=_DEVICE)
        x = torch.where((s["mask"][..., v // 32] >> (v % 32).int() & 1) != 0, x, -math.inf)
    return torch.where((t < counts[..., None])[..., None], x, 0.0).to(_TYPES[case["type"]])


def run(state):
    case = state["case"]
    op, H = case["op"], case.get("heads")
    if own:
        from paper_2503_05330_amd import verify
        if op == "adjust":
            return verify.adjust(state["logits"], state["tokens"], state["path_len"], state["counts"], state["prompt"], state["prompt_len"],
                                 state["penalties"], state["bias"], state["mask"])
        x, Hk = state["qkv"], case["kv_heads"]
        if op == "prompt":
            return verify.prompt_attend(x[..., :H, :], x[..., H:H + Hk, :], x[..., H + Hk:, :], state["offsets"])
        if op == "rotate":
            return verify.rotate(x[..., :H + Hk, :], state["positions"], state["rotary"])
        cache, start, counts = state["cache"], state["start"], state["counts"]
        q = cache.write_rotated(0, x[..., :H, :], x[..., H:H + Hk, :], x[..., H + Hk:, :], state["rotary"], state["positions"], start, counts)
        return (q, *cache.read(0, case["step"], start, counts))
    if op == "rotate":
        return _turned(state["qkv"][..., :H + case["kv_heads"], :], state["positions"], case)
    return {"prompt": _plain_prompt, "place": _plain_place, "adjust": _plain_adjust}[op](state)


# ----------------------------------------------------------------------------------------------------------- exact

def _held64(x, fp8):
    """The values that a cache holds of x, from the format's definition: three bits behind the leading one, exponents down
    to -6, below which the spacing stays 2^-9."""
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


def _turned64(x, positions, case):
    """Pairs as complex numbers, times e^(i angle)."""
    R = case["rotated"]
    per_token = torch.tensor([case["base"] ** (-2.0 * i / R) for i in range(R // 2)], dtype=torch.float64, device=_DEVICE)
    over = case["original"] * per_token / (2 * math.pi)                                  # turns over the original length
    share = torch.where(over >= 4, 1.0, torch.where(over <= 1, 0.0, (over - 1) / 3)) if case["original"] else torch.zeros_like(over)
    per_token = share * per_token + (1 - share) * per_token / case["factor"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=_DEVICE), positions.double()[..., None] * per_token)[..., None, :]
    y = x.double().clone()
    if case["interleaved"]:
        z = torch.complex(y[..., 0:R:2], y[..., 1:R:2]) * turn
        y[..., 0:R:2], y[..., 1:R:2] = z.real, z.imag
    else:
        z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * turn
        y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
    return y


def _exact_adjust(s):
    case = s["case"]
    P, N, n, V = s["logits"].shape
    out = torch.zeros((P, N, n, V), dtype=torch.float64, device=_DEVICE)
    path_len, prompt_len = s["path_len"].tolist(), s["prompt_len"].tolist()
    counts = s["counts"].tolist() if s["counts"] is not None else [[n] * N] * P
    for p in range(P):
        rep, pres, freq = s["penalties"][p].double().unbind()
        asked = torch.bincount(s["prompt"][p, :prompt_len[p]], minlength=V) > 0
        for i in range(N):
            for t in range(counts[p][i]):
                times = torch.bincount(s["tokens"][p, i, :path_len[p][i] - counts[p][i] + t + 1], minlength=V)
                x = s["logits"][p, i, t].double()
                x = torch.where(asked | (times > 0), x * torch.where(x > 0, 1 / rep, rep), x) - times * freq - (times > 0) * pres
                if s["bias"] is not None:
                    x = x + s["bias"][p].double()
                if s["mask"] is not None:
                    allowed = s["mask"][p, i, t][:, None].bitwise_right_shift(torch.arange(32, device=_DEVICE, dtype=torch.int32)).bitwise_and(1)
                    x = x.masked_fill(allowed.flatten()[:V] == 0, -math.inf)
                out[p, i, t] = x
    return out


def exact(case, seed):
    if case["op"] == "adjust" and case["problems"] * case["paths"] * case["step"] > 20000:
        return None                                      # (a row after the other: it would take too long)
    s = _inputs(case, seed)
    if case["op"] == "adjust":
        return _exact_adjust(s)
    H, Hk, D, x = case["heads"], case["kv_heads"], case["dim"], s["qkv"]
    if case["op"] == "rotate":
        return _turned64(x[..., :H + Hk, :], s["positions"], case)
    if case["op"] == "place":
        turned = _turned64(x[..., :H + Hk, :], s["positions"], case)
        live = torch.arange(case["step"], device=_DEVICE) < (s["counts"][..., None] if s["counts"] is not None else case["step"])
        # the keys are of the cache's type, as a projection's are, before they are held
        k, v = turned[..., H:, :].to(x.dtype).double(), x[..., H + Hk:, :].double()
        return (turned[..., :H, :], *(torch.where(live[..., None, None], _held64(y, case["fp8"]), 0.0) for y in (k, v)))
    out = torch.empty((len(x), H, D), dtype=torch.float64, device=_DEVICE)
    offsets = s["offsets"].tolist()
    for a, b in zip(offsets, offsets[1:]):
        hidden = torch.ones((b - a, b - a), dtype=torch.bool, device=_DEVICE).triu(1)
        for h in range(H):
            q, k, v = (x[a:b, at].double() for at in (h, H + h // (H // Hk), H + Hk + h // (H // Hk)))
            weight = torch.softmax((q @ k.T / math.sqrt(D)).masked_fill(hidden, -math.inf), -1)
            out[a:b, h] = weight @ v
    return out


# ------------------------------------------------------------------------------------------------------------ work

def work(case):
    """prompt: queries, keys and values once, outputs; two products over what each token sees.  rotate: queries and keys once.  place: those and
    the values, what the cache holds of keys and values written and read again, all written.  adjust: each live logit and its bias
    once, its bit of the mask, the tokens; every logit written."""
    if case["op"] == "adjust":
        rows, V, e = case["problems"] * case["paths"] * case["step"], case["vocab"], _TYPES[case["type"]].itemsize
        live = 15 / 16 * (1 + case["step"]) / 2 / case["step"] if case["ragged"] else 1
        tokens = case["problems"] * (case["prompt"] * 3 / 4 + case["paths"] * (max(case["step"], case["path"] // 4) + case["path"]) / 2)
        return {"bytes": rows * V * e * (1 + live) + (rows * live * V / 8 if case["mask"] else 0) + 4 * tokens +
                (4 * case["problems"] * V if case["bias"] else 0), "flops": rows * live * V * (3 if case["bias"] else 2)}
    H, Hk, D = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "prompt":
        lengths = _lengths(case)
        return {"bytes": sum(lengths) * 4 * (H + Hk) * D, "flops": sum(x * (x + 1) // 2 for x in lengths) * 4 * D * H}
    if case["op"] == "rotate":
        return {"bytes": case["tokens"] * (H + Hk) * D * 4, "flops": case["tokens"] * (H + Hk) * case["rotated"] * 3}
    tokens = case["problems"] * case["paths"] * case["step"]
    live = 15 / 16 * (1 + case["step"]) / 2 / case["step"] if case["ragged"] else 1
    held = 2 * Hk * (D + 1 if case["fp8"] else 2 * D)                                    # bytes of a token, K and V
    return {"bytes": tokens * (4 * H * D + 4 * Hk * D) + tokens * live * (4 * Hk * D + 2 * held),
            "flops": tokens * (H + Hk) * case["rotated"] * 3}

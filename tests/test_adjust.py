"""Penalties, biases and masks on logits against a plain implementation in 64 bits."""
import pytest
import torch

from paper_2503_05330_amd import binding, verify
from test_verify import BF, F16, F32, gen, ints, normal, same  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu
HALF = {BF: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}


def plain(logits, tokens, path_len, counts, prompt, prompt_len, penalties, bias, mask):
    """The result in 64 bits, and what 32-bit steps may be off by beside the last rounding."""
    P, N, n, V = logits.shape
    out, loose = torch.zeros(logits.shape, dtype=torch.float64), torch.zeros(logits.shape, dtype=torch.float64)
    for p in range(P):
        rep, pres, freq = penalties[p].double().tolist() if penalties is not None else (1.0, 0.0, 0.0)
        asked = set(prompt[p, :(prompt_len[p] if prompt_len is not None else None)].tolist()) if prompt is not None else set()
        for i in range(N):
            count = n if counts is None else min(max(counts[p][i], 0), n)
            for t in range(count):
                x = logits[p, i, t].double().cpu()
                times = torch.zeros(V, dtype=torch.float64)
                if tokens is not None:
                    sees = max(0, min(max(path_len[p][i], 0), tokens.shape[-1]) - count + t + 1)
                    for v in tokens[p, i, :sees].tolist():
                        if 0 <= v < V:
                            times[v] += 1
                said = times > 0
                for v in asked:
                    if 0 <= v < V:
                        said[v] = True
                size = x.abs().nan_to_num(0, 0, 0)
                x = torch.where(said, torch.where(x > 0, x / rep, x * rep), x)
                size = size + x.abs().nan_to_num(0, 0, 0)
                x = torch.where(times > 0, x - (freq * times + pres), x)
                size = size + torch.where(times > 0, (abs(freq) * times + abs(pres)), 0.0) * 2
                if bias is not None:
                    b = (bias if bias.dim() == 1 else bias[p]).double().cpu()
                    x, size = x + b, size + b.abs().nan_to_num(0, 0, 0)
                if mask is not None:
                    words = (mask if mask.dim() == 1 else mask[p, i, t]).cpu().long()
                    v = torch.arange(V)
                    x = torch.where((words[v // 32] >> v % 32) & 1 == 1, x, -torch.inf)
                out[p, i, t], loose[p, i, t] = x, size
    return out, loose


def check(logits, tokens=None, path_len=None, counts=None, prompt=None, prompt_len=None, penalties=None, bias=None, mask=None, out=None):
    lists = lambda t: None if t is None else ints(t)
    given = (logits, tokens, lists(path_len), lists(counts), prompt, lists(prompt_len), penalties, bias, mask)
    got = verify.adjust(*given, out=out)
    want, size = plain(logits, tokens, path_len, counts, prompt, prompt_len, penalties, bias, mask)
    dtype = logits.dtype
    assert got.dtype == dtype and got.shape == logits.shape
    result, want = got.double().cpu(), want.to(want.device)
    high = float(torch.finfo(dtype).max) * (1 + HALF[dtype])
    want = torch.where(want.abs() >= high, torch.sign(want) * torch.inf, want)            # what rounds to an infinity
    finite = want.isfinite()
    assert same(result[~finite], want[~finite])
    # one rounding to the type (also below its smallest normal number), and one of 32 bits for each step
    tiny = float(torch.finfo(dtype).tiny) * HALF[dtype] * 2
    error = (result - want).abs() - HALF[dtype] * want.abs() * (1 + 2.0 ** -20) - 2.0 ** -23 * size - tiny
    assert error[finite].max().item() <= 0 if finite.any() else True, error[finite].max().item()
    mine = logits.clone()                                 # in place: the same
    assert verify.adjust(mine, *given[1:], out=mine) is mine
    assert same(mine, got)
    return got


def texts(gen, shape, vocab):
    return (torch.rand(shape, generator=gen, device="cuda") ** 3 * vocab).int()


def some_mask(gen, shape):
    return torch.randint(-1 << 31, 1 << 31, shape, generator=gen, device="cuda", dtype=torch.int64).int()


SHAPES = [  # P, N, n, V, tokens, prompt
    (1, 1, 1, 1, 1, 1), (1, 4, 1, 1000, 64, 256), (2, 3, 5, 4099, 40, 7), (1, 2, 17, 9001, 300, 50), (3, 1, 33, 77, 33, 3), (1, 1, 2, 152064, 600, 2000),
    (2, 2, 3, 31, 9, 9), (1, 3, 4, 32, 200, 0), (1, 2, 2, 50257, 2, 30), (5, 7, 2, 8200, 90, 100)]


@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("ragged", [False, True])
def test_all_together(gen, shape, dtype, ragged):
    P, N, n, V, T, U = SHAPES[shape]
    print(SHAPES[shape], dtype, ragged, flush=True)
    logits = normal(gen, (P, N, n, V), dtype) * 3
    tokens, prompt = texts(gen, (P, N, T), V), texts(gen, (P, U), V)
    path_len = [[max(1, T - 3 * (p + i)) for i in range(N)] for p in range(P)]
    counts = [[(p + 2 * i) % (n + 1) for i in range(N)] for p in range(P)] if ragged else None
    prompt_len = [max(0, U - p) for p in range(P)] if ragged else None
    penalties = torch.tensor([[1.2, 0.5, 0.25], [0.8, -0.3, 0.1], [1.0, 0.0, 0.0], [3.0, 0.0, 0.7], [1.0, 1.5, 0.0]], device="cuda")[:P].contiguous()
    bias, mask = normal(gen, (P, V), F32), some_mask(gen, (P, N, n, -(-V // 32)))
    if ragged:
        bias, mask = bias[0], mask[0, 0, 0]               # one for all
    check(logits, tokens, path_len, counts, prompt, prompt_len, penalties, bias, mask)
    check(logits, tokens, path_len, counts, prompt, prompt_len, penalties)
    check(logits, tokens, path_len, counts, None, None, penalties, None, mask)
    check(logits, None, None, counts, prompt, prompt_len, penalties, bias)
    check(logits, None, None, counts, None, None, None, bias, mask)


def test_the_newest_tokens_count_from_their_position_on(gen):
    """Drafted tokens that repeat each other and the history; a path that is shorter than its count."""
    V = 100
    logits = torch.full((1, 3, 4, V), 2.0, device="cuda")
    tokens = ints([[[5, 5, 7, 9, 7, 7, 11, 0], [1, 2, 3, 4, 5, 6, 7, 8], [8, 8, 8, 8, 8, 8, 8, 8]]])
    penalties = torch.tensor([[1.0, 0.0, 1.0]], device="cuda")
    got = check(logits, tokens, [[7, 2, 8]], [[4, 4, 2]], None, None, penalties)
    # path 0: the history 5 5 7, then 9, 7, 7, 11
    assert got[0, 0, :, 7].tolist() == [1.0, 0.0, -1.0, -1.0] and got[0, 0, :, 5].tolist() == [0.0] * 4
    assert got[0, 0, :, 9].tolist() == [1.0] * 4 and got[0, 0, :, 11].tolist() == [2.0, 2.0, 2.0, 1.0]
    # path 1 has two tokens in all, so its first two positions see none
    assert got[0, 1, :, 1].tolist() == [2.0, 2.0, 1.0, 1.0] and got[0, 1, :, 2].tolist() == [2.0, 2.0, 2.0, 1.0]
    assert got[0, 2, :, 8].tolist() == [-5.0, -6.0, 0.0, 0.0] and not got[0, 2, 2:].any()


@pytest.mark.parametrize("dtype", [BF, F16, F32])
def test_infinities_nan_and_rows_that_nothing_is_left_of(gen, dtype):
    V = 70
    logits = normal(gen, (1, 2, 3, V), dtype)
    logits[0, 0, :, 3], logits[0, 0, :, 4], logits[0, 0, :, 5] = torch.nan, torch.inf, -torch.inf
    logits[0, 1, 0] = torch.nan
    logits[0, 1, 1, :4] = float(torch.finfo(dtype).max)
    tokens, prompt = ints([[[3, 4, 5, 6, 40], [0, 1, 2, 0, 1]]]), ints([[4, 5, 6, 2, 69]])
    penalties = torch.tensor([[0.5, 0.5, 0.5]], device="cuda")
    mask = torch.full((1, 2, 3, 3), -1, dtype=torch.int32, device="cuda")
    mask[0, 0, 1], mask[0, 1, 0] = 0, 0                   # nothing may be picked
    mask[0, 0, 2, 0] &= ~(1 << 3 | 1 << 4)                # what is odd may not
    bias = normal(gen, (V,), F32)
    bias[6], bias[7], bias[5] = -torch.inf, torch.inf, torch.inf
    for b in (None, bias):
        got = check(logits, tokens, [[5, 5]], None, prompt, None, penalties, b, mask)
        assert (got[0, 0, 1] == -torch.inf).all() and (got[0, 1, 0] == -torch.inf).all()
        picked, probs = verify.targets(got)
        assert picked[0, 0, 1] == -1 and probs[0, 0, 1] == 0 and picked[0, 1, 0] == -1
        assert picked[0, 0, 2] not in (3, 4)


def test_tokens_that_are_none_count_for_nothing(gen):
    logits = normal(gen, (1, 1, 2, 1000), BF)
    tokens, prompt = ints([[[-1, 1000, 1 << 30, -(1 << 31), 5, (1 << 31) - 1]]]), ints([[-7, 1003, 999, 1024]])
    check(logits, tokens, [[6]], None, prompt, None, torch.tensor([[1.5, 0.25, 0.25]], device="cuda"))


@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("offset,vocab,stride", [(0, 100, 104), (1, 1001, 1003), (3, 517, 520), (5, 3, 11), (2, 5000, 5001), (7, 33000, 33001)])
def test_rows_at_any_alignment(gen, dtype, offset, vocab, stride):
    wide, to = normal(gen, (2, 3, 2, stride), dtype), torch.full((2, 3, 2, stride + 6), 9.0, dtype=dtype, device="cuda")
    offset = min(offset, stride - vocab)
    tokens, prompt = texts(gen, (2, 3, 50), vocab)[..., 3:], texts(gen, (2, 40), vocab)[:, 1:]
    out = to[..., 3:3 + vocab]
    check(wide[..., offset:offset + vocab], tokens, [[47, 3, 30]] * 2, [[2, 1, 0]] * 2, prompt, None, torch.tensor([[1.5, 0.25, 0.125]] * 2, device="cuda"),
          normal(gen, (2, vocab + 3), F32)[:, 1:vocab + 1], some_mask(gen, (2, 3, 2, -(-vocab // 32) + 2))[..., 1:], out)
    assert (to[..., :3] == 9).all() and (to[..., 3 + vocab:] == 9).all()


def test_long_histories(gen):
    """More of one token than 16 bits count, and histories of a hundred thousand tokens."""
    V, T = 50000, 120000
    tokens = texts(gen, (1, 2, T), V)
    tokens[0, 0, 1000:90000] = 77
    logits = normal(gen, (1, 2, 2, V), F32)
    got = check(logits, tokens, [[T, T - 11]], None, texts(gen, (1, 100000), V), None, torch.tensor([[1.0, 0.0, 1e-3]], device="cuda"))
    assert got[0, 0, 0, 77] < -80


def test_many_paths(gen):
    """More workgroups than one launch takes, and places beyond 2^32 bytes."""
    P, V = 1 << 16, 40000
    logits = torch.ones((P, 1, 1, V), dtype=BF, device="cuda")
    tokens = torch.arange(P, dtype=torch.int32, device="cuda")[:, None, None] % V
    penalties = torch.zeros((P, 3), device="cuda")
    penalties[:, 0], penalties[:, 1] = 1, 2
    verify.adjust(logits, tokens, torch.ones((P, 1), dtype=torch.int32, device="cuda"), None, None, None, penalties, out=logits)
    assert (logits.gather(-1, tokens[:, :, None].long()) == -1).all()
    assert logits[-1, 0, 0].float().sum().item() == V - 2 and int((logits == -1).sum()) == P


def test_another_stream_and_graph_replays(gen):
    P, N, n, V = 2, 3, 4, 5000
    logits, tokens, prompt = normal(gen, (P, N, n, V), BF), texts(gen, (P, N, 60), V), texts(gen, (P, 70), V)
    path_len, counts = ints([[60, 40, 5]] * P), ints([[4, 2, 0]] * P)
    penalties, mask = torch.tensor([[1.25, 0.5, 0.25]] * P, device="cuda"), some_mask(gen, (P, N, n, 157))
    call = lambda: verify.adjust(logits, tokens, path_len, counts, prompt, None, penalties, None, mask)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = call()
    torch.cuda.current_stream().wait_stream(side)
    assert same(there, call())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(4):
        logits.copy_(normal(gen, logits.shape, BF))
        tokens.copy_(texts(gen, tokens.shape, V))
        path_len -= 1
        graph.replay()
        torch.cuda.synchronize()
        assert same(out, call())


def test_arguments_that_are_refused(gen):
    x, tokens, length = normal(gen, (2, 3, 4, 100), BF), texts(gen, (2, 3, 9), 100), ints([[9] * 3] * 2)
    penalties, bias, mask = torch.ones((2, 3), device="cuda"), torch.zeros((2, 100), device="cuda"), some_mask(gen, (2, 3, 4, 4))
    wants = lambda t: t.clone().requires_grad_()
    verify.adjust(x, tokens, length, None, None, None, penalties, bias, mask)
    for call, error in [
        (lambda: verify.adjust(x[0]), TypeError), (lambda: verify.adjust(x.double()), TypeError), (lambda: verify.adjust(x.cpu()), TypeError),
        (lambda: verify.adjust(x, tokens, None, penalties=penalties), ValueError), (lambda: verify.adjust(x, tokens[:1], length), ValueError),
        (lambda: verify.adjust(x, tokens.long(), length), TypeError), (lambda: verify.adjust(x, tokens, length[:1]), ValueError),
        (lambda: verify.adjust(x, tokens, length.cpu()), TypeError), (lambda: verify.adjust(x, counts=ints([1])), ValueError),
        (lambda: verify.adjust(x, penalties=penalties[:1]), ValueError), (lambda: verify.adjust(x, penalties=penalties.half()), TypeError),
        (lambda: verify.adjust(x, bias=bias[:, :99]), ValueError), (lambda: verify.adjust(x, bias=bias.half()), TypeError),
        (lambda: verify.adjust(x, bias=bias[:1]), ValueError), (lambda: verify.adjust(x, mask=mask[..., :3]), ValueError),
        (lambda: verify.adjust(x, mask=mask.long()), TypeError), (lambda: verify.adjust(x, mask=mask[:1]), ValueError),
        (lambda: verify.adjust(x, prompt=tokens), ValueError), (lambda: verify.adjust(x, out=x[..., :50]), ValueError),
        (lambda: verify.adjust(x[..., :50], out=x[..., 20:70]), ValueError), (lambda: verify.adjust(x, out=x.float()), ValueError),
        (lambda: verify.adjust(x[..., ::2]), ValueError), (lambda: verify.adjust(wants(x)), TypeError),
        (lambda: verify.adjust(x, bias=wants(bias)), TypeError), (lambda: verify.adjust(x.repeat(1, 1, 9, 1)), binding.CsdError),
        (lambda: verify.adjust(x, out=torch.zeros((), dtype=BF, device="cuda").expand(2, 3, 4, 100)), ValueError),
        (lambda: verify.adjust(x, out=torch.zeros(100, dtype=BF, device="cuda").expand(2, 3, 4, 100)), binding.CsdError),
    ]:
        with pytest.raises(error):
            call()

"""The verifying pass's operators (cache, attention over it, targets) against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2503_05330_amd import binding, verify

pytestmark = pytest.mark.gpu

BF, F16, F32 = torch.bfloat16, torch.float16, torch.float32
ROUND = {BF: 2.0 ** -8, F16: 2.0 ** -11}                 # half a unit in the last place, relative


def held(x, fp8):
    """What a cache holds of x [..., head_dim]: x, or what its e4m3 codes and scale stand for, in 64 bits."""
    x = x.double().cpu()
    if not fp8:
        return x
    size = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1, keepdim=True)
    power = torch.full_like(size, -126.0)
    for e in range(-126, 128):                           # the least power of two that takes the largest to 448
        power = torch.where(size > 448 * 2.0 ** power, power + 1, power)
    power = torch.where(size == 0, 0.0, power)
    y = (x * 2.0 ** -power).clamp(-448, 448)
    grain = 2.0 ** ((torch.frexp(y)[1].double() - 1).clamp(min=-6) - 3)
    return torch.where(y.isnan(), y, torch.round(y / grain) * grain * 2.0 ** power)


def same(a, b):
    """Equal, with NaN equal to NaN."""
    return torch.equal(torch.nan_to_num(a.double().cpu(), nan=1e300), torch.nan_to_num(b.double().cpu(), nan=1e300))


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


@pytest.fixture
def gen():
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    return g


# ------------------------------------------------------------------------------------------------------------ cache

@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dim,kv_heads,P,N,n,cap", [(128, 8, 2, 3, 1, 37), (64, 1, 1, 5, 9, 64), (96, 3, 3, 2, 17, 45), (256, 2, 1, 2, 70, 101),
                                                    (128, 2, 2, 1, 8, 32), (64, 5, 1, 70, 2, 3)])
def test_written_rows_are_read_back_and_others_stay(gen, dtype, fp8, dim, kv_heads, P, N, n, cap):
    print(dtype, fp8, dim, kv_heads, P, N, n, cap, flush=True)
    c = verify.PathCache(P, N, 0, cap, kv_heads, kv_heads, dim, 1, n_layers=2, dtype=dtype, fp8=fp8)
    want = [torch.zeros((2, P, N, cap, kv_heads, dim), dtype=torch.float64) for _ in range(2)]
    zero = torch.zeros((P, N, cap, kv_heads, dim), dtype=dtype, device="cuda")
    for layer in range(2):
        c.write(layer, zero, zero)
    for turn in range(3):                                # the later ones write over parts of the earlier ones
        layer = turn % 2
        if turn == 1:                                    # slices of a projection's output
            kv = normal(gen, (P, N, n, 3 * kv_heads, dim), dtype)
            k, v = kv[..., kv_heads:2 * kv_heads, :], kv[..., 2 * kv_heads:, :]
        else:
            k, v = normal(gen, (P, N, n, kv_heads, dim), dtype) * 100, normal(gen, (P, N, n, kv_heads, dim), dtype) / 1000
        start = torch.randint(0, cap - n + 1, (P, N), generator=gen, device="cuda", dtype=torch.int32)
        counts = torch.randint(0, n + 1, (P, N), generator=gen, device="cuda", dtype=torch.int32) if turn else None
        c.write(layer, k, v, start, counts)
        got = c.read(layer, n, start, counts)
        for x, y, z in zip((k, v), want, got):
            x = held(x, fp8)
            for p in range(P):
                for i in range(N):
                    m, s = n if counts is None else int(counts[p, i]), int(start[p, i])
                    y[layer, p, i, s:s + m] = x[p, i, :m]
                    assert not z[p, i, m:].any()
                    assert same(z[p, i, :m], x[p, i, :m].to(dtype))
    for layer in range(2):
        for y, z in zip(want, c.read(layer, cap)):
            assert same(z, y[layer].to(dtype))
    assert c.status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_prompts_are_held_apart_from_paths(gen, fp8):
    P, N, T, U, H, D = 3, 2, 50, 40, 2, 64
    c = verify.PathCache(P, N, T, U, H, H, D, 1, fp8=fp8)
    pk, pv = normal(gen, (P, T, H, D), BF), normal(gen, (P, T, H, D), BF)
    k, v = normal(gen, (P, N, U, H, D), BF), normal(gen, (P, N, U, H, D), BF)
    c.write_prompt(0, pk[:, :30], pv[:, :30])
    c.write(0, k, v)
    c.write_prompt(0, pk[:, 20:], pv[:, 20:], ints([20] * P))
    for x, y in zip((pk, pv), c.read_prompt(0, T)):
        assert same(held(x, fp8).to(BF), y)
    for x, y in zip((k, v), c.read(0, U)):
        assert same(held(x, fp8).to(BF), y)
    got = c.read_prompt(0, 9, ints([0, 45, 49]), ints([9, 9, 3]))[0]      # past the end: zeros
    assert same(got[0], held(pk[0, :9], fp8).to(BF))
    assert same(got[1, :5], held(pk[1, 45:], fp8).to(BF)) and not got[1, 5:].any()
    assert same(got[2, :1], held(pk[2, 49:], fp8).to(BF)) and not got[2, 1:].any()


@pytest.mark.parametrize("dtype", [BF, F16])
def test_eight_bit_codes_of_special_values(dtype):
    """Infinities saturate, NaN stays, zero and the smallest and largest numbers keep their scales; every 16-bit number that
    an e4m3 number stands for comes back as it is, and halves between two of them go to the even one."""
    D, big = 64, float(torch.finfo(dtype).max)
    rows = torch.zeros((9, D), dtype=torch.float64)
    rows[1, 0], rows[1, 1], rows[1, 2] = float("inf"), float("-inf"), 3.0
    rows[2, 5], rows[2, 6] = float("nan"), 1.0
    rows[3, 0], rows[3, 1] = float("inf"), float("nan")                  # nothing finite but zeros
    rows[4, 0], rows[4, 1], rows[4, 2] = big, -big / 3, big / 1000
    rows[5, :3] = float(torch.finfo(dtype).tiny)
    rows[6] = torch.arange(D) / 8 + 8                                      # halves at 16 .. : spacing there is 2 * 2^-k
    rows[7, 0], rows[7, 1:] = 448.0, torch.arange(1, D) * 2.0 ** -10       # down to half of the smallest code
    rows[8, 0], rows[8, 1] = 449.0, 448.0                                  # the next power of two
    x = rows.to(dtype).cuda().reshape(1, 1, 9, 1, D)
    c = verify.PathCache(1, 1, 0, 16, 1, 1, D, 1, dtype=dtype, fp8=True)
    c.write(0, x, x.flip(-1))
    k, v = c.read(0, 9)
    assert same(k, held(x, True).to(dtype)) and same(v, held(x.flip(-1), True).to(dtype))


@pytest.mark.parametrize("dtype,least,most", [(BF, -133, 127), (F16, -24, 15)])
@pytest.mark.parametrize("odd", [False, True])
def test_eight_bit_codes_at_every_size(gen, dtype, least, most, odd):
    """Tokens of every magnitude of the type, subnormal ones among them, each rounded once to what its scale allows; a token
    with an infinity beside them changes nothing."""
    D = 128
    sizes = 2.0 ** torch.arange(least, most + 1, device="cuda", dtype=torch.float64)
    x = torch.rand((len(sizes), D), generator=gen, device="cuda", dtype=torch.float64) * sizes[:, None]
    x = (x * torch.sign(torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.float64))).to(dtype)
    x[:, :D // 4] *= 2.0 ** -9                           # the codes' own subnormal numbers
    if odd:
        x[::8, 5] = float("inf")
    c = verify.PathCache(1, 1, 0, len(x), 1, 1, D, 1, dtype=dtype, fp8=True)
    c.write(0, x[None, None, :, None], x.flip(-1)[None, None, :, None])
    k, v = c.read(0, len(x))
    want = held(x, True).to(dtype)
    assert same(k[0, 0, :, 0], want) and same(v[0, 0, :, 0], want.flip(-1))


@pytest.mark.parametrize("prompt", [False, True])
def test_positions_outside_of_the_cache_are_dropped_and_reported(gen, prompt):
    P, N, cap, H, D = 2, 2, 40, 2, 64
    c = verify.PathCache(P, N, cap, cap, H, H, D, 1)
    lead = (P,) if prompt else (P, N)
    write, read = (c.write_prompt, c.read_prompt) if prompt else (c.write, c.read)
    zero = torch.zeros((*lead, cap, H, D), dtype=BF, device="cuda")
    c.write_prompt(0, zero if prompt else zero[:, 0], zero if prompt else zero[:, 0])
    c.write(0, zero[:, None].expand(P, N, cap, H, D).contiguous() if prompt else zero, zero[:, None].expand(P, N, cap, H, D).contiguous() if prompt else zero)
    assert c.status() == 0
    k = normal(gen, (*lead, 12, H, D), BF)
    start = ints([-5, 33]) if prompt else ints([[-5, 33], [2 ** 31 - 5, -2 ** 31]])
    write(0, k, k, start)
    assert c.status() == binding.STATUS_CAPACITY
    want = torch.zeros((*lead, cap, H, D), dtype=BF, device="cuda")
    flat, src = want.view(-1, cap, H, D), k.view(-1, 12, H, D)
    flat[0, :7], flat[1, 33:] = src[0, 5:], src[1, :7]
    got = read(0, cap)
    assert torch.equal(got[0], want) and torch.equal(got[1], want)
    other = (c.read if prompt else c.read_prompt)(0, cap)
    assert not other[0].any() and not other[1].any()


# -------------------------------------------------------------------------------------------------------- attention

def plain_attend(q, prompt, path, prompt_len, path_len, counts, scale):
    """out, lse, and sum_x w_x |v_x|, all in 64 bits; prompt, path: (k, v) in 64 bits."""
    P, N, n, H, D = q.shape
    G = H // prompt[0].shape[-2]
    out = torch.zeros((P, N, n, H, D), dtype=torch.float64)
    lse = torch.full((P, N, n, H), -torch.inf, dtype=torch.float64)
    size = torch.zeros_like(out)
    for p in range(P):
        for i in range(N):
            for t in range(counts[p][i]):
                sees = max(0, path_len[p][i] - counts[p][i] + t + 1)
                k, v = (torch.cat([a[p, :prompt_len[p]], b[p, i, :sees]]).repeat_interleave(G, 1) for a, b in zip(prompt, path))
                if len(k) == 0:
                    continue
                s = (k * q[p, i, t].double()).sum(-1) * scale               # [tokens][H]
                lse[p, i, t] = torch.logsumexp(s, 0)
                w = torch.softmax(s, 0)[..., None]
                out[p, i, t], size[p, i, t] = (w * v).sum(0), (w * v.abs()).sum(0)
    return out, lse, size


def check_attend(gen, P, N, n, H, Hk, D, prompt_len, path_len, counts, dtype=BF, fp8=False, caps=None, bounds=(0, 0), poison=None, scale=None,
                 layer=0, fused=True):
    T, U = caps or (max(prompt_len), max(max(map(max, path_len)), n))
    scale = D ** -0.5 if scale is None else scale
    c = verify.PathCache(P, N, T, U, H, Hk, D, n, n_layers=layer + 1, dtype=dtype, fp8=fp8)
    c._buf.fill_(255)                                    # what is not written is NaN, with scales that are none
    pk, pv = normal(gen, (P, max(T, 1), Hk, D), dtype), normal(gen, (P, max(T, 1), Hk, D), dtype)
    k, v = normal(gen, (P, N, U, Hk, D), dtype), normal(gen, (P, N, U, Hk, D), dtype)
    if poison is not None:
        poison(pk, pv, k, v)
    lengths = ints(prompt_len)
    if T:
        c.write_prompt(layer, pk, pv, None, lengths)     # no more than the lengths
    c.write(layer, k, v, None, ints(path_len))
    if fused:
        q = normal(gen, (P, N, n, H + 2 * Hk, D), dtype)[..., :H, :]
    else:
        q = normal(gen, (P, N, n, H, D), dtype)
    lse = torch.full((P, N, n, H), 77.0, device="cuda")
    out = torch.full((P, N, n, H, D), 77.0, dtype=dtype, device="cuda")
    got = c.attend(layer, q, lengths, ints(path_len), None if counts is None else ints(counts), scale, out, lse, *bounds)
    assert got is out
    counts = counts or [[n] * N] * P
    held_prompt, held_path = (held(pk, fp8), held(pv, fp8)), (held(k, fp8), held(v, fp8))
    want, want_lse, size = plain_attend(q.cpu(), held_prompt, held_path, prompt_len, path_len, counts, scale)
    # rounding of the weights and of the result to the type; scores and sums in 32 bits; half precision's smallest weights
    tokens = T + U
    length = lambda x: x.nan_to_num(0, 0, 0).norm(dim=-1).max().item()
    score = abs(scale) * length(q.double()) * max(length(held_prompt[0]), length(held_path[0]))
    loose = 2 * ((D + 4) * 2.0 ** -24 * score + (tokens + 8) * 2.0 ** -24)
    high = max(x.nan_to_num(0, 0, 0).abs().max().item() for x in (held_prompt[1], held_path[1]))
    error = ROUND[dtype] * (want.abs() + size) + loose * size + tokens * 2.0 ** -24 * high
    got, lse = got.double().cpu(), lse.double().cpu()
    finite = want.isfinite()
    assert torch.equal(torch.nan_to_num(got[~finite], nan=1e300), torch.nan_to_num(want[~finite].to(dtype).double(), nan=1e300))
    worst = ((got - want).abs() - error)[finite].max().item()
    assert worst <= 0, worst
    empty = want_lse == -torch.inf
    assert torch.equal(empty, lse == -torch.inf) and not got[empty].any()
    fine = want_lse.isfinite()
    assert ((lse - want_lse).abs()[fine] <= loose + 2.0 ** -22 * (1 + want_lse.abs()[fine])).all()
    return c


SHAPES = [  # P, N, n, H, Hk, D, prompt lengths, path lengths, counts
    (1, 4, 1, 8, 2, 128, [70], [[1, 2, 33, 64]], None),
    (1, 3, 9, 8, 2, 128, [31], [[9, 40, 10]], [[9, 0, 3]]),
    (2, 3, 5, 14, 2, 64, [0, 33], [[5, 7, 64], [37, 6, 5]], [[5, 1, 2], [3, 5, 4]]),
    (1, 2, 17, 28, 4, 128, [257], [[17, 300]], [[17, 11]]),
    (2, 2, 3, 6, 6, 96, [65, 1], [[3, 50], [4, 31]], None),
    (1, 2, 2, 4, 1, 256, [96], [[2, 77]], None),
    (1, 2, 33, 5, 1, 64, [40], [[33, 64]], [[33, 30]]),
    (1, 1, 1, 1, 1, 64, [0], [[1]], None),
    (3, 2, 2, 4, 2, 64, [0, 0, 5], [[0, 1], [2, 0], [0, 0]], [[1, 2], [2, 1], [2, 0]]),   # rows that see nothing, or less than is new
    (1, 5, 1, 8, 8, 128, [1500], [[700, 1, 650, 1000, 33]], None),                         # long axes: split and joined
    (1, 70, 4, 4, 2, 64, [600], [[4 + i % 7 for i in range(70)]], [[i % 5 for i in range(70)]]),
]


@pytest.mark.parametrize("dtype,fp8", [(BF, False), (BF, True), (F16, False), (F16, True)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention(gen, shape, dtype, fp8):
    print(SHAPES[shape], dtype, fp8, flush=True)
    check_attend(gen, *SHAPES[shape], dtype=dtype, fp8=fp8, layer=shape % 2, fused=shape % 3 > 0)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("P,N,H,Hk,prompt,path", [(33, 8, 4, 4, 573, 16), (33, 31, 8, 8, 36, 31), (13, 4, 8, 8, 1143, 251), (13, 6, 8, 8, 1104, 553)])
def test_more_items_of_prompts_and_of_paths_than_are_dealt_at_once(gen, P, N, H, Hk, prompt, path, fp8):
    """Some hundred workgroups each of prompts' and of paths' items, the longer ones the prompts' or the paths'."""
    lengths = [prompt - 31 * p % prompt for p in range(P)]
    paths = [[1 + (p * N + i) * 53 % path for i in range(N)] for p in range(P)]
    counts = [[int((p + i) % 5 > 0) for i in range(N)] for p in range(P)]
    check_attend(gen, P, N, 1, H, Hk, 64, lengths, paths, counts, fp8=fp8, caps=(prompt, path))


@pytest.mark.parametrize("P,N,n,H,Hk,D", [(7, 5, 2, 8, 2, 64), (15, 3, 3, 4, 1, 128), (23, 2, 4, 8, 1, 64)])
def test_problems_and_heads_that_are_no_multiple_of_eight(gen, P, N, n, H, Hk, D):
    paths = [[n + (p * N + i) * 7 % 30 for i in range(N)] for p in range(P)]
    check_attend(gen, P, N, n, H, Hk, D, [9 * p % 66 for p in range(P)], paths, None, caps=(65, 40))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("caps", [(64, 64), (2048, 64), (640, 1024)])
def test_lengths_anywhere_below_the_capacities(gen, caps, fp8):
    """A launch is shaped by the capacities, or by the bounds; lengths are what they are."""
    for prompt, paths in ((0, [[1, 2, 3]]), (64, [[64, 33, 32]]), (min(caps[0], 600), [[2, 60, min(caps[1], 900)]])):
        for bounds in ((0, 0), (1, 1)):
            check_attend(gen, 1, 3, 2, 8, 2, 64, [prompt], paths, [[1, 2, 2]], fp8=fp8, caps=caps, bounds=bounds)


@pytest.mark.parametrize("dtype,fp8", [(BF, False), (BF, True), (F16, False)])
@pytest.mark.parametrize("prompt_len", [40, 700])
def test_what_a_token_does_not_see_does_not_reach_it(gen, dtype, fp8, prompt_len):
    """Infinities and NaN in the newest tokens' keys and values: rejected drafts' places, and later tokens of the step."""
    def poison(pk, pv, k, v):
        v[0, 0, 35, :, 3], k[0, 0, 36, :, 5] = float("nan"), float("nan")
        v[0, 1, 31, :, 0], v[0, 1, 33, :, 1] = float("inf"), float("-inf")
        v[0, 2, 12], k[0, 2, 12] = float("nan"), float("inf")             # beyond the length
        pv[0, prompt_len - 1, :, 7] = float("inf")                         # seen by all
    check_attend(gen, 1, 3, 6, 8, 2, 64, [prompt_len], [[37, 34, 12]], [[6, 6, 4]], dtype=dtype, fp8=fp8, caps=(prompt_len, 64), poison=poison)


@pytest.mark.parametrize("dtype,fp8", [(BF, False), (BF, True), (F16, True)])
def test_values_and_keys_of_very_different_sizes(gen, dtype, fp8):
    """Weights that are concentrated on single tokens, and values (so scales) that differ by 2^18."""
    def poison(pk, pv, k, v):
        k[:, :, ::5] *= 6
        v[:, :, ::3] *= 2.0 ** 9
        pv[:, 1::3] *= 2.0 ** -9
        v[:, :, 7], pv[:, 4] = 0, 0
    check_attend(gen, 1, 2, 3, 4, 2, 64, [100], [[64, 61]], None, dtype=dtype, fp8=fp8, poison=poison)


def test_scores_far_below_and_above_zero(gen):
    def poison(pk, pv, k, v):
        k *= 40
        pk *= 40
    for scale in (1.0, -0.5):
        check_attend(gen, 1, 2, 3, 4, 2, 64, [100], [[64, 61]], None, poison=poison, scale=scale)


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("fp8", [False, True])
def test_a_scale_of_zero_weighs_all_that_is_seen_alike(gen, dtype, fp8):
    check_attend(gen, 1, 2, 3, 4, 2, 128, [100], [[64, 61]], None, dtype=dtype, fp8=fp8, scale=0.0)


def test_a_cache_beyond_32_bit_offsets(gen):
    """A path whose keys and values start behind 4 GB, and one of a million tokens that all weigh the same."""
    U, D, Hk = 1 << 20, 128, 4
    c = verify.PathCache(1, 3, 0, U, Hk, Hk, D, 2)
    assert c._buf.numel() > 3 << 31
    c._buf.zero_()
    k = torch.zeros((1, 3, 2, Hk, D), dtype=BF, device="cuda")
    v = torch.ones_like(k) * 2.0 ** 14 * torch.arange(1, Hk + 1, device="cuda", dtype=BF)[:, None]
    length = ints([[5, U - 1, U]])
    c.write(0, k, v, length - 2)
    got = c.read(0, 2, length - 2)
    assert torch.equal(got[0], k) and torch.equal(got[1], v)
    out = c.attend(0, normal(gen, (1, 3, 2, Hk, D), BF), None, length)
    tokens = torch.tensor([[4, 5], [U - 2, U - 1], [U - 1, U]], dtype=torch.float64)
    want = torch.arange(1, Hk + 1) * 2.0 ** 14 * torch.tensor([1, 2]) [None, :, None] / tokens[..., None]
    assert ((out[0].double().cpu() - want[..., None]).abs() <= (ROUND[BF] + 2.0 ** -12) * want[..., None]).all()


def test_another_stream_and_graph_replays(gen):
    P, N, n, H, Hk, D, T, U = 1, 4, 3, 8, 2, 64, 700, 600
    c = verify.PathCache(P, N, T, U, H, Hk, D, n, fp8=True)
    pk, k = normal(gen, (P, T, Hk, D), BF), normal(gen, (P, N, U, Hk, D), BF)
    new, q = normal(gen, (P, N, n, Hk, D), BF), normal(gen, (P, N, n, H, D), BF)
    logits = normal(gen, (P, N, n, 5001), BF)
    length, total = ints([[300, 17, 5, 590]]), ints([[303, 20, 8, 593]])
    prompt_len = ints([690])

    def program():
        c.write(0, new, new, length)
        return c.attend(0, q, prompt_len, total), *verify.targets(logits)
    c.write_prompt(0, pk, pk)
    c.write(0, k, k)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        program()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = program()
    torch.cuda.synchronize()
    for turn in range(4):                                # other inputs and lengths at each replay
        new.copy_(normal(gen, new.shape, BF))
        q.copy_(normal(gen, q.shape, BF))
        logits.copy_(normal(gen, logits.shape, BF))
        length += 1
        total += 1
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        want = program()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), turn


def test_the_same_call_gives_the_same_bits(gen):
    c = verify.PathCache(1, 6, 3000, 500, 8, 2, 128, 4)
    for write, shape in ((c.write_prompt, (1, 3000, 2, 128)), (c.write, (1, 6, 500, 2, 128))):
        write(0, normal(gen, shape, BF), normal(gen, shape, BF))
    q, length = normal(gen, (1, 6, 4, 8, 128), BF), ints([[500, 400, 300, 4, 100, 5]])
    first = c.attend(0, q, None, length)
    for _ in range(5):
        assert torch.equal(first, c.attend(0, q, None, length))


def test_arguments_that_are_refused(gen):
    c = verify.PathCache(2, 3, 16, 16, 8, 2, 64, 4)
    q, length = normal(gen, (2, 3, 4, 8, 64), BF), ints([[4] * 3] * 2)
    k = normal(gen, (2, 3, 4, 2, 64), BF)
    with pytest.raises(TypeError):
        c.attend(0, q.half(), None, length)
    with pytest.raises(TypeError):
        c.attend(0, q, None, length.long())
    with pytest.raises(TypeError):
        c.attend(0, q.cpu(), None, length)
    with pytest.raises(ValueError):
        c.attend(0, q[:, :2], None, length)
    with pytest.raises(ValueError):
        c.attend(0, q, None, length[:1].contiguous())
    with pytest.raises(TypeError):
        c.attend(0, q.transpose(1, 2).contiguous().transpose(1, 2), None, length)      # paths not evenly spaced
    with pytest.raises(ValueError):
        c.attend(0, torch.cat([q, q], -1).view(-1)[4:4 + q.numel()].view(q.shape), None, length)   # 8 bytes off
    for bad in (dict(layer=1), dict(layer=-1), dict(scale=float("nan")), dict(prompt_bound=-1)):
        with pytest.raises(binding.CsdError) as err:
            c.attend(**{**dict(layer=0, q=q, prompt_len=None, path_len=length), **bad})
        assert err.value.code == binding.ERR_INVALID_ARG
    with pytest.raises(binding.CsdError):                # more than max_step
        c.attend(0, normal(gen, (2, 3, 5, 8, 64), BF), None, length)
    with pytest.raises(binding.CsdError):                # a path's length is needed
        c.attend(0, q, None, None)
    with pytest.raises(ValueError):
        c.write(0, k, k[:, :, :3])
    with pytest.raises(ValueError):
        c.write(0, normal(gen, (2, 3, 4, 3, 64), BF), k)
    with pytest.raises(binding.CsdError):
        c.write(2, k, k)
    with pytest.raises(binding.CsdError):
        c.read(0, 0)
    with pytest.raises(TypeError):
        verify.PathCache(1, 1, 1, 1, 1, 1, 64, 1, dtype=F32)
    with pytest.raises(TypeError):
        verify.targets(length)
    with pytest.raises(TypeError):
        verify.targets(normal(gen, (3, 100), BF), normal(gen, (3, 100), BF))
    with pytest.raises(TypeError):
        verify.targets(normal(gen, (100, 3), BF).t())
    with pytest.raises(binding.CsdError):
        verify.targets(normal(gen, (3, 100), BF), inv_temperature=0.0)
    with pytest.raises(binding.CsdError):
        verify.targets(torch.empty((0, 100), dtype=BF, device="cuda"))


# ----------------------------------------------------------------------------------------------------------- targets

def check_targets(logits, noise=None, inv_temperature=1.0):
    tokens, probs = verify.targets(logits, noise, inv_temperature)
    x = logits.float().cpu().reshape(-1, logits.shape[-1])
    x = torch.where(x.isnan(), -torch.inf, x)
    y = x * np.float32(inv_temperature)
    z = x if noise is None else y + noise.cpu().reshape(x.shape)         # as it is rounded
    z = torch.where(z.isnan(), -torch.inf, z)
    best = z.amax(-1, keepdim=True)
    want = (z == best).int().argmax(-1)                  # the first
    some = best[:, 0] > -torch.inf
    y = x.double() * np.float32(inv_temperature)
    weight = torch.where(y.amax(-1, keepdim=True) == torch.inf, (y == torch.inf).double(), (y - y.amax(-1, keepdim=True)).exp())
    prob = torch.where(some, weight.gather(1, want[:, None])[:, 0] / weight.sum(-1), 0.0)
    assert tokens.dtype == torch.int32 and tokens.shape == logits.shape[:-1] == probs.shape
    assert torch.equal(tokens.cpu().reshape(-1).long(), torch.where(some, want, -1))
    # y and its distance to the largest are rounded once each, and the product with log2(e): |y| and |y - top| times 2^-24;
    # then the exponentials and their sum, of which a thread, a wave and a workgroup add up their parts
    finite = torch.where(y.isfinite(), y.abs(), 0.0).amax(-1)
    bound = (2.0 ** -24 * (6 * finite + 40 + x.shape[1] / 512)) * prob
    assert ((probs.double().cpu().reshape(-1) - prob).abs() <= bound + 1e-37).all()


@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("noisy", [False, True])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 2), (2, 7), (5, 8), (4, 1000), (3, 4099), (2, 32000), (1, 152064), (600, 777), (7, 60001), (520, 152064)])
def test_targets(gen, dtype, noisy, rows, vocab):
    print(dtype, noisy, rows, vocab, flush=True)
    x = (normal(gen, (rows, vocab), F32) * 3).to(dtype)
    noise = -(-torch.rand((rows, vocab), generator=gen, device="cuda").clamp(min=1e-30).log()).log() if noisy else None
    check_targets(x, noise, 0.7 if noisy else 1.0)
    if rows > 1:
        check_targets(x.view(1, rows, vocab), None if noise is None else noise.view(1, rows, vocab), 2.5)


@pytest.mark.parametrize("dtype", [BF, F16, F32])
@pytest.mark.parametrize("offset,vocab,stride", [(0, 100, 104), (1, 1001, 1003), (3, 517, 520), (7, 9, 9), (5, 3, 11), (2, 5000, 5001)])
def test_rows_at_any_alignment(gen, dtype, offset, vocab, stride):
    data = normal(gen, (6 * stride + 8,), F32)
    x = data.to(dtype)[offset:offset + 6 * stride].view(6, stride)[:, :vocab]
    noise = normal(gen, (6 * stride + 8,), F32)[1:1 + 6 * stride].view(6, stride)[:, :vocab]
    check_targets(x)
    check_targets(x, noise, 1.5)


def test_ties_infinities_and_rows_without_a_token(gen):
    inf, nan = float("inf"), float("nan")
    x = normal(gen, (12, 3001), BF)
    x[0] = 0                                             # all equal
    x[1, 5::700] = 9                                     # equal ones in different threads
    x[2] = -inf
    x[3] = nan
    x[4] = -inf
    x[4, 2999] = -5
    x[5, 77], x[5, 78] = nan, 3.5
    x[6, 100], x[6, 2000] = inf, inf
    x[7] = torch.finfo(BF).min                           # masked by the type's lowest value
    x[7, 1234] = 0
    x[8] = torch.finfo(BF).min
    x[9, ::2] = -inf
    x[10, :8], x[10, 8:] = nan, -inf
    x[11, 3000] = 300
    check_targets(x)
    check_targets(x, torch.zeros(x.shape, device="cuda"), 1.0)
    noise = normal(gen, x.shape, F32)
    noise[0, 3], noise[1, 4], noise[9, 2] = inf, nan, inf
    check_targets(x, noise, 1.0)


def test_calls_in_native_code_and_in_python_do_the_same(gen, monkeypatch):
    class Never:
        def __getattr__(self, name):
            return lambda *args: None
    c = verify.PathCache(2, 3, 70, 50, 8, 2, 64, 4, n_layers=2, fp8=True)
    kv = normal(gen, (2, 3, 9, 6, 64), BF)
    k, v = kv[..., 2:4, :], kv[..., 4:, :]
    pk = normal(gen, (2, 90, 2, 64), BF)[:, 10:80]
    q, start = normal(gen, (2, 3, 4, 8, 64), BF), ints([[0, 5, 41], [7, 8, 30]])
    counts, length = ints([[9, 4, 9], [0, 9, 1]]), ints([[9, 9, 50], [8, 17, 31]])
    logits, noise = normal(gen, (2, 3, 4, 501), F16)[..., 100:], normal(gen, (2, 3, 4, 501), F32)[..., :401]

    def calls():
        for layer in range(2):
            for write, shape in ((c.write, (2, 3, 50, 2, 64)), (c.write_prompt, (2, 70, 2, 64))):
                zero = torch.zeros(shape, dtype=BF, device="cuda")
                write(layer, zero, zero)
        c.write(1, k, v, start, counts)
        c.write_prompt(1, pk, pk.flip(-1), None, ints([70, 33]))
        yield from c.read(1, 12, start)
        yield from c.read_prompt(0, 70)
        yield from c.read_prompt(1, 70, None, ints([50, 70]))
        yield c.attend(1, q, ints([70, 33]), length, ints([[4, 1, 2], [0, 3, 4]]))
        yield c.attend(1, q, None, length, None, 0.3, prompt_bound=70, path_bound=50)
        yield from verify.targets(logits, noise, 0.9)
        yield from verify.targets(logits.float())
    native = list(calls())
    assert verify._native is not None and len(native) == 12
    monkeypatch.setattr(verify, "_native", Never())
    assert all(torch.equal(a, b) for a, b in zip(native, calls()))

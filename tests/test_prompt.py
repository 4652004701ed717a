"""Attention of packed prompts to themselves, and their way into the cache, against plain implementations in 64 bits."""
import pytest
import torch

from paper_2503_05330_amd import binding, verify
from test_verify import BF, F16, ROUND, gen, held, ints, normal, same  # noqa: F401 (gen: a fixture)

pytestmark = pytest.mark.gpu


def plain(q, k, v, offsets, scale):
    """out, lse and sum of |weight * value| of q [T][H][D], k, v [T][Hk][D], in 64 bits; zeros (lse -inf) for tokens of no sequence."""
    T, H, D = q.shape
    G = H // k.shape[1]
    q, k, v = (x.double() for x in (q, k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)))
    out, size = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((T, H), -torch.inf, dtype=torch.float64, device=q.device)
    for a, b in zip(offsets, offsets[1:]):
        hidden = torch.ones((b - a, b - a), dtype=torch.bool, device=q.device).triu(1)
        for h in range(H):
            s = (q[a:b, h] @ k[a:b, h].T * scale).masked_fill(hidden, -torch.inf)
            lse[a:b, h] = torch.logsumexp(s, -1)
            w = torch.softmax(s, -1)
            odd = ~v[a:b, h].isfinite()
            fine = torch.where(odd, 0.0, v[a:b, h])
            out[a:b, h], size[a:b, h] = w @ fine, w @ fine.abs()
            for x in odd.any(-1).nonzero()[:, 0].tolist():                # seen by the tokens from x on
                out[a + x:b, h] += torch.where(odd[x], w[x:, x, None] * v[a + x, h], 0.0)
    return out, lse, size


def check(gen, lengths, H, Hk, D, dtype=BF, fused=True, poison=None, scale=None, before=0, behind=0):
    T = before + sum(lengths) + behind
    offsets = [before]
    for x in lengths:
        offsets.append(offsets[-1] + x)
    scale = D ** -0.5 if scale is None else scale
    if fused:
        qkv = normal(gen, (T, H + 2 * Hk, D), dtype)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    else:
        q, k, v = normal(gen, (T, H, D), dtype), normal(gen, (Hk, T, D), dtype).transpose(0, 1), normal(gen, (T, Hk, D), dtype)
    if poison is not None:
        poison(q, k, v)
    out = torch.full((T, H, D), 77.0, dtype=dtype, device="cuda")
    lse = torch.full((T, H), 77.0, device="cuda")
    assert verify.prompt_attend(q, k, v, ints(offsets), scale, out, lse) is out
    inside = slice(before, T - behind)
    for x in (out, lse):                                  # tokens of no sequence: left as they were
        assert (x[:before] == 77).all() and (x[T - behind:] == 77).all()
    want, want_lse, size = (x[inside] for x in plain(q, k, v, offsets, scale))
    got, lse = out[inside].double(), lse[inside].double()
    # weights and results are rounded to the type; scores and sums in 32 bits; half precision's smallest weights
    longest = max(lengths)
    size_of = lambda x: x[inside].double().nan_to_num(0, 0, 0).norm(dim=-1).max().item()
    loose = 2 * ((D + 4) * 2.0 ** -24 * abs(scale) * size_of(q) * size_of(k) + (longest + 8) * 2.0 ** -24)
    high = v[inside].double().nan_to_num(0, 0, 0).abs().max().item()
    error = ROUND[dtype] * (want.abs() + size) + loose * size + longest * 2.0 ** -24 * high
    finite = want.isfinite()
    assert same(got[~finite], want[~finite].to(dtype))
    assert ((got - want).abs() - error)[finite].max().item() <= 0, ((got - want).abs() - error)[finite].max().item()
    fine = want_lse.isfinite()
    assert ((lse - want_lse).abs()[fine] <= loose + 2.0 ** -22 * (1 + want_lse.abs()[fine])).all()
    return q, k, v, ints(offsets), out


SHAPES = [  # lengths, H, Hk, D
    ([1], 1, 1, 64),
    ([1, 2, 31, 32, 33], 8, 2, 128),
    ([63, 0, 64, 65, 0, 127], 4, 4, 64),
    ([128, 129, 1, 200], 28, 4, 128),
    ([0, 0, 5], 14, 2, 64),
    ([255, 256, 257], 4, 1, 96),
    ([97, 300], 3, 3, 256),
    ([70] * 9, 16, 2, 128),
    ([1] * 65, 12, 12, 64),
    ([511, 513], 6, 2, 64),
    ([40, 33], 512, 1, 64),                               # more heads of a group than rows of a tile
    ([1500], 8, 8, 128),
    ([777, 331], 6, 3, 96),
    ([700], 8, 2, 256),
]


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention_of_prompts(gen, shape, dtype):
    print(SHAPES[shape], dtype, flush=True)
    check(gen, *SHAPES[shape], dtype=dtype, fused=shape % 3 > 0)


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("length", [2300, 4100])
def test_long_prompts(gen, length, D):
    check(gen, [length, 3], 4, 2, D)


def test_tokens_before_and_behind_the_sequences_are_left(gen):
    for before, behind in ((1, 0), (0, 1), (130, 70), (37, 300)):
        check(gen, [40, 0, 90], 8, 2, 128, before=before, behind=behind)


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("G,D", [(1, 64), (4, 128), (7, 128), (3, 96), (2, 256)])
def test_what_a_token_does_not_see_does_not_reach_it(gen, dtype, G, D):
    """Infinities and NaN in later tokens, in other sequences, and in tokens that nobody sees."""
    def poison(q, k, v):
        v[35, :, 3], k[36, :, 5] = float("nan"), float("nan")
        v[31, :, 0], v[33, :, 1], v[64, :, D - 1] = float("inf"), float("-inf"), float("inf")
        k[150, :, 1] = float("inf")
        v[199], k[199] = float("nan"), float("nan")       # the last of its sequence
        k[260:], v[260:] = float("nan"), float("inf")     # behind all sequences
    lengths = [200, 60]
    q, k, v, offsets, out = check(gen, lengths, 2 * G, 2, D, dtype=dtype, poison=poison, behind=20)
    assert out[:35].isfinite()[:, :, 2].all() and out[200:260].isfinite().all()


def test_a_row_whose_scores_are_all_minus_infinity_is_zero(gen):
    q = normal(gen, (70, 2, 64), BF)
    q[..., 0], q[..., 1:] = 1, 0
    k, v = torch.zeros_like(q), normal(gen, (70, 2, 64), BF)
    k[:5, :, 0] = -torch.inf
    lse = torch.zeros((70, 2), device="cuda")
    out = verify.prompt_attend(q, k, v, ints([0, 70]), 1.0, lse=lse)
    assert not out[:5].any() and (lse[:5] == -torch.inf).all()
    assert torch.equal(out[5], v[5]) and (lse[5] == 0).all() and out.isfinite().all()


def test_scores_far_below_and_above_zero(gen):
    def poison(q, k, v):
        k *= 40
    for scale in (1.0, -0.5, 0.0):
        check(gen, [130, 61], 4, 2, 64, poison=poison, scale=scale)


@pytest.mark.parametrize("dtype", [BF, F16])
def test_values_of_very_different_sizes(gen, dtype):
    def poison(q, k, v):
        k[::5] *= 6
        v[::3] *= 2.0 ** 9
        v[1::3] *= 2.0 ** -9
    check(gen, [164, 61], 4, 2, 128, dtype=dtype, poison=poison)


def test_strides_beyond_32_bit_offsets(gen):
    """Tokens and heads so far apart that their places pass 2^32 bytes."""
    D, T = 64, 130
    buf = torch.empty((T, 1 << 24), dtype=BF, device="cuda")
    q, k, v = (buf[:, i * 64:(i + 2) * 64].unflatten(-1, (2, D)) for i in (0, 2, 4))
    for x in (q, k, v):
        x.copy_(normal(gen, (T, 2, D), BF))
    got = verify.prompt_attend(q, k, v, ints([0, T]))
    assert torch.equal(got, verify.prompt_attend(*(x.contiguous() for x in (q, k, v)), ints([0, T])))
    assert buf.stride(0) * 2 * T > 1 << 32


def test_many_sequences_and_the_same_bits(gen):
    lengths = [(7 * i) % 40 for i in range(500)]
    q, k, v, offsets, out = check(gen, lengths, 4, 2, 64)
    for _ in range(3):
        assert torch.equal(verify.prompt_attend(q, k, v, offsets)[:], out)


def test_offsets_that_make_no_sense_stay_inside(gen):
    """Descending, negative and too large offsets: results are unspecified, but nothing else is touched."""
    q = normal(gen, (64, 4, 64), BF)
    room = torch.full((256, 4, 64), 5.0, dtype=BF, device="cuda")
    cache = verify.PathCache(3, 1, 40, 1, 4, 4, 64, 1)
    for offsets in ([0, 64, 10, 30], [-5, 20, 10 ** 9, 64], [70, 80, -1, 3], [64, 64, 64, 0]):
        verify.prompt_attend(q, q, q, ints(offsets), out=room[96:160])
        assert (room[:96] == 5).all() and (room[160:] == 5).all()
        cache.write_packed(0, q, q, ints(offsets))


def test_another_stream_and_graph_replays(gen):
    lengths, H, Hk, D = [70, 200, 5], 8, 2, 128
    T = sum(lengths)
    offsets = ints([0, 70, 270, 275])
    qkv = normal(gen, (T, H + 2 * Hk, D), BF)
    call = lambda: verify.prompt_attend(qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], offsets)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = call()
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(there, call())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(4):
        qkv.copy_(normal(gen, qkv.shape, BF))
        if i == 2:
            offsets.copy_(ints([0, 100, 101, 275]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call())


# ---------------------------------------------------------------------------------------------- packed prompts to the cache

@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lengths,Hk,D", [([5], 2, 64), ([8, 0, 9, 31], 8, 128), ([40, 33, 1], 3, 96), ([7, 40], 1, 256), ([1] * 20, 12, 64)])
def test_packed_prompts_are_written(gen, dtype, fp8, lengths, Hk, D):
    P, T, cap = len(lengths), sum(lengths), 40
    c = verify.PathCache(P, 1, cap, 1, Hk, Hk, D, 1, n_layers=2, dtype=dtype, fp8=fp8)
    old = normal(gen, (P, cap, Hk, D), dtype)
    c.write_prompt(0, old, old)
    c.write_prompt(1, old, old)
    offsets = [3]
    for x in lengths:
        offsets.append(offsets[-1] + x)
    kv = normal(gen, (T + 5, 2 * Hk, D), dtype)
    c.write_packed(1, kv[:, :Hk], kv[:, Hk:], ints(offsets))
    assert c.status() == 0
    for x, got in zip((kv[:, :Hk], kv[:, Hk:]), c.read_prompt(1, cap)):
        want = held(old, fp8)
        for p, n in enumerate(lengths):
            want[p, :n] = held(x[offsets[p]:offsets[p + 1]], fp8)
        assert same(got, want.to(dtype))
    for got in c.read_prompt(0, cap):
        assert same(got, held(old, fp8).to(dtype))


def test_packed_prompts_beyond_the_capacity_are_dropped_and_reported(gen):
    c = verify.PathCache(2, 1, 33, 1, 2, 2, 64, 1)
    k = normal(gen, (70, 2, 64), BF)
    c.write_packed(0, k, k, ints([0, 50, 70]))
    assert c.status() == binding.STATUS_CAPACITY
    got = c.read_prompt(0, 33)[0]
    assert same(got[0], k[:33]) and same(got[1, :20], k[50:])


# --------------------------------------------------------------------------------------------------------- refusals

def test_arguments_that_are_refused(gen):
    q, k, offsets = normal(gen, (10, 8, 64), BF), normal(gen, (10, 2, 64), BF), ints([0, 10])
    empty = verify.prompt_attend(q[:0], k[:0], k[:0], ints([0, 0]))
    assert empty.shape == (0, 8, 64)
    wants = lambda t: t.clone().requires_grad_()
    for call, error in [
        (lambda: verify.prompt_attend(q.float(), k.float(), k.float(), offsets), TypeError),
        (lambda: verify.prompt_attend(q, k.half(), k, offsets), TypeError),
        (lambda: verify.prompt_attend(q, k, k[:5], offsets), ValueError),
        (lambda: verify.prompt_attend(q[:5], k, k, offsets), ValueError),
        (lambda: verify.prompt_attend(q[None], k, k, offsets), TypeError),
        (lambda: verify.prompt_attend(q, k[..., :32], k, offsets), ValueError),
        (lambda: verify.prompt_attend(q, k, k, offsets.long()), TypeError),
        (lambda: verify.prompt_attend(q, k, k, offsets[:1]), ValueError),
        (lambda: verify.prompt_attend(q, k, k, offsets.cpu()), TypeError),
        (lambda: verify.prompt_attend(q.cpu(), k, k, offsets), TypeError),
        (lambda: verify.prompt_attend(q, k, k, offsets, out=q), ValueError),
        (lambda: verify.prompt_attend(q, k, k, offsets, out=torch.empty((10, 8, 32), dtype=BF, device="cuda")), ValueError),
        (lambda: verify.prompt_attend(q, k, k, offsets, lse=torch.empty((10, 8), dtype=BF, device="cuda")), TypeError),
        (lambda: verify.prompt_attend(q[..., :7, :], k, k, offsets), binding.CsdError),
        (lambda: verify.prompt_attend(q[..., ::2], k[..., ::2], k[..., ::2], offsets), TypeError),
        (lambda: verify.prompt_attend(q, k, k, offsets, scale=float("nan")), binding.CsdError),
        (lambda: verify.prompt_attend(wants(q), k, k, offsets), TypeError),
        (lambda: verify.prompt_attend(q, k, wants(k), offsets), TypeError),
    ]:
        with pytest.raises(error):
            call()
    c = verify.PathCache(1, 1, 16, 1, 8, 2, 64, 1)
    for call, error in [(lambda: c.write_packed(0, k, k[:5], offsets), ValueError), (lambda: c.write_packed(1, k, k, offsets), binding.CsdError),
                        (lambda: c.write_packed(0, q, q, offsets), ValueError), (lambda: c.write_packed(0, k, k, offsets[:1]), ValueError),
                        (lambda: c.write_packed(0, k.half(), k.half(), offsets), TypeError), (lambda: c.write_packed(0, wants(k), k, offsets), TypeError)]:
        with pytest.raises(error):
            call()
    with torch.no_grad():
        verify.prompt_attend(wants(q), k, k, offsets)


def test_packed_keys_of_more_axes_are_refused(gen):
    c, k = verify.PathCache(1, 1, 16, 1, 8, 2, 64, 1), normal(gen, (2, 5, 2, 64), BF)
    with pytest.raises(ValueError):                                                                     # (whose length is not that of the tokens)
        c.write_packed(0, k, k, ints([0, 10]))


def test_scales_beyond_32_bits_are_refused(gen):
    q, k = normal(gen, (3, 2, 64), BF), normal(gen, (3, 2, 64), BF)
    for scale in (3e38, -3e38):                                                                         # (times log2 e)
        with pytest.raises(binding.CsdError):
            verify.prompt_attend(q, k, k, ints([0, 3]), scale=scale)


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("lengths,H,Hk", [([261], 512, 8), ([259, 262], 512, 8), ([1100], 128, 32)])
def test_launches_that_fill_the_chip(gen, lengths, H, Hk, D, dtype):
    """(more than 512 tiles of 256 rows, of 4096 rows a sequence and more: the largest workgroups)"""
    rows = sum(lengths) * H // Hk
    assert rows >= 4096 * len(lengths) and rows // 256 * Hk >= 512
    check(gen, lengths, H, Hk, D, dtype=dtype)


# kv heads and heads of each that take sequences of 200 and 60 tokens through every kind of workgroup
FORMS = [(2, 4), (128, 1), (192, 1), (16, 32)]


@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("Hk,G", FORMS)
def test_every_workgroup_with_odd_tokens(gen, Hk, G, D, dtype):
    def poison(q, k, v):
        v[35, :, 3], k[150, :, 5] = float("nan"), float("nan")
        v[31, :, 0], v[100, :, 1], v[130, :, D - 1] = float("inf"), float("-inf"), float("inf")
        v[199], k[199] = float("nan"), float("nan")
    print(Hk, G, D, dtype, flush=True)
    *_, out = check(gen, [200, 60], Hk * G, Hk, D, dtype=dtype, poison=poison, behind=20)
    assert out[:150].isfinite()[:, :, 2].all() and out[200:260].isfinite().all()


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("Hk,G", FORMS)
def test_every_workgroup_with_tokens_that_weigh_nothing(gen, Hk, G, D):
    """Scores of -inf for all that a wave sees, of some rows and of all."""
    T, H = 270, Hk * G
    q, k, v = torch.zeros((T, H, D), dtype=BF, device="cuda"), torch.zeros((T, Hk, D), dtype=BF, device="cuda"), normal(gen, (T, Hk, D), BF)
    q[..., 0] = 1
    counts = torch.ones(T, dtype=torch.bool, device="cuda")
    counts[:70] = counts[128:192] = counts[200:210] = False
    k[~counts, :, 0] = -torch.inf
    lse = torch.zeros((T, H), device="cuda")
    out = verify.prompt_attend(q, k, v, ints([0, 210, T]), 1.0, lse=lse)
    for a, b in ((0, 210), (210, T)):
        n = counts[a:b].double().cumsum(0)
        x = torch.where(counts[a:b, None, None], v[a:b].double(), 0.0)
        # weights of one, exact; sums in 32 bits; one rounding
        want, error = x.cumsum(0) / n.clamp(min=1)[:, None, None], x.abs().cumsum(0) * 280 * 2.0 ** -24 / n.clamp(min=1)[:, None, None]
        want, error = (t.repeat_interleave(G, 1) for t in (want, error + ROUND[BF] * want.abs()))
        assert ((out[a:b].double() - want).abs() <= error * (1 + 2.0 ** -7)).all()
        assert ((lse[a:b].double() - n.log()[:, None]).abs()[n > 0] <= 2.0 ** -20 * 6).all() and (lse[a:b][n == 0] == -torch.inf).all()
    assert not out[:70].any()


@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("lengths,G", [([32] * 40, 4), ([96] * 25, 4), ([5] * 33, 1), ([64, 1, 33] * 21, 3)])
def test_many_sequences_of_few_tiles(gen, lengths, G, D):
    check(gen, lengths, 8 * G, 8, D)

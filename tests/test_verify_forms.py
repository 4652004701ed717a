"""Attention over the cache in every form that a launch can take, with every size of heads, against a plain form in 64 bits."""
import ctypes
import random

import pytest
import torch

import test_verify
from paper_2503_05330_amd import binding, verify
from test_verify import BF, F16, check_attend, gen  # noqa: F401 (gen: a fixture)

DIMS = (64, 96, 128, 256)
TYPES = ((BF, False), (BF, True), (F16, False), (F16, True))

# P, N, n, heads, kv heads, prompt and path capacities; then the form: joined, solo; groups of 32 query rows that a workgroup
# takes of a path and of a prompt (1, 2 or 4; of a solo path: its waves'; 0: prompts have no items); whether paths and prompts are split
FORMS = [
    ((2, 3, 3, 10, 2, 100, 100), (0, 0, 1, 0, 0, 0)),
    ((1, 3, 9, 8, 2, 31, 40), (0, 0, 2, 0, 0, 0)),
    ((1, 2, 33, 5, 1, 40, 64), (0, 0, 4, 0, 0, 0)),
    ((50, 5, 1, 8, 8, 52, 63), (0, 1, 1, 0, 0, 0)),
    ((40, 3, 9, 12, 3, 0, 40), (0, 1, 2, 0, 0, 0)),
    ((1, 1, 17, 4, 1, 100, 100), (0, 1, 4, 0, 0, 0)),
    ((1, 3, 1, 2, 1, 0, 1500), (1, 0, 1, 0, 1, 0)),
    ((1, 3, 1, 3, 1, 600, 700), (1, 0, 1, 1, 1, 1)),
    ((40, 3, 1, 8, 8, 1000, 700), (1, 0, 1, 1, 0, 0)),
    ((1, 2, 9, 2, 1, 600, 1500), (1, 0, 1, 2, 1, 1)),
    ((1, 3, 5, 5, 1, 40, 1500), (1, 0, 1, 4, 1, 0)),
    ((1, 1, 17, 2, 1, 600, 700), (1, 0, 2, 2, 1, 1)),
    ((8, 1, 17, 8, 4, 600, 300), (1, 0, 2, 2, 0, 1)),
    ((1, 2, 17, 2, 1, 40, 700), (1, 0, 2, 4, 1, 0)),
    ((8, 5, 17, 14, 2, 300, 700), (1, 0, 4, 4, 1, 0)),
    ((20, 3, 17, 8, 2, 600, 300), (1, 0, 4, 4, 0, 1)),
    ((1, 5, 1, 7, 1, 1000, 300), (1, 1, 1, 1, 1, 1)),
    ((1, 3, 3, 4, 1, 1000, 300), (1, 1, 1, 2, 1, 1)),
    ((1, 3, 5, 5, 1, 300, 1500), (1, 1, 1, 4, 1, 1)),
    ((1, 2, 17, 2, 1, 600, 300), (1, 1, 2, 4, 1, 1)),
    ((1, 1, 17, 4, 1, 0, 700), (1, 1, 4, 0, 1, 0)),
    ((1, 1, 17, 5, 1, 300, 40), (1, 1, 4, 4, 0, 1)),
]


def groups(rows):
    return 1 if rows <= 32 else 2 if rows <= 64 else 4


def lengths(P, N, n, T, U):
    """Ragged, the longest of them the capacities: of prompts, of paths, counts."""
    prompt = [T - 53 * p % T if T else 0 for p in range(P)]
    path = [[U - 37 * (p * N + i) % (3 * U // 4) for i in range(N)] for p in range(P)]
    counts = [[n if (p * N + i) % 4 != 3 else 0 if p % 2 == 0 else n // 2 for i in range(N)] for p in range(P)]
    return prompt, path, counts


@pytest.mark.parametrize("form", range(len(FORMS)))
def test_the_form_is_the_one_that_is_meant(form):
    (P, N, n, H, Hk, T, U), want = FORMS[form]
    counts, G = lengths(P, N, n, T, U)[2], H // Hk
    for D in DIMS:
        for dtype, fp8 in TYPES:
            got = verify.attend_form(verify.CacheConfig(P, N, T, U, 1, H, Hk, D, n, verify.TYPES[dtype], fp8), n)
            prompts = groups(max(map(sum, counts)) * G) if got.prompt_splits else 0
            assert (got.joined, got.solo, groups(max(map(max, counts)) * G), prompts, got.path_splits > 1, got.prompt_splits > 1) == want


def test_all_forms_are_there():
    forms = [want for _, want in FORMS]
    assert {x[:3] for x in forms} == {(j, s, g) for j in (0, 1) for s in (0, 1) for g in (1, 2, 4)}
    assert {x[3] for x in forms if x[0]} == {0, 1, 2, 4}
    assert {x[4:] for x in forms if x[0]} == {(a, b) for a in (0, 1) for b in (0, 1)}


def test_parts_have_room_in_the_cache():
    """What the parts of a call of any size take of memory, and what a cache of these limits has beside its keys and values."""
    rng, lib, size = random.Random(5), verify.load(), ctypes.c_size_t()
    spread = lambda lo, hi: int(round(2 ** rng.uniform(lo, hi)))
    for _ in range(20000):
        Hk, G, n = spread(0, 4), rng.randint(1, 8), rng.randint(1, 33)
        P, N, T, U = spread(0, 7), spread(0, 7), spread(0, 14) if rng.random() < 0.8 else 0, spread(0, 14)
        cfg = verify.CacheConfig(P, N, T, U, 1, Hk * G, Hk, rng.choice(DIMS), n, 0, rng.randint(0, 1))
        assert lib.csd_cache_bytes(ctypes.byref(cfg), ctypes.byref(size)) == binding.OK
        blocks = P * Hk * (-(-T // 32) + N * -(-U // 32))
        room = size.value - blocks * 64 * (cfg.head_dim + 1 if cfg.fp8 else 2 * cfg.head_dim)
        calls = [(n, 0, 0), (rng.randint(1, n), 0, 0), (rng.randint(1, n), spread(0, 14), spread(0, 14)), (1, 1, 1 << 24)]
        for m, prompt_bound, path_bound in calls:
            form = verify.attend_form(cfg, m, prompt_bound, path_bound)
            parts = (form.prompt_splits + form.path_splits) * P * N * m * Hk * G if form.joined else 0
            assert parts * (cfg.head_dim + 1) * 4 <= room, (cfg, m)


def test_forms_of_calls_that_are_refused():
    cfg = verify.CacheConfig(1, 2, 40, 40, 1, 4, 2, 64, 5, 0, 0)
    for args in ((0,), (6,), (1, -1), (1, 0, -1)):
        with pytest.raises(binding.CsdError) as err:
            verify.attend_form(cfg, *args)
        assert err.value.code == binding.ERR_INVALID_ARG
    with pytest.raises(binding.CsdError):
        verify.attend_form(verify.CacheConfig(1, 2, 40, 40, 1, 4, 3, 64, 5, 0, 0), 1)
    assert verify.load().csd_attend_form_of(ctypes.byref(cfg), 1, 0, 0, None) == binding.ERR_INVALID_ARG


def attend64(q, prompt, path, prompt_len, path_len, counts, scale):
    """test_verify.plain_attend on the GPU, all heads of a token at once."""
    P, N, n, H, D = q.shape
    G = H // prompt[0].shape[-2]
    q = q.cuda().double()
    prompt, path = ([x.cuda().repeat_interleave(G, -2) for x in pair] for pair in (prompt, path))
    out, size = (torch.zeros((P, N, n, H, D), dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((P, N, n, H), -torch.inf, dtype=torch.float64, device="cuda")
    for p in range(P):
        for i in range(N):
            sees = [max(0, path_len[p][i] - counts[p][i] + t + 1) for t in range(counts[p][i])]
            most = max(sees, default=0)
            k, v = (torch.cat([a[p, :prompt_len[p]], b[p, i, :most]]) for a, b in zip(prompt, path))
            for t, x in enumerate(sees):
                x += prompt_len[p]
                if x == 0:
                    continue
                s = (k[:x] * q[p, i, t]).sum(-1) * scale                    # [tokens][H]
                lse[p, i, t] = torch.logsumexp(s, 0)
                w = torch.softmax(s, 0)[..., None]
                out[p, i, t], size[p, i, t] = (w * v[:x]).sum(0), (w * v[:x].abs()).sum(0)
    return out.cpu(), lse.cpu(), size.cpu()


@pytest.mark.gpu
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_attention_in_every_form(gen, monkeypatch, form, D):
    """Ragged lengths; then with infinities and NaN in the newest tokens, which some rows see, in the prompts' last, which all see,
    and where nothing has been written."""
    monkeypatch.setattr(test_verify, "plain_attend", attend64)
    P, N, n, H, Hk, T, U = FORMS[form][0]
    prompt, path, counts = lengths(P, N, n, T, U)

    def poison(pk, pv, k, v):
        for p in range(P):
            for i in range(N):
                end, kind = path[p][i], (p * N + i) % 4
                at = max(0, end - (1 + n // 3))          # seen by the later rows alone, where there are several
                if kind == 0:
                    v[p, i, at, :, 3], v[p, i, end - 1, :, D - 1] = float("inf"), float("nan")
                elif kind == 1:
                    k[p, i, end - 1, :, 5] = float("nan")
                elif kind == 2:
                    v[p, i, at, :, 40], v[p, i, max(0, at - 40), 0, 1] = float("-inf"), float("inf")
            if T and p % 2 == 0:
                pv[p, prompt[p] - 1, :, 7] = float("inf")
    large = P * Hk * (T + N * U) * D > 5e7
    for dtype, fp8 in TYPES[1:3] if large else TYPES:
        print(FORMS[form], D, dtype, fp8, flush=True)
        for poisons in (None, poison):
            check_attend(gen, P, N, n, H, Hk, D, prompt, path, counts, dtype=dtype, fp8=fp8, caps=(T, U), poison=poisons)

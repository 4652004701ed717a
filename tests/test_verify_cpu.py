"""Host-side checks of the verifying pass's operators that need no GPU: exports, sizes, refusals before anything is enqueued."""
import ctypes
import os
import re

import pytest

from paper_2503_05330_amd import binding as b
from paper_2503_05330_amd import verify

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
GOOD = dict(n_problems=2, n_paths=16, prompt_cap=1000, path_cap=100, n_layers=3, n_heads=32, n_kv_heads=8, head_dim=128,
            max_step=9, type=verify.BF16, fp8=0)


@pytest.fixture(scope="module")
def lib():
    return verify.load()


def config(**change):
    values = {**GOOD, **change}
    return verify.CacheConfig(*[values[name] for name, _ in verify.CacheConfig._fields_])


def test_exports_every_declared_symbol(lib):
    header = open(os.path.join(ROOT, "include", "csd_verify.h")).read()
    declared = sorted(set(re.findall(r"^int\s+(csd_[a-z_]+)\s*\(", header, re.M)))
    assert declared == sorted(verify.EXPORTS)
    for name in declared:
        assert hasattr(lib, name)


def test_header_compiles_as_c(tmp_path):
    import subprocess
    source = tmp_path / "x.c"
    source.write_text('#include "csd_verify.h"\nint main(void) { return sizeof(csd_heads) == 32 ? 0 : 1; }\n')
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(tmp_path / "x")])
    subprocess.check_call([str(tmp_path / "x")])


@pytest.mark.parametrize("fp8", [0, 1])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_a_cache_takes_what_its_tokens_take(lib, fp8, dim):
    out = ctypes.c_size_t(0)
    assert lib.csd_cache_bytes(ctypes.byref(config(fp8=fp8, head_dim=dim)), ctypes.byref(out)) == b.OK
    tokens = 3 * 2 * (1024 + 16 * 128)                   # whole blocks of 32
    held = tokens * 8 * 2 * (dim + 1 if fp8 else 2 * dim)
    parts = 2 * (2 * 16 * 9 * 32) + (1 << 16)
    assert held + parts * (dim + 1) * 4 <= out.value <= held + parts * (dim + 1) * 4 + 4096


def test_configurations_that_are_refused(lib):
    out = ctypes.c_size_t(0)
    for bad in (dict(n_problems=0), dict(n_paths=0), dict(prompt_cap=-1), dict(path_cap=0), dict(n_layers=0), dict(n_layers=2000),
                dict(n_heads=0), dict(n_heads=33), dict(n_kv_heads=0), dict(n_heads=1024), dict(head_dim=0), dict(head_dim=-64),
                dict(max_step=0), dict(max_step=34), dict(type=2), dict(type=-1), dict(fp8=2), dict(path_cap=(1 << 24) + 1),
                dict(prompt_cap=(1 << 24) + 1), dict(n_problems=1 << 13, n_paths=1 << 12),
                dict(n_problems=1 << 13, n_paths=1 << 9, n_kv_heads=1, n_heads=1),
                dict(n_problems=1 << 10, n_paths=1 << 10, n_layers=1024, path_cap=1 << 24, n_kv_heads=1)):
        assert lib.csd_cache_bytes(ctypes.byref(config(**bad)), ctypes.byref(out)) == b.ERR_INVALID_ARG, bad
    for unknown in (32, 80, 192, 512):
        assert lib.csd_cache_bytes(ctypes.byref(config(head_dim=unknown)), ctypes.byref(out)) == b.ERR_UNIMPLEMENTED
    assert lib.csd_cache_bytes(None, ctypes.byref(out)) == b.ERR_INVALID_ARG
    assert lib.csd_cache_bytes(ctypes.byref(config()), None) == b.ERR_INVALID_ARG
    for fine in (dict(prompt_cap=0), dict(n_heads=8), dict(max_step=33), dict(type=verify.F16, fp8=1), dict(head_dim=64)):
        assert lib.csd_cache_bytes(ctypes.byref(config(**fine)), ctypes.byref(out)) == b.OK, fine


def test_null_and_misaligned_arguments_are_refused(lib):
    h, cfg, big = ctypes.c_void_p(), config(), 1 << 40
    assert lib.csd_cache_create(ctypes.byref(cfg), None, big, None, ctypes.byref(h)) == b.ERR_INVALID_ARG
    assert lib.csd_cache_create(ctypes.byref(cfg), 256, 4096, None, ctypes.byref(h)) == b.ERR_WORKSPACE
    assert lib.csd_cache_create(ctypes.byref(cfg), 128, big, None, ctypes.byref(h)) == b.ERR_WORKSPACE
    assert lib.csd_cache_create(ctypes.byref(cfg), 256, big, None, None) == b.ERR_INVALID_ARG
    assert h.value is None
    heads = verify.Heads(4096, 1024, 1024, 128)
    hp = ctypes.byref(heads)
    for fn, args in ((lib.csd_cache_destroy, (None,)), (lib.csd_cache_write, (None, 0, hp, hp, None, None, 1, None)),
                     (lib.csd_cache_write_prompt, (None, 0, hp, hp, None, None, 1, None)),
                     (lib.csd_cache_read, (None, 0, None, None, 1, 4096, 4096, None)),
                     (lib.csd_cache_read_prompt, (None, 0, None, None, 1, 4096, 4096, None)),
                     (lib.csd_attend, (None, 0, hp, None, 4096, None, 1, 1.0, 0, 0, 4096, None, None)),
                     (lib.csd_cache_status, (None, None, None))):
        assert fn(*args) == b.ERR_INVALID_ARG
    size = ctypes.c_size_t(0)
    for rows, vocab in ((0, 10), (1 << 23, 10), (1, 0), (1, 1 << 29), (-1, 5)):
        assert lib.csd_targets_bytes(rows, vocab, ctypes.byref(size)) == b.ERR_INVALID_ARG
    assert lib.csd_targets_bytes(1, 10, None) == b.ERR_INVALID_ARG
    good = dict(logits=4096, type=0, rows=2, vocab=10, stride=10, noise=None, noise_stride=0, inv=1.0, tokens=4096, probs=4096)

    def targets(**change):
        v = {**good, **change}
        return lib.csd_targets(v["logits"], v["type"], v["rows"], v["vocab"], v["stride"], v["noise"], v["noise_stride"], v["inv"],
                               v["tokens"], v["probs"], None, 0, None)
    for bad in (dict(logits=None), dict(type=3), dict(type=-1), dict(rows=0), dict(vocab=0), dict(stride=-1), dict(logits=4097),
                dict(type=2, logits=4098), dict(noise=4098), dict(noise=4096, noise_stride=-1), dict(inv=0.0), dict(inv=-1.0),
                dict(inv=float("nan")), dict(inv=float("inf")), dict(tokens=None), dict(probs=None)):
        assert targets(**bad) == b.ERR_INVALID_ARG, bad


def test_rows_of_targets_share_a_launch_of_less_than_two_to_the_32_threads(lib):
    size = ctypes.c_size_t()
    for rows in (1 << 19, (1 << 19) + 1, 1 << 20, 1 << 22):                # (a scratch: eight workgroups of 512 threads a row)
        assert lib.csd_targets_bytes(rows, 152064, ctypes.byref(size)) == 0
        assert (rows * 8 * 512 < 1 << 32) if size.value else (rows * 512 < 1 << 32)


def test_tensors_of_the_host_are_refused(lib):
    import torch
    with pytest.raises(TypeError):
        verify.targets(torch.zeros(3, 100, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        verify._heads(torch.zeros(2, 3, 4, 8, 64, dtype=torch.bfloat16), torch.bfloat16, (2, 3), 8, 64)

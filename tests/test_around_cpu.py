"""Host-side checks of the operators around the cache that need no GPU: refusals before anything is enqueued, rotations' frequencies."""
import ctypes
import math
import os

import pytest
import torch

from paper_2503_05330_amd import binding as b
from paper_2503_05330_amd import verify

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    return verify.load()


def test_structures_have_the_header_s_layout(tmp_path):
    import subprocess
    source = tmp_path / "x.c"
    fields = [("csd_rotary", "d_turns", verify.RotaryConfig.turns), ("csd_rotary", "amplitude", verify.RotaryConfig.amplitude)]
    a = verify.Adjustment
    fields += [("csd_adjustment", "d_" + n, getattr(a, n)) for n in ("logits", "out", "counts", "penalties", "tokens", "path_len", "prompt", "prompt_len", "bias", "mask")]
    fields += [("csd_adjustment", n, getattr(a, n)) for n in ("n_problems", "type", "logit_stride", "out_stride", "token_stride", "path_cap", "prompt_cap",
                                                             "bias_stride", "mask_stride")]
    checks = "".join("if (offsetof(%s, %s) != %d) return %d;\n" % (s, n, f.offset, i + 1) for i, (s, n, f) in enumerate(fields))
    sizes = "if (sizeof(csd_rotary) != %d || sizeof(csd_adjustment) != %d) return 99;\n" % (ctypes.sizeof(verify.RotaryConfig), ctypes.sizeof(a))
    source.write_text('#include <stddef.h>\n#include "csd_verify.h"\nint main(void) {\n%s%sreturn 0; }\n' % (checks, sizes))
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(source), "-o", str(tmp_path / "x")])
    subprocess.check_call([str(tmp_path / "x")])


def test_turns_of_a_rotation(lib):
    for dim, base, factor, original, low, high in ((64, 10000.0, 1.0, 0, 1, 4), (128, 500000.0, 8.0, 8192, 1, 4), (16, 2.0, 0.5, 10, 0.25, 0.5), (512, 1e6, 3.0, 100, 1, 32)):
        out = (ctypes.c_double * (dim // 2))()
        assert lib.csd_rotary_turns(dim, base, factor, original, low, high, ctypes.addressof(out)) == b.OK
        for i, got in enumerate(out):
            f = base ** (-2 * i / dim) / (2 * math.pi)
            keep = min(1.0, max(0.0, (original * f - low) / (high - low))) if original else 0.0
            assert math.isclose(got, keep * f + (1 - keep) * f / factor, rel_tol=1e-14)
    room = ctypes.addressof((ctypes.c_double * 512)())
    good = dict(dim=64, base=10000.0, factor=1.0, original=0.0, low=1.0, high=4.0, out=room)
    nan, inf = float("nan"), float("inf")
    for bad in (dict(dim=0), dict(dim=8), dict(dim=24), dict(dim=528), dict(dim=-16), dict(base=1.0), dict(base=nan), dict(base=inf), dict(factor=0.0),
                dict(factor=-1.0), dict(factor=nan), dict(original=-1.0), dict(original=nan), dict(high=1.0), dict(low=5.0), dict(low=nan), dict(out=None)):
        assert lib.csd_rotary_turns(*{**good, **bad}.values()) == b.ERR_INVALID_ARG, bad


def test_rotations_on_the_host():
    r = verify.Rotary(32, base=100.0, device="cpu")
    assert r.turns.dtype == torch.float64 and math.isclose(r.turns[3].item(), 100.0 ** (-6 / 32) / (2 * math.pi), rel_tol=1e-14)
    given = verify.Rotary(32, frequencies=[1.0] * 16, amplitude=2.0, device="cpu")
    assert (given.turns == 1 / (2 * math.pi)).all() and given.amplitude == 2.0
    for bad in (lambda: verify.Rotary(32, frequencies=[1.0] * 15, device="cpu"), lambda: verify.Rotary(24, frequencies=[1.0] * 12, device="cpu"),
                lambda: verify.Rotary(32, amplitude=float("inf"), device="cpu")):
        with pytest.raises(ValueError):
            bad()
    for bad in (dict(dim=20), dict(dim=32, base=0.5), dict(dim=32, factor=0.0), dict(dim=32, original=5, low=3, high=2)):
        with pytest.raises((b.CsdError, ValueError)):
            verify.Rotary(**bad, device="cpu")


def test_arguments_of_a_rotation_that_are_refused(lib):
    good = dict(turns=4096, dim=64, interleaved=0, amplitude=1.0, x=4096, x_token=512, x_head=64, at=4096, tokens=3, heads=8, head_dim=64, type=0, out=8192,
                out_token=512, out_head=64)

    def call(**change):
        v = {**good, **change}
        how = verify.RotaryConfig(v["turns"], v["dim"], v["interleaved"], v["amplitude"])
        x, out = verify.Heads(v["x"], 0, v["x_token"], v["x_head"]), verify.Heads(v["out"], 0, v["out_token"], v["out_head"])
        return lib.csd_rotate(ctypes.byref(how), ctypes.byref(x), v["at"], v["tokens"], v["heads"], v["head_dim"], v["type"], ctypes.byref(out), None)
    for bad in (dict(turns=None), dict(turns=4100), dict(dim=0), dict(dim=24), dict(dim=80), dict(dim=-16), dict(interleaved=2), dict(amplitude=float("nan")),
                dict(x=None), dict(x=4104), dict(x_token=4), dict(x_head=-8), dict(at=None), dict(at=4097), dict(tokens=-1), dict(tokens=(1 << 24) + 1),
                dict(heads=0), dict(heads=1025), dict(head_dim=60), dict(head_dim=520), dict(type=2), dict(type=-1), dict(out=None), dict(out=8200),
                dict(out_token=-8), dict(out=4096, out_token=1024), dict(out=4096, out_head=128)):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    assert call(tokens=0, x=None, out=None, at=None) == b.OK                             # nothing to do
    assert lib.csd_rotate(None, None, None, 1, 1, 64, 0, None, None) == b.ERR_INVALID_ARG


def test_results_of_a_rotation_at_one_place_are_refused(lib):
    how, x = verify.RotaryConfig(4096, 64, 0, 1.0), verify.Heads(4096, 0, 0, 0)                       # (what is read may be)
    for token, head in ((0, 64), (512, 0), (512, 56), (504, 64), (64, 128), (56, 192), (64, 184)):
        out = verify.Heads(1 << 20, 0, token, head)
        assert lib.csd_rotate(ctypes.byref(how), ctypes.byref(x), 4096, 3, 8, 64, 0, ctypes.byref(out), None) == b.ERR_INVALID_ARG, (token, head)


def test_arguments_of_attention_of_prompts_that_are_refused(lib):
    good = dict(q=4096, k=8192, v=16384, stride=512, head=64, type=0, n_heads=8, n_kv_heads=2, head_dim=64, offsets=4096, sequences=2, tokens=10, scale=0.1, out=4096, lse=None)

    def call(**change):
        x = {**good, **change}
        heads = [ctypes.byref(verify.Heads(x[n], 0, x["stride"], x["head"])) for n in "qkv"]
        return lib.csd_prompt_attend(*heads, x["type"], x["n_heads"], x["n_kv_heads"], x["head_dim"], x["offsets"], x["sequences"], x["tokens"], x["scale"], x["out"],
                                     x["lse"], None)
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(q=4100), dict(stride=4), dict(stride=-8), dict(stride=(1 << 24) + 8), dict(head=4), dict(type=2), dict(type=-1),
                dict(n_heads=7), dict(n_heads=0), dict(n_heads=1024), dict(n_kv_heads=0), dict(head_dim=0), dict(offsets=None), dict(offsets=4098), dict(sequences=0),
                dict(sequences=(1 << 20) + 1), dict(tokens=-1), dict(tokens=(1 << 24) + 1), dict(scale=float("inf")), dict(out=None), dict(out=4104), dict(lse=4098),
                dict(tokens=1 << 24, n_heads=512, n_kv_heads=4)):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    for unknown in (32, 80, 192):
        assert call(head_dim=unknown) == b.ERR_UNIMPLEMENTED
    assert call(tokens=0, q=None, k=None, v=None, out=None) == b.OK
    assert lib.csd_prompt_attend(None, None, None, 0, 8, 2, 64, 4096, 1, 1, 1.0, 4096, None, None) == b.ERR_INVALID_ARG
    heads, how = verify.Heads(4096, 512, 512, 64), verify.RotaryConfig(4096, 64, 0, 1.0)
    h = ctypes.byref(heads)
    assert lib.csd_cache_write_packed(None, 0, h, h, 4096, 1, None) == b.ERR_INVALID_ARG
    assert lib.csd_cache_write_rotated(None, 0, ctypes.byref(how), h, h, h, 4096, None, None, 1, 4096, None) == b.ERR_INVALID_ARG


def test_arguments_of_adjust_that_are_refused(lib):
    good = dict(n_problems=2, n_paths=3, n=4, vocab=100, type=0, logits=4096, logit_stride=100, out=1 << 20, out_stride=100, counts=None, penalties=4096, tokens=4096,
                token_stride=8, path_cap=8, path_len=4096, prompt=4096, prompt_stride=8, prompt_cap=8, prompt_len=None, bias=4096, bias_stride=100, mask=4096, mask_stride=4)

    def call(**change):
        return lib.csd_adjust(ctypes.byref(verify.Adjustment(*{**good, **change}.values())), None)
    for bad in (dict(n_problems=0), dict(n_paths=-1), dict(n=0), dict(n=34), dict(vocab=0), dict(vocab=1 << 29), dict(n_problems=1 << 12, n_paths=1 << 10), dict(type=3),
                dict(type=-1), dict(logits=None), dict(logits=4097), dict(type=2, logits=4098), dict(out=None), dict(out=4097), dict(logit_stride=-1), dict(out_stride=99),
                dict(out_stride=-100), dict(out=4096, out_stride=104), dict(counts=4098), dict(penalties=4097), dict(tokens=4098), dict(token_stride=-1), dict(path_cap=-1),
                dict(path_cap=(1 << 24) + 1), dict(path_len=None), dict(path_len=4098), dict(prompt=4098), dict(prompt_stride=-1), dict(prompt_cap=-1), dict(prompt_len=4098),
                dict(bias=4098), dict(bias_stride=-1), dict(mask=4098), dict(mask_stride=-1)):
        assert call(**bad) == b.ERR_INVALID_ARG, bad
    assert lib.csd_adjust(None, None) == b.ERR_INVALID_ARG


def test_tensors_of_the_host_are_refused(lib):
    x, at = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: verify.rotate(x, at, verify.Rotary(64, device="cpu")), lambda: verify.prompt_attend(x, x, x, at), lambda: verify.adjust(x[None])):
        with pytest.raises(TypeError):
            call()

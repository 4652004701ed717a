"""Where the attention of prompts reads a tile's keys and values from, worked out on the host; and that tokens and heads may lie at any distance."""
import os
import shutil
import subprocess

import pytest
import torch

from paper_2503_05330_amd import build, verify
from test_verify import BF, F16, gen, ints, normal, same  # noqa: F401 (gen: a fixture)

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "csd_prompt.cuh"
using namespace csd::verify;

// Row r of a tile (rows of a block: r % 32) lies in LDS at r * kRow, chunk j of it at place j ^ swizzle(r % 32): so the 16 bytes that go to place
// `to` are chunk (to / 16 % kChunks) ^ swizzle of token to / kRow.
template <int D, int WAVES>
int wrong() {
  typedef Rows<D, false> R;
  typedef TileLoads<R, WAVES> Loads;
  const int64_t strides[] = {0, 1 << 24, (1 << 24) - 8, (1 << 24) - 24};
  int bad = 0;
  for (int s = 0; s < 260; ++s) {
    const int64_t stride = s < 4 ? strides[s] : D + 8 * (s - 4);
    std::vector<int> seen(2 * R::kHalf / 16);
    for (int wave = 0; wave < WAVES; ++wave)
      for (int lane = 0; lane < 64; ++lane) {
        const Loads loads(stride, wave, lane);
        for (int x = 0; x < Loads::kPieces; ++x) {
          const int to = 1024 * (WAVES * x + wave) + 16 * lane;
          if (to >= 2 * R::kHalf) continue;
          ++seen[to / 16];
          const int token = to / R::kRow, chunk = to % R::kRow / 16 ^ R::swizzle(token & 31);
          const int64_t from = 2 * Loads::wave_at(x, stride) + (int64_t)loads.lane_at(x);
          if (from != token * stride * 2 + 16 * chunk) {
            if (!bad) printf("heads of %d, %d waves, stride %lld: token %d, chunk %d is read at %lld\n", D, WAVES, (long long)stride, token, chunk, (long long)from);
            ++bad;
          }
          for (int left : {1, 31, 33, 63})               // (tokens that are not there: the last one)
            if (Loads::place(x, stride, left, wave, lane) != (uint32_t)((token < left ? token : left - 1) * stride * 2 + 16 * chunk)) ++bad;
        }
      }
    for (int n : seen) bad += n != 1;
  }
  return bad;
}
int main() { return wrong<64, 4>() || wrong<96, 4>() || wrong<128, 4>() || wrong<128, 8>() || wrong<256, 4>(); }
"""


def test_every_16_bytes_come_from_their_own_place(tmp_path):
    """Strides of all multiples of 8, and the largest: heads of every size, every number of waves that there is."""
    source = tmp_path / "places.hip"
    source.write_text(PROGRAM)
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    flags = [x for x in build.HIPCC_FLAGS if not x.startswith("--offload") and x not in ("-Xclang", "-target-feature", "-packed-fp32-ops")]
    subprocess.check_call([hipcc, *flags, "--cuda-host-only", "-I", os.path.join(build.ROOT, "include"), "-I", os.path.join(build.HERE, "csrc"), str(source), "-o",
                           str(tmp_path / "places")])
    run = subprocess.run([str(tmp_path / "places")], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout


# kv heads and heads of each that take sequences of 200, 60 and 129 tokens through every kind of workgroup
FORMS = [(2, 4), (128, 1), (192, 1), (16, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("D", [64, 96, 128, 256])
@pytest.mark.parametrize("Hk,G", FORMS)
def test_tokens_at_any_distance(gen, Hk, G, D, dtype):
    """Keys and values whose rows are 8, 16, 24 .. elements longer than their heads, NaN between them and nothing behind the last: the same bits as
    of contiguous copies."""
    lengths = [200, 60, 129]
    T, H, offsets = sum(lengths), Hk * G, ints([0, 200, 260, 389])
    q, k, v = normal(gen, (T, H, D), dtype), normal(gen, (T, Hk, D), dtype), normal(gen, (T, Hk, D), dtype)
    want = verify.prompt_attend(q, k, v, offsets)
    assert want.isfinite().all()
    for more in (8, 16, 24, 40):
        print(Hk, G, D, dtype, more, flush=True)

        def spread(x):
            n = T * (x[0].numel() + more) - more             # the last token's values end where the storage does
            flat = torch.full((n,), torch.nan, dtype=dtype, device="cuda")
            return flat.as_strided(x.shape, (x[0].numel() + more, D, 1)).copy_(x)
        assert same(verify.prompt_attend(spread(q), spread(k), spread(v), offsets), want)
        apart = [torch.full((T, x.shape[1], D + more), torch.nan, dtype=dtype, device="cuda")[..., :D].copy_(x) for x in (q, k, v)]
        assert same(verify.prompt_attend(*apart, offsets), want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F16])
@pytest.mark.parametrize("lengths,H,Hk,D", [([1100], 128, 32, 128), ([1100], 128, 32, 256), ([2500, 70], 8, 2, 256), ([2500, 70], 8, 2, 64)])
def test_long_rows_at_any_distance(gen, lengths, H, Hk, D, dtype):
    T, offsets = sum(lengths), [0]
    for x in lengths:
        offsets.append(offsets[-1] + x)
    q, k, v = normal(gen, (T, H, D), dtype), normal(gen, (T, Hk, D), dtype), normal(gen, (T, Hk, D), dtype)
    want = verify.prompt_attend(q, k, v, ints(offsets))
    for gate in (8, 16, 24):                                 # a projection that leaves other numbers behind its heads
        wide = torch.full((T, (H + 2 * Hk) * D + gate), torch.nan, dtype=dtype, device="cuda")
        heads = [wide[:, a * D:(a + n) * D].unflatten(-1, (n, D)).copy_(x) for a, n, x in ((0, H, q), (H, Hk, k), (H + Hk, Hk, v))]
        assert same(verify.prompt_attend(*heads, ints(offsets)), want)

// csd — host side of attention of whole prompts: argument checks, the launch.
#include <cmath>

#include "csd_prompt.cuh"

extern "C" int csd_prompt_attend(const csd_heads* q, const csd_heads* k, const csd_heads* v, int32_t type, int32_t n_heads, int32_t n_kv_heads,
                                 int32_t head_dim, const int32_t* d_offsets, int32_t sequences, int64_t tokens, float scale, void* d_out, float* d_lse,
                                 void* stream) {
  using namespace csd::verify;
  constexpr float kLog2E = 1.44269504088896340736f;
  if (n_kv_heads <= 0 || n_heads <= 0 || n_heads > CSD_MAX_HEADS || n_heads % n_kv_heads || head_dim <= 0) return CSD_ERR_INVALID_ARG;
  if ((type != CSD_BF16 && type != CSD_F16) || sequences <= 0 || sequences > CSD_MAX_SEQUENCES || tokens < 0 || tokens > CSD_MAX_PACKED_TOKENS || !std::isfinite(scale * kLog2E))
    return CSD_ERR_INVALID_ARG;
  auto bad = [](const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  for (const csd_heads* h : {q, k, v})
    if (!h || (tokens && !h->data) || bad(h->data, 16) || h->token_stride < 0 || h->head_stride < 0 || h->token_stride % 8 || h->head_stride % 8)
      return CSD_ERR_INVALID_ARG;
  if (k->token_stride > 1 << 24 || v->token_stride > 1 << 24) return CSD_ERR_INVALID_ARG;
  if (!d_offsets || bad(d_offsets, 4) || (tokens && !d_out) || bad(d_out, 16) || bad(d_lse, 4)) return CSD_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 256) return CSD_ERR_UNIMPLEMENTED;
  const int32_t G = n_heads / n_kv_heads;
  const int64_t tiles = tokens * G / 128 + sequences;
  if (tiles * n_kv_heads > 1 << 23) return CSD_ERR_INVALID_ARG;
  if (tokens == 0) return CSD_OK;
  const PromptArgs a{*q, *k, *v, d_offsets, sequences, (int32_t)tokens, n_kv_heads, G, (int32_t)tiles, false, scale * kLog2E, d_out, d_lse};
  hipStream_t st = static_cast<hipStream_t>(stream);
  switch (head_dim) {
    case 64: prompt_64(a, type == CSD_F16, st); break;
    case 96: prompt_96(a, type == CSD_F16, st); break;
    case 128: prompt_128(a, type == CSD_F16, st); break;
    default: prompt_256(a, type == CSD_F16, st);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CSD_OK : csd::hip_fail(e, "csd_prompt_attend");
}

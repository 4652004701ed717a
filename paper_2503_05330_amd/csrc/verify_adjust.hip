// csd — logits as they are sampled from: penalties for repeated tokens, biases, masks.
//
// A workgroup takes a stretch of the vocabulary of one path, all its positions.  How often the prompt and the path have said each token of the
// stretch is counted in LDS once: bits 0 .. 29 of a token's word count what the path said before its newest tokens, bit 30 says that one
// of these is the token (then they are looked through up to the row's position), bit 31 that the prompt has it.  Most words are zero: such
// logits are copied, with their bias and bit of the mask.
#include "csd_launch.h"
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

constexpr uint32_t kNew = 1u << 30, kPrompt = 1u << 31;

template <class E>
__global__ __launch_bounds__(512) void adjust_kernel(csd_adjustment a, int32_t first_path, int32_t parts, int32_t per) {
  constexpr int kThreads = 512;
  extern __shared__ uint32_t words[];                    // of the stretch's tokens
  __shared__ int32_t newest[CSD_MAX_VERIFY_STEP];
  const int32_t path = first_path + blockIdx.x / (uint32_t)parts, part = blockIdx.x % (uint32_t)parts, p = path / a.n_paths;
  const int32_t from = part * per, size = a.vocab - from < per ? a.vocab - from : per;
  int32_t count = a.d_counts ? a.d_counts[path] : a.n;
  count = count < 0 ? 0 : count > a.n ? a.n : count;
  const bool penalties = a.d_penalties != nullptr;
  float repetition = 1, presence = 0, frequency = 0;
  int32_t before = 0, path_len = 0;                      // tokens before the newest ones; the newest: before .. before + count - 1, where they are there
  if (penalties) {
    repetition = a.d_penalties[3 * (int64_t)p];
    presence = a.d_penalties[3 * (int64_t)p + 1];
    frequency = a.d_penalties[3 * (int64_t)p + 2];
    for (int32_t x = threadIdx.x; x < per; x += kThreads) words[x] = 0;
    if (a.d_tokens) {
      path_len = a.d_path_len[path];
      path_len = path_len < 0 ? 0 : path_len > a.path_cap ? a.path_cap : path_len;
      before = path_len - count;
    }
    const int32_t* const said = a.d_tokens ? a.d_tokens + path * a.token_stride : nullptr;
    if (threadIdx.x < CSD_MAX_VERIFY_STEP) {
      const int32_t at = before + (int32_t)threadIdx.x;
      newest[threadIdx.x] = said && (int32_t)threadIdx.x < count && at >= 0 ? said[at] : -1;
    }
    __syncthreads();
    if (count) {
      for (int32_t x = threadIdx.x; x < before; x += kThreads) {
        const uint32_t v = (uint32_t)said[x] - (uint32_t)from;
        if (v < (uint32_t)size) atomicAdd(&words[v], 1u);
      }
      if (a.d_prompt) {
        int32_t length = a.d_prompt_len ? a.d_prompt_len[p] : a.prompt_cap;
        length = length < 0 ? 0 : length > a.prompt_cap ? a.prompt_cap : length;
        const int32_t* const prompt = a.d_prompt + p * a.prompt_stride;
        for (int32_t x = threadIdx.x; x < length; x += kThreads) {
          const uint32_t v = (uint32_t)prompt[x] - (uint32_t)from;
          if (v < (uint32_t)size) atomicOr(&words[v], kPrompt);
        }
      }
      if ((int32_t)threadIdx.x < count) {
        const uint32_t v = (uint32_t)newest[threadIdx.x] - (uint32_t)from;
        if (v < (uint32_t)size) atomicOr(&words[v], kNew);
      }
    }
    __syncthreads();
  }
  for (int32_t t = 0; t < a.n; ++t) {
    const int64_t row = (int64_t)path * a.n + t;
    const E* const x = static_cast<const E*>(a.d_logits) + row * a.logit_stride + from;
    E* const out = static_cast<E*>(a.d_out) + row * a.out_stride + from;
    const float* const bias = a.d_bias ? a.d_bias + p * a.bias_stride + from : nullptr;
    const uint32_t* const mask = a.d_mask ? a.d_mask + row * a.mask_stride : nullptr;
    for (int32_t v = threadIdx.x; v < size; v += kThreads) {
      float y = 0;
      if (t < count) {
        y = (float)x[v];
        if (penalties) {
          const uint32_t word = words[v];
          if (word) {
            int32_t times = word & (kNew - 1);
            if (word & kNew)
              for (int32_t i = 0; i <= t; ++i) times += newest[i] == from + v;
            if (times || (word & kPrompt)) y = y > 0 ? y / repetition : y * repetition;
            if (times) y -= frequency * (float)times + presence;
          }
        }
        if (bias) y += bias[v];
        if (mask && !(mask[(from + v) / 32] >> ((from + v) % 32) & 1)) y = -INFINITY;
      }
      out[v] = (E)y;
    }
  }
}

constexpr int32_t kMostLogits = 8192, kLeastLogits = 1024;

}  // namespace
}  // namespace verify
}  // namespace csd

extern "C" int csd_adjust(const csd_adjustment* adjustment, void* stream) {
  using namespace csd::verify;
  if (!adjustment) return CSD_ERR_INVALID_ARG;
  const csd_adjustment& a = *adjustment;
  if (a.n_problems <= 0 || a.n_paths <= 0 || a.n < 1 || a.n > CSD_MAX_VERIFY_STEP || a.vocab <= 0 || a.vocab > CSD_MAX_VOCAB) return CSD_ERR_INVALID_ARG;
  const int64_t paths = (int64_t)a.n_problems * a.n_paths;
  if (paths * a.n > CSD_MAX_TARGET_ROWS || a.type < CSD_BF16 || a.type > CSD_F32) return CSD_ERR_INVALID_ARG;
  const uintptr_t element = a.type == CSD_F32 ? 4 : 2;
  auto bad = [](const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  if (!a.d_logits || !a.d_out || bad(a.d_logits, element) || bad(a.d_out, element) || a.logit_stride < 0 || a.out_stride < 0) return CSD_ERR_INVALID_ARG;
  if (paths * a.n > 1 && a.out_stride < a.vocab) return CSD_ERR_INVALID_ARG;
  if (a.d_logits == a.d_out && paths * a.n > 1 && a.logit_stride != a.out_stride) return CSD_ERR_INVALID_ARG;
  for (const void* p : {(const void*)a.d_counts, (const void*)a.d_penalties, (const void*)a.d_tokens, (const void*)a.d_path_len, (const void*)a.d_prompt,
                        (const void*)a.d_prompt_len, (const void*)a.d_bias, (const void*)a.d_mask})
    if (bad(p, 4)) return CSD_ERR_INVALID_ARG;
  if (a.d_tokens && (!a.d_path_len || a.token_stride < 0 || a.path_cap < 0 || a.path_cap > CSD_MAX_CACHE_TOKENS)) return CSD_ERR_INVALID_ARG;
  if (a.d_prompt && (a.prompt_stride < 0 || a.prompt_cap < 0 || a.prompt_cap > CSD_MAX_CACHE_TOKENS)) return CSD_ERR_INVALID_ARG;
  if ((a.d_bias && a.bias_stride < 0) || (a.d_mask && a.mask_stride < 0)) return CSD_ERR_INVALID_ARG;
  // stretches: as long as leaves some 1024 workgroups
  int64_t parts = (1024 + paths - 1) / paths;
  const int64_t most = (a.vocab + kLeastLogits - 1) / kLeastLogits, least = (a.vocab + kMostLogits - 1) / kMostLogits;
  parts = parts < least ? least : parts > most ? most : parts;
  const int32_t per = (int32_t)(((a.vocab + parts - 1) / parts + 31) / 32 * 32);
  parts = (a.vocab + per - 1) / per;
  const uint32_t lds = a.d_penalties ? (uint32_t)per * 4 : 0;
  auto* kernel = a.type == CSD_BF16 ? adjust_kernel<__bf16> : a.type == CSD_F16 ? adjust_kernel<_Float16> : adjust_kernel<float>;
  const int64_t together = ((int64_t)1 << 22) / parts;                // paths of a launch of less than 2^32 threads
  for (int64_t first = 0; first < paths; first += together) {
    const int64_t here = paths - first < together ? paths - first : together;
    kernel<<<(uint32_t)(here * parts), 512, lds, static_cast<hipStream_t>(stream)>>>(a, (int32_t)first, (int32_t)parts, per);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CSD_OK : csd::hip_fail(e, "csd_adjust");
}

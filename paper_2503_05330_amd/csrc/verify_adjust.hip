// csd — logits as they are sampled from: penalties for repeated tokens, biases, masks.
//
// x -> x / r or x r where the token was said, - (frequency c + presence) where the path said it c times, + bias, -inf where masked.
//
// A workgroup takes a stretch of the vocabulary of one path, all its positions.  How often the prompt and the path have said each token of the
// stretch is counted in LDS once: bits 0 .. 29 of a token's word count what the path said before its newest tokens, bit 30 says that one
// of these is the token (then they are looked through up to the row's position), bit 31 that the prompt has it.  Most words are zero: such
// logits are copied, with their bias and bit of the mask.  Every workgroup of a path reads all of the prompt's and the path's tokens, from L2; the
// logits' first vectors are asked for before the counting.
//
// What bounds it: memory, and the counting where positions are few.  64 paths x up to 17 positions of 152064 in bfloat16, a prompt of 4096 tokens, paths
// of up to 4096, masks: 110 .. 119 us, 4.4 TB/s (a copy reaches 5.2); with all positions there 155, 133 without penalties.  1024 paths x 1 position
// 180; 166 without masks, 115 without penalties.  (Every lane reads the words of its eight logits at once: 70 .. 85 % of LDS's cycles are conflicts.)  3 x 13 x 5 of 50257
// in 32 bits, biases: 15.6 us, 4.1 TB/s; 4 x 32000: 5.5 us, a launch and three round trips.
#include "csd_verify.cuh"

namespace csd {
namespace verify {
namespace {

constexpr uint32_t kNew = 1u << 30, kPrompt = 1u << 31;

constexpr int kAdjustThreads = 512;                            // (256 .. 1024: no faster)

// Tokens that the workgroup looks at: the first few of each thread are asked for at once, so that they are on their way together with all else.
struct Tokens {
  typedef int32_t Four __attribute__((ext_vector_type(4), aligned(4)));
  static constexpr int kAhead = 3;
  const int32_t* from;
  int32_t length;
  Four first[kAhead];
  __device__ void ask(Four (&x)[kAhead], int32_t x0) const {
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int32_t at = x0 + s * kAdjustThreads;
      x[s] = 4 * at + 3 < length ? *reinterpret_cast<const Four*>(from + 4 * at) : Four{};
    }
  }
  __device__ Tokens(const int32_t* from, int32_t length) : from(from), length(length) { ask(first, threadIdx.x); }
  // calls f with each
  template <class F>
  __device__ void each(F f) const {
    const int32_t fours = length / 4;
    Four x[kAhead];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) x[s] = first[s];
    for (int32_t x0 = threadIdx.x; x0 < fours; x0 += kAhead * kAdjustThreads) {
      if (x0 != (int32_t)threadIdx.x) ask(x, x0);
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        if (x0 + s * kAdjustThreads >= fours) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) f((uint32_t)x[s][i]);
      }
    }
    if ((int32_t)threadIdx.x < length - 4 * fours) f((uint32_t)from[4 * fours + threadIdx.x]);
  }
};

template <class E>
__global__ __launch_bounds__(kAdjustThreads) void adjust_kernel(csd_adjustment a, int32_t first_path, int32_t parts, int32_t per) {
  extern __shared__ __align__(32) uint32_t words[];      // of the stretch's tokens
  __shared__ int32_t newest[CSD_MAX_VERIFY_STEP];
  const int32_t path = first_path + blockIdx.x / (uint32_t)parts, part = blockIdx.x % (uint32_t)parts, p = path / a.n_paths;
  const int32_t from = part * per, size = a.vocab - from < per ? a.vocab - from : per;
  int32_t count = a.d_counts ? a.d_counts[path] : a.n;
  count = count < 0 ? 0 : count > a.n ? a.n : count;
  const bool penalties = a.d_penalties != nullptr;
  float repetition = 1, presence = 0, frequency = 0;
  int32_t before = 0;                                    // tokens before the newest ones, which are before .. before + count - 1, where they are there
  const int32_t* said = nullptr;
  if (penalties && count && a.d_tokens) {
    int32_t path_len = a.d_path_len[path];
    path_len = path_len < 0 ? 0 : path_len > a.path_cap ? a.path_cap : path_len;
    before = path_len - count;
    said = a.d_tokens + path * a.token_stride;
  }
  int32_t length = 0;
  if (penalties && count && a.d_prompt) {
    length = a.d_prompt_len ? a.d_prompt_len[p] : a.prompt_cap;
    length = length < 0 ? 0 : length > a.prompt_cap ? a.prompt_cap : length;
  }
  const Tokens path_tokens(said, before), prompt_tokens(a.d_prompt + p * a.prompt_stride, length);

  const float* const bias = a.d_bias ? a.d_bias + p * a.bias_stride + from : nullptr;
  const int64_t first_row = (int64_t)path * a.n;
  const E* const in = static_cast<const E*>(a.d_logits) + first_row * a.logit_stride + from;
  E* const out = static_cast<E*>(a.d_out) + first_row * a.out_stride + from;
  // bit i: logit at + i of row t may be picked (at: a multiple of eight, from the stretch's first)
  const auto allowed = [&](int32_t t, int32_t at) -> uint32_t {
    return a.d_mask ? reinterpret_cast<const uint8_t*>(a.d_mask + (first_row + t) * a.mask_stride)[(from + at) / 8] : 0xff;
  };
  typedef E Eight __attribute__((ext_vector_type(8), aligned(sizeof(E))));
  typedef float EightFloats __attribute__((ext_vector_type(8), aligned(4)));
  typedef uint32_t EightWords __attribute__((ext_vector_type(8)));
  constexpr int kAhead = 2;
  const int32_t eights = size / 8, all = count * eights;
  Eight x[kAhead];
  uint32_t bits[kAhead];
  int32_t t[kAhead], at[kAhead];
  const auto ask = [&](int32_t x0) {
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int32_t item = x0 + s * kAdjustThreads < all ? x0 + s * kAdjustThreads : x0;
      t[s] = item / eights;
      at[s] = 8 * (item - t[s] * eights);
      x[s] = *reinterpret_cast<const Eight*>(in + t[s] * a.logit_stride + at[s]);
      bits[s] = allowed(t[s], at[s]);
    }
  };
  if ((int32_t)threadIdx.x < all) ask(threadIdx.x);

  if (penalties) {
    repetition = a.d_penalties[3 * (int64_t)p];
    presence = a.d_penalties[3 * (int64_t)p + 1];
    frequency = a.d_penalties[3 * (int64_t)p + 2];
    for (int32_t x = threadIdx.x; x < per / 4; x += kAdjustThreads) reinterpret_cast<uint4*>(words)[x] = uint4{};
    if (threadIdx.x < CSD_MAX_VERIFY_STEP) {
      const int32_t at = before + (int32_t)threadIdx.x;
      newest[threadIdx.x] = said && (int32_t)threadIdx.x < count && at >= 0 ? said[at] : -1;
    }
    __syncthreads();
    path_tokens.each([&](uint32_t token) {
      const uint32_t v = token - (uint32_t)from;
      if (v < (uint32_t)size) atomicAdd(&words[v], 1u);
    });
    prompt_tokens.each([&](uint32_t token) {
      const uint32_t v = token - (uint32_t)from;
      if (v < (uint32_t)size) atomicOr(&words[v], kPrompt);
    });
    if ((int32_t)threadIdx.x < count) {
      const uint32_t v = (uint32_t)newest[threadIdx.x] - (uint32_t)from;
      if (v < (uint32_t)size) atomicOr(&words[v], kNew);
    }
    __syncthreads();
  }
  const auto adjusted = [&](float y, uint32_t word, int32_t t, int32_t v) {
    int32_t times = word & (kNew - 1);
    if (word & kNew)
      for (int32_t i = 0; i <= t; ++i) times += newest[i] == v;
    if (times || (word & kPrompt)) y = y > 0 ? y / repetition : y * repetition;
    if (times) y -= frequency * (float)times + presence;
    return y;
  };
  for (int32_t x0 = threadIdx.x; x0 < all; x0 += kAhead * kAdjustThreads) {
    if (x0 != (int32_t)threadIdx.x) ask(x0);
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      if (x0 + s * kAdjustThreads >= all) break;
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = (float)x[s][i];
      if (penalties) {
        const EightWords word = *reinterpret_cast<const EightWords*>(words + at[s]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (word[i]) y[i] = adjusted(y[i], word[i], t[s], from + at[s] + i);
      }
      if (bias) {
        const EightFloats b = *reinterpret_cast<const EightFloats*>(bias + at[s]);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] += b[i];
      }
      Eight z;
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = (E)(bits[s] >> i & 1 ? y[i] : -INFINITY);
      *reinterpret_cast<Eight*>(out + t[s] * a.out_stride + at[s]) = z;
    }
  }
  // the vocabulary's last few, and the rows of positions that there are none of
  const int32_t rest = size % 8;
  if ((int32_t)threadIdx.x < count * rest) {
    const int32_t t = threadIdx.x / rest, i = threadIdx.x - t * rest, at = eights * 8 + i;
    float y = (float)in[t * a.logit_stride + at];
    if (penalties && words[at]) y = adjusted(y, words[at], t, from + at);
    if (bias) y += bias[at];
    out[t * a.out_stride + at] = (E)(allowed(t, eights * 8) >> i & 1 ? y : -INFINITY);
  }
  for (int32_t t = count; t < a.n; ++t) {
    for (int32_t x = threadIdx.x; x < eights; x += kAdjustThreads) *reinterpret_cast<Eight*>(out + t * a.out_stride + 8 * x) = Eight{};
    if ((int32_t)threadIdx.x < rest) out[t * a.out_stride + eights * 8 + threadIdx.x] = (E)0.0f;
  }
}

constexpr int32_t kLeastStretch = 1024;

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
  // Stretches: as long as leaves some 1024 workgroups, up to a bound.  Short ones read and count the tokens more often, which weighs with few positions;
  // long ones have more in LDS, and fewer workgroups a CU.  us with 2048, 4096 and 8192 logits, vocabulary 152064, 4096 + 4096 tokens, masks:
  // 1024 paths x 1 position 373, 261, 180; 256 x 4 141, 116, 114; 128 x 8 107, 110, 119; 64 x 17 117, 130, 146.
  const int32_t longest = a.n <= 4 ? 8192 : a.n < 8 ? 4096 : 2048;
  int64_t parts = (1024 + paths - 1) / paths;
  const int64_t most = (a.vocab + kLeastStretch - 1) / kLeastStretch, least = (a.vocab + longest - 1) / longest;
  parts = parts < least ? least : parts > most ? most : parts;
  const int32_t per = (int32_t)(((a.vocab + parts - 1) / parts + 31) / 32 * 32);
  parts = (a.vocab + per - 1) / per;
  const uint32_t lds = a.d_penalties ? (uint32_t)per * 4 : 0;
  auto* kernel = a.type == CSD_BF16 ? adjust_kernel<__bf16> : a.type == CSD_F16 ? adjust_kernel<_Float16> : adjust_kernel<float>;
  const int64_t together = ((int64_t)1 << 22) / parts;                // paths of a launch of less than 2^32 threads
  for (int64_t first = 0; first < paths; first += together) {
    const int64_t here = paths - first < together ? paths - first : together;
    kernel<<<(uint32_t)(here * parts), kAdjustThreads, lds, static_cast<hipStream_t>(stream)>>>(a, (int32_t)first, (int32_t)parts, per);
  }
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CSD_OK : csd::hip_fail(e, "csd_adjust");
}

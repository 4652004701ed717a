// csd — attention of whole prompts, heads of 128.
#include "csd_prompt.cuh"

namespace csd {
namespace verify {

void prompt_128(const PromptArgs& a, bool f16, hipStream_t st) { prompt_of<128>(a, f16, st); }

}  // namespace verify
}  // namespace csd

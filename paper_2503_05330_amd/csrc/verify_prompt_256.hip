// csd — attention of whole prompts, heads of 256.
#include "csd_prompt.cuh"

namespace csd {
namespace verify {

void prompt_256(const PromptArgs& a, bool f16, hipStream_t st) { prompt_of<256>(a, f16, st); }

}  // namespace verify
}  // namespace csd

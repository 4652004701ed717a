// csd — attention over the cache, heads of 64.
#include "csd_attend_rows.cuh"

namespace csd {
namespace verify {

void attend_64(const AttendArgs& a, const AttendLaunch& how, hipStream_t st) { attend_of<64>(a, how, st); }

}  // namespace verify
}  // namespace csd

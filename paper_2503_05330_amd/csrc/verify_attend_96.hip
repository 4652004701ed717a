// csd — attention over the cache, heads of 96.
#include "csd_attend_rows.cuh"

namespace csd {
namespace verify {

void attend_96(const AttendArgs& a, const AttendLaunch& how, hipStream_t st) { attend_of<96>(a, how, st); }

}  // namespace verify
}  // namespace csd

// csd — attention over the cache, heads of 256.
#include "csd_attend_rows.cuh"

namespace csd {
namespace verify {

void attend_256(const AttendArgs& a, const AttendLaunch& how, hipStream_t st) { attend_of<256>(a, how, st); }

}  // namespace verify
}  // namespace csd

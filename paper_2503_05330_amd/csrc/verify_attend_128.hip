// csd — attention over the cache, heads of 128.
#include "csd_attend_rows.cuh"

namespace csd {
namespace verify {

void attend_128(const AttendArgs& a, const AttendLaunch& how, hipStream_t st) { attend_of<128>(a, how, st); }

}  // namespace verify
}  // namespace csd

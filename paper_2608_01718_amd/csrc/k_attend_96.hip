// k_attend_96.hip -- the attention kernels of heads padded to 96 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<96, kWhole>(const AttendArgs&, const AttendPlan&, hipStream_t);
}  // namespace lacache

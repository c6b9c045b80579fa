// k_attend_128.hip -- the attention kernels of heads padded to 128 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<128, kWhole>(const AttendArgs&, const AttendPlan&, hipStream_t);
}  // namespace lacache

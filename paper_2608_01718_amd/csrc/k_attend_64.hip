// k_attend_64.hip -- the attention kernels of heads padded to 64 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<64, kWhole>(const AttendArgs&, const AttendPlan&, hipStream_t);
}  // namespace lacache

// k_attend_256.hip -- the attention kernels of heads padded to 256 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<256, kWhole>(const AttendArgs&, const AttendPlan&, hipStream_t);
}  // namespace lacache

// k_attend_192.hip -- the attention kernels of heads padded to 192 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<192, kWhole>(const AttendArgs&, const AttendPlan&, hipStream_t);
}  // namespace lacache

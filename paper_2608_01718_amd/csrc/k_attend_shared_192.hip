// k_attend_shared_192.hip -- the attention kernels of batches that share prefixes, heads padded to 192 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<192, kPrefix>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend<192, kOwn>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
}  // namespace lacache

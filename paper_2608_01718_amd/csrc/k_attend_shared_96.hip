// k_attend_shared_96.hip -- the attention kernels of batches that share prefixes, heads padded to 96 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<96, kPrefix>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend<96, kOwn>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend_both<96>(const AttendArgs&, const AttendPartPlan&, const AttendPartPlan&, hipStream_t);
}  // namespace lacache

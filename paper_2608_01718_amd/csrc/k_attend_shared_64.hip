// k_attend_shared_64.hip -- the attention kernels of batches that share prefixes, heads padded to 64 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<64, kPrefix>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend<64, kOwn>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend_both<64>(const AttendArgs&, const AttendPartPlan&, const AttendPartPlan&, hipStream_t);
}  // namespace lacache

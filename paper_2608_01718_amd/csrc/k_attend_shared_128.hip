// k_attend_shared_128.hip -- the attention kernels of batches that share prefixes, heads padded to 128 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<128, kPrefix>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend<128, kOwn>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend_both<128>(const AttendArgs&, const AttendPartPlan&, const AttendPartPlan&, hipStream_t);
}  // namespace lacache

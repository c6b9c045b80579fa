// k_attend_shared_256.hip -- the attention kernels of batches that share prefixes, heads padded to 256 columns.
#include "attend_wide.hpp"

namespace lacache {
template hipError_t launch_attend<256, kPrefix>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
template hipError_t launch_attend<256, kOwn>(const AttendArgs&, const AttendPartPlan&, hipStream_t);
}  // namespace lacache

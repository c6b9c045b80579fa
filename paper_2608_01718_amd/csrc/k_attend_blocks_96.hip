// k_attend_blocks_96.hip -- attention over lists of pages, heads padded to 96 columns.
#include "attend_blocks.hpp"

namespace lacache {
template hipError_t launch_blocks<96>(const BlocksArgs&, int64_t, hipStream_t);
}  // namespace lacache

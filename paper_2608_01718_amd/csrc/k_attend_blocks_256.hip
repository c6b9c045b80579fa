// k_attend_blocks_256.hip -- attention over lists of pages, heads padded to 256 columns.
#include "attend_blocks.hpp"

namespace lacache {
template hipError_t launch_blocks<256>(const BlocksArgs&, int64_t, hipStream_t);
}  // namespace lacache

// k_attend_blocks_64.hip -- attention over lists of pages, heads padded to 64 columns.
#include "attend_blocks.hpp"

namespace lacache {
template hipError_t launch_blocks<64>(const BlocksArgs&, int64_t, hipStream_t);
}  // namespace lacache

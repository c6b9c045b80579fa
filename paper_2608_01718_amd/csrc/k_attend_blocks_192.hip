// k_attend_blocks_192.hip -- attention over lists of pages, heads padded to 192 columns.
#include "attend_blocks.hpp"

namespace lacache {
template hipError_t launch_blocks<192>(const BlocksArgs&, int64_t, hipStream_t);
}  // namespace lacache

// k_attend_blocks_128.hip -- attention over lists of pages, heads padded to 128 columns.
#include "attend_blocks.hpp"

namespace lacache {
template hipError_t launch_blocks<128>(const BlocksArgs&, int64_t, hipStream_t);
}  // namespace lacache

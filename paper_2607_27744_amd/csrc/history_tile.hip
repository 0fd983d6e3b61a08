// The tiled history attention over K/V in bf16.
#include "history_tile.h"

namespace rocs {

hipError_t launch_history_tile(const HistArgs& a, hipStream_t s) { return launch_tile<false>(a, s); }

}  // namespace rocs

// The kernel for the shared rows of groups with many rows, head_dim 64, 8-bit cache.
#include "attend_many.h"

namespace codecomp { template int launch_many_shared_of<64, true>(const ManyArgs&, hipStream_t); }

// The kernel for the shared rows of groups with many rows, head_dim 64, bf16 cache.
#include "attend_many.h"

namespace codecomp { template int launch_many_shared_of<64, false>(const ManyArgs&, hipStream_t); }

// The kernel for the shared rows of groups with many rows, head_dim 128, bf16 cache.
#include "attend_many.h"

namespace codecomp { template int launch_many_shared_of<128, false>(const ManyArgs&, hipStream_t); }

#include "attend_many.h"

namespace codecomp {
template int launch_many_of<64, false>(const ManyArgs&, hipStream_t);
}

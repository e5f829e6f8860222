#include "attend_many.h"

namespace codecomp {
template int launch_many_of<128, false>(const ManyArgs&, hipStream_t);
}

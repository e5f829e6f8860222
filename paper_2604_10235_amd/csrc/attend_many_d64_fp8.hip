#include "attend_many.h"

namespace codecomp {
template int launch_many_of<64, true>(const ManyArgs&, hipStream_t);
}

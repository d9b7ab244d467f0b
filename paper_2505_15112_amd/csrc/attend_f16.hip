// attend_f16.hip -- the walk of linear attention for f16 activations.
#include "attend_walk.hpp"

namespace ls {
template hipError_t launch_walk<_Float16>(const Walks&, bool, hipStream_t);
}  // namespace ls

// attend_f32.hip -- the walk of linear attention for f32 activations.
#include "attend_walk.hpp"

namespace ls {
template hipError_t launch_walk<float>(const Walks&, bool, hipStream_t);
}  // namespace ls

// attend_bf16.hip -- the walk of linear attention for bf16 activations.
#include "attend_walk.hpp"

namespace ls {
template hipError_t launch_walk<__bf16>(const Walks&, bool, hipStream_t);
}  // namespace ls

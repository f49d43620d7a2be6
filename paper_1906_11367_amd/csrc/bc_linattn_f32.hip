// The walk of linear attention on fp32 tensors.
#include "bc_linattn_walk.hpp"

namespace bc {
namespace linattn {
hipError_t launch_walk_f32(const Walk& w, const Walk* beside, hipStream_t s) { return launch_walk_dt<kF32>(w, beside, s); }
}  // namespace linattn
}  // namespace bc

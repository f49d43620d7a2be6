// The walk of linear attention on fp32 tensors.
#include "bc_linattn_walk.hpp"

namespace bc {
namespace linattn {
hipError_t launch_decays_f32(const DecayArgs& a, hipStream_t s) { return launch_decays_dt<kF32>(a, s); }
hipError_t launch_walk_f32(const Walk& w, hipStream_t s) { return launch_walk_dt<kF32>(w, s); }
}  // namespace linattn
}  // namespace bc

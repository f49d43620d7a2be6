// The walk of linear attention on bf16 tensors.
#include "bc_linattn_walk.hpp"

namespace bc {
namespace linattn {
hipError_t launch_decays_bf16(const DecayArgs& a, hipStream_t s) { return launch_decays_dt<kBF16>(a, s); }
hipError_t launch_walk_bf16(const Walk& w, hipStream_t s) { return launch_walk_dt<kBF16>(w, s); }
}  // namespace linattn
}  // namespace bc

// The walk of linear attention on bf16 tensors.
#include "bc_linattn_walk.hpp"

namespace bc {
namespace linattn {
hipError_t launch_walk_bf16(const Walk& w, const Walk* beside, hipStream_t s) { return launch_walk_dt<kBF16>(w, beside, s); }
}  // namespace linattn
}  // namespace bc

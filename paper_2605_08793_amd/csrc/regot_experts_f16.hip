// Products grouped by expert, of numbers of type f16.
#include "regot_experts_launch.hpp"

namespace regot {
void expert_tiles_f16(const GroupArgs &A, const TilePlan &P, hipStream_t s) { launch_tiles<REGOT_F16>(A, P, s); }
}  // namespace regot

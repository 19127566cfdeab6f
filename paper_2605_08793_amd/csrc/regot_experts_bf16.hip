// Products grouped by expert, of numbers of type bf16.
#include "regot_experts_launch.hpp"

namespace regot {
void expert_tiles_bf16(const GroupArgs &A, const TilePlan &P, hipStream_t s) { launch_tiles<REGOT_BF16>(A, P, s); }
}  // namespace regot

// fp32 instances of the attention weights' kernels.
#include "mass_kernel.h"

namespace ftcnn {

hipError_t launch_mass_f32(const MassPlan &pl, const MassArgs &a, hipStream_t st) { return mass_pick<float>(pl, a, st); }

}  // namespace ftcnn

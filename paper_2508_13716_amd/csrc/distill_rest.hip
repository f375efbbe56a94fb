// capgnn_distill's kernels with the teacher's remaining probability as one more outcome.  (A file of their own: with all sixteen sets in one
// the compiler gave some of them a kilobyte of scratch memory a thread.)
#include "distill.h"

namespace capgnn {

DistillLaunch distill_launch_rest(bool z_bf16, bool dz_bf16) { return distill_launch_of<true>(z_bf16, dz_bf16); }

}  // namespace capgnn

// Direct-to-LDS products of 16-bit matrices: FORM_KK, END_SCORES_GRAD.
#include "linear_pp_kernel.h"
namespace mg {
hipError_t launch_linear_dma_kk_scores_grad(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream) { return launch_linear_dma<FORM_KK, END_SCORES_GRAD>(dtype, tile, args, slices, stream); }
}  // namespace mg

// Direct-to-LDS products of 16-bit matrices: FORM_NN, END_STORE.
#include "linear_pp_kernel.h"
namespace mg {
hipError_t launch_linear_dma_nn_store(int dtype, int tile, const LinearArgs &args, int slices, hipStream_t stream) { return launch_linear_dma<FORM_NN, END_STORE>(dtype, tile, args, slices, stream); }
}  // namespace mg

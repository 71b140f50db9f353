// 8-bit operands straight into LDS (block_dma_kernel.h): sums over experts' rows.
#include "internal.h"
#include "block_dma_kernel.h"
namespace mg {
hipError_t launch_block_dma_sum(const BlockArgs &args, int sums, int tile, hipStream_t stream) { return launch_block_dma<BLOCK_SUM>(args, sums, tile, stream); }
}  // namespace mg

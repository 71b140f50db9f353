// 8-bit operands straight into LDS (block_dma_kernel.h): the products of rows that belong to experts.
#include "internal.h"
#include "block_dma_kernel.h"
namespace mg {
hipError_t launch_block_dma_rows(const BlockArgs &args, int sums, int tile, hipStream_t stream) { return launch_block_dma<BLOCK_ROWS>(args, sums, tile, stream); }
}  // namespace mg

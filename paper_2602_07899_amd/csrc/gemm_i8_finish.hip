// Products of activation codes with weight codes on int8 MFMA with a bias, an activation and a second matrix behind them: the
// tiles of gemm_i8.hip with another epilogue.  The classes of activations are kernels of their own: an activation is written out for
// each of a lane's 64 to 160 outputs, and code that a tile runs once is fetched cold.
#include "contraction.h"

namespace tlq {

template <int NSTAGE, int CLASS, int HALVES, int JB>
__global__ __launch_bounds__(HALVES * 256) void gemm_i8_finish_kernel(GemmDev a) {
  gemm_dma_body<Int8, NSTAGE, EPI_FINISH + CLASS, false, false, HALVES, JB>(a);
}

template <int CLASS>
static hipError_t launch(const GemmDev& d, GemmTile tile, unsigned blocks, hipStream_t stream) {
  if (!tile.small && tile.tok_blocks == 3) gemm_i8_finish_kernel<2, CLASS, 2, 3><<<blocks, 512, 0, stream>>>(d);
  else if (!tile.small && tile.tok_blocks == 5) gemm_i8_finish_kernel<2, CLASS, 2, 5><<<blocks, 512, 0, stream>>>(d);
  else if (!tile.small) gemm_i8_finish_kernel<2, CLASS, 2, 4><<<blocks, 512, 0, stream>>>(d);
  else if ((int64_t)d.tiles_o * d.tiles_t <= 256) gemm_i8_finish_kernel<4, CLASS, 1, 4><<<blocks, 256, 0, stream>>>(d);
  else gemm_i8_finish_kernel<2, CLASS, 1, 4><<<blocks, 256, 0, stream>>>(d);
  return hipGetLastError();
}

hipError_t launch_dma_i8_finish(const GemmDev& d, GemmTile tile, unsigned blocks, hipStream_t stream) {
  const int c = act_class(d.fin.act);
  if (c == kActNone) return launch<kActNone>(d, tile, blocks, stream);
  return c == kActErf ? launch<kActErf>(d, tile, blocks, stream) : launch<kActGate>(d, tile, blocks, stream);
}

}  // namespace tlq

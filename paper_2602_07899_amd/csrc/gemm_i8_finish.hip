// Products of activation codes with weight codes on int8 MFMA with a bias, an activation and a second matrix behind them: the
// tiles of gemm_i8.hip with another epilogue.  Activations are kernels of their own: an activation is written out for
// each of a lane's 32 to 160 outputs, and code that a tile runs once is fetched cold.  Bound by the matrix instructions and the
// LDS reads that feed them, as without an epilogue: 10,240 x 5120 x 13824 with SiLU and a second matrix 647 us behind other work, 2.24
// POP/s (a large library product of codes reaches 2.01; the second matrix adds 283 MB).  By latency where
// tiles are few; then they are 128 x 64, one a CU, as in gemm_half.hip: 128 x 128 and these, us, tokens x channels x outputs:
// 613 x 1096 x 1399 14.4 9.7, 512 x 1024 x 1024 10.8 7.7, 300 x 4096 x 2048 26.6 16.9, 8000 x 1096 x 250 19.1 12.3; 288 of
// them would be a second round, 1100 x 1000 x 2000 stays 15.5.
#include "contraction.h"

namespace tlq {

template <int NSTAGE, int ACT, int HALVES, int JB>
__global__ __launch_bounds__(HALVES * 256) void gemm_i8_finish_kernel(GemmDev a) {
  gemm_dma_body<Int8, NSTAGE, EPI_FINISH + ACT, false, false, HALVES, JB>(a);
}

template <int ACT>
static hipError_t launch(const GemmDev& d, GemmTile tile, unsigned blocks, hipStream_t stream) {
  if (!tile.small && tile.tok_blocks == 3) gemm_i8_finish_kernel<2, ACT, 2, 3><<<blocks, 512, 0, stream>>>(d);
  else if (!tile.small && tile.tok_blocks == 5) gemm_i8_finish_kernel<2, ACT, 2, 5><<<blocks, 512, 0, stream>>>(d);
  else if (!tile.small) gemm_i8_finish_kernel<2, ACT, 2, 4><<<blocks, 512, 0, stream>>>(d);
  else if (tile.tok_blocks == 2) gemm_i8_finish_kernel<4, ACT, 1, 2><<<blocks, 256, 0, stream>>>(d);
  else if ((int64_t)d.tiles_o * d.tiles_t <= 256) gemm_i8_finish_kernel<4, ACT, 1, 4><<<blocks, 256, 0, stream>>>(d);
  else gemm_i8_finish_kernel<2, ACT, 1, 4><<<blocks, 256, 0, stream>>>(d);
  return hipGetLastError();
}

hipError_t launch_dma_i8_finish(const GemmDev& d, GemmTile tile, unsigned blocks, hipStream_t stream) {
  switch (d.fin.act) {
    case TLQ_ACT_NONE: return launch<kActNone>(d, tile, blocks, stream);
    case TLQ_ACT_SILU: return launch<kActSilu>(d, tile, blocks, stream);
    case TLQ_ACT_GELU_TANH: return launch<kActTanh>(d, tile, blocks, stream);
    default: return launch<kActErf>(d, tile, blocks, stream);
  }
}

}  // namespace tlq

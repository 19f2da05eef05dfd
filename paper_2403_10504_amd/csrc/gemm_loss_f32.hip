// gemm_dl instantiations with the loss epilogues: fp32 tiles.
#include "gemm_dl.h"

namespace atom {

hipError_t gemm_loss_f32_64(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s) {
  return dl::launch_loss<float, 64, 64>(g, akc, bkc, epi, s);
}
hipError_t gemm_loss_f32_32(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s) {
  return dl::launch_loss<float, 32, 32>(g, akc, bkc, epi, s);
}

}  // namespace atom

// gemm_dl instantiations with the loss epilogues: 64x64 tiles.
#include "gemm_dl.h"

namespace atom {

hipError_t gemm_loss_64(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s) {
  return dl::launch_loss<bf16_t, 64, 64>(g, akc, bkc, epi, s);
}

}  // namespace atom

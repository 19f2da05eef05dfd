// gemm_dl instantiations for fp32 operands in three bf16 planes: 256x192 tiles.
#include "gemm_dl.h"

namespace atom {

hipError_t gemm_planes_192(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s) {
  return dl::launch_planes<256, 192>(g, akc, bkc, epi, s);
}

}  // namespace atom

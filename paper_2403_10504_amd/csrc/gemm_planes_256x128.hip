// gemm_dl instantiations for fp32 operands in three bf16 planes: 256x128 tiles.
#include "gemm_dl.h"

namespace atom {

hipError_t gemm_planes_256x128(const GemmArgs& g, bool akc, bool bkc, int epi, hipStream_t s) {
  return dl::launch_planes<256, 128>(g, akc, bkc, epi, s);
}

}  // namespace atom

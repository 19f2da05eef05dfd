// gemm_dl instantiations for the Newton-Schulz products: 64x64 tiles.
#include "gemm_dl.h"

namespace atom {

hipError_t gemm_ns_64(const GemmArgs& g, int planes, int batch, bool akc, bool bkc, int epi, hipStream_t s) {
  return planes == 1 ? dl::launch_ns<64, 1>(g, batch, akc, bkc, epi, s) : dl::launch_ns<64, 3>(g, batch, akc, bkc, epi, s);
}

}  // namespace atom

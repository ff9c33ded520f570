// The product of 8-bit codes, int32 partials of pieces of K.
#include "gemm_i8.hpp"

namespace hxf {

hipError_t gemm_i8_split(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
  return launch_i8_cfg<EPI_F32, true>(a, p, st);
}

}  // namespace hxf

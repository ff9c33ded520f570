// The product of 8-bit codes with a gate and an up weight, int32 partials of pieces of K.
#include "gemm_i8.hpp"

namespace hxf {

hipError_t gemm_i8_split_swiglu(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
  return launch_i8_cfg<EPI_SWIGLU, true>(a, p, st);
}

}  // namespace hxf

// The product of 8-bit codes, SwiGLU of a gate and an up weight.
#include "gemm_i8.hpp"

namespace hxf {

hipError_t gemm_i8_swiglu(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
  return launch_i8_cfg<EPI_SWIGLU, false>(a, p, st);
}

}  // namespace hxf

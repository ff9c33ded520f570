// The product of 8-bit codes, fp32 output.
#include "gemm_i8.hpp"

namespace hxf {

hipError_t gemm_i8_f32(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
  return launch_i8_cfg<EPI_F32, false>(a, p, st);
}

}  // namespace hxf

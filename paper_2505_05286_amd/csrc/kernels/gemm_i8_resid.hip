// The product of 8-bit codes, added to an fp32 residual.
#include "gemm_i8.hpp"

namespace hxf {

hipError_t gemm_i8_resid(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
  return launch_i8_cfg<EPI_RESID, false>(a, p, st);
}

}  // namespace hxf

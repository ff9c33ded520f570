// The product of 8-bit codes, bf16 output.
#include "gemm_i8.hpp"

namespace hxf {

hipError_t gemm_i8_bf16(const GemmI8Args& a, const GemmI8Plan& p, hipStream_t st) {
  return launch_i8_cfg<EPI_BF16, false>(a, p, st);
}

}  // namespace hxf

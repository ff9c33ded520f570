// What the launches of the 8-bit cache's operators hold, at the limits that the header states: threads of a dimension
// under 2^32, counts of them exact.
#include <cstdio>
#include <cstdlib>

#include "kernels/kernels.hpp"

using namespace hxf;

#define CHECK(c)                                         \
  do {                                                   \
    if (!(c)) {                                          \
      std::printf("line %d: %s\n", __LINE__, #c);        \
      std::exit(1);                                      \
    }                                                    \
  } while (0)

int main() {
  const int64_t k28 = int64_t(1) << 28, k26 = int64_t(1) << 26, k24 = int64_t(1) << 24;
  CHECK(launch_fits(k24 - 1, 256) && !launch_fits(k24, 256));
  CHECK(kv8_write_fits(k28 - 16, 1, 1) && !kv8_write_fits(k28 - 15, 1, 1));
  CHECK(kv8_write_fits(1, 65533, 1) && !kv8_write_fits(1, 65534, 1) && !kv8_write_fits(1, int64_t(1) << 30, int64_t(1) << 30));
  // decode: a wavefront for each item; heads four to a workgroup of the join, which short tables do without
  CHECK(kv8_decode_fits(k26 - 3073, 1) && !kv8_decode_fits(k26 - 3072, 1));
  CHECK(kv8_decode_fits((k26 - 3073) / 8, 8) && !kv8_decode_fits(k26 / 8, 8));
  CHECK(kv8_decode_join_fits(k24 - 1, 4, 9) && !kv8_decode_join_fits(k24, 1, 9) && kv8_decode_join_fits(k24, 4, 8));
  CHECK(kv8_decode_join_fits(k24 / 8 - 1, 32, 1000) && !kv8_decode_join_fits(k24 / 8, 32, 1000));
  // prefill: four wavefronts for each unit and head
  CHECK(kv8_prefill_fits(k24 - 2, 0, 128, 1) && !kv8_prefill_fits(k24 - 1, 0, 128, 1));
  CHECK(kv8_prefill_fits(1000, 32 * (k24 / 8 - 1002), 32, 8) && !kv8_prefill_fits(1000, 32 * (k24 / 8 - 1001), 32, 8));
  std::puts("ok");
}

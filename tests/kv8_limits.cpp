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
  CHECK(kv8_decode_fits(k26 - kKv8Resident - 1, 1) && !kv8_decode_fits(k26 - kKv8Resident, 1));
  CHECK(kv8_decode_fits((k26 - kKv8Resident - 1) / 8, 8) && !kv8_decode_fits(k26 / 8, 8));
  CHECK(kv8_decode_join_fits(k24 - 1, 4, 9) && !kv8_decode_join_fits(k24, 1, 9) && kv8_decode_join_fits(k24, 4, 8));
  CHECK(kv8_decode_join_fits(k24 / 8 - 1, 32, 1000) && !kv8_decode_join_fits(k24 / 8, 32, 1000));
  // prefill: four wavefronts for each unit and head
  CHECK(kv8_prefill_fits(k24 - 2, 0, 128, 1) && !kv8_prefill_fits(k24 - 1, 0, 128, 1));
  CHECK(kv8_prefill_fits(1000, 32 * (k24 / 8 - 1002), 32, 8) && !kv8_prefill_fits(1000, 32 * (k24 / 8 - 1001), 32, 8));
  // the planning launch's blocks where row0 goes up and down between 0 and T: S / 2 sequences of T rows
  const int64_t S = 1 << 15, T = 1 << 20;
  const int q = 8, cap = (int)kv8_prefill_unit_cap(S, T, q, 1);
  int64_t all = 0;
  int base = 0;
  for (int64_t s = 0; s < S; s += 256) {
    const int more = (int)(128 * (T / q));
    all += more;
    base += kv8_prefill_take(base, more, cap);
    CHECK(base >= 0 && base <= cap);
  }
  CHECK(all > INT32_MAX && base == cap);
  // and where it ascends: all of them, whatever the lengths are
  for (int64_t n = 1; n < 3000; n = n * 3 + 1) {
    const int64_t rows = n * 300, blocks = 300 * ((n + q - 1) / q);
    CHECK(kv8_prefill_take(0, (int)blocks, (int)kv8_prefill_unit_cap(300, rows, q, 8)) == blocks);
  }
  std::puts("ok");
}

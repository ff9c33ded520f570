// The work splits of the 8-bit cache's attention, as its kernels make them, over many batches: every page and every
// key tile once, and never more items, units and slots than the launch and the workspace hold.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "kernels/kernels.hpp"

using namespace hxf;

#define CHECK(c)                                                      \
  do {                                                                \
    if (!(c)) {                                                       \
      std::printf("line %d: %s (case %d)\n", __LINE__, #c, g_case);   \
      std::exit(1);                                                   \
    }                                                                 \
  } while (0)

static int g_case = 0;

static void decode(const std::vector<int>& pages, int hkv) {
  const int64_t S = (int64_t)pages.size();
  int64_t total = 0, items = 0;
  int longest = 0;
  for (int p : pages) total += p, longest = std::max(longest, p);
  const int64_t t = kv8_target_pages(total, S, hkv, longest);
  CHECK(t >= (longest <= kKv8WholePages ? longest : kKv8MinPages));   // short tables: no stream is cut
  const int target = (int)std::min<int64_t>(t, int64_t(1) << 27);
  for (int p : pages) {
    const int n = kv8_parts(p, target);
    CHECK((n == 0) == (p == 0));
    if (p == 0) continue;
    const int len = (p + n - 1) / n;
    CHECK(len == kv8_part_pages(p, target) && (len <= target || (int64_t)len * len <= p / 8));
    CHECK((int64_t)(n - 1) * len < p && (int64_t)n * len >= p);   // no part is empty, and all are covered
    items += (int64_t)n * hkv;
  }
  CHECK(items <= kv8_decode_items(S, hkv));
}

static void prefill(const std::vector<int>& rows, const std::vector<int64_t>& pos, int hkv, int group, int64_t pad) {
  const int q = kPrefillPairs / group;
  int64_t T = pad, blocks = 0;
  std::vector<int> all;
  for (size_t s = 0; s < rows.size(); ++s) {
    T += rows[s];
    for (int r = 0; r < rows[s]; r += q) {
      const int64_t end = std::min<int64_t>(pos[s] + std::min(r + q, rows[s]), int64_t(1) << 30);
      all.push_back((int)((std::max<int64_t>(end, 0) + 63) / 64 * 2));
      ++blocks;
    }
  }
  const int64_t cap = kv8_prefill_unit_cap((int64_t)rows.size(), T, q, hkv);
  const int64_t slots = kv8_prefill_slots((int64_t)rows.size(), T, q, hkv);
  if (!kv8_prefill_cuts(blocks, hkv)) {
    CHECK(blocks < cap);
    return;
  }
  CHECK(blocks <= kCus && blocks * hkv < kPrefillCutUnits);
  const int shift = kv8_prefill_shift(1 << 26 >> (pad % 3));   // of long tables, whatever the blocks are
  uint64_t total = 0;
  for (int t : all) total += kv8_prefill_size(t, shift);
  CHECK(total < (uint64_t(1) << 31));
  const uint32_t share = kv8_prefill_share((uint32_t)total, hkv);
  int64_t units = 0;
  uint32_t at = 0;
  for (int t : all) {
    const uint32_t size = kv8_prefill_size(t, shift);
    const Kv8Cut c = kv8_prefill_cut(at, size, share);
    CHECK(c.parts >= 1);
    int end = 0;
    for (int k = 0; k < c.parts; ++k) {   // successive, even, none of several empty or far beyond a share
      const int t0 = kv8_prefill_part_tile(c, at, share, shift, t, k), t1 = kv8_prefill_part_tile(c, at, share, shift, t, k + 1);
      CHECK(t0 == end && t0 % 2 == 0 && t1 % 2 == 0 && (t1 > t0 || c.parts == 1));
      CHECK(t1 - t0 <= ((int64_t)share + kPrefillMinTiles) << (shift + 1));
      end = t1;
    }
    CHECK(end == t);
    units += c.parts;
    at += size;
  }
  CHECK(units <= blocks + kv8_prefill_streams(hkv) && units < cap && units < slots && units <= kCus + kPrefillResident);
}

int main() {
  std::mt19937_64 r(1);
  auto log_int = [&](double hi) { return (int64_t)std::exp(std::uniform_real_distribution<double>(0, std::log(hi))(r)); };
  for (g_case = 0; g_case < 4000; ++g_case) {
    const int hkv = (int)log_int(17), S = (int)log_int(3000);
    const double hi = g_case % 5 == 0 ? 6e7 : g_case % 2 ? 40 : 3000;
    std::vector<int> pages(S);
    for (int& p : pages) p = r() % 7 == 0 ? 0 : (int)log_int(hi);
    if (g_case % 11 == 0) pages[0] = 1 << 26;
    decode(pages, hkv);
    const int group = 1 + (int)(r() % 16), n = (int)log_int(300);
    std::vector<int> rows(n);
    std::vector<int64_t> pos(n);
    const double rows_hi = g_case % 3 ? 20 : 2000;
    for (int s = 0; s < n; ++s) {
      rows[s] = r() % 3 == 0 ? 0 : (int)log_int(rows_hi);
      pos[s] = g_case % 4 == 0 ? (int64_t)log_int(1e9) : (int64_t)log_int(30000) - 5;
    }
    prefill(rows, pos, hkv, group, (int64_t)(r() % 50));
  }
  std::puts("ok");
}

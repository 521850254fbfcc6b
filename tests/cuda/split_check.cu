// Checks at_split_over (k_attend.cuh), which tells the merge of the recomputed attention weights which CTAs hold
// parts of an item, on the host:
//   splits  every item of random runs of items, cut into equal shares as the kernel cuts them: first and last must
//           be the CTAs that hold its first and its last unit, and the call false where that is one CTA;
//   stale   numbers that no split makes (memory that a CTA which gave up a wait never wrote): whatever they are,
//           no CTA past the last one may come out.
// Prints one line per class and exits non-zero on any mismatch.  Test code only; no GPU is used.
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "k_attend.cuh"

int main() {
  std::mt19937_64 rng(7);
  long long bad = 0, split = 0, whole = 0;
  for (int run = 0; run < 4000; ++run) {
    const uint32_t ctas = run % 3 == 0 ? 152 : 1 + rng() % 200;
    const int items = 1 + rng() % 300;
    const uint32_t most = run % 2 ? 40 : 4;
    std::vector<uint32_t> n(items);
    uint64_t total = 0;
    for (auto& x : n) total += x = 1 + rng() % most;
    const uint32_t per = static_cast<uint32_t>((total + ctas - 1) / ctas);
    uint32_t u = 0;
    for (int i = 0; i < items; u += n[i++]) {
      uint32_t a = 0, b = 0;
      while ((a + 1) * per <= u) ++a;
      b = a;
      while ((b + 1) * per <= u + n[i] - 1) ++b;
      uint32_t first = ~0u, last = ~0u;
      const bool over = bkv::at_split_over(u, n[i], per, ctas, first, last);
      if (over != (a < b) || (over && (first != a || last != b || last >= ctas))) ++bad;
      (over ? split : whole) += 1;
    }
  }
  std::printf("splits: %lld split and %lld whole items, %lld mismatches\n", split, whole, bad);
  long long out = 0, tried = 0;
  auto stale = [&](uint32_t u, uint32_t n, uint32_t per, uint32_t ctas) {
    uint32_t first = 0, last = 0;
    ++tried;
    if (bkv::at_split_over(u, n, per, ctas, first, last) && (first >= last || last >= ctas)) ++out;
  };
  const uint32_t edges[] = {0, 1, 2, 151, 152, 153, 0x3F800000u, 0x7FFFFFFFu, 0x80000000u, 0xFF800000u, 0xFFFFFFFEu,
                            0xFFFFFFFFu};
  for (uint32_t u : edges)
    for (uint32_t per : edges)
      for (uint32_t n : {1u, 2u, 3u, 128u, 4096u, 0x7FFFFFFFu})
        for (uint32_t ctas : {1u, 152u}) stale(u, n, per, ctas);
  for (int i = 0; i < 4000000; ++i)
    stale(static_cast<uint32_t>(rng()), 1 + rng() % 5000, i % 2 ? 1 + rng() % 100000 : static_cast<uint32_t>(rng()), 152);
  std::printf("stale: %lld numbers, %lld past the last CTA\n", tried, out);
  return bad || out || split == 0 || whole == 0;
}

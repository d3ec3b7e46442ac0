// Host program: every element that the norm kernels' loads of rows of odd width touch, for all small shapes.  Prints each
// access outside an array of n rows; returns 1 if there is one.
#include <cstdio>

#include "../../paper_2601_02360_b200/csrc/sl_norm_rows.cuh"

int main() {
  int bad = 0;
  for (uint32_t d = 1; d <= 40; ++d) {
    if (d % 8 == 0) continue;
    for (uint32_t gap = 0; gap <= 16; gap += 8)                 // rows lie d + gap elements apart
      for (uint32_t n = 1; n <= 24; ++n)
        for (uint32_t lanes = 1; lanes <= 4; lanes *= 2)
          for (uint64_t r = 0; r < n; ++r)
            for (uint32_t lane = 0; lane < lanes; ++lane) {
              const auto c = sl::columns_of<8, 2, true>(r, lane, lanes, d);
              const bool near_end = sl::near_array_end(r, n, sl::rows_near_end(d));
              const int64_t end = (int64_t)(n - 1) * (d + gap) + d;
              for (int k = 0; k < 2; ++k)
                for (int e = 0; e < 8; ++e) {
                  if (!c.by_vector(k, near_end) && !(c.any(k) && c.has(k, e))) continue;      // not read
                  const int64_t at = (int64_t)r * (d + gap) + c.safe(k) + e;
                  if ((at < 0 || at >= end) && bad++ < 20)
                    std::printf("n %u d %u gap %u row %llu lane %u of %u: element %lld of %lld\n", n, d, gap, (unsigned long long)r, lane, lanes,
                                (long long)at, (long long)end);
                }
            }
  }
  return bad ? 1 : 0;
}

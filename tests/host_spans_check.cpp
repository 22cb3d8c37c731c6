// Host-side check of what counts as shared memory (csrc/spans.h), built and run by
// tests/test_spans_host.py (host compiler only, no device code).
//
// Every layout of up to three rows in a small range, against the bytes that each side
// has: sharing is never missed, and what shares nothing is told apart wherever the two
// lie in columns of one buffer.
#include <cstdio>
#include <set>

#include "../paper_2602_10729_amd/csrc/spans.h"

namespace {

using bo::share;
using bo::Span;

std::set<int> bytes_of(int at, int rows, int width, int pitch) {
  std::set<int> s;
  for (int r = 0; r < rows; ++r)
    for (int i = 0; i < width; ++i) s.insert(at + r * pitch + i);
  return s;
}
const void* address(uint64_t at) { return reinterpret_cast<const void*>(at); }

}  // namespace

int main() {
  int failures = 0;
  long missed = 0, apart = 0, refused = 0;
  for (int wa = 1; wa <= 4; ++wa)
    for (int wb = 1; wb <= 4; ++wb)
      for (int ra = 1; ra <= 3; ++ra)
        for (int rb = 1; rb <= 3; ++rb)
          for (int sa = wa; sa <= 8; ++sa)
            for (int sb = wb; sb <= 8; ++sb)
              for (int d = -26; d <= 26; ++d) {
                const std::set<int> x = bytes_of(100, ra, wa, sa), y = bytes_of(100 + d, rb, wb, sb);
                bool real = false;
                for (int v : y) real = real || x.count(v);
                const Span a{address(1000), ra, wa, sa}, b{address(1000 + d), rb, wb, sb};
                const bool got = share(a, b);
                if (got != share(b, a)) ++failures;
                if (real && !got) ++missed;
                apart += !real && !got;
                refused += !real && got;
                // columns of one buffer: equal pitches, or one side a single row
                const int pitch = ra > 1 ? sa : sb, off = ((d % pitch) + pitch) % pitch;
                const bool columns = (ra == 1 || rb == 1 || sa == sb) && (ra > 1 || rb > 1) &&
                                     off >= wa && pitch - off >= wb;
                if ((columns || (ra == 1 && rb == 1)) && got != real) ++failures;
              }
  if (missed) std::printf("%ld shared layouts were missed\n", missed);
  const int64_t far = (int64_t)1 << 40;
  // one row in the columns that a far matrix leaves, and in those that it has
  const Span matrix{address(1 << 20), 1000, 4096, far};
  if (share(matrix, {address((1 << 20) + 999 * far + 4096), 1, far - 4096, 0})) ++failures;
  if (!share(matrix, {address((1 << 20) + 999 * far + 4095), 1, 1, 0})) ++failures;
  if (share({nullptr, 3, 4, 4}, matrix) || share({address(1 << 20), 0, 4, 4}, matrix)) ++failures;
  // every second row beside other columns of every row
  if (share({address(1000 + 16), 4, 16, 64}, {address(1000), 8, 16, 32})) ++failures;
  if (!share({address(1000 + 15), 4, 16, 64}, {address(1000), 8, 16, 32})) ++failures;
  if (missed || failures) {
    std::printf("%d failures\n", failures);
    return 1;
  }
  std::printf("spans ok: %ld apart, %ld counted as shared without a byte\n", apart, refused);
  return 0;
}

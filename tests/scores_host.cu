// Which keys a row sees, on the host (the kernels' own function): inside the sequence, and as the definition says.
#include <cstdio>
#include <cstdlib>

#include "paged.cuh"

int main() {
  srand(3);
  const int odd[] = {0, 1, -1, -0x7fffffff - 1, 0x7fffffff, 1 << 30, (1 << 30) - 1, -5};
  long checked = 0;
  for (int trial = 0; trial < 500000; ++trial) {
    auto some = [&](int most) { return rand() % 5 ? rand() % (most + 4) - 2 : odd[rand() % 8]; };
    const int len = rand() % 10 ? rand() % 200 : (rand() % 2 ? 1 << 30 : 0);
    const long long pos = len && rand() % 6 ? rand() % len : (rand() % 2 ? -1 : -1000000000000ll);
    const int lo = some(len), hi = some(len);
    const bool has_lo = rand() % 2, has_hi = rand() % 2;
    const int window = rand() % 2 ? 0 : rand() % 4 ? 1 + rand() % 100 : 0x7fffffff;
    const sd::Scores sc{0.f, nullptr, window, has_lo ? &lo : nullptr, has_hi ? &hi : nullptr};
    const sd::Span v = sd::visible(sc, 0, pos, len);
    long long first = 0, last = pos;
    if (window && pos - window + 1 > first) first = pos - window + 1;
    if (has_lo && lo > first) first = lo;
    if (has_hi) last = hi;
    if (last > len - 1) last = len - 1;
    if (pos < 0 || first > last) {
      if (v.lo != 0 || v.hi != -1) { printf("%d..%d for nothing\n", v.lo, v.hi); return 1; }
    } else if (v.lo != first || v.hi != last || v.lo < 0 || v.hi >= len) {
      printf("%d..%d for %lld..%lld of %d\n", v.lo, v.hi, first, last, len);
      return 1;
    }
    ++checked;
  }
  printf("ok %ld\n", checked);
  return 0;
}

// How many keys one sum goes over where results are fp32, on the host (the launches' own functions).
#include <cstdio>
#include <cstdlib>

#include "attn_launch.cuh"

int main() {
  srand(5);
  auto some = [](int64_t lo, int64_t hi) {                       // over the logarithm
    const double x = rand() / (double)RAND_MAX;
    return (int64_t)(lo * pow((double)hi / lo, x));
  };
  long limited = 0, kept = 0;
  for (int trial = 0; trial < 300000; ++trial) {
    const int64_t max_len = some(1, 1 << 30), slot_rows = some(1, 9), units = some(1, 60000), rows = units * slot_rows;
    const int chunk = pick_split(some(100, 1000), units, rows, max_len), now = split_sums(chunk, units, rows, max_len);
    const int64_t splits = (max_len + now - 1) / now;
    if (now % 64 || now < 1 || now > chunk) { printf("%d keys, before %d\n", now, chunk); return 1; }
    if (splits > 65535 || (splits > 1 && rows * splits > kPartSlots)) { printf("%lld splits of %lld rows\n", (long long)splits, (long long)rows); return 1; }
    if (units <= kPartSlots && (max_len + kSumKeys - 1) / kSumKeys * rows <= kPartSlots) {
      if (now > kSumKeys) { printf("%d keys with room for fewer\n", now); return 1; }
      ++limited;
    } else if (now == chunk) {
      ++kept;
    }
    if (chunk <= kSumKeys && now != chunk) { printf("%d keys for %d\n", now, chunk); return 1; }
  }
  printf("ok %ld %ld\n", limited, kept);
  return 0;
}

// Runs the index functions of the calls on pages on the host (they are the kernels' own), over lengths and page numbers of which some are wrong.
#include <cstdio>
#include <cstdlib>

#include "pages.cuh"

int main() {
  srand(5);
  long checked = 0;
  const int odd[] = {0, 1, -1, 7, 8, 9, 127, 128, 129, 0x7fffffff, -0x7fffffff - 1, 1 << 30, (1 << 30) + 1};
  for (int trial = 0; trial < 200000; ++trial) {
    const int shift = 3 + rand() % 5, columns = 1 + rand() % 20, n_pages = 1 + rand() % 50;
    int status = 0;
    const sd::Books b{nullptr, nullptr, nullptr, 3, columns, n_pages, shift, &status};
    auto some = [&] { return rand() % 4 ? rand() % ((columns << shift) + 3) - 1 : odd[rand() % 13]; };
    const int length = some(), target = some();
    const bool fine = length >= 0 && length <= columns << shift && target >= 0 && target <= columns << shift;
    const sd::Resize r = sd::resize_of(b, length, target);
    if (r.ok != fine) { printf("ok %d for %d -> %d of %d\n", r.ok, length, target, columns << shift); return 1; }
    if (r.have < 0 || r.want < 0 || r.have > columns || r.want > columns || r.part >= columns) { printf("columns %d %d %d\n", r.have, r.want, r.part); return 1; }
    if (!fine && (r.have || r.want || r.part != -1)) { printf("work for a wrong row\n"); return 1; }
    if (fine) {
      const int pl = 1 << shift, kept = length < target ? length : target;
      if (r.have != (length + pl - 1) / pl || r.want != (target + pl - 1) / pl) { printf("columns of %d, %d\n", length, target); return 1; }
      if (r.part != (kept % pl ? kept / pl : -1) || (r.part >= 0 && (r.part >= r.have || r.part >= r.want))) { printf("part %d\n", r.part); return 1; }
    }
    const int p = some();
    if (b.is_page(p) != (p >= 0 && p < n_pages)) { printf("page %d\n", p); return 1; }
    ++checked;
  }
  // the longest table: 2^30 positions
  int status = 0;
  const sd::Books b{nullptr, nullptr, nullptr, 1, 1 << 23, 10, 7, &status};
  if (!b.is_length(1 << 30) || b.is_length((1 << 30) + 1) || b.columns_of(1 << 30) != 1 << 23 || b.row(0) != nullptr) { printf("long table\n"); return 1; }
  printf("ok %ld\n", checked);
  return 0;
}

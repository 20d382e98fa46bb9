// Runs the batch description's index functions on the host (they are the kernels' own) over random tables, some entries
// of which are wrong, and checks that every index they hand out lies inside its array.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "paged.cuh"

int main() {
  srand(7);
  long checked = 0;
  for (int trial = 0; trial < 3000; ++trial) {
    const int shift = 3 + rand() % 5, page_len = 1 << shift, n_pages = 1 + rand() % 40, heads = 1 + rand() % 5;
    const int n_seqs = 1 + rand() % 6, columns = 1 + rand() % 9;
    std::vector<int> pages(n_seqs * columns), len(n_seqs), first(n_seqs + 1, 0);
    for (int& p : pages) p = rand() % 8 ? rand() % n_pages : rand() % 3 - 1 + (rand() % 2 ? n_pages : 0) - (rand() % 5 == 0 ? 1 << 30 : 0);
    for (int s = 0; s < n_seqs; ++s) {
      len[s] = rand() % 10 ? rand() % (columns * page_len + 1) : (rand() % 2 ? 0x7fffffff : -5);
      first[s + 1] = first[s] + rand() % 9;
    }
    int status = 0;
    const int n_tokens = first[n_seqs];
    const sd::BatchView b{pages.data(), first.data(), len.data(), n_seqs, columns, n_tokens, 8, n_pages, page_len, shift, heads, &status};
    for (int s = 0; s < n_seqs; ++s) {
      const int l = b.seq_len(s);
      if (l < 0 || l > columns * page_len) { printf("length %d\n", l); return 1; }
      if (len[s] > columns * page_len && !(status & sd::STATUS_BAD_BATCH)) { printf("long sequence not reported\n"); return 1; }
      for (int pos = 0; pos < l; ++pos) {
        const int before = status;
        const int pg = b.page_of(s, pos);
        const int entry = pages[s * columns + pos / page_len];
        const bool good = entry >= 0 && entry < n_pages;
        if (good != (pg >= 0) || (good && pg != entry)) { printf("page %d for entry %d of %d\n", pg, entry, n_pages); return 1; }
        if (!good) { if (!(status & sd::STATUS_BAD_BATCH)) { printf("bad page not reported (%d)\n", before); return 1; } continue; }
        const int g = rand() % heads;
        const size_t e = b.entry(pg, g, pos);
        if (e != ((size_t)pg * heads + g) * page_len + pos % page_len || e >= (size_t)n_pages * heads * page_len) { printf("entry %zu\n", e); return 1; }
        ++checked;
      }
    }
  }
  // a pool with more than 2^32 elements: entries are 64-bit
  int status = 0, table[1] = {0x7ffffffe}, first[2] = {0, 1}, len[1] = {1};
  const sd::BatchView b{table, first, len, 1, 1, 1, 1, 0x7fffffff, 128, 7, 100, &status};
  if (b.entry(b.page_of(0, 0), 99, 127) != ((size_t)0x7ffffffe * 100 + 99) * 128 + 127) { printf("64-bit entry\n"); return 1; }
  printf("ok %ld\n", checked);
  return 0;
}

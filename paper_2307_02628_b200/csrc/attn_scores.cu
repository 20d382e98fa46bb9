// Attention over the paged cache with capped, biased or masked scores: the forms of the kernels that do it, compiled beside the others.
#include "attn_launch.cuh"

namespace sd {

int attention_with_scores(sd_cache* c, int l, const sd_batch* b, const sd_heads* q, float scale, const sd_heads* out, const Scores& sc) {
  return cache_attention<true>(c, l, b, q, scale, out, sc);
}

}  // namespace sd

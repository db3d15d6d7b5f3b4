// Where the rows of a ragged batch lie: a pool of pages is a packed cache whose
// "sequences" are the pages (Dims::batch of them) and whose capacity is a
// page's rows, a multiple of 64, so that no 64-row key tile and no 32-row value
// tile crosses a page.  Sequence s's new tokens are rows cu[s] .. cu[s + 1] - 1
// of the inputs and take the last positions of its ctx[s] rows; its row t lies
// in page pages[s max_pages + t / capacity].
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.h"

namespace bgtq {
namespace paged {

// What the arrays of a batch say is read on the device: a sequence whose
// numbers contradict each other or the host's bounds is not `ok`.
struct Seq {
  int first, n, len;  // its tokens in the inputs, its rows (the new ones among them)
  bool ok;
};
__device__ __forceinline__ Seq make_seq(const PagedBatch& b, int c0, int c1, int len) {
  Seq s;
  s.first = min(max(c0, 0), b.n_tokens);
  s.n = max(min(c1, b.n_tokens) - s.first, 0);
  s.len = len;
  s.ok = c0 == s.first && c1 - c0 == s.n && s.n <= b.max_new && len >= s.n && len <= b.max_ctx;
  return s;
}
__device__ __forceinline__ Seq seq_of(const PagedBatch& b, int s) {
  return make_seq(b, b.cu[s], b.cu[s + 1], b.ctx[s]);
}

// The page of row t of sequence s, -1 where the table names none of the pool.
__device__ __forceinline__ int page_of(const PagedBatch& b, int n_pages, int page_rows, int s, int t) {
  const int p = b.pages[static_cast<size_t>(s) * b.max_pages + t / page_rows];
  return static_cast<uint32_t>(p) < static_cast<uint32_t>(n_pages) ? p : -1;
}

// Item `want` of a list that has count(sequence) items of each sequence in
// turn: its sequence (-1 behind the end) and its number there.  Called with
// whole waves, the same `want` in each lane; the results are wave-uniform.  64
// sequences at a time: their three numbers, one scan, one ballot.
template <class F>
__device__ __forceinline__ int find_item(const PagedBatch& b, int want, const F& count, int& number, Seq& seq) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < b.n_seqs; base += 64) {
    const int s = min(base + lane, b.n_seqs - 1);
    const Seq q = seq_of(b, s);
    const int mine = base + lane < b.n_seqs ? count(q) : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int x = __shfl_up(upto, o);
      upto += lane >= o ? x : 0;
    }
    const uint64_t at = __builtin_amdgcn_ballot_w64(upto > want);
    if (at != 0) {
      const int l = __builtin_ctzll(at);
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      number = want - (of(upto) - of(mine));
      seq = {of(q.first), of(q.n), of(q.len), of(q.ok) != 0};
      return base + l;
    }
    want -= __builtin_amdgcn_readlane(upto, 63);
  }
  number = 0;
  seq = {0, 0, 0, false};
  return -1;
}

}  // namespace paged
}  // namespace bgtq

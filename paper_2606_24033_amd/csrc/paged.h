// Where the rows of a ragged batch lie: a pool of pages is a packed cache whose
// "sequences" are the pages (Dims::batch of them) and whose capacity is a
// page's rows, a multiple of 64, so that no 64-row key tile and no 32-row value
// tile crosses a page.  Sequence s's new tokens are rows cu[s] .. cu[s + 1] - 1
// of the inputs and take the last positions of its ctx[s] rows; its row t lies
// in page pages[s max_pages + t / capacity].
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "layout.h"

namespace bgtq {
namespace paged {

// What the arrays of a batch say is read on the device: a sequence whose
// numbers contradict each other or the host's bounds is not `ok`.  Its tokens
// lie inside the inputs all the same, for any 32-bit offsets.
struct Seq {
  int first, n, len;  // its tokens in the inputs, its rows (the new ones among them)
  bool ok;
};
__host__ __device__ __forceinline__ Seq make_seq(const PagedBatch& b, int c0, int c1, int len) {
  const auto inside = [&](int c) { return c < 0 ? 0 : c < b.n_tokens ? c : b.n_tokens; };
  Seq s;
  s.first = inside(c0);
  const int last = inside(c1);  // (both in 0 .. n_tokens: the difference fits)
  s.n = last > s.first ? last - s.first : 0;
  s.len = len;
  s.ok = c0 == s.first && c1 == last && c0 <= c1 && s.n <= b.max_new && len >= s.n && len <= b.max_ctx;
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

// Page (-1: none) and place of input row r0 + tk of a ragged batch, r0 the same
// in the wave, tk < ROWS.  The sequence of r0 by a search 64 sequences at a time,
// the rows' own by one ballot each over the 64 sequences from there on.
template <int ROWS = 16>
__device__ __forceinline__ int2 page_of_row(const PagedBatch& b, int n_pages, int page_rows, int r0, int tk) {
  const int lane = threadIdx.x & 63, last = b.n_seqs - 1;
  int s0 = last;
  for (int base = 0; base < b.n_seqs; base += 64) {
    const uint64_t past = __builtin_amdgcn_ballot_w64(base + lane <= last && b.cu[min(base + lane, last) + 1] > r0);
    if (past != 0) {
      s0 = base + __builtin_ctzll(past);
      break;
    }
  }
  const int end = s0 + lane <= last ? b.cu[min(s0 + lane, last) + 1] : 0x7FFFFFFF;
  int s = s0;
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    const int n = __builtin_popcountll(__builtin_amdgcn_ballot_w64(end <= r0 + j));
    s = tk == j ? s0 + n : s;
  }
  s = min(s, last);
  // (64 sequences behind s0 end before the row: empty ones among them)
  while (s < last && b.cu[s + 1] <= r0 + tk) ++s;
  const Seq q = seq_of(b, s);
  const int i = r0 + tk - q.first;
  if (!q.ok || i < 0 || i >= q.n) return make_int2(-1, 0);
  const int t = q.len - q.n + i;
  return make_int2(page_of(b, n_pages, page_rows, s, t), t % page_rows);
}

// Value tile `want` of the new rows of a ragged batch: its page (-1: none), the
// first row of that tile in the sequence, and the rows [lo, hi) that are new.
struct Tile {
  int page, P0, lo, hi;
  size_t in0;  // input row of the sequence's row 0 (it may lie before the inputs)
};
__device__ __forceinline__ bool tile_of(const PagedBatch& b, int n_pages, int page_rows, int want, Tile& t) {
  int number;
  Seq q;
  const int s = find_item(
      b, want, [](const Seq& x) { return x.ok && x.n > 0 ? (x.len - 1) / kTile - (x.len - x.n) / kTile + 1 : 0; },
      number, q);
  if (s < 0) return false;
  const int wp = q.len - q.n;
  t.P0 = (wp / kTile + number) * kTile;
  t.lo = max(t.P0, wp) - t.P0;
  t.hi = min(t.P0 + kTile, q.len) - t.P0;
  t.page = page_of(b, n_pages, page_rows, s, t.P0);
  t.in0 = static_cast<size_t>(static_cast<long>(q.first) - wp);
  return t.page >= 0;
}

}  // namespace paged
}  // namespace bgtq

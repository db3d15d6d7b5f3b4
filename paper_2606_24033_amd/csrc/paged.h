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
  bool taken;  // not ok, but only because an earlier sequence claims some of its tokens
};
__host__ __device__ __forceinline__ Seq make_seq(const PagedBatch& b, int c0, int c1, int len) {
  const auto inside = [&](int c) { return c < 0 ? 0 : c < b.n_tokens ? c : b.n_tokens; };
  Seq s;
  s.first = inside(c0);
  const int last = inside(c1);  // (both in 0 .. n_tokens: the difference fits)
  s.n = last > s.first ? last - s.first : 0;
  s.len = len;
  s.ok = c0 == s.first && c1 == s.first + s.n && s.n <= b.max_new && len >= s.n && len <= b.max_ctx;
  s.taken = false;
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

// The sequences of a wave's 64 lanes, from `base` on in turn (the last one again
// behind the end): one that claims inputs' rows of an earlier one is not ok
// either, so that the ok ones share no row.  Offsets that never fall and stay
// inside the inputs keep them apart by themselves; what that costs is a ballot.
struct Apart {
  bool fell = false;  // an offset so far falls or lies outside
  int high = 0;       // the end of the sequences so far, where one does
  __device__ __forceinline__ void keep(int base, int c0, int c1, Seq& q) {
    if (!fell) {
      if (__builtin_amdgcn_ballot_w64(c0 != q.first || c1 != q.first + q.n) == 0) return;
      fell = true;
      high = base > 0 ? __builtin_amdgcn_readlane(c0, 0) : 0;
    }
    const int lane = threadIdx.x & 63;
    int upto = q.ok ? c1 : 0;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int x = __shfl_up(upto, o);
      upto = lane >= o ? max(upto, x) : upto;
    }
    const int x = __shfl_up(upto, 1), before = max(high, lane > 0 ? x : 0);
    q.taken = q.ok && q.n > 0 && c0 < before;
    q.ok = q.ok && !q.taken;
    high = max(high, __builtin_amdgcn_readlane(upto, 63));
  }
};

// Item `want` of a list that has count(sequence) items of each sequence in
// turn: its sequence (-1 behind the end) and its number there.  Called with
// whole waves, the same `want` in each lane; the results are wave-uniform.  64
// sequences at a time: their three numbers, one scan, one ballot.
template <class F>
__device__ __forceinline__ int find_item(const PagedBatch& b, int want, const F& count, int& number, Seq& seq) {
  const int lane = threadIdx.x & 63;
  Apart apart;
  for (int base = 0; base < b.n_seqs; base += 64) {
    const int s = min(base + lane, b.n_seqs - 1), c0 = b.cu[s], c1 = b.cu[s + 1];
    Seq q = make_seq(b, c0, c1, b.ctx[s]);
    apart.keep(base, c0, c1, q);
    const int mine = base + lane < b.n_seqs ? count(q) : 0;
    int upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(upto, o);
      upto += lane >= o ? y : 0;
    }
    const uint64_t at = __builtin_amdgcn_ballot_w64(upto > want);
    if (at != 0) {
      const int l = __builtin_ctzll(at);
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      number = want - (of(upto) - of(mine));
      seq = {of(q.first), of(q.n), of(q.len), true, false};
      return base + l;
    }
    want -= __builtin_amdgcn_readlane(upto, 63);
  }
  number = 0;
  seq = {0, 0, 0, false, false};
  return -1;
}

// The sequence that input row r0 + tk of a ragged batch belongs to (-1: none), r0
// the same in the wave; rows from number `need` on are of no interest.  64
// sequences at a time, then those of them that claim any of the rows.
__device__ __forceinline__ int seq_of_row(const PagedBatch& b, int r0, int tk, int need, Seq& seq) {
  const int lane = threadIdx.x & 63, last = b.n_seqs - 1;
  int at = -1;
  Apart apart;
  for (int base = 0; base <= last; base += 64) {
    const int s = min(base + lane, last), c0 = b.cu[s], c1 = b.cu[s + 1], len = b.ctx[s];
    Seq q = make_seq(b, c0, c1, len);
    apart.keep(base, c0, c1, q);
    const int end = apart.fell ? apart.high : __builtin_amdgcn_readlane(c1, 63);
    if (end <= r0) continue;
    const bool any = base + lane <= last && q.ok && c0 < c1 && c1 > r0 && c0 - need < r0;
    for (uint64_t some = __builtin_amdgcn_ballot_w64(any); some != 0; some &= some - 1) {
      const int l = __builtin_ctzll(some);
      const int first = __builtin_amdgcn_readlane(c0, l), behind = __builtin_amdgcn_readlane(c1, l);
      const int rows = __builtin_amdgcn_readlane(len, l);
      if (first <= r0 + tk && r0 + tk < behind) {
        at = base + l;
        seq = {first, behind - first, rows, true, false};
      }
    }
    // (what follows starts behind `end`)
    if (__builtin_amdgcn_ballot_w64(at < 0 && tk < need) == 0 || end >= r0 + need) break;
  }
  return at;
}

// Page (-1: none) and place of input row r0 + tk, tk < ROWS.
template <int ROWS = 16>
__device__ __forceinline__ int2 page_of_row(const PagedBatch& b, int n_pages, int page_rows, int r0, int tk) {
  Seq q = {};
  const int s = seq_of_row(b, r0, tk, ROWS, q);
  if (s < 0) return make_int2(-1, 0);
  const int t = q.len - q.n + r0 + tk - q.first;
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

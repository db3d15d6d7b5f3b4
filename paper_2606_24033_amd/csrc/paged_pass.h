// The attention passes of cross_impl.h and cross_tile.h over pages: which query
// rows of a ragged batch a workgroup takes, which cache rows each of them sees,
// and what happens to a logit before the softmax.
//
// Query row r of a sequence is head r % G of its new token r / G.  A unit is
// (block of query rows, KV head, split of the key axis).  Blocks are numbered
// sequence after sequence; the host knows only an upper bound of their number
// (it has no lengths), so the last workgroups may have none.  A call may run two
// passes, for sequences of few and of many query rows: a pass takes the
// sequences with lo < rows <= hi.
#pragma once
#include <hip/hip_runtime.h>

#include "kernels.h"
#include "layout.h"
#include "paged.h"

namespace bgtq {
namespace paged {

struct WholeCache {  // not this: every query row sees rows [0, len) of a cache
  static constexpr bool kPaged = false, kMods = false;
};
template <bool MODS>  // MODS: capped logits, a bias
struct Mode : PagedPass {
  static constexpr bool kPaged = true, kMods = MODS;
};

// A page's number read ahead of its use, in a vector register: one that the
// compiler sees to be uniform it waits for at once, and for every load before it.
__device__ __forceinline__ int page_ahead(const PagedBatch& b, int seq, int t, int page_rows) {
  uint32_t at = 0;
  asm volatile("" : "+v"(at));
  const int32_t* row = b.pages + static_cast<size_t>(seq) * b.max_pages + t / page_rows;
  return *reinterpret_cast<const int32_t*>(reinterpret_cast<const uint8_t*>(row) + at);
}

struct Unit {
  int seq, r0, kvh, split;  // r0: its first query row
  Seq q;
};

// The place among the partials of new token i's head `head` (of hq).
__device__ __forceinline__ size_t part_row(const PagedPass& p, const Unit& u, int hq, int i, int head) {
  return (p.direct ? static_cast<size_t>(u.seq) * p.most + i : static_cast<size_t>(u.q.first + i)) * hq + head;
}

// A sequence's blocks of R query rows in the pass.  (One whose numbers make no
// sense has one in the pass of the smallest, which answers for it, and one whose
// tokens are taken has one in the pass of its rows.)
template <int R>
__device__ __forceinline__ int blocks_of(const PagedPass& p, int group, const Seq& q) {
  if (!q.ok && !q.taken) return p.lo == 0 && q.n > 0 ? 1 : 0;
  const int rows = q.n * group;  // (below 2^31: the host checks)
  return rows > p.lo && rows <= p.hi ? (q.ok ? (rows + R - 1) / R : 1) : 0;
}

template <int R>
__device__ __forceinline__ bool find_block(const PagedPass& p, int group, int block, Unit& u) {
  if (p.direct) {  // no sequence has more than one block
    u.seq = block;
    u.q = seq_of(p.b, block);
    u.r0 = 0;
    return blocks_of<R>(p, group, u.q) > 0;
  }
  int number;
  u.seq = find_item(p.b, block, [&](const Seq& q) { return blocks_of<R>(p, group, q); }, number, u.q);
  u.r0 = number * R;
  return u.seq >= 0;
}

// KV heads vary fastest, then splits: the workgroups of a block go to all XCDs,
// however many blocks there turn out to be.  Blocks from the last one down: a
// chunk's late ones see the most rows.
__device__ __forceinline__ int unit_at(const PagedPass& p, const Dims& d, int n_splits, int item, Unit& u) {  // the block
  u.kvh = item % d.n_kv;
  item /= d.n_kv;
  u.split = item % n_splits;
  return p.n_blocks - 1 - item / n_splits;
}
template <int R>
__device__ __forceinline__ bool unit_of(const PagedPass& p, const Dims& d, int n_splits, int item, Unit& u) {
  return find_block<R>(p, d.group, unit_at(p, d, n_splits, item, u), u);
}

// The rows of a sequence that a call cannot answer for are not numbers.
__device__ __forceinline__ void refuse(const Unit& u, const Dims& d, int kvh, void* out, int out_dtype, int tid, int threads) {
  const int per = d.group * kHeadDim;
  const size_t stride = static_cast<size_t>(d.n_kv) * per;
  for (long i = tid; i < static_cast<long>(u.q.n) * per; i += threads) {
    const size_t at = (u.q.first + i / per) * stride + static_cast<size_t>(kvh) * per + i % per;
    if (out_dtype == 1) static_cast<uint16_t*>(out)[at] = 0x7FC0;
    else static_cast<float*>(out)[at] = __builtin_nanf("");
  }
}

// What new token i of a sequence sees: rows [0, end(i)), end never falls.
struct Sight {
  int pos0, see;  // position of token 0; rows that all of them see
  __device__ __forceinline__ int pos(int i) const { return pos0 + i; }
  __device__ __forceinline__ int end(int i) const { return max(pos0 + i + 1, see); }
};
__device__ __forceinline__ Sight sight_of(const PagedPass& p, const Unit& u, int seq) {
  return {u.q.len - u.q.n, p.m.prefix ? min(p.m.prefix[seq], u.q.len) : 0};
}

// Radii (fp16) of four tokens, zero from number `left` on.
__device__ __forceinline__ uint2 seen(const uint2& r, int left) {
  return make_uint2((left > 0 ? r.x & 0xFFFFu : 0u) | (left > 1 ? r.x & 0xFFFF0000u : 0u),
                    (left > 2 ? r.y & 0xFFFFu : 0u) | (left > 3 ? r.y & 0xFFFF0000u : 0u));
}

// A base-2 logit x = log2 e q k / sqrt(d) after the cap, C tanh(x / C) with
// C = cap log2 e, and the bias, -slope |distance|.  The cap is x P(z) / Q(z),
// z = (x / C)^2, |x| up to 8.2 C, beyond which tanh is 1 to 2^-22.6.  P and Q of
// degree 4 are the least largest relative error of tanh(y) / y up to there (8e-9;
// fitted by reweighted least squares); in fp32 2^-21.7, whatever the cap.  One
// transcendental instruction and 15 others.  (1 - t) / (1 + t), t = 2^(-2 |y| log2 e),
// has two and 7, but loses 2^-24 C of small logits: all of them at a cap of 1e7.
// cap: 2^-100 .. 2^100 (0: none), so that C, 1 / C and 8.2 C are normal numbers; a
// cap beyond either end changes no output that one at the end does not.
__device__ __forceinline__ float changed(float cap, float slope, float x, float distance) {
  constexpr float kLog2 = 1.4426950408889634f;
  if (cap > 0.f) {
    const float c = cap * kLog2, inv = 1.f / c;
    const float xc = fminf(fmaxf(x, -8.2f * c), 8.2f * c), y = xc * inv, z = y * y;
    float p = fmaf(z, 1.4842521e-08f, 2.1638720e-05f), q = fmaf(z, 8.3714156e-07f, 3.3865857e-04f);
    p = fmaf(z, p, 3.5567754e-03f);
    q = fmaf(z, q, 2.6108639e-02f);
    p = fmaf(z, p, 0.13432199f);
    q = fmaf(z, q, 0.46765524f);
    p = fmaf(z, p, 1.f);
    q = fmaf(z, q, 1.f);
    x = x == x ? xc * p * __builtin_amdgcn_rcpf(q) : x;  // (the bounds pass over what is not a number)
  }
  return fmaf(-slope, fabsf(distance), x);
}

}  // namespace paged
}  // namespace bgtq

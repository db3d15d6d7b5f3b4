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

// A sequence's blocks of R query rows in the pass.
template <int R>
__device__ __forceinline__ int blocks_of(const PagedPass& p, int group, const Seq& q) {
  const int rows = q.n * group;  // (below 2^31: the host checks)
  return q.ok && rows > p.lo && rows <= p.hi ? (rows + R - 1) / R : 0;
}

// Whether the pass answers for a refused sequence: that of the smallest, or, of
// one whose tokens are taken, that of its rows.
__device__ __forceinline__ bool answers(const PagedPass& p, int group, const Seq& q) {
  return !q.ok && q.n > 0 && (q.taken ? q.n * group > p.lo && q.n * group <= p.hi : p.lo == 0);
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

// The rows of a sequence that a call cannot answer for are not numbers.
__device__ __forceinline__ void refuse(const Seq& q, const Dims& d, int kvh, const CrossCall& call, int tid, int threads) {
  const int per = d.group * kHeadDim;
  const size_t stride = static_cast<size_t>(d.n_kv) * per;
  for (long i = tid; i < static_cast<long>(q.n) * per; i += threads) {
    const size_t at = (q.first + i / per) * stride + static_cast<size_t>(kvh) * per + i % per;
    if (call.out_dtype == 1) static_cast<uint16_t*>(call.out)[at] = 0x7FC0;
    else static_cast<float*>(call.out)[at] = __builtin_nanf("");
  }
}

// Refused sequences of a pass whose blocks are numbered over all sequences: they
// have none, for the list to stay within the grid whatever the offsets say.
// Block 0's workgroups answer for them: a wave looks at every threads / 64-th 64
// sequences, and goes through all of them where it finds one that is at fault.
// (Rows next to or among those that it has written once are not written again:
// numbers of all sizes, as uninitialized ones, claim every row over and over.)
__device__ __forceinline__ void answer_refused(const PagedPass& p, const Dims& d, int kvh, const CrossCall& call, int threads) {
  const PagedBatch& b = p.b;
  const int lane = threadIdx.x & 63;
  bool fault = false;
  for (int base = threadIdx.x & ~63; base < b.n_seqs; base += threads) {
    const int s = min(base + lane, b.n_seqs - 1), c0 = b.cu[s], c1 = b.cu[s + 1];
    const Seq q = make_seq(b, c0, c1, b.ctx[s]);
    fault = fault || c0 != q.first || c1 != q.first + q.n || answers(p, d.group, q);
  }
  if (__builtin_amdgcn_ballot_w64(fault) == 0) return;
  Apart apart;
  int done0 = 0, done1 = 0;
  const auto write = [&](int from, int to) {
    if (from < to) refuse({from, to - from, 0, false, false}, d, kvh, call, lane, 64);
  };
  for (int base = 0; base < b.n_seqs; base += 64) {
    const int s = min(base + lane, b.n_seqs - 1), c0 = b.cu[s], c1 = b.cu[s + 1];
    Seq q = make_seq(b, c0, c1, b.ctx[s]);
    apart.keep(base, c0, c1, q);
    for (uint64_t some = __builtin_amdgcn_ballot_w64(base + lane < b.n_seqs && answers(p, d.group, q)); some != 0; some &= some - 1) {
      const int l = __builtin_ctzll(some);
      const int from = __builtin_amdgcn_readlane(q.first, l), to = from + __builtin_amdgcn_readlane(q.n, l);
      if (done0 < done1 && from <= done1 && to >= done0) {
        write(from, min(to, done0));
        write(max(from, done1), to);
        done0 = min(done0, from);
        done1 = max(done1, to);
      } else {
        write(from, to);
        if (to - from > done1 - done0) {
          done0 = from;
          done1 = to;
        }
      }
    }
  }
}

// The unit of a block (unit_at), with whole waves; false: it has no rows.  (Blocks
// of 8 rows are single tokens', always direct.)
template <int R>
__device__ __forceinline__ bool find_unit(const PagedPass& p, const Dims& d, const CrossCall& call, int block, Unit& u, int threads) {
  if (R == 8 || p.direct) {  // no sequence has more than one block
    u.seq = block;
    u.q = seq_of(p.b, block);
    u.r0 = 0;
    if (u.split == 0 && answers(p, d.group, u.q)) refuse(u.q, d, u.kvh, call, threadIdx.x, threads);
    return blocks_of<R>(p, d.group, u.q) > 0;
  }
  if constexpr (R == 8) return false;
  if (block == 0 && u.split == 0) answer_refused(p, d, u.kvh, call, threads);
  int number;
  u.seq = find_item(p.b, block, [&](const Seq& q) { return blocks_of<R>(p, d.group, q); }, number, u.q);
  u.r0 = number * R;
  return u.seq >= 0;
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

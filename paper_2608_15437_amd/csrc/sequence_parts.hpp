// Which rows a workgroup of a walk over ragged sequences takes: a sequence, or
// a part of a long one.
#pragma once

#include "common.hpp"
#include "sequence.hpp"

namespace mmbev {
namespace {

constexpr int kPartStep = 64;  // parts begin at multiples of this from their sequence's start

// Positions run over the rows in use, from the last row backwards where the
// call is reversed; sequence k in that order begins at bound(k).
struct Order {
  const int64_t* offsets;
  int64_t ahead[2];  // offsets of this lane's sequence, if it is one of the first 64
  int32_t used, B, reversed;
  __device__ __forceinline__ int32_t clamped(int64_t o) const {
    const int32_t c = o < 0 ? 0 : o > used ? used : (int32_t)o;
    return reversed ? used - c : c;
  }
  __device__ __forceinline__ int32_t bound(int32_t k) const { return clamped(offsets[reversed ? B - k : k]); }
  __device__ __forceinline__ int32_t row(int32_t p) const { return reversed ? used - 1 - p : p; }
  __device__ __forceinline__ int32_t sequence(int32_t k) const { return reversed ? B - 1 - k : k; }
};

__device__ __forceinline__ Order order_of(const Ranges& a) {
  Order o;
  o.offsets = a.offsets;
  o.B = a.B;
  o.reversed = a.reversed;
  // all of these loads before the first is waited for
  const int k = min((int)(threadIdx.x & 63), a.B - 1);
  o.ahead[0] = a.offsets[a.reversed ? a.B - k : k];
  o.ahead[1] = a.offsets[a.reversed ? a.B - k - 1 : k + 1];
  const int64_t end = a.offsets[a.B];
  o.used = end < 0 ? 0 : end > a.rows ? (int32_t)a.rows : (int32_t)end;
  return o;
}

// A run of rows that one workgroup walks: a sequence, or a part of one.
struct Part {
  int32_t lo, hi;  // positions
  int32_t b;       // sequence
  int32_t next;    // where the sequence's next part ends, if this one goes on
  int32_t end;     // and the sequence
  int32_t before;  // parts that go on (into another of their sequence) before this one
  bool began;      // a part of the sequence comes before it
  bool goes_on;    // and after it
};

// The r-th longest of up to 256 sequences that are not longer than `most`
// (ties: the first ones first), found bit by bit: the largest length that more
// than r of them reach.  False: there are no more than r.

__device__ __forceinline__ bool find_longest(Part& q, const Order& o, int32_t most, int32_t r) {
  constexpr int N = kOrderedSequences / 64;
  const int lane = threadIdx.x & 63;
  int32_t n[N], s0[N];
  int32_t there = 0;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    n[u] = -1;
    s0[u] = 0;
    if (64 * u < o.B) {
      const int32_t k = 64 * u + lane;
      s0[u] = o.bound(min(k, o.B - 1));
      const int32_t len = max(o.bound(min(k, o.B - 1) + 1) - s0[u], 0);
      n[u] = k < o.B && len <= most ? len : -1;
    }
    there += __popcll(__ballot(n[u] >= 0));
  }
  if (r >= there) return false;
  auto reach = [&](int32_t len) {
    int32_t c = 0;
#pragma unroll
    for (int u = 0; u < N; ++u) c += __popcll(__ballot(n[u] >= len));
    return c;
  };
  int32_t len = 0;
  for (int32_t bit = most > 0 ? 1 << (31 - __builtin_clz(most)) : 0; bit; bit >>= 1)
    if (reach(len | bit) > r) len |= bit;
  int32_t tie = r - reach(len + 1);
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const uint64_t same = __ballot(n[u] == len);
    const int c = __popcll(same);
    if (tie >= 0 && tie < c) {
      const int at = __builtin_ctzll(__ballot(n[u] == len && (int32_t)count_below(same) == tie));
      q.lo = __builtin_amdgcn_readlane(s0[u], at);
      q.hi = q.lo + len;
      q.b = o.sequence(64 * u + at);
    }
    tie -= c;
  }
  return true;
}

// A workgroup's share is the rows in use over a.cuts.  Sequences longer than
// two shares are cut into equal parts of at most one, in whole chunks; the
// others are walked whole.  There are at most a.cuts + B parts, of which at
// most a.cuts go on.  Finds part `index`: the cut sequences' parts come first,
// then the whole ones, the longest first where there are more than the chip
// takes at once (so that the last ones to begin are short).  Or, `going_on`,
// the part of that number among those that go on.  False if there are fewer.
// Every wave looks for itself, 64 sequences at a time: loads, a sum over the
// lanes and ballots, about a microsecond.
__device__ __forceinline__ bool find_part(Part& q, const Order& o, const Ranges& a, int32_t index, bool going_on) {
  q.before = 0;
  q.began = q.goes_on = false;
  if (!a.cuts) {
    q.lo = o.bound(index);
    q.hi = max(o.bound(index + 1), q.lo);
    q.b = o.sequence(index);
    return true;
  }
  const int32_t each = (int32_t)(((int64_t)o.used + a.cuts - 1) / a.cuts);
  const int32_t share = max((int32_t)(((int64_t)each + kPartStep - 1) / kPartStep * kPartStep), a.least);
  const int32_t most = (int32_t)min((int64_t)share * 2, (int64_t)INT32_MAX);
  const int lane = threadIdx.x & 63;
  int32_t seen = 0, cut = 0;
  for (int32_t k0 = 0; k0 < o.B; k0 += 64) {
    const int32_t k = min(k0 + lane, o.B - 1);
    const int32_t s0 = k0 == 0 ? o.clamped(o.ahead[0]) : o.bound(k);
    const int32_t n = max((k0 == 0 ? o.clamped(o.ahead[1]) : o.bound(k + 1)) - s0, 0);
    const uint32_t parts = k0 + lane < o.B && n > most ? (uint32_t)(((int64_t)n + share - 1) / share) : 0u;
    const uint64_t cuts = __ballot(parts != 0);
    if (cuts == 0) continue;
    const uint32_t count = parts - (going_on && parts ? 1u : 0u), upto = wave_inclusive_sum(count);
    const uint32_t all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    if ((uint32_t)(index - seen) < all) {
      const int at = __builtin_ctzll(__ballot(upto > (uint32_t)(index - seen)));
      const int32_t n0 = __builtin_amdgcn_readlane(s0, at), len = __builtin_amdgcn_readlane(n, at);
      const int32_t c = __builtin_amdgcn_readlane((int)parts, at);
      const int32_t j = index - seen - (int32_t)__builtin_amdgcn_readlane((int)(upto - count), at);
      const int32_t step = (int32_t)((((int64_t)len + c - 1) / c + kPartStep - 1) / kPartStep * kPartStep);  // <= share
      q.lo = n0 + j * step;
      q.hi = j + 1 < c ? q.lo + step : n0 + len;
      q.end = n0 + len;
      q.next = j + 2 < c ? q.hi + step : q.end;
      q.b = o.sequence(k0 + at);
      q.before = going_on ? index : index - cut - __popcll(cuts & ((1ull << at) - 1));
      q.began = j > 0 && q.before <= a.cuts;  // more parts than that go on only where the offsets break their contract
      q.goes_on = j + 1 < c;
      return true;
    }
    seen += (int32_t)all;
    cut += __popcll(cuts);
  }
  if (going_on) return false;
  if (a.longest_first) return find_longest(q, o, most, index - seen);
  int32_t r = index - seen;
  for (int32_t k0 = 0; k0 < o.B; k0 += 64) {
    const int32_t k = min(k0 + lane, o.B - 1);
    const int32_t s0 = o.bound(k), n = max(o.bound(k + 1) - s0, 0);
    const uint64_t whole = __ballot(k0 + lane < o.B && n <= most);
    const int c = __popcll(whole);
    if (r < c) {
      const int at = __builtin_ctzll(__ballot((whole >> lane & 1) && (int32_t)count_below(whole) == r));
      q.lo = __builtin_amdgcn_readlane(s0, at);
      q.hi = q.lo + __builtin_amdgcn_readlane(n, at);
      q.b = o.sequence(k0 + at);
      return true;
    }
    r -= c;
  }
  return false;
}

}  // namespace
}  // namespace mmbev

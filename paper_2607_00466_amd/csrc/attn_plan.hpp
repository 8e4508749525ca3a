// How a batch's attention is cut into work: what each request shares, and two
// lines of equal units that are dealt to the workgroups in equal stretches.
//
// A request's cached slots are [0, reach), read with its group, and
// [max(reach, lens - window), lens), its own.  Every workgroup works the plan
// out for itself from lens and the groups (a few thousand cycles, no launch of
// its own, and no host copy of the lengths, so that a graph can replay a step
// while the lengths grow).
//
//   own line     for each head tile, for each request: tiles of kTile slots
//   shared line  for each kv head, for each group, for each row tile: tiles
//
// A part of a row is a stretch that one workgroup holds.
#pragma once

#include "attn_common.hpp"

namespace eldr {

constexpr int kTile = 128;  // slots of a unit; units start at multiples of it

struct Groups {
  const int32_t *lens, *start, *prefix;
  int32_t R, n, window;  // n: groups (0 where a window forbids sharing)
};

// The plan in LDS.
struct Plan {
  int *own;     // [R + 1] own units before each request
  int *reach;   // [R] slots read with the group
  int *group;   // [R] the request's group, -1: none
  int *shared;  // [n + 1] shared units (row tiles x slot tiles) before each group
  int *first;   // [n] the group's first request that holds anything: the prefix is read through its row (R: none does)
  int *len;     // [R] cached slots
  int *start;   // [n + 1] the groups' first requests

  // own, reach, group and shared: what moe_attn_decode leaves for its join
  static __host__ __device__ int kept(int R, int n) { return 3 * R + 1 + n + 1; }
  static __host__ __device__ size_t bytes(int R, int n) { return sizeof(int) * ((size_t)kept(R, n) + n + R + n + 1); }
};

// out[0] = 0, out[i + 1] = sum of f(0 .. i), by THREADS threads, i ascending a thread.
template <int THREADS, typename F>
__device__ __forceinline__ void sums(int n, int* out, int* waves, F f) {
  const int t = threadIdx.x, lane = t % kWave, wave = t / kWave;
  const int per = (n + THREADS - 1) / THREADS;
  int mine = 0;
  for (int i = t * per; i < min(n, t * per + per); ++i) mine += f(i);
  const int upto = wave_sum_before(mine);
  if (lane == kWave - 1) waves[wave] = upto;
  __syncthreads();
  int at = upto - mine;
#pragma unroll
  for (int w = 0; w < THREADS / kWave; ++w) at += w < wave ? waves[w] : 0;
  if (t == 0) out[0] = 0;
  for (int i = t * per; i < min(n, t * per + per); ++i) {
    at += f(i);
    out[i + 1] = at;
  }
  __syncthreads();
}

// Tiles that [lo, hi) touches.
__device__ __forceinline__ int tiles_of(int lo, int hi) {
  return hi > lo ? (hi + kTile - 1) / kTile - lo / kTile : 0;
}

__device__ __forceinline__ int clamp_len(int n, int capacity) { return min(max(n, 0), capacity); }

// First slot of a request's own part.
__device__ __forceinline__ int own_from(int n, int reach, int window) {
  return window > 0 ? max(0, n - window) : min(reach, n);
}

// Works the plan out.  `lds`: Plan::bytes of LDS; `waves`: THREADS / 64 ints of
// LDS; G: query heads a kv head; row_tile: rows of a shared unit.  What is read
// from memory is asked for at once, and the rest is LDS.
template <int THREADS>
__device__ __forceinline__ Plan make_plan(const Groups& gr, int capacity, int G, int row_tile, int* lds, int* waves) {
  Plan p;
  p.own = lds;
  p.reach = p.own + gr.R + 1;
  p.group = p.reach + gr.R;
  p.shared = p.group + gr.R;
  p.first = p.shared + gr.n + 1;
  p.len = p.first + gr.n;
  p.start = p.len + gr.R;
  // until the requests know their reach: the slots that a group shares where `first`
  // will be, and the first request where `shared` will be
  int *least = p.first, *holder = p.shared;
  for (int r = threadIdx.x; r < gr.R; r += THREADS) p.len[r] = clamp_len(gr.lens[r], capacity);
  for (int g = threadIdx.x; g < gr.n; g += THREADS) {
    least[g] = clamp_len(gr.prefix[g], capacity);
    holder[g] = gr.R;
    p.start[g] = min(max(gr.start[g], 0), gr.R);
  }
  if (gr.n > 0 && threadIdx.x == 0) p.start[gr.n] = min(max(gr.start[gr.n], 0), gr.R);
  __syncthreads();
  for (int r = threadIdx.x; r < gr.R; r += THREADS) {
    int group = -1;
    if (gr.n > 0) {
      // the last group that starts at or before r (the first one may not)
      int lo = 0, hi = gr.n;
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (p.start[mid] <= r) lo = mid;
        else hi = mid;
      }
      const int s = p.start[lo], e = p.start[lo + 1];
      // an empty member reads nothing, does not shorten what the others share, and
      // its row of the block table may name anything
      if (s <= r && r < e && e - s > 1 && p.len[r] > 0) {
        group = lo;
        atomicMin(&least[lo], p.len[r]);
        if (r == s || p.len[r - 1] == 0) atomicMin(&holder[lo], r);  // (a member that follows one that holds something is not the first)
      }
    }
    p.group[r] = group;
  }
  __syncthreads();
  for (int r = threadIdx.x; r < gr.R; r += THREADS) p.reach[r] = p.group[r] < 0 ? 0 : least[p.group[r]];
  __syncthreads();
  for (int g = threadIdx.x; g < gr.n; g += THREADS) p.first[g] = holder[g];
  // (a barrier of the sums comes before `first` is read and `shared` written)
  sums<THREADS>(gr.R, p.own, waves,
                [&](int r) { return tiles_of(own_from(p.len[r], p.reach[r], gr.window), p.len[r]); });
  if (gr.n > 0)
    sums<THREADS>(gr.n, p.shared, waves, [&](int g) {
      const int members = p.start[g + 1] - p.start[g];
      return p.first[g] < gr.R ? (members * G + row_tile - 1) / row_tile * tiles_of(0, p.reach[p.first[g]]) : 0;
    });
  else if (threadIdx.x == 0)
    p.shared[0] = 0;
  __syncthreads();
  return p;
}

// The last i of [0, n) with at[i] <= v; at[0] <= v.
__device__ __forceinline__ int last_at(const int* at, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (at[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// A line of units dealt to workgroups in stretches whose lengths differ by one
// at most: w has [first(w), first(w + 1)), the first `longer` ones each + 1 units.
// No workgroup is without a unit: the join counts on it.
struct Deal {
  int wgs, each, longer;
  __device__ __forceinline__ Deal(int units, int most) {
    wgs = min(units, most);
    each = wgs > 0 ? (int)((uint32_t)units / (uint32_t)wgs) : 1;
    longer = units - each * wgs;
  }
  __device__ __forceinline__ int first(int w) const { return w * each + min(w, longer); }
  __device__ __forceinline__ int owner(int u) const {
    const int in_longer = longer * (each + 1);
    return u < in_longer ? (int)((uint32_t)u / (uint32_t)(each + 1))
                         : longer + (int)((uint32_t)(u - in_longer) / (uint32_t)each);
  }
};

}  // namespace eldr

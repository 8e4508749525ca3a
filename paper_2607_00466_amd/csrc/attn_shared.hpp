// The shared part of moe_attn_decode: a group's prefix against the query rows
// of all its members, its keys and values read once for 128 rows.
//
// With members x G rows on a kv head the products outweigh the bytes (at 64
// members of 8 heads each, 512 rows and 1024 flop a byte), so this is an MFMA
// kernel: the prefix goes through LDS in stages of 64 slots, double-buffered
// (the next stage's loads are in flight in registers while this one is used),
// and every wave takes 32 rows (16 where D is 256) of the tile and one half of
// each stage.  Four waves' rows by two halves: LDS is read at the rate at which
// the matrix cores use it up, and the tile is no larger than it has to be, since
// each workgroup leaves a part of every row it held.
//
// The products and the softmax are as in the other kernel: S^T = K Q^T, weights
// used where the product left them, in two bf16 parts.  (Here the second part's
// product costs: 64 behind 8192 48.8 -> 51.5 us, 64 behind 65536 127 -> 144, the
// whole call; with one part these outputs' error was 1.3 times their rounding's.)
//
// Measured: 64 requests (32 heads over 4 of 128) against 8192 shared slots 28 us,
// against 65536 132 to 146 us (470 to 520 TFLOP/s of the formula's products; a library
// product 1400): a stage takes a workgroup 1.9 to 2.1 us.  (With one part 25 and 113 us,
// 1.5 a stage, of which its two waves a SIMD spent half in MFMAs and exponents and the
// rest in the dependences between them.)  Starting (plan, queries, first stage) takes
// 6 us and handing over the parts 3.  Stages of 128 slots measured the same (4% faster
// at D = 64), more stages in flight too.
#pragma once

#include "attn_plan.hpp"
#include "attn_tile.hpp"

namespace eldr {

constexpr int kSharedThreads = 512;
constexpr int kSharedWaves = kSharedThreads / kWave;
constexpr int kRowWaves = 4;      // waves side by side over the rows
constexpr int kSharedWgs = 256;   // one a CU
constexpr int kStage = 64;        // slots in LDS at a time

template <int D>
struct SharedTile {
  static constexpr int kQ = D == 256 ? 1 : 2;             // 16-row tiles a wave
  static constexpr int kRowsWg = kRowWaves * kQ * kRows;  // rows of a workgroup
  static constexpr int kChunks = D / 8;                   // 16-byte pieces of a row in LDS
  static constexpr int kPieces = kStage * kChunks / kSharedThreads;  // a thread stages, of keys and of values
  static constexpr int kStageBytes = kStage * D * 2;      // of one cache
  static constexpr int kAhead = D == 256 ? 1 : 2;         // stages in flight
  static constexpr int kMergeWords = kQ * (D / 16 * 4 + 2);
  static constexpr int kBytes = 4 * kStageBytes > kRowWaves * kMergeWords * kWave * 4 ? 4 * kStageBytes
                                                                                      : kRowWaves * kMergeWords * kWave * 4;
  // Where piece c of row r lies: rows are rotated against each other so that 16
  // rows' pieces of one column, and one row's 16 pieces, fall on different banks.
  static __device__ __forceinline__ uint32_t at(int r, int c) {
    const int turn = D == 64 ? (r >> 1) & 7 : r & 15;
    return (uint32_t)(r * kChunks + (c ^ turn)) * 16;
  }
};

// A thread's share of one stage of one cache, on its way from HBM to LDS.  Wave
// w stages slots [8 w, 8 w + 8), half of a 16-slot tile, so all in one page:
// pass i's piece is piece lane % kChunks of slot 8 w + lane / kChunks + i kRowsPass.
template <int D, bool FP8>
struct Piece {
  using S = SharedTile<D>;
  typedef typename std::conditional<FP8, u32x2, u32x4>::type Raw;
  static constexpr int kElem = FP8 ? 1 : 2;
  static constexpr int kRowsPass = kWave / S::kChunks;
  Raw raw[S::kPieces];
  __device__ __forceinline__ void load(const char* tile, uint32_t off) {
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) raw[i] = *reinterpret_cast<const Raw*>(tile + off + i * kRowsPass * D * kElem);
  }
  // live: the lane's slots that count come before it (of pass i: before live - i kRowsPass)
  __device__ __forceinline__ void store(char* stage, const uint32_t (&at)[S::kPieces], bool whole, int live) const {
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
      u32x4 x;
      if constexpr (FP8)
        x = u32x4{fp8_pair<false>(raw[i][0]), fp8_pair<true>(raw[i][0]), fp8_pair<false>(raw[i][1]), fp8_pair<true>(raw[i][1])};
      else
        x = raw[i];
      // slots that do not count become zeros: their bits may be NaN
      if (!whole) x = keep_if(i * kRowsPass < live, x);
      *reinterpret_cast<u32x4*>(stage + at[i]) = x;
    }
  }
};

struct SharedArgs {
  const uint16_t* q;
  const char *k_cache, *v_cache;
  Groups gr;
  const float* k_scale;
  float *rows_part, *rest_part;  // [R * Hq][D + 4], [kSharedWgs][kRowsWg][D + 4]
  float scale;
  int32_t Hq, G;
};

// Rows [row0, row0 + kRowsWg) of a group's members (requests from `first` on) on kv
// head h, against slots [k0, k1) of the prefix, through row table_row of the block
// table; k0 is a multiple of kTile.
struct SharedSegment {
  int first, table_row, rows, row0, h, k0, k1;
};

template <int D, bool FP8>
__device__ __forceinline__ void attend_shared(const SharedArgs& a, const Pages& pg, const SharedSegment& sg, char* lds,
                                              float* part, bool by_row) {
  using S = SharedTile<D>;
  constexpr int kK = D / 32, kV = D / 16, kElem = FP8 ? 1 : 2;
  const int lane = threadIdx.x % kWave, n = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int half = wave / kRowWaves, wave_row = sg.row0 + wave % kRowWaves * S::kQ * kRows;
  const bool live = wave_row < sg.rows;  // the wave has rows
  const float unit = a.scale * kLog2e * (FP8 && a.k_scale ? a.k_scale[sg.h] : 1.0f);
  u32x4 q[S::kQ][kK];
#pragma unroll
  for (int t = 0; t < S::kQ; ++t) {
    const int row = wave_row + t * kRows + n;
    const bool there = row < sg.rows;
    const int req = sg.first + (there ? row / a.G : 0), head = sg.h * a.G + (there ? row % a.G : 0);
    const uint16_t* src = a.q + ((int64_t)req * a.Hq + head) * D;
#pragma unroll
    for (int s = 0; s < kK; ++s) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + s * 32 + g * 8);
      q[t][s] = keep_if(there, x);
    }
  }
  float m[S::kQ], l[S::kQ];  // reference, and this lane's part of the sum, of row n
  f32x4 acc[S::kQ][kV];
#pragma unroll
  for (int t = 0; t < S::kQ; ++t) {
    m[t] = -INFINITY, l[t] = 0.0f;
#pragma unroll
    for (int c = 0; c < kV; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int32_t* table = pg.table + (int64_t)sg.table_row * pg.max_blocks;
  // stage i on its way: set i % kAhead
  Piece<D, FP8> next_k[S::kAhead], next_v[S::kAhead];
  const int my_row = lane / S::kChunks;  // of the wave's eight, in pass 0
  const uint32_t off = (uint32_t)((wave % 2 * 8 + my_row) * D + lane % S::kChunks * 8) * kElem;
  uint32_t put[S::kPieces];
#pragma unroll
  for (int i = 0; i < S::kPieces; ++i) put[i] = S::at(wave * 8 + my_row + i * Piece<D, FP8>::kRowsPass, lane % S::kChunks);
  // The pages of 64 16-slot tiles (a window), lane i the i-th's, asked for one
  // window ahead: a scalar load a stage would be waited for with every LDS read.
  // present[w % 2]: which tiles of window w count and have a page.
  constexpr int kWindow = kWave * 16;
  const auto look_up = [&](int window) {
    const int slot = window * kWindow + lane * 16;
    return slot < sg.k1 ? table[slot >> pg.shift] : -1;
  };
  int pages = look_up(sg.k0 / kWindow), pages_next = look_up(sg.k0 / kWindow + 1);
  uint64_t present[2];
  present[0] = present[1] = __ballot(pg.has(pages));
  // which of stage k's four tiles are there
  const auto tiles_there = [&](int k) { return (uint32_t)(present[k / kWindow % 2] >> (k / 16 % kWave)) & 15u; };
  const int64_t head_at = (int64_t)sg.h << pg.shift;
  const int in_page = (1 << pg.shift) - 1;
  const auto fetch = [&](int set, int k) {
    if (k % kWindow == 0 && k != sg.k0) {
      pages = pages_next;
      pages_next = look_up(k / kWindow + 1);
      present[k / kWindow % 2] = __ballot(pg.has(pages));
    }
    const int slot = k + wave / 2 * 16;
    int page = __builtin_amdgcn_readlane(pages, slot / 16 % kWave);
    page = pg.has(page) ? page : 0;
    const int64_t at = (page * pg.block_stride + (head_at + (slot & in_page)) * D) * kElem;
    next_k[set].load(a.k_cache + at, off);
    next_v[set].load(a.v_cache + at, off);
  };
  // stage k from its set to the buffer
  const auto store = [&](int set, int k, char* to) {
    const uint32_t there = tiles_there(k);
    const bool whole = there == 15u && k + kStage <= sg.k1;
    const int live = (there >> (wave / 2) & 1u) ? sg.k1 - (k + wave * 8 + my_row) : 0;
    next_k[set].store(to, put, whole, live);
    next_v[set].store(to + S::kStageBytes, put, whole, live);
  };
  // where the lane's operands lie in a stage (the swizzle repeats every 16 rows)
  uint32_t k_at[kK], v_at[4];
#pragma unroll
  for (int i = 0; i < kK; ++i) k_at[i] = S::at(half * kStep + n, i * 4 + g);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    v_at[j] = S::kStageBytes + (D == 64 ? S::at(half * kStep + 4 * g + j, n / 2) + (n % 2) * 8
                                        : S::at(half * kStep + 4 * g + j, n * (kV / 8)));
  constexpr uint32_t kTileBytes = kRows * D * 2;  // 16 slots
#pragma unroll
  for (int i = 0; i < S::kAhead; ++i)
    if (sg.k0 + i * kStage < sg.k1) fetch(i, sg.k0 + i * kStage);
  store(0, sg.k0, lds);
  __syncthreads();
  // one stage: k's slots lie in buffer `stage`; set (of k) is free again
  const auto use = [&](int k, int set, int next_set, char* stage, char* other) {
    if (k + S::kAhead * kStage < sg.k1) fetch(set, k + S::kAhead * kStage);
    const int k_mine = k + half * kStep;
    const uint32_t there = tiles_there(k) >> (2 * half);
    if (live && k_mine < sg.k1) {
      f32x4 s[S::kQ][2];
#pragma unroll
      for (int t = 0; t < S::kQ; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kK; ++i) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(stage + k_at[i] + b * kTileBytes);
#pragma unroll
          for (int t = 0; t < S::kQ; ++t) s[t][b] = mfma16x16x32(x, q[t][i], s[t][b]);
        }
      }
      const bool whole = (there & 3u) == 3u && k_mine + kStep <= sg.k1;
      const auto keep = [&](int j) { return (there >> (j / 4) & 1u) && k_mine + (j / 4) * 16 + 4 * g + j % 4 < sg.k1; };
      u32x4 most[S::kQ], rest[S::kQ];
#pragma unroll
      for (int t = 0; t < S::kQ; ++t) {
        const Weights p = softmax_step(s[t], unit, whole, keep, m[t], l[t], [&](float f) {
#pragma unroll
          for (int c = 0; c < kV; ++c) acc[t][c] *= f;
        });
        most[t] = p.most, rest[t] = p.rest;
      }
      // eight value columns a lane at a time (four where D is 64)
      constexpr int kCols = kV < 8 ? kV : 8;
#pragma unroll
      for (int w = 0; w < kV / kCols; ++w) {
        Values<kCols * 16, false> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // (neighbouring pieces of a row differ in the lowest bit of their place)
          const char* from = stage + ((v_at[j % 4] ^ (w * 16)) + (j / 4) * kTileBytes);
          if constexpr (D == 64) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(from);
            v.raw[j][0] = x[0], v.raw[j][1] = x[1];
          } else {
            const u32x4 x = *reinterpret_cast<const u32x4*>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) v.raw[j][i] = x[i];
          }
        }
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          const u32x4 x = v.operand(c);
#pragma unroll
          for (int t = 0; t < S::kQ; ++t) acc[t][w * kCols + c] = mfma16x16x32(x, most[t], acc[t][w * kCols + c]);
#pragma unroll
          for (int t = 0; t < S::kQ; ++t) acc[t][w * kCols + c] = mfma16x16x32(x, rest[t], acc[t][w * kCols + c]);
        }
      }
    }
    if (k + kStage < sg.k1) store(next_set, k + kStage, other);
    __syncthreads();
  };
  char* const buffers[2] = {lds, lds + 2 * S::kStageBytes};
  for (int k = sg.k0; k < sg.k1; k += 2 * kStage) {
    use(k, 0, 1 % S::kAhead, buffers[0], buffers[1]);
    if (k + kStage < sg.k1) use(k + kStage, 1 % S::kAhead, 0, buffers[1], buffers[0]);
  }
  // The halves add up: each hands the other the row tile that it does not finish
  // (tile t is finished by half t; with one tile the second half only hands over),
  // lane by lane.
  const auto spot = [&](int t) {
    return reinterpret_cast<float*>(lds) + (wave % kRowWaves * S::kQ + t) * (kV * 4 + 2) * kWave + lane;
  };
#pragma unroll
  for (int t = 0; t < S::kQ; ++t) {
    if (t == half) continue;
    float* to = spot(t);
    to[0] = m[t], to[kWave] = l[t];
#pragma unroll
    for (int c = 0; c < kV; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) to[(2 + c * 4 + i) * kWave] = acc[t][c][i];
  }
  __syncthreads();
  f32x4 sum[kV];
  float top = -INFINITY, total = 0.0f;
#pragma unroll
  for (int t = 0; t < S::kQ; ++t) {
    if (t != half) continue;
    const float* from = spot(t);
    const float m1 = from[0];
    top = fmaxf(m[t], m1);
    const bool none = top == -INFINITY;
    const float f0 = none ? 0.0f : exp2_fast(m[t] - top), f1 = none ? 0.0f : exp2_fast(m1 - top);
    total = l[t] * f0 + from[kWave] * f1;
#pragma unroll
    for (int c = 0; c < kV; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[c][i] = acc[t][c][i] * f0 + from[(2 + c * 4 + i) * kWave] * f1;
  }
  total += __shfl_xor(total, 16);
  total += __shfl_xor(total, 32);
  __syncthreads();
  // through LDS once more, so that the parts are written as whole lines
  constexpr int kPitch = D + 4;
  float* tile = reinterpret_cast<float*>(lds);
  if (half < S::kQ) {
    float* row = tile + (wave % kRowWaves * S::kQ * kRows + half * kRows + n) * kPitch;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < kV; c += 4)
        *reinterpret_cast<f32x4*>(row + (4 * g + i) * kV + c) = f32x4{sum[c][i], sum[c + 1][i], sum[c + 2][i], sum[c + 3][i]};
    if (g == 0) *reinterpret_cast<f32x4*>(row + D) = f32x4{top, total, 0.0f, 0.0f};
  }
  __syncthreads();
  constexpr int kQuads = kPitch / 4;
  const int live_rows = min(S::kRowsWg, sg.rows - sg.row0);
  for (int e = threadIdx.x; e < live_rows * kQuads; e += kSharedThreads) {
    const int r = e / kQuads, row = sg.row0 + r;
    const int64_t q_row = (int64_t)(sg.first + row / a.G) * a.Hq + sg.h * a.G + row % a.G;
    *reinterpret_cast<f32x4*>(part + (by_row ? q_row : (int64_t)r) * kPitch + (e - r * kQuads) * 4) =
        *reinterpret_cast<const f32x4*>(tile + e * 4);
  }
  __syncthreads();
}

template <int D, bool FP8>
__global__ __launch_bounds__(kSharedThreads, 2) void attn_shared_kernel(SharedArgs a, Pages pg) {
  using S = SharedTile<D>;
  extern __shared__ char lds_shared[];
  __shared__ int waves[kSharedWaves];
  const int capacity = pg.capacity();
  const Plan plan = make_plan<kSharedThreads>(a.gr, capacity, a.G, S::kRowsWg, reinterpret_cast<int*>(lds_shared + S::kBytes), waves);
  const int n = a.gr.n, row = plan.shared[n];
  const Deal deal(row * pg.Hkv, kSharedWgs);
  const int w = (int)blockIdx.x % kNumXcd * (kSharedWgs / kNumXcd) + (int)blockIdx.x / kNumXcd;
  if (w >= deal.wgs) return;
  int u = __builtin_amdgcn_readfirstlane(deal.first(w));
  const int end = __builtin_amdgcn_readfirstlane(deal.first(w + 1));
  while (u < end) {
    const int h = u / row, v = u - h * row;
    const int grp = last_at(plan.shared, n, v);
    const int first = plan.start[grp], members = plan.start[grp + 1] - first;
    const int table_row = plan.first[grp], reach = plan.reach[table_row], per = tiles_of(0, reach), in = v - plan.shared[grp];
    const int tile = in / per, t = in - tile * per;
    const int tiles = __builtin_amdgcn_readfirstlane(min(per - t, end - u));
    SharedSegment sg{first, table_row, members * a.G, tile * S::kRowsWg, h, t * kTile, min((t + tiles) * kTile, reach)};
    int* f = reinterpret_cast<int*>(&sg);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(sg) / 4); ++i) f[i] = __builtin_amdgcn_readfirstlane(f[i]);
    const bool begins = sg.k0 == 0;
    attend_shared<D, FP8>(a, pg, sg, lds_shared,
                          begins ? a.rows_part : a.rest_part + (int64_t)w * S::kRowsWg * (D + 4), begins);
    u += tiles;
  }
}

}  // namespace eldr

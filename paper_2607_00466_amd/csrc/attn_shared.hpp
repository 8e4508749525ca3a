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
// The softmax is as in the other kernel: S^T = K Q^T, weights used where the
// product left them.  Its maximum is taken of the raw scores and the scale
// enters the exponent's multiply-add (a negative scale is turned into a
// positive one by the sign of q).
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

// A thread's share of one stage of one cache, on its way from HBM to LDS.
template <int D, bool FP8>
struct Piece {
  using S = SharedTile<D>;
  typedef typename std::conditional<FP8, u32x2, u32x4>::type Raw;
  Raw raw[S::kPieces];
  __device__ __forceinline__ void load(const char* const (&rows)[S::kPieces], const bool (&ok)[S::kPieces], uint32_t off) {
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
      Raw x = {};
      if (ok[i]) x = *reinterpret_cast<const Raw*>(rows[i] + off);
      raw[i] = x;
    }
  }
  __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
      const int p = threadIdx.x + i * kSharedThreads;
      u32x4 x;
      if constexpr (FP8)
        x = u32x4{fp8_pair<false>(raw[i][0]), fp8_pair<true>(raw[i][0]), fp8_pair<false>(raw[i][1]), fp8_pair<true>(raw[i][1])};
      else
        x = raw[i];
      *reinterpret_cast<u32x4*>(lds + S::at(p / S::kChunks, p % S::kChunks)) = x;
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

// Rows [row0, row0 + kRowsWg) of a group's members on kv head h, against slots
// [k0, k1) of the prefix; k0 is a multiple of kTile.
struct SharedSegment {
  int table_row, rows, row0, h, k0, k1;
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
  const float unit0 = a.scale * kLog2e * (FP8 && a.k_scale ? a.k_scale[sg.h] : 1.0f);
  const float unit = fabsf(unit0);
  const uint32_t flip = unit0 < 0.0f ? 0x80008000u : 0u;
  u32x4 q[S::kQ][kK];
#pragma unroll
  for (int t = 0; t < S::kQ; ++t) {
    const int row = wave_row + t * kRows + n;
    const bool there = row < sg.rows;
    const int req = sg.table_row + (there ? row / a.G : 0), head = sg.h * a.G + (there ? row % a.G : 0);
    const uint16_t* src = a.q + ((int64_t)req * a.Hq + head) * D;
#pragma unroll
    for (int s = 0; s < kK; ++s) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(src + s * 32 + g * 8);
      q[t][s] = there ? x ^ flip : u32x4{0u, 0u, 0u, 0u};
    }
  }
  float m[S::kQ], l[S::kQ];  // maximum (raw) and this lane's part of the sum of row n
  f32x4 acc[S::kQ][kV];
#pragma unroll
  for (int t = 0; t < S::kQ; ++t) {
    m[t] = -INFINITY, l[t] = 0.0f;
#pragma unroll
    for (int c = 0; c < kV; ++c) acc[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int32_t* table = pg.table + (int64_t)sg.table_row * pg.max_blocks;
  // the rows that this wave stages in pass i lie in one 16-slot tile, so in one page
  constexpr int kRowsPass = kSharedThreads / S::kChunks, kRowsWave = kWave / S::kChunks;
  const int in_row = (threadIdx.x % S::kChunks) * 8 * kElem;
  const int row_in_wave = lane / S::kChunks;
  Piece<D, FP8> next_k, next_v;
  const auto fetch = [&](int k) {
    const char *kp[S::kPieces], *vp[S::kPieces];
    bool ok[S::kPieces];
#pragma unroll
    for (int i = 0; i < S::kPieces; ++i) {
      const int first = k + i * kRowsPass + wave * kRowsWave;  // the wave's first row: a slot
      const int page = first < sg.k1 ? table[first >> pg.shift] : -1;
      const bool has = pg.has(page);
      const int64_t at = pg.row(has ? page : 0, sg.h, first) * kElem;
      kp[i] = a.k_cache + at;
      vp[i] = a.v_cache + at;
      ok[i] = has && first + row_in_wave < sg.k1;
    }
    const uint32_t off = (uint32_t)(row_in_wave * D * kElem + in_row);
    next_k.load(kp, ok, off);
    next_v.load(vp, ok, off);
  };
  char* stage = lds;
  fetch(sg.k0);
  next_k.store(stage);
  next_v.store(stage + S::kStageBytes);
  __syncthreads();
  for (int k = sg.k0; k < sg.k1; k += kStage) {
    char* other = lds + (stage == lds ? 2 * S::kStageBytes : 0);
    const bool more = k + kStage < sg.k1;
    if (more) fetch(k + kStage);
    const int k_mine = k + half * kStep;
    if (live && k_mine < sg.k1) {
      const char *ks = stage, *vs = stage + S::kStageBytes;
      const int r0 = half * kStep;
      f32x4 s[S::kQ][2];
#pragma unroll
      for (int t = 0; t < S::kQ; ++t) s[t][0] = s[t][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kK; ++i) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const u32x4 x = *reinterpret_cast<const u32x4*>(ks + S::at(r0 + 16 * b + n, i * 4 + g));
#pragma unroll
          for (int t = 0; t < S::kQ; ++t) s[t][b] = mfma16x16x32(x, q[t][i], s[t][b]);
        }
      }
      const int next = (k_mine + 16) >> pg.shift;
      const bool has0 = pg.has(table[k_mine >> pg.shift]), has1 = next < pg.max_blocks && pg.has(table[next]);
      if (!(has0 && has1 && k_mine + kStep <= sg.k1)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool keep = (j < 4 ? has0 : has1) && k_mine + (j / 4) * 16 + 4 * g + j % 4 < sg.k1;
#pragma unroll
          for (int t = 0; t < S::kQ; ++t) s[t][j / 4][j % 4] = keep ? s[t][j / 4][j % 4] : -INFINITY;
        }
      }
      u32x4 p[S::kQ];
#pragma unroll
      for (int t = 0; t < S::kQ; ++t) {
        float top = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])),
                          fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (__any(top > m[t])) {
          const float m2 = fmaxf(m[t], top);
          const float back = m2 == -INFINITY ? 0.0f : exp2_fast((m[t] - m2) * unit);
          m[t] = m2;
          l[t] *= back;
#pragma unroll
          for (int c = 0; c < kV; ++c) acc[t][c] *= back;
        }
        const float base = m[t] == -INFINITY ? 0.0f : m[t] * unit;
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = exp2_fast(fmaf(s[t][j / 4][j % 4], unit, -base));
          l[t] += x[j];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) p[t][i] = pack_bf16(x[2 * i], x[2 * i + 1]);
      }
      // eight value columns a lane at a time (four where D is 64)
      constexpr int kCols = kV < 8 ? kV : 8;
#pragma unroll
      for (int w = 0; w < kV / kCols; ++w) {
        Values<kCols * 16, false> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = r0 + (j / 4) * 16 + 4 * g + j % 4;
          if constexpr (D == 64) {
            const u32x2 x = *reinterpret_cast<const u32x2*>(vs + S::at(r, n / 2) + (n % 2) * 8);
            v.raw[j][0] = x[0], v.raw[j][1] = x[1];
          } else {
            const u32x4 x = *reinterpret_cast<const u32x4*>(vs + S::at(r, n * (kV / 8) + w));
#pragma unroll
            for (int i = 0; i < 4; ++i) v.raw[j][i] = x[i];
          }
        }
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          const u32x4 x = v.operand(c);
#pragma unroll
          for (int t = 0; t < S::kQ; ++t) acc[t][w * kCols + c] = mfma16x16x32(x, p[t], acc[t][w * kCols + c]);
        }
      }
    }
    if (more) {
      next_k.store(other);
      next_v.store(other + S::kStageBytes);
    }
    stage = other;
    __syncthreads();
  }
  // the second half's waves hand their state to the first half's, lane by lane
  float* swap = reinterpret_cast<float*>(lds) + (wave % kRowWaves) * S::kMergeWords * kWave + lane;
  if (half == 1) {
#pragma unroll
    for (int t = 0; t < S::kQ; ++t) {
      float* to = swap + t * (kV * 4 + 2) * kWave;
      to[0] = m[t], to[kWave] = l[t];
#pragma unroll
      for (int c = 0; c < kV; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) to[(2 + c * 4 + i) * kWave] = acc[t][c][i];
    }
  }
  __syncthreads();
  if (half == 0 && live) {
#pragma unroll
    for (int t = 0; t < S::kQ; ++t) {
      const float* from = swap + t * (kV * 4 + 2) * kWave;
      const float m1 = from[0], m2 = fmaxf(m[t], m1);
      const bool none = m2 == -INFINITY;
      const float f0 = none ? 0.0f : exp2_fast((m[t] - m2) * unit), f1 = none ? 0.0f : exp2_fast((m1 - m2) * unit);
      float sum = l[t] * f0 + from[kWave] * f1;
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      const int row = wave_row + t * kRows + n;
      if (row < sg.rows) {
        const int64_t q_row = (int64_t)(sg.table_row + row / a.G) * a.Hq + sg.h * a.G + row % a.G;
        float* to = part + (by_row ? q_row : (int64_t)(row - sg.row0)) * (D + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < kV; c += 4) {
            f32x4 x;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = acc[t][c + e][i] * f0 + from[(2 + (c + e) * 4 + i) * kWave] * f1;
            *reinterpret_cast<f32x4*>(to + (4 * g + i) * kV + c) = x;
          }
        if (g == 0) to[D] = none ? -INFINITY : m2 * unit, to[D + 1] = sum;
      }
    }
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
  const int R = a.gr.R, n = a.gr.n, row = plan.shared[n];
  const Deal deal = deal_of((int64_t)row * pg.Hkv, kSharedWgs);
  if ((int)blockIdx.x >= deal.wgs) return;
  int u = __builtin_amdgcn_readfirstlane(deal.first(blockIdx.x));
  const int end = __builtin_amdgcn_readfirstlane(deal.first(blockIdx.x + 1));
  while (u < end) {
    const int h = u / row, v = u - h * row;
    const int grp = last_at(plan.shared, n, v);
    const int first = max(a.gr.start[grp], 0), members = min(a.gr.start[grp + 1], R) - first;
    const int reach = plan.least[grp], per = tiles_of(0, reach), in = v - plan.shared[grp];
    const int tile = in / per, t = in - tile * per;
    const int tiles = __builtin_amdgcn_readfirstlane(min(per - t, end - u));
    SharedSegment sg{first, members * a.G, tile * S::kRowsWg, h, t * kTile, min((t + tiles) * kTile, reach)};
    int* f = reinterpret_cast<int*>(&sg);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(sg) / 4); ++i) f[i] = __builtin_amdgcn_readfirstlane(f[i]);
    const bool begins = sg.k0 == 0;
    attend_shared<D, FP8>(a, pg, sg, lds_shared,
                          begins ? a.rows_part : a.rest_part + (int64_t)blockIdx.x * S::kRowsWg * (D + 4), begins);
    u += tiles;
  }
}

}  // namespace eldr

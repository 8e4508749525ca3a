// moe_kv_append_int8: norms, rotation and the write of new tokens into pages of
// 8-bit integers that share a scale, page by page and head by head.
//
// A scale needs the largest value of all of the page's new rows before the first
// code can be written, so a page's rows of one kv head (a tile) are one wave's
// work, or one workgroup's where pages have more than 16 slots: the rows are
// normed and turned, kept in registers where they fit (16 slots a wave, 64 a
// workgroup; past that they are worked out again), their largest magnitude is
// found by exchanges between lanes, and the codes follow.  The queries, which no
// scale ties together, are turned by further workgroups of the same launch.
//
// Bound by bytes for prompts: 16 of up to 1000 tokens (64 heads over 8 of 64, from fp32,
// 192 MB read and written) 42 us, 4.5 TB/s; 32 over 4 of 128 in bf16 (128 MB) 31.9; pages
// of 64 slots 32.3.  By a chain of dependent loads for a decode batch: 64 tokens 5.7 us
// (the request, its page, position and scale, then rows; with the angles asked for after
// the norm and divisions for the codes 6.7), 1000 requests of one token 24 (36 while each
// wave looked its request up among all; its bytes are 4: a tile of one row has work for
// 4 to 16 of a wave's lanes).  Pages whose scale grows have their held codes read and
// written besides: 64 tokens of which half the keys' and 78% of the values' pages grow 6.4
// where none grows any more 6.2, 16 prompts the same.  A wave that takes several of a page's tiles one
// after another needs a quarter more registers: 3 to 7% faster for prompts, but only
// with spills, and without them 18% slower at D = 256; runs of 1 to 3 tokens 12 -> 18 us.
//
// Which page a wave takes is worked out on the device, from query_start and lens
// (a captured graph replays steps of growing lengths): request r has the units
// from unit_of(r) on, at least as many as its tokens touch pages.
#include "append_rows.hpp"
#include "eldr_kv_cache.h"

namespace eldr {

constexpr int kQuantThreads = 256;

struct QuantArgs {
  Rotation turns;
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;
  const int32_t *query_start, *lens;
  uint16_t* q_out;
  const float *q_norm, *k_norm;  // [D] or null
  int8_t *k_cache, *v_cache;
  float *k_scale, *v_scale;
  float eps;
  int32_t R, Hq;
  int32_t unit_shift, unit_more;  // unit_of
  int32_t tiles, tile_blocks;     // units * 2 Hkv, and the workgroups they take
  int32_t q_lanes;                // threads that share a token's queries
  // Units before those of request r, whose tokens begin at `start`: a unit for each
  // token, or one for each whole page of tokens before and two more a request.  (n
  // tokens touch at most n pages, and at most the whole pages in n, and 2.)
  __device__ __forceinline__ int unit_of(int r, int start) const { return (start >> unit_shift) + r * unit_more; }
  __device__ __forceinline__ int start_of(int r) const { return min(max(query_start[r], 0), turns.T); }
};

// The last request that f, which does not fall, gives at most `most` (0 if none
// does); by one wave.
template <typename F>
__device__ __forceinline__ int last_request(int R, int most, F f) {
  constexpr int kBatch = 4;  // loads in flight
  int count = 0;
  for (int r0 = 0; r0 < R; r0 += kBatch * kWave) {
    int at[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) at[b] = f(min(r0 + b * kWave + (int)(threadIdx.x % kWave), R - 1));
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
      count += __popcll(__ballot(r0 + b * kWave + (int)(threadIdx.x % kWave) < R && at[b] <= most));
  }
  return max(count - 1, 0);
}

// The largest x of a wave, in all lanes.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int m = 1; m < kWave; m *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, m));
  return x;
}

// The scale of a page that holds values of `scale` already and gets ones of up to
// top: scale 2^n, n >= 0 the smallest with 127 scale 2^n >= top; `back` = 2^-n.
__device__ __forceinline__ float grown(float scale, float top, float& back) {
  const double most = 127.0 * (double)scale, need = (double)top;
  int n = 0;
  if (need > most) {
    n = ilogb(need) - ilogb(most);       // 2^n most has need's exponent
    n += ldexp(most, n) < need ? 1 : 0;
  }
  back = (float)ldexp(1.0, -n);
  return (float)ldexp((double)scale, n);
}

// What turns values into codes of a page.
struct Coder {
  float by, scale, inverse;  // values times `by` are in units of `scale`
  bool none;                 // the scale is 0, or NaN
  // (2^64: where the scale's inverse would be infinite, or a remainder below fp32's range)
  __device__ __forceinline__ explicit Coder(float page_scale)
      : by(page_scale < 0x1p-60f ? 0x1p64f : 1.0f), scale(page_scale * by), inverse(1.0f / scale), none(!(page_scale > 0.0f)) {}
  // round(x / scale) within +-127.  The quotient is the correctly rounded one, so that
  // codes equal those of the definition: two steps from the product with the inverse.
  // (No magnitude is over 127 scale and its rounding; quotients too small for the
  // steps to be exact round to 0.)
  __device__ __forceinline__ uint32_t code(float x) const {
    x *= by;
    float c = x * inverse;
    c = fmaf(fmaf(-c, scale, x), inverse, c);
    c = fmaf(fmaf(-c, scale, x), inverse, c);
    c = fminf(fmaxf(rintf(c), -127.0f), 127.0f);
    return (uint32_t)(none ? 0 : (int)c) & 0xffu;
  }
  __device__ __forceinline__ u32x2 codes(const float (&x)[8]) const {
    u32x2 v;
#pragma unroll
    for (int w = 0; w < 2; ++w) v[w] = code(x[4 * w]) | code(x[4 * w + 1]) << 8 | code(x[4 * w + 2]) << 16 | code(x[4 * w + 3]) << 24;
    return v;
  }
};

// Held codes under a scale that is 2^n as large: back = 2^-n.
__device__ __forceinline__ u32x4 codes_again(u32x4 old, float back) {
  u32x4 v;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t word = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const float c = (float)(int8_t)(old[w] >> (8 * b));
      word |= ((uint32_t)(int)rintf(c * back) & 0xffu) << (8 * b);
    }
    v[w] = word;
  }
  return v;
}

// A page's new rows: `rows` of them from token t0 on, to offsets from o0 on.
struct PageRows {
  int page, t0, o0, rows;
};

// One tile: the rows of kind `kind`, a kv head's keys (below Hkv) or values, by
// WAVES waves.
template <typename In, int D, bool INTERLEAVED, int WAVES>
__device__ __forceinline__ void quantise_tile(const QuantArgs& a, const Pages& pg, const PageRows& p, int kind, uint32_t* tops) {
  constexpr int kLanes = D / 16;                       // of a row
  constexpr int kRowsPass = WAVES * kWave / kLanes;    // 64 / kLanes a wave
  constexpr int kHold = kLanes / 4;                    // passes in registers: 16 rows a wave
  const int id = threadIdx.x % (WAVES * kWave), chunk = id % kLanes, row0 = id / kLanes;
  const int wave = threadIdx.x / kWave;
  const bool is_v = kind >= pg.Hkv;
  const int h = is_v ? kind - pg.Hkv : kind;
  float* scale_at = (is_v ? a.v_scale : a.k_scale) + (int64_t)p.page * pg.Hkv + h;
  const float old = p.o0 > 0 ? *scale_at : 0.0f;
  const bool turns = !is_v && chunk * 16 < a.turns.rot;
  const Runs at(chunk, a.turns.rot / 2, turns && !INTERLEAVED);
  const float* weight = is_v ? nullptr : a.k_norm;
  float wx[8], wy[8];
  if (weight) {
    load8(weight + at.e0, wx);
    load8(weight + at.e1, wy);
  }
  const In* src = reinterpret_cast<const In*>(is_v ? a.v : a.k) + (int64_t)h * D;
  const int64_t stride = is_v ? a.v_stride : a.k_stride;
  const auto load = [&](int row, float (&x)[8], float (&y)[8]) {
    const int t = p.t0 + row;
    // what the row needs is asked for before any of it is worked on
    Raw8<In> r[2];
    r[0].load(src + t * stride + at.e0);
    r[1].load(src + t * stride + at.e1);
    float c[8], s[8];
    if (turns) load_angles(a.turns, t, chunk, c, s);
    r[0].get(x);
    r[1].get(y);
    if (weight) {
      const float i = row_scale(x, y, kLanes, a.eps);
      norm8(x, i, wx);
      norm8(y, i, wy);
    }
    if (turns) turn_runs<INTERLEAVED>(x, y, c, s);
  };
  uint32_t top = 0;  // largest magnitude's bits: a NaN's are above infinity's
  const auto see = [&](const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  };
  float hx[kHold][8], hy[kHold][8];
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    const int row = row0 + i * kRowsPass;
    if (row < p.rows) {
      load(row, hx[i], hy[i]);
      see(hx[i]);
      see(hy[i]);
    }
  }
  for (int row = row0 + kHold * kRowsPass; row < p.rows; row += kRowsPass) {
    float x[8], y[8];
    load(row, x, y);
    see(x);
    see(y);
  }
  top = wave_max(top);
  if constexpr (WAVES > 1) {
    tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = max(top, tops[w]);
  }
  float scale = __uint_as_float(top) * (1.0f / 127.0f), back = 0.0f;
  if (old > 0.0f && top < 0x7f800000u) scale = grown(old, __uint_as_float(top), back);
  const bool finite = top < 0x7f800000u && (__float_as_uint(old) & 0x7fffffffu) < 0x7f800000u;
  if (!finite) scale = __builtin_nanf("");
  if constexpr (WAVES > 1) __syncthreads();  // (the old scale is read before the new one is written)
  if (id == 0) *scale_at = scale;
  int8_t* rows_at = (is_v ? a.v_cache : a.k_cache) + pg.row(p.page, h, p.o0);
  // held rows, where the scale changed: from the page's first slot on
  if (p.o0 > 0 && finite && back != 1.0f) {
    u32x4* piece = reinterpret_cast<u32x4*>(rows_at - p.o0 * D);
    for (int i = id; i < p.o0 * kLanes; i += WAVES * kWave) piece[i] = codes_again(piece[i], back);
  }
  const Coder coder(scale);
  const auto store = [&](int row, const float (&x)[8], const float (&y)[8]) {
    int8_t* dst = rows_at + row * D;
    *reinterpret_cast<u32x2*>(dst + at.e0) = coder.codes(x);
    *reinterpret_cast<u32x2*>(dst + at.e1) = coder.codes(y);
  };
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    const int row = row0 + i * kRowsPass;
    if (row < p.rows) store(row, hx[i], hy[i]);
  }
  for (int row = row0 + kHold * kRowsPass; row < p.rows; row += kRowsPass) {
    float x[8], y[8];
    load(row, x, y);
    store(row, x, y);
  }
}

// A wave's (or workgroup's) tile: which page and rows it is.
template <typename In, int D, bool INTERLEAVED, int WAVES>
__device__ __forceinline__ void quantise_page(const QuantArgs& a, const Pages& pg, int block, uint32_t* tops) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int tile = WAVES == 1 ? block * (kQuantThreads / kWave) + wave : block;
  if (tile >= a.tiles) return;
  const int kinds = 2 * pg.Hkv, u = tile / kinds;
  // (a decode batch: request u's own token)
  int r = min(u, a.R - 1);
  if (a.unit_more != 0 || a.start_of(r) > u || a.start_of(r + 1) <= u)
    r = last_request(a.R, u, [&](int i) { return a.unit_of(i, a.start_of(i)); });
  const int start = a.start_of(r), tokens = max(a.start_of(r + 1) - start, 0);
  const int held = min(max(a.lens[r], 0), pg.capacity());
  const int page_at = (held >> pg.shift) + u - a.unit_of(r, start);  // of the request's pages
  if (u < a.unit_of(r, start) || page_at >= pg.max_blocks) return;
  const int first = max(held, page_at << pg.shift), end = min(held + tokens, (page_at + 1) << pg.shift);
  if (first >= end) return;
  const int page = pg.table[(int64_t)r * pg.max_blocks + page_at];
  if (!pg.has(page)) return;
  const PageRows p{page, start + first - held, first & ((1 << pg.shift) - 1), end - first};
  quantise_tile<In, D, INTERLEAVED, WAVES>(a, pg, p, tile - u * kinds, tops);
}

// Queries: as in moe_kv_append, several heads a thread with the angles it has read.
template <typename In, int D, bool INTERLEAVED>
__device__ __forceinline__ void turn_queries(const QuantArgs& a, uint32_t block) {
  constexpr int kLanes = D / 16;
  if (!a.q_out) return;  // (the rest of a grid's last row)
  const int64_t id = (int64_t)block * kQuantThreads + threadIdx.x, th = id / kLanes;
  const int chunk = (int)(id % kLanes), t = (int)(th / a.q_lanes);
  if (t >= min(a.turns.T, a.start_of(a.R)) || t < a.start_of(0)) return;
  const bool turns = chunk * 16 < a.turns.rot;
  float c[8], s[8], wx[8], wy[8];
  if (turns) load_angles(a.turns, t, chunk, c, s);
  const Runs at(chunk, a.turns.rot / 2, turns && !INTERLEAVED);
  if (a.q_norm) {
    load8(a.q_norm + at.e0, wx);
    load8(a.q_norm + at.e1, wy);
  }
  for (int h = (int)(th - (int64_t)t * a.q_lanes); h < a.Hq; h += a.q_lanes) {
    const In* src = reinterpret_cast<const In*>(a.q) + t * a.q_stride + (int64_t)h * D;
    float x[8], y[8];
    load8(src + at.e0, x);
    load8(src + at.e1, y);
    if (a.q_norm) {
      const float i = row_scale(x, y, kLanes, a.eps);
      norm8(x, i, wx);
      norm8(y, i, wy);
    }
    if (turns) turn_runs<INTERLEAVED>(x, y, c, s);
    uint16_t* dst = a.q_out + ((int64_t)t * a.Hq + h) * D;
    store8_bf16(dst + at.e0, x);
    store8_bf16(dst + at.e1, y);
  }
}

template <typename In, int D, bool INTERLEAVED, int WAVES>
__global__ __launch_bounds__(kQuantThreads) void kv_append_int8_kernel(QuantArgs a, Pages pg) {
  __shared__ uint32_t tops[kQuantThreads / kWave];
  const uint32_t block = grid_block();
  if (block < (uint32_t)a.tile_blocks) quantise_page<In, D, INTERLEAVED, WAVES>(a, pg, (int)block, tops);
  else turn_queries<In, D, INTERLEAVED>(a, block - a.tile_blocks);
}

template <typename In, int D>
void launch_int8(const QuantArgs& a, const Pages& pg, bool interleaved, dim3 grid, hipStream_t s) {
  const bool wave = pg.shift == 4;
  const auto kernel = wave ? interleaved ? kv_append_int8_kernel<In, D, true, 1> : kv_append_int8_kernel<In, D, false, 1>
                           : interleaved ? kv_append_int8_kernel<In, D, true, 4> : kv_append_int8_kernel<In, D, false, 4>;
  hipLaunchKernelGGL(kernel, grid, dim3(kQuantThreads), 0, s, a, pg);
}

}  // namespace eldr

extern "C" int moe_kv_append_int8(const void* q, const void* k, const void* v, int64_t q_stride,
                                  int64_t k_stride, int64_t v_stride, int32_t in_type, int32_t T,
                                  const int32_t* positions, int32_t n_axes, const int32_t* pair_axis,
                                  const float* cos_table, const float* sin_table, int32_t max_pos,
                                  int32_t rot, int32_t interleaved, const int32_t* query_start,
                                  const int32_t* block_table, const int32_t* lens, moe_attn_dims d,
                                  const float* q_norm, const float* k_norm, float eps, uint16_t* q_out,
                                  void* k_cache, void* v_cache, float* k_scale, float* v_scale,
                                  void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  if (d.kv_type != MOE_KV_INT8) return MOE_ERR_INVALID;
  const AppendCheck check{q, k, v, q_stride, k_stride, v_stride, in_type, T, positions, n_axes, pair_axis,
                          cos_table, sin_table, max_pos, rot, q_out, k_cache, v_cache};
  if ((st = check.sizes(d)) != MOE_OK) return st;
  if (!norms_finite(eps)) return MOE_ERR_INVALID;
  if (T == 0 || d.R == 0) return MOE_OK;
  if (!query_start || !lens || (d.max_blocks > 0 && !block_table) || (d.num_blocks > 0 && (!k_scale || !v_scale)))
    return MOE_ERR_INVALID;
  if ((st = check.pointers(d)) != MOE_OK) return st;
  if (!aligned4(query_start) || !aligned4(block_table) || !aligned4(lens) || !aligned4(k_scale) || !aligned4(v_scale) ||
      !aligned16(q_norm) || !aligned16(k_norm))
    return MOE_ERR_UNSUPPORTED;
  eldr::QuantArgs a;
  a.turns = check.rotation();
  a.q = q, a.k = k, a.v = v;
  a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride;
  a.query_start = query_start, a.lens = lens;
  a.q_out = q_out;
  a.q_norm = q_norm, a.k_norm = k_norm, a.eps = eps;
  a.k_cache = static_cast<int8_t*>(k_cache), a.v_cache = static_cast<int8_t*>(v_cache);
  a.k_scale = k_scale, a.v_scale = v_scale;
  a.R = d.R, a.Hq = d.Hq;
  const eldr::Pages pg = pages_of(d, block_table);
  // as few units as hold every page: a unit for each token where requests have few
  const int64_t by_page = ((int64_t)T >> pg.shift) + 2 * (int64_t)d.R;
  const bool by_token = T <= by_page;
  a.unit_shift = by_token ? 0 : pg.shift, a.unit_more = by_token ? 0 : 2;
  const int64_t units = d.num_blocks == 0 || d.max_blocks == 0 ? 0 : by_token ? T : by_page;
  const int64_t tiles = units * 2 * d.Hkv;
  constexpr int kWaves = eldr::kQuantThreads / eldr::kWave;
  const int64_t tile_blocks = pg.shift == 4 ? (tiles + kWaves - 1) / kWaves : tiles;
  // as few threads a token as still fill the chip: 2048 for each CU
  constexpr int64_t kFull = 256 * 2048;
  const int lanes = d.D / 16;
  a.q_lanes = d.Hq;
  while (a.q_lanes > 4 && (int64_t)T * ((a.q_lanes + 1) / 2) * lanes >= kFull / 2) a.q_lanes = (a.q_lanes + 1) / 2;
  const int64_t q_blocks =
      q_out ? ((int64_t)T * a.q_lanes * lanes + eldr::kQuantThreads - 1) / eldr::kQuantThreads : 0;
  if (tiles > 0x7fffffffLL - kWaves || tile_blocks + q_blocks > 0x7fffffffLL) return MOE_ERR_UNSUPPORTED;
  if (tile_blocks + q_blocks == 0) return MOE_OK;
  a.tiles = (int32_t)tiles, a.tile_blocks = (int32_t)tile_blocks;
  const dim3 grid = grid_of(tile_blocks + q_blocks);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool inter = interleaved != 0;
  if (in_type == MOE_IN_FP32) {
    if (d.D == 64) eldr::launch_int8<float, 64>(a, pg, inter, grid, s);
    else if (d.D == 128) eldr::launch_int8<float, 128>(a, pg, inter, grid, s);
    else eldr::launch_int8<float, 256>(a, pg, inter, grid, s);
  } else {
    if (d.D == 64) eldr::launch_int8<uint16_t, 64>(a, pg, inter, grid, s);
    else if (d.D == 128) eldr::launch_int8<uint16_t, 128>(a, pg, inter, grid, s);
    else eldr::launch_int8<uint16_t, 256>(a, pg, inter, grid, s);
  }
  return launch_status();
}

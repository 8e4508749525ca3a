// moe_kv_evict: the slots that stay, and the compaction of the cache.
//
// Two launches.  kv_select, a workgroup a (request, kv head): the budget-th
// largest key by a radix selection (8 bits a pass over 32-bit keys that order
// as the rule does), then one bit a slot in LDS for "stays", and from the
// bits' prefix counts the i-th slot that leaves below the budget and the i-th
// that stays past it, which is its new content.  kv_move copies those rows:
// sources lie past the budget and destinations below it, so no row is both
// read and written and the copies need no order.
#include "attn_common.hpp"

namespace eldr {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / kWave;
constexpr int kMoveThreads = 256;
constexpr int kMoveSlots = 256;  // slots below the budget that a move workgroup looks at

struct EvictArgs {
  const float* weights;
  const int32_t *pos, *lens, *seen, *protect;
  int32_t* src;
  int32_t* new_lens;
  float* weights_out;
  int32_t* pos_out;
  int32_t N, budget, recent, words;  // words: 64-slot words of the bit array (ceil(N / 64))
};

// A slot's rank key: protected slots above every weight; then the weights in
// their order (both zeros alike); NaN last.
__device__ __forceinline__ uint32_t slot_key(float w, bool sure) {
  if (sure) return 0xffffffffu;
  if (w != w) return 0u;
  const uint32_t b = __float_as_uint(w + 0.0f);  // -0 becomes +0
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

// Exclusive sum over the workgroup's threads in order; total to every thread.
__device__ __forceinline__ int block_scan(int v, int* lds, int& total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int x = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == kWave - 1) lds[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kSelectWaves; ++w) {
    const int t = lds[w];
    before += w < wave ? t : 0;
    total += t;
  }
  return before + x - v;
}

// The bit position of the k-th set bit (k from 0) of m.
__device__ __forceinline__ int nth_bit(uint64_t m, int k) {
  int at = 0;
#pragma unroll
  for (int w = 32; w; w >>= 1) {
    const int c = __popcll(m & ((1ull << w) - 1));
    if (k >= c) {
      k -= c;
      m >>= w;
      at += w;
    }
  }
  return at;
}

__global__ __launch_bounds__(kSelectThreads) void kv_select_kernel(EvictArgs a, int Hkv) {
  extern __shared__ uint64_t bits[];                       // [words] slot stays
  int* before = reinterpret_cast<int*>(bits + a.words);    // [words] slots before the word that move here
  __shared__ int hist[256], lds[kSelectWaves], found[2];
  const int r = blockIdx.x / Hkv;
  const int64_t row = (int64_t)blockIdx.x * a.N;
  const int n = min(max(a.lens[r], 0), a.N);
  const int t = threadIdx.x, lane = t % kWave;
  int32_t* src = a.src + (int64_t)blockIdx.x * a.budget;
  if (t == 0 && blockIdx.x % Hkv == 0) a.new_lens[r] = min(n, a.budget);
  if (n <= a.budget) {
    for (int i = t; i < a.budget; i += kSelectThreads) src[i] = i < n ? i : -1;
    if (a.weights_out != a.weights)
      for (int i = t; i < n; i += kSelectThreads) a.weights_out[row + i] = a.weights[row + i];
    if (a.pos_out != a.pos)
      for (int i = t; i < n; i += kSelectThreads) a.pos_out[row + i] = a.pos[row + i];
    return;
  }
  const int protect = a.protect ? a.protect[r] : 0;
  // positions from here on are the last `recent` ones (64 bits: no overflow)
  const int64_t recent_from = (int64_t)a.seen[r] - a.recent;
  const auto key_of = [&](int i) {
    return slot_key(a.weights[row + i], i < protect || a.pos[row + i] >= recent_from);
  };
  // the budget-th largest key, and how many of its equals stay
  uint32_t prefix = 0;
  int want = a.budget;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = t; i < 256; i += kSelectThreads) hist[i] = 0;
    __syncthreads();
    for (int i = t; i < n; i += kSelectThreads) {
      const uint32_t k = key_of(i);
      if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    // bins from the top: the first whose running sum reaches `want`
    const int c = t < 256 ? hist[255 - t] : 0;
    int total;
    const int above = block_scan(c, lds, total);
    if (t < 256 && above < want && above + c >= want) {
      found[0] = 255 - t;
      found[1] = want - above;
    }
    __syncthreads();
    prefix = (prefix << 8) | (uint32_t)found[0];
    want = found[1];
  }
  // who stays: keys above it, and of its equals the first `want` by slot
  int equals = 0;
  for (int i0 = 0; i0 < n; i0 += kSelectThreads) {
    const int i = i0 + t;
    const uint32_t k = i < n ? key_of(i) : 0u;
    const bool eq = i < n && k == prefix;
    int total;
    const int rank = block_scan(eq ? 1 : 0, lds, total);
    const bool stays = i < n && (k > prefix || (eq && equals + rank < want));
    const uint64_t m = __ballot(stays);
    if (lane == 0 && i0 + t < a.N) bits[(i0 + t) / 64] = m;
    equals += total;
  }
  __syncthreads();
  // counts before each word: of leaving slots below the budget, and of staying ones from it on
  const int words = (n + 63) / 64;
  const auto holes_of = [&](int w) -> uint64_t {
    const int left = a.budget - w * 64;
    const uint64_t below = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0ull;
    return ~bits[w] & below;
  };
  const auto movers_of = [&](int w) -> uint64_t {
    const int left = a.budget - w * 64;
    const uint64_t below = left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0ull;
    return bits[w] & ~below;
  };
  // words below the budget's count holes, the budget's own word and later ones movers;
  // the word that holds the budget has both: its holes follow all earlier ones, its movers come first
  const int edge = a.budget / 64;
  int holes_before_edge = 0;
  {
    int carry = 0;
    for (int w0 = 0; w0 < edge; w0 += kSelectThreads) {
      const int w = w0 + t;
      int total;
      const int x = block_scan(w < edge ? (int)__popcll(holes_of(w)) : 0, lds, total);
      if (w < edge) before[w] = carry + x;
      carry += total;
    }
    holes_before_edge = carry;
    carry = 0;
    for (int w0 = edge; w0 < words; w0 += kSelectThreads) {
      const int w = w0 + t;
      int total;
      const int x = block_scan(w < words ? (int)__popcll(movers_of(w)) : 0, lds, total);
      if (w < words) before[w] = carry + x;
      carry += total;
    }
  }
  __syncthreads();
  for (int i = t; i < a.budget; i += kSelectThreads) {
    const int w = i / 64;
    int from = i;
    const uint64_t holes = holes_of(w);
    if ((holes >> (i % 64)) & 1ull) {
      const int rank = (w < edge ? before[w] : holes_before_edge) + (int)__popcll(holes & ((1ull << (i % 64)) - 1));
      // the last word whose movers start at or before the rank-th
      int lo = edge, hi = words - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (before[mid] <= rank) lo = mid;
        else hi = mid - 1;
      }
      from = lo * 64 + nth_bit(movers_of(lo), rank - before[lo]);
    }
    src[i] = from;
    a.weights_out[row + i] = a.weights[row + from];
    a.pos_out[row + i] = a.pos[row + from];
  }
  // in place, slots past the budget are still read above
  __syncthreads();
  for (int i = a.budget + t; i < n; i += kSelectThreads) {
    a.weights_out[row + i] = 0.0f;
    a.pos_out[row + i] = -1;
  }
}

// One workgroup a (request, kv head, run of kMoveSlots slots): the moved ones
// are listed in LDS, then 16 bytes a thread, a row's pieces on neighbouring
// lanes, keys and values in turn.
__global__ __launch_bounds__(kMoveThreads) void kv_move_kernel(EvictArgs a, Pages pg, void* k_cache, void* v_cache,
                                                               int row_shift, int elem) {
  __shared__ int to[kMoveSlots], from[kMoveSlots], count;
  const int rh = blockIdx.y, r = rh / pg.Hkv, h = rh % pg.Hkv;
  if (min(max(a.lens[r], 0), a.N) <= a.budget) return;
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  const int i = blockIdx.x * kMoveSlots + threadIdx.x;
  if (i < a.budget) {
    const int s = a.src[(int64_t)rh * a.budget + i];
    if (s != i) {
      const int at = atomicAdd(&count, 1);  // any order: the rows are copied independently
      to[at] = i;
      from[at] = s;
    }
  }
  __syncthreads();
  const int pieces = count << row_shift;  // of 16 bytes, of one cache
  for (int p = threadIdx.x; p < 2 * pieces; p += kMoveThreads) {
    const bool is_v = p >= pieces;
    const int q = is_v ? p - pieces : p;
    const int m = q >> row_shift, off = (q & ((1 << row_shift) - 1)) * 16;
    const int bt = pg.page(r, to[m]), bf = pg.page(r, from[m]);
    if (!pg.has(bt) || !pg.has(bf)) continue;
    char* cache = reinterpret_cast<char*>(is_v ? v_cache : k_cache);
    const u32x4 x = *reinterpret_cast<const u32x4*>(cache + pg.row(bf, h, from[m]) * elem + off);
    *reinterpret_cast<u32x4*>(cache + pg.row(bt, h, to[m]) * elem + off) = x;
  }
}

}  // namespace eldr

extern "C" int moe_kv_evict(const float* weights, const int32_t* pos, const int32_t* lens,
                            const int32_t* seen, const int32_t* protect, const int32_t* block_table,
                            moe_attn_dims d, int32_t budget, int32_t recent, void* k_cache,
                            void* v_cache, int32_t* src, int32_t* new_lens, float* weights_out,
                            int32_t* pos_out, void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  if (budget < 1 || recent < 0) return MOE_ERR_INVALID;
  if (d.R == 0) return MOE_OK;
  if (!lens || !seen || !src || !new_lens || new_lens == lens) return MOE_ERR_INVALID;
  if (d.max_blocks > 0 && (!weights || !pos || !block_table || !weights_out || !pos_out)) return MOE_ERR_INVALID;
  if (d.num_blocks > 0 && (!k_cache || !v_cache)) return MOE_ERR_INVALID;
  if (budget > MOE_ATTN_MAX_TOKENS || (int64_t)d.R * d.Hkv > 65535) return MOE_ERR_UNSUPPORTED;
  if (!aligned16(weights) || !aligned16(weights_out) || !aligned16(k_cache) || !aligned16(v_cache) ||
      !aligned4(pos) || !aligned4(pos_out) || !aligned4(lens) || !aligned4(seen) || !aligned4(protect) ||
      !aligned4(block_table) || !aligned4(src) || !aligned4(new_lens))
    return MOE_ERR_UNSUPPORTED;
  eldr::EvictArgs a;
  a.weights = weights, a.pos = pos, a.lens = lens, a.seen = seen, a.protect = protect;
  a.src = src, a.new_lens = new_lens, a.weights_out = weights_out, a.pos_out = pos_out;
  a.N = d.num_blocks == 0 ? 0 : d.max_blocks * d.block_size, a.budget = budget, a.recent = recent;
  a.words = (a.N + 63) / 64;
  const size_t lds = (size_t)a.words * 12;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (lds > 60 * 1024 &&
      hipFuncSetAttribute(reinterpret_cast<const void*>(eldr::kv_select_kernel),
                          hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
    (void)hipGetLastError();
    return MOE_ERR_HIP;
  }
  hipLaunchKernelGGL(eldr::kv_select_kernel, dim3(d.R * d.Hkv), dim3(eldr::kSelectThreads), lds, s, a, d.Hkv);
  st = launch_status();
  if (st != MOE_OK || a.N <= budget) return st;
  const int elem = d.kv_type == MOE_KV_FP8 ? 1 : 2;
  const int row_shift = __builtin_ctz((unsigned)(d.D * elem / 16));
  const dim3 grid((budget + eldr::kMoveSlots - 1) / eldr::kMoveSlots, d.R * d.Hkv);
  hipLaunchKernelGGL(eldr::kv_move_kernel, grid, dim3(eldr::kMoveThreads), 0, s, a,
                     pages_of(d, block_table), k_cache, v_cache, row_shift, elem);
  return launch_status();
}

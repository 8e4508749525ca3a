// moe_kv_evict: the slots that stay, and the compaction of the cache.
//
// Selection, a row (request and kv head) at a time: keys of 32 bits that order
// as the rule does, and the budget-th largest of them by a radix selection, 8
// bits a pass.  Rows of up to 32,768 slots (kv_select) keep their keys in
// registers, in one wave to 16 of them: a pass is an LDS histogram and one
// barrier, after which every wave finds the digit by itself.  Longer rows
// (kv_select_long) read their keys again for each pass.  Then one bit a slot in
// LDS says "stays", and the prefix counts of the bits pair the i-th slot that
// leaves below the budget with the i-th that stays past it.
//
// kv_move copies those rows: sources lie past the budget and destinations below
// it, so no row is both read and written and the copies need no order.  Where the
// table holds no more than 64 slots over the budget (one made for the budget and for
// what the steps append), kv_select copies them itself and there is no second launch.
// Both choices go by the table, whose width the host knows, not by the lengths, which
// only the device does: a table far wider than its requests' caches pays for it.
//
// Measured: 256 caches of 4 heads, one token each past 1024, 16.6 us (a lane's
// loads, four barriers and the launch; 48 us with keys read again for each digit and
// the move by itself) in tables of 1040 slots, 18 in 2048, 29 in 4096 and 8192 (a
// selection of 1024 lanes of 8 keys for rows of 1025), 44 in 32,768 and 46 in 65,536
// (keys read again); letting each row's length decide who moves it gained 0 to 2 us
// there and cost others 1 to 3%.  64 of up to 4096 cut to 2048 15 us and the move 35
// (172 MB, 4.9 TB/s, a large copy's rate).
#include "attn_common.hpp"

namespace eldr {

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / kWave;
constexpr int kShortRow = 16 * 32 * 64;            // slots of a row whose keys fit 16 waves
constexpr int kFewMoves = 64;                      // rows that kv_select copies itself
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

// The row is within its budget: nothing changes.
__device__ __forceinline__ void keep_all(const EvictArgs& a, int64_t row, int32_t* src, int n, int t, int threads) {
  for (int i = t; i < a.budget; i += threads) src[i] = i < n ? i : -1;
  if (a.weights_out == a.weights && a.pos_out == a.pos) return;
  constexpr int kBatch = 8;  // in flight together
  for (int i0 = t; i0 < n; i0 += kBatch * threads) {
    float weight[kBatch];
    int pos[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int i = min(i0 + b * threads, n - 1);
      weight[b] = a.weights[row + i];
      pos[b] = a.pos[row + i];
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int i = i0 + b * threads;
      if (i >= n) break;
      a.weights_out[row + i] = weight[b];
      a.pos_out[row + i] = pos[b];
    }
  }
}

// Of the 64 slots of word w: those below the budget.
__device__ __forceinline__ uint64_t below_budget(int w, int budget) {
  const int left = budget - w * 64;
  return left >= 64 ? ~0ull : left > 0 ? (1ull << left) - 1 : 0ull;
}

// Copies the keys' and values' row of slot `from` to slot `to`, 16 bytes a lane:
// pieces [0, 2 << row_shift), keys first.
__device__ __forceinline__ void copy_piece(const Pages& pg, void* k_cache, void* v_cache, int r, int h, int to, int from, int piece,
                                           int row_shift, int elem) {
  const int bt = pg.page(r, to), bf = pg.page(r, from);
  if (!pg.has(bt) || !pg.has(bf)) return;
  char* cache = reinterpret_cast<char*>(piece >> row_shift ? v_cache : k_cache);
  const int off = (piece & ((1 << row_shift) - 1)) * 16;
  const u32x4 x = *reinterpret_cast<const u32x4*>(cache + pg.row(bf, h, from) * elem + off);
  *reinterpret_cast<u32x4*>(cache + pg.row(bt, h, to) * elem + off) = x;
}

// One row by WAVES waves, KEYS slots a lane: n <= WAVES * KEYS * 64.  Slot i is
// key i / THREADS of thread i % THREADS, so a ballot covers 64 neighbouring slots.
template <int WAVES, int KEYS, bool MOVES>
__global__ __launch_bounds__(WAVES * kWave) void kv_select_kernel(EvictArgs a, Pages pg, void* k_cache, void* v_cache, int row_shift,
                                                                  int elem) {
  constexpr int kThreads = WAVES * kWave, kWords = WAVES * KEYS, kDigits = 256;
  __shared__ int hist[4][kDigits];          // a pass each; bin d counts digit 255 - d
  __shared__ uint64_t stays[kWords], ties[kWords];
  __shared__ int before[kWords];            // holes, or movers, before the word's
  __shared__ uint16_t movers[kWords * 32 < 2 * kFewMoves ? 2 * kFewMoves : kWords * 32];  // staying slots past the budget
  __shared__ int holes_at_edge;
  const int r = blockIdx.x / pg.Hkv, h = blockIdx.x % pg.Hkv;
  const int64_t row = (int64_t)blockIdx.x * a.N;
  const int n = min(max(a.lens[r], 0), a.N), budget = a.budget;
  const int t = threadIdx.x, lane = t % kWave, wave = __builtin_amdgcn_readfirstlane(t / kWave);
  int32_t* src = a.src + (int64_t)blockIdx.x * budget;
  if (t == 0 && h == 0) a.new_lens[r] = min(n, budget);
  if (n <= budget) {
    keep_all(a, row, src, n, t, kThreads);
    return;
  }
  const int protect = a.protect ? a.protect[r] : 0;
  // positions from here on are the last `recent` ones (64 bits: no overflow)
  const int64_t recent_from = (int64_t)a.seen[r] - a.recent;
  // f(k) for the keys that the row has, eight at a time
  const auto each_key = [&](auto f) {
#pragma unroll
    for (int k0 = 0; k0 < KEYS; k0 += 8) {
      if (k0 * kThreads < n) {
#pragma unroll
        for (int k = k0; k < k0 + 8; ++k) f(k);
      }
    }
  };
  uint32_t key[KEYS];
  each_key([&](int k) {
    const int i = min(k * kThreads + t, n - 1);
    key[k] = slot_key(a.weights[row + i], i < protect || a.pos[row + i] >= recent_from);
  });
  for (int i = t; i < 4 * kDigits; i += kThreads) (&hist[0][0])[i] = 0;
  __syncthreads();
  // The digits of the budget-th largest key from the top.  `all`: the keys that
  // share the digits found so far all stay, so no further digit is needed.
  uint32_t prefix = 0;
  int want = budget, shift = 32;
  bool all = false;
  for (int pass = 0; pass < 4 && !all; ++pass) {
    const int above_bits = shift;
    shift -= 8;
    each_key([&](int k) {
      if (k * kThreads + t < n && (pass == 0 || key[k] >> above_bits == prefix))
        atomicAdd(&hist[pass][255 - (int)(key[k] >> shift & 255u)], 1);
    });
    __syncthreads();
    // four bins a lane, largest digits first: the first bin at which the running sum reaches `want`
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    const i32x4 c = *reinterpret_cast<const i32x4*>(&hist[pass][4 * lane]);
    const int mine = c[0] + c[1] + c[2] + c[3], upto = wave_sum_before(mine);
    const int at = __builtin_ctzll(__ballot(upto >= want));
    int above = __builtin_amdgcn_readlane(upto - mine, at), bin = 4 * at;
    int count = __builtin_amdgcn_readlane(c[0], at);
#pragma unroll
    for (int b = 1; b < 4; ++b) {
      if (above + count >= want) break;
      above += count;
      ++bin;
      count = __builtin_amdgcn_readlane(c[b], at);
    }
    prefix = prefix << 8 | (uint32_t)(255 - bin);
    want -= above;
    all = want == count;
  }
  // every key above the digits found stays; of the others that share all 32 bits, the first `want` by slot
  each_key([&](int k) {
    const bool real = k * kThreads + t < n;
    const uint32_t x = key[k] >> shift;
    const uint64_t m = __ballot(real && (all ? x >= prefix : x > prefix));
    const uint64_t e = __ballot(real && !all && x == prefix);
    if (lane == 0) stays[k * WAVES + wave] = m, ties[k * WAVES + wave] = e;
  });
  __syncthreads();
  // a wave's work on words, then everybody's on slots
  const int words = (n + 63) / 64, edge = budget / 64;
  if (wave == 0) {
    constexpr int kPer = (kWords + kWave - 1) / kWave;  // words a lane
    const int w0 = lane * kPer, w1 = min(w0 + kPer, words);
    if (!all) {
      int mine = 0;
      for (int w = w0; w < w1; ++w) mine += (int)__popcll(ties[w]);
      int left = want - (wave_sum_before(mine) - mine);
      for (int w = w0; w < w1; ++w) {
        const uint64_t m = ties[w];
        const int c = (int)__popcll(m);
        if (left >= c) stays[w] |= m;
        else if (left > 0) stays[w] |= m & ((1ull << nth_bit(m, left)) - 1);
        left -= c;
      }
    }
    // holes before each word below the edge (in the low half), movers before each from it on
    int mine = 0;
    for (int w = w0; w < w1; ++w) {
      const uint64_t below = below_budget(w, budget);
      mine += w < edge ? (int)__popcll(~stays[w] & below) : (int)__popcll(stays[w] & ~below) << 16;
    }
    int at = wave_sum_before(mine);
    if (lane == kWave - 1) holes_at_edge = at & 0xffff;
    at -= mine;
    for (int w = w0; w < w1; ++w) {
      const uint64_t below = below_budget(w, budget);
      before[w] = w < edge ? at & 0xffff : at >> 16;
      at += w < edge ? (int)__popcll(~stays[w] & below) : (int)__popcll(stays[w] & ~below) << 16;
    }
  }
  __syncthreads();
  for (int w = edge + wave; w < words; w += WAVES) {
    const uint64_t m = stays[w] & ~below_budget(w, budget);
    if (m >> lane & 1) movers[before[w] + (int)__popcll(m & ((1ull << lane) - 1))] = (uint16_t)(w * 64 + lane);
  }
  __syncthreads();
  const bool same_w = a.weights_out == a.weights, same_p = a.pos_out == a.pos;
  // Batches, so that a batch's loads are in flight together.  Nothing read here is
  // written before the barrier by another thread: a slot below the budget is read
  // by its own thread alone.
  constexpr int kBatch = 8;
  for (int i0 = t; i0 < budget; i0 += kBatch * kThreads) {
    int from[kBatch], pos[kBatch];
    float weight[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int i = min(i0 + b * kThreads, budget - 1), w = i / 64;
      const uint64_t holes = ~stays[w] & below_budget(w, budget);
      const int rank = (w < edge ? before[w] : holes_at_edge) + (int)__popcll(holes & ((1ull << (i % 64)) - 1));
      const bool hole = holes >> (i % 64) & 1;
      from[b] = hole ? movers[rank] : i;
      if (MOVES && hole) movers[rank + kFewMoves] = (uint16_t)i;  // where the rank-th goes
      weight[b] = a.weights[row + from[b]];
      pos[b] = a.pos[row + from[b]];
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int i = i0 + b * kThreads;
      if (i >= budget) break;
      src[i] = from[b];
      if (from[b] != i || !same_w) a.weights_out[row + i] = weight[b];
      if (from[b] != i || !same_p) a.pos_out[row + i] = pos[b];
    }
  }
  // in place, slots past the budget are still read above
  __syncthreads();
  for (int i = budget + t; i < n; i += kThreads) {
    a.weights_out[row + i] = 0.0f;
    a.pos_out[row + i] = -1;
  }
  if constexpr (MOVES) {
    const int last = words - 1;
    const int count = before[last] + (int)__popcll(stays[last] & ~below_budget(last, budget));
    const int pieces = 2 << row_shift;
    for (int p = t; p < count * pieces; p += kThreads) {
      const int m = p / pieces;
      copy_piece(pg, k_cache, v_cache, r, h, movers[m + kFewMoves], movers[m], p - m * pieces, row_shift, elem);
    }
  }
}

__global__ __launch_bounds__(kSelectThreads) void kv_select_long_kernel(EvictArgs a, int Hkv) {
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
    keep_all(a, row, src, n, t, kSelectThreads);
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
  const auto holes_of = [&](int w) { return ~bits[w] & below_budget(w, a.budget); };
  const auto movers_of = [&](int w) { return bits[w] & ~below_budget(w, a.budget); };
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

// One workgroup a (request, kv head, run of kMoveSlots slots): the moved rows'
// offsets are listed in LDS, pages looked up once a row, then 16 bytes a thread
// and four of them in flight, a row's pieces on neighbouring lanes.
__global__ __launch_bounds__(kMoveThreads) void kv_move_kernel(EvictArgs a, Pages pg, char* k_cache, char* v_cache, int row_shift,
                                                               int elem) {
  __shared__ int64_t to[kMoveSlots], from[kMoveSlots];  // bytes
  __shared__ int count;
  const int rh = blockIdx.y, r = rh / pg.Hkv, h = rh % pg.Hkv;
  if (min(max(a.lens[r], 0), a.N) <= a.budget) return;
  if (threadIdx.x == 0) count = 0;
  __syncthreads();
  const int i = blockIdx.x * kMoveSlots + threadIdx.x;
  if (i < a.budget) {
    const int s = a.src[(int64_t)rh * a.budget + i];
    if (s != i) {
      const int bt = pg.page(r, i), bf = pg.page(r, s);
      if (pg.has(bt) && pg.has(bf)) {
        const int at = atomicAdd(&count, 1);  // any order: the rows are copied independently
        to[at] = pg.row(bt, h, i) * elem;
        from[at] = pg.row(bf, h, s) * elem;
      }
    }
  }
  __syncthreads();
  const int pieces = count << row_shift;  // of one cache
  constexpr int kBatch = 4;
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    char* cache = v ? v_cache : k_cache;
    for (int p0 = threadIdx.x; p0 < pieces; p0 += kBatch * kMoveThreads) {
      u32x4 x[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int p = min(p0 + b * kMoveThreads, pieces - 1);
        x[b] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x4*>(cache + from[p >> row_shift] + (p & ((1 << row_shift) - 1)) * 16));
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int p = p0 + b * kMoveThreads;
        if (p < pieces) *reinterpret_cast<u32x4*>(cache + to[p >> row_shift] + (p & ((1 << row_shift) - 1)) * 16) = x[b];
      }
    }
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
  if (d.kv_type == MOE_KV_INT8) return MOE_ERR_UNSUPPORTED;  // (a moved row would need its new page's scale)
  if (budget < 1 || recent < 0) return MOE_ERR_INVALID;
  if (d.R == 0) return MOE_OK;
  if (!lens || !seen || !src || !new_lens || new_lens == lens) return MOE_ERR_INVALID;
  if (d.max_blocks > 0 && (!weights || !pos || !block_table || !weights_out || !pos_out)) return MOE_ERR_INVALID;
  if (d.num_blocks > 0 && (!k_cache || !v_cache)) return MOE_ERR_INVALID;
  if (budget > MOE_ATTN_MAX_TOKENS || (int64_t)d.R * d.Hkv > 65535) return MOE_ERR_UNSUPPORTED;
  if (!aligned4(weights) || !aligned4(weights_out) || !aligned16(k_cache) || !aligned16(v_cache) ||
      !aligned4(pos) || !aligned4(pos_out) || !aligned4(lens) || !aligned4(seen) || !aligned4(protect) ||
      !aligned4(block_table) || !aligned4(src) || !aligned4(new_lens))
    return MOE_ERR_UNSUPPORTED;
  eldr::EvictArgs a;
  a.weights = weights, a.pos = pos, a.lens = lens, a.seen = seen, a.protect = protect;
  a.src = src, a.new_lens = new_lens, a.weights_out = weights_out, a.pos_out = pos_out;
  a.N = d.num_blocks == 0 ? 0 : d.max_blocks * d.block_size, a.budget = budget, a.recent = recent;
  a.words = (a.N + 63) / 64;
  const eldr::Pages pg = pages_of(d, block_table);
  const int elem = d.kv_type == MOE_KV_FP8 ? 1 : 2;
  const int row_shift = __builtin_ctz((unsigned)(d.D * elem / 16));
  const bool moves = a.N - budget <= eldr::kFewMoves;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const dim3 rows(d.R * d.Hkv);
#define ELDR_SELECT(W, K)                                                                                        \
  do {                                                                                                           \
    if (moves)                                                                                                   \
      hipLaunchKernelGGL((eldr::kv_select_kernel<W, K, true>), rows, dim3(W * eldr::kWave), 0, s, a, pg, k_cache, \
                         v_cache, row_shift, elem);                                                              \
    else                                                                                                         \
      hipLaunchKernelGGL((eldr::kv_select_kernel<W, K, false>), rows, dim3(W * eldr::kWave), 0, s, a, pg, k_cache, \
                         v_cache, row_shift, elem);                                                              \
  } while (0)
  // eight keys a lane, while 16 waves can hold the row so
  if (a.N <= 8 * 64) {
    ELDR_SELECT(1, 8);
  } else if (a.N <= 4 * 8 * 64) {
    ELDR_SELECT(4, 8);
  } else if (a.N <= 16 * 8 * 64) {
    ELDR_SELECT(16, 8);
  } else if (a.N <= eldr::kShortRow) {
    ELDR_SELECT(16, 32);
  } else {
    const size_t lds = (size_t)a.words * 12;
    if (lds > 60 * 1024 &&
        hipFuncSetAttribute(reinterpret_cast<const void*>(eldr::kv_select_long_kernel),
                            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) {
      (void)hipGetLastError();
      return MOE_ERR_HIP;
    }
    hipLaunchKernelGGL(eldr::kv_select_long_kernel, rows, dim3(eldr::kSelectThreads), lds, s, a, d.Hkv);
  }
#undef ELDR_SELECT
  st = launch_status();
  if (st != MOE_OK || a.N <= budget || (moves && a.N <= eldr::kShortRow)) return st;
  const dim3 grid((budget + eldr::kMoveSlots - 1) / eldr::kMoveSlots, d.R * d.Hkv);
  hipLaunchKernelGGL(eldr::kv_move_kernel, grid, dim3(eldr::kMoveThreads), 0, s, a, pg, static_cast<char*>(k_cache),
                     static_cast<char*>(v_cache), row_shift, elem);
  return launch_status();
}

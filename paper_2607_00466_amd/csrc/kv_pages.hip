// moe_kv_fork and moe_kv_compact: rows and pages of the paged cache copied in all
// layers at once, block tables beside them.
//
// Both are copies, bound by bytes where there are many and by a chain of three
// dependent loads (who, which page, its rows) where there are few: one launch, a
// workgroup for one fork or moving page and a run of layers, 16-byte pieces, four
// of a thread's in flight.  Measured: 64 forks in 48 layers (46 MB read and written)
// 11.4 us, 32 requests' pages compacted in 48 layers (533 MB) 115 us, 4.6 TB/s of a
// large copy's 4.74 to 4.93; 4 forks in one layer 3.4.
//
// Compaction has a workgroup for every page and run of layers, moving or not, which is
// what a pool much larger than what moves costs: 32 pages of 4 x 16 x 128 in 8 bits out
// of 100,000 32 us in one layer and 62 in 8, out of 130,000 in 48 layers (102 GB) 455 (a
// copy of them: 11); 1000 of those 640 (332).
#include <algorithm>

#include "attn_common.hpp"
#include "eldr_kv_cache.h"

namespace eldr {

constexpr int kPageThreads = 256;
constexpr int kPieceBytes = 16;

// The caches of all layers, in bytes.
struct Layers {
  char *k_cache, *v_cache;
  float *k_scale, *v_scale;  // [layers, num_blocks, Hkv], or null
  int64_t layer_bytes, block_bytes;
  int32_t count, Hkv, num_blocks;
  int32_t head_pieces;       // of a page and head
};

// Pieces [0, pieces) of each kv head of page `from`, of the keys and the values of
// layer `layer`, to page `to`; the page's scales too.  `take` of `share` workgroups.
// ONCE: by non-temporal loads and stores, for what is not read again soon (32 requests'
// pages in 48 layers, 533 MB: 121 -> 115 us; 64 forks of 16 pages in 48 layers lose by
// them, 12 -> 16, since each page is read for four copies).
template <bool ONCE>
__device__ __forceinline__ void copy_page(const Layers& c, int layer, int from, int to, int pieces, int take, int share) {
  const int64_t at = (int64_t)layer * c.layer_bytes;
  const char *ks = c.k_cache + at + from * c.block_bytes, *vs = c.v_cache + at + from * c.block_bytes;
  char *kd = c.k_cache + at + to * c.block_bytes, *vd = c.v_cache + at + to * c.block_bytes;
  const int of_cache = c.Hkv * pieces, all = 2 * of_cache;
  constexpr int kBatch = 4;
  for (int i0 = take * kPageThreads * kBatch + threadIdx.x; i0 < all; i0 += share * kPageThreads * kBatch) {
    u32x4 x[kBatch];
    char* dst[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int i = min(i0 + b * kPageThreads, all - 1);
      const bool is_v = i >= of_cache;
      const int j = is_v ? i - of_cache : i, h = j / pieces;
      const int64_t off = (int64_t)(h * c.head_pieces + (j - h * pieces)) * kPieceBytes;
      const u32x4* src = reinterpret_cast<const u32x4*>((is_v ? vs : ks) + off);
      x[b] = ONCE ? __builtin_nontemporal_load(src) : *src;
      dst[b] = (is_v ? vd : kd) + off;
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (i0 + b * kPageThreads >= all) break;
      if (ONCE) __builtin_nontemporal_store(x[b], reinterpret_cast<u32x4*>(dst[b]));
      else *reinterpret_cast<u32x4*>(dst[b]) = x[b];
    }
  }
  if (c.k_scale && take == 0) {
    const int64_t row = (int64_t)layer * c.num_blocks;
    for (int h = threadIdx.x; h < 2 * c.Hkv; h += kPageThreads) {
      float* s = h < c.Hkv ? c.k_scale : c.v_scale;
      const int i = h < c.Hkv ? h : h - c.Hkv;
      s[(row + to) * c.Hkv + i] = s[(row + from) * c.Hkv + i];
    }
  }
}

// A workgroup: fork blockIdx.x, layers [run blockIdx.y, + run), share blockIdx.z.
__global__ __launch_bounds__(kPageThreads) void kv_fork_kernel(const int32_t* parent, const int32_t* child, const int32_t* page,
                                                               int32_t* table, int32_t* lens, Pages pg, Layers c, int R, int run) {
  const int f = blockIdx.x, p = parent[f], to_row = child[f];
  if ((uint32_t)p >= (uint32_t)R || (uint32_t)to_row >= (uint32_t)R || p == to_row) return;
  const int n = min(max(lens[p], 0), pg.capacity());
  const int full = n >> pg.shift, rest = n & ((1 << pg.shift) - 1);
  const int32_t* from_table = table + (int64_t)p * pg.max_blocks;
  int from = -1, to = -1;
  if (rest > 0) {
    from = from_table[full];
    to = page[f];
  }
  const bool copies = pg.has(from) && pg.has(to);
  if (blockIdx.y == 0 && blockIdx.z == 0) {
    int32_t* to_table = table + (int64_t)to_row * pg.max_blocks;
    for (int j = threadIdx.x; j < pg.max_blocks; j += kPageThreads)
      to_table[j] = j < full ? from_table[j] : j == full && copies ? to : -1;
    if (threadIdx.x == 0) lens[to_row] = n;
  }
  if (!copies) return;
  const int pieces = rest * (c.head_pieces >> pg.shift);
  for (int l = blockIdx.y * run; l < min(c.count, (int)(blockIdx.y + 1) * run); ++l)
    copy_page<false>(c, l, from, to, pieces, blockIdx.z, gridDim.z);
}

// Where page b is afterwards, -1: nowhere.
__device__ __forceinline__ int page_after(const Pages& pg, const int32_t* remap, int b) {
  if (!pg.has(b)) return -1;
  const int to = remap[b];
  if (!pg.has(to)) return -1;
  // a page that is held does not receive another
  return to == b || pg.has(remap[to]) ? b : to;
}

// Workgroups: a page's run of layers each (or a share of one layer), then the block table.
__global__ __launch_bounds__(kPageThreads) void kv_compact_kernel(const int32_t* remap, const int32_t* table, int32_t* table_out,
                                                                  int64_t entries, Pages pg, Layers c, int run, int runs, int share) {
  const int parts = runs * share;
  const int64_t moves = (int64_t)pg.num_blocks * parts;
  const uint32_t block = grid_block();
  if (block >= moves) {
    const int64_t i = (block - moves) * kPageThreads + threadIdx.x;
    if (i < entries) table_out[i] = page_after(pg, remap, table[i]);
    return;
  }
  const int b = (int)(block / (uint32_t)parts), part = (int)(block - (uint32_t)b * (uint32_t)parts);
  const int l0 = part / share * run, take = part % share;
  const int to = page_after(pg, remap, b);
  if (to < 0 || to == b) return;
  for (int l = l0; l < min(c.count, l0 + run); ++l) copy_page<true>(c, l, b, to, c.head_pieces, take, share);
}

}  // namespace eldr

namespace eldr_host {

// The checks of the caches of several layers, and the kernels' view of them.
inline int layers_of(const moe_attn_dims& d, int32_t layers, int64_t layer_stride, void* k_cache, void* v_cache, float* k_scale,
                     float* v_scale, eldr::Layers& c) {
  if (layers < 0 || layer_stride < 0) return MOE_ERR_INVALID;
  if (layers > MOE_KV_MAX_LAYERS || layer_stride % 16 != 0) return MOE_ERR_UNSUPPORTED;
  const int64_t dense = (int64_t)d.Hkv * d.block_size * d.D, block = d.block_stride ? d.block_stride : dense;
  const int64_t span = (int64_t)d.num_blocks * block;
  if (layer_stride == 0) layer_stride = span;
  // a layer lies behind the one before, or beside it inside the block stride
  if (layers > 1 && layer_stride < span && (layer_stride < dense || layer_stride > block / layers)) return MOE_ERR_INVALID;
  const bool int8 = d.kv_type == MOE_KV_INT8;
  if (layers > 0 && d.num_blocks > 0 && (!k_cache || !v_cache || (int8 && (!k_scale || !v_scale)))) return MOE_ERR_INVALID;
  if (!aligned16(k_cache) || !aligned16(v_cache) || (int8 && (!aligned4(k_scale) || !aligned4(v_scale)))) return MOE_ERR_UNSUPPORTED;
  const int elem = d.kv_type == MOE_KV_BF16 ? 2 : 1;
  c.k_cache = static_cast<char*>(k_cache), c.v_cache = static_cast<char*>(v_cache);
  c.k_scale = int8 ? k_scale : nullptr, c.v_scale = int8 ? v_scale : nullptr;
  c.layer_bytes = layer_stride * elem, c.block_bytes = block * elem;
  c.count = layers, c.Hkv = d.Hkv, c.num_blocks = d.num_blocks;
  c.head_pieces = d.block_size * d.D * elem / eldr::kPieceBytes;
  return MOE_OK;
}

// How a page of all layers is dealt: a workgroup copies `run` layers, or one of
// `share` parts of a layer, some 64 KB.
struct PageDeal {
  int run, runs, share;
  explicit PageDeal(const eldr::Layers& c) {
    constexpr int64_t kBytes = 1 << 16;
    const int64_t page = (int64_t)2 * c.Hkv * c.head_pieces * eldr::kPieceBytes;
    run = (int)std::max<int64_t>(1, std::min<int64_t>(kBytes / page, c.count));
    runs = (c.count + run - 1) / run;
    share = (int)std::min<int64_t>((page + kBytes - 1) / kBytes, 256);
  }
};

}  // namespace eldr_host

extern "C" int moe_kv_fork(const int32_t* parent, const int32_t* child, const int32_t* page, int32_t F, int32_t* block_table,
                           int32_t* lens, moe_attn_dims d, int32_t layers, int64_t layer_stride, void* k_cache, void* v_cache,
                           float* k_scale, float* v_scale, void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  if (F < 0) return MOE_ERR_INVALID;
  if (F > MOE_KV_MAX_FORKS) return MOE_ERR_UNSUPPORTED;
  eldr::Layers c;
  if ((st = layers_of(d, layers, layer_stride, k_cache, v_cache, k_scale, v_scale, c)) != MOE_OK) return st;
  if (F == 0 || d.R == 0) return MOE_OK;
  if (!parent || !child || !page || !lens || (d.max_blocks > 0 && !block_table)) return MOE_ERR_INVALID;
  if (!aligned4(parent) || !aligned4(child) || !aligned4(page) || !aligned4(lens) || !aligned4(block_table))
    return MOE_ERR_UNSUPPORTED;
  const PageDeal deal(c);
  const dim3 grid((unsigned)F, (unsigned)std::max(deal.runs, 1), (unsigned)deal.share);  // (no layer: the table alone)
  hipLaunchKernelGGL(eldr::kv_fork_kernel, grid, dim3(eldr::kPageThreads), 0, reinterpret_cast<hipStream_t>(stream), parent, child,
                     page, block_table, lens, pages_of(d, nullptr), c, d.R, deal.run);
  return launch_status();
}

extern "C" int moe_kv_compact(const int32_t* remap, const int32_t* block_table, int32_t* table_out, moe_attn_dims d, int32_t layers,
                              int64_t layer_stride, void* k_cache, void* v_cache, float* k_scale, float* v_scale, void* stream) {
  using namespace eldr_host;
  int st = check_attn_dims(d);
  if (st != MOE_OK) return st;
  eldr::Layers c;
  if ((st = layers_of(d, layers, layer_stride, k_cache, v_cache, k_scale, v_scale, c)) != MOE_OK) return st;
  const int64_t entries = (int64_t)d.R * d.max_blocks;
  if (entries == 0 && d.num_blocks == 0) return MOE_OK;
  if ((d.num_blocks > 0 && !remap) || (entries > 0 && (!block_table || !table_out))) return MOE_ERR_INVALID;
  if (!aligned4(remap) || !aligned4(block_table) || !aligned4(table_out)) return MOE_ERR_UNSUPPORTED;
  const PageDeal deal(c);
  const int64_t blocks = (int64_t)d.num_blocks * deal.runs * deal.share + (entries + eldr::kPageThreads - 1) / eldr::kPageThreads;
  if (blocks > 0x7fffffffLL) return MOE_ERR_UNSUPPORTED;
  if (blocks == 0) return MOE_OK;
  hipLaunchKernelGGL(eldr::kv_compact_kernel, grid_of(blocks), dim3(eldr::kPageThreads), 0, reinterpret_cast<hipStream_t>(stream), remap,
                     block_table, table_out, entries, pages_of(d, nullptr), c, deal.run, deal.runs, deal.share);
  return launch_status();
}

// What the attention kernels share: the paged cache's addresses, its two value
// types, and the host's checks of moe_attn_dims.
#pragma once

#include "common.hpp"
#include "eldr_attention.h"

namespace eldr {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A load through the scalar cache: p is the same for the whole wave, and nothing
// writes there while the kernel runs.  (Without the constant address space the
// compiler has to use a vector load, whose wait also waits for every tile that
// was asked for before it.)
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *reinterpret_cast<const __attribute__((address_space(4))) T*>(reinterpret_cast<uintptr_t>(p));
}

// The kernels' view of one cache: pages of block_size = 1 << shift slots.
struct Pages {
  const int32_t* table;  // [R, max_blocks]
  int64_t block_stride;  // elements
  int32_t shift, max_blocks, num_blocks, Hkv, D;

  // Slots a request can have.
  __device__ __forceinline__ int capacity() const { return max_blocks << shift; }
  // The page of slot j of request r; outside [0, num_blocks) where it is absent.
  __device__ __forceinline__ int page(int r, int j) const {
    return table[(int64_t)r * max_blocks + (j >> shift)];
  }
  __device__ __forceinline__ bool has(int b) const { return (uint32_t)b < (uint32_t)num_blocks; }
  // Element offset of slot j's row of kv head h in page b.
  __device__ __forceinline__ int64_t row(int b, int h, int j) const {
    return (int64_t)b * block_stride + (int64_t)((h << shift) + (j & ((1 << shift) - 1))) * D;
  }
};

// Inclusive sum over a wave's lanes, by data-parallel moves: within rows of 16,
// then each row's last sum to the rows after it.
__device__ __forceinline__ int wave_sum_before(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15, to rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast 31, to rows 2 and 3
  return x;
}

// Between LDS that some lanes of a wave wrote and other lanes of it read, or the
// other way round.  The hardware keeps a wave's LDS operations in order, so no wait
// comes of this: it keeps the compiler from moving one of them past it.
__device__ __forceinline__ void wave_handover() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Round to nearest even; two values in one word, the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const bf16x2 v = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, v);
}

}  // namespace eldr

namespace eldr_host {

inline bool power_of_two(int32_t v) { return v > 0 && (v & (v - 1)) == 0; }

// The shape that every attention call shares.
inline int check_attn_dims(const moe_attn_dims& d) {
  if (d.R < 0 || d.Hq <= 0 || d.Hkv <= 0 || d.D <= 0 || d.block_size <= 0 || d.max_blocks < 0 ||
      d.num_blocks < 0 || d.block_stride < 0 || d.Hq % d.Hkv != 0)
    return MOE_ERR_INVALID;
  if (d.kv_type != MOE_KV_BF16 && d.kv_type != MOE_KV_FP8 && d.kv_type != MOE_KV_INT8) return MOE_ERR_INVALID;
  const int64_t dense = (int64_t)d.Hkv * d.block_size * d.D;
  if (d.block_stride != 0 && d.block_stride < dense) return MOE_ERR_INVALID;
  if (d.R > MOE_ATTN_MAX_R || d.Hq > MOE_ATTN_MAX_HEADS) return MOE_ERR_UNSUPPORTED;
  if (d.D != 64 && d.D != 128 && d.D != 256) return MOE_ERR_UNSUPPORTED;
  if (!power_of_two(d.block_size) || d.block_size < MOE_ATTN_MIN_BLOCK || d.block_size > MOE_ATTN_MAX_BLOCK)
    return MOE_ERR_UNSUPPORTED;
  if ((int64_t)d.max_blocks * d.block_size > MOE_ATTN_MAX_TOKENS) return MOE_ERR_UNSUPPORTED;
  // rows start at multiples of 16 bytes
  if (d.block_stride % 16 != 0) return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

inline eldr::Pages pages_of(const moe_attn_dims& d, const int32_t* table) {
  eldr::Pages p;
  p.table = table;
  p.block_stride = d.block_stride ? d.block_stride : (int64_t)d.Hkv * d.block_size * d.D;
  p.shift = __builtin_ctz((unsigned)d.block_size);
  p.max_blocks = d.max_blocks;
  p.num_blocks = d.num_blocks;
  p.Hkv = d.Hkv;
  p.D = d.D;
  return p;
}

}  // namespace eldr_host

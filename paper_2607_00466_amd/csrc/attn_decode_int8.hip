// moe_attn_decode's kernels for pages of 8-bit integers.
#include "attn_decode.hpp"

namespace eldr {

int launch_decode_int8(int D, const DecodeArgs& a, const Pages& pg, float* ws, hipStream_t s) {
  return D == 64    ? launch_decode<64, kKvInt8>(a, pg, ws, s)
         : D == 128 ? launch_decode<128, kKvInt8>(a, pg, ws, s)
                    : launch_decode<256, kKvInt8>(a, pg, ws, s);
}

}  // namespace eldr

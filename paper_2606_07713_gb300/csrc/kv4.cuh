// The 4-bit cache of keys and values: its numbers and its layout, shared by the kernels that write
// it, read it back and attend over it.
//
// Numbers.  32 neighbouring features of one head and token share the scale s = bf16(max|x| / 7);
// a feature is the code rint(x / s) in [-7, 7] and stands for code * s.  (Four bits and half a
// bit of scale a value.  bf16 scales keep the range of bf16 inputs; a scale that underflows to
// zero gives codes of zero; a group with a member that is not finite gets a NaN scale.)
//
// Layout.  A pool [pages, heads, page / 16] of blocks; a block holds 16 tokens of one head in
// 9 (dk + dv) contiguous bytes: key codes (8 dk), value codes (8 dv), key scales (dk), value
// scales (dv bytes).  Codes are stored as code + 8 in the order in which the attention kernel's
// matrix instructions want them, so that a lane's operands are whole 32-bit words:
//   keys     word (token, t, g): features 32 g + 8 t + e, e < 8; even e in nibbles 0..3, odd e in
//            nibbles 4..7.  (w >> 4 j) & 0x000f000f then is the feature pair e = 2 j, 2 j + 1.
//   values   word (h, c, t, g): features 32 g + 4 c + j, j < 4, of token 8 h + 2 t in nibbles
//            0..3 and of token 8 h + 2 t + 1 in nibbles 4..7.  (w >> 4 j) & 0x000f000f then is
//            the token pair of one feature.
//   scales   [token][group], bf16.
// A token owns whole 16-bit words, so tokens of one block may be written by different threads.
#pragma once
#include <cstdint>

namespace moa {
namespace kv4 {

constexpr int kBlock = 16;   // tokens of a block
constexpr int kGroup = 32;   // features that share a scale
constexpr unsigned kErrIndex = 7u;  // MOA_ERR_DEVICE_INDEX

__host__ __device__ constexpr int block_bytes(int dk, int dv) { return 9 * (dk + dv); }
__host__ __device__ constexpr int value_codes(int dk) { return 8 * dk; }
__host__ __device__ constexpr int key_scales(int dk, int dv) { return 8 * (dk + dv); }
__host__ __device__ constexpr int value_scales(int dk, int dv) { return 8 * (dk + dv) + dk; }

// Byte offsets inside a block.
__device__ __forceinline__ int key_word(int token, int t, int g, int groups) {
  return ((token * 4 + t) * groups + g) * 4;
}
__device__ __forceinline__ int value_word(int dk, int token, int c, int g, int groups) {
  return value_codes(dk) + ((((token >> 3) * 8 + c) * 4 + ((token & 7) >> 1)) * groups + g) * 4;
}

}  // namespace kv4
}  // namespace moa

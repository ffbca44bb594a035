// Rows held in 4 bits (KVC_KV4): what a row stands for and where its bytes are, for the host and
// the device.
//
// A row of D elements (K rotated, or V) is held in groups of 32.  A group x has a scale
// s = max|x| / 7 rounded to 7 significant bits and to a multiple of 2^-20 at the finest, 9344 at
// most, and codes c = rint(x / s) in -7..7; it stands for s * c.  The scale is stored as the
// binary16 number s / 16, the code as the nibble c + 8.  These limits make every product
// (c + 64 + 8) * (s / 16), 72 * (s / 16) and c * (s / 16) a binary16 number, so that one fused
// multiply-add turns a nibble into an exact operand of the tensor cores: (64 + n) * m - 72 * m
// with m = s / 16 and 64 + n the binary16 pattern 0x5400 | n << 4.  (With an 8-bit scale 72 * m
// would need 12 bits; with s itself instead of s / 16 it would pass 65504 from s = 910 on.)
// A group with an infinity or a NaN gets a NaN scale and stands for NaN.
//
// A tile is the 16 rows of one (page, layer, KV head) of K or of V, 9 D bytes: codes, then scales.
//   K: row-major, D / 2 bytes of codes a row; scales [slot][D / 32].  Lane (g, t) of a warp takes 8
//      dims of each group, [32 w + 8 t, 32 w + 8 t + 8) as its word w, of rows g and g + 8: its
//      D / 32 words side by side, one 16-byte (D = 128) or 8-byte (D = 64) load a row.  A step of
//      the product then stays within a group, so that a scale can come in behind it.
//   V: dims in 8 pieces of D / 8; a piece of one row is D / 16 bytes, dim d in nibble d % (D / 8).
//      Lane (g, t) takes piece g of rows 2t, 2t + 1 and of rows 2t + 8, 2t + 9, each pair side by
//      side; scales [D / 32][slot], so that those of a pair are one 4-byte load.
// A page holds [layer][KV head][K, V] tiles: both of a head come with one copy of 18 D bytes.
#pragma once

#include <stddef.h>
#include <stdint.h>

#ifdef __CUDACC__
#define KV4_FN __host__ __device__ inline
#else
#define KV4_FN inline
#endif

namespace kvc {
namespace kv4 {

constexpr int ROWS = 16;    // of a tile: positions of a page
constexpr int GROUP = 32;   // elements that share a scale
constexpr int CODE_MAX = 7;
constexpr float SCALE_MAX = 9344.f;     // 73 * 128: 7 * 9344 / 16 * 16 < 65504
constexpr int SCALE_BITS = 7;           // significant bits of a scale
constexpr int SCALE_FINEST_EXP = -20;   // scales are multiples of 2^-20

KV4_FN size_t tile_bytes(int D) { return (size_t)9 * D; }
KV4_FN size_t page_bytes(int D, int layers, int heads) { return tile_bytes(D) * 2 * heads * layers; }
// Byte offset in the pool of a tile (kv: 0 = K, 1 = V).
KV4_FN size_t tile_at(int D, int layers, int heads, int page, int layer, int head, int kv) {
  return ((((size_t)page * layers + layer) * heads + head) * 2 + kv) * tile_bytes(D);
}

// Byte offsets within a tile; 8 codes are a 32-bit word, dim d in nibble d % 8.
// 8 codes (4 bytes) from dim d (a multiple of 8) of a K row.
KV4_FN int k_codes(int D, int slot, int d) {
  return slot * (D / 2) + (d % GROUP / 8 * (D / GROUP) + d / GROUP) * 4;
}
// Piece p of the 8 (D / 16 bytes each) that make up the codes of a K row.
KV4_FN int k_piece(int D, int slot, int p) { return slot * (D / 2) + p * (D / 16); }
KV4_FN int k_scale(int D, int slot, int group) { return ROWS * D / 2 + (slot * (D / GROUP) + group) * 2; }
// Piece g (dims [g D / 8, (g + 1) D / 8)) of a V row.
KV4_FN int v_piece(int D, int slot, int g) {
  return (slot >> 3) * (D * 4) + (g * 4 + ((slot & 7) >> 1)) * (D / 8) + (slot & 1) * (D / 16);
}
// 8 codes (4 bytes) from dim d (a multiple of 8) of a V row.
KV4_FN int v_codes(int D, int slot, int d) { return v_piece(D, slot, d / (D / 8)) + d % (D / 8) / 2; }
KV4_FN int v_scale(int D, int slot, int group) { return ROWS * D / 2 + (group * ROWS + slot) * 2; }

}  // namespace kv4
}  // namespace kvc

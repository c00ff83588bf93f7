// Rows and matrices in 8-bit floating point, in plain C++ (a host compiler can check it).
#pragma once

#include "kv_cache.h"

namespace moqe {

// A row's codes are e4m3, 128 to a block; a block's scale is a power of two 2^e, e in [-120, 120], stored as the byte 127 + e: what the matrix cores take as an operand's scale.
constexpr int F8_BLOCK = 128;
MOQE_HD int f8_blocks(int d) { return (d + F8_BLOCK - 1) / F8_BLOCK; }

// Packed matrices.  Tiles of 16 rows x 128 columns, row tile major, in the order of a 16x16x128 operand: lane 16 q + r has columns 16 q .. 16 q + 15 (first kilobyte) and
// 64 + 16 q .. (second) of row r, so a wave reads a tile with two coalesced loads of 16 bytes a lane.  (Which columns a lane has is free as long as both operands agree: their 128
// columns have one scale.)  A gated pair has its tiles in turn, gate tile j at 2 j and up tile j at 2 j + 1, so that a lane holds both values of a feature.
// Scales follow: [row tile][group of 4 blocks][row][4], so that a lane gets four blocks' scales of its row in one dword.
struct F8Packed {
  int tiles, blocks, groups;         // row tiles (both matrices of a pair), 128-column blocks, groups of 4 blocks
  size_t scale_off, total;
};
MOQE_HD F8Packed f8_packed(int n, int k, int gated) {
  F8Packed p;
  p.tiles = (n + 15) / 16 * (gated ? 2 : 1);
  p.blocks = f8_blocks(k);
  p.groups = (p.blocks + 3) / 4;
  p.scale_off = size_t(p.tiles) * p.blocks * 2048;
  p.total = p.scale_off + (size_t(p.tiles) * p.groups * 64 + 255) / 256 * 256;
  return p;
}
// Byte of (row of its tile, column of its block) inside a tile.
MOQE_HD uint32_t f8_code_at(uint32_t row, uint32_t col) { return col / 64 * 1024 + (col % 64 / 16 * 16 + row) * 16 + col % 16; }
MOQE_HD size_t f8_scale_at(const F8Packed& p, size_t tile, uint32_t row, uint32_t block) { return p.scale_off + (tile * p.groups + block / 4) * 64 + row * 4 + block % 4; }

}  // namespace moqe

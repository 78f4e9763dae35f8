// Microscaled 4-bit floating point: blocks of 32 values along the contraction, one power-of-two scale a block (a byte: exponent + 127),
// each value e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives).  Layouts, conversions and the launchers of mx.hip and mx_product.hip.
#pragma once
#include "wave.hpp"

namespace bigmac {

constexpr int MX_BLOCK = 32, MX_STEP = 64, MX_CHUNK = 256;   // values: per scale, per matrix instruction, per dword of four scales of a lane

// Rows: codes [rows][cols / 2], value 2i in the low half of byte i; scales [cols / 256, rounded up][rows][8]: of 8 bytes the first four
// belong to the even blocks and the other four to the odd ones, unused bytes 0.  A lane of a matrix instruction holds the even or the odd
// block of a row and reads the scales of four instructions as one dword; the scales that a tile's rows need at a time are whole lines.
// (A row's scales one after another cost a line per row: 16 KB of lines beside the 48 KB of operands of 128 rows x 256 columns.)
inline size_t mx_scale_bytes(long cols) { return (size_t)((cols + MX_CHUNK - 1) / MX_CHUNK) * 8; }
__device__ __forceinline__ size_t mx_scale_at(long rows, long row, unsigned block) { return ((size_t)(block >> 3) * rows + row) * 8 + (block & 1) * 4 + ((block & 7) >> 1); }

// Weights: 32 output columns x 64 inputs are the 1 KB that a wavefront feeds to one matrix instruction, lane l's 16 bytes (column l % 32,
// inputs 32 (l / 32) .. + 31) one after another.  A strip of 32 columns: [n_in / 64][64 lanes][16] codes, behind them its scales,
// [n_in / 256, rounded up][64 lanes][4]: byte j of a lane for its j-th instruction of the 256 inputs.  [groups][n_out / 32] strips.
// (With the scales behind all codes the strips lie a power of two apart where n_in is one, and wavefronts that read the same inputs of
// different strips meet on a few of the L2's channels.)
inline __host__ __device__ size_t mx_strip_bytes(long n_in) { return (size_t)(n_in / MX_STEP) * 1024 + (size_t)((n_in + MX_CHUNK - 1) / MX_CHUNK) * 256; }
inline size_t mx_packed_bytes(long groups, long n_in, long n_out) { return (size_t)groups * (n_out / 32) * mx_strip_bytes(n_in); }

// Scale byte of a block from the largest magnitude's bits: floor(log2) - 2, not under 2^-127; 255 where the block holds an infinity or NaN.
__device__ __forceinline__ unsigned mx_scale_byte(unsigned top_bits) {
  const unsigned e = top_bits >> 23;
  return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
// 2^-(byte - 127), by which the block's values are multiplied (exact); bytes 0 .. 252
__device__ __forceinline__ float mx_inverse(unsigned byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float mx_scale(unsigned byte) {   // 2^(byte - 127), NaN for 255
  return __uint_as_float(byte == 255u ? 0x7FC00000u : byte ? byte << 23 : 0x00400000u);
}
// eight values as codes, nearest, ties to the even code, saturated (the hardware's conversion does all three)
__device__ __forceinline__ unsigned mx_codes8(const float* f, unsigned byte) {
  const float inv = mx_inverse(byte);
  unsigned r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[0] * inv, f[1] * inv, 1.0f, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[2] * inv, f[3] * inv, 1.0f, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[4] * inv, f[5] * inv, 1.0f, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[6] * inv, f[7] * inv, 1.0f, 3);
  return byte == 255u ? 0u : r;
}
typedef float f32x2v_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void mx_values8(unsigned codes, float scale, float* f) {
  f32x2v_t v;
  v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0); f[0] = v.x * scale; f[1] = v.y * scale;
  v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1); f[2] = v.x * scale; f[3] = v.y * scale;
  v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2); f[4] = v.x * scale; f[5] = v.y * scale;
  v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3); f[6] = v.x * scale; f[7] = v.y * scale;
}

constexpr long MX_MAX_BLOCKS = 0xFFFFFF;   // of 256 threads: a launch has under 2^32 threads

enum MxEpilogue { MX_STORE_BF16 = 0, MX_STORE_F32 = 1, MX_GELU_CODES = 2 };
// C = A W[group] (+ bias[group]) over ragged or dense rows
struct MxProduct {
  const uint8_t *codes, *scales;   // A: rows x n_in
  const uint8_t* packed;           // W: [groups] of n_in x n_out
  const bf16_t* bias;              // [groups][n_out] or NULL
  const int* offsets;              // device [groups + 1], or NULL: one group of all rows
  const int* tile_map;             // device, with offsets: from an MxMapJob of mx_tile_rows rows
  void* out;                       // [rows][n_out] bf16 or fp32, or codes
  uint8_t* out_scales;             // MX_GELU_CODES: of the rows of codes
  int rows, groups, n_in, n_out, epilogue;
  int tile_rows;                   // from mx_tile_rows, as the tile map's
};
int mx_tile_rows(int rows, int groups, int n_in, int n_out, int epilogue);   // 32, 64 or 128
int check_mx_product(const MxProduct& p);   // BIGMAC_ERR_TOO_LARGE where its launch would be; before anything is launched
int launch_mx_product(const MxProduct& p, hipStream_t s);
// The row tiles of a ragged product: map[0] = how many, then from map[4] on (group, first row, end of the group's rows, 0) of each, groups in order
struct MxMapJob {
  const int* offsets;              // device [groups + 1]
  int* map;                        // device, mx_map_ints(rows, groups); NULL: no job
  int rows, groups, tile_rows;
};
// upper bound of the row tiles (ascending offsets keep it by themselves, others are cut off at it)
inline __host__ __device__ long mx_most_tiles(long rows, long groups, int tile_rows) { return rows / tile_rows + (groups < rows ? groups : rows); }
inline size_t mx_map_ints(long rows, long groups) { return 4 + 4 * ((size_t)rows / 32 + groups + 1); }   // for every tile height
// maps (optional): one or two tile maps, by workgroups of the same launch
int launch_mx_quantize(long rows, long cols, int dtype, const void* src, uint8_t* codes, uint8_t* scales, hipStream_t s, const MxMapJob* maps = nullptr);

}  // namespace bigmac

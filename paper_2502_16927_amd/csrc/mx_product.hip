// Products of microscaled 4-bit operands on the scaled matrix instructions: C[m, n] = sum_k A[m, k] W[group][k, n], exact products of
// the held values, fp32 sums; rows grouped by expert (ragged) or dense.  v_mfma_scale_f32_32x32x64: lane l holds the 32 values of one
// block (row or column l % 32, block l / 32 of the 64 inputs) and that block's scale, one byte of a dword that serves four instructions.
//
// The results are worked out transposed (the weights are the instruction's first operand), so a lane holds 16 columns of one row:
// a block of 32 hidden columns lies in lanes l and l + 32, which is what the GELU epilogue needs to make 4-bit rows of it.
#include <algorithm>
#include <type_traits>

#include "mx.hpp"
#include "gemm_core.hpp"

namespace bigmac {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t scalar_buffer(size_t at, size_t bytes) {
  const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)at), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(((size_t)hi << 32) | lo), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}
template <int J>
__device__ __forceinline__ f32x16_t mx_mfma(const u32x4_t& w, unsigned ws, const u32x4_t& a, unsigned as, f32x16_t c) {
  const i32x8_t W = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0}, A = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, c, 4, 4, J, (int)ws, J, (int)as);   // 4: e2m1
}
// a value that an LDS read written in assembly delivers: usable behind the wait in front of this call
template <typename T>
__device__ __forceinline__ void hold(T& v) { asm volatile("" : "+v"(v)); }
template <int OFFSET>
__device__ __forceinline__ void lds_read_b32(unsigned addr, unsigned& v) { asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFFSET) : "memory"); }

// GELU for 4-bit results: a polynomial of degree 5 for log2 of the normal tail (minimax of the tail's absolute error, of |a| times it past
// 1: under 7e-7, so within 7e-7 of |a| and of 1).  That is 2^-15 of a block's largest value where this is 2^-5 or more; smaller blocks with an input past 1,
// which may hold the far tail alone (18 % off at -6), take gelu_tail_f (inputs up to 1: 2^-17 of the result).  The polynomial falls without end, so
// |a| needs no limit.  max(a, 0) on the bits as an integer: one instruction.  The vector ALU is what bounds a product with this epilogue: for
// the 131072 x 4096 hidden values of a 16384-token call every instruction per value is 16 us, and a matrix instruction leaves it about half of its time.
__device__ __forceinline__ float gelu_mx_f(float a) {
  const float x = fabsf(a);
  float q = fmaf(x, -5.002595082e-04f, 7.282377832e-03f);
  q = fmaf(x, q, -5.234324002e-02f);
  q = fmaf(x, q, -4.594140765e-01f);
  q = fmaf(x, q, -1.151052049e+00f);
  q = fmaf(x, q, -1.000001856e+00f);
  return fmaf(-x, __builtin_amdgcn_exp2f(q), __int_as_float(max(__float_as_int(a), 0)));
}
// GELU for blocks of small values: e^(a^2 / 2) times the tail as t times a polynomial of degree 7 in t = 1 / (1 + 0.3 |a|) (minimax of the relative
// error, 1.7e-7; with the roundings of a^2 and of the exponential within 1e-5 of the result down to 2^-124).  2^32 keeps the exponential of the
// far tail from being flushed to 0.
constexpr unsigned MX_GELU_SMALL = 0x3D000000u, MX_GELU_NEAR = 0x3F800000u;   // 2^-5 and 1, by their bits
__device__ __forceinline__ float gelu_tail_f(float a) {
  const float x = fabsf(a), t = __builtin_amdgcn_rcpf(fmaf(x, 0.3f, 1.0f));
  float q = fmaf(t, 3.542370350e-02f, -1.561583233e-01f);
  q = fmaf(t, q, 2.045565844e-01f);
  q = fmaf(t, q, -5.203384629e-02f);
  q = fmaf(t, q, 1.276916891e-01f);
  q = fmaf(t, q, 1.001759707e-01f);
  q = fmaf(t, q, 1.207121328e-01f);
  q = fmaf(t, q, 1.196320074e-01f);
  const float e = __builtin_amdgcn_exp2f(fmaf(x * -0.72134752f, x, 32.0f));
  return fmaf(-(q * t * x * e), 0x1p-32f, __int_as_float(max(__float_as_int(a), 0)));
}
// largest magnitude of 16 values, NaN if one is
__device__ __forceinline__ float top_of(const float (&f)[16]) {
  float t = f[0];
#pragma unroll
  for (int v = 0; v < 16; v += 2) asm("v_maximum3_f32 %0, |%1|, |%2|, |%0|" : "+v"(t) : "v"(f[v]), "v"(f[v + 1]));
  return t;
}
// eight values over 2^(byte - 127), byte 1 .. 254: the conversion divides by its scale operand
__device__ __forceinline__ unsigned mx_codes8_scaled(const float* f, unsigned byte) {
  const float scale = __uint_as_float(byte << 23);
  unsigned r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[0], f[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[2], f[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[4], f[5], scale, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[6], f[7], scale, 3);
  return byte == 255u ? 0u : r;
}

// Which tile a workgroup has, and what it needs of it
struct MxTile {
  int group, m0, m_rows, strip0;   // strip0: first 32 columns of the workgroup
  bool valid;
};
// Tiles of BM rows x `parts` parts of the columns.  Consecutive workgroups go to the 8 XCDs in turn: each XCD gets a run of consecutive tiles,
// column parts fastest.  strip0: which part.
template <int BM>
__device__ __forceinline__ MxTile mx_part(const MxProduct& p, int parts) {
  MxTile t;
  const int tiles = p.offsets ? table_at(p.tile_map, 0) : (p.rows + BM - 1) / BM;
  const unsigned total = (unsigned)tiles * (unsigned)parts, per_xcd = (total + 7) / 8, slot = blockIdx.x >> 3, id = (blockIdx.x & 7) * per_xcd + slot;
  t.valid = slot < per_xcd && id < total;
  if (!t.valid) return t;
  const int tile = (int)(id / (unsigned)parts);
  t.strip0 = (int)(id % (unsigned)parts);
  int m_end = p.rows;
  t.group = 0;
  t.m0 = tile * BM;
  if (p.offsets) {
    t.group = table_at(p.tile_map, 4 + 4 * tile);
    t.m0 = table_at(p.tile_map, 5 + 4 * tile);
    m_end = table_at(p.tile_map, 6 + 4 * tile);
    t.valid = t.m0 >= 0 && t.m0 < m_end;   // (offsets out of order or past the rows: nothing outside the buffers is touched)
  }
  t.m_rows = min(m_end - t.m0, BM);
  return t;
}
// ... the parts STRIPS x 32 columns each; strip0: the first 32 columns
template <int BM, int STRIPS>
__device__ __forceinline__ MxTile mx_tile(const MxProduct& p) {
  MxTile t = mx_part<BM>(p, (p.n_out / 32 + STRIPS - 1) / STRIPS);
  t.strip0 *= STRIPS;
  return t;
}

// A row of 128 bytes in the LDS as eight pieces of 16, in places that put 16 consecutive rows' equal pieces on all banks
__device__ __forceinline__ unsigned piece_place(unsigned row, unsigned piece) { return row * 128u + (piece ^ ((row >> 1) & 7u)) * 16u; }

// Results leave as whole lines.  A sub-tile of 32 x 32 lies in the lanes as: row l % 32, columns 8 q + 4 (l / 32) + 0 .. 3 in values 4 q .. 4 q + 3.
// bf16 and fp32: through 4 KB of the wavefront's own, 32 rows x 128 bytes.  (Stored from where they lie, 32 bytes of a row at a time, they
// were four requests a line; the 8 and 1 bytes of the 4-bit epilogue 16 and 8.)
template <int PIECES = 8>   // of 16 bytes: a line, or half of one
__device__ __forceinline__ void strip_out(char* strip, const MxProduct& p, int row0, int rows, size_t col_byte, size_t row_bytes, int lane) {
#pragma unroll
  for (int i = 0; i < PIECES / 2; ++i) {
    const unsigned q = i * 64 + lane, row = q / PIECES, piece = q % PIECES;
    const uint4 v = *(const uint4*)(strip + piece_place(row, piece));
    if ((int)row < rows) *(uint4*)((char*)p.out + (size_t)(row0 + (int)row) * row_bytes + col_byte + piece * 16) = v;
  }
}
template <int NS>
__device__ __forceinline__ void mx_store(const MxProduct& p, const f32x16_t (&acc)[NS], const float (&bias)[NS][16], int row0, int rows, int col0, char* strip, int lane,
                                         std::integral_constant<int, MX_STORE_BF16>) {
  const int half = lane >> 5;
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      float f[8];
#pragma unroll
      for (int v = 0; v < 8; ++v) f[v] = acc[j][8 * s + v] + bias[j][8 * s + v];
      // quads 2 s and 2 s + 1: the lower lane takes all eight columns of the first, the upper one of the second
      const auto r0 = __builtin_amdgcn_permlane32_swap(f2bf_pair(f[0], f[1]), f2bf_pair(f[4], f[5]), false, false);
      const auto r1 = __builtin_amdgcn_permlane32_swap(f2bf_pair(f[2], f[3]), f2bf_pair(f[6], f[7]), false, false);
      *(uint4*)(strip + piece_place(lane & 31, j * 4 + s * 2 + half)) = make_uint4(r0[0], r1[0], r0[1], r1[1]);
    }
  strip_out<4 * NS>(strip, p, row0, rows, (size_t)col0 * 2, (size_t)p.n_out * 2, lane);
}
template <int NS>
__device__ __forceinline__ void mx_store(const MxProduct& p, const f32x16_t (&acc)[NS], const float (&bias)[NS][16], int row0, int rows, int col0, char* strip, int lane,
                                         std::integral_constant<int, MX_STORE_F32>) {
#pragma unroll
  for (int j = 0; j < NS; ++j) {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *(float4*)(strip + piece_place(lane & 31, 2 * q + (lane >> 5))) = make_float4(acc[j][4 * q] + bias[j][4 * q], acc[j][4 * q + 1] + bias[j][4 * q + 1],
                                                                                    acc[j][4 * q + 2] + bias[j][4 * q + 2], acc[j][4 * q + 3] + bias[j][4 * q + 3]);
    strip_out(strip, p, row0, rows, (size_t)(col0 + 32 * j) * 4, (size_t)p.n_out * 4, lane);
  }
}
// GELU and 4 bits of 32 rows x 64 columns: a block of a row per lane, the first 32 columns in the lower lanes; bytes: both blocks' scales.
// TAIL false: every block by gelu_mx_f; small: whether a block of this lane's may need the other form (its row, `live`, is one of the tile's: the
// others' values count for nothing).  TAIL true: the blocks that need it by gelu_tail_f.  Which form a block has depends on its own values only.
template <int NS, bool TAIL>
__device__ __forceinline__ uint4 mx_gelu_blocks(const f32x16_t (&acc)[NS], const float (&bias)[NS][16], bool biased, bool live, bool& small, unsigned (&bytes)[NS]) {
  static_assert(NS == 2, "a lane for each block");
  uint2 half_block[NS];   // lower lane: columns 0 .. 15 of a block, upper lane: 16 .. 31
  unsigned least = ~0u;
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    float f[16];
    auto inputs = [&]() {
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] = acc[j][v];
      if (biased)
#pragma unroll
        for (int v = 0; v < 16; ++v) f[v] += bias[j][v];
    };
    auto block_top = [&]() {   // bits of the largest magnitude (a NaN is the largest, with its sign or without)
      const unsigned mine = __float_as_uint(top_of(f));
      const auto both = __builtin_amdgcn_permlane32_swap(mine, mine, false, false);
      return max(both[0], both[1]) & 0x7FFFFFFFu;
    };
    inputs();
    const unsigned top_input = TAIL ? block_top() : 0u;   // (of sums that an addition has read: assembly reads no matrix instruction's result)
#pragma unroll
    for (int v = 0; v < 16; ++v) f[v] = gelu_mx_f(f[v]);
    unsigned top = block_top();
    if constexpr (TAIL) {
      if (top < MX_GELU_SMALL && top_input > MX_GELU_NEAR) {   // (both lanes of a block or none)
        inputs();
#pragma unroll
        for (int v = 0; v < 16; ++v) f[v] = gelu_tail_f(f[v]);
        top = block_top();
      }
    }
    least = min(least, top);
    // the smallest scale here is 2^-126: values of a block under 2^-124 that 2^-127 would hold better
    bytes[j] = max(mx_scale_byte(top), 1u);
    // halfword q: this lane's four columns of quad q; lower lane: the lower and the upper lane's of quads 0 and 1, upper lane: of quads 2 and 3
    const auto r = __builtin_amdgcn_permlane32_swap(mx_codes8_scaled(f, bytes[j]), mx_codes8_scaled(f + 8, bytes[j]), false, false);
    half_block[j] = make_uint2((r[0] & 0xFFFFu) | (r[1] << 16), (r[0] >> 16) | (r[1] & 0xFFFF0000u));
  }
  if constexpr (!TAIL) small |= live && least < MX_GELU_SMALL;
  const auto x = __builtin_amdgcn_permlane32_swap(half_block[0].x, half_block[1].x, false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(half_block[0].y, half_block[1].y, false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}
// GELU and 4 bits of MT x 32 rows x 64 columns, `put` stores a sub-tile's blocks.  First every block by the short form; then, in wavefronts with a
// small block that has an input past 1, all over again with the other form where it is needed.  (Decided block by block on the way the branches
// between the blocks cost 14 us of a 16384-token call; so it is 4.)
template <int MT, int NS, typename Put>
__device__ __forceinline__ void mx_gelu_tile(f32x16_t (&acc)[MT][NS], const float (&bias)[NS][16], bool biased, int rows, int lane, Put&& put) {
  bool small = false;
  unsigned bytes[NS];
#pragma unroll
  for (int i = 0; i < MT; ++i)
    if (i * 32 < rows) {
      const uint4 block = mx_gelu_blocks<NS, false>(acc[i], bias, biased, i * 32 + (lane & 31) < rows, small, bytes);
      put(i, block, bytes);
    }
  if (__builtin_expect(__any(small), 0)) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NS; ++j) hold(acc[i][j]);   // (or the compiler keeps every value of the first pass, out of registers)
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NS; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) top = fmaxf(top, fabsf(acc[i][j][v] + bias[j][v]));
    if (__any(top > 1.0f)) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
        if (i * 32 < rows) {
          const uint4 block = mx_gelu_blocks<NS, true>(acc[i], bias, true, true, small, bytes);   // (without biases: zeros)
          put(i, block, bytes);
        }
    }
  }
}
// biases of the columns a lane holds of the 32 NS from `strip` on (bias NULL: zeros)
template <int NS>
__device__ __forceinline__ void mx_bias(const MxProduct& p, const MxTile& t, int strip, float (&bias)[NS][16], int lane) {
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[j][v] = 0.0f;
  if (!p.bias) return;
#pragma unroll
  for (int j = 0; j < NS; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const uint2 b = *(const uint2*)(p.bias + (size_t)t.group * p.n_out + (strip + j) * 32 + 8 * q + 4 * (lane >> 5));
      bias[j][4 * q] = __uint_as_float(b.x << 16); bias[j][4 * q + 1] = __uint_as_float(b.x & 0xFFFF0000u);
      bias[j][4 * q + 2] = __uint_as_float(b.y << 16); bias[j][4 * q + 3] = __uint_as_float(b.y & 0xFFFF0000u);
    }
}

// MT x 32 rows, 4 wavefronts side by side with NS x 32 columns each (NS 1: 64 rows without the GELU epilogue).
//
// Weights go from memory to registers as they lie there (1 KB per instruction operand, whole lines), each wavefront its own columns'.
// Rows go straight to the LDS in chunks of 256 inputs, three stages: while chunk c is multiplied, chunk c + 1 has landed or is about
// to and chunk c + 2 is requested.  A chunk's step: the MT NS instructions of 64 inputs, between them the LDS reads of the next
// step's fragments, behind them the next chunk's weights of the same step, into the registers that have just been read.
//
// At 131072 rows, 1024 -> 4096 with GELU and 4096 -> 1024 without, it takes 402 to 423 and 277 to 284 us in a call of the FFN (2.7 and 3.9 PFLOP/s).  What
// bounds it, measured before the scales of 256 columns lay together, each product over and over (389 and 304 us, matrix cores busy 31 and 39 % at 2.2 GHz):
// without the epilogues 259 and 270 us (53 % at 1.9 GHz), without the loop's requests too 190 (78 % at 1.8 GHz), without its LDS reads too 160: power holds the
// clock down, and the requests cost as much as the epilogue.  Two workgroups share a CU.
// Slower or level: one persistent workgroup walking many tiles with its operands requested a tile ahead (917 us a 16384-token call against 873),
// 256 x 256 tiles by eight wavefronts (960 against 819), 64-row tiles (885 against 797), 32 columns a wavefront (888 against 874), weights two
// chunks ahead (807 against 796), the rows of a tile kept in the LDS for all columns (803 against 799); for 32-row tiles weights two chunks ahead
// and eight wavefronts with half of the inputs each (+0.2 and +0.6 us at 512 -> 1024 to 4096 -> 4096: their CU is bound by what it takes in).
constexpr int MX_STAGES = 3;
// the scales of a tile's rows for the 256 inputs of a chunk
__device__ __forceinline__ __amdgpu_buffer_rsrc_t chunk_scales(const MxProduct& p, const MxTile& t, int chunk) {
  return scalar_buffer((size_t)p.scales + ((size_t)chunk * p.rows + t.m0) * 8, (size_t)t.m_rows * 8);
}
constexpr unsigned mx_stage_bytes(int mt) { return mt * 4096 + 1024; }   // codes; 256 dwords of scales (past the tile's rows: zeros)
template <int MT, int NS, int EPI>
__device__ __forceinline__ void mx_tile_product(const MxProduct& p, const MxTile& t, uint4* ring, uint4* staging, uint8_t* out_scales) {
  constexpr int STAGES = MX_STAGES;
  constexpr unsigned CODES = MT * 4096, STAGE = mx_stage_bytes(MT);
  const unsigned ring_at = lds_address(ring);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int strips = p.n_out / 32, strip0 = t.strip0 + wave * NS;
  const int steps = p.n_in / MX_STEP, chunks = (steps + 3) / 4;
  const unsigned row_bytes = (unsigned)p.n_in / 2;
  const auto ba = scalar_buffer((size_t)p.codes + (size_t)t.m0 * row_bytes, (size_t)t.m_rows * row_bytes);
  const unsigned strip_bytes = (unsigned)mx_strip_bytes(p.n_in), scales_at = (unsigned)steps * 1024u;   // of a strip of the weights
  __amdgpu_buffer_rsrc_t bw[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const bool there = strip0 + j < strips;   // past the last column: empty ranges, zeros
    const size_t strip = (size_t)t.group * strips + (there ? strip0 + j : 0);
    bw[j] = scalar_buffer((size_t)p.packed + strip * strip_bytes, there ? strip_bytes : 0);
  }

  // LDS place q (16 bytes) of a stage: row q / 8, piece (q % 8) ^ (row / 2 % 8) of it: 16 consecutive rows at one piece lie on all banks
  constexpr int DMA = MT;                   // 16-byte requests of a lane per chunk, 32 rows each
  const unsigned swizzle = (threadIdx.x >> 4) & 7;
  const unsigned a_off = (threadIdx.x >> 3) * row_bytes + ((threadIdx.x & 7) ^ swizzle) * 16u, a_pass = 32u * row_bytes;
  // Past the last chunk: out of range, zeros that nobody reads.  (Requested all the same: with a branch in the loop the compiler moves
  // the matrix instructions in front of it, which it takes for arithmetic like any other, behind it, and keeps their operands.)
  auto request = [&](int chunk, unsigned stage) {
    const unsigned at = chunk < chunks ? 0u : 0x80000000u;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int i = 0; i < DMA; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(ba, (__attribute__((address_space(3))) void*)(ring + stage / 16 + i * 256 + wave * 64), 16,
                                               (a_off + i * a_pass + (unsigned)chunk * 128u) | at, 0, 0, 0);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(chunk_scales(p, t, chunk), (__attribute__((address_space(3))) void*)(ring + stage / 16 + CODES / 16 + wave * 16), 4,
                                             (threadIdx.x * 4u) | at, 0, 0, 0);
#endif
    asm volatile("" ::: "memory");
  };
  u32x4_t w[NS][4], fa[2][MT];
  unsigned ws[NS], as[MT], ws_next[NS], as_next[MT];
  const unsigned w_off = (unsigned)lane * 16u, ws_off = (unsigned)lane * 4u;
  auto load_w = [&](int chunk, auto ks) {
    constexpr int J = decltype(ks)::value;
#pragma unroll
    for (int j = 0; j < NS; ++j) w[j][J] = __builtin_amdgcn_raw_buffer_load_b128(bw[j], chunk * 4 + J < steps ? (unsigned)(chunk * 4 + J) * 1024u + w_off : 0x80000000u, 0, 0);
  };
  auto load_ws = [&](int chunk) {
#pragma unroll
    for (int j = 0; j < NS; ++j) ws_next[j] = __builtin_amdgcn_raw_buffer_load_b32(bw[j], scales_at + (unsigned)chunk * 256u + ws_off, 0, 0);
  };
  const unsigned fa_at = ring_at + (unsigned)(lane & 31) * 128u + (((unsigned)lane >> 5) ^ (((unsigned)lane >> 1) & 7)) * 16u;
  const unsigned as_at = ring_at + CODES + (unsigned)(lane & 31) * 8u + ((unsigned)lane >> 5) * 4u;
  auto read_a = [&](auto n, auto ks, unsigned stage) {   // fragment n of step ks
    constexpr int i = decltype(n)::value, J = decltype(ks)::value;
    lds_read_b128<i * 4096>((fa_at ^ (J * 32)) + stage, fa[J & 1][i]);
  };
  auto read_scales = [&](unsigned stage) {
    static_for<0, MT>([&](auto n) { lds_read_b32<decltype(n)::value * 256>(as_at + stage, as_next[decltype(n)::value]); });
  };
  f32x16_t acc[MT][NS];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NS; ++j) acc[i][j] = f32x16_t{0};
  auto multiply = [&](auto n, auto ks) {
    constexpr int i = decltype(n)::value / NS, j = decltype(n)::value % NS, J = decltype(ks)::value;
    acc[i][j] = mx_mfma<J>(w[j][J], ws[j], fa[J & 1][i], as[i], acc[i][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  // The fragments of a step.  A chunk's first ones and its scales are waited for at the end of the chunk in front of it: registers that an LDS
  // read still under way will write must not be there where the loop closes, because the compiler, which knows nothing of the read,
  // copies values between registers there.
  auto arrived = [&](auto ks) {
    constexpr int J = decltype(ks)::value;
    if constexpr (J == 0) {
#pragma unroll
      for (int i = 0; i < MT; ++i) as[i] = as_next[i];
#pragma unroll
      for (int j = 0; j < NS; ++j) ws[j] = ws_next[j];
    } else {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < MT; ++i) hold(fa[J & 1][i]);
    }
  };
  auto first_arrived = [&]() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      hold(fa[0][i]);
      hold(as_next[i]);
    }
  };
  // one step of 64 inputs; meanwhile the next step's fragments are read, behind step 3 the next chunk's first
  auto step = [&](auto ks, unsigned stage, unsigned next_stage, int chunk) {
    constexpr int J = decltype(ks)::value;
    arrived(ks);
    if constexpr (J == 3) {
      // The next chunk's rows have landed: behind its requests came this chunk's weights (5 NS), all but the last of which have been
      // used, the requests of the chunk after it (DMA + 1) and so far 4 NS of the next chunk's weights.  And everyone has read
      // the fragments of this chunk, whose stage takes the requests of the next turn.
      BIGMAC_WAIT_VMCNT(DMA + 1 + 4 * NS);
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      read_scales(next_stage);
    }
    static_for<0, MT * NS>([&](auto n) {
      multiply(n, ks);
      if constexpr (decltype(n)::value < MT) {
        if constexpr (J < 3) read_a(n, std::integral_constant<int, J + 1>{}, stage);
        else read_a(n, std::integral_constant<int, 0>{}, next_stage);
      }
    });
    load_w(chunk + 1, ks);
    if constexpr (J == 0) load_ws(chunk + 1);
    asm volatile("" ::: "memory");
    if constexpr (J == 3) first_arrived();
  };
  constexpr std::integral_constant<int, 0> I0{};
  constexpr std::integral_constant<int, 1> I1{};
  constexpr std::integral_constant<int, 2> I2{};
  constexpr std::integral_constant<int, 3> I3{};
  request(0, 0);
  request(1, STAGE);
  load_ws(0);
  load_w(0, I0);
  load_w(0, I1);
  load_w(0, I2);
  load_w(0, I3);
  asm volatile("" ::: "memory");
  BIGMAC_WAIT_VMCNT(DMA + 1 + 5 * NS);   // chunk 0 (younger: chunk 1's requests, the weights)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_scales(0);
  static_for<0, MT>([&](auto n) { read_a(n, I0, 0); });
  first_arrived();
  const int whole = steps / 4;              // chunks of four steps
  unsigned stage = 0;
#pragma clang loop unroll(disable)
  for (int c = 0; c < whole; ++c) {
    const unsigned next = stage + STAGE == STAGES * STAGE ? 0 : stage + STAGE, after = next + STAGE == STAGES * STAGE ? 0 : next + STAGE;
    request(c + 2, after);
    step(I0, stage, next, c);
    step(I1, stage, next, c);
    step(I2, stage, next, c);
    step(I3, stage, next, c);
    stage = next;
  }
  // one to three steps more; the fragments of the first are there (of a chunk that is not: zeros or old ones, not used)
  const int left = steps - whole * 4;
  arrived(I0);
  if (left > 0) {
    static_for<0, MT * NS>([&](auto n) { multiply(n, I0); });
    auto one = [&](auto ks) {
      static_for<0, MT>([&](auto n) { read_a(n, ks, stage); });
      arrived(ks);
      static_for<0, MT * NS>([&](auto n) { multiply(n, ks); });
    };
    if (left > 1) one(I1);
    if (left > 2) one(I2);
  }

  BIGMAC_WAIT_VMCNT(0);                     // what is on its way to the LDS past the last chunk (zeros) arrives before the workgroup may end
  const bool there = strip0 < strips;       // (strips are whole pairs)
  float bias[NS][16];
  mx_bias<NS>(p, t, there ? strip0 : t.strip0, bias, lane);
  if constexpr (EPI == MX_GELU_CODES) {
    if (there)
      mx_gelu_tile<MT, NS>(acc, bias, p.bias != nullptr, t.m_rows, lane, [&](int i, const uint4& block, const unsigned (&bytes)[NS]) {
        *(uint4*)((char*)staging + piece_place(i * 32 + (lane & 31), wave * 2 + (lane >> 5))) = block;
        out_scales[(i * 32 + (lane & 31)) * 8 + (lane >> 5) * 4 + wave] = (uint8_t)(lane < 32 ? bytes[0] : bytes[1]);   // blocks 2 wave and 2 wave + 1: see mx.hpp
      });
    __syncthreads();
    const size_t row_out = (size_t)p.n_out / 2;
    const int pieces = min(8, strips - t.strip0);   // of the workgroup's 256 columns, 32 each
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const unsigned q = i * 256 + threadIdx.x, row = q >> 3, piece = q & 7;
      const uint4 v = *(const uint4*)((const char*)staging + piece_place(row, piece));
      if ((int)row < t.m_rows && (int)piece < pieces) *(uint4*)((uint8_t*)p.out + (size_t)(t.m0 + (int)row) * row_out + (size_t)t.strip0 * 16 + piece * 16) = v;
    }
    // (bytes of blocks past the last column are whatever the LDS held: nobody reads them)
    if ((int)threadIdx.x < t.m_rows)
      *(uint2*)(p.out_scales + mx_scale_at(p.rows, t.m0 + (int)threadIdx.x, t.strip0)) = *(const uint2*)(out_scales + threadIdx.x * 8);
  } else {
    if (!there) return;
#pragma unroll
    for (int i = 0; i < MT; ++i)
      if (i * 32 < t.m_rows)
        mx_store<NS>(p, acc[i], bias, t.m0 + i * 32, t.m_rows - i * 32, strip0 * 32, (char*)staging + wave * 4096, lane, std::integral_constant<int, EPI>{});
  }
}

template <int MT, int NS, int EPI>
__global__ __launch_bounds__(256, MT == 4 ? 2 : MT == 2 ? 3 : 4) void mx_product_kernel(MxProduct p) {
  constexpr int BM = MT * 32;
  __shared__ uint4 ring[MX_STAGES * mx_stage_bytes(MT) / 16];
  __shared__ uint4 staging[(EPI == MX_GELU_CODES ? BM * 128 : 4 * 4096) / 16];
  __shared__ __align__(16) uint8_t out_scales[EPI == MX_GELU_CODES ? BM * 8 : 8];
  const MxTile t = mx_tile<BM, 4 * NS>(p);
  if (!t.valid) return;
  if constexpr (MT > 1) {   // the last rows of a group
    if (t.m_rows <= 32) return mx_tile_product<1, NS, EPI>(p, t, ring, staging, out_scales);
  }
  if constexpr (MT == 4) {
    if (t.m_rows <= 64) return mx_tile_product<2, NS, EPI>(p, t, ring, staging, out_scales);
    if (t.m_rows <= 96) return mx_tile_product<3, NS, EPI>(p, t, ring, staging, out_scales);
  }
  mx_tile_product<MT, NS, EPI>(p, t, ring, staging, out_scales);
}

// Few tiles, long rows: 32 rows x 64 columns per workgroup, its four wavefronts each a quarter of the inputs, their sums joined in the
// LDS in the wavefronts' order.  With 64 columns a row tile's operands are re-read four times as often as with 256, but nothing waits for a
// serial walk over all inputs.  Both operands go straight to registers, a chunk ahead; no barrier before the join.
template <int EPI>
__global__ __launch_bounds__(256, 2) void mx_split_kernel(MxProduct p) {
  constexpr int NS = 2;
  __shared__ float join[3][NS * 16][64];
  __shared__ uint4 staging[4096 / 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const MxTile t = mx_tile<32, NS>(p);
  if (!t.valid) return;
  const int strips = p.n_out / 32, steps = p.n_in / MX_STEP, chunks = (steps + 3) / 4;
  const unsigned row_bytes = (unsigned)p.n_in / 2;
  const auto ba = scalar_buffer((size_t)p.codes + (size_t)t.m0 * row_bytes, (size_t)t.m_rows * row_bytes);
  const unsigned strip_bytes = (unsigned)mx_strip_bytes(p.n_in), scales_at = (unsigned)steps * 1024u;   // of a strip of the weights
  __amdgpu_buffer_rsrc_t bw[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) bw[j] = scalar_buffer((size_t)p.packed + ((size_t)t.group * strips + t.strip0 + j) * strip_bytes, strip_bytes);
  const unsigned a_off = (unsigned)(lane & 31) * row_bytes + ((unsigned)lane >> 5) * 16u, s_off = (unsigned)(lane & 31) * 8u + ((unsigned)lane >> 5) * 4u;
  struct Chunk {
    u32x4_t w[NS][4], a[4];
    unsigned ws[NS], as;
  };
  // (past the last input: weights out of range, zeros; the rows' codes are another row's, their scales are cut off below)
  auto load = [&](Chunk& c, int chunk) {
#pragma unroll
    for (int j = 0; j < NS; ++j) {
      c.ws[j] = __builtin_amdgcn_raw_buffer_load_b32(bw[j], scales_at + (unsigned)chunk * 256u + lane * 4u, 0, 0);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
        c.w[j][ks] = __builtin_amdgcn_raw_buffer_load_b128(bw[j], chunk * 4 + ks < steps ? (unsigned)(chunk * 4 + ks) * 1024u + lane * 16u : 0x80000000u, 0, 0);
    }
    c.as = __builtin_amdgcn_raw_buffer_load_b32(chunk_scales(p, t, chunk), s_off, 0, 0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) c.a[ks] = __builtin_amdgcn_raw_buffer_load_b128(ba, a_off + (unsigned)chunk * 128u + ks * 32u, 0, 0);
  };
  f32x16_t accs[1][NS], (&acc)[NS] = accs[0];
#pragma unroll
  for (int j = 0; j < NS; ++j) acc[j] = f32x16_t{0};
  const unsigned last_mask = steps & 3 ? (1u << (8 * (steps & 3))) - 1u : ~0u;   // (a scale byte of 255 there would make NaN of the weights' zeros)
  auto multiply = [&](const Chunk& c, int chunk) {
    const unsigned as = chunk + 1 == chunks ? c.as & last_mask : c.as;
    static_for<0, NS>([&](auto n) {
      constexpr int j = decltype(n)::value;
      static_for<0, 4>([&](auto ks) { acc[j] = mx_mfma<decltype(ks)::value>(c.w[j][decltype(ks)::value], c.ws[j], c.a[decltype(ks)::value], as, acc[j]); });
    });
  };
  const int first = chunks * wave / 4, last = chunks * (wave + 1) / 4;            // this wavefront's chunks
  Chunk one, two;
  if (first < last) {
    load(one, first);
    int c = first;
    for (; c + 1 < last; c += 2) {
      load(two, c + 1);
      multiply(one, c);
      load(one, min(c + 2, last - 1));
      multiply(two, c + 1);
    }
    if (c < last) multiply(one, c);
  }
  if (wave > 0)
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) join[wave - 1][j * 16 + v][lane] = acc[j][v];
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[j][v] += join[w][j * 16 + v][lane];
  float bias[NS][16];
  mx_bias<NS>(p, t, t.strip0, bias, lane);
  if constexpr (EPI == MX_GELU_CODES) {
    mx_gelu_tile<1, NS>(accs, bias, p.bias != nullptr, t.m_rows, lane, [&](int, const uint4& block, const unsigned (&bytes)[NS]) {
      const int row = lane & 31, strip = t.strip0 + (lane >> 5);
      if (row < t.m_rows) {
        *(uint4*)((uint8_t*)p.out + (size_t)(t.m0 + row) * (p.n_out / 2) + (size_t)strip * 16) = block;
        p.out_scales[mx_scale_at(p.rows, t.m0 + row, strip)] = (uint8_t)(lane < 32 ? bytes[0] : bytes[1]);
      }
    });
  } else {
    mx_store<NS>(p, acc, bias, t.m0, t.m_rows, t.strip0 * 32, (char*)staging, lane, std::integral_constant<int, EPI>{});
  }
}

long most_tiles(const MxProduct& p, int tile_rows) {
  return p.offsets ? mx_most_tiles(p.rows, p.groups, tile_rows) : ((long)p.rows + tile_rows - 1) / tile_rows;
}
// A quarter of the inputs per wavefront, for few tiles and a long walk: us without and with at 4096 inputs, 1024 columns: 1 row 8.4, 6.1;
// 500 (64 tiles of 256 columns) 10.0, 8.3; 8 groups of 32 (32) 12.8, 10.9; 16 of 16 (64) 13.2, 12.3; 8 of 125 (128) 13.1, 15.6; at 1024 inputs within 0.4.
long even_tiles(long rows, long groups, int tile_rows) {   // rows spread evenly over the groups
  const long busy = std::min(rows, groups), each = (rows + busy - 1) / busy;
  return busy * ((each + tile_rows - 1) / tile_rows);
}
bool worth_splitting(long rows, long groups, int n_in, int n_out) { return n_in >= 2048 && even_tiles(rows, groups, 32) * ((n_out + 255) / 256) <= 64; }
bool splits(const MxProduct& p) { return p.tile_rows == 32 && worth_splitting(p.rows, p.groups, p.n_in, p.n_out); }
long product_blocks(const MxProduct& p) {
  const int columns = splits(p) ? 64 : p.tile_rows == 64 && p.epilogue != MX_GELU_CODES ? 128 : 256;
  return (most_tiles(p, p.tile_rows) * ((p.n_out + columns - 1) / columns) + 7) / 8 * 8;
}
template <int MT>
void launch_of(const MxProduct& p, dim3 grid, hipStream_t s) {
  if (p.epilogue == MX_GELU_CODES) mx_product_kernel<MT, 2, MX_GELU_CODES><<<grid, 256, 0, s>>>(p);
  else if (p.epilogue == MX_STORE_F32) mx_product_kernel<MT, 2, MX_STORE_F32><<<grid, 256, 0, s>>>(p);
  else mx_product_kernel<MT, 2, MX_STORE_BF16><<<grid, 256, 0, s>>>(p);
}
void launch_64(const MxProduct& p, dim3 grid, hipStream_t s) {
  if (p.epilogue == MX_GELU_CODES) mx_product_kernel<2, 2, MX_GELU_CODES><<<grid, 256, 0, s>>>(p);
  else if (p.epilogue == MX_STORE_F32) mx_product_kernel<2, 1, MX_STORE_F32><<<grid, 256, 0, s>>>(p);
  else mx_product_kernel<2, 1, MX_STORE_BF16><<<grid, 256, 0, s>>>(p);
}
void launch_split(const MxProduct& p, dim3 grid, hipStream_t s) {
  if (p.epilogue == MX_GELU_CODES) mx_split_kernel<MX_GELU_CODES><<<grid, 256, 0, s>>>(p);
  else if (p.epilogue == MX_STORE_F32) mx_split_kernel<MX_STORE_F32><<<grid, 256, 0, s>>>(p);
  else mx_split_kernel<MX_STORE_BF16><<<grid, 256, 0, s>>>(p);
}

}  // namespace

// Rows per tile, from rows spread evenly over the groups.  What a CU takes in per 256 inputs: 48 KB for 128 rows x 256 columns, 24 KB for 64 x 128,
// 36 KB for 32 x 256, at 64 bytes a clock.  us on both sides, two operands' sizes and rows each:
// up to 32 rows a group: 32 (64 groups of 4, 1024 -> 4096 -> 1024: 59.1 with 128, 58.3 with 32; 256 groups of 2, 512 -> 1024 -> 512: 34.3, 32.7);
// 128 from three quarters of the CUs on (4096 -> 1024: 4096 rows, 128 tiles: 16.3 with 128, 13.8 with 64; 8192, 256 tiles: 21.5, 22.5), but not for a
// second round of few tiles unless the inputs are long (1024 -> 1024, 9216 rows, 288 tiles: 12.5, 11.9; 12288, 384: 12.6, 13.5; 4096 -> 1024,
// 288: 28.2, 29.5); else 64 (2048 rows 4096 -> 1024: 10.8 with 32, 10.0 with 64; 200 rows 1024 -> 4096: 5.6, 4.4), where the inputs are not
// split (500 rows 4096 -> 1024: 9.0 with 64, 7.5), and with the GELU epilogue, whose tiles keep 256 columns, only where there are enough
// of them (FFN 256 -> 1024 -> 256, 8 groups of 125: 13.0 with 64, 12.0 with 32; 1536 -> 6144 -> 1536, 8 of 125: 32.3 with 32, 29.9 with 64).
int mx_tile_rows(int rows, int groups, int n_in, int n_out, int epilogue) {
  const long parts = (n_out + 255) / 256, tiles = even_tiles(rows, groups, 128) * parts;
  if ((rows + groups - 1) / groups <= 32) return 32;
  if (tiles >= 192 && (n_in >= 2048 || tiles <= 256 || tiles >= 384)) return 128;
  if (worth_splitting(rows, groups, n_in, n_out)) return 32;
  return epilogue == MX_GELU_CODES && even_tiles(rows, groups, 64) * parts < 256 ? 32 : 64;
}

int check_mx_product(const MxProduct& p) { return product_blocks(p) > MX_MAX_BLOCKS ? BIGMAC_ERR_TOO_LARGE : BIGMAC_OK; }

int launch_mx_product(const MxProduct& p, hipStream_t s) {
  const dim3 grid((unsigned)product_blocks(p));
  if (splits(p)) launch_split(p, grid, s);
  else if (p.tile_rows == 128) launch_of<4>(p, grid, s);
  else if (p.tile_rows == 64) launch_64(p, grid, s);
  else launch_of<1>(p, grid, s);
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

}  // namespace bigmac

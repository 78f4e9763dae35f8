// Products of microscaled 4-bit operands on the scaled matrix instructions: C[m, n] = sum_k A[m, k] W[group][k, n], exact products of
// the held values, fp32 sums; rows grouped by expert (ragged) or dense.  v_mfma_scale_f32_32x32x64: lane l holds the 32 values of one
// block (row or column l % 32, block l / 32 of the 64 inputs) and that block's scale, one byte of a dword that serves four instructions.
//
// The results are worked out transposed (the weights are the instruction's first operand), so a lane holds 16 columns of one row:
// a block of 32 hidden columns lies in lanes l and l + 32, which is what the GELU epilogue needs to make 4-bit rows of it.
#include <type_traits>

#include "mx.hpp"
#include "tile_map.hpp"

namespace bigmac {

namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef const int __attribute__((address_space(4))) * table_ptr_t;
__device__ __forceinline__ int table_at(const int* table, int i) { return ((table_ptr_t)(unsigned long long)table)[i]; }

typedef unsigned int q4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t scalar_buffer(size_t at, size_t bytes) {
  const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)at), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(((size_t)hi << 32) | lo), 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}
template <int J>
__device__ __forceinline__ f32x16_t mx_mfma(const q4_t& w, unsigned ws, const q4_t& a, unsigned as, f32x16_t c) {
  const i32x8_t W = {(int)w.x, (int)w.y, (int)w.z, (int)w.w, 0, 0, 0, 0}, A = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(W, A, c, 4, 4, J, (int)ws, J, (int)as);   // 4: e2m1
}

// 16-byte piece index in the LDS of piece c (of 8) of a row of 256 4-bit values: 16 consecutive rows at one piece lie on 16 different
// groups of 4 banks
__device__ __forceinline__ int piece_at(int row, int c) { return row * 8 + (c ^ ((row >> 1) & 7)); }

// MT x 32 rows, 4 wavefronts side by side with NS x 32 columns each
template <int MT, int NS, int EPI>
__global__ __launch_bounds__(256, 2) void mx_product_kernel(MxProduct p) {
  constexpr int BM = MT * 32, STRIPS = 4 * NS;
  constexpr int PIECES = BM * 8 / 256;   // of A per thread and chunk
  __shared__ uint4 a_codes[2][BM * 8];
  __shared__ unsigned a_scales[2][BM * 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int strips = p.n_out / 32, gx = (strips + STRIPS - 1) / STRIPS;
  const int tiles = p.offsets ? table_at(p.tile_map, 0) : (p.rows + BM - 1) / BM;
  // consecutive workgroups go to the 8 XCDs in turn: each XCD gets a run of consecutive tiles, column tiles fastest
  const long total = (long)tiles * gx;
  const long per_xcd = (total + 7) / 8, slot = blockIdx.x >> 3;
  const long id = (long)(blockIdx.x & 7) * per_xcd + slot;
  if (slot >= per_xcd || id >= total) return;
  const int tile = (int)(id / gx), strip0 = (int)(id % gx) * STRIPS + wave * NS;
  int group = 0, m0 = tile * BM, m_end = p.rows;
  if (p.offsets) {
    group = table_at(p.tile_map, TILE_MAP_HEADER + p.groups + 2 * tile);
    m0 = table_at(p.tile_map, TILE_MAP_HEADER + p.groups + 1 + 2 * tile);
    m_end = table_at(p.offsets, group + 1);
  }
  const int m_rows = min(m_end - m0, BM);
  const int steps = p.n_in / MX_STEP, chunks = (steps + 3) / 4;
  const unsigned row_bytes = (unsigned)p.n_in / 2, scale_bytes = (unsigned)chunks * 8;
  const auto ba = scalar_buffer((size_t)p.codes + (size_t)m0 * row_bytes, (size_t)m_rows * row_bytes);
  const auto bs = scalar_buffer((size_t)p.scales + (size_t)m0 * scale_bytes, (size_t)m_rows * scale_bytes);
  const size_t scales_at = (size_t)p.groups * p.n_in * p.n_out / 2;
  __amdgpu_buffer_rsrc_t bw[NS], bws[NS];
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    const bool there = strip0 + j < strips;   // past the last column: empty ranges, zeros
    const size_t strip = (size_t)group * strips + (there ? strip0 + j : 0);
    bw[j] = scalar_buffer((size_t)p.packed + strip * steps * 1024, there ? (size_t)steps * 1024 : 0);
    bws[j] = scalar_buffer((size_t)p.packed + scales_at + strip * chunks * 256, there ? (size_t)chunks * 256 : 0);
  }

  q4_t ra[PIECES], rw[2][NS][4];
  unsigned ras = 0, rws[2][NS];
  auto load_a = [&](int chunk) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int q = i * 256 + threadIdx.x;
      ra[i] = __builtin_amdgcn_raw_buffer_load_b128(ba, (unsigned)(q >> 3) * row_bytes + (unsigned)chunk * 128u + (unsigned)(q & 7) * 16u, 0, 0);
    }
    if (threadIdx.x < BM * 2) ras = __builtin_amdgcn_raw_buffer_load_b32(bs, (unsigned)(threadIdx.x >> 1) * scale_bytes + (unsigned)chunk * 8u + (threadIdx.x & 1) * 4u, 0, 0);
  };
  auto store_a = [&](int buf) {
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
      const int q = i * 256 + threadIdx.x;
      a_codes[buf][piece_at(q >> 3, q & 7)] = make_uint4(ra[i].x, ra[i].y, ra[i].z, ra[i].w);
    }
    if (threadIdx.x < BM * 2) a_scales[buf][threadIdx.x] = ras;
  };
  auto load_w = [&](int chunk, auto buf) {
    constexpr int b = decltype(buf)::value;
#pragma unroll
    for (int j = 0; j < NS; ++j) {
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) rw[b][j][ks] = __builtin_amdgcn_raw_buffer_load_b128(bw[j], (unsigned)(chunk * 4 + ks) * 1024u + (unsigned)lane * 16u, 0, 0);
      rws[b][j] = __builtin_amdgcn_raw_buffer_load_b32(bws[j], (unsigned)chunk * 256u + (unsigned)lane * 4u, 0, 0);
    }
  };
  f32x16_t acc[MT][NS];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.0f;
  auto step = [&](int buf, auto wbuf, auto ks, const unsigned (&as)[MT]) {
    constexpr int b = decltype(wbuf)::value, J = decltype(ks)::value;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint4 q = a_codes[buf][piece_at(i * 32 + (lane & 31), 2 * J + (lane >> 5))];
      const q4_t a = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int j = 0; j < NS; ++j) acc[i][j] = mx_mfma<J>(rw[b][j][J], rws[b][j], a, as[i], acc[i][j]);
    }
  };
  auto compute = [&](int chunk, int buf, auto wbuf) {
    unsigned as[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) as[i] = a_scales[buf][(i * 32 + (lane & 31)) * 2 + (lane >> 5)];
    const int left = steps - chunk * 4;   // instructions past the last input are left out
    step(buf, wbuf, std::integral_constant<int, 0>{}, as);
    if (left > 1) step(buf, wbuf, std::integral_constant<int, 1>{}, as);
    if (left > 2) step(buf, wbuf, std::integral_constant<int, 2>{}, as);
    if (left > 3) step(buf, wbuf, std::integral_constant<int, 3>{}, as);
  };
  constexpr std::integral_constant<int, 0> B0{};
  constexpr std::integral_constant<int, 1> B1{};
  load_a(0);
  load_w(0, B0);
  store_a(0);
  __syncthreads();
  for (int c = 0; c < chunks; c += 2) {   // (loads past the last chunk are out of range: zeros)
    load_a(c + 1);
    load_w(c + 1, B1);
    compute(c, 0, B0);
    if (c + 1 >= chunks) break;
    store_a(1);
    __syncthreads();
    load_a(c + 2);
    load_w(c + 2, B0);
    compute(c + 1, 1, B1);
    store_a(0);
    __syncthreads();
  }

  // lane l: row l % 32 of a sub-tile, columns 8 q + 4 (l / 32) + 0 .. 3 of a strip in values 4 q .. 4 q + 3
  const int half = lane >> 5;
#pragma unroll
  for (int j = 0; j < NS; ++j) {
    if (strip0 + j >= strips) break;
    const int col0 = (strip0 + j) * 32;
    float bias[16];
#pragma unroll
    for (int v = 0; v < 16; ++v) bias[v] = 0.0f;
    if (p.bias)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint2 b = *(const uint2*)(p.bias + (size_t)group * p.n_out + col0 + 8 * q + 4 * half);
        bias[4 * q] = __uint_as_float(b.x << 16); bias[4 * q + 1] = __uint_as_float(b.x & 0xFFFF0000u);
        bias[4 * q + 2] = __uint_as_float(b.y << 16); bias[4 * q + 3] = __uint_as_float(b.y & 0xFFFF0000u);
      }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int row = i * 32 + (lane & 31);
      const bool live = row < m_rows;
      const size_t at = (size_t)(m0 + row);
      float f[16];
#pragma unroll
      for (int v = 0; v < 16; ++v) f[v] = acc[i][j][v] + bias[v];
      if (EPI == MX_GELU_CODES) {
        unsigned top = 0;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
          f[v] = gelu_f(f[v]);
          top = max(top, __float_as_uint(f[v]) & 0x7FFFFFFFu);
        }
        top = max(top, from_lane_xor<32>(top, lane));
        const unsigned byte = mx_scale_byte(top);
        const unsigned lo = mx_codes8(f, byte), hi = mx_codes8(f + 8, byte);   // halfword q: this lane's four columns of quad q
        // the lower lane puts columns 0 .. 15 together, the upper one 16 .. 31: one exchange
        const unsigned got = from_lane_xor<32>(half ? lo : hi, lane);
        const unsigned mine = half ? hi : lo;
        const unsigned even = half ? got : mine, odd = half ? mine : got;      // quads of the lower lane, of the upper lane
        if (live) {
          *(uint2*)((uint8_t*)p.out + at * (p.n_out / 2) + col0 / 2 + 8 * half) =
              make_uint2((even & 0xFFFFu) | (odd << 16), (even >> 16) | (odd & 0xFFFF0000u));
          if (!half) p.out_scales[at * ((p.n_out + MX_CHUNK - 1) / MX_CHUNK * 8) + mx_scale_at((unsigned)col0 / 32)] = (uint8_t)byte;
        }
      } else if (live) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const size_t to = at * p.n_out + col0 + 8 * q + 4 * half;
          if (EPI == MX_STORE_F32) *(float4*)((float*)p.out + to) = make_float4(f[4 * q], f[4 * q + 1], f[4 * q + 2], f[4 * q + 3]);
          else *(uint2*)((bf16_t*)p.out + to) = make_uint2(f2bf_pair(f[4 * q], f[4 * q + 1]), f2bf_pair(f[4 * q + 2], f[4 * q + 3]));
        }
      }
    }
  }
}

template <int MT, int NS>
int launch_of(const MxProduct& p, hipStream_t s) {
  const long tiles = p.offsets ? (long)p.rows / (MT * 32) + p.groups : ((long)p.rows + MT * 32 - 1) / (MT * 32);
  const long gx = (p.n_out / 32 + 4 * NS - 1) / (4 * NS);
  const long blocks = (tiles * gx + 7) / 8 * 8;
  if (blocks > 0x7FFFFFFFl / 256 * 255) return BIGMAC_ERR_TOO_LARGE;
  const dim3 grid((unsigned)blocks);
  if (p.epilogue == MX_GELU_CODES) mx_product_kernel<MT, NS, MX_GELU_CODES><<<grid, 256, 0, s>>>(p);
  else if (p.epilogue == MX_STORE_F32) mx_product_kernel<MT, NS, MX_STORE_F32><<<grid, 256, 0, s>>>(p);
  else mx_product_kernel<MT, NS, MX_STORE_BF16><<<grid, 256, 0, s>>>(p);
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

}  // namespace

int mx_tile_rows(int rows, int groups) {
  const int even = rows / groups;
  return even > 64 ? 128 : even > 32 ? 64 : 32;
}

int launch_mx_product(const MxProduct& p, hipStream_t s) {
  switch (mx_tile_rows(p.rows, p.groups)) {
    case 32: return launch_of<1, 2>(p, s);
    case 64: return launch_of<2, 2>(p, s);
    default: return launch_of<4, 2>(p, s);
  }
}

}  // namespace bigmac

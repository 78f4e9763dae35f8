// Rows and weights into microscaled 4-bit floating point and back, and the C entry points of the 4-bit path.
//
// Conversions are bound by HBM: 2 or 4 bytes read, 17/32 of a byte written per value (back: the other way round).  Rows: eight
// consecutive values a lane (16 bytes of bf16), a block's largest magnitude over four neighbouring lanes by register moves, the
// comparison on the magnitudes' bits, which also finds infinities and NaN.  Weights: blocks run down the columns, so a lane takes
// four columns x 32 inputs (reads of 512 or 1024 contiguous bytes a wavefront) and has whole blocks to itself.
#include <algorithm>

#include "mx.hpp"

namespace bigmac {

namespace {

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* f);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* f) {
  const float4 a = *(const float4*)p, b = *(const float4*)(p + 4);
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <>
__device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float* f) { unpack_bf16x8(*(const uint4*)p, f); }
__device__ __forceinline__ void put8(float* p, const float* f) {
  *(float4*)p = make_float4(f[0], f[1], f[2], f[3]);
  *(float4*)(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void put8(bf16_t* p, const float* f) { *(uint4*)p = pack_bf16x8(f); }

// The tile map by one workgroup of 256 threads, up to 1024 groups: tiles in front of every group (four groups a thread, a scan over the
// wavefronts), then each thread finds the groups of every 256th tile.  Whatever the offsets hold, nothing is written past the map: counts wrap,
// and the tiles are cut off at the most that ascending offsets make; the products leave out tiles outside their rows.
__device__ __forceinline__ void build_mx_map(const MxMapJob& job) {
  __shared__ unsigned before[1025], wave_total[4];
  __shared__ int start[1025];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g0 = threadIdx.x * 4;
  unsigned count[4], sum = 0;
  int edge[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) edge[i] = job.offsets[min(g0 + i, job.groups)];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int g = g0 + i;
    count[i] = g < job.groups ? (unsigned)max((long)edge[i + 1] - edge[i] + job.tile_rows - 1, 0l) / (unsigned)job.tile_rows : 0;
    sum += count[i];
  }
  unsigned upto = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned o = __shfl_up(upto, d, 64);
    if (lane >= d) upto += o;
  }
  if (lane == 63) wave_total[wave] = upto;
  __syncthreads();
  unsigned at = upto - sum;
  for (int w = 0; w < wave; ++w) at += wave_total[w];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    before[g0 + i] = at;
    start[g0 + i] = edge[i];
    at += count[i];
  }
  if (threadIdx.x == 255) {
    before[1024] = min(at, (unsigned)mx_most_tiles(job.rows, job.groups, job.tile_rows));
    start[1024] = edge[4];
    job.map[0] = (int)before[1024];
  }
  __syncthreads();
  const unsigned tiles = before[1024];
  for (unsigned i = threadIdx.x; i < tiles; i += 256) {
    int lo = 0, hi = job.groups;           // the last group that starts at or in front of tile i: groups without rows start where the next one does
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (before[mid] <= i) lo = mid;
      else hi = mid;
    }
    *(int4*)(job.map + 4 + 4 * (size_t)i) = make_int4(lo, (int)((unsigned)start[lo] + (i - before[lo]) * (unsigned)job.tile_rows), min(start[lo + 1], job.rows), 0);
  }
}
__global__ __launch_bounds__(256) void mx_map_kernel(MxMapJob job) { build_mx_map(job); }

constexpr int ROW_TURNS = 4;   // rows a thread takes

// 1 << log_tx threads side by side on a row, the others on further rows
template <typename T>
__global__ __launch_bounds__(256) void mx_quantize_kernel(const T* __restrict__ src, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, long rows,
                                                          int cols, int log_tx, int scale_bytes, MxMapJob map0, MxMapJob map1) {
  if (map0.map && blockIdx.x >= gridDim.x - (map1.map ? 2 : 1)) {
    if (blockIdx.x == gridDim.x - 1) build_mx_map(map0);
    else build_mx_map(map1);
    return;
  }
  const int tx = threadIdx.x & ((1 << log_tx) - 1), ty = threadIdx.x >> log_tx, rows_at_once = 256 >> log_tx;
  const int pieces = cols / 8;
  for (int p = tx; p < scale_bytes * 4; p += 1 << log_tx) {   // (a multiple of 4 pieces; past the row's end only the unused scale bytes)
#pragma unroll
    for (int j = 0; j < ROW_TURNS; ++j) {
      const long row = ((long)blockIdx.x * ROW_TURNS + j) * rows_at_once + ty;
      if (row >= rows) break;
      uint8_t* to = scales + mx_scale_at(rows, row, (unsigned)p / 4);
      if (p >= pieces) {
        if ((p & 3) == 0) *to = 0;
        continue;
      }
      float f[8];
      load8(src + row * cols + (long)p * 8, f);
      unsigned top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7FFFFFFFu);
      top = max(top, from_lane_xor<1>(top, 0));
      top = max(top, from_lane_xor<2>(top, 0));
      const unsigned byte = mx_scale_byte(top);
      *(unsigned*)(codes + row * (cols / 2) + (long)p * 4) = mx_codes8(f, byte);
      if ((p & 3) == 0) *to = (uint8_t)byte;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, T* __restrict__ dst, long rows,
                                                            int cols, int log_tx) {
  const int tx = threadIdx.x & ((1 << log_tx) - 1), ty = threadIdx.x >> log_tx, rows_at_once = 256 >> log_tx;
  const int pieces = cols / 8;
  for (int p = tx; p < pieces; p += 1 << log_tx) {
#pragma unroll
    for (int j = 0; j < ROW_TURNS; ++j) {
      const long row = ((long)blockIdx.x * ROW_TURNS + j) * rows_at_once + ty;
      if (row >= rows) break;
      float f[8];
      mx_values8(*(const unsigned*)(codes + row * (cols / 2) + (long)p * 4), mx_scale(scales[mx_scale_at(rows, row, (unsigned)p / 4)]), f);
      put8(dst + row * cols + (long)p * 8, f);
    }
  }
}

// A thread's part of the weights: four output columns, one block out of each of up to four matrix instructions
struct PackPlace {
  long group;
  int col, chunk, half;
  bool any;
};
__device__ __forceinline__ PackPlace pack_place(long groups, int n_in, int n_out) {
  const int quads = n_out / 4, chunks2 = (n_in + MX_CHUNK - 1) / MX_CHUNK * 2;
  const long id = (long)blockIdx.x * 256 + threadIdx.x;
  PackPlace t;
  t.any = id < groups * chunks2 * quads;
  t.col = (int)(id % quads) * 4;
  const long rest = id / quads;
  t.half = (int)(rest & 1);
  t.chunk = (int)(rest % chunks2) >> 1;
  t.group = rest / chunks2;
  return t;
}
__device__ __forceinline__ void load4(const float* p, float* f) {
  const float4 a = *(const float4*)p;
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
}
__device__ __forceinline__ void load4(const bf16_t* p, float* f) {
  const uint2 a = *(const uint2*)p;
  f[0] = __uint_as_float(a.x << 16); f[1] = __uint_as_float(a.x & 0xFFFF0000u);
  f[2] = __uint_as_float(a.y << 16); f[3] = __uint_as_float(a.y & 0xFFFF0000u);
}
__device__ __forceinline__ void put4(float* p, const float* f) { *(float4*)p = make_float4(f[0], f[1], f[2], f[3]); }
__device__ __forceinline__ void put4(bf16_t* p, const float* f) { *(uint2*)p = make_uint2(f2bf_pair(f[0], f[1]), f2bf_pair(f[2], f[3])); }

template <typename T>
__global__ __launch_bounds__(256) void mx_pack_kernel(const T* __restrict__ w, uint8_t* __restrict__ packed, long groups, int n_in, int n_out) {
  const PackPlace t = pack_place(groups, n_in, n_out);
  if (!t.any) return;
  const int steps = n_in / MX_STEP;
  const size_t strip = (size_t)(t.group * (n_out / 32) + t.col / 32) * mx_strip_bytes(n_in);
  const int lane = t.half * 32 + t.col % 32;
  unsigned bytes[4] = {0, 0, 0, 0};
#pragma unroll 1
  for (int j = 0; j < 4; ++j) {
    const int step = t.chunk * 4 + j;
    if (step >= steps) break;
    const T* from = w + (t.group * n_in + step * MX_STEP + t.half * MX_BLOCK) * n_out + t.col;
    float f[4][32];
#pragma unroll
    for (int k = 0; k < 32; ++k) {
      float v[4];
      load4(from + (long)k * n_out, v);
#pragma unroll
      for (int c = 0; c < 4; ++c) f[c][k] = v[c];
    }
    uint4* to = (uint4*)(packed + strip + (size_t)step * 1024) + lane;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      unsigned top = 0;
#pragma unroll
      for (int k = 0; k < 32; ++k) top = max(top, __float_as_uint(f[c][k]) & 0x7FFFFFFFu);
      const unsigned byte = mx_scale_byte(top);
      to[c] = make_uint4(mx_codes8(f[c], byte), mx_codes8(f[c] + 8, byte), mx_codes8(f[c] + 16, byte), mx_codes8(f[c] + 24, byte));
      bytes[c] |= byte << (8 * j);
    }
  }
  *(uint4*)(packed + strip + (size_t)steps * 1024 + t.chunk * 256 + lane * 4) = make_uint4(bytes[0], bytes[1], bytes[2], bytes[3]);
}

template <typename T>
__global__ __launch_bounds__(256) void mx_unpack_kernel(const uint8_t* __restrict__ packed, T* __restrict__ w, long groups, int n_in, int n_out) {
  const PackPlace t = pack_place(groups, n_in, n_out);
  if (!t.any) return;
  const int steps = n_in / MX_STEP;
  const size_t strip = (size_t)(t.group * (n_out / 32) + t.col / 32) * mx_strip_bytes(n_in);
  const int lane = t.half * 32 + t.col % 32;
  const uint4 b = *(const uint4*)(packed + strip + (size_t)steps * 1024 + t.chunk * 256 + lane * 4);
  const unsigned bytes[4] = {b.x, b.y, b.z, b.w};
#pragma unroll 1
  for (int j = 0; j < 4; ++j) {
    const int step = t.chunk * 4 + j;
    if (step >= steps) break;
    T* to = w + (t.group * n_in + step * MX_STEP + t.half * MX_BLOCK) * n_out + t.col;
    const uint4* from = (const uint4*)(packed + strip + (size_t)step * 1024) + lane;
    uint4 q[4];
    float scale[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      q[c] = from[c];
      scale[c] = mx_scale((bytes[c] >> (8 * j)) & 255u);
    }
#pragma unroll
    for (int k8 = 0; k8 < 4; ++k8) {
      float f[4][8];
#pragma unroll
      for (int c = 0; c < 4; ++c) mx_values8(k8 == 0 ? q[c].x : k8 == 1 ? q[c].y : k8 == 2 ? q[c].z : q[c].w, scale[c], f[c]);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float v[4] = {f[0][k], f[1][k], f[2][k], f[3][k]};
        put4(to + (long)(k8 * 8 + k) * n_out, v);
      }
    }
  }
}

struct RowGrid {
  long blocks;
  int log_tx;
};
RowGrid row_grid(long rows, long pieces) {
  int log_tx = 2;
  while (log_tx < 8 && (1l << log_tx) < pieces) ++log_tx;
  const long per_block = (long)ROW_TURNS * (256 >> log_tx);
  return {(rows + per_block - 1) / per_block, log_tx};
}

bool aligned(std::initializer_list<const void*> ps) {
  for (const void* q : ps)
    if ((size_t)q & 15) return false;
  return true;
}
constexpr long MAX_ROWS = 1l << 30, MAX_COLS = 1l << 24;
int check_rows(int64_t rows, int64_t cols, int dtype) {
  if (rows < 1 || cols < 32 || cols % 32 || (dtype != BIGMAC_F32 && dtype != BIGMAC_BF16)) return BIGMAC_ERR_INVALID_ARG;
  return rows > MAX_ROWS || cols > MAX_COLS || row_grid(rows, cols / 8).blocks >= MX_MAX_BLOCKS - 1 ? BIGMAC_ERR_TOO_LARGE : BIGMAC_OK;
}
long pack_blocks(long groups, long n_in, long n_out) { return (groups * ((n_in + MX_CHUNK - 1) / MX_CHUNK) * 2 * (n_out / 4) + 255) / 256; }
int check_weights(int32_t groups, int32_t n_in, int32_t n_out) {
  if (groups < 1 || n_in < 64 || n_in % 64 || n_out < 64 || n_out % 64) return BIGMAC_ERR_INVALID_ARG;
  return groups > 1024 || n_in > MAX_COLS || n_out > MAX_COLS || pack_blocks(groups, n_in, n_out) > MX_MAX_BLOCKS ? BIGMAC_ERR_TOO_LARGE : BIGMAC_OK;
}
int check_mx(const bigmac_mx_dims* D) {
  if (!D || D->rows < 1 || (D->out_dtype != BIGMAC_F32 && D->out_dtype != BIGMAC_BF16)) return BIGMAC_ERR_INVALID_ARG;
  const int rc = check_weights(D->groups, D->n_in, D->n_out);
  return rc ? rc : D->rows > MAX_ROWS ? BIGMAC_ERR_TOO_LARGE : BIGMAC_OK;
}
size_t mx_map_bytes(int rows, int groups) { return align_up(mx_map_ints(rows, groups) * 4); }

struct FfnPlan {
  size_t x_codes, x_scales, h_codes, h_scales, up_map, down_map, total;
};
FfnPlan plan_ffn(const bigmac_dims& D) {
  const Widths W = widths(D);
  const size_t rows = (size_t)D.T * D.k;
  FfnPlan p;
  p.x_codes = 0;
  p.x_scales = align_up(rows * W.win / 2);
  p.h_codes = p.x_scales + align_up(rows * mx_scale_bytes(W.win));
  p.h_scales = p.h_codes + align_up(rows * W.hid / 2);
  p.up_map = p.h_scales + align_up(rows * mx_scale_bytes(W.hid));
  p.down_map = p.up_map + mx_map_bytes((int)rows, D.N);
  p.total = p.down_map + mx_map_bytes((int)rows, D.N);
  return p;
}
// A product as far as sizes go, for ragged rows or dense ones
MxProduct product_of(const bigmac_mx_dims& D, const int32_t* offsets) {
  MxProduct p{};
  p.offsets = offsets;
  p.rows = D.rows; p.groups = D.groups; p.n_in = D.n_in; p.n_out = D.n_out;
  p.epilogue = D.out_dtype == BIGMAC_F32 ? MX_STORE_F32 : MX_STORE_BF16;
  p.tile_rows = mx_tile_rows(D.rows, D.groups, D.n_in, D.n_out, p.epilogue);
  return p;
}
constexpr int32_t SOME_OFFSETS = 0;   // its address: where only the sizes of a ragged product are asked for
// The FFN's two products as far as sizes and offsets (not NULL) go, or the code of what is too large; before anything is launched
int ffn_products(const bigmac_dims& D, const int32_t* offsets, MxProduct& up, MxProduct& down) {
  const Widths W = widths(D);
  int rc = check_weights(D.N, W.win, W.hid);
  if (!rc) rc = check_rows((int64_t)D.T * D.k, W.win, BIGMAC_BF16);
  if (rc) return rc;
  up.n_in = W.win; up.n_out = W.hid; up.epilogue = MX_GELU_CODES;
  down.n_in = W.hid; down.n_out = W.win; down.epilogue = MX_STORE_BF16;
  for (MxProduct* p : {&up, &down}) {
    p->offsets = offsets;
    p->rows = D.T * D.k; p->groups = D.N;
    p->tile_rows = mx_tile_rows(p->rows, p->groups, p->n_in, p->n_out, p->epilogue);
    rc = check_mx_product(*p);
    if (rc) return rc;
  }
  return BIGMAC_OK;
}

}  // namespace

int launch_mx_quantize(long rows, long cols, int dtype, const void* src, uint8_t* codes, uint8_t* scales, hipStream_t s, const MxMapJob* maps) {
  const int scale_bytes = (int)mx_scale_bytes(cols);
  const RowGrid g = row_grid(rows, cols / 8);
  const MxMapJob map0 = maps ? maps[0] : MxMapJob{}, map1 = maps ? maps[1] : MxMapJob{};
  const unsigned blocks = (unsigned)g.blocks + (map0.map ? 1 : 0) + (map1.map ? 1 : 0);
  if (dtype == BIGMAC_BF16) mx_quantize_kernel<bf16_t><<<blocks, 256, 0, s>>>((const bf16_t*)src, codes, scales, rows, (int)cols, g.log_tx, scale_bytes, map0, map1);
  else mx_quantize_kernel<float><<<blocks, 256, 0, s>>>((const float*)src, codes, scales, rows, (int)cols, g.log_tx, scale_bytes, map0, map1);
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

size_t mx_ffn_ws_bytes(const bigmac_dims& D) {
  MxProduct up{}, down{};
  return ffn_products(D, &SOME_OFFSETS, up, down) == BIGMAC_OK ? plan_ffn(D).total : 0;
}

}  // namespace bigmac

using namespace bigmac;

extern "C" {

size_t bigmac_mx_scale_bytes(int64_t cols) { return cols < 32 || cols % 32 || cols > MAX_COLS ? 0 : mx_scale_bytes(cols); }

size_t bigmac_mx_packed_bytes(int32_t groups, int32_t n_in, int32_t n_out) {
  return check_weights(groups, n_in, n_out) == BIGMAC_OK ? mx_packed_bytes(groups, n_in, n_out) : 0;
}

int bigmac_mx_quantize(int64_t rows, int64_t cols, int32_t dtype, const void* src, void* codes, void* scales, void* stream) {
  const int rc = check_rows(rows, cols, dtype);
  if (rc) return rc;
  if (!src || !codes || !scales || !aligned({src, codes, scales})) return BIGMAC_ERR_INVALID_ARG;
  return launch_mx_quantize(rows, cols, dtype, src, (uint8_t*)codes, (uint8_t*)scales, (hipStream_t)stream);
}

int bigmac_mx_dequantize(int64_t rows, int64_t cols, const void* codes, const void* scales, int32_t dtype, void* dst, void* stream) {
  const int rc = check_rows(rows, cols, dtype);
  if (rc) return rc;
  if (!dst || !codes || !scales || !aligned({dst, codes, scales})) return BIGMAC_ERR_INVALID_ARG;
  const RowGrid g = row_grid(rows, cols / 8);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == BIGMAC_BF16) mx_dequantize_kernel<bf16_t><<<(unsigned)g.blocks, 256, 0, s>>>((const uint8_t*)codes, (const uint8_t*)scales, (bf16_t*)dst, rows, (int)cols, g.log_tx);
  else mx_dequantize_kernel<float><<<(unsigned)g.blocks, 256, 0, s>>>((const uint8_t*)codes, (const uint8_t*)scales, (float*)dst, rows, (int)cols, g.log_tx);
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

int bigmac_mx_pack(int32_t groups, int32_t n_in, int32_t n_out, int32_t dtype, const void* w, void* packed, void* stream) {
  const int rc = check_weights(groups, n_in, n_out);
  if (rc) return rc;
  if ((dtype != BIGMAC_F32 && dtype != BIGMAC_BF16) || !w || !packed || !aligned({w, packed})) return BIGMAC_ERR_INVALID_ARG;
  const unsigned blocks = (unsigned)pack_blocks(groups, n_in, n_out);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == BIGMAC_BF16) mx_pack_kernel<bf16_t><<<blocks, 256, 0, s>>>((const bf16_t*)w, (uint8_t*)packed, groups, n_in, n_out);
  else mx_pack_kernel<float><<<blocks, 256, 0, s>>>((const float*)w, (uint8_t*)packed, groups, n_in, n_out);
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

int bigmac_mx_unpack(int32_t groups, int32_t n_in, int32_t n_out, const void* packed, int32_t dtype, void* w, void* stream) {
  const int rc = check_weights(groups, n_in, n_out);
  if (rc) return rc;
  if ((dtype != BIGMAC_F32 && dtype != BIGMAC_BF16) || !w || !packed || !aligned({w, packed})) return BIGMAC_ERR_INVALID_ARG;
  const unsigned blocks = (unsigned)pack_blocks(groups, n_in, n_out);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == BIGMAC_BF16) mx_unpack_kernel<bf16_t><<<blocks, 256, 0, s>>>((const uint8_t*)packed, (bf16_t*)w, groups, n_in, n_out);
  else mx_unpack_kernel<float><<<blocks, 256, 0, s>>>((const uint8_t*)packed, (float*)w, groups, n_in, n_out);
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

size_t bigmac_mx_workspace_bytes(const bigmac_mx_dims* D) {
  return check_mx(D) == BIGMAC_OK && check_mx_product(product_of(*D, &SOME_OFFSETS)) == BIGMAC_OK ? mx_map_bytes(D->rows, D->groups) : 0;
}

int bigmac_mx_product(const bigmac_mx_dims* D, const void* codes, const void* scales, const int32_t* offsets, const void* packed, const void* bias, void* out,
                      void* ws, size_t ws_bytes, void* stream) {
  int rc = check_mx(D);
  if (rc) return rc;
  if (!codes || !scales || !packed || !out || !aligned({codes, scales, packed, bias, out})) return BIGMAC_ERR_INVALID_ARG;
  if (!offsets && D->groups != 1) return BIGMAC_ERR_INVALID_ARG;
  hipStream_t s = (hipStream_t)stream;
  MxProduct p = product_of(*D, offsets);
  p.codes = (const uint8_t*)codes; p.scales = (const uint8_t*)scales; p.packed = (const uint8_t*)packed; p.bias = (const bf16_t*)bias;
  p.out = out;
  if (offsets) {
    if (!ws || !aligned({ws})) return BIGMAC_ERR_INVALID_ARG;
    if (ws_bytes < mx_map_bytes(D->rows, D->groups)) return BIGMAC_ERR_WORKSPACE;
    p.tile_map = (const int*)ws;
  }
  rc = check_mx_product(p);
  if (rc) return rc;
  if (offsets) {
    mx_map_kernel<<<1, 256, 0, s>>>(MxMapJob{offsets, (int*)ws, D->rows, D->groups, p.tile_rows});
    BIGMAC_CHECK_LAUNCH();
  }
  return launch_mx_product(p, s);
}

int bigmac_mx_grouped_ffn(const bigmac_dims* D, const void* x_perm, const int32_t* expert_offsets, const void* w1, const void* w2, const void* b1, const void* b2,
                          void* o_perm, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_dims(D);
  if (rc) return rc;
  if (D->dtype != BIGMAC_BF16) return BIGMAC_ERR_UNSUPPORTED;
  MxProduct up{}, down{};
  if (!expert_offsets) return BIGMAC_ERR_INVALID_ARG;
  rc = ffn_products(*D, expert_offsets, up, down);
  if (rc) return rc;
  if (!x_perm || !w1 || !w2 || !o_perm || !ws || !aligned({x_perm, w1, w2, b1, b2, o_perm, ws})) return BIGMAC_ERR_INVALID_ARG;
  const FfnPlan plan = plan_ffn(*D);
  if (ws_bytes < plan.total) return BIGMAC_ERR_WORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  const int rows = up.rows;
  uint8_t* base = (uint8_t*)ws;
  up.codes = base + plan.x_codes; up.scales = base + plan.x_scales; up.packed = (const uint8_t*)w1; up.bias = (const bf16_t*)b1;
  up.out = base + plan.h_codes; up.out_scales = base + plan.h_scales;
  down.codes = base + plan.h_codes; down.scales = base + plan.h_scales; down.packed = (const uint8_t*)w2; down.bias = (const bf16_t*)b2;
  down.out = o_perm;
  MxMapJob maps[2] = {{expert_offsets, (int*)(base + plan.up_map), rows, D->N, up.tile_rows}, {}};
  if (down.tile_rows != up.tile_rows) maps[1] = {expert_offsets, (int*)(base + plan.down_map), rows, D->N, down.tile_rows};
  up.tile_map = maps[0].map;
  down.tile_map = maps[1].map ? maps[1].map : maps[0].map;
  rc = launch_mx_quantize(rows, up.n_in, BIGMAC_BF16, x_perm, base + plan.x_codes, base + plan.x_scales, s, maps);
  if (!rc) rc = launch_mx_product(up, s);
  return rc ? rc : launch_mx_product(down, s);
}

}  // extern "C"

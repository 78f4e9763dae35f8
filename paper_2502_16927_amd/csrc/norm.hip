// The norms on both sides of a block, with the block's gate and residual scale:
//     z = alpha x + g * n_post(y)        u = n_pre(z as stored)
//     n(v) = w (v - m) rstd + b,   rstd = 1 / sqrt(mean((v - m)^2) + eps),   m = mean(v) (layer norm) or 0 (RMS norm)
// and their gradients.  With v^ = (v - m) rstd and c the gradient of n(v), a = c w:
//     n'(c) = rstd (a - mean(a) - v^ mean(a v^))   (RMS norm: without mean(a)),   dw = sum_t c v^,   db = sum_t c
//     dZ = dz + n_pre'(du);   dx = alpha dZ;   dn = g dZ;   dy = n_post'(dn);   dg = dZ n_post(y), summed over what g is broadcast over
//
// What bounds them: HBM.  A row passes through registers once: a wavefront (up to 512 columns) or 2 to 16 of one workgroup hold it,
// 8 columns a lane, so every tensor is read once and written once, and the statistics of the backward are worked out again from the
// rows that it reads anyway instead of being stored.  (16 columns a lane: 154 registers forward, 234 backward, two wavefronts a SIMD.)  32768 rows
// of 4096, bf16 stream, fp32 y: forward 242 us (5.6 TB/s), backward 428 us (5.0 TB/s; a large copy reaches 4.9, a sum of two tensors 6.05).  Wider rows
// are slower: 16384 of 8192 252 and 672 us (5.3 and 3.2 TB/s, see the backward), 26208 of 5120, whose lanes are half idle, 345 and 940.  Vectors (weights, channel
// gate) stay in registers over the rows of a persistent workgroup.  Sums and statistics are fp32; a layer norm's variance is
// taken behind its mean.  Rows are addressed as buffers (range = the row): a lane past the end of the row loads zeros and its
// stores are dropped, and the two halves of an fp32 piece and the one of a bf16 piece are the same code without a branch.
#include <algorithm>
#include <cmath>

#include "wave.hpp"

namespace bigmac {

namespace {

constexpr unsigned PAST = 0x80000000u;   // offset outside every row

struct NormArgs {
  const void *x, *y, *gate, *du, *dz;    // x: the stream in front of the branch (forward), behind it (backward: z)
  const float *post_w, *post_b, *pre_w, *pre_b;
  void *z, *u;                           // forward
  void *dx, *dy, *dgate;                 // backward
  float* part;                           // backward: [workgroups][vectors][d]
  int T, d, x_f32, y_f32, u_f32, layer, gate_kind;
  float eps, alpha, inv_d;
};

typedef unsigned int q4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* base, int row, int d, int f32) {
  const size_t bytes = (size_t)d * (f32 ? 4 : 2);
  const size_t at = (size_t)base + (size_t)row * bytes;
  const unsigned lo = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)at), hi = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32));
  return __builtin_amdgcn_make_buffer_rsrc((void*)(((size_t)hi << 32) | lo), 0, base ? (int)bytes : 0, 0x00020000);
}

// 8 consecutive elements as they lie in memory: one piece of 16 bytes (bf16) or two (fp32)
struct Raw8 {
  q4_t q[2];
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int col, int f32) {
    const unsigned at = (unsigned)col * (f32 ? 4u : 2u);
    q[0] = __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0);
    q[1] = __builtin_amdgcn_raw_buffer_load_b128(r, f32 ? at + 16u : PAST, 0, 0);
  }
  __device__ __forceinline__ void values(int f32, float* f) const {
    if (f32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(q[i >> 2][i & 3]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(i & 1 ? q[0][i >> 1] & 0xFFFF0000u : q[0][i >> 1] << 16);
    }
  }
};
// stores 8 elements; rounded: what the row then holds
__device__ __forceinline__ void store8(__amdgpu_buffer_rsrc_t r, int col, int f32, const float* f, float* rounded = nullptr) {
  if (f32) {
    q4_t a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = __float_as_uint(f[i]);
      b[i] = __float_as_uint(f[4 + i]);
    }
    __builtin_amdgcn_raw_buffer_store_b128(a, r, (unsigned)col * 4u, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b128(b, r, (unsigned)col * 4u + 16u, 0, 0);
    if (rounded)
#pragma unroll
    for (int i = 0; i < 8; ++i) rounded[i] = f[i];
  } else {
    q4_t a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = f2bf_pair(f[2 * i], f[2 * i + 1]);
    __builtin_amdgcn_raw_buffer_store_b128(a, r, (unsigned)col * 2u, 0, 0);
    if (rounded)
#pragma unroll
    for (int i = 0; i < 8; ++i) rounded[i] = __uint_as_float(i & 1 ? a[i >> 1] & 0xFFFF0000u : a[i >> 1] << 16);
  }
}

// Sums of M values over the W wavefronts that hold a row, the same in all of them.  box: [2][rows of the workgroup][W][M],
// the two halves in turn, so that one barrier per sum is enough.
template <int W, int M, int SLOTS>
__device__ __forceinline__ void row_sums(float (&v)[M], float* box, int& turn, int slot, int wave_in_row, int lane) {
#pragma unroll
  for (int m = 0; m < M; ++m) v[m] = wave_sum(v[m], lane);
  if (W == 1) return;
  constexpr int MAX_M = 4;
  float* mine = box + ((turn & 1) * SLOTS + slot) * W * MAX_M;
  ++turn;
  if (lane == 0)
#pragma unroll
    for (int m = 0; m < M; ++m) mine[wave_in_row * MAX_M + m] = v[m];
  __syncthreads();
#pragma unroll
  for (int m = 0; m < M; ++m) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) s += mine[w * MAX_M + m];
    v[m] = s;
  }
}

__device__ __forceinline__ void load_vector(const float* p, int d, int col, float none, float (&f)[8]) {
  const auto r = row_buffer(p, 0, d, 1);
  Raw8 q;
  q.load(r, col, 1);
  q.values(1, f);
  if (!p)
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = none;
}

// W wavefronts per row, 8 columns per lane
template <int W>
struct RowShape {
  static constexpr int WAVES = W < 4 ? 4 : W, THREADS = WAVES * 64, SLOTS = WAVES / W;   // rows a workgroup holds at a time
};

template <int W, bool POST, bool PRE>
__global__ __launch_bounds__((RowShape<W>::THREADS)) void norm_forward_kernel(NormArgs p) {
  using S = RowShape<W>;
  __shared__ float box[W > 1 ? 2 * S::SLOTS * W * 4 : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int slot = wave / W, wir = wave % W;
  const int col = (wir * 64 + lane) * 8;
  const float in_row = col < p.d ? 1.0f : 0.0f;
  float pw[8], qw[8], cg[8];
  if (POST) load_vector(p.post_w, p.d, col, 1.0f, pw);
  if (PRE) load_vector(p.pre_w, p.d, col, 1.0f, qw);
  if (POST) load_vector(p.gate_kind == BIGMAC_GATE_CHANNEL ? (const float*)p.gate : nullptr, p.d, col, 1.0f, cg);
  int turn = 0;
  // every wavefront makes the same number of turns: the barriers of the sums are the workgroup's
  for (int first = blockIdx.x * S::SLOTS; first < p.T; first += gridDim.x * S::SLOTS) {
    const int row = first + slot;
    const bool live = row < p.T;
    const int at = live ? row : 0;
    auto buffer = [&](const void* base, int f32) { return row_buffer(live ? base : nullptr, at, p.d, f32); };
    Raw8 rx, ry, rg;
    const auto bx = buffer(p.x, p.x_f32), by = buffer(p.y, p.y_f32), bg = buffer(p.gate_kind == BIGMAC_GATE_FULL ? p.gate : nullptr, p.u_f32);
    if (POST) ry.load(by, col, p.y_f32);
    rx.load(bx, col, p.x_f32);
    if (POST && p.gate_kind == BIGMAC_GATE_FULL) rg.load(bg, col, p.u_f32);
    float token_gate = 1.0f;
    if (POST && p.gate_kind == BIGMAC_GATE_TOKEN) token_gate = ((const float*)p.gate)[at];

    // mean and reciprocal root of a row held in registers
    auto centre = [&](float (&f)[8]) {   // subtracts the mean of a layer norm, returns rstd
      if (p.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0] += f[i];
        row_sums<W, 1, S::SLOTS>(s, box, turn, slot, wir, lane);
        const float m = s[0] * p.inv_d;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = in_row * (f[i] - m);
      }
      float s[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] = fmaf(f[i], f[i], s[0]);
      row_sums<W, 1, S::SLOTS>(s, box, turn, slot, wir, lane);
      return 1.0f / sqrtf(fmaf(s[0], p.inv_d, p.eps));
    };
    auto affine = [&](float (&f)[8], float rstd, const float (&w)[8], const float* bias) {
      float b[8];
      if (bias) load_vector(bias, p.d, col, 0.0f, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = bias ? fmaf(f[i] * rstd, w[i], b[i]) : f[i] * rstd * w[i];
    };

    float z[8];
    if (POST) {
      float n[8];
      ry.values(p.y_f32, n);
      const float rstd = centre(n);
      affine(n, rstd, pw, p.post_b);
      const auto bz = buffer(p.z, p.x_f32);
      float f[8], g[8];
      rx.values(p.x_f32, f);
      if (p.gate_kind == BIGMAC_GATE_FULL) rg.values(p.u_f32, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float gate = p.gate_kind == BIGMAC_GATE_FULL ? g[i] : cg[i] * token_gate;
        f[i] = fmaf(gate, n[i], p.alpha * f[i]);
      }
      store8(bz, col, p.x_f32, f, z);
    } else {
      rx.values(p.x_f32, z);
    }
    if (PRE) {
      // (columns past the row hold alpha * 0 + gate * 0: zero)
      const float rstd = centre(z);
      affine(z, rstd, qw, p.pre_b);
      const auto bu = buffer(p.u, p.u_f32);
      store8(bu, col, p.u_f32, z);
    }
  }
}

// Vectors of partial sums, in this order as far as the call has them: du z^, dn y^ (with a channel gate dZ y^), du, dn (dZ)
// Four wavefronts a SIMD without biases: 32768 x 4096 471 -> 443 us, although with both norms 10 registers spill there (1 with 4 wavefronts a row); with biases
// too many would, 43 -> 50 us at 6001 x 1024.  16 wavefronts a row (past 4096 columns) are 1024 threads, 128 registers whatever is asked for: with both norms 56
// spill, with biases 81, and 16384 x 8192 takes 672 and 845 us (3.2 and 2.5 TB/s).
template <int W, bool POST, bool PRE, bool BIAS>
__global__ __launch_bounds__((RowShape<W>::THREADS), BIAS ? 1 : 4) void norm_backward_kernel(NormArgs p) {
  using S = RowShape<W>;
  constexpr int VECTORS = ((POST ? 1 : 0) + (PRE ? 1 : 0)) * (BIAS ? 2 : 1);
  __shared__ float box[W > 1 ? 2 * S::SLOTS * W * 4 : 1];
  __shared__ float4 join[S::SLOTS > 1 ? (S::SLOTS - 1) * W * 64 * 2 : 1];   // the slots' sums on their way into the first slot's, 8 columns per lane
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int slot = wave / W, wir = wave % W;
  const int col = (wir * 64 + lane) * 8;
  const float in_row = col < p.d ? 1.0f : 0.0f;
  float pw[8], qw[8], cg[8];
  if (POST) load_vector(p.post_w, p.d, col, 1.0f, pw);
  if (PRE) load_vector(p.pre_w, p.d, col, 1.0f, qw);
  if (POST) load_vector(p.gate_kind == BIGMAC_GATE_CHANNEL ? (const float*)p.gate : nullptr, p.d, col, 1.0f, cg);
  float sum[VECTORS][8];
#pragma unroll
  for (int k = 0; k < VECTORS; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[k][i] = 0.0f;
  constexpr int AT_PRE = 0, AT_POST = PRE ? 1 : 0, AT_BIAS = (POST ? 1 : 0) + (PRE ? 1 : 0);
  int turn = 0;
  for (int first = blockIdx.x * S::SLOTS; first < p.T; first += gridDim.x * S::SLOTS) {
    const int row = first + slot;
    const bool live = row < p.T;
    const int at = live ? row : 0;
    auto buffer = [&](const void* base, int f32) { return row_buffer(live ? base : nullptr, at, p.d, f32); };
    Raw8 rz, ry, rdu, rdz, rg;
    const auto bz = buffer(p.x, p.x_f32), by = buffer(p.y, p.y_f32), bdu = buffer(p.du, p.y_f32), bdz = buffer(p.dz, p.x_f32);
    const auto bg = buffer(p.gate_kind == BIGMAC_GATE_FULL ? p.gate : nullptr, p.u_f32);
    if (PRE) rz.load(bz, col, p.x_f32);
    if (PRE) rdu.load(bdu, col, p.y_f32);
    if (POST) ry.load(by, col, p.y_f32);
    rdz.load(bdz, col, p.x_f32);
    if (POST && p.gate_kind == BIGMAC_GATE_FULL) rg.load(bg, col, p.u_f32);
    float token_gate = 1.0f;
    if (POST && p.gate_kind == BIGMAC_GATE_TOKEN && live) token_gate = ((const float*)p.gate)[at];

    float z[8], du[8], y[8];
    if (PRE) {
      rz.values(p.x_f32, z);
      rdu.values(p.y_f32, du);
    }
    if (POST) ry.values(p.y_f32, y);
    float mean_a = 0.0f;
    if (p.layer) {   // means first: of z, of du w_pre, of y
      float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (PRE) s[0] += z[i], s[1] = fmaf(du[i], qw[i], s[1]);
        if (POST) s[2] += y[i];
      }
      row_sums<W, 3, S::SLOTS>(s, box, turn, slot, wir, lane);
      mean_a = s[1] * p.inv_d;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (PRE) z[i] = in_row * (z[i] - s[0] * p.inv_d);
        if (POST) y[i] = in_row * (y[i] - s[2] * p.inv_d);
      }
    }
    float s[3] = {0.0f, 0.0f, 0.0f};   // sums of squares of z and y, of du w_pre z
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (PRE) s[0] = fmaf(z[i], z[i], s[0]), s[1] = fmaf(du[i] * qw[i], z[i], s[1]);
      if (POST) s[2] = fmaf(y[i], y[i], s[2]);
    }
    row_sums<W, 3, S::SLOTS>(s, box, turn, slot, wir, lane);
    float dZ[8];
    {
      const float r = PRE && live ? 1.0f / sqrtf(fmaf(s[0], p.inv_d, p.eps)) : 0.0f;   // (no row: nothing that an eps of 0 makes infinite)
      const float c = s[1] * r * p.inv_d;   // mean(a z^)
      const auto bdx = buffer(p.dx, p.x_f32);
      rdz.values(p.x_f32, dZ);
      float out[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (PRE) {
          const float zh = z[i] * r;
          dZ[i] = fmaf(r, du[i] * qw[i] - mean_a - zh * c, dZ[i]);
          sum[AT_PRE][i] = fmaf(du[i], zh, sum[AT_PRE][i]);
          if (BIAS) sum[AT_BIAS][i] += du[i];
        }
        if (!live) dZ[i] = 0.0f;   // (no row: adds nothing to the sums, whatever the weights hold)
        out[i] = p.alpha * dZ[i];
      }
      store8(bdx, col, p.x_f32, out);
    }
    if (POST) {
      const float r = live ? 1.0f / sqrtf(fmaf(s[2], p.inv_d, p.eps)) : 0.0f;
      const auto bdg = buffer(p.gate_kind == BIGMAC_GATE_FULL ? p.dgate : nullptr, p.u_f32);
      float q[3] = {0.0f, 0.0f, 0.0f};   // sums of e, of e y^, of dZ n(y);  e = dn w_post
      float b[8];
      if (BIAS) load_vector(p.post_b, p.d, col, 0.0f, b);
      float g[8], dg[8];
      if (p.gate_kind == BIGMAC_GATE_FULL) rg.values(p.u_f32, g);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[i] *= r;
        const float n = BIAS ? fmaf(pw[i], y[i], b[i]) : pw[i] * y[i];
        dg[i] = in_row * (dZ[i] * n);
        q[2] += dg[i];
        const float gate = p.gate_kind == BIGMAC_GATE_FULL ? g[i] : cg[i] * token_gate;
        const float dn = gate * dZ[i];
        const float counted = p.gate_kind == BIGMAC_GATE_CHANNEL ? dZ[i] : dn;
        sum[AT_POST][i] = fmaf(counted, y[i], sum[AT_POST][i]);
        if (BIAS) sum[AT_BIAS + (PRE ? 1 : 0)][i] += counted;
        const float e = in_row * (dn * pw[i]);
        dZ[i] = e;
        q[0] += e;
        q[1] = fmaf(e, y[i], q[1]);
      }
      if (p.gate_kind == BIGMAC_GATE_FULL) store8(bdg, col, p.u_f32, dg);
      row_sums<W, 3, S::SLOTS>(q, box, turn, slot, wir, lane);
      if (p.gate_kind == BIGMAC_GATE_TOKEN && live && wir == 0 && lane == 0) ((float*)p.dgate)[row] = q[2];
      const float mean_e = p.layer ? q[0] * p.inv_d : 0.0f, c = q[1] * p.inv_d;
      const auto bdy = buffer(p.dy, p.u_f32);
      float out[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] = r * (dZ[i] - mean_e - y[i] * c);
      store8(bdy, col, p.u_f32, out);
    }
  }
  // the workgroup's sums: the other slots' added to the first slot's in their order
#pragma unroll
  for (int k = 0; k < VECTORS; ++k) {
    float* f = sum[k];
    if (S::SLOTS > 1) {
      const int mine = wir * 64 + lane;
      __syncthreads();
      if (slot > 0) {
        float4* to = join + ((slot - 1) * W * 64 + mine) * 2;
        to[0] = make_float4(f[0], f[1], f[2], f[3]);
        to[1] = make_float4(f[4], f[5], f[6], f[7]);
      }
      __syncthreads();
      if (slot == 0)
#pragma unroll
        for (int o = 0; o < S::SLOTS - 1; ++o) {
          const float4 a = join[(o * W * 64 + mine) * 2], c = join[(o * W * 64 + mine) * 2 + 1];
          f[0] += a.x; f[1] += a.y; f[2] += a.z; f[3] += a.w;
          f[4] += c.x; f[5] += c.y; f[6] += c.z; f[7] += c.w;
        }
    }
    if (slot == 0 && col < p.d) {
      float4* to = (float4*)(p.part + ((size_t)blockIdx.x * VECTORS + k) * p.d + col);
      to[0] = make_float4(f[0], f[1], f[2], f[3]);
      to[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
  }
}

// The workgroups' sums of a vector, 16 columns per workgroup: 64 groups of threads each add every 64th workgroup's, 4 columns a thread,
// then the groups' are added in order, four and four and then sixteen.  (64 columns per workgroup: 16 x 2 of them at 1024 columns, 13.8 us.)
struct NormReduce {
  const float* part;
  const float *post_w, *post_b, *channel_gate;   // channel gate: NULL if the gate is none
  float *d_pre_w, *d_pre_b, *d_post_w, *d_post_b, *d_gate;
  int workgroups, vectors, d, pre, post, beta;
};
__global__ __launch_bounds__(256) void norm_reduce_kernel(NormReduce p) {
  __shared__ float4 box[2][64][4];
  __shared__ float fours[2][16][16];
  const int quad = threadIdx.x & 3, group = threadIdx.x >> 2;
  const int col = blockIdx.x * 16 + quad * 4;
  const bool post = p.pre ? blockIdx.y == 1 : true;      // which side's vectors
  const bool bias = p.vectors == 2 * (p.pre + p.post);
  const int k0 = post && p.pre ? 1 : 0, k1 = p.pre + p.post + k0;
  float4 s0 = make_float4(0.f, 0.f, 0.f, 0.f), s1 = s0;
  if (col < p.d)
#pragma unroll 4
    for (int g = group; g < p.workgroups; g += 64) {
      const float4 a = *(const float4*)(p.part + ((size_t)g * p.vectors + k0) * p.d + col);
      s0.x += a.x; s0.y += a.y; s0.z += a.z; s0.w += a.w;
      if (bias) {
        const float4 b = *(const float4*)(p.part + ((size_t)g * p.vectors + k1) * p.d + col);
        s1.x += b.x; s1.y += b.y; s1.z += b.z; s1.w += b.w;
      }
    }
  box[0][group][quad] = s0;
  box[1][group][quad] = s1;
  __syncthreads();
  const int c = threadIdx.x & 15, part = threadIdx.x >> 4;   // one column a thread from here on
#pragma unroll
  for (int v = 0; v < 2; ++v) {
    float t = 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) t += ((const float*)box[v][part * 4 + g])[c];
    fours[v][part][c] = t;
  }
  __syncthreads();
  if (part > 0 || blockIdx.x * 16 + c >= p.d) return;
  float t0 = 0.0f, t1 = 0.0f;
#pragma unroll
  for (int g = 0; g < 16; ++g) {
    t0 += fours[0][g][c];
    t1 += fours[1][g][c];
  }
  const int n = blockIdx.x * 16 + c;
  auto put = [&](float* to, float v) { if (to) to[n] = p.beta ? to[n] + v : v; };
  if (!post) {
    put(p.d_pre_w, t0);
    put(p.d_pre_b, t1);
    return;
  }
  const float g = p.channel_gate ? p.channel_gate[n] : 1.0f;
  put(p.d_post_w, g * t0);
  put(p.d_post_b, g * t1);
  if (p.channel_gate) {
    const float w = p.post_w ? p.post_w[n] : 1.0f;
    put(p.d_gate, p.post_b ? fmaf(w, t0, p.post_b[n] * t1) : w * t0);
  }
}

int check_norm(const bigmac_norm_dims* D) {
  if (!D) return BIGMAC_ERR_INVALID_ARG;
  if (D->T < 1 || D->d < 8 || D->d % 8) return BIGMAC_ERR_INVALID_ARG;
  for (int t : {D->x_dtype, D->y_dtype, D->u_dtype})
    if (t != BIGMAC_F32 && t != BIGMAC_BF16) return BIGMAC_ERR_INVALID_ARG;
  if (D->kind != BIGMAC_NORM_RMS && D->kind != BIGMAC_NORM_LAYER) return BIGMAC_ERR_INVALID_ARG;
  if (D->parts & ~(BIGMAC_NORM_PRE | BIGMAC_NORM_POST | BIGMAC_NORM_ACCUMULATE) || !(D->parts & (BIGMAC_NORM_PRE | BIGMAC_NORM_POST))) return BIGMAC_ERR_INVALID_ARG;
  if (D->gate < BIGMAC_GATE_NONE || D->gate > BIGMAC_GATE_FULL) return BIGMAC_ERR_INVALID_ARG;
  if (D->gate != BIGMAC_GATE_NONE && !(D->parts & BIGMAC_NORM_POST)) return BIGMAC_ERR_INVALID_ARG;
  if (!(D->eps >= 0.0f) || !std::isfinite(D->eps) || !std::isfinite(D->alpha)) return BIGMAC_ERR_INVALID_ARG;
  if (!(D->parts & BIGMAC_NORM_POST) && D->alpha != 1.0f) return BIGMAC_ERR_INVALID_ARG;
  if (D->d > 8192 || D->T > 1 << 30) return BIGMAC_ERR_TOO_LARGE;
  return BIGMAC_OK;
}
bool aligned(std::initializer_list<const void*> ps) {
  for (const void* q : ps)
    if ((size_t)q & 15) return false;
  return true;
}
int check_params(const bigmac_norm_dims& D, const bigmac_norm_params* P) {
  if (!P) return BIGMAC_ERR_INVALID_ARG;
  const bool post = D.parts & BIGMAC_NORM_POST, pre = D.parts & BIGMAC_NORM_PRE;
  if (post != (P->post_w != nullptr) || pre != (P->pre_w != nullptr)) return BIGMAC_ERR_INVALID_ARG;
  if ((P->post_b && !post) || (P->pre_b && !pre)) return BIGMAC_ERR_INVALID_ARG;
  if ((D.gate != BIGMAC_GATE_NONE) != (P->gate != nullptr)) return BIGMAC_ERR_INVALID_ARG;
  return aligned({P->post_w, P->post_b, P->pre_w, P->pre_b, P->gate}) ? BIGMAC_OK : BIGMAC_ERR_INVALID_ARG;
}
// wavefronts per row: a lane holds 8 columns
int waves_per_row(int d) {
  int w = 1;
  while (w * 512 < d) w *= 2;
  return w;
}
constexpr int BACKWARD_WORKGROUPS = 512;
int backward_workgroups(const bigmac_norm_dims& D) {
  const int w = waves_per_row(D.d), slots = w < 4 ? 4 / w : 1;
  // at least four rows a slot: a workgroup's sums are written and read once more, and cost as much as about two rows
  const int wanted = (D.T + 4 * slots - 1) / (4 * slots);
  return std::min(wanted, BACKWARD_WORKGROUPS);
}
int bias_vectors(const bigmac_norm_params& P) { return P.post_b || P.pre_b ? 2 : 1; }

NormArgs norm_args(const bigmac_norm_dims& D, const bigmac_norm_params& P) {
  NormArgs a{};
  a.gate = P.gate;
  a.post_w = P.post_w; a.post_b = P.post_b; a.pre_w = P.pre_w; a.pre_b = P.pre_b;
  a.T = D.T; a.d = D.d;
  a.x_f32 = D.x_dtype == BIGMAC_F32; a.y_f32 = D.y_dtype == BIGMAC_F32; a.u_f32 = D.u_dtype == BIGMAC_F32;
  a.layer = D.kind == BIGMAC_NORM_LAYER;
  a.gate_kind = D.gate;
  a.eps = D.eps; a.alpha = D.alpha; a.inv_d = 1.0f / (float)D.d;
  return a;
}

template <int W>
void forward_of(const NormArgs& a, bool post, bool pre, hipStream_t s) {
  using S = RowShape<W>;
  // a persistent grid of what the chip holds: eight workgroups of 256 threads a CU
  const int grid = std::min((a.T + S::SLOTS - 1) / S::SLOTS, 256 * 32 / S::WAVES);
  if (post && pre) norm_forward_kernel<W, true, true><<<grid, S::THREADS, 0, s>>>(a);
  else if (post) norm_forward_kernel<W, true, false><<<grid, S::THREADS, 0, s>>>(a);
  else norm_forward_kernel<W, false, true><<<grid, S::THREADS, 0, s>>>(a);
}
template <int W>
void backward_of(const NormArgs& a, bool post, bool pre, bool bias, int grid, hipStream_t s) {
  constexpr int THREADS = RowShape<W>::THREADS;
  if (bias) {
    if (post && pre) norm_backward_kernel<W, true, true, true><<<grid, THREADS, 0, s>>>(a);
    else if (post) norm_backward_kernel<W, true, false, true><<<grid, THREADS, 0, s>>>(a);
    else norm_backward_kernel<W, false, true, true><<<grid, THREADS, 0, s>>>(a);
  } else {
    if (post && pre) norm_backward_kernel<W, true, true, false><<<grid, THREADS, 0, s>>>(a);
    else if (post) norm_backward_kernel<W, true, false, false><<<grid, THREADS, 0, s>>>(a);
    else norm_backward_kernel<W, false, true, false><<<grid, THREADS, 0, s>>>(a);
  }
}

}  // namespace

}  // namespace bigmac

using namespace bigmac;

extern "C" {

size_t bigmac_norm_workspace_bytes(const bigmac_norm_dims* D) {
  if (check_norm(D) != BIGMAC_OK) return 0;
  const size_t sides = (D->parts & BIGMAC_NORM_POST ? 1 : 0) + (D->parts & BIGMAC_NORM_PRE ? 1 : 0);
  return align_up((size_t)backward_workgroups(*D) * sides * 2 * D->d * 4);
}

int bigmac_norm_forward(const bigmac_norm_dims* D, const bigmac_norm_params* P, const void* x, const void* y, void* z, void* u, void* stream) {
  int rc = check_norm(D);
  if (rc) return rc;
  rc = check_params(*D, P);
  if (rc) return rc;
  const bool post = D->parts & BIGMAC_NORM_POST, pre = D->parts & BIGMAC_NORM_PRE;
  if (!x || post != (y != nullptr) || post != (z != nullptr) || pre != (u != nullptr) || !aligned({x, y, z, u})) return BIGMAC_ERR_INVALID_ARG;
  NormArgs a = norm_args(*D, *P);
  a.x = x; a.y = y; a.z = z; a.u = u;
  hipStream_t s = (hipStream_t)stream;
  switch (waves_per_row(D->d)) {
    case 1: forward_of<1>(a, post, pre, s); break;
    case 2: forward_of<2>(a, post, pre, s); break;
    case 4: forward_of<4>(a, post, pre, s); break;
    case 8: forward_of<8>(a, post, pre, s); break;
    default: forward_of<16>(a, post, pre, s); break;
  }
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

int bigmac_norm_backward(const bigmac_norm_dims* D, const bigmac_norm_params* P, const void* z, const void* y, const void* du, const void* dz,
                         void* dx, void* dy, void* d_gate, float* d_post_w, float* d_post_b, float* d_pre_w, float* d_pre_b,
                         void* ws, size_t ws_bytes, void* stream) {
  int rc = check_norm(D);
  if (rc) return rc;
  rc = check_params(*D, P);
  if (rc) return rc;
  const bool post = D->parts & BIGMAC_NORM_POST, pre = D->parts & BIGMAC_NORM_PRE, bias = bias_vectors(*P) == 2;
  if ((!pre && !dz) || !dx || !ws) return BIGMAC_ERR_INVALID_ARG;
  if (pre != (z != nullptr) || pre != (du != nullptr) || pre != (d_pre_w != nullptr)) return BIGMAC_ERR_INVALID_ARG;
  if (post != (y != nullptr) || post != (dy != nullptr) || post != (d_post_w != nullptr)) return BIGMAC_ERR_INVALID_ARG;
  if ((P->post_b != nullptr) != (d_post_b != nullptr) || (P->pre_b != nullptr) != (d_pre_b != nullptr)) return BIGMAC_ERR_INVALID_ARG;
  if ((P->gate != nullptr) != (d_gate != nullptr)) return BIGMAC_ERR_INVALID_ARG;
  if (!aligned({z, y, du, dz, dx, dy, d_gate, d_post_w, d_post_b, d_pre_w, d_pre_b, ws})) return BIGMAC_ERR_INVALID_ARG;
  const int workgroups = backward_workgroups(*D), vectors = ((post ? 1 : 0) + (pre ? 1 : 0)) * (bias ? 2 : 1);
  if (ws_bytes < bigmac_norm_workspace_bytes(D)) return BIGMAC_ERR_WORKSPACE;
  NormArgs a = norm_args(*D, *P);
  a.x = z; a.y = y; a.du = du; a.dz = dz; a.dx = dx; a.dy = dy; a.dgate = d_gate; a.part = (float*)ws;
  hipStream_t s = (hipStream_t)stream;
  switch (waves_per_row(D->d)) {
    case 1: backward_of<1>(a, post, pre, bias, workgroups, s); break;
    case 2: backward_of<2>(a, post, pre, bias, workgroups, s); break;
    case 4: backward_of<4>(a, post, pre, bias, workgroups, s); break;
    case 8: backward_of<8>(a, post, pre, bias, workgroups, s); break;
    default: backward_of<16>(a, post, pre, bias, workgroups, s); break;
  }
  BIGMAC_CHECK_LAUNCH();
  NormReduce r{};
  r.part = a.part;
  r.post_w = P->post_w; r.post_b = P->post_b;
  r.channel_gate = D->gate == BIGMAC_GATE_CHANNEL ? (const float*)P->gate : nullptr;
  r.d_pre_w = d_pre_w; r.d_pre_b = d_pre_b; r.d_post_w = d_post_w; r.d_post_b = d_post_b;
  r.d_gate = D->gate == BIGMAC_GATE_CHANNEL ? (float*)d_gate : nullptr;
  r.workgroups = workgroups; r.vectors = vectors; r.d = D->d; r.pre = pre; r.post = post;
  r.beta = D->parts & BIGMAC_NORM_ACCUMULATE ? 1 : 0;
  norm_reduce_kernel<<<dim3((D->d + 15) / 16, (pre ? 1 : 0) + (post ? 1 : 0)), 256, 0, s>>>(r);
  BIGMAC_CHECK_LAUNCH();
  return BIGMAC_OK;
}

}  // extern "C"

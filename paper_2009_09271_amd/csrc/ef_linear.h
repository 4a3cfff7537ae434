// HIP kernels of the checkpointed linear layer (gfx950): activations kept in 8 bits, and the products that
// write and read them.
//
// A checkpoint of x [n][c] is codes [n][32 G] and one scale byte per group of 32 columns of a row, G =
// ceil(c / 32).  A group's scale is a power of two 2^e: the smallest (e >= kLeastExp) under which its largest
// magnitude still fits the code, so no value saturates and each is off by at most half a step.  Powers of two
// make the decoded value code * 2^e exact in bfloat16 (at most seven significant bits, never subnormal), so the
// matrix instructions take it as it is and a product with it rounds only where it sums.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/efsparse.h"

namespace efs {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// the same at any address that an element may have: rows of odd lengths start anywhere
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kGroup = 32;       // columns that share a scale
constexpr int kLeastExp = -100;  // smallest exponent of a group: 2^-100 times any code is a normal bfloat16

// ---------------------------------------------------------------------------------------------
// Elements: eight neighbours of a row at a time.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ float bf16_f(uint32_t lo16) { return __uint_as_float(lo16 << 16); }

// (one rounding to nearest, ties to even; a NaN stays one)
__device__ __forceinline__ uint32_t f_bf16x2(float a, float b) {
  const __bf16 x = (__bf16)a, y = (__bf16)b;
  return (uint32_t)__builtin_bit_cast(uint16_t, x) | (uint32_t)__builtin_bit_cast(uint16_t, y) << 16;
}

// v = the `cnt` (of eight) elements from p + at on; the rest 0.
template <int DT>
__device__ __forceinline__ void load8(const void* p, int64_t at, int cnt, float (&v)[8]) {
  if (DT == EF_F32) {
    const float* q = static_cast<const float*>(p) + at;
    if (cnt >= 8) {
      const u32x4 a = *reinterpret_cast<const u32x4u*>(q), b = *reinterpret_cast<const u32x4u*>(q + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = __uint_as_float(a[j]);
        v[j + 4] = __uint_as_float(b[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < cnt ? q[j] : 0.0f;
    }
  } else {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (cnt >= 8) {
      const u32x4 a = *reinterpret_cast<const u32x4u*>(q);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[2 * j] = __uint_as_float(a[j] << 16);
        v[2 * j + 1] = __uint_as_float(a[j] & 0xFFFF0000u);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < cnt ? bf16_f(q[j]) : 0.0f;
    }
  }
}

template <int DT>
__device__ __forceinline__ void store8(void* p, int64_t at, int cnt, const float (&v)[8]) {
  if (DT == EF_F32) {
    float* q = static_cast<float*>(p) + at;
    if (cnt >= 8) {
      u32x4 a, b;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = __float_as_uint(v[j]);
        b[j] = __float_as_uint(v[j + 4]);
      }
      *reinterpret_cast<u32x4u*>(q) = a;
      *reinterpret_cast<u32x4u*>(q + 4) = b;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < cnt) q[j] = v[j];
    }
  } else {
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    u32x4 a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = f_bf16x2(v[2 * j], v[2 * j + 1]);
    if (cnt >= 8) {
      *reinterpret_cast<u32x4u*>(q) = a;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < cnt) q[j] = (uint16_t)(a[j / 2] >> (16 * (j & 1)));
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Codes.
// ---------------------------------------------------------------------------------------------
// The scale byte of a group whose largest magnitude has these bits.  A group with an infinity or a NaN has
// scale byte 255 and codes 0, which decode to NaN: a step that overflowed stays visible.
__device__ __forceinline__ uint32_t group_scale(uint32_t amax, int fmt) {
  if (amax >= 0x7F800000u) return 255u;
  const int e = (int)(amax >> 23) - 127;
  const uint32_t m = amax & 0x7FFFFFu;
  // int8: largest code in [64, 127], one exponent up where 1.9921875 * 64 = 127.5 and more would round to 128;
  // e4m3: largest in (224, 448], 448 = 1.75 * 2^8
  const int x = fmt == EF_CKPT_INT8 ? e - 6 + (m >= 0x7F0000u ? 1 : 0) : e - 8 + (m > 0x600000u ? 1 : 0);
  return (uint32_t)((x < kLeastExp ? kLeastExp : x) + 127);
}

// Eight codes of a group with scale byte s, in order from the low byte of [0].
__device__ __forceinline__ u32x2 encode8(const float (&v)[8], uint32_t s, int fmt) {
  u32x2 q = {0u, 0u};
  if (s == 255u) return q;
  const float r = __uint_as_float((254u - s) << 23);  // 2^-e
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (fmt == EF_CKPT_INT8) {
      uint32_t w = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) w |= ((uint32_t)(int)rintf(v[4 * h + j] * r) & 255u) << (8 * j);
      q[h] = w;
    } else {
      int w = 0;
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * r, v[4 * h + 1] * r, w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * r, v[4 * h + 3] * r, w, true);
      q[h] = (uint32_t)w;
    }
  }
  return q;
}

__device__ __forceinline__ void decode8(u32x2 q, uint32_t s, int fmt, float (&v)[8]) {
  const float r = __uint_as_float(s << 23);  // 2^e; scale byte 255: infinity, and 0 * infinity is NaN
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (fmt == EF_CKPT_INT8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * h + j] = (float)((int32_t)(q[h] << (24 - 8 * j)) >> 24) * r;
    } else {
      const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], false);
      const auto b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[h], true);
      v[4 * h] = a[0] * r;
      v[4 * h + 1] = a[1] * r;
      v[4 * h + 2] = b[0] * r;
      v[4 * h + 3] = b[1] * r;
    }
  }
}

// The largest magnitude bits over the four lanes (eight columns each) that hold a group.
__device__ __forceinline__ uint32_t group_amax(const float (&v)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(v[j]) & 0x7FFFFFFFu);
  m = max(m, (uint32_t)__shfl_xor((int)m, 1));
  return max(m, (uint32_t)__shfl_xor((int)m, 2));
}

// ---------------------------------------------------------------------------------------------
// Activations, in float32.
// ---------------------------------------------------------------------------------------------
constexpr float kGeluA = 0.7978845608028654f;  // sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

__device__ __forceinline__ float act_value(float z, int act) {
  switch (act) {
    case EF_ACT_RELU: return z < 0.0f ? 0.0f : z;  // (a NaN stays one)
    case EF_ACT_GELU: return 0.5f * z * erfcf(-0.70710678118654752f * z);
    case EF_ACT_GELU_TANH: return z / (1.0f + expf(-2.0f * kGeluA * (z + kGeluB * z * z * z)));
    case EF_ACT_SILU: return z / (1.0f + expf(-z));
    default: return z;
  }
}

// The derivative.  Far out, where it is 0 or 1 to float32, z is held at a bound: no product there overflows.
__device__ __forceinline__ float act_slope(float z, int act) {
  switch (act) {
    case EF_ACT_RELU: return z > 0.0f ? 1.0f : (z <= 0.0f ? 0.0f : z);
    case EF_ACT_GELU: {
      z = z > 16.0f ? 16.0f : (z < -16.0f ? -16.0f : z);
      return 0.5f * erfcf(-0.70710678118654752f * z) + z * 0.3989422804014327f * expf(-0.5f * z * z);
    }
    case EF_ACT_GELU_TANH: {
      z = z > 16.0f ? 16.0f : (z < -16.0f ? -16.0f : z);
      const float t = expf(-2.0f * kGeluA * (z + kGeluB * z * z * z)), p = 1.0f / (1.0f + t);
      const float q = t > 1e30f ? 1.0f : t * p;  // 1 - p
      return p + z * p * q * (2.0f * kGeluA) * (1.0f + 3.0f * kGeluB * z * z);
    }
    case EF_ACT_SILU: {
      z = z > 128.0f ? 128.0f : (z < -128.0f ? -128.0f : z);
      const float t = expf(-z), p = 1.0f / (1.0f + t);
      const float q = t > 1e30f ? 1.0f : t * p;
      return p + z * p * q;
    }
    default: return 1.0f;
  }
}

// ---------------------------------------------------------------------------------------------
// The elementwise passes.  Four neighbouring lanes hold a group of 32 columns; a workgroup of 256 lanes is
// `tx` lanes wide (a power of two, enough for a row where that is at most 256) and 256 / tx rows high.
// ---------------------------------------------------------------------------------------------
struct Kept {
  uint8_t* codes;   // [rows][32 G]
  uint8_t* scales;  // [rows][G]
  int32_t G;
  int32_t fmt;
};

template <int DT>
__global__ __launch_bounds__(256) void k_ckpt_pack(int64_t n, int32_t c, const void* x, int64_t ldx, Kept k, int txs) {
  const int tx = threadIdx.x & ((1 << txs) - 1), ty = threadIdx.x >> txs;
  const int64_t row = (int64_t)blockIdx.x * (256 >> txs) + ty;
  const int32_t col = ((int32_t)(blockIdx.y << txs) + tx) * 8;
  if (row >= n || col >= k.G * kGroup) return;  // (whole groups: 4 lanes, 32 columns)
  float v[8];
  load8<DT>(x, row * ldx + col, c - col, v);
  const uint32_t s = group_scale(group_amax(v), k.fmt);
  *reinterpret_cast<u32x2u*>(k.codes + row * k.G * kGroup + col) = encode8(v, s, k.fmt);
  if ((col & (kGroup - 1)) == 0) k.scales[row * k.G + col / kGroup] = (uint8_t)s;
}

template <int DT>
__global__ __launch_bounds__(256) void k_ckpt_unpack(int64_t n, int32_t c, Kept k, void* y, int64_t ldy, int txs) {
  const int tx = threadIdx.x & ((1 << txs) - 1), ty = threadIdx.x >> txs;
  const int64_t row = (int64_t)blockIdx.x * (256 >> txs) + ty;
  const int32_t col = ((int32_t)(blockIdx.y << txs) + tx) * 8;
  if (row >= n || col >= c) return;
  float v[8];
  decode8(*reinterpret_cast<const u32x2u*>(k.codes + row * k.G * kGroup + col), k.scales[row * k.G + col / kGroup],
          k.fmt, v);
  store8<DT>(y, row * ldy + col, c - col, v);
}

// dz = dy * act'(x^), rounded once.
template <int DT>
__global__ __launch_bounds__(256) void k_ckpt_act_backward(int64_t n, int32_t c, int act, Kept k, const void* dy,
                                                           int64_t lddy, void* dz, int64_t lddz, int txs) {
  const int tx = threadIdx.x & ((1 << txs) - 1), ty = threadIdx.x >> txs;
  const int64_t row = (int64_t)blockIdx.x * (256 >> txs) + ty;
  const int32_t col = ((int32_t)(blockIdx.y << txs) + tx) * 8;
  if (row >= n || col >= c) return;
  float v[8], z[8];
  load8<DT>(dy, row * lddy + col, c - col, v);
  decode8(*reinterpret_cast<const u32x2u*>(k.codes + row * k.G * kGroup + col), k.scales[row * k.G + col / kGroup],
          k.fmt, z);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] *= act_slope(z[j], act);
  store8<DT>(dz, row * lddz + col, c - col, v);
}

// ---------------------------------------------------------------------------------------------
// The products' epilogue: eight columns of a row of C in float32, four neighbouring lanes a group.
// ---------------------------------------------------------------------------------------------
enum : int { K_FWD = 0, K_DGRAD = 1, K_WGRAD = 2 };

struct Epi {
  void* out;          // y / dx / dw
  int64_t ldo;
  const void* bias;   // forward: [N], or null
  const void* res;    // forward, dgrad: added last, or null
  int64_t ldr;
  Kept k;             // forward: written where codes is not null; dgrad: read where act is not EF_ACT_NONE
  int32_t act;
  int32_t add;        // wgrad: dw += product
};

// KIND the product, DT the type of out, bias and res.
template <int KIND, int DT>
__device__ __forceinline__ void epilogue8(const Epi& a, int64_t row, int32_t col, bool row_ok, int32_t N,
                                          float (&v)[8]) {
  const int cnt = row_ok ? N - col : 0;  // columns of this lane that exist (8 or more: all)
  if (KIND == K_FWD) {
    if (a.bias) {
      float b[8];
      load8<DT>(a.bias, col, N - col, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += b[j];
    }
    if (a.k.codes) {  // (every lane of a group takes part)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < cnt ? v[j] : 0.0f;
      const uint32_t s = group_scale(group_amax(v), a.k.fmt);
      if (row_ok && col < a.k.G * kGroup) {
        *reinterpret_cast<u32x2u*>(a.k.codes + row * a.k.G * kGroup + col) = encode8(v, s, a.k.fmt);
        if ((col & (kGroup - 1)) == 0) a.k.scales[row * a.k.G + col / kGroup] = (uint8_t)s;
      }
    }
    if (a.act != EF_ACT_NONE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = act_value(v[j], a.act);
    }
  }
  if (cnt <= 0) return;
  if (KIND == K_DGRAD && a.act != EF_ACT_NONE) {
    float z[8];
    decode8(*reinterpret_cast<const u32x2u*>(a.k.codes + row * a.k.G * kGroup + col),
            a.k.scales[row * a.k.G + col / kGroup], a.k.fmt, z);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= act_slope(z[j], a.act);
  }
  if (KIND != K_WGRAD && a.res) {
    float r[8];
    load8<DT>(a.res, row * a.ldr + col, cnt, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += r[j];
  }
  if (KIND == K_WGRAD && a.add) {
    float r[8];
    load8<DT>(a.out, row * a.ldo + col, cnt, r);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = r[j] + v[j];
  }
  store8<DT>(a.out, row * a.ldo + col, cnt, v);
}

// ---------------------------------------------------------------------------------------------
// The product for every type, order and alignment, in float32: C[m][n] = sum_k A(m, k) B(n, k).
//   forward  A = x  [n][i] (k along the row), B = W [o][i] (k along the row)
//   dgrad    A = dy [n][o] (k along the row), B = W [o][i] (k down the rows)
//   wgrad    A = dy [t][o] (k down the rows), B = the checkpoint [t][i] (k down the rows)
// A workgroup has 128 x 128 of C, four wavefronts 64 x 64 each, and steps of 16 along k: the tiles of the next
// step are loaded into registers while this one is multiplied, and stored to the other half of the LDS as
// float32 [k][m], whatever the order in memory.
// ---------------------------------------------------------------------------------------------
struct Mat {
  const void* p;
  int64_t ld;
};

constexpr int kAnyTile = 128, kAnyK = 16, kAnyPitch = 132;  // (132: rows eight apart land 32 banks apart)
constexpr int kSlabPitch = 68;  // epilogue: a wavefront's 32 x 64 floats

// Eight elements along the contiguous direction of a tile of A or B: ROWS of the matrix down, 8 columns across.
template <int DT>
__device__ __forceinline__ void load_chunk(const Mat& a, int64_t row, int64_t rows, int64_t col, int64_t cols, float (&v)[8]) {
  const int64_t left = cols - col;
  load8<DT>(a.p, row * a.ld + col, row < rows ? (int)(left < 8 ? left : 8) : 0, v);
}

template <int KIND, int DT, int DO>
__global__ __launch_bounds__(256) void k_linear_any(int32_t M, int32_t N, int32_t K, Mat A, Mat B, Kept BK, Epi ep) {
  constexpr bool AKC = KIND != K_WGRAD, BKC = KIND == K_FWD, B8 = KIND == K_WGRAD;
  constexpr int kTileF = kAnyK * kAnyPitch;
  __shared__ __align__(16) float sm[4 * 32 * kSlabPitch > 4 * kTileF ? 4 * 32 * kSlabPitch : 4 * kTileF];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int32_t tn = (N + kAnyTile - 1) / kAnyTile;
  const int64_t m0 = (int64_t)(blockIdx.x / tn) * kAnyTile, n0 = (int64_t)(blockIdx.x % tn) * kAnyTile;
  const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  float av[8], bv[8];
  // tile element of this thread's chunk: (line, 8 along k) or (k, 8 along the line)
  const int kc_l = t >> 1, kc_k = (t & 1) * 8, ks_k = t >> 4, ks_l = (t & 15) * 8;
  auto fetch = [&](int64_t k0) {
    if (AKC) load_chunk<DT>(A, m0 + kc_l, M, k0 + kc_k, K, av);
    else load_chunk<DT>(A, k0 + ks_k, K, m0 + ks_l, M, av);
    if (B8) {
      const int64_t row = k0 + ks_k, col = n0 + ks_l;
#pragma unroll
      for (int j = 0; j < 8; ++j) bv[j] = 0.0f;
      if (row < K && col < N)
        decode8(*reinterpret_cast<const u32x2u*>(BK.codes + row * BK.G * kGroup + col),
                BK.scales[row * BK.G + col / kGroup], BK.fmt, bv);
    } else if (BKC) {
      load_chunk<DT>(B, n0 + kc_l, N, k0 + kc_k, K, bv);
    } else {
      load_chunk<DT>(B, k0 + ks_k, K, n0 + ks_l, N, bv);
    }
  };
  auto put = [&](float* s, bool kc, const float (&v)[8]) {
    if (kc) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s[(kc_k + j) * kAnyPitch + kc_l] = v[j];
    } else {
      *reinterpret_cast<f32x4*>(s + ks_k * kAnyPitch + ks_l) = f32x4{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<f32x4*>(s + ks_k * kAnyPitch + ks_l + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
  };
  f32x16 acc[2][2];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;
  const int steps = (int)(((int64_t)K + kAnyK - 1) / kAnyK);
  if (steps) fetch(0);
  for (int s = 0; s < steps; ++s) {
    float* sa = sm + (s & 1) * 2 * kTileF;
    float* sb = sa + kTileF;
    put(sa, AKC, av);
    put(sb, BKC, bv);
    __syncthreads();  // (the other half was last read before the previous barrier's step ended)
    if (s + 1 < steps) fetch((int64_t)(s + 1) * kAnyK);
#pragma unroll
    for (int k = 0; k < kAnyK; k += 2) {
      const int row = (k + (lane >> 5)) * kAnyPitch + (lane & 31);
      const float a0 = sa[row + wm], a1 = sa[row + wm + 32], b0 = sb[row + wn], b1 = sb[row + wn + 32];
      acc[0][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a0, b0, acc[0][0], 0, 0, 0);
      acc[0][1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a0, b1, acc[0][1], 0, 0, 0);
      acc[1][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a1, b0, acc[1][0], 0, 0, 0);
      acc[1][1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a1, b1, acc[1][1], 0, 0, 0);
    }
  }
  __syncthreads();
  // a wavefront's 64 x 64 through its own part of the LDS, 32 rows at a time: lanes that hold single columns
  // (four rows each) hand over to lanes that hold eight columns of a row
  float* slab = sm + wave * 32 * kSlabPitch;
#pragma unroll
  for (int a = 0; a < 2; ++a) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        slab[((r >> 2) * 8 + (lane >> 5) * 4 + (r & 3)) * kSlabPitch + b * 32 + (lane & 31)] = acc[a][b][r];
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int rr = q * 8 + (lane >> 3), cc = (lane & 7) * 8;
      const f32x4 lo = *reinterpret_cast<const f32x4*>(slab + rr * kSlabPitch + cc);
      const f32x4 hi = *reinterpret_cast<const f32x4*>(slab + rr * kSlabPitch + cc + 4);
      float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      const int64_t row = m0 + wm + a * 32 + rr;
      epilogue8<KIND, DO>(ep, row, (int32_t)(n0 + wn + cc), row < M, N, v);
    }
    __syncthreads();
  }
}

// The bias gradient: db[o] (+)= sum over the rows of dy[., o], in float32: a workgroup has 32 columns, eight
// lanes down, each lane's rows in order, the eight sums in order.
template <int DT, int DO>
__global__ __launch_bounds__(256) void k_bias_grad(int64_t n, int32_t o, const void* dy, int64_t ld, void* db, int add) {
  __shared__ float part[8][32];
  const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
  const int64_t col = (int64_t)blockIdx.x * 32 + c;
  float s = 0.0f;
  if (col < o)
    for (int64_t row = r; row < n; row += 8)
      s += DT == EF_F32 ? static_cast<const float*>(dy)[row * ld + col]
                        : bf16_f(static_cast<const uint16_t*>(dy)[row * ld + col]);
  part[r][c] = s;
  __syncthreads();
  if (r == 0 && col < o) {
#pragma unroll
    for (int j = 1; j < 8; ++j) s += part[j][c];
    if (DO == EF_F32) {
      float* q = static_cast<float*>(db) + col;
      *q = add ? *q + s : s;
    } else {
      static_cast<uint16_t*>(db)[col] = (uint16_t)f_bf16x2(s, 0.0f);
    }
  }
}

}  // namespace efs

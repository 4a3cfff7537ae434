// HIP kernels of the checkpointed linear layer (gfx950): activations kept in 8 bits, and the products that
// write and read them.
//
// A checkpoint of x [n][c] is codes [n][32 G] and one scale byte per group of 32 columns of a row, G =
// ceil(c / 32).  A group's scale is a power of two 2^e: the smallest (e >= kLeastExp) under which its largest
// magnitude still fits the code, so each value is off by at most half a step (values that would round to 2^128 are held at
// the largest finite code, off by less than a step).  Powers of two
// make the decoded value code * 2^e exact in bfloat16 (at most seven significant bits, never subnormal), so the
// matrix instructions take it as it is and a product with it rounds only where it sums.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/efsparse.h"

namespace efs {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// the same at any address that an element may have: rows of odd lengths start anywhere
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kGroup = 32;       // columns that share a scale
constexpr int kLeastExp = -100;  // smallest exponent of a group: 2^-100 times any code is a normal bfloat16
// scale byte of the highest exponent of a group of finite values (122, 120), under which the codes 64 and 256 would stand for
// 2^128, and the largest magnitude below, 63 * 2^122 and 240 * 2^120
constexpr uint32_t kTopInt8 = 249, kTopE4m3 = 247;
constexpr float kMostInt8 = 0x1.F8p127f, kMostE4m3 = 0x1.Ep127f;

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

// ONCE: past the caches
template <bool ONCE>
__device__ __forceinline__ void store16(u32x4 a, void* p) {
  if (ONCE) __builtin_nontemporal_store(a, static_cast<u32x4u*>(p));
  else *static_cast<u32x4u*>(p) = a;
}

template <int DT, bool ONCE = false>
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
      store16<ONCE>(a, q);
      store16<ONCE>(b, q + 4);
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
      store16<ONCE>(a, q);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < cnt) q[j] = (uint16_t)(a[j / 2] >> (16 * (j & 1)));
    }
  }
}

// Eight neighbours of a row as they are stored, for loads that are used later.
template <int DT>
struct Raw {
  static constexpr int W = DT == EF_F32 ? 8 : 4;
  uint32_t r[W];

  // ONCE: past the caches
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const void* p, int64_t at, int cnt) {
    if (cnt >= 8) {
      const u32x4u* from = reinterpret_cast<const u32x4u*>(static_cast<const char*>(p) + at * (W / 2));
#pragma unroll
      for (int j = 0; j < W / 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) r[4 * j + i] = (ONCE ? __builtin_nontemporal_load(from + j) : from[j])[i];
    } else {
      float v[8];
      load8<DT>(p, at, cnt, v);
#pragma unroll
      for (int j = 0; j < W; ++j) r[j] = DT == EF_F32 ? __float_as_uint(v[j]) : f_bf16x2(v[2 * j % 8], v[(2 * j + 1) % 8]);
    }
  }
  __device__ __forceinline__ float value(int j) const {
    if (DT == EF_F32) return __uint_as_float(r[j % W]);
    return __uint_as_float(j & 1 ? r[j / 2 % W] & 0xFFFF0000u : r[j / 2 % W] << 16);
  }
};

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
__device__ __forceinline__ u32x2 encode8(const float (&x)[8], uint32_t s, int fmt) {
  u32x2 q = {0u, 0u};
  if (s == 255u) return q;
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = x[j];
  if (__builtin_expect(s >= kTopE4m3, 0)) {  // a finite value does not come back as an infinity
    const float most = fmt == EF_CKPT_E4M3 ? kMostE4m3 : s == kTopInt8 ? kMostInt8 : 0x1.FFFFFEp127f;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __builtin_amdgcn_fmed3f(v[j], -most, most);
  }
  const float r = __uint_as_float((254u - s) << 23);  // 2^-e
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (fmt == EF_CKPT_INT8) {
      uint32_t b[4];  // added to 1.5 * 2^23 the product is rounded to a whole number, its low byte the code
#pragma unroll
      for (int j = 0; j < 4; ++j) b[j] = __float_as_uint(fmaf(v[4 * h + j], r, 12582912.0f));
      q[h] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0C0C0400u),
                                   __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), 0x05040100u);
    } else {
      int w = 0;
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * r, v[4 * h + 1] * r, w, false);
      w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * r, v[4 * h + 3] * r, w, true);
      q[h] = (uint32_t)w;
    }
  }
  return q;
}

// The signed bytes 2 HI and 2 HI + 1 of w as floats.  (Written out: from the conversion itself the compiler keeps a whole
// step's bytes of the weight gradient apart, and spills.)
template <int HI>
__device__ __forceinline__ void bytes(uint32_t w, float* a, float* b) {
  if (HI) {
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_2" : "=v"(*a) : "v"(w));
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_3" : "=v"(*b) : "v"(w));
  } else {
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_0" : "=v"(*a) : "v"(w));
    asm("v_cvt_f32_i32_sdwa %0, sext(%1) dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:BYTE_1" : "=v"(*b) : "v"(w));
  }
}

__device__ __forceinline__ void decode8(u32x2 q, uint32_t s, int fmt, float (&v)[8]) {
  const float r = __uint_as_float(s << 23);  // 2^e; scale byte 255: infinity, and 0 * infinity is NaN
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (fmt == EF_CKPT_INT8) {
      bytes<0>(q[h], &v[4 * h], &v[4 * h + 1]);
      bytes<1>(q[h], &v[4 * h + 2], &v[4 * h + 3]);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[4 * h + j] *= r;
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
constexpr float kLog2e = 1.4426950408889634f;

// The normal distribution function, from its tail: with a = |z| and E = exp(-a^2 / 2), Phi(-a) = E Q(a), and
// Q(a) = erfcx(a / sqrt 2) / 2 as t P(t), t = 1 / (1 + 0.235 a), P the polynomial of degree 7 fitted to the least
// relative error over a <= 16 (1.2e-7; with the float32 roundings Phi is off by 2.6e-7 at most, and by 1.6e-6 of
// itself down to z = -5).  E serves the density too.  Against the math library's erfc and exp the backward pass of 16384 x 4096
// in bfloat16 went from 143 to 72 us, and to 58 with the other steps: 5.8 TB/s.
__device__ __forceinline__ float normal_cdf(float z, float* density) {
  const float a = fabsf(z), E = __builtin_amdgcn_exp2f(a * a * (-0.5f * kLog2e));
  const float t = __builtin_amdgcn_rcpf(fmaf(0.235f, a, 1.0f));
  float q = fmaf(-0.064110115f, t, 0.21003315f);
  q = fmaf(q, t, -0.1455516f);
  q = fmaf(q, t, 0.17967904f);
  q = fmaf(q, t, 0.0355675f);
  q = fmaf(q, t, 0.097955726f);
  q = fmaf(q, t, 0.092617f);
  q = fmaf(q, t, 0.09380927f);
  const float lo = E * (q * t);
  *density = E * 0.3989422804014327f;
  return z < 0.0f ? lo : 1.0f - lo;
}

// 1 / (1 + 2^t): the logistic function of u at t = -u log2 e
__device__ __forceinline__ float logistic2(float t) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t)); }

// (1 + tanh x) / 2 is the logistic function of 2 x: its t for GELU's x at z
__device__ __forceinline__ float gelu_t(float z) {
  constexpr float a = -2.0f * kGeluA * kLog2e;
  return z * fmaf(a * kGeluB * z, z, a);
}

__device__ __forceinline__ void act_value(float (&v)[8], int act) {
  float d;
  switch (act) {
    case EF_ACT_RELU:
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] < 0.0f ? 0.0f : v[j];  // (a NaN stays one)
      break;
    case EF_ACT_GELU:
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= normal_cdf(v[j], &d);
      break;
    case EF_ACT_GELU_TANH:
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= logistic2(gelu_t(v[j]));
      break;
    case EF_ACT_SILU:
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= logistic2(-kLog2e * v[j]);
      break;
  }
}

// v *= the derivative at z.  (The logistic function at -u is taken by itself: 1 minus that at u would cancel.)
__device__ __forceinline__ void act_slope(float (&v)[8], const float (&z)[8], int act) {
  switch (act) {
    case EF_ACT_RELU:
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = z[j] > 0.0f ? v[j] : v[j] * (z[j] <= 0.0f ? 0.0f : z[j]);
      break;
    case EF_ACT_GELU:
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float d;
        const float p = normal_cdf(z[j], &d);
        v[j] *= fmaf(z[j], d, p);
      }
      break;
    case EF_ACT_GELU_TANH:
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        // (held where the derivative is 0 or 1 to float32: the square of a larger z could overflow; a NaN comes back in)
        const float x = __builtin_amdgcn_fmed3f(z[j], -16.0f, 16.0f), t = gelu_t(x), p = logistic2(t), q = logistic2(-t);
        v[j] *= fmaf(x * p * q, 2.0f * kGeluA * fmaf(3.0f * kGeluB * x, x, 1.0f), fmaf(z[j], 0.0f, p));
      }
      break;
    case EF_ACT_SILU:
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float p = logistic2(-kLog2e * z[j]), q = logistic2(kLog2e * z[j]);
        v[j] *= fmaf(z[j] * p, q, p);
      }
      break;
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

// What is read once and by nobody else goes past the caches (16384 x 4096 in bfloat16: pack 42 -> 34 us, unpack 34 -> 31;
// two or four rows a lane: 46 and 49 us); so does what act_backward writes (67 -> 65).
template <int DT>
__global__ __launch_bounds__(256) void k_ckpt_pack(int64_t n, int32_t c, const void* x, int64_t ldx, Kept k, int txs) {
  const int tx = threadIdx.x & ((1 << txs) - 1), ty = threadIdx.x >> txs;
  const int64_t row = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * (256 >> txs) + ty;
  const int32_t col = ((int32_t)(blockIdx.y << txs) + tx) * 8;
  if (row >= n || col >= k.G * kGroup) return;  // (whole groups: 4 lanes, 32 columns)
  Raw<DT> raw;
  raw.template load<true>(x, row * ldx + col, c - col);
  float v[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = raw.value(j);
  const uint32_t s = group_scale(group_amax(v), k.fmt);
  *reinterpret_cast<u32x2*>(k.codes + row * k.G * kGroup + col) = encode8(v, s, k.fmt);
  if ((col & (kGroup - 1)) == 0) k.scales[row * k.G + col / kGroup] = (uint8_t)s;
}

// ACT: y = dy * act'(x^), rounded once (y may be dy); else y = x^.
template <int DT, bool ACT>
__global__ __launch_bounds__(256) void k_ckpt_unpack(int64_t n, int32_t c, int act, Kept k, const void* dy, int64_t lddy, void* y,
                                                     int64_t ldy, int txs) {
  const int tx = threadIdx.x & ((1 << txs) - 1), ty = threadIdx.x >> txs;
  const int64_t row = ((int64_t)blockIdx.z * gridDim.x + blockIdx.x) * (256 >> txs) + ty;
  const int32_t col = ((int32_t)(blockIdx.y << txs) + tx) * 8;
  if (row >= n || col >= c) return;
  const u32x2* from = reinterpret_cast<const u32x2*>(k.codes + row * k.G * kGroup + col);
  const u32x2 q = ACT ? *from : __builtin_nontemporal_load(from);
  const uint32_t s = k.scales[row * k.G + col / kGroup];
  float v[8], z[8];
  Raw<DT> raw;
  if (ACT) raw.load(dy, row * lddy + col, c - col);
  decode8(q, s, k.fmt, z);
  if (ACT) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = raw.value(j);
    act_slope(v, z, act);
  }
  store8<DT, ACT>(y, row * ldy + col, c - col, ACT ? v : z);
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
  int32_t add;        // wgrad: dw += product, db += sum
  void* db;           // wgrad: [M], the sums of A's lines, or null
};

// What the epilogue reads beside C for eight columns of a row, loaded ahead of its use; KIND the product, DT the type
// of out, bias and res.
template <int KIND, int DT>
struct Side {
  Raw<DT> old;  // res, or the old dw
  u32x2 q;      // dgrad: the kept codes and their scale
  uint32_t s;

  // cnt of the eight columns exist (8 or more: all; 0 or less: none)
  __device__ __forceinline__ void load(const Epi& a, int64_t row, int32_t col, int cnt) {
    if (cnt <= 0) return;
    if (KIND == K_DGRAD && a.act != EF_ACT_NONE) {
      q = *reinterpret_cast<const u32x2*>(a.k.codes + row * a.k.G * kGroup + col);
      s = a.k.scales[row * a.k.G + col / kGroup];
    }
    if (KIND == K_WGRAD) {
      if (a.add) old.load(a.out, row * a.ldo + col, cnt);
    } else if (a.res) {
      old.load(a.res, row * a.ldr + col, cnt);
    }
  }
};

template <int KIND, int DT>
__device__ __forceinline__ void load_bias(const Epi& a, int32_t col, int32_t N, float (&b)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) b[j] = 0.0f;
  if (KIND == K_FWD && a.bias) load8<DT>(a.bias, col, N - col, b);
}

// Four neighbouring lanes hold a group of 32 columns and call this together.
template <int KIND, int DT>
__device__ __forceinline__ void epilogue8(const Epi& a, int64_t row, int32_t col, int cnt, float (&v)[8], const float (&b)[8],
                                          const Side<KIND, DT>& side) {
  if (KIND == K_FWD) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += b[j];
    if (a.k.codes) {
      if (cnt < 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < cnt ? v[j] : 0.0f;
      const uint32_t s = group_scale(group_amax(v), a.k.fmt);
      if (cnt > -kGroup && col < a.k.G * kGroup) {  // (the group's columns behind the last one: code 0)
        *reinterpret_cast<u32x2*>(a.k.codes + row * a.k.G * kGroup + col) = encode8(v, s, a.k.fmt);
        if ((col & (kGroup - 1)) == 0) a.k.scales[row * a.k.G + col / kGroup] = (uint8_t)s;
      }
    }
    act_value(v, a.act);
  }
  if (cnt <= 0) return;
  if (KIND == K_DGRAD && a.act != EF_ACT_NONE) {
    float z[8];
    decode8(side.q, side.s, a.k.fmt, z);
    act_slope(v, z, a.act);
  }
  if (KIND == K_WGRAD ? a.add != 0 : a.res != nullptr) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = side.old.value(j) + v[j];
  }
  store8<DT>(a.out, row * a.ldo + col, cnt, v);
}

// No column of this row: less than any distance to the last column's group.
constexpr int kNoRow = -0x40000000;

template <int DO>
__device__ __forceinline__ void store_db(const Epi& a, int64_t m, float s) {
  if (DO == EF_F32) {
    float* q = static_cast<float*>(a.db) + m;
    *q = a.add ? *q + s : s;
  } else {
    static_cast<uint16_t*>(a.db)[m] = (uint16_t)f_bf16x2(s, 0.0f);
  }
}

// The sums of a product whose k is split over workgroups: partial C [split][M][Np] floats, Np = N rounded up to
// a group, then (wgrad) partial db [split][M].
struct Split {
  float* part;     // null: not split
  float* part_db;
  int64_t plane;   // M * Np
  int32_t Np;
  int32_t per;     // steps per split
  int32_t splits;
};

// A wavefront's T times 32 x 64 of C, handed over R times 32 rows at a time through its own part of the LDS (a
// wavefront's reads and writes of the LDS keep their order): from lanes that hold single columns, four rows each, to
// lanes that hold eight columns of a row.  Eight rows a turn, in a loop that stays a loop: unrolled, the epilogue was
// 100 KB of instructions, more than their cache holds.  What it reads beside C is loaded a turn ahead.
constexpr int kSlabPitch = 68;
constexpr int slab_bytes(int waves, int R) { return waves * R * 32 * kSlabPitch * 4; }
template <int KIND, int DO, int T, int R>
__device__ __forceinline__ void finish(const f32x16 (&acc)[T][2], char* lds, int wave, int lane, int64_t row0, int64_t col0, int32_t M,
                                       int32_t N, const Epi& ep, const Split& sp, int64_t split) {
  float* slab = reinterpret_cast<float*>(lds) + wave * R * 32 * kSlabPitch;
  const int32_t col = (int32_t)col0 + (lane & 7) * 8;
  const float* from = slab + (lane >> 3) * kSlabPitch + (lane & 7) * 8;
  float bias[8];
  if (!sp.part) load_bias<KIND, DO>(ep, col, N, bias);
#pragma unroll
  for (int p = 0; p < T / R; ++p) {
    const int64_t top = row0 + p * R * 32 + (lane >> 3);
    Side<KIND, DO> even, odd;
    auto ahead = [&](Side<KIND, DO>& side, int q) {
      const int64_t row = top + q * 8;
      side.load(ep, row, col, row < M ? N - col : kNoRow);
    };
    auto turn = [&](const Side<KIND, DO>& side, int q) {
      const int64_t row = top + q * 8;
      const f32x4 lo = *reinterpret_cast<const f32x4*>(from + q * 8 * kSlabPitch);
      const f32x4 hi = *reinterpret_cast<const f32x4*>(from + q * 8 * kSlabPitch + 4);
      if (sp.part) {
        if (row < M && col < sp.Np) {
          float* to = sp.part + split * sp.plane + row * sp.Np + col;
          *reinterpret_cast<f32x4*>(to) = lo;
          *reinterpret_cast<f32x4*>(to + 4) = hi;
        }
      } else {
        float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        epilogue8<KIND, DO>(ep, row, col, row < M ? N - col : kNoRow, v, bias, side);
      }
    };
    if (!sp.part) ahead(even, 0);
#pragma unroll
    for (int a = 0; a < R; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          slab[(a * 32 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3)) * kSlabPitch + b * 32 + (lane & 31)] = acc[p * R + a][b][r];
    asm volatile("" ::: "memory");
#pragma unroll 1
    for (int q = 0; q < R * 4; q += 2) {
      if (!sp.part) ahead(odd, q + 1);
      turn(even, q);
      if (!sp.part && q + 2 < R * 4) ahead(even, q + 2);
      turn(odd, q + 1);
    }
    asm volatile("" ::: "memory");
  }
}

// wgrad, the wavefronts of the first column of tiles: the sums of A's lines that went by; two lanes hold a line.
template <int DO, int T>
__device__ __forceinline__ void finish_db(const float (&s)[T], int lane, int64_t m0, int32_t M, const Epi& ep, const Split& sp,
                                          int64_t split) {
#pragma unroll
  for (int a = 0; a < T; ++a) {
    const float t = s[a] + __shfl_xor(s[a], 32);
    const int64_t m = m0 + a * 32 + lane;
    if (lane < 32 && m < M) {
      if (sp.part) sp.part_db[split * M + m] = t;
      else store_db<DO>(ep, m, t);
    }
  }
}

struct Mat {
  const void* p;
  int64_t ld;
};

// ---------------------------------------------------------------------------------------------
// The products, C[m][n] = sum_k A(m, k) B(n, k), on bfloat16 matrix instructions with float32 sums:
//   forward  A = x  [n][i] (k along the row), B = W [o][i] (k along the row)
//   dgrad    A = dy [n][o] (k along the row), B = W [o][i] (k down the rows)
//   wgrad    A = dy [t][o] (k down the rows), B = the checkpoint [t][i] (k down the rows)
//
// k_linear_bf16, for bfloat16 matrices whose rows start on 16 bytes.  A workgroup has BM x BN of C, WM x WN wavefronts,
// and steps of 64 along k; a wavefront has BM / WM rows and 64 columns of C in accumulators of 32 x 32.  A's tiles take
// turns in three parts of the LDS, B's in two: 256 x 256 fills its 160 KB, one workgroup a CU, and 128 x 128 half of it,
// two a CU.  Operands go from memory to the LDS without passing registers (16 bytes a lane; what lies outside the matrix
// arrives as zeros by the buffer's bounds), in the order that they have in memory:
//   k along the row   [line][64]: 16-byte chunk c of line r at place c ^ (r >> 1 & 7), so that sixteen lines' reads
//                     of one k fall on different banks (two lines span them all); read 16 bytes a lane
//   k down the rows   [64][line]: 64-byte unit u of row k at place u ^ (k & 3), so that four rows' reads do; read
//                     by the transposing load, which hands four k of one line to a lane
//   checkpoint        as k down the rows: its codes pass through registers, where they become bfloat16
// A step's last fragments are read before the barrier that releases its parts, and the next step's first ones
// after it, among the last fragments' instructions: the matrix pipes have work while the LDS changes hands.
//
// What bounds it: the matrix instructions, and the chip's power under them (1.5 to 1.7 GHz while they run).  Kernel
// times of n, i, o after a warm-up (the first 60 passes are up to 10 % slower), and the share of the cycles in which the
// matrix pipes work:
//   forward 8192, 4096, 16384, GELU and checkpoint  920 us, 1.19 PFLOP/s, 67 % (the loop alone 93 %; the epilogue
//           takes 34 thousand cycles of a tile's 191, the start 18)
//   dgrad   8192, 4096, 4096, GELU                  241 to 250 us, 1.1 PFLOP/s, 65 %
//   wgrad   8192, 4096, 16384                       970 to 1000 us, 1.1 PFLOP/s, 60 % (decoding the codes, and waits for them)
//   forward 4096, 768, 768 on 128 x 128 tiles       13 to 15 us, 192 workgroups, 12 steps: mostly start and epilogue
// Tried: four wavefronts of 128 x 128 on 256 x 256 (1788 thousand cycles against 1531), the L2 warmed a step ahead (1789
// against 1687 then), a fourth part for the 128 x 128 tiles' operands (14.8 us against 12.4).
// ---------------------------------------------------------------------------------------------
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

#define EF_LDS __attribute__((address_space(3)))

constexpr int kBK = 64;                    // k per step
constexpr int kFar = 0x7FFFFFF0;           // a byte offset outside every buffer: reads give zeros
constexpr int64_t kFastLd = (int64_t)1 << 21;  // leading dimensions up to this keep a tile's offsets in 31 bits

// (the host pass does not know the buffer type)
#if defined(__HIP_DEVICE_COMPILE__)
#define EF_BUFFER(P, BYTES) __builtin_amdgcn_make_buffer_rsrc((void*)(P), 0, (int)(BYTES), 0x00020000)
#define EF_BUFFER_B128(R, OFF) __builtin_amdgcn_raw_buffer_load_b128(R, OFF, 0, 0)
#define EF_BUFFER_B8(R, OFF) __builtin_amdgcn_raw_buffer_load_b8(R, OFF, 0, 0)
#else
#define EF_BUFFER(P, BYTES) (BYTES)
#define EF_BUFFER_B128(R, OFF) (u32x4{(uint32_t)(R), (uint32_t)(OFF), 0u, 0u})
#define EF_BUFFER_B8(R, OFF) ((uint32_t)(R))
#endif

// 16 bytes a lane from offset `off` of a buffer to the LDS, the lanes side by side from lds on; what lies outside the
// buffer arrives as zeros.  Written out: the compiler, which cannot tell the parts of the LDS apart, would let
// later reads of the LDS wait for it.  It has no result register; the wait before the barrier covers it.  (It overwrites m0,
// which the compiler keeps for uses of its own and warns of; nothing else in these kernels has one.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void buffer_to_lds(const char* base, uint32_t bytes, const char* lds, int off) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const u32x4 r = {(uint32_t)b, (uint32_t)(b >> 32), bytes, 0x00020000u};
  const uint32_t at = (uint32_t)reinterpret_cast<uintptr_t>((EF_LDS const char*)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(off), "s"(r) : "memory", "m0");
#endif
}
#pragma clang diagnostic pop

// One operand's way into the LDS.  KC: k along the row.  LINES rows of C (or columns) per tile, NW wavefronts.
// (K is at most 2^30 here: 32 bits hold every k.)
template <bool KC, int LINES, int NW>
struct Stream {
  static constexpr int J = LINES * kBK * 2 / 1024 / NW;  // loads per wavefront and step, 1024 bytes each
  static_assert(NW % 2 == 0, "a wavefront's loads are all of even or all of odd eights of lines");
  const char* base;
  int64_t step;   // bytes from one step to the next
  int ld2, K;
  int left;       // KC: bytes from base to the end of the matrix's last line; else bytes of a row from base on
  int off[J];
  int chunk8;     // KC: first k of this lane's chunk

  __device__ __forceinline__ void init(const Mat& m, int64_t line0, int64_t lines, int k, int wave, int lane) {
    ld2 = (int)m.ld * 2;
    K = k;
    if (KC) {
      base = static_cast<const char*>(m.p) + line0 * ld2;
      step = kBK * 2;
      const int have = lines - line0 < LINES ? (int)(lines - line0) : LINES;
      left = (have - 1) * ld2 + k * 2;
      chunk8 = ((lane & 7) ^ ((wave & 1) * 4 + (lane >> 4))) * 8;  // (eight lines a load: r >> 1 & 7 of line r)
#pragma unroll
      for (int j = 0; j < J; ++j) off[j] = ((j * NW + wave) * 8 + (lane >> 3)) * ld2 + chunk8 * 2;
    } else {
      constexpr int CH = LINES / 8, R = 64 / CH;  // chunks per row, rows per load
      base = static_cast<const char*>(m.p) + line0 * 2;
      step = (int64_t)kBK * ld2;
      left = (int)(lines - line0) * 2;
      chunk8 = 0;
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const int row = (j * NW + wave) * R + lane / CH, chunk = (lane % CH) ^ ((row & 3) << 2);
        off[j] = chunk * 16 < left ? row * ld2 + chunk * 16 : kFar;
      }
    }
  }

  // The tile of step s: where it begins, and how much of what follows belongs to the matrix (behind the last step:
  // nothing, and the loads give zeros that nothing reads).
  struct Aim {
    const char* from;
    uint32_t bytes;
    bool in;
  };
  __device__ __forceinline__ Aim aim(int s) const {
    const int kleft = K - s * kBK;
    const int n = KC ? (kleft > 0 ? left - s * (kBK * 2) : 0) : ((kleft < kBK ? kleft : kBK) - 1) * ld2 + left;
    return {base + s * step, (uint32_t)(n > 0 && kleft > 0 ? n : 0), !KC || chunk8 < kleft};
  }
  // part j of it into lds (LINES * 128 bytes in all)
  __device__ __forceinline__ void load(int j, const Aim& a, char* lds, int wave) const {
    buffer_to_lds(a.from, a.bytes, lds + (j * NW + wave) * 1024, a.in ? off[j] : kFar);
  }
};

// A checkpoint's way: NT threads, LINES columns per tile; a thread has J chunks of sixteen codes, half a group each,
// in registers, and passes them on as bfloat16 in quarters of a step.  (Neighbours write 32 bytes apart: a fifth of the
// LDS's cycles are bank conflicts, and hide.  Halves in turns, which leaves none: 998 -> 1028 us with loads of half the
// size, 1045 with selects, wgrad of 8192, 4096, 16384.)
template <int FMT, int LINES, int NT>
struct StreamKept {
  static constexpr int J = kBK * LINES / 16 / NT;
  static_assert(J == 2, "four times eight codes");
  struct Codes {
    u32x4 q[J];
    uint32_t s[J];
  };
  const uint8_t *codes, *scales;
  int32_t K, row_bytes, G, left;
  int off[J], soff[J], to[J];

  __device__ __forceinline__ void init(const Kept& k, int64_t line0, int rows, int tid) {
    row_bytes = k.G * kGroup;
    G = k.G;
    K = rows;
    codes = k.codes + line0;
    scales = k.scales + line0 / kGroup;
    left = row_bytes - (int32_t)line0;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int id = j * NT + tid, row = id / (LINES / 16), c = id % (LINES / 16);
      const bool in = c * 16 < left;
      off[j] = in ? row * row_bytes + c * 16 : kFar;
      soff[j] = in ? row * G + c / 2 : kFar;
      to[j] = row * LINES * 2 + (((c >> 1) ^ (row & 3)) << 6) + (c & 1) * 32;
    }
  }
  // the codes of a step (outside the matrix: zeros, as the scales, and 0 * 0 is what they decode to)
  __device__ __forceinline__ void fetch(int step, Codes& c) const {
    const int kleft = K - step * kBK, rows = kleft < kBK ? kleft : kBK;
    const int nc = (rows - 1) * row_bytes + left, ns = (rows - 1) * G + left / kGroup;  // (no rows: 0 or less)
    const auto rc = EF_BUFFER(codes + (int64_t)step * kBK * row_bytes, nc > 0 ? nc : 0);
    const auto rs = EF_BUFFER(scales + (int64_t)step * kBK * G, ns > 0 ? ns : 0);
#pragma unroll
    for (int j = 0; j < J; ++j) {
      c.q[j] = EF_BUFFER_B128(rc, off[j]);
      c.s[j] = EF_BUFFER_B8(rs, soff[j]);
    }
  }
  // codes 2 h and 2 h + 1 of quarter f
  __device__ __forceinline__ uint32_t pair(const Codes& c, int f, int h) const {
    const uint32_t w = c.q[f >> 1][(f & 1) * 2 + (h >> 1)];
    const float r = __uint_as_float(c.s[f >> 1] << 23);
    if (FMT == EF_CKPT_INT8) {
      float a, b;
      if (h & 1) bytes<1>(w, &a, &b);
      else bytes<0>(w, &a, &b);
      a *= r;
      b *= r;
      return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);  // (exact: the low halves are zeros)
    }
    // (a scale of infinity gives NaN for every code: the conversion takes the scale's exponent, and the highest one for NaN)
    return __builtin_bit_cast(uint32_t, h & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, r, true)
                                              : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, r, false));
  }
  __device__ __forceinline__ void put(int f, u32x4 w, char* lds) const {
    *reinterpret_cast<u32x4*>(lds + to[f >> 1] + (f & 1) * 16) = w;
  }
};

// A wavefront's fragments of one operand: T of 32 lines by 16 k, eight k a lane; BK k per tile.
template <bool KC, int LINES, int T, int BK = kBK>
struct Reader {
  int off[KC ? BK / 16 : T];
  __device__ __forceinline__ void init(int line0, int lane) {
    if (KC) {
#pragma unroll
      for (int ks = 0; ks < BK / 16; ++ks)
        off[ks] = (line0 + (lane & 31)) * BK * 2 + (((ks * 2 + (lane >> 5)) ^ (BK == 64 ? (lane >> 1) & 7 : (lane >> 2) & 3)) << 4);
    } else {
      const int x = (lane >> 2) & 3;
#pragma unroll
      for (int t = 0; t < T; ++t)
        off[t] = ((lane >> 5) * 8 + x) * LINES * 2 + (((line0 / 32 + t) ^ x) << 6) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    }
  }
  __device__ __forceinline__ bf16x8 read(const char* lds, int ks, int t) const {
    if (KC) return *reinterpret_cast<const bf16x8*>(lds + off[ks] + t * 32 * BK * 2);
    const char* p = lds + off[t] + ks * 16 * LINES * 2;
    const bf16x4 a = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((EF_LDS s16x4*)p));
    const bf16x4 b = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((EF_LDS s16x4*)(p + 4 * LINES * 2)));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// s plus the eight elements of a fragment, in float32 (two at a time against ones)
__device__ __forceinline__ float add8(bf16x8 f, float s) {
  const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
#pragma unroll
  for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{f[2 * j], f[2 * j + 1]}, one, s, false);
  return s;
}

// What workgroup b of a product does: a tile of C and a part of k.  In an order in which those that run at one time on an
// XCD (workgroups b, b + 8, b + 16, ...) share what they read: each XCD has a run of the work, one part of k after the
// other, its tiles in bands of eight rows of tiles.
struct Share {
  uint32_t m, n, z;
};
__device__ __forceinline__ Share share_of(uint32_t b, uint32_t tm, uint32_t tn, uint32_t splits) {
  const uint32_t tiles = tm * tn, T = tiles * splits, q = T / 8, rest = T % 8, x = b % 8;
  const uint32_t id = x * q + (x < rest ? x : rest) + b / 8, z = id / tiles, t = id - z * tiles;
  const uint32_t band = t / (8 * tn), h = tm - band * 8 < 8 ? tm - band * 8 : 8, in = t - band * 8 * tn;
  return {band * 8 + in % h, in / h, z};
}

template <int KIND, int DO, int FMT, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(WM* WN * 64, 2) void k_linear_bf16(int32_t M, int32_t N, int32_t K, Mat A, Mat B, Kept BK, Epi ep, Split sp) {
  constexpr bool AKC = KIND != K_WGRAD, BKC = KIND == K_FWD, B8 = KIND == K_WGRAD;
  constexpr int NW = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  static_assert(TN == 2, "the epilogue hands over 64 columns a wavefront");
  constexpr int kA = BM * kBK * 2, kB = BN * kBK * 2;
  __shared__ __align__(1024) char lds[3 * kA + 2 * kB];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Share my = share_of(blockIdx.x, ((uint32_t)M + BM - 1) / BM, ((uint32_t)N + BN - 1) / BN, sp.splits);
  const int64_t m0 = (int64_t)my.m * BM, n0 = (int64_t)my.n * BN;
  const int wm = wave / WN * (BM / WM), wn = wave % WN * 64;
  const int all = (K + kBK - 1) / kBK, s0 = (int)my.z * sp.per, s1 = s0 + sp.per < all ? s0 + sp.per : all;

  Stream<AKC, BM, NW> sa;
  sa.init(A, m0, M, K, wave, lane);
  Stream<BKC, BN, NW> sb;
  using SK = StreamKept<FMT, BN, NW * 64>;
  SK sk;
  if (B8) sk.init(BK, n0, K, tid);
  else sb.init(B, n0, N, K, wave, lane);
  Reader<AKC, BM, TM> ra;
  Reader<BKC, BN, TN> rb;
  ra.init(wm, lane);
  rb.init(wn, lane);

  f32x16 acc[TM][TN];
#pragma unroll
  for (int a = 0; a < TM; ++a)
#pragma unroll
    for (int b = 0; b < TN; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;
  // db: the workgroups of the first column of tiles add up A's lines as they go by, each of the wavefronts that share
  // them the slices ks = wave % WN of every step.
  const int sum_slice = KIND == K_WGRAD && ep.db && n0 == 0 ? wave % WN : -1;
  float bs[TM];
#pragma unroll
  for (int a = 0; a < TM; ++a) bs[a] = 0.0f;
  bf16x8 fa[2][TM], fb[2][TN];
  // One slice: the matrix instructions of the fragments h, and between them, one by one, the reads of the next ones
  // (slice ks of the tiles from_a and from_b, where there are `more`) and whatever else there is to do.  Pinned in this
  // order: left to itself the compiler gathers the reads before their use.
  constexpr int kMul = TM * TN;
  auto slice = [&](auto more, int h, const char* from_a, const char* from_b, int ks, auto&& between) {
#pragma unroll
    for (int i = 0; i < kMul; ++i) {
      const int a = i / TN, b = i % TN;
      acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[h][a], fb[h][b], acc[a][b], 0, 0, 0);
      if constexpr (decltype(more)::value) {
        if (i < TN) fb[h ^ 1][i] = rb.read(from_b, ks, i);
        else if (i - TN < TM) fa[h ^ 1][i - TN] = ra.read(from_a, ks, i - TN);
        if (i == kMul - 1)
#pragma unroll
          for (int t = kMul - TN; t < TM; ++t) fa[h ^ 1][t] = ra.read(from_a, ks, t);
      }
      between(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Tiles of A take turns in three parts of the LDS, those of B in two.  Behind the barrier that ends step s its last
  // fragments' instructions (slice 3) are to be issued, and its parts of the LDS are free: for step s + 2 of B, loaded
  // in slice 3, and step s + 3 of A, loaded in the slices after that, which have more than a step to arrive.  The
  // address unit takes 16 cycles for a load, and a wavefront that finds it busy issues nothing: one load every kGap
  // matrix instructions.  A checkpoint's codes are loaded a step before their first use and go into the LDS a quarter a
  // slice.  (They are waited for earlier than that: the compiler widens the loaded scale bytes at the end of the loop of
  // two steps, so that every second step waits there for loads that it has just issued, and its waits for codes do not
  // count the loads written as asm, so that they reach A's tiles too.)
  using SA = Stream<AKC, BM, NW>;
  using SB = Stream<BKC, BN, NW>;
  typename SK::Codes codes[2];
  u32x4 w;
  auto quarter = [&](int i, const typename SK::Codes& c, int f, char* to) {
    constexpr int P = 4 / (kMul / 2);
    if (i < kMul / 2) {
#pragma unroll
      for (int h = 0; h < P; ++h) w[i * P + h] = sk.pair(c, f, i * P + h);
    }
    if (i == kMul / 2) sk.put(f, w, to);
  };
  constexpr int kGap = SA::J <= kMul / 2 ? 2 : 1;
  auto decode = [&](const typename SK::Codes& c, int f0, int f1, char* to) {
#pragma unroll
    for (int f = f0; f < f1; ++f) {
#pragma unroll
      for (int h = 0; h < 4; ++h) w[h] = sk.pair(c, f, h);
      sk.put(f, w, to);
    }
  };
  char* const b0 = lds;  // (first: offsets within B's parts fit the instructions)
  char* const b1 = lds + kB;
  char *a0 = lds + 2 * kB, *a1 = a0 + kA, *a2 = a1 + kA;
  if (B8) {
    sk.fetch(s0, codes[0]);
    sk.fetch(s0 + 1, codes[1]);
  }
  {
    const auto a = sa.aim(s0), a_next = sa.aim(s0 + 1);
    typename SB::Aim b{}, b_next{};  // (a checkpoint has no Stream)
    if constexpr (!B8) {
      b = sb.aim(s0);
      b_next = sb.aim(s0 + 1);
    }
#pragma unroll
    for (int j = 0; j < SA::J; ++j) {
      sa.load(j, a, a0, wave);
      if (!B8) sb.load(j, b, b0, wave);
    }
#pragma unroll
    for (int j = 0; j < SA::J; ++j) {
      sa.load(j, a_next, a1, wave);
      if (!B8) sb.load(j, b_next, b1, wave);
    }
  }
  if (B8) {
    decode(codes[0], 0, 4, b0);
    decode(codes[1], 0, 1, b1);
    sk.fetch(s0 + 2, codes[0]);
  }
  // The first fragments wait for the first step's tiles alone (a checkpoint's codes have passed already): the barrier that
  // ends it waits for the second's.  n, i, o = 4096, 768, 768: 14.6 -> 14.1 us.
  if (B8) __builtin_amdgcn_s_waitcnt(0);
  else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * SA::J) : "memory");
  asm volatile("s_barrier" ::: "memory");
#pragma unroll
  for (int t = 0; t < TM; ++t) fa[0][t] = ra.read(a0, 0, t);
#pragma unroll
  for (int t = 0; t < TN; ++t) fb[0][t] = rb.read(b0, 0, t);
  // Step s in a0 and cur, s + 1 in a1 and nxt (of its checkpoint, in `now`, a quarter); `then` has the codes of s + 2.
  auto sum = [&](int h, int ks) {
    if (KIND == K_WGRAD && sum_slice >= 0 && (WN == 4 ? ks == sum_slice : (ks & 1) == sum_slice)) {
#pragma unroll
      for (int a = 0; a < TM; ++a) bs[a] = add8(fa[h][a], bs[a]);
    }
  };
  auto advance = [&](int s, char* cur, char* nxt, typename SK::Codes& now, typename SK::Codes& then) {
    const auto a = sa.aim(s + 2);
#pragma unroll
    for (int ks = 0; ks < 3; ++ks) {
      slice(std::true_type{}, ks & 1, a0, cur, ks + 1, [&](int i) {
        const int j = (ks * kMul + i) / kGap;
        if (i % kGap == 0 && j < SA::J) sa.load(j, a, a2, wave);
        if (B8) quarter(i, now, ks + 1, nxt);
      });
      sum(ks & 1, ks);
    }
    // This wavefront's part of the next step has arrived (all but the last loads, of A behind it), and its last reads
    // of this one.
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(SA::J) : "memory");
    typename SB::Aim b{};
    if constexpr (!B8) b = sb.aim(s + 2);
    slice(std::true_type{}, 1, a1, nxt, 0, [&](int i) {
      if (B8 && i == 0) sk.fetch(s + 3, now);
      if (!B8 && i % kGap == 0 && i / kGap < SB::J) sb.load(i / kGap, b, cur, wave);
      if (B8) quarter(i, then, 0, cur);
    });
    sum(1, 3);
    char* x = a0;
    a0 = a1;
    a1 = a2;
    a2 = x;
  };
  static_assert(SA::J == SB::J && kMul / kGap >= SB::J, "B's loads fit a slice");
  int s = s0;
  for (; s + 2 < s1; s += 2) {
    advance(s, b0, b1, codes[1], codes[0]);
    advance(s + 1, b1, b0, codes[0], codes[1]);
  }
  const char* last = b0;
  if (s + 1 < s1) {
    advance(s, b0, b1, codes[1], codes[0]);
    last = b1;
  }
#pragma unroll
  for (int ks = 0; ks < 3; ++ks) {
    slice(std::true_type{}, ks & 1, a0, last, ks + 1, [](int) {});
    sum(ks & 1, ks);
  }
  slice(std::false_type{}, 1, a0, last, 0, [](int) {});
  sum(1, 3);
  __builtin_amdgcn_s_waitcnt(0);
  __syncthreads();
  static_assert(slab_bytes(NW, 2) <= sizeof(lds), "the epilogue's part of the LDS");
  if (KIND == K_WGRAD && ep.db && n0 == 0) {  // the wavefronts' sums of a line, in order
    float* share = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int a = 0; a < TM; ++a) share[(wave * TM + a) * 64 + lane] = bs[a];
    __syncthreads();
    if (wn == 0) {
#pragma unroll
      for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int z = 1; z < WN; ++z) bs[a] += share[((wave + z) * TM + a) * 64 + lane];
      finish_db<DO>(bs, lane, m0 + wm, M, ep, sp, my.z);
    }
    __syncthreads();
  }
  finish<KIND, DO, TM, 2>(acc, lds, wave, lane, m0 + wm, n0 + wn, M, N, ep, sp, my.z);
}

// ---------------------------------------------------------------------------------------------
// The same products for every type and alignment.  Operands pass through registers, two steps of 32 ahead.  A float32
// value goes into the LDS as three bfloat16 numbers, hi + mid + lo: rounded to nearest three times, which leaves
// nothing of its 24 bits.  Of the nine products of two such sums the six that matter are taken; what is left out is
// 2^-23 of the product at most.  A checkpoint's values are bfloat16 numbers, so against them three products are the
// whole.  (Against the matrix instructions for float32, a sixteenth as fast: n, i, o = 1021, 771, 1285, dgrad
// 49 -> 44 us, and 31 with the steps since; 2043, 1285, 771, wgrad 87 -> 38 us, and 35; each with its join.)  An infinity has no such parts: it comes out as NaN.
// A workgroup has 128 x 128 of C, four wavefronts of 64 x 64.
// ---------------------------------------------------------------------------------------------
constexpr int kAnyTile = 128, kAnyK = 32;
constexpr int kPlane = kAnyTile * kAnyK * 2;

// Eight float32 values as hi + mid + lo, each rounded to the nearest bfloat16.  hi is held at the largest one: a finite
// value does not round to an infinity, and what is not finite goes on into mid and lo.
__device__ __forceinline__ void split8(const Raw<EF_F32>& r, u32x4 (&w)[3]) {
#pragma unroll
  for (int h = 0; h < 4; ++h) {
    float x = r.value(2 * h), y = r.value(2 * h + 1);
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      w[p][h] = p ? f_bf16x2(x, y) : f_bf16x2(__builtin_amdgcn_fmed3f(x, -0x1.FEp127f, 0x1.FEp127f), __builtin_amdgcn_fmed3f(y, -0x1.FEp127f, 0x1.FEp127f));
      x -= __uint_as_float(w[p][h] << 16);
      y -= __uint_as_float(w[p][h] & 0xFFFF0000u);
    }
  }
}
__device__ __forceinline__ void split8(const Raw<EF_BF16>& r, u32x4 (&w)[3]) { w[0] = u32x4{r.r[0], r.r[1], r.r[2], r.r[3]}; }

// Where a thread's two chunks of eight elements of a step lie: eight k of a line where KC, else eight lines of a k.
template <bool KC>
struct Places {
  __device__ __forceinline__ static int line(int t, int j) { return KC ? (j * 256 + t) / 4 : (t & 15) * 8; }
  __device__ __forceinline__ static int k(int t, int j) { return KC ? (t & 3) * 8 : (j * 256 + t) / 16; }
  __device__ __forceinline__ static int lds(int t, int j) {
    const int l = line(t, j), r = k(t, j);
    return KC ? l * kAnyK * 2 + (((t & 3) ^ ((l >> 2) & 3)) << 4) : r * kAnyTile * 2 + (((t >> 2 & 3) ^ (r & 3)) << 6) + (t & 3) * 16;
  }
};

// One operand: its chunks in registers, P bfloat16 numbers a value in the LDS.  Lines behind the last one are not
// kept out: they repeat the last line, or line 0, or are what follows the row in memory (up to seven elements, so not
// in the last step, whose last row may end the matrix), and reach only rows and columns of C that nobody stores.
// Taken one by one, the last lines' elements made the workgroups at the edge wait for memory in each step (dgrad of
// 1021, 771, 1285 in bfloat16, unsplit: 63 -> 28 us).
template <int DT, bool KC, int P>
struct Chunks {
  using At = Places<KC>;
  const char* p[2];  // this thread's chunks of the next step
  int64_t step;      // bytes from one step to the next
  int64_t ld;
  int cnt;           // !KC: lines that the chunks have
  bool narrow;       // !KC: rows of under eight elements
  Raw<DT> raw[2][2];

  __device__ __forceinline__ void init(const Mat& m, int64_t line0, int64_t lines, int64_t k0, int t) {
    constexpr int S = DT == EF_F32 ? 4 : 2;
    ld = m.ld * S;
    narrow = !KC && m.ld < 8;
    step = KC ? kAnyK * S : kAnyK * ld;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int64_t l = line0 + At::line(t, j);
      const int64_t k = k0 + At::k(t, j);
      cnt = lines - l < 8 ? (int)(lines - l) : 8;
      if (KC && l >= lines) l = lines - 1;
      if (!KC && cnt <= 0) {
        l = 0;
        cnt = lines < 8 ? (int)lines : 8;
      }
      p[j] = static_cast<const char*>(m.p) + (KC ? l * ld + k * S : k * ld + l * S);
    }
  }
  // left: k from this step's first on; WHOLE: more than the step's, and rows that are not narrow
  template <bool WHOLE>
  __device__ __forceinline__ void fetch(int set, int64_t left, int t) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t mine = left - At::k(t, j);
      int n = 8;
      if (!WHOLE && (left <= kAnyK || narrow)) n = KC ? (mine < 8 ? (int)mine : 8) : (mine > 0 ? cnt : 0);
      raw[set][j].load(p[j], 0, n);
      p[j] += step;
    }
  }
  __device__ __forceinline__ void put(int set, char* lds, int t) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const Raw<DT>& r = raw[set][j];
      char* to = lds + At::lds(t, j);
      if (P == 1) {
        *reinterpret_cast<u32x4*>(to) = u32x4{r.r[0], r.r[1], r.r[2], r.r[3]};
      } else {
        u32x4 w[3];
        split8(r, w);
#pragma unroll
        for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4*>(to + p * kPlane) = w[p];
      }
    }
  }
};

struct KeptChunks {
  using At = Places<false>;
  const uint8_t *q[2], *s[2];
  int64_t qstep, sstep;
  u32x2 code[2][2];
  uint32_t scale[2][2];

  __device__ __forceinline__ void init(const Kept& m, int64_t line0, int64_t k0, int t) {
    const int64_t row = (int64_t)m.G * kGroup;
    qstep = kAnyK * row;
    sstep = kAnyK * (int64_t)m.G;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      int64_t l = line0 + At::line(t, j);
      if (l >= row) l = 0;
      q[j] = m.codes + (k0 + At::k(t, j)) * row + l;
      s[j] = m.scales + (k0 + At::k(t, j)) * m.G + l / kGroup;
    }
  }
  template <bool WHOLE>
  __device__ __forceinline__ void fetch(int set, int64_t left, int t) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      code[set][j] = u32x2{0u, 0u};
      scale[set][j] = 0u;
      if (WHOLE || At::k(t, j) < left) {
        code[set][j] = *reinterpret_cast<const u32x2*>(q[j]);
        scale[set][j] = *s[j];
      }
      q[j] += qstep;
      s[j] += sstep;
    }
  }
  __device__ __forceinline__ void put(int set, char* lds, int fmt, int t) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float v[8];
      decode8(code[set][j], scale[set][j], fmt, v);
      u32x4 w;
#pragma unroll
      for (int h = 0; h < 4; ++h) w[h] = __builtin_amdgcn_perm(__float_as_uint(v[2 * h + 1]), __float_as_uint(v[2 * h]), 0x07060302u);
      *reinterpret_cast<u32x4*>(lds + At::lds(t, j)) = w;
    }
  }
};

template <int KIND, int DT, int DO>
__global__ __launch_bounds__(256, 2) void k_linear_any(int32_t M, int32_t N, int32_t K, Mat A, Mat B, Kept BK, Epi ep, Split sp) {
  constexpr bool AKC = KIND != K_WGRAD, BKC = KIND == K_FWD, B8 = KIND == K_WGRAD;
  constexpr int PA = DT == EF_F32 ? 3 : 1, PB = B8 ? 1 : PA;
  constexpr int kTiles = (PA + PB) * kPlane, kSlabs = slab_bytes(4, 1);
  __shared__ __align__(1024) char lds[kTiles > kSlabs ? kTiles : kSlabs];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const Share my = share_of(blockIdx.x, ((uint32_t)M + kAnyTile - 1) / kAnyTile, ((uint32_t)N + kAnyTile - 1) / kAnyTile, sp.splits);
  const int64_t m0 = (int64_t)my.m * kAnyTile, n0 = (int64_t)my.n * kAnyTile;
  const int wm = (wave >> 1) * 64, wn = (wave & 1) * 64;
  Chunks<DT, AKC, PA> ca;
  Chunks<DT, BKC, PB> cb;
  KeptChunks ck;
  Reader<AKC, kAnyTile, 2, kAnyK> ra;
  Reader<BKC, kAnyTile, 2, kAnyK> rb;
  ra.init(wm, lane);
  rb.init(wn, lane);
  f32x16 acc[2][2];
#pragma unroll
  for (int a = 0; a < 2; ++a)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.0f;
  const bool sums = KIND == K_WGRAD && ep.db && n0 == 0 && wn == 0;
  float bs[2] = {0.0f, 0.0f};
  const int64_t all = ((int64_t)K + kAnyK - 1) / kAnyK;
  const int64_t s0 = (int64_t)my.z * sp.per, s1 = s0 + sp.per < all ? s0 + sp.per : all;
  ca.init(A, m0, M, s0 * kAnyK, t);
  if (B8) ck.init(BK, n0, s0 * kAnyK, t);
  else cb.init(B, n0, N, s0 * kAnyK, t);
  auto fetch = [&](auto whole, int64_t s, int set) {
    constexpr bool W = decltype(whole)::value;
    const int64_t left = K - s * kAnyK;
    ca.template fetch<W>(set, left, t);
    if (B8) ck.template fetch<W>(set, left, t);
    else cb.template fetch<W>(set, left, t);
  };
  auto step = [&](auto whole, int64_t s, int set) {
    __builtin_amdgcn_sched_barrier(0);  // (nothing of this step into the one before it: its loads would be waited for there)
    __syncthreads();
    ca.put(set, lds, t);
    if (B8) ck.put(set, lds + PA * kPlane, BK.fmt, t);
    else cb.put(set, lds + PA * kPlane, t);
    __syncthreads();
    if (decltype(whole)::value || s + 2 < s1) fetch(whole, s + 2, set);
#pragma unroll
    for (int ks = 0; ks < kAnyK / 16; ++ks) {
      bf16x8 fa[PA][2], fb[PB][2];
#pragma unroll
      for (int p = 0; p < PA; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) fa[p][i] = ra.read(lds + p * kPlane, ks, i);
#pragma unroll
      for (int p = 0; p < PB; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i) fb[p][i] = rb.read(lds + (PA + p) * kPlane, ks, i);
#pragma unroll
      for (int d = PA + PB - 2; d >= 0; --d)  // the least products first
#pragma unroll
        for (int p = 0; p < PA; ++p)
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
              if (d < 3 && d - p >= 0 && d - p < PB)
                acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[p][a], fb[d - p][b], acc[a][b], 0, 0, 0);
      if (sums) {
#pragma unroll
        for (int p = PA - 1; p >= 0; --p)
#pragma unroll
          for (int a = 0; a < 2; ++a) bs[a] = add8(fa[p][a], bs[a]);
      }
    }
  };
  // The steps whose chunks are whole (all but the last one) in a loop without branches: where some lanes load elements
  // and others chunks, the compiler waits for everything that is under way, and two steps ahead become one.  (float32,
  // dgrad of 8192, 4096, 1024: 393 -> 371 us, 1.1 PFLOP/s in bfloat16 products; 4096, 768, 768 forward: 38.5 -> 36.5.)
  const bool narrow = ca.narrow || (!B8 && cb.narrow);
  const int64_t whole = narrow ? s0 : s1 < all ? s1 : all - 1;
  int64_t s = s0;
  if (s0 + 3 < whole) {
    fetch(std::true_type{}, s0, 0);
    fetch(std::true_type{}, s0 + 1, 1);
    for (; s + 3 < whole; s += 2) {
      step(std::true_type{}, s, 0);
      step(std::true_type{}, s + 1, 1);
    }
  } else {
    if (s0 < s1) fetch(std::false_type{}, s0, 0);
    if (s0 + 1 < s1) fetch(std::false_type{}, s0 + 1, 1);
  }
  for (; s < s1; s += 2) {
    step(std::false_type{}, s, 0);
    if (s + 1 < s1) step(std::false_type{}, s + 1, 1);
  }
  __syncthreads();
  finish<KIND, DO, 2, 1>(acc, lds, wave, lane, m0 + wm, n0 + wn, M, N, ep, sp, my.z);
  if (sums) finish_db<DO>(bs, lane, m0 + wm, M, ep, sp, my.z);
}

// ---------------------------------------------------------------------------------------------
// The forward product of a few tokens (up to 16 TT): the weights are read once, and that bounds it.  A workgroup
// has 16 OT output features and splits k over its eight wavefronts; each takes the weights' rows as the first
// operand and the tokens as the second, straight from memory to registers, 16 bytes a lane, eight loads of the
// weights in flight (sixteen: 8.6 us against 8.1, past the caches 10.2); float32 as in k_linear_any.  4096 x 4096
// weights in bfloat16, one token: 8.1 to 9 us, about 4 TB/s, of which 3 us are the launch and the last loads' latency.
// The eight partial sums are added in order through the LDS.  Up to 32 tokens: with those weights 32 take 13.1 us here and
// 33 12.7 on tiles (16: 9.6), in float32 27.5 and 34.0.
// ---------------------------------------------------------------------------------------------
constexpr int kFewWaves = 8;
constexpr int kFewTokens = 32;

template <int DT, int TT, int OT>
__global__ __launch_bounds__(kFewWaves * 64) void k_linear_few(int32_t n, int32_t N, int32_t K, Mat X, Mat W, Epi ep) {
  __shared__ f32x4 red[kFewWaves][TT][OT][64];
  constexpr int S = DT == EF_F32 ? 4 : 2, P = DT == EF_F32 ? 3 : 1, U = 16 / S / OT;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t o0 = (int64_t)blockIdx.x * 16 * OT;
  const int64_t ldw = W.ld * S, ldx = X.ld * S;
  const int64_t have = N - o0 < 16 * OT ? N - o0 : 16 * OT;
  const auto rw = EF_BUFFER(static_cast<const char*>(W.p) + o0 * ldw, (have - 1) * ldw + (int64_t)K * S);
  const auto rx = EF_BUFFER(X.p, (int64_t)(n - 1) * ldx + (int64_t)K * S);
  const int kl = (lane >> 4) * 8;
  const int per = ((K + 32 * kFewWaves - 1) / (32 * kFewWaves) + 3) / 4 * 4;  // steps of 32 per wavefront: whole 256-byte runs
  const int c0 = wave * per, c1 = c0 + per;
  f32x4 acc[TT][OT];
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int o = 0; o < OT; ++o) acc[t][o] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  auto fetch = [&](auto r, int off, bool in) {
    Raw<DT> v;
#pragma unroll
    for (int h = 0; h < S / 2; ++h) {
      const u32x4 a = EF_BUFFER_B128(r, in ? off + h * 16 : kFar);
#pragma unroll
      for (int j = 0; j < 4; ++j) v.r[4 * h + j] = a[j];
    }
    return v;
  };
  for (int c = c0; c < c1 && c * 32 < K; c += U) {
    Raw<DT> w[U][OT], x[U][TT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (c + u) * 32 + kl;
      const bool in = k < K && c + u < c1;
#pragma unroll
      for (int o = 0; o < OT; ++o) w[u][o] = fetch(rw, (int)((o * 16 + (lane & 15)) * ldw) + k * S, in);
#pragma unroll
      for (int t = 0; t < TT; ++t) x[u][t] = fetch(rx, (int)((t * 16 + (lane & 15)) * ldx) + k * S, in);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      u32x4 wp[OT][3], xp[TT][3];
#pragma unroll
      for (int o = 0; o < OT; ++o) split8(w[u][o], wp[o]);
#pragma unroll
      for (int t = 0; t < TT; ++t) split8(x[u][t], xp[t]);
#pragma unroll
      for (int d = P == 1 ? 0 : 2; d >= 0; --d)  // the least products first
#pragma unroll
        for (int p = 0; p <= d; ++p)
#pragma unroll
          for (int o = 0; o < OT; ++o)
#pragma unroll
            for (int t = 0; t < TT; ++t)
              acc[t][o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wp[o][p]), __builtin_bit_cast(bf16x8, xp[t][d - p]),
                                                                 acc[t][o], 0, 0, 0);
    }
  }
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int o = 0; o < OT; ++o) red[wave][t][o][lane] = acc[t][o];
  __syncthreads();
  // eight outputs of a token per lane; four neighbouring lanes a group where OT is 2
  if (tid >= TT * 16 * OT * 2) return;
  const int q = tid % (OT * 2), token = tid / (OT * 2);
  const int32_t col = (int32_t)o0 + q * 8;
  const int cnt = token < n ? N - col : kNoRow;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
  for (int z = 0; z < kFewWaves; ++z) {
    const f32x4* p = red[z][token >> 4][q >> 1] + (q & 1) * 32 + (token & 15);
    const f32x4 lo = p[0], hi = p[16];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] += lo[j];
      v[j + 4] += hi[j];
    }
  }
  float b[8];
  Side<K_FWD, DT> side;
  load_bias<K_FWD, DT>(ep, col, N, b);
  side.load(ep, token, col, cnt);
  epilogue8<K_FWD, DT>(ep, token, col, cnt, v, b, side);
}

// The splits' sums in order, then the epilogue.  Np / 8 lanes a row, whole groups side by side.
template <int KIND, int DO>
__global__ __launch_bounds__(256) void k_linear_join(int32_t M, int32_t N, Split sp, Epi ep) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int32_t w = sp.Np / 8;
  const int64_t row = id / w;
  const int32_t col = (int32_t)(id - row * w) * 8;
  const bool in = row < M;
  if (KIND == K_WGRAD && !in) {  // the lanes behind the last row: db
    const int64_t m = id - (int64_t)M * w;
    if (!ep.db || m >= M) return;
    float t = 0.0f;
    for (int z = 0; z < sp.splits; ++z) t += sp.part_db[(int64_t)z * M + m];
    store_db<DO>(ep, m, t);
    return;
  }
  const int cnt = in ? N - col : kNoRow;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0}, b[8];
  Side<KIND, DO> side;
  load_bias<KIND, DO>(ep, col, N, b);
  side.load(ep, row, col, cnt);
  if (in)
    for (int z = 0; z < sp.splits; ++z) {
      const float* p = sp.part + z * sp.plane + row * sp.Np + col;
      const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] += lo[j];
        v[j + 4] += hi[j];
      }
    }
  epilogue8<KIND, DO>(ep, row, col, cnt, v, b, side);
}

}  // namespace efs

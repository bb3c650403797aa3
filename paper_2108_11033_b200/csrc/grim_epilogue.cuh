// What follows a product: bias, activation, residual (grim_bcr_linear).  The device code that every multiply kernel ends with.
//
// p = (W X)_rq + bias_r in fp32;  y = act(p) + residual_rq, rounded once;  p itself, rounded, where it is asked for.
// Kernels call this where they store, on values that are still in registers or shared memory, so the epilogue costs its own
// operands' bytes and no pass.  An access to the residual comes before the store to Y by the same thread: they may be one matrix.
#pragma once
#include <cuda_bf16.h>

#include "grim_device.cuh"
#include "grim_internal.h"

namespace grim {

// The pieces that activations and gates are made of.  2^x and 1/x by the special function unit are within 2 and 1 ulp; the product with
// log2 e rounds by u (2^-24, half an ulp) and its constant by 0.23 u, so e^-x is within (1.23 |x| + 4) u of itself.
constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float exp2_(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float inverse(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Two operations in one instruction, each rounded as the single one is.  Gates and their gradients are bound by the number of
// instructions: the recurrence's gradient, 2048 x 16384 in bf16, 75 -> 73 us, 8192 x 2048 in fp32 62 -> 60; forward its time stays.
__device__ __forceinline__ void mul2(float& r0, float& r1, float a0, float a1, float b0, float b1) {
  asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 c, a, b;\nmov.b64 {%0, %1}, c;\n}"
      : "=f"(r0), "=f"(r1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void add2(float& r0, float& r1, float a0, float a1, float b0, float b1) {
  asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 c, a, b;\nmov.b64 {%0, %1}, c;\n}"
      : "=f"(r0), "=f"(r1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}

__device__ __forceinline__ void fma2(float& r0, float& r1, float a0, float a1, float b0, float b1, float c0, float c1) {
  asm("{\n.reg .b64 a, b, c;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 c, a, b, c;\n"
      "mov.b64 {%0, %1}, c;\n}"
      : "=f"(r0), "=f"(r1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}

// The smaller, the larger of two numbers, NaN if one is.
__device__ __forceinline__ float min_nan(float a, float b) {
  float y;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// sigmoid(v) = a = 1 / (1 + e) and 1 - sigmoid(v) = k = e a, e = e^-v: neither is a difference, so both keep their relative precision; e is
// bounded where a would leave the range of 1 / x, so that a is never below 2.4e-35 (1.8e-35 without FAST).  FAST, for values of eight bits:
// e within (1.23 |v| + 4) u; otherwise within 4 u.  (Selecting by v's sign between 1 / (1 + e^-|v|) and its complement costs two selects and a comparison more, on the unit
// that a bf16 recurrence keeps busiest: 2048 x 16384 46.5 -> 45.1 us.)
template <bool FAST = false>
__device__ __forceinline__ void sigmoid_pair(float v, float& a, float& k) {
  const float e = FAST ? exp2_(min_nan(v * -kLog2e, 115.f)) : expf(min_nan(-v, 80.f));
  a = inverse(1.f + e);
  k = e * a;
}

// The same for two values.
template <bool FAST>
__device__ __forceinline__ void sigmoid_pair2(float v0, float v1, float& a0, float& a1, float& k0, float& k1) {
  float e0, e1, d0, d1;
  if (FAST) {
    mul2(e0, e1, v0, v1, -kLog2e, -kLog2e);
    e0 = exp2_(min_nan(e0, 115.f));
    e1 = exp2_(min_nan(e1, 115.f));
  } else {
    e0 = expf(min_nan(-v0, 80.f));
    e1 = expf(min_nan(-v1, 80.f));
  }
  add2(d0, d1, e0, e1, 1.f, 1.f);
  a0 = inverse(d0);
  a1 = inverse(d1);
  mul2(k0, k1, e0, e1, a0, a1);
}

// Up to 0.6 a polynomial in v^2 for tanh(v) / v, fitted for the least largest relative error (0.05 u; 1.7 u as evaluated); from there on
// 1 - 2 / (1 + e^2|v|), whose difference does not cancel (within 8 u at 0.6, less beyond).  Both without a branch.
__device__ __forceinline__ float tanh_(float v) {
  const float s = v * v, a = fabsf(v);
  float p = -0.005852168425917625f;
  p = fmaf(p, s, 0.02075362764298916f);
  p = fmaf(p, s, -0.05376870557665825f);
  p = fmaf(p, s, 0.13331688940525055f);
  p = fmaf(p, s, -0.3333328366279602f);
  p = fmaf(p, s, 1.f);
  const float far = copysignf(fmaf(-2.f, inverse(1.f + exp2_(a * (2.f * kLog2e))), 1.f), v);
  return a <= 0.6f ? v * p : far;
}

// e = e^(-v^2 / 2) and the normal distribution's Phi(v).  Its tail is e t P(t), t = 1 / (1 + 0.3 |v|): P of degree 7 fitted for the least
// largest relative error of the tail on 0 .. 14 (2.5 u; 6.5 u as evaluated, if e is exact), so nothing cancels on either side.  e's exponent is
// rounded three times, which takes the tail to 11 u of itself up to |v| = 3, 34 u up to 6, 127 u up to 12; of 1 it is 4.2 u.
__device__ __forceinline__ float normal(float v, float& e) {
  const float t = inverse(fmaf(fabsf(v), 0.3f, 1.f));
  e = exp2_(v * v * (-0.5f * kLog2e));
  float p = 0.0713493674993515f;
  p = fmaf(p, t, -0.3144046366214752f);
  p = fmaf(p, t, 0.4127030074596405f);
  p = fmaf(p, t, -0.1073622927069664f);
  p = fmaf(p, t, 0.2571198642253876f);
  p = fmaf(p, t, 0.1998282372951508f);
  p = fmaf(p, t, 0.2415076643228531f);
  p = fmaf(p, t, 0.2392586171627045f);
  const float tail = 0.5f * (e * t) * p;
  return v >= 0.f ? 1.f - tail : tail;
}

// The same for two values.  Where a thread has eight (a bf16 piece) the gradient of gelu takes this: 4096 x 8192 40 -> 39 us, 64 x 100003
// 12.5 -> 11.7.  Where it has four (fp32) memory is the bound and the pairs' registers cost more: 62 -> 64.
__device__ __forceinline__ void normal_pair(float v0, float v1, float& y0, float& y1, float& e0, float& e1) {
  float t0, t1, p0, p1;
  fma2(t0, t1, fabsf(v0), fabsf(v1), 0.3f, 0.3f, 1.f, 1.f);
  t0 = inverse(t0);
  t1 = inverse(t1);
  mul2(e0, e1, v0, v1, v0, v1);
  mul2(e0, e1, e0, e1, -0.5f * kLog2e, -0.5f * kLog2e);
  e0 = exp2_(e0);
  e1 = exp2_(e1);
  fma2(p0, p1, t0, t1, 0.0713493674993515f, 0.0713493674993515f, -0.3144046366214752f, -0.3144046366214752f);
  fma2(p0, p1, p0, p1, t0, t1, 0.4127030074596405f, 0.4127030074596405f);
  fma2(p0, p1, p0, p1, t0, t1, -0.1073622927069664f, -0.1073622927069664f);
  fma2(p0, p1, p0, p1, t0, t1, 0.2571198642253876f, 0.2571198642253876f);
  fma2(p0, p1, p0, p1, t0, t1, 0.1998282372951508f, 0.1998282372951508f);
  fma2(p0, p1, p0, p1, t0, t1, 0.2415076643228531f, 0.2415076643228531f);
  fma2(p0, p1, p0, p1, t0, t1, 0.2392586171627045f, 0.2392586171627045f);
  mul2(t0, t1, t0, t1, e0, e1);
  mul2(t0, t1, t0, t1, 0.5f, 0.5f);
  mul2(p0, p1, p0, p1, t0, t1);
  fma2(t0, t1, p0, p1, -1.f, -1.f, 1.f, 1.f);
  y0 = v0 >= 0.f ? t0 : p0;
  y1 = v1 >= 0.f ? t1 : p1;
}

constexpr float kSqrt2OverPi = 0.79788456f, kInvSqrt2Pi = 0.39894228f, kGeluCubic = 0.044715f;

// The branch on the activation is taken once for N values.  (relu keeps NaN.)
template <int N>
__device__ __forceinline__ void act_values(int act, float (&v)[N]) {
  switch (act) {
    case GRIM_ACT_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
      break;
    case GRIM_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] *= inverse(1.f + exp2_(v[i] * -kLog2e));
      break;
    case GRIM_ACT_GELU:
#pragma unroll
      for (int i = 0; i < N; ++i) { float e; v[i] *= normal(v[i], e); }
      break;
    case GRIM_ACT_GELU_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = 0.5f * v[i] * (1.f + tanh_(kSqrt2OverPi * fmaf(kGeluCubic * v[i] * v[i], v[i], v[i])));
      break;
    case GRIM_ACT_SIGMOID:
#pragma unroll
      for (int i = 0; i < N; ++i) { float k; sigmoid_pair(v[i], v[i], k); }
      break;
    case GRIM_ACT_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = tanh_(v[i]);
      break;
    default: break;
  }
}

// act'(p)
template <int N>
__device__ __forceinline__ void act_slopes(int act, const float (&p)[N], float (&d)[N]) {
  switch (act) {
    case GRIM_ACT_RELU:
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] = p[i] > 0.f ? 1.f : 0.f;
      break;
    case GRIM_ACT_SILU:
#pragma unroll
      for (int i = 0; i < N; ++i) {
        // q (1 + c k), c = p but no less than -88.  e = e^-c stays finite there (2^126.96), and from 2^126 on q leaves the range of
        // 1 / x and is 0: so the slope goes to 0 and does not grow with p.  NaN stays NaN.
        const float c = max_nan(p[i], -88.f), e = exp2_(c * -kLog2e), q = inverse(1.f + e);
        d[i] = q * fmaf(c, e * q, 1.f);
      }
      break;
    case GRIM_ACT_GELU:
      if constexpr (N >= 8) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          float y0, y1, e0, e1;
          normal_pair(p[i], p[i + 1], y0, y1, e0, e1);
          mul2(e0, e1, e0, e1, p[i], p[i + 1]);
          fma2(d[i], d[i + 1], e0, e1, kInvSqrt2Pi, kInvSqrt2Pi, y0, y1);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) { float e; const float phi = normal(p[i], e); d[i] = fmaf(p[i] * e, kInvSqrt2Pi, phi); }
      }
      break;
    case GRIM_ACT_GELU_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) {
        // (1 + t) / 2 + (1 - t^2) (3 a / 2 - r), a = r + 0.044715 r c^2, r = sqrt(2 / pi) c: little cancels, |a| >= |r|.  Beyond 16 the slope is 0 or 1: c is p kept within it, so that 1 - t^2 = 0 never meets an a that is infinite.
        const float c = max_nan(min_nan(p[i], 16.f), -16.f), r = kSqrt2OverPi * c, a = fmaf(kGeluCubic * c * c, r, r), t = tanh_(a);
        d[i] = fmaf(fmaf(-t, t, 1.f), fmaf(1.5f, a, -r), fmaf(0.5f, t, 0.5f));
      }
      break;
    case GRIM_ACT_SIGMOID:
#pragma unroll
      for (int i = 0; i < N; ++i) { float q, k; sigmoid_pair(p[i], q, k); d[i] = q * k; }
      break;
    case GRIM_ACT_TANH:
#pragma unroll
      for (int i = 0; i < N; ++i) { const float t = tanh_(p[i]); d[i] = fmaf(-t, t, 1.f); }
      break;
    default:
#pragma unroll
      for (int i = 0; i < N; ++i) d[i] = 1.f;
  }
}

// An element as memory holds it (float, or the bits of a bf16) and as a number.
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(unsigned short v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void narrow(float v, float& out) { out = v; }
__device__ __forceinline__ void narrow(float v, unsigned short& out) { out = __bfloat16_as_ushort(__float2bfloat16_rn(v)); }

__device__ __forceinline__ float epi_load(const void* m, int64_t at, int dtype) {
  return dtype == GRIM_F32 ? static_cast<const float*>(m)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(m)[at]);
}
__device__ __forceinline__ void epi_store(void* m, int64_t at, int dtype, float v) {
  if (dtype == GRIM_F32) static_cast<float*>(m)[at] = v;
  else static_cast<__nv_bfloat16*>(m)[at] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// What becomes of p = v (bias included) at row, column q of the output; the caller stores the result.
__device__ __forceinline__ float epilogue(const Epilogue& e, int dtype, float v, int64_t row, int64_t q) {
  float r = 0.f;
  if (e.res) r = epi_load(e.res, row * e.res_ld + q, dtype);
  if (e.pre) epi_store(e.pre, row * e.pre_ld + q, dtype, v);
  float t[1] = {v};
  act_values<1>(e.act, t);
  return e.res ? t[0] + r : t[0];
}

// Four neighbouring columns, n of them there.
__device__ __forceinline__ void epilogue4(const Epilogue& e, int dtype, float (&v)[4], int64_t row, int64_t q, int n) {
  float r[4] = {0.f, 0.f, 0.f, 0.f};
  if (e.res) {
    const int64_t at = row * e.res_ld + q;
    if (dtype == GRIM_F32 && n == 4 && reinterpret_cast<uintptr_t>(static_cast<const float*>(e.res) + at) % 16 == 0) {
      const float4 f = *reinterpret_cast<const float4*>(static_cast<const float*>(e.res) + at);
      r[0] = f.x; r[1] = f.y; r[2] = f.z; r[3] = f.w;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) r[i] = epi_load(e.res, at + i, dtype);
    }
  }
  if (e.pre) {
    const int64_t at = row * e.pre_ld + q;
    if (dtype == GRIM_F32 && n == 4 && reinterpret_cast<uintptr_t>(static_cast<float*>(e.pre) + at) % 16 == 0) {
      *reinterpret_cast<float4*>(static_cast<float*>(e.pre) + at) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) epi_store(e.pre, at + i, dtype, v[i]);
    }
  }
  act_values<4>(e.act, v);
  if (e.res) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += r[i];
  }
}

// Columns [q, q + n) of a row of the residual are on their way into L2 while the multiplies run.
__device__ __forceinline__ void residual_ahead(const SpmmArgs& a, int64_t row, int64_t q, int n) {
  const Epilogue& e = a.e;
  if (!e.res || !e.vec || row < 0 || q >= a.ncols) return;
  const unsigned esz = a.y_dtype == GRIM_F32 ? 4u : 2u, bytes = (unsigned)min((int64_t)n, a.ncols - q) * esz & ~15u;
  if (bytes) ptx::bulk_prefetch_l2(static_cast<const uint8_t*>(e.res) + (row * e.res_ld + q) * esz, bytes);
}

// A warp's 32 x 32 piece of the output, left in shared memory by row with a pitch of 33 floats (bias included).  Residual, P and Y
// go in 16-byte vectors, a warp instruction taking eight (bf16) or four (fp32) rows of 32 columns, where they are aligned and all
// columns are there.  The residual of a piece is fetched while the piece before it is worked on (the first one while the
// multiplies run): one trip to memory after the other cost 110 us at 8192^2 x 1024 in bf16, this, bias
// and gelu included, 8 (115.5 -> 123.5; the residual alone 2, gelu alone 2.5).
struct PieceRes { uint4 v[8]; };

// row: the output row of piece row `lane`, below 0 for none; q: the piece's first column, a multiple of 32.
__device__ __forceinline__ void piece_fetch(const SpmmArgs& a, PieceRes& pr, int row, int64_t q, int lane) {
  const Epilogue& e = a.e;
  if (!e.res || !e.vec || q + 31 >= a.ncols) return;
  if (a.y_dtype == GRIM_F32) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = __shfl_sync(0xffffffffu, row, i * 4 + (lane >> 3));
      if (r >= 0) pr.v[i] = *reinterpret_cast<const uint4*>(static_cast<const float*>(e.res) + r * e.res_ld + q + (lane & 7) * 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = __shfl_sync(0xffffffffu, row, i * 8 + (lane >> 2));
      if (r >= 0) pr.v[i] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(e.res) + r * e.res_ld + q + (lane & 3) * 8);
    }
  }
}

__device__ __forceinline__ void put8(void* m, int64_t at, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(m) + at) = make_uint4(two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7]));
}

__device__ __forceinline__ void piece_store(const SpmmArgs& a, PieceRes& pr, const float* piece, int row, int64_t q, int lane) {
  const Epilogue& e = a.e;
  if (e.vec && q + 31 < a.ncols) {
    if (a.y_dtype == GRIM_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int rl = i * 4 + (lane >> 3), c = (lane & 7) * 4;
        const int r = __shfl_sync(0xffffffffu, row, rl);
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = piece[rl * 33 + c + k];
        if (e.pre && r >= 0) *reinterpret_cast<float4*>(static_cast<float*>(e.pre) + r * e.pre_ld + q + c) = make_float4(v[0], v[1], v[2], v[3]);
        act_values<4>(e.act, v);
        if (e.res) {
          v[0] += __uint_as_float(pr.v[i].x); v[1] += __uint_as_float(pr.v[i].y);
          v[2] += __uint_as_float(pr.v[i].z); v[3] += __uint_as_float(pr.v[i].w);
        }
        if (r >= 0) *reinterpret_cast<float4*>(static_cast<float*>(a.Y) + r * a.y_sr + q + c) = make_float4(v[0], v[1], v[2], v[3]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int rl = i * 8 + (lane >> 2), c = (lane & 3) * 8;
        const int r = __shfl_sync(0xffffffffu, row, rl);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = piece[rl * 33 + c + k];
        if (e.pre && r >= 0) put8(e.pre, r * e.pre_ld + q + c, v);
        act_values<8>(e.act, v);
        if (e.res) {
          const uint32_t w[4] = {pr.v[i].x, pr.v[i].y, pr.v[i].z, pr.v[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) { v[2 * k] += __uint_as_float(w[k] << 16); v[2 * k + 1] += __uint_as_float(w[k] & 0xFFFF0000u); }
        }
        if (r >= 0) put8(a.Y, r * a.y_sr + q + c, v);
      }
    }
    return;
  }
  const bool there = q + lane < a.ncols;
  const int64_t c = q + lane;
#pragma unroll 1
  for (int r0 = 0; r0 < 32; r0 += 8) {
    float v[8], res[8];
    int rows[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      rows[i] = __shfl_sync(0xffffffffu, row, r0 + i);
      v[i] = piece[(r0 + i) * 33 + lane];
      res[i] = 0.f;
      if (e.res && there && rows[i] >= 0) res[i] = epi_load(e.res, rows[i] * e.res_ld + c, a.y_dtype);
    }
    if (e.pre && there) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (rows[i] >= 0) epi_store(e.pre, rows[i] * e.pre_ld + c, a.y_dtype, v[i]);
    }
    act_values<8>(e.act, v);
    if (there) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (rows[i] >= 0) epi_store(a.Y, rows[i] * a.y_sr + c, a.y_dtype, e.res ? v[i] + res[i] : v[i]);
    }
  }
}

// N rows' values of one column, one thread (neighbouring lanes hold neighbouring columns): the residuals are requested together.
// rows below 0 are none.
template <int N>
__device__ __forceinline__ void column_store(const SpmmArgs& a, float (&v)[N], const int (&rows)[N], int64_t q) {
  const Epilogue& e = a.e;
  float res[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    res[i] = 0.f;
    if (e.res && rows[i] >= 0) res[i] = epi_load(e.res, rows[i] * e.res_ld + q, a.y_dtype);
  }
  if (e.pre) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (rows[i] >= 0) epi_store(e.pre, rows[i] * e.pre_ld + q, a.y_dtype, v[i]);
  }
  act_values<N>(e.act, v);
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (rows[i] >= 0) epi_store(a.Y, rows[i] * a.y_sr + q * a.y_sq, a.y_dtype, e.res ? v[i] + res[i] : v[i]);
}

}  // namespace grim

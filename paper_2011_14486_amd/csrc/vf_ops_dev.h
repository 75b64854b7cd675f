// Device pieces that the sequence operators share: typed loads and stores of eight elements, and the
// microscaled formats.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vf.h"

namespace vfo {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// two floats -> packed bfloat16 pair, ties to even (v_cvt_pk_bf16_f32)
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ uint16_t round_bf16(float a) { return (uint16_t)pack2(a, 0.0f); }
__device__ __forceinline__ float bf16_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// Eight elements at an address that is aligned to one element only: global memory takes wide accesses at
// any alignment, so that odd widths and row distances need no path of their own.
typedef uint32_t u16x8 __attribute__((ext_vector_type(4), aligned(2)));
struct __attribute__((packed, aligned(4))) f32v4 { float v[4]; };

__device__ __forceinline__ void load8(const uint16_t *p, float (&v)[8]) {
  const u16x8 q = *reinterpret_cast<const u16x8 *>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(q[i] << 16);
    v[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float *p, float (&v)[8]) {
  const f32v4 a = reinterpret_cast<const f32v4 *>(p)[0], b = reinterpret_cast<const f32v4 *>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = a.v[i];
    v[4 + i] = b.v[i];
  }
}
__device__ __forceinline__ float load1(const uint16_t *p) { return bf16_f32(*p); }
__device__ __forceinline__ float load1(const float *p) { return *p; }
// Eight elements as they are in memory, fetched before they are needed; the last n of a row with zeros behind them.
template <typename T> struct raw8 { uint32_t w[2 * sizeof(T)]; };
__device__ __forceinline__ void fetch8(const uint16_t *p, int n, raw8<uint16_t> &r) {
  if (n >= 8) {
    const u16x8 q = *reinterpret_cast<const u16x8 *>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = q[i];
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) r.w[i] = (2 * i < n ? p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
}
__device__ __forceinline__ void fetch8(const float *p, int n, raw8<float> &r) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (n >= 4 * h + 4) {
      const f32v4 q = reinterpret_cast<const f32v4 *>(p)[h];
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[4 * h + i] = __float_as_uint(q.v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) r.w[4 * h + i] = 4 * h + i < n ? __float_as_uint(p[4 * h + i]) : 0u;
    }
  }
}
__device__ __forceinline__ void unpack8(const raw8<uint16_t> &r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(r.w[i] << 16);
    v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack8(const raw8<float> &r, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
}
// elements 0..n-1 of eight, zeros behind them
template <typename T>
__device__ __forceinline__ void load_upto8(const T *p, int n, float (&v)[8]) {
  if (n >= 8) {
    load8(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = i < n ? load1(p + i) : 0.0f;
}

__device__ __forceinline__ void store8(uint16_t *p, const float (&v)[8]) {
  u16x8 q;
#pragma unroll
  for (int i = 0; i < 4; ++i) q[i] = pack2(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<u16x8 *>(p) = q;
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
  f32v4 a, b;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a.v[i] = v[i];
    b.v[i] = v[4 + i];
  }
  reinterpret_cast<f32v4 *>(p)[0] = a;
  reinterpret_cast<f32v4 *>(p)[1] = b;
}
__device__ __forceinline__ void store1(uint16_t *p, float v) { *p = round_bf16(v); }
__device__ __forceinline__ void store1(float *p, float v) { *p = v; }
template <typename T>
__device__ __forceinline__ void store_upto8(T *p, int n, const float (&v)[8]) {
  if (n >= 8) {
    store8(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i < n) store1(p + i, v[i]);
}

// ---- scalar functions of the scan ----
__device__ __forceinline__ float silu(float x) { return x * __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
// log(1 + e^x) = max(x, 0) + log(1 + u), u = e^-|x| <= 1, by log(1 + u) = 2 artanh(s), s = u / (2 + u) <= 1 / 3: eight terms of
// s^(2 k + 1) / (2 k + 1), the first one left out 1e-9 of the sum, and no loss where u is small
__device__ __forceinline__ float softplus(float x) {
  const float u = __expf(-fabsf(x)), s = u * __builtin_amdgcn_rcpf(2.0f + u), s2 = s * s;
  float t = 2.0f / 15.0f;
  t = fmaf(t, s2, 2.0f / 13.0f);
  t = fmaf(t, s2, 2.0f / 11.0f);
  t = fmaf(t, s2, 2.0f / 9.0f);
  t = fmaf(t, s2, 2.0f / 7.0f);
  t = fmaf(t, s2, 2.0f / 5.0f);
  t = fmaf(t, s2, 2.0f / 3.0f);
  t = fmaf(t, s2, 2.0f);
  return fmaf(s, t, fmaxf(x, 0.0f));
}

// ---- microscaled formats ----
// E4M3: sign, 4 exponent bits, 3 fraction bits, largest 448 = 1.75 * 2^8; E2M1: largest 6 = 1.5 * 2^2.
template <int FMT> struct mx;
template <> struct mx<VF_E4M3> { static constexpr int emax = 8, bytes32 = 32; static constexpr float most = 448.0f; };
template <> struct mx<VF_E2M1> { static constexpr int emax = 2, bytes32 = 16; static constexpr float most = 6.0f; };

// The scale byte of a block whose largest magnitude has these bits: with the exponent field x the power
// of two below the magnitude is 2^(x - 127), so the byte is x - emax, at least 0 (a field of 0 is zero or a
// subnormal number, whose exponent is far below that); infinities and NaN have field 255 and give NaN.
template <int FMT>
__device__ __forceinline__ int scale_byte(uint32_t top) {
  const int x = (int)(top >> 23) & 255;
  const int b = x - mx<FMT>::emax;
  return x == 255 ? 255 : b < 0 ? 0 : b;
}
// Codes of eight values under a scale byte (<= 252, or 255: all codes zero, the scale says NaN).  2^(127 - byte)
// is a normal number for all of them, and the product with it is exact unless it falls below the format's
// smallest numbers by far.
template <int FMT>
__device__ __forceinline__ void codes8(const float (&v)[8], int byte, uint32_t (&out)[2]) {
  const float inv = byte == 255 ? 0.0f : __uint_as_float((uint32_t)(254 - byte) << 23);
  float q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // (the largest magnitudes of a block lie up to 2^(emax + 1) and are cut to the format's largest number)
    q[i] = fminf(fmaxf(v[i] * inv, -mx<FMT>::most), mx<FMT>::most);
    if (byte == 255) q[i] = 0.0f;
  }
  if constexpr (FMT == VF_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
      out[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], w, true);
    }
  } else {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[0], q[1], 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[2], q[3], 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[4], q[5], 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, q[6], q[7], 1.0f, 3);
    out[0] = w;
    out[1] = 0;
  }
}
// Largest magnitude of a block's 32 values, eight in each of four neighbouring lanes, as bits: magnitudes compare
// as integers, NaN above infinity above the rest.
__device__ __forceinline__ uint32_t block_top(const float (&v)[8]) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
    t = b > t ? b : t;
  }
  uint32_t o = (uint32_t)__shfl_xor((int)t, 1);
  t = o > t ? o : t;
  o = (uint32_t)__shfl_xor((int)t, 2);
  return o > t ? o : t;
}
// Quantizes chunk `c` (columns 8c .. 8c + 7) of a row; four neighbouring lanes hold one block.
template <int FMT>
__device__ __forceinline__ void quantize_chunk(const float (&v)[8], int c, bool on, uint8_t *codes_row, uint8_t *scales_row) {
  const int byte = scale_byte<FMT>(block_top(v));
  uint32_t w[2];
  codes8<FMT>(v, byte, w);
  if (!on) return;
  if constexpr (FMT == VF_E4M3) reinterpret_cast<uint2 *>(codes_row)[c] = make_uint2(w[0], w[1]);
  else reinterpret_cast<uint32_t *>(codes_row)[c] = w[0];
  if ((c & 3) == 0) scales_row[c >> 2] = (uint8_t)byte;
}

}  // namespace vfo

// Shared declarations of the matrix products of svgear_linear and its backward pass (internal).
#pragma once
#include "common.h"

namespace svgear {

// One operand of a product: rows of `pitch` elements, 16-byte aligned, whole 16-byte chunks.
struct Operand {
  const void* p;
  int64_t pitch;
};

// Strides of a [B,N,columns] tensor.
struct Rows {
  int64_t b, n;
};

// out[r][c] = sum_k Q[r][k] P[c][k], r < R rows, c < C columns, k < K. Where an operand has k contiguous, the last
// 16-byte chunk of its rows holds zeros behind the values; where it has k over rows, its last chunk is readable.
struct LinearArgs {
  Operand P, Q;
  int64_t K;
  int R, C;
  int tile;      // tile of the tile kernel: 64, 128, or (bf16) 256 rows and columns; 0: the kernel of few rows
  bool even;     // for it: rows of the operands are as the tile kernel needs them
  int splits;    // K in so many parts, each into its own slice of `partial`
  float* partial;  // [splits][R][C] or null
  // epilogue: row r is token r - b*n of batch entry b = r / n
  int n;
  const void* bias;
  const void* gate;
  const void* residual;
  void* pre;
  void* y;
  Rows gst, rst, yst;
  int act;
  bool wide;  // every row of y, gate, residual and pre, and bias, 16-byte aligned, C a multiple of 8
};

// How the contraction index lies in the operands: contiguous in both (forward), in Q alone (dx), in neither (dw).
enum { kContractBoth = 0, kContractQ = 1, kContractNone = 2 };

int launch_linear_bf16(const LinearArgs& a, int form, hipStream_t s);
int launch_linear_f32(const LinearArgs& a, int form, hipStream_t s);
// The same for few rows (kContractBoth), operands at any alignment. Up to 4 in bf16: 4 / 8 rows of 5120 by 5120 18.5 / 33 us,
// by tiles of 64 22 / 22; up to 8 in fp32, which needs no unpacking: 27 / 35 us and 42 / 42.
static inline int few_rows(svgear_dtype dt) { return dt == SVGEAR_F32 ? 8 : 4; }
int launch_linear_rows(const LinearArgs& a, svgear_dtype dt, hipStream_t s);
// y from the partial products of `splits` parts.
int launch_linear_merge(const LinearArgs& a, svgear_dtype dt, hipStream_t s);

// ---- activations, fp32
// z / (1 + e^-v): silu for v = z; for v = 2u the tanh form of gelu, since (1 + tanh u) / 2 = 1 / (1 + e^-2u)
__device__ __forceinline__ float gelu_tanh_arg(float z) {
  const float z2 = fminf(z * z, 1e30f);  // (large z: the limit is the same, and nothing is infinity times zero)
  return 1.5957691216057308f * (z + 0.044715f * z * z2);
}
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == SVGEAR_ACT_SILU) return z / (1.f + expf(-z));
  if (act == SVGEAR_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
  if (act == SVGEAR_ACT_GELU_TANH) return z / (1.f + expf(-gelu_tanh_arg(z)));
  return z;
}
// slope, and the value in `a`
__device__ __forceinline__ float act_slope(int act, float z, float& a) {
  if (act == SVGEAR_ACT_NONE) {
    a = z;
    return 1.f;
  }
  if (act == SVGEAR_ACT_GELU) {
    const float cdf = 0.5f * erfcf(-0.70710678118654752f * z);
    a = z * cdf;
    return cdf + z * (0.39894228040143268f * expf(-0.5f * z * z));
  }
  // z s(v): slope s + z s (1 - s) v', with s (1 - s) = e^-|v| / (1 + e^-|v|)^2, which loses nothing on either side
  float v = z, dv = 1.f;
  if (act == SVGEAR_ACT_GELU_TANH) {
    v = gelu_tanh_arg(z);
    dv = 1.5957691216057308f * (1.f + 0.134145f * fminf(z * z, 1e30f));
  }
  const float e = expf(-fabsf(v)), r = 1.f / (1.f + e);
  const float s = v >= 0.f ? r : e * r;
  a = z * s;
  return s + z * (e * r * r) * dv;
}

template <typename T>
__device__ __forceinline__ float load_as_f32(const T* p);
template <>
__device__ __forceinline__ float load_as_f32<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_as_f32<bf16_t>(const bf16_t* p) { return bf16_to_f32(*p); }

// Eight consecutive elements, 16-byte aligned.
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
  v[4] = __uint_as_float(u.z << 16), v[5] = __uint_as_float(u.z & 0xffff0000u);
  v[6] = __uint_as_float(u.w << 16), v[7] = __uint_as_float(u.w & 0xffff0000u);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
}

// The epilogue of one element.
template <typename T>
__device__ __forceinline__ void finish1(const LinearArgs& a, const T* bias, const T* gate, const T* res, T* pre, T* y, float v) {
  if (bias) v += load_as_f32(bias);
  if (pre) store1(pre, v);
  if (a.act != SVGEAR_ACT_NONE) v = act_value(a.act, v);
  if (gate) v *= load_as_f32(gate);
  if (res) v += load_as_f32(res);
  store1(y, v);
}

// The epilogue of eight consecutive columns c.. of row r (those < C; wide: all of them are, c is a multiple of 8).
template <typename T>
__device__ __forceinline__ void finish8(const LinearArgs& a, int r, int c, float (&v)[8]) {
  const int b = a.n >= a.R ? 0 : r / a.n, t = r - b * a.n;
  T* y = static_cast<T*>(a.y) + (int64_t)b * a.yst.b + (int64_t)t * a.yst.n + c;
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + (int64_t)b * a.gst.b + (int64_t)t * a.gst.n + c : nullptr;
  const T* res = a.residual ? static_cast<const T*>(a.residual) + (int64_t)b * a.rst.b + (int64_t)t * a.rst.n + c : nullptr;
  T* pre = a.pre ? static_cast<T*>(a.pre) + (int64_t)r * a.C + c : nullptr;
  const T* bias = a.bias ? static_cast<const T*>(a.bias) + c : nullptr;
  float w[8];
  if (a.wide) {
    if (bias) {
      load8(bias, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
    if (pre) store8(pre, v);
    if (a.act != SVGEAR_ACT_NONE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = act_value(a.act, v[i]);
    }
    if (gate) {
      load8(gate, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    if (res) {
      load8(res, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += w[i];
    }
    store8(y, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < a.C) finish1<T>(a, bias ? bias + i : nullptr, gate ? gate + i : nullptr, res ? res + i : nullptr, pre ? pre + i : nullptr, y + i, v[i]);
}

template <typename T>
__device__ __forceinline__ void finish1(const LinearArgs& a, int r, int c, float v) {
  const int b = a.n >= a.R ? 0 : r / a.n, t = r - b * a.n;
  finish1<T>(a, a.bias ? static_cast<const T*>(a.bias) + c : nullptr,
             a.gate ? static_cast<const T*>(a.gate) + (int64_t)b * a.gst.b + (int64_t)t * a.gst.n + c : nullptr,
             a.residual ? static_cast<const T*>(a.residual) + (int64_t)b * a.rst.b + (int64_t)t * a.rst.n + c : nullptr,
             a.pre ? static_cast<T*>(a.pre) + (int64_t)r * a.C + c : nullptr,
             static_cast<T*>(a.y) + (int64_t)b * a.yst.b + (int64_t)t * a.yst.n + c, v);
}

// Eight consecutive columns of a part's product.
__device__ __forceinline__ void store_partial8(const LinearArgs& a, int64_t part, int r, int c, const float (&v)[8]) {
  float* o = a.partial + (part * a.R + r) * a.C + c;
  if (a.C % 8 == 0) {
    store8(o, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < a.C) o[i] = v[i];
  }
}

}  // namespace svgear

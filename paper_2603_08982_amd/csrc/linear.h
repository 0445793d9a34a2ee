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
  int tile;      // tile of the tile kernel: 64, 128, or (bf16) 256 rows and columns, (fp32) 32 rows of 128; 0: the kernel of few rows
  bool by_element;  // the tile kernel copies P by the fp32 element (rows of any alignment and length); tiles of 32 and 64 rows only
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
};

// How the contraction index lies in the operands: contiguous in both (forward), in Q alone (dx), in neither (dw).
enum { kContractBoth = 0, kContractQ = 1, kContractNone = 2 };

int launch_linear_bf16(const LinearArgs& a, int form, hipStream_t s);
int launch_linear_f32(const LinearArgs& a, int form, hipStream_t s);
// The same for few rows (kContractBoth), operands at any alignment. Up to 4 in bf16: 4 / 8 rows of 5120 by 5120 16.7 / 22.9 us,
// by tiles of 64 18.7 / 19.0; up to 8 in fp32: 27 / 35 us and 41 / 41.
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
// e^x and 1/x. For bf16 results the hardware's exponential of x log2(e) and its reciprocal: off by 2^-17 where x is near 88,
// by 2^-22 around 0, beside the 2^-8 of the result's rounding (of dz too, in front of the sums of dbias and dgate, which are
// rounded so themselves); a third of the instructions.
template <typename T>
__device__ __forceinline__ float act_exp(float x) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(x * 1.44269504f);
  return expf(x);
}
template <typename T>
__device__ __forceinline__ float act_inverse(float x) {
  if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(x);
  return 1.f / x;
}
template <typename T>
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == SVGEAR_ACT_SILU) return z * act_inverse<T>(1.f + act_exp<T>(-z));
  if (act == SVGEAR_ACT_GELU) return 0.5f * z * erfcf(-0.70710678118654752f * z);
  if (act == SVGEAR_ACT_GELU_TANH) return z * act_inverse<T>(1.f + act_exp<T>(-gelu_tanh_arg(z)));
  return z;
}
// slope, and the value in `a`
template <typename T>
__device__ __forceinline__ float act_slope(int act, float z, float& a) {
  if (act == SVGEAR_ACT_NONE) {
    a = z;
    return 1.f;
  }
  if (act == SVGEAR_ACT_GELU) {
    const float cdf = 0.5f * erfcf(-0.70710678118654752f * z);
    a = z * cdf;
    return __builtin_fmaf(z, 0.39894228040143268f * act_exp<T>(-0.5f * z * z), cdf);
  }
  // z s(v): slope s + z s (1 - s) v', with s (1 - s) = e^-|v| / (1 + e^-|v|)^2, which loses nothing on either side
  float v = z, dv = 1.f;
  if (act == SVGEAR_ACT_GELU_TANH) {
    v = gelu_tanh_arg(z);
    dv = 1.5957691216057308f * __builtin_fmaf(0.134145f, fminf(z * z, 1e30f), 1.f);
  }
  const float e = act_exp<T>(-fabsf(v)), r = act_inverse<T>(1.f + e);
  const float s = v >= 0.f ? r : e * r;
  a = z * s;
  return __builtin_fmaf(z * (e * r * r), dv, s);
}

template <typename T>
__device__ __forceinline__ float load_as_f32(const T* p);
template <>
__device__ __forceinline__ float load_as_f32<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_as_f32<bf16_t>(const bf16_t* p) { return bf16_to_f32(*p); }

// 16 bytes at the alignment of their elements: global memory is read and written 16 bytes a lane at any address (rows of odd
// lengths by the element instead: 1,541 x 2,103 of 1,003 with a full epilogue in bf16 52 us, 31 this way; 1 x 5,001 of 1,003 11.5 and 8.5;
// 3 x 3,001 of 5,121 39 and 15).
typedef float float4_any __attribute__((ext_vector_type(4), aligned(4), may_alias));
typedef uint32_t uint4_any __attribute__((ext_vector_type(4), aligned(2), may_alias));
__device__ __forceinline__ uint4 load16(const void* p) {
  const uint4_any u = *static_cast<const uint4_any*>(p);
  return make_uint4(u.x, u.y, u.z, u.w);
}

// Eight consecutive elements.
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4_any a = *reinterpret_cast<const float4_any*>(p), b = *reinterpret_cast<const float4_any*>(p + 4);
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) {
  const uint4 u = load16(p);
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
  v[4] = __uint_as_float(u.z << 16), v[5] = __uint_as_float(u.z & 0xffff0000u);
  v[6] = __uint_as_float(u.w << 16), v[7] = __uint_as_float(u.w & 0xffff0000u);
}
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f32_to_bf16(v); }
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4_any*>(p) = float4_any{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<float4_any*>(p + 4) = float4_any{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<uint4_any*>(p) = uint4_any{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7])};
}

// Eight consecutive elements as they lie in memory.
template <typename T>
struct Eight;
template <>
struct Eight<bf16_t> {
  uint4 u;
  __device__ __forceinline__ void load(const bf16_t* p) { u = load16(p); }
  __device__ __forceinline__ float get(int i) const {
    const uint32_t w = i < 2 ? u.x : i < 4 ? u.y : i < 6 ? u.z : u.w;
    return __uint_as_float((i & 1) ? (w & 0xffff0000u) : (w << 16));
  }
};
template <>
struct Eight<float> {
  float v[8];
  __device__ __forceinline__ void load(const float* p) { load8(p, v); }
  __device__ __forceinline__ float get(int i) const { return v[i]; }
};

// Element offsets of row r: token t of batch entry b.
struct Place {
  int64_t y, gate, res;
  Place() = default;
  __device__ __forceinline__ Place(const LinearArgs& a, int r) {
    const int b = a.n >= a.R ? 0 : r / a.n, t = r - b * a.n;
    y = (int64_t)b * a.yst.b + (int64_t)t * a.yst.n;
    gate = (int64_t)b * a.gst.b + (int64_t)t * a.gst.n;
    res = (int64_t)b * a.rst.b + (int64_t)t * a.rst.n;
  }
};

// The epilogue of one element.
template <typename T>
__device__ __forceinline__ void finish1(const LinearArgs& a, int r, int c, float v) {
  const Place p(a, r);
  if (a.bias) v += load_as_f32(static_cast<const T*>(a.bias) + c);
  if (a.pre) store1(static_cast<T*>(a.pre) + (int64_t)r * a.C + c, v);
  if (a.act != SVGEAR_ACT_NONE) v = act_value<T>(a.act, v);
  if (a.gate) v *= load_as_f32(static_cast<const T*>(a.gate) + p.gate + c);
  if (a.residual) v += load_as_f32(static_cast<const T*>(a.residual) + p.res + c);
  store1(static_cast<T*>(a.y) + p.y + c, v);
}

// The epilogue of eight consecutive columns c.. of row r, all of them < C.
template <typename T>
__device__ __forceinline__ void finish8(const LinearArgs& a, int r, int c, float (&v)[8], const float (&bias)[8]) {
  const Place p(a, r);
  Eight<T> gate, res;
  if (a.gate) gate.load(static_cast<const T*>(a.gate) + p.gate + c);
  if (a.residual) res.load(static_cast<const T*>(a.residual) + p.res + c);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] += bias[i];
  if (a.pre) store8(static_cast<T*>(a.pre) + (int64_t)r * a.C + c, v);
  if (a.act != SVGEAR_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_value<T>(a.act, v[i]);
  }
  if (a.gate) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= gate.get(i);
  }
  if (a.residual) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += res.get(i);
  }
  store8(static_cast<T*>(a.y) + p.y + c, v);
}

// Eight consecutive columns of a part's product.
__device__ __forceinline__ void store_partial8(const LinearArgs& a, int64_t part, int r, int c, const float (&v)[8]) {
  float* o = a.partial + (part * a.R + r) * a.C + c;
  if (c + 8 <= a.C) {
    store8(o, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < a.C) o[i] = v[i];
  }
}

}  // namespace svgear

// Shared declarations of dense attention with masks and its backward pass (internal).
#pragma once
#include "common.h"

namespace svgear {

// Division of 0 <= n < 2^31 by a number that a launch has once: n / d = (2 n mul / 2^32) / 2^shift with mul = 2^(31 + shift) / d rounded
// up, 2^shift >= d, exact, since what the rounding adds, n / 2^(31 + shift) at most, is below 1 / d of the quotient. (A workgroup divides
// eight times before it knows its first address; the instructions of a division are some twenty, one waiting for the other.)
struct Divider {
  uint32_t mul = 1u << 31;
  int shift = 0;
  Divider() = default;
  explicit Divider(int d) {
    while (((int64_t)1 << shift) < d) ++shift;
    mul = (uint32_t)((((uint64_t)1 << (31 + shift)) + d - 1) / d);
  }
  friend __device__ __forceinline__ int operator/(int n, const Divider& d) { return (int)(__umulhi(2u * (unsigned)n, d.mul) >> d.shift); }
};

// Queries of the H / Hk heads that share a key head are one run of rows: row r of key head hk is token r / G of head
// hk G + r % G, G = H / Hk. Rows of a document see the keys [0, hi) of it, hi growing with the token (see Rows below).
struct DenseArgs {
  const void* q;
  const void* k;
  const void* v;
  const void* dy;
  void* o;  // dq in the backward pass
  void* dk;
  void* dv;
  float* lse;           // forward: out or null
  const float* lse_in;  // backward
  float* delta;         // [B,H,Nq]: sum over d of dy o
  Strides qst, kst, vst, yst, ost, dkst, dvst;
  const int32_t* q_offsets;  // [B or 1, n_docs + 1], or null: one document of all rows
  const int32_t* k_offsets;
  const int32_t* prefix;  // [B or 1, n_docs] or null
  const float* slopes;    // [H] or null
  int n_docs;
  bool docs_shared, causal;
  float scale, cap;
  int B, H, Hk, G, Nq, Nk;
  Divider by_hk, by_g, by_slots, by_splits;
  int slots, splits;  // tiles a key head has at most, parts that the other side's rows are cut into
  float* part;        // where splits > 1: [splits][B Hk rows][d] (dk, then dv in the backward pass)
  float2* part_ml;    // forward: maximum and sum of each
  int32_t* marks;     // with a causal mask: [splits][B Hk][slots][4], see dense_again.hip
};

constexpr int kDenseWaves = 4;
constexpr int kDenseRows = 32 * kDenseWaves;  // rows (queries, or keys for their gradients) of a workgroup in bf16

// Tiles of `per` rows that `rows` rows in n_docs documents (0: not cut) take at most: a document starts a tile, and so do the
// rows before the first and behind the last document.
static inline int64_t dense_slots(int64_t rows, int n_docs, int per) { return n_docs ? rows / per + n_docs + 2 : ceil_div(rows, per); }

enum { kDenseForward = 0, kDenseDq = 1, kDenseDkv = 2 };
int launch_dense_bf16(const DenseArgs& a, int d, hipStream_t s);
int launch_dense_f32(const DenseArgs& a, int d, hipStream_t s);
int launch_dense_backward_bf16(const DenseArgs& a, int d, int what, hipStream_t s);
int launch_dense_backward_far_cap(const DenseArgs& a, int d, int what, hipStream_t s);  // (bf16, with caps over kFarCap)
int launch_dense_backward_f32(const DenseArgs& a, int d, int what, hipStream_t s);
// The rows that a causal launch of `what` has marked, once their parts are joined.
int launch_dense_again(const DenseArgs& a, svgear_dtype dt, int d, int what, hipStream_t s);

}  // namespace svgear

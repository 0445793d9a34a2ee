// Kernels of dense attention with masks and of its gradients, for both types.
//
//   x_ij = log2(e) (cap tanh(scale q_i k_j / cap) - slope |p_i - j|), p_ij = 2^(x_ij - m_i), o_i = sum_j p_ij v_j / sum_j p_ij
//   backward: p_ij = e^(s_ij - lse_i), ds_ij = p_ij (dy_i v_j - dy_i o_i) (1 - tanh^2),
//   dq_i = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i, dv_j = sum_i p_ij dy_i
//
// A wave owns 32 rows (queries; keys for dk and dv) as columns of the matrix products, in registers, and the workgroup's four
// waves share tiles of the other side's rows, which go from global memory straight into LDS, the next under the present one:
//   X^T = tile columns^T  (32 x 32: a register holds tile rows 8 (r / 4) + 4 (lane / 32) + r % 4 of column lane % 32)
//   acc^T += tile^T X     (those registers are operands as they stand; bf16 reads the tile transposed with ds_read_b64_tr_b16)
// No atomics: dq is made by a pass over the keys, dk and dv by one over the queries, which finds the scores again (7 products
// instead of 5); where one side has few rows, the other is cut into parts that are added in a fixed order.
#pragma once
#include <type_traits>

#include "dense_attention.h"

namespace svgear {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16* lds_v4i16_ptr;

__device__ __forceinline__ bf16x8 as_bf16x8(uint4 v) {
  union { uint4 u; bf16x8 b; } c;
  c.u = v;
  return c.b;
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)(p);
}
// value held by lane ^ 32
__device__ __forceinline__ float swap32(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ float uniform(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
// A pointer that all lanes share, in scalar registers.
__device__ __forceinline__ const void* uniform_ptr(const void* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const void*>(((uint64_t)hi << 32) | lo);
}

__device__ __forceinline__ void clear(f32x16& v) {
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = 0.f;
}

// Tile row that register r of a product holds in lane half lh.
__device__ __forceinline__ int row_of(int r, int lh) { return 8 * (r >> 2) + 4 * lh + (r & 3); }

// ---- tiles in LDS and the products with them
// The 16-byte chunks of row r are permuted by XOR with swz(r), so that 16 rows of one chunk (the plain reads) and 4 rows of
// four chunks (the transposed reads) both lie in different banks.
template <typename T, int D, int BLOCKS = sizeof(T) == 2 ? 2 : 1>
struct Tile {
  static constexpr bool kHalf = sizeof(T) == 2;
  static constexpr int kBlocks = BLOCKS;  // of 32 rows
  static constexpr int kRows = 32 * kBlocks;
  static constexpr int kRowBytes = D * (int)sizeof(T);
  static constexpr int kBytes = kRows * kRowBytes;
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kRowsPerCopy = 64 / kChunks;
  static constexpr int kCopies = kRows / kRowsPerCopy / kDenseWaves;  // of a wave
  static constexpr int DB = D / 32;

  static __device__ __forceinline__ int swz(int r) {
    if constexpr (!kHalf) return r & (kChunks - 1);
    else if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return ((r & 2) << 1) | ((r >> 2) & 3);
  }

  // a row of 32 columns, in registers: operand of X
  struct Column {
    std::conditional_t<kHalf, bf16x8, float4> v[kHalf ? D / 16 : D / 8];
    __device__ __forceinline__ void load(const T* row, int lh) {
#pragma unroll
      for (int s = 0; s < (kHalf ? D / 16 : D / 8); ++s) {
        if constexpr (kHalf) v[s] = as_bf16x8(*reinterpret_cast<const uint4*>(row + 16 * s + 8 * lh));
        else v[s] = *reinterpret_cast<const float4*>(row + lh * (D / 2) + 4 * s);
      }
    }
  };

  int row_off, tr_off;  // this lane's first operands of the plain and of the transposed reads
  __device__ __forceinline__ Tile(int lane) {
    const int li = lane & 31, lh = lane >> 5;
    if constexpr (kHalf) {
      row_off = li * kRowBytes + ((lh ^ swz(li)) << 4);
      const int r = lane & 15, g = lane >> 4, row = 4 * (g >> 1) + (r >> 2);
      tr_off = row * kRowBytes + (((2 * (g & 1) + ((r & 3) >> 1)) ^ swz(row)) << 4) + (r & 1) * 8;
    } else {
      row_off = li * kRowBytes + (((lh * (kChunks / 2)) ^ swz(li)) << 4);
      tr_off = 0;
    }
  }

  // X^T of block kb of a tile
  __device__ __forceinline__ void rows_times(const unsigned char* tile, int kb, const Column& c, f32x16& x) const {
    const unsigned char* t = tile + kb * 32 * kRowBytes;
    if constexpr (kHalf) {
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*reinterpret_cast<const uint4*>(t + (row_off ^ (s << 5)))), c.v[s], x, 0, 0, 0);
    } else {
#pragma unroll
      for (int s = 0; s < D / 8; ++s) {
        const float4 a = *reinterpret_cast<const float4*>(t + (row_off ^ (s << 4)));
        x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, c.v[s].x, x, 0, 0, 0);
        x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, c.v[s].y, x, 0, 0, 0);
        x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, c.v[s].z, x, 0, 0, 0);
        x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, c.v[s].w, x, 0, 0, 0);
      }
    }
  }

  // the same with the columns in LDS, each lane's operands where it put them (see park)
  static constexpr int kParked = 32 * kRowBytes;  // bytes of a wave
  static __device__ __forceinline__ void park(unsigned char* to, const Column& c, int lane) {
#pragma unroll
    for (int s = 0; s < kParked / 1024; ++s) *reinterpret_cast<std::conditional_t<kHalf, bf16x8, float4>*>(to + s * 1024 + lane * 16) = c.v[s];
  }
  __device__ __forceinline__ void rows_times(const unsigned char* tile, int kb, const unsigned char* parked, f32x16& x, int lane) const {
    static_assert(kHalf, "bf16 columns alone are parked");
    const unsigned char* t = tile + kb * 32 * kRowBytes;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*reinterpret_cast<const uint4*>(t + (row_off ^ (s << 5)))),
                                                  as_bf16x8(*reinterpret_cast<const uint4*>(parked + s * 1024 + lane * 16)), x, 0, 0, 0);
  }

  // acc^T += block kb of a tile, transposed, times X (bf16: rounded to it)
  __device__ __forceinline__ void transposed_times(const unsigned char* tile, int kb, const f32x16& x, f32x16 (&acc)[DB], int lane) const {
    const unsigned char* t = tile + kb * 32 * kRowBytes;
    if constexpr (kHalf) {
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        const bf16x8 b = as_bf16x8(make_uint4(pack2_bf16(x[8 * ks], x[8 * ks + 1]), pack2_bf16(x[8 * ks + 2], x[8 * ks + 3]),
                                              pack2_bf16(x[8 * ks + 4], x[8 * ks + 5]), pack2_bf16(x[8 * ks + 6], x[8 * ks + 7])));
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const int off = tr_off ^ (db << 6);
          union { struct { v4i16 a, b; } s; bf16x8 v; } u;
          u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(t + ks * 16 * kRowBytes + off));
          u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(t + (ks * 16 + 8) * kRowBytes + (off ^ 32)));
          acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(u.v, b, acc[db], 0, 0, 0);
        }
      }
    } else {
      // columns DB i .. of row i of the accumulators, so that a lane reads what it needs of a tile row at once
      const int li = lane & 31, lh = lane >> 5;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int row = row_of(r, lh);
        if constexpr (DB == 4) {
          const float4 a = *reinterpret_cast<const float4*>(t + row * kRowBytes + ((li ^ swz(row)) << 4));
          acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, x[r], acc[0], 0, 0, 0);
          acc[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, x[r], acc[1], 0, 0, 0);
          acc[2] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, x[r], acc[2], 0, 0, 0);
          acc[3] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, x[r], acc[3], 0, 0, 0);
        } else {
          const float2 a = *reinterpret_cast<const float2*>(t + row * kRowBytes + (((li >> 1) ^ swz(row)) << 4) + (li & 1) * 8);
          acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, x[r], acc[0], 0, 0, 0);
          acc[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, x[r], acc[1], 0, 0, 0);
        }
      }
    }
  }

  // f(first of four columns, their values) for what the lane's accumulators hold of its row
  template <typename F>
  static __device__ __forceinline__ void each_four(const f32x16 (&acc)[DB], int lh, F f) {
    if constexpr (kHalf) {
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          f(32 * db + 8 * g + 4 * lh, make_float4(acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]));
    } else if constexpr (DB == 4) {
#pragma unroll
      for (int r = 0; r < 16; ++r) f(4 * row_of(r, lh), make_float4(acc[0][r], acc[1][r], acc[2][r], acc[3][r]));
    } else {
#pragma unroll
      for (int r = 0; r < 16; r += 2) f(2 * row_of(r, lh), make_float4(acc[0][r], acc[1][r], acc[0][r + 1], acc[1][r + 1]));
    }
  }
};

__device__ __forceinline__ void store_four(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store_four(bf16_t* p, float4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack2_bf16(v.x, v.y), pack2_bf16(v.z, v.w));
}

// Rows of a tensor as 16-byte chunks of lanes: row `at` of tile rows from `first` on, those behind `last` as `last`.
// (32-bit offsets within a tile: the entry points hold strides to what that takes.)
template <typename Z, typename T, typename RowOffset>
__device__ __forceinline__ void copy_tile(const T* base, uint32_t lds, int wave, int lane, RowOffset offset) {
#pragma unroll
  for (int i = 0; i < Z::kCopies; ++i) {
    const int inst = i * kDenseWaves + wave, row = inst * Z::kRowsPerCopy + lane / Z::kChunks;
    const int chunk = (lane % Z::kChunks) ^ Z::swz(row);
    async_copy_16B(base + offset(row) + chunk * (16 / (int)sizeof(T)), (uint32_t)uniform((int)(lds + inst * 1024)));
  }
}

// ---- documents and masks
__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return min(max(v, lo), hi); }

// The tile that slot t of batch entry b stands for: rows [first, end) of document doc (-1: rows of no document).
struct Place {
  int first, end, doc;
};
// Document c's tiles begin at slot floor(start_c rows / per) + c, which leaves room for what precedes it and needs no list; rows
// before the first and behind the last document count as documents. Lanes look at 64 documents at once. Offsets out of range
// are taken as the nearest in range.
__device__ __forceinline__ Place place_of(const int32_t* offsets, int n_docs, int N, int G, int per, int t, int lane) {
  if (!offsets) return {t * per, N * G, 0};
  const int all = n_docs + 2;
  int c = -1;
  for (int c0 = 0; c0 < all; c0 += 64) {
    const int i = c0 + lane;
    bool before = false;
    if (i < all) {
      const int start = i == 0 ? 0 : clamp_to(offsets[i - 1], 0, N);
      before = (int64_t)start * G / per + i <= t;
    }
    const unsigned long long votes = __ballot(before);
    c += __popcll(votes);
    if (votes != ~0ull) break;
  }
  c = max(c, 0);
  const int start = c == 0 ? 0 : clamp_to(offsets[c - 1], 0, N), end = c == all - 1 ? N : clamp_to(offsets[c], 0, N);
  Place p;
  const int64_t first = (int64_t)start * G + (t - ((int64_t)start * G / per + c)) * per;
  p.first = uniform((int)(first < 0 ? 0 : first < INT32_MAX ? first : INT32_MAX));
  p.end = uniform(end * G);
  p.doc = uniform(c >= 1 && c <= n_docs ? c - 1 : -1);
  return p;
}

// A document: its first query and key, how many of each, and what each query sees.
struct Document {
  int q0, nq, k0, nk, prefix;
  bool causal;
  __device__ __forceinline__ explicit Document(const DenseArgs& a) : causal(a.causal) {}
  __device__ __forceinline__ Document(const DenseArgs& a, int b, int doc) {
    const int64_t row = a.docs_shared ? 0 : b;
    q0 = 0, nq = a.Nq, k0 = 0, nk = a.Nk, prefix = 0;
    causal = a.causal;
    if (doc < 0) {
      nq = nk = 0;
      return;
    }
    if (a.q_offsets) {
      const int32_t* o = a.q_offsets + row * (a.n_docs + 1) + doc;
      q0 = clamp_to(o[0], 0, a.Nq);
      nq = clamp_to(o[1], q0, a.Nq) - q0;
    }
    if (a.k_offsets) {
      const int32_t* o = a.k_offsets + row * (a.n_docs + 1) + doc;
      k0 = clamp_to(o[0], 0, a.Nk);
      nk = clamp_to(o[1], k0, a.Nk) - k0;
    }
    if (a.prefix) prefix = clamp_to(a.prefix[row * a.n_docs + doc], 0, nk);
    q0 = uniform(q0), nq = uniform(nq), k0 = uniform(k0), nk = uniform(nk), prefix = uniform(prefix);
  }
  // where the document's query i stands among its keys: the last query at the last key
  __device__ __forceinline__ int position(int i) const { return i + nk - nq; }
  // query i sees the keys [0, seen(i)), which grows with i
  __device__ __forceinline__ int seen(int i) const { return causal ? clamp_to(max(prefix, position(i) + 1), 0, nk) : nk; }
  // key j is seen by the queries [first_seer(j), nq), which grows with j
  __device__ __forceinline__ int first_seer(int j) const { return causal && j >= prefix ? max(j - (nk - nq), 0) : 0; }
};

// Workgroup to (key head of the batch, slot): consecutive logical indexes, which share keys or queries, on one XCD.
__device__ __forceinline__ bool dense_index(const DenseArgs& a, int& bh, int& slot) {
  const unsigned total = (unsigned)(a.B * a.Hk) * (unsigned)a.slots, per = (total + 7) / 8, wg = long_grid_index();
  const unsigned logical = (wg & 7) * per + (wg >> 3);
  if ((wg >> 3) >= per || logical >= total) return false;
  bh = (int)(logical / (unsigned)a.slots);
  slot = (int)(logical - (unsigned)bh * (unsigned)a.slots);
  return true;
}

// tanh from the hardware's exponential and reciprocal. For bf16 1 - 2 / (e^2x + 1), off by some 2^-23 of 1, which moves a score of
// cap 50 by 1e-5 beside the 2^-9 that its weight's rounding is off by. For fp32 (1 - e) / (1 + e) with e = e^-2|x|, and below 0.3,
// where 1 - e would lose digits, the series, whose next term is 3e-9 of the result there.
template <typename T>
__device__ __forceinline__ float tanh_of(float x) {
  if constexpr (sizeof(T) == 2) {
    return 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * (2.f * kLog2e)) + 1.f);
  } else {
    const float a = fabsf(x), e = __builtin_amdgcn_exp2f(a * (-2.f * kLog2e)), z = x * x;
    const float far = copysignf((1.f - e) * __builtin_amdgcn_rcpf(1.f + e), x);
    float p = __builtin_fmaf(z, 0.0035921280f, -0.0088632356f);
    p = __builtin_fmaf(z, p, 0.0218694885f);
    p = __builtin_fmaf(z, p, -0.0539682540f);
    p = __builtin_fmaf(z, p, 0.1333333333f);
    p = __builtin_fmaf(z, p, -0.3333333333f);
    return a < 0.3f ? __builtin_fmaf(x * z, p, x) : far;
  }
}

// Products to exponents of 2, of a query at `dist` from the key. The cap's derivative is 1 - tanh^2.
template <typename T, bool CAP, bool SLOPES>
struct Scores {
  float c, cap2;
  __device__ __forceinline__ Scores(const DenseArgs& a) : c(CAP ? a.scale / a.cap : a.scale * kLog2e), cap2(a.cap * kLog2e) {}
  // tanh (or the product itself)
  __device__ __forceinline__ float inner(float s) const { return CAP ? tanh_of<T>(s * c) : s; }
  // exponent less `less`
  __device__ __forceinline__ float outer(float in, float dist, float slope, float less) const {
    if (SLOPES) less = __builtin_fmaf(slope, fabsf(dist), less);
    return __builtin_fmaf(in, CAP ? cap2 : c, -less);
  }
  __device__ __forceinline__ float keeps(float in) const { return __builtin_fmaf(-in, in, 1.f); }
};

// ---- forward: 128 queries a workgroup
template <typename T, int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, 2)
dense_forward_kernel(DenseArgs a) {
  using Z = Tile<T, D>;
  constexpr int DB = D / 32, BN = Z::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes];  // two of K, two of V
  int bh, slot;
  if (!dense_index(a, bh, slot)) return;
  if (a.causal) slot = a.slots - 1 - slot;  // the longest first
  const int b = bh / a.Hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const int32_t* qo = a.q_offsets ? a.q_offsets + (a.docs_shared ? 0 : (int64_t)b * (a.n_docs + 1)) : nullptr;
  const Place at = place_of(qo, a.n_docs, a.Nq, a.G, kDenseRows, slot, lane);
  if (at.first >= at.end) return;
  const Document doc(a, b, at.doc);

  const int wave_row = at.first + 32 * wave, row = wave_row + li, row_c = min(row, at.end - 1);
  const bool active = wave_row < at.end;
  const int token = row_c / a.G, head = hk * a.G + (row_c - token * a.G);
  const int pos = doc.position(token - doc.q0), hi = doc.seen(token - doc.q0);
  // keys that every row of this wave sees, that some row of it sees, and of the workgroup
  const int hi_all = doc.seen(min(wave_row, at.end - 1) / a.G - doc.q0), hi_any = doc.seen(min(wave_row + 31, at.end - 1) / a.G - doc.q0);
  const int hi_wg = doc.seen((min(at.first + kDenseRows, at.end) - 1) / a.G - doc.q0);
  const int split = blockIdx.y, tiles = (hi_wg + BN - 1) / BN;
  const int t_lo = (int)((int64_t)tiles * split / a.splits), t_hi = (int)((int64_t)tiles * (split + 1) / a.splits);

  typename Z::Column q;
  q.load(static_cast<const T*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n, lh);
  const float slope = SLOPES ? a.slopes[head] * kLog2e : 0.f;
  SVGEAR_WAIT_VMCNT(0);  // (the copies below are not seen by the compiler, which would wait for them inside the loop)

  const Z z(lane);
  const Scores<T, CAP, SLOPES> scores(a);
  const uint32_t lds = lds_address(smem);
  const T* kp = static_cast<const T*>(a.k) + b * a.kst.b + hk * a.kst.h + doc.k0 * a.kst.n;
  const T* vp = static_cast<const T*>(a.v) + b * a.vst.b + hk * a.vst.h + doc.k0 * a.vst.n;
  auto issue = [&](int t) __attribute__((always_inline)) {
    const int last = hi_wg - 1 - t * BN;  // (keys that no row here sees are not read)
    copy_tile<Z>(kp + (int64_t)t * BN * a.kst.n, lds + (t & 1) * Z::kBytes, wave, lane,
                    [&](int r) { return (int64_t)min(r, last) * a.kst.n; });
    copy_tile<Z>(vp + (int64_t)t * BN * a.vst.n, lds + (2 + (t & 1)) * Z::kBytes, wave, lane,
                    [&](int r) { return (int64_t)min(r, last) * a.vst.n; });
  };

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(acc[db]);
  float m = -INFINITY, l = 0.f;
  if (t_lo < t_hi) issue(t_lo);
  for (int t = t_lo; t < t_hi; ++t) {
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
    if (t + 1 < t_hi) issue(t + 1);
    if (!active || t * BN >= hi_any) continue;
    const unsigned char* kt = smem + (t & 1) * Z::kBytes;
    const unsigned char* vt = smem + (2 + (t & 1)) * Z::kBytes;
    f32x16 x[Z::kBlocks];
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < Z::kBlocks; ++kb) {
      clear(x[kb]);
      z.rows_times(kt, kb, q, x[kb]);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = t * BN + 32 * kb + row_of(r, lh);
        x[kb][r] = scores.outer(scores.inner(x[kb][r]), (float)(pos - j), slope, 0.f);
      }
    }
    if ((t + 1) * BN > hi_all) {
#pragma unroll
      for (int kb = 0; kb < Z::kBlocks; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (t * BN + 32 * kb + row_of(r, lh) >= hi) x[kb][r] = -INFINITY;
    }
#pragma unroll
    for (int kb = 0; kb < Z::kBlocks; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[kb][r]);
    mx = fmaxf(mx, swap32(mx));
    if (__any(mx > m)) {
      const float m_new = fmaxf(m, mx), alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
      m = m_new;
    }
    const float m_use = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int kb = 0; kb < Z::kBlocks; ++kb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        x[kb][r] = __builtin_amdgcn_exp2f(x[kb][r] - m_use);
        l += x[kb][r];
      }
      z.transposed_times(vt, kb, x[kb], acc, lane);
    }
  }

  if (!active) return;
  l += swap32(l);
  if (row >= at.end) return;
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.B * a.Hk * a.Nq * a.G, out = split * rows + (int64_t)bh * a.Nq * a.G + row;
    if (lh == 0) a.part_ml[out] = make_float2(m, l);
    Z::each_four(acc, lh, [&](int d, float4 v) { store_four(a.part + out * D + d, v); });
    return;
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  T* o = static_cast<T*>(a.o) + b * a.ost.b + head * a.ost.h + token * a.ost.n;
  Z::each_four(acc, lh, [&](int d, float4 v) { store_four(o + d, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv)); });
  if (a.lse && lh == 0) a.lse[((int64_t)b * a.H + head) * a.Nq + token] = (m + log2f(l)) * kLn2;
}

// ---- the queries' gradients: 128 queries a workgroup, a pass over the keys
template <typename T, int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, sizeof(T) == 4 && D == 128 ? 1 : 2)
dense_dq_kernel(DenseArgs a) {
  using Z = Tile<T, D>;
  constexpr int DB = D / 32, BN = Z::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes];
  int bh, slot;
  if (!dense_index(a, bh, slot)) return;
  if (a.causal) slot = a.slots - 1 - slot;
  const int b = bh / a.Hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const int32_t* qo = a.q_offsets ? a.q_offsets + (a.docs_shared ? 0 : (int64_t)b * (a.n_docs + 1)) : nullptr;
  const Place at = place_of(qo, a.n_docs, a.Nq, a.G, kDenseRows, slot, lane);
  if (at.first >= at.end) return;
  const Document doc(a, b, at.doc);

  const int wave_row = at.first + 32 * wave, row = wave_row + li, row_c = min(row, at.end - 1);
  const bool active = wave_row < at.end;
  const int token = row_c / a.G, head = hk * a.G + (row_c - token * a.G);
  const int pos = doc.position(token - doc.q0), hi = doc.seen(token - doc.q0);
  const int hi_all = doc.seen(min(wave_row, at.end - 1) / a.G - doc.q0), hi_any = doc.seen(min(wave_row + 31, at.end - 1) / a.G - doc.q0);
  const int hi_wg = doc.seen((min(at.first + kDenseRows, at.end) - 1) / a.G - doc.q0);
  const int split = blockIdx.y, tiles = (hi_wg + BN - 1) / BN;
  const int t_lo = (int)((int64_t)tiles * split / a.splits), t_hi = (int)((int64_t)tiles * (split + 1) / a.splits);

  typename Z::Column q, dy;
  q.load(static_cast<const T*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n, lh);
  dy.load(static_cast<const T*>(a.dy) + b * a.yst.b + head * a.yst.h + token * a.yst.n, lh);
  const int64_t stat = ((int64_t)b * a.H + head) * a.Nq + token;
  const float lse2 = a.lse_in[stat] * kLog2e, delta = a.delta[stat];
  const float slope = SLOPES ? a.slopes[head] * kLog2e : 0.f;
  SVGEAR_WAIT_VMCNT(0);

  const Z z(lane);
  const Scores<T, CAP, SLOPES> scores(a);
  const uint32_t lds = lds_address(smem);
  const T* kp = static_cast<const T*>(a.k) + b * a.kst.b + hk * a.kst.h + doc.k0 * a.kst.n;
  const T* vp = static_cast<const T*>(a.v) + b * a.vst.b + hk * a.vst.h + doc.k0 * a.vst.n;
  auto issue = [&](int t) __attribute__((always_inline)) {
    const int last = hi_wg - 1 - t * BN;
    copy_tile<Z>(kp + (int64_t)t * BN * a.kst.n, lds + (t & 1) * Z::kBytes, wave, lane,
                    [&](int r) { return (int64_t)min(r, last) * a.kst.n; });
    copy_tile<Z>(vp + (int64_t)t * BN * a.vst.n, lds + (2 + (t & 1)) * Z::kBytes, wave, lane,
                    [&](int r) { return (int64_t)min(r, last) * a.vst.n; });
  };

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(acc[db]);
  if (t_lo < t_hi) issue(t_lo);
  for (int t = t_lo; t < t_hi; ++t) {
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
    if (t + 1 < t_hi) issue(t + 1);
    if (!active || t * BN >= hi_any) continue;
    const unsigned char* kt = smem + (t & 1) * Z::kBytes;
    const unsigned char* vt = smem + (2 + (t & 1)) * Z::kBytes;
    const bool masked = (t + 1) * BN > hi_all;
#pragma unroll
    for (int kb = 0; kb < Z::kBlocks; ++kb) {
      f32x16 x, dp;
      clear(x);
      clear(dp);
      z.rows_times(kt, kb, q, x);
      z.rows_times(vt, kb, dy, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int j = t * BN + 32 * kb + row_of(r, lh);
        const float in = scores.inner(x[r]);
        float ds = __builtin_amdgcn_exp2f(scores.outer(in, (float)(pos - j), slope, lse2)) * (dp[r] - delta);
        if (CAP) ds *= scores.keeps(in);
        x[r] = masked && j >= hi ? 0.f : ds;
      }
      z.transposed_times(kt, kb, x, acc, lane);
    }
  }

  if (!active || row >= at.end) return;
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.B * a.Hk * a.Nq * a.G, out = split * rows + (int64_t)bh * a.Nq * a.G + row;
    Z::each_four(acc, lh, [&](int d, float4 v) { store_four(a.part + out * D + d, v); });
    return;
  }
  T* o = static_cast<T*>(a.o) + b * a.ost.b + head * a.ost.h + token * a.ost.n;
  const float f = a.scale;
  Z::each_four(acc, lh, [&](int d, float4 v) { store_four(o + d, make_float4(v.x * f, v.y * f, v.z * f, v.w * f)); });
}

// ---- the keys' and values' gradients: 128 keys a workgroup, a pass over the queries of all heads that share them
template <typename T, int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, sizeof(T) == 4 && D == 128 ? 1 : 2)
dense_dkv_kernel(DenseArgs a) {
  // Two waves a SIMD, one's exponentials under the other's products, leave 256 registers: at d = 128 in bf16 the accumulators
  // take 128 and the keys 32, and the values wait in LDS, under tiles of 32 rows.
  constexpr bool kPark = sizeof(T) == 2 && D == 128;
  using Z = Tile<T, D, kPark ? 1 : sizeof(T) == 2 ? 2 : 1>;
  constexpr int DB = D / 32, BN = Z::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes + (kPark ? kDenseWaves * Z::kParked : 0)];  // two of Q, two of dy
  __shared__ __attribute__((aligned(256))) float stats[2][4][64];  // of a tile's rows: log-sum-exp, delta, slope, position
  int bh, slot;
  if (!dense_index(a, bh, slot)) return;
  const int b = bh / a.Hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const int32_t* ko = a.k_offsets ? a.k_offsets + (a.docs_shared ? 0 : (int64_t)b * (a.n_docs + 1)) : nullptr;
  const Place at = place_of(ko, a.n_docs, a.Nk, 1, kDenseRows, slot, lane);
  if (at.first >= at.end) return;
  const Document doc(a, b, at.doc);

  const int wave_key = at.first + 32 * wave, key = wave_key + li, key_c = min(key, at.end - 1);
  const bool active = wave_key < at.end;
  // rows of the document [from, end) see key j of it; rows from `from_all` on see all keys of this wave, from from_any on one of them
  const int j = key_c - doc.k0, from = doc.first_seer(j) * a.G, end = doc.nq * a.G;
  const int from_all = doc.first_seer(min(wave_key + 31, at.end - 1) - doc.k0) * a.G;
  const int from_any = doc.first_seer(min(wave_key, at.end - 1) - doc.k0) * a.G;
  const int first_tile = doc.first_seer(at.first - doc.k0) * a.G / BN, tiles_end = (end + BN - 1) / BN;
  const int tiles = max(tiles_end - first_tile, 0), split = blockIdx.y;
  const int t_lo = first_tile + (int)((int64_t)tiles * split / a.splits), t_hi = first_tile + (int)((int64_t)tiles * (split + 1) / a.splits);

  typename Z::Column k, v;
  unsigned char* parked = smem + 4 * Z::kBytes + (kPark ? wave * Z::kParked : 0);
  k.load(static_cast<const T*>(a.k) + b * a.kst.b + hk * a.kst.h + key_c * a.kst.n, lh);
  v.load(static_cast<const T*>(a.v) + b * a.vst.b + hk * a.vst.h + key_c * a.vst.n, lh);
  if constexpr (kPark) Z::park(parked, v, lane);
  SVGEAR_WAIT_VMCNT(0);

  const Z z(lane);
  const Scores<T, CAP, SLOPES> scores(a);
  const uint32_t lds = lds_address(smem), lds_stats = lds_address(stats);
  const T* qp = static_cast<const T*>(a.q) + b * a.qst.b + hk * a.G * a.qst.h + doc.q0 * a.qst.n;
  const T* yp = static_cast<const T*>(a.dy) + b * a.yst.b + hk * a.G * a.yst.h + doc.q0 * a.yst.n;
  const int64_t stat0 = ((int64_t)b * a.H + hk * a.G) * a.Nq + doc.q0;
  auto issue = [&](int t) __attribute__((always_inline)) {
    auto offset = [&](int r, const Strides& st) {
      const int row = min(t * BN + r, end - 1), token = a.G == 1 ? row : row / a.G;
      return (row - token * a.G) * st.h + token * st.n;
    };
    copy_tile<Z>(qp, lds + (t & 1) * Z::kBytes, wave, lane, [&](int r) { return offset(r, a.qst); });
    copy_tile<Z>(yp, lds + (2 + (t & 1)) * Z::kBytes, wave, lane, [&](int r) { return offset(r, a.yst); });
    const int row = min(t * BN + lane, end - 1), token = a.G == 1 ? row : row / a.G;
    const uint32_t to = (uint32_t)uniform((int)(lds_stats + ((t & 1) * 4 + wave) * 256));
    if (wave < 2) async_copy_4B((wave == 0 ? a.lse_in : a.delta) + stat0 + (int64_t)(row - token * a.G) * a.Nq + token, to);
    if (SLOPES && wave == 2) async_copy_4B(a.slopes + hk * a.G + row - token * a.G, to);
    if (SLOPES && wave == 3) stats[t & 1][3][lane] = (float)doc.position(token);
  };

  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(dk[db]), clear(dv[db]);
  if (t_lo < t_hi) issue(t_lo);
  for (int t = t_lo; t < t_hi; ++t) {
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
    if (t + 1 < t_hi) issue(t + 1);
    if (!active || (t + 1) * BN <= from_any) continue;
    const unsigned char* qt = smem + (t & 1) * Z::kBytes;
    const unsigned char* yt = smem + (2 + (t & 1)) * Z::kBytes;
    const bool masked = t * BN < from_all || (t + 1) * BN > end;
#pragma unroll
    for (int kb = 0; kb < Z::kBlocks; ++kb) {
      f32x16 x, dp;
      clear(x);
      clear(dp);
      z.rows_times(qt, kb, k, x);
      if constexpr (kPark) z.rows_times(yt, kb, parked, dp, lane);
      else z.rows_times(yt, kb, v, dp);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        auto of_rows = [&](int what) { return *reinterpret_cast<const float4*>(&stats[t & 1][what][32 * kb + 8 * g + 4 * lh]); };
        const float4 ls = of_rows(0), de = of_rows(1);
        const float lse[4] = {ls.x, ls.y, ls.z, ls.w}, delta[4] = {de.x, de.y, de.z, de.w};
        float slope[4] = {0.f, 0.f, 0.f, 0.f}, dist[4] = {0.f, 0.f, 0.f, 0.f};
        if (SLOPES) {
          const float4 sl = of_rows(2), po = of_rows(3);
          slope[0] = sl.x * kLog2e, slope[1] = sl.y * kLog2e, slope[2] = sl.z * kLog2e, slope[3] = sl.w * kLog2e;
          dist[0] = po.x - (float)j, dist[1] = po.y - (float)j, dist[2] = po.z - (float)j, dist[3] = po.w - (float)j;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 4 * g + i, row = t * BN + 32 * kb + row_of(r, lh);
          const float in = scores.inner(x[r]);
          float p = __builtin_amdgcn_exp2f(scores.outer(in, dist[i], slope[i], lse[i] * kLog2e));
          float ds = p * (dp[r] - delta[i]);
          if (CAP) ds *= scores.keeps(in);
          if (masked && (row < from || row >= end)) p = ds = 0.f;
          x[r] = p;
          dp[r] = ds;
        }
      }
      z.transposed_times(yt, kb, x, dv, lane);
      z.transposed_times(qt, kb, dp, dk, lane);
    }
  }

  if (!active || key >= at.end) return;
  const float f = a.scale;
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.B * a.Hk * a.Nk, out = split * rows + (int64_t)bh * a.Nk + key;
    Z::each_four(dk, lh, [&](int d, float4 u) { store_four(a.part + out * D + d, make_float4(u.x * f, u.y * f, u.z * f, u.w * f)); });
    Z::each_four(dv, lh, [&](int d, float4 u) { store_four(a.part + (a.splits * rows + out) * D + d, u); });
    return;
  }
  T* ok = static_cast<T*>(a.dk) + b * a.dkst.b + hk * a.dkst.h + key * a.dkst.n;
  T* ov = static_cast<T*>(a.dv) + b * a.dvst.b + hk * a.dvst.h + key * a.dvst.n;
  Z::each_four(dk, lh, [&](int d, float4 u) { store_four(ok + d, make_float4(u.x * f, u.y * f, u.z * f, u.w * f)); });
  Z::each_four(dv, lh, [&](int d, float4 u) { store_four(ov + d, u); });
}

template <typename T, int D, bool CAP, bool SLOPES, int WHAT>
int launch_dense_mode(const DenseArgs& a, hipStream_t s) {
  const int64_t groups = ceil_div((int64_t)a.B * a.Hk * a.slots, 8) * 8;
  const dim3 grid = long_grid(groups, a.splits);
  if constexpr (WHAT == kDenseForward) dense_forward_kernel<T, D, CAP, SLOPES><<<grid, 64 * kDenseWaves, 0, s>>>(a);
  else if constexpr (WHAT == kDenseDq) dense_dq_kernel<T, D, CAP, SLOPES><<<grid, 64 * kDenseWaves, 0, s>>>(a);
  else dense_dkv_kernel<T, D, CAP, SLOPES><<<grid, 64 * kDenseWaves, 0, s>>>(a);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

template <typename T, int D, int WHAT>
int launch_dense_width(const DenseArgs& a, hipStream_t s) {
  if (a.cap > 0.f) return a.slopes ? launch_dense_mode<T, D, true, true, WHAT>(a, s) : launch_dense_mode<T, D, true, false, WHAT>(a, s);
  return a.slopes ? launch_dense_mode<T, D, false, true, WHAT>(a, s) : launch_dense_mode<T, D, false, false, WHAT>(a, s);
}
template <typename T, int WHAT>
int launch_dense(const DenseArgs& a, int d, hipStream_t s) {
  return d == 64 ? launch_dense_width<T, 64, WHAT>(a, s) : launch_dense_width<T, 128, WHAT>(a, s);
}

}  // namespace
}  // namespace svgear

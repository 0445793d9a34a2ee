// Kernels of dense attention with masks and of its gradients, for both types.
//
//   x_ij = log2(e) (cap tanh(scale q_i k_j / cap) - slope |p_i - j|), p_ij = 2^(x_ij - m_i), o_i = sum_j p_ij v_j / sum_j p_ij
//   backward: p_ij = e^(s_ij - lse_i), ds_ij = p_ij (dy_i v_j - dy_i o_i) (1 - tanh^2),
//   dq_i = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i, dv_j = sum_i p_ij dy_i
//
// A wave owns 32 rows (queries; keys for dk and dv; 64 in bf16's backward pass) as columns of the matrix products, in registers, and reads tiles of the other
// side's rows, which go from global memory straight into LDS, the next under the present one:
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

// 16 bytes of zeros in LDS: rows behind the last one of a tile that is multiplied by weights of 0, which an infinity there would not survive
__device__ __forceinline__ void clear_16B(uint32_t lds) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  uint32_t zero;
  asm volatile("v_mov_b32 %0, 0" : "=v"(zero));  // (the compiler would keep four registers of them through the loop)
  *(__attribute__((address_space(3))) u32x4*)(uintptr_t)lds = u32x4{zero, zero, zero, zero};
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
    // fp32: in accumulation registers from here on, which leaves the others to the vector unit (dk and dv at d = 128 spilled up to 38: the
    // gradients of 2 x 24 heads, 37 queries over 9,389 keys 781 us, 732 so)
    __device__ __forceinline__ void keep() {
#pragma unroll
      for (int s = 0; s < D / 8; ++s) asm volatile("" : "+a"(v[s].x), "+a"(v[s].y), "+a"(v[s].z), "+a"(v[s].w));
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

  // X^T of a tile (fp32; the kernels in bf16 have their products among what else they do)
  __device__ __forceinline__ void rows_times(const unsigned char* tile, const Column& c, f32x16& x) const {
    static_assert(!kHalf, "fp32");
#pragma unroll
    for (int s = 0; s < D / 8; ++s) {
      const float4 a = *reinterpret_cast<const float4*>(tile + (row_off ^ (s << 4)));
      x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, c.v[s].x, x, 0, 0, 0);
      x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, c.v[s].y, x, 0, 0, 0);
      x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, c.v[s].z, x, 0, 0, 0);
      x = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, c.v[s].w, x, 0, 0, 0);
    }
  }

  // columns that wait in LDS, each lane's operands where it put them
  static constexpr int kParked = 32 * kRowBytes;  // bytes of a wave
  static __device__ __forceinline__ void park(unsigned char* to, const Column& c, int lane) {
#pragma unroll
    for (int s = 0; s < kParked / 1024; ++s) *reinterpret_cast<std::conditional_t<kHalf, bf16x8, float4>*>(to + s * 1024 + lane * 16) = c.v[s];
  }

  // acc^T += a tile, transposed, times X (fp32). Columns DB i .. of row i of the accumulators, so that a lane reads what it needs of a
  // tile row at once.
  __device__ __forceinline__ void transposed_times(const unsigned char* tile, const f32x16& x, f32x16 (&acc)[DB], int lane) const {
    static_assert(!kHalf, "fp32");
    const int li = lane & 31, lh = lane >> 5;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = row_of(r, lh);
      if constexpr (DB == 4) {
        const float4 a = *reinterpret_cast<const float4*>(tile + row * kRowBytes + ((li ^ swz(row)) << 4));
        acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, x[r], acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, x[r], acc[1], 0, 0, 0);
        acc[2] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.z, x[r], acc[2], 0, 0, 0);
        acc[3] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.w, x[r], acc[3], 0, 0, 0);
      } else {
        const float2 a = *reinterpret_cast<const float2*>(tile + row * kRowBytes + (((li >> 1) ^ swz(row)) << 4) + (li & 1) * 8);
        acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x, x[r], acc[0], 0, 0, 0);
        acc[1] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.y, x[r], acc[1], 0, 0, 0);
      }
    }
  }

  // Whether a wave's accumulators hold an infinity or a NaN: nothing else keeps 0 times itself from 0.
  static __device__ __forceinline__ bool unbounded(const f32x16 (&acc)[DB]) {
    float zero = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) zero = __builtin_fmaf(acc[db][r], 0.f, zero);
    return __any(!(zero == 0.f));
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

// A value that is found again where it is used: the compiler otherwise keeps what follows from it in registers through the loop.
__device__ __forceinline__ int again(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// ---- documents and masks
__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return min(max(v, lo), hi); }

// A document: its first query and key, how many of each, and what each query sees.
struct Document {
  int q0, nq, k0, nk, prefix;
  bool causal;
  // where the document's query i stands among its keys: the last query at the last key
  __device__ __forceinline__ int position(int i) const { return i + nk - nq; }
  // query i sees the keys [0, seen(i)), which grows with i
  __device__ __forceinline__ int seen(int i) const { return causal ? clamp_to(max(prefix, position(i) + 1), 0, nk) : nk; }
  // key j is seen by the queries [first_seer(j), nq), which grows with j
  __device__ __forceinline__ int first_seer(int j) const { return causal && j >= prefix ? max(j - (nk - nq), 0) : 0; }
};

// The tile that slot t of a head of batch entry b stands for: rows [first, end) of a document, of which the tile has the first `per`
// (QUERIES: rows of queries; otherwise keys). Rows of no document are those of one that has nothing.
// Document c's tiles begin at slot floor(start_c rows / per) + c, which leaves room for what precedes it and needs no list; the rows
// before the first and behind the last document count as documents. A lane looks at a document each, and all that is to be known of
// it comes with one round of loads (three, one after the other, took 2 us of every workgroup). Where there are more than 64, rounds before
// it look at 64 of them and leave those from one to the next (65,536 documents of single tokens, 8 heads of 64: 64 documents after 64 took
// 192 ms, so 3.3). Offsets out of range are taken as the nearest in range.
struct Found {
  int first, end;
  Document doc;
};
template <bool QUERIES>
__device__ __forceinline__ Found find_tile(const DenseArgs& a, int b, int per, int t, int lane) {
  const int64_t row = a.docs_shared ? 0 : b, pitch = a.n_docs + 1;
  const int32_t* own = QUERIES ? a.q_offsets : a.k_offsets;
  const int32_t* other = QUERIES ? a.k_offsets : a.q_offsets;
  const int n_own = QUERIES ? a.Nq : a.Nk, n_other = QUERIES ? a.Nk : a.Nq, G = QUERIES ? a.G : 1;
  if (own) own += row * pitch;
  if (other) other += row * pitch;
  const int all = own ? a.n_docs + 2 : 1;  // (without offsets the one document alone)
  int c = 0, start = 0, end = 0, lo = 0, hi = 0, prefix = 0;
  int before = 0;
  for (int left = all; left > 64;) {
    const int step = (left + 63) / 64, i = before + lane * step;
    const bool in = lane * step < left;
    const int v_start = in && i > 0 ? clamp_to(own[i - 1], 0, n_own) : 0;
    const int skip = max(__popcll(__ballot(in && (int64_t)v_start * G / per + i <= t)) - 1, 0) * step;
    before += skip;
    left = min(step, left - skip);
  }
  // (a loop from a number that the compiler does not know had the kernels behind it keep 30 registers of addresses)
  for (int c0 = 0; c0 < all; c0 += 64) {
    const int i = before + c0 + lane, d = own ? i - 1 : i;  // its number among the documents
    const bool real = d >= 0 && d < a.n_docs;
    const int v_start = own && i > 0 && i < all ? clamp_to(own[i - 1], 0, n_own) : 0;
    const int v_end = own && i < all - 1 ? clamp_to(own[i], 0, n_own) : n_own;
    const int v_lo = real && other ? clamp_to(other[d], 0, n_other) : 0;
    const int v_hi = !real ? 0 : other ? clamp_to(other[d + 1], 0, n_other) : n_other;
    const int v_prefix = real && a.prefix ? a.prefix[row * a.n_docs + d] : 0;
    const unsigned long long votes = __ballot(i < all && (int64_t)v_start * G / per + i <= t);
    const int found = __popcll(votes);
    if (found == 0) break;
    c = before + c0 + found - 1;
    start = __builtin_amdgcn_readlane(v_start, found - 1);
    end = __builtin_amdgcn_readlane(v_end, found - 1);
    lo = __builtin_amdgcn_readlane(v_lo, found - 1);
    hi = max(__builtin_amdgcn_readlane(v_hi, found - 1), lo);
    prefix = __builtin_amdgcn_readlane(v_prefix, found - 1);
    if (found < 64) break;
  }
  const bool real = !own || (c >= 1 && c <= a.n_docs);
  const int n = real ? max(end - start, 0) : 0;
  Found f;
  const int64_t first = (int64_t)start * G + (t - ((int64_t)start * G / per + c)) * per;
  f.first = first < 0 ? 0 : first < INT32_MAX ? (int)first : INT32_MAX;
  f.end = end * G;
  f.doc.q0 = QUERIES ? start : lo, f.doc.nq = QUERIES ? n : hi - lo;
  f.doc.k0 = QUERIES ? lo : start, f.doc.nk = QUERIES ? hi - lo : n;
  f.doc.prefix = clamp_to(prefix, 0, f.doc.nk);
  f.doc.causal = a.causal;
  return f;
}

// Where part `split` of `splits` begins among so many tiles: 2^25 and a few at most, and 64 parts.
__device__ __forceinline__ int part_begin(int tiles, int split, int splits) {
  return splits == 1 ? split * tiles : (int)((unsigned)tiles * (unsigned)split / (unsigned)splits);
}

// Workgroup to (key head of the batch, slot). Workgroups go to the 8 XCDs in turn: each takes whole heads, whose keys and values (or
// queries) its L2 then holds once, and the heads that are left over when each has as many are dealt out by the slot, so that tiles
// of different lengths (documents, the triangle of a causal mask) fall on all of them alike.
__device__ __forceinline__ bool dense_index(const DenseArgs& a, int& bh, int& slot, int& split) {
  const unsigned heads = (unsigned)(a.B * a.Hk), slots = (unsigned)a.slots, whole = heads / 8, rest = heads % 8;
  const unsigned wg = long_grid_index(), xcd = wg & 7, all = wg >> 3, i = (unsigned)((int)all / a.by_splits);
  split = (int)(all - i * (unsigned)a.splits);
  if (i < whole * slots) {
    const unsigned h = (unsigned)((int)i / a.by_slots);
    bh = (int)(h * 8 + xcd);
    slot = (int)(i - h * slots);
    return true;
  }
  const unsigned r = (i - whole * slots) * 8 + xcd;
  if (rest == 0 || r >= rest * slots) return false;
  slot = (int)(r / rest);
  bh = (int)(whole * 8 + (r - (unsigned)slot * rest));
  return true;
}

// tanh from the hardware's exponential and reciprocal. NEAR: 1 - 2 / (e^2x + 1), off by up to 2.7e-7 of 1 (half steps of the sum and
// of its exponential, a step of each), however small x is. Otherwise (1 - e) / (1 + e) with e = e^-2|x|, and below 0.3, where 1 - e would lose
// digits, the series, whose next term is 3e-9 of the result there: off by some 10 half steps of the result.
template <bool NEAR>
__device__ __forceinline__ float tanh_of(float x) {
  if constexpr (NEAR) {
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

// What a call's cap is. With a cap a score is off by what its tanh is off by, times the cap: in bf16 the short form is good for caps up to
// 256, which it moves by 7e-5 at most, beside the 2^-9 that a weight's rounding is off by. (At 1e6 that would be 0.3.) The long form
// is some ten operations more a pair: gradients of 4,000 causal tokens of 40 heads, 8 key heads of 128, 1,180 us with a cap of 50 or 256, 1,535 with
// one of 1,000; the forward pass, whose whole tiles take a series with both, 204 and 207.
enum { kCapNone = 0, kCapNear = 1, kCapFar = 2 };
constexpr float kFarCap = 256.f;

// Products to exponents of 2, of a query at `dist` from the key. The cap's derivative is 1 - tanh^2.
template <typename T, int CAP, bool SLOPES>
struct Scores {
  float c, cap2;
  __device__ __forceinline__ Scores(const DenseArgs& a) : c(CAP ? a.scale / a.cap : a.scale * kLog2e), cap2(a.cap * kLog2e) {}
  // tanh (or the product itself)
  __device__ __forceinline__ float inner(float s) const { return CAP ? tanh_of<sizeof(T) == 2 && CAP == kCapNear>(s * c) : s; }
  // exponent less `less`
  __device__ __forceinline__ float outer(float in, float dist, float slope, float less) const {
    if (SLOPES) less = __builtin_fmaf(slope, fabsf(dist), less);
    return __builtin_fmaf(in, CAP ? cap2 : c, -less);
  }
  __device__ __forceinline__ float keeps(float in) const { return __builtin_fmaf(-in, in, 1.f); }
};

// The mark of a wave of a workgroup (bh, slot) and its part: whether what it found is unbounded.
__device__ __forceinline__ int32_t* mark_of(const DenseArgs& a, int part, int bh, int slot, int wave) {
  return a.marks + (((int64_t)part * (a.B * a.Hk) + bh) * a.slots + slot) * kDenseWaves + wave;
}

// f(cap, slopes) as types, for what a call has; FAR: caps over kFarCap by themselves
template <bool FAR = false, typename F>
int by_scores(const DenseArgs& a, F f) {
  auto with = [&](auto cap) -> int { return a.slopes ? f(cap, std::true_type{}) : f(cap, std::false_type{}); };
  if constexpr (FAR)
    if (a.cap > kFarCap) return with(std::integral_constant<int, kCapFar>{});
  return a.cap > 0.f ? with(std::integral_constant<int, kCapNear>{}) : with(std::integral_constant<int, kCapNone>{});
}
// Workgroups of a launch: those of dense_index.
inline dim3 dense_grid(const DenseArgs& a) { return long_grid(ceil_div((int64_t)a.B * a.Hk * a.slots, 8) * 8 * a.splits, 1); }

}  // namespace
}  // namespace svgear

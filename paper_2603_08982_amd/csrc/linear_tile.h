// The tile kernel of the matrix products, for bf16 and fp32 (internal; see linear.hip for the operators).
//
// out[r][c] = sum_k Q[r][k] P[c][k]. A workgroup makes a tile of BC columns by BR rows; its waves hold
// their shares as 32 x 32 MFMA blocks whose row index is c, so that a lane ends with four consecutive
// columns of one row. K is walked in steps of 128 bytes per row (64 bf16, 32 fp32), two steps' tiles in
// LDS: the copies of the next step, straight from global memory, run under the products of this one.
//
// An operand whose contraction index is contiguous lies in LDS as rows of 128 bytes; a lane's fragment is one
// 16-byte chunk. One whose contraction index runs over rows (dx: w; dw: both) lies there as it does in
// memory, a row for each k; bf16 fragments are then read with the LDS transpose read, fp32 ones element by
// element (the fp32 matrix cores take 16 times as long for a step, so the reads are hidden).
// Bank conflicts: chunks of 16 bytes are XORed with bits of the row; the copy's lanes pick the global chunk
// that belongs into their slot.
#pragma once
#include <type_traits>

#include "linear.h"

namespace svgear {
namespace {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16* lds_v4i16_ptr;

__device__ uint4 g_zero_chunk[1];  // what chunks past the end of K read

__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)(p);
}

// 16 bytes of a fragment
struct Frag {
  union {
    uint4 u;
    float f[4];
    bf16x8 b;
    struct { v4i16 lo, hi; } h;
  };
};

// One operand's tile: E extent (rows of the output's r or c), contraction contiguous or over rows.
template <typename T, int E, bool OVER_ROWS, int WAVES>
struct Tile {
  static constexpr int ES = sizeof(T);
  static constexpr int BK = 128 / ES;                        // k of a step
  static constexpr int CH = 16 / ES;                         // elements of a chunk
  static constexpr int ROWB = OVER_ROWS ? E * ES : 128;      // bytes of an LDS row
  static constexpr int CPR = ROWB / 16;                      // its chunks
  static constexpr int BYTES = E * 128;
  static constexpr int COPIES = BYTES / 1024 / WAVES;        // wave-wide copies of 1 KB, each wave
  static_assert(BYTES % (1024 * WAVES) == 0, "copies must split evenly over the waves");

  static __device__ __forceinline__ int swz(int row) {
    if (!OVER_ROWS) return (row >> 1) & 7;
    if (ES == 4) return ((row >> 2) & 1) << 3;
    return ROWB >= 256 ? (row & 3) << 2 : (row & 2) << 1;
  }

  uint32_t off[COPIES];   // byte offset of the lane's chunk from the tile's first row / step's first k
  int kk[COPIES];         // its k within the step
  const unsigned char* base;  // wave-uniform: the step's first element
  int64_t step;               // bytes from step to step

  // e0: first row of the output this tile covers, limit: their number; k0: first k.
  __device__ __forceinline__ void init(const Operand& o, int e0, int limit, int64_t k0, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const int slot = (wave + i * WAVES) * 64 + lane, row = slot / CPR, chunk = (slot % CPR) ^ swz(row);
      if (!OVER_ROWS) {
        // rows past the last repeat it: what they give is never stored
        off[i] = (uint32_t)(min(row, limit - 1 - e0) * (int64_t)(o.pitch * ES) + chunk * 16);
        kk[i] = chunk * CH;
      } else {
        const int last = (limit - 1 - e0) / CH;  // chunks past the last likewise
        off[i] = (uint32_t)(row * (int64_t)(o.pitch * ES) + min(chunk, last) * 16);
        kk[i] = row;
      }
    }
    const int64_t first = OVER_ROWS ? k0 * o.pitch + e0 : e0 * o.pitch + k0;
    base = static_cast<const unsigned char*>(o.p) + first * ES;
    step = (OVER_ROWS ? BK * o.pitch : (int64_t)BK) * ES;
  }
  // Copies the step whose first element is `base` into lds and goes on; `left`: k that remain.
  __device__ __forceinline__ void copy(uint32_t lds, int64_t left, int wave) {
    if (left >= BK) {
#pragma unroll
      for (int i = 0; i < COPIES; ++i)
        async_copy_16B(base, off[i], __builtin_amdgcn_readfirstlane(lds + (wave + i * WAVES) * 1024));
    } else {
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {
        const void* src = kk[i] < left ? static_cast<const void*>(base + off[i]) : static_cast<const void*>(g_zero_chunk);
        async_copy_16B(src, __builtin_amdgcn_readfirstlane(lds + (wave + i * WAVES) * 1024));
      }
    }
    base += step;
  }
};

// Reads of one wave's fragments: NB blocks of 32 from e = first.
template <typename T, int E, bool OVER_ROWS, int NB>
struct Reader {
  static constexpr int ES = sizeof(T);
  static constexpr int ROWB = OVER_ROWS ? E * ES : 128;
  static constexpr int NO = !OVER_ROWS ? 4 : NB;
  int off[NO];

  __device__ __forceinline__ void init(int first, int lane) {
    const int li = lane & 31, lh = lane >> 5;
    if (!OVER_ROWS) {  // chunk 2s + lh of row li, by s
#pragma unroll
      for (int s = 0; s < NO; ++s) off[s] = (first + li) * 128 + (((2 * s + lh) ^ ((li >> 1) & 7)) << 4);
    } else if (ES == 2) {
      // transpose read: lane r of a group of 16 addresses k = r/4 and columns 4 (r%4) ..; it gets column r of
      // k 0..3. Groups: (column half, k half)
      const int r = lane & 15, half = (lane >> 4) & 1, row = 8 * lh + (r >> 2);
      const int x = ROWB >= 256 ? (row & 3) << 2 : (row & 2) << 1;
#pragma unroll
      for (int i = 0; i < NO; ++i)
        off[i] = row * ROWB + ((((first + 32 * i) / 8 + 2 * half + ((r & 3) >> 1)) ^ x) << 4) + (r & 1) * 8;
    } else {  // k = 4 lh + j: row's swizzle is lh alone
#pragma unroll
      for (int i = 0; i < NO; ++i) off[i] = lh * 4 * ROWB + (((first + 32 * i + li) * 4) ^ (lh << 7));
    }
  }
  // Fragment of block i, contraction step s (16 bf16 or 8 fp32 of k): the lane's 16 bytes are k = half lh of it.
  __device__ __forceinline__ Frag get(const unsigned char* lds, int i, int s) const {
    Frag f;
    if constexpr (!OVER_ROWS) {
      f.u = *reinterpret_cast<const uint4*>(lds + off[s] + i * 32 * 128);
    } else if constexpr (ES == 2) {
      const unsigned char* p = lds + off[i] + s * 16 * ROWB;
      f.h.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(p));
      f.h.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(p + 4 * ROWB));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f.f[j] = *reinterpret_cast<const float*>(lds + off[i] + (8 * s + j) * ROWB);
    }
    return f;
  }
};

template <typename T>
__device__ __forceinline__ void multiply(const Frag& p, const Frag& q, f32x16& acc) {
  if constexpr (sizeof(T) == 2) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p.b, q.b, acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(p.f[j], q.f[j], acc, 0, 0, 0);
  }
}

// WC x WR waves, each TC x TR blocks of 32 x 32.
template <typename T, int FORM, int TC, int TR, int WC, int WR>
__global__ void __launch_bounds__(64 * WC * WR, WC * WR / 4)
linear_tile_kernel(LinearArgs a, int tiles_c, int tiles_r) {
  constexpr int WAVES = WC * WR, BC = 32 * TC * WC, BR = 32 * TR * WR;
  constexpr bool P_ROWS = FORM != kContractBoth, Q_ROWS = FORM == kContractNone;
  typedef Tile<T, BC, P_ROWS, WAVES> PT;
  typedef Tile<T, BR, Q_ROWS, WAVES> QT;
  constexpr int BK = PT::BK, STAGE = PT::BYTES + QT::BYTES;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wc = wave % WC, wr = wave / WC;

  // Tile of this workgroup. Workgroups go to the 8 XCDs in turn: each XCD gets a run of tiles of its own, in
  // order of 8 tile rows a column at a time, so that what runs on it together shares both operands in its L2.
  const int tiles = tiles_c * tiles_r, bid = blockIdx.x;
  const int xcd = bid & 7, per = tiles >> 3, more = tiles & 7;
  const int t = xcd * per + min(xcd, more) + (bid >> 3);
  const int band = t / (8 * tiles_c), band_r = min(8, tiles_r - 8 * band), in_band = t - band * 8 * tiles_c;
  const int r0 = (8 * band + in_band % band_r) * BR, c0 = in_band / band_r * BC;

  const int64_t steps = (a.K + BK - 1) / BK, part = blockIdx.y;
  const int64_t s0 = steps * part / a.splits, s1 = steps * (part + 1) / a.splits;
  int64_t left = a.K - s0 * BK;  // k from the next copy's first on
  const int n = (int)(s1 - s0);

  PT pt;
  QT qt;
  pt.init(a.P, c0, a.C, s0 * BK, wave, lane);
  qt.init(a.Q, r0, a.R, s0 * BK, wave, lane);
  Reader<T, BC, P_ROWS, TC> pr;
  Reader<T, BR, Q_ROWS, TR> qr;
  pr.init(wc * 32 * TC, lane);
  qr.init(wr * 32 * TR, lane);
  const uint32_t lds0 = lds_address(smem);
  auto copy = [&](int buf) __attribute__((always_inline)) {
    pt.copy(lds0 + buf * STAGE, left, wave);
    qt.copy(lds0 + buf * STAGE + PT::BYTES, left, wave);
    left -= BK;
  };

  f32x16 acc[TC][TR];
#pragma unroll
  for (int i = 0; i < TC; ++i)
#pragma unroll
    for (int j = 0; j < TR; ++j) acc[i][j] = f32x16{};

  copy(0);
  SVGEAR_WAIT_VMCNT(0);
  __syncthreads();
  for (int k = 0; k < n; ++k) {
    if (k + 1 < n) copy((k + 1) & 1);
    const unsigned char* ps = smem + (k & 1) * STAGE;
    const unsigned char* qs = ps + PT::BYTES;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      Frag pf[TC], qf[TR];
#pragma unroll
      for (int i = 0; i < TC; ++i) pf[i] = pr.get(ps, i, s);
#pragma unroll
      for (int j = 0; j < TR; ++j) qf[j] = qr.get(qs, j, s);
#pragma unroll
      for (int i = 0; i < TC; ++i)
#pragma unroll
        for (int j = 0; j < TR; ++j) multiply<T>(pf[i], qf[j], acc[i][j]);
    }
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
  }

  // a lane's block holds columns 8g + 4lh + 0..3 of row li
  const int li = lane & 31, lh = lane >> 5;
#pragma unroll
  for (int j = 0; j < TR; ++j) {
    const int r = r0 + (wr * TR + j) * 32 + li;
    if (r >= a.R) continue;
#pragma unroll
    for (int i = 0; i < TC; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int c = c0 + (wc * TC + i) * 32 + 8 * g + 4 * lh;
        if (c >= a.C) continue;
        const float4 v = make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
        if (a.partial) {
          float* o = a.partial + (part * a.R + r) * a.C + c;
          if (a.C % 4 == 0) {
            *reinterpret_cast<float4*>(o) = v;
          } else {
            o[0] = v.x;
            if (c + 1 < a.C) o[1] = v.y;
            if (c + 2 < a.C) o[2] = v.z;
            if (c + 3 < a.C) o[3] = v.w;
          }
        } else {
          finish4<T>(a, r, c, v);
        }
      }
  }
}

template <typename T, int FORM, int TC, int TR, int WC, int WR>
int launch_tiles(const LinearArgs& a, hipStream_t s) {
  constexpr int BC = 32 * TC * WC, BR = 32 * TR * WR, lds = 2 * (BC + BR) * 128;
  const int tc = (int)ceil_div(a.C, BC), tr = (int)ceil_div(a.R, BR);
  if ((int64_t)tc * tr > INT32_MAX) return SVGEAR_ERR_UNSUPPORTED;
  auto kern = linear_tile_kernel<T, FORM, TC, TR, WC, WR>;
  if (lds > 65536)
    SVGEAR_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  kern<<<dim3((unsigned)(tc * tr), (unsigned)a.splits), 64 * WC * WR, lds, s>>>(a, tc, tr);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

template <typename T>
int launch_linear(const LinearArgs& a, int form, hipStream_t s) {
  switch (form) {
    case kContractBoth: return launch_tiles<T, kContractBoth, 2, 2, 2, 2>(a, s);
    case kContractQ: return launch_tiles<T, kContractQ, 2, 2, 2, 2>(a, s);
    default: return launch_tiles<T, kContractNone, 2, 2, 2, 2>(a, s);
  }
}

}  // namespace
}  // namespace svgear

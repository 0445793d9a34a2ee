// The tile kernel of the matrix products, for bf16 and fp32 (internal; see linear.hip for the operators).
//
// out[r][c] = sum_k Q[r][k] P[c][k]. A workgroup makes a tile of BC columns by BR rows; its waves hold
// their shares as 32 x 32 MFMA blocks whose row index is c, so that a lane ends with four consecutive
// columns of one row. K is walked in steps of 128 bytes per row (64 bf16, 32 fp32); the copies of later steps' tiles,
// straight from global memory into LDS, run under the products of this one.
//
// An operand whose contraction index is contiguous lies in LDS as rows of 128 bytes; a lane's fragment is one
// 16-byte chunk. One whose contraction index runs over rows (dx: w; dw: both) lies there as it does in
// memory, a row for each k; bf16 fragments are then read with the LDS transpose read, fp32 ones element by
// element (the fp32 matrix cores take 16 times as long for a step, so the reads are hidden).
// Bank conflicts: chunks of 16 bytes are XORed with bits of the row; the copy's lanes pick the global chunk
// that belongs into their slot (none are left: SQ_LDS_BANK_CONFLICT is 0).
//
// What bounds it, 256 x 256 tiles, 37,800 x 15,360 of 5,120 in bf16 (4.35 ms, 1,368 TFLOP/s; the library's product 4.1): the
// matrix cores are busy 82 % of the cycles, at the 1.43 GHz that the power limit leaves; 8 to 10 us of each tile's 120
// are its prologue and epilogue. With the copies left out the loop takes 17 % less, with the LDS reads left out 4 %.
// Steps that brought it there from 6.3 ms: fragments read and tiles copied under the products (5.3; the copies all at once stall
// the waves: in two shares 4.9), tiles in the order below (4.6), the third buffer of P (4.4). 8 waves of 64 x 128 and 4
// of 128 x 128, copies earlier, later or in turn, and wave priorities all come to the same within 2 %.
// fp32, 8,192 x 2,048 of 2,048 in tiles of 128: 0.49 ms, 139 TFLOP/s (the library's 140): the fp32 matrix cores.
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

// One operand's tile: E extent (rows of the output's r or c), contraction contiguous or over rows; copied by G bytes a lane: 16, or
// one fp32 element, for rows at any alignment and of any length.
template <typename T, int E, bool OVER_ROWS, int WAVES, int G>
struct Tile {
  static constexpr int ES = sizeof(T);
  static constexpr int BK = 128 / ES;                        // k of a step
  static constexpr int CH = 16 / ES;                         // elements of a chunk
  static constexpr int ROWB = OVER_ROWS ? E * ES : 128;      // bytes of an LDS row
  static constexpr int CPR = ROWB / 16;                      // its chunks
  static constexpr int BYTES = E * 128;
  static constexpr int COPIES = BYTES / (64 * G) / WAVES;    // wave-wide copies, each wave
  static_assert(BYTES % (64 * G * WAVES) == 0, "copies must split evenly over the waves");
  static_assert(G == 16 || (G == 4 && ES == 4), "chunks or fp32 elements");
  static_assert(!OVER_ROWS || ES == 2 || ROWB >= 256, "the chunk swizzle needs 16 chunks in a row");

  static __device__ __forceinline__ int swz(int row) {
    if (!OVER_ROWS) return (row >> 1) & 7;
    if (ES == 4) return ((row >> 2) & 1) << 3;
    return ROWB >= 256 ? (row & 3) << 2 : (row & 2) << 1;
  }

  uint32_t off[COPIES];   // byte offset of the lane's G bytes from the tile's first row / step's first k
  int kk[COPIES];         // its k within the step
  const unsigned char* base;  // wave-uniform: the step's first element
  int64_t step;               // bytes from step to step

  // e0: first row of the output this tile covers, limit: their number; k0: first k.
  __device__ __forceinline__ void init(const Operand& o, int e0, int limit, int64_t k0, int wave, int lane) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const int slot = ((wave + i * WAVES) * 64 + lane) * G / 16, row = slot / CPR, chunk = (slot % CPR) ^ swz(row);
      const int part = G == 16 ? 0 : lane & 3;  // element of the chunk
      if (!OVER_ROWS) {
        // rows past the last repeat it: what they give is never stored
        off[i] = (uint32_t)(min(row, limit - 1 - e0) * (int64_t)(o.pitch * ES) + chunk * 16 + part * G);
        kk[i] = chunk * CH + part;
      } else {
        const int last = limit - 1 - e0;  // chunks (elements) past the last likewise
        off[i] = (uint32_t)(row * (int64_t)(o.pitch * ES) + (G == 16 ? min(chunk, last / CH) * 16 : min(chunk * CH + part, last) * ES));
        kk[i] = row;
      }
    }
    const int64_t first = OVER_ROWS ? k0 * o.pitch + e0 : e0 * o.pitch + k0;
    base = static_cast<const unsigned char*>(o.p) + first * ES;
    step = (OVER_ROWS ? BK * o.pitch : (int64_t)BK) * ES;
  }
  // Copy i of the step whose first element is `base` into lds; LAST: the last step, `left` k of which exist.
  template <bool LAST>
  __device__ __forceinline__ void copy(int i, uint32_t lds, int left, int wave) const {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + (wave + i * WAVES) * (64 * G));
    const void* from = LAST && kk[i] >= left ? static_cast<const void*>(g_zero_chunk) : static_cast<const void*>(base + off[i]);
    if constexpr (G == 4)
      async_copy_4B(from, to);
    else if constexpr (!LAST)
      async_copy_16B(base, off[i], to);
    else
      async_copy_16B(from, to);
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

// All waves' LDS reads are done and may be overwritten; copies in flight stay in flight.
__device__ __forceinline__ void workgroup_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <typename T>
__device__ __forceinline__ void multiply(const Frag& p, const Frag& q, f32x16& acc) {
  if constexpr (sizeof(T) == 2) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(p.b, q.b, acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(p.f[j], q.f[j], acc, 0, 0, 0);
  }
}

// WC x WR waves, each TC x TR blocks of 32 x 32. Registers for as many workgroups on a CU as the LDS holds: one of 256 x 256, two
// or more of the others. PG: bytes a lane of P's copies.
template <typename T, int FORM, int TC, int TR, int WC, int WR, int PG>
__global__ void __launch_bounds__(64 * WC * WR, (TC * TR > 2 ? WC * WR / 4 : WC * WR / 2))
linear_tile_kernel(LinearArgs a, int tiles_c, int tiles_r) {
  constexpr int WAVES = WC * WR, BC = 32 * TC * WC, BR = 32 * TR * WR;
  constexpr bool P_ROWS = FORM != kContractBoth, Q_ROWS = FORM == kContractNone;
  typedef Tile<T, BC, P_ROWS, WAVES, PG> PT;
  typedef Tile<T, BR, Q_ROWS, WAVES, 16> QT;
  constexpr int BK = PT::BK, LDS = 3 * PT::BYTES + 2 * QT::BYTES;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wc = wave % WC, wr = wave / WC;

  // Tile of this workgroup. Tiles are numbered column by column in bands of 16 tile rows, and 256 at a time run
  // together: 16 x 16 tiles, which read 32 panels of the operands out of the 256 MB cache behind the L2s.
  // Workgroups go to the 8 XCDs in turn; each gets 8 x 4 tiles of those, so that its L2 serves 32 tiles with 12
  // panels. What is left of 256 goes to them in runs. (Each XCD with a run of tiles of its own from the start: 68 panels
  // at a time, 37,800 x 15,360 of 5,120 4.9 instead of 4.6 ms.)
  const int tiles = tiles_c * tiles_r, bid = (int)long_grid_index(), xcd = bid & 7, whole = tiles & ~255;
  if (bid >= tiles) return;
  int t;
  if (bid < whole) {
    const int i = (bid & 255) >> 3;
    t = (bid & ~255) + (4 * (xcd >> 1) + (i >> 3)) * 16 + 8 * (xcd & 1) + (i & 7);
  } else {
    const int per = (tiles - whole) >> 3, more = (tiles - whole) & 7;
    t = whole + xcd * per + min(xcd, more) + ((bid - whole) >> 3);
  }
  const int band = t / (16 * tiles_c), band_r = min(16, tiles_r - 16 * band), in_band = t - band * 16 * tiles_c;
  const int r0 = (16 * band + in_band % band_r) * BR, c0 = in_band / band_r * BC;

  const int64_t steps = (a.K + BK - 1) / BK, part = blockIdx.y;
  const int64_t s0 = steps * part / a.splits, s1 = steps * (part + 1) / a.splits;
  const int left = (int)min((int64_t)BK, a.K - (s1 - 1) * BK);  // k of the last step
  const int n = (int)(s1 - s0);

  PT pt;
  QT qt;
  pt.init(a.P, c0, a.C, s0 * BK, wave, lane);
  qt.init(a.Q, r0, a.R, s0 * BK, wave, lane);
  Reader<T, BC, P_ROWS, TC> pr;
  Reader<T, BR, Q_ROWS, TR> qr;
  pr.init(wc * 32 * TC, lane);
  qr.init(wr * 32 * TR, lane);
  f32x16 acc[TC][TR];
#pragma unroll
  for (int i = 0; i < TC; ++i)
#pragma unroll
    for (int j = 0; j < TR; ++j) acc[i][j] = f32x16{};

  // The main loop's step k is four contraction steps. Under the products of each, the fragments of the next one
  // are read, across steps too: the workgroup's barrier lies before the last products of a step, when all its
  // fragments are in registers. Copies: P has three buffers and Q two, so P's of step k+2 go out under the first
  // products of step k and Q's behind its barrier, and none is waited for sooner than three contraction steps later.
  Frag pf[2][TC], qf[2][TR];
  const uint32_t lds0 = lds_address(smem);
  enum { kNo, kFull, kLast };
  constexpr std::integral_constant<int, kNo> no{};
  constexpr std::integral_constant<int, kFull> full{};
  constexpr std::integral_constant<int, kLast> last{};
  constexpr std::true_type yes{};
  constexpr std::false_type none{};
  auto copy_p = [&](int i, int slot, auto mode) __attribute__((always_inline)) {
    pt.template copy<mode.value == kLast>(i, lds0 + slot * PT::BYTES, left, wave);
    if (i == PT::COPIES - 1) pt.base += pt.step;
  };
  auto copy_q = [&](int i, int slot, auto mode) __attribute__((always_inline)) {
    qt.template copy<mode.value == kLast>(i, lds0 + 3 * PT::BYTES + slot * QT::BYTES, left, wave);
    if (i == QT::COPIES - 1) qt.base += qt.step;
  };
  auto read = [&](int i, int p_slot, int q_slot, int s, int set) __attribute__((always_inline)) {
    if (i < TC) pf[set][i] = pr.get(smem + p_slot * PT::BYTES, i, s);
    else if (i < TC + TR) qf[set][i - TC] = qr.get(smem + 3 * PT::BYTES + q_slot * QT::BYTES, i - TC, s);
  };
  // products of `set`; between them the reads of the other set's fragments, and what `more` does at each
  constexpr int BLOCKS = TC * TR;
  auto step = [&](int set, auto reads, int p_slot, int q_slot, int s, auto more) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < BLOCKS; ++m) {
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (reads.value) {
        constexpr int PER = (TC + TR + BLOCKS - 1) / BLOCKS;
#pragma unroll
        for (int i = 0; i < PER; ++i) read(m * PER + i, p_slot, q_slot, s, set ^ 1);
      }
      more(m);
      multiply<T>(pf[set][m / TR], qf[set][m % TR], acc[m / TR][m % TR]);
    }
  };
  auto nothing = [](int) {};
  // `share` copies spread evenly over a contraction step's products
  auto spread = [&](int m, int share, auto go) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < share; ++i)
      if (i * BLOCKS / share == m) go(i);
  };
  int slot = 0;  // k % 3
  auto iterate = [&](int k, auto mode, auto next) __attribute__((always_inline)) {
    constexpr int H = PT::COPIES / 2;
    const int before = slot == 0 ? 2 : slot - 1, after = slot == 2 ? 0 : slot + 1;
    step(0, yes, slot, k & 1, 1, [&](int m) __attribute__((always_inline)) {
      if constexpr (mode.value != kNo) spread(m, H, [&](int i) { copy_p(i, before, mode); });
    });
    step(1, yes, slot, k & 1, 2, [&](int m) __attribute__((always_inline)) {
      if constexpr (mode.value != kNo) spread(m, PT::COPIES - H, [&](int i) { copy_p(H + i, before, mode); });
    });
    step(0, yes, slot, k & 1, 3, nothing);
    if constexpr (next.value) {
      if constexpr (mode.value != kNo)
        SVGEAR_WAIT_VMCNT(PT::COPIES);
      else
        SVGEAR_WAIT_VMCNT(0);
      workgroup_barrier();
      step(1, yes, after, (k + 1) & 1, 0, [&](int m) __attribute__((always_inline)) {
        if constexpr (mode.value != kNo) spread(m, QT::COPIES, [&](int i) { copy_q(i, k & 1, mode); });
      });
    } else {
      step(1, none, 0, 0, 0, nothing);
    }
    slot = after;
  };
  auto copies = [&](int to, auto mode) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < PT::COPIES; ++i) copy_p(i, to, mode);
#pragma unroll
    for (int i = 0; i < QT::COPIES; ++i) copy_q(i, to, mode);
  };
  if (n == 1) {
    copies(0, last);
    SVGEAR_WAIT_VMCNT(0);
  } else {
    copies(0, full);
    if (n == 2) copies(1, last);
    else copies(1, full);
    SVGEAR_WAIT_VMCNT(PT::COPIES + QT::COPIES);
  }
  workgroup_barrier();
#pragma unroll
  for (int i = 0; i < TC + TR; ++i) read(i, 0, 0, 0, 0);
  int k = 0;
  for (; k + 3 < n; ++k) iterate(k, full, yes);
  if (k + 2 < n) iterate(k++, last, yes);
  if (k + 1 < n) iterate(k++, no, yes);
  iterate(k, no, none);
  __syncthreads();

  // A wave's 32 rows at a time go through its own part of LDS, so that what is read and written of a row is one
  // run of 16-byte pieces: block i, group g of a lane are columns 32i + 8g + 4lh + 0..3 of row li.
  constexpr int COLS = 32 * TC, CHUNKS = COLS / 4;
  static_assert(32 * COLS * 4 * WAVES <= LDS, "the waves' parts must fit");
  unsigned char* own = smem + wave * (32 * COLS * 4);
  const int li = lane & 31, lh = lane >> 5;
  auto stage = [&](int j) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < TC; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<float4*>(own + li * (COLS * 4) + (((8 * i + 2 * g + lh) ^ (li & (CHUNKS - 1))) << 4)) =
            make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  const int rw = r0 + wr * TR * 32;  // the wave's first row
  constexpr int LANES = COLS / 8, ROWS = 64 / LANES, PASSES = 32 / ROWS;  // LANES share a row, eight columns each
  const int sub = lane / LANES, at = 2 * (lane % LANES), c = c0 + wc * COLS + (lane % LANES) * 8;
  auto staged = [&](int q, float (&v)[8]) __attribute__((always_inline)) {
    const int row = q * ROWS + sub, x = row & (CHUNKS - 1);
    const float4 lo = *reinterpret_cast<const float4*>(own + row * (COLS * 4) + ((at ^ x) << 4));
    const float4 hi = *reinterpret_cast<const float4*>(own + row * (COLS * 4) + (((at + 1) ^ x) << 4));
    v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
  };
  const bool whole8 = c + 8 <= a.C;
  // columns behind the last whole eight: eight lanes a row
  const int first_tail = a.C % 8 && !a.partial ? (a.C & ~7) - c0 - wc * COLS : -1;
  float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (a.bias && !a.partial && whole8) load8(static_cast<const T*>(a.bias) + c, bias);
  const bool plain = sizeof(T) == 2 && a.act == SVGEAR_ACT_NONE && !a.pre && !a.partial;
#pragma unroll
  for (int j = 0; j < TR; ++j) {
    if (plain) {
      // bf16 (fp32 has no registers for it), no activation: gate and residual of all 32 rows are on their way together (18,900 x 5,120 of 5,120 with both: 885 us
      // a pass at a time, 776 together)
      Eight<T> gate[PASSES], res[PASSES];
      int64_t to[PASSES];
#pragma unroll
      for (int q = 0; q < PASSES; ++q) {
        const int r = min(rw + j * 32 + q * ROWS + sub, a.R - 1), b = a.n >= a.R ? 0 : r / a.n, t = r - b * a.n;
        to[q] = (int64_t)b * a.yst.b + (int64_t)t * a.yst.n;
        if (whole8) {
          if (a.gate) gate[q].load(static_cast<const T*>(a.gate) + (int64_t)b * a.gst.b + (int64_t)t * a.gst.n + c);
          if (a.residual) res[q].load(static_cast<const T*>(a.residual) + (int64_t)b * a.rst.b + (int64_t)t * a.rst.n + c);
        }
      }
      stage(j);
#pragma unroll
      for (int q = 0; q < PASSES; ++q) {
        float v[8];
        staged(q, v);
        if (rw + j * 32 + q * ROWS + sub >= a.R || !whole8) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += bias[i];
        if (a.gate) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] *= gate[q].get(i);
        }
        if (a.residual) {
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] += res[q].get(i);
        }
        store8(static_cast<T*>(a.y) + to[q] + c, v);
      }
    } else {
      stage(j);
#pragma unroll 1
      for (int q = 0; q < PASSES; ++q) {
        float v[8];
        staged(q, v);
        const int r = rw + j * 32 + q * ROWS + sub;
        if (r >= a.R || c >= a.C) continue;
        if (a.partial)
          store_partial8(a, part, r, c, v);
        else if (whole8)
          finish8<T>(a, r, c, v, bias);
      }
    }
    if (first_tail >= 0 && first_tail < COLS) {
#pragma unroll 1
      for (int q = 0; q < 32; q += 8) {
        const int row = q + (lane >> 3), col = first_tail + (lane & 7), r = rw + j * 32 + row, e = c0 + wc * COLS + col;
        if (r < a.R && e < a.C)
          finish1<T>(a, r, e, *reinterpret_cast<const float*>(own + row * (COLS * 4) + (((col >> 2) ^ (row & (CHUNKS - 1))) << 4) + (col & 3) * 4));
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

template <typename T, int FORM, int TC, int TR, int WC, int WR, int PG = 16>
int launch_tiles(const LinearArgs& a, hipStream_t s) {
  constexpr int BC = 32 * TC * WC, BR = 32 * TR * WR, lds = (3 * BC + 2 * BR) * 128;
  const int tc = (int)ceil_div(a.C, BC), tr = (int)ceil_div(a.R, BR);
  if ((int64_t)tc * tr > 1 << 30) return SVGEAR_ERR_UNSUPPORTED;
  auto kern = linear_tile_kernel<T, FORM, TC, TR, WC, WR, PG>;
  if (lds > 65536)
    SVGEAR_HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
  kern<<<long_grid(tc * tr, a.splits), 64 * WC * WR, lds, s>>>(a, tc, tr);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

template <typename T, int FORM>
int launch_form(const LinearArgs& a, hipStream_t s) {
  if constexpr (sizeof(T) == 4 && FORM != kContractNone) {
    if (a.by_element)
      return a.tile == 32 ? launch_tiles<T, FORM, 1, 1, 4, 1, 4>(a, s) : a.tile == 64 ? launch_tiles<T, FORM, 1, 1, 2, 2, 4>(a, s) : SVGEAR_ERR_UNSUPPORTED;
  }
  if (a.by_element) return SVGEAR_ERR_UNSUPPORTED;
  switch (a.tile) {
    case 32:
      if constexpr (sizeof(T) == 4 && FORM != kContractNone) return launch_tiles<T, FORM, 1, 1, 4, 1>(a, s);
      break;
    case 64: return launch_tiles<T, FORM, 1, 1, 2, 2>(a, s);
    // 8 waves, not 4 of 64 x 64: twice the waves for prologue and epilogue (fp32, 5,120 x 4,096 of 256: 91 us against 111; bf16,
    // 5,120 x 5,120 of 16: 20 against 23; at large K the two are within 2 %, at 6,000 x 4,000 of 2,048 4 of 64 x 64 gain 4 %)
    case 128: return launch_tiles<T, FORM, 1, 2, 4, 2>(a, s);
    case 256:
      if constexpr (sizeof(T) == 2) return launch_tiles<T, FORM, 2, 4, 4, 2>(a, s);
      break;
  }
  return SVGEAR_ERR_UNSUPPORTED;
}

template <typename T>
int launch_linear(const LinearArgs& a, int form, hipStream_t s) {
  switch (form) {
    case kContractBoth: return launch_form<T, kContractBoth>(a, s);
    case kContractQ: return launch_form<T, kContractQ>(a, s);
    default: return launch_form<T, kContractNone>(a, s);
  }
}

}  // namespace
}  // namespace svgear

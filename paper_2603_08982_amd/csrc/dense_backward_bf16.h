// The gradients of dense attention with masks in bf16: a workgroup owns 128 rows, 64 each of its two waves, which share the other side's
// tiles.
//
// A wave has a SIMD to itself, with 512 registers, and an operand that it reads from a tile goes into two products (with 32 rows a wave,
// two waves a SIMD, the reads of LDS took as long as the products). What it computes from one pair of sums it issues between the products of the
// next, and the operands are read AHEAD pairs of products before their own (2: as fast; 4: registers spill).
// 9,450 packed tokens of 16 heads, warm: delta 14 us, dq 637 (1,100 TFLOP/s), dk and dv 868 (1,080), the matrix cores busy 47 and 45 % of the
// cycles at 2.1 GHz (the whole call with 32 rows a wave for dk and dv 1,833 us, then 1,646; for dq too 1,626, then 1,534). Of dk's and dv's
// time the copies are 80 us, the exponentials 55, the differences 50, the operands' reads 80.
// A cap's tanh makes the vector unit the bound: 4,000 causal tokens of 40 heads, 8 key heads, 1,195 us (with two waves a SIMD 1,100). dk and dv
// at d = 128 spill registers in their loop there: 8 with a cap, 11 with slopes too, 4 with slopes alone (far caps 0 and 6).
#pragma once
#include "dense_tile.h"

namespace svgear {
namespace {

constexpr int kWaves = 2;  // of a workgroup

// f(0), f(1), .. f(N - 1) with constants (a loop of this length over so much is not unrolled)
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// Products whose sums are kept in vector registers (x) and in accumulation registers (acc): the compiler, which is free to choose, moves
// half of the accumulators between the two kinds in every step. It does not know of these instructions' latency: a sum that is read by
// another kind of instruction is read behind `settled` (11 cycles of 4 at least after the last product; here 20), and the two
// idle ones before a product are for an operand that was just written.
__device__ __forceinline__ void product(f32x16& x, const bf16x8& a, const bf16x8& b, bool first) {
  if (first) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(x) : "v"(a), "v"(b));
  else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x) : "v"(a), "v"(b));
}
// The same with the columns in accumulation registers (`keep`).
__device__ __forceinline__ void product_kept(f32x16& x, const bf16x8& a, const bf16x8& b, bool first) {
  if (first) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(x) : "v"(a), "a"(b));
  else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x) : "v"(a), "a"(b));
}
__device__ __forceinline__ void keep(bf16x8& b) { asm volatile("" : "+a"(b)); }
__device__ __forceinline__ void settled(f32x16 (&x)[2]) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(x[0]), "+v"(x[1])); }
__device__ __forceinline__ void accumulate(f32x16& acc, const bf16x8& a, const bf16x8& b) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// Behind the last products of a loop, and in it: what the compiler moves as it leaves the loop comes before any other statement.
__device__ __forceinline__ void settled_all() { asm volatile("s_nop 15\n\ts_nop 3" ::: "memory"); }
__device__ __forceinline__ void settled_acc(f32x16& acc) { asm volatile("s_nop 15\n\ts_nop 3" : "+a"(acc)); }

// ---- the queries' gradients: a pass over the keys
// A tile of 64 keys is 6 x 16 products of 32 cycles at d = 128: of its first and second 32 keys, those of k and q, of v and dy, and of
// ds and k. The exponentials lie between those of v and dy, ds = p (dp - delta) between what follows.
template <int D, int CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kWaves, 1)
dense_dq_kernel(DenseArgs a) {
  using T = bf16_t;
  using Z = Tile<T, D>;
  constexpr int DB = D / 32, KS = D / 16, BN = Z::kRows, ROWB = Z::kRowBytes, AHEAD = 3;
  static_assert(kWaves * 64 == kDenseRows && 2 * DB == KS, "the tiles of the other kernels; as many pairs of products each");
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes];  // two of K, two of V
  int bh, slot, split;
  if (!dense_index(a, bh, slot, split)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<true>(a, b, kDenseRows, a.causal ? a.slots - 1 - slot : slot, lane);  // causal: the longest first
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int wave_row = at.first + 64 * wave;
  const bool active = wave_row < at.end;
  const int hi_all = uniform(doc.seen(min(wave_row, at.end - 1) / a.by_g - doc.q0));
  const int hi_wg = uniform(doc.seen((min(at.first + kDenseRows, at.end) - 1) / a.by_g - doc.q0));
  const int tiles = (hi_wg + BN - 1) / BN;
  const int t_lo = uniform(part_begin(tiles, split, a.splits)), t_hi = uniform(part_begin(tiles, split + 1, a.splits));

  const Z z(lane);
  const Scores<T, CAP, SLOPES> scores(a);
  const uint32_t lds = lds_address(smem);
  const T* kp = static_cast<const T*>(a.k) + b * a.kst.b + hk * a.kst.h + doc.k0 * a.kst.n;
  const T* vp = static_cast<const T*>(a.v) + b * a.vst.b + hk * a.vst.h + doc.k0 * a.vst.n;
  // Rows of a whole tile lie at one offset of the lane from addresses that the wave shares; in the last tile, rows behind the last key
  // that a query here sees are not read.
  constexpr int kCopies = BN / Z::kRowsPerCopy / kWaves, kStep = kWaves * Z::kRowsPerCopy;
  const int copy_row = wave * Z::kRowsPerCopy + lane / Z::kChunks;
  auto issue_rows = [&](int t, const T* base, int64_t st, int buffer) __attribute__((always_inline)) {
    const T* rows = static_cast<const T*>(uniform_ptr(base + (int64_t)t * BN * st));
    const uint32_t to = (uint32_t)uniform((int)(lds + buffer * Z::kBytes + wave * 1024));
    const int last = hi_wg - 1 - t * BN;
    if (last >= BN - 1) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        async_copy_16B(rows + (int64_t)(i * kStep) * st, (uint32_t)copy_row * (uint32_t)st * 2u + ((lane % Z::kChunks) ^ Z::swz(i * kStep + copy_row)) * 16,
                       to + i * kWaves * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        async_copy_16B(rows, (uint32_t)min(i * kStep + copy_row, last) * (uint32_t)st * 2u + ((lane % Z::kChunks) ^ Z::swz(i * kStep + copy_row)) * 16,
                       to + i * kWaves * 1024);
    }
  };
  auto issue = [&](int t) __attribute__((always_inline)) {
    issue_rows(t, kp, a.kst.n, t & 1);
    issue_rows(t, vp, a.vst.n, 2 + (t & 1));
  };
  if (t_lo < t_hi) issue(t_lo);

  typename Z::Column q[2], dy[2];
  int pos[2], hi[2];
  float lse2[2], delta[2], slope[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const int row = min(wave_row + 32 * c + li, at.end - 1), token = row / a.by_g, head = hk * a.G + (row - token * a.G);
    pos[c] = doc.position(token - doc.q0), hi[c] = doc.seen(token - doc.q0);
    q[c].load(static_cast<const T*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n, lh);
    dy[c].load(static_cast<const T*>(a.dy) + b * a.yst.b + head * a.yst.h + token * a.yst.n, lh);
    const int64_t stat = ((int64_t)b * a.H + head) * a.Nq + token;
    lse2[c] = a.lse_in[stat] * kLog2e, delta[c] = a.delta[stat];
    slope[c] = SLOPES ? a.slopes[head] * kLog2e : 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) keep(q[c].v[s]), keep(dy[c].v[s]);
  }

  f32x16 acc[2][DB];
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int db = 0; db < DB; ++db) clear(acc[c][db]);

  for (int t = t_lo; t < t_hi; ++t) {
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
    if (t + 1 < t_hi) issue(t + 1);
    const bool masked = (t + 1) * BN > hi_all;
    const unsigned char* kt = smem + (t & 1) * Z::kBytes;
    const unsigned char* vt = smem + (2 + (t & 1)) * Z::kBytes;
    constexpr int N = 6 * KS;
    bf16x8 op[N];
    // pairs of products: KS each of k q and v dy of the first 32 keys, of the second, and of ds k of both
    auto rd = [&](int i) __attribute__((always_inline)) {
      const int phase = i / KS, s = i % KS;
      if (phase < 4) {
        op[i] = as_bf16x8(*reinterpret_cast<const uint4*>((phase & 1 ? vt : kt) + (phase >> 1) * 32 * ROWB + (z.row_off ^ (s << 5))));
      } else {
        const unsigned char* from16 = kt + (phase - 4) * 32 * ROWB + (s / DB) * 16 * ROWB;
        const int off = z.tr_off ^ ((s % DB) << 6);
        union { struct { v4i16 a, b; } s; bf16x8 v; } x;
        x.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(from16 + off));
        x.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(from16 + 8 * ROWB + (off ^ 32)));
        op[i] = x.v;
      }
    };
    f32x16 x[2][2], dp[2][2];  // of a block, of a column
    uint32_t dsk[2][2][8];
    auto weights = [&](int blk, int e) __attribute__((always_inline)) {  // of registers 2 e, 2 e + 1
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int r = 2 * e; r < 2 * e + 2; ++r) {
          const float in = scores.inner(x[blk][c][r]);
          const float dist = SLOPES ? (float)(pos[c] - (t * BN + 32 * blk + row_of(r, lh))) : 0.f;
          const float p = __builtin_amdgcn_exp2f(scores.outer(in, dist, slope[c], lse2[c]));
          x[blk][c][r] = CAP ? p * scores.keeps(in) : p;
        }
    };
    auto differences = [&](int blk, int e) __attribute__((always_inline)) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
        dsk[blk][c][e] = pack2_bf16(x[blk][c][2 * e] * (dp[blk][c][2 * e] - delta[c]), x[blk][c][2 * e + 1] * (dp[blk][c][2 * e + 1] - delta[c]));
    };
    // What keys that a row does not see have is taken out where there are such (a branch that no accumulator's value goes through: in one
    // that it did, the compiler would move it).
    auto hide = [&](int blk) __attribute__((always_inline)) {
      if (!masked) return;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int limit = hi[c] - (t * BN + 32 * blk + 4 * lh);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (row_of(2 * e, 0) >= limit) dsk[blk][c][e] &= 0xffff0000u;
          if (row_of(2 * e + 1, 0) >= limit) dsk[blk][c][e] &= 0xffffu;
        }
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rd(i);
    each<N>([&](auto group) __attribute__((always_inline)) {
      constexpr int i = decltype(group)::value, phase = i / KS, s = i % KS, E = 8 / KS;
      __builtin_amdgcn_sched_barrier(0);
      if (i == 4 * KS) hide(0);
      if (i == 5 * KS) hide(1);
      if (i + AHEAD < N) rd(i + AHEAD);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (phase < 4) {
          if (phase & 1) product_kept(dp[phase >> 1][c], op[i], dy[c].v[s], s == 0);
          else product_kept(x[phase >> 1][c], op[i], q[c].v[s], s == 0);
        } else {
          const uint32_t(&w)[8] = dsk[phase == 5][c];
          constexpr int q4 = (s / DB) * 4;
          accumulate(acc[c][s % DB], op[i], as_bf16x8(make_uint4(w[q4], w[q4 + 1], w[q4 + 2], w[q4 + 3])));
        }
      }
      // sums of the phase before, behind its last products and this group's
      if (s == 0 && (phase == 1 || phase == 3)) settled(x[phase >> 1]);
      if (s == 0 && (phase == 2 || phase == 4)) settled(dp[phase / 2 - 1]);
#pragma unroll
      for (int e = s * E; e < (s + 1) * E; ++e) {
        if (phase == 1 || phase == 3) weights(phase >> 1, e);
        if (phase == 2 || phase == 4) differences(phase / 2 - 1, e);
      }
    });
    __builtin_amdgcn_sched_barrier(0);
    if (t + 1 == t_hi) settled_all();
  }

#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int db = 0; db < DB; ++db) settled_acc(acc[c][db]);
  if (!active) return;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    if (a.marks) {
      const bool spoiled = Z::unbounded(acc[c]);
      if (lane == 0) *mark_of(a, split, bh, slot, 2 * wave + c) = spoiled;
    }
    const int row = wave_row + 32 * c + li, token = row / a.by_g, head = hk * a.G + (row - token * a.G);
    if (row >= at.end) continue;
    if (a.splits > 1) {
      const int64_t rows = (int64_t)a.B * a.Hk * a.Nq * a.G, out = split * rows + (int64_t)bh * a.Nq * a.G + row;
      Z::each_four(acc[c], lh, [&](int d, float4 v) { store_four(a.part + out * D + d, v); });
      continue;
    }
    T* o = static_cast<T*>(a.o) + b * a.ost.b + head * a.ost.h + token * a.ost.n;
    const float f = a.scale;
    Z::each_four(acc[c], lh, [&](int d, float4 v) { store_four(o + d, make_float4(v.x * f, v.y * f, v.z * f, v.w * f)); });
  }
}

// ---- the keys' and values' gradients: 128 keys a workgroup, a pass over the queries of all heads that share them
// Of a wave's registers the accumulators take 256 at d = 128 and the keys 64, and the values wait in LDS. A step of 32 queries is 4 x 16
// products of 32 cycles; the exponentials lie between the products of dy and v, ds = p (dp - delta) between those of p and dy.
template <int D, int CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kWaves, 1)
dense_dkv_kernel(DenseArgs a) {
  constexpr bool kPark = D == 128;
  using T = bf16_t;
  using Z = Tile<T, D, kPark ? 1 : 2>;
  constexpr int DB = D / 32, KS = D / 16, BN = Z::kRows, ROWB = Z::kRowBytes, AHEAD = 3;
  static_assert(kWaves * 64 == kDenseRows, "the tiles of the other kernels");
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes + (kPark ? 2 * kWaves * Z::kParked : 0)];  // two of Q, two of dy
  __shared__ __attribute__((aligned(256))) float stats[2][4][64];  // of a tile's rows: log-sum-exp, delta, slope, distance from the workgroup's first key
  int bh, slot, split;
  if (!dense_index(a, bh, slot, split)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<false>(a, b, kDenseRows, slot, lane);
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int wave_key = at.first + 64 * wave;
  const bool active = wave_key < at.end;
  // rows of the document [from, end) see key j of it; rows from `from_all` on see all keys of this wave
  const int end = doc.nq * a.G;
  int from[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) from[kb] = doc.first_seer(min(wave_key + 32 * kb + li, at.end - 1) - doc.k0) * a.G;
  const int from_all = uniform(doc.first_seer(min(wave_key + 63, at.end - 1) - doc.k0) * a.G);
  const int first_tile = doc.first_seer(at.first - doc.k0) * a.G / BN, tiles_end = (end + BN - 1) / BN;
  const int tiles = max(tiles_end - first_tile, 0);
  const int t_lo = uniform(first_tile + part_begin(tiles, split, a.splits)), t_hi = uniform(first_tile + part_begin(tiles, split + 1, a.splits));

  const Z z(lane);
  const Scores<T, CAP, SLOPES> scores(a);
  const uint32_t lds = lds_address(smem), lds_stats = lds_address(stats);
  const T* qp = static_cast<const T*>(a.q) + b * a.qst.b + hk * a.G * a.qst.h + doc.q0 * a.qst.n;
  const T* yp = static_cast<const T*>(a.dy) + b * a.yst.b + hk * a.G * a.yst.h + doc.q0 * a.yst.n;
  const int64_t stat0 = ((int64_t)b * a.H + hk * a.G) * a.Nq + doc.q0;
  // Where the strides leave a tile's offsets within 32 bits, rows lie at an offset of the lane from an address that the wave shares: at the
  // same one in every whole tile, if a key head has one query head.
  constexpr int kCopies = BN / Z::kRowsPerCopy / kWaves, kStep = kWaves * Z::kRowsPerCopy;
  const int copy_row = wave * Z::kRowsPerCopy + lane / Z::kChunks;
  auto is_near = [&](const Strides& st) { return st.n < (1 << 24) && (a.G == 1 || (a.G <= (1 << 24) && st.h < (1 << 24) && a.G * st.h <= (1 << 29))); };
  const bool near = is_near(a.qst) && is_near(a.yst);
  auto issue_rows = [&](int t) __attribute__((always_inline)) {
    const uint32_t q_to = (uint32_t)uniform((int)(lds + (t & 1) * Z::kBytes + wave * 1024)), y_to = q_to + 2 * Z::kBytes;
    auto chunk = [&](int i) { return ((lane % Z::kChunks) ^ Z::swz(i * kStep + copy_row)) * 16; };
    if (near && a.G == 1 && (t + 1) * BN <= end) {
      const T* q = static_cast<const T*>(uniform_ptr(qp + (int64_t)t * BN * a.qst.n));
      const T* y = static_cast<const T*>(uniform_ptr(yp + (int64_t)t * BN * a.yst.n));
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        async_copy_16B(q + (int64_t)(i * kStep) * a.qst.n, (uint32_t)copy_row * (uint32_t)a.qst.n * 2u + chunk(i), q_to + i * kWaves * 1024);
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        async_copy_16B(y + (int64_t)(i * kStep) * a.yst.n, (uint32_t)copy_row * (uint32_t)a.yst.n * 2u + chunk(i), y_to + i * kWaves * 1024);
      return;
    }
    const int token0 = uniform(t * BN / a.by_g);
    const T* q = static_cast<const T*>(uniform_ptr(qp + token0 * a.qst.n));
    const T* y = static_cast<const T*>(uniform_ptr(yp + token0 * a.yst.n));
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int row = min(t * BN + i * kStep + copy_row, end - 1), token = row / a.by_g, h = row - token * a.G, ahead = token - token0;
      if (near) {
        async_copy_16B(q, (__umul24(h, (uint32_t)a.qst.h) + __umul24(ahead, (uint32_t)a.qst.n)) * 2u + chunk(i), q_to + i * kWaves * 1024);
        async_copy_16B(y, (__umul24(h, (uint32_t)a.yst.h) + __umul24(ahead, (uint32_t)a.yst.n)) * 2u + chunk(i), y_to + i * kWaves * 1024);
      } else {
        async_copy_16B(q + h * a.qst.h + ahead * a.qst.n + chunk(i) / 2, q_to + i * kWaves * 1024);
        async_copy_16B(y + h * a.yst.h + ahead * a.yst.n + chunk(i) / 2, y_to + i * kWaves * 1024);
      }
    }
  };
  // Rows behind the document's last one: q's are that row's once more, whose products are masked, those of dy are cleared by the wave that
  // has copied them (as they are copied, lane by lane, it cost 4 % where heads share keys).
  auto clear_rows = [&](int t) __attribute__((always_inline)) {
    asm volatile("" ::: "memory");  // (behind the wait for the copies)
    const uint32_t to = (uint32_t)uniform((int)(lds + (2 + (t & 1)) * Z::kBytes + wave * 1024));
#pragma unroll
    for (int i = 0; i < kCopies; ++i)
      if (t * BN + i * kStep + copy_row >= end) clear_16B(to + i * kWaves * 1024 + lane * 16);
  };
  auto issue = [&](int t) __attribute__((always_inline)) {
    issue_rows(t);
    const int row = min(t * BN + lane, end - 1), token = row / a.by_g;
    const uint32_t to = (uint32_t)uniform((int)(lds_stats + ((t & 1) * 4 + wave) * 256));
    async_copy_4B((wave == 0 ? a.lse_in : a.delta) + stat0 + (int64_t)(row - token * a.G) * a.Nq + token, to);
    if (SLOPES && wave == 0) async_copy_4B(a.slopes + hk * a.G + row - token * a.G, to + 512);
    // (less a key's place among the workgroup's afterwards: as numbers of fp32, positions past 2^24 would lose what they differ by)
    if (SLOPES && wave == 1) stats[t & 1][3][lane] = (float)(doc.position(token) - (at.first - doc.k0));
  };
  if (t_lo < t_hi) issue(t_lo);

  typename Z::Column k[2], v[2];
  unsigned char* parked = smem + 4 * Z::kBytes + (kPark ? 2 * wave * Z::kParked : 0);
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    const int key = min(wave_key + 32 * kb + li, at.end - 1);
    k[kb].load(static_cast<const T*>(a.k) + b * a.kst.b + hk * a.kst.h + key * a.kst.n, lh);
    v[kb].load(static_cast<const T*>(a.v) + b * a.vst.b + hk * a.vst.h + key * a.vst.n, lh);
    if constexpr (kPark) Z::park(parked + kb * Z::kParked, v[kb], lane);
  }

  f32x16 dk[2][DB], dv[2][DB];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int db = 0; db < DB; ++db) clear(dk[kb][db]), clear(dv[kb][db]);

  // The products of 32 rows with the wave's keys: groups of two, 0 .. KS: q k, .. 2 KS: dy v, then p dy and ds q by 16 rows and 32 columns
  auto rows_of_tile = [&](int t, int rb, bool masked) __attribute__((always_inline)) {
    constexpr int N = 2 * KS + 4 * DB;
    const unsigned char* qt = smem + (t & 1) * Z::kBytes + rb * 32 * ROWB;
    const unsigned char* yt = smem + (2 + (t & 1)) * Z::kBytes + rb * 32 * ROWB;
    bf16x8 op[N], pv[KS][2];
    auto rd = [&](int i) __attribute__((always_inline)) {
      if (i < 2 * KS) {
        const int s = i < KS ? i : i - KS;
        op[i] = as_bf16x8(*reinterpret_cast<const uint4*>((i < KS ? qt : yt) + (z.row_off ^ (s << 5))));
        if (kPark && i >= KS)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) pv[s][kb] = as_bf16x8(*reinterpret_cast<const uint4*>(parked + kb * Z::kParked + s * 1024 + lane * 16));
      } else {
        const int u = i - 2 * KS, w = u < 2 * DB ? u : u - 2 * DB, off = z.tr_off ^ ((w % DB) << 6);
        const unsigned char* from16 = (u < 2 * DB ? yt : qt) + (w / DB) * 16 * ROWB;
        union { struct { v4i16 a, b; } s; bf16x8 v; } x;
        x.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(from16 + off));
        x.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(from16 + 8 * ROWB + (off ^ 32)));
        op[i] = x.v;
      }
    };
    auto of_rows = [&](int what, int g) { return *reinterpret_cast<const float4*>(&stats[t & 1][what][32 * rb + 8 * g + 4 * lh]); };
    f32x16 x[2], dp[2];
    uint32_t pk[2][8], dsk[2][8];
    // What rows that do not see a key have is taken out where there are such (branches that no accumulator's value goes through: in one
    // that it did, the compiler would move it).
    auto hide = [&](uint32_t (&c)[2][8]) __attribute__((always_inline)) {
      if (!masked) return;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        const int lo = from[kb] - (t * BN + 32 * rb + 4 * lh);
        const unsigned count = (unsigned)max(end - from[kb], 0);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if ((unsigned)(row_of(2 * e, 0) - lo) >= count) c[kb][e] &= 0xffff0000u;
          if ((unsigned)(row_of(2 * e + 1, 0) - lo) >= count) c[kb][e] &= 0xffffu;
        }
      }
    };
    float4 st[2], sl, po;
    auto weights = [&](int e) __attribute__((always_inline)) {  // of registers 2 e, 2 e + 1
      const int g = e >> 1, w = 2 * (e & 1);
      if (w == 0 && SLOPES) sl = of_rows(2, g), po = of_rows(3, g);
      if (w == 0 && g < 3) st[(g + 1) & 1] = of_rows(0, g + 1);
      const float lse[2] = {(w ? st[g & 1].z : st[g & 1].x) * kLog2e, (w ? st[g & 1].w : st[g & 1].y) * kLog2e};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        float p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = 2 * e + i;
          const float in = scores.inner(x[kb][r]);
          const float slope = SLOPES ? (w ? (i ? sl.w : sl.z) : (i ? sl.y : sl.x)) * kLog2e : 0.f;
          const float dist = SLOPES ? (w ? (i ? po.w : po.z) : (i ? po.y : po.x)) - (float)(64 * wave + 32 * kb + li) : 0.f;
          p[i] = __builtin_amdgcn_exp2f(scores.outer(in, dist, slope, lse[i]));
          x[kb][r] = CAP ? p[i] * scores.keeps(in) : p[i];
        }
        pk[kb][e] = pack2_bf16(p[0], p[1]);
      }
    };
    auto differences = [&](int e) __attribute__((always_inline)) {
      const int g = e >> 1, w = 2 * (e & 1);
      if (w == 0 && g < 3) st[(g + 1) & 1] = of_rows(1, g + 1);
      const float delta[2] = {w ? st[g & 1].z : st[g & 1].x, w ? st[g & 1].w : st[g & 1].y};
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        float ds[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int r = 2 * e + i;
          ds[i] = x[kb][r] * (dp[kb][r] - delta[i]);
        }
        dsk[kb][e] = pack2_bf16(ds[0], ds[1]);
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rd(i);
    each<N>([&](auto group) __attribute__((always_inline)) {
      constexpr int i = decltype(group)::value;
      __builtin_amdgcn_sched_barrier(0);
      if (i == 2 * KS) hide(pk);
      if (i == 2 * KS + 2 * DB) hide(dsk);
      if (i + AHEAD < N) rd(i + AHEAD);
      if (i == KS - 1) st[0] = of_rows(0, 0);
      if (i == 2 * KS - 1) st[0] = of_rows(1, 0);
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        if (i < KS) product(x[kb], op[i], k[kb].v[i], i == 0);
        else if (i < 2 * KS) product(dp[kb], op[i], kPark ? pv[i - KS][kb] : v[kb].v[i - KS], i == KS);
        else {
          const int u = i - 2 * KS, w = u < 2 * DB ? u : u - 2 * DB, q4 = (w / DB) * 4;
          const uint32_t(&c)[8] = u < 2 * DB ? pk[kb] : dsk[kb];
          f32x16& acc = u < 2 * DB ? dv[kb][w % DB] : dk[kb][w % DB];
          accumulate(acc, op[i], as_bf16x8(make_uint4(c[q4], c[q4 + 1], c[q4 + 2], c[q4 + 3])));
        }
      }
      if (i == KS) settled(x);
      if (i == 2 * KS) settled(dp);
      constexpr int E = 8 / KS, F = 8 / (2 * DB);
      if (i >= KS && i < 2 * KS)
#pragma unroll
        for (int e = (i - KS) * E; e < (i - KS + 1) * E; ++e) weights(e);
      if (i >= 2 * KS && i < 2 * KS + 2 * DB)
#pragma unroll
        for (int e = (i - 2 * KS) * F; e < (i - 2 * KS + 1) * F; ++e) differences(e);
    });
    __builtin_amdgcn_sched_barrier(0);
  };

  for (int t = t_lo; t < t_hi; ++t) {
    SVGEAR_WAIT_VMCNT(0);
    if ((t + 1) * BN > end) clear_rows(t);
    __syncthreads();
    if (t + 1 < t_hi) issue(t + 1);
    const bool masked = t * BN < from_all || (t + 1) * BN > end;
#pragma unroll
    for (int rb = 0; rb < Z::kBlocks; ++rb) rows_of_tile(t, rb, masked);
    if (t + 1 == t_hi) settled_all();
  }

#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int db = 0; db < DB; ++db) settled_acc(dk[kb][db]), settled_acc(dv[kb][db]);
  if (!active) return;
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) {
    if (a.marks) {
      const bool spoiled = Z::unbounded(dk[kb]) || Z::unbounded(dv[kb]);
      if (lane == 0) *mark_of(a, split, bh, slot, 2 * wave + kb) = spoiled;
    }
    const int key = wave_key + 32 * kb + li;
    if (key >= at.end) continue;
    const float f = a.scale;
    if (a.splits > 1) {
      const int64_t rows = (int64_t)a.B * a.Hk * a.Nk, out = split * rows + (int64_t)bh * a.Nk + key;
      Z::each_four(dk[kb], lh, [&](int d, float4 u) { store_four(a.part + out * D + d, make_float4(u.x * f, u.y * f, u.z * f, u.w * f)); });
      Z::each_four(dv[kb], lh, [&](int d, float4 u) { store_four(a.part + (a.splits * rows + out) * D + d, u); });
      continue;
    }
    T* ok = static_cast<T*>(a.dk) + b * a.dkst.b + hk * a.dkst.h + key * a.dkst.n;
    T* ov = static_cast<T*>(a.dv) + b * a.dvst.b + hk * a.dvst.h + key * a.dvst.n;
    Z::each_four(dk[kb], lh, [&](int d, float4 u) { store_four(ok + d, make_float4(u.x * f, u.y * f, u.z * f, u.w * f)); });
    Z::each_four(dv[kb], lh, [&](int d, float4 u) { store_four(ov + d, u); });
  }
}

template <int D, int CAP, bool SLOPES>
int launch_gradients(const DenseArgs& a, int what, hipStream_t s) {
  if (what == kDenseDq) dense_dq_kernel<D, CAP, SLOPES><<<dense_grid(a), 64 * kWaves, 0, s>>>(a);
  else dense_dkv_kernel<D, CAP, SLOPES><<<dense_grid(a), 64 * kWaves, 0, s>>>(a);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

}  // namespace
}  // namespace svgear

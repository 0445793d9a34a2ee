// The gradients of dense attention with masks in bf16: the workgroup's four waves own 128 rows and share the other side's tiles.
#include "dense_tile.h"

namespace svgear {
namespace {

// ---- the queries' gradients: 128 queries a workgroup, a pass over the keys
template <int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, 2)
dense_dq_kernel(DenseArgs a) {
  using T = bf16_t;
  using Z = Tile<T, D>;
  constexpr int DB = D / 32, BN = Z::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes];
  int bh, slot;
  if (!dense_index(a, bh, slot)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<true>(a, b, kDenseRows, a.causal ? a.slots - 1 - slot : slot, lane);  // causal: the longest first
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int wave_row = at.first + 32 * wave, row = wave_row + li, row_c = min(row, at.end - 1);
  const bool active = wave_row < at.end;
  const int token = row_c / a.by_g, head = hk * a.G + (row_c - token * a.G);
  const int pos = doc.position(token - doc.q0), hi = doc.seen(token - doc.q0);
  const int hi_all = doc.seen(min(wave_row, at.end - 1) / a.by_g - doc.q0), hi_any = doc.seen(min(wave_row + 31, at.end - 1) / a.by_g - doc.q0);
  const int hi_wg = doc.seen((min(at.first + kDenseRows, at.end) - 1) / a.by_g - doc.q0);
  const int split = blockIdx.y, tiles = (hi_wg + BN - 1) / BN;
  const int t_lo = part_begin(tiles, split, a.splits), t_hi = part_begin(tiles, split + 1, a.splits);

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

  if (!active) return;
  if (a.marks) {
    const bool spoiled = Z::unbounded(acc);
    if (lane == 0) *mark_of(a, split, bh, slot, wave) = spoiled;
  }
  if (row >= at.end) return;
  if (a.splits > 1) {
    const int64_t rows = (int64_t)a.B * a.Hk * a.Nq * a.G, out = split * rows + (int64_t)bh * a.Nq * a.G + row;
    Z::each_four(acc, lh, [&](int d, float4 v) { store_four(a.part + out * D + d, v); });
    return;
  }
  T* o = static_cast<T*>(a.o) + b * a.ost.b + head * a.ost.h + token * a.ost.n;
  const float f = a.scale;
  Z::each_four(acc, lh, [&](int d, float4 v) { store_four(o + d, make_float4(v.x * f, v.y * f, v.z * f, v.w * f)); });
}

// f(0), f(1), .. f(N - 1) with constants (a loop of this length over so much is not unrolled)
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// ---- the keys' and values' gradients: 128 keys a workgroup, a pass over the queries of all heads that share them
// A wave has 64 keys and a SIMD to itself: 512 registers, of which the accumulators take 256 at d = 128 and the keys 64, and the values
// wait in LDS. An operand read from a tile goes into two products (with 32 keys a wave, two waves a SIMD, the reads of LDS took longer
// than the products). A step of 32 queries is 4 x 16 products of 32 cycles; the exponentials lie between the products of dy and v, the
// differences from delta between those of p and dy, and the operands are read AHEAD pairs of products before their own.
constexpr int kDkvWaves = 2;

// Products whose sums are kept in vector registers (x) and in accumulation registers (acc): the compiler, which is free to choose, moves
// half of the accumulators between the two kinds in every step. It does not know of these instructions' latency: a sum that is read by
// another kind of instruction is read behind `settled` (11 cycles of 4 at least after the last product; here 20), and the two
// idle ones before a product are for an operand that was just written.
__device__ __forceinline__ void product(f32x16& x, const bf16x8& a, const bf16x8& b, bool first) {
  if (first) asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, 0" : "=&v"(x) : "v"(a), "v"(b));
  else asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+v"(x) : "v"(a), "v"(b));
}
__device__ __forceinline__ void settled(f32x16 (&x)[2]) { asm volatile("s_nop 15\n\ts_nop 3" : "+v"(x[0]), "+v"(x[1])); }
__device__ __forceinline__ void accumulate(f32x16& acc, const bf16x8& a, const bf16x8& b) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
__device__ __forceinline__ void settled_acc(f32x16& acc) { asm volatile("s_nop 15\n\ts_nop 3" : "+a"(acc)); }

template <int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDkvWaves, 1)
dense_dkv_kernel(DenseArgs a) {
  constexpr bool kPark = D == 128;
  using T = bf16_t;
  using Z = Tile<T, D, kPark ? 1 : 2>;
  constexpr int DB = D / 32, KS = D / 16, BN = Z::kRows, ROWB = Z::kRowBytes, AHEAD = 3;
  static_assert(kDkvWaves * 64 == kDenseRows, "the tiles of the other kernels");
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes + (kPark ? 2 * kDkvWaves * Z::kParked : 0)];  // two of Q, two of dy
  __shared__ __attribute__((aligned(256))) float stats[2][4][64];  // of a tile's rows: log-sum-exp, delta, slope, position
  int bh, slot;
  if (!dense_index(a, bh, slot)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<false>(a, b, kDenseRows, slot, lane);
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int wave_key = at.first + 64 * wave;
  const bool active = wave_key < at.end;
  // rows of the document [from, end) see key j of it; rows from `from_all` on see all keys of this wave
  const int j0 = wave_key + li - doc.k0, end = doc.nq * a.G;
  int from[2];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb) from[kb] = doc.first_seer(min(wave_key + 32 * kb + li, at.end - 1) - doc.k0) * a.G;
  const int from_all = uniform(doc.first_seer(min(wave_key + 63, at.end - 1) - doc.k0) * a.G);
  const int first_tile = doc.first_seer(at.first - doc.k0) * a.G / BN, tiles_end = (end + BN - 1) / BN;
  const int tiles = max(tiles_end - first_tile, 0), split = blockIdx.y;
  const int t_lo = uniform(first_tile + part_begin(tiles, split, a.splits)), t_hi = uniform(first_tile + part_begin(tiles, split + 1, a.splits));

  const Z z(lane);
  const Scores<T, CAP, SLOPES> scores(a);
  const uint32_t lds = lds_address(smem), lds_stats = lds_address(stats);
  const T* qp = static_cast<const T*>(a.q) + b * a.qst.b + hk * a.G * a.qst.h + doc.q0 * a.qst.n;
  const T* yp = static_cast<const T*>(a.dy) + b * a.yst.b + hk * a.G * a.yst.h + doc.q0 * a.yst.n;
  const int64_t stat0 = ((int64_t)b * a.H + hk * a.G) * a.Nq + doc.q0;
  // Rows of a whole tile lie at one offset of the lane from addresses that the wave shares, where a key head has one query head and
  // the strides leave the offsets within 32 bits.
  constexpr int kCopies = BN / Z::kRowsPerCopy / kDkvWaves, kStep = kDkvWaves * Z::kRowsPerCopy;
  const int copy_row = wave * Z::kRowsPerCopy + lane / Z::kChunks;
  const bool even = a.G == 1 && a.qst.n <= (1 << 24) && a.yst.n <= (1 << 24);
  auto issue_rows = [&](int t, const T* base, const Strides& st, int buffer) __attribute__((always_inline)) {
    const uint32_t to = (uint32_t)uniform((int)(lds + buffer * Z::kBytes + wave * 1024));
    if (even && (t + 1) * BN <= end) {
      const T* rows = static_cast<const T*>(uniform_ptr(base + (int64_t)t * BN * st.n));
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        async_copy_16B(rows + (int64_t)(i * kStep) * st.n, (uint32_t)copy_row * (uint32_t)st.n * 2u + ((lane % Z::kChunks) ^ Z::swz(i * kStep + copy_row)) * 16,
                       to + i * kDkvWaves * 1024);
    } else {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int r = i * kStep + copy_row, row = min(t * BN + r, end - 1), token = row / a.by_g;
        async_copy_16B(base + (row - token * a.G) * st.h + token * st.n + ((lane % Z::kChunks) ^ Z::swz(r)) * 8, to + i * kDkvWaves * 1024);
      }
    }
  };
  auto issue = [&](int t) __attribute__((always_inline)) {
    issue_rows(t, qp, a.qst, t & 1);
    issue_rows(t, yp, a.yst, 2 + (t & 1));
    const int row = min(t * BN + lane, end - 1), token = row / a.by_g;
    const uint32_t to = (uint32_t)uniform((int)(lds_stats + ((t & 1) * 4 + wave) * 256));
    async_copy_4B((wave == 0 ? a.lse_in : a.delta) + stat0 + (int64_t)(row - token * a.G) * a.Nq + token, to);
    if (SLOPES && wave == 0) async_copy_4B(a.slopes + hk * a.G + row - token * a.G, to + 512);
    if (SLOPES && wave == 1) stats[t & 1][3][lane] = (float)doc.position(token);
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
          const float dist = SLOPES ? (w ? (i ? po.w : po.z) : (i ? po.y : po.x)) - (float)(j0 + 32 * kb) : 0.f;
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
    __syncthreads();
    if (t + 1 < t_hi) issue(t + 1);
    const bool masked = t * BN < from_all || (t + 1) * BN > end;
#pragma unroll
    for (int rb = 0; rb < Z::kBlocks; ++rb) rows_of_tile(t, rb, masked);
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

template <int D>
int launch(const DenseArgs& a, int what, hipStream_t s) {
  return by_scores(a, [&](auto cap, auto slopes) -> int {
    constexpr bool C = decltype(cap)::value, S = decltype(slopes)::value;
    if (what == kDenseDq) dense_dq_kernel<D, C, S><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    else dense_dkv_kernel<D, C, S><<<dense_grid(a), 64 * kDkvWaves, 0, s>>>(a);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  });
}

}  // namespace

int launch_dense_backward_bf16(const DenseArgs& a, int d, int what, hipStream_t s) { return d == 64 ? launch<64>(a, what, s) : launch<128>(a, what, s); }
}  // namespace svgear

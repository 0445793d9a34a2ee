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

// ---- the keys' and values' gradients: 128 keys a workgroup, a pass over the queries of all heads that share them
template <int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, 2)
dense_dkv_kernel(DenseArgs a) {
  // Two waves a SIMD, one's exponentials under the other's products, leave 256 registers: at d = 128 in bf16 the accumulators
  // take 128 and the keys 32, and the values wait in LDS, under tiles of 32 rows.
  constexpr bool kPark = D == 128;
  using T = bf16_t;
  using Z = Tile<T, D, kPark ? 1 : 2>;
  constexpr int DB = D / 32, BN = Z::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes + (kPark ? kDenseWaves * Z::kParked : 0)];  // two of Q, two of dy
  __shared__ __attribute__((aligned(256))) float stats[2][4][64];  // of a tile's rows: log-sum-exp, delta, slope, position
  int bh, slot;
  if (!dense_index(a, bh, slot)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<false>(a, b, kDenseRows, slot, lane);
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int wave_key = at.first + 32 * wave, key = wave_key + li, key_c = min(key, at.end - 1);
  const bool active = wave_key < at.end;
  // rows of the document [from, end) see key j of it; rows from `from_all` on see all keys of this wave, from from_any on one of them
  const int j = key_c - doc.k0, from = doc.first_seer(j) * a.G, end = doc.nq * a.G;
  const int from_all = doc.first_seer(min(wave_key + 31, at.end - 1) - doc.k0) * a.G;
  const int from_any = doc.first_seer(min(wave_key, at.end - 1) - doc.k0) * a.G;
  const int first_tile = doc.first_seer(at.first - doc.k0) * a.G / BN, tiles_end = (end + BN - 1) / BN;
  const int tiles = max(tiles_end - first_tile, 0), split = blockIdx.y;
  const int t_lo = first_tile + part_begin(tiles, split, a.splits), t_hi = first_tile + part_begin(tiles, split + 1, a.splits);

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
      const int row = min(t * BN + r, end - 1), token = row / a.by_g;
      return (row - token * a.G) * st.h + token * st.n;
    };
    copy_tile<Z>(qp, lds + (t & 1) * Z::kBytes, wave, lane, [&](int r) { return offset(r, a.qst); });
    copy_tile<Z>(yp, lds + (2 + (t & 1)) * Z::kBytes, wave, lane, [&](int r) { return offset(r, a.yst); });
    const int row = min(t * BN + lane, end - 1), token = row / a.by_g;
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
        if (CAP || SLOPES) __builtin_amdgcn_sched_barrier(0);  // (four rows after four: together they take registers that are not there)
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

  if (!active) return;
  if (a.marks) {
    const bool spoiled = Z::unbounded(dk) || Z::unbounded(dv);
    if (lane == 0) *mark_of(a, split, bh, slot, wave) = spoiled;
  }
  if (key >= at.end) return;
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

template <int D>
int launch(const DenseArgs& a, int what, hipStream_t s) {
  return by_scores(a, [&](auto cap, auto slopes) -> int {
    constexpr bool C = decltype(cap)::value, S = decltype(slopes)::value;
    if (what == kDenseDq) dense_dq_kernel<D, C, S><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    else dense_dkv_kernel<D, C, S><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  });
}

}  // namespace

int launch_dense_backward_bf16(const DenseArgs& a, int d, int what, hipStream_t s) { return d == 64 ? launch<64>(a, what, s) : launch<128>(a, what, s); }
}  // namespace svgear

// The gradients of dense attention with masks in fp32.
#include "dense_solo.h"

namespace svgear {
namespace {

// ---- the queries' gradients: 32 queries a workgroup, a pass over the keys
template <int D, int CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, D == 64 ? 2 : 1)
dense_dq_f32_kernel(DenseArgs a) {
  using Z = Tile<float, D>;
  using S = Solo<D>;
  constexpr int DB = D / 32, BN = S::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[kDenseWaves * S::kWave];  // of a wave: a tile of K, one of V
  int bh, slot, split;
  if (!dense_index(a, bh, slot, split)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<true>(a, b, S::kRows, a.causal ? a.slots - 1 - slot : slot, lane);  // causal: the longest first
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int row = min(at.first + li, at.end - 1), token = row / a.by_g, head = hk * a.G + (row - token * a.G);
  const int pos = doc.position(token - doc.q0), hi = doc.seen(token - doc.q0);
  const int hi_all = doc.seen(at.first / a.by_g - doc.q0), hi_any = doc.seen((min(at.first + S::kRows, at.end) - 1) / a.by_g - doc.q0);
  const int tiles = (hi_any + BN - 1) / BN;
  const int t_lo = part_begin(tiles, split, a.splits), t_hi = part_begin(tiles, split + 1, a.splits);

  typename Z::Column q, dy;
  q.load(static_cast<const float*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n, lh);
  dy.load(static_cast<const float*>(a.dy) + b * a.yst.b + head * a.yst.h + token * a.yst.n, lh);
  const int64_t stat = ((int64_t)b * a.H + head) * a.Nq + token;
  const float lse2 = a.lse_in[stat] * kLog2e, delta = a.delta[stat];
  const float slope = SLOPES ? a.slopes[head] * kLog2e : 0.f;
  SVGEAR_WAIT_VMCNT(0);

  const Z z(lane);
  const Scores<float, CAP, SLOPES> scores(a);
  const unsigned char* kt = smem + wave * S::kWave;
  const unsigned char* vt = kt + Z::kBytes;
  const uint32_t lds = lds_address(kt);
  const float* kp = static_cast<const float*>(a.k) + b * a.kst.b + hk * a.kst.h + doc.k0 * a.kst.n;
  const float* vp = static_cast<const float*>(a.v) + b * a.vst.b + hk * a.vst.h + doc.k0 * a.vst.n;
  auto issue = [&](const float* base, int64_t st, int t, uint32_t to) __attribute__((always_inline)) {
    const int last = hi_any - 1 - t * BN;
    copy_solo<D>(base + (int64_t)t * BN * st, to, lane, [&](int r) { return (int64_t)min(r, last) * st; });
  };

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(acc[db]);
  int t = t_lo + wave;
  if (t < t_hi) {
    issue(vp, a.vst.n, t, lds + Z::kBytes);
    issue(kp, a.kst.n, t, lds);
  }
  for (; t < t_hi; t += kDenseWaves) {
    const bool more = t + kDenseWaves < t_hi;
    f32x16 x, dp;
    clear(x);
    clear(dp);
    SVGEAR_WAIT_VMCNT(S::kCopies);  // V has landed, which was issued first
    asm volatile("" ::: "memory");
    z.rows_times(vt, dy, dp);
    SVGEAR_WAIT_VMCNT(0);
    asm volatile("" ::: "memory");
    if (more) issue(vp, a.vst.n, t + kDenseWaves, lds + Z::kBytes);
    z.rows_times(kt, q, x);
    const bool masked = (t + 1) * BN > hi_all;
    const int base = t * BN + 4 * lh, limit = hi - base;
    const float ahead = (float)(pos - base);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float in = scores.inner(x[r]);
      float ds = __builtin_amdgcn_exp2f(scores.outer(in, ahead - (float)row_of(r, 0), slope, lse2)) * (dp[r] - delta);
      if (CAP) ds *= scores.keeps(in);
      x[r] = masked && row_of(r, 0) >= limit ? 0.f : ds;
    }
    z.transposed_times(kt, x, acc, lane);
    if (more) issue(kp, a.kst.n, t + kDenseWaves, lds);
  }

  if (a.marks) {
    const bool spoiled = Z::unbounded(acc);
    if (lane == 0) *mark_of(a, split, bh, slot, wave) = spoiled;
  }
  const int64_t rows = (int64_t)a.B * a.Hk * a.Nq * a.G, part0 = split * rows + (int64_t)bh * a.Nq * a.G + at.first;
  meet<D>(smem, acc, wave, lane, [](int, int) { return 1.f; }, [&](int r, int d, float4 v) {
    if (at.first + r >= at.end) return;
    if (a.splits > 1) {
      store_four(a.part + (part0 + r) * D + d, v);
      return;
    }
    const int tok = (at.first + r) / a.by_g, hd = hk * a.G + (at.first + r - tok * a.G);
    store_four(static_cast<float*>(a.o) + b * a.ost.b + hd * a.ost.h + tok * a.ost.n + d, times(v, a.scale));
  });
}

// ---- the keys' and values' gradients: 32 keys a workgroup, a pass over the queries of all heads that share them
template <int D, int CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, D == 64 ? 2 : 1)
dense_dkv_f32_kernel(DenseArgs a) {
  using Z = Tile<float, D>;
  using S = Solo<D>;
  constexpr int DB = D / 32, BN = S::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[kDenseWaves * S::kWave];  // of a wave: a tile of Q, one of dy
  __shared__ __attribute__((aligned(256))) float stats_s[kDenseWaves][4][64];           // of its rows: log-sum-exp, delta, slope, distance from the first key
  int bh, slot, split;
  if (!dense_index(a, bh, slot, split)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<false>(a, b, S::kRows, slot, lane);
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  // rows of the document [from, end) see key j of it; from from_all on all keys of this workgroup, from from_any on one of them
  const int key = min(at.first + li, at.end - 1), j = key - doc.k0, from = doc.first_seer(j) * a.G, end = doc.nq * a.G;
  const int from_all = doc.first_seer(min(at.first + S::kRows, at.end) - 1 - doc.k0) * a.G;
  const int first_tile = doc.first_seer(at.first - doc.k0) * a.G / BN;
  const int tiles = max((end + BN - 1) / BN - first_tile, 0);
  const int t_lo = first_tile + part_begin(tiles, split, a.splits), t_hi = first_tile + part_begin(tiles, split + 1, a.splits);

  typename Z::Column k, v;
  k.load(static_cast<const float*>(a.k) + b * a.kst.b + hk * a.kst.h + key * a.kst.n, lh);
  v.load(static_cast<const float*>(a.v) + b * a.vst.b + hk * a.vst.h + key * a.vst.n, lh);
  if (D == 128) k.keep(), v.keep();
  SVGEAR_WAIT_VMCNT(0);

  const Z z(lane);
  const Scores<float, CAP, SLOPES> scores(a);
  const unsigned char* qt = smem + wave * S::kWave;
  const unsigned char* yt = qt + Z::kBytes;
  float (*stats)[64] = stats_s[wave];
  const uint32_t lds = lds_address(qt), lds_stats = lds_address(stats);
  const float* qp = static_cast<const float*>(a.q) + b * a.qst.b + hk * a.G * a.qst.h + doc.q0 * a.qst.n;
  const float* yp = static_cast<const float*>(a.dy) + b * a.yst.b + hk * a.G * a.yst.h + doc.q0 * a.yst.n;
  const int64_t stat0 = ((int64_t)b * a.H + hk * a.G) * a.Nq + doc.q0;
  // (the heads of a key head divide the rows of a copy, and the strides leave a lane's offset within 32 bits)
  constexpr int64_t kNear = 1 << 24;
  const bool even = Z::kRowsPerCopy % a.G == 0 && a.qst.n <= kNear && a.yst.n <= kNear && (a.G == 1 || (a.qst.h <= kNear && a.yst.h <= kNear));
  auto issue = [&](const float* base, const Strides& st, int t, uint32_t to) __attribute__((always_inline)) {
    if (even && (t + 1) * BN <= end) {
      const int l = again(lane), r = l / Z::kChunks, token = r / a.by_g;
      copy_solo<D>(base + (t * BN) / a.by_g * st.n, Z::kRowsPerCopy / a.by_g * st.n,
                   ((uint32_t)(r - token * a.G) * (uint32_t)st.h + (uint32_t)token * (uint32_t)st.n) * 4u, to, l);
      return;
    }
    copy_solo<D>(base, to, again(lane), [&](int r) {
      const int row = min(t * BN + r, end - 1), token = row / a.by_g;
      return (row - token * a.G) * st.h + token * st.n;
    });
  };
  constexpr int kStats = 2 + SLOPES;
  auto issue_stats = [&](int t) __attribute__((always_inline)) {
    const int row = min(t * BN + (again(lane) & 31), end - 1), token = row / a.by_g;
    const int64_t stat = stat0 + (int64_t)(row - token * a.G) * a.Nq + token;
    async_copy_4B(a.lse_in + stat, (uint32_t)uniform((int)lds_stats));
    async_copy_4B(a.delta + stat, (uint32_t)uniform((int)(lds_stats + 256)));
    if (SLOPES) {
      async_copy_4B(a.slopes + hk * a.G + row - token * a.G, (uint32_t)uniform((int)(lds_stats + 512)));
      // (positions past 2^24 would lose as numbers of fp32 what they differ by)
      stats[3][lane] = (float)(doc.position(token) - (at.first - doc.k0));
    }
  };

  f32x16 dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(dk[db]), clear(dv[db]);
  int t = t_lo + wave;
  if (t < t_hi) {
    issue(yp, a.yst, t, lds + Z::kBytes);
    issue_stats(t);
    issue(qp, a.qst, t, lds);
  }
  for (; t < t_hi; t += kDenseWaves) {
    const bool more = t + kDenseWaves < t_hi, masked = t * BN < from_all || (t + 1) * BN > end;
    f32x16 x, dp;
    clear(x);
    clear(dp);
    SVGEAR_WAIT_VMCNT(S::kCopies + kStats);  // dy has landed, which was issued first
    asm volatile("" ::: "memory");
    if ((t + 1) * BN > end) clear_solo<D>(lds + Z::kBytes, end - t * BN, again(lane));
    z.rows_times(yt, v, dp);
    SVGEAR_WAIT_VMCNT(0);
    asm volatile("" ::: "memory");
    z.rows_times(qt, k, x);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if (CAP || SLOPES) __builtin_amdgcn_sched_barrier(0);  // (four rows after four: together they take registers that are not there)
      auto of_rows = [&](int what) { return *reinterpret_cast<const float4*>(&stats[what][8 * g + 4 * lh]); };
      const float4 ls = of_rows(0), de = of_rows(1);
      const float lse[4] = {ls.x, ls.y, ls.z, ls.w}, delta[4] = {de.x, de.y, de.z, de.w};
      float slope[4] = {0.f, 0.f, 0.f, 0.f}, dist[4] = {0.f, 0.f, 0.f, 0.f};
      if (SLOPES) {
        const float4 sl = of_rows(2), po = of_rows(3);
        slope[0] = sl.x * kLog2e, slope[1] = sl.y * kLog2e, slope[2] = sl.z * kLog2e, slope[3] = sl.w * kLog2e;
        dist[0] = po.x - (float)li, dist[1] = po.y - (float)li, dist[2] = po.z - (float)li, dist[3] = po.w - (float)li;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * g + i, row = t * BN + row_of(r, lh);
        const float in = scores.inner(x[r]);
        float p = __builtin_amdgcn_exp2f(scores.outer(in, dist[i], slope[i], lse[i] * kLog2e));
        float ds = p * (dp[r] - delta[i]);
        if (CAP) ds *= scores.keeps(in);
        if (masked && (row < from || row >= end)) p = ds = 0.f;
        x[r] = p;
        dp[r] = ds;
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    z.transposed_times(yt, x, dv, lane);
    __builtin_amdgcn_sched_barrier(0);
    if (more) {
      issue(yp, a.yst, t + kDenseWaves, lds + Z::kBytes);
      issue_stats(t + kDenseWaves);
    }
    z.transposed_times(qt, dp, dk, lane);
    if (more) issue(qp, a.qst, t + kDenseWaves, lds);
  }

  if (a.marks) {
    const bool spoiled = Z::unbounded(dk) || Z::unbounded(dv);
    if (lane == 0) *mark_of(a, split, bh, slot, wave) = spoiled;
  }
  const int64_t rows = (int64_t)a.B * a.Hk * a.Nk, part0 = split * rows + (int64_t)bh * a.Nk + at.first;
  auto put = [&](void* to, const Strides& st, int64_t part, float f) {
    return [=, &a](int r, int d, float4 u) {
      if (at.first + r >= at.end) return;
      if (a.splits > 1) store_four(a.part + (part + r) * D + d, times(u, f));
      else store_four(static_cast<float*>(to) + b * st.b + hk * st.h + (at.first + r) * st.n + d, times(u, f));
    };
  };
  auto one = [](int, int) { return 1.f; };
  meet<D>(smem, dk, wave, lane, one, put(a.dk, a.dkst, part0, a.scale));
  __syncthreads();
  meet<D>(smem, dv, wave, lane, one, put(a.dv, a.dvst, a.splits * rows + part0, 1.f));
}

template <int D>
int launch(const DenseArgs& a, int what, hipStream_t s) {
  return by_scores(a, [&](auto cap, auto slopes) -> int {
    constexpr int C = decltype(cap)::value;
    constexpr bool S = decltype(slopes)::value;
    if (what == kDenseDq) dense_dq_f32_kernel<D, C, S><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    else dense_dkv_f32_kernel<D, C, S><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  });
}

}  // namespace

int launch_dense_backward_f32(const DenseArgs& a, int d, int what, hipStream_t s) { return d == 64 ? launch<64>(a, what, s) : launch<128>(a, what, s); }
}  // namespace svgear

// Dense attention with masks in bf16.
//
// What bounds it: the matrix cores and the vector unit alike. A step of a wave (64 keys, 32 queries, d = 128) is 32 products of 32
// cycles, and 32 exponentials a lane at a quarter of the rate with their scaling, maximum, sum and conversion, some 950 cycles.
// So a wave issues the exponentials of a tile between the products of the next tile's scores, and the next tile's maximum between
// the products with the values; two workgroups share a CU and fill what is left. 9,450 packed tokens of 40 heads take 1,075 us, 1,090
// TFLOP/s with the matrix cores busy 58 % of the cycles at 1.7 GHz, the power limit's clock. Where there are few tiles of keys, what
// precedes the first products counts as much as they do: 2 x 37,800 queries over texts of at most 512 758 us, of a workgroup's 29,000 cycles 12,500
// in the loop. (Rows by way of LDS, 256 bytes of a row at a time, change nothing there; nor do workgroups that take several tiles of queries.)
#include <cfloat>

#include "dense_tile.h"

namespace svgear {
namespace {

// log2 headroom before the running maximum is refreshed; none at d = 64, where the weight of a row's largest score is then exactly 1
template <int D>
constexpr float kHeadroom = D == 64 ? 0.f : 8.f;

// A row of results: the lanes l and l + 32 hold alternate fours of its columns; they exchange halves and store 16 bytes each.
template <int DB>
__device__ __forceinline__ void store_whole(bf16_t* o, const f32x16 (&acc)[DB], float f, int lh, bool live) {
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      const f32x16& x = acc[db];
      const uint32_t a0 = pack2_bf16(x[4 * g] * f, x[4 * g + 1] * f), a1 = pack2_bf16(x[4 * g + 2] * f, x[4 * g + 3] * f);
      const uint32_t b0 = pack2_bf16(x[4 * g + 4] * f, x[4 * g + 5] * f), b1 = pack2_bf16(x[4 * g + 6] * f, x[4 * g + 7] * f);
      const auto u = __builtin_amdgcn_permlane32_swap(a0, b0, false, false), v = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
      if (live) *reinterpret_cast<uint4*>(o + 32 * db + 8 * g + 8 * lh) = make_uint4(u[0], v[0], u[1], v[1]);
    }
}

template <int D, int CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, 2)
dense_forward_bf16_kernel(DenseArgs a) {
  using Z = Tile<bf16_t, D>;
  constexpr int DB = D / 32, KS = D / 16, BN = Z::kRows, ROWB = Z::kRowBytes;
  constexpr int AHEAD = CAP && !SLOPES ? 3 : 4;  // operands read before the product that takes them; as many as registers are left
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes];  // two of K, two of V
  int bh, slot, split;
  if (!dense_index(a, bh, slot, split)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<true>(a, b, kDenseRows, a.causal ? a.slots - 1 - slot : slot, lane);  // causal: the longest first
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int wave_row = at.first + 32 * wave, row = min(wave_row + li, at.end - 1);
  const int token = row / a.by_g, head = hk * a.G + (row - token * a.G);
  const int pos = doc.position(token - doc.q0) - 4 * lh, hi = doc.seen(token - doc.q0) - 4 * lh;  // (less what a lane's first key is)
  // keys that every row of this wave sees, and that some row of the workgroup sees
  const int hi_all = uniform(doc.seen(min(wave_row, at.end - 1) / a.by_g - doc.q0));
  const int hi_wg = uniform(doc.seen((min(at.first + kDenseRows, at.end) - 1) / a.by_g - doc.q0));
  const int tiles = (hi_wg + BN - 1) / BN;
  const int t_lo = uniform(part_begin(tiles, split, a.splits)), t_hi = uniform(part_begin(tiles, split + 1, a.splits));

  const float slope = SLOPES ? a.slopes[head] * kLog2e : 0.f;

  const Z z(lane);
  const uint32_t lds = lds_address(smem);
  const bf16_t* kp = static_cast<const bf16_t*>(a.k) + b * a.kst.b + hk * a.kst.h + doc.k0 * a.kst.n;
  const bf16_t* vp = static_cast<const bf16_t*>(a.v) + b * a.vst.b + hk * a.vst.h + doc.k0 * a.vst.n;
  // Rows of a whole tile lie at one offset of the lane from addresses that the wave shares; in the last tile, rows behind the last key
  // that a query here sees are not read: K's are that key's once more, whose scores are masked, V's are 0.
  const int copy_row = wave * Z::kRowsPerCopy + lane / Z::kChunks, copy_chunk = ((lane % Z::kChunks) ^ Z::swz(copy_row)) * 16;
  constexpr int kStep = kDenseWaves * Z::kRowsPerCopy;
  static_assert(kStep % 16 == 0, "all copies of a lane have one chunk");
  const uint32_t k_lane = (uint32_t)copy_row * (uint32_t)a.kst.n * 2u + copy_chunk, v_lane = (uint32_t)copy_row * (uint32_t)a.vst.n * 2u + copy_chunk;
  auto issue = [&](int t, const bf16_t* base, int64_t st, uint32_t at_lane, int buffer, bool values) __attribute__((always_inline)) {
    const bf16_t* rows = static_cast<const bf16_t*>(uniform_ptr(base + (int64_t)t * BN * st));
    const uint32_t to = (uint32_t)uniform((int)(lds + buffer * Z::kBytes + wave * 1024));
    const int last = hi_wg - 1 - t * BN;
    if (last >= BN - 1) {
#pragma unroll
      for (int i = 0; i < Z::kCopies; ++i) async_copy_16B(rows + (int64_t)(i * kStep) * st, at_lane, to + i * kDenseWaves * 1024);
    } else {
      const int l = again(lane), mine = wave * Z::kRowsPerCopy + l / Z::kChunks, chunk = ((l % Z::kChunks) ^ Z::swz(mine)) * 16;
#pragma unroll
      for (int i = 0; i < Z::kCopies; ++i) {
        if (values && i * kStep + mine > last) clear_16B(to + i * kDenseWaves * 1024 + l * 16);
        else async_copy_16B(rows, (uint32_t)min(i * kStep + mine, last) * (uint32_t)st * 2u + chunk, to + i * kDenseWaves * 1024);
      }
    }
  };
  auto issue_k = [&](int t) __attribute__((always_inline)) { issue(t, kp, a.kst.n, k_lane, (t - t_lo) & 1, false); };
  auto issue_v = [&](int t) __attribute__((always_inline)) { issue(t, vp, a.vst.n, v_lane, 2 + ((t - t_lo) & 1), true); };

  // the first tiles are on their way while the queries are fetched
  if (t_lo < t_hi) {
    issue_k(t_lo);
    issue_v(t_lo);
  }
  typename Z::Column q;
  q.load(static_cast<const bf16_t*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n, lh);
  if (a.scale < 0.f) {  // (the maximum is that of the unscaled scores)
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      union { bf16x8 v; uint4 u; } c;
      c.v = q.v[s];
      c.u.x ^= 0x80008000u, c.u.y ^= 0x80008000u, c.u.z ^= 0x80008000u, c.u.w ^= 0x80008000u;
      q.v[s] = c.v;
    }
  }

  Scores<bf16_t, CAP, SLOPES> scores_of(a);
  scores_of.c = uniform(fabsf(scores_of.c));
  scores_of.cap2 = uniform(scores_of.cap2);
  // A cap's tanh between the products: cap2 tanh(z) = z P(z^2) cap2 for |z| <= 0.5, P the best fit of degree 3, off by 6e-7 of it at
  // most; in products s, whose factor c is in the coefficients. A tile with a larger one takes the exponential and the reciprocal,
  // two more operations at a quarter of the rate, and so does every tile where a factor is so large that a coefficient would be (8,704 tokens of 40 heads, 8 key heads, causal, the kernel: 440 us so, 390 by the series).
  constexpr bool SERIES = CAP && !SLOPES;
  float series[4];
  if (SERIES) {
    constexpr float p[4] = {0.99999946f, -0.33326376f, 0.13190912f, -0.04441858f};
    float f = scores_of.c * scores_of.cap2;
#pragma unroll
    for (int i = 0; i < 4; ++i, f *= scores_of.c * scores_of.c) series[i] = uniform(p[i] * f);
  }
  auto by_series = [&](float s, float add) __attribute__((always_inline)) {
    const float u = s * s;
    float p = series[3];
#pragma unroll
    for (int i = 2; i >= 0; --i) p = __builtin_fmaf(p, u, series[i]);
    return __builtin_fmaf(s, p, add);
  };
  bool raw = false;  // whether the scores whose maximum is known are still products, for the series
  // (infinite where no tile takes the series: no product times it is 0.5 or less; a series' tile has no other use for it)
  const float c0 = SERIES && !(fabsf(series[3]) <= FLT_MAX) ? INFINITY : scores_of.c;
  f32x16 acc[DB], sA[2], sB[2];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(acc[db]);
#pragma unroll
  for (int k = 0; k < 2; ++k) clear(sA[k]), clear(sB[k]);
  float m = -INFINITY;
  uint32_t pk[2][8];
  float cc = c0;  // factor still to be applied to the scores whose maximum is known

  float ls[2] = {0.f, 0.f};
  auto weigh = [&](const f32x16 (&sc)[2], int e, float neg_m, auto raw_tag) __attribute__((always_inline)) {
    constexpr bool RAW = decltype(raw_tag)::value;
    const int k = e >> 3, r = 2 * (e & 7);
    const float p0 = __builtin_amdgcn_exp2f(RAW ? by_series(sc[k][r], neg_m) : __builtin_fmaf(sc[k][r], cc, neg_m));
    const float p1 = __builtin_amdgcn_exp2f(RAW ? by_series(sc[k][r + 1], neg_m) : __builtin_fmaf(sc[k][r + 1], cc, neg_m));
    pk[k][r >> 1] = pack2_bf16(p0, p1);
    ls[e & 1] += p0 + p1;
  };
  // Scores of the K tile in `buffer` into sn, and between those products, with EXPS, the weights of the scores sc into pk
  auto scores = [&](int buffer, f32x16 (&sn)[2], const f32x16 (&sc)[2], auto exps_tag, auto raw_tag) __attribute__((always_inline)) {
    constexpr bool EXPS = decltype(exps_tag)::value;
    const unsigned char* kt = smem + buffer * Z::kBytes;
    bf16x8 kf[2 * KS];
    auto rd = [&](int i) { kf[i] = as_bf16x8(*reinterpret_cast<const uint4*>(kt + (i & 1) * 32 * ROWB + (z.row_off ^ ((i >> 1) << 5)))); };
    clear(sn[0]);
    clear(sn[1]);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rd(i);
    const float neg_m = m == -INFINITY ? 0.f : -m;
    constexpr int E = 16 / (2 * KS);  // pairs of scores per product
#pragma unroll
    for (int i = 0; i < 2 * KS; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i + AHEAD < 2 * KS) rd(i + AHEAD);
      sn[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i], q.v[i >> 1], sn[i & 1], 0, 0, 0);
      if constexpr (EXPS) {
#pragma unroll
        for (int e = i * E; e < (i + 1) * E; ++e) weigh(sc, e, neg_m, raw_tag);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto max_pair = [&](const f32x16 (&sn)[2], float& mx, int e) __attribute__((always_inline)) {
    const int k = e >> 3, r = 2 * (e & 7);
    mx = fmaxf(fmaxf(mx, sn[k][r]), sn[k][r + 1]);
  };
  float most = 0.f;  // of a tile's products, for the series
  auto most_pair = [&](const f32x16 (&sn)[2], int e) __attribute__((always_inline)) {
    const int k = e >> 3, r = 2 * (e & 7);
    if (SERIES) most = fmaxf(fmaxf(most, fabsf(sn[k][r])), fabsf(sn[k][r + 1]));
  };
  // The running maximum covers the scores sn of the keys' tile t afterwards; where there is more to them than a factor, they are exponents.
  auto settle = [&](int t, f32x16 (&sn)[2], float mx, auto whole_tag) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(whole_tag)::value;  // seen by all rows of the wave, as the caller knows
    const bool masked = !WHOLE && (t + 1) * BN > hi_all;
    cc = c0;
    raw = SERIES && !masked && !__any(!(most * c0 <= 0.5f));
    if ((CAP && !raw) || SLOPES || masked) {
      asm volatile("");  // (a branch: found for every tile, and chosen from, it would cost as much as if it were needed)
      const int limit = masked ? hi - t * BN : INT32_MAX;  // (constants on the other side of the comparisons)
      const float ahead = (float)(pos - t * BN);
      mx = -INFINITY;
      cc = 1.f;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = 32 * k + row_of(r, 0);
          const float x = scores_of.outer(scores_of.inner(sn[k][r]), ahead - (float)j, slope, 0.f);
          sn[k][r] = !WHOLE && j >= limit ? -INFINITY : x;
          mx = fmaxf(mx, sn[k][r]);
        }
    }
    mx = fmaxf(mx, swap32(mx));
    const float ms = raw ? by_series(mx, 0.f) : mx * cc;
    if (__any(ms > m + kHeadroom<D>)) {
      const float m_new = fmaxf(m, ms), alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
#pragma unroll
      for (int u = 0; u < 2; ++u) ls[u] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
      m = m_new;
    }
  };
  // O^T += V^T P^T with the V tile in `buffer`, and between those products, with MORE, the maximum of the next scores sn
  auto values = [&](int buffer, const f32x16 (&sn)[2], auto more_tag) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more_tag)::value && !SLOPES;
    constexpr int N = 4 * DB;
    bf16x8 vf[N];
    auto rd = [&](int i) {
      const unsigned char* at = smem + (2 + buffer) * Z::kBytes + (i / DB) * 16 * ROWB;
      const int off = z.tr_off ^ ((i % DB) << 6);
      union { struct { v4i16 a, b; } s; bf16x8 v; } u;
      u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(at + off));
      u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(at + 8 * ROWB + (off ^ 32)));
      vf[i] = u.v;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rd(i);
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    most = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i + AHEAD < N) rd(i + AHEAD);
      const int ks = i / DB, k = ks >> 1, u4 = (ks & 1) * 4;
      const bf16x8 bp = as_bf16x8(make_uint4(pk[k][u4], pk[k][u4 + 1], pk[k][u4 + 2], pk[k][u4 + 3]));
      acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], bp, acc[i % DB], 0, 0, 0);
      if (MORE && i >= N / 4) {
#pragma unroll
        for (int e = (i - N / 4) * 16 / (3 * N / 4); e < (i + 1 - N / 4) * 16 / (3 * N / 4); ++e) max_pair(sn, mx[e & 3], e), most_pair(sn, e);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
  };

  // Step t takes the weights of its scores and its values, and finds the scores of step t + 1; K(t + 2) and V(t + 1) are copied
  // meanwhile, over K(t) and V(t - 1), which step t - 1 was the last to read.
  if (t_lo < t_hi) {
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
    if (t_lo + 1 < t_hi) issue_k(t_lo + 1);
    scores(0, sA, sB, std::false_type{}, std::false_type{});
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; ++e) max_pair(sA, mx, e), most_pair(sA, e);
    settle(t_lo, sA, mx, std::false_type{});
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
    auto step = [&](int t, int parity, f32x16 (&s_now)[2], f32x16 (&s_next)[2], auto whole_tag) __attribute__((always_inline)) {
      if (t + 2 < t_hi) issue(t + 2, kp, a.kst.n, k_lane, parity, false);
      issue(t + 1, vp, a.vst.n, v_lane, 2 + (parity ^ 1), true);
      if (SERIES && raw) scores(parity ^ 1, s_next, s_now, std::true_type{}, std::integral_constant<bool, SERIES>{});
      else scores(parity ^ 1, s_next, s_now, std::true_type{}, std::false_type{});
      const float next = values(parity, s_next, std::true_type{});
      settle(t + 1, s_next, next, whole_tag);
      SVGEAR_WAIT_VMCNT(0);
      __syncthreads();
    };
    int t = t_lo;
    const int whole = min(t_hi, hi_all / BN);  // up to here without a mask for this wave
    for (; t + 2 < whole; t += 2) {
      step(t, 0, sA, sB, std::true_type{});
      step(t + 1, 1, sB, sA, std::true_type{});
    }
    for (; t + 2 < t_hi; t += 2) {
      step(t, 0, sA, sB, std::false_type{});
      step(t + 1, 1, sB, sA, std::false_type{});
    }
    auto last = [&](int parity, const f32x16 (&s)[2]) __attribute__((always_inline)) {
      const float neg_m = m == -INFINITY ? 0.f : -m;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (SERIES && raw) weigh(s, e, neg_m, std::integral_constant<bool, SERIES>{});
        else weigh(s, e, neg_m, std::false_type{});
      }
      __builtin_amdgcn_sched_barrier(0);
      values(parity, s, std::false_type{});
    };
    if (t + 1 < t_hi) {
      step(t, 0, sA, sB, std::false_type{});
      last(1, sB);
    } else {
      last(0, sA);
    }
  }

  if (a.marks) {
    const bool spoiled = Z::unbounded(acc);
    if (lane == 0) *mark_of(a, split, bh, slot, wave) = spoiled;
  }
  float l = ls[0] + ls[1];
  l += swap32(l);
  const int l2 = again(lane), out_row = min(wave_row + (l2 & 31), at.end - 1), out_token = out_row / a.by_g;
  const int out_head = hk * a.G + (out_row - out_token * a.G);
  const bool live = wave_row + (l2 & 31) < at.end;
  if (a.splits > 1) {
    if (!live) return;
    const int64_t rows = (int64_t)a.B * a.Hk * a.Nq * a.G, out = split * rows + (int64_t)bh * a.Nq * a.G + out_row;
    if (l2 < 32) a.part_ml[out] = make_float2(m, l);
    Z::each_four(acc, l2 >> 5, [&](int d, float4 v) { store_four(a.part + out * D + d, v); });
    return;
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
  store_whole(static_cast<bf16_t*>(a.o) + b * a.ost.b + out_head * a.ost.h + out_token * a.ost.n, acc, inv, l2 >> 5, live);
  if (live && a.lse && l2 < 32) a.lse[((int64_t)b * a.H + out_head) * a.Nq + out_token] = (m + log2f(l)) * kLn2;
}

template <int D>
int launch(const DenseArgs& a, hipStream_t s) {
  return by_scores<true>(a, [&](auto cap, auto slopes) -> int {
    dense_forward_bf16_kernel<D, decltype(cap)::value, decltype(slopes)::value><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  });
}

}  // namespace

int launch_dense_bf16(const DenseArgs& a, int d, hipStream_t s) { return d == 64 ? launch<64>(a, s) : launch<128>(a, s); }
}  // namespace svgear

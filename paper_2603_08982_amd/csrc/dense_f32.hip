// Dense attention with masks in fp32.
#include "dense_solo.h"

namespace svgear {
namespace {

template <int D, int CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, D == 64 ? 2 : 1)
dense_forward_f32_kernel(DenseArgs a) {
  using Z = Tile<float, D>;
  using S = Solo<D>;
  constexpr int DB = D / 32, BN = S::kRows;
  __shared__ __attribute__((aligned(256))) unsigned char smem[kDenseWaves * S::kWave];  // of a wave: a tile of K, one of V
  __shared__ float ml[kDenseWaves][2][32];                                              // of a wave: maximum, sum of each row
  int bh, slot, split;
  if (!dense_index(a, bh, slot, split)) return;
  const int b = bh / a.by_hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const Found at = find_tile<true>(a, b, S::kRows, a.causal ? a.slots - 1 - slot : slot, lane);  // causal: the longest first
  if (at.first >= at.end) return;
  const Document& doc = at.doc;

  const int row = min(at.first + li, at.end - 1), token = row / a.by_g, head = hk * a.G + (row - token * a.G);
  const int pos = doc.position(token - doc.q0), hi = doc.seen(token - doc.q0);
  // keys that every row sees, and that some row sees
  const int hi_all = doc.seen(at.first / a.by_g - doc.q0), hi_any = doc.seen((min(at.first + S::kRows, at.end) - 1) / a.by_g - doc.q0);
  const int tiles = (hi_any + BN - 1) / BN;
  const int t_lo = part_begin(tiles, split, a.splits), t_hi = part_begin(tiles, split + 1, a.splits);

  typename Z::Column q;
  q.load(static_cast<const float*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n, lh);
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
    const int last = hi_any - 1 - t * BN;  // (keys that no row here sees are not read)
    copy_solo<D>(base + (int64_t)t * BN * st, to, lane, [&](int r) { return (int64_t)min(r, last) * st; });
  };

  f32x16 acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(acc[db]);
  float m = -INFINITY, l = 0.f;
  int t = t_lo + wave;
  if (t < t_hi) {
    issue(kp, a.kst.n, t, lds);
    issue(vp, a.vst.n, t, lds + Z::kBytes);
  }
  for (; t < t_hi; t += kDenseWaves) {
    SVGEAR_WAIT_VMCNT(S::kCopies);  // K has landed
    asm volatile("" ::: "memory");
    const bool more = t + kDenseWaves < t_hi;
    f32x16 x;
    clear(x);
    z.rows_times(kt, q, x);
    if (more) issue(kp, a.kst.n, t + kDenseWaves, lds);
    float mx = -INFINITY;
    const int base = t * BN + 4 * lh, limit = hi - base;
    const float ahead = (float)(pos - base);
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = scores.outer(scores.inner(x[r]), ahead - (float)row_of(r, 0), slope, 0.f);
    if ((t + 1) * BN > hi_all) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (row_of(r, 0) >= limit) x[r] = -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, x[r]);
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
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r] = __builtin_amdgcn_exp2f(x[r] - m_use);
      s[r & 3] += x[r];
    }
    l += (s[0] + s[1]) + (s[2] + s[3]);
    if (more) SVGEAR_WAIT_VMCNT(S::kCopies);  // V has landed; the next K may be on its way
    else SVGEAR_WAIT_VMCNT(0);
    asm volatile("" ::: "memory");
    if ((t + 1) * BN > hi_any) clear_solo<D>(lds + Z::kBytes, hi_any - t * BN, again(lane));
    z.transposed_times(vt, x, acc, lane);
    if (more) issue(vp, a.vst.n, t + kDenseWaves, lds + Z::kBytes);
  }

  if (a.marks) {
    const bool spoiled = Z::unbounded(acc);
    if (lane == 0) *mark_of(a, split, bh, slot, wave) = spoiled;
  }
  l += swap32(l);
  if (lh == 0) ml[wave][0][li] = m, ml[wave][1][li] = l;
  const int64_t rows = (int64_t)a.B * a.Hk * a.Nq * a.G, part0 = split * rows + (int64_t)bh * a.Nq * a.G + at.first;
  auto top = [&](int r) {
    float M = ml[0][0][r];
#pragma unroll
    for (int w = 1; w < kDenseWaves; ++w) M = fmaxf(M, ml[w][0][r]);
    return M;
  };
  auto share = [&](int w, int r) { return ml[w][0][r] == -INFINITY ? (ml[w][1][r] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(ml[w][0][r] - top(r)); };
  meet<D>(smem, acc, wave, lane, share, [&](int r, int d, float4 v) {
    if (at.first + r >= at.end) return;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kDenseWaves; ++w) sum = __builtin_fmaf(share(w, r), ml[w][1][r], sum);
    if (a.splits > 1) {
      store_four(a.part + (part0 + r) * D + d, v);
      if (d == 0) a.part_ml[part0 + r] = make_float2(top(r), sum);
      return;
    }
    const int tok = (at.first + r) / a.by_g, hd = hk * a.G + (at.first + r - tok * a.G);
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    store_four(static_cast<float*>(a.o) + b * a.ost.b + hd * a.ost.h + tok * a.ost.n + d, times(v, inv));
    if (a.lse && d == 0) a.lse[((int64_t)b * a.H + hd) * a.Nq + tok] = (top(r) + log2f(sum)) * kLn2;
  });
}

template <int D>
int launch(const DenseArgs& a, hipStream_t s) {
  return by_scores(a, [&](auto cap, auto slopes) -> int {
    dense_forward_f32_kernel<D, decltype(cap)::value, decltype(slopes)::value><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  });
}

}  // namespace

int launch_dense_f32(const DenseArgs& a, int d, hipStream_t s) { return d == 64 ? launch<64>(a, s) : launch<128>(a, s); }
}  // namespace svgear

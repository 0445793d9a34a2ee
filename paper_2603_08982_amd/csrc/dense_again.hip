// What is left to do with a causal mask where a masked value is an infinity or a NaN.
#include "dense_tile.h"

namespace svgear {
namespace {

// ---- Masked values that are unbounded
// A masked weight is 0, and 0 times an infinity or a NaN is a NaN: a product on the matrix cores lets such a value through to rows that do
// not see it. So with a causal mask a wave that ends with such a value leaves a mark. The kernels here, behind the others, look at the
// marked waves' rows: where one that some of them do not see holds such a value, they find the 32 again, from memory, by the vector unit,
// each row of the other side for those alone that see it, up to where every sum is a NaN. Without a mark they read that and end. (Checks
// of the tiles themselves, in the loops that copy them, cost registers that are not there.) The two halves of a wave have half of a
// row's columns each. Without a mark a launch costs its length: 8,704 tokens of 40 heads with a prefix 397 -> 404 us, the gradients of
// 8 heads of 1,531 tokens in fp32 121 -> 129 (two launches). A marked wave takes some 2 us a key.
__device__ __forceinline__ float4 load_four(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load_four(const bf16_t* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u));
}
// half of the columns of a row
template <int D>
struct Half {
  float4 v[D / 8];
  __device__ __forceinline__ void set(float f) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) v[i] = make_float4(f, f, f, f);
  }
  template <typename T>
  __device__ __forceinline__ void add(float f, const T* row) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      const float4 u = load_four(row + 4 * i);
      v[i].x = __builtin_fmaf(f, u.x, v[i].x), v[i].y = __builtin_fmaf(f, u.y, v[i].y);
      v[i].z = __builtin_fmaf(f, u.z, v[i].z), v[i].w = __builtin_fmaf(f, u.w, v[i].w);
    }
  }
  __device__ __forceinline__ void scale(float f) {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) v[i].x *= f, v[i].y *= f, v[i].z *= f, v[i].w *= f;
  }
  // whether nothing but NaN can follow
  __device__ __forceinline__ bool lost() const {
    bool all = true;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) all = all && v[i].x != v[i].x && v[i].y != v[i].y && v[i].z != v[i].z && v[i].w != v[i].w;
    return all;
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row) const {
#pragma unroll
    for (int i = 0; i < D / 8; ++i) store_four(row + 4 * i, v[i]);
  }
};
template <int D, typename T>
__device__ __forceinline__ float dot_halves(const T* a, const T* b) {
  float s = 0.f;
#pragma unroll 8
  for (int d = 0; d < D / 2; d += 4) {
    const float4 u = load_four(a + d), v = load_four(b + d);
    s = __builtin_fmaf(u.x, v.x, s), s = __builtin_fmaf(u.y, v.y, s), s = __builtin_fmaf(u.z, v.z, s), s = __builtin_fmaf(u.w, v.w, s);
  }
  return s + swap32(s);
}

// Whether one of rows [lo, hi), `rn` apart, is unbounded: D / 4 lanes a row. (Up to 2^30 rows, behind a prefix: no count of their elements.)
template <int D, typename T>
__device__ __forceinline__ bool unbounded_rows(const T* rows, int64_t rn, int lo, int hi, int lane) {
  constexpr int L = D / 4;
  float zero = 0.f;
  for (int r = lo + lane / L; r < hi; r += 64 / L) {
    const float4 u = load_four(rows + r * rn + lane % L * 4);
    for (float x : {u.x, u.y, u.z, u.w}) zero = __builtin_fmaf(x, 0.f, zero);
  }
  return __any(!(zero == 0.f));
}

// A query's output over its keys [0, hi); j_hi: the most that one of the wave has.
template <typename T, int D, int CAP, bool SLOPES>
__device__ __forceinline__ void again_forward(const T* q, const T* k, int64_t kn, const T* v, int64_t vn, int j_hi, int hi, int pos,
                                              float slope, const DenseArgs& a, T* o, float* lse, bool live) {
  const Scores<float, CAP, SLOPES> scores(a);  // (fp32's, which is right for all caps)
  const int at = (threadIdx.x & 32) ? D / 2 : 0;
  Half<D> acc;
  acc.set(0.f);
  float m = -INFINITY, l = 0.f;
  for (int j = 0; j < j_hi; ++j) {
    if (j % 64 == 63 && __all(acc.lost() || l != l || j >= hi)) break;
    const float x = scores.outer(scores.inner(dot_halves<D>(q + at, k + j * kn + at)), (float)(pos - j), slope, 0.f);
    if (j >= hi) continue;
    const float m_new = fmaxf(m, x), use = m_new == -INFINITY ? 0.f : m_new;
    const float f = __builtin_amdgcn_exp2f(m - use), p = __builtin_amdgcn_exp2f(x - use);
    l = __builtin_fmaf(l, f, p);
    acc.scale(f);
    acc.add(p, v + j * vn + at);
    m = m_new;
  }
  if (!live) return;
  acc.scale(l > 0.f ? 1.f / l : l == 0.f ? 0.f : l);
  acc.store(o + at);
  if (lse && at == 0) *lse = (m + log2f(l)) * kLn2;
}

// A query's gradient.
template <typename T, int D, int CAP, bool SLOPES>
__device__ __forceinline__ void again_dq(const T* q, const T* dy, const T* k, int64_t kn, const T* v, int64_t vn, int j_hi, int hi,
                                         int pos, float slope, float lse2, float delta, const DenseArgs& a, T* o, bool live) {
  const Scores<float, CAP, SLOPES> scores(a);  // (fp32's, which is right for all caps)
  const int at = (threadIdx.x & 32) ? D / 2 : 0;
  Half<D> acc;
  acc.set(0.f);
  for (int j = 0; j < j_hi; ++j) {
    if (j % 64 == 63 && __all(acc.lost() || j >= hi)) break;
    const float in = scores.inner(dot_halves<D>(q + at, k + j * kn + at)), dp = dot_halves<D>(dy + at, v + j * vn + at);
    if (j >= hi) continue;
    float ds = __builtin_amdgcn_exp2f(scores.outer(in, (float)(pos - j), slope, lse2)) * (dp - delta);
    if (CAP) ds *= scores.keeps(in);
    acc.add(ds, k + j * kn + at);
  }
  if (!live) return;
  acc.scale(a.scale);
  acc.store(o + at);
}

// A key's gradient (DK), or a value's, over the rows [r_lo, r_hi) from `from` on: token r / G of head r % G.
template <typename T, int D, int CAP, bool SLOPES, bool DK>
__device__ __forceinline__ void again_dkv(const T* k, const T* v, const T* q, int64_t qh, int64_t qn, const T* dy, int64_t yh, int64_t yn,
                                          const float* lse, const float* delta, const float* slopes, int r_lo, int r_hi, int from, int ahead,
                                          const DenseArgs& a, T* o, bool live) {
  const Scores<float, CAP, SLOPES> scores(a);  // (fp32's, which is right for all caps)
  const int at = (threadIdx.x & 32) ? D / 2 : 0;
  Half<D> acc;
  acc.set(0.f);
  for (int r = r_lo; r < r_hi; ++r) {
    if (r % 64 == 63 && __all(acc.lost())) break;
    const int token = r / a.by_g, h = r - token * a.G;
    const T* qr = q + h * qh + token * qn;
    const T* yr = dy + h * yh + token * yn;
    const int64_t stat = (int64_t)h * a.Nq + token;
    const float in = scores.inner(dot_halves<D>(k + at, qr + at)), dp = DK ? dot_halves<D>(v + at, yr + at) : 0.f;
    if (r < from) continue;
    const float p = __builtin_amdgcn_exp2f(scores.outer(in, (float)(token + ahead), SLOPES ? slopes[h] * kLog2e : 0.f, lse[stat] * kLog2e));
    if (DK) acc.add(p * (dp - delta[stat]) * (CAP ? scores.keeps(in) : 1.f), qr + at);
    else acc.add(p, yr + at);
  }
  if (!live) return;
  if (DK) acc.scale(a.scale);
  acc.store(o + at);
}

// The rows of the workgroups' waves that have left a mark in a part of theirs. WHAT as of the kernel that left it, on the same grid.
// SOLO: a workgroup's waves share 32 rows (fp32).
template <typename T, int D, int CAP, bool SLOPES, int WHAT>
__global__ void __launch_bounds__(64 * kDenseWaves)
dense_again_kernel(DenseArgs a) {
  constexpr bool SOLO = sizeof(T) == 4;
  int bh, slot, split;
  if (!dense_index(a, bh, slot, split) || split > 0) return;
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), b = bh / a.by_hk, hk = bh - b * a.Hk;
  if (SOLO && wave > 0) return;
  const int tile = a.causal && WHAT != kDenseDkv ? a.slots - 1 - slot : slot;
  const Found at = find_tile<WHAT != kDenseDkv>(a, b, SOLO ? 32 : kDenseRows, tile, lane);
  const int first = at.first + 32 * wave;
  if (first >= at.end) return;
  bool marked = false;
  for (int s = 0; s < a.splits; ++s)
    for (int w = SOLO ? 0 : wave; w <= (SOLO ? kDenseWaves - 1 : wave); ++w) marked |= *mark_of(a, s, bh, slot, w) != 0;
  if (!marked) return;

  const Document& doc = at.doc;
  const int own = min(first + (lane & 31), at.end - 1);
  const bool live = first + (lane & 31) < at.end;
  const T* kp = static_cast<const T*>(a.k) + b * a.kst.b + hk * a.kst.h;
  const T* vp = static_cast<const T*>(a.v) + b * a.vst.b + hk * a.vst.h;
  if constexpr (WHAT == kDenseDkv) {
    const T* qp = static_cast<const T*>(a.q) + b * a.qst.b + hk * a.G * a.qst.h + doc.q0 * a.qst.n;
    const T* yp = static_cast<const T*>(a.dy) + b * a.yst.b + hk * a.G * a.yst.h + doc.q0 * a.yst.n;
    const int64_t stat0 = ((int64_t)b * a.H + hk * a.G) * a.Nq + doc.q0;
    const int j = own - doc.k0, from = doc.first_seer(j) * a.G, end = doc.nq * a.G, ahead = doc.position(0) - j;
    const int r_lo = doc.first_seer(first - doc.k0) * a.G;
    // tokens that the wave has read for nothing: a workgroup's tiles begin at, or up to 64 rows before, the first that sees its first key
    const int lo = max(0, doc.first_seer(at.first - doc.k0) - 64), hi = min(doc.nq, doc.first_seer(min(first + 32, at.end) - 1 - doc.k0));
    bool found = false;
    for (int h = 0; h < a.G; ++h)
      found = found || unbounded_rows<D>(qp + h * a.qst.h, a.qst.n, lo, hi, lane) || unbounded_rows<D>(yp + h * a.yst.h, a.yst.n, lo, hi, lane);
    if (!found) return;
    const float* slopes = SLOPES ? a.slopes + hk * a.G : nullptr;
    again_dkv<T, D, CAP, SLOPES, true>(kp + own * a.kst.n, vp + own * a.vst.n, qp, a.qst.h, a.qst.n, yp, a.yst.h, a.yst.n, a.lse_in + stat0,
                                       a.delta + stat0, slopes, r_lo, end, from, ahead, a,
                                       static_cast<T*>(a.dk) + b * a.dkst.b + hk * a.dkst.h + own * a.dkst.n, live);
    again_dkv<T, D, CAP, SLOPES, false>(kp + own * a.kst.n, vp + own * a.vst.n, qp, a.qst.h, a.qst.n, yp, a.yst.h, a.yst.n, a.lse_in + stat0,
                                        a.delta + stat0, slopes, r_lo, end, from, ahead, a,
                                        static_cast<T*>(a.dv) + b * a.dvst.b + hk * a.dvst.h + own * a.dvst.n, live);
  } else {
    const int token = own / a.by_g, head = hk * a.G + (own - token * a.G);
    const int pos = doc.position(token - doc.q0), hi = doc.seen(token - doc.q0), hi_any = doc.seen((min(first + 32, at.end) - 1) / a.by_g - doc.q0);
    const float slope = SLOPES ? a.slopes[head] * kLog2e : 0.f;
    const int64_t stat = ((int64_t)b * a.H + head) * a.Nq + token;
    const T* q = static_cast<const T*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n;
    T* o = static_cast<T*>(a.o) + b * a.ost.b + head * a.ost.h + token * a.ost.n;
    kp += doc.k0 * a.kst.n;
    vp += doc.k0 * a.vst.n;
    // keys that the wave has read for nothing: a workgroup's tiles end at, or up to 64 keys behind, the last that its last row sees
    const int lo = doc.seen(first / a.by_g - doc.q0), past = doc.seen((min(at.first + (SOLO ? 32 : kDenseRows), at.end) - 1) / a.by_g - doc.q0) + 64;
    if (!unbounded_rows<D>(WHAT == kDenseDq ? kp : vp, WHAT == kDenseDq ? a.kst.n : a.vst.n, lo, min(past, doc.nk), lane)) return;
    if constexpr (WHAT == kDenseForward) {
      again_forward<T, D, CAP, SLOPES>(q, kp, a.kst.n, vp, a.vst.n, hi_any, hi, pos, slope, a, o, a.lse ? a.lse + stat : nullptr, live);
    } else {
      again_dq<T, D, CAP, SLOPES>(q, static_cast<const T*>(a.dy) + b * a.yst.b + head * a.yst.h + token * a.yst.n, kp, a.kst.n, vp, a.vst.n, hi_any, hi,
                                  pos, slope, a.lse_in[stat] * kLog2e, a.delta[stat], a, o, live);
    }
  }
}

template <typename T, int D, int WHAT>
int launch(const DenseArgs& a, hipStream_t s) {
  return by_scores(a, [&](auto cap, auto slopes) -> int {
    dense_again_kernel<T, D, decltype(cap)::value, decltype(slopes)::value, WHAT><<<dense_grid(a), 64 * kDenseWaves, 0, s>>>(a);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  });
}
template <typename T, int D>
int launch_what(const DenseArgs& a, int what, hipStream_t s) {
  return what == kDenseForward ? launch<T, D, kDenseForward>(a, s) : what == kDenseDq ? launch<T, D, kDenseDq>(a, s) : launch<T, D, kDenseDkv>(a, s);
}

}  // namespace

int launch_dense_again(const DenseArgs& a, svgear_dtype dt, int d, int what, hipStream_t s) {
  if (dt == SVGEAR_F32) return d == 64 ? launch_what<float, 64>(a, what, s) : launch_what<float, 128>(a, what, s);
  return d == 64 ? launch_what<bf16_t, 64>(a, what, s) : launch_what<bf16_t, 128>(a, what, s);
}
}  // namespace svgear

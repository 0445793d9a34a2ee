// svgear_attention and svgear_attention_backward: argument checks, how many parts the work is cut into, and the small kernels
// around those of dense_tile.h.
#include "dense_attention.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

#include "linear.h"

namespace svgear {
namespace {

constexpr int64_t kMaxDenseRows = (int64_t)1 << 30;
constexpr int kMaxDocs = 1 << 20;
constexpr int64_t kMaxKeyStride = 1 << 24;
constexpr int kThreads = 256;

// Where a row of `part` goes: row r of key head (b, hk) is token r / G of head hk G + r % G.
struct Out {
  void* p;
  Strides st;
  int N, G, Hk;
};
__device__ __forceinline__ int64_t out_offset(const Out& o, int64_t u, int& head, int& token, int& b) {
  const int per = o.N * o.G;
  const int bh = (int)(u / per), r = (int)(u - (int64_t)bh * per);
  b = bh / o.Hk;
  token = r / o.G;
  head = (bh - b * o.Hk) * o.G + (r - token * o.G);
  return (int64_t)b * o.st.b + (int64_t)head * o.st.h + (int64_t)token * o.st.n;
}

// The parts of every row of the forward pass, in their order: a thread per eight columns.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
dense_merge_kernel(const float* part, const float2* ml, int splits, int64_t rows, Out o, float* lse) {
  const int64_t u = (int64_t)long_grid_index() * kThreads + threadIdx.x, row = u / (D / 8);
  if (row >= rows) return;
  const int d = 8 * (int)(u % (D / 8));
  float M = -INFINITY, l = 0.f, acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  // (eight parts' loads at a time: one after the other, 50 parts of 320 rows took 22 us)
  constexpr int U = 8;
  for (int s = 0; s < splits; s += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) M = fmaxf(M, ml[min(s + u, splits - 1) * rows + row].x);
  }
  for (int s = 0; s < splits; s += U) {
    float2 p[U];
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = min(s + u, splits - 1) * rows + row;
      p[u] = ml[at];
      load8(part + at * D + d, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= splits || (p[u].x == -INFINITY && p[u].y == 0.f)) continue;  // no key there
      const float w = __builtin_amdgcn_exp2f(p[u].x - M);
      l = __builtin_fmaf(w, p[u].y, l);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(w, v[u][i], acc[i]);
    }
  }
  const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] *= inv;
  int head, token, b;
  store8(static_cast<T*>(o.p) + out_offset(o, row, head, token, b) + d, acc);
  if (lse && d == 0) lse[((int64_t)b * o.Hk * o.G + head) * o.N + token] = (M + log2f(l)) * 0.6931471805599453f;
}

// out = factor * the parts of every row, added in their order.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
dense_sum_kernel(const float* part, int splits, int64_t rows, float factor, Out first, Out second) {
  const int64_t u = (int64_t)long_grid_index() * kThreads + threadIdx.x, row = u / (D / 8);
  if (row >= rows) return;
  const Out& o = blockIdx.y ? second : first;
  if (blockIdx.y) part += splits * rows * D;
  const int d = 8 * (int)(u % (D / 8));
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    float v[8];
    load8(part + (s * rows + row) * D + d, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] += v[i];
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] *= factor;
  int head, token, b;
  store8(static_cast<T*>(o.p) + out_offset(o, row, head, token, b) + d, acc);
}

// delta = sum over d of dy o: D / 8 lanes a row.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
dense_delta_kernel(const T* dy, Strides yst, const T* o, Strides ost, int H, int N, int64_t rows, float* delta) {
  constexpr int L = D / 8;
  const int64_t row = ((int64_t)long_grid_index() * kThreads + threadIdx.x) / L;
  const int d = 8 * (int)(threadIdx.x % L);
  float s = 0.f;
  if (row < rows) {
    const int bh = (int)(row / N), n = (int)(row - (int64_t)bh * N);
    float a[8], c[8];
    load8(dy + head_base(yst, bh, H) + n * yst.n + d, a);
    load8(o + head_base(ost, bh, H) + n * ost.n + d, c);
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(a[i], c[i], s);
  }
#pragma unroll
  for (int q = 1; q < L; q <<= 1) s += __shfl_xor(s, q);
  if (row < rows && d == 0) delta[row] = s;
}

// ---- how many parts the rows of the other side are cut into: so many that some 512 workgroups (two a CU) have work, but two
// tiles a part at least. `own`: rows a key head has on the workgroups' side, `other`: on the other. Where a head's rows are one
// tile (single tokens), the parts cost little and are finer, four tiles each, so that pasts of different lengths even out.
int rows_of_tile(svgear_dtype dt) { return dt == SVGEAR_F32 ? 32 : kDenseRows; }
int parts_of(int64_t heads, int64_t own, int64_t other, int n_docs, svgear_dtype dt) {
  const int64_t tiles = heads * ceil_div(own, rows_of_tile(dt)), each = ceil_div(other, n_docs > 1 ? n_docs : 1), most = ceil_div(each, 128);
  const int64_t wanted = own <= kDenseRows ? std::max<int64_t>(512 / tiles, std::min<int64_t>(1024 / tiles, most / 2)) : 512 / tiles;
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(wanted, most), 64));
}

struct Sizes {
  svgear_dtype dt;
  int B, H, Hk;
  int64_t Nq, Nk;
  int d, n_docs;
};
bool sizes_ok(const Sizes& z) {
  if ((z.dt != SVGEAR_F32 && z.dt != SVGEAR_BF16) || z.B <= 0 || z.H <= 0 || z.Hk <= 0 || z.H % z.Hk || z.Nq <= 0 || z.Nk <= 0 ||
      (z.d != 64 && z.d != 128) || z.n_docs < 0 || z.n_docs > kMaxDocs || z.Nq > kMaxDenseRows || z.Nk > kMaxDenseRows ||
      z.B > kMaxDenseRows || z.H > kMaxDenseRows)
    return false;
  const int64_t heads = (int64_t)z.B * z.Hk;
  if ((int64_t)z.B * z.H > kMaxDenseRows || (z.H / z.Hk) * z.Nq > kMaxDenseRows) return false;
  const int64_t q = dense_slots((z.H / z.Hk) * z.Nq, z.n_docs, rows_of_tile(z.dt)), k = dense_slots(z.Nk, z.n_docs, rows_of_tile(z.dt));
  return heads * std::max(q, k) <= kMaxDenseRows && (__int128)z.B * z.H * z.Nq <= ((__int128)1 << 40) &&
         (__int128)heads * z.Nk <= ((__int128)1 << 40);
}
// Marks of a launch (whether or not it is a causal one): a wave of each tile and part.
size_t mark_bytes(const Sizes& z, int64_t heads, int64_t rows, int splits) {
  return z.Nq > 1 ? align_up((size_t)heads * dense_slots(rows, z.n_docs, rows_of_tile(z.dt)) * splits * kDenseWaves * sizeof(int32_t), 256) : 0;
}
size_t part_bytes(int splits, int64_t rows, int d, int tensors) {
  return splits > 1 ? align_up((size_t)splits * rows * d * sizeof(float) * tensors, 256) : 0;
}
int64_t q_rows(const Sizes& z) { return (int64_t)z.B * z.H * z.Nq; }
int64_t k_rows(const Sizes& z) { return (int64_t)z.B * z.Hk * z.Nk; }
int parts_over_keys(const Sizes& z) { return parts_of((int64_t)z.B * z.Hk, z.Nq * (z.H / z.Hk), z.Nk, z.n_docs, z.dt); }
int parts_over_queries(const Sizes& z) { return parts_of((int64_t)z.B * z.Hk, z.Nk, z.Nq * (z.H / z.Hk), z.n_docs, z.dt); }

// [B,H,N,d]: 16-byte aligned, strides multiples of 16 bytes (that of a dimension of one element does not matter).
bool tensor_ok(const void* p, const int64_t st[3], const Sizes& z, int64_t H, int64_t N) {
  if (!p || !st || reinterpret_cast<uintptr_t>(p) % 16) return false;
  const int64_t n[3] = {z.B, H, N};
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && (st[i] < 0 || st[i] > kMaxStride || (st[i] * (int64_t)esize(z.dt)) % 16)) return false;
  return true;
}
// An output's rows may not meet: the strides, the smallest first, each span what is within it.
bool output_ok(const void* p, const int64_t st[3], const Sizes& z, int64_t H, int64_t N) {
  if (!tensor_ok(p, st, z, H, N)) return false;
  std::pair<int64_t, int64_t> s[3] = {{st[0], z.B}, {st[1], H}, {st[2], N}};
  std::sort(s, s + 3);
  __int128 span = z.d;
  for (const auto& i : s) {
    if (i.second == 1) continue;
    if (i.first < span) return false;
    span += (__int128)(i.second - 1) * i.first;
  }
  return true;
}
Strides strides_of(const int64_t st[3], const Sizes& z, int64_t H, int64_t N) {
  return Strides{z.B > 1 ? st[0] : 0, H > 1 ? st[1] : 0, N > 1 ? st[2] : 0};
}

// Factors of the scores that fp32 has: those of the exponents, log2(e) scale, or log2(e) cap and scale / cap.
bool factors_ok(float scale, float cap) {
  if (!std::isfinite(scale) || !std::isfinite(cap) || cap < 0.f) return false;
  const float s = std::fabs(scale), log2e = 1.4426950408889634f;
  if (cap == 0.f) return std::isfinite(s * log2e);
  return std::isfinite(cap * log2e) && std::isfinite(s * log2e) && std::isfinite(s / cap) && (s == 0.f || s / cap >= FLT_MIN);
}

// The arguments that both passes share.
int fill(DenseArgs& a, const Sizes& z, const void* q, const int64_t qst[3], const void* k, const int64_t kst[3], const void* v,
         const int64_t vst[3], float scale, float cap, const float* slopes, unsigned flags, const int32_t* q_offsets,
         const int32_t* k_offsets, const int32_t* prefix) {
  if (!sizes_ok(z) || !tensor_ok(q, qst, z, z.H, z.Nq) || !tensor_ok(k, kst, z, z.Hk, z.Nk) || !tensor_ok(v, vst, z, z.Hk, z.Nk) ||
      !factors_ok(scale, cap) ||
      (flags & ~(SVGEAR_ATTENTION_CAUSAL | SVGEAR_ATTENTION_SHARED_DOCUMENTS)) ||
      (prefix && !(flags & SVGEAR_ATTENTION_CAUSAL)) || reinterpret_cast<uintptr_t>(slopes) % 4 ||
      reinterpret_cast<uintptr_t>(q_offsets) % 4 || reinterpret_cast<uintptr_t>(k_offsets) % 4 || reinterpret_cast<uintptr_t>(prefix) % 4)
    return SVGEAR_ERR_INVALID;
  // (a tile's keys are addressed by 32-bit byte offsets)
  if (z.Nk > 1 && (kst[2] > kMaxKeyStride || vst[2] > kMaxKeyStride)) return SVGEAR_ERR_INVALID;
  const bool some = q_offsets || k_offsets, both = q_offsets && k_offsets;
  if ((z.n_docs > 0) != some || (!both && z.n_docs > 1)) return SVGEAR_ERR_INVALID;
  a.q = q, a.k = k, a.v = v;
  a.qst = strides_of(qst, z, z.H, z.Nq);
  a.kst = strides_of(kst, z, z.Hk, z.Nk);
  a.vst = strides_of(vst, z, z.Hk, z.Nk);
  a.q_offsets = q_offsets, a.k_offsets = k_offsets, a.prefix = prefix, a.slopes = slopes;
  a.n_docs = std::max(z.n_docs, 1);
  a.docs_shared = flags & SVGEAR_ATTENTION_SHARED_DOCUMENTS;
  a.causal = (flags & SVGEAR_ATTENTION_CAUSAL) && z.Nq > 1;  // (a single query stands at the last key)
  a.scale = scale, a.cap = cap;
  a.B = z.B, a.H = z.H, a.Hk = z.Hk, a.G = z.H / z.Hk, a.Nq = (int)z.Nq, a.Nk = (int)z.Nk;
  a.by_hk = Divider(a.Hk), a.by_g = Divider(a.G);
  return SVGEAR_OK;
}
bool space_ok(const void* ws, size_t ws_bytes, size_t need) {
  return need == 0 || (ws && reinterpret_cast<uintptr_t>(ws) % 256 == 0 && ws_bytes >= need);
}
int launch(const DenseArgs& a, const Sizes& z, int what, hipStream_t s) {
  if (what == kDenseForward) return z.dt == SVGEAR_F32 ? launch_dense_f32(a, z.d, s) : launch_dense_bf16(a, z.d, s);
  return z.dt == SVGEAR_F32 ? launch_dense_backward_f32(a, z.d, what, s) : launch_dense_backward_bf16(a, z.d, what, s);
}

template <typename T, int D>
int merge(const DenseArgs& a, int64_t rows, hipStream_t s) {
  const Out o{a.o, a.ost, a.Nq, a.G, a.Hk};
  dense_merge_kernel<T, D><<<long_grid(ceil_div(rows * (D / 8), kThreads), 1), kThreads, 0, s>>>(a.part, a.part_ml, a.splits, rows, o, a.lse);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}
template <typename T, int D>
int sum(const DenseArgs& a, int64_t rows, float factor, const Out& first, const Out* second, hipStream_t s) {
  dense_sum_kernel<T, D><<<long_grid(ceil_div(rows * (D / 8), kThreads), second ? 2 : 1), kThreads, 0, s>>>(
      a.part, a.splits, rows, factor, first, second ? *second : first);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}
template <typename T, int D>
int find_delta(const DenseArgs& a, const void* o, const Strides& ost, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.H * a.Nq;
  dense_delta_kernel<T, D><<<long_grid(ceil_div(rows * (D / 8), kThreads), 1), kThreads, 0, s>>>(
      static_cast<const T*>(a.dy), a.yst, static_cast<const T*>(o), ost, a.H, a.Nq, rows, a.delta);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}
// f(type, head dimension) for a call's
template <typename F>
int by_kind(const Sizes& z, F f) {
  using std::integral_constant;
  if (z.dt == SVGEAR_F32) return z.d == 64 ? f(float{}, integral_constant<int, 64>{}) : f(float{}, integral_constant<int, 128>{});
  return z.d == 64 ? f(bf16_t{}, integral_constant<int, 64>{}) : f(bf16_t{}, integral_constant<int, 128>{});
}

}  // namespace
}  // namespace svgear

using namespace svgear;

extern "C" size_t svgear_attention_workspace(svgear_dtype dt, int B, int H, int Hk, int64_t Nq, int64_t Nk, int d, int n_docs) {
  const Sizes z{dt, B, H, Hk, Nq, Nk, d, n_docs};
  if (!sizes_ok(z)) return 0;
  const int splits = parts_over_keys(z);
  return mark_bytes(z, (int64_t)B * Hk, Nq * (H / Hk), splits) + part_bytes(splits, q_rows(z), d, 1) +
         (splits > 1 ? align_up((size_t)splits * q_rows(z) * sizeof(float2), 256) : 0);
}

extern "C" int svgear_attention(const void* q, const int64_t qstride[3], const void* k, const int64_t kstride[3], const void* v,
                                const int64_t vstride[3], svgear_dtype dt, int B, int H, int Hk, int64_t Nq, int64_t Nk, int d,
                                float scale, float cap, const float* slopes, unsigned flags, int n_docs,
                                const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* prefix, void* o,
                                const int64_t ostride[3], float* lse, void* ws, size_t ws_bytes, void* stream) {
  const Sizes z{dt, B, H, Hk, Nq, Nk, d, n_docs};
  DenseArgs a{};
  const int rc = fill(a, z, q, qstride, k, kstride, v, vstride, scale, cap, slopes, flags, q_offsets, k_offsets, prefix);
  if (rc != SVGEAR_OK) return rc;
  if (!output_ok(o, ostride, z, H, Nq) || reinterpret_cast<uintptr_t>(lse) % 4) return SVGEAR_ERR_INVALID;
  const void* ins[] = {q, k, v, slopes, q_offsets, k_offsets, prefix};
  for (const void* i : ins)
    if (o == i || (lse && lse == i)) return SVGEAR_ERR_INVALID;
  if (o == lse) return SVGEAR_ERR_INVALID;
  if (!space_ok(ws, ws_bytes, svgear_attention_workspace(dt, B, H, Hk, Nq, Nk, d, n_docs))) return SVGEAR_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  a.o = o;
  a.ost = strides_of(ostride, z, H, Nq);
  a.lse = lse;
  a.slots = (int)dense_slots(Nq * a.G, q_offsets ? n_docs : 0, rows_of_tile(dt));
  a.by_slots = Divider(a.slots);
  a.splits = parts_over_keys(z);
  a.by_splits = Divider(a.splits);
  Workspace w(ws, ws_bytes);
  if (a.causal) a.marks = w.take<int32_t>(mark_bytes(z, (int64_t)B * Hk, Nq * a.G, a.splits) / sizeof(int32_t));
  if (a.splits > 1) {
    a.part = w.take<float>((size_t)a.splits * q_rows(z) * d);
    a.part_ml = w.take<float2>((size_t)a.splits * q_rows(z));
  }
  int done = launch(a, z, kDenseForward, s);
  if (done == SVGEAR_OK && a.splits > 1)
    done = by_kind(z, [&](auto t, auto dim) { return merge<decltype(t), decltype(dim)::value>(a, q_rows(z), s); });
  return done == SVGEAR_OK && a.causal ? launch_dense_again(a, dt, d, kDenseForward, s) : done;
}

extern "C" size_t svgear_attention_backward_workspace(svgear_dtype dt, int B, int H, int Hk, int64_t Nq, int64_t Nk, int d, int n_docs) {
  const Sizes z{dt, B, H, Hk, Nq, Nk, d, n_docs};
  if (!sizes_ok(z)) return 0;
  return align_up((size_t)q_rows(z) * sizeof(float), 256) +
         std::max(mark_bytes(z, (int64_t)B * Hk, Nq * (H / Hk), parts_over_keys(z)) + part_bytes(parts_over_keys(z), q_rows(z), d, 1),
                  mark_bytes(z, (int64_t)B * Hk, Nk, parts_over_queries(z)) + part_bytes(parts_over_queries(z), k_rows(z), d, 2));
}

extern "C" int svgear_attention_backward(const void* dy, const int64_t dystride[3], const void* q, const int64_t qstride[3],
                                         const void* k, const int64_t kstride[3], const void* v, const int64_t vstride[3],
                                         const void* o, const int64_t ostride[3], const float* lse, svgear_dtype dt, int B,
                                         int H, int Hk, int64_t Nq, int64_t Nk, int d, float scale, float cap,
                                         const float* slopes, unsigned flags, int n_docs, const int32_t* q_offsets,
                                         const int32_t* k_offsets, const int32_t* prefix, void* dq, const int64_t dqstride[3],
                                         void* dk, const int64_t dkstride[3], void* dv, const int64_t dvstride[3], void* ws,
                                         size_t ws_bytes, void* stream) {
  const Sizes z{dt, B, H, Hk, Nq, Nk, d, n_docs};
  DenseArgs a{};
  const int rc = fill(a, z, q, qstride, k, kstride, v, vstride, scale, cap, slopes, flags, q_offsets, k_offsets, prefix);
  if (rc != SVGEAR_OK) return rc;
  if (!tensor_ok(dy, dystride, z, H, Nq) || !tensor_ok(o, ostride, z, H, Nq) || !lse || reinterpret_cast<uintptr_t>(lse) % 4 ||
      (!dq && !dk && !dv) || !dk != !dv || (dq && !output_ok(dq, dqstride, z, H, Nq)) || (dk && !output_ok(dk, dkstride, z, Hk, Nk)) ||
      (dv && !output_ok(dv, dvstride, z, Hk, Nk)))
    return SVGEAR_ERR_INVALID;
  const void* ins[] = {dy, q, k, v, o, lse, slopes, q_offsets, k_offsets, prefix};
  const void* outs[] = {dq, dk, dv};
  for (int i = 0; i < 3; ++i) {
    if (!outs[i]) continue;
    for (const void* in : ins)
      if (outs[i] == in) return SVGEAR_ERR_INVALID;
    for (int j = 0; j < i; ++j)
      if (outs[i] == outs[j]) return SVGEAR_ERR_INVALID;
  }
  if (!space_ok(ws, ws_bytes, svgear_attention_backward_workspace(dt, B, H, Hk, Nq, Nk, d, n_docs))) return SVGEAR_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Workspace w(ws, ws_bytes);
  a.dy = dy;
  a.yst = strides_of(dystride, z, H, Nq);
  a.lse_in = lse;
  a.delta = w.take<float>((size_t)q_rows(z));
  // marks and parts of either launch, one after the other in the same room
  auto room = [&](int64_t rows) {
    char* p = w.base + w.used;
    const size_t marks = a.causal ? mark_bytes(z, (int64_t)B * Hk, rows, a.splits) : 0;
    a.marks = a.causal ? reinterpret_cast<int32_t*>(p) : nullptr;
    a.part = reinterpret_cast<float*>(p + marks);
  };
  const Strides ost = strides_of(ostride, z, H, Nq);
  int done = by_kind(z, [&](auto t, auto dim) { return find_delta<decltype(t), decltype(dim)::value>(a, o, ost, s); });
  if (done != SVGEAR_OK) return done;
  if (dq) {
    a.o = dq;
    a.ost = strides_of(dqstride, z, H, Nq);
    a.slots = (int)dense_slots(Nq * a.G, q_offsets ? n_docs : 0, rows_of_tile(dt));
    a.by_slots = Divider(a.slots);
    a.splits = parts_over_keys(z);
    a.by_splits = Divider(a.splits);
    room(Nq * a.G);
    done = launch(a, z, kDenseDq, s);
    if (done != SVGEAR_OK) return done;
    if (a.splits > 1) {
      const Out out{dq, a.ost, a.Nq, a.G, Hk};
      done = by_kind(z, [&](auto t, auto dim) { return sum<decltype(t), decltype(dim)::value>(a, q_rows(z), scale, out, nullptr, s); });
      if (done != SVGEAR_OK) return done;
    }
    if (a.causal) done = launch_dense_again(a, dt, d, kDenseDq, s);
    if (done != SVGEAR_OK) return done;
  }
  if (!dk) return SVGEAR_OK;
  a.dk = dk, a.dv = dv;
  a.dkst = strides_of(dkstride, z, Hk, Nk);
  a.dvst = strides_of(dvstride, z, Hk, Nk);
  a.slots = (int)dense_slots(Nk, k_offsets ? n_docs : 0, rows_of_tile(dt));
  a.by_slots = Divider(a.slots);
  a.splits = parts_over_queries(z);
  a.by_splits = Divider(a.splits);
  room(Nk);
  done = launch(a, z, kDenseDkv, s);
  if (done == SVGEAR_OK && a.splits > 1) {
    const Out out_k{dk, a.dkst, a.Nk, 1, Hk}, out_v{dv, a.dvst, a.Nk, 1, Hk};
    done = by_kind(z, [&](auto t, auto dim) { return sum<decltype(t), decltype(dim)::value>(a, k_rows(z), 1.f, out_k, &out_v, s); });
  }
  return done == SVGEAR_OK && a.causal ? launch_dense_again(a, dt, d, kDenseDkv, s) : done;
}

// Dense attention with masks in bf16: the kernel of dense_tile.h with its phases laid over each other.
//
// What bounds it: the matrix cores and the vector unit alike. A step of a wave (64 keys, 32 queries, d = 128) is 32 products of 32
// cycles, and 32 exponentials a lane at a quarter of the rate with their scaling, maximum, sum and conversion, some 900 cycles.
// So a wave issues the exponentials of a tile between the products of the next tile's scores, and the next tile's maximum between
// the products with the values; two workgroups share a CU and fill what is left. A workgroup goes on to further tiles of
// queries of its head without a pause: the next queries are loaded when the last scores of the present ones are done, and the
// keys and values of the next step are on their way whatever tile it is of, since with few keys the start of a tile (lookups, first
// copies) takes as long as its steps.
#include "dense_tile.h"

namespace svgear {
namespace {

// log2 headroom before the running maximum is refreshed; none at d = 64, where the weight of a row's largest score is then exactly 1
template <int D>
constexpr float kHeadroom = D == 64 ? 0.f : 8.f;

// A tile of queries: its rows, its document, and its steps (tiles of keys) in this part of them.
struct QueryTile {
  Place at;
  int i;            // of the workgroup's run
  int t0, steps;    // first tile of keys, and how many
  int seen;         // keys of the document that its rows see
  int q0, nq, k0, nk, prefix;
};

template <int D, bool CAP, bool SLOPES>
__global__ void __launch_bounds__(64 * kDenseWaves, 2)
dense_forward_bf16_kernel(DenseArgs a) {
  using Z = Tile<bf16_t, D>;
  constexpr int DB = D / 32, KS = D / 16, BN = Z::kRows, ROWB = Z::kRowBytes, AHEAD = 4;
  __shared__ __attribute__((aligned(256))) unsigned char smem[4 * Z::kBytes];  // two of K, two of V
  int bh, run;
  if (!dense_index(a, bh, run)) return;
  if (a.causal) run = a.slots - 1 - run;  // the longest first
  const int b = bh / a.Hk, hk = bh - b * a.Hk;
  const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5, wave = uniform(tid >> 6);
  const int32_t* qo = a.q_offsets ? a.q_offsets + (a.docs_shared ? 0 : (int64_t)b * (a.n_docs + 1)) : nullptr;
  const int split = blockIdx.y;
  const int64_t part_rows = (int64_t)a.B * a.Hk * a.Nq * a.G;

  auto document = [&](const QueryTile& c) {
    Document d(a);
    d.q0 = c.q0, d.nq = c.nq, d.k0 = c.k0, d.nk = c.nk, d.prefix = c.prefix;
    return d;
  };
  // a row's output: what it has summed, or nothing
  auto store_row = [&](int row, const f32x16 (&acc)[DB], float m, float l) __attribute__((always_inline)) {
    if (a.splits > 1) {
      const int64_t out = split * part_rows + (int64_t)bh * a.Nq * a.G + row;
      if (lh == 0) a.part_ml[out] = make_float2(m, l);
      Z::each_four(acc, lh, [&](int d, float4 v) {
        __builtin_amdgcn_sched_barrier(0);  // (one after the other: together they take registers that the loop then misses)
        store_four(a.part + out * D + d, v);
      });
      return;
    }
    const int token = row / a.G, head = hk * a.G + (row - token * a.G);
    const float inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    bf16_t* o = static_cast<bf16_t*>(a.o) + b * a.ost.b + head * a.ost.h + token * a.ost.n;
    Z::each_four(acc, lh, [&](int d, float4 v) {
      __builtin_amdgcn_sched_barrier(0);
      store_four(o + d, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
    });
    if (a.lse && lh == 0) a.lse[((int64_t)b * a.H + head) * a.Nq + token] = (m + log2f(l)) * kLn2;
  };
  // The first tile from the run's i-th on that has steps; those that see no key (or none of this part) are written here. False: none.
  auto seek = [&](QueryTile& c) {
    for (; c.i < a.run; ++c.i) {
      if (c.at.first + kDenseRows < c.at.end) {  // the next tile of the same document
        c.at.first += kDenseRows;
      } else {
        const Place p = place_of(qo, a.n_docs, a.Nq, a.G, kDenseRows, run * a.run + c.i, lane);
        if (p.first >= p.end || p.first < c.at.end) continue;  // an empty slot
        c.at = p;
        const Document d(a, b, p.doc);
        c.q0 = d.q0, c.nq = d.nq, c.k0 = d.k0, c.nk = d.nk, c.prefix = d.prefix;
      }
      const int end = min(c.at.first + kDenseRows, c.at.end);
      c.seen = document(c).seen((end - 1) / a.G - c.q0);
      const int tiles = (c.seen + BN - 1) / BN;
      c.t0 = (int)((int64_t)tiles * split / a.splits);
      c.steps = (int)((int64_t)tiles * (split + 1) / a.splits) - c.t0;
      if (c.steps > 0) return true;
      f32x16 none[DB];
#pragma unroll
      for (int db = 0; db < DB; ++db) clear(none[db]);
      const int row = c.at.first + 32 * wave + li;
      if (row < end) store_row(row, none, -INFINITY, 0.f);
    }
    return false;
  };

  const Z z(lane);
  const uint32_t lds = lds_address(smem);
  const bf16_t* kb = static_cast<const bf16_t*>(a.k) + b * a.kst.b + hk * a.kst.h;
  const bf16_t* vb = static_cast<const bf16_t*>(a.v) + b * a.vst.b + hk * a.vst.h;
  auto issue = [&](const QueryTile& c, int t, const bf16_t* base, int64_t st, int buffer) __attribute__((always_inline)) {
    const int key = (c.t0 + t) * BN, last = c.seen - 1 - key;  // (keys that no row here sees are not read)
    copy_tile<Z>(base + ((int64_t)c.k0 + key) * st, lds + buffer * Z::kBytes, wave, lane, [&](int r) { return min(r, last) * st; });
  };
  auto row_of_lane = [&](const QueryTile& c) { return min(c.at.first + 32 * wave + li, c.at.end - 1); };

  typename Z::Column q;
  auto load_queries = [&](const QueryTile& c) __attribute__((always_inline)) {
    const int row = row_of_lane(c), token = row / a.G, head = hk * a.G + (row - token * a.G);
    q.load(static_cast<const bf16_t*>(a.q) + b * a.qst.b + head * a.qst.h + token * a.qst.n, lh);
    if (a.scale < 0.f) {  // (the maximum is that of the unscaled scores)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        union { bf16x8 v; uint4 u; } c2;
        c2.v = q.v[s];
        c2.u.x ^= 0x80008000u, c2.u.y ^= 0x80008000u, c2.u.z ^= 0x80008000u, c2.u.w ^= 0x80008000u;
        q.v[s] = c2.v;
      }
    }
  };
  // what this lane's query sees, and what all of the wave's do
  int pos = 0, hi = 0, hi_all = 0;
  float slope = 0.f;
  auto look_at_row = [&](const QueryTile& c) __attribute__((always_inline)) {
    const Document d = document(c);
    const int row = row_of_lane(c), token = row / a.G;
    pos = d.position(token - c.q0);
    hi = d.seen(token - c.q0);
    hi_all = d.seen(min(c.at.first + 32 * wave, c.at.end - 1) / a.G - c.q0);
    if (SLOPES) slope = a.slopes[hk * a.G + (row - token * a.G)] * kLog2e;
  };

  Scores<bf16_t, CAP, SLOPES> scores_of(a);
  scores_of.c = fabsf(scores_of.c);
  const float c0 = scores_of.c;
  f32x16 acc[DB], sA[2], sB[2];
#pragma unroll
  for (int db = 0; db < DB; ++db) clear(acc[db]);
#pragma unroll
  for (int k = 0; k < 2; ++k) clear(sA[k]), clear(sB[k]);
  float m = -INFINITY;
  uint32_t pk[2][8];
  float cc = c0;  // factor still to be applied to the scores whose maximum is known

  float ls[4] = {0.f, 0.f, 0.f, 0.f};
  auto weigh = [&](const f32x16 (&sc)[2], int e, float neg_m) __attribute__((always_inline)) {
    const int k = e >> 3, r = 2 * (e & 7);
    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[k][r], cc, neg_m));
    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[k][r + 1], cc, neg_m));
    pk[k][r >> 1] = pack2_bf16(p0, p1);
    ls[e & 3] += p0 + p1;
  };
  // Scores of the K tile in `buffer` into sn, and between those products, with EXPS, the weights of the scores sc into pk
  auto scores = [&](int buffer, f32x16 (&sn)[2], const f32x16 (&sc)[2], auto exps_tag) __attribute__((always_inline)) {
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
        for (int e = i * E; e < (i + 1) * E; ++e) weigh(sc, e, neg_m);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto max_pair = [&](const f32x16 (&sn)[2], float& mx, int e) __attribute__((always_inline)) {
    const int k = e >> 3, r = 2 * (e & 7);
    mx = fmaxf(fmaxf(mx, sn[k][r]), sn[k][r + 1]);
  };
  // The running maximum covers the scores sn of the keys' tile t afterwards; where there is more to them than a factor, they are exponents.
  auto settle = [&](int t, f32x16 (&sn)[2], float mx, auto whole_tag) __attribute__((always_inline)) {
    constexpr bool WHOLE = decltype(whole_tag)::value;  // seen by all rows of the wave, as the caller knows
    const bool masked = !WHOLE && (t + 1) * BN > hi_all;
    cc = c0;
    if (CAP || SLOPES || masked) {
      const int limit = masked ? hi - t * BN - 4 * lh : INT32_MAX;  // (constants on the other side of the comparisons)
      const float ahead = (float)(pos - t * BN - 4 * lh);
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
    const float ms = mx * cc;
    if (__any(ms > m + kHeadroom<D>)) {
      const float m_new = fmaxf(m, ms), alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
#pragma unroll
      for (int u = 0; u < 4; ++u) ls[u] *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[db][r] *= alpha;
      m = m_new;
    }
  };
  // O^T += V^T P^T with the V tile that v_off points into, and between those products, with MORE, the maximum of the next scores sn
  int v_off = 2 * Z::kBytes + z.tr_off;
  auto values = [&](const f32x16 (&sn)[2], auto more_tag) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more_tag)::value && !CAP && !SLOPES;
    constexpr int N = 4 * DB;
    bf16x8 vf[N];
    auto rd = [&](int i) {
      const unsigned char* at = smem + (i / DB) * 16 * ROWB;
      const int off = v_off ^ ((i % DB) << 6);
      union { struct { v4i16 a, b; } s; bf16x8 v; } u;
      u.s.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(at + off));
      u.s.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(at + 8 * ROWB + (off ^ 32)));
      vf[i] = u.v;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) rd(i);
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_barrier(0);
      if (i + AHEAD < N) rd(i + AHEAD);
      const int ks = i / DB, k = ks >> 1, u4 = (ks & 1) * 4;
      const bf16x8 bp = as_bf16x8(make_uint4(pk[k][u4], pk[k][u4 + 1], pk[k][u4 + 2], pk[k][u4 + 3]));
      acc[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[i], bp, acc[i % DB], 0, 0, 0);
      if (MORE && i >= N / 4) {
#pragma unroll
        for (int e = (i - N / 4) * 16 / (3 * N / 4); e < (i + 1 - N / 4) * 16 / (3 * N / 4); ++e) max_pair(sn, mx[e & 3], e);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
  };

  // Step t of a tile takes the weights of its scores and its values, and finds the scores of step t + 1; K(t + 2) and V(t + 1) are
  // copied meanwhile, over K(t) and V(t - 1), which step t - 1 was the last to read. In the last step both K buffers and one of V's are
  // free for the first steps of the next tile, whose queries are loaded.
  QueryTile now;
  now.at = Place{0, 0, -1};
  now.i = 0;
  now.q0 = now.nq = now.k0 = now.nk = now.prefix = 0;
  bool more = seek(now);
  auto start = [&](const QueryTile& c, int v_buffer) __attribute__((always_inline)) {
    issue(c, 0, kb, a.kst.n, 0);
    issue(c, 0, vb, a.vst.n, v_buffer);
    if (c.steps > 1) issue(c, 1, kb, a.kst.n, 1);
    load_queries(c);
  };
  int v_buffer = 2;  // that the present step's values are in
  if (more) {
    start(now, v_buffer);
    look_at_row(now);
  }
  while (more) {
    SVGEAR_WAIT_VMCNT(0);
    __syncthreads();
    scores(0, sA, sB, std::false_type{});
    {
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) max_pair(sA, mx, e);
      settle(now.t0, sA, mx, std::false_type{});
    }
    __syncthreads();  // everyone is done with the first K tile before it is copied over
    auto step = [&](int t, int parity, f32x16 (&s_now)[2], f32x16 (&s_next)[2], auto whole_tag) __attribute__((always_inline)) {
      if (t + 2 < now.steps) issue(now, t + 2, kb, a.kst.n, parity);
      issue(now, t + 1, vb, a.vst.n, v_buffer ^ 1);
      scores(parity ^ 1, s_next, s_now, std::true_type{});
      const float mx = values(s_next, std::true_type{});
      settle(now.t0 + t + 1, s_next, mx, whole_tag);
      v_buffer ^= 1;
      v_off ^= Z::kBytes;
      SVGEAR_WAIT_VMCNT(0);
      __syncthreads();
    };
    int t = 0;
    const int whole = min(now.steps, hi_all / BN - now.t0);  // steps without a mask for this wave
    for (; t + 2 < whole; t += 2) {
      step(t, 0, sA, sB, std::true_type{});
      step(t + 1, 1, sB, sA, std::true_type{});
    }
    for (; t + 2 < now.steps; t += 2) {
      step(t, 0, sA, sB, std::false_type{});
      step(t + 1, 1, sB, sA, std::false_type{});
    }
    if (t + 1 < now.steps) {
      step(t, 0, sA, sB, std::false_type{});
#pragma unroll
      for (int k = 0; k < 2; ++k) sA[k] = sB[k];
    }
    // the last step
    QueryTile next = now;
    ++next.i;
    more = seek(next);
    if (more) start(next, v_buffer ^ 1);
    {
      const float neg_m = m == -INFINITY ? 0.f : -m;
#pragma unroll
      for (int e = 0; e < 16; ++e) weigh(sA, e, neg_m);
    }
    __builtin_amdgcn_sched_barrier(0);
    values(sB, std::false_type{});
    __builtin_amdgcn_sched_barrier(0);
    float l = (ls[0] + ls[1]) + (ls[2] + ls[3]);
    l += swap32(l);
    const int row = now.at.first + 32 * wave + li;
    if (row < now.at.end) store_row(row, acc, m, l);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int db = 0; db < DB; ++db) clear(acc[db]);
#pragma unroll
    for (int u = 0; u < 4; ++u) ls[u] = 0.f;
    m = -INFINITY;
    v_buffer ^= 1;
    v_off ^= Z::kBytes;
    now = next;
    if (more) look_at_row(now);
  }
}

template <int D, bool CAP, bool SLOPES>
int launch_bf16_mode(const DenseArgs& a, hipStream_t s) {
  const int64_t groups = ceil_div((int64_t)a.B * a.Hk * a.slots, 8) * 8;
  dense_forward_bf16_kernel<D, CAP, SLOPES><<<long_grid(groups, a.splits), 64 * kDenseWaves, 0, s>>>(a);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}
template <int D>
int launch_bf16_width(const DenseArgs& a, hipStream_t s) {
  if (a.cap > 0.f) return a.slopes ? launch_bf16_mode<D, true, true>(a, s) : launch_bf16_mode<D, true, false>(a, s);
  return a.slopes ? launch_bf16_mode<D, false, true>(a, s) : launch_bf16_mode<D, false, false>(a, s);
}

}  // namespace

int launch_dense_bf16(const DenseArgs& a, int d, hipStream_t s) { return d == 64 ? launch_bf16_width<64>(a, s) : launch_bf16_width<128>(a, s); }
}  // namespace svgear

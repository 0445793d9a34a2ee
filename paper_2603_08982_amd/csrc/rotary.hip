// RMS norm of queries and keys and their rotation by the token's position on up to three axes, and the
// backward pass of both.
//
//   u = x f weight, f = rsqrt(mean(x^2) + eps);  pair p turned by position[axis(p)] * inv_freq[p]
//
// One pass over the data: a wave holds all heads of a token (or its share of them) in registers, 16 bytes a
// load, so the mean over a token's heads costs no second read; the angles of a token are found once, one pair
// a lane, and shared by its heads through LDS. Bound by memory: two tensors of 75,600 tokens of 40 heads of 128, bf16, norm over
// the token: 600 us, 5.2 TB/s, as a plain copy; a single token 7 us, the launch and three dependent loads.
#include "common.h"

#include <math.h>

namespace svgear {
namespace {

constexpr int kMaxHeads = 128;
constexpr int64_t kMaxTokens = 1 << 30;
constexpr int kRotWaves = 8;  // waves of a workgroup, at most; of the backward pass in bf16 up to 64 heads of 128:
constexpr int kRotBackWaves = 16;
// Workgroups of the backward pass, at most; each leaves a partial dweight. One on each CU, three tokens of 40 heads of 128 at a
// time (15 waves, all that its registers allow): two tensors of 75,600 tokens take 1,019 us (1,014 with a multiplication an element
// less, as the rest of these); two on each of one token (five waves: a third does not fit the four SIMDs) 1,052, and with 768 to
// 1,536 of these, a part of which waits, 1,271 to 1,396.
constexpr int kBackwardGroups = 256;

struct RotaryArgs {
  const void* src[2];     // x (forward), x of the norm (backward)
  const void* dy[2];      // backward only
  void* dst[2];
  const void* weight[2];
  Strides sst[2], yst[2], dst_st[2];
  const double* inv_freq;
  const int32_t* positions;
  int64_t pos_b;
  float* partial[2];  // backward: [workgroups][columns of weight], or null
  int tokens, N, n_rot, H, d;
  int sec0, sec01, pairs;
  int first, plane, width;  // grid: tokens of a time step, of a row
  int waves_per_token, its;
  int rows;  // backward: workgroups, rows of `partial`
  float eps, sign;
};

// V consecutive elements of T as they lie in memory: 16 bytes, or one element.
template <typename T, int V>
struct Chunk;
template <>
struct Chunk<bf16_t, 8> {
  uint4 r;
  __device__ __forceinline__ float get(int i) const {
    const uint32_t u = i < 2 ? r.x : i < 4 ? r.y : i < 6 ? r.z : r.w;
    return __uint_as_float((i & 1) ? (u & 0xffff0000u) : (u << 16));
  }
  static __device__ __forceinline__ Chunk of(const float* v) {
    return Chunk{make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]))};
  }
};
template <>
struct Chunk<float, 4> {
  float4 r;
  __device__ __forceinline__ float get(int i) const { return i == 0 ? r.x : i == 1 ? r.y : i == 2 ? r.z : r.w; }
  static __device__ __forceinline__ Chunk of(const float* v) { return Chunk{make_float4(v[0], v[1], v[2], v[3])}; }
};
template <>
struct Chunk<bf16_t, 1> {
  bf16_t r;
  __device__ __forceinline__ float get(int) const { return bf16_to_f32(r); }
  static __device__ __forceinline__ Chunk of(const float* v) { return Chunk{f32_to_bf16(v[0])}; }
};
template <>
struct Chunk<float, 1> {
  float r;
  __device__ __forceinline__ float get(int) const { return r; }
  static __device__ __forceinline__ Chunk of(const float* v) { return Chunk{v[0]}; }
};

// Heads a wave holds: `its` times 64 / (d / 2V); enough for 40 heads of 128 in 16-byte chunks.
template <typename T, int V>
constexpr int kMaxIts = V == 1 ? 16 : V == 4 ? 10 : 5;
// Backward: it holds two tensors, turned gradients and the sums of dweight, so a wave takes fewer heads and a token more
// waves: few of them up to 64 heads of 128, twice as many beyond.
template <typename T, int V>
constexpr int kFewIts = V == 1 ? 8 : V == 4 ? 2 : 1;
template <int V, int IT>
constexpr int kBackWaves = V == 8 && IT == 1 ? kRotBackWaves : kRotWaves;

enum { kNormNone = 0, kNormHead = 1, kNormToken = 2 };

// What a lane works on: V pairs of every head that falls to it, elements ea.. and eb.. of the head. Halves:
// pairs p0.. are elements p0.. and P + p0..; what lies beyond the rotated pairs is 2V consecutive elements.
// Interleaved: 2V consecutive elements.
template <int V, bool HALVES>
struct Lane {
  int sub, p0, ea, eb, per_wave;  // head within the wave's step; first pair; first elements; heads a step
  __device__ __forceinline__ Lane(int lane, int d, int pairs) {
    const int units = d / (2 * V);
    const int u = lane % units;
    sub = lane / units;
    per_wave = 64 / units;
    p0 = u * V;
    ea = HALVES && p0 < pairs ? p0 : 2 * p0;
    eb = HALVES ? (p0 < pairs ? p0 + pairs : 2 * p0 + V) : 2 * p0 + V;
  }
};

// cos and sin of the token's angles, one pair a lane, into the wave's LDS row; pairs that are not rotated get
// (1, 0). The angle in turns, fp64, less its nearest whole number: exact, so far positions keep their phase.
__device__ __forceinline__ void find_angles(const RotaryArgs& a, int b, int n, int lane, float2* row) {
  float2 cs = make_float2(1.f, 0.f);
  if (lane < a.pairs && n < a.n_rot) {
    const int axis = lane < a.sec0 ? 0 : lane < a.sec01 ? 1 : 2;
    int pos;
    if (a.positions) {
      pos = a.positions[(int64_t)b * a.pos_b + (int64_t)n * 3 + axis];
    } else {
      const int i = a.first + n, t = i / a.plane, rest = i - t * a.plane, h = rest / a.width;
      pos = axis == 0 ? t : axis == 1 ? h : rest - h * a.width;
    }
    const double turns = (double)pos * a.inv_freq[lane] * 0.15915494309189533577;
    const float f = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.f * f, &s, &c);
    cs = make_float2(c, a.sign * s);
  }
  if (2 * lane < a.d) row[lane] = cs;
}

// Turns the first `rotated` of the lane's pairs (with halves all or none; the others stay as they are, infinities
// too). xa, xb: the elements of the two chunks; interleaved: pairs lie within a chunk, the first V/2 of them in xa.
template <int V, bool HALVES>
__device__ __forceinline__ void turn(float (&xa)[V], float (&xb)[V], const float2 (&cs)[V], int rotated) {
  if (HALVES) {
    if (rotated <= 0) return;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float u = __builtin_fmaf(xa[i], cs[i].x, -xb[i] * cs[i].y), v = __builtin_fmaf(xa[i], cs[i].y, xb[i] * cs[i].x);
      xa[i] = u;
      xb[i] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float* x = i < V / 2 ? xa + 2 * i : xb + 2 * (i - V / 2);
      const float u = __builtin_fmaf(x[0], cs[i].x, -x[1] * cs[i].y), v = __builtin_fmaf(x[0], cs[i].y, x[1] * cs[i].x);
      if (i < rotated) x[0] = u, x[1] = v;
    }
  }
}

// Sum over the lanes that share a head (a head's mean) or over the wave and the other waves of the token.
template <int NORM>
__device__ __forceinline__ float sum_over(float v, int units, int wpt, int wave, int lane, float* slots) {
  const int upto = NORM == kNormHead ? units : 64;
  for (int o = 1; o < upto; o <<= 1) v += __shfl_xor(v, o);
  if (NORM == kNormToken && wpt > 1) {  // wpt is the workgroup's: every wave gets here as often
    __syncthreads();
    if (lane == 0) slots[wave] = v;
    __syncthreads();
    const int w0 = wave - wave % wpt;
    v = 0.f;
    for (int w = 0; w < wpt; ++w) v += slots[w0 + w];
  }
  return v;
}

// A workgroup's waves are tokens times waves_per_token; blockIdx.y is the tensor.
template <typename T, int V, int NORM, bool HALVES>
__global__ void __launch_bounds__(64 * kRotWaves)
rotary_kernel(RotaryArgs a) {
  constexpr int IT = kMaxIts<T, V>;
  __shared__ float2 rows[kRotWaves][64];
  __shared__ float slots[kRotWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wpt = a.waves_per_token, per_group = (blockDim.x >> 6) / wpt;
  const int token = (int)long_grid_index() * per_group + wave / wpt;
  const bool on = token < a.tokens;
  const int k = blockIdx.y;
  const int b = on ? token / a.N : 0, n = on ? token - b * a.N : 0;
  const Lane<V, HALVES> at(lane, a.d, a.pairs);
  const T* src = static_cast<const T*>(a.src[k]) + (int64_t)b * a.sst[k].b + (int64_t)n * a.sst[k].n;
  T* dst = static_cast<T*>(a.dst[k]) + (int64_t)b * a.dst_st[k].b + (int64_t)n * a.dst_st[k].n;
  const T* weight = static_cast<const T*>(a.weight[k]);
  const int h0 = (wave % wpt) * a.its * at.per_wave + at.sub;
  const int H = on ? a.H : 0;

  Chunk<T, V> xa[IT], xb[IT];
  float sum[IT];  // of squares: by head, or all in sum[0]
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int h = h0 + it * at.per_wave;
    if (it < a.its && h < H) {
      const T* p = src + (int64_t)h * a.sst[k].h;
      xa[it] = *reinterpret_cast<const Chunk<T, V>*>(p + at.ea);
      xb[it] = *reinterpret_cast<const Chunk<T, V>*>(p + at.eb);
    }
  }
  if (on) find_angles(a, b, n, lane, rows[wave]);
  __syncthreads();
  float2 cs[V];
#pragma unroll
  for (int i = 0; i < V; ++i) cs[i] = rows[wave][at.p0 + i];
  const int rotated = (n < a.n_rot ? a.pairs : 0) - at.p0;

  float all = 0.f;
  if (NORM != kNormNone) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      sum[it] = 0.f;
      if (it < a.its && h0 + it * at.per_wave < H) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          sum[it] = __builtin_fmaf(xa[it].get(i), xa[it].get(i), sum[it]);
          sum[it] = __builtin_fmaf(xb[it].get(i), xb[it].get(i), sum[it]);
        }
      }
      if (NORM == kNormToken) all += sum[it];
    }
    if (NORM == kNormToken) {
      all = sum_over<NORM>(all, 64, wpt, wave, lane, slots);
      all = 1.f / sqrtf(all / (float)(a.H * a.d) + a.eps);
    }
  }
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int h = h0 + it * at.per_wave;
    if (it >= a.its) break;
    float f = all;
    if (NORM == kNormHead) {
      f = sum_over<NORM>(sum[it], a.d / (2 * V), 1, wave, lane, nullptr);
      f = 1.f / sqrtf(f / (float)a.d + a.eps);
    }
    if (h >= H) continue;
    float va[V], vb[V];
#pragma unroll
    for (int i = 0; i < V; ++i) va[i] = xa[it].get(i), vb[i] = xb[it].get(i);
    if (NORM != kNormNone) {
#pragma unroll
      for (int i = 0; i < V; ++i) va[i] *= f, vb[i] *= f;
      if (weight) {
        const T* w = weight + (NORM == kNormToken ? h * a.d : 0);
        const Chunk<T, V> wa = *reinterpret_cast<const Chunk<T, V>*>(w + at.ea);
        const Chunk<T, V> wb = *reinterpret_cast<const Chunk<T, V>*>(w + at.eb);
#pragma unroll
        for (int i = 0; i < V; ++i) va[i] *= wa.get(i), vb[i] *= wb.get(i);
      }
    }
    turn<V, HALVES>(va, vb, cs, rotated);
    T* o = dst + (int64_t)h * a.dst_st[k].h;
    *reinterpret_cast<Chunk<T, V>*>(o + at.ea) = Chunk<T, V>::of(va);
    *reinterpret_cast<Chunk<T, V>*>(o + at.eb) = Chunk<T, V>::of(vb);
  }
}

// Backward with a norm. Every workgroup takes tokens at a distance and keeps its sums of du x f in registers
// until the end, then leaves them, its waves' tokens added in order, as one row of `partial`. A lane has some 17
// vector instructions an element, with the turned gradients kept for the second use; the first version, which
// turned them twice and packed by hand, had some 40 and was bound by them.
template <typename T, int V, int NORM, bool HALVES, int IT>
__global__ void __launch_bounds__((64 * kBackWaves<V, IT>))
rotary_backward_kernel(RotaryArgs a) {
  constexpr int AT = NORM == kNormToken ? IT : 1;  // a head's weight is shared by all heads
  constexpr int MW = kBackWaves<V, IT>;
  __shared__ float2 rows[2][MW][64];
  __shared__ float2 slots[2][MW];
  constexpr int Q = V == 1 ? 2 : 4;  // sums of a lane that go through LDS at a time
  __shared__ float acc_s[MW][64][Q];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wpt = a.waves_per_token, per_group = (blockDim.x >> 6) / wpt, first = wave - wave % wpt;
  const int k = blockIdx.y, units = a.d / (2 * V);
  const Lane<V, HALVES> at(lane, a.d, a.pairs);
  const T* weight = static_cast<const T*>(a.weight[k]);
  const int h0 = (wave % wpt) * a.its * at.per_wave + at.sub;
  float acc[AT][2 * V];
  Chunk<T, V> wa[AT], wb[AT];
#pragma unroll
  for (int it = 0; it < AT; ++it) {
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) acc[it][i] = 0.f;
    const int h = h0 + it * at.per_wave;
    float one[V];
#pragma unroll
    for (int i = 0; i < V; ++i) one[i] = 1.f;
    wa[it] = wb[it] = Chunk<T, V>::of(one);
    if (weight && it < a.its && (NORM == kNormHead || h < a.H)) {
      const T* w = weight + (NORM == kNormToken ? h * a.d : 0);
      wa[it] = *reinterpret_cast<const Chunk<T, V>*>(w + at.ea);
      wb[it] = *reinterpret_cast<const Chunk<T, V>*>(w + at.eb);
    }
  }

  // A token's rows are on their way and its angles found while the one before it is finished. LDS rows and slots of every
  // second token are others, so that the one barrier of a token orders both.
  struct Token {
    const T *x, *dy;
    T* dx;
    int b, n, H;
  };
  auto place = [&](int t0) __attribute__((always_inline)) {
    const int token = t0 + wave / wpt;
    Token t;
    const bool on = token < a.tokens;
    t.b = on ? token / a.N : 0;
    t.n = on ? token - t.b * a.N : 0;
    t.H = on ? a.H : 0;
    t.x = static_cast<const T*>(a.src[k]) + (int64_t)t.b * a.sst[k].b + (int64_t)t.n * a.sst[k].n;
    t.dy = static_cast<const T*>(a.dy[k]) + (int64_t)t.b * a.yst[k].b + (int64_t)t.n * a.yst[k].n;
    t.dx = static_cast<T*>(a.dst[k]) + (int64_t)t.b * a.dst_st[k].b + (int64_t)t.n * a.dst_st[k].n;
    return t;
  };
  Chunk<T, V> xa[IT], xb[IT], ya[IT], yb[IT], na[IT], nb[IT];  // x and dy of the token, x of the next
  auto load_dy = [&](const Token& t) __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int h = h0 + it * at.per_wave;
      if (it < a.its && h < t.H) {
        const T* q = t.dy + (int64_t)h * a.yst[k].h;
        ya[it] = *reinterpret_cast<const Chunk<T, V>*>(q + at.ea);
        yb[it] = *reinterpret_cast<const Chunk<T, V>*>(q + at.eb);
      }
    }
  };
  auto load_x = [&](const Token& t) __attribute__((always_inline)) {
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int h = h0 + it * at.per_wave;
      if (it < a.its && h < t.H) {
        const T* p = t.x + (int64_t)h * a.sst[k].h;
        na[it] = *reinterpret_cast<const Chunk<T, V>*>(p + at.ea);
        nb[it] = *reinterpret_cast<const Chunk<T, V>*>(p + at.eb);
      }
    }
  };
  const int stride = gridDim.x * per_group;
  int turn_of = 0;
  Token now = place(blockIdx.x * per_group);
  load_x(now);
  load_dy(now);
  if (now.H && wave == first) find_angles(a, now.b, now.n, lane, rows[0][first]);
  __syncthreads();
  for (int t0 = blockIdx.x * per_group; t0 < a.tokens; t0 += stride, turn_of ^= 1) {
    const int n = now.n, H = now.H;
    float2 cs[V];
#pragma unroll
    for (int i = 0; i < V; ++i) cs[i] = rows[turn_of][first][at.p0 + i];
#pragma unroll
    for (int it = 0; it < IT; ++it) xa[it] = na[it], xb[it] = nb[it];
    const int rotated = (n < a.n_rot ? a.pairs : 0) - at.p0;

    float ua[IT][V], ub[IT][V];  // du
    float xx[IT], gx[IT];        // sums of x^2 and g x, by head or all in [0]
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      xx[it] = gx[it] = 0.f;
      if (it < a.its && h0 + it * at.per_wave < H) {
        const int iw = NORM == kNormToken ? it : 0;
#pragma unroll
        for (int i = 0; i < V; ++i) ua[it][i] = ya[it].get(i), ub[it][i] = yb[it].get(i);
        turn<V, HALVES>(ua[it], ub[it], cs, rotated);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float x0 = xa[it].get(i), x1 = xb[it].get(i);
          xx[it] = __builtin_fmaf(x0, x0, xx[it]);
          xx[it] = __builtin_fmaf(x1, x1, xx[it]);
          gx[it] = __builtin_fmaf(ua[it][i] * x0, wa[iw].get(i), gx[it]);
          gx[it] = __builtin_fmaf(ub[it][i] * x1, wb[iw].get(i), gx[it]);
        }
      }
      if (NORM == kNormToken && it > 0) xx[0] += xx[it], gx[0] += gx[it];
    }
    T* const dst = now.dx;
    if (t0 + stride < a.tokens) {
      now = place(t0 + stride);
      load_x(now);
      load_dy(now);
      if (now.H && wave == first) find_angles(a, now.b, now.n, lane, rows[turn_of ^ 1][first]);
    }
    // f and mean(g x f): dx = f (g - x f mean(g x f)). Neither f^3 nor f^2, which leave fp32 from |x| of 1e13 on, nor their
    // products with a mean, which do for gradients that are small too.
    float f = 0.f, c = 0.f;
    if (NORM == kNormToken) {
      for (int o = 1; o < 64; o <<= 1) xx[0] += __shfl_xor(xx[0], o), gx[0] += __shfl_xor(gx[0], o);
      if (wpt > 1 && lane == 0) slots[turn_of][wave] = make_float2(xx[0], gx[0]);
    }
    __syncthreads();
    if (NORM == kNormToken) {
      if (wpt > 1) {
        xx[0] = gx[0] = 0.f;
        for (int w = 0; w < wpt; ++w) xx[0] += slots[turn_of][first + w].x, gx[0] += slots[turn_of][first + w].y;
      }
      const float inv = 1.f / (float)(a.H * a.d);
      f = 1.f / sqrtf(xx[0] * inv + a.eps);
      c = f * (gx[0] * inv);
    }
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int h = h0 + it * at.per_wave;
      if (it >= a.its) break;
      if (NORM == kNormHead) {
        for (int o = 1; o < units; o <<= 1) xx[it] += __shfl_xor(xx[it], o), gx[it] += __shfl_xor(gx[it], o);
        const float inv = 1.f / (float)a.d;
        f = 1.f / sqrtf(xx[it] * inv + a.eps);
        c = f * (gx[it] * inv);
      }
      if (h >= H) continue;
      const int ia = NORM == kNormToken ? it : 0;
      float ga[V], gb[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float x0 = f * xa[it].get(i), x1 = f * xb[it].get(i);
        acc[ia][i] = __builtin_fmaf(ua[it][i], x0, acc[ia][i]);
        acc[ia][V + i] = __builtin_fmaf(ub[it][i], x1, acc[ia][V + i]);
        ga[i] = f * __builtin_fmaf(-c, x0, ua[it][i] * wa[ia].get(i));
        gb[i] = f * __builtin_fmaf(-c, x1, ub[it][i] * wb[ia].get(i));
      }
      T* o = dst + (int64_t)h * a.dst_st[k].h;
      *reinterpret_cast<Chunk<T, V>*>(o + at.ea) = Chunk<T, V>::of(ga);
      *reinterpret_cast<Chunk<T, V>*>(o + at.eb) = Chunk<T, V>::of(gb);
    }
  }
  if (!a.partial[k]) return;

  float* out = a.partial[k] + (int64_t)blockIdx.x * (NORM == kNormToken ? a.H * a.d : a.d);
  if (NORM == kNormHead) {  // the heads of a wave, then the waves
#pragma unroll
    for (int i = 0; i < 2 * V; ++i)
      for (int o = units; o < 64; o <<= 1) acc[0][i] += __shfl_xor(acc[0][i], o);
  }
#pragma unroll
  for (int it = 0; it < AT; ++it) {
    if (it >= a.its) break;
    const int h = h0 + it * at.per_wave;
#pragma unroll
    for (int q = 0; q < 2 * V; q += Q) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < Q; ++i) acc_s[wave][lane][i] = acc[it][q + i];
      __syncthreads();
      const bool mine = NORM == kNormToken ? wave < wpt && h < a.H : wave == 0 && lane < units;
      if (!mine) continue;
#pragma unroll
      for (int i = 0; i < Q; ++i) {
        float v = 0.f;
        for (int w = NORM == kNormToken ? wave : 0; w < (int)(blockDim.x >> 6); w += NORM == kNormToken ? wpt : 1) v += acc_s[w][lane][i];
        out[(NORM == kNormToken ? h * a.d : 0) + (q + i < V ? at.ea + q + i : at.eb + q + i - V)] = v;
      }
    }
  }
}

// (the stride of a dimension of one element does not matter)
bool aligned_strides(const int64_t st[3], size_t es, const void* p, int64_t B, int64_t H, int64_t N) {
  if (reinterpret_cast<uintptr_t>(p) % 16) return false;
  const int64_t n[3] = {B, H, N};
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && (st[i] < 0 || st[i] > kMaxStride || (st[i] * (int64_t)es) % 16)) return false;
  return true;
}

// An output's rows may not meet: the strides, the smallest first, each span what is within it.
bool rows_apart(const int64_t st[3], int64_t B, int64_t H, int64_t N, int64_t d) {
  int64_t s[3] = {st[0], st[1], st[2]}, n[3] = {B, H, N};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (s[j] < s[i]) {
        const int64_t t = s[i], u = n[i];
        s[i] = s[j], n[i] = n[j], s[j] = t, n[j] = u;
      }
  __int128 span = d;
  for (int i = 0; i < 3; ++i) {
    if (n[i] == 1) continue;
    if (s[i] < span) return false;
    span += (__int128)(n[i] - 1) * s[i];
  }
  return true;
}

struct Shape {
  int B, H;
  int64_t N, n_tail;
  int d;
};

// Whether output k lies where an input or the other output does, other than the input it may replace (at its own strides; that
// of a dimension of one element does not matter).
bool meets(void* const* out, const int64_t (*ost)[3], const void* const* own, const int64_t (*own_st)[3], const void* const* other,
           int n, int k, const Shape& z) {
  for (int j = 0; j < n; ++j) {
    if (j != k && (out[k] == out[j] || out[k] == own[j])) return true;
    if (other && out[k] == other[j]) return true;
  }
  return out[k] == own[k] && ((z.B > 1 && ost[k][0] != own_st[k][0]) || (z.H > 1 && ost[k][1] != own_st[k][1]) ||
                              (z.N > 1 && ost[k][2] != own_st[k][2]));
}

int fill_args(RotaryArgs& a, int n_tensors, svgear_dtype dt, const Shape& z, const double* inv_freq,
              const int sections[3], const int64_t grid[3], int64_t first, const int32_t* positions,
              int64_t positions_stride_b, unsigned flags, float eps) {
  if (n_tensors < 1 || n_tensors > 2 || (dt != SVGEAR_F32 && dt != SVGEAR_BF16) || z.B <= 0 || z.H <= 0 ||
      z.H > kMaxHeads || z.N <= 0 || z.n_tail < 0 || z.n_tail >= z.N || z.N > kMaxTokens || (int64_t)z.B * z.N > kMaxTokens ||
      (z.d != 64 && z.d != 128) || !sections || (flags & ~7u) || ((flags & 3u) == 3u) || !(eps >= 0.f))
    return SVGEAR_ERR_INVALID;
  for (int i = 0; i < 3; ++i)
    if (sections[i] < 0 || sections[i] > z.d / 2) return SVGEAR_ERR_INVALID;
  a.sec0 = sections[0];
  a.sec01 = sections[0] + sections[1];
  a.pairs = a.sec01 + sections[2];
  if (a.pairs > z.d / 2 || (a.pairs > 0 && !inv_freq)) return SVGEAR_ERR_INVALID;
  const int64_t n_rot = z.N - z.n_tail;
  if (positions) {
    if (z.B > 1 && positions_stride_b != 0 && (positions_stride_b < 3 * n_rot || positions_stride_b > kMaxStride)) return SVGEAR_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(positions) % 4) return SVGEAR_ERR_INVALID;
    a.plane = a.width = 1;
  } else {
    if (!grid) return SVGEAR_ERR_INVALID;
    for (int i = 0; i < 3; ++i)
      if (grid[i] < 1 || grid[i] > INT32_MAX) return SVGEAR_ERR_INVALID;
    if (grid[1] * grid[2] > INT32_MAX || grid[0] * (grid[1] * grid[2]) > INT32_MAX || first < 0 ||
        first > INT32_MAX - n_rot || first + n_rot > grid[0] * grid[1] * grid[2])
      return SVGEAR_ERR_INVALID;
    a.plane = (int)(grid[1] * grid[2]);
    a.width = (int)grid[2];
    a.first = (int)first;
  }
  a.inv_freq = inv_freq;
  a.positions = positions;
  a.pos_b = positions_stride_b;
  a.tokens = (int)(z.B * z.N);
  a.N = (int)z.N;
  a.n_rot = (int)n_rot;
  a.H = z.H;
  a.d = z.d;
  a.eps = eps;
  return SVGEAR_OK;
}

// 16-byte chunks serve halves too where the pairs are whole chunks.
bool wide_pairs(svgear_dtype dt, int pairs, unsigned flags) {
  return !(flags & SVGEAR_ROTARY_HALVES) || pairs % (dt == SVGEAR_F32 ? 4 : 8) == 0;
}

// How a token's heads lie in waves; the threads of a workgroup, of `waves` waves if that is not fewer than a token's.
int plan_waves(RotaryArgs& a, int V, int max_its, int waves) {
  const int per_wave = 64 / (a.d / (2 * V));
  a.waves_per_token = (int)ceil_div(a.H, per_wave * max_its);
  a.its = (int)ceil_div(a.H, per_wave * a.waves_per_token);
  return 64 * a.waves_per_token * (a.waves_per_token >= waves ? 1 : waves / a.waves_per_token);
}

template <typename T, int V, int NORM, bool HALVES>
int launch_mode(RotaryArgs& a, int n_tensors, bool backward, hipStream_t s) {
  if constexpr (NORM != kNormNone) {
    if (backward) {
      constexpr int few = kFewIts<T, V>;
      const bool wide = a.H > kRotWaves * few * (64 / (a.d / (2 * V)));
      const int threads = plan_waves(a, V, wide ? 2 * few : few, wide ? kBackWaves<V, 2 * few> : kBackWaves<V, few>);
      a.rows = (int)ceil_div(a.tokens, threads / 64 / a.waves_per_token);
      if (a.rows > kBackwardGroups / n_tensors) a.rows = kBackwardGroups / n_tensors;
      const dim3 grid((unsigned)a.rows, (unsigned)n_tensors);
      if (wide)
        rotary_backward_kernel<T, V, NORM, HALVES, 2 * few><<<grid, threads, 0, s>>>(a);
      else
        rotary_backward_kernel<T, V, NORM, HALVES, few><<<grid, threads, 0, s>>>(a);
      SVGEAR_LAUNCH_CHECK();
      return SVGEAR_OK;
    }
  }
  const int threads = plan_waves(a, V, kMaxIts<T, V>, 4);
  const int64_t groups = ceil_div(a.tokens, threads / 64 / a.waves_per_token);
  rotary_kernel<T, V, NORM, HALVES><<<long_grid(groups, n_tensors), threads, 0, s>>>(a);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

template <typename T, int V, int NORM>
int launch_pairs(RotaryArgs& a, int n_tensors, unsigned flags, bool backward, hipStream_t s) {
  if (flags & SVGEAR_ROTARY_HALVES) return launch_mode<T, V, NORM, true>(a, n_tensors, backward, s);
  if constexpr (V == 1) return SVGEAR_ERR_INVALID;  // interleaved pairs always lie in whole chunks
  else return launch_mode<T, V, NORM, false>(a, n_tensors, backward, s);
}

template <typename T, int V>
int launch_width(RotaryArgs& a, int n_tensors, unsigned flags, bool backward, hipStream_t s) {
  if (flags & SVGEAR_ROTARY_NORM_HEAD) return launch_pairs<T, V, kNormHead>(a, n_tensors, flags, backward, s);
  if (flags & SVGEAR_ROTARY_NORM_TOKEN) return launch_pairs<T, V, kNormToken>(a, n_tensors, flags, backward, s);
  return launch_pairs<T, V, kNormNone>(a, n_tensors, flags, backward, s);
}

int launch_rotary(RotaryArgs& a, svgear_dtype dt, int n_tensors, unsigned flags, bool backward, hipStream_t s) {
  const bool wide = wide_pairs(dt, a.pairs, flags);
  if (dt == SVGEAR_F32)
    return wide ? launch_width<float, 4>(a, n_tensors, flags, backward, s) : launch_width<float, 1>(a, n_tensors, flags, backward, s);
  return wide ? launch_width<bf16_t, 8>(a, n_tensors, flags, backward, s) : launch_width<bf16_t, 1>(a, n_tensors, flags, backward, s);
}

// Rows that the backward pass leaves in `partial` for a tensor: no more than there are tokens.
int64_t partial_rows(int n_tensors, int B, int64_t N) {
  const int64_t tokens = (int64_t)B * N, most = kBackwardGroups / n_tensors;
  return tokens < most ? tokens : most;
}

}  // namespace
}  // namespace svgear

using namespace svgear;

extern "C" int svgear_rotary(int n_tensors, const void* const* src, const int64_t (*sstride)[3], void* const* dst,
                             const int64_t (*dstride)[3], const void* const* weight, svgear_dtype dt, int B, int H,
                             int64_t N, int64_t n_tail, int d, const double* inv_freq, const int sections[3],
                             const int64_t grid[3], int64_t first, const int32_t* positions,
                             int64_t positions_stride_b, unsigned flags, float eps, void* stream) {
  RotaryArgs a{};
  const Shape z{B, H, N, n_tail, d};
  const int rc = fill_args(a, n_tensors, dt, z, inv_freq, sections, grid, first, positions,
                           positions_stride_b, flags, eps);
  if (rc != SVGEAR_OK) return rc;
  if (!src || !sstride || !dst || !dstride) return SVGEAR_ERR_INVALID;
  for (int k = 0; k < n_tensors; ++k) {
    if (!src[k] || !dst[k] || !aligned_strides(sstride[k], esize(dt), src[k], B, H, N) ||
        !aligned_strides(dstride[k], esize(dt), dst[k], B, H, N) || !rows_apart(dstride[k], B, H, N, d))
      return SVGEAR_ERR_INVALID;
    a.src[k] = src[k];
    a.dst[k] = dst[k];
    a.weight[k] = weight ? weight[k] : nullptr;
    if (a.weight[k] && (!(flags & 3u) || reinterpret_cast<uintptr_t>(a.weight[k]) % 16)) return SVGEAR_ERR_INVALID;
    if (meets(dst, dstride, src, sstride, nullptr, n_tensors, k, z)) return SVGEAR_ERR_INVALID;
    a.sst[k] = Strides{sstride[k][0], sstride[k][1], sstride[k][2]};
    a.dst_st[k] = Strides{dstride[k][0], dstride[k][1], dstride[k][2]};
  }
  a.sign = 1.f;
  return launch_rotary(a, dt, n_tensors, flags, false, static_cast<hipStream_t>(stream));
}

extern "C" size_t svgear_rotary_backward_workspace(int n_tensors, int B, int H, int64_t N, int d) {
  if (n_tensors < 1 || n_tensors > 2 || B <= 0 || H <= 0 || H > kMaxHeads || N <= 0 || N > kMaxTokens ||
      (int64_t)B * N > kMaxTokens || (d != 64 && d != 128))
    return 0;
  return (size_t)n_tensors * align_up((size_t)partial_rows(n_tensors, B, N) * H * d * sizeof(float), 256);
}

extern "C" int svgear_rotary_backward(int n_tensors, const void* const* dy, const int64_t (*dystride)[3],
                                      const void* const* src, const int64_t (*sstride)[3], void* const* dx,
                                      const int64_t (*dxstride)[3], const void* const* weight, void* const* dweight,
                                      svgear_dtype dt, int B, int H, int64_t N, int64_t n_tail, int d,
                                      const double* inv_freq, const int sections[3], const int64_t grid[3],
                                      int64_t first, const int32_t* positions, int64_t positions_stride_b,
                                      unsigned flags, float eps, void* ws, size_t ws_bytes, void* stream) {
  RotaryArgs a{};
  const Shape z{B, H, N, n_tail, d};
  const int rc = fill_args(a, n_tensors, dt, z, inv_freq, sections, grid, first, positions,
                           positions_stride_b, flags, eps);
  if (rc != SVGEAR_OK) return rc;
  const bool norm = flags & 3u;
  if (!dy || !dystride || !dx || !dxstride || (norm && (!src || !sstride))) return SVGEAR_ERR_INVALID;
  bool any = false;
  for (int k = 0; k < n_tensors; ++k) {
    if (!dy[k] || !dx[k] || !aligned_strides(dystride[k], esize(dt), dy[k], B, H, N) ||
        !aligned_strides(dxstride[k], esize(dt), dx[k], B, H, N) || !rows_apart(dxstride[k], B, H, N, d))
      return SVGEAR_ERR_INVALID;
    a.weight[k] = weight ? weight[k] : nullptr;
    if (a.weight[k] && (!norm || reinterpret_cast<uintptr_t>(a.weight[k]) % 16)) return SVGEAR_ERR_INVALID;
    if (dweight && dweight[k]) {
      if (!norm || reinterpret_cast<uintptr_t>(dweight[k]) % esize(dt)) return SVGEAR_ERR_INVALID;
      any = true;
    }
    a.dy[k] = dy[k];
    a.yst[k] = Strides{dystride[k][0], dystride[k][1], dystride[k][2]};
    a.dst[k] = dx[k];
    a.dst_st[k] = Strides{dxstride[k][0], dxstride[k][1], dxstride[k][2]};
    if (norm) {
      if (!src[k] || !aligned_strides(sstride[k], esize(dt), src[k], B, H, N)) return SVGEAR_ERR_INVALID;
      if (meets(dx, dxstride, dy, dystride, src, n_tensors, k, z)) return SVGEAR_ERR_INVALID;
      a.src[k] = src[k];
      a.sst[k] = Strides{sstride[k][0], sstride[k][1], sstride[k][2]};
    } else {  // the forward kernel with the angles' signs turned
      if (meets(dx, dxstride, dy, dystride, nullptr, n_tensors, k, z)) return SVGEAR_ERR_INVALID;
      a.src[k] = dy[k];
      a.sst[k] = a.yst[k];
    }
  }
  for (int k = 0; any && k < n_tensors; ++k)
    for (int j = 0; j < n_tensors; ++j)
      if (dweight[k] && (dweight[k] == dx[j] || (j != k && dweight[k] == dweight[j]))) return SVGEAR_ERR_INVALID;
  a.sign = -1.f;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Workspace w(ws, ws_bytes);
  if (any) {
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < svgear_rotary_backward_workspace(n_tensors, B, H, N, d))
      return SVGEAR_ERR_WORKSPACE;
    for (int k = 0; k < n_tensors; ++k) a.partial[k] = dweight[k] ? w.take<float>((size_t)partial_rows(n_tensors, B, N) * H * d) : nullptr;
  }
  const int done = launch_rotary(a, dt, n_tensors, flags, true, s);
  if (done != SVGEAR_OK || !any) return done;
  const int cols = (flags & SVGEAR_ROTARY_NORM_TOKEN) ? H * d : d;
  if (n_tensors == 2 && a.partial[0] && a.partial[1])
    return sum_rows(a.partial[0], dweight[0], a.partial[1], dweight[1], a.rows, cols, 1, dt, s);
  const int k = a.partial[0] ? 0 : 1;
  return sum_rows(a.partial[k], dweight[k], nullptr, nullptr, a.rows, cols, 1, dt, s);
}

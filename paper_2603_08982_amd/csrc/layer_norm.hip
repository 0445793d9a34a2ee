// svgear_layer_norm and svgear_layer_norm_backward: mean, variance, modulation and their gradients in one pass over the rows.
//
//   h = (x - mean) rstd,  u = h w + b,  y = u (1 + scale) + shift
//   du = dy (1 + scale),  g = du w,  dx = rstd (g - mean(g) - h mean(g h))
//   columns: S1 = sum dy, S2 = sum dy h over the rows of a batch entry; dshift = S1, dscale = w S2 + b S1,
//   dbias = sum over entries of (1 + scale) S1, dweight = of (1 + scale) S2
//
// What bounds it: memory. x is read and y written once; the gradients read x and dy and write dx once.
// A row is dealt to a team: L lanes of a wave for short rows (64 / L rows a wave at a time), else `wpr` whole waves with CH
// runs of eight columns a lane. A team stays with its columns and walks over rows, so that weights, modulation and, in the
// backward pass, the sums of its columns stay in registers; the next row is on its way while the present one is reduced.
// A row's statistics take one exchange between its waves: each finds its own mean and the squares' sum around that (so that a
// mean far from zero costs nothing), and those of the waves are joined around the row's mean.
// Registers hold all that up to 16,384 columns in the forward pass and, with a modulation of entries, up to 8,192 in fp32's and whole chunks of
// 16,384 in bf16's backward pass. Wider rows spill 96 registers and more, and a token's modulation in the backward pass does from 1,025
// columns in bf16 and 8,193 in fp32: 9,450 x 5,120 in bf16, gradients with a modulation of entries 79 us, of tokens 487 for a copy's 115; 3,000
// rows of 16,384 in bf16 forward 37 us, backward 80, of 16,392 columns 128 and 590.
#include <algorithm>
#include <type_traits>

#include "linear.h"

namespace svgear {
namespace {

constexpr int kMaxNormWidth = 1 << 15;
constexpr int64_t kMaxNormRows = 1 << 30;
constexpr int kNormWaves = 4;  // waves of a workgroup whose teams are a wave or less
constexpr int kEntriesOfOne = 4;  // entries whose sums one workgroup joins: a second launch costs as much

enum { kModNone = SVGEAR_NORM_PLAIN, kModEntry = SVGEAR_NORM_BATCH, kModToken = SVGEAR_NORM_TOKEN };

struct NormArgs {
  const void* x;
  const void* dy;
  const void* weight;
  const void* bias;
  const void* scale;
  const void* shift;
  void* y;  // dx in the backward pass
  void* dscale;
  void* dshift;  // of tokens, dense
  float* partial;  // [entries][parts][2][c]
  Rows xst, dyst, yst, sst, hst;
  int64_t R;    // rows of an entry (a batch entry where each has its own modulation, else all)
  int64_t n;    // tokens of a batch entry
  int entries, c, wpr, groups, parts;  // groups: workgroups of an entry
  float eps;
};

// ---- sums over L lanes
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float v) {
  const int moved = __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false);
  return v + __int_as_float(moved);
}
template <int L>
__device__ __forceinline__ float team_sum(float v) {
  if constexpr (L == 64) {  // rows of 16 lanes, then their last lanes on to the next rows: six vector adds, no LDS
    v = dpp_add<0x111, 0xf>(v);
    v = dpp_add<0x112, 0xf>(v);
    v = dpp_add<0x114, 0xf>(v);
    v = dpp_add<0x118, 0xf>(v);
    v = dpp_add<0x142, 0xa>(v);
    v = dpp_add<0x143, 0xc>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
  } else {
#pragma unroll
    for (int o = 1; o < L; o <<= 1) v += __shfl_xor(v, o);
    return v;
  }
}

// ---- eight columns of which `n` are within the row; WHOLE: all of them or none (a comparison for each element otherwise)
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_some(Eight<T>& v, const T* p, int n) {
  if (n >= 8) {
    v.load(p);
  } else if constexpr (WHOLE) {
    __builtin_memset(&v, 0, sizeof(v));
  } else {
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = i < n ? p[i] : T(0);
    __builtin_memcpy(&v, t, sizeof(t));
  }
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void store_some(T* p, const float (&v)[8], int n) {
  if (n >= 8) {
    store8(p, v);
  } else if constexpr (!WHOLE) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) store1(p + i, v[i]);
  }
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_floats(float (&f)[8], const void* p, int64_t at, int n) {
  Eight<T> v;
  load_some<WHOLE>(v, static_cast<const T*>(p) + at, n);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = v.get(i);
}

// Where a lane's columns and a team's rows are.
template <int L, int CH>
struct Team {
  int col[CH], n[CH];  // first of eight columns, and how many of them are in the row
  float inv_here;      // 1 / columns of this wave's share (a lane team: of the row)
  float here;
  int wave, lane, entry;
  int64_t first, step;  // rows first + team, then on by step

  __device__ __forceinline__ Team(const NormArgs& a) {
    const int tid = threadIdx.x;
    lane = tid & 63;
    wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool waves = L == 64 && a.wpr > 1;
    const unsigned wg = long_grid_index();
    entry = (int)(wg / (unsigned)a.groups);
    const int g = (int)(wg - (unsigned)entry * (unsigned)a.groups);
    first = waves ? g : ((int64_t)g * kNormWaves + wave) * (64 / L);
    step = waves ? a.groups : (int64_t)a.groups * kNormWaves * (64 / L);
    int mine = 0;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int row = waves ? k * a.wpr + wave : k;
      col[k] = 8 * (row * L + lane % L);
      n[k] = min(max(a.c - col[k], 0), 8);
      mine += min(max(a.c - 8 * row * L, 0), 8 * L);
    }
    here = (float)mine;
    inv_here = mine > 0 ? 1.f / (float)mine : 0.f;
  }
};

// Row r of an entry as (batch entry, token).
struct Where {
  int64_t b, t;
  __device__ __forceinline__ Where(const NormArgs& a, int entry, int64_t r) {
    if (a.entries > 1) {
      b = entry;
      t = r;
    } else if (r < a.n) {
      b = 0;
      t = r;
    } else {
      b = (uint32_t)r / (uint32_t)a.n;
      t = r - b * a.n;
    }
  }
  __device__ __forceinline__ int64_t at(const Rows& st) const { return b * st.b + t * st.n; }
};

// Mean and the sum of squares around it of this wave's share of a row (a lane team: of the row).
template <bool WHOLE, typename T, int L, int CH>
__device__ __forceinline__ void share_statistics(const Team<L, CH>& at, const Eight<T> (&x)[CH], float& mean, float& m2) {
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < CH; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[k].get(i);  // (zeros behind the row's end)
  mean = team_sum<L>(s) * at.inv_here;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < CH; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float d = i < (WHOLE ? at.n[k] & 8 : at.n[k]) ? x[k].get(i) - mean : 0.f;
      s = __builtin_fmaf(d, d, s);
    }
  m2 = team_sum<L>(s);
}

template <typename T, int L, int CH, int MOD, int MAXW, bool WHOLE>
__global__ void __launch_bounds__(64 * MAXW)
layer_norm_kernel(NormArgs a) {
  __shared__ float4 slots[2][MAXW];
  const Team<L, CH> at(a);
  if (at.entry >= a.entries) return;
  const bool waves = L == 64 && a.wpr > 1;
  const int team = L == 64 ? 0 : at.lane / L;
  const float inv_c = 1.f / (float)a.c;

  // y = h f + o
  float f[CH][8], o[CH][8];
#pragma unroll
  for (int k = 0; k < CH; ++k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[k][i] = 1.f, o[k][i] = 0.f;
    if (a.weight) load_floats<WHOLE, T>(f[k], a.weight, at.col[k], at.n[k]);
    if (a.bias) load_floats<WHOLE, T>(o[k], a.bias, at.col[k], at.n[k]);
    if (MOD == kModEntry) {
      if (a.scale) {
        float s[8];
        load_floats<WHOLE, T>(s, a.scale, at.entry * a.sst.b + at.col[k], at.n[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[k][i] *= 1.f + s[i], o[k][i] *= 1.f + s[i];
      }
      if (a.shift) {
        float s[8];
        load_floats<WHOLE, T>(s, a.shift, at.entry * a.hst.b + at.col[k], at.n[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[k][i] += s[i];
      }
    }
  }

  Eight<T> next[CH], sc[CH], sh[CH];
  auto load = [&](int64_t base) {
    const int64_t r = base + team;
    if (r >= a.R) return;
    const Where w(a, at.entry, r);
    const T* p = static_cast<const T*>(a.x) + w.at(a.xst);
#pragma unroll
    for (int k = 0; k < CH; ++k) load_some<WHOLE>(next[k], p + at.col[k], at.n[k]);
  };
  load(at.first);
  int turn = 0;
  for (int64_t base = at.first; base < a.R; base += at.step, turn ^= 1) {
    Eight<T> x[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) x[k] = next[k];
    const int64_t r = base + team;
    const bool valid = r < a.R;
    const Where w(a, at.entry, valid ? r : a.R - 1);
    if (MOD == kModToken && valid) {
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        if (a.scale) load_some<WHOLE>(sc[k], static_cast<const T*>(a.scale) + w.at(a.sst) + at.col[k], at.n[k]);
        if (a.shift) load_some<WHOLE>(sh[k], static_cast<const T*>(a.shift) + w.at(a.hst) + at.col[k], at.n[k]);
      }
    }
    if (base + at.step < a.R) load(base + at.step);
    float mean, m2;
    share_statistics<WHOLE, T, L, CH>(at, x, mean, m2);
    if (waves) {
      if (at.lane == 0) slots[turn][at.wave] = make_float4(mean, m2, at.here, 0.f);
      __syncthreads();
      float s = 0.f, q = 0.f;
      for (int v = 0; v < a.wpr; ++v) s = __builtin_fmaf(slots[turn][v].x, slots[turn][v].z, s);
      mean = s * inv_c;
      for (int v = 0; v < a.wpr; ++v) {
        const float4 p = slots[turn][v];
        q += __builtin_fmaf(p.z * (p.x - mean), p.x - mean, p.y);
      }
      m2 = q;
    }
    const float rstd = 1.f / sqrtf(m2 * inv_c + a.eps);
    if (!valid) continue;
    T* y = static_cast<T*>(a.y) + w.at(a.yst);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[i] = __builtin_fmaf((x[k].get(i) - mean) * rstd, f[k][i], o[k][i]);
        if (MOD == kModToken) {
          if (a.scale) v[i] *= 1.f + sc[k].get(i);
          if (a.shift) v[i] += sh[k].get(i);
        }
      }
      if (at.n[k] > 0) store_some<WHOLE>(y + at.col[k], v, at.n[k]);
    }
  }
}

template <typename T, int L, int CH, int MOD, int MAXW, bool WHOLE>
__global__ void __launch_bounds__(64 * MAXW)
layer_norm_backward_kernel(NormArgs a) {
  __shared__ float4 slots[2][MAXW];
  const Team<L, CH> at(a);
  if (at.entry >= a.entries) return;
  const bool waves = L == 64 && a.wpr > 1;
  const int team = L == 64 ? 0 : at.lane / L;
  const float inv_c = 1.f / (float)a.c;

  // g = dy f; u = h f + o for the gradient of a token's scale
  float f[CH][8], o[MOD == kModToken ? CH : 1][8], s1[CH][8], s2[CH][8];
#pragma unroll
  for (int k = 0; k < CH; ++k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[k][i] = 1.f, s1[k][i] = s2[k][i] = 0.f;
    if (a.weight) load_floats<WHOLE, T>(f[k], a.weight, at.col[k], at.n[k]);
    if (MOD == kModToken) {
#pragma unroll
      for (int i = 0; i < 8; ++i) o[k][i] = 0.f;
      if (a.bias) load_floats<WHOLE, T>(o[k], a.bias, at.col[k], at.n[k]);
    }
    if (MOD == kModEntry && a.scale) {
      float s[8];
      load_floats<WHOLE, T>(s, a.scale, at.entry * a.sst.b + at.col[k], at.n[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[k][i] *= 1.f + s[i];
    }
  }

  Eight<T> nx[CH], ny[CH];
  auto load = [&](int64_t base) {
    const int64_t r = base + team;
    if (r >= a.R) return;
    const Where w(a, at.entry, r);
    const T* px = static_cast<const T*>(a.x) + w.at(a.xst);
    const T* py = static_cast<const T*>(a.dy) + w.at(a.dyst);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      load_some<WHOLE>(nx[k], px + at.col[k], at.n[k]);
      load_some<WHOLE>(ny[k], py + at.col[k], at.n[k]);
    }
  };
  load(at.first);
  int turn = 0;
  for (int64_t base = at.first; base < a.R; base += at.step, turn ^= 1) {
    Eight<T> x[CH], dy[CH], sc[MOD == kModToken ? CH : 1];
#pragma unroll
    for (int k = 0; k < CH; ++k) x[k] = nx[k], dy[k] = ny[k];
    const int64_t r = base + team;
    const bool valid = r < a.R;
    const Where w(a, at.entry, valid ? r : a.R - 1);
    if (MOD == kModToken && valid && a.scale) {
#pragma unroll
      for (int k = 0; k < CH; ++k) load_some<WHOLE>(sc[k], static_cast<const T*>(a.scale) + w.at(a.sst) + at.col[k], at.n[k]);
    }
    if (base + at.step < a.R) load(base + at.step);
    auto du_of = [&](int k, int i) __attribute__((always_inline)) {
      const float v = dy[k].get(i);
      return MOD == kModToken && a.scale ? v * (1.f + sc[k].get(i)) : v;
    };
    float mean, m2;
    share_statistics<WHOLE, T, L, CH>(at, x, mean, m2);
    float ga = 0.f, gx = 0.f;  // sums of g and of g (x - mean)
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (WHOLE || i < at.n[k]) {  // (dy is 0 behind the row's end)
          const float g = du_of(k, i) * f[k][i];
          ga += g;
          gx = __builtin_fmaf(g, x[k].get(i) - mean, gx);
        }
    ga = team_sum<L>(ga);
    gx = team_sum<L>(gx);
    if (waves) {
      if (at.lane == 0) {
        slots[turn][at.wave] = make_float4(mean, m2, ga, gx);
      }
      __syncthreads();
      // (a wave's columns are eight runs of the lanes from its own on, as in Team)
      float s = 0.f;
      auto share = [&](int v) {
        int mine = 0;
#pragma unroll
        for (int k = 0; k < CH; ++k) mine += min(max(a.c - 8 * (k * a.wpr + v) * 64, 0), 512);
        return (float)mine;
      };
      for (int v = 0; v < a.wpr; ++v) s = __builtin_fmaf(slots[turn][v].x, share(v), s);
      mean = s * inv_c;
      m2 = ga = gx = 0.f;
      for (int v = 0; v < a.wpr; ++v) {
        const float4 p = slots[turn][v];
        const float d = p.x - mean;
        m2 += __builtin_fmaf(share(v) * d, d, p.y);
        ga += p.z;
        gx += __builtin_fmaf(d, p.z, p.w);
      }
    }
    const float rstd = 1.f / sqrtf(m2 * inv_c + a.eps);
    if (!valid) continue;
    const float mg = ga * inv_c, mgh = gx * rstd * inv_c;  // means of g and g h
    T* dx = a.y ? static_cast<T*>(a.y) + w.at(a.yst) : nullptr;
    const int64_t dense = (w.b * a.n + w.t) * a.c;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      float v[8], ds[8], db[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float h = (x[k].get(i) - mean) * rstd, du = du_of(k, i);
        s1[k][i] += du;
        s2[k][i] = __builtin_fmaf(du, h, s2[k][i]);
        v[i] = rstd * (__builtin_fmaf(du, f[k][i], -mg) - h * mgh);
        if (MOD == kModToken) {
          db[i] = dy[k].get(i);
          ds[i] = db[i] * __builtin_fmaf(h, f[k][i], o[k][i]);
        }
      }
      if (at.n[k] > 0) {
        if (dx) store_some<WHOLE>(dx + at.col[k], v, at.n[k]);
        if (MOD == kModToken && a.dscale) store_some<WHOLE>(static_cast<T*>(a.dscale) + dense + at.col[k], ds, at.n[k]);
        if (MOD == kModToken && a.dshift) store_some<WHOLE>(static_cast<T*>(a.dshift) + dense + at.col[k], db, at.n[k]);
      }
    }
  }
  if (!a.partial) return;

  // one row of sums for each wave of the workgroup, or for all its waves together where they share rows
  const int g = (int)(long_grid_index() - (unsigned)at.entry * (unsigned)a.groups);
  const int64_t part = (int64_t)at.entry * a.parts + (waves ? g : g * kNormWaves + at.wave);
  float* out = a.partial + part * 2 * a.c;
#pragma unroll
  for (int k = 0; k < CH; ++k) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int q = L; q < 64; q <<= 1) s1[k][i] += __shfl_xor(s1[k][i], q), s2[k][i] += __shfl_xor(s2[k][i], q);
    }
    if (at.n[k] > 0 && (L == 64 || at.lane < L)) {
      store_some<WHOLE>(out + at.col[k], s1[k], at.n[k]);
      store_some<WHOLE>(out + a.c + at.col[k], s2[k], at.n[k]);
    }
  }
}

// ---- the columns' sums, joined: 16 columns a workgroup, 64 runs of parts, each every 64th, then those in order
// An entry takes a workgroup some 1.6 us, whatever its parts are, so the entries are dealt out to workgroups too. Each then leaves its
// sums for dweight and dbias where its first entry's part 0 was, which nobody else reads, and a second launch joins those (16,384 entries of
// two tokens of 24, the whole call: one workgroup for all entries 26 ms, dealt out 0.2).
struct NormSums {
  float* partial;
  int64_t joined_pitch;  // elements from a part to the next, of the second launch
  const void* weight;
  const void* bias;
  const void* scale;  // of entries
  int64_t scale_b;
  void* dweight;
  void* dbias;
  void* dscale;
  void* dshift;
  int entries, parts, c, dealt;
};
template <typename T, bool JOINED>  // (a pitch that the compiler does not see made of c: 7.1 us for 5.0 at 2 x 777 rows of 1,541)
__global__ void __launch_bounds__(1024)
layer_norm_sums_kernel(NormSums a) {
  __shared__ float s[2][64][17];
  const int x = threadIdx.x & 15, y = threadIdx.x >> 4, c = blockIdx.x * 16 + x;
  const bool in = c < a.c;
  float w = 1.f, b = 0.f, t1 = 0.f, t2 = 0.f;
  if (y == 0 && in) {
    if (a.weight) w = load_as_f32(static_cast<const T*>(a.weight) + c);
    if (a.bias) b = load_as_f32(static_cast<const T*>(a.bias) + c);
  }
  for (int e = blockIdx.y; e < a.entries; e += a.dealt) {
    const float* p = a.partial + (int64_t)e * a.parts * 2 * a.c + c;
    float v1 = 0.f, v2 = 0.f;
    if (in)
#pragma unroll 8
      for (int i = y; i < a.parts; i += 64) {
        const int64_t at = JOINED ? i * a.joined_pitch : (int64_t)i * 2 * a.c;
        v1 += p[at], v2 += p[at + a.c];
      }
    s[0][y][x] = v1;
    s[1][y][x] = v2;
    __syncthreads();
    if (y == 0 && in) {
#pragma unroll 16
      for (int k = 1; k < 64; ++k) v1 += s[0][k][x], v2 += s[1][k][x];
      const float f = a.scale ? 1.f + load_as_f32(static_cast<const T*>(a.scale) + e * a.scale_b + c) : 1.f;
      t1 = __builtin_fmaf(f, v1, t1);
      t2 = __builtin_fmaf(f, v2, t2);
      if (a.dshift) store1(static_cast<T*>(a.dshift) + (int64_t)e * a.c + c, v1);
      if (a.dscale) store1(static_cast<T*>(a.dscale) + (int64_t)e * a.c + c, __builtin_fmaf(w, v2, b * v1));
    }
    __syncthreads();
  }
  if (y == 0 && in && a.dealt == 1) {
    if (a.dbias) store1(static_cast<T*>(a.dbias) + c, t1);
    if (a.dweight) store1(static_cast<T*>(a.dweight) + c, t2);
  } else if (y == 0 && in && (a.dbias || a.dweight)) {
    float* p = a.partial + (int64_t)blockIdx.y * a.parts * 2 * a.c + c;
    p[0] = t1;
    p[a.c] = t2;
  }
}

// ---- host side
// Lanes or waves of a team, runs of eight columns a lane.
struct Shape {
  int lanes, wpr, ch;
};
Shape shape_of(int c, svgear_dtype dt) {
  const int runs = (int)ceil_div(c, 8);
  for (int l = 8; l < 64; l *= 2)
    if (runs <= l) return {l, 1, 1};
  // up to 64 bytes a lane (75,600 x 5,120 in bf16: 300 us; with half of it and as much on its way 314, with a quarter 350), fp32
  // rows of over 16 waves 128
  int ch = 1;
  while (runs > 64 * ch && ch < (dt == SVGEAR_F32 && runs <= 64 * 2 * 16 ? 2 : 4)) ch *= 2;
  return {64, (int)ceil_div(runs, 64 * ch), ch};
}

struct Plan {
  Shape z;
  int64_t entries, rows;  // of an entry
  int groups, parts, mod;
};
// mod: kModToken also where each batch entry is a single token (its modulation is then read as a token's)
Plan plan_norm(svgear_dtype dt, int64_t B, int64_t N, int c, int mod, bool backward) {
  Plan p{};
  p.z = shape_of(c, dt);
  p.mod = mod;
  p.entries = mod == kModEntry ? B : 1;
  p.rows = mod == kModEntry ? N : B * N;
  const int per_group = p.z.wpr > 1 ? 1 : kNormWaves * (64 / p.z.lanes), waves = p.z.wpr > 1 ? p.z.wpr : kNormWaves;
  // One round of workgroups that stay, of so many waves a CU that some 30 KB of rows are on their way to it: 75,600 x 5,120 forward
  // with 3 / 6 / 9 / 12 waves of 4 KB 465 / 319 / 300 / 307 us. Backward a workgroup leaves a row of sums, which is worth three rows
  // of x at least (2 x 777 rows of 1,541 in fp32, with 4 / 3 / 2 of them 21.4 / 20.2 / 21.9 us).
  const int lane_bytes = 8 * p.z.ch * (int)esize(dt);
  const int resident = std::max(1, std::min((backward ? 384 : 576) / lane_bytes, backward ? 20 : 24) / waves);
  const int64_t wanted = std::max<int64_t>(256 * resident / p.entries, 1), most = ceil_div(p.rows, per_group * (backward ? 3 : 1));
  p.groups = (int)std::min(wanted, most);
  p.parts = p.groups * (p.z.wpr > 1 ? 1 : kNormWaves);
  return p;
}

template <typename T, int L, int CH, int MAXW>
int launch_shape(const NormArgs& a, const Plan& p, bool backward, hipStream_t s) {
  const dim3 grid = long_grid(p.entries * p.groups, 1);
  const int threads = 64 * (p.z.wpr > 1 ? p.z.wpr : kNormWaves);
  auto by_mod = [&](auto whole) {
    constexpr bool W = decltype(whole)::value;
    if (backward) {
      if (p.mod == kModToken) layer_norm_backward_kernel<T, L, CH, kModToken, MAXW, W><<<grid, threads, 0, s>>>(a);
      else layer_norm_backward_kernel<T, L, CH, kModEntry, MAXW, W><<<grid, threads, 0, s>>>(a);
    } else {
      if (p.mod == kModToken) layer_norm_kernel<T, L, CH, kModToken, MAXW, W><<<grid, threads, 0, s>>>(a);
      else layer_norm_kernel<T, L, CH, kModEntry, MAXW, W><<<grid, threads, 0, s>>>(a);
    }
  };
  if (a.c % 8 == 0) by_mod(std::true_type{});
  else by_mod(std::false_type{});
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

template <typename T>
int launch_norm(NormArgs& a, const Plan& p, bool backward, hipStream_t s) {
  a.entries = (int)p.entries;
  a.R = p.rows;
  a.wpr = p.z.wpr;
  a.groups = p.groups;
  a.parts = p.parts;
  if (p.z.lanes == 8) return launch_shape<T, 8, 1, kNormWaves>(a, p, backward, s);
  if (p.z.lanes == 16) return launch_shape<T, 16, 1, kNormWaves>(a, p, backward, s);
  if (p.z.lanes == 32) return launch_shape<T, 32, 1, kNormWaves>(a, p, backward, s);
  if (p.z.ch == 1) return launch_shape<T, 64, 1, kNormWaves>(a, p, backward, s);
  if (p.z.ch == 2 && p.z.wpr <= 8) return launch_shape<T, 64, 2, 8>(a, p, backward, s);
  // (two runs a lane are one wave in bf16, four are nine waves at least in fp32)
  if constexpr (sizeof(T) == 4) {
    if (p.z.ch == 2) return launch_shape<T, 64, 2, 16>(a, p, backward, s);
  } else {
    if (p.z.wpr <= 8) return launch_shape<T, 64, 4, 8>(a, p, backward, s);
  }
  return launch_shape<T, 64, 4, 16>(a, p, backward, s);
}

bool norm_sizes_ok(svgear_dtype dt, int B, int64_t N, int c, float eps) {
  return (dt == SVGEAR_F32 || dt == SVGEAR_BF16) && B > 0 && N > 0 && N <= kMaxNormRows && (int64_t)B * N <= kMaxNormRows && c > 0 &&
         c <= kMaxNormWidth && eps >= 0.f && eps < INFINITY;
}
bool in_ok(const void* p, const int64_t st[2], svgear_dtype dt) {
  return p && st && st[0] >= 0 && st[1] >= 0 && st[0] <= kMaxStride && st[1] <= kMaxStride && reinterpret_cast<uintptr_t>(p) % esize(dt) == 0;
}
bool out_ok(const void* p, const int64_t st[2], svgear_dtype dt, int64_t B, int64_t N, int64_t width) {
  if (!in_ok(p, st, dt)) return false;
  const bool b_inner = (B > 1 && N > 1) ? st[0] < st[1] : B > 1;
  const int64_t inner = b_inner ? st[0] : st[1], n_inner = b_inner ? B : N, outer = b_inner ? st[1] : st[0], n_outer = b_inner ? N : B;
  if (n_inner > 1 && inner < width) return false;
  return n_outer == 1 || outer >= (n_inner > 1 ? (__int128)(n_inner - 1) * inner : 0) + width;
}
bool vector_ok(const void* p, svgear_dtype dt) { return reinterpret_cast<uintptr_t>(p) % esize(dt) == 0; }
// Strides of one batch entry and of one token do not matter.
Rows rows_of(const int64_t st[2], int64_t B, int64_t N) { return Rows{B > 1 ? st[0] : 0, N > 1 ? st[1] : 0}; }
bool same_rows(const int64_t p[2], const int64_t q[2], int64_t B, int64_t N) { return (B == 1 || p[0] == q[0]) && (N == 1 || p[1] == q[1]); }

// The modulation of batch entries of one token each is that of tokens.
int of_tokens(int modulation, int64_t N) { return modulation == kModEntry && N == 1 ? (int)kModToken : modulation; }

}  // namespace
}  // namespace svgear

using namespace svgear;

extern "C" int svgear_layer_norm(const void* x, const int64_t xstride[2], const void* weight, const void* bias, const void* scale,
                                 const int64_t sstride[2], const void* shift, const int64_t hstride[2], svgear_dtype dt, int B,
                                 int64_t N, int c, float eps, void* y, const int64_t ystride[2], void* stream) {
  if (!norm_sizes_ok(dt, B, N, c, eps) || !in_ok(x, xstride, dt) || !vector_ok(weight, dt) || !vector_ok(bias, dt) ||
      (scale && !in_ok(scale, sstride, dt)) || (shift && !in_ok(shift, hstride, dt)) || !out_ok(y, ystride, dt, B, N, c))
    return SVGEAR_ERR_INVALID;
  if (y == weight || y == bias || y == scale || y == shift || (y == x && !same_rows(xstride, ystride, B, N))) return SVGEAR_ERR_INVALID;
  NormArgs a{};
  a.x = x, a.weight = weight, a.bias = bias, a.scale = scale, a.shift = shift, a.y = y;
  a.xst = rows_of(xstride, B, N);
  a.yst = rows_of(ystride, B, N);
  if (scale) a.sst = rows_of(sstride, B, N);
  if (shift) a.hst = rows_of(hstride, B, N);
  a.n = N;
  a.c = c;
  a.eps = eps;
  const bool tokens = N == 1 || (scale && sstride[1] != 0) || (shift && hstride[1] != 0);
  const Plan p = plan_norm(dt, B, N, c, !scale && !shift ? kModNone : tokens ? kModToken : kModEntry, false);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return dt == SVGEAR_F32 ? launch_norm<float>(a, p, false, s) : launch_norm<bf16_t>(a, p, false, s);
}

extern "C" size_t svgear_layer_norm_backward_workspace(svgear_dtype dt, int B, int64_t N, int c, int modulation) {
  if (!norm_sizes_ok(dt, B, N, c, 0.f) || modulation < kModNone || modulation > kModToken) return 0;
  const Plan p = plan_norm(dt, B, N, c, of_tokens(modulation, N), true);
  return align_up((size_t)(p.entries * p.parts) * 2 * c * sizeof(float), 256);
}

extern "C" int svgear_layer_norm_backward(const void* dy, const int64_t dystride[2], const void* x, const int64_t xstride[2],
                                          const void* weight, const void* bias, const void* scale, const int64_t sstride[2],
                                          int modulation, svgear_dtype dt, int B, int64_t N, int c, float eps, void* dx,
                                          const int64_t dxstride[2], void* dweight, void* dbias, void* dscale, void* dshift,
                                          void* ws, size_t ws_bytes, void* stream) {
  if (!norm_sizes_ok(dt, B, N, c, eps) || !in_ok(dy, dystride, dt) || !in_ok(x, xstride, dt) || !vector_ok(weight, dt) ||
      !vector_ok(bias, dt) || (scale && !in_ok(scale, sstride, dt)) || (dx && !out_ok(dx, dxstride, dt, B, N, c)) ||
      !vector_ok(dweight, dt) || !vector_ok(dbias, dt) || !vector_ok(dscale, dt) || !vector_ok(dshift, dt) ||
      (!dx && !dweight && !dbias && !dscale && !dshift) || modulation < kModNone || modulation > kModToken)
    return SVGEAR_ERR_INVALID;
  if (modulation == kModNone && (scale || dscale || dshift)) return SVGEAR_ERR_INVALID;
  if (modulation == kModEntry && scale && N > 1 && sstride[1] != 0) return SVGEAR_ERR_INVALID;
  const void* outs[5] = {dx, dweight, dbias, dscale, dshift};
  const void* ins[5] = {dy, x, weight, bias, scale};
  for (int i = 0; i < 5; ++i) {
    if (!outs[i]) continue;
    for (int j = 0; j < 5; ++j)
      if ((j != i && outs[i] == outs[j]) || (outs[i] == ins[j] && !(i == 0 && j == 0 && same_rows(dystride, dxstride, B, N))))
        return SVGEAR_ERR_INVALID;
  }
  const int mod = of_tokens(modulation, N);
  const bool sums = dweight || dbias || (mod == kModEntry && (dscale || dshift));
  if (sums && (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < svgear_layer_norm_backward_workspace(dt, B, N, c, modulation)))
    return SVGEAR_ERR_WORKSPACE;
  NormArgs a{};
  a.dy = dy, a.x = x, a.weight = weight, a.bias = bias, a.scale = scale, a.y = dx;
  a.dyst = rows_of(dystride, B, N);
  a.xst = rows_of(xstride, B, N);
  if (dx) a.yst = rows_of(dxstride, B, N);
  if (scale) a.sst = rows_of(sstride, B, N);
  if (mod == kModToken) a.dscale = dscale, a.dshift = dshift;
  a.n = N;
  a.c = c;
  a.eps = eps;
  if (sums) a.partial = static_cast<float*>(ws);
  const Plan p = plan_norm(dt, B, N, c, mod, true);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int rc = dt == SVGEAR_F32 ? launch_norm<float>(a, p, true, s) : launch_norm<bf16_t>(a, p, true, s);
  if (rc != SVGEAR_OK || !sums) return rc;
  NormSums z{};
  z.partial = a.partial, z.weight = weight, z.bias = bias, z.dweight = dweight, z.dbias = dbias;
  z.entries = (int)p.entries, z.parts = p.parts, z.c = c;
  if (mod == kModEntry) {
    z.scale = scale, z.scale_b = a.sst.b;
    z.dscale = dscale, z.dshift = dshift;
  }
  const unsigned blocks = (unsigned)ceil_div(c, 16);
  const unsigned dealt = z.entries <= kEntriesOfOne ? 1u : std::min((unsigned)z.entries, std::max(2048u / blocks, 8u));
  auto launch = [&](unsigned workgroups, auto joined) -> int {
    z.dealt = (int)workgroups;
    if (dt == SVGEAR_F32) layer_norm_sums_kernel<float, decltype(joined)::value><<<dim3(blocks, workgroups), 1024, 0, s>>>(z);
    else layer_norm_sums_kernel<bf16_t, decltype(joined)::value><<<dim3(blocks, workgroups), 1024, 0, s>>>(z);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  };
  const int summed = launch(dealt, std::false_type{});
  if (summed != SVGEAR_OK || dealt == 1 || (!dweight && !dbias)) return summed;
  z.joined_pitch = (int64_t)z.parts * 2 * c;
  z.entries = 1, z.parts = (int)dealt;
  z.weight = z.bias = z.scale = nullptr;
  z.dscale = z.dshift = nullptr;
  return launch(1, std::true_type{});
}

// svgear_linear and svgear_linear_backward: argument checks, the copies of operands that the tile kernel
// cannot read in place, and what is done element by element.
#include "linear.h"

namespace svgear {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxWidth = 1 << 21;
constexpr int64_t kMaxRows = 1 << 30;
constexpr int64_t kMaxPitch = 1 << 21;  // a tile's rows are addressed by 32-bit byte offsets: 256 rows of 8 MB

// ---- rows copied to an even, 16-byte aligned pitch, zeros behind the values; a 16-byte piece a thread, one or two operands
struct PackJob {
  const void* src;
  void* dst;
  Rows st;
  int64_t pitch, pieces;  // of a row of dst; in all
  int n, rows, width;
};
template <typename T>
__global__ void __launch_bounds__(kThreads)
pack_rows_kernel(PackJob a, PackJob b) {
  constexpr int CH = 16 / sizeof(T);
  const PackJob& p = blockIdx.y ? b : a;
  const int64_t across = p.pitch / CH;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < p.pieces; i += (int64_t)gridDim.x * kThreads) {
    const int r = (int)(i / across), col = (int)(i - r * across) * CH, e = p.n >= p.rows ? 0 : r / p.n;
    const T* s = static_cast<const T*>(p.src) + (int64_t)e * p.st.b + (int64_t)(r - e * p.n) * p.st.n + col;
    uint4 u;
    if (col + CH <= p.width) {
      u = load16(s);
    } else {
      T v[CH];
#pragma unroll
      for (int k = 0; k < CH; ++k) v[k] = col + k < p.width ? s[k] : T(0);
      __builtin_memcpy(&u, v, 16);
    }
    *reinterpret_cast<uint4*>(static_cast<T*>(p.dst) + (int64_t)r * p.pitch + col) = u;
  }
}

// ---- out[g][c] = sum over i of part[g][i][c]: 32 runs of rows, each every 32nd, then those in order
constexpr int kSumThreads = 1024;
template <typename T>
__global__ void __launch_bounds__(kSumThreads)
sum_rows_kernel(const float* part, T* out, const float* part2, T* out2, int rows, int cols, int groups) {
  __shared__ float s[32][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  if (blockIdx.z) part = part2, out = out2;
  for (int g = blockIdx.y; g < groups; g += gridDim.y) {
    const float* p = part + (int64_t)g * rows * cols;
    float v = 0.f;
    if (c < cols)
#pragma unroll 8
      for (int i = y; i < rows; i += 32) v += p[(int64_t)i * cols + c];
    s[y][x] = v;
    __syncthreads();
    if (y == 0 && c < cols) {
#pragma unroll
      for (int k = 1; k < 32; ++k) v += s[k][x];
      store1(out + (int64_t)g * cols + c, v);
    }
    __syncthreads();
  }
}

// ---- the epilogue on partial products
template <typename T>
__global__ void __launch_bounds__(kThreads)
linear_merge_kernel(LinearArgs a, int runs) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int r = (int)(i / runs), c = (int)(i % runs) * 8;
  if (r >= a.R) return;
  const bool whole8 = c + 8 <= a.C;
  float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int p = 0; p < a.splits; ++p) {
    const float* o = a.partial + ((int64_t)p * a.R + r) * a.C + c;
    if (whole8) {
      float w[8];
      load8(o, w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += w[k];
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (c + k < a.C) v[k] += o[k];
    }
  }
  if (whole8) {
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (a.bias) load8(static_cast<const T*>(a.bias) + c, bias);
    finish8<T>(a, r, c, v, bias);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (c + k < a.C) finish1<T>(a, r, c + k, v[k]);
  }
}

// ---- dz, the partial sums of dbias, and dgate
// eight elements, those of them that exist, others 0
template <typename T>
__device__ __forceinline__ void load_values(const T* p, int left, float (&v)[8]) {
  if (left >= 8) {
    load8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < left ? load_as_f32(p + i) : 0.f;
  }
}
template <typename T>
__device__ __forceinline__ void store_values(T* p, int left, const float (&v)[8]) {
  if (left >= 8) {
    store8(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < left) store1(p + i, v[i]);
  }
}

struct GradientArgs {
  const void* dy;
  const void* pre;   // or null
  const void* gate;  // or null
  void* dz;          // [R][pitch], or null
  void* dgate;       // [R][C] where the gate is of tokens, or null
  float* sum_dz;     // [blocks][C] or null
  float* sum_da;     // [blocks][C] or null: a batch entry's blocks together
  Rows yst, gst;
  int64_t pitch;
  int C, n, act;
  int blocks, blocks_b, rows_block;  // blocks, those of a batch entry, rows of a block
};

// A workgroup takes 256 columns of a run of rows of one batch entry, 8 a thread, its 8 half waves every eighth row. WHOLE: C is a
// multiple of 8.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads)
linear_gradient_kernel(GradientArgs a) {
  constexpr int V = 8, LANES = 32, WAYS = kThreads / LANES;
  __shared__ float s[2][WAYS][LANES * V + 4];
  const int x = threadIdx.x % LANES, way = threadIdx.x / LANES;
  const int c0 = blockIdx.y * LANES * V, c = c0 + x * V, left = WHOLE ? 8 : a.C - c;
  const int block = (int)long_grid_index();
  if (block >= a.blocks) return;
  const int b = block / a.blocks_b, first = block % a.blocks_b * a.rows_block;
  const int last = min(first + a.rows_block, a.n);
  const T* dy = static_cast<const T*>(a.dy) + (int64_t)b * a.yst.b + c;
  const T* gate = a.gate ? static_cast<const T*>(a.gate) + (int64_t)b * a.gst.b + c : nullptr;
  const int64_t r0 = (int64_t)b * a.n;
  float sz[V], sa[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sz[i] = sa[i] = 0.f;
  if (c < a.C) {
    float g[V];
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = 1.f;
    const bool one_gate = gate && a.gst.n == 0;
    if (one_gate) load_values(gate, left, g);
    for (int t = first + way; t < last; t += WAYS) {
      float d[V], z[V], act[V];
      load_values(dy + (int64_t)t * a.yst.n, left, d);
      if (a.pre) load_values(static_cast<const T*>(a.pre) + (r0 + t) * a.C + c, left, z);
      if (gate && !one_gate) load_values(gate + (int64_t)t * a.gst.n, left, g);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const float y = d[i];
        act[i] = 0.f;
        if (a.pre) d[i] = y * act_slope<T>(a.act, z[i], act[i]);
        act[i] *= y;
        if (gate) d[i] *= g[i];
        sz[i] += d[i];
        sa[i] += act[i];
      }
      // dz for the products, in the tensors' type: the matrix cores take bf16 at ten times fp32's rate (1,590 and 151 TFLOP/s).
      // In bf16 that rounding makes the error of dx and dw against 64 bits 2.35e-3, 1.66e-3 with their own rounding alone
      // (9,450 x 20,480 of 5,120); dz as the sum of two bf16 values would take each product twice. The sums here take it as
      // it is. (Its rows are whole 16-byte pieces, zeros behind the values.)
      if (a.dz) store_values(static_cast<T*>(a.dz) + (r0 + t) * a.pitch + c, WHOLE ? V : (int)min(a.pitch - c, (int64_t)V), d);
      if (a.dgate) store_values(static_cast<T*>(a.dgate) + (r0 + t) * a.C + c, left, act);
    }
  }
  if (!a.sum_dz && !a.sum_da) return;
#pragma unroll
  for (int i = 0; i < V; ++i) s[0][way][x * V + i] = sz[i], s[1][way][x * V + i] = sa[i];
  __syncthreads();
  for (int i = threadIdx.x; i < LANES * V; i += kThreads) {
    if (c0 + i >= a.C) break;
    float z = 0.f, v = 0.f;
#pragma unroll
    for (int w = 0; w < WAYS; ++w) z += s[0][w][i], v += s[1][w][i];
    if (a.sum_dz) a.sum_dz[(int64_t)block * a.C + c0 + i] = z;
    if (a.sum_da) a.sum_da[(int64_t)block * a.C + c0 + i] = v;
  }
}

// ---- host side
int64_t chunk(svgear_dtype dt) { return dt == SVGEAR_F32 ? 4 : 8; }
int64_t even_pitch(int64_t width, svgear_dtype dt) { return ceil_div(width, chunk(dt)) * chunk(dt); }

// Whether the tile kernel can read these rows where they are.
bool in_place(const void* p, int64_t pitch, int64_t width, svgear_dtype dt) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && pitch % chunk(dt) == 0 && width % chunk(dt) == 0 && pitch <= kMaxPitch;
}
// [B,N,width] as one run of rows: their distance, or -1.
int64_t run_pitch(const int64_t st[2], int B, int64_t N) {
  if (B == 1) return st[1];
  if (N == 1) return st[0];
  return st[0] == (__int128)N * st[1] ? st[1] : -1;
}
bool rows_in_place(const void* p, const int64_t st[2], int B, int64_t N, int64_t width, svgear_dtype dt) {
  const int64_t pitch = run_pitch(st, B, N);
  return pitch >= 0 && in_place(p, pitch, width, dt);
}
size_t packed_bytes(int64_t rows, int64_t width, svgear_dtype dt) {
  return align_up((size_t)rows * even_pitch(width, dt) * esize(dt), 256);
}

// The copies that a call needs, made by one launch.
struct Packing {
  PackJob job[2] = {};
  int jobs = 0;
  void add(const void* src, Rows st, int64_t n, int64_t rows, int64_t width, svgear_dtype dt, Workspace& w, Operand& out) {
    out.pitch = even_pitch(width, dt);
    void* dst = w.take<unsigned char>((size_t)rows * out.pitch * esize(dt));
    out.p = dst;
    job[jobs++] = PackJob{src, dst, st, out.pitch, rows * (out.pitch / chunk(dt)), (int)n, (int)rows, (int)width};
  }
  int launch(svgear_dtype dt, hipStream_t s) const {
    if (jobs == 0) return SVGEAR_OK;
    int64_t blocks = 1;
    for (int k = 0; k < jobs; ++k)
      if (ceil_div(job[k].pieces, kThreads) > blocks) blocks = ceil_div(job[k].pieces, kThreads);
    const dim3 grid((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20), (unsigned)jobs);
    if (dt == SVGEAR_F32)
      pack_rows_kernel<uint32_t><<<grid, kThreads, 0, s>>>(job[0], job[1]);
    else
      pack_rows_kernel<bf16_t><<<grid, kThreads, 0, s>>>(job[0], job[1]);
    SVGEAR_LAUNCH_CHECK();
    return SVGEAR_OK;
  }
};

// Whether the tile kernel reads the weights where they are by the element: fp32 rows that it cannot read by 16 bytes, where the
// product has few rows, so that a copy costs more than four times the loads (forward and dx, us with the copy and without it: 60 rows, 14,453 in,
// 4,239 out 188 / 189 and 106 / 98; 128 rows, 3,723 in, 5,001 out 83 / 85 and 65 / 64; 256 rows 121 / 124 and 115 / 107; 384 rows 162 / 161 and
// 160 / 167).
bool by_element(const void* w, int64_t w_stride, int64_t d_in, svgear_dtype dt, int64_t rows) {
  return dt == SVGEAR_F32 && rows <= 256 && w_stride <= kMaxPitch && !in_place(w, w_stride, d_in, dt);
}

// What of svgear_linear's operands goes through the workspace. Few rows: x only, where its batches are not one run of rows.
struct Copies {
  bool x, w;
};
Copies operand_copies(const void* x, const int64_t xstride[2], const void* w, int64_t w_stride, svgear_dtype dt, int B,
                      int64_t N, int64_t d_in) {
  if (B * N <= few_rows(dt)) return Copies{run_pitch(xstride, B, N) < 0, false};
  return Copies{!rows_in_place(x, xstride, B, N, d_in, dt), !in_place(w, w_stride, d_in, dt) && !by_element(w, w_stride, d_in, dt, B * N)};
}

bool sizes_ok(svgear_dtype dt, int B, int64_t N, int d_in, int d_out) {
  return (dt == SVGEAR_F32 || dt == SVGEAR_BF16) && B > 0 && N > 0 && N <= kMaxRows && (int64_t)B * N <= kMaxRows &&
         d_in > 0 && d_out > 0 && d_in <= kMaxWidth && d_out <= kMaxWidth;
}
bool input_ok(const void* p, const int64_t st[2], svgear_dtype dt) {
  return p && st && st[0] >= 0 && st[1] >= 0 && st[0] <= kMaxStride && st[1] <= kMaxStride && reinterpret_cast<uintptr_t>(p) % esize(dt) == 0;
}
bool output_ok(const void* p, const int64_t st[2], svgear_dtype dt, int64_t B, int64_t N, int64_t width) {
  if (!input_ok(p, st, dt)) return false;
  const bool b_inner = st[0] < st[1];
  const int64_t inner = b_inner ? st[0] : st[1], n_inner = b_inner ? B : N, outer = b_inner ? st[1] : st[0],
                n_outer = b_inner ? N : B;
  if (n_inner > 1 && inner < width) return false;
  return n_outer == 1 || outer >= (n_inner > 1 ? (__int128)(n_inner - 1) * inner : 0) + width;
}

int launch(const LinearArgs& a, svgear_dtype dt, int form, hipStream_t s) {
  const int rc = a.tile == 0 ? launch_linear_rows(a, dt, s) : dt == SVGEAR_F32 ? launch_linear_f32(a, form, s) : launch_linear_bf16(a, form, s);
  if (rc != SVGEAR_OK || !a.partial) return rc;
  return launch_linear_merge(a, dt, s);
}

// Tile and number of parts of K of a product: the least of an estimate in microseconds. m tiles on the CU that has most
// of them take their steps in turn, max(alone, m * step) each (a single workgroup waits for its own copies and barriers;
// 256 x 256: one at a time), `once` for their prologues and epilogues, `first` for those that nothing hides; joining parts costs a launch and their products'
// way to memory and back. The constants are measured. Both sides of the choices, us, MI355X, bf16, C x R of K: 5120 x 256 of 4096
// in tiles of 64 / 128 / 128 in 3 parts: 30 / 34 / 25; 2048 x 512 of 2048 in 64 / 128: 12 / 17; 5120 x 2000 of 5120 in 128 / 256:
// 118 / 100; 2048 x 4000 of 6000: 106 / 114. fp32, 1000 x 1554 of 640 in 64 / 128: 27 / 45, 1536 x 2103 of 1024 73 / 69, 1541 x 2103 of 1003 with a full epilogue 90 / 88; 1000 x 700 of 3000
// in 64, one part / 4: 56 / 46.
// Up to 32 rows in fp32, whose matrix cores the idle rows of a tile of 64 would keep busy, have one of 32 x 128 (30,720 x 9 of 5,120:
// 169 us by 64, 119; 5,120 x 32 of 5,120 39 and 28; for more rows it is no faster, nor is
// it in bf16; the weights' gradient, whose rows are d_out, has none).
// Few rows (forward only) go to the kernel that reads the weights straight into registers.
struct Plan {
  int tile, splits;
};
// element: by_element's rows, for which there are tiles of 32 and 64 alone. K is cut for them as for aligned rows, so that results
// do not depend on where the weights lie (every tile adds a part's products in one order). That costs something where aligned
// rows have tiles of 128, some 2 % of the sizes of 9 to 256 rows (200 rows, 8,192 in, 5,120 out at an odd address, in 4 parts and
// in 3: 212 and 222 us; 100 rows, 20,480 in, 8,192 out, 2 and 8: 391 and 420).
Plan plan_product(int64_t R, int64_t C, int64_t K, svgear_dtype dt, int form, bool element) {
  if (form == kContractBoth && R <= few_rows(dt)) return Plan{0, 1};
  struct Kind {
    int tile, rows, cols;
    double alone, step, once, first;
  };
  static const Kind bf16[] = {{64, 64, 64, 0.40, 0.19, 1.0, 0.0}, {128, 128, 128, 0.50, 0.475, 1.5, 0.0}, {256, 256, 256, 1.3, 1.3, 9.0, 0.0}};
  static const Kind f32[] = {{64, 64, 64, 0.56, 0.53, 1.0, 0.0}, {128, 128, 128, 1.9, 1.85, 2.0, 10.0}, {32, 32, 128, 0.6, 0.55, 1.0, 0.0}};
  const Kind* kinds = dt == SVGEAR_F32 ? f32 : bf16;
  const int64_t steps = ceil_div(K, dt == SVGEAR_F32 ? 32 : 64);
  Plan best{64, 1};
  double least = 1e300;
  for (int i = 0; i < 3; ++i) {
    const Kind& k = kinds[i];
    if (k.rows == 32 && (R > 32 || form == kContractNone)) continue;
    const int64_t tiles = ceil_div(R, k.rows) * ceil_div(C, k.cols);
    for (int p = 1; p <= 16 && (p == 1 || (steps >= 4 * p && tiles < 1024)); ++p) {
      const double m = (double)ceil_div(tiles * p, 256), each = m * k.step;
      double us = (double)ceil_div(steps, p) * (each > k.alone ? each : k.alone) + m * k.once + k.first;
      if (p > 1) us += 4.0 + (double)p * (double)R * (double)C * 8.0 / 5e6;
      if (us < least) {
        least = us;
        best = Plan{k.tile, p};
      }
    }
  }
  if (element && best.tile == 128) best.tile = 64;
  return best;
}
size_t parts_bytes(int64_t R, int64_t C, int64_t K, svgear_dtype dt, int form, bool element) {
  const int p = plan_product(R, C, K, dt, form, element).splits;
  return p > 1 ? align_up((size_t)p * R * C * sizeof(float), 256) : 0;
}
void set_product(LinearArgs& a, const Operand& P, const Operand& Q, int64_t R, int64_t C, int64_t K, svgear_dtype dt,
                 int form, bool element, Workspace& w) {
  a.P = P;
  a.Q = Q;
  a.R = (int)R;
  a.C = (int)C;
  a.K = K;
  const Plan plan = plan_product(R, C, K, dt, form, element);
  a.by_element = element && plan.tile != 0;
  a.tile = plan.tile;
  a.splits = plan.splits;
  a.partial = a.splits > 1 ? w.take<float>((size_t)a.splits * R * C) : nullptr;
}

// Rows of a workgroup of linear_gradient_kernel, its workgroups of a batch entry: 128 rows where that makes 1,024 workgroups
// or more, down to 8 where it does not (fp32, 1,554 x 1,000 values: 12.4 us with 32 rows, 9.7 with 8).
int gradient_rows(int B, int64_t N, int d_out) {
  int rows = 128;
  while (rows > 8 && (int64_t)B * ceil_div(N, rows) * ceil_div(d_out, 256) < 1024) rows /= 2;
  return rows;
}
// Batch entries of one token each count as tokens of one entry, dgate included: its row is their own.
bool one_token_each(int B, int64_t N) { return N == 1 && B > 1; }
int gradient_blocks(int B, int64_t N, int d_out) { return (int)ceil_div(N, gradient_rows(B, N, d_out)); }

}  // namespace

int sum_rows(const float* part, void* out, const float* part2, void* out2, int rows, int cols, int groups, svgear_dtype dt,
             hipStream_t s) {
  const dim3 grid((unsigned)ceil_div(cols, 32), (unsigned)(groups < 65535 ? groups : 65535), part2 ? 2 : 1);
  if (dt == SVGEAR_F32)
    sum_rows_kernel<float><<<grid, kSumThreads, 0, s>>>(part, static_cast<float*>(out), part2, static_cast<float*>(out2), rows, cols, groups);
  else
    sum_rows_kernel<bf16_t><<<grid, kSumThreads, 0, s>>>(part, static_cast<bf16_t*>(out), part2, static_cast<bf16_t*>(out2), rows, cols, groups);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

int launch_linear_merge(const LinearArgs& a, svgear_dtype dt, hipStream_t s) {
  const int runs = (int)ceil_div(a.C, 8);
  const unsigned blocks = (unsigned)ceil_div((int64_t)a.R * runs, kThreads);
  if (dt == SVGEAR_F32)
    linear_merge_kernel<float><<<blocks, kThreads, 0, s>>>(a, runs);
  else
    linear_merge_kernel<bf16_t><<<blocks, kThreads, 0, s>>>(a, runs);
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

}  // namespace svgear

using namespace svgear;

extern "C" size_t svgear_linear_workspace(const void* x, const int64_t xstride[2], const void* w, int64_t w_stride,
                                          svgear_dtype dt, int B, int64_t N, int d_in, int d_out) {
  if (!sizes_ok(dt, B, N, d_in, d_out) || !input_ok(x, xstride, dt) || !w || w_stride < d_in ||
      w_stride > kMaxStride)
    return 0;
  const Copies copies = operand_copies(x, xstride, w, w_stride, dt, B, N, d_in);
  size_t bytes = 0;
  if (copies.x) bytes += packed_bytes((int64_t)B * N, d_in, dt);
  if (copies.w) bytes += packed_bytes(d_out, d_in, dt);
  return bytes + parts_bytes((int64_t)B * N, d_out, d_in, dt, kContractBoth, by_element(w, w_stride, d_in, dt, (int64_t)B * N));
}

extern "C" int svgear_linear(const void* x, const int64_t xstride[2], const void* w, int64_t w_stride,
                             const void* bias, svgear_dtype dt, int B, int64_t N, int d_in, int d_out, svgear_act act,
                             const void* gate, const int64_t gstride[2], const void* residual,
                             const int64_t rstride[2], void* pre, void* y, const int64_t ystride[2], void* ws,
                             size_t ws_bytes, void* stream) {
  if (!sizes_ok(dt, B, N, d_in, d_out) || !input_ok(x, xstride, dt) || !w || reinterpret_cast<uintptr_t>(w) % esize(dt) ||
      w_stride < d_in || w_stride > kMaxStride || !output_ok(y, ystride, dt, B, N, d_out) || (int)act < 0 || (int)act > (int)SVGEAR_ACT_GELU_TANH ||
      (gate && !input_ok(gate, gstride, dt)) || (residual && !input_ok(residual, rstride, dt)) ||
      reinterpret_cast<uintptr_t>(bias) % esize(dt) || reinterpret_cast<uintptr_t>(pre) % esize(dt))
    return SVGEAR_ERR_INVALID;
  if (y == x || y == w || y == gate || y == bias || (pre && (pre == y || pre == x || pre == w || pre == gate || pre == residual || pre == bias)))
    return SVGEAR_ERR_INVALID;
  if (residual == y && ((B > 1 && rstride[0] != ystride[0]) || (N > 1 && rstride[1] != ystride[1])))
    return SVGEAR_ERR_INVALID;
  const size_t need = svgear_linear_workspace(x, xstride, w, w_stride, dt, B, N, d_in, d_out);
  if (need && (!ws || reinterpret_cast<uintptr_t>(ws) % 256 || ws_bytes < need)) return SVGEAR_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Workspace space(ws, ws_bytes);
  const int64_t M = (int64_t)B * N;
  Operand X{x, run_pitch(xstride, B, N)}, W{w, w_stride};
  const Copies copies = operand_copies(x, xstride, w, w_stride, dt, B, N, d_in);
  Packing packing;
  if (copies.x) packing.add(x, Rows{xstride[0], xstride[1]}, N, M, d_in, dt, space, X);
  if (copies.w) packing.add(w, Rows{0, w_stride}, d_out, d_out, d_in, dt, space, W);
  const int rc = packing.launch(dt, s);
  if (rc != SVGEAR_OK) return rc;
  LinearArgs a{};
  set_product(a, W, X, M, d_out, d_in, dt, kContractBoth, by_element(w, w_stride, d_in, dt, M), space);
  a.n = (int)N;
  a.bias = bias;
  a.gate = gate;
  a.residual = residual;
  a.pre = pre;
  a.y = y;
  a.yst = Rows{ystride[0], ystride[1]};
  if (gate) a.gst = Rows{gstride[0], gstride[1]};
  if (residual) a.rst = Rows{rstride[0], rstride[1]};
  a.act = act;
  return launch(a, dt, kContractBoth, s);
}

extern "C" size_t svgear_linear_backward_workspace(const void* dy, const int64_t dystride[2], const void* x,
                                                   const int64_t xstride[2], const void* w, int64_t w_stride,
                                                   svgear_dtype dt, int B, int64_t N, int d_in, int d_out) {
  if (!sizes_ok(dt, B, N, d_in, d_out) || !input_ok(dy, dystride, dt) || (x && !input_ok(x, xstride, dt)) ||
      (w && (w_stride < d_in || w_stride > kMaxStride)))
    return 0;
  const int64_t M = (int64_t)B * N;
  size_t bytes = 256 + packed_bytes(M, d_out, dt);  // dz
  const bool fold = one_token_each(B, N);
  const int gb = fold ? 1 : B;
  bytes += 2 * align_up((size_t)gb * gradient_blocks(gb, fold ? B : N, d_out) * d_out * sizeof(float), 256);
  if (x) {
    if (!rows_in_place(x, xstride, B, N, d_in, dt)) bytes += packed_bytes(M, d_in, dt);
    bytes += parts_bytes(d_out, d_in, M, dt, kContractNone, false);
  }
  if (w) {
    const bool element = by_element(w, w_stride, d_in, dt, M);
    if (!in_place(w, w_stride, d_in, dt) && !element) bytes += packed_bytes(d_out, d_in, dt);
    bytes += parts_bytes(M, d_in, d_out, dt, kContractQ, element);
  }
  return bytes;
}

extern "C" int svgear_linear_backward(const void* dy, const int64_t dystride[2], const void* x,
                                      const int64_t xstride[2], const void* w, int64_t w_stride, const void* pre,
                                      svgear_dtype dt, int B, int64_t N, int d_in, int d_out, svgear_act act,
                                      const void* gate, const int64_t gstride[2], void* dx, const int64_t dxstride[2],
                                      void* dw, void* dbias, void* dgate, void* ws, size_t ws_bytes, void* stream) {
  const uintptr_t es = esize(dt);
  if (!sizes_ok(dt, B, N, d_in, d_out) || !input_ok(dy, dystride, dt) || (!dx && !dw && !dbias && !dgate) ||
      (dw && !x) || (x && !input_ok(x, xstride, dt)) || (dx && !w) ||
      (w && (w_stride < d_in || w_stride > kMaxStride || reinterpret_cast<uintptr_t>(w) % es)) || (int)act < 0 ||
      (int)act > (int)SVGEAR_ACT_GELU_TANH || (gate && !input_ok(gate, gstride, dt)) || (dgate && !gate) ||
      ((act != SVGEAR_ACT_NONE || dgate) && !pre) || (dx && !output_ok(dx, dxstride, dt, B, N, d_in)) ||
      reinterpret_cast<uintptr_t>(pre) % es || reinterpret_cast<uintptr_t>(dw) % es ||
      reinterpret_cast<uintptr_t>(dbias) % es || reinterpret_cast<uintptr_t>(dgate) % es)
    return SVGEAR_ERR_INVALID;
  const void* ins[] = {dy, x, w, pre, gate};
  void* outs[] = {dx, dw, dbias, dgate};
  for (int i = 0; i < 4; ++i) {
    for (const void* in : ins)
      if (outs[i] && outs[i] == in) return SVGEAR_ERR_INVALID;
    for (int j = 0; j < i; ++j)
      if (outs[i] && outs[i] == outs[j]) return SVGEAR_ERR_INVALID;
  }
  if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 ||
      ws_bytes < svgear_linear_backward_workspace(dy, dystride, x, xstride, w, w_stride, dt, B, N, d_in, d_out))
    return SVGEAR_ERR_WORKSPACE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  Workspace space(ws, ws_bytes);
  const int64_t M = (int64_t)B * N;

  // dz, unless it is dy itself and dy can be read where it is
  Operand dz{dy, run_pitch(dystride, B, N)};
  const bool same = act == SVGEAR_ACT_NONE && !gate;
  const bool make = (dx || dw) && !(same && rows_in_place(dy, dystride, B, N, d_out, dt));
  const bool fold = one_token_each(B, N), token_gate = gate && (gstride[1] != 0 || fold);
  const int gb = fold ? 1 : B, gn = fold ? B : (int)N;
  if (make || dbias || dgate) {
    GradientArgs g{};
    g.dy = dy;
    g.pre = act != SVGEAR_ACT_NONE || dgate ? pre : nullptr;
    g.gate = gate;
    if (make) {
      dz.pitch = even_pitch(d_out, dt);
      g.dz = space.take<unsigned char>((size_t)M * dz.pitch * es);
      dz.p = g.dz;
    }
    g.pitch = even_pitch(d_out, dt);
    g.yst = fold ? Rows{0, dystride[0]} : Rows{dystride[0], dystride[1]};
    if (gate) g.gst = fold ? Rows{0, gstride[0]} : Rows{gstride[0], gstride[1]};
    g.C = d_out;
    g.n = gn;
    g.act = act;
    g.rows_block = gradient_rows(gb, gn, d_out);
    g.blocks_b = gradient_blocks(gb, gn, d_out);
    g.blocks = gb * g.blocks_b;
    const size_t sums = (size_t)g.blocks * d_out;
    if (dbias) g.sum_dz = space.take<float>(sums);
    if (dgate && !token_gate) g.sum_da = space.take<float>(sums);
    if (dgate && token_gate) g.dgate = dgate;
    const dim3 grid = long_grid(g.blocks, ceil_div(d_out, 256));
    const bool whole = d_out % 8 == 0;
    if (dt == SVGEAR_F32)
      whole ? linear_gradient_kernel<float, true><<<grid, kThreads, 0, s>>>(g) : linear_gradient_kernel<float, false><<<grid, kThreads, 0, s>>>(g);
    else
      whole ? linear_gradient_kernel<bf16_t, true><<<grid, kThreads, 0, s>>>(g) : linear_gradient_kernel<bf16_t, false><<<grid, kThreads, 0, s>>>(g);
    SVGEAR_LAUNCH_CHECK();
    const bool together = dbias && g.sum_da && gb == 1;
    if (dbias) {
      const int rc = sum_rows(g.sum_dz, dbias, together ? g.sum_da : nullptr, together ? dgate : nullptr, g.blocks, d_out, 1, dt, s);
      if (rc != SVGEAR_OK) return rc;
    }
    if (g.sum_da && !together) {
      const int rc = sum_rows(g.sum_da, dgate, nullptr, nullptr, g.blocks_b, d_out, gb, dt, s);
      if (rc != SVGEAR_OK) return rc;
    }
  }

  Operand W{w, w_stride}, X{x, dw ? run_pitch(xstride, B, N) : 0};
  Packing packing;
  const bool element = dx && by_element(w, w_stride, d_in, dt, M);
  if (dx && !in_place(w, w_stride, d_in, dt) && !element) packing.add(w, Rows{0, w_stride}, d_out, d_out, d_in, dt, space, W);
  if (dw && !rows_in_place(x, xstride, B, N, d_in, dt))
    packing.add(x, Rows{xstride[0], xstride[1]}, N, M, d_in, dt, space, X);
  const int packed = packing.launch(dt, s);
  if (packed != SVGEAR_OK) return packed;
  if (dx) {
    LinearArgs a{};
    set_product(a, W, dz, M, d_in, d_out, dt, kContractQ, element, space);
    a.n = (int)N;
    a.y = dx;
    a.yst = Rows{dxstride[0], dxstride[1]};
    const int rc = launch(a, dt, kContractQ, s);
    if (rc != SVGEAR_OK) return rc;
  }
  if (dw) {
    LinearArgs a{};
    set_product(a, X, dz, d_out, d_in, M, dt, kContractNone, false, space);
    a.n = d_out;
    a.y = dw;
    a.yst = Rows{0, d_in};
    const int rc = launch(a, dt, kContractNone, s);
    if (rc != SVGEAR_OK) return rc;
  }
  return SVGEAR_OK;
}

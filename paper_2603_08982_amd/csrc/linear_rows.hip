// The matrix product of a few rows (single tokens, a time embedding, a modulation): every weight is read once for
// all of them, so it is bound by memory, and by latency where the weights are few.
//
// out[r][c] = sum_k Q[r][k] P[c][k]. A wave reads whole rows of weights, 1 KB at a time and several rows and pieces in
// flight, and multiplies them with the rows of Q on the vector ALU, bf16 by pairs. The waves of a workgroup have the same few columns and K in turn, their
// sums are added in order. Workgroups are small, so that all CUs get the same share of the weights: with the 16
// columns that a matrix instruction wants for each, 5,120 columns are 320 shares for 256 CUs (1 row of 5120 by 5120,
// bf16: 18.3 us that way, 12.9 this way; by 30,720: 66 and 60 us, 5.2 TB/s).
#include "linear.h"

namespace svgear {
namespace {

constexpr int kMaxWaves = 8;

// 16 bytes of a row: elements k.. of it, those < K, others 0; WHOLE: all or none of them.
template <typename T, bool WHOLE>
__device__ __forceinline__ uint4 load_piece(const T* row, int64_t k, int64_t K) {
  constexpr int CH = 16 / sizeof(T);
  if constexpr (WHOLE) {
    return k < K ? load16(row + k) : make_uint4(0, 0, 0, 0);
  } else {
    if (k + CH <= K) return load16(row + k);
    T e[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) e[i] = k + i < K ? row[k + i] : T(0);
    uint4 u;
    __builtin_memcpy(&u, e, 16);
    return u;
  }
}

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
// acc + the products of two pieces, bf16 by pairs (exact products, fp32 sums).
template <typename T>
__device__ __forceinline__ float multiply_piece(uint4 x, uint4 w, float acc) {
  const uint32_t a[4] = {x.x, x.y, x.z, x.w}, b[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      acc = __builtin_fmaf(__uint_as_float(a[i]), __uint_as_float(b[i]), acc);
    } else {
      union { uint32_t u; bf16x2v v; } p, q;
      p.u = a[i], q.u = b[i];
      acc = __builtin_amdgcn_fdot2_f32_bf16(p.v, q.v, acc, false);
    }
  }
  return acc;
}

// NR rows or fewer, CW columns a workgroup. WHOLE: K is a whole number of pieces.
template <typename T, int NR, int CW, bool WHOLE>
__global__ void __launch_bounds__(64 * kMaxWaves)
linear_rows_kernel(LinearArgs a) {
  constexpr int CH = 16 / sizeof(T), STEP = 64 * CH, U = 8 / CW;  // eight pieces of weights in flight
  __shared__ float sums[kMaxWaves][NR][CW];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int c0 = blockIdx.x * CW;
  const T* p[CW];
  const T* q[NR];
  float acc[NR][CW];
  // rows and columns past the last repeat it: what they give is not stored
#pragma unroll
  for (int c = 0; c < CW; ++c) p[c] = static_cast<const T*>(a.P.p) + (int64_t)min(c0 + c, a.C - 1) * a.P.pitch;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    q[r] = static_cast<const T*>(a.Q.p) + (int64_t)min(r, a.R - 1) * a.Q.pitch;
#pragma unroll
    for (int c = 0; c < CW; ++c) acc[r][c] = 0.f;
  }
  for (int64_t k = (int64_t)wave * STEP * U + lane * CH; k < a.K; k += (int64_t)waves * STEP * U) {
    uint4 w[U][CW];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int c = 0; c < CW; ++c) w[u][c] = load_piece<T, WHOLE>(p[c], k + u * STEP, a.K);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      uint4 x[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) x[r] = load_piece<T, WHOLE>(q[r], k + u * STEP, a.K);
#pragma unroll
      for (int c = 0; c < CW; ++c)
#pragma unroll
        for (int r = 0; r < NR; ++r) acc[r][c] = multiply_piece<T>(x[r], w[u][c], acc[r][c]);
    }
  }
#pragma unroll
  for (int r = 0; r < NR; ++r)
#pragma unroll
    for (int c = 0; c < CW; ++c) {
      float v = acc[r][c];
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
      if (lane == 0) sums[wave][r][c] = v;
    }
  __syncthreads();
  const int r = threadIdx.x / CW, c = threadIdx.x % CW;
  if (r < NR && r < a.R && c0 + c < a.C) {
    float v = 0.f;
    for (int w = 0; w < waves; ++w) v += sums[w][r][c];
    finish1<T>(a, r, c0 + c, v);
  }
}

template <typename T, int NR, int CW>
void launch_kernel(const LinearArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)ceil_div(a.C, CW);
  // two waves where they are enough for the GPU, more where columns are few and K is long
  const int64_t steps = ceil_div(a.K, (int64_t)(64 * 16 / sizeof(T)) * (8 / CW));
  int waves = grid >= 1024 ? 2 : kMaxWaves;
  while (waves > 1 && waves > steps) waves /= 2;
  if (a.K % (16 / sizeof(T)) == 0)
    linear_rows_kernel<T, NR, CW, true><<<grid, 64 * waves, 0, s>>>(a);
  else
    linear_rows_kernel<T, NR, CW, false><<<grid, 64 * waves, 0, s>>>(a);
}

template <typename T>
int launch_type(const LinearArgs& a, hipStream_t s) {
  // four columns a workgroup where they still are 1,024 of them, or where more rows than two make rereading those dear
  const bool many = a.C >= 4096 || a.R > 2;
  if (a.R <= 1) many ? launch_kernel<T, 1, 4>(a, s) : launch_kernel<T, 1, 1>(a, s);
  else if (a.R <= 2) many ? launch_kernel<T, 2, 4>(a, s) : launch_kernel<T, 2, 1>(a, s);
  else if (a.R <= 4) launch_kernel<T, 4, 4>(a, s);
  else if constexpr (sizeof(T) == 4) launch_kernel<T, 8, 4>(a, s);
  else return SVGEAR_ERR_UNSUPPORTED;
  SVGEAR_LAUNCH_CHECK();
  return SVGEAR_OK;
}

}  // namespace

int launch_linear_rows(const LinearArgs& a, svgear_dtype dt, hipStream_t s) {
  return dt == SVGEAR_F32 ? launch_type<float>(a, s) : launch_type<bf16_t>(a, s);
}

}  // namespace svgear

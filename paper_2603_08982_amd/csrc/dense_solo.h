// Dense attention and its gradients in fp32: a workgroup owns 32 rows, and its four waves take the other side's tiles in turn,
// each with buffers of its own, and meet once, at the end.
//
// What bounds it: the fp32 matrix cores, 64 cycles for a product of two rows of the contraction, so that copies, softmax and LDS
// reads hide behind the products of the wave itself and of the other wave of its SIMD (d = 64). Waves that share nothing need no
// barrier in the loop, and a workgroup of 32 rows is small enough that short documents and the triangle of a causal mask leave no CU
// behind (2 x 6 heads of 1,237 tokens in three documents 49 us; with 128 rows to a workgroup and shared tiles 61). There the matrix cores
// are busy 30 % of the cycles: 464 workgroups, the longest of which share a SIMD; with twice the parts it takes longer.
#pragma once
#include "dense_tile.h"

namespace svgear {
namespace {

template <int D>
struct Solo {
  using Z = Tile<float, D>;
  static constexpr int kRows = 32, kCopies = kRows / Z::kRowsPerCopy;  // of a workgroup and of a tile; copies of a tile
  static constexpr int kWave = 2 * Z::kBytes;                          // LDS of a wave
  static constexpr int kPitch = D + 4;                                 // floats of a row where the waves meet
  static_assert(kRows * kPitch * 4 <= kWave, "a wave's rows fit where its tiles were");
};

// 32 rows to a wave's tile; offset(row) in elements.
template <int D, typename RowOffset>
__device__ __forceinline__ void copy_solo(const float* base, uint32_t lds, int lane, RowOffset offset) {
  using Z = Tile<float, D>;
  // every read of what lay there has returned
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < Solo<D>::kCopies; ++i) {
    __builtin_amdgcn_sched_barrier(0);  // (one address at a time)
    const int row = i * Z::kRowsPerCopy + lane / Z::kChunks, chunk = (lane % Z::kChunks) ^ Z::swz(row);
    async_copy_16B(base + offset(row) + chunk * 4, (uint32_t)uniform((int)(lds + i * 1024)));
  }
}

// The same where all 32 rows are there and a lane's row of copy i is i * step elements from that of the first: one offset a lane,
// `at_lane` bytes, from addresses that the wave shares.
template <int D>
__device__ __forceinline__ void copy_solo(const float* base, int64_t step, uint32_t at_lane, uint32_t lds, int lane) {
  using Z = Tile<float, D>;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < Solo<D>::kCopies; ++i) {
    __builtin_amdgcn_sched_barrier(0);
    const int chunk = (lane % Z::kChunks) ^ Z::swz(i * Z::kRowsPerCopy + lane / Z::kChunks);
    async_copy_16B(uniform_ptr(base + i * step), at_lane + chunk * 16, (uint32_t)uniform((int)(lds + i * 1024)));
  }
}

// Rows [from, 32) of a wave's tile, whose copies have landed, are 0.
template <int D>
__device__ __forceinline__ void clear_solo(uint32_t lds, int from, int lane) {
  constexpr int C = Tile<float, D>::kChunks;
  for (int e = from * C + lane; e < Solo<D>::kRows * C; e += 64) clear_16B(lds + e * 16);
}

// The waves' sums of 32 rows, added in their order by all threads: out(row, first of four columns, their sum), each wave's times
// weight(wave, row).
template <int D, typename Weight, typename Put>
__device__ __forceinline__ void meet(unsigned char* smem, const f32x16 (&acc)[D / 32], int wave, int lane, Weight weight, Put put) {
  using Z = Tile<float, D>;
  constexpr int P = Solo<D>::kPitch;
  float* mine = reinterpret_cast<float*>(smem + wave * Solo<D>::kWave) + (lane & 31) * P;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  Z::each_four(acc, lane >> 5, [&](int d, float4 v) { store_four(mine + d, v); });
  __syncthreads();
  for (int u = threadIdx.x; u < 32 * (D / 4); u += 64 * kDenseWaves) {
    const int row = u / (D / 4), d = 4 * (u % (D / 4));
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kDenseWaves; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem + w * Solo<D>::kWave) + row * P + d);
      const float f = weight(w, row);
      s.x = __builtin_fmaf(f, v.x, s.x), s.y = __builtin_fmaf(f, v.y, s.y), s.z = __builtin_fmaf(f, v.z, s.z), s.w = __builtin_fmaf(f, v.w, s.w);
    }
    put(row, d, s);
  }
}
__device__ __forceinline__ float4 times(float4 v, float f) { return make_float4(v.x * f, v.y * f, v.z * f, v.w * f); }

}  // namespace
}  // namespace svgear

// Products of bf16 or fp16 matrices into fp32 parts (matmul.hpp has the main loop): what the linear loss and
// the gradient of the patch embedding have in common.  Where the tiles of the result are fewer than the
// compute units, k is split and every part leaves its own sums; the caller's last kernel joins them in
// a fixed order.
#include "mae_device.hpp"
#include "mae_kernels.hpp"
#include "matmul.hpp"

namespace mae {

namespace {

using namespace mm;

template <int TM, int TN, int WGM, int WGN, bool kAlongA, bool kHalf>
__global__ __launch_bounds__(64 * WGM * WGN) void matmul_kernel(MatmulArgs a) {
  using T = Tile<TM, TN, WGM, WGN, kAlongA, false, kHalf>;
  __shared__ __attribute__((aligned(1024))) u32x4 lds[T::kLdsBytes / 16];
  const int M = a.rows ? min(uniform(*a.rows), (int)a.M) : (int)a.M;
  const int K = a.depth ? min(uniform(*a.depth), (int)a.K) : (int)a.K;
  const uint32_t tiles_n = (uint32_t)((a.N + T::BN - 1) / T::BN);
  const uint32_t tiles = (uint32_t)((a.M + T::BM - 1) / T::BM) * tiles_n;
  const uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t part = id / tiles, tile = id - part * tiles;
  const uint32_t tm = tile / tiles_n, tn = tile - tm * tiles_n;
  const int m0 = (int)tm * T::BM, n0 = (int)tn * T::BN;
  if (m0 >= M) return;
  const int rows_m = min(T::BM, M - m0), rows_n = min(T::BN, a.N - n0);
  // this part's share of the slices of k
  const int slices = (K + kSlice - 1) / kSlice, share = (slices + a.parts - 1) / a.parts;
  const int s0 = uniform(min((int)part * share, slices)), s1 = uniform(min(s0 + share, slices));
  const int64_t k0 = (int64_t)s0 * kSlice;
  const int depth = uniform(min(s1 * kSlice, K) - min(s0 * kSlice, K));
  const Operand A{kAlongA ? a.A + m0 * a.lda + k0 : a.A + k0 * a.lda + m0, a.lda, rows_m};
  const Operand B{a.B + k0 * a.ldb + n0, a.ldb, rows_n};
  f32x16 acc[TM][TN];
  T::template run<0>(T::source(A, B, depth), lds, acc);

  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int wm = wave / WGN, wn = wave % WGN;
  float* out = a.out + ((int64_t)part * a.M + m0) * a.N + n0;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = wm * 32 * TM + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
      if (r >= rows_m) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int c = wn * 32 * TN + 32 * j + (lane & 31);
        if (c >= rows_n) continue;
        float* p = out + (int64_t)r * a.N + c;
        *p = a.accumulate ? *p + acc[i][j][e] : acc[i][j][e];
      }
    }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int TM, int TN, int WGM, int WGN>
void launch_sized(const MatmulArgs& a, bool along, bool half, hipStream_t stream) {
  constexpr int BM = 32 * TM * WGM, BN = 32 * TN * WGN;
  const dim3 grid((uint32_t)(ceil_div(a.M, BM) * ceil_div(a.N, BN) * a.parts)), block(64 * WGM * WGN);
  if (along) hipLaunchKernelGGL((matmul_kernel<TM, TN, WGM, WGN, true, true>), grid, block, 0, stream, a);
  else if (half) hipLaunchKernelGGL((matmul_kernel<TM, TN, WGM, WGN, false, true>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((matmul_kernel<TM, TN, WGM, WGN, false, false>), grid, block, 0, stream, a);
}

}  // namespace

int matmul_side(int64_t M, int N) {
  if (M <= 64 || N <= 64) return 64;
  if (M <= 512 || N <= 128) return 128;
  return 256;
}

int matmul_parts(int64_t M, int N, int64_t K, int side) {
  const int64_t tiles = ceil_div(M, side) * ceil_div(N, side);
  const int64_t slices = ceil_div(K, kSlice);
  int64_t parts = 256 / tiles;
  if (parts > slices / 4) parts = slices / 4;
  return parts < 1 ? 1 : (int)parts;
}

hipError_t launch_matmul(const MatmulArgs& a, MatmulKind kind, int side, hipStream_t stream) {
  const bool along = kind == MatmulKind::kHalfAlong, half = kind != MatmulKind::kBf16Across;
  if (side == 256) launch_sized<4, 2, 2, 4>(a, along, half, stream);
  else if (side == 128) launch_sized<2, 1, 2, 4>(a, along, half, stream);
  else launch_sized<1, 1, 2, 2>(a, along, half, stream);
  return hipGetLastError();
}

}  // namespace mae

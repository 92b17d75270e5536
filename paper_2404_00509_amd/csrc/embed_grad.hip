// Gradients of the patch embedding of the visible tokens: with g = the gradient of the tokens [M, E],
//   grad_weight[e, d] = sum over m of g[m, e] visible[m, d]
//   grad_bias[e]      = sum over m of g[m, e]
//   grad_pos[l, e]    = sum over the rows m with ids_keep[m] = l of g[m, e]
//
// All three are one product of two matrices with few results and a long sum (768 x 768 over 200 k rows): g^T times the
// rows of `visible`, and g^T times a matrix that is 1 at column ids_keep[m] of row m, which is made in LDS and never
// exists in memory; grad_bias is the sum of grad_pos, or without that a single column of ones (by positions always, so that
// it has the same bits with and without grad_pos, weight and bias alone take 22 % longer at 21,312 rows, 588 -> 1024, 256
// patches, 2 % at the headline batch, and several times as long with thousands of patches).  Both operands lie with the
// sum's index as their row number and are multiplied as they lie (matmul.hpp, "across k").  The products are exact, sums
// fp32.  The sum's index is split over the compute units; a second kernel adds the parts in a fixed order.
//
// (Sorting the rows by their index and adding up the rows of each took seven launches and 181 us beside 208 for the
// weight, 200,704 rows, 768 -> 768, 196 patches; as columns of the product they cost a third more tiles.)
#include "mae_device.hpp"
#include "mae_kernels.hpp"
#include "matmul.hpp"

namespace mae {

namespace {

using namespace mm;

constexpr int kThreads = 256;

// What a pass over rows that are not all finite takes in place of g: a count of +infinity and NaN, of -infinity and NaN, or
// what is finite.
enum Filter { kUp, kDown, kFinite };
__device__ inline u32x4 filtered(u32x4 v, int filter) {
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    uint32_t out = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t x = v[w] >> (16 * h) & 0xFFFFu, size = x & 0x7FFFu;
      const bool counts = size > 0x7F80u || x == (filter == kUp ? 0x7F80u : 0xFF80u);
      out |= (filter == kFinite ? (size < 0x7F80u ? x : 0u) : counts ? 0x3F80u : 0u) << (16 * h);
    }
    v[w] = out;
  }
  return v;
}

// Part s of the sums: weight_acc[s][e][d], pos_acc[s][e][l].
// In a product with zeros an infinity of one position is a NaN in all others (0 * inf).  That is how it is noticed: then the
// tile is made again from the finite values, and infinities and NaN are added to the sums of their own positions (three
// passes without loads in flight: 200,704 rows of NaN, 768 -> 768, 2.3 ms instead of 0.27; nothing where all is finite).
template <int TM, int TN, int WGM, int WGN>
__global__ __launch_bounds__(64 * WGM * WGN) void embed_products_kernel(EmbedGradArgs a) {
  using T = Tile<TM, TN, WGM, WGN, false, false>;
  __shared__ __attribute__((aligned(1024))) u32x4 lds[T::kLdsBytes / 16];
  const int tiles_d = a.grad_weight ? (a.D + T::BN - 1) / T::BN : 0;
  const int tiles_l = a.pos_columns ? (a.pos_columns + T::BN - 1) / T::BN : 0;
  const uint32_t tiles_n = (uint32_t)(tiles_d + tiles_l), tiles = tiles_n * (uint32_t)((a.E + T::BM - 1) / T::BM);
  const uint32_t id = xcd_remap(blockIdx.x, gridDim.x);
  const uint32_t part = id / tiles, tile = id - part * tiles;
  const int tm = (int)(tile / tiles_n), tn = (int)(tile - (uint32_t)tm * tiles_n);
  const int m0 = tm * T::BM, rows_m = min(T::BM, a.E - m0);
  // this part's share of the slices
  const int K = (int)a.K, slices = (K + kSlice - 1) / kSlice, share = (slices + a.parts - 1) / a.parts;
  const int s0 = uniform(min((int)part * share, slices)), s1 = uniform(min(s0 + share, slices));
  const int64_t k0 = (int64_t)s0 * kSlice;
  const int depth = uniform(min(s1 * kSlice, K) - min(s0 * kSlice, K));
  const Operand A{a.g + k0 * a.ld + m0, a.ld, rows_m};
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int wm = wave / WGN, wn = wave % WGN;
  f32x16 acc[TM][TN];
  float* out;
  int ld, rows_n;
  if (tn < tiles_d) {
    const int n0 = tn * T::BN;
    rows_n = min(T::BN, a.D - n0);
    const Operand B{a.visible + k0 * a.D + n0, a.D, rows_n};
    T::template run<0>(T::source(A, B, depth), lds, acc);
    ld = a.D;
    out = a.weight_acc + ((int64_t)part * a.E + m0) * ld + n0;
  } else {
    const int n0 = (tn - tiles_d) * T::BN;
    rows_n = min(T::BN, a.pos_columns - n0);
    const typename T::Ones ones{a.ids ? a.ids + k0 : nullptr, n0, a.pos_columns};
    T::template run<0, true>(T::source(A, A, depth), lds, acc, ones);
    ld = a.pos_columns;
    out = a.pos_acc + ((int64_t)part * a.E + m0) * ld + n0;
    if (a.ids) {  // (without, every row has its 1 in the one column that is used)
      bool nan = false;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) nan |= acc[i][j][e] != acc[i][j][e];
      uint32_t* seen = reinterpret_cast<uint32_t*>(lds);
      __syncthreads();  // every wavefront is done with the ring
      const bool any = __any(nan) != 0;
      if (lane == 0) seen[wave] = any ? 1u : 0u;
      __syncthreads();
      uint32_t found = 0;
#pragma unroll
      for (int w = 0; w < WGM * WGN; ++w) found |= seen[w];
      if (uniform((int)found) != 0) {
        constexpr int kSums = TM * TN * 16, kWords = (kSums + 31) / 32;
        uint32_t up[kWords] = {}, down[kWords] = {};  // a bit per sum of this lane
        __syncthreads();
#pragma unroll 1
        for (int filter = kUp; filter <= kFinite; ++filter) {
          T::run_filtered(A, depth, lds, acc, ones, [&](u32x4 v) { return filtered(v, filter); });
#pragma unroll
          for (int n = 0; n < kSums; ++n) {
            const uint32_t bit = acc[n / 16 / TN][n / 16 % TN][n % 16] > 0.f ? 1u << (n % 32) : 0u;
            if (filter == kUp) up[n / 32] |= bit;
            if (filter == kDown) down[n / 32] |= bit;
          }
        }
#pragma unroll
        for (int n = 0; n < kSums; ++n) {
          float sum = acc[n / 16 / TN][n / 16 % TN][n % 16];
          if (up[n / 32] >> (n % 32) & 1u) sum += __builtin_inff();
          if (down[n / 32] >> (n % 32) & 1u) sum -= __builtin_inff();
          acc[n / 16 / TN][n / 16 % TN][n % 16] = sum;
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const int r = wm * 32 * TM + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
      if (r >= rows_m) continue;
#pragma unroll
      for (int j = 0; j < TN; ++j) {
        const int c = wn * 32 * TN + 32 * j + (lane & 31);
        if (c < rows_n) out[(int64_t)r * ld + c] = acc[i][j][e];
      }
    }
}

// The parts joined.  Where the rows do not begin on 16-byte boundaries the product kernel, which reads whole chunks of
// 8 columns, ends one row earlier, and the last row's products are added here.
// Workgroups [0, for_pos): grad_pos and grad_bias, a wavefront per column e of g.  The rest: grad_weight, four values per lane.
__global__ __launch_bounds__(kThreads) void embed_join_kernel(EmbedGradArgs a, uint32_t for_pos) {
  if (blockIdx.x < for_pos) {
    const int lane = threadIdx.x % kWave;
    const int e = (int)blockIdx.x * (kThreads / kWave) + (int)threadIdx.x / kWave;
    if (e >= a.E) return;
    const int64_t stride = (int64_t)a.E * a.pos_columns;
    const bool rest = a.K < a.M;
    const float g = rest ? __uint_as_float((uint32_t)a.g[a.K * a.ld + e] << 16) : 0.f;
    const int id = rest && a.ids ? min(max(a.ids[a.K], 0), a.pos_columns - 1) : 0;
    double bias = 0.0;
    for (int l = lane; l < a.pos_columns; l += kWave) {
      const float* p = a.pos_acc + (int64_t)e * a.pos_columns + l;
      float s = rest && id == l ? g : 0.f;
#pragma unroll 8
      for (int k = 0; k < a.parts; ++k) s += p[k * stride];
      if (a.grad_pos) a.grad_pos[(int64_t)l * a.E + e] = s;
      bias += (double)s;
    }
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1) bias += __shfl_xor(bias, off, kWave);
    if (a.grad_bias && lane == 0) a.grad_bias[e] = (float)bias;
    return;
  }
  const int64_t total = (int64_t)a.E * a.D / 4, stride = (int64_t)a.E * a.D;
  for (int64_t i = (int64_t)(blockIdx.x - for_pos) * kThreads + threadIdx.x; i < total;
       i += (int64_t)(gridDim.x - for_pos) * kThreads) {
    f32x4 s = *reinterpret_cast<const f32x4*>(a.weight_acc + i * 4);
#pragma unroll 8
    for (int k = 1; k < a.parts; ++k) s += *reinterpret_cast<const f32x4*>(a.weight_acc + k * stride + i * 4);
    if (a.K < a.M) {
      const int64_t e = i * 4 / a.D, d = i * 4 - e * a.D;
      const float g = __uint_as_float((uint32_t)a.g[a.K * a.ld + e] << 16);
      const u32x2 v = *reinterpret_cast<const u32x2*>(a.visible + a.K * a.D + d);
      s += g * f32x4{bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)};
    }
    *reinterpret_cast<f32x4*>(a.grad_weight + i * 4) = s;
  }
}

// g with rows of ld = E rounded up to 8 values, for an E that is no multiple of 4
__global__ __launch_bounds__(kThreads) void embed_pad_kernel(EmbedGradArgs a, const uint16_t* src, uint16_t* dst) {
  const int64_t total = a.M * a.ld;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
    const int64_t r = i / a.ld, c = i - r * a.ld;
    dst[i] = c < a.E ? src[r * a.E + c] : (uint16_t)0;
  }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

int64_t tiles_of(int side, int E, int weight_columns, int pos_columns) {
  return ceil_div(E, side) * (ceil_div(weight_columns, side) + ceil_div(pos_columns, side));
}

template <int TM, int TN, int WGM, int WGN>
void launch_products(const EmbedGradArgs& a, uint32_t blocks, hipStream_t stream) {
  hipLaunchKernelGGL((embed_products_kernel<TM, TN, WGM, WGN>), dim3(blocks), dim3(64 * WGM * WGN), 0, stream, a);
}

}  // namespace

EmbedGradPlan embed_grad_plan(int64_t M, int D, int E, int L) {
  EmbedGradPlan p{};
  p.ld = E % 4 == 0 ? E : (int)ceil_div(E, 8) * 8;
  p.K = p.ld % 8 != 0 || D % 8 != 0 ? M - 1 : M;
  // Side of the tiles by the number of products; as many parts as fill the compute units, of four slices at least.
  // us for tiles of 64 / 128 / 256, 768 -> 768, 196 patches: 784 rows 14.4 / 19.5 / 31, 1568 17.4 / 21.3 / 32, 3136
  // 23.4 / 24.0 / 33, 6272 30.0 / 26.3 / 37.4, 12544 44.8 / 35.4 / 43.2, 25088 73 / 54.7 / 55.2, 50176 130 / 93 / 83,
  // 200704 - / 347 / 271; 192 -> 384, 100 patches: 50000 rows 30.6 / 28.3 / 38; 192 -> 192: 8192 rows 12.2 / 14.1 / 21
  const int64_t work = M * E * (D + L);
  p.side = work < 2300000000 ? 64 : work < 19000000000 ? 128 : 256;
  const int64_t tiles = tiles_of(p.side, E, D, L);
  int64_t parts = (p.side == 256 ? 256 : 512) / tiles;
  if (parts > ceil_div(p.K, kSlice) / 4) parts = ceil_div(p.K, kSlice) / 4;
  p.parts = (int)(parts < 1 ? 1 : parts);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t was = at;
    at += up256(bytes);
    return was;
  };
  p.padded = take(p.ld != E ? (size_t)M * p.ld * 2 : 0);
  p.weight_acc = take((size_t)p.parts * E * D * 4);
  p.pos_acc = take((size_t)p.parts * E * L * 4);
  p.bytes = at;
  return p;
}

hipError_t launch_embed_grad(EmbedGradArgs a, const EmbedGradPlan& p, uint16_t* padded, hipStream_t stream) {
  a.ld = p.ld;
  a.K = p.K;
  a.parts = p.parts;
  if (p.ld != a.E) {
    const int64_t blocks = ceil_div(a.M * p.ld, kThreads);
    hipLaunchKernelGGL(embed_pad_kernel, dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), dim3(kThreads), 0, stream, a,
                       a.g, padded);
    a.g = padded;
  }
  const uint32_t blocks = (uint32_t)(tiles_of(p.side, a.E, a.grad_weight ? a.D : 0, a.pos_columns) * p.parts);
  if (p.side == 256) launch_products<4, 2, 2, 4>(a, blocks, stream);
  else if (p.side == 128) launch_products<2, 1, 2, 4>(a, blocks, stream);
  else launch_products<1, 1, 2, 2>(a, blocks, stream);
  const uint32_t for_pos = a.pos_columns ? (uint32_t)ceil_div(a.E, kThreads / kWave) : 0;
  const int64_t for_weight = a.grad_weight ? ceil_div((int64_t)a.E * a.D / 4, kThreads) : 0;
  hipLaunchKernelGGL(embed_join_kernel, dim3(for_pos + (uint32_t)(for_weight < 4096 ? for_weight : 4096)), dim3(kThreads), 0,
                     stream, a, for_pos);
  return hipGetLastError();
}

}  // namespace mae

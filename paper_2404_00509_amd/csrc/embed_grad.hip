// Gradients of the patch embedding of the visible tokens: with g = the gradient of the tokens [M, E],
//   grad_weight[e, d] = sum over m of g[m, e] visible[m, d]
//   grad_bias[e]      = sum over m of g[m, e]
//   grad_pos[l, e]    = sum over the rows m with ids_keep[m] = l of g[m, e]
//
// grad_weight is a product of two matrices with few results and a long sum (768 x 768 over 200 k rows):
// both operands lie with the sum's index as their row number and are multiplied as they lie (matmul.hpp,
// "across k"); k is split over the compute units, the parts are added in a fixed order.
// grad_pos: rows are sorted by their patch index (counting sort, stable, so that every sum has one order and
// nothing depends on scheduling), then the rows of an index are added up by several workgroups whose parts are
// joined.  grad_bias is the sum of all those parts.  Every gradient row is read once more for it.
#include "mae_device.hpp"
#include "mae_kernels.hpp"
#include "matmul.hpp"

namespace mae {

namespace {

using namespace mm;

constexpr int kThreads = 256;

__device__ inline int clamp_id(int id, int L) { return min(max(id, 0), L - 1); }

// ---- rows by patch index ---------------------------------------------------------------------------
// counts[chunk][l]: rows of the chunk with index l
__global__ __launch_bounds__(kThreads) void embed_count_kernel(EmbedGradArgs a) {
  extern __shared__ int32_t hist[];
  for (int l = threadIdx.x; l < a.L; l += kThreads) hist[l] = 0;
  __syncthreads();
  const int64_t from = (int64_t)blockIdx.x * a.chunk_rows, to = min(from + a.chunk_rows, a.M);
  for (int64_t r = from + threadIdx.x; r < to; r += kThreads) atomicAdd(&hist[clamp_id(a.ids[r], a.L)], 1);
  __syncthreads();
  for (int l = threadIdx.x; l < a.L; l += kThreads) a.counts[(int64_t)blockIdx.x * a.L + l] = hist[l];
}

// counts[chunk][l] -> rows with index l in earlier chunks; totals[l] -> their number
__global__ __launch_bounds__(kThreads) void embed_chunks_kernel(EmbedGradArgs a) {
  const int l = blockIdx.x * kThreads + threadIdx.x;
  if (l >= a.L) return;
  constexpr int kBatch = 16;  // loads in flight
  int32_t s = 0;
  for (int c0 = 0; c0 < a.chunks; c0 += kBatch) {
    int32_t n[kBatch];
#pragma unroll
    for (int c = 0; c < kBatch; ++c) n[c] = c0 + c < a.chunks ? a.counts[(int64_t)(c0 + c) * a.L + l] : 0;
#pragma unroll
    for (int c = 0; c < kBatch; ++c) {
      if (c0 + c < a.chunks) a.counts[(int64_t)(c0 + c) * a.L + l] = s;
      s += n[c];
    }
  }
  a.starts[l + 1] = s;  // (turned into starts by the next kernel)
}

// starts[0 .. L]: prefix sums of the totals, by one workgroup
__global__ __launch_bounds__(kThreads) void embed_starts_kernel(EmbedGradArgs a) {
  __shared__ int32_t wave_sum[kThreads / kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int32_t carry = 0;
  for (int base = 0; base < a.L; base += kThreads) {
    const int l = base + threadIdx.x;
    int32_t v = l < a.L ? a.starts[l + 1] : 0;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
      const int32_t up = __shfl_up(v, off, kWave);
      if (lane >= off) v += up;
    }
    if (lane == kWave - 1) wave_sum[wave] = v;
    __syncthreads();
    int32_t before = carry;
    for (int w = 0; w < wave; ++w) before += wave_sum[w];
    for (int w = 0; w < kThreads / kWave; ++w) carry += wave_sum[w];
    if (l < a.L) a.starts[l + 1] = before + v;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.starts[0] = 0;
}

// order[starts[l] + k]: the k-th row with index l
__global__ __launch_bounds__(kThreads) void embed_order_kernel(EmbedGradArgs a) {
  extern __shared__ int32_t next[];  // [L], then the ids of kThreads rows
  int32_t* id_of = next + a.L;
  for (int l = threadIdx.x; l < a.L; l += kThreads)
    next[l] = a.starts[l] + a.counts[(int64_t)blockIdx.x * a.L + l];
  const int64_t from = (int64_t)blockIdx.x * a.chunk_rows, to = min(from + a.chunk_rows, a.M);
  for (int64_t base = from; base < to; base += kThreads) {
    const int64_t r = base + threadIdx.x;
    const int n = (int)min((int64_t)kThreads, to - base);
    const int id = r < to ? clamp_id(a.ids[r], a.L) : -1;
    __syncthreads();
    id_of[threadIdx.x] = id;
    __syncthreads();
    int rank = 0, same = 0;  // rows with this index in front of this one, and in all
    for (int k = 0; k < n; ++k) {
      const bool eq = id_of[k] == id;
      same += eq ? 1 : 0;
      rank += eq && k < (int)threadIdx.x ? 1 : 0;
    }
    if (r < to) a.order[next[id] + rank] = (int32_t)r;
    __syncthreads();
    if (r < to && rank == same - 1) next[id] += same;  // the last of them
  }
}

// parts[l][share][e]: sums over a share of the rows with index l; 256 columns per workgroup, four per
// lane, rows in turn by the four wavefronts
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(EmbedGradArgs a) {
  __shared__ f32x4 sums[kThreads / kWave][kWave];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int share = blockIdx.x % a.shares, l = blockIdx.x / a.shares;
  const int c = blockIdx.y * 256 + 4 * lane;
  const int64_t first = a.order ? a.starts[l] : 0, end = a.order ? a.starts[l + 1] : a.M;
  const int64_t per = (end - first + a.shares - 1) / a.shares;
  const int64_t from = first + share * per, to = min(from + per, end);
  const bool in = c < a.ld;  // (ld is a multiple of 4)
  f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int64_t k = from + wave; k < to; k += 4 * 4) {
    u32x2 raw[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      raw[u] = u32x2{0u, 0u};
      const int64_t at = k + 4 * u;
      if (at < to && in) {
        const int64_t row = a.order ? (int64_t)a.order[at] : at;
        raw[u] = *reinterpret_cast<const u32x2*>(a.g + row * a.ld + c);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      s += f32x4{bf16_lo(raw[u].x), bf16_hi(raw[u].x), bf16_lo(raw[u].y), bf16_hi(raw[u].y)};
  }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && in) {
    s = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    *reinterpret_cast<f32x4*>(a.pos_parts + ((int64_t)l * a.shares + share) * a.ld + c) = s;
  }
}

// grad_pos: the shares of an index joined
__global__ __launch_bounds__(kThreads) void embed_pos_kernel(EmbedGradArgs a) {
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= (int64_t)a.L * a.E) return;
  const int l = (int)(i / a.E), e = (int)(i - (int64_t)l * a.E);
  double s = 0.0;
  for (int k = 0; k < a.shares; ++k) s += (double)a.pos_parts[((int64_t)l * a.shares + k) * a.ld + e];
  a.grad_pos[i] = (float)s;
}

// grad_bias: all parts joined, 16 columns by 16 lanes
__global__ __launch_bounds__(kThreads) void embed_bias_kernel(EmbedGradArgs a) {
  __shared__ double part[16][17];
  const int col = threadIdx.x % 16, r = threadIdx.x / 16;
  const int e = blockIdx.x * 16 + col;
  double s = 0.0;
  if (e < a.E)
    for (int64_t k = r; k < (int64_t)a.L * a.shares; k += 16) s += (double)a.pos_parts[k * a.ld + e];
  part[r][col] = s;
  __syncthreads();
  if (r == 0 && e < a.E) {
    for (int k = 1; k < 16; ++k) s += part[k][col];
    a.grad_bias[e] = (float)s;
  }
}

// grad_weight: the parts of the split joined, and the last row's products where the rows do not begin on
// 16-byte boundaries (the product kernel reads whole chunks of 8 columns, so it ends one row earlier)
__global__ __launch_bounds__(kThreads) void embed_weight_kernel(EmbedGradArgs a) {
  const int64_t total = (int64_t)a.E * a.D / 4, stride = (int64_t)a.E * a.D;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
    f32x4 s = *reinterpret_cast<const f32x4*>(a.weight_acc + i * 4);
    for (int k = 1; k < a.parts; ++k) s += *reinterpret_cast<const f32x4*>(a.weight_acc + k * stride + i * 4);
    if (a.last_row) {
      const int64_t e = i * 4 / a.D, d = i * 4 - e * a.D;
      const float g = __uint_as_float((uint32_t)a.g[(a.M - 1) * a.ld + e] << 16);
      const u32x2 v = *reinterpret_cast<const u32x2*>(a.visible + (a.M - 1) * a.D + d);
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

}  // namespace

EmbedGradPlan embed_grad_plan(int64_t M, int D, int E, int L, bool by_index) {
  EmbedGradPlan p;
  p.ld = E % 4 == 0 ? E : (int)ceil_div(E, 8) * 8;
  p.last_row = p.ld % 8 != 0 || D % 8 != 0;
  p.rows = by_index ? L : 1;
  p.side = matmul_side(E, D);
  p.parts = matmul_parts(E, D, M, p.side);
  p.chunk_rows = (int)ceil_div(ceil_div(M, 256), kThreads) * kThreads;
  p.chunks = (int)ceil_div(M, p.chunk_rows);
  const int64_t tasks = (int64_t)p.rows * ceil_div(p.ld, 256);
  int64_t shares = ceil_div(4096, tasks);
  if (shares > ceil_div(M, (int64_t)p.rows * 16)) shares = ceil_div(M, (int64_t)p.rows * 16);
  p.shares = (int)(shares < 1 ? 1 : shares);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t was = at;
    at += up256(bytes);
    return was;
  };
  p.padded = take(p.ld != E ? (size_t)M * p.ld * 2 : 0);
  p.counts = take(by_index ? (size_t)p.chunks * L * 4 : 0);
  p.starts = take(by_index ? (size_t)(L + 1) * 4 : 0);
  p.order = take(by_index ? (size_t)M * 4 : 0);
  p.pos_parts = take((size_t)p.rows * p.shares * p.ld * 4);
  p.weight_acc = take((size_t)p.parts * E * D * 4);
  p.bytes = at;
  return p;
}

hipError_t launch_embed_grad(EmbedGradArgs a, const EmbedGradPlan& p, uint16_t* padded, hipStream_t stream) {
  a.ld = p.ld;
  a.parts = p.parts;
  a.shares = p.shares;
  a.chunks = p.chunks;
  a.chunk_rows = p.chunk_rows;
  a.last_row = p.last_row;
  const dim3 block(kThreads);
  if (p.ld != a.E) {
    const int64_t blocks = ceil_div(a.M * p.ld, kThreads);
    hipLaunchKernelGGL(embed_pad_kernel, dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), block, 0, stream, a, a.g,
                       padded);
    a.g = padded;
  }
  if (a.grad_weight) {
    MatmulArgs m{};
    m.A = a.g, m.lda = p.ld, m.B = a.visible, m.ldb = a.D;
    m.M = a.E, m.N = a.D, m.K = p.last_row ? a.M - 1 : a.M;
    m.out = a.weight_acc, m.parts = p.parts;
    hipError_t e = launch_matmul(m, MatmulKind::kBf16Across, p.side, stream);
    if (e != hipSuccess) return e;
    const int64_t blocks = ceil_div((int64_t)a.E * a.D / 4, kThreads);
    hipLaunchKernelGGL(embed_weight_kernel, dim3((uint32_t)(blocks < 65536 ? blocks : 65536)), block, 0, stream, a);
  }
  if (a.grad_pos || a.grad_bias) {
    a.L = p.rows;
    if (a.order) {
      const size_t bins = (size_t)a.L * sizeof(int32_t);
      hipLaunchKernelGGL(embed_count_kernel, dim3((uint32_t)a.chunks), block, bins, stream, a);
      hipLaunchKernelGGL(embed_chunks_kernel, dim3((uint32_t)ceil_div(a.L, kThreads)), block, 0, stream, a);
      hipLaunchKernelGGL(embed_starts_kernel, dim3(1), block, 0, stream, a);
      hipLaunchKernelGGL(embed_order_kernel, dim3((uint32_t)a.chunks), block, bins + kThreads * sizeof(int32_t), stream,
                         a);
    }
    hipLaunchKernelGGL(embed_sum_kernel, dim3((uint32_t)(a.L * a.shares), (uint32_t)ceil_div(a.ld, 256)), block, 0,
                       stream, a);
    if (a.grad_pos)
      hipLaunchKernelGGL(embed_pos_kernel, dim3((uint32_t)ceil_div((int64_t)a.L * a.E, kThreads)), block, 0, stream, a);
    if (a.grad_bias)
      hipLaunchKernelGGL(embed_bias_kernel, dim3((uint32_t)ceil_div(a.E, 16)), block, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace mae

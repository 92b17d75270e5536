// Layer norm of token rows, forward and backward (Sec. 2, Sec. 5: the ViT encoder that works on the
// embedded tokens begins and ends its blocks with it).
//
//   h = (x - mean) rstd, rstd = 1 / sqrt(mean((x - mean)^2) + eps);  y = h w + b
//   grad_x = rstd (g - mean(g) - h mean(g h)) with g = grad_y w
//   grad_w = sum over rows of grad_y h;  grad_b = sum over rows of grad_y
//
// Bound by HBM: every value is read once and written once.  A row lies in the registers of 16 lanes
// (up to 64 values), of a wavefront (up to 2048) or of a workgroup (up to 8192), four neighbouring
// values per lane and step, so that mean and variance take two passes over registers instead of memory:
// no difference of two large sums, as one pass with sums of squares would have.  A
// wavefront takes rows in turn and keeps weight, bias and its share of their gradients in
// registers; the shares of a workgroup are added through LDS, those of the workgroups by a second
// kernel in a fixed order, in double precision, so results do not depend on scheduling.
#include "mae_device.hpp"
#include "mae_kernels.hpp"

namespace mae {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// rows that are no multiple of four values start at any multiple of the value's size
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));

constexpr int kThreads = 256;

// Four values, the first n of them where n < 4 (zeros behind).
template <bool kBf16>
__device__ inline f32x4 load4(const void* p, int64_t at, int n) {
  f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
  if (n >= 4) {
    if (kBf16) {
      const u32x2 raw = *reinterpret_cast<const u32x2_a2*>(static_cast<const uint16_t*>(p) + at);
      return f32x4{bf16_lo(raw.x), bf16_hi(raw.x), bf16_lo(raw.y), bf16_hi(raw.y)};
    }
    return *reinterpret_cast<const f32x4_a4*>(static_cast<const float*>(p) + at);
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < n)
      v[j] = kBf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at + j] << 16)
                   : static_cast<const float*>(p)[at + j];
  return v;
}
template <bool kBf16>
__device__ inline void store4(void* p, int64_t at, f32x4 v, int n) {
  if (n >= 4) {
    if (kBf16)
      *reinterpret_cast<u32x2_a2*>(static_cast<uint16_t*>(p) + at) =
          u32x2{pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w)};
    else
      *reinterpret_cast<f32x4_a4*>(static_cast<float*>(p) + at) = v;
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j)
    if (j < n) {
      if (kBf16) static_cast<uint16_t*>(p)[at + j] = (uint16_t)bf16_rne(v[j]);
      else static_cast<float*>(p)[at + j] = v[j];
    }
}

__device__ inline float sum4(f32x4 v) { return (v.x + v.y) + (v.z + v.w); }

// Sum over the kLanes lanes that hold a row; `slots`: 4 floats of LDS per use for rows of a workgroup.
template <int kLanes>
__device__ inline float row_sum(float v, float* slots) {
#pragma unroll
  for (int off = (kLanes < kWave ? kLanes : kWave) / 2; off > 0; off >>= 1) v += __shfl_xor(v, off, kWave);
  if constexpr (kLanes > kWave) {
    if (threadIdx.x % kWave == 0) slots[threadIdx.x / kWave] = v;
    __syncthreads();
    v = (slots[0] + slots[1]) + (slots[2] + slots[3]);
  }
  return v;
}

// NV: groups of four values per lane.
template <int kLanes, int NV, bool kBf16In, bool kBf16Out>
__global__ __launch_bounds__(kThreads) void layer_norm_kernel(NormArgs a) {
  constexpr int kRows = kThreads / kLanes;  // rows of a workgroup at a time
  __shared__ float slots[2][2][4];
  const int lane = threadIdx.x % kLanes;
  const int D = a.D;
  const float count = (float)D;
  f32x4 w[NV], b[NV];
  int n[NV];  // values of each group that exist
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = 4 * (lane + v * kLanes);
    n[v] = min(4, D - c);
    w[v] = f32x4{1.f, 1.f, 1.f, 1.f};
    b[v] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (a.weight && n[v] > 0) w[v] = load4<false>(a.weight, c, n[v]);
    if (a.bias && n[v] > 0) b[v] = load4<false>(a.bias, c, n[v]);
  }
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.M; row0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = row0 + threadIdx.x / kLanes;
    const bool live = row < a.M;
    const int64_t at = row * D;
    f32x4 x[NV];
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      x[v] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (live && n[v] > 0) x[v] = load4<kBf16In>(a.x, at + 4 * (lane + v * kLanes), n[v]);
      s += sum4(x[v]);
    }
    const float mean = row_sum<kLanes>(s, slots[turn][0]) / count;
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[v][j] = j < n[v] ? x[v][j] - mean : 0.f;
      ss += (x[v].x * x[v].x + x[v].y * x[v].y) + (x[v].z * x[v].z + x[v].w * x[v].w);
    }
    const float rstd = 1.0f / sqrtf(row_sum<kLanes>(ss, slots[turn][1]) / count + a.eps);
    turn ^= 1;
    if (!live) continue;
    if (lane == 0) {
      if (a.mean_out) a.mean_out[row] = mean;
      if (a.rstd_out) a.rstd_out[row] = rstd;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (n[v] > 0)
        store4<kBf16Out>(a.y, at + 4 * (lane + v * kLanes), x[v] * rstd * w[v] + b[v], n[v]);
  }
}

// kParams: the gradients of weight and bias are wanted.
template <int kLanes, int NV, bool kBf16In, bool kBf16Out, bool kParams>
__global__ __launch_bounds__(kThreads) void layer_norm_grad_kernel(NormArgs a) {
  constexpr int kRows = kThreads / kLanes;
  __shared__ float slots[2][2][4];
  __shared__ f32x4 shares[kParams && kLanes <= kWave ? kThreads / kWave : 1][2 * kWave];
  const int lane = threadIdx.x % kLanes;
  const int D = a.D;
  const float count = (float)D;
  f32x4 w[NV], gw[NV], gb[NV];
  int n[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = 4 * (lane + v * kLanes);
    n[v] = min(4, D - c);
    w[v] = f32x4{1.f, 1.f, 1.f, 1.f};
    gw[v] = gb[v] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (a.weight && n[v] > 0) w[v] = load4<false>(a.weight, c, n[v]);
  }
  int turn = 0;
  for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.M; row0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = row0 + threadIdx.x / kLanes;
    const bool live = row < a.M;
    const int64_t at = row * D;
    const float mean = live ? a.mean[row] : 0.f, rstd = live ? a.rstd[row] : 0.f;
    f32x4 h[NV], g[NV];
    float s = 0.f, sh = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      h[v] = g[v] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (live && n[v] > 0) {
        const int64_t e = at + 4 * (lane + v * kLanes);
        h[v] = load4<kBf16In>(a.x, e, n[v]);
        g[v] = load4<kBf16Out>(a.grad_y, e, n[v]);
      }
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      h[v] = (h[v] - mean) * rstd;
      if (kParams) {  // (groups' values that do not exist hold a zero gradient)
        gw[v] += g[v] * h[v];
        gb[v] += g[v];
      }
      g[v] *= w[v];
      s += sum4(g[v]);
      sh += sum4(g[v] * h[v]);
    }
    const float mg = row_sum<kLanes>(s, slots[turn][0]) / count;
    const float mgh = row_sum<kLanes>(sh, slots[turn][1]) / count;
    turn ^= 1;
    if (!live || !a.grad_x) continue;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (n[v] > 0)
        store4<kBf16In>(a.grad_x, at + 4 * (lane + v * kLanes), (g[v] - mg - h[v] * mgh) * rstd, n[v]);
  }
  if constexpr (kParams) {
    // the workgroup's sums: [gridDim.x][2][D rounded up to 4]
    float* out = a.partials + (int64_t)blockIdx.x * 2 * a.padded;
    if constexpr (kLanes > kWave) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = 4 * (lane + v * kLanes);
        if (n[v] > 0) {
          *reinterpret_cast<f32x4*>(out + c) = gw[v];
          *reinterpret_cast<f32x4*>(out + a.padded + c) = gb[v];
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int off = kLanes; off < kWave; off <<= 1) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            gw[v][j] += __shfl_xor(gw[v][j], off, kWave);
            gb[v][j] += __shfl_xor(gb[v][j], off, kWave);
          }
        }
        const int wave = threadIdx.x / kWave, l = threadIdx.x % kWave;
        __syncthreads();
        shares[wave][l] = gw[v];
        shares[wave][kWave + l] = gb[v];
        __syncthreads();
        if (threadIdx.x < 2 * kWave && l < kLanes) {
          const f32x4 sum = (shares[0][threadIdx.x] + shares[1][threadIdx.x]) +
                            (shares[2][threadIdx.x] + shares[3][threadIdx.x]);
          const int c = 4 * (l + v * kLanes);
          if (c < D) *reinterpret_cast<f32x4*>(out + (threadIdx.x / kWave) * a.padded + c) = sum;
        }
      }
    }
  }
}

// Sum of the workgroups' shares: 16 columns by 16 lanes each.
__global__ __launch_bounds__(kThreads) void layer_norm_params_kernel(NormArgs a) {
  __shared__ double part[16][17];
  const int col = threadIdx.x % 16, r = threadIdx.x / 16;
  const int c = blockIdx.x * 16 + col;  // of the 2 * padded columns
  double s = 0.0;
  if (c < 2 * a.padded)
    for (int p = r; p < a.num_partials; p += 16) s += (double)a.partials[(int64_t)p * 2 * a.padded + c];
  part[r][col] = s;
  __syncthreads();
  if (r == 0 && c < 2 * a.padded) {
    for (int k = 1; k < 16; ++k) s += part[k][col];
    const int d = c < a.padded ? c : c - a.padded;
    float* out = c < a.padded ? a.grad_weight : a.grad_bias;
    if (out && d < a.D) out[d] = (float)s;
  }
}

template <int kLanes, int NV>
void launch_forward(const NormArgs& a, int blocks, hipStream_t stream) {
  const dim3 grid(blocks), block(kThreads);
  if (a.x_bf16) {
    if (a.y_bf16) hipLaunchKernelGGL((layer_norm_kernel<kLanes, NV, true, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((layer_norm_kernel<kLanes, NV, true, false>), grid, block, 0, stream, a);
  } else {
    if (a.y_bf16) hipLaunchKernelGGL((layer_norm_kernel<kLanes, NV, false, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((layer_norm_kernel<kLanes, NV, false, false>), grid, block, 0, stream, a);
  }
}

template <int kLanes, int NV, bool kParams>
void launch_backward(const NormArgs& a, int blocks, hipStream_t stream) {
  const dim3 grid(blocks), block(kThreads);
  if (a.x_bf16) {
    if (a.y_bf16)
      hipLaunchKernelGGL((layer_norm_grad_kernel<kLanes, NV, true, true, kParams>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((layer_norm_grad_kernel<kLanes, NV, true, false, kParams>), grid, block, 0, stream, a);
  } else {
    if (a.y_bf16)
      hipLaunchKernelGGL((layer_norm_grad_kernel<kLanes, NV, false, true, kParams>), grid, block, 0, stream, a);
    else
      hipLaunchKernelGGL((layer_norm_grad_kernel<kLanes, NV, false, false, kParams>), grid, block, 0, stream, a);
  }
}

// lanes per row
int norm_lanes(int D) { return D <= 64 ? 16 : D <= 2048 ? 64 : 256; }

template <int kLanes, int NV>
void launch_either(const NormArgs& a, int blocks, bool grad, hipStream_t stream) {
  if (!grad) launch_forward<kLanes, NV>(a, blocks, stream);
  else if (a.partials) launch_backward<kLanes, NV, true>(a, blocks, stream);
  else launch_backward<kLanes, NV, false>(a, blocks, stream);
}

void launch_sized(const NormArgs& a, int blocks, bool grad, hipStream_t stream) {
  const int groups = (a.D + 3) / 4;
  if (a.D <= 64) return launch_either<16, 1>(a, blocks, grad, stream);
  if (a.D <= 2048) {
    switch ((groups + 63) / 64) {
      case 1: return launch_either<64, 1>(a, blocks, grad, stream);
      case 2: return launch_either<64, 2>(a, blocks, grad, stream);
      case 3: return launch_either<64, 3>(a, blocks, grad, stream);
      case 4: return launch_either<64, 4>(a, blocks, grad, stream);
      case 5: return launch_either<64, 5>(a, blocks, grad, stream);
      case 6: return launch_either<64, 6>(a, blocks, grad, stream);
      default: return launch_either<64, 8>(a, blocks, grad, stream);
    }
  }
  switch ((groups + 255) / 256) {
    case 3: return launch_either<256, 3>(a, blocks, grad, stream);
    case 4: return launch_either<256, 4>(a, blocks, grad, stream);
    case 5:
    case 6: return launch_either<256, 6>(a, blocks, grad, stream);
    default: return launch_either<256, 8>(a, blocks, grad, stream);
  }
}

int norm_blocks(int64_t M, int D, int most) {
  const int rows = kThreads / norm_lanes(D);
  const int64_t blocks = (M + rows - 1) / rows;
  return (int)(blocks < most ? blocks : most);
}

}  // namespace

int norm_partials(int64_t M, int D) { return norm_blocks(M, D, 1024); }

hipError_t launch_layer_norm(const NormArgs& a, hipStream_t stream) {
  launch_sized(a, norm_blocks(a.M, a.D, 2048), false, stream);
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(const NormArgs& a, hipStream_t stream) {
  launch_sized(a, norm_blocks(a.M, a.D, 1024), true, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.partials) return e;
  hipLaunchKernelGGL(layer_norm_params_kernel, dim3((2 * a.padded + 15) / 16), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mae

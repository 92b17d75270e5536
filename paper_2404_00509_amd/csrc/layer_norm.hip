// Layer norm of token rows, forward and backward (Sec. 2, Sec. 5: the ViT encoder that works on the
// embedded tokens begins and ends its blocks with it).
//
//   h = (x - mean) rstd, rstd = 1 / sqrt(mean((x - mean)^2) + eps);  y = h w + b
//   grad_x = rstd (g - mean(g) - h mean(g h)) with g = grad_y w
//   grad_w = sum over rows of grad_y h;  grad_b = sum over rows of grad_y
//
// Bound by HBM: every value is read once and written once.  A row lies in the registers of 16 lanes (up to 384 values), a
// wavefront (1536) or a workgroup of 256 (6144) or 512 lanes, four neighbouring values per lane and step, so that mean and
// variance take two passes over registers instead of memory: no difference of two large sums, as one pass with sums of
// squares would have.  A group of lanes takes rows in turn, up to two at once, with the loads of the next ones on their way, and keeps
// weight, bias and its share of their gradients in registers; sums over lanes go through DPP moves, not LDS.  The
// shares of a workgroup are added through LDS, those of the workgroups by a second kernel in a fixed order, in double
// precision, so results do not depend on scheduling.
// 204,800 x 768 in bf16: forward 123 us (630 MB, 5.1 TB/s; 215 us without the loads ahead and with shuffles through LDS),
// backward 185 us (945 MB, 5.1 TB/s), 6 of them for the join; a copy of several GB runs at 4.7 TB/s on this card.
#include "mae_device.hpp"
#include "mae_kernels.hpp"

namespace mae {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// rows that are no multiple of four values start at any multiple of the value's size
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));

// Four values as they lie in memory.
template <bool kBf16>
struct Raw {
  using Type = f32x4;
};
template <>
struct Raw<true> {
  using Type = u32x2;
};

// The first n (none, or 1 to 4) of four values, zeros behind.
template <bool kBf16>
__device__ inline typename Raw<kBf16>::Type load4(const void* p, int64_t at, int n) {
  if constexpr (kBf16) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (n >= 4) return *reinterpret_cast<const u32x2_a2*>(q);
    u32x2 v = u32x2{0u, 0u};
    if (n > 0) v.x = q[0];
    if (n > 1) v.x |= (uint32_t)q[1] << 16;
    if (n > 2) v.y = q[2];
    return v;
  } else {
    const float* q = static_cast<const float*>(p) + at;
    if (n >= 4) return *reinterpret_cast<const f32x4_a4*>(q);
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
    if (n > 0) v.x = q[0];
    if (n > 1) v.y = q[1];
    if (n > 2) v.z = q[2];
    return v;
  }
}
__device__ inline f32x4 values(f32x4 v) { return v; }
__device__ inline f32x4 values(u32x2 v) { return f32x4{bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y)}; }

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

// v plus that of the lane `kBy` places further round in its group of 16: no trip through LDS, as shuffles take.
template <int kBy>
__device__ inline float add_rotated(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 | kBy, 0xF, 0xF, true));
}
__device__ inline float lane_value(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}
// Sum over the kLanes lanes that hold a row; `slots`: kSlots floats of LDS per use for rows of a workgroup.
constexpr int kSlots = 8;
template <int kLanes>
__device__ inline float row_sum(float v, float* slots) {
  v = add_rotated<1>(add_rotated<2>(add_rotated<4>(add_rotated<8>(v))));
  if constexpr (kLanes >= kWave)
    v = (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
  if constexpr (kLanes > kWave) {
    if (threadIdx.x % kWave == 0) slots[threadIdx.x / kWave] = v;
    __syncthreads();
    v = (slots[0] + slots[1]) + (slots[2] + slots[3]);
    if constexpr (kLanes > 4 * kWave) v += (slots[4] + slots[5]) + (slots[6] + slots[7]);
  }
  return v;
}

// of a workgroup
template <int kLanes>
constexpr int threads() { return kLanes > 256 ? kLanes : 256; }
// Rows that a group of lanes has in hand at a time, beside as many whose loads are on their way.
template <int kLanes, int NV>
constexpr int rows_at_once() { return kLanes <= kWave && NV <= 3 ? 2 : 1; }

// NV: groups of four values per lane.
template <int kLanes, int NV, bool kBf16In, bool kBf16Out>
__global__ __launch_bounds__(threads<kLanes>()) void layer_norm_kernel(NormArgs a) {
  constexpr int R = rows_at_once<kLanes, NV>();
  constexpr int kThreads = threads<kLanes>();
  constexpr int kRows = kThreads / kLanes * R;  // of a workgroup at a time
  __shared__ float slots[2][2][kSlots];
  const int lane = threadIdx.x % kLanes;
  const int D = a.D;
  const float count = (float)D;
  f32x4 w[NV], b[NV];
  int n[NV];  // values of each group that exist
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = 4 * (lane + v * kLanes);
    n[v] = max(0, min(4, D - c));
    w[v] = f32x4{1.f, 1.f, 1.f, 1.f};
    b[v] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (a.weight) w[v] = load4<false>(a.weight, c, n[v]);
    if (a.bias) b[v] = load4<false>(a.bias, c, n[v]);
  }
  typename Raw<kBf16In>::Type next[R][NV];
  const auto load = [&](int64_t row0) {
#pragma unroll
    for (int u = 0; u < R; ++u)
#pragma unroll
      for (int v = 0; v < NV; ++v)
        next[u][v] = load4<kBf16In>(a.x, (row0 + u) * D + 4 * (lane + v * kLanes), row0 + u < a.M ? n[v] : 0);
  };
  int64_t row0 = (int64_t)blockIdx.x * kRows + (int)threadIdx.x / kLanes * R;
  const int64_t step = (int64_t)gridDim.x * kRows;
  load(row0);
  int turn = 0;
  // (rows of a workgroup: all lanes of it take the same number of turns)
  for (; row0 < a.M; row0 += step) {
    f32x4 x[R][NV];
    float s[R];
#pragma unroll
    for (int u = 0; u < R; ++u) {
      s[u] = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        x[u][v] = values(next[u][v]);
        s[u] += sum4(x[u][v]);
      }
    }
    load(row0 + step);
    float mean[R], rstd[R];
#pragma unroll
    for (int u = 0; u < R; ++u) mean[u] = row_sum<kLanes>(s[u], slots[turn][0]) / count;
#pragma unroll
    for (int u = 0; u < R; ++u) {
      s[u] = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[u][v][j] = j < n[v] ? x[u][v][j] - mean[u] : 0.f;
        s[u] += sum4(x[u][v] * x[u][v]);
      }
    }
#pragma unroll
    for (int u = 0; u < R; ++u) rstd[u] = 1.0f / sqrtf(row_sum<kLanes>(s[u], slots[turn][1]) / count + a.eps);
    turn ^= 1;
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const int64_t row = row0 + u;
      if (row >= a.M) continue;
      if (lane == 0) {
        if (a.mean_out) a.mean_out[row] = mean[u];
        if (a.rstd_out) a.rstd_out[row] = rstd[u];
      }
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (n[v] > 0) store4<kBf16Out>(a.y, row * D + 4 * (lane + v * kLanes), x[u][v] * rstd[u] * w[v] + b[v], n[v]);
    }
  }
}

// kParams: the gradients of weight and bias are wanted.
template <int kLanes, int NV, bool kBf16In, bool kBf16Out, bool kParams>
__global__ __launch_bounds__(threads<kLanes>()) void layer_norm_grad_kernel(NormArgs a) {
  constexpr int R = rows_at_once<kLanes, NV>();
  constexpr int kThreads = threads<kLanes>();
  constexpr int kRows = kThreads / kLanes * R;
  __shared__ float slots[2][2][kSlots];
  __shared__ f32x4 shares[kParams && kLanes <= kWave ? kThreads / kWave : 1][2 * kWave];
  const int lane = threadIdx.x % kLanes;
  const int D = a.D;
  const float count = (float)D;
  f32x4 w[NV], gw[NV], gb[NV];
  int n[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = 4 * (lane + v * kLanes);
    n[v] = max(0, min(4, D - c));
    w[v] = f32x4{1.f, 1.f, 1.f, 1.f};
    gw[v] = gb[v] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (a.weight) w[v] = load4<false>(a.weight, c, n[v]);
  }
  typename Raw<kBf16In>::Type next_x[R][NV];
  typename Raw<kBf16Out>::Type next_g[R][NV];
  float next_mean[R], next_rstd[R];
  const auto load = [&](int64_t row0) {
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const bool live = row0 + u < a.M;
      next_mean[u] = live ? a.mean[row0 + u] : 0.f;
      next_rstd[u] = live ? a.rstd[row0 + u] : 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int64_t at = (row0 + u) * D + 4 * (lane + v * kLanes);
        next_x[u][v] = load4<kBf16In>(a.x, at, live ? n[v] : 0);
        next_g[u][v] = load4<kBf16Out>(a.grad_y, at, live ? n[v] : 0);
      }
    }
  };
  int64_t row0 = (int64_t)blockIdx.x * kRows + (int)threadIdx.x / kLanes * R;
  const int64_t step = (int64_t)gridDim.x * kRows;
  load(row0);
  int turn = 0;
  for (; row0 < a.M; row0 += step) {
    f32x4 h[R][NV], g[R][NV];
    float rstd[R], s[R], sh[R];
#pragma unroll
    for (int u = 0; u < R; ++u) {
      rstd[u] = next_rstd[u];
      s[u] = sh[u] = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        h[u][v] = (values(next_x[u][v]) - next_mean[u]) * rstd[u];
        g[u][v] = values(next_g[u][v]);
        // (values that do not exist have a zero gradient; mean and rstd may be so large that h is none that can meet it)
#pragma unroll
        for (int j = 0; j < 4; ++j) h[u][v][j] = j < n[v] ? h[u][v][j] : 0.f;
        if (kParams) {
          gw[v] += g[u][v] * h[u][v];
          gb[v] += g[u][v];
        }
        g[u][v] *= w[v];
        s[u] += sum4(g[u][v]);
        sh[u] += sum4(g[u][v] * h[u][v]);
      }
    }
    load(row0 + step);
    float mg[R], mgh[R];
#pragma unroll
    for (int u = 0; u < R; ++u) {
      mg[u] = row_sum<kLanes>(s[u], slots[turn][0]) / count;
      mgh[u] = row_sum<kLanes>(sh[u], slots[turn][1]) / count;
    }
    turn ^= 1;
    if (!a.grad_x) continue;
#pragma unroll
    for (int u = 0; u < R; ++u) {
      const int64_t row = row0 + u;
      if (row >= a.M) continue;
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (n[v] > 0)
          store4<kBf16In>(a.grad_x, row * D + 4 * (lane + v * kLanes), (g[u][v] - mg[u] - h[u][v] * mgh[u]) * rstd[u],
                          n[v]);
    }
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

// Sum of the workgroups' shares: 32 columns by 32 lanes each, sixteen loads in flight per lane.
constexpr int kJoinThreads = 1024, kJoinColumns = 32, kJoinRows = kJoinThreads / kJoinColumns;
__global__ __launch_bounds__(kJoinThreads) void layer_norm_params_kernel(NormArgs a) {
  __shared__ double part[kJoinRows][kJoinColumns + 1];
  const int col = threadIdx.x % kJoinColumns, r = threadIdx.x / kJoinColumns;
  const int c = blockIdx.x * kJoinColumns + col, columns = 2 * a.padded;
  const float* from = a.partials + min(c, columns - 1);
  double s = 0.0;
  constexpr int kBatch = 16;
  for (int p0 = r; p0 < a.num_partials; p0 += kJoinRows * kBatch) {
    float v[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
      v[k] = from[(int64_t)min(p0 + kJoinRows * k, a.num_partials - 1) * columns];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) s += p0 + kJoinRows * k < a.num_partials ? (double)v[k] : 0.0;
  }
  part[r][col] = s;
  __syncthreads();
  if (r == 0 && c < columns) {
    for (int k = 1; k < kJoinRows; ++k) s += part[k][col];
    const int d = c < a.padded ? c : c - a.padded;
    float* out = c < a.padded ? a.grad_weight : a.grad_bias;
    if (out && d < a.D) out[d] = (float)s;
  }
}

template <int kLanes, int NV>
void launch_forward(const NormArgs& a, int blocks, hipStream_t stream) {
  const dim3 grid(blocks), block(threads<kLanes>());
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
  const dim3 grid(blocks), block(threads<kLanes>());
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

// Lanes per row: as few as leave a lane six groups of four values at most.  GB/s of the backward pass in bf16 with the next
// larger number: 192 values 4970 by 16 lanes, 4120 by 64; 384 4690 / 3840; 2048 5090 by 256, 3810 by 64; 5000 4390 by 256,
// 3460 by 512; 8192 3940 by 512, 3400 by 256.
int norm_lanes(int D) { return D <= 384 ? 16 : D <= 1536 ? 64 : D <= 6144 ? 256 : 512; }

template <int kLanes, int NV>
void launch_either(const NormArgs& a, int blocks, bool grad, hipStream_t stream) {
  if (!grad) launch_forward<kLanes, NV>(a, blocks, stream);
  else if (a.partials) launch_backward<kLanes, NV, true>(a, blocks, stream);
  else launch_backward<kLanes, NV, false>(a, blocks, stream);
}

void launch_sized(const NormArgs& a, int blocks, bool grad, hipStream_t stream) {
  const int groups = (a.D + 3) / 4;
  if (a.D <= 384) {
    switch ((groups + 15) / 16) {
      case 1: return launch_either<16, 1>(a, blocks, grad, stream);
      case 2: return launch_either<16, 2>(a, blocks, grad, stream);
      case 3: return launch_either<16, 3>(a, blocks, grad, stream);
      case 4: return launch_either<16, 4>(a, blocks, grad, stream);
      default: return launch_either<16, 6>(a, blocks, grad, stream);
    }
  }
  if (a.D <= 1536) {
    switch ((groups + 63) / 64) {
      case 2: return launch_either<64, 2>(a, blocks, grad, stream);
      case 3: return launch_either<64, 3>(a, blocks, grad, stream);
      case 4: return launch_either<64, 4>(a, blocks, grad, stream);
      case 5: return launch_either<64, 5>(a, blocks, grad, stream);
      default: return launch_either<64, 6>(a, blocks, grad, stream);
    }
  }
  if (a.D <= 6144) {
    switch ((groups + 255) / 256) {
      case 2: return launch_either<256, 2>(a, blocks, grad, stream);
      case 3: return launch_either<256, 3>(a, blocks, grad, stream);
      case 4: return launch_either<256, 4>(a, blocks, grad, stream);
      default: return launch_either<256, 6>(a, blocks, grad, stream);
    }
  }
  return launch_either<512, 4>(a, blocks, grad, stream);
}

int norm_blocks(int64_t M, int D, int most) {
  const int lanes = norm_lanes(D);
  const int rows = (lanes > 256 ? 1 : 256 / lanes) * ((D + 3) / 4 <= 3 * lanes && lanes <= kWave ? 2 : 1);  // rows_at_once
  const int64_t blocks = (M + rows - 1) / rows;
  return (int)(blocks < most ? blocks : most);
}

}  // namespace

// Workgroups of the backward kernel: every one leaves 2 D sums that another kernel reads, so that few rows take fewer of
// them than could have a row of their own.  us of the backward pass with / without that, bf16: 700 x 4096 14.7 / 19.9, 4000 x
// 4096 28.4 / 32.2, 4000 x 1024 12.6 / 15.9, 4000 x 8192 54 / 64.
int norm_partials(int64_t M, int D) {
  const int64_t most = M / 10;
  return norm_blocks(M, D, most < 256 ? 256 : most < 1024 ? (int)most : 1024);
}

hipError_t launch_layer_norm(const NormArgs& a, hipStream_t stream) {
  launch_sized(a, norm_blocks(a.M, a.D, 2048), false, stream);
  return hipGetLastError();
}

hipError_t launch_layer_norm_grad(const NormArgs& a, hipStream_t stream) {
  launch_sized(a, a.partials ? a.num_partials : norm_blocks(a.M, a.D, 1024), true, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.partials) return e;
  hipLaunchKernelGGL(layer_norm_params_kernel, dim3((2 * a.padded + kJoinColumns - 1) / kJoinColumns),
                     dim3(kJoinThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mae

// Dropout of token rows with no stored mask, added to a residual: the keyed draws of the library are
// made again wherever they are needed, so the backward pass is the same call on the gradient.
//
//   value i of the tensor (or the i-th group of rows, "drop path") draws 32 bits: half i mod 2 of
//   mix64(key + GAMMA (i / 2 + 1));  kept iff the draw >= p 2^32;  y = kept ? x / (1 - p) : 0, + residual
//
// Bound by HBM; a 64-bit mix (two 64-bit products) serves two values, beside 16-byte loads and stores
// of eight (bf16) or twice four (fp32) values per lane.  Values that are dropped are selected away, not multiplied by
// zero, so an infinity or a NaN among them does not reach the result; groups that are dropped are not read.
// 204,800 x 768 in bf16 with a residual (944 MB): 159 us, 5.9 TB/s; 147,492 x 1017 by single rows 150 (314 where a lane's
// eight values that lie in two rows went one by one).
#include "mae_device.hpp"
#include "mae_kernels.hpp"

namespace mae {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// tensors begin at any multiple of their values' size (rows cut out of a batch)
typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));

constexpr int kThreads = 256;
constexpr int kVec = 8;                    // values per lane and step
constexpr int kChunk = kThreads * kVec;    // values of a workgroup per step

struct Values {
  float v[kVec];
};

template <bool kBf16>
__device__ inline Values load8(const void* p, int64_t at) {
  Values r;
  if (kBf16) {
    const u32x4 raw = *reinterpret_cast<const u32x4_a2*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      r.v[2 * j] = bf16_lo(raw[j]);
      r.v[2 * j + 1] = bf16_hi(raw[j]);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 raw = *reinterpret_cast<const f32x4_a4*>(static_cast<const float*>(p) + at + 4 * h);
#pragma unroll
      for (int j = 0; j < 4; ++j) r.v[4 * h + j] = raw[j];
    }
  }
  return r;
}
template <bool kBf16>
__device__ inline void store8(void* p, int64_t at, const Values& r) {
  if (kBf16) {
    *reinterpret_cast<u32x4_a2*>(static_cast<uint16_t*>(p) + at) =
        u32x4{pack_bf16x2(r.v[0], r.v[1]), pack_bf16x2(r.v[2], r.v[3]), pack_bf16x2(r.v[4], r.v[5]),
              pack_bf16x2(r.v[6], r.v[7])};
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<f32x4_a4*>(static_cast<float*>(p) + at + 4 * h) =
          f32x4{r.v[4 * h], r.v[4 * h + 1], r.v[4 * h + 2], r.v[4 * h + 3]};
  }
}
template <bool kBf16>
__device__ inline float load1(const void* p, int64_t at) {
  return kBf16 ? __uint_as_float((uint32_t)static_cast<const uint16_t*>(p)[at] << 16)
               : static_cast<const float*>(p)[at];
}
template <bool kBf16>
__device__ inline void store1(void* p, int64_t at, float v) {
  if (kBf16) static_cast<uint16_t*>(p)[at] = (uint16_t)bf16_rne(v);
  else static_cast<float*>(p)[at] = v;
}

__device__ inline uint64_t pair_draw(uint64_t key, uint64_t pair) { return mix64(key + kGamma * (pair + 1)); }
// whether value (or group) i is kept
__device__ inline bool kept(const DropoutArgs& a, uint64_t i) {
  const uint64_t z = pair_draw(a.key, i >> 1);
  return (uint64_t)(uint32_t)((i & 1) ? z >> 32 : z) >= a.threshold;
}

// kOdd: value 0 of the tensor has an odd index, so that eight values touch five pairs.
template <bool kBf16, bool kOdd>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropoutArgs a) {
  for (int64_t at = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kVec; at < a.count;
       at += (int64_t)gridDim.x * kChunk) {
    const uint64_t i = a.first + (uint64_t)at;
    if (at + kVec <= a.count) {
      Values x = load8<kBf16>(a.x, at);
      Values r;
      if (a.residual) r = load8<kBf16>(a.residual, at);
      uint64_t z = pair_draw(a.key, i >> 1);
#pragma unroll
      for (int j = 0; j < kVec; ++j) {
        constexpr int kShift = kOdd ? 1 : 0;
        if (j > 0 && ((j + kShift) & 1) == 0) z = pair_draw(a.key, (i >> 1) + (uint64_t)((j + kShift) >> 1));
        const uint32_t bits = (uint32_t)(((j + kShift) & 1) ? z >> 32 : z);
        x.v[j] = (uint64_t)bits >= a.threshold ? x.v[j] * a.scale : 0.f;
        if (a.residual) x.v[j] += r.v[j];
      }
      store8<kBf16>(a.y, at, x);
    } else {
      for (int64_t e = at; e < a.count; ++e) {
        float v = kept(a, a.first + (uint64_t)e) ? load1<kBf16>(a.x, e) * a.scale : 0.f;
        if (a.residual) v += load1<kBf16>(a.residual, e);
        store1<kBf16>(a.y, e, v);
      }
    }
  }
}

// One draw per `span` consecutive values (whole rows).  What is dropped is not read.
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void drop_path_kernel(DropoutArgs a) {
  for (int64_t start = (int64_t)blockIdx.x * kChunk; start < a.count; start += (int64_t)gridDim.x * kChunk) {
    // group of the workgroup's first value, and that value's place in it
    const uint64_t from = a.first + (uint64_t)start;  // counted from the start of group a.group0
    const uint64_t g0 = from / a.span, rest = from % a.span;
    const int off = threadIdx.x * kVec;
    const int64_t at = start + off;
    if (at >= a.count) continue;
    auto group = [&](int o) -> uint64_t {
      const uint64_t r = rest + (uint64_t)o;
      if (a.span >= (uint64_t)kChunk) return g0 + (r >= a.span ? 1 : 0);  // (o < kChunk: one border at most)
      return g0 + (uint64_t)((uint32_t)r / (uint32_t)a.span);
    };
    const uint64_t ga = group(off);
    if (at + kVec <= a.count && a.span >= kVec) {
      // values of this lane that lie in group ga; the others in the next one
      const uint64_t left = (ga - g0 + 1) * a.span - (rest + (uint64_t)off);
      const bool first = kept(a, a.group0 + ga);
      const bool second = left >= (uint64_t)kVec ? first : kept(a, a.group0 + ga + 1);
      Values x;
#pragma unroll
      for (int j = 0; j < kVec; ++j) x.v[j] = 0.f;
      if (first || second) {
        x = load8<kBf16>(a.x, at);
#pragma unroll
        for (int j = 0; j < kVec; ++j) x.v[j] = ((uint64_t)j < left ? first : second) ? x.v[j] * a.scale : 0.f;
      }
      if (a.residual) {
        const Values r = load8<kBf16>(a.residual, at);
#pragma unroll
        for (int j = 0; j < kVec; ++j) x.v[j] += r.v[j];
      }
      store8<kBf16>(a.y, at, x);
    } else {
      for (int j = 0; j < kVec && at + j < a.count; ++j) {
        float v = kept(a, a.group0 + group(off + j)) ? load1<kBf16>(a.x, at + j) * a.scale : 0.f;
        if (a.residual) v += load1<kBf16>(a.residual, at + j);
        store1<kBf16>(a.y, at + j, v);
      }
    }
  }
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  const int64_t chunks = (a.count + kChunk - 1) / kChunk;
  const dim3 grid((uint32_t)(chunks < (1 << 20) ? chunks : 1 << 20)), block(kThreads);
  if (a.span) {
    if (a.bf16) hipLaunchKernelGGL((drop_path_kernel<true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((drop_path_kernel<false>), grid, block, 0, stream, a);
  } else if (a.first & 1) {
    if (a.bf16) hipLaunchKernelGGL((dropout_kernel<true, true>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((dropout_kernel<false, true>), grid, block, 0, stream, a);
  } else {
    if (a.bf16) hipLaunchKernelGGL((dropout_kernel<true, false>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((dropout_kernel<false, false>), grid, block, 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace mae

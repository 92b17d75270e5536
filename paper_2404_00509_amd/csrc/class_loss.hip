// Softmax cross entropy of a linear head over many classes (the finetuning recipe's loss, Sec. 3, Sec. 5.2, with
// its label smoothing), with the gradients of tokens, weight and bias, and without ever
// holding the logits of a large call: they are made on the matrix cores tile by tile and reduced; for the gradient
// something of them is kept where there is room, and the rest made again.
//
//   l = x W^T + b;  loss_n = lse(l_n) - (1 - s) l_n,y - s mean(l_n);  loss = mean of loss_n
//   g = (softmax(l) - (1 - s) onehot(y) - s / V) grad_scale / count
//   grad_x = g W, grad_W = g^T x, grad_b = sum over rows of g
//
//   pack      rows whose label is no class are left out: the others' labels and tokens one after the other, and
//             their count, which the later kernels read from memory.  What such a row holds (NaN, infinities) touches
//             nothing.  For the gradient also the largest magnitudes among tokens and weight
//   stats     tiles of logits -> per row and tile the maximum, the sum of exponentials under it, the sum of logits
//             (smoothing) and the label's logit.  For the gradient also, without bias and smoothing, the exponentials of
//             the first piece of the classes, else all logits of a small call (class_plan)
//   rows      the tiles of a row joined -> maximum, 1 / sum, the row's loss.  Beside it, for the gradient, tokens and
//             weight as fp16
//   grad      what is kept, or tiles of logits again -> g as fp16 [rows, classes of the piece], sums of its columns in
//             fp32; one workgroup joins the loss (without gradient: a launch of its own)
//   products  g W (g along k, W across k) and g^T x (both across k) in one launch; few tiles: k is split
//   finish    grad_bias, and the parts of a split joined, scaled, rounded once to bf16
//
// The loss alone of a few rows (one tile of 64) takes two launches: stats on the tokens as they are, rows.
//
// The gradient goes through the vocabulary in pieces, so g takes M x piece values of the workspace.
// Logits are made as W x^T: a lane then holds up to 64 classes of one row, and the
// reductions over classes stay in registers up to the last two steps.
//
// Types.  Logits: products of the bf16 operands, fp32 sums.  Maxima, exponentials and their sums: fp32; sums over rows of
// the loss: double precision.  g, an operand of two products, is fp16 and not bf16: |g| <= 1, so that as 2^15 g it
// loses at most 2^-11 of a value down to 2^-29, an eighth of what bf16 would, and less than the bf16 outputs
// do by their own rounding (with bf16 gradients were up to 1.5 times as far from the exact ones as results that are
// rounded once, now within 1 %).  Kept exponentials are 2^15 exp as fp16 likewise, under the maximum of their group of
// classes; the label's g is made from its logit, and there is no smoothing, so that nothing cancels; nor a bias, whose
// gradient is a sum of g in single precision.  What is below 2^-40 of g becomes 0.  The other operand has to be fp16 too: scaled
// by the power of two that puts its largest value just under 2^15, a bf16 number down to 2^-31 of the largest is exact (to the
// smallest there is, where the largest is below 2^-112).  Where values lie further apart than that (too_wide; one token of
// 1e15 among tokens around 1, say), both products are of bf16 instead, with g rounded to it: found out on the device, at a
// percent of a small call's time (4096 x 768 over 1000 classes 69.2 -> 70.0 us), nothing of a large one's.
//
// 16,384 x 1024 over 32,003 classes, a tenth of the rows left out, 2.90 TFLOP: 3.1 ms (3.6 to 3.7 with the logits made
// again).  pack 28 us, stats 1050 (0.92 PFLOP/s; 915 if nothing is kept), rows 58, grad 362 (1.9 GB, 5.2 TB/s), products 1630
// (1.19 PFLOP/s).  What bounds it is the main loop (matmul.hpp), and beside it in stats the exponentials: a tile of
// 256 x 256 with 16 slices takes 33 us, 26 of them in the loop, and storing exponentials 5 more.  Small calls are bound by
// their launches: 64 x 192 over 1000 classes 28 us for six, 4.5 us each.
#include "mae_device.hpp"
#include "mae_kernels.hpp"
#include "matmul.hpp"

namespace mae {

namespace {

using namespace mm;

typedef f32x4 f32x4_a4 __attribute__((aligned(4)));
typedef int32_t i32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -__builtin_inff();
constexpr int kGExponent = 15;
constexpr float kGScale = 1 << kGExponent;  // of g as fp16
// Of logits in their sum: of up to 2^20 classes that are ruled out by the lowest float as their bias, it stays a float.
constexpr float kSumScale = 0x1p-20f;
// What stats leaves of the first piece for its gradient
enum Keep { kKeepNone, kKeepLogits, kKeepExp };

// exp(v) for v <= 0
__device__ inline float exp_neg(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }

// rows that take part
__device__ inline int row_count(const ClassArgs& a) { return a.count ? uniform(*a.count) : (int)a.M; }

// ---- powers of two that bring the operands into the range of fp16 ---------------------------------------
constexpr int kPackThreads = 256;

// Of finite magnitudes as bf16 bits: in the low half the largest; in the high half the smallest that the largest of any eight
// neighbours is, where these are not all zero, counted down from infinity, so that both halves are maxima (of nothing: 0).
__device__ inline uint32_t both(uint32_t a, uint32_t b) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
__device__ inline uint32_t range_of(u32x4 v) {
  uint32_t peak = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t lo = v[k] & 0x7FFFu, hi = (v[k] >> 16) & 0x7FFFu;
    if (lo < 0x7F80u) peak = max(peak, lo);
    if (hi < 0x7F80u) peak = max(peak, hi);
  }
  return peak > 0 ? (0x7F80u - peak) << 16 | peak : 0u;
}
__device__ inline int32_t most_of(uint32_t range) { return (int32_t)(range & 0xFFFFu); }
__device__ inline int32_t least_of(uint32_t range) { return 0x7F80 - (int32_t)(range >> 16); }
__device__ inline uint32_t over_lanes(uint32_t range) {
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) range = both(range, (uint32_t)__shfl_xor((int)range, off, kWave));
  return range;
}
// The workgroup's to memory.
__device__ inline void leave_range(uint32_t range, uint32_t* slots, uint32_t* out) {
  range = over_lanes(range);
  __syncthreads();
  if (threadIdx.x % kWave == 0) slots[threadIdx.x / kWave] = range;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kPackThreads / kWave; ++w) range = both(range, slots[w]);
    *out = range;
  }
}
// Of the workgroups [from, to), by all lanes of a wavefront
__device__ inline uint32_t range_among(const uint32_t* ranges, int from, int to) {
  uint32_t range = 0;
  for (int i = from + (int)(threadIdx.x % kWave); i < to; i += kWave) range = both(range, ranges[i]);
  return over_lanes(range);
}
// Whether an operand goes beyond what an fp16 copy holds.  With the largest value just under 2^15, eight neighbours of which
// the largest is 2^-25 of that are at most 2^-15 of it off (half a step of fp16's smallest numbers), a sixteenth of what g
// loses by its rounding; what is smaller still would lose more, and in the end everything.
__device__ inline bool too_wide(uint32_t range) { return (most_of(range) >> 7) - (least_of(range) >> 7) > 24; }
// The factor that brings values of which `peak` is the largest under 2^15, as an exponent of two: fp16 holds
// 2^15 times what is under 2.  At most 2^126 and at least 2^-113, so that it is a float and so is its inverse.
__device__ inline int half_exponent(int32_t peak) {
  const int e = (peak >> 7) - 127;  // 2^e <= the largest value < 2^(e + 1)
  return min(14 - e, 126);
}

__device__ inline uint32_t half_pair(float lo, float hi) {
  typedef float in2 __attribute__((ext_vector_type(2)));
  typedef _Float16 out2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((in2{lo, hi}), out2));
}

// grad_scale / count
__device__ inline double grad_factor(const ClassArgs& a) {
  const int n = *a.count;
  return n > 0 ? (double)a.grad_scale / (double)n : 0.0;
}
// What g is multiplied by if it is bf16: at most 1 / rows, so that sums over rows stay floats wherever the operand's values are.
__device__ inline int wide_exponent(const ClassArgs& a) { return *a.count > 1 ? __clz(*a.count - 1) - 32 : 0; }

// A product's sum to a gradient: a factor in [0.5, 1), and the powers of two of grad_scale, of the number of rows and of the
// operands, none of which need be a float by itself (an upstream derivative of 1e38, operands of 1e-30).
struct Scale {
  float factor;
  int exponent;
  __device__ inline float operator()(float v) const { return ldexpf(v * factor, exponent); }
};
__device__ inline Scale product_scale(const ClassArgs& a, bool by_weight) {
  const int from = by_weight ? a.pack_blocks : 0, to = by_weight ? a.num_ranges : a.pack_blocks;
  const int of_half = kGExponent + half_exponent(most_of(range_among(a.ranges, from, to)));
  int e;
  const double m = frexp(grad_factor(a), &e);
  return Scale{(float)m, e - (*a.wide ? wide_exponent(a) : of_half)};
}

// ---- pack -----------------------------------------------------------------------------------------
// Workgroups from pack_blocks on look for the range of the weight's magnitudes.
__global__ __launch_bounds__(kPackThreads) void class_pack_kernel(ClassArgs a) {
  __shared__ int32_t wave_sum[kPackThreads / kWave];
  __shared__ uint32_t wave_range[kPackThreads / kWave];
  __shared__ int32_t map[kPackThreads];
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  uint32_t range = 0;
  if ((int)blockIdx.x >= a.pack_blocks) {
    const u32x4* w = reinterpret_cast<const u32x4*>(a.weight);
    const int64_t n = (int64_t)a.V * a.D / 8, step = (int64_t)(a.num_ranges - a.pack_blocks) * kPackThreads;
    constexpr int kBatch = 4;  // loads in flight
    for (int64_t i = (int64_t)((int)blockIdx.x - a.pack_blocks) * kPackThreads + tid; i < n; i += kBatch * step) {
      u32x4 v[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) v[k] = i + k * step < n ? w[i + k * step] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int k = 0; k < kBatch; ++k) range = both(range, range_of(v[k]));
    }
    leave_range(range, wave_range, a.ranges + blockIdx.x);
    return;
  }
  const int64_t row0 = (int64_t)blockIdx.x * a.pack_rows;
  const int64_t end = min(row0 + a.pack_rows, a.M);
  auto is_class = [&](int32_t label) { return (uint32_t)label < (uint32_t)a.V ? 1 : 0; };
  // rows in front of this workgroup's that take part (row0 is a multiple of 4)
  int32_t before = 0;
#pragma unroll 4
  for (int64_t r = 4 * tid; r < row0; r += 4 * kPackThreads) {
    const i32x4_a4 l = *reinterpret_cast<const i32x4_a4*>(a.labels + r);
    before += (is_class(l.x) + is_class(l.y)) + (is_class(l.z) + is_class(l.w));
  }
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) before += __shfl_xor(before, off, kWave);
  if (lane == 0) wave_sum[wave] = before;
  __syncthreads();
  int32_t at = 0;
  for (int w = 0; w < kPackThreads / kWave; ++w) at += wave_sum[w];
  for (int64_t base = row0; base < end; base += kPackThreads) {
    const int64_t r = base + tid;
    const bool in = r < end && is_class(a.labels[r]);
    const uint64_t votes = __ballot(in);
    __syncthreads();
    if (lane == 0) wave_sum[wave] = __popcll(votes);
    __syncthreads();
    int32_t slot = at + __popcll(votes & ((1ull << lane) - 1));
    for (int w = 0; w < wave; ++w) slot += wave_sum[w];
    for (int w = 0; w < kPackThreads / kWave; ++w) at += wave_sum[w];
    if (in) {
      a.label_of[slot] = a.labels[r];
      a.row_of[slot] = (int32_t)r;
    }
    if (r < end && !in && a.row_loss) a.row_loss[r] = 0.f;
    map[tid] = in ? slot : -1;
    __syncthreads();
    // the tokens, 16 bytes per lane, several loads in flight
    const int per_row = a.D / 8, chunks = (int)min((int64_t)kPackThreads, end - base) * per_row;
    const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.tokens) + base * a.D);
    constexpr int kBatch = 8;
    for (int i0 = tid; i0 < chunks; i0 += kBatch * kPackThreads) {
      u32x4 v[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) v[k] = src[min(i0 + k * kPackThreads, chunks - 1)];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int i = i0 + k * kPackThreads;
        if (i >= chunks) break;
        const int row = i / per_row, c = i - row * per_row, to = map[row];
        if (to >= 0) {
          if (a.ranges) range = both(range, range_of(v[k]));
          reinterpret_cast<u32x4*>(a.packed + (int64_t)to * a.D)[c] = v[k];
        } else if (a.grad_tokens) {
          reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.grad_tokens) + (base + row) * a.D)[c] = u32x4{0u, 0u, 0u, 0u};
        }
      }
    }
  }
  if (end == a.M && tid == 0) *a.count = at;
  if (a.ranges) leave_range(range, wave_range, a.ranges + blockIdx.x);
}

// ---- tiles of logits --------------------------------------------------------------------------------
// acc[i][j][e]: class 32 (wm TM + i) + 8 (e / 4) + 4 (lane / 32) + e % 4 of the tile, row 32 (wn TN + j) + lane % 32.
template <int TM, int TN>
__device__ inline void add_bias(const float* bias, int first, int V, int lane, f32x16 (&acc)[TM][TN]) {
  if (!bias) return;
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int v = first + 32 * i + 8 * q + 4 * (lane >> 5);
      f32x4 b = f32x4{0.f, 0.f, 0.f, 0.f};
      if (v + 4 <= V) {
        b = *reinterpret_cast<const f32x4_a4*>(bias + v);
      } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
          if (v + k < V) b[k] = bias[v + k];
      }
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][j][4 * q + k] += b[k];
    }
}

template <int TM, int TN, int WGM, int WGN>
struct Logits : Tile<TM, TN, WGM, WGN, true, true> {
  using Base = Tile<TM, TN, WGM, WGN, true, true>;

  // Where tile number `id` lies; classes [first, first + classes).
  struct Place {
    int tv, tn;          // column and row of the grid of tiles
    int c0;              // first class, counted from `first`
    int64_t n0;          // first row
    int rows_v, rows_n;  // that exist
    typename Base::Source source;
  };
  __device__ static inline Place place(const ClassArgs& a, uint32_t id, uint32_t tiles, int count, int first, int classes) {
    const uint32_t tiles_v = (uint32_t)((classes + Base::BM - 1) / Base::BM);
    uint32_t tn, tv;
    grouped(xcd_remap(id, tiles), tiles / tiles_v, tiles_v, &tn, &tv);
    Place p;
    p.tv = (int)tv;
    p.tn = (int)tn;
    p.c0 = (int)tv * Base::BM;
    p.n0 = (int64_t)tn * Base::BN;
    p.rows_v = min(Base::BM, classes - p.c0);
    p.rows_n = min(Base::BN, count - (int)p.n0);
    const Operand W{static_cast<const uint16_t*>(a.weight) + (int64_t)(first + p.c0) * a.D, a.D, p.rows_v};
    const Operand X{a.packed + p.n0 * a.D, a.D, p.rows_n};
    p.source = Base::source(W, X, a.D);
    return p;
  }
  __device__ static inline uint32_t tiles(int count, int classes) {
    return (uint32_t)((count + Base::BN - 1) / Base::BN) * (uint32_t)((classes + Base::BM - 1) / Base::BM);
  }

  // The tile's logits to memory or back, as they lie in the lanes.
  template <bool kStore>
  __device__ static inline void logits_of(const ClassArgs& a, const Place& at, int wave, int lane, f32x16 (&acc)[TM][TN]) {
    const int64_t tile = (int64_t)at.tn * a.stat_tiles + at.tv;
    f32x4* p = reinterpret_cast<f32x4*>(a.logits) + (tile * (WGM * WGN) + wave) * (TM * TN * 4 * kWave) + lane;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4* to = p + ((i * TN + j) * 4 + q) * kWave;
          if (kStore) {
            *to = f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
          } else {
            const f32x4 v = *to;
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][j][4 * q + k] = v[k];
          }
        }
  }

  // Rows 32 j .. + 31 of a wavefront's values as fp16 to g (kWide: as bf16, times `down`).  A lane has every second group of
  // four classes of its row: the halves of the wavefront swap theirs, so that each has groups of eight, 16 bytes.  (Through
  // strips of LDS, 256 bytes along a row at a time: 3 % of a call over 32,003 classes more.)
  template <int j, bool kWide = false>
  __device__ static inline void store_block(const ClassArgs& a, const Place& at, int wave, int lane,
                                            const f32x16 (&acc)[TM][TN], float down = 1.f) {
    const auto pair = [&](float lo, float hi) { return kWide ? pack_bf16x2(lo * down, hi * down) : half_pair(lo, hi); };
    const int wm = wave / WGN, wn = wave % WGN;
    const int row = wn * 32 * TN + j * 32 + (lane & 31), c = at.c0 + wm * 32 * TM + 8 * (lane >> 5);
    uint16_t* to = a.g + (at.n0 + row) * (int64_t)a.piece_ld + c;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int q = 0; q < 4; q += 2) {
        u32x4 v;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const auto swapped = __builtin_amdgcn_permlane32_swap(
              pair(acc[i][j][4 * q + 2 * k], acc[i][j][4 * q + 2 * k + 1]),
              pair(acc[i][j][4 * q + 4 + 2 * k], acc[i][j][4 * q + 5 + 2 * k]), false, false);
          v[k] = swapped[0];
          v[2 + k] = swapped[1];
        }
        if (row < at.rows_n && c + 32 * i + 8 * q < a.piece_ld) *reinterpret_cast<u32x4*>(to + 32 * i + 8 * q) = v;
      }
  }
};

template <int TM, int TN, int WGM, int WGN, int kKeep>
__global__ __launch_bounds__(64 * WGM * WGN) void class_stats_kernel(ClassArgs a) {
  using T = Logits<TM, TN, WGM, WGN>;
  __shared__ __attribute__((aligned(1024))) u32x4 lds[T::kLdsBytes / 16];
  const int count = row_count(a);
  const uint32_t tiles = T::tiles(count, a.V);
  if (blockIdx.x >= tiles) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int wm = wave / WGN, wn = wave % WGN;
  // beside the epilogue of a tile the next one's first slices are brought in; the epilogue has the ring's last place
  float* part = reinterpret_cast<float*>(lds + 4 * T::kSlots);  // [WGM][BN][3]
  static_assert(WGM * T::BN * 3 * 4 <= T::kPlaceBytes, "room in a place");
  typename T::Place next = T::place(a, blockIdx.x, tiles, count, 0, a.V);
  T::template fill<0, 4>(next.source, lds);
  for (uint32_t id = blockIdx.x; id < tiles; id += gridDim.x) {
    const typename T::Place at = next;
    f32x16 acc[TM][TN];
    T::template run<4>(at.source, lds, acc);
    const int v0 = at.c0, rows_v = at.rows_v, rows_n = at.rows_n;
    const int64_t n0 = at.n0;
    const int first = v0 + wm * 32 * TM;
    __syncthreads();  // every wavefront is done with the ring
    if (id + gridDim.x < tiles) {
      next = T::place(a, id + gridDim.x, tiles, count, 0, a.V);
      T::template fill<0, 4>(next.source, lds);
    }
    add_bias<TM, TN>(a.bias, first, a.V, lane, acc);
    if (kKeep == kKeepLogits) T::template logits_of<true>(a, at, wave, lane, acc);
    const int half = 4 * (lane >> 5);
    const int classes = a.V - first - half;  // class 32 i + 8 (e / 4) + e % 4 of this lane exists if below
    unroll<TN>([&](auto j_tag) {
      constexpr int j = decltype(j_tag)::value;
      const int r = wn * 32 * TN + j * 32 + (lane & 31);
      const int y = r < rows_n ? a.label_of[n0 + r] - first - half : -1;
      float sl = 0.f;
      if (a.logit_sums) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            sl += 32 * i + 8 * (e >> 2) + (e & 3) < classes ? acc[i][j][e] * kSumScale : 0.f;
      }
      if (rows_v < T::BM) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i][j][e] = 32 * i + 8 * (e >> 2) + (e & 3) < classes ? acc[i][j][e] : kNegInf;
      }
      // the label's logit: few rows have theirs among a wavefront's classes
      const bool mine = y >= 0 && y < 32 * TM && (y & 4) == 0;
      if (__any(mine)) {
        float own = 0.f;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) own = 32 * i + 8 * (e >> 2) + (e & 3) == y ? acc[i][j][e] : own;
        if (mine) a.label_logit[n0 + r] = own;
      }
      float m = acc[0][j][0];
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) m = fmaxf(m, acc[i][j][e]);
      m = fmaxf(m, __shfl_xor(m, 32, kWave));
      const float from = m == kNegInf ? 0.f : m;  // (a tile of -inf only adds nothing; a NaN reaches the sum)
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float v = exp_neg(acc[i][j][e] - from);
          s += v;
          if (kKeep == kKeepExp) acc[i][j][e] = v * kGScale;
        }
      s += __shfl_xor(s, 32, kWave);
      sl += __shfl_xor(sl, 32, kWave);
      if (lane < 32) {
        float* p = part + (wm * T::BN + r) * 3;
        p[0] = m;
        p[1] = s;
        p[2] = sl;
      }
      if (kKeep == kKeepExp && v0 < a.piece_classes) {  // (pieces are whole tiles, or all classes)
        if (lane < 32 && r < rows_n) a.tops[(n0 + r) * (int64_t)a.top_ld + at.tv * WGM + wm] = m;
        T::template store_block<j>(a, at, wave, lane, acc);
      }
    });
    __syncthreads();
    for (int r = tid; r < rows_n; r += T::kThreads) {
      float m = kNegInf, s = 0.f, sl = 0.f;
#pragma unroll
      for (int w = 0; w < WGM; ++w) m = fmaxf(m, part[(w * T::BN + r) * 3]);
#pragma unroll
      for (int w = 0; w < WGM; ++w) {
        const float* p = part + (w * T::BN + r) * 3;
        s += p[0] == kNegInf ? p[1] : p[1] * exp_neg(p[0] - m);
        sl += p[2];
      }
      const int64_t to = (n0 + r) * (int64_t)a.stat_tiles + at.tv;
      reinterpret_cast<f32x2*>(a.stats)[to] = f32x2{m, s};
      if (a.logit_sums) a.logit_sums[to] = sl;
    }
    __syncthreads();
  }
}

// ---- rows -------------------------------------------------------------------------------------------
// One row by one wavefront: its loss; maximum and 1 / sum to memory.
__device__ inline float join_row(const ClassArgs& a, int64_t slot, int lane) {
  const f32x2* st = reinterpret_cast<const f32x2*>(a.stats) + slot * a.stat_tiles;
  const float own = a.label_logit[slot];
  float m = kNegInf, s = 0.f, sl = 0.f;
  constexpr int kBatch = 8;  // loads in flight
  for (int t0 = lane; t0 < a.stat_tiles; t0 += kBatch * kWave) {
    f32x2 p[kBatch];
    float top = m;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      p[k] = st[min(t0 + k * kWave, a.stat_tiles - 1)];
      if (t0 + k * kWave >= a.stat_tiles) p[k] = f32x2{kNegInf, 0.f};
      top = fmaxf(top, p[k].x);
    }
    if (a.logit_sums) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        if (t0 + k * kWave < a.stat_tiles) sl += a.logit_sums[slot * a.stat_tiles + t0 + k * kWave];
    }
    // (-inf: nothing under it, or a NaN that reaches the sum)
    s = m == kNegInf ? s : s * exp_neg(m - top);
#pragma unroll
    for (int k = 0; k < kBatch; ++k) s += p[k].x == kNegInf ? p[k].y : p[k].y * exp_neg(p[k].x - top);
    m = top;
  }
  float top = m;
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
  s = m == kNegInf ? s : s * exp_neg(m - top);
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) {
    s += __shfl_xor(s, off, kWave);
    sl += __shfl_xor(sl, off, kWave);
  }
  float v = (top + logf(s)) - (1.0f - a.smoothing) * own;
  if (a.logit_sums) v -= a.smoothing * (sl / ((float)a.V * kSumScale));
  if (lane == 0 && a.ranges) {
    a.row_max[slot] = top;
    a.row_inv[slot] = 1.0f / s;
  }
  return v;
}

constexpr int kRowThreads = 256, kRowWaves = kRowThreads / kWave;
// Workgroups from row_blocks on make the fp16 copies, eight values per lane, and find out whether they do.
__global__ __launch_bounds__(kRowThreads) void class_rows_kernel(ClassArgs a) {
  if ((int)blockIdx.x >= a.row_blocks) {
    const uint32_t of_t = range_among(a.ranges, 0, a.pack_blocks), of_w = range_among(a.ranges, a.pack_blocks, a.num_ranges);
    const int64_t of_tokens = (int64_t)*a.count * (a.D / 8), of_weight = (int64_t)a.V * (a.D / 8);
    const float ft = ldexpf(1.0f, half_exponent(most_of(of_t))), fw = ldexpf(1.0f, half_exponent(most_of(of_w)));
    const int64_t step = (int64_t)((int)gridDim.x - a.row_blocks) * kRowThreads;
    for (int64_t i = (int64_t)((int)blockIdx.x - a.row_blocks) * kRowThreads + threadIdx.x; i < of_tokens + of_weight;
         i += step) {
      const bool t = i < of_tokens;
      const int64_t at = t ? i : i - of_tokens;
      const u32x4 v = t ? reinterpret_cast<const u32x4*>(a.packed)[at] : reinterpret_cast<const u32x4*>(a.weight)[at];
      const float f = t ? ft : fw;
      u32x4 out;
#pragma unroll
      for (int k = 0; k < 4; ++k) out[k] = half_pair(bf16_lo(v[k]) * f, bf16_hi(v[k]) * f);
      reinterpret_cast<u32x4*>(t ? a.half_tokens : a.half_weight)[at] = out;
    }
    // (behind the loop: in front of it the compiler would not read the number of rows before it has stored this)
    if ((int)blockIdx.x == a.row_blocks && threadIdx.x == 0) *a.wide = too_wide(of_t) || too_wide(of_w) ? 1 : 0;
    return;
  }
  __shared__ double sums[kRowWaves];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int count = *a.count;
  double loss = 0.0;
  for (int64_t slot = (int64_t)blockIdx.x * kRowWaves + wave; slot < count; slot += (int64_t)a.row_blocks * kRowWaves) {
    const float v = join_row(a, slot, lane);
    loss += (double)v;
    if (lane == 0 && a.row_loss) a.row_loss[a.row_of[slot]] = v;
  }
  if (lane == 0) sums[wave] = loss;
  __syncthreads();
  if (threadIdx.x == 0) a.partials[blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
}

// The loss from the workgroups' shares, by the first kRowThreads threads of a workgroup; `sums`: kRowWaves of LDS.
__device__ inline void join_losses(const ClassArgs& a, double* sums) {
  const int tid = threadIdx.x, count = *a.count;
  double s = 0.0;
  if (tid < kRowThreads)
    for (int i = tid; i < a.row_blocks; i += kRowThreads) s += a.partials[i];
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) s += __shfl_xor(s, off, kWave);
  if (tid < kRowThreads && tid % kWave == 0) sums[tid / kWave] = s;
  __syncthreads();
  if (tid == 0) *a.loss = count > 0 ? (float)(((sums[0] + sums[1]) + (sums[2] + sums[3])) / (double)count) : 0.f;
  __syncthreads();
}
__global__ __launch_bounds__(kRowThreads) void class_loss_kernel(ClassArgs a) {
  __shared__ double sums[kRowWaves];
  join_losses(a, sums);
}

// The rows of a call that did not pack any: one workgroup.
constexpr int kFewThreads = 1024, kFewRows = 64;
__global__ __launch_bounds__(kFewThreads) void class_few_rows_kernel(ClassArgs a) {
  __shared__ float losses[kFewRows];
  __shared__ int32_t in_rows[kFewRows];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  for (int row = wave; row < (int)a.M; row += kFewThreads / kWave) {
    const bool in = (uint32_t)a.labels[row] < (uint32_t)a.V;
    const float v = in ? join_row(a, row, lane) : 0.f;
    if (lane == 0) {
      losses[row] = v;
      in_rows[row] = in ? 1 : 0;
      if (a.row_loss) a.row_loss[row] = v;
    }
  }
  __syncthreads();
  if (wave > 0) return;
  static_assert(kFewRows == kWave, "a lane per row");
  double s = lane < (int)a.M ? (double)losses[lane] : 0.0;
  int n = lane < (int)a.M ? in_rows[lane] : 0;
#pragma unroll
  for (int off = kWave / 2; off > 0; off >>= 1) {
    s += __shfl_xor(s, off, kWave);
    n += __shfl_xor(n, off, kWave);
  }
  if (lane == 0) *a.loss = n > 0 ? (float)(s / (double)n) : 0.f;
}

// ---- the gradient of the logits, one piece of the classes -------------------------------------------------
// One step of adding kCount values over the 32 lanes of half a wavefront: lanes whose bit kMask is set go on
// with the upper half of the values, the others with the lower half.
template <int kCount, int kMask>
__device__ inline void halve(float* v, int lane) {
  if constexpr (kCount > 1) {
#pragma unroll
    for (int k = 0; k < kCount / 2; ++k) {
      const bool up = (lane & kMask) != 0;
      const float send = up ? v[k] : v[k + kCount / 2];
      const float keep = up ? v[k + kCount / 2] : v[k];
      v[k] = keep + __shfl_xor(send, kMask, kWave);
    }
  } else {
    v[0] += __shfl_xor(v[0], kMask, kWave);
  }
}

// kKept: from the logits that stats has kept (of all classes), a tile per workgroup.
template <int TM, int TN, int WGM, int WGN, bool kKept>
__global__ __launch_bounds__(64 * WGM * WGN) void class_grad_kernel(ClassArgs a) {
  using T = Logits<TM, TN, WGM, WGN>;
  // beside the epilogue of a tile the next one's first slices are brought in; the epilogue has the ring's last place
  constexpr int kRoomBytes = WGN * T::BM * 4;
  static_assert(kRoomBytes <= T::kPlaceBytes, "room in a place");
  __shared__ __attribute__((aligned(1024))) u32x4 lds[(kKept ? kRoomBytes : T::kLdsBytes) / 16];
  const int count = uniform(*a.count);
  const bool wide = uniform(*a.wide) != 0;
  const float down = ldexpf(1.0f / kGScale, wide_exponent(a));
  const uint32_t tiles = T::tiles(count, a.piece_classes);
  // (with the first piece: the loss, by a workgroup that has no more tiles than any other)
  if (a.piece_first == 0 && blockIdx.x == gridDim.x - 1) join_losses(a, reinterpret_cast<double*>(lds));
  if (blockIdx.x >= tiles) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int wm = wave / WGN, wn = wave % WGN;
  float* columns = reinterpret_cast<float*>(lds + (kKept ? 0 : 4 * T::kSlots));
  typename T::Place next = T::place(a, blockIdx.x, tiles, count, a.piece_first, a.piece_classes);
  if (!kKept) T::template fill<0, 4>(next.source, lds);
  for (uint32_t id = blockIdx.x; id < tiles; id += gridDim.x) {
    const typename T::Place at = next;
    f32x16 acc[TM][TN];
    if constexpr (kKept) T::template logits_of<false>(a, at, wave, lane, acc);
    else T::template run<4>(at.source, lds, acc);
    const int c0 = at.c0, rows_v = at.rows_v, rows_n = at.rows_n;
    const int64_t n0 = at.n0;
    const int first = a.piece_first + c0 + wm * 32 * TM;
    if constexpr (!kKept) {
      __syncthreads();  // every wavefront is done with the ring
      if (id + gridDim.x < tiles) {
        next = T::place(a, id + gridDim.x, tiles, count, a.piece_first, a.piece_classes);
        T::template fill<0, 4>(next.source, lds);
      }
      add_bias<TM, TN>(a.bias, first, a.V, lane, acc);
    }

    const float uniform = a.smoothing / (float)a.V * kGScale, label = (1.0f - a.smoothing) * kGScale;
    const int half = 4 * (lane >> 5);
    const int classes = a.piece_first + a.piece_classes - first - half;  // of the piece, from this lane's first one on
    unroll<TN>([&](auto j_tag) {
      constexpr int j = decltype(j_tag)::value;
      const int r = wn * 32 * TN + j * 32 + (lane & 31);
      const bool live = r < rows_n;  // (a row that does not exist gets zeros)
      const float m = live ? a.row_max[n0 + r] : __builtin_inff(), inv = live ? a.row_inv[n0 + r] * kGScale : 0.f;
      const float off = live ? uniform : 0.f;
      const int y = live ? a.label_of[n0 + r] - first - half : -1;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = exp_neg(acc[i][j][e] - m) * inv - off;
      if (__any(y >= 0 && y < 32 * TM)) {  // few rows have their label among a wavefront's classes
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i][j][e] -= 32 * i + 8 * (e >> 2) + (e & 3) == y ? label : 0.f;
      }
      if (rows_v < T::BM) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[i][j][e] = 32 * i + 8 * (e >> 2) + (e & 3) < classes ? acc[i][j][e] : 0.f;
      }
      if (wide) T::template store_block<j, true>(a, at, wave, lane, acc, down);
      else T::template store_block<j>(a, at, wave, lane, acc);
    });
    if (a.column_sums) {
      // sums over the tile's rows: over j in registers, over 32 lanes by halving, over wavefronts through LDS
      float v[16 * TM];
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float s = acc[i][0][e];
#pragma unroll
          for (int j = 1; j < TN; ++j) s += acc[i][j][e];
          v[16 * i + e] = s;
        }
      constexpr int N = 16 * TM;
      halve<N, 16>(v, lane);
      halve<(N > 1 ? N / 2 : 1), 8>(v, lane);
      halve<(N > 2 ? N / 4 : 1), 4>(v, lane);
      halve<(N > 4 ? N / 8 : 1), 2>(v, lane);
      halve<(N > 8 ? N / 16 : 1), 1>(v, lane);
      // the index of what is left: the lane's bits from the top down, then k
      constexpr int kLeft = N >= 32 ? N / 32 : 1;
      int base = 0;
      {
        int n = N;
#pragma unroll
        for (int mask = 16; mask > 0; mask >>= 1)
          if (n > 1) {
            n >>= 1;
            if (lane & mask) base += n;
          }
      }
#pragma unroll
      for (int k = 0; k < kLeft; ++k) {
        const int at = base + k, i = at >> 4, e = at & 15;
        const int c = wm * 32 * TM + 32 * i + 8 * (e >> 2) + half + (e & 3);
        columns[wn * T::BM + c] = v[k];  // (lanes that hold the same sum write the same value)
      }
      __syncthreads();
      for (int c = tid; c < rows_v; c += T::kThreads) {
        float s = columns[c];
#pragma unroll
        for (int w = 1; w < WGN; ++w) s += columns[w * T::BM + c];
        a.column_sums[(int64_t)at.tn * a.piece_classes + c0 + c] = s;
      }
    }
    __syncthreads();
  }
}

// ---- the same from the exponentials that stats has kept of the first piece (no smoothing) ---------------------
// A workgroup: kKeptRows rows by 256 classes, eight classes of every eighth row per lane.
constexpr int kKeptThreads = 256, kKeptColumns = 256, kKeptRows = 32;
__global__ __launch_bounds__(kKeptThreads) void class_kept_kernel(ClassArgs a) {
  constexpr int kLanesPerRow = kKeptColumns / 8, kStep = kKeptThreads / kLanesPerRow, kTurns = kKeptRows / kStep;
  __shared__ double sums[kRowWaves];
  if (blockIdx.x == gridDim.x - 1) join_losses(a, sums);
  const int count = uniform(*a.count);
  const bool wide = uniform(*a.wide) != 0;
  const float down = ldexpf(1.0f / kGScale, wide_exponent(a));
  const uint32_t chunks = (uint32_t)((a.piece_classes + kKeptColumns - 1) / kKeptColumns);
  const int64_t row0 = (int64_t)(blockIdx.x / chunks) * kKeptRows + (int)threadIdx.x / kLanesPerRow;
  const int c = (int)(blockIdx.x % chunks) * kKeptColumns + (int)(threadIdx.x % kLanesPerRow) * 8;
  if (row0 >= count || c >= a.piece_ld) return;
  f16x8 e[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t)
    if (row0 + t * kStep < count) e[t] = *reinterpret_cast<const f16x8*>(a.g + (row0 + t * kStep) * a.piece_ld + c);
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int64_t row = row0 + t * kStep;
    if (row >= count) break;
    const float m = a.row_max[row], inv = a.row_inv[row];
    const int y = a.label_of[row] - c;
    const float scale = exp_neg(a.tops[row * a.top_ld + c / a.top_classes] - m) * inv;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = (float)e[t][k] * scale;
    if (y >= 0 && y < 8) {  // (the label's anew from its logit: what is left of 1 - exp / sum has no digits to lose)
      const float own = exp_neg(a.label_logit[row] - m) * (inv * kGScale) - kGScale;
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = k == y ? own : v[k];
    }
    u32x4 out;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < a.piece_classes ? v[k] : 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      out[k] = wide ? pack_bf16x2(v[2 * k] * down, v[2 * k + 1] * down) : half_pair(v[2 * k], v[2 * k + 1]);
    *reinterpret_cast<u32x4*>(a.g + row * a.piece_ld + c) = out;
  }
}

// ---- products ---------------------------------------------------------------------------------------
// Part s of the sums over k of A(m, k) B[k][n], B with k as its row number; k is split into parts.
struct Product {
  const uint16_t* A;       // "along": A[m][k]; otherwise A[k][m]
  const uint16_t* B;       // fp16 copy
  const uint16_t* B_wide;  // bf16, if that would not do
  int64_t lda, ldb;   // values from row to row
  int M, N, K, parts;
  const int32_t* rows;    // nullable: only so many m (device memory)
  const int32_t* depth;   // nullable: only so many k
  float* acc;             // [parts][M][N]
  bool accumulate;        // to what is there
  uint16_t* out;          // nullable: with one part, bf16 results instead of sums
  const int32_t* row_of;  // nullable: rows of `out` that the m go to
  bool by_weight;         // B is the weight's copy (tokens' otherwise)
};

template <int TM, int TN, int WGM, int WGN, bool kAlongA, bool kWide>
__device__ inline void product_tile(const ClassArgs& a, const Product& p, uint32_t block, uint32_t blocks, u32x4* lds) {
  using T = Tile<TM, TN, WGM, WGN, kAlongA, false, !kWide>;
  const int M = p.rows ? min(uniform(*p.rows), p.M) : p.M;
  const int K = p.depth ? min(uniform(*p.depth), p.K) : p.K;
  const uint32_t tiles_n = (uint32_t)((p.N + T::BN - 1) / T::BN);
  const uint32_t tiles = (uint32_t)((p.M + T::BM - 1) / T::BM) * tiles_n;
  const uint32_t id = xcd_remap(block, blocks);
  const uint32_t part = id / tiles, tile = id - part * tiles;
  const uint32_t tm = tile / tiles_n, tn = tile - tm * tiles_n;
  const int m0 = (int)tm * T::BM, n0 = (int)tn * T::BN;
  if (m0 >= M) return;
  const int rows_m = min(T::BM, M - m0), rows_n = min(T::BN, p.N - n0);
  // this part's share of the slices of k
  const int slices = (K + kSlice - 1) / kSlice, share = (slices + p.parts - 1) / p.parts;
  const int s0 = uniform(min((int)part * share, slices)), s1 = uniform(min(s0 + share, slices));
  const int64_t k0 = (int64_t)s0 * kSlice;
  const int depth = uniform(min(s1 * kSlice, K) - min(s0 * kSlice, K));
  const Operand A{kAlongA ? p.A + m0 * p.lda + k0 : p.A + k0 * p.lda + m0, p.lda, rows_m};
  const Operand B{(kWide ? p.B_wide : p.B) + k0 * p.ldb + n0, p.ldb, rows_n};
  f32x16 acc[TM][TN];
  T::template run<0>(T::source(A, B, depth), lds, acc);

  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int wm = wave / WGN, wn = wave % WGN;
  float* sums = p.acc + ((int64_t)part * p.M + m0) * p.N + n0;
  const bool final = p.out && p.parts == 1;
  if (!final || p.accumulate) {
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
          float* at = sums + (int64_t)r * p.N + c;
          if (p.accumulate) acc[i][j][e] += *at;
          if (!final) *at = acc[i][j][e];
        }
      }
    if (!final) return;
  }
  // results through a strip of LDS per wavefront, 32 rows at a time: 16 bytes per lane along a row (N is a multiple of 8)
  const Scale scaled = product_scale(a, p.by_weight);
  constexpr int kPitch = 32 * TN + 8;
  static_assert(WGM * WGN * 32 * kPitch * 2 <= T::kLdsBytes, "room for the strips");
  uint16_t* strip = reinterpret_cast<uint16_t*>(lds) + wave * 32 * kPitch;
  __syncthreads();  // every wavefront is done with the staged operands
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e)
        strip[(8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * kPitch + 32 * j + (lane & 31)] =
            (uint16_t)bf16_rne(scaled(acc[i][j][e]));
    __builtin_amdgcn_wave_barrier();
    constexpr int kLanesPerRow = 4 * TN, kRowsPerRep = kWave / kLanesPerRow;
#pragma unroll
    for (int rep = 0; rep < 32 / kRowsPerRep; ++rep) {
      const int sr = rep * kRowsPerRep + lane / kLanesPerRow, col = (lane % kLanesPerRow) * 8;
      const int r = wm * 32 * TM + 32 * i + sr, c = wn * 32 * TN + col;
      if (r >= rows_m || c >= rows_n) continue;
      const int64_t row = p.row_of ? p.row_of[m0 + r] : m0 + r;
      *reinterpret_cast<u32x4*>(p.out + row * p.N + n0 + c) = *reinterpret_cast<const u32x4*>(strip + sr * kPitch + col);
    }
  }
}

// The first `of_tokens` workgroups make g W, the others g^T x.
template <int TM, int TN, int WGM, int WGN>
__global__ __launch_bounds__(64 * WGM * WGN) void class_products_kernel(ClassArgs a, Product tokens, Product weight,
                                                                        uint32_t of_tokens) {
  __shared__ __attribute__((aligned(1024))) u32x4 lds[Tile<TM, TN, WGM, WGN, true, false, true>::kLdsBytes / 16];
  const bool wide = uniform(*a.wide) != 0, first = blockIdx.x < of_tokens;
  const uint32_t block = first ? blockIdx.x : blockIdx.x - of_tokens, blocks = first ? of_tokens : gridDim.x - of_tokens;
  if (wide) {
    if (first) product_tile<TM, TN, WGM, WGN, true, true>(a, tokens, block, blocks, lds);
    else product_tile<TM, TN, WGM, WGN, false, true>(a, weight, block, blocks, lds);
  } else {
    if (first) product_tile<TM, TN, WGM, WGN, true, false>(a, tokens, block, blocks, lds);
    else product_tile<TM, TN, WGM, WGN, false, false>(a, weight, block, blocks, lds);
  }
}

// ---- finish -----------------------------------------------------------------------------------------
constexpr int kFinishThreads = 256;

// eight values at `at` of the first of `parts` arrays that lie `stride` values apart, added up and scaled, as bf16
__device__ inline u32x4 joined(const float* p, int64_t at, int64_t stride, int parts, const Scale& scaled) {
  f32x4 lo = f32x4{0.f, 0.f, 0.f, 0.f}, hi = lo;
  for (int s = 0; s < parts; ++s) {
    lo += *reinterpret_cast<const f32x4*>(p + s * stride + at);
    hi += *reinterpret_cast<const f32x4*>(p + s * stride + at + 4);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    lo[k] = scaled(lo[k]);
    hi[k] = scaled(hi[k]);
  }
  return u32x4{pack_bf16x2(lo.x, lo.y), pack_bf16x2(lo.z, lo.w), pack_bf16x2(hi.x, hi.y), pack_bf16x2(hi.z, hi.w)};
}

// Workgroups [0, for_bias): grad_bias of the piece, 64 classes by four wavefronts.  [for_bias, + for_weight):
// grad_weight of the piece from its parts.  The rest: grad_tokens from its parts.
__global__ __launch_bounds__(kFinishThreads) void class_finish_kernel(ClassArgs a, uint32_t for_bias, uint32_t for_weight) {
  const int per_row = a.D / 8;
  uint32_t block = blockIdx.x;
  if (block < for_bias) {
    __shared__ float part[4][64];
    const int col = threadIdx.x % 64, r = threadIdx.x / 64;
    const int c = (int)block * 64 + col;
    const int tiles = (*a.count + a.grad_rows - 1) / a.grad_rows;
    float s = 0.f;
    if (c < a.piece_classes)
      for (int t = r; t < tiles; t += 4) s += a.column_sums[(int64_t)t * a.piece_classes + c];
    part[r][col] = s;
    __syncthreads();
    if (r == 0 && c < a.piece_classes)
      a.grad_bias[a.piece_first + c] =
          (float)((double)((part[0][col] + part[1][col]) + (part[2][col] + part[3][col])) *
                  (grad_factor(a) / (double)kGScale));
    return;
  }
  block -= for_bias;
  if (block < for_weight) {
    const Scale scaled = product_scale(a, false);
    const int64_t total = (int64_t)a.piece_classes * per_row;
    for (int64_t i = (int64_t)block * kFinishThreads + threadIdx.x; i < total; i += (int64_t)for_weight * kFinishThreads)
      *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.grad_weight) + (int64_t)a.piece_first * a.D + i * 8) =
          joined(a.weight_acc, i * 8, (int64_t)a.piece_classes * a.D, a.weight_parts, scaled);
    return;
  }
  block -= for_weight;
  const uint32_t blocks = gridDim.x - for_bias - for_weight;
  const Scale scaled = product_scale(a, true);
  const int64_t total = (int64_t)*a.count * per_row;
  for (int64_t i = (int64_t)block * kFinishThreads + threadIdx.x; i < total; i += (int64_t)blocks * kFinishThreads) {
    const int64_t slot = i / per_row;
    const int c = (int)(i - slot * per_row) * 8;
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(a.grad_tokens) + (int64_t)a.row_of[slot] * a.D + c) =
        joined(a.tokens_acc, slot * a.D + c, a.M * a.D, a.tokens_parts, scaled);
  }
}

}  // namespace

// ---- host ---------------------------------------------------------------------------------------------
namespace {

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t up256(size_t n) { return (n + 255) & ~size_t(255); }

// Side of the tiles of logits: the largest of which there are enough.  Loss alone, us for 64 / 128 / 256: 2048 x 768 over
// 1000 classes 21.9 / 24.5 / 36, 4096 28.5 / 27.6 / 41, 8192 43 / 36.4 / 43.5, 16384 68 / 54.4 / 50.0; 1024 x 1024
// over 8192 42.6 / 34.2 / 39.8; 512 x 768 over 21,841 45 / 36.2 / 35.6; 2048 x 1024 over 32,003 228 / 166 / 134.
int logits_side(int64_t M, int V) {
  if (M <= 64 || ceil_div(M, 128) * ceil_div(V, 128) < 192) return 64;
  if (M <= 256 || ceil_div(M, 256) * ceil_div(V, 256) < 256) return 128;
  return 256;
}

// Parts that k is split into: as many as give every compute unit a tile, of four slices at least.
int product_parts(int64_t M, int N, int64_t K, int side, int64_t slots) {
  const int64_t tiles = ceil_div(M, side) * ceil_div(N, side);
  int64_t parts = slots / tiles;
  if (parts > ceil_div(K, kSlice) / 4) parts = ceil_div(K, kSlice) / 4;
  return parts < 1 ? 1 : (int)parts;
}

}  // namespace

// Side of the tiles of the two products of a piece, the largest of which there are enough.  Whole calls, us for 64 / 128 /
// 256: 512 x 768 over 1000 classes 43.8 / 47.0 / 60, 1024 44.1 / 48.3 / 61, 2048 59.1 / 60.3 / 70, 4096 75.8 / 69.4 / 78.5,
// 16384 199 / 177 / 182; 128 x 1024 over 32,003 128 / 119 / 136, 512 x 768 over 21,841 149 / 137 / 137, 2048 x 1024 over
// 32,003 714 / 598 / 555.
static int products_side(int64_t M, int D, int V) {
  const auto tiles = [&](int side) { return (ceil_div(M, side) + ceil_div(V, side)) * ceil_div(D, side); };
  if (M <= 64 || V <= 64 || tiles(128) < 128) return 64;
  return M <= 256 || tiles(256) < 256 ? 128 : 256;
}

// What stats keeps for the gradient, so that the logits need not be made again.  Without bias and smoothing: exponentials of
// the first piece, as fp16 in the place of its g.  Else, as a bias's gradient is to have single precision and p - s / V
// may cancel: the logits in fp32 if they fit the caches with room to spare, 64 MiB.  us of whole calls with the logits made
// again / in fp32 / exponentials: 768 values, 1000 classes, 4096 rows 72.2 / 67.1 / 64.8, 16384 179 / 175 / 163, 32768
// 320 / 328 / 284; 512 x 768 over 32,003 182 / 172 / 159, 16384 x 1024 over 32,003 4070 / - / 3390.
constexpr int64_t kMostLogits = int64_t(1) << 24;

ClassPlan class_plan(int64_t M, int D, int V, bool bias, bool smooth, bool grad) {
  ClassPlan p{};
  p.few = !grad && M <= kFewRows;
  p.side = logits_side(M, V);
  p.stat_tiles = (int)ceil_div(V, p.side);
  p.pack_rows = (int)ceil_div(ceil_div(M, 1024), 16) * 16;
  p.row_blocks = (int)(ceil_div(M, kRowWaves) < 2048 ? ceil_div(M, kRowWaves) : 2048);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t was = at;
    at += up256(bytes);
    return was;
  };
  const size_t m = (size_t)M;
  p.stats = take(m * p.stat_tiles * 8);
  p.logit_sums = take(smooth ? m * p.stat_tiles * 4 : 0);
  p.label_logit = take(m * 4);
  if (!p.few) {
    p.count = take(2 * sizeof(int32_t));
    p.wide = p.count + sizeof(int32_t);  // (in one cache line: both are read where a kernel begins)
    p.label_of = take(m * 4);
    p.row_of = take(m * 4);
    p.packed = take(m * D * 2);
    p.partials = take((size_t)p.row_blocks * 8);
  }
  if (grad) {
    // g of a piece takes at most 1 GiB, or 1024 classes
    const int64_t most = (int64_t(1) << 29) / M / 256 * 256;
    p.piece = (int)(most < 1024 ? 1024 : most < V ? most : V);
    if (p.piece > V) p.piece = V;
    p.piece_ld = (int)ceil_div(p.piece, 64) * 64;
    const int64_t padded = ceil_div(M, p.side) * ceil_div(V, p.side) * p.side * p.side;
    p.keep = !bias && !smooth ? kKeepExp : padded <= kMostLogits ? kKeepLogits : kKeepNone;
    p.top_ld = (int)ceil_div(p.piece, p.side) * 2;
    p.logits = take(p.keep == kKeepLogits ? (size_t)padded * 4 : 0);
    p.tops = take(p.keep == kKeepExp ? m * p.top_ld * 4 : 0);
    p.products_side = products_side(M, D, p.piece);
    // (the tiles for grad_weight alone fill the compute units: the others, in the same launch, are split less)
    const bool many = ceil_div(p.piece, p.products_side) * ceil_div(D, p.products_side) >= 256;
    p.tokens_parts = product_parts(M, D, p.piece, p.products_side, many ? 128 : 256);
    p.weight_parts = product_parts(p.piece, D, M, p.products_side, 256);
    const int64_t for_weight = ceil_div((int64_t)V * D / 8, kPackThreads * 4);
    const int num_weight_ranges = (int)(for_weight < 1024 ? for_weight : 1024);
    p.num_ranges = (int)ceil_div(M, p.pack_rows) + num_weight_ranges;
    p.ranges = take((size_t)p.num_ranges * 4);
    p.row_max = take(m * 4);
    p.row_inv = take(m * 4);
    p.half_tokens = take(m * D * 2);
    p.half_weight = take((size_t)V * D * 2);
    p.g = take(m * p.piece_ld * 2);
    p.column_sums = take(bias ? (size_t)ceil_div(M, p.side) * p.piece * 4 : 0);
    if (p.tokens_parts > 1 || p.piece < V) p.tokens_acc = take(m * D * 4 * p.tokens_parts);
    if (p.weight_parts > 1) p.weight_acc = take((size_t)p.piece * D * 4 * p.weight_parts);
  }
  p.bytes = at;
  return p;
}

namespace {
// Workgroups that walk the tiles: as many as fit on the compute units, or one per tile.
template <class T>
uint32_t walkers(int64_t M, int classes) {
  const int64_t tiles = ceil_div(M, T::BN) * ceil_div(classes, T::BM);
  constexpr int kPerUnit = 160 * 1024 / T::kLdsBytes;
  return (uint32_t)(tiles < 256 * kPerUnit ? tiles : 256 * kPerUnit);
}
template <int TM, int TN, int WGM, int WGN>
void launch_stats(const ClassArgs& a, int keep, hipStream_t stream) {
  using T = Logits<TM, TN, WGM, WGN>;
  const dim3 grid(walkers<T>(a.M, a.V)), block(T::kThreads);
  if (keep == kKeepLogits) hipLaunchKernelGGL((class_stats_kernel<TM, TN, WGM, WGN, kKeepLogits>), grid, block, 0, stream, a);
  else if (keep == kKeepExp) hipLaunchKernelGGL((class_stats_kernel<TM, TN, WGM, WGN, kKeepExp>), grid, block, 0, stream, a);
  else hipLaunchKernelGGL((class_stats_kernel<TM, TN, WGM, WGN, kKeepNone>), grid, block, 0, stream, a);
}
void launch_kept(const ClassArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(class_kept_kernel, dim3((uint32_t)(ceil_div(a.M, kKeptRows) * ceil_div(a.piece_classes, kKeptColumns))),
                     dim3(kKeptThreads), 0, stream, a);
}
template <int TM, int TN, int WGM, int WGN>
void launch_grad(const ClassArgs& a, int keep, hipStream_t stream) {
  using T = Logits<TM, TN, WGM, WGN>;
  if (keep == kKeepLogits) {
    const dim3 grid((uint32_t)(ceil_div(a.M, T::BN) * ceil_div(a.V, T::BM)));
    hipLaunchKernelGGL((class_grad_kernel<TM, TN, WGM, WGN, true>), grid, dim3(T::kThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL((class_grad_kernel<TM, TN, WGM, WGN, false>), dim3(walkers<T>(a.M, a.piece_classes)),
                       dim3(T::kThreads), 0, stream, a);
  }
}
template <int TM, int TN, int WGM, int WGN>
void launch_products(const ClassArgs& a, const Product& tokens, const Product& weight, hipStream_t stream) {
  constexpr int BM = 32 * TM * WGM, BN = 32 * TN * WGN;
  const auto blocks = [&](const Product& p) {
    return p.A ? (uint32_t)(ceil_div(p.M, BM) * ceil_div(p.N, BN) * p.parts) : 0u;
  };
  const uint32_t of_tokens = blocks(tokens), of_weight = blocks(weight);
  hipLaunchKernelGGL((class_products_kernel<TM, TN, WGM, WGN>), dim3(of_tokens + of_weight), dim3(64 * WGM * WGN), 0,
                     stream, a, tokens, weight, of_tokens);
}
uint32_t finish_blocks(int64_t values) {
  const int64_t blocks = ceil_div(values / 8, kFinishThreads);
  return (uint32_t)(blocks < 1 ? 1 : blocks < 2048 ? blocks : 2048);
}
}  // namespace

hipError_t launch_class_loss(ClassArgs a, const ClassPlan& p, hipStream_t stream) {
  a.pack_rows = p.pack_rows;
  a.stat_tiles = p.stat_tiles;
  a.pack_blocks = (int)ceil_div(a.M, p.pack_rows);
  a.num_ranges = p.num_ranges;
  a.row_blocks = p.row_blocks;
  const bool grad = a.ranges != nullptr;
  if (!p.few)
    hipLaunchKernelGGL(class_pack_kernel, dim3((uint32_t)(grad ? p.num_ranges : a.pack_blocks)), dim3(kPackThreads), 0,
                       stream, a);
  a.piece_first = 0;
  a.piece_classes = p.piece;
  a.piece_ld = p.piece_ld;
  a.top_ld = p.top_ld;
  a.top_classes = p.side / 2;
  if (p.side == 256) launch_stats<4, 2, 2, 4>(a, p.keep, stream);
  else if (p.side == 128) launch_stats<2, 1, 2, 4>(a, p.keep, stream);
  else launch_stats<1, 1, 2, 2>(a, p.keep, stream);
  if (p.few) {
    hipLaunchKernelGGL(class_few_rows_kernel, dim3(1), dim3(kFewThreads), 0, stream, a);
    return hipGetLastError();
  }
  const int64_t for_halves = ceil_div((a.M + a.V) * a.D / 8, kRowThreads);
  hipLaunchKernelGGL(class_rows_kernel,
                     dim3((uint32_t)(p.row_blocks + (grad ? (for_halves < 4096 ? for_halves : 4096) : 0))),
                     dim3(kRowThreads), 0, stream, a);
  if (!grad) hipLaunchKernelGGL(class_loss_kernel, dim3(1), dim3(kRowThreads), 0, stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !grad) return e;

  a.grad_rows = p.side;
  a.tokens_parts = p.tokens_parts;
  a.weight_parts = p.weight_parts;
  if (!a.grad_bias) a.column_sums = nullptr;
  for (int first = 0; first < a.V; first += p.piece) {
    a.piece_first = first;
    a.piece_classes = a.V - first < p.piece ? a.V - first : p.piece;
    const bool last = first + a.piece_classes == a.V;
    if (p.keep == kKeepExp && first == 0) launch_kept(a, stream);
    else if (p.side == 256) launch_grad<4, 2, 2, 4>(a, p.keep, stream);
    else if (p.side == 128) launch_grad<2, 1, 2, 4>(a, p.keep, stream);
    else launch_grad<1, 1, 2, 2>(a, p.keep, stream);
    Product tokens{}, weight{};
    if (a.grad_tokens) {
      // rows: packed rows; k: classes of the piece (g holds zeros up to a multiple of 8 behind them)
      tokens.A = a.g, tokens.lda = p.piece_ld;
      tokens.B = a.half_weight + (int64_t)first * a.D, tokens.ldb = a.D, tokens.by_weight = true;
      tokens.B_wide = static_cast<const uint16_t*>(a.weight) + (int64_t)first * a.D;
      tokens.M = (int)a.M, tokens.N = a.D, tokens.K = a.piece_classes, tokens.rows = a.count;
      tokens.parts = p.tokens_parts, tokens.acc = a.tokens_acc, tokens.accumulate = first > 0;
      if (last) tokens.out = static_cast<uint16_t*>(a.grad_tokens), tokens.row_of = a.row_of;
    }
    if (a.grad_weight) {
      weight.A = a.g, weight.lda = p.piece_ld, weight.B = a.half_tokens, weight.ldb = a.D;
      weight.B_wide = a.packed;
      weight.M = a.piece_classes, weight.N = a.D, weight.K = (int)a.M, weight.depth = a.count;
      weight.parts = p.weight_parts, weight.acc = a.weight_acc;
      weight.out = static_cast<uint16_t*>(a.grad_weight) + (int64_t)first * a.D;
    }
    if (a.grad_tokens || a.grad_weight) {
      if (p.products_side == 256) launch_products<4, 2, 2, 4>(a, tokens, weight, stream);
      else if (p.products_side == 128) launch_products<2, 1, 2, 4>(a, tokens, weight, stream);
      else launch_products<1, 1, 2, 2>(a, tokens, weight, stream);
    }
    const uint32_t for_bias = a.grad_bias ? (uint32_t)ceil_div(a.piece_classes, 64) : 0;
    const uint32_t for_weight =
        a.grad_weight && p.weight_parts > 1 ? finish_blocks((int64_t)a.piece_classes * a.D) : 0;
    const uint32_t for_tokens = a.grad_tokens && p.tokens_parts > 1 && last ? finish_blocks(a.M * a.D) : 0;
    if (for_bias + for_weight + for_tokens > 0)
      hipLaunchKernelGGL(class_finish_kernel, dim3(for_bias + for_weight + for_tokens), dim3(kFinishThreads), 0, stream, a,
                         for_bias, for_weight);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace mae

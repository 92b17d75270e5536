// Tiles of products of bf16 or fp16 matrices on the matrix cores (v_mfma_f32_32x32x16_bf16, _f16, fp32
// sums): the main loop that the linear loss and the gradient of the patch embedding share.  Each kernel
// has its own epilogue.
//
//   C[m, n] = sum over k of A(m, k) B(n, k)
//
// Either operand may lie in memory with its k contiguous (rows of m or n: "along k") or with its k as
// the row number (columns of m or n: "across k", as both operands of a weight's gradient do).  The
// slices of both go to LDS as they lie in memory (global_load_lds_dwordx4, no trip through registers).
// An operand along k is read back with ds_read_b128: a lane takes 8 consecutive k of one row.  One
// across k is read with ds_read_b64_tr_b16: 16 lanes read four rows of 16 columns and each gets the four
// k of one column, so that two of them give the same 8 consecutive k, and nothing is transposed in memory.
//
// LDS layout of a slice of 64 k (both kinds take 128 bytes per m or n).  Along k: a row of eight
// 16-byte chunks, the chunk's place XORed with bits 1..3 of the row: 16 rows of one chunk column fall
// into 16 different 16-byte bank groups.  Across k: 64 rows of R columns; half a wavefront reads four
// consecutive rows, 64 bytes of each, so the place of a 64-byte block is XORed with the row's number in
// its group of four (for R = 64, whose rows are half a turn of the banks, with bit 1 of it): the four
// blocks fall into four different quarters of the banks.  Direct loads write lane l to slot l, so
// the swizzle is applied on the global side.
//
// Fragment reads are inline assembly, so that the compiler does not make each of them wait for every
// direct load in flight; the code waits on lgkmcnt itself before it uses what was read, in straight lines, and
// every build goes through the assembly of the library for registers that are touched in between (spilled or moved,
// as under more register pressure they are) and refuses them.
//
// What bounds it.  A slice of a 256 x 256 tile takes 1.62 us on the 256 compute units together (1.3 PFLOP/s): its
// multiplies alone take 1.00 us at 2.28 GHz, with the reads beside them 1.31 us at 1.8 GHz, with the loads too 1.62 us at
// 1.45 to 1.75 GHz, where 2048 of 2350 to 2800 cycles multiply: the card's clock falls with the power of the three together.
// Tried: four wavefronts of 128 x 128 (a third less to read, but a wavefront alone on its SIMD waits for its own
// loads: 1.7 us), loads at other multiplies for each wavefront (branches: 1.85 us), reads behind the first one, two or four of
// eight multiplies instead of six (the same), rows on an odd number of lines (the same).
#pragma once

#include "mae_device.hpp"

namespace mae {
namespace mm {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kSlice = 64;  // k per stage

// What lanes fetch in place of what lies behind the end of k.
static __device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};

template <int kOff>
__device__ static inline u32x4 read_along(uint32_t addr) {
  u32x4 v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(kOff) : "memory");
  return v;
}
template <int kOff>
__device__ static inline u32x2 read_across(uint32_t addr) {
  u32x2 v;
  asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(kOff) : "memory");
  return v;
}

// s_waitcnt immediate: vmcnt(n) and lgkmcnt(0), expcnt not waited for
constexpr int wait_vm(int n) { return (n & 0xF) | ((n >> 4) << 14) | 0x0070; }

// A value that is the same in all lanes, as one that the compiler knows to be so.
__device__ static inline int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

__device__ static inline const char* uniform(const uint16_t* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  return reinterpret_cast<const char*>((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// Tiles in the order in which workgroups take them: the rows of the grid of tiles in groups of kGroup, column by
// column within a group, so that the 32 tiles that an XCD works on at a time share kGroup panels of one operand and
// few of the other.  (A linear loss and its gradients of 8184 rows and 32003 classes of 1024 values, on one card: 2 panels
// 3.74 ms, 4 and 8 3.73, 6 3.74, 16 3.76: the loads come early enough for any of them.)
constexpr uint32_t kGroup = 8;
__device__ static inline void grouped(uint32_t id, uint32_t rows, uint32_t cols, uint32_t* row, uint32_t* col) {
  const uint32_t group = id / (kGroup * cols);
  const uint32_t first = group * kGroup, size = min(kGroup, rows - first);
  const uint32_t in = id - first * cols;
  *col = in / size;
  *row = first + in - *col * size;
}

template <int v>
struct Tag {
  static constexpr int value = v;
};
template <int N, class F>
__device__ static inline void unroll(F&& f) {
  if constexpr (N > 0) {
    unroll<N - 1>(f);
    f(Tag<N - 1>{});
  }
}

// One operand of a tile.
struct Operand {
  const uint16_t* p;  // along k: element (first row of the tile, first k); across k: (first k, first column)
  int64_t ld;         // elements from row to row
  int limit;          // rows (along k) or columns (across k) of the tile that exist, at least 1
};

// A tile of (32 TM WGM) x (32 TN WGN) results by WGM x WGN wavefronts, square.
// Requirements: along k: k up to a multiple of 8 can be read and holds finite values where the other
// operand's are zero; across k: whole chunks of 8 columns up to `limit` rounded up to 8 can be read
// in every row.  Addresses are multiples of 4 bytes.
//
// LDS is a ring of five places for a slice of one operand: A0 B0 A1 B1 A2, then B2 in A0's place, A3 in B0's and so
// on.  When slice s is done, B of s + 2 is requested first, which has the whole of s + 1 to arrive, then A of
// s + 3, which has two slices.  (With two places for both operands together, which is what fits with 256 x 256 results, the
// last loads of a slice have a third of one.)
template <int TM, int TN, int WGM, int WGN, bool kAlongA, bool kAlongB, bool kHalf = false>
struct Tile {
  static constexpr int kThreads = 64 * WGM * WGN;
  static constexpr int BM = 32 * TM * WGM, BN = 32 * TN * WGN;
  static_assert(BM == BN, "places of the ring hold either operand");
  static constexpr int kSlots = BM * 8;         // 16-byte slots of a place
  static constexpr int NL = kSlots / kThreads;  // direct loads per lane and place
  static constexpr int kPlaceBytes = kSlots * 16;
  static constexpr int kPlaces = 5;
  static constexpr int kLdsBytes = kPlaces * kPlaceBytes;
  static_assert(kSlots % kThreads == 0 && NL % 2 == 0, "halves of whole wave-wide loads");
  static_assert(3 * NL <= 63, "vmcnt range");

  // what the chunk's place is XORed with in row k of an operand across k
  template <int R>
  __device__ static inline int swizzle(int k) {
    return R >= 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
  }
  // which chunk of its row slot `s` of an operand of R rows or columns holds, and that row
  template <int R, bool kAlong>
  __device__ static inline void slot_place(int s, int* row, int* chunk) {
    if (kAlong) {
      *row = s / 8;
      *chunk = (s % 8) ^ ((*row >> 1) & 7);
    } else {
      constexpr int kChunks = R / 8;
      *row = s / kChunks;
      *chunk = (s % kChunks) ^ swizzle<R>(*row);
    }
  }

  // What a lane needs to bring in the slices of a tile's operands.
  struct Source {
    const char *a, *b;           // first slice
    uint32_t step_a, step_b;     // bytes from slice to slice
    uint32_t off_a[NL], off_b[NL];  // this lane's chunks of a slice
    int K, nk, tail;
  };
  __device__ static inline Source source(const Operand& A, const Operand& B, int K) {
    const int lane = threadIdx.x % kWave;
    const int wave = uniform((int)threadIdx.x / kWave);
    Source s;
    s.a = uniform(A.p);
    s.b = uniform(B.p);
    s.step_a = kAlongA ? kSlice * 2 : kSlice * 2 * (uint32_t)uniform((int)A.ld);
    s.step_b = kAlongB ? kSlice * 2 : kSlice * 2 * (uint32_t)uniform((int)B.ld);
    s.K = K;
    s.nk = (K + kSlice - 1) / kSlice;
    s.tail = K % kSlice;
#pragma unroll
    for (int q = 0; q < NL; ++q) {
      const int slot = (wave * NL + q) * kWave + lane;
      int row, chunk;
      slot_place<BM, kAlongA>(slot, &row, &chunk);
      if (kAlongA) row = min(row, A.limit - 1);
      else if (8 * chunk >= A.limit) chunk = 0;  // (any columns that exist: their results are not used)
      s.off_a[q] = (uint32_t)(row * A.ld + 8 * chunk) * 2u;
      slot_place<BN, kAlongB>(slot, &row, &chunk);
      if (kAlongB) row = min(row, B.limit - 1);
      else if (8 * chunk >= B.limit) chunk = 0;
      s.off_b[q] = (uint32_t)(row * B.ld + 8 * chunk) * 2u;
    }
    return s;
  }

  // Loads q0 .. q1 of a slice of one operand into a place of the ring.
  template <bool kA>
  __device__ static inline void issue(const Source& s, u32x4* lds, int it, int place, int q0, int q1) {
    constexpr bool kAlong = kA ? kAlongA : kAlongB;
    const int lane = threadIdx.x % kWave;
    const int wave = uniform((int)threadIdx.x / kWave);
    u32x4* dst = lds + place * kSlots + wave * NL * kWave;
    const char* base = (kA ? s.a : s.b) + (uint64_t)(uint32_t)it * (kA ? s.step_a : s.step_b);
    asm("" : "+s"(base));
#pragma unroll
    for (int q = q0; q < q1; ++q) {
      const char* src = base + (kA ? s.off_a[q] : s.off_b[q]);
      if ((it + 1) * kSlice > s.K) {  // (a load for every lane, whatever it holds: the waits count them)
        int row, chunk;
        slot_place<BM, kAlong>((wave * NL + q) * kWave + lane, &row, &chunk);
        if (kAlong ? 8 * chunk >= s.tail : row >= s.tail) src = reinterpret_cast<const char*>(&kZeros);
      }
      __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)src,
                                       (void __attribute__((address_space(3)))*)(dst + q * kWave), 16, 0, 0);
    }
  }
  // Slices `from` .. `to` of the ring's first five (A0 B0 A1 B1 A2), as far as there are any.
  template <int kFrom, int kTo>
  __device__ static inline void fill(const Source& s, u32x4* lds) {
    unroll<kTo - kFrom>([&](auto tag) {
      constexpr int n = kFrom + decltype(tag)::value;
      if (n / 2 < s.nk) issue<n % 2 == 0>(s, lds, n / 2, n, 0, NL);
    });
  }

  // A second operand that is not in memory: row k of it is 1 at column ids[k] - first and 0 elsewhere (ids null: at
  // column 0), so that the product adds up the columns of A whose k has the same id.  ids outside [0, count) are
  // clamped into it.
  struct Ones {
    const int32_t* ids;  // of this tile's first k
    int first, count;
  };

  // The tile's sums.  kAhead: slices of the ring that fill() has been called for already (0 or 4); no
  // wavefront uses what the others' places hold any more.
  // kOnes: B is made in LDS: the ring's places 0 to 2 are A's, 3 and 4 hold B, zero but for 64 values that the first
  // wavefront moves from slice to slice.
  template <int kAhead, bool kOnes = false>
  __device__ static inline void run(const Source& src, u32x4* lds, f32x16 (&acc)[TM][TN], Ones ones = {}) {
    static_assert(!kOnes || (kAhead == 0 && !kAlongB && !kHalf), "bf16 ones, across k");
    const int lane = threadIdx.x % kWave;
    const int wave = uniform((int)threadIdx.x / kWave);
    const int wm = wave / WGN, wn = wave % WGN;
    const int nk = src.nk;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    if (nk == 0) return;

    // fragment addresses inside a place (bytes)
    const uint32_t lds_base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) u32x4*)lds;
    const uint32_t c0 = (uint32_t)((lane >> 5) ^ ((lane >> 1) & 7)) * 16u;
    const int g = lane >> 4, i16 = lane & 15;
    uint32_t fa_at[kAlongA ? 1 : TM], fb_at[kAlongB ? 1 : TN];
    if constexpr (kAlongA) {
      fa_at[0] = lds_base + (uint32_t)(wm * 32 * TM + (lane & 31)) * 128u + c0;
    } else {
#pragma unroll
      for (int t = 0; t < TM; ++t) fa_at[t] = lds_base + across_at<BM>(wm * TM + t, g, i16);
    }
    if constexpr (kAlongB) {
      fb_at[0] = lds_base + (uint32_t)(wn * 32 * TN + (lane & 31)) * 128u + c0;
    } else {
#pragma unroll
      for (int t = 0; t < TN; ++t) fb_at[t] = lds_base + across_at<BN>(wn * TN + t, g, i16);
    }

    u32x4 fa[2][TM], fb[2][TN];
    // Read number r of sub-step ks: the operands' reads one after the other.
    constexpr int kReadsA = kAlongA ? TM : 2 * TM, kReadsB = kAlongB ? TN : 2 * TN, kReads = kReadsA + kReadsB;
    auto read_one = [&](uint32_t a_bytes, uint32_t b_bytes, auto ks_tag, auto r_tag, int set) {
      constexpr int ks = decltype(ks_tag)::value, r = decltype(r_tag)::value;
      if constexpr (r < kReadsA) read_part<BM, kAlongA, ks, r>(fa_at, a_bytes, fa[set]);
      else read_part<BN, kAlongB, ks, r - kReadsA>(fb_at, b_bytes, fb[set]);
    };
    auto read_frags = [&](int a_place, int b_place, auto ks_tag, int set) {
      unroll<kReads>([&](auto r) {
        read_one((uint32_t)a_place * kPlaceBytes, (uint32_t)b_place * kPlaceBytes, ks_tag, r, set);
      });
      __builtin_amdgcn_sched_barrier(0);
    };
    auto arrive = [&](int set) {
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
      for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(fa[set][i]));
#pragma unroll
      for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(fb[set][j]));
    };
    auto multiply_one = [&](int set, int i, int j) {
      if constexpr (kHalf)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, fa[set][i]),
                                                           __builtin_bit_cast(f16x8, fb[set][j]), acc[i][j], 0, 0, 0);
      else
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[set][i]),
                                                            __builtin_bit_cast(bf16x8, fb[set][j]), acc[i][j], 0, 0, 0);
    };
    auto multiply = [&](int set) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) multiply_one(set, i, j);
    };
    // The multiplies of one set of fragments; behind each of the first ones a share of the reads of the other set
    // (sub-step ks of the slice in these places), behind the last ones `loads`, one by one.
    constexpr int kMul = TM * TN;
    constexpr int kReadMul = kMul >= 8 ? kMul * 3 / 4 : kMul;  // multiplies that reads follow
    auto step = [&](int set, int a_place, int b_place, auto ks_tag, auto&& load) {
      const uint32_t a_bytes = (uint32_t)a_place * kPlaceBytes, b_bytes = (uint32_t)b_place * kPlaceBytes;
      unroll<kMul>([&](auto m_tag) {
        constexpr int m = decltype(m_tag)::value;
        multiply_one(set, m / TN, m % TN);
        __builtin_amdgcn_sched_barrier(0);
        constexpr int r0 = m < kReadMul ? kReads * m / kReadMul : kReads;
        constexpr int r1 = m < kReadMul ? kReads * (m + 1) / kReadMul : kReads;
        unroll<r1 - r0>([&](auto r) {
          read_one(a_bytes, b_bytes, ks_tag, Tag<r0 + decltype(r)::value>{}, set ^ 1);
        });
        constexpr int l0 = (NL / 2) * m / kMul, l1 = (NL / 2) * (m + 1) / kMul;
        if constexpr (l1 > l0) load(l0, l1);
        __builtin_amdgcn_sched_barrier(0);
      });
      arrive(set ^ 1);
    };

    // ones: byte of this lane's 1 in either place (-1: none), and the id of the slice after the last one made
    int at_one[2] = {-1, -1}, next_id = 0;
    auto load_id = [&](int it) {
      const int k = it * kSlice + lane;
      if (ones.ids) next_id = ones.ids[min(k, src.K - 1)];
    };
    auto make_ones = [&](int it) {  // (next_id is that of slice `it`)
      if (wave != 0) return;
      char* place = reinterpret_cast<char*>(lds + (3 + (it & 1)) * kSlots);
      const int old = (it & 1) ? at_one[1] : at_one[0];
      if (old >= 0) *reinterpret_cast<uint16_t*>(place + old) = 0;
      const int c = min(max(next_id, 0), ones.count - 1) - ones.first;
      int at = -1;
      if (it * kSlice + lane < src.K && c >= 0 && c < BN) {
        at = lane * BN * 2 + (((c >> 3) ^ swizzle<BN>(lane)) * 16) + (c & 7) * 2;
        *reinterpret_cast<uint16_t*>(place + at) = 0x3F80;
      }
      if (it & 1) at_one[1] = at;
      else at_one[0] = at;
      if (it + 1 < nk) load_id(it + 1);
    };

    if constexpr (kOnes) {
      unroll<3>([&](auto n) {
        if (decltype(n)::value < nk) issue<true>(src, lds, decltype(n)::value, decltype(n)::value, 0, NL);
      });
      for (int i = threadIdx.x; i < 2 * kSlots; i += kThreads) lds[3 * kSlots + i] = u32x4{0u, 0u, 0u, 0u};
      load_id(0);
      __syncthreads();
      make_ones(0);
      __syncthreads();  // (waits for the loads of all three slices as well)
    } else {
      fill<kAhead, 5>(src, lds);
      // slice 0 has landed; of what was issued here the rest may be on its way
      static_assert(kAhead == 0 || kAhead == 4, "none, or whole slices of both operands");
      constexpr int kRest = kAhead == 4 ? 1 : 3;
      if (nk > 2) __builtin_amdgcn_s_waitcnt(wait_vm(kRest * NL));
      else if (nk > 1) __builtin_amdgcn_s_waitcnt(wait_vm((kRest - 1) * NL));
      else __builtin_amdgcn_s_waitcnt(wait_vm(0));
      __builtin_amdgcn_s_barrier();
    }
    read_frags(0, kOnes ? 3 : 1, Tag<0>{}, 0);
    arrive(0);

    // A slice is four sub-steps of 16 k; the fragments of a sub-step are read while the one before it is
    // multiplied, across slices too; the loads that refill the ring are spread over all four.
    // Places of the ring: A and B of this slice, of the next one, and A of the one after it.
    auto after = [](int place) { return place + 1 == kPlaces ? 0 : place + 1; };
    int pa = 0, pb = kOnes ? 3 : 1;
    for (int it = 0; it + 1 < nk; ++it) {
      int na, nb, ma;
      if constexpr (kOnes) {
        na = pa == 2 ? 0 : pa + 1;
        nb = 7 - pb;
        ma = na == 2 ? 0 : na + 1;
        make_ones(it + 1);
      } else {
        na = after(pb);
        nb = after(na);
        ma = after(nb);
      }
      constexpr int kHalfNL = NL / 2;
      const bool more = it + 2 < nk;
      step(0, pa, pb, Tag<1>{}, [&](int q0, int q1) {
        if constexpr (kOnes) {
          if (it >= 1 && more) issue<true>(src, lds, it + 2, ma, q0, q1);
        } else {
          if (it >= 1) issue<false>(src, lds, it + 1, nb, kHalfNL + q0, kHalfNL + q1);
        }
      });
      step(1, pa, pb, Tag<2>{}, [&](int q0, int q1) {
        if (it >= 1 && more) issue<true>(src, lds, it + 2, ma, q0 + (kOnes ? kHalfNL : 0), q1 + (kOnes ? kHalfNL : 0));
      });
      step(0, pa, pb, Tag<3>{}, [&](int q0, int q1) {
        if constexpr (!kOnes)
          if (it >= 1 && more) issue<true>(src, lds, it + 2, ma, kHalfNL + q0, kHalfNL + q1);
      });
      // the next slice has landed (the A behind it may be on its way) for all wavefronts, and all have read what
      // they need of this one
      if (more) __builtin_amdgcn_s_waitcnt(wait_vm(NL));
      else __builtin_amdgcn_s_waitcnt(wait_vm(0));
      __builtin_amdgcn_s_barrier();
      step(1, na, nb, Tag<0>{}, [&](int q0, int q1) {  // (B of slice it + 2 goes where A of this one was)
        if constexpr (!kOnes)
          if (more) issue<false>(src, lds, it + 2, pa, q0, q1);
      });
      pa = na;
      pb = nb;
    }
    // The last slice (behind the end of k it holds zeros).
    read_frags(pa, pb, Tag<1>{}, 1);
    multiply(0);
    arrive(1);
    read_frags(pa, pb, Tag<2>{}, 0);
    multiply(1);
    arrive(0);
    read_frags(pa, pb, Tag<3>{}, 1);
    multiply(0);
    arrive(1);
    multiply(1);
  }

  // The product with the ones by values that pass through `filter` (eight bf16 at a time) on their way to LDS: K rows
  // of A through registers, a slice at a time.  For what is rare, so of few registers and little code; no wavefront uses the
  // ring any more.
  template <class F>
  __device__ static inline void run_filtered(const Operand& A, int K, u32x4* lds, f32x16 (&acc)[TM][TN], const Ones& ones,
                                             F&& filter) {
    static_assert(!kAlongA && !kAlongB && !kHalf, "bf16 ones, across k");
    typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
    const int lane = threadIdx.x % kWave, wave = uniform((int)threadIdx.x / kWave);
    const int wm = wave / WGN, wn = wave % WGN;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const uint32_t lds_base = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) u32x4*)lds;
    const int g = lane >> 4, i16 = lane & 15;
#pragma unroll 1
    for (int k0 = 0; k0 < K; k0 += kSlice) {
#pragma unroll 1
      for (int slot = threadIdx.x; slot < kSlots; slot += kThreads) {
        int row, chunk;
        slot_place<BM, false>(slot, &row, &chunk);
        u32x4 v = u32x4{0u, 0u, 0u, 0u};
        int c = -1;  // of this chunk's columns, the one whose 1 this row has
        if (k0 + row < K) {
          const int from = 8 * chunk < A.limit ? 8 * chunk : 0;
          v = filter(*reinterpret_cast<const u32x4_a4*>(A.p + (int64_t)(k0 + row) * A.ld + from));
          c = min(max(ones.ids[k0 + row], 0), ones.count - 1) - ones.first - 8 * chunk;
        }
        lds[slot] = v;
        const uint32_t one = (c & 1) ? 0x3F800000u : 0x3F80u;
#pragma unroll
        for (int w = 0; w < 4; ++w) v[w] = c >= 0 && (c >> 1) == w ? one : 0u;
        lds[kSlots + slot] = v;
      }
      __syncthreads();
#pragma unroll 1
      for (uint32_t ks = 0; ks < kSlice / 16; ++ks) {
        u32x4 fa[TM], fb[TN];
        uint32_t at[TM];
#pragma unroll
        for (int t = 0; t < TM; ++t) at[t] = lds_base + across_at<BM>(wm * TM + t, g, i16);
        unroll<2 * TM>([&](auto r) { read_part<BM, false, 0, decltype(r)::value>(at, ks * 32 * BM, fa); });
#pragma unroll
        for (int t = 0; t < TN; ++t) at[t] = lds_base + across_at<BN>(wn * TN + t, g, i16);
        unroll<2 * TN>([&](auto r) { read_part<BN, false, 0, decltype(r)::value>(at, kPlaceBytes + ks * 32 * BN, fb); });
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(fa[i]));
#pragma unroll
        for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(fb[j]));
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[i]),
                                                                __builtin_bit_cast(bf16x8, fb[j]), acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      __syncthreads();
    }
  }

 private:
  // where lane (g, i) of a 32-column block reads: row i / 4 of its group of four, columns 16 (g % 2) + 4 (i % 4)
  template <int R>
  __device__ static inline uint32_t across_at(int block, int g, int i) {
    const int k = (g >> 1) * 8 + (i >> 2);
    const int chunk = (block * 4 + (g & 1) * 2 + ((i & 3) >> 1)) ^ swizzle<R>(k);
    return (uint32_t)(k * R * 2 + chunk * 16 + (i & 1) * 8);
  }
  template <int R, bool kAlong, int ks, int r, int T, int N>
  __device__ static inline void read_part(const uint32_t (&at)[N], uint32_t place, u32x4 (&f)[T]) {
    if constexpr (kAlong) {
      f[r] = read_along<r * 4096>((at[0] ^ (32u * ks)) + place);
    } else {
      constexpr int t = r / 2;
      const u32x2 v = read_across<ks * 32 * R + (r % 2) * 8 * R>(at[t] + place);
      if constexpr (r % 2 == 0) f[t] = u32x4{v.x, v.y, f[t].z, f[t].w};
      else f[t] = u32x4{f[t].x, f[t].y, v.x, v.y};
    }
  }
};

}  // namespace mm
}  // namespace mae

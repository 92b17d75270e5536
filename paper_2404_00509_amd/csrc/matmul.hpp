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
// direct load in flight; the code waits on lgkmcnt itself before it uses what was read.
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

// One operand of a tile.
struct Operand {
  const uint16_t* p;  // along k: element (first row of the tile, first k); across k: (first k, first column)
  int64_t ld;         // elements from row to row
  int limit;          // rows (along k) or columns (across k) of the tile that exist, at least 1
};

// A tile of (32 TM WGM) x (32 TN WGN) results by WGM x WGN wavefronts.
// Requirements: along k: k up to a multiple of 8 can be read and holds finite values where the other
// operand's are zero; across k: whole chunks of 8 columns up to `limit` rounded up to 8 can be read
// in every row.  Addresses are multiples of 4 bytes.
template <int TM, int TN, int WGM, int WGN, int STAGES, bool kAlongA, bool kAlongB, bool kHalf = false>
struct Tile {
  static constexpr int kThreads = 64 * WGM * WGN;
  static constexpr int BM = 32 * TM * WGM, BN = 32 * TN * WGN;
  static constexpr int kSlotsA = BM * 8, kSlots = (BM + BN) * 8;  // 16-byte slots per stage
  static constexpr int NL = kSlots / kThreads;                    // direct loads per lane and stage
  static constexpr int kStageBytes = kSlots * 16;
  static constexpr int kLdsBytes = STAGES * kStageBytes;
  static_assert(kSlots % kThreads == 0 && kSlotsA % kWave == 0, "whole wave-wide loads of one operand");
  static_assert(NL * (STAGES - 1) <= 63, "vmcnt range");

  // which chunk of its row slot `s` of an operand of R rows or columns holds, and that row
  template <int R, bool kAlong>
  __device__ static inline void slot_place(int s, int* row, int* chunk) {
    if (kAlong) {
      *row = s / 8;
      *chunk = (s % 8) ^ ((*row >> 1) & 7);
    } else {
      constexpr int kChunks = R / 8;
      *row = s / kChunks;
      *chunk = (s % kChunks) ^ (R >= 128 ? (*row & 3) << 2 : ((*row >> 1) & 1) << 2);
    }
  }

  __device__ static inline void run(const Operand& A, const Operand& B, int K, u32x4* lds,
                                    f32x16 (&acc)[TM][TN]) {
    const int tid = threadIdx.x;
    const int lane = tid % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wm = wave / WGN, wn = wave % WGN;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const int nk = (K + kSlice - 1) / kSlice;
    if (nk == 0) return;
    const int tail = K % kSlice;

    // what this lane brings in per stage, as bytes from the operand's first element of the slice
    uint32_t off[NL];
#pragma unroll
    for (int q = 0; q < NL; ++q) {
      const int s0 = (wave * NL + q) * kWave;  // (the same operand for all lanes)
      int row, chunk;
      if (s0 < kSlotsA) {
        slot_place<BM, kAlongA>(s0 + lane, &row, &chunk);
        if (kAlongA) row = min(row, A.limit - 1);
        else if (8 * chunk >= A.limit) chunk = 0;  // (any columns that exist: their results are not used)
        off[q] = (uint32_t)(row * A.ld + 8 * chunk) * 2u;
      } else {
        slot_place<BN, kAlongB>(s0 - kSlotsA + lane, &row, &chunk);
        if (kAlongB) row = min(row, B.limit - 1);
        else if (8 * chunk >= B.limit) chunk = 0;
        off[q] = (uint32_t)(row * B.ld + 8 * chunk) * 2u;
      }
    }
    // bytes from slice to slice
    const uint32_t step_a = kAlongA ? kSlice * 2 : kSlice * 2 * (uint32_t)uniform((int)A.ld);
    const uint32_t step_b = kAlongB ? kSlice * 2 : kSlice * 2 * (uint32_t)uniform((int)B.ld);
    const char* const first_a = uniform(A.p);
    const char* const first_b = uniform(B.p);

    auto issue = [&](int it, int stage, int q0, int q1) {
      u32x4* dst = lds + stage * kSlots + wave * NL * kWave;
      const char* a_base = first_a + (uint64_t)(uint32_t)it * step_a;
      const char* b_base = first_b + (uint64_t)(uint32_t)it * step_b;
      asm("" : "+s"(a_base), "+s"(b_base));
      if ((it + 1) * kSlice <= K) {
#pragma unroll
        for (int q = q0; q < q1; ++q) {
          const char* base = (wave * NL + q) * kWave < kSlotsA ? a_base : b_base;
          __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)(base + off[q]),
                                           (void __attribute__((address_space(3)))*)(dst + q * kWave), 16, 0, 0);
        }
      } else {
        // (a load for every lane, whatever it holds: the waits count them)
#pragma unroll
        for (int q = q0; q < q1; ++q) {
          const int s0 = (wave * NL + q) * kWave;
          int row, chunk;
          bool behind;
          const char* src;
          if (s0 < kSlotsA) {
            slot_place<BM, kAlongA>(s0 + lane, &row, &chunk);
            behind = kAlongA ? 8 * chunk >= tail : row >= tail;
            src = a_base + off[q];
          } else {
            slot_place<BN, kAlongB>(s0 - kSlotsA + lane, &row, &chunk);
            behind = kAlongB ? 8 * chunk >= tail : row >= tail;
            src = b_base + off[q];
          }
          if (behind) src = reinterpret_cast<const char*>(&kZeros);
          __builtin_amdgcn_global_load_lds((const void __attribute__((address_space(1)))*)src,
                                           (void __attribute__((address_space(3)))*)(dst + q * kWave), 16, 0, 0);
        }
      }
    };

    // fragment addresses inside a stage (bytes)
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
      fb_at[0] = lds_base + (uint32_t)(BM + wn * 32 * TN + (lane & 31)) * 128u + c0;
    } else {
#pragma unroll
      for (int t = 0; t < TN; ++t) fb_at[t] = lds_base + BM * 128 + across_at<BN>(wn * TN + t, g, i16);
    }

    u32x4 fa[2][TM], fb[2][TN];
    auto read_frags = [&](int stage, auto ks_tag, int set) {
      constexpr int ks = decltype(ks_tag)::value;
      const uint32_t st = (uint32_t)stage * kStageBytes;
      read_operand<BM, TM, kAlongA, ks>(fa_at, st, fa[set]);
      read_operand<BN, TN, kAlongB, ks>(fb_at, st, fb[set]);
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
    auto multiply = [&](int set, int from, int to) {
#pragma unroll
      for (int i = from; i < to; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
          if constexpr (kHalf)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, fa[set][i]),
                                                               __builtin_bit_cast(f16x8, fb[set][j]), acc[i][j], 0, 0,
                                                               0);
          else
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, fa[set][i]),
                                                                __builtin_bit_cast(bf16x8, fb[set][j]), acc[i][j], 0,
                                                                0, 0);
    };
    // slice `next` has landed for all wavefronts, and all have read what they need of the one before
    auto turn = [&](int next) {
      if (next + STAGES - 1 <= nk) __builtin_amdgcn_s_waitcnt(wait_vm(NL * (STAGES - 2)));
      else __builtin_amdgcn_s_waitcnt(wait_vm(0));
      __builtin_amdgcn_s_barrier();
    };

#pragma unroll
    for (int s = 0; s < STAGES; ++s)
      if (s < nk) issue(s, s, 0, NL);
    if (nk >= STAGES) __builtin_amdgcn_s_waitcnt(wait_vm(NL * (STAGES - 1)));
    else __builtin_amdgcn_s_waitcnt(wait_vm(0));
    __builtin_amdgcn_s_barrier();
    read_frags(0, Tag<0>{}, 0);
    arrive(0);

    // A slice is four sub-steps of 16 k; the fragments of a sub-step are read while the one before it is
    // multiplied, across slices too; the loads that refill a stage come in three parts.
    constexpr int kLoads1 = 3 * NL / 8, kLoads2 = 6 * NL / 8;
    int cur = 0;
    for (int it = 0; it + 1 < nk; ++it) {
      const bool more = it >= 1 && it + STAGES - 1 < nk;
      const int prv = cur == 0 ? STAGES - 1 : cur - 1;
      auto sub = [&](auto ks_tag) {
        constexpr int ks = decltype(ks_tag)::value;
        read_frags(cur, Tag<ks + 1>{}, (ks + 1) & 1);
        multiply(ks & 1, 0, 1);
        __builtin_amdgcn_sched_barrier(0);
        if (more && ks == 0) issue(it + STAGES - 1, prv, kLoads1, kLoads2);
        if (more && ks == 1) issue(it + STAGES - 1, prv, kLoads2, NL);
        __builtin_amdgcn_sched_barrier(0);
        multiply(ks & 1, 1, TM);
        arrive((ks + 1) & 1);
      };
      sub(Tag<0>{});
      sub(Tag<1>{});
      sub(Tag<2>{});
      const int nxt = cur + 1 == STAGES ? 0 : cur + 1;
      turn(it + 1);
      read_frags(nxt, Tag<0>{}, 0);
      multiply(1, 0, 1);
      __builtin_amdgcn_sched_barrier(0);
      if (it + STAGES < nk) issue(it + STAGES, cur, 0, kLoads1);
      __builtin_amdgcn_sched_barrier(0);
      multiply(1, 1, TM);
      arrive(0);
      cur = nxt;
    }
    const int left = tail ? (tail + 15) / 16 : 4;  // sub-steps of the last slice that hold values
    if (left > 1) read_frags(cur, Tag<1>{}, 1);
    multiply(0, 0, TM);
    if (left > 1) {
      arrive(1);
      if (left > 2) read_frags(cur, Tag<2>{}, 0);
      multiply(1, 0, TM);
    }
    if (left > 2) {
      arrive(0);
      if (left > 3) read_frags(cur, Tag<3>{}, 1);
      multiply(0, 0, TM);
    }
    if (left > 3) {
      arrive(1);
      multiply(1, 0, TM);
    }
  }

 private:
  template <int v>
  struct Tag {
    static constexpr int value = v;
  };
  // where lane (g, i) of a 32-column block reads: row i / 4 of its group of four, columns 16 (g % 2) + 4 (i % 4)
  template <int R>
  __device__ static inline uint32_t across_at(int block, int g, int i) {
    const int k = (g >> 1) * 8 + (i >> 2);
    const int swizzle = R >= 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
    const int chunk = (block * 4 + (g & 1) * 2 + ((i & 3) >> 1)) ^ swizzle;
    return (uint32_t)(k * R * 2 + chunk * 16 + (i & 1) * 8);
  }
  template <int R, int T, bool kAlong, int ks, int N>
  __device__ static inline void read_operand(const uint32_t (&at)[N], uint32_t st, u32x4 (&f)[T]) {
    if constexpr (kAlong) {
      const uint32_t v = (at[0] ^ (32u * ks)) + st;
      f[0] = read_along<0>(v);
      if constexpr (T >= 2) f[1] = read_along<4096>(v);
      if constexpr (T >= 3) f[2] = read_along<8192>(v);
      if constexpr (T >= 4) f[3] = read_along<12288>(v);
    } else {
#pragma unroll
      for (int t = 0; t < T; ++t) {
        const u32x2 lo = read_across<ks * 32 * R>(at[t] + st);
        const u32x2 hi = read_across<ks * 32 * R + 8 * R>(at[t] + st);
        f[t] = u32x4{lo.x, lo.y, hi.x, hi.y};
      }
    }
  }
};

}  // namespace mm
}  // namespace mae

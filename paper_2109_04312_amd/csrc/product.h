// What every product of token rows and weights is made of (proj_mfma.hip, linear_mfma.hip): workgroup shapes, the
// swizzled tiles of a stage, operand fragments, one stage's products, and sums of several token ranges.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "arrival.h"
#include "d2l.h"
#include "mfma_common.h"

namespace mate {

// A pointer the compiler can keep in scalar registers (the value is the same in every lane).
__device__ inline const char* uniform_ptr(const void* p) {
  const unsigned long long v = reinterpret_cast<unsigned long long>(p);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)v), hi = __builtin_amdgcn_readfirstlane((unsigned)(v >> 32));
  return reinterpret_cast<const char*>(((unsigned long long)hi << 32) | lo);
}

// Workgroup shape: kA x 64 rows of operand A by kB x 64 rows of operand B, kWA x kWB wavefronts; kGroups such
// sets of wavefronts share the contraction (stage k belongs to group k mod kGroups, each group has its own
// ring of stages) and add their accumulators at the end.
//
// Two groups are for products with so few tiles that a CU has one: alone, four wavefronts read LDS and
// multiply in turns (0.6 us a stage of 128 x 128 where the matrix pipe needs 0.2), and two workgroups on a
// CU drift apart so that one reads while the other multiplies.  Two groups of one workgroup would read at the
// same time, because every stage has a barrier; so they are kept half a stage apart (kAlternate): a second
// barrier between reading and multiplying, and group 1 one barrier behind.  dX at 8 x 512 tokens and 768
// wide 26.4 -> 21.8 us, its weight gradient 35.3 -> 32.9, that of the output projection 29.2 -> 24.6; in
// step they gained 0 to 2.  (The 128 x 64 shape with its shorter stages, three of them, is better in step.)
//
// Eight wavefronts on one tile (256 x 256) are kept apart in the same way, the upper four half a slice behind
// the lower four, where the weights' products use them: 1024 -> 3072 features at 2 x 8192 tokens 97.5 -> 93.0
// us, 3072 -> 1024 81.7 -> 78.5.  In the weight gradient, whose operands are both read through the slower
// transposing reads, the reads of one half outlast the products of the other: 111 -> 117 us, so not there.
template <int kA_, int kB_, int kWA_, int kWB_, int kStages_, int kPerCU_, int kGroups_ = 1>
struct Shape {
  static constexpr int kA = kA_, kB = kB_, kWA = kWA_, kWB = kWB_, kStages = kStages_, kPerCU = kPerCU_, kGroups = kGroups_;
  static constexpr int kWaves = kWA * kWB, kAllWaves = kWaves * kGroups, kThreads = 64 * kAllWaves;
  static constexpr int kRowsA = 64 * kA, kRowsB = 64 * kB;
  static constexpr int kFA = 4 * kA / kWA, kFB = 4 * kB / kWB;  // 16-row blocks of a wavefront
  static constexpr int kOutB = kFB / kGroups;                   // and those of B that it stores
  static constexpr bool kAlternate = kGroups == 2 && kStages == 2;
  static constexpr int kStageBytes = (kA + kB) * kTileBytes, kRingBytes = kStages * kStageBytes, kLds = kGroups * kRingBytes;
  static constexpr int kLoadsA = 8 * kA / kWaves, kLoadsB = 8 * kB / kWaves, kLoads = kLoadsA + kLoadsB;
  static_assert(8 * kA % kWaves == 0 && 8 * kB % kWaves == 0, "loads must divide evenly");
  static_assert(4 * kA % kWA == 0 && 4 * kB % kWB == 0 && kFA % 2 == 0 && kFB % kGroups == 0, "blocks must divide evenly");
  static_assert(kGroups == 1 || kGroups == 2, "the exchange is between two groups");
};

// Load instruction i of a wavefront brings eight rows of one tile: which tile, which row this lane's
// 16 bytes belong to, and which 16-byte chunk of it.
struct LoadUnit {
  int tile, row, chunk;
};
template <int kWaves>
__device__ __forceinline__ LoadUnit load_unit(int wave, int lane, int i) {
  const int u = wave + kWaves * i;
  LoadUnit l;
  l.tile = u >> 3;
  l.row = (u & 7) * 8 + (lane >> 3);
  l.chunk = (lane & 7) ^ swz(l.row & 15);
  return l;
}
template <int kWaves>
__device__ __forceinline__ int load_dst(int wave, int i) {
  const int u = wave + kWaves * i;
  return (u >> 3) * kTileBytes + (u & 7) * 8 * 128;
}

// Operand fragment of 16 rows and 32 of k.  Lane l = 16 q + r: row r, k = 8 q .. 8 q + 7.
struct FragOffsets {
  int plain[2];      // per 32-wide k slice
  int trans[2][4];   // [first / second four of k][16-column block of a tile]; a k slice is 32 rows further
};
template <bool kTransposed>
__device__ __forceinline__ void frag_offsets(FragOffsets& f, int lane) {
  const int r = lane & 15, q = lane >> 4;
  if (!kTransposed) {
#pragma unroll
    for (int k = 0; k < 2; ++k) f.plain[k] = r * 128 + (((4 * k + q) ^ swz(r)) << 4);
  } else {
    // 16 lanes read 4 rows x 16 columns: lane i addresses row i / 4, columns 4 (i % 4) .., and receives
    // column i of the four rows
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = 8 * q + 4 * h + (r >> 2);
#pragma unroll
      for (int c = 0; c < 4; ++c)
        f.trans[h][c] = row * 128 + (((2 * c + ((r & 3) >> 1)) ^ swz(row & 15)) << 4) + ((r & 1) << 3);
    }
  }
}
template <bool kTransposed>
__device__ __forceinline__ bf16x8 read_frag(const char* tiles, const FragOffsets& f, int block, int k) {
  if (!kTransposed) return read_plain(tiles + block * 16 * 128, f.plain[k]);
  const char* t = tiles + (block >> 2) * kTileBytes + k * 32 * 128;
  return read_transposed(t, f.trans[0][block & 3], f.trans[1][block & 3]);
}

// One stage (64 of k): two slices of 32.
// `issue` starts the loads of a later stage.  Where the stage's operands are plain it does so behind the operand
// reads: its instructions (eight for 256 x 256, each with an address and m0) then cost the wavefront time in which its
// reads travel, not time before them.  256 x 256 at 16384 x 3072 x 1024 2590 -> 2539 cycles a stage (2885 while the reads had bank
// conflicts); whole products in 128 x 64 with two groups 5 to 9 % shorter, 128 x 128 with two groups 2 to 5, 192 x 128 1 to 2.
// Transposing reads are twice as many instructions, and behind them the loads come too late: all gradients with `issue` behind
// the reads take 3 to 6 % more in the mean.  And 128 x 128 with one group: 5 % less to 7 % more, none in the mean.
// kHalves: `next_landed` is called where this wavefront's share of the next stage must have landed.
// kAlternate: `reading` is called while the fragments travel and the other group multiplies.
template <class S, bool kTA, bool kTB, bool kHalves, class Issue, class PerSlice, class Next, class Reading>
__device__ __forceinline__ void contract_stage(const char* stage, const FragOffsets& fa, const FragOffsets& fb, int wa,
                                               int wb, f32x4 (&acc)[S::kFA][S::kFB], Issue&& issue, PerSlice&& per_slice,
                                               Next&& next_landed, Reading&& reading) {
  const char* ta = stage + (kTA ? 0 : wa * S::kFA * 16 * 128);
  const char* tb = stage + S::kA * kTileBytes + (kTB ? 0 : wb * S::kFB * 16 * 128);
  constexpr bool kIssueLate = !kTA && (S::kGroups > 1 || S::kFA * S::kFB != 16);
  bf16x8 a[2][S::kFA], b[2][S::kFB];
  auto read_slice = [&](int k) {
#pragma unroll
    for (int i = 0; i < S::kFA; ++i) a[k][i] = read_frag<kTA>(ta, fa, (kTA ? wa * S::kFA : 0) + i, k);
#pragma unroll
    for (int j = 0; j < S::kFB; ++j) b[k][j] = read_frag<kTB>(tb, fb, (kTB ? wb * S::kFB : 0) + j, k);
  };
  if (!kIssueLate) issue();
  if constexpr (kHalves) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (k) barrier_no_fence();
      __builtin_amdgcn_sched_barrier(0);
      read_slice(k);
      if (kIssueLate && !k) issue();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (k) next_landed();
      __builtin_amdgcn_sched_barrier(0);
      barrier_no_fence();  // from here on the other half reads
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int i = 0; i < S::kFA; ++i)
#pragma unroll
        for (int j = 0; j < S::kFB; ++j) acc[i][j] = mfma16(a[k][i], b[k][j], acc[i][j]);
      per_slice(b[k]);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(0);
    }
    return;
  }
  read_slice(0);
  if constexpr (S::kAlternate) {
    read_slice(1);
    if (kIssueLate) issue();
    reading();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    barrier_no_fence();  // from here on the other group reads
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k == 0 && !S::kAlternate) {
      read_slice(1);  // the second slice travels while the first is contracted
      if (kIssueLate) issue();
    }
#pragma unroll
    for (int i = 0; i < S::kFA; ++i)
#pragma unroll
      for (int j = 0; j < S::kFB; ++j) acc[i][j] = mfma16(a[k][i], b[k][j], acc[i][j]);
    if constexpr (!S::kAlternate) per_slice(b[k]);
  }
  if constexpr (S::kAlternate) {
    per_slice(b[0]);
    per_slice(b[1]);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
  }
}
// The two groups' accumulators: each wavefront gives half of its blocks of B to its counterpart in the
// other group, through LDS, and keeps the sum of the other half.  (Group 0 stores blocks 0 .. kOutB - 1.)
template <class S>
__device__ __forceinline__ void add_groups(f32x4 (&acc)[S::kFA][S::kFB], f32x4 (&out)[S::kFA][S::kOutB], char* lds, int group,
                                           int wave, int lane) {
  if constexpr (S::kGroups == 1) {
#pragma unroll
    for (int i = 0; i < S::kFA; ++i)
#pragma unroll
      for (int j = 0; j < S::kOutB; ++j) out[i][j] = acc[i][j];
  } else {
    constexpr int kBlocks = S::kFA * S::kOutB;
    static_assert(2 * S::kWaves * kBlocks * 1024 <= S::kLds, "the exchange must fit the stages");
    f32x4* x = reinterpret_cast<f32x4*>(lds) + lane;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::kFA; ++i)
#pragma unroll
      for (int j = 0; j < S::kOutB; ++j)
        x[((group * S::kWaves + wave) * kBlocks + i * S::kOutB + j) * 64] = group ? acc[i][j] : acc[i][j + S::kOutB];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < S::kFA; ++i)
#pragma unroll
      for (int j = 0; j < S::kOutB; ++j) {
        const f32x4 other = x[(((1 - group) * S::kWaves + wave) * kBlocks + i * S::kOutB + j) * 64];
        out[i][j] = group ? other + acc[i][j + S::kOutB] : acc[i][j] + other;
      }
  }
}

// Partial sums of a weight gradient (one fp32 matrix per token range, see below), added in range order
// by the workgroups behind the tiles of the product that follows: a launch of its own took 11 to 14 us
// on the benchmark layer, 5 of them the launch, while the product leaves compute units idle at its end.
struct RangeSums {
  const float* part;       // [splits][n] partial sums, n a multiple of 4
  const float* part_bias;  // [splits][n_bias]
  float *out, *out_bias;   // out_bias may be null
  size_t n;
  int n_bias, splits, blocks;  // blocks: workgroups that share the work (0: nothing to add)
};
__device__ __forceinline__ void add_ranges(const RangeSums& s, int block, int threads) {
  const size_t stride = (size_t)s.blocks * threads, first = (size_t)block * threads + threadIdx.x;
  const f32x4* part = reinterpret_cast<const f32x4*>(s.part);
  for (size_t i = first; i < s.n / 4; i += stride) {
    f32x4 v = part[i];
    for (int k0 = 1; k0 < s.splits; k0 += 4) {  // four at a time, all loaded before the first is added
      f32x4 x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = part[(size_t)min(k0 + e, s.splits - 1) * (s.n / 4) + i];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (k0 + e < s.splits) v += x[e];
    }
    reinterpret_cast<f32x4*>(s.out)[i] = v;
  }
  if (s.out_bias)
    for (size_t i = first; i < (size_t)s.n_bias; i += stride) {
      float v = s.part_bias[i];
      for (int k = 1; k < s.splits; ++k) v += s.part_bias[(size_t)k * s.n_bias + i];
      s.out_bias[i] = v;
    }
}

// The same inside the launch: the range of a tile that is done last adds them all.
constexpr int kMaxRanges = 8;
struct RangeMerge {
  float* part;                  // [splits][tiles][the tile's registers]
  float* part_bias;             // [splits][bias_stride]
  unsigned long long* arrived;  // [tiles][kMaxRanges]
  unsigned long long ticket;    // see arrival.h
  int splits, tiles, bias_stride;
};
// Ranges are added in pairs, pairs of pairs and so on: of two, the one that comes first leaves its registers
// as they are ([wavefront][block][half][lane] pairs, in the place of its lowest range) and ends, the other adds
// them to its own.  (One workgroup that adds all of them waits for 64 KB of far memory per range.)  False: this workgroup has left its own.
// `row`: first row of the wavefront's blocks of B, whose sums `bias_sum` are if it has any.
template <class S>
__device__ __forceinline__ bool merge_ranges(const RangeMerge& m, int split, int tile, int row, bool has_bias, f32x4 (&sum)[S::kFA][S::kOutB],
                                             float (&bias_sum)[S::kFB], int wave_id) {
  constexpr int kTile = S::kRowsA * S::kRowsB, kBlocks = S::kFA * S::kOutB;
  static_assert(kTile == S::kAllWaves * kBlocks * 256, "the registers are the tile");
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, quarter = lane >> 4;
  __shared__ int second;
  for (int level = 0; (1 << level) < m.splits; ++level) {
    const int node = split >> level, other = (node ^ 1) << level;
    if (other >= m.splits) continue;
    unsigned long long* const word = m.arrived + (size_t)tile * kMaxRanges + (kMaxRanges - (kMaxRanges >> level)) + (node >> 1);
    auto place = [&](int range) { return m.part + ((size_t)range * m.tiles + tile) * kTile + wave_id * kBlocks * 256 + lane * 2; };
    auto bias_place = [&](int range) { return m.part_bias + (size_t)range * m.bias_stride + row + r; };
    if (tid == 0) second = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == m.ticket;
    __syncthreads();
    if (!second) {
      float* const mine = place(node << level);
#pragma unroll
      for (int y = 0; y < kBlocks; ++y)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          put_pair<true>(mine + y * 256 + h * 128, sum[y / S::kOutB][y % S::kOutB][2 * h], sum[y / S::kOutB][y % S::kOutB][2 * h + 1]);
      if (has_bias && quarter == 0)
#pragma unroll
        for (int j = 0; j < S::kFB; ++j)
          __hip_atomic_store(bias_place(node << level) + j * 16, bias_sum[j], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      publish_partials();
      if (tid == 0) second = __hip_atomic_exchange(word, m.ticket, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == m.ticket;
      __syncthreads();
      if (!second) return false;
    }
    const float* const theirs = place(other);
    float2 v[kBlocks][2];
#pragma unroll
    for (int y = 0; y < kBlocks; ++y)
#pragma unroll
      for (int h = 0; h < 2; ++h) v[y][h] = get_pair<true>(theirs + y * 256 + h * 128);
#pragma unroll
    for (int y = 0; y < kBlocks; ++y) sum[y / S::kOutB][y % S::kOutB] += f32x4{v[y][0].x, v[y][0].y, v[y][1].x, v[y][1].y};
    if (has_bias)
#pragma unroll
      for (int j = 0; j < S::kFB; ++j)
        bias_sum[j] += __hip_atomic_load(bias_place(other) + j * 16, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    // (cleared again, so that a captured launch, which is replayed with its old ticket, finds none of its own)
    if (tid == 0) __hip_atomic_store(word, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();  // (everyone has looked at `second`)
  }
  return true;
}

// Which of the 64 tokens from position n0 of the sequence at flags[seq] on are padding (or past its end):
// one bit each.  `total` = bytes of the flags array, which is read 64 bytes at a time.
__device__ __forceinline__ unsigned long long pad_mask(const unsigned char* flags, size_t total, size_t seq, int n0, int N) {
  const int n = min(64, N - n0);
  const size_t first = seq + n0;
  unsigned long long bits = 0;
  if (total >= 64) {
    const size_t at = first < total - 64 ? first : total - 64;  // the 64 bytes must lie inside the array
    unsigned w[16];
    __builtin_memcpy(w, flags + at, 64);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned two = w[i] & 0xfefefefeu;  // a byte of 2 or more leaves a bit here: collect it in bit 7
      const unsigned pad = (((two & 0x7f7f7f7fu) + 0x7f7f7f7fu) | two) & 0x80808080u;
      bits |= (unsigned long long)(((pad >> 7) * 0x10204080u) >> 28) << (4 * i);
    }
    bits >>= (int)(first - at);
  } else {
    for (int i = 0; i < n; ++i) bits |= (unsigned long long)(flags[first + i] >= 2) << i;
  }
  return n < 64 ? bits | ~0ull << n : bits;
}

}  // namespace mate

// The products of a layer's feed-forward half and their gradients, bf16 MFMA (gfx950):
//   forward:  z = x w^T + bias,  y = act(z) + residual, and what the backward needs of them (z in bf16 or in 8 bits, y in 8 bits);
//   dx:       (dy w) act'(z) + the residual's gradient, z the pre-activation that x came from;
//   dw:       sum over tokens of dy^T x, x in bf16 or in 8 bits.
// The main loop is that of the projections (product.h): C[b, a] = sum_k B[b, k] A[a, k], a contiguous in the output, so that a lane holds
// four consecutive features of a token.  Rows are flat tokens here, and widths any multiple of 8: a last
// stage of fewer than 64 terms repeats the last 16 bytes or rows and is then cleared in LDS, in both operands (zero times whatever a
// row ends in would do for numbers, not for infinities).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "activation.h"
#include "d2l.h"
#include "eight_bits.h"
#include "launch.h"
#include "mfma_common.h"
#include "product.h"
#include "tile_deal.h"

namespace mate {
namespace {

// ======================================================================================
// Products with the weights: forward, dx
// ======================================================================================
// What a tile's first loads need: kernel arguments of their own, as plain values arrive in registers with the wavefront.
struct LinearStart {
  const unsigned short* w;    // forward: [O][K];  dx: [K][O], read transposed
  const unsigned short* tok;  // [T][K]
  int T, O, K;                // tokens, features out, contraction length
  TileDeal deal;
};
struct LinearArgs : LinearStart {
  const unsigned char* flags;   // [T] or null
  const unsigned short* add;    // [T][O] or null: residual, or the residual's gradient
  int act;
  const float* bias;            // forward: [O] or null
  const void* z_in;             // dx: pre-activation [T][O], bf16, or codes if z_in_scales is not null
  const unsigned char* z_in_scales;
  unsigned short* y;            // [T][O]
  void* z;                      // forward: bf16, or codes if z_scales is not null; or null
  unsigned char *z_scales, *y_codes, *y_scales;
  RangeSums ranges;
};

// Eight consecutive features of a token, in two words of codes or four of bf16, and a lane's four features of each block of a pair in the
// accumulators' layout: exchanging quarters between the two blocks' words turns one into the other, both ways.
struct Pair { unsigned u[2]; };
__device__ __forceinline__ Pair exchange(unsigned x, unsigned y) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
  return {{r[0], r[1]}};
}

template <class S, bool kGrad>
__device__ __forceinline__ void linear_tile(const LinearStart& p, const LinearArgs& a, char* lds, int t0, int f0) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_id = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = wave_id / S::kWaves, wave = wave_id - group * S::kWaves;
  const int wa = wave / S::kWB, wb = wave - wa * S::kWB;
  const int r = lane & 15, quarter = lane >> 4;
  char* const ring = lds + group * S::kRingBytes;
  const int rows = min(S::kRowsB, p.T - t0), feats = min(S::kRowsA, p.O - f0);

  // ---- operand streams: per load a wave-uniform base and a 32-bit lane offset -----------------------
  unsigned off[S::kLoads];
#pragma unroll
  for (int i = 0; i < S::kLoadsA; ++i) {   // (features past the last, or the last eight, repeat those, and are not stored)
    const LoadUnit l = load_unit<S::kWaves>(wave, lane, i);
    off[i] = kGrad ? (unsigned)l.row * (unsigned)p.O * 2 + (unsigned)min(64 * l.tile + 8 * l.chunk, feats - 8) * 2
                   : (unsigned)min(64 * l.tile + l.row, feats - 1) * (unsigned)p.K * 2 + l.chunk * 16;
  }
#pragma unroll
  for (int i = 0; i < S::kLoadsB; ++i) {   // (tokens past the end repeat the last one)
    const LoadUnit l = load_unit<S::kWaves>(wave, lane, i);
    off[S::kLoadsA + i] = (unsigned)min(64 * l.tile + l.row, rows - 1) * (unsigned)p.K * 2 + l.chunk * 16;
  }
  const char* const w0 = reinterpret_cast<const char*>(kGrad ? p.w + f0 : p.w + (size_t)f0 * p.K);
  const char* const x0 = reinterpret_cast<const char*>(p.tok + (size_t)t0 * p.K);
  const size_t w_step = kGrad ? (size_t)64 * p.O * 2 : 128;
  const char *w_ptr = w0 + group * w_step, *x_ptr = x0 + group * 128;   // of the next stage
  const int stages = (p.K + 63) >> 6, nk = (stages + S::kGroups - 1) / S::kGroups;   // nk: this group's, the last one short or empty
  const int short_k = 64 * ((nk - 1) * S::kGroups + group);   // its first term
  const bool is_short = short_k + 64 > p.K;
  auto issue_stage = [&](int g) {
    char* st = ring + (g % S::kStages) * S::kStageBytes;
    if (__builtin_expect(g == nk - 1 && is_short, 0)) {
      const int row0 = min(short_k, p.K - 1);
      const char *w_base = uniform_ptr(kGrad ? w0 + (size_t)row0 * p.O * 2 : w0), *x_base = uniform_ptr(x0);
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i) {
        const bool is_a = i < S::kLoadsA;
        const int y = is_a ? i : i - S::kLoadsA;
        const LoadUnit l = load_unit<S::kWaves>(wave, lane, y);
        unsigned o = off[i];
        if (kGrad && is_a) o -= (unsigned)(l.row - (min(short_k + l.row, p.K - 1) - row0)) * (unsigned)p.O * 2;
        else o += (unsigned)min(short_k + 8 * l.chunk, p.K - 8) * 2 - l.chunk * 16;
        load_to_lds_16(is_a ? w_base : x_base, o, st + (is_a ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, y));
      }
      return;
    }
    const char *w_base = uniform_ptr(w_ptr), *x_base = uniform_ptr(x_ptr);
#pragma unroll
    for (int i = 0; i < S::kLoadsA; ++i) load_to_lds_16(w_base, off[i], st + load_dst<S::kWaves>(wave, i));
#pragma unroll
    for (int i = 0; i < S::kLoadsB; ++i)
      load_to_lds_16(x_base, off[S::kLoadsA + i], st + S::kA * kTileBytes + load_dst<S::kWaves>(wave, i));
    w_ptr += S::kGroups * w_step;
    x_ptr += S::kGroups * 128;
  };
  // My share of the short stage, landed, is zero from the last term on.
  auto clear_short = [&]() {
    char* st = ring + ((nk - 1) % S::kStages) * S::kStageBytes;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const bool is_a = i < S::kLoadsA;
      const int y = is_a ? i : i - S::kLoadsA;
      const LoadUnit l = load_unit<S::kWaves>(wave, lane, y);
      if (short_k + (kGrad && is_a ? l.row : 8 * l.chunk) >= p.K)
        *reinterpret_cast<uint4*>(st + (is_a ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, y) + lane * 16) = make_uint4(0, 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  constexpr bool kHalves = S::kGroups == 1 && S::kWaves == 8 && S::kStages == 2;
#pragma unroll
  for (int s = 0; s < S::kStages - 1; ++s)
    if (s < nk) issue_stage(s);

  // While the first stages travel: which tokens are padding, and the bias of this lane's features.
  const unsigned char* const fl = a.flags ? a.flags + t0 : nullptr;
  bool any = !fl;
  const int j0 = wb * S::kFB + group * S::kOutB;  // first block of tokens that this wavefront stores
  int row[S::kOutB];
  unsigned pad_bits = 0;
#pragma unroll
  for (int j = 0; j < S::kOutB; ++j) row[j] = min((j0 + j) * 16 + r, rows - 1);
  if (fl) {
#pragma unroll
    for (int i = 0; i < S::kB; ++i) any |= fl[min(64 * i + lane, rows - 1)] < 2;
#pragma unroll
    for (int j = 0; j < S::kOutB; ++j) pad_bits |= (unsigned)(fl[row[j]] >= 2) << j;
  }
  f32x4 bias[S::kFA];
#pragma unroll
  for (int i = 0; i < S::kFA; ++i) bias[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (!kGrad && a.bias)
#pragma unroll
    for (int i = 0; i < S::kFA; ++i) bias[i] = *reinterpret_cast<const f32x4*>(a.bias + f0 + min((wa * S::kFA + i) * 16 + 4 * quarter, feats - 4));

  f32x4 acc[S::kFA][S::kFB];
#pragma unroll
  for (int i = 0; i < S::kFA; ++i)
#pragma unroll
    for (int j = 0; j < S::kFB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (__any(any)) {  // (a tile of padding only is stored as zeros without arithmetic)
    FragOffsets fa, fb;
    frag_offsets<kGrad>(fa, lane);
    frag_offsets<false>(fb, lane);
    // the second half, or group, follows one barrier behind
    const bool apart = kHalves || S::kAlternate, second = kHalves ? wave >= 4 : group == 1;
    if (kHalves) {
      wait_vmcnt_le<0>(0);
      if (is_short && nk == 1) clear_short();
    }
    if (apart && second) barrier_no_fence();
    for (int ks = 0; ks < nk; ++ks) {
      // stage ks has landed: everything but the younger stages' loads (fewer near the end)
      if (!kHalves) {
        wait_vmcnt_le<S::kLoads * (S::kStages - 2)>(min(S::kStages - 2, nk - 1 - ks) * S::kLoads);
        if (__builtin_expect(is_short && ks == nk - 1, 0)) clear_short();
      }
      barrier_no_fence();  // ... for every wavefront, and everyone is done with stage ks - 1
      contract_stage<S, kGrad, false, kHalves>(ring + (ks % S::kStages) * S::kStageBytes, fa, fb, wa, wb, acc,
                                               [&]() { if (ks + S::kStages - 1 < nk) issue_stage(ks + S::kStages - 1); },
                                               [](const bf16x8 (&)[S::kFB]) {},
                                               [&]() {
                                                 wait_vmcnt_le<0>(0);
                                                 if (__builtin_expect(is_short && ks == nk - 2, 0)) clear_short();
                                               },
                                               []() {});
    }
    if (apart && !second) barrier_no_fence();
  }
  f32x4 sum[S::kFA][S::kOutB];
  add_groups<S>(acc, sum, lds, group, wave, lane);

  // ---- epilogue, in fp32 until a result is rounded.  A lane holds features 16 i + 4 quarter .. + 3 of token 16 j + r; memory is read
  // and written in eight consecutive ones, 64 of a token's bytes per instruction (32 of codes).  A pair of blocks is a block of one
  // scale, its 32 values in the four quarters. ----
  const int scales = scale_blocks(p.O);
  const int lane_feature = (quarter & 1) * 16 + (quarter >> 1) * 8;   // first of the eight, in the pair
  auto magnitude_across = [](unsigned m) {
    const Pair x = exchange(m, m);
    m = max(x.u[0], x.u[1]);
    const auto y = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return max((unsigned)y[0], (unsigned)y[1]);
  };
  with_activation(a.act, [&](auto kind) {
    constexpr int kAct = decltype(kind)::value;
#pragma unroll
    for (int i = 0; i < S::kFA; i += 2) {
      const int fw = (wa * S::kFA + i) * 16;       // first feature of the pair in the tile
      if (fw >= feats) break;
      const bool stored = fw + lane_feature < feats;
      const bool real[2] = {fw + 4 * quarter < feats, fw + 16 + 4 * quarter < feats};   // this lane's four features of each block
      const size_t at0 = (size_t)t0 * p.O + f0 + fw + lane_feature, scale0 = (size_t)t0 * scales + (f0 + fw) / kScaleBlock;
      u32x4 add[S::kOutB], zb[S::kOutB];
      unsigned zs[S::kOutB];
#pragma unroll
      for (int j = 0; j < S::kOutB; ++j) {
        const size_t at = at0 + (size_t)row[j] * p.O;
        add[j] = zb[j] = u32x4{0, 0, 0, 0};
        zs[j] = 1;
        if (stored && a.add) add[j] = *reinterpret_cast<const u32x4*>(a.add + at);
        if (kGrad && kAct != kActNone) {
          if (a.z_in_scales) {
            zs[j] = a.z_in_scales[scale0 + (size_t)row[j] * scales];
            if (stored) {
              const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const unsigned char*>(a.z_in) + at);
              zb[j][0] = w.x;
              zb[j][1] = w.y;
            }
          } else if (stored) {
            zb[j] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(a.z_in) + at);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < S::kOutB; ++j) {
        const bool pad = (pad_bits >> j) & 1u, store = stored && (j0 + j) * 16 + r < rows;
        const size_t at = at0 + (size_t)row[j] * p.O, scale_at = scale0 + (size_t)row[j] * scales;
        const Pair add_lo = exchange(add[j][0], add[j][2]), add_hi = exchange(add[j][1], add[j][3]);
        float v[8], z[8];
        if (kGrad && kAct != kActNone) {
          if (a.z_in_scales) {
            const Pair c = exchange(zb[j][0], zb[j][1]);
            const f32x4 lo = from_codes(c.u[0], scale_value(zs[j])), hi = from_codes(c.u[1], scale_value(zs[j]));
#pragma unroll
            for (int e = 0; e < 4; ++e) { z[e] = lo[e]; z[4 + e] = hi[e]; }
          } else {
            const Pair lo = exchange(zb[j][0], zb[j][2]), hi = exchange(zb[j][1], zb[j][3]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              z[4 * h] = low_bf16(lo.u[h]); z[4 * h + 1] = high_bf16(lo.u[h]);
              z[4 * h + 2] = low_bf16(hi.u[h]); z[4 * h + 3] = high_bf16(hi.u[h]);
            }
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const f32x4 c = sum[i + h][j] + bias[i + h];
          const float more[4] = {low_bf16(add_lo.u[h]), high_bf16(add_lo.u[h]), low_bf16(add_hi.u[h]), high_bf16(add_hi.u[h])};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x;
            if constexpr (kGrad) {
              x = kAct == kActNone ? c[e] : c[e] * slope<kAct>(z[4 * h + e]);
            } else {
              z[4 * h + e] = pad || !real[h] ? 0.f : c[e];
              x = activate<kAct>(c[e]);
            }
            if (a.add) x += more[e];
            v[4 * h + e] = pad || !real[h] ? 0.f : x;
          }
        }
        auto store_bf16 = [&](unsigned short* to, const float (&x)[8]) {
          const Pair lo = exchange(pack2(x[0], x[1]), pack2(x[4], x[5])), hi = exchange(pack2(x[2], x[3]), pack2(x[6], x[7]));
          if (store) *reinterpret_cast<u32x4*>(to + at) = u32x4{lo.u[0], hi.u[0], lo.u[1], hi.u[1]};
        };
        auto store_8bit = [&](unsigned char* to, unsigned char* to_scales, float (&x)[8]) {
          const unsigned s = scale_byte(block_magnitude(x, magnitude_across));
          const float scale = scale_value(s);
          const Pair c = exchange(to_codes(x[0], x[1], x[2], x[3], scale), to_codes(x[4], x[5], x[6], x[7], scale));
          if (store) *reinterpret_cast<uint2*>(to + at) = make_uint2(c.u[0], c.u[1]);
          if (store && quarter == 0) to_scales[scale_at] = (unsigned char)s;
        };
        if (!kGrad && a.z) {
          if (a.z_scales) store_8bit(static_cast<unsigned char*>(a.z), a.z_scales, z);
          else store_bf16(static_cast<unsigned short*>(a.z), z);
        }
        store_bf16(a.y, v);
        if (!kGrad && a.y_codes) store_8bit(a.y_codes, a.y_scales, v);
      }
    }
  });
}

template <class S, bool kGrad>
__global__ __launch_bounds__(S::kThreads, S::kAllWaves / 4 * S::kPerCU) void linear_kernel(const unsigned short* w, const unsigned short* tok, int T,
                                                                                         int O, int K, int token_tiles, int feature_tiles,
                                                                                         int whole_rows, int by_feature, LinearArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const LinearStart p = {w, tok, T, O, K, {token_tiles, feature_tiles, whole_rows, by_feature}};
  const int x = blockIdx.x, y = blockIdx.y + kMostGridY * blockIdx.z, behind = y - p.deal.grid_y();
  if (behind < 0) {
    int token_tile, feature_tile;
    if (dealt_tile(p.deal, x, y, token_tile, feature_tile)) linear_tile<S, kGrad>(p, a, lds, token_tile * S::kRowsB, feature_tile * S::kRowsA);
  } else if (behind * p.deal.grid_x() < a.ranges.blocks) {
    add_ranges(a.ranges, behind * p.deal.grid_x() + x, S::kThreads);   // behind the tiles: partial sums of dw
  }
}

template <class S>
long tiles_of(const LinearArgs& a) {
  return (a.T + (long)S::kRowsB - 1) / S::kRowsB * ((a.O + S::kRowsA - 1) / S::kRowsA);
}

template <class S, bool kGrad>
hipError_t launch_product(LinearArgs a, hipStream_t stream) {
  TileDeal& d = a.deal;
  d.tokens = (int)((a.T + (long)S::kRowsB - 1) / S::kRowsB);
  d.features = (a.O + S::kRowsA - 1) / S::kRowsA;
  d.by_feature = a.O > a.T && d.features >= 8;   // (every XCD reads all of the other operand: the smaller one)
  d.rows = (d.by_feature ? d.features : d.tokens) / 8;
  const int x = d.grid_x();
  int range_rows = 0;
  if (a.ranges.splits) {
    range_rows = (int)(std::max<size_t>(1, std::min<size_t>(1024 * 256 / S::kThreads, a.ranges.n / 4 / S::kThreads)) + x - 1) / x;
    a.ranges.blocks = range_rows * x;
  }
  const int y = d.grid_y() + range_rows;
  const dim3 grid(x, std::min(y, kMostGridY), (y + kMostGridY - 1) / kMostGridY);
  const hipError_t e = allow_lds<&linear_kernel<S, kGrad>>(S::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((linear_kernel<S, kGrad>), grid, dim3(S::kThreads), S::kLds, stream, a.w, a.tok, a.T, a.O, a.K, d.tokens, d.features, d.rows,
                     d.by_feature, a);
  return hipGetLastError();
}

//                        features x tokens, wavefronts, stages, workgroups per CU, groups
using Tile256 = Shape<4, 4, 2, 4, 2, 1>;
using Tile128 = Shape<2, 2, 2, 2, 2, 2>;
using Tile128x2 = Shape<2, 2, 2, 2, 2, 1, 2>;
using Tile64 = Shape<2, 1, 2, 2, 3, 2>;
using Tile64x2 = Shape<2, 1, 2, 2, 3, 1, 2>;
template <bool kGrad>
hipError_t run_product(const LinearArgs& a, hipStream_t stream) {
  typedef hipError_t (*Launch)(LinearArgs, hipStream_t);
  double best = 1e30;
  Launch launch = nullptr;
  auto offer = [&](auto shape, double c1, double c2, double e) {
    typedef decltype(shape) S;
    const long n = (tiles_of<S>(a) + 255) / 256;
    const double cost = (a.K + 63) / 64 * ((n / 2) * c2 + (n % 2) * c1) + e * n;
    if (cost < best) {
      best = cost;
      launch = launch_product<S, kGrad>;
    }
  };
  offer(Tile256(), 1.37, 3.14, 5.33);
  offer(Tile128(), 0.62, 1.09, 1.1);
  offer(Tile128x2(), 0.47, 1.2, 1.86);
  offer(Tile64(), 0.46, 0.74, 0.53);
  offer(Tile64x2(), 0.39, 0.8, 0.71);
  return launch(a, stream);
}

// ======================================================================================
// Gradient with respect to the weights
// ======================================================================================
// Both operands are token-major, so their 64-token x 64-column tiles go into LDS as they are and both are read transposed.  A
// workgroup owns a tile of dw and a range of the token blocks; partial sums of the ranges are added in a fixed order
// afterwards (no atomics: the result is bit-reproducible).  The bias gradient rides along in the workgroups of the first
// column tile.  Rows of pad tokens are cleared in LDS after a block has landed, and blocks of padding only are skipped.
struct WeightGradArgs {
  const unsigned short *g, *x;   // [T][F], [T][E]
  const unsigned char* flags;    // [T] or null
  float *out, *out_bias;         // [F][E], [F] or null (final when splits == 1)
  float *part, *part_bias;       // [splits][F][E], [splits][F]
  int T, F, E;
  int splits, per_split;         // ranges of 64-token blocks
};
constexpr int kMostBlocks = 1024;   // of a range

template <class S>
__global__ __launch_bounds__(S::kThreads, S::kAllWaves / 4 * S::kPerCU) void linear_wgrad_kernel(WeightGradArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_id = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = wave_id / S::kWaves, wave = wave_id - group * S::kWaves;
  char* const ring = lds + group * S::kRingBytes;
  const int e_tiles = (a.E + S::kRowsA - 1) / S::kRowsA, tiles = ((a.F + S::kRowsB - 1) / S::kRowsB) * e_tiles;
  // XCD q = block % 8 takes a contiguous piece of the list ordered by token range first: workgroups that stream the same tokens share an L2
  const int total = tiles * a.splits, per_xcd = (total + 7) >> 3;
  const int q = blockIdx.x & 7, jx = blockIdx.x >> 3, idx = q * per_xcd + jx;
  if (jx >= per_xcd || idx >= total) return;
  const int split = idx / tiles, tile = idx - split * tiles;
  const int ft = tile / e_tiles, et = tile - ft * e_tiles;
  const int f0 = ft * S::kRowsB, e0 = et * S::kRowsA;
  const int wa = wave / S::kWB, wb = wave - wa * S::kWB;
  const int total_blocks = (int)((a.T + 63L) / 64);
  const bool share = total_blocks <= kMostBlocks;   // every workgroup lists all blocks and takes its share of the live ones
  const int s_begin = share ? 0 : split * a.per_split, s_end = share ? total_blocks : min(total_blocks, s_begin + a.per_split);

  __shared__ unsigned long long live_mask[kMostBlocks];   // pad tokens of the blocks with any other token, in order
  __shared__ int live_block[kMostBlocks];
  __shared__ int wave_live[S::kAllWaves];
  int n_live = 0;
  for (int s0 = s_begin; s0 < s_end; s0 += S::kThreads) {
    const int s = s0 + tid;
    unsigned long long mask = ~0ull;
    if (s < s_end) {
      if (a.flags) mask = pad_mask(a.flags, (size_t)a.T, 0, s * 64, a.T);
      else mask = a.T - s * 64 < 64 ? ~0ull << (a.T - s * 64) : 0;
    }
    const unsigned long long ballot = __ballot(mask != ~0ull);
    if (lane == 0) wave_live[wave_id] = __popcll(ballot);
    __syncthreads();
    int at = n_live + __popcll(ballot & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < S::kAllWaves; ++w) {
      if (w < wave_id) at += wave_live[w];
      n_live += wave_live[w];
    }
    if (mask != ~0ull) {
      live_mask[at] = mask;
      live_block[at] = s;
    }
    __syncthreads();
  }
  n_live = __builtin_amdgcn_readfirstlane(n_live);
  const int i_begin = share ? n_live * split / a.splits : 0, i_end = share ? n_live * (split + 1) / a.splits : n_live;

  // ---- operand streams: X tiles (columns e0 ..) then G tiles (columns f0 ..); columns past the last eight repeat those and are not stored
  const unsigned x_stride = (unsigned)a.E * 2, g_stride = (unsigned)a.F * 2;
  unsigned off[S::kLoads];
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) {
    const bool is_x = i < S::kLoadsA;
    const LoadUnit l = load_unit<S::kWaves>(wave, lane, is_x ? i : i - S::kLoadsA);
    off[i] = (unsigned)l.row * (is_x ? x_stride : g_stride) + (unsigned)min((is_x ? e0 : f0) + 64 * l.tile + 8 * l.chunk, (is_x ? a.E : a.F) - 8) * 2;
  }
  const int last_block = total_blocks - 1, last_rows = a.T - 64 * last_block;
  auto issue_stage = [&](int block, int slot) {
    char* st = ring + slot * S::kStageBytes;
    block = __builtin_amdgcn_readfirstlane(block);
    const char* const x_base = uniform_ptr(reinterpret_cast<const char*>(a.x) + (size_t)block * 64 * x_stride);
    const char* const g_base = uniform_ptr(reinterpret_cast<const char*>(a.g) + (size_t)block * 64 * g_stride);
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const bool is_x = i < S::kLoadsA;
      const int y = is_x ? i : i - S::kLoadsA;
      unsigned o = off[i];
      if (block == last_block)   // rows past the end repeat the last one, and are cleared like pad rows
        o -= (unsigned)max(0, load_unit<S::kWaves>(wave, lane, y).row - (last_rows - 1)) * (is_x ? x_stride : g_stride);
      load_to_lds_16(is_x ? x_base : g_base, o, st + (is_x ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, y));
    }
  };

  f32x4 acc[S::kFA][S::kFB];
#pragma unroll
  for (int i = 0; i < S::kFA; ++i)
#pragma unroll
    for (int j = 0; j < S::kFB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float bias_acc[S::kFB];
#pragma unroll
  for (int j = 0; j < S::kFB; ++j) bias_acc[j] = 0.f;
  const bool do_bias = a.out_bias && et == 0 && wa == 0;
  FragOffsets fo;
  frag_offsets<true>(fo, lane);

#pragma unroll
  for (int k = 0; k + 1 < S::kStages; ++k)
    if (i_begin + group + k * S::kGroups < i_end) issue_stage(live_block[i_begin + group + k * S::kGroups], k);
  auto land = [&](int i, int it) {
    wait_vmcnt_le<S::kLoads * (S::kStages - 2)>(max(0, min(S::kStages - 2, (i_end - 1 - i) / S::kGroups)) * S::kLoads);
    const unsigned long long padmask = S::kGroups == 1 || i < i_end ? live_mask[i] : ~0ull;   // (an odd last block leaves group 1 padding only)
    if (padmask) {
      char* st = ring + (it % S::kStages) * S::kStageBytes;
#pragma unroll
      for (int l = 0; l < S::kLoads; ++l) {
        const int y = l < S::kLoadsA ? l : l - S::kLoadsA;
        if ((padmask >> load_unit<S::kWaves>(wave, lane, y).row) & 1ull)
          *reinterpret_cast<uint4*>(st + (l < S::kLoadsA ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, y) + lane * 16) =
              make_uint4(0, 0, 0, 0);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  };
  if (S::kAlternate && group == 1) barrier_no_fence();  // group 1 follows one barrier behind
  for (int i0 = i_begin, it = 0; i0 < i_end; i0 += S::kGroups, ++it) {
    const int i = i0 + group, ahead = i + (S::kStages - 1) * S::kGroups;
    const int next = live_block[min(ahead, i_end - 1)];
    land(i, it);
    barrier_no_fence();          // landed for everyone; and everyone is done with the block before it
    contract_stage<S, true, true, false>(ring + (it % S::kStages) * S::kStageBytes, fo, fo, wa, wb, acc,
                                         [&]() { if (ahead < i_end) issue_stage(next, (it + S::kStages - 1) % S::kStages); },
                                         [&](const bf16x8 (&g)[S::kFB]) {
                                           if (do_bias) {
#pragma unroll
                                             for (int j = 0; j < S::kFB; ++j) bias_acc[j] = sum8(g[j], bias_acc[j]);
                                           }
                                         },
                                         []() {}, []() {});
  }
  if (S::kAlternate && group == 0) barrier_no_fence();
  f32x4 sum[S::kFA][S::kOutB];
  add_groups<S>(acc, sum, lds, group, wave, lane);

  const int r = lane & 15, quarter = lane >> 4;
  if (a.out_bias && et == 0) {
    if (S::kGroups > 1) {  // the other group's column sums
      float* x = reinterpret_cast<float*>(lds);
      __syncthreads();
      if (do_bias && group)
#pragma unroll
        for (int j = 0; j < S::kFB; ++j) x[(wb * S::kFB + j) * 64 + lane] = bias_acc[j];
      __syncthreads();
      if (do_bias && !group)
#pragma unroll
        for (int j = 0; j < S::kFB; ++j) bias_acc[j] += x[(wb * S::kFB + j) * 64 + lane];
    }
    if (do_bias && !group) {
      float* bd = a.splits > 1 ? a.part_bias + (size_t)split * a.F : a.out_bias;
#pragma unroll
      for (int j = 0; j < S::kFB; ++j) {
        const float b = quad_sum(bias_acc[j]);
        const int f = f0 + (wb * S::kFB + j) * 16 + r;
        if (quarter == 0 && f < a.F) bd[f] = b;
      }
    }
  }
  // a lane holds columns 16 i + 4 quarter .. + 3 of row 16 j + r
  float* const to = (a.splits > 1 ? a.part + (size_t)split * a.F * a.E : a.out) + (size_t)f0 * a.E;
#pragma unroll
  for (int j = 0; j < S::kOutB; ++j) {
    const int f = (wb * S::kFB + group * S::kOutB + j) * 16 + r;
#pragma unroll
    for (int i = 0; i < S::kFA; ++i) {
      const int e = e0 + (wa * S::kFA + i) * 16 + 4 * quarter;
      if (f < a.F - f0 && e < a.E) *reinterpret_cast<f32x4*>(to + (size_t)f * a.E + e) = sum[i][j];
    }
  }
}

// For a weight gradient that no product follows.
__global__ __launch_bounds__(256) void add_weight_ranges_kernel(RangeSums s) { add_ranges(s, blockIdx.x, 256); }

using Wgrad256 = Shape<4, 4, 2, 4, 2, 1>;
using Wgrad128 = Shape<2, 2, 2, 2, 2, 1, 2>;

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }
struct WeightGradPlan {
  int splits, per_split, tile;
  size_t bias_off, total;
};
WeightGradPlan plan_weight_grad(int T, int F, int E) {
  WeightGradPlan p = {};
  const int blocks = (int)((T + 63L) / 64);
  constexpr int kSlots = 256;
  double best = 1e30;
  for (int tile : {256, 128}) {
    const long tiles = (long)((F + tile - 1) / tile) * ((E + tile - 1) / tile);
    // enough workgroups for the chip, but ranges of at least eight token blocks
    const int want = (int)std::max<long>({1, std::min(std::max(1L, kSlots / tiles), blocks / 8L), (blocks + kMostBlocks - 1L) / kMostBlocks});
    const int per = (blocks + want - 1) / want, splits = (blocks + per - 1) / per;
    const double rounds = (double)((tiles * splits + kSlots - 1) / kSlots);
    const double cost = rounds * per * (tile == 256 ? 1.9 : 0.7) + (splits > 1 ? splits * 8.0 * F * E / 5.2e6 : 0.0);
    if (cost < best) {
      best = cost;
      p.tile = tile;
      p.per_split = per;
      p.splits = splits;
    }
  }
  p.bias_off = p.splits > 1 ? align256((size_t)p.splits * F * E * 4) : 0;
  p.total = p.bias_off + (p.splits > 1 ? align256((size_t)p.splits * F * 4) : 0) + 256;
  return p;
}
template <class S>
hipError_t launch_weight_grad(const WeightGradArgs& a, hipStream_t stream) {
  const long tiles = (long)((a.F + S::kRowsB - 1) / S::kRowsB) * ((a.E + S::kRowsA - 1) / S::kRowsA);
  const hipError_t e = allow_lds<&linear_wgrad_kernel<S>>(S::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(linear_wgrad_kernel<S>, dim3((unsigned)(8 * ((tiles * a.splits + 7) / 8))), dim3(S::kThreads), S::kLds, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_linear(const LinearCall& c, hipStream_t stream) {
  LinearArgs a = {};
  a.w = static_cast<const unsigned short*>(c.w);
  a.tok = static_cast<const unsigned short*>(c.x);
  a.T = c.T; a.O = c.F; a.K = c.E;
  a.flags = c.flags;
  a.add = static_cast<const unsigned short*>(c.residual);
  a.act = c.act;
  a.bias = c.bias;
  a.y = static_cast<unsigned short*>(c.y);
  a.z = c.z;
  a.z_scales = c.z_scales;
  a.y_codes = c.y_codes;
  a.y_scales = c.y_scales;
  return run_product<false>(a, stream);
}

size_t linear_bwd_workspace(int T, int E, int F, bool codes) {
  return plan_weight_grad(T, F, E).total + (codes ? align256((size_t)T * E * 2) : 0) + 16;   // (the caller's address may be any)
}

hipError_t launch_linear_bwd(const LinearBwdCall& c, hipStream_t stream) {
  LinearArgs a = {};
  if (c.dw) {
    const WeightGradPlan p = plan_weight_grad(c.T, c.F, c.E);
    char* ws = static_cast<char*>(c.workspace);
    ws += -reinterpret_cast<uintptr_t>(ws) & 15;
    WeightGradArgs w = {};
    w.g = static_cast<const unsigned short*>(c.dy);
    w.x = static_cast<const unsigned short*>(c.x);
    if (c.x_scales) {
      void* values = ws + p.total;
      const hipError_t e = launch_checkpoint_unpack(static_cast<const unsigned char*>(c.x), c.x_scales, c.T, c.E, false, values, stream);
      if (e != hipSuccess) return e;
      w.x = static_cast<const unsigned short*>(values);
    }
    w.flags = c.flags;
    w.out = c.dw;
    w.out_bias = c.dbias;
    w.T = c.T; w.F = c.F; w.E = c.E;
    w.splits = p.splits;
    w.per_split = p.per_split;
    w.part = reinterpret_cast<float*>(ws);
    w.part_bias = reinterpret_cast<float*>(ws + p.bias_off);
    const hipError_t e = p.tile == 256 ? launch_weight_grad<Wgrad256>(w, stream) : launch_weight_grad<Wgrad128>(w, stream);
    if (e != hipSuccess) return e;
    if (p.splits > 1) a.ranges = {w.part, w.part_bias, w.out, w.out_bias, (size_t)c.F * c.E, c.F, p.splits, 0};
  }
  if (!c.dx) {
    if (!a.ranges.splits) return hipSuccess;
    a.ranges.blocks = (int)std::max<size_t>(1, std::min<size_t>(1024, a.ranges.n / 4 / 256));
    hipLaunchKernelGGL(add_weight_ranges_kernel, dim3(a.ranges.blocks), dim3(256), 0, stream, a.ranges);
    return hipGetLastError();
  }
  a.w = static_cast<const unsigned short*>(c.w);
  a.tok = static_cast<const unsigned short*>(c.dy);
  a.T = c.T; a.O = c.E; a.K = c.F;
  a.flags = c.flags;
  a.add = static_cast<const unsigned short*>(c.residual);
  a.act = c.z ? c.act : kActNone;
  a.z_in = c.z;
  a.z_in_scales = c.z_scales;
  a.y = static_cast<unsigned short*>(c.dx);
  return run_product<true>(a, stream);
}

}  // namespace mate

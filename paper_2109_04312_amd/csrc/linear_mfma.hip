// The products of a layer's feed-forward half and their gradients, bf16 MFMA (gfx950):
//   forward:  z = x w^T + bias,  y = act(z) + residual, and what the backward needs of them (z in bf16 or in 8 bits, y in 8 bits);
//   dx:       (dy w) act'(z) + a gradient that reached z on another way, z the pre-activation that x came from (without one: that reached x);
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
#include "linear_plan.h"
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
  const unsigned short* add;    // [T][O] or null: residual, or the gradient that is added to dx
  int act;
  const float* bias;            // forward: [O] or null
  const void* z_in;             // dx: pre-activation [T][O], bf16, or codes if z_in_scales is not null
  const unsigned char* z_in_scales;
  unsigned short* y;            // [T][O]
  void* z;                      // forward: bf16, or codes if z_scales is not null; or null
  unsigned char *z_scales, *y_codes, *y_scales;
  int far;                      // y passes the memory-side cache
  RangeSums ranges;
};

// ---- epilogue ------------------------------------------------------------------------------------
// A wavefront's part of a token tensor: rows of its tokens from its first feature on.  Lanes past the last token or feature read zeros and
// write nothing, by the range that the hardware checks, so that no branch stands around an access: the compiler
// counts what is under way, and waits for a read and not for the writes behind it.
struct Part {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ Part(const void* p, int bytes_each, int width, int t_first, int f_first, int T)
      : rsrc(__builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(uniform_ptr(static_cast<const char*>(p) + ((size_t)t_first * width + f_first) * bytes_each)), 0,
            p ? __builtin_amdgcn_readfirstlane((min(T - t_first, 64) * width - f_first) * bytes_each) : 0, 0x00027000)) {}
  __device__ __forceinline__ u32x4 load16(unsigned at) const { return __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, 0, 0); }
  __device__ __forceinline__ uint2 load8(unsigned at) const {
    const auto v = __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, 0, 0);
    return make_uint2(v[0], v[1]);
  }
  __device__ __forceinline__ unsigned load1(unsigned at) const { return __builtin_amdgcn_raw_buffer_load_b8(rsrc, at, 0, 0); }
  template <int kAux = 0>
  __device__ __forceinline__ void store16(unsigned at, u32x4 v) const { __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, at, 0, kAux); }
  template <int kAux = 0>
  __device__ __forceinline__ void store8(unsigned at, unsigned x, unsigned y) const {
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    __builtin_amdgcn_raw_buffer_store_b64(u32x2{x, y}, rsrc, at, 0, kAux);
  }
  __device__ __forceinline__ void store1(unsigned at, unsigned x) const { __builtin_amdgcn_raw_buffer_store_b8((unsigned char)x, rsrc, at, 0, 0); }
};
constexpr unsigned kNowhere = 0x7fffffffu;   // an offset past every part's end
constexpr int kNonTemporal = 2;
// What the backward pass reads (z, codes) is written past the caches, and so is a y that would not be there any more when the next product
// comes to it.  us, y of every size in the caches and past them, 1024 -> 4096 alone and with the product that reads it: 134 MB 153 and
// 136, 270 and 248; 67 MB 70 and 65, 137 and 140; 34 MB 36 and 34, 70 and 73.
constexpr size_t kFarBytes = 96u << 20;

// A wavefront's kFA x kNB blocks of 16 features x 16 tokens, in fp32 until a result is rounded.  They go through LDS, 16 tokens at a time
// (kArea such chunks where there is room), so that a lane holds eight consecutive features of a token: memory is read and written 16 bytes a
// lane, 256 of a token's bytes side by side, and four lanes hold the block of a scale.  Chunk c of 16 bytes of row r lies at slot
// c ^ r ^ (c >> 4): both the accumulators' columns of 16 rows and rows of eight features are free of bank conflicts.
// What is read from memory is read kAhead steps ahead, into registers that the operands no longer need.
enum ZKind { kZNone = 0, kZBf16 = 1, kZCodes = 2 };   // of the pre-activation that is read
template <int kFA, int kNB, int kArea, bool kGrad, int kZ, bool kAdd, int kAct>
__device__ __forceinline__ void finish_as(const LinearStart& p, const LinearArgs& a, const f32x4 (&sum)[kFA][kNB], char* area, int t_first, int f_first) {
  constexpr int kLanes = 2 * kFA, kTokens = 64 / kLanes, kSteps = 16 / kTokens, kRow = kFA * 64, kChunkBytes = 16 * kRow;
  constexpr int kPhase = kArea * kSteps, kAhead = kPhase % 4 == 0 ? 4 : 2;
  static_assert(kNB % kArea == 0 && 64 % kLanes == 0 && kPhase % kAhead == 0, "whole chunks and rows");
  const int lane = threadIdx.x & 63, r = lane & 15, quarter = lane >> 4;
  const int token = lane / kLanes, f_lane = 8 * (lane % kLanes), c = f_lane / 4, scales = scale_blocks(p.O);
  const bool real = f_first + f_lane < p.O;
  f32x4 bias[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  if (!kGrad && a.bias) {
    const f32x4* b = reinterpret_cast<const f32x4*>(a.bias + min(f_first + f_lane, p.O - 8));
    bias[0] = b[0];
    bias[1] = b[1];
  }
  // Padding of the wavefront's tokens, a bit each.
  unsigned long long pads = 0;
  if (a.flags) pads = __ballot(a.flags[min(t_first + lane, p.T - 1)] >= 2);
  const bool masked = pads || f_first + 16 * kFA > p.O;   // does any value not count?
  const Part add(a.add, 2, p.O, t_first, f_first, p.T), y(a.y, 2, p.O, t_first, f_first, p.T);
  const Part z_in(a.z_in, kZ == kZCodes ? 1 : 2, p.O, t_first, f_first, p.T), z_in_scale(a.z_in_scales, 1, scales, t_first, f_first / kScaleBlock, p.T);
  const Part z_out(a.z, a.z_scales ? 1 : 2, p.O, t_first, f_first, p.T), z_scale(a.z_scales, 1, scales, t_first, f_first / kScaleBlock, p.T);
  const Part y_code(a.y_codes, 1, p.O, t_first, f_first, p.T), y_scale(a.y_scales, 1, scales, t_first, f_first / kScaleBlock, p.T);
  // Offsets of a step's values, in elements, and of its scales.
  const unsigned at0 = real ? (unsigned)(token * p.O + f_lane) : kNowhere / 2, at_step = (unsigned)(kTokens * p.O);
  const unsigned scale0 = real ? (unsigned)(token * scales + f_lane / kScaleBlock) : kNowhere, scale_step = (unsigned)(kTokens * scales);
  auto at = [&](int step) { return at0 + (real ? step * at_step : 0u); };
  auto scale_at = [&](int step) { return scale0 + (real ? step * scale_step : 0u); };
  struct Read {
    u32x4 add, z;
    unsigned scale;
  };
  auto fetch = [&](int step) {
    Read x;
    if (kAdd) x.add = add.load16(2 * at(step));
    if (kZ == kZBf16) x.z = z_in.load16(2 * at(step));
    if (kZ == kZCodes) {
      const uint2 w = z_in.load8(at(step));
      x.z = u32x4{w.x, w.y, 0, 0};
      x.scale = z_in_scale.load1(scale_at(step));
    }
    return x;
  };
  const int from = token * kRow + ((c ^ token ^ (c >> 4)) << 4);
  enum { kFarY = 1, kZ16 = 2, kZ8 = 4, kY8 = 8 };
  const int results = __builtin_amdgcn_readfirstlane((a.far ? kFarY : 0) | (a.z ? a.z_scales ? kZ8 : kZ16 : 0) | (a.y_codes ? kY8 : 0));
  Read x[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) x[k] = fetch(k);
#pragma unroll 1
  for (int j0 = 0; j0 < kNB; j0 += kArea) {
#pragma unroll
    for (int k = 0; k < kNB; k += kArea)
      if (k == j0) {
#pragma unroll
        for (int j = 0; j < kArea; ++j)
#pragma unroll
          for (int i = 0; i < kFA; ++i) {
            const int c = 4 * i + quarter;
            *reinterpret_cast<f32x4*>(area + j * kChunkBytes + r * kRow + ((c ^ r ^ (c >> 4)) << 4)) = sum[i][k + j];
          }
      }
#pragma unroll 1
    for (int s0 = 0; s0 < kPhase; s0 += kAhead) {
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int step = j0 * kSteps + s0 + k;
        // rows kTokens (step % kSteps) + token of a chunk: the step's bits and the token's do not meet
        const int in_chunk = (s0 + k) % kSteps * kTokens;
        const char* const chunk = area + (s0 + k) / kSteps * kChunkBytes + in_chunk * kRow;
        const f32x4 lo = *reinterpret_cast<const f32x4*>(chunk + (from ^ (in_chunk << 4))), hi = *reinterpret_cast<const f32x4*>(chunk + (from ^ (in_chunk << 4) ^ 16));
        const Read now = x[k];
        float v[8], z[8];
        if (kZ == kZCodes) {
          const f32x4 z_lo = from_codes(now.z[0], scale_value(now.scale)), z_hi = from_codes(now.z[1], scale_value(now.scale));
#pragma unroll
          for (int e = 0; e < 4; ++e) { z[e] = z_lo[e]; z[4 + e] = z_hi[e]; }
        }
        if (kZ == kZBf16)
#pragma unroll
          for (int e = 0; e < 4; ++e) { z[2 * e] = low_bf16(now.z[e]); z[2 * e + 1] = high_bf16(now.z[e]); }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float s = e < 4 ? lo[e % 4] : hi[e % 4];
          if constexpr (kGrad) {
            v[e] = kZ == kZNone ? s : s * slope<kAct>(z[e]);
          } else {
            z[e] = s + bias[e / 4][e % 4];
            v[e] = activate<kAct>(z[e]);
          }
        }
        if (kAdd)
#pragma unroll
          for (int e = 0; e < 4; ++e) { v[2 * e] += low_bf16(now.add[e]); v[2 * e + 1] += high_bf16(now.add[e]); }
        if (masked) {
          const bool counts = real && !((pads >> (step * kTokens + token)) & 1);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = counts ? v[e] : 0.f;
            if (!kGrad) z[e] = counts ? z[e] : 0.f;
          }
        }
        x[k] = fetch(step + kAhead);   // (past the last step: zeros)
        auto words = [](const float (&x)[8]) { return u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])}; };
        auto store_8bit = [&](const Part& codes, const Part& scales_of, float (&x)[8]) {
          const unsigned s = scale_byte(block_magnitude(x, quad_maximum));
          const float scale = scale_value(s);
          codes.store8<kNonTemporal>(at(step), to_codes(x[0], x[1], x[2], x[3], scale), to_codes(x[4], x[5], x[6], x[7], scale));
          scales_of.store1(lane & 3 ? kNowhere : scale_at(step), s);
        };
        int wanted = results;
        asm volatile("" : "+s"(wanted));   // (tested as a number: lane masks of what never changes would be kept, and made again in every step)
        if (wanted & kFarY) y.store16<kNonTemporal>(2 * at(step), words(v));
        else y.store16(2 * at(step), words(v));
        if (!kGrad && (wanted & kZ16)) z_out.store16<kNonTemporal>(2 * at(step), words(z));
        if (!kGrad && (wanted & kZ8)) store_8bit(z_out, z_scale, z);   // (last, as it may change z)
        if (!kGrad && (wanted & kY8)) store_8bit(y_code, y_scale, v);
      }
    }
  }
}
template <int kFA, int kNB, int kArea, bool kGrad>
__device__ __forceinline__ void finish(const LinearStart& p, const LinearArgs& a, const f32x4 (&sum)[kFA][kNB], char* area, int t_first, int f_first) {
  if (f_first >= p.O || t_first >= p.T) return;   // (the whole wavefront)
  auto as = [&](auto z, auto kind) {
    constexpr int kZ = decltype(z)::value, kAct = decltype(kind)::value;
    if (a.add) finish_as<kFA, kNB, kArea, kGrad, kZ, true, kAct>(p, a, sum, area, t_first, f_first);
    else finish_as<kFA, kNB, kArea, kGrad, kZ, false, kAct>(p, a, sum, area, t_first, f_first);
  };
  typedef std::integral_constant<int, kZNone> NoZ;
  if constexpr (kGrad) {
    if (a.act == kActNone) as(NoZ(), std::integral_constant<int, kActNone>());
    else with_activation(a.act, [&](auto kind) {
      if constexpr (decltype(kind)::value != kActNone) {
        if (a.z_in_scales) as(std::integral_constant<int, kZCodes>(), kind);
        else as(std::integral_constant<int, kZBf16>(), kind);
      }
    });
  } else {
    with_activation(a.act, [&](auto kind) { as(NoZ(), kind); });
  }
}

// One group, two stages of 64 terms: a wavefront reads a slice of 32 terms from LDS while it multiplies the slice before, also across
// the one barrier of a stage, which stands between its two slices: there everyone has read the second one, so that the stage's space can be
// filled again, and the next stage, issued a stage ago, has landed.  Reads and loads are dealt among the products one by one: the
// eight wavefronts' loads of a stage take the address unit half of its products' time, and issued together they keep everyone from multiplying.
// `prepare(s)` is called before the loads of stage s, `load(s, i)` issues one of them (stages 0 and 1 are under way), `landed(s)` is
// called when all of this wavefront's have landed, before others see them; `per_slice` gets operand B of each slice.
template <class S, bool kTA, bool kTB, class Prepare, class Load, class Landed, class PerSlice>
__device__ __forceinline__ void contract_pipelined(const char* ring, int nk, const FragOffsets& fa, const FragOffsets& fb, int wa, int wb,
                                                   f32x4 (&acc)[S::kFA][S::kFB], Prepare&& prepare, Load&& load, Landed&& landed,
                                                   PerSlice&& per_slice) {
  bf16x8 a[2][S::kFA], b[2][S::kFB];
  auto read_a = [&](const char* stage, int k, int i) {
    a[k][i] = read_frag<kTA>(stage + (kTA ? 0 : wa * S::kFA * 16 * 128), fa, (kTA ? wa * S::kFA : 0) + i, k);
  };
  auto read_b = [&](const char* stage, int k, int j) {
    b[k][j] = read_frag<kTB>(stage + S::kA * kTileBytes + (kTB ? 0 : wb * S::kFB * 16 * 128), fb, (kTB ? wb * S::kFB : 0) + j, k);
  };
  // Multiplies slice k; reads slice 1 - k of `stage`; and issues the loads of stage s.
  auto part = [&](auto slice, const char* stage, int s) {
    constexpr int k = decltype(slice)::value, kEach = (S::kLoads + S::kFA - 1) / S::kFA;
#pragma unroll
    for (int i = 0; i < S::kFA; ++i) {
      if (k == 1 && s < nk)
#pragma unroll
        for (int l = i * kEach; l < min((i + 1) * kEach, S::kLoads); ++l) load(s, l);
#pragma unroll
      for (int j = i * S::kFB / S::kFA; j < (i + 1) * S::kFB / S::kFA; ++j) read_b(stage, 1 - k, j);
      read_a(stage, 1 - k, i);
#pragma unroll
      for (int j = 0; j < S::kFB; ++j) acc[i][j] = mfma16(a[k][i], b[k][j], acc[i][j]);
      __builtin_amdgcn_sched_barrier(0);
    }
    per_slice(b[k]);
  };
  // lgkmcnt(0), in the form that the compiler takes account of: with asm it waits for the next slice's reads before the first product
  constexpr int kReadsDone = 0xc07f;
  wait_vmcnt_le<S::kLoads>(nk > 1 ? S::kLoads : 0);
  landed(0);
  barrier_no_fence();
#pragma unroll
  for (int j = 0; j < S::kFB; ++j) read_b(ring, 0, j);
#pragma unroll
  for (int i = 0; i < S::kFA; ++i) read_a(ring, 0, i);
  __builtin_amdgcn_s_waitcnt(kReadsDone);
  for (int s = 0; s < nk; ++s) {
    const char *now = ring + (s & 1) * S::kStageBytes, *next = ring + (~s & 1) * S::kStageBytes;
    __builtin_amdgcn_sched_barrier(0);
    part(std::integral_constant<int, 0>(), now, 0);
    __builtin_amdgcn_s_waitcnt(kReadsDone);
    if (s + 1 < nk) {
      wait_vmcnt_le<0>(0);
      landed(s + 1);
    }
    barrier_no_fence();
    __builtin_amdgcn_sched_barrier(0);
    if (s + 2 < nk) prepare(s + 2);
    part(std::integral_constant<int, 1>(), next, s + 2);   // (behind the last stage it reads whatever is there, for nothing)
    __builtin_amdgcn_s_waitcnt(kReadsDone);
  }
}

// A tile, over the terms from stage `first` on, up to term k_end; merge(sums): whether this workgroup is the one that goes on with them.
template <class S, bool kGrad, class Merge>
__device__ __forceinline__ void linear_tile(const LinearStart& p, const LinearArgs& a, char* lds, int t0, int f0, int first, int k_end, Merge&& merge) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_id = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = wave_id / S::kWaves, wave = wave_id - group * S::kWaves;
  const int wa = wave / S::kWB, wb = wave - wa * S::kWB;
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
  const char *w_ptr = w0 + (first + group) * w_step, *x_ptr = x0 + (size_t)(first + group) * 128;   // of the next stage
  const int stages = ((k_end + 63) >> 6) - first, nk = (stages + S::kGroups - 1) / S::kGroups;   // nk: this group's, the last one short or empty
  const int short_k = 64 * (first + (nk - 1) * S::kGroups + group);   // its first term
  const bool is_short = short_k + 64 > k_end;
  // Before a stage's loads: the short one's repeat the last 16 bytes, or rows (no other stage follows).
  auto prepare_stage = [&](int g) {
    if (__builtin_expect(g == nk - 1 && is_short, 0)) {
      const int row0 = min(short_k, k_end - 1);
      w_ptr = kGrad ? w0 + (size_t)row0 * p.O * 2 : w0;
      x_ptr = x0;
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i) {
        const bool is_a = i < S::kLoadsA;
        const LoadUnit l = load_unit<S::kWaves>(wave, lane, is_a ? i : i - S::kLoadsA);
        if (kGrad && is_a) off[i] -= (unsigned)(l.row - (min(short_k + l.row, k_end - 1) - row0)) * (unsigned)p.O * 2;
        else off[i] += (unsigned)min(short_k + 8 * l.chunk, k_end - 8) * 2 - l.chunk * 16;
      }
    }
  };
  auto load_one = [&](int g, int i) {
    char* st = ring + (g % S::kStages) * S::kStageBytes;
    const bool is_a = i < S::kLoadsA;
    load_to_lds_16(uniform_ptr(is_a ? w_ptr : x_ptr), off[i],
                   st + (is_a ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, is_a ? i : i - S::kLoadsA));
    if (i == S::kLoads - 1) {
      w_ptr += S::kGroups * w_step;
      x_ptr += S::kGroups * 128;
    }
  };
  auto issue_stage = [&](int g) {
    prepare_stage(g);
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) load_one(g, i);
  };
  // My share of the short stage, landed, is zero from the last term on.
  auto clear_short = [&]() {
    char* st = ring + ((nk - 1) % S::kStages) * S::kStageBytes;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const bool is_a = i < S::kLoadsA;
      const int y = is_a ? i : i - S::kLoadsA;
      const LoadUnit l = load_unit<S::kWaves>(wave, lane, y);
      if (short_k + (kGrad && is_a ? l.row : 8 * l.chunk) >= k_end)
        *reinterpret_cast<uint4*>(st + (is_a ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, y) + lane * 16) = make_uint4(0, 0, 0, 0);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  constexpr bool kPipelined = S::kGroups == 1 && S::kStages == 2;
#pragma unroll
  for (int s = 0; s < (kPipelined ? S::kStages : S::kStages - 1); ++s)
    if (s < nk) issue_stage(s);

  // While the first stages travel: is any token of the tile not padding (every wavefront looks at all of them)?
  bool any = !a.flags;
  if (a.flags) {
#pragma unroll
    for (int i = 0; i < S::kB; ++i) any |= a.flags[t0 + min(64 * i + lane, rows - 1)] < 2;
  }

  f32x4 acc[S::kFA][S::kFB];
#pragma unroll
  for (int i = 0; i < S::kFA; ++i)
#pragma unroll
    for (int j = 0; j < S::kFB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (__any(any)) {  // (a tile of padding only is stored as zeros without arithmetic)
    FragOffsets fa, fb;
    frag_offsets<kGrad>(fa, lane);
    frag_offsets<false>(fb, lane);
    if constexpr (kPipelined) {
      contract_pipelined<S, kGrad, false>(ring, nk, fa, fb, wa, wb, acc, prepare_stage, load_one,
                                          [&](int s) { if (__builtin_expect(is_short && s == nk - 1, 0)) clear_short(); },
                                          [](const bf16x8 (&)[S::kFB]) {});
    } else {
    // the second group follows one barrier behind
    const bool apart = S::kAlternate, second = group == 1;
    if (apart && second) barrier_no_fence();
    for (int ks = 0; ks < nk; ++ks) {
      // stage ks has landed: everything but the younger stages' loads (fewer near the end)
      wait_vmcnt_le<S::kLoads * (S::kStages - 2)>(min(S::kStages - 2, nk - 1 - ks) * S::kLoads);
      if (__builtin_expect(is_short && ks == nk - 1, 0)) clear_short();
      barrier_no_fence();  // ... for every wavefront, and everyone is done with stage ks - 1
      contract_stage<S, kGrad, false, false>(ring + (ks % S::kStages) * S::kStageBytes, fa, fb, wa, wb, acc,
                                             [&]() { if (ks + S::kStages - 1 < nk) issue_stage(ks + S::kStages - 1); },
                                             [](const bf16x8 (&)[S::kFB]) {}, []() {}, []() {});
    }
    if (apart && !second) barrier_no_fence();
    }
  } else {
    wait_vmcnt_le<0>(0);   // (the first stages' loads, which the compiler does not know of: their place is scratch from here on)
  }
  f32x4 sum[S::kFA][S::kOutB];
  add_groups<S>(acc, sum, lds, group, wave, lane);
  if (!merge(sum, wave_id)) return;

  constexpr int kWaveArea = S::kLds / S::kAllWaves / 1024 * 1024, kFit = std::min(S::kOutB, kWaveArea / (S::kFA * 1024));
  constexpr int kArea = S::kOutB % kFit == 0 ? kFit : kFit - 1;
  __syncthreads();   // (everyone is done with the stages)
  finish<S::kFA, S::kOutB, kArea, kGrad>(p, a, sum, lds + wave_id * kWaveArea, t0 + (wb * S::kFB + group * S::kOutB) * 16, f0 + wa * S::kFA * 16);
}

template <class S, bool kGrad>
__device__ __forceinline__ void linear_tile(const LinearStart& p, const LinearArgs& a, char* lds, int t0, int f0) {
  linear_tile<S, kGrad>(p, a, lds, t0, f0, 0, p.K, [](f32x4 (&)[S::kFA][S::kOutB], int) { return true; });
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
void deal_tiles(LinearArgs& a) {
  TileDeal& d = a.deal;
  d.tokens = (int)((a.T + (long)S::kRowsB - 1) / S::kRowsB);
  d.features = (a.O + S::kRowsA - 1) / S::kRowsA;
  d.by_feature = a.O > a.T && d.features >= 8;   // (every XCD reads all of the other operand: the smaller one)
  d.rows = (d.by_feature ? d.features : d.tokens) / 8;
  a.far = (size_t)a.T * a.O * 2 > kFarBytes;
}
template <class S, bool kGrad>
hipError_t launch_product(LinearArgs a, hipStream_t stream) {
  deal_tiles<S>(a);
  const TileDeal& d = a.deal;
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
template <bool kGrad>
hipError_t launch_product(ProductForm form, const LinearArgs& a, hipStream_t stream) {
  switch (form) {
    case kProduct256: return launch_product<Tile256, kGrad>(a, stream);
    case kProduct128: return launch_product<Tile128, kGrad>(a, stream);
    case kProduct128x2: return launch_product<Tile128x2, kGrad>(a, stream);
    case kProduct64: return launch_product<Tile64, kGrad>(a, stream);
    case kProduct64x2: return launch_product<Tile64x2, kGrad>(a, stream);
  }
  return hipErrorInvalidValue;
}

// Few tiles of a long contraction: each is shared by the workgroups of several ranges of it, whose sums the launch adds.  Ranges of all
// tiles follow each other, so that every XCD has the same tiles in each.
template <class S, bool kGrad>
__device__ __forceinline__ void split_tile(const LinearStart& p, const LinearArgs& a, const RangeMerge& m, char* lds, int range, int token_tile, int feature_tile) {
  const int stages = (p.K + 63) >> 6;
  linear_tile<S, kGrad>(p, a, lds, token_tile * S::kRowsB, feature_tile * S::kRowsA, stages * range / m.splits,
                        min(p.K, 64 * (stages * (range + 1) / m.splits)), [&](f32x4 (&sum)[S::kFA][S::kOutB], int wave_id) {
                          float none[S::kFB] = {};
                          return merge_ranges<S>(m, range, token_tile * p.deal.features + feature_tile, 0, false, sum, none, wave_id);
                        });
}
template <class S, bool kGrad>
__global__ __launch_bounds__(S::kThreads, S::kAllWaves / 4 * S::kPerCU) void linear_split_kernel(const unsigned short* w, const unsigned short* tok, int T,
                                                                                               int O, int K, int token_tiles, int feature_tiles,
                                                                                               int whole_rows, int by_feature, RangeMerge m, LinearArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const LinearStart p = {w, tok, T, O, K, {token_tiles, feature_tiles, whole_rows, by_feature}};
  int y, token_tile, feature_tile;
  const int range = uniform_div(blockIdx.y, p.deal.grid_y(), y);
  if (dealt_tile(p.deal, blockIdx.x, y, token_tile, feature_tile)) split_tile<S, kGrad>(p, a, m, lds, range, token_tile, feature_tile);
}
template <class S>
RangeMerge merge_in(void* workspace, size_t tiles, int splits, unsigned long long ticket) {
  RangeMerge m = {static_cast<float*>(workspace), nullptr, nullptr, ticket, splits, (int)tiles, 0};
  m.arrived = reinterpret_cast<unsigned long long*>(m.part + (size_t)splits * tiles * S::kRowsA * S::kRowsB);
  return m;
}
template <class S, bool kGrad>
hipError_t launch_split(LinearArgs a, int splits, void* workspace, unsigned long long ticket, hipStream_t stream) {
  deal_tiles<S>(a);
  const TileDeal& d = a.deal;
  const RangeMerge m = merge_in<S>(workspace, (size_t)d.tokens * d.features, splits, ticket);
  const hipError_t e = allow_lds<&linear_split_kernel<S, kGrad>>(S::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((linear_split_kernel<S, kGrad>), dim3(d.grid_x(), d.grid_y() * splits), dim3(S::kThreads), S::kLds, stream, a.w, a.tok, a.T, a.O, a.K,
                     d.tokens, d.features, d.rows, d.by_feature, m, a);
  return hipGetLastError();
}

// ---- few tokens ------------------------------------------------------------------------------------
// Where tiles of 128 features leave most units idle, what takes time is latency, and how much a unit can read at a time (some 35 GB/s).
// A workgroup has 4 to 32 features and 16 to 64 tokens; its wavefronts share the contraction, each a piece of it, and read operands straight from
// memory into registers.  Their sums are added through LDS, in the order of the wavefronts.
// kRows < 16: where 16 features a workgroup leave units without one, a workgroup has 8 or 4, and the 16 rows of an operand are those at 2
// or 4 places of the contraction, each multiplied with the tokens at all of these places, of which one product in 2 or 4 counts (there
// is time for that).
template <int kRows, int kFA, int kFB>
__global__ __launch_bounds__(512) void few_kernel(const unsigned short* w, const unsigned short* tok, int T, int O, int K, LinearArgs a) {
  constexpr int kWaves = 8, kParts = 16 / kRows, kBlocks = kFA * kFB;
  constexpr int kDepth = std::max(1, 4 / kParts / (kFB > 2 ? 2 : 1) / kFA);   // steps whose loads travel together
  static_assert((kParts == 1 || kFA == 1) && kBlocks <= kWaves, "a wavefront for each block of results");
  __shared__ f32x4 part[kWaves][kBlocks][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
  const int f0 = blockIdx.x * (kRows * kFA), t0 = blockIdx.y * (16 * kFB);
  const int first = 64 * (r / kRows) + 8 * q;   // of this lane's terms of the weights in a step
  const unsigned short *rows_w[kFA], *rows_x[kFB];
#pragma unroll
  for (int i = 0; i < kFA; ++i) rows_w[i] = w + (size_t)min(f0 + 16 * i + r % kRows, O - 1) * K + first;
#pragma unroll
  for (int j = 0; j < kFB; ++j) rows_x[j] = tok + (size_t)min(t0 + 16 * j + r, T - 1) * K + 8 * q;
  f32x4 acc[kParts][kFA][kFB];
#pragma unroll
  for (int s = 0; s < kParts; ++s)
#pragma unroll
    for (int i = 0; i < kFA; ++i)
#pragma unroll
      for (int j = 0; j < kFB; ++j) acc[s][i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  bf16x8 fw[kDepth][kFA][2], fx[kDepth][kParts][kFB][2];
  auto multiply = [&](int d) {
#pragma unroll
    for (int s = 0; s < kParts; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kFA; ++i)
#pragma unroll
          for (int j = 0; j < kFB; ++j) acc[s][i][j] = mfma16_apart(fw[d][i][h], fx[d][s][j][h], acc[s][i][j]);
  };
  constexpr int kTerms = 64 * kParts;   // of a step
  auto load = [&](int d, int c, auto&& one) {   // one(address, first term)
    const int at = c * kTerms;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int i = 0; i < kFA; ++i) fw[d][i][h] = one(rows_w[i] + at + 32 * h, at + first + 32 * h);
#pragma unroll
      for (int s = 0; s < kParts; ++s)
#pragma unroll
        for (int j = 0; j < kFB; ++j) fx[d][s][j][h] = one(rows_x[j] + at + 64 * s + 32 * h, at + 64 * s + 8 * q + 32 * h);
    }
  };
  const int steps = (K + kTerms - 1) / kTerms, each = (steps + kWaves - 1) / kWaves, end = min(steps, (wave + 1) * each), whole = min(end, K / kTerms);
  int c = wave * each;
  for (; c + kDepth <= whole; c += kDepth) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) load(d, c + d, [](const unsigned short* p, int) { return *reinterpret_cast<const bf16x8*>(p); });
#pragma unroll
    for (int d = 0; d < kDepth; ++d) multiply(d);
  }
  for (; c < end; c += kDepth) {   // the last ones: what is past the end is zero
    const int stop = min(K, end * kTerms);
#pragma unroll
    for (int d = 0; d < kDepth; ++d)
      load(d, c + d, [&](const unsigned short* p, int k) { return k < stop ? *reinterpret_cast<const bf16x8*>(p) : bf16x8{}; });
#pragma unroll
    for (int d = 0; d < kDepth; ++d) multiply(d);
  }
  // Rows 4 q .. + 3 of a product: kRows = 4: features 0 .. 3 at place q; 8: features 4 (q % 2) .. + 3 at place q / 2.
#pragma unroll
  for (int i = 0; i < kFA; ++i)
#pragma unroll
    for (int j = 0; j < kFB; ++j) {
      f32x4 x = acc[0][i][j];
#pragma unroll
      for (int s = 1; s < kParts; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = q * kParts / 4 == s ? acc[s][i][j][e] : x[e];
      part[wave][i * kFB + j][lane] = x;
    }
  __syncthreads();
  const bool codes = kFA == 2 && (a.z_scales || a.y_codes);
  if (wave >= kBlocks && !codes) return;
  f32x4 z = {0.f, 0.f, 0.f, 0.f}, y = z;
  if (wave < kBlocks) {
    z = part[0][wave][lane];
#pragma unroll
    for (int v = 1; v < kWaves; ++v) z += part[v][wave][lane];
    if (kParts > 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) z[e] = kParts == 4 ? quad_sum(z[e]) : half_sum(z[e]);
    const int i = wave / kFB, t = t0 + 16 * (wave - i * kFB) + r, f = f0 + 16 * i + 4 * q;   // a lane's four features of a token
    const bool real = t < T && f < O && 4 * q < kRows;
    if (!codes && !real) return;
    const size_t at = (size_t)t * O + f;
    uint2 add = make_uint2(0, 0);
    if (a.add && real) add = *reinterpret_cast<const uint2*>(a.add + at);
    if (a.bias && real) z += *reinterpret_cast<const f32x4*>(a.bias + f);
    const bool pad = !real || (a.flags && a.flags[t] >= 2);
    with_activation(a.act, [&](auto kind) {
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = activate<decltype(kind)::value>(z[e]);
    });
    if (a.add) y += f32x4{low_bf16(add.x), high_bf16(add.x), low_bf16(add.y), high_bf16(add.y)};
    if (pad) y = z = f32x4{0.f, 0.f, 0.f, 0.f};
    if (real) {
      if (a.z && !a.z_scales) *reinterpret_cast<uint2*>(static_cast<unsigned short*>(a.z) + at) = make_uint2(pack2(z[0], z[1]), pack2(z[2], z[3]));
      *reinterpret_cast<uint2*>(a.y + at) = make_uint2(pack2(y[0], y[1]), pack2(y[2], y[3]));
    }
  }
  if constexpr (kFA == 2) {
    // 8 bits: the workgroup's 32 features of a token have one scale.  Through LDS, so that four lanes have a token, eight features each.
    if (!codes) return;
    constexpr int kTokens = 16 * kFB;
    static_assert(2 * kTokens * 32 * sizeof(float) <= sizeof(part) && 4 * kTokens <= 512, "room for both, and a thread for eight values");
    f32x4* const staged = &part[0][0][0];   // [z, y][token][four features]
    __syncthreads();                        // (the sums have been read)
    if (wave < kBlocks) {
      const int i = wave / kFB, to = (16 * (wave - i * kFB) + r) * 8 + 4 * i + q;
      staged[to] = z;
      staged[kTokens * 8 + to] = y;
    }
    __syncthreads();
    if ((int)threadIdx.x >= 4 * kTokens) return;
    const int token = threadIdx.x >> 2, t = t0 + token, f = f0 + 8 * (threadIdx.x & 3), scales = scale_blocks(O);
    const bool real = t < T && f < O;
    auto keep = [&](const f32x4* from, unsigned char* to, unsigned char* scales_to) {
      const f32x4 lo = from[token * 8 + 2 * (threadIdx.x & 3)], hi = from[token * 8 + 2 * (threadIdx.x & 3) + 1];
      float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      const unsigned s = scale_byte(block_magnitude(v, quad_maximum));
      const float scale = scale_value(s);
      if (!real) return;
      *reinterpret_cast<uint2*>(to + (size_t)t * O + f) = make_uint2(to_codes(v[0], v[1], v[2], v[3], scale), to_codes(v[4], v[5], v[6], v[7], scale));
      if ((threadIdx.x & 3) == 0) scales_to[(size_t)t * scales + f / kScaleBlock] = (unsigned char)s;
    };
    if (a.z_scales) keep(staged, static_cast<unsigned char*>(a.z), a.z_scales);
    if (a.y_codes) keep(staged + kTokens * 8, a.y_codes, a.y_scales);
  }
}
template <int kRows, int kFA, int kFB>
hipError_t launch_few(LinearArgs a, hipStream_t stream) {
  const dim3 grid((a.O + kRows * kFA - 1) / (kRows * kFA), (a.T + 16 * kFB - 1) / (16 * kFB));
  hipLaunchKernelGGL((few_kernel<kRows, kFA, kFB>), grid, dim3(512), 0, stream, a.w, a.tok, a.T, a.O, a.K, a);
  return hipGetLastError();
}
hipError_t launch_few(const FewForm& f, const LinearArgs& a, hipStream_t stream) {
  if (f.blocks == 2) return f.tokens == 1 ? launch_few<16, 2, 1>(a, stream) : f.tokens == 2 ? launch_few<16, 2, 2>(a, stream) : launch_few<16, 2, 4>(a, stream);
  if (f.rows < 16) return f.rows == 4 ? launch_few<4, 1, 1>(a, stream) : launch_few<8, 1, 1>(a, stream);
  return f.tokens == 1 ? launch_few<16, 1, 1>(a, stream) : f.tokens == 2 ? launch_few<16, 1, 2>(a, stream) : launch_few<16, 1, 4>(a, stream);
}
// ======================================================================================
// Gradient with respect to the weights
// ======================================================================================
// Both operands are token-major, so their 64-token x 64-column tiles go into LDS as they are and both are read transposed.  A
// workgroup owns a tile of dw and a range of the token blocks; the ranges' sums are added in a fixed order (no atomic
// additions: the result is bit-reproducible), in the launch (kMerge) or after it.  The bias gradient rides along in the workgroups of the first
// column tile.  Rows of pad tokens are cleared in LDS after a block has landed, and blocks of padding only are skipped.
// x in 8 bits (kCodes) passes through registers: 16 codes of a token and their scale become bf16 (exactly, but for values below 2^-130) on the way to LDS.  That takes
// a stage a third of a microsecond longer, in every tile that reads them; where a copy in bf16, written and read again, takes
// less, the values are copied into the workspace first.  (us, dw with a copy and so: 16384 tokens, 4096 x 1024 178 and 151, 1024 x 4096 139 and 152,
// 4072 tokens, 2048 x 768 36 and 59.)
struct WeightGradArgs {
  const unsigned short* g;       // [T][F]
  const void* x;                 // [T][E], bf16, or codes if x_scales is not null
  const unsigned char* x_scales;
  const unsigned char* flags;    // [T] or null
  float *out, *out_bias;         // [F][E], [F] or null
  float *part, *part_bias;       // the ranges' sums (splits > 1)
  unsigned long long *arrived, ticket;
  int T, F, E;
  int splits, per_split;         // ranges of 64-token blocks
};
template <class S, bool kMerge, bool kCodes>
__device__ __forceinline__ void weight_grad_tile(const WeightGradArgs& a, char* lds, int workgroup) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave_id = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = wave_id / S::kWaves, wave = wave_id - group * S::kWaves;
  char* const ring = lds + group * S::kRingBytes;
  const int e_tiles = (a.E + S::kRowsA - 1) / S::kRowsA, f_tiles = (a.F + S::kRowsB - 1) / S::kRowsB, tiles = f_tiles * e_tiles;
  // XCD q = workgroup % 8 takes a contiguous piece of the list ordered by token range first: workgroups that stream the same tokens share an L2
  const int total = tiles * a.splits, per_xcd = (total + 7) >> 3;
  const int q = workgroup & 7, jx = workgroup >> 3, idx = q * per_xcd + jx;
  if (jx >= per_xcd || idx >= total) return;
  const int split = idx / tiles, tile = idx - split * tiles;
  const int ft = tile / e_tiles, et = tile - ft * e_tiles;
  const int f0 = ft * S::kRowsB, e0 = et * S::kRowsA;
  const int wa = wave / S::kWB, wb = wave - wa * S::kWB;
  const int total_blocks = (int)((a.T + 63L) / 64);
  constexpr int kList = kMerge ? kMergeBlocks : kMostBlocks;
  const bool share = kMerge || total_blocks <= kList;   // every workgroup lists all blocks and takes its share of the live ones
  const int s_begin = share ? 0 : split * a.per_split, s_end = share ? total_blocks : min(total_blocks, s_begin + a.per_split);

  __shared__ unsigned long long live_mask[kList];   // pad tokens of the blocks with any other token, in order
  __shared__ int live_block[kList];
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
  const int last_block = total_blocks - 1, last_rows = a.T - 64 * last_block;

  // ---- operand streams: X tiles (columns e0 ..) then G tiles (columns f0 ..); columns past the last eight repeat those and are not
  // stored, rows past the end repeat the last one and are cleared like pad rows
  const unsigned x_stride = (unsigned)a.E * 2, g_stride = (unsigned)a.F * 2;
  constexpr int kFirst = kCodes ? S::kLoadsA : 0;   // loads that go straight to LDS
  unsigned off[S::kLoads];
#pragma unroll
  for (int i = kFirst; i < S::kLoads; ++i) {
    const bool is_x = i < S::kLoadsA;
    const LoadUnit l = load_unit<S::kWaves>(wave, lane, is_x ? i : i - S::kLoadsA);
    off[i] = (unsigned)l.row * (is_x ? x_stride : g_stride) + (unsigned)min((is_x ? e0 : f0) + 64 * l.tile + 8 * l.chunk, (is_x ? a.E : a.F) - 8) * 2;
  }
  auto issue_stage = [&](int block, int slot) {
    char* st = ring + slot * S::kStageBytes;
    block = __builtin_amdgcn_readfirstlane(block);
    const char* const x_base = uniform_ptr(static_cast<const char*>(a.x) + (size_t)block * 64 * x_stride);
    const char* const g_base = uniform_ptr(reinterpret_cast<const char*>(a.g) + (size_t)block * 64 * g_stride);
#pragma unroll
    for (int i = kFirst; i < S::kLoads; ++i) {
      const bool is_x = i < S::kLoadsA;
      const int y = is_x ? i : i - S::kLoadsA;
      unsigned o = off[i];
      if (block == last_block) o -= (unsigned)max(0, load_unit<S::kWaves>(wave, lane, y).row - (last_rows - 1)) * (is_x ? x_stride : g_stride);
      load_to_lds_16(is_x ? x_base : g_base, o, st + (is_x ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, y));
    }
  };
  // Codes: a lane has 16 columns of a row, kUnits times; four lanes a row, sixteen rows and one tile of 64 columns a wavefront.
  constexpr int kUnits = kCodes ? S::kA * 4 / S::kWaves : 0, kUnitsHere = kCodes ? kUnits : 1;
  static_assert(!kCodes || (S::kA * 4 % S::kWaves == 0 && S::kStages == 2), "codes divide evenly, and are one stage ahead of their values");
  struct Raw { unsigned w[4], scale; } raw[kUnitsHere];
  const int scales = scale_blocks(a.E);
  auto unit_tile = [&](int u) { return (wave + S::kWaves * u) >> 2; };
  auto unit_row = [&](int u) { return ((wave + S::kWaves * u) & 3) * 16 + (lane >> 2); };
  auto unit_column = [&](int u) { return e0 + 64 * unit_tile(u) + 16 * (lane & 3); };
  auto read_codes = [&](int block) {
    block = __builtin_amdgcn_readfirstlane(block);
    const unsigned char* const base = static_cast<const unsigned char*>(a.x) + (size_t)block * 64 * a.E;
    const unsigned char* const scale_base = a.x_scales + (size_t)block * 64 * scales;
    const int most = block == last_block ? last_rows - 1 : 63;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int row = min(unit_row(u), most), column = unit_column(u);
      // (rows begin at multiples of 8: two halves, the second one past the row's end repeats the last eight)
      const uint2 lo = *reinterpret_cast<const uint2*>(base + (unsigned)row * (unsigned)a.E + min(column, a.E - 8));
      const uint2 hi = *reinterpret_cast<const uint2*>(base + (unsigned)row * (unsigned)a.E + min(column + 8, a.E - 8));
      raw[u].w[0] = lo.x; raw[u].w[1] = lo.y; raw[u].w[2] = hi.x; raw[u].w[3] = hi.y;
      raw[u].scale = scale_base[(unsigned)row * (unsigned)scales + min(column, a.E - 8) / kScaleBlock];
    }
  };
  auto write_values = [&](unsigned long long padmask, int slot) {
    char* const st = ring + slot * S::kStageBytes;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int row = unit_row(u), chunk = 2 * (lane & 3);
      const bool pad = (padmask >> row) & 1ull;
      const float scale = scale_value(raw[u].scale);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint2 lo = bf16_from_codes(raw[u].w[2 * h], scale), hi = bf16_from_codes(raw[u].w[2 * h + 1], scale);
        const uint4 v = pad ? make_uint4(0, 0, 0, 0) : make_uint4(lo.x, lo.y, hi.x, hi.y);
        *reinterpret_cast<uint4*>(st + unit_tile(u) * kTileBytes + row * 128 + (((chunk + h) ^ swz(row & 15)) << 4)) = v;
      }
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

  // this group's blocks: i_begin + group, + kGroups, ...  (An odd last block leaves group 1 a block of padding only.)
  auto pads_of = [&](int i) { return i < i_end ? live_mask[min(i, i_end - 1)] : ~0ull; };
#pragma unroll
  for (int k = 0; k + 1 < S::kStages; ++k)
    if (i_begin + group + k * S::kGroups < i_end) issue_stage(live_block[i_begin + group + k * S::kGroups], k);
  auto block_at = [&](int i) { return live_block[min(i, i_end - 1)]; };
  if (kCodes && i_begin < i_end) {
    read_codes(block_at(i_begin + group));
    write_values(pads_of(i_begin + group), 0);
    read_codes(block_at(i_begin + group + S::kGroups));
  }
  auto land = [&](int i, int it) {
    wait_vmcnt_le<S::kLoads * (S::kStages - 2)>(max(0, min(S::kStages - 2, (i_end - 1 - i) / S::kGroups)) * S::kLoads);
    const unsigned long long padmask = pads_of(i);
    if (padmask) {
      char* st = ring + (it % S::kStages) * S::kStageBytes;
#pragma unroll
      for (int l = kFirst; l < S::kLoads; ++l) {
        const int y = l < S::kLoadsA ? l : l - S::kLoadsA;
        if ((padmask >> load_unit<S::kWaves>(wave, lane, y).row) & 1ull)
          *reinterpret_cast<uint4*>(st + (l < S::kLoadsA ? 0 : S::kA * kTileBytes) + load_dst<S::kWaves>(wave, y) + lane * 16) =
              make_uint4(0, 0, 0, 0);
      }
    }
    if (padmask || kCodes) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };
  if (S::kAlternate && group == 1) barrier_no_fence();  // group 1 follows one barrier behind
  for (int i0 = i_begin, it = 0; i0 < i_end; i0 += S::kGroups, ++it) {
    const int i = i0 + group, ahead = i + (S::kStages - 1) * S::kGroups;
    const int next = block_at(ahead), later = kCodes ? block_at(ahead + S::kGroups) : 0;
    const unsigned long long next_pads = kCodes ? pads_of(ahead) : 0;
    land(i, it);
    barrier_no_fence();          // landed for everyone; and everyone is done with the block before it
    contract_stage<S, true, true, false>(ring + (it % S::kStages) * S::kStageBytes, fo, fo, wa, wb, acc,
                                         [&]() {
                                           // (the codes have landed with this stage; behind loads to LDS, which the compiler does not
                                           // see, it would wait for those as well)
                                           if (kCodes && i0 + S::kGroups < i_end) write_values(next_pads, (it + 1) % S::kStages);
                                           if (ahead < i_end) issue_stage(next, (it + S::kStages - 1) % S::kStages);
                                           if (kCodes && i0 + S::kGroups < i_end) read_codes(later);
                                         },
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
  float bias_sum[S::kFB];   // of row 16 j + r, in group 0's wavefronts of the first columns
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
#pragma unroll
    for (int j = 0; j < S::kFB; ++j) bias_sum[j] = quad_sum(bias_acc[j]);
  }
  const bool has_bias = do_bias && !group;
  if constexpr (kMerge) {
    const RangeMerge m = {a.part, a.part_bias, a.arrived, a.ticket, a.splits, tiles, f_tiles * S::kRowsB};
    if (a.splits > 1 && !merge_ranges<S>(m, split, tile, f0 + wb * S::kFB * 16, has_bias, sum, bias_sum, wave_id)) return;
  }
  const bool partial = !kMerge && a.splits > 1;
  if (has_bias) {
    float* bd = partial ? a.part_bias + (size_t)split * a.F : a.out_bias;
#pragma unroll
    for (int j = 0; j < S::kFB; ++j) {
      const int f = f0 + (wb * S::kFB + j) * 16 + r;
      if (quarter == 0 && f < a.F) bd[f] = bias_sum[j];
    }
  }
  // a lane holds columns 16 i + 4 quarter .. + 3 of row 16 j + r
  float* const to = (partial ? a.part + (size_t)split * a.F * a.E : a.out) + (size_t)f0 * a.E;
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
template <class S, bool kMerge, bool kCodes>
__global__ __launch_bounds__(S::kThreads, S::kAllWaves / 4 * S::kPerCU) void weight_grad_kernel(WeightGradArgs a) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  weight_grad_tile<S, kMerge, kCodes>(a, lds, blockIdx.x);
}

// For a weight gradient that no product follows.
__global__ __launch_bounds__(256) void add_weight_ranges_kernel(RangeSums s) { add_ranges(s, blockIdx.x, 256); }

template <class S, bool kCodes>
__global__ __launch_bounds__(S::kThreads, S::kAllWaves / 4) void linear_bwd_kernel(WeightGradArgs w, LinearArgs a, RangeMerge m, int w_groups) {
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  static_assert(S::kThreads == Wgrad128::kThreads, "one workgroup size for both");
  if ((int)blockIdx.x < w_groups) {
    weight_grad_tile<Wgrad128, true, kCodes>(w, lds, blockIdx.x);
  } else {
    int x, token_tile, feature_tile, at = blockIdx.x - w_groups;
    const int range = S::kB == 1 && m.splits > 1 ? uniform_div(at, a.deal.grid_x() * a.deal.grid_y(), at) : 0;
    const int y = uniform_div(at, a.deal.grid_x(), x);
    if (!dealt_tile(a.deal, x, y, token_tile, feature_tile)) return;
    if constexpr (S::kB == 1)
      if (m.splits > 1) return split_tile<S, true>(a, a, m, lds, range, token_tile, feature_tile);
    linear_tile<S, true>(a, a, lds, token_tile * S::kRowsB, feature_tile * S::kRowsA);
  }
}

template <class S, bool kMerge, bool kCodes>
hipError_t launch_weight_grad(const WeightGradArgs& a, hipStream_t stream) {
  const long tiles = tiles_of_size(a.F, a.E, S::kRowsA);
  static_assert(S::kRowsA == S::kRowsB, "square tiles");
  const hipError_t e = allow_lds<&weight_grad_kernel<S, kMerge, kCodes>>(S::kLds);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((weight_grad_kernel<S, kMerge, kCodes>), dim3((unsigned)(8 * ((tiles * a.splits + 7) / 8))), dim3(S::kThreads), S::kLds, stream, a);
  return hipGetLastError();
}
template <class S, bool kCodes>
hipError_t launch_both(const WeightGradArgs& w, LinearArgs a, int dx_splits, void* dx_workspace, hipStream_t stream) {
  deal_tiles<S>(a);
  const int w_groups = (int)((tiles_of_size(w.F, w.E, 128) * w.splits + 7) / 8 * 8);   // (whole rounds of XCDs, so that the products' tiles are dealt as ever)
  constexpr int kLds = std::max(S::kLds, Wgrad128::kLds);
  const hipError_t e = allow_lds<&linear_bwd_kernel<S, kCodes>>(kLds);
  if (e != hipSuccess) return e;
  const RangeMerge m = merge_in<S>(dx_workspace, (size_t)a.deal.tokens * a.deal.features, dx_splits, w.ticket);
  hipLaunchKernelGGL((linear_bwd_kernel<S, kCodes>), dim3(w_groups + a.deal.grid_x() * a.deal.grid_y() * dx_splits), dim3(S::kThreads), kLds, stream, w, a, m,
                     w_groups);
  return hipGetLastError();
}
template <bool kCodes>
hipError_t run_backward(const BackwardPlan& p, const WeightGradArgs& w, LinearArgs a, void* dx_workspace, hipStream_t stream) {
  if (p.one_launch && w.out) {
    if (!a.y) return launch_weight_grad<Wgrad128, true, kCodes>(w, stream);
    return p.product.rows == 128 ? launch_both<Tile128x2, kCodes>(w, a, 1, nullptr, stream)
                                 : launch_both<TileSplit, kCodes>(w, a, p.dx_splits, dx_workspace, stream);
  }
  if (a.y && p.dx_splits > 1) return launch_split<TileSplit, true>(a, p.dx_splits, dx_workspace, w.ticket, stream);   // (without dw)
  if (w.out) {
    const hipError_t e = p.tile == 256 ? launch_weight_grad<Wgrad256, false, kCodes>(w, stream) : launch_weight_grad<Wgrad128, false, kCodes>(w, stream);
    if (e != hipSuccess) return e;
    if (p.splits > 1) a.ranges = {w.part, w.part_bias, w.out, w.out_bias, (size_t)w.F * w.E, w.F, p.splits, 0};
  }
  if (a.y) return launch_product<true>(p.product.form, a, stream);
  if (!a.ranges.splits) return hipSuccess;
  a.ranges.blocks = (int)std::max<size_t>(1, std::min<size_t>(1024, a.ranges.n / 4 / 256));
  hipLaunchKernelGGL(add_weight_ranges_kernel, dim3(a.ranges.blocks), dim3(256), 0, stream, a.ranges);
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
  const ForwardPlan p = plan_forward(a.T, a.O, a.K, a.z_scales || a.y_codes);
  if (p.few.form.rows) return launch_few(p.few.form, a, stream);
  if (!p.split.splits) return launch_product<false>(p.tiles.form, a, stream);
  char* ws = static_cast<char*>(c.workspace);
  return launch_split<TileSplit, false>(a, p.split.splits, ws + (-reinterpret_cast<uintptr_t>(ws) & 15), c.ticket, stream);
}
size_t linear_workspace(int T, int E, int F, bool codes) {
  const ForwardPlan p = plan_forward(T, F, E, codes);
  return p.split.splits ? p.split.bytes + 16 : 0;   // (the caller's address may be any)
}

size_t linear_bwd_workspace(int T, int E, int F, bool codes) { return plan_backward(T, E, F, codes).total; }   // (the caller's address may be any)
size_t linear_bwd_dx_workspace(int T, int E, int F) { return plan_backward(T, E, F, false).dx_bytes; }

hipError_t launch_linear_bwd(const LinearBwdCall& c, hipStream_t stream) {
  const BackwardPlan p = plan_backward(c.T, c.E, c.F, c.x_scales != nullptr);
  LinearArgs a = {};
  a.w = static_cast<const unsigned short*>(c.w);
  a.tok = static_cast<const unsigned short*>(c.dy);
  a.T = c.T; a.O = c.E; a.K = c.F;
  a.flags = c.flags;
  a.add = static_cast<const unsigned short*>(c.residual);
  a.act = c.act;
  a.z_in = c.z;
  a.z_in_scales = c.z_scales;
  a.y = static_cast<unsigned short*>(c.dx);
  WeightGradArgs w = {};
  w.g = static_cast<const unsigned short*>(c.dy);
  w.x = c.x;
  w.x_scales = c.x_scales;
  w.flags = c.flags;
  w.out = c.dw;
  w.out_bias = c.dbias;
  w.T = c.T; w.F = c.F; w.E = c.E;
  w.splits = p.splits;
  w.per_split = p.per_split;
  w.ticket = c.ticket;
  char* ws = static_cast<char*>(c.workspace);
  ws += -reinterpret_cast<uintptr_t>(ws) & 15;
  w.part = reinterpret_cast<float*>(ws);
  w.part_bias = reinterpret_cast<float*>(ws + p.bias_off);
  w.arrived = reinterpret_cast<unsigned long long*>(ws + p.words_off);
  if (c.dw && c.x_scales && p.copy) {
    const hipError_t e = launch_checkpoint_unpack(static_cast<const unsigned char*>(c.x), c.x_scales, c.T, c.E, false, ws + p.copy_off, stream);
    if (e != hipSuccess) return e;
    w.x = ws + p.copy_off;
    w.x_scales = nullptr;
  }
  void* const dx_workspace = c.dw ? ws + p.dx_off : ws;
  return w.x_scales ? run_backward<true>(p, w, a, dx_workspace, stream) : run_backward<false>(p, w, a, dx_workspace, stream);
}

}  // namespace mate

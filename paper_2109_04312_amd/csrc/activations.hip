// Activations on their own: kept in 8 bits and brought back (eight_bits.h), and dz = dy act'(z) for a product whose gradient
// is not joined to the next one's.  All three read and write each value once and are bound by memory.
//
// A thread takes 16 features of a token, so that a pair of lanes holds a block of one scale and exchanges its maximum by one DPP
// move; 16 codes are one store.  A workgroup takes whole rows: units are counted within it, where a quotient by the units of a row
// is a product of 32-bit numbers, and offsets of whole rows are 64-bit.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "activation.h"
#include "eight_bits.h"
#include "launch.h"

namespace mate {
namespace {

constexpr int kThreads = 256, kUnit = 16;

// Which rows a workgroup takes, and the units of a row (two to a scale block).
struct RowDeal {
  int rows, E;
  int each;            // rows of a workgroup
  unsigned units, by;  // of a row; 2^32 / units, rounded up
};
RowDeal deal_rows(int rows, int E) {
  RowDeal d;
  d.rows = rows;
  d.E = E;
  d.units = 2u * scale_blocks(E);
  d.by = (unsigned)(((1ull << 32) + d.units - 1) / d.units);
  // four units a thread once there are enough for the chip: their loads travel together
  const size_t total = (size_t)rows * d.units;
  const unsigned want = total >= (size_t)4 * kThreads * 1024 ? 4 * kThreads : kThreads;
  d.each = (int)std::max(1u, want / d.units);
  return d;
}
unsigned groups_of(const RowDeal& d) { return (unsigned)((d.rows + (long)d.each - 1) / d.each); }

// A thread's unit: its row (of the tensor), first feature and how many of 16 are features (0, 8 or 16).
struct Unit {
  size_t row;
  int first, n;
};
__device__ __forceinline__ Unit unit_at(const RowDeal& d, unsigned i, int here) {
  const unsigned r = __umulhi(i, d.by);
  // (i < 2^16 and units <= 2^12: the rounding of `by` cannot reach the next quotient)
  Unit u;
  u.row = (size_t)blockIdx.x * d.each + r;
  u.first = (int)(i - r * d.units) * kUnit;
  u.n = (int)r < here ? max(0, min(kUnit, d.E - u.first)) : 0;
  return u;
}
// A quotient by one is no product of 32-bit numbers: a row has two units at least.

struct alignas(8) Words2 { unsigned w[2]; };
struct alignas(8) Words4 { unsigned w[4]; };   // (rows of codes begin at multiples of 8)

template <bool kF32>
__device__ __forceinline__ void load_values(const void* x, const RowDeal& d, const Unit& u, float (&v)[kUnit]) {
#pragma unroll
  for (int e = 0; e < kUnit; ++e) v[e] = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (8 * h < u.n) {
      if (kF32) {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + u.row * d.E + u.first + 8 * h);
        const f32x4 a = p[0], b = p[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[8 * h + e] = a[e]; v[8 * h + 4 + e] = b[e]; }
      } else {
        const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(x) + u.row * d.E + u.first + 8 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) { v[8 * h + 2 * e] = low_bf16(w[e]); v[8 * h + 2 * e + 1] = high_bf16(w[e]); }
      }
    }
}
template <bool kF32>
__device__ __forceinline__ void store_values(void* x, const RowDeal& d, const Unit& u, const float (&v)[kUnit]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    if (8 * h < u.n) {
      if (kF32) {
        f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(x) + u.row * d.E + u.first + 8 * h);
        p[0] = f32x4{v[8 * h], v[8 * h + 1], v[8 * h + 2], v[8 * h + 3]};
        p[1] = f32x4{v[8 * h + 4], v[8 * h + 5], v[8 * h + 6], v[8 * h + 7]};
      } else {
        u32x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack2(v[8 * h + 2 * e], v[8 * h + 2 * e + 1]);
        *reinterpret_cast<u32x4*>(static_cast<unsigned short*>(x) + u.row * d.E + u.first + 8 * h) = w;
      }
    }
}
// 16 codes of a unit, fewer at a row's end
__device__ __forceinline__ Words4 load_codes(const unsigned char* codes, const RowDeal& d, const Unit& u) {
  const unsigned char* p = codes + u.row * d.E + u.first;
  Words4 w = {};
  if (u.n == kUnit) w = *reinterpret_cast<const Words4*>(p);
  else if (u.n) {
    const Words2 t = *reinterpret_cast<const Words2*>(p);
    w.w[0] = t.w[0];
    w.w[1] = t.w[1];
  }
  return w;
}
__device__ __forceinline__ void store_codes(unsigned char* codes, const RowDeal& d, const Unit& u, const Words4& w) {
  unsigned char* p = codes + u.row * d.E + u.first;
  if (u.n == kUnit) *reinterpret_cast<Words4*>(p) = w;
  else if (u.n) *reinterpret_cast<Words2*>(p) = Words2{{w.w[0], w.w[1]}};
}
__device__ __forceinline__ size_t scale_at(const RowDeal& d, const Unit& u) { return u.row * (d.units / 2) + u.first / kScaleBlock; }

// Calls f(unit) for every unit of this workgroup, all lanes of a wavefront together.
template <int kDepth, class Load, class Rest>
__device__ __forceinline__ void each_unit(const RowDeal& d, Load&& load, Rest&& rest) {
  const int here = (int)min((size_t)d.each, (size_t)d.rows - (size_t)blockIdx.x * d.each);
  const unsigned n = (unsigned)d.each * d.units;
  for (unsigned i0 = threadIdx.x; i0 < n + threadIdx.x; i0 += kDepth * kThreads) {
    Unit u[kDepth];
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      u[k] = unit_at(d, min(i0 + k * kThreads, n), here);   // (n: past the last row)
      load(k, u[k]);
    }
#pragma unroll
    for (int k = 0; k < kDepth; ++k) rest(k, u[k]);
  }
}

template <bool kF32, int kDepth>
__global__ __launch_bounds__(kThreads) void pack_kernel(const void* x, const unsigned char* flags, unsigned char* codes, unsigned char* scales,
                                                        RowDeal d) {
  float v[kDepth][kUnit];
  each_unit<kDepth>(
      d,
      [&](int k, Unit u) {
        if (u.n && flags && flags[u.row] >= 2) u.n = 0;   // a row of padding is zeros, whatever it holds
        load_values<kF32>(x, d, u, v[k]);
      },
      [&](int k, const Unit& u) {
        const unsigned m = block_magnitude(v[k], [](unsigned m) { return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false)); });
        const unsigned s = scale_byte(m);
        const float scale = scale_value(s);
        Words4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w.w[e] = to_codes(v[k][4 * e], v[k][4 * e + 1], v[k][4 * e + 2], v[k][4 * e + 3], scale);
        store_codes(codes, d, u, w);
        if (u.n && !(u.first & kUnit)) scales[scale_at(d, u)] = (unsigned char)s;
      });
}

template <bool kF32, int kDepth>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const unsigned char* codes, const unsigned char* scales, void* x, RowDeal d) {
  Words4 w[kDepth];
  unsigned s[kDepth];
  each_unit<kDepth>(
      d,
      [&](int k, const Unit& u) {
        w[k] = load_codes(codes, d, u);
        s[k] = u.n ? scales[scale_at(d, u)] : 1;
      },
      [&](int k, const Unit& u) {
        float v[kUnit];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x4 f = from_codes(w[k].w[e], scale_value(s[k]));
#pragma unroll
          for (int y = 0; y < 4; ++y) v[4 * e + y] = f[y];
        }
        store_values<kF32>(x, d, u, v);
      });
}

template <bool kCodes, int kDepth>
__global__ __launch_bounds__(kThreads) void activation_bwd_kernel(const void* dy, const void* z, const unsigned char* scales, const unsigned char* flags,
                                                                  void* dz, int act, RowDeal d) {
  with_activation(act, [&](auto kind) {
    float g[kDepth][kUnit], v[kCodes ? 1 : kDepth][kUnit];
    Words4 w[kDepth];
    unsigned s[kDepth];
    bool pad[kDepth];
    each_unit<kDepth>(
        d,
        [&](int k, Unit u) {
          pad[k] = u.n && flags && flags[u.row] >= 2;
          if (pad[k]) u.n = 0;
          load_values<false>(dy, d, u, g[k]);
          if constexpr (kCodes) {
            w[k] = load_codes(static_cast<const unsigned char*>(z), d, u);
            s[k] = u.n ? scales[scale_at(d, u)] : 1;
          } else {
            load_values<false>(z, d, u, v[k]);
          }
        },
        [&](int k, const Unit& u) {
          float r[kUnit];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f32x4 f;
            if constexpr (kCodes) f = from_codes(w[k].w[e], scale_value(s[k]));
            else f = f32x4{v[k][4 * e], v[k][4 * e + 1], v[k][4 * e + 2], v[k][4 * e + 3]};
#pragma unroll
            for (int y = 0; y < 4; ++y) r[4 * e + y] = pad[k] ? 0.f : g[k][4 * e + y] * slope<decltype(kind)::value>(f[y]);
          }
          store_values<false>(dz, d, u, r);
        });
  });
}

// Four units a thread where a workgroup has them.
template <class One, class Four>
hipError_t launch_rows(const RowDeal& d, One&& one, Four&& four) {
  if ((size_t)d.each * d.units > kThreads) four(dim3(groups_of(d)));
  else one(dim3(groups_of(d)));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_checkpoint_pack(const void* x, const unsigned char* flags, int rows, int E, bool f32, unsigned char* codes, unsigned char* scales,
                                  hipStream_t stream) {
  const RowDeal d = deal_rows(rows, E);
  auto run = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, x, flags, codes, scales, d); };
  return launch_rows(
      d, [&](dim3 g) { f32 ? run(pack_kernel<true, 1>, g) : run(pack_kernel<false, 1>, g); },
      [&](dim3 g) { f32 ? run(pack_kernel<true, 4>, g) : run(pack_kernel<false, 4>, g); });
}

hipError_t launch_checkpoint_unpack(const unsigned char* codes, const unsigned char* scales, int rows, int E, bool f32, void* x, hipStream_t stream) {
  const RowDeal d = deal_rows(rows, E);
  auto run = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, codes, scales, x, d); };
  return launch_rows(
      d, [&](dim3 g) { f32 ? run(unpack_kernel<true, 1>, g) : run(unpack_kernel<false, 1>, g); },
      [&](dim3 g) { f32 ? run(unpack_kernel<true, 4>, g) : run(unpack_kernel<false, 4>, g); });
}

hipError_t launch_activation_bwd(const void* dy, const void* z, const unsigned char* z_scales, const unsigned char* flags, int rows, int E, int act,
                                 void* dz, hipStream_t stream) {
  const RowDeal d = deal_rows(rows, E);
  auto run = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, dy, z, z_scales, flags, dz, act, d); };
  return launch_rows(
      d, [&](dim3 g) { z_scales ? run(activation_bwd_kernel<true, 1>, g) : run(activation_bwd_kernel<false, 1>, g); },
      [&](dim3 g) { z_scales ? run(activation_bwd_kernel<true, 4>, g) : run(activation_bwd_kernel<false, 4>, g); });
}

}  // namespace mate

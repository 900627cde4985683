// Activations on their own: kept in 8 bits and brought back (eight_bits.h), and dz = dy act'(z) for a product whose gradient
// is not joined to the next one's.  All three read and write each value once and are bound by memory.
//
// A thread takes 8 features of a token, so that a wavefront's 16-byte accesses are side by side (of 16, in two accesses each, only every other 16
// bytes: activations of 16384 x 4096 from 16 bits 84 us, so 74), and four lanes hold a block of one scale and exchange its maximum by
// two DPP moves.  A workgroup takes whole rows: units are counted within it, where a quotient by the units of a row
// is a product of 32-bit numbers, and offsets of whole rows are 64-bit.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "activation.h"
#include "eight_bits.h"
#include "launch.h"
#include "row_deal.h"

namespace mate {
namespace {

constexpr int kThreads = kRowThreads, kUnits = kScaleBlock / kUnit;   // kUnits: of a scale block

// A thread's unit: its row (of the tensor), first feature, and whether there are features there.
struct Unit {
  size_t row;
  int first;
  bool some;
};
__device__ __forceinline__ Unit unit_at(const RowDeal& d, long first, unsigned i, int here) {
  const unsigned r = __umulhi(i, d.by);   // (i <= 2^13 and units <= 2^13: the rounding of `by` cannot reach the next quotient)
  Unit u;
  u.row = (size_t)first + r;
  u.first = (int)(i - r * d.units) * kUnit;
  u.some = (int)r < here && u.first < d.E;
  return u;
}

template <bool kF32>
__device__ __forceinline__ void load_values(const void* x, const RowDeal& d, const Unit& u, float (&v)[kUnit]) {
#pragma unroll
  for (int e = 0; e < kUnit; ++e) v[e] = 0.f;
  if (!u.some) return;
  const size_t at = u.row * d.E + u.first;
  if (kF32) {
    const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + at);
    const f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
  } else {
    const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(x) + at);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[2 * e] = low_bf16(w[e]); v[2 * e + 1] = high_bf16(w[e]); }
  }
}
template <bool kF32>
__device__ __forceinline__ void store_values(void* x, const RowDeal& d, const Unit& u, const float (&v)[kUnit]) {
  if (!u.some) return;
  const size_t at = u.row * d.E + u.first;
  if (kF32) {
    f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(x) + at);
    p[0] = f32x4{v[0], v[1], v[2], v[3]};
    p[1] = f32x4{v[4], v[5], v[6], v[7]};
  } else {
    *reinterpret_cast<u32x4*>(static_cast<unsigned short*>(x) + at) = u32x4{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7])};
  }
}
__device__ __forceinline__ uint2 load_codes(const unsigned char* codes, const RowDeal& d, const Unit& u) {
  return u.some ? *reinterpret_cast<const uint2*>(codes + u.row * d.E + u.first) : make_uint2(0, 0);
}
__device__ __forceinline__ size_t scale_at(const RowDeal& d, const Unit& u) { return u.row * (d.units / kUnits) + u.first / kScaleBlock; }
__device__ __forceinline__ void values_of(const uint2& w, unsigned s, float (&v)[kUnit]) {
  const f32x4 a = from_codes(w.x, scale_value(s)), b = from_codes(w.y, scale_value(s));
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
}

// Calls load and then rest for every unit of this workgroup, kDepth of them at a time, all lanes of a wavefront together.
template <int kDepth, class Load, class Rest>
__device__ __forceinline__ void each_unit(const RowDeal& d, Load&& load, Rest&& rest) {
  const long first = first_row(d, blockIdx.x, blockIdx.y);
  const int here = rows_from(d, first);
  const unsigned n = (unsigned)d.each * d.units;
  for (unsigned i0 = threadIdx.x; i0 < n + threadIdx.x; i0 += kDepth * kThreads) {
    Unit u[kDepth];
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      u[k] = unit_at(d, first, min(i0 + k * kThreads, n), here);   // (n: past the last row)
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
        if (u.some && flags && flags[u.row] >= 2) u.some = false;   // a row of padding is zeros, whatever it holds
        load_values<kF32>(x, d, u, v[k]);
      },
      [&](int k, const Unit& u) {
        const unsigned s = scale_byte(block_magnitude(v[k], quad_maximum));
        if (!u.some) return;
        const float scale = scale_value(s);
        *reinterpret_cast<uint2*>(codes + u.row * d.E + u.first) =
            make_uint2(to_codes(v[k][0], v[k][1], v[k][2], v[k][3], scale), to_codes(v[k][4], v[k][5], v[k][6], v[k][7], scale));
        if (u.first % kScaleBlock == 0) scales[scale_at(d, u)] = (unsigned char)s;
      });
}

template <bool kF32, int kDepth>
__global__ __launch_bounds__(kThreads) void unpack_kernel(const unsigned char* codes, const unsigned char* scales, void* x, RowDeal d) {
  uint2 w[kDepth];
  unsigned s[kDepth];
  each_unit<kDepth>(
      d,
      [&](int k, const Unit& u) {
        w[k] = load_codes(codes, d, u);
        s[k] = u.some ? scales[scale_at(d, u)] : 1;
      },
      [&](int k, const Unit& u) {
        float v[kUnit];
        values_of(w[k], s[k], v);
        store_values<kF32>(x, d, u, v);
      });
}

template <bool kCodes, int kDepth>
__global__ __launch_bounds__(kThreads) void activation_bwd_kernel(const void* dy, const void* z, const unsigned char* scales, const unsigned char* flags,
                                                                  void* dz, int act, RowDeal d) {
  with_activation(act, [&](auto kind) {
    float g[kDepth][kUnit], v[kDepth][kUnit];
    uint2 w[kDepth];
    unsigned s[kDepth];
    bool pad[kDepth];
    each_unit<kDepth>(
        d,
        [&](int k, Unit u) {
          pad[k] = u.some && flags && flags[u.row] >= 2;
          if (pad[k]) u.some = false;
          load_values<false>(dy, d, u, g[k]);
          if constexpr (kCodes) {
            w[k] = load_codes(static_cast<const unsigned char*>(z), d, u);
            s[k] = u.some ? scales[scale_at(d, u)] : 1;
          } else {
            load_values<false>(z, d, u, v[k]);
          }
        },
        [&](int k, const Unit& u) {
          if (kCodes) values_of(w[k], s[k], v[k]);
          float r[kUnit];
#pragma unroll
          for (int e = 0; e < kUnit; ++e) r[e] = pad[k] ? 0.f : g[k][e] * slope<decltype(kind)::value>(v[k][e]);
          store_values<false>(dz, d, u, r);
        });
  });
}

// launch(grid, units that a thread has under way): as many as there are.
template <class Launch>
hipError_t launch_rows(const RowDeal& d, Launch&& launch) {
  const size_t units = (size_t)d.each * d.units;
  const dim3 grid = groups_of(d);
  if (units <= kThreads) launch(grid, std::integral_constant<int, 1>());
  else if (units <= 2 * kThreads) launch(grid, std::integral_constant<int, 2>());
  else launch(grid, std::integral_constant<int, 4>());
  return hipGetLastError();
}

}  // namespace

hipError_t launch_checkpoint_pack(const void* x, const unsigned char* flags, int rows, int E, bool f32, unsigned char* codes, unsigned char* scales,
                                  hipStream_t stream) {
  const RowDeal d = deal_rows(rows, E, kScaleBlock);
  auto run = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, x, flags, codes, scales, d); };
  return launch_rows(d, [&](dim3 g, auto depth) {
    constexpr int k = decltype(depth)::value;
    f32 ? run(pack_kernel<true, k>, g) : run(pack_kernel<false, k>, g);
  });
}

hipError_t launch_checkpoint_unpack(const unsigned char* codes, const unsigned char* scales, int rows, int E, bool f32, void* x, hipStream_t stream) {
  const RowDeal d = deal_rows(rows, E, kScaleBlock);
  auto run = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, codes, scales, x, d); };
  return launch_rows(d, [&](dim3 g, auto depth) {
    constexpr int k = decltype(depth)::value;
    f32 ? run(unpack_kernel<true, k>, g) : run(unpack_kernel<false, k>, g);
  });
}

hipError_t launch_activation_bwd(const void* dy, const void* z, const unsigned char* z_scales, const unsigned char* flags, int rows, int E, int act,
                                 void* dz, hipStream_t stream) {
  const RowDeal d = deal_rows(rows, E, kScaleBlock);
  auto run = [&](auto kernel, dim3 grid) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, dy, z, z_scales, flags, dz, act, d); };
  return launch_rows(d, [&](dim3 g, auto depth) {
    constexpr int k = decltype(depth)::value;
    z_scales ? run(activation_bwd_kernel<true, k>, g) : run(activation_bwd_kernel<false, k>, g);
  });
}

}  // namespace mate

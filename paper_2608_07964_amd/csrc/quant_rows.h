// A step's activations to e4m3 (see quant8.h), shared by the launch that does
// only that (quant8.hip) and the grouping of small steps (permute.hip), which
// has them done by further workgroups of its own launch.
#pragma once

#include "eb_internal.h"
#include "eb_numeric.h"
#include "quant8.h"

namespace eb {
namespace {

typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

// Eight bf16 values as floats.
struct Eight {
  float v[8];
  __device__ __forceinline__ void from(const u32x4& u) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  // the largest finite magnitude; infinities become NaN, which the maximum passes over
  __device__ __forceinline__ float amax() {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      v[i] = nan_if_infinite(v[i]);
      a = fmaxf(a, fabsf(v[i]));
    }
    return a;
  }
  __device__ __forceinline__ u32x2 quantised(float inv) const {
    return (u32x2){pack_e4m3x4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                   pack_e4m3x4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
  }
};

// Largest value over the 16 lanes of a DPP row.
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0xB1, 0xF, 0xF, true)));
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x4E, 0xF, 0xF, true)));
  v = fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x141, 0xF, 0xF, true)));
  return fmaxf(v, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x140, 0xF, 0xF, true)));
}

// The activations of a step's tokens, each once (the grouped GEMM reads a
// token's row through the grouping).  One wavefront per (token, 512 columns):
// 16 lanes hold a block of 128, and the four blocks' exponents are one word of
// the scales, sa[piece][token].  Wavefront wv of the step.
__device__ __forceinline__ void quantize_row_piece(const RunTable& rt, long long wv, int pieces, int tokens,
                                                   uint8_t* __restrict__ qa, uint32_t* __restrict__ sa) {
  const int total = rt.tok_base[rt.n], lane = threadIdx.x & 63;
  if (wv >= (long long)total * pieces) return;
  const int g = (int)(wv / pieces), piece = (int)(wv - (long long)g * pieces);
  const int rho = find_entry(rt.tok_base, rt.n, g), t = g - rt.tok_base[rho], H = rt.H;
  const int col = piece * 512 + lane * 8;
  const bool in = col < H;
  const bf16_t* a = in_global(static_cast<const bf16_t*>(rt.a[rho])) + (size_t)t * H;
  Eight x;
  x.from(in ? *reinterpret_cast<const u32x4*>(a + col) : (u32x4){0, 0, 0, 0});
  const int e8 = scale_exponent(row16_max(x.amax()));
  if (in) *reinterpret_cast<u32x2*>(qa + (size_t)g * H + col) = x.quantised(inverse_scale(e8));
  const uint32_t word = (uint32_t)__builtin_amdgcn_readlane(e8, 0) | (uint32_t)__builtin_amdgcn_readlane(e8, 16) << 8 |
                        (uint32_t)__builtin_amdgcn_readlane(e8, 32) << 16 |
                        (uint32_t)__builtin_amdgcn_readlane(e8, 48) << 24;
  if (lane == 0) sa[(size_t)piece * tokens + g] = word;
}

}  // namespace
}  // namespace eb

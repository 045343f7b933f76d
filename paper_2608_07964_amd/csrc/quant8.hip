// Quantisation to e4m3 with power-of-two scales (see quant8.h): a step's
// activations by row and 128 columns, weights by blocks of 128 x 128.
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
  __device__ __forceinline__ float amax() const {
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmaxf(a, finite_magnitude(v[i]));
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
// the scales, sa[piece][token].
template <class RTA>
__global__ __launch_bounds__(256) void quantize_rows_kernel(RTA rta, int pieces, int tokens, uint8_t* __restrict__ qa,
                                                            uint32_t* __restrict__ sa) {
  const RunTable& rt = rta.get();
  const int total = rt.tok_base[rt.n], lane = threadIdx.x & 63;
  const long long wv = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
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

// Eight consecutive values of a source row.
template <typename TS>
__device__ __forceinline__ Eight load8(const TS* p);
template <>
__device__ __forceinline__ Eight load8<bf16_t>(const bf16_t* p) {
  Eight x;
  x.from(*reinterpret_cast<const u32x4*>(p));
  return x;
}
template <>
__device__ __forceinline__ Eight load8<float>(const float* p) {
  Eight x;
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) x.v[i] = v[i];
  return x;
}

// One workgroup per 128 x 128 block: thread t holds columns 8 (t % 16) .. + 7 of
// rows t / 16 + 16 i.
template <typename TS>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const TS* __restrict__ src, uint8_t* __restrict__ q,
                                                              float* __restrict__ scales, int K) {
  __shared__ float part[4];
  const size_t row0 = (size_t)blockIdx.y * 128 + (threadIdx.x >> 4);  // row of all the matrices
  const size_t at = row0 * K + (size_t)blockIdx.x * 128 + (threadIdx.x & 15) * 8;
  Eight x[8];
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = load8(src + at + (size_t)i * 16 * K);
#pragma unroll
  for (int i = 0; i < 8; ++i) a = fmaxf(a, x[i].amax());
  a = row16_max(a);
  a = fmaxf(a, __shfl_xor(a, 16, 64));
  a = fmaxf(a, __shfl_xor(a, 32, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = a;
  __syncthreads();
  const int e8 = scale_exponent(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
  const float inv = inverse_scale(e8);
#pragma unroll
  for (int i = 0; i < 8; ++i) *reinterpret_cast<u32x2*>(q + at + (size_t)i * 16 * K) = x[i].quantised(inv);
  if (threadIdx.x == 0) scales[(size_t)blockIdx.y * (K / 128) + blockIdx.x] = scale_value(e8);
}

__global__ __launch_bounds__(256) void copy_scales_kernel(const float* __restrict__ src, float* __restrict__ dst,
                                                          size_t n) {
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i < n) dst[i] = src[i];
}

template <class RTA>
hipError_t quantize_rows_impl(RTA a, int H, int grid_tokens, int tokens, uint8_t* qa, uint32_t* sa, hipStream_t s) {
  const int pieces = (H + 511) / 512;
  const long long waves = (long long)grid_tokens * pieces;
  prof_start(EB_K_PERM_GATHER, s);
  if (waves > 0)
    hipLaunchKernelGGL(quantize_rows_kernel<RTA>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a, pieces,
                       tokens, qa, sa);
  prof_stop(EB_K_PERM_GATHER, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const RunTable& rt, int tokens, uint8_t* qa, uint32_t* sa, hipStream_t s) {
  return quantize_rows_impl(ByValue<RunTable>{rt}, rt.H, rt.tok_base[rt.n], tokens, qa, sa, s);
}
hipError_t launch_quantize_rows_dev(const RunTable* rt, int H, int tokens, uint8_t* qa, uint32_t* sa, hipStream_t s) {
  return quantize_rows_impl(InMemory<RunTable>{rt}, H, tokens, tokens, qa, sa, s);
}

hipError_t launch_copy_scales(const float* src, void* dst, size_t bytes, hipStream_t s) {
  const size_t n = bytes / sizeof(float);
  hipLaunchKernelGGL(copy_scales_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, src,
                     static_cast<float*>(dst), n);
  return hipGetLastError();
}

hipError_t launch_quantize_blocks(int src_dtype, int n, int N, int K, const void* src, void* q, float* scales,
                                  hipStream_t s) {
  // a grid's y dimension holds 65535 row blocks
  for (long long b = 0, all = (long long)n * (N / 128); b < all; b += 65535) {
    const long long rows = all - b < 65535 ? all - b : 65535;
    const size_t at = (size_t)b * 128 * K;
    float* sc = scales + (size_t)b * (K / 128);
    uint8_t* to = static_cast<uint8_t*>(q) + at;
    if (src_dtype == EB_DTYPE_BF16)
      hipLaunchKernelGGL(quantize_blocks_kernel<bf16_t>, dim3(K / 128, (unsigned)rows), dim3(256), 0, s,
                         static_cast<const bf16_t*>(src) + at, to, sc, K);
    else
      hipLaunchKernelGGL(quantize_blocks_kernel<float>, dim3(K / 128, (unsigned)rows), dim3(256), 0, s,
                         static_cast<const float*>(src) + at, to, sc, K);
  }
  return hipGetLastError();
}

}  // namespace eb

// Choice of experts from router logits with scores, a balance bias and expert
// groups, for a batch of micro-batches:
//
//   s   = 1 / (1 + e^-z)  or  softmax(z)            the routing weights' source
//   c   = s + balance                               what the choice goes by
//   of G groups of E/G consecutive experts the topk_group with the largest
//   group score stay (the sum of the group's 1 or 2 largest c)
//   idx = the k largest c of the groups that stay, w = scale * s[idx] (over
//   their sum where renormalised), counts
//
// Order: larger first, then the lower id (group, expert); NaN after every
// number.
//
// Neighbours in this order are often closer than fp32 resolves (256 scores in
// (0, 1), two million tokens an hour), and a pick decided by rounding depends
// on the library's exp.  So a token is first chosen in fp32 together with the
// distance of every decision that was made: the gap between the last group
// kept and the first left out, and between each pick and the next.  Where one
// is within the error bound of the fp32 scores (kMargin*), the token is chosen
// again from fp64 scores.  About 1 token in 100 of 256 experts takes that path.
//
// A team of W lanes takes a token.  Its lanes are dealt to the groups (a power
// of two each), so a lane holds V experts of one group: e = group M + j + i LPG
// for lane j of the group's LPG lanes, and a group's two largest are a
// reduction over LPG lanes.  A pick is one maximum of unsigned order keys over
// the lane's V values and the team, then the lowest id that has it.
#include "eb_internal.h"
#include "eb_numeric.h"

namespace eb {
namespace {

// Bounds of the error of c in fp32, relative to (largest s of the row + |c|).
// Sigmoid: s(1-s)|z| < 0.23 bounds what the rounded exponent does to s, exp2,
// the sum and the reciprocal add an ulp each, s + balance half an ulp: below
// 2^-22.  Softmax: its denominator is a sum of E <= 1024 terms, 32 in a lane
// and then 6 levels: 38 roundings and the exponential's, below 2^-18.
constexpr float kMarginSigmoid = 0x1p-21f, kMarginSoftmax = 0x1p-17f;
// Sums of the picked scores below this are formed in fp64 (fp32 scores near
// its smallest numbers have few digits).
constexpr float kTiny = 1e-30f;

// Order-preserving unsigned keys: NaN 1, then -inf .. inf; 0 is no value.
__device__ __forceinline__ uint32_t order_key(float v) {
  if (!(v == v)) return 1u;
  const uint32_t u = __float_as_uint(v == 0.f ? 0.f : v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ uint64_t order_key(double v) {
  if (!(v == v)) return 1ull;
  const uint64_t u = (uint64_t)__double_as_longlong(v == 0.0 ? 0.0 : v);
  return (u >> 63) ? ~u : (u | (1ull << 63));
}
__device__ __forceinline__ float key_float(uint32_t o) {
  return o <= 1u ? __builtin_nanf("") : __uint_as_float((o & 0x80000000u) ? (o ^ 0x80000000u) : ~o);
}

// Value of the lane `off` away by XOR, off a power of two below W: within 16
// lanes by DPP (for off 4 and 8 a mirror, which serves a reduction whose
// values are already equal within groups of off lanes).
template <int OFF>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (OFF == 1) return __builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);
  else if constexpr (OFF == 2) return __builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);
  else if constexpr (OFF == 4) return __builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true);
  else if constexpr (OFF == 8) return __builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true);
  else return __shfl_xor((int)v, OFF, 64);
}
template <int OFF>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  return ((uint64_t)lane_xor<OFF>((uint32_t)(v >> 32)) << 32) | lane_xor<OFF>((uint32_t)v);
}
template <int OFF>
__device__ __forceinline__ float lane_xor(float v) { return __uint_as_float(lane_xor<OFF>(__float_as_uint(v))); }
template <int OFF>
__device__ __forceinline__ double lane_xor(double v) {
  return __longlong_as_double((long long)lane_xor<OFF>((uint64_t)__double_as_longlong(v)));
}
// All-reduce over the team, in a fixed pattern.
template <int W, class T, class Op>
__device__ __forceinline__ T team_reduce(T v, Op op) {
  v = op(v, lane_xor<1>(v));
  v = op(v, lane_xor<2>(v));
  v = op(v, lane_xor<4>(v));
  v = op(v, lane_xor<8>(v));
  if constexpr (W == 64) {
    v = op(v, lane_xor<16>(v));
    v = op(v, lane_xor<32>(v));
  }
  return v;
}

__device__ __forceinline__ float sigmoid_of(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-z * 1.44269504088896341f));
}
__device__ __forceinline__ double sigmoid_of(double z) { return 1.0 / (1.0 + exp(-z)); }
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ double exp_of(double x) { return exp(x); }

// What the lanes of a team hold: lane `sub`'s experts are first + i step for
// i < V, those below `end` (the end of its group).
struct TeamMap {
  int sub, lpg, group, first, end;
};

__device__ __forceinline__ float magnitude(float v) { return fabsf(v); }
__device__ __forceinline__ double magnitude(double v) { return fabs(v); }

// The k picks of one token in type R (float or double): lane r < k returns pick
// r's expert in *pick and its routing weight in *w.  close: a decision was
// within the error bound of float, or the picks' sum where fp32 loses digits.
template <int W, int V, class R>
__device__ __forceinline__ void choose(const eb_router& p, const TeamMap& m, int E, int k, const float* __restrict__ z,
                                       const float* __restrict__ balance, int* pick, float* w, bool* close) {
  using Key = decltype(order_key(R(0)));
  const auto maxk = [](Key a, Key b) { return a > b ? a : b; };
  const auto maxr = [](R a, R b) { return a > b ? a : b; };
  const R ninf = -(R)INFINITY;
  // softmax: the row's largest logit and denominator.  A row of -inf alone has
  // s = 0; NaN and +inf logits make every s of the row NaN.
  R mx = ninf, denom = 1, top = 1;
  const bool soft = p.score == EB_SCORE_SOFTMAX;
  R c[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = m.first + i * m.lpg;
    c[i] = e < m.end ? (R)z[e] : ninf;
  }
  if (soft) {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mx = maxr(mx, c[i]);
      nan |= !(c[i] == c[i]);
    }
    mx = team_reduce<W>(mx, maxr);
    denom = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) denom += mx == ninf ? (R)0 : exp_of(c[i] - mx);
    if (nan) denom = (R)__builtin_nan("");
    denom = team_reduce<W>(denom, [](R a, R b) { return a + b; });
    if (denom == 0) denom = 1;  // a row of -inf alone
    top = 1 / denom;
  }
  auto score = [&](R v) -> R {
    if (!soft) return sigmoid_of(v);
    return (mx == ninf ? (R)0 : exp_of(v - mx)) / denom;
  };
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = m.first + i * m.lpg;
    if (e < m.end) {
      c[i] = score(c[i]);
      if (balance) c[i] += (R)balance[e];
    }
  }
  const R margin = (R)(soft ? kMarginSoftmax : kMarginSigmoid);
  bool near = false;
  // group choice
  bool kept = m.group < p.n_group;
  if (p.topk_group < p.n_group) {
    R b1 = ninf, b2 = ninf;  // the lane's, then the group's, two largest (NaN counts as -inf)
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const R v = m.first + i * m.lpg < m.end && c[i] == c[i] ? c[i] : ninf;
      b2 = maxr(b2, v < b1 ? v : b1);
      b1 = maxr(b1, v);
    }
    for (int off = 1; off < m.lpg; off <<= 1) {
      const R o1 = __shfl_xor(b1, off, W), o2 = __shfl_xor(b2, off, W);
      b2 = maxr(maxr(b2, o2), o1 < b1 ? o1 : b1);
      b1 = maxr(b1, o1);
    }
    R gs = p.group_top == 2 ? b1 + b2 : b1;
    if (!(gs == gs)) gs = ninf;
    int before = 0;
    for (int g = 0; g < p.n_group; ++g) {
      const R o = __shfl(gs, g * m.lpg, W);
      before += o > gs || (o == gs && g < m.group);
    }
    const bool real = kept;
    kept = real && before < p.topk_group;
    // the last group kept against the first left out, each at its worst
    const R err = gs - gs == 0 ? margin * (2 * top + magnitude(b1) + (p.group_top == 2 ? magnitude(b2) : 0)) : 0;
    const R in = team_reduce<W>(kept ? err - gs : ninf, maxr);
    const R out = team_reduce<W>(real && !kept ? gs + err : ninf, maxr);
    if (!(-in > out)) near = true;
  }
  Key key[V];
#pragma unroll
  for (int i = 0; i < V; ++i) key[i] = kept && m.first + i * m.lpg < m.end ? order_key(c[i]) : (Key)0;
  R last = 0;
  const bool more = k < E;
  int mine = 0;
  for (int r = 0; r < k + 1; ++r) {
    if (r == k && (sizeof(R) == 8 || !more)) break;
    Key best = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) best = maxk(best, key[i]);
    best = team_reduce<W>(best, maxk);
    if constexpr (sizeof(R) == 4) {
      const R v = key_float(best);
      // equal or close values, NaN and no value at all (the extra round's) alike
      if (r > 0 && best != 0 && !(last - v > margin * (2 * top + magnitude(last) + magnitude(v)))) near = true;
      last = v;
    }
    if (r == k) break;
    uint32_t at = ~0u;
#pragma unroll
    for (int i = V - 1; i >= 0; --i)
      if (key[i] == best) at = (uint32_t)(m.first + i * m.lpg);
    const uint32_t lane_at = at;
    at = team_reduce<W>(at, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
    if (lane_at == at) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (m.first + i * m.lpg == (int)at) key[i] = 0;
    }
    if (m.sub == r) mine = (int)at;
  }
  mine = min(max(mine, 0), E - 1);
  R weight = m.sub < k ? score((R)z[mine]) : (R)0;
  if (p.norm_topk) {
    const R sum = team_reduce<W>(weight, [](R a, R b) { return a + b; });
    if (sum != 0) weight = weight / sum;
    near = near || sum < (R)kTiny;
  }
  *pick = mine;
  *w = (float)weight * p.scale;
  *close = near;
}

// One workgroup per 32-token block of the batch.  OWN: every entry of the batch
// has one block, whose workgroup writes the entry's counts; else they were
// cleared before and are added to.
constexpr int kSelectTokens = 32;
template <int W, int V, bool OWN, class RBA>
__global__ __launch_bounds__(256) void select_kernel(RBA rba, eb_router p, int E, int k) {
  __shared__ int hist[1024];
  const RouteBatch& rb = rba.get();
  if ((int)blockIdx.x >= rb.blk0[rb.n]) return;  // past the live blocks
  const int ei = find_entry(rb.blk0, rb.n, blockIdx.x);
  const int t0 = (blockIdx.x - rb.blk0[ei]) * kSelectTokens;
  const int rows = min(rb.tok0[ei + 1] - rb.tok0[ei] - t0, kSelectTokens);
  const float* __restrict__ z = in_global(static_cast<const float*>(rb.e[ei].z)) + (size_t)t0 * E;
  const float* __restrict__ balance = in_global(rb.e[ei].balance);
  int32_t* __restrict__ idx = in_global(rb.e[ei].idx) + (size_t)t0 * k;
  float* __restrict__ w = in_global(rb.e[ei].w) + (size_t)t0 * k;
  for (int e = threadIdx.x; e < E; e += 256) hist[e] = 0;
  __syncthreads();
  TeamMap m;
  m.sub = threadIdx.x % W;
  m.lpg = W;
  while (m.lpg * p.n_group > W) m.lpg >>= 1;
  m.group = m.sub / m.lpg;
  const int M = E / p.n_group;
  m.first = m.group * M + m.sub % m.lpg;
  m.end = m.group < p.n_group ? (m.group + 1) * M : 0;
  // whole teams leave the loop together, but not all teams of a wavefront: the
  // exchanges stay within a team
  for (int t = threadIdx.x / W; t < rows; t += 256 / W) {
    int e;
    float we;
    bool close;
    const float* zt = z + (size_t)t * E;
    choose<W, V, float>(p, m, E, k, zt, balance, &e, &we, &close);
    if (team_reduce<W>((uint32_t)close, [](uint32_t a, uint32_t b) { return a | b; }))
      choose<W, V, double>(p, m, E, k, zt, balance, &e, &we, &close);
    if (m.sub < k) {
      idx[(size_t)t * k + m.sub] = e;
      w[(size_t)t * k + m.sub] = we;
      atomicAdd(&hist[e], 1);
    }
  }
  __syncthreads();
  int32_t* __restrict__ counts = in_global(rb.e[ei].counts);
  for (int e = threadIdx.x; e < E; e += 256) {
    if (OWN) counts[e] = hist[e];
    else if (hist[e]) atomicAdd(&counts[e], hist[e]);
  }
}

// counts = 0 for every live entry.
template <class RBA>
__global__ __launch_bounds__(256) void counts_clear_kernel(RBA rba, int E) {
  const RouteBatch& rb = rba.get();
  if ((int)blockIdx.x >= rb.n) return;
  int32_t* __restrict__ counts = in_global(rb.e[blockIdx.x].counts);
  for (int e = threadIdx.x; e < E; e += 256) counts[e] = 0;
}

template <int W, int V, class RBA>
void select_launch_v(RBA rba, const eb_router& p, int E, int k, int grid, bool own, hipStream_t s) {
  if (own)
    hipLaunchKernelGGL((select_kernel<W, V, true, RBA>), dim3(grid), dim3(256), 0, s, rba, p, E, k);
  else
    hipLaunchKernelGGL((select_kernel<W, V, false, RBA>), dim3(grid), dim3(256), 0, s, rba, p, E, k);
}

// Experts a lane of a W-lane team holds.
int lane_experts(const eb_router& p, int E, int W) {
  int lpg = W;
  while (lpg > 1 && lpg * p.n_group > W) lpg >>= 1;
  const int M = E / p.n_group;
  return lpg * p.n_group > W ? 1 << 20 : (M + lpg - 1) / lpg;
}

template <class RBA>
hipError_t select_batch(RBA rba, const eb_router& p, int E, int k, int grid_entries, int grid_blocks, bool own,
                        hipStream_t s) {
  prof_start(EB_K_ROUTE_TOPK, s);
  if (!own && grid_entries > 0)
    hipLaunchKernelGGL((counts_clear_kernel<RBA>), dim3(grid_entries), dim3(256), 0, s, rba, E);
  if (grid_blocks > 0) {
    const int v16 = lane_experts(p, E, 16), v64 = lane_experts(p, E, 64);
    if (v16 <= 4) select_launch_v<16, 4>(rba, p, E, k, grid_blocks, own, s);
    else if (v16 <= 8) select_launch_v<16, 8>(rba, p, E, k, grid_blocks, own, s);
    else if (v16 <= 16) select_launch_v<16, 16>(rba, p, E, k, grid_blocks, own, s);
    else if (v64 <= 8) select_launch_v<64, 8>(rba, p, E, k, grid_blocks, own, s);
    else select_launch_v<64, 32>(rba, p, E, k, grid_blocks, own, s);
  }
  prof_stop(EB_K_ROUTE_TOPK, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_select_batch(const eb_router& p, int E, int k, const RouteBatch& rb, hipStream_t s) {
  bool one = true;
  for (int i = 0; i < rb.n; ++i) one = one && rb.blk0[i + 1] - rb.blk0[i] == 1;
  return select_batch(ByValue<RouteBatch>{rb}, p, E, k, rb.n, rb.blk0[rb.n], one, s);
}

hipError_t launch_select_batch_dev(const eb_router& p, int E, int k, const RouteBatch* rb, int max_entries, int T,
                                   hipStream_t s) {
  return select_batch(InMemory<RouteBatch>{rb}, p, E, k, max_entries, max_entries * ((T + 31) / 32), T >= 1 && T <= 32,
                      s);
}

}  // namespace eb

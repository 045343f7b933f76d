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
// of two each), so a lane holds up to V consecutive experts of one group: lane j
// of the group's LPG lanes those from group M + j V on, and a group's two
// largest are a reduction over LPG lanes.  A pick is one maximum over the lane's
// values and the team.  The fp32 choice needs no order among equal values (they
// are close, so fp64 decides) and takes the values as they are; the fp64 choice
// has a wavefront to itself and goes by unsigned order keys.
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

// Order-preserving unsigned key: NaN 1, then -inf .. inf; 0 is no value.
__device__ __forceinline__ uint64_t order_key(double v) {
  if (!(v == v)) return 1ull;
  const uint64_t u = (uint64_t)__double_as_longlong(v == 0.0 ? 0.0 : v);
  return (u >> 63) ? ~u : (u | (1ull << 63));
}

// Exchange of a reduction whose values are already equal within groups of OFF
// lanes: each lane gets the value of the neighbouring group.  Within 16 lanes by
// DPP (4 and 8 as mirrors), beyond by the swaps of rows and halves.
template <int OFF>
__device__ __forceinline__ uint32_t lane_xor(uint32_t v) {
  if constexpr (OFF == 1) return __builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true);
  else if constexpr (OFF == 2) return __builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true);
  else if constexpr (OFF == 4) return __builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true);
  else if constexpr (OFF == 8) return __builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true);
  else if constexpr (OFF == 16) {
    // [0] rows 0 0 2 2, [1] rows 1 1 3 3 of v
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return (threadIdx.x & 16) ? r[0] : r[1];
  } else {
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (threadIdx.x & 32) ? r[0] : r[1];
  }
}
template <int OFF>
__device__ __forceinline__ uint64_t lane_xor(uint64_t v) {
  return ((uint64_t)lane_xor<OFF>((uint32_t)(v >> 32)) << 32) | lane_xor<OFF>((uint32_t)v);
}
template <int OFF>
__device__ __forceinline__ int lane_xor(int v) { return (int)lane_xor<OFF>((uint32_t)v); }
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

// What a lane of a team holds: experts first + i for i < V, those below end (the
// end of its group).  Lanes past the last group hold none.
struct TeamMap {
  int sub, lpg, group, first, end;
};
template <int W, int V>
__device__ __forceinline__ TeamMap team_map(const eb_router& p, int E, int sub) {
  TeamMap m;
  m.sub = sub;
  m.lpg = W;
  while (m.lpg * p.n_group > W) m.lpg >>= 1;
  m.group = sub / m.lpg;
  const int M = E / p.n_group;
  m.first = m.group * M + (sub % m.lpg) * V;
  m.end = m.group < p.n_group ? (m.group + 1) * M : 0;
  return m;
}

__device__ __forceinline__ float magnitude(float v) { return fabsf(v); }
__device__ __forceinline__ double magnitude(double v) { return fabs(v); }

// The row's scores.  softmax: over the row's largest logit and denominator; a
// row of -inf alone has s = 0, NaN and +inf logits make every s of the row NaN.
template <bool SOFT, class R>
struct Scores {
  R mx, inv;  // inv: 1 / denominator, 0 for a row of -inf alone
  __device__ __forceinline__ R of(R z) const {
    if constexpr (!SOFT) return sigmoid_of(z);
    return exp_of(z - mx) * inv;
  }
  // an upper bound of the row's scores
  __device__ __forceinline__ R top() const { return SOFT ? inv : (R)1; }
};
template <bool SOFT, int W, int V, class R>
__device__ __forceinline__ Scores<SOFT, R> row_scores(const R (&z)[V]) {
  Scores<SOFT, R> s{0, 1};
  if constexpr (SOFT) {
    const auto maxr = [](R a, R b) { return a > b ? a : b; };
    bool nan = false;
    R mx = -(R)INFINITY, sum = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      mx = maxr(mx, z[i]);
      nan |= !(z[i] == z[i]);
    }
    mx = team_reduce<W>(mx, maxr);
    s.mx = mx == -(R)INFINITY ? (R)0 : mx;  // e^(-inf - 0) = 0
#pragma unroll
    for (int i = 0; i < V; ++i) sum += exp_of(z[i] - s.mx);
    if (nan) sum = (R)__builtin_nan("");
    sum = team_reduce<W>(sum, [](R a, R b) { return a + b; });
    s.inv = sum == 0 ? (R)0 : 1 / sum;
  }
  return s;
}

// The lane's V values of a row (none: past its end); vec: in 16-byte loads.
template <int V>
__device__ __forceinline__ void load_lane(float (&c)[V], const TeamMap& m, bool vec, const float* __restrict__ row,
                                          float none) {
  if (V % 4 == 0 && vec) {
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      float4 v = make_float4(none, none, none, none);
      if (m.first + i < m.end) v = *reinterpret_cast<const float4*>(row + m.first + i);
      c[i] = v.x;
      c[i + 1] = v.y;
      c[i + 2] = v.z;
      c[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = m.first + i < m.end ? row[m.first + i] : none;
  }
}

// The two largest c of the lane's group in b1, b2 (NaN left out).
template <int W, int V>
__device__ __forceinline__ void group_best(const TeamMap& m, const float (&c)[V], float* b1, float* b2) {
  float x = c[0], y = -INFINITY;
#pragma unroll
  for (int i = 1; i < V; ++i) {
    y = __builtin_amdgcn_fmed3f(x, y, c[i]);  // x >= y: the middle one is the new second
    x = fmaxf(x, c[i]);
  }
  for (int off = 1; off < m.lpg; off <<= 1) {
    const float o1 = __shfl_xor(x, off, W), o2 = __shfl_xor(y, off, W);
    y = fmaxf(__builtin_amdgcn_fmed3f(x, y, o1), o2);
    x = fmaxf(x, o1);
  }
  *b1 = x;
  *b2 = y;
}
template <int W, int V>
__device__ __forceinline__ void group_best(const TeamMap& m, const double (&c)[V], double* b1, double* b2) {
  const auto maxr = [](double a, double b) { return a > b ? a : b; };
  double x = -INFINITY, y = x;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const double v = c[i] == c[i] ? c[i] : -INFINITY;
    y = maxr(y, v < x ? v : x);
    x = maxr(x, v);
  }
  for (int off = 1; off < m.lpg; off <<= 1) {
    const double o1 = __shfl_xor(x, off, W), o2 = __shfl_xor(y, off, W);
    y = maxr(maxr(y, o2), o1 < x ? o1 : x);
    x = maxr(x, o1);
  }
  *b1 = x;
  *b2 = y;
}

// Routing weight of the team's lane r < k from the score s of its pick.
template <int W, class R>
__device__ __forceinline__ R weight_of(const eb_router& p, bool mine, R s, R* sum) {
  const R w = mine ? s : (R)0;
  *sum = team_reduce<W>(w, [](R a, R b) { return a + b; });
  return p.norm_topk && *sum != 0 ? w / *sum : w;
}

// The k picks of one token in fp32: lane r < k of the team returns pick r's
// expert in *pick and its routing weight in *w.  Returns whether the token has
// to be chosen in fp64: a decision within the error bound, values that fp32
// comparisons do not settle (NaN, picks at -inf), or a sum of scores where fp32
// loses digits.
// bal: the lane's balance values, -inf where it has no expert; picks: 16 words of LDS of the team's own.
template <bool SOFT, int W, int V>
__device__ __forceinline__ bool choose_fp32(const eb_router& p, const TeamMap& m, int E, int k, bool vec,
                                            const float* __restrict__ z, const float (&bal)[V], volatile int* picks,
                                            int* pick, float* w) {
  // max as a median: fmaxf first quiets what an exchange brings
  const auto maxf = [](float a, float b) { return __builtin_amdgcn_fmed3f(a, b, INFINITY); };
  const float ninf = -INFINITY;
  float c[V];
  load_lane(c, m, vec, z, ninf);
  const Scores<SOFT, float> sc = row_scores<SOFT, W, V>(c);
  bool near = false;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    c[i] = sc.of(c[i]) + bal[i];
    near |= !(c[i] == c[i]);
  }
  const float margin = SOFT ? kMarginSoftmax : kMarginSigmoid, floor = 2 * margin * sc.top();
  if (p.topk_group < p.n_group) {
    float b1, b2;
    group_best<W, V>(m, c, &b1, &b2);
    const float gs = p.group_top == 2 ? b1 + b2 : b1;
    int before = 0;
    for (int g = 0; g < p.n_group; ++g) before += __shfl(gs, g * m.lpg, W) > gs;
    const bool real = m.group < p.n_group, kept = real && before < p.topk_group;
    // the last group kept against the first left out, each at its worst
    const float err = floor + margin * (fabsf(b1) + (p.group_top == 2 ? fabsf(b2) : 0.f));
    const float in = team_reduce<W>(kept ? err - gs : ninf, maxf);
    const float out = team_reduce<W>(real && !kept ? gs + err : ninf, maxf);
    near |= !(-in > out) || (real && !(gs - gs == 0.f));
#pragma unroll
    for (int i = 0; i < V; ++i) c[i] = kept ? c[i] : ninf;
  }
  // the k largest and the one after them: lane r keeps the r-th value (lane 15
  // none where k = 16: the last comparison is made from `best`)
  float own = ninf, best = ninf;
  int given = 0;
  for (int r = 0;; ++r) {
    float top = c[0];
#pragma unroll
    for (int i = 1; i < V; ++i) top = fmaxf(top, c[i]);
    const float prev = best;
    best = team_reduce<W>(top, maxf);
    if (r == k) {  // the best that was not picked, if any is left
      near |= best != ninf && !(prev - best > floor + margin * (fabsf(prev) + fabsf(best)));
      break;
    }
    own = m.sub == r ? best : own;
    // the lane that holds it gives it up.  Equal values: a second one of the
    // same lane comes next, at a distance of 0; one of another lane is given up
    // too and counts twice
    bool found = false;
    int at = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const bool hit = c[i] == best && !found;
      at = hit ? i : at;
      c[i] = hit ? ninf : c[i];
      found = found || hit;
    }
    if (found) picks[r] = m.first + at;
    given += found;
  }
  near |= team_reduce<W>(given, [](int a, int b) { return a + b; }) != k;
  const float before = __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(own), 0x111, 0xF, 0xF, true));
  if (m.sub > 0 && m.sub < k) near |= !(before - own > floor + margin * (fabsf(before) + fabsf(own)));
  if (m.sub < k) near |= own == ninf;
  const int mine = m.sub < k ? min(max(picks[m.sub], 0), E - 1) : 0;
  *pick = mine;
  float sum;
  const float we = weight_of<W>(p, m.sub < k, sc.of(z[mine]), &sum);
  *w = we * p.scale;
  near |= p.norm_topk && !(sum >= kTiny);
  return team_reduce<W>((uint32_t)near, [](uint32_t a, uint32_t b) { return a | b; }) != 0;
}

// The same from fp64 scores by a whole wavefront: decided.
template <bool SOFT, int V>
__device__ __forceinline__ void choose_fp64(const eb_router& p, int E, int k, const float* __restrict__ z,
                                            const float* __restrict__ balance, int* pick, float* w) {
  const TeamMap m = team_map<64, V>(p, E, threadIdx.x & 63);
  const auto maxk = [](uint64_t a, uint64_t b) { return a > b ? a : b; };
  const double ninf = -INFINITY;
  double c[V];
#pragma unroll
  for (int i = 0; i < V; ++i) c[i] = m.first + i < m.end ? (double)z[m.first + i] : ninf;
  const Scores<SOFT, double> sc = row_scores<SOFT, 64, V>(c);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = m.first + i;
    c[i] = e < m.end ? sc.of(c[i]) + (balance ? (double)balance[e] : 0.0) : ninf;
  }
  bool kept = m.group < p.n_group;
  if (p.topk_group < p.n_group) {
    double b1, b2;
    group_best<64, V>(m, c, &b1, &b2);
    double gs = p.group_top == 2 ? b1 + b2 : b1;
    if (!(gs == gs)) gs = ninf;
    int before = 0;
    for (int g = 0; g < p.n_group; ++g) {
      const double o = __shfl(gs, g * m.lpg, 64);
      before += o > gs || (o == gs && g < m.group);
    }
    kept = kept && before < p.topk_group;
  }
  uint64_t key[V];
#pragma unroll
  for (int i = 0; i < V; ++i) key[i] = kept && m.first + i < m.end ? order_key(c[i]) : 0ull;
  int mine = 0;
  for (int r = 0; r < k; ++r) {
    uint64_t best = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) best = maxk(best, key[i]);
    best = team_reduce<64>(best, maxk);
    int lane_at = 0x7fffffff;
#pragma unroll
    for (int i = V - 1; i >= 0; --i)
      if (key[i] == best) lane_at = m.first + i;
    const int at = team_reduce<64>(lane_at, [](int a, int b) { return a < b ? a : b; });
    if (lane_at == at) {
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (m.first + i == at) key[i] = 0;
    }
    if (m.sub == r) mine = at;
  }
  *pick = mine = min(max(mine, 0), E - 1);
  double sum;
  *w = (float)weight_of<64>(p, m.sub < k, sc.of((double)z[mine]), &sum) * p.scale;
}

// SUB workgroups of TH threads per 32-token block of the batch; VX experts a
// lane in the fp64 choice.  OWN (SUB 1): every entry of the batch has one block, whose
// workgroup writes the entry's counts; else they were cleared before and are
// added to.
constexpr int kSelectTokens = 32;
template <bool SOFT, int W, int V, int VX, int TH, int SUB, bool OWN, class RBA>
__global__ __launch_bounds__(TH) void select_kernel(RBA rba, eb_router p, int E, int k) {
  __shared__ int hist[1024];
  __shared__ int picks[TH / W][kMaxSlots];
  const RouteBatch& rb = rba.get();
  if ((int)blockIdx.x >= rb.blk0[rb.n]) return;  // past the live blocks
  const int ei = find_entry(rb.blk0, rb.n, blockIdx.x);
  const int t0 = (blockIdx.x - rb.blk0[ei]) * kSelectTokens + blockIdx.y * (kSelectTokens / SUB);
  const int rows = min(rb.tok0[ei + 1] - rb.tok0[ei] - t0, kSelectTokens / SUB);
  if (rows <= 0) return;
  const float* __restrict__ z = in_global(static_cast<const float*>(rb.e[ei].z)) + (size_t)t0 * E;
  const float* __restrict__ balance = in_global(rb.e[ei].balance);
  int32_t* __restrict__ idx = in_global(rb.e[ei].idx) + (size_t)t0 * k;
  float* __restrict__ w = in_global(rb.e[ei].w) + (size_t)t0 * k;
  for (int e = threadIdx.x; e < E; e += TH) hist[e] = 0;
  __syncthreads();
  const TeamMap m = team_map<W, V>(p, E, threadIdx.x % W);
  // rows, groups and lanes start on 16 bytes
  const bool vec = E % 4 == 0 && (E / p.n_group) % 4 == 0 && (reinterpret_cast<uintptr_t>(z) & 15) == 0;
  float bal[V];
  if (balance) load_lane(bal, m, vec && (reinterpret_cast<uintptr_t>(balance) & 15) == 0, balance, -INFINITY);
  else
#pragma unroll
    for (int i = 0; i < V; ++i) bal[i] = m.first + i < m.end ? 0.f : -INFINITY;
  auto store = [&](int t, int r, int e, float we) {
    idx[(size_t)t * k + r] = e;
    w[(size_t)t * k + r] = we;
    atomicAdd(&hist[e], 1);
  };
  // a wavefront's tokens at t .. t + 64 / W - 1: its teams stay together
  constexpr int PER = 64 / W, STEP = TH / W;
  for (int t = (threadIdx.x >> 6) * PER; t < rows; t += STEP) {
    const int tt = t + (threadIdx.x & 63) / W;
    const bool live = tt < rows;
    int e;
    float we;
    const bool again = choose_fp32<SOFT, W, V>(p, m, E, k, vec, z + (size_t)min(tt, rows - 1) * E, bal,
                                         picks[threadIdx.x / W], &e, &we);
    if (live && !again && m.sub < k) store(tt, m.sub, e, we);
    unsigned long long left = __ballot(live && again && m.sub == 0);
    while (left) {
      const int tx = t + (__ffsll(left) - 1) / W;
      left &= left - 1;
      choose_fp64<SOFT, VX>(p, E, k, z + (size_t)tx * E, balance, &e, &we);
      if ((int)(threadIdx.x & 63) < k) store(tx, threadIdx.x & 63, e, we);
    }
  }
  __syncthreads();
  int32_t* __restrict__ counts = in_global(rb.e[ei].counts);
  for (int e = threadIdx.x; e < E; e += TH) {
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

template <bool SOFT, int W, int V, int VX, int TH, int SUB, class RBA>
void select_launch_s(RBA rba, const eb_router& p, int E, int k, int grid, bool own, hipStream_t s) {
  if (own)
    hipLaunchKernelGGL((select_kernel<SOFT, W, V, VX, TH, 1, true, RBA>), dim3(grid), dim3(TH), 0, s, rba, p, E, k);
  else
    hipLaunchKernelGGL((select_kernel<SOFT, W, V, VX, TH, SUB, false, RBA>), dim3(grid, SUB), dim3(TH), 0, s, rba, p, E, k);
}
template <int W, int V, int VX, int TH, int SUB, class RBA>
void select_launch(RBA rba, const eb_router& p, int E, int k, int grid, bool own, hipStream_t s) {
  if (p.score == EB_SCORE_SOFTMAX) select_launch_s<true, W, V, VX, TH, SUB>(rba, p, E, k, grid, own, s);
  else select_launch_s<false, W, V, VX, TH, SUB>(rba, p, E, k, grid, own, s);
}

// Experts a lane of a W-lane team holds at most (0: more groups than lanes).
int lane_experts(const eb_router& p, int E, int W) {
  if (p.n_group > W) return 0;
  int lpg = W;
  while (lpg * p.n_group > W) lpg >>= 1;
  return (E / p.n_group + lpg - 1) / lpg;
}

// Most 32-token blocks for which a token gets a whole wavefront.
constexpr int kWholeWaveBlocks = 256;

template <class RBA>
hipError_t select_batch(RBA rba, const eb_router& p, int E, int k, int grid_entries, int grid_blocks, bool own,
                        hipStream_t s) {
  prof_start(EB_K_ROUTE_TOPK, s);
  if (!own && grid_entries > 0)
    hipLaunchKernelGGL((counts_clear_kernel<RBA>), dim3(grid_entries), dim3(256), 0, s, rba, E);
  if (grid_blocks > 0) {
    // a lane's 16 experts in a quarter of a wavefront are at most 4 in a whole one
    const int v16 = lane_experts(p, E, 16), v64 = lane_experts(p, E, 64);
    if (grid_blocks <= kWholeWaveBlocks && v64 <= 4) {
      if (v64 <= 1) select_launch<64, 1, 1, 1024, 2>(rba, p, E, k, grid_blocks, own, s);
      else select_launch<64, 4, 4, 1024, 2>(rba, p, E, k, grid_blocks, own, s);
    } else if (v16 > 0 && v16 <= 4) {
      select_launch<16, 4, 4, 256, 1>(rba, p, E, k, grid_blocks, own, s);
    } else if (v16 > 0 && v16 <= 8) {
      select_launch<16, 8, 4, 256, 1>(rba, p, E, k, grid_blocks, own, s);
    } else if (v16 > 0 && v16 <= 16) {
      select_launch<16, 16, 4, 256, 1>(rba, p, E, k, grid_blocks, own, s);
    } else if (v64 <= 8) {
      select_launch<64, 8, 8, 256, 1>(rba, p, E, k, grid_blocks, own, s);
    } else {
      select_launch<64, 32, 32, 256, 1>(rba, p, E, k, grid_blocks, own, s);
    }
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

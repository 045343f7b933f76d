// Shared by the grouped expert GEMMs (gemm.hip: fp32 and bf16 experts,
// gemm_fp8.hip: 8-bit experts): waits and barriers, buffer descriptors, the
// LDS swizzle and the persistent launches' item walk.
#pragma once

#include "eb_internal.h"
#include "eb_numeric.h"

namespace eb {
namespace {

enum { MODE_GATEUP = 0, MODE_DOWN = 1 };
constexpr int kXcds = 8;

// 128-byte LDS rows hold eight 16-byte chunks; logical chunk c of row r sits
// at c ^ ((r >> 1) & 7).  A ds_read_b128 phase of 16 lanes reads 16
// consecutive rows at one logical chunk: two rows share each 256-byte bank
// window, and the XOR spreads the 8 rows of each parity over 8 chunks, so the
// 16 reads hit 16 distinct 16-byte groups of the 64 banks.
__device__ __forceinline__ int swz(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

// s_waitcnt immediates (gfx9 encoding: vmcnt bits 3:0 and 15:14, expcnt
// 6:4, lgkmcnt 11:8).  Issued through the builtin so that the compiler's own
// wait insertion sees them and does not add conservative waits of its own.
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
constexpr int kWaitLgkm0 = 15 | (3 << 14) | (7 << 4);

// Bare workgroup barrier: this wave's outstanding buffer->LDS loads stay in
// flight across it (a fenced __syncthreads would drain them).
__device__ __forceinline__ void bar() {
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// Barrier that orders LDS accesses only: a wave's LDS reads and writes are done
// when it arrives, its global stores need not be (__syncthreads would wait for
// an item's output stores, 3 to 6 us with every CU storing).
__device__ __forceinline__ void bar_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(kWaitLgkm0);
  bar();
}

// A wavefront-uniform pointer the compiler cannot prove uniform, in scalar
// registers (a buffer descriptor in vector registers costs a loop per load).
template <class T>
__device__ __forceinline__ const T* uniform(const T* p) {
  const uint64_t v = (uint64_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return (const T*)(((uint64_t)hi << 32) | lo);
}

// Raw buffer descriptor over [base, base + bytes) (bytes < 2^32); offsets
// past the end read zeros.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes, 0x00020000);
}

// Float pair to packed bf16, round to nearest even (one hardware conversion).
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){a, b}, bf16x2));
}

// m-tiles per block of the item order (see grouped_gemm_bf16): a window of
// the 32 items one XCD runs at a time then spans 4 m-tiles x 8 n-tiles, so
// it streams 4 activation and 8 weight tiles instead of 32 and 1.
constexpr int kMBlock = 4;

// A group record by a scalar load (i uniform): it does not queue behind the
// vector loads in flight.  The records are written by an earlier launch.
__device__ __forceinline__ int4 scalar_record(const int4* p, int i) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 v = reinterpret_cast<const __attribute__((address_space(4))) i32x4*>((uintptr_t)p)[i];
  return make_int4(v.x, v.y, v.z, v.w);
}

// Position of an item inside its group's list: column tile and m-tile.
struct Tile2 {
  int ni, mi;
};
__device__ __forceinline__ Tile2 item_tile(int local, int mt, int n_ntiles) {
  const int mb = local / (kMBlock * n_ntiles);
  const int gm = min(kMBlock, mt - mb * kMBlock);
  const int rb = local - mb * kMBlock * n_ntiles;
  const int ni = rb / gm;
  return Tile2{ni, mb * kMBlock + (rb - ni * gm)};
}

// One thread's view of the item counters: the XCD whose range it draws from.
// Each XCD's counter has a cache line of its own, and another XCD's counter is
// read before it is drawn from: when every workgroup drew from all eight in
// one line on its way out, those 2000 atomics ran one after the other (gate/up
// at H = 2048, F = 1408: one token on 64 + 2 experts 37 -> 23 us, 80 tokens on
// three layers of 60 + 4 172 -> 165, 12 x 256 on five of 64 + 2 768 -> 764).
//
// The list's last n_tiles[0] - n_tiles[1] row blocks are small ones the scan
// set aside: their items are taken once the others are gone, so that the
// launch ends on short items.  They are split into eighths like the others
// (drawn by all XCDs from one counter, every XCD streamed from every expert:
// a launch of 256 items of K = 7168 took 220 instead of 158 us).
//
// A split-K launch has few, long items (32 per m-tile, of K = 7168, at
// H = 4096, F = 14336), and those of a small group, bound by streaming their
// weights, are hardly shorter than the others: they overlap better with the
// others' matrix work than with each other.  Setting them aside pays there only
// where the last round of items would leave most workgroups idle, or where all
// fit one round (every XCD then has some of them); else they stay in the queue.
// Down launch of 8 experts, 2 picks a token, in us, always set aside / by this
// rule / never: 2.0 rounds (128 tokens at each of two layers) 356 / 308 / 315;
// 4.0 rounds (64 at each of four) 646 / 583 / 603; 1.12 rounds (512 at one)
// 227 / 229 / 343; 2.25 rounds (384 at each of two) 437 / 438 / 480.
struct ItemQueue {
  int32_t* ctr;
  long long main;  // items before the ones set aside
  int total, xcd, victim, per_xcd;  // victim: XCD range drawn from, + kXcds for its set-aside range
  // Every item has a workgroup by number, nothing is drawn: the counters are
  // neither drawn from nor read (15 reads in turn on each workgroup's way out:
  // fp32 down launch of 774 tokens on three layers of 8 experts, H = 256,
  // F = 128, 14.2 -> 8.2 us).
  bool numbered;
  __device__ __forceinline__ ItemQueue(const GroupedProblem& p, int nsub)
      : ctr(p.work_ctr), total(p.n_tiles[0] * nsub), xcd(blockIdx.x % kXcds), victim(blockIdx.x % kXcds),
        per_xcd(gridDim.x / kXcds) {
    const int last = total % (int)gridDim.x;  // items of the last, partial round
    const bool aside = p.ksplit == 1 || total <= (int)gridDim.x || (last > 0 && 2 * last <= (int)gridDim.x);
    main = aside ? (long long)p.n_tiles[1] * nsub : total;
    numbered = main == total && total <= kXcds * per_xcd;
  }
  __device__ __forceinline__ int bound(int x) const {  // first item of range x; bound(2 kXcds) = total
    return x < kXcds ? (int)((x * main) / kXcds) : (int)(main + ((x - kXcds) * (total - main)) / kXcds);
  }
  __device__ __forceinline__ int32_t* counter() const {
    return ctr + (victim < kXcds ? victim * kWorkStride : (victim - kXcds) * kWorkStride + kWorkTail);
  }
  __device__ __forceinline__ int draw() const { return numbered ? 0 : atomicAdd(counter(), 1); }
  // The first items of an XCD's range go to its workgroups by number (drawn,
  // the first few to start would each hold a second item while others have
  // none), the rest through its counter.
  __device__ __forceinline__ int drawn(int got) const { return bound(victim) + got + (victim < kXcds ? per_xcd : 0); }
  // item index from a value drawn from victim's counter, or -1 once everything
  // is taken: the own range, the other XCDs', then the set-aside ones alike
  __device__ __forceinline__ int settle(int got) {
    if (numbered) return -1;
    int it = drawn(got);
    while (it >= bound(victim + 1)) {
      if (victim < kXcds) {
        victim = victim + 1 == kXcds ? 0 : victim + 1;
        if (victim == xcd) victim += kXcds;
      } else {
        victim = victim + 1 == 2 * kXcds ? kXcds : victim + 1;
        if (victim == xcd + kXcds) return -1;
      }
      it = drawn(__hip_atomic_load(counter(), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
      if (it < bound(victim + 1)) it = drawn(draw());
    }
    return it;
  }
  __device__ __forceinline__ int first() {
    const int it = bound(xcd) + (int)(blockIdx.x / kXcds);
    return it < bound(xcd + 1) ? it : settle(draw());
  }
};

inline int persistent_grid() {
  static int grid = 0;
  if (grid == 0) {
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess ||
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
      cus = 256;
    grid = (cus + kXcds - 1) / kXcds * kXcds;
  }
  return grid;
}

}  // namespace
}  // namespace eb

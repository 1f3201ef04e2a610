// Queries and keys brought to unit mean square and rotated, K and V on into the cache:
//   y = x rsqrt(mean(x^2) + eps) w,  mean over a head's D values or over all of a token's
//   (y0, y1) -> (y0 c - y1 s, y0 s + y1 c) for each pair, rounded once.
// A few operations per byte, so what bounds it is HBM: each row is read once, held in
// registers over the sum, and written once.
//
// Per head: lanes hold eight neighbouring values, a lane group (a power of two of them) a head,
// a warp kHeads heads of each group of one token and tensor, whose table row and weights the
// lanes load once.  Across the heads: a group of whole warps holds a token's row, up to four
// vectors of eight values a thread, and the warps' sums meet in shared memory.
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "hsa_internal.cuh"
#include "hsa_ptx.cuh"
#include "hsa_tma.cuh"

namespace hsa {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxD = 256;
constexpr int kHeads = 4;        // heads of a lane group at a time
constexpr int kHeadBlocks = 3;   // blocks per SM of the kernel per head
constexpr float kDown = 0x1p-80f;
// Tokens per SM from which on the ring takes them.  Replayed from a graph, whose steps are about
// 2.05 us, ring / group of warps: bf16 40 x 128, 16 to 150 tokens 6.2 / 6.2 us, 200 8.2 / 8.2, 300
// 8.2 / 10.3, 600 10.2 / 14.4, 5000 55 / 109; fp32 16 tokens 8.2 / 6.2, 150 8.2 / 8.2, 300 10.3 /
// 12.3, 5000 113 / 142; bf16 8 x 128 up to 600 tokens 6.2 / 6.2, 5000 20.5 / 22.8; 4 x 64, where a
// warp holds a row and the ring's blocks are one warp, up to 150 tokens 6.2 / 4.1, 1200 8.2 / 6.2,
// 5000 18.6 / 14.4.
constexpr int kRingTokens = 1;

__device__ __forceinline__ uint4 ld16(const void *p) {
  uint4 v;   // not the read-only path: the rows may be written in place
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// Brings a range into L2; 16-byte aligned, its size a multiple of 16.
__device__ __forceinline__ void bulk_prefetch(const void *src, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src), "r"(bytes) : "memory");
}

// Eight neighbouring values as they are stored.
template <bool kF32>
struct Eight {
  uint4 w[kF32 ? 2 : 1];
};
template <bool kF32>
__device__ __forceinline__ Eight<kF32> load8(const uint8_t *p) {
  Eight<kF32> v;
  v.w[0] = ld16(p);
  if (kF32) v.w[kF32 ? 1 : 0] = ld16(p + 16);
  return v;
}
template <bool kF32>
__device__ __forceinline__ void store8(uint8_t *p, const Eight<kF32> &v) {
  reinterpret_cast<uint4 *>(p)[0] = v.w[0];
  if (kF32) reinterpret_cast<uint4 *>(p)[kF32 ? 1 : 0] = v.w[kF32 ? 1 : 0];
}
// Eight values in 32 bits, the even ones apart from the odd: (x0, x2), (x4, x6), (x1, x3),
// (x5, x7), so that two pairs turn in one packed instruction.
struct Values {
  uint64_t a[2], b[2];
};
template <bool kF32>
__device__ __forceinline__ Values unpack8(const Eight<kF32> &v) {
  Values x;
  const uint4 &p = v.w[0], &q = v.w[kF32 ? 1 : 0];
  if (kF32) {
    x.a[0] = pack2(p.x, p.z), x.b[0] = pack2(p.y, p.w);
    x.a[1] = pack2(q.x, q.z), x.b[1] = pack2(q.y, q.w);
  } else {
    constexpr uint32_t kHigh = 0xffff0000u;
    x.a[0] = pack2(p.x << 16, p.y << 16), x.b[0] = pack2(p.x & kHigh, p.y & kHigh);
    x.a[1] = pack2(p.z << 16, p.w << 16), x.b[1] = pack2(p.z & kHigh, p.w & kHigh);
  }
  return x;
}
template <bool kF32>
__device__ __forceinline__ Eight<kF32> pack8(const Values &x) {
  Eight<kF32> v;
  if (kF32) {
    v.w[0] = make_uint4((uint32_t)x.a[0], (uint32_t)x.b[0], x.a[0] >> 32, x.b[0] >> 32);
    v.w[kF32 ? 1 : 0] = make_uint4((uint32_t)x.a[1], (uint32_t)x.b[1], x.a[1] >> 32, x.b[1] >> 32);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      w[2 * i] = pack_bf16(lo_f(x.a[i]), lo_f(x.b[i]));
      w[2 * i + 1] = pack_bf16(hi_f(x.a[i]), hi_f(x.b[i]));
    }
    v.w[0] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}
__device__ __forceinline__ uint64_t twice(float f) {
  return pack2(__float_as_uint(f), __float_as_uint(f));
}

__device__ __forceinline__ float squares(const Values &x) {
  const uint64_t s = fma2(x.b[1], x.b[1], fma2(x.a[1], x.a[1], fma2(x.b[0], x.b[0],
                                                                    mul2(x.a[0], x.a[0]))));
  return lo_f(s) + hi_f(s);
}
// The squares of x 2^-80.
__device__ __forceinline__ float small_squares(Values x) {
  const uint64_t f = twice(kDown);
#pragma unroll
  for (int i = 0; i < 2; ++i) x.a[i] = mul2(x.a[i], f), x.b[i] = mul2(x.b[i], f);
  return squares(x);
}
// 1 / sqrt(x) for x >= 1e-30: the approximation (within 2^-22), and where the result keeps more
// than eight bits a step of Newton's method after it; zero for infinity.
template <bool kF32>
__device__ __forceinline__ float inverse_root(float x) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  if (kF32) r = r > 0.f ? fmaf(0.5f * r, fmaf(-x * r, r, 1.f), r) : r;
  return r;
}

// What a lane keeps of the weights and of the table's row for its eight dimensions.
struct Turn {
  Values w;
  uint64_t c[2], s[2], minus_s[2];   // of its pairs 0, 1 and 2, 3
};
__device__ __forceinline__ Values values_of(const float4 &x, const float4 &y) {
  Eight<true> v;
  v.w[0] = make_uint4(__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(x.z),
                      __float_as_uint(x.w));
  v.w[1] = make_uint4(__float_as_uint(y.x), __float_as_uint(y.y), __float_as_uint(y.z),
                      __float_as_uint(y.w));
  return unpack8<true>(v);
}
__device__ __forceinline__ Values weights_at(const float *p) {
  if (!p) return Values{{twice(1.f), twice(1.f)}, {twice(1.f), twice(1.f)}};
  return values_of(__ldg(reinterpret_cast<const float4 *>(p)),
                   __ldg(reinterpret_cast<const float4 *>(p) + 1));
}
// (cos, sin) of four pairs at p.
__device__ __forceinline__ void turn_by(Turn &t, const float4 &x, const float4 &y) {
  const Values v = values_of(x, y);
#pragma unroll
  for (int i = 0; i < 2; ++i)
    t.c[i] = v.a[i], t.s[i] = v.b[i], t.minus_s[i] = v.b[i] ^ 0x8000000080000000ull;
}

// x r (r: one over the root), times the weights, turned.
template <bool kF32>
__device__ __forceinline__ Eight<kF32> normed(Values x, float r, const Turn &t, bool turn) {
  const uint64_t f = twice(r);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    x.a[i] = mul2(mul2(x.a[i], f), t.w.a[i]);
    x.b[i] = mul2(mul2(x.b[i], f), t.w.b[i]);
    if (turn) {
      const uint64_t a = x.a[i], b = x.b[i];
      x.a[i] = fma2(a, t.c[i], mul2(b, t.minus_s[i]));
      x.b[i] = fma2(a, t.s[i], mul2(b, t.c[i]));
    }
  }
  return pack8<kF32>(x);
}

struct Args {
  const uint8_t *x[3];             // q, k, v
  uint8_t *y[3];
  long long in_row[3], out_row[3]; // bytes from a token's row to the next
  const float *weight[2], *table;
  const int32_t *tidx, *kidx;
  unsigned *err;
  int H[3], first[4];              // heads; units of a token before q, k, v, and all
  Divider units;
  unsigned items;                  // n units
  int D, table_rows, k_rows, lpr_log2;
  float eps, inv;                  // inv = 1 / values of a mean

  __device__ int tensor_of(int unit) const {
    return unit < first[1] ? 0 : unit < first[2] ? 1 : 2;
  }
};

// Where token j's row of tensor `of` goes, and its table row; -1: nothing to write.  Index -1
// is a place that holds no token; others out of range are reported.
struct Place {
  long long to;
  int trow;
};
__device__ __forceinline__ Place place_of(const Args &a, int of, unsigned j) {
  Place p{(long long)j, 0};
  const int slot = a.kidx ? __ldg(a.kidx + j) : (int)j;
  if (of && a.kidx) {
    p.to = slot >= 0 && slot < a.k_rows ? slot : -1;
    if (slot < -1 || slot >= a.k_rows) set_error(a.err, kErrIndex);
  }
  if (a.table) {
    p.trow = a.tidx ? __ldg(a.tidx + j) : slot;
    if (p.trow < 0 || p.trow >= a.table_rows) {
      if (p.trow != -1) set_error(a.err, kErrIndex);
      p.to = -1;
    }
  }
  return p;
}

// Lanes that share a head: known to the compiler for D = 64 and 128 (kLog), or any.
template <int kLog>
__device__ __forceinline__ int log_lanes(const Args &a) {
  return kLog >= 0 ? kLog : a.lpr_log2;
}

// One over the roots of the mean squares of kN heads that a lane holds parts of, s: the lane's
// sums.  Where a sum overflows (rare), from those of x 2^-80, next to which eps is nothing.  All
// lanes call it.
template <bool kF32, int kLog, int kN>
__device__ __forceinline__ void head_roots(const Args &a, const Eight<kF32> (&v)[kN],
                                           float (&r)[kN]) {
  const int log = log_lanes<kLog>(a);
  float s[kN];
#pragma unroll
  for (int y = 0; y < kN; ++y) s[y] = squares(unpack8<kF32>(v[y]));
#pragma unroll
  for (int o = 0; o < (kLog >= 0 ? kLog : 5); ++o)
    if (kLog >= 0 || o < log)
#pragma unroll
      for (int y = 0; y < kN; ++y) s[y] += __shfl_xor_sync(0xffffffffu, s[y], 1 << o);
  bool down = false;
#pragma unroll
  for (int y = 0; y < kN; ++y) {
    r[y] = inverse_root<kF32>(fmaf(s[y], a.inv, a.eps));
    down |= s[y] == INFINITY;
  }
  if (__any_sync(0xffffffffu, down)) {
#pragma unroll 1
    for (int y = 0; y < kN; ++y) {
      float z = 0.f, was = 0.f;
#pragma unroll
      for (int i = 0; i < kN; ++i)
        if (i == y) z = small_squares(unpack8<kF32>(v[i])), was = s[i];
      for (int o = 0; o < log; ++o) z += __shfl_xor_sync(0xffffffffu, z, 1 << o);
      z = inverse_root<kF32>(z * a.inv) * kDown;
#pragma unroll
      for (int i = 0; i < kN; ++i)
        if (i == y && was == INFINITY) r[i] = z;
    }
  }
}

// A unit is the kHeads lane groups' heads of one token and tensor.  The grid is the blocks that
// are resident, so that each warp asks for its next unit's rows, into L2, before it takes the
// present one: the loads that it waits for are then short ones.  bf16, 40 heads of each, D = 128,
// 18900 tokens: 179 us, 0.96 of HBM's measured rate; without asking ahead 189, and with 32 blocks
// per SM in turn instead, whose number hides the latency then, 193.  fp32 428 us, 0.80; 20 heads of
// D = 256 191, 0.90; 40 of D = 96 and of 80, where a quarter and more of a group's lanes hold
// nothing, 180 both, 0.72 and 0.60.
template <bool kF32, int kLog>
__global__ void __launch_bounds__(kThreads, kHeadBlocks) norm_heads_kernel(const Args a) {
  pdl_wait();
  pdl_trigger();
  constexpr int kVec = kF32 ? 32 : 16;
  const int log = log_lanes<kLog>(a), lane = threadIdx.x & 31, c = lane & ((1 << log) - 1);
  const int group = lane >> log, groups = 32 >> log;
  const int vecs8 = kLog >= 0 ? 1 << kLog : a.D / 8;
  const bool in = kLog >= 0 || c < vecs8;
  const unsigned warps = gridDim.x * (kThreads / 32);
  for (unsigned long long i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i < a.items;
       i += warps) {
    const unsigned j = quotient((unsigned)i, a.units);
    const int u = (unsigned)i - j * a.units.d;
    const int of = a.tensor_of(u);
    const int h0 = (u - a.first[of]) * groups * kHeads + group;
    if (i + warps < a.items && lane == 0) {
      const unsigned next = (unsigned)i + warps, nj = quotient(next, a.units);
      const int nu = next - nj * a.units.d, nof = a.tensor_of(nu);
      const int nh = (nu - a.first[nof]) * groups * kHeads;
      bulk_prefetch(a.x[nof] + (long long)nj * a.in_row[nof] + (size_t)nh * vecs8 * kVec,
                    min(groups * kHeads, a.H[nof] - nh) * vecs8 * kVec);
    }
    const Place place = place_of(a, of, j);
    if (place.to < 0) continue;
    Eight<kF32> v[kHeads] = {};
    const uint8_t *src = a.x[of] + (long long)j * a.in_row[of] + c * kVec;
    uint8_t *dst = a.y[of] + place.to * a.out_row[of] + c * kVec;
#pragma unroll
    for (int y = 0; y < kHeads; ++y)
      if (in && h0 + y * groups < a.H[of])
        v[y] = load8<kF32>(src + (size_t)(h0 + y * groups) * vecs8 * kVec);
    if (of < 2) {
      Turn t;
      t.w = weights_at(in && a.weight[of] ? a.weight[of] + 8 * c : nullptr);
      if (in && a.table) {
        const float4 *row = reinterpret_cast<const float4 *>(a.table + (size_t)place.trow * a.D);
        turn_by(t, __ldg(row + 2 * c), __ldg(row + 2 * c + 1));
      }
      float r[kHeads];
      head_roots<kF32, kLog, kHeads>(a, v, r);
#pragma unroll
      for (int y = 0; y < kHeads; ++y)
        v[y] = normed<kF32>(unpack8<kF32>(v[y]), r[y], t, a.table != nullptr);
    }
#pragma unroll
    for (int y = 0; y < kHeads; ++y)
      if (in && h0 + y * groups < a.H[of])
        store8<kF32>(dst + (size_t)(h0 + y * groups) * vecs8 * kVec, v[y]);
  }
}

// A unit is one token's row of one tensor, taken by kT threads of a block: fewer tokens than SMs,
// where the ring has nothing to run ahead of, and rows that leave it no stages.
constexpr int kVectors = 4;      // vectors of eight values a thread

template <bool kF32, int kT>
__global__ void __launch_bounds__(kT < kThreads ? kThreads : kT)
norm_row_kernel(const Args a) {
  constexpr int kBlock = kT < kThreads ? kThreads : kT, kVec = kF32 ? 32 : 16;
  __shared__ float sh[2][kBlock / 32];
  pdl_wait();
  pdl_trigger();
  const int sub = threadIdx.x % kT;
  const unsigned i = blockIdx.x * (kBlock / kT) + threadIdx.x / kT;
  const int vecs8 = a.D / 8;
  Eight<kF32> v[kVectors] = {};
  int of = 0;
  unsigned j = 0;
  Place p{-1, 0};
  if (i < a.items) {
    j = quotient(i, a.units);
    of = i - j * a.units.d;
    p = place_of(a, of, j);
  }
  const int vecs = p.to < 0 ? 0 : a.H[of] * vecs8;
  const uint8_t *src = a.x[of] + (long long)j * a.in_row[of];
#pragma unroll
  for (int y = 0; y < kVectors; ++y)
    if (sub + y * kT < vecs) v[y] = load8<kF32>(src + (size_t)(sub + y * kT) * kVec);
  auto total = [&](bool small, float (&part)[kBlock / 32]) {
    float s = 0.f;
#pragma unroll
    for (int y = 0; y < kVectors; ++y) {
      const Values x = unpack8<kF32>(v[y]);
      s += small ? small_squares(x) : squares(x);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (kT > 32) {
      if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = s;
      __syncthreads();
      s = 0.f;
#pragma unroll
      for (int w = 0; w < kT / 32; ++w) s += part[threadIdx.x / kT * (kT / 32) + w];
    }
    return s;
  };
  const float inv = of < 2 ? 1.f / (float)(a.H[of] * a.D) : 0.f;
  const float s = total(false, sh[0]);
  float r = inverse_root<kF32>(fmaf(s, inv, a.eps));
  const bool down = s == INFINITY;
  if (__syncthreads_or(down)) {   // rare
    const float z = total(true, sh[1]);
    if (down) r = inverse_root<kF32>(z * inv) * kDown;
  }
  uint8_t *dst = a.y[of] + p.to * a.out_row[of];
#pragma unroll
  for (int y = 0; y < kVectors; ++y) {
    const int at = sub + y * kT;
    if (at >= vecs) continue;
    if (of < 2) {
      Turn t;
      t.w = weights_at(a.weight[of] ? a.weight[of] + 8 * at : nullptr);
      if (a.table) {
        const float4 *row = reinterpret_cast<const float4 *>(a.table + (size_t)p.trow * a.D);
        const int q = 2 * (at % vecs8);
        turn_by(t, __ldg(row + q), __ldg(row + q + 1));
      }
      v[y] = normed<kF32>(unpack8<kF32>(v[y]), r, t, a.table != nullptr);
    }
    store8<kF32>(dst + (size_t)at * kVec, v[y]);
  }
}

// Across the heads, many tokens: a block takes whole tokens, one after the other, and their rows
// of q, k, v and the table come by bulk copies into a ring of stages, so that what is in flight
// does not depend on registers and occupancy; v goes out again without passing through them.  A
// thread holds the same kY vectors of q and of k of every token, so that their weights stay in
// registers, and (a head's vectors divide the block's threads) one place in a head.  bf16, 40 heads
// of each, D = 128: 18900 tokens 182 us, 0.94 of HBM's measured rate (a group of warps per row
// 397); fp32 395 us, 0.87.
constexpr int kMostStages = 8;
constexpr int kRingThreads = 512;   // at most

struct RingArgs {
  Args a;
  int n, stages, stage;       // tokens; stages of `stage` bytes
  int inject_stall;           // test hook (hsa_test.h)
  int bytes[4], at[4];        // of q, k, v and the table's row in a stage
  float inv[2];               // 1 / values of q's and k's mean
};

template <bool kF32, int kY>
__global__ void __maxnreg__((kY == 1 ? 64 : 96)) norm_ring_kernel(const RingArgs z) {
  constexpr int kVec = kF32 ? 32 : 16, kMostWarps = kRingThreads / 32;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint64_t full[kMostStages];
  __shared__ __align__(16) float part[2][2][kMostWarps];
  __shared__ int abort_flag;
  const Args &a = z.a;
  const int threads = blockDim.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const bool leads = threadIdx.x == 0;
  if (leads) {
    for (int s = 0; s < z.stages; ++s) mbar_init(&full[s], 2);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // a block may have fewer threads than these: those of warps that are not there stay zero
  for (int i = threadIdx.x; i < 4 * kMostWarps; i += threads) (&part[0][0][0])[i] = 0.f;
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int step = gridDim.x;
  auto slot_of = [&](int j) { return a.kidx ? __ldg(a.kidx + j) : j; };
  auto trow_of = [&](int j, int slot) { return a.tidx ? __ldg(a.tidx + j) : slot; };
  auto load_rows = [&](int j, int s) {
    mbar_expect_tx(&full[s], z.bytes[0] + z.bytes[1] + z.bytes[2]);
#pragma unroll
    for (int i = 0; i < 3; ++i)
      if (z.bytes[i])
        bulk_load(smem_addr(smem) + s * z.stage + z.at[i], a.x[i] + (long long)j * a.in_row[i],
                  z.bytes[i], &full[s]);
  };
  auto load_table = [&](int trow, int s) {
    if (a.table && trow >= 0 && trow < a.table_rows) {
      mbar_expect_tx(&full[s], z.bytes[3]);
      bulk_load(smem_addr(smem) + s * z.stage + z.at[3], a.table + (size_t)trow * a.D, z.bytes[3],
                &full[s]);
    } else {
      mbar_arrive(&full[s]);
    }
  };
  if (leads) {
    for (int s = 0, j = blockIdx.x; s < z.stages && j < z.n; ++s, j += step) load_rows(j, s);
    for (int s = 0, j = blockIdx.x; s < z.stages && j < z.n; ++s, j += step)
      if (z.inject_stall != 1 || s)   // test hook: the first token's never comes
        load_table(trow_of(j, slot_of(j)), s);
  }
  const int vecs8 = a.D / 8, in_head = threadIdx.x % vecs8;
  Values w[2][kY];
  bool mine[2][kY];
#pragma unroll
  for (int of = 0; of < 2; ++of)
#pragma unroll
    for (int y = 0; y < kY; ++y) {
      const int at = threadIdx.x + y * threads;
      mine[of][y] = at < a.H[of] * vecs8;
      w[of][y] = weights_at(mine[of][y] && a.weight[of] ? a.weight[of] + 8 * at : nullptr);
    }
  int s = 0;                  // the present stage
  uint32_t phase = 0;
  int loaded = z.stages * step + blockIdx.x;   // the next token to load
  int late_trow = -1;         // its table row
  int slot = 0, trow = 0;
  if ((int)blockIdx.x < z.n) {
    slot = slot_of(blockIdx.x);
    trow = trow_of(blockIdx.x, slot);
  }
  for (int j = blockIdx.x, it = 0; j < z.n; j += step, ++it) {
    // the next token's places, and the table's row of the token that this stage takes next
    int slot_next = 0, trow_next = 0, trow_far = -1;
    if (j + step < z.n) {
      slot_next = slot_of(j + step);
      trow_next = trow_of(j + step, slot_next);
    }
    if (leads && j + z.stages * step < z.n)
      trow_far = trow_of(j + z.stages * step, slot_of(j + z.stages * step));
    bool all = true, kv = true;   // whether q, and whether k and v are written
    if (a.kidx && (slot < 0 || slot >= a.k_rows)) {
      kv = false;
      if (leads && slot != -1) set_error(a.err, kErrIndex);
    }
    if (a.table && (trow < 0 || trow >= a.table_rows)) {
      all = kv = false;
      if (leads && trow != -1) set_error(a.err, kErrIndex);
    }
    mbar_wait(&full[s], phase, &abort_flag, a.err);
    const uint8_t *stage = smem + s * z.stage;
    if (leads && z.bytes[2] && kv)
      bulk_store(a.y[2] + (long long)slot * a.out_row[2], smem_addr(stage) + z.at[2], z.bytes[2]);
    Eight<kF32> v[2][kY] = {};
    float sum[2], r[2];
#pragma unroll
    for (int of = 0; of < 2; ++of) {
      sum[of] = 0.f;
#pragma unroll
      for (int y = 0; y < kY; ++y) {
        if (mine[of][y]) {
          const uint4 *p = reinterpret_cast<const uint4 *>(
              stage + z.at[of] + (threadIdx.x + y * threads) * kVec);
          v[of][y].w[0] = p[0];
          if (kF32) v[of][y].w[kF32 ? 1 : 0] = p[kF32 ? 1 : 0];
        }
        sum[of] += squares(unpack8<kF32>(v[of][y]));
      }
    }
    Turn t;
    if (a.table) {
      const float4 *p = reinterpret_cast<const float4 *>(stage + z.at[3]) + 2 * in_head;
      turn_by(t, p[0], p[1]);
    }
    auto total = [&]() {
#pragma unroll
      for (int of = 0; of < 2; ++of) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) sum[of] += __shfl_xor_sync(0xffffffffu, sum[of], o);
        if (lane == 0) part[it & 1][of][warp] = sum[of];
      }
      __syncthreads();
#pragma unroll
      for (int of = 0; of < 2; ++of) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kMostWarps / 4; ++i) {   // those of warps that are not there are zero
          const float4 q = reinterpret_cast<const float4 *>(part[it & 1][of])[i];
          x.x += q.x, x.y += q.y, x.z += q.z, x.w += q.w;
        }
        sum[of] = (x.x + x.y) + (x.z + x.w);
      }
    };
    total();
    // every thread has left the stage before: it takes the next token to load
    if (leads && it > 0 && loaded < z.n && !*(volatile int *)&abort_flag) {
      bulk_stores_read();
      const int late = s == 0 ? z.stages - 1 : s - 1;
      load_rows(loaded, late);
      load_table(late_trow, late);
      loaded += step;
    }
    const bool down[2] = {sum[0] == INFINITY, sum[1] == INFINITY};
#pragma unroll
    for (int of = 0; of < 2; ++of) r[of] = inverse_root<kF32>(fmaf(sum[of], z.inv[of], a.eps));
    if (down[0] || down[1]) {   // rare, and the same for all threads
#pragma unroll
      for (int of = 0; of < 2; ++of) {
        sum[of] = 0.f;
#pragma unroll
        for (int y = 0; y < kY; ++y) sum[of] += small_squares(unpack8<kF32>(v[of][y]));
      }
      __syncthreads();
      total();
#pragma unroll
      for (int of = 0; of < 2; ++of)
        if (down[of]) r[of] = inverse_root<kF32>(sum[of] * z.inv[of]) * kDown;
    }
#pragma unroll
    for (int of = 0; of < 2; ++of) {
      uint8_t *out = a.y[of] + (long long)(of ? slot : j) * a.out_row[of];
#pragma unroll
      for (int y = 0; y < kY; ++y)
        if (mine[of][y] && (of ? kv : all)) {
          t.w = w[of][y];
          store8<kF32>(out + (size_t)(threadIdx.x + y * threads) * kVec,
                       normed<kF32>(unpack8<kF32>(v[of][y]), r[of], t, a.table != nullptr));
        }
    }
    late_trow = trow_far;
    slot = slot_next;
    trow = trow_next;
    if (++s == z.stages) s = 0, phase ^= 1;
  }
  if (leads) bulk_stores_written();
  if (leads && abort_flag) {   // a wait ran out: copies in flight land before the block ends
    const int count = (loaded - (int)blockIdx.x) / step;
    for (int i = max(0, count - z.stages); i < count && blockIdx.x + i * step < (unsigned)z.n; ++i)
      mbar_wait(&full[i % z.stages], i / z.stages & 1, &abort_flag, a.err, false);
  }
}

template <bool kF32>
void launch_row(const Args &a, int threads, cudaStream_t s) {
  auto go = [&](auto kernel, int t) {
    const int block = t < kThreads ? kThreads : t;
    const unsigned per = block / t;
    launch_pdl(kernel, dim3((a.items + per - 1) / per), dim3(block), 0, s, a);
  };
  switch (threads) {
    case 32: return go(norm_row_kernel<kF32, 32>, 32);
    case 64: return go(norm_row_kernel<kF32, 64>, 64);
    case 128: return go(norm_row_kernel<kF32, 128>, 128);
    case 256: return go(norm_row_kernel<kF32, 256>, 256);
    case 512: return go(norm_row_kernel<kF32, 512>, 512);
    default: return go(norm_row_kernel<kF32, 1024>, 1024);
  }
}

// Registers of a ring kernel's thread, which may from now on use all of an SM's shared memory on
// this device; 0 where that failed.
template <bool kF32, int kY>
int ring_registers() {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  int regs = known[dev].load(std::memory_order_acquire);
  if (regs) return regs;
  cudaFuncAttributes f;
  if (cudaFuncSetAttribute(norm_ring_kernel<kF32, kY>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           226 * 1024 - 1024) != cudaSuccess ||
      cudaFuncGetAttributes(&f, norm_ring_kernel<kF32, kY>) != cudaSuccess)
    return 0;
  known[dev].store(regs = (f.numRegs + 7) & ~7, std::memory_order_release);
  return regs;
}

// Launches the ring for n tokens where it is the better: false where the other kernel takes the
// call, for few tokens, rows that 512 threads or two stages do not hold, or head dimensions whose
// vectors do not divide as many threads.
template <bool kF32>
bool launch_ring(const Args &a, int n, bool with_v, cudaStream_t s) {
  constexpr int kRoom = 227 * 1024, kOwn = 1024 + 1024;   // an SM's; a block's, and its statics
  const int vecs8 = a.D / 8, most = std::max(a.H[0], a.H[1]) * vecs8;
  if (n < kRingTokens * sm_count()) return false;
  int unit = 32;                                          // whole warps and whole heads
  while (unit % vecs8) unit += 32;
  const int y = most <= kRingThreads ? 1 : 2;
  const int threads = ((most + y - 1) / y + unit - 1) / unit * unit;
  if (threads > kRingThreads) return false;
  const int regs = y == 1 ? ring_registers<kF32, 1>() : ring_registers<kF32, 2>();
  if (!regs) return false;
  RingArgs z;
  z.a = a;
  z.n = n;
  z.stage = 0;
  z.inject_stall = attention_stall();
  for (int i = 0; i < 4; ++i) {
    z.bytes[i] = i == 3 ? (a.table ? 4 * a.D : 0)
                 : i == 2 && !with_v ? 0 : a.H[i] * a.D * (kF32 ? 4 : 2);
    z.at[i] = z.stage;
    z.stage += z.bytes[i];
  }
  for (int i = 0; i < 2; ++i) z.inv[i] = 1.f / (float)(a.H[i] * a.D);
  z.stage = (z.stage + 127) & ~127;
  int nb = std::min(4, 65536 / (regs * threads));
  for (; nb >= 1; --nb) {
    z.stages = std::min(kMostStages, (kRoom / nb - kOwn) / z.stage);
    if (z.stages >= 3 || (nb == 1 && z.stages == 2)) break;
  }
  if (nb < 1) return false;
  const int blocks = std::min(n, nb * sm_count());
  launch_pdl(y == 1 ? norm_ring_kernel<kF32, 1> : norm_ring_kernel<kF32, 2>, dim3(blocks),
             dim3(threads), (size_t)z.stages * z.stage, s, z);
  return true;
}

}  // namespace
}  // namespace hsa

using namespace hsa;

extern "C" int hsa_qk_norm_rope(const void *q, long long q_row, const void *k, long long k_row,
                                const void *v, long long v_row, const float *q_weight,
                                const float *k_weight, float eps, int across, const float *table,
                                const int32_t *table_idx, int table_rows, int n, int Hq, int Hkv,
                                int D, hsa_dtype dtype, void *q_out, void *k_out, void *v_out,
                                const int32_t *k_idx, int k_rows, hsa_stream_t stream) {
  if (n < 0 || Hq < 1 || Hkv < 1 || D < 8 || (D & 7) || k_rows < 0) return HSA_ERR_INVALID_ARG;
  if (dtype != HSA_BF16 && dtype != HSA_F32) return HSA_ERR_INVALID_ARG;
  if (!(eps >= 1e-30f) || !std::isfinite(eps)) return HSA_ERR_INVALID_ARG;
  if (table ? table_rows < 1 : table_idx != nullptr) return HSA_ERR_INVALID_ARG;
  const int size = dtype == HSA_F32 ? 4 : 2, step = 16 / size;
  const int H[3] = {Hq, Hkv, Hkv};
  const long long rows[3] = {q_row, k_row, v_row};
  for (int i = 0; i < (v ? 3 : 2); ++i)
    if (rows[i] < (long long)H[i] * D || rows[i] % step || rows[i] > (1LL << 31))
      return HSA_ERR_INVALID_ARG;
  if (D > kMaxD || Hq > (1 << 20) || Hkv > (1 << 20)) return HSA_ERR_UNSUPPORTED;
  const int most = Hq > Hkv ? Hq : Hkv;
  if (across && (long long)most * (D / 8) > 1024 * kVectors) return HSA_ERR_UNSUPPORTED;
  if (!v != !v_out) return HSA_ERR_INVALID_ARG;
  if (n == 0) return HSA_OK;
  if (!q || !k || !q_out || !k_out || !aligned16(q) || !aligned16(k) || !aligned16(v) ||
      !aligned16(q_out) || !aligned16(k_out) || !aligned16(v_out) || !aligned16(q_weight) ||
      !aligned16(k_weight) || !aligned16(table))
    return HSA_ERR_INVALID_ARG;
  Args a;
  const void *in[3] = {q, k, v};
  void *out[3] = {q_out, k_out, v_out};
  a.lpr_log2 = 0;
  while ((1 << a.lpr_log2) * 8 < D) ++a.lpr_log2;
  const int heads = across ? 0 : (32 >> a.lpr_log2) * kHeads;
  a.first[0] = 0;
  for (int i = 0; i < 3; ++i) {
    a.x[i] = static_cast<const uint8_t *>(in[i]);
    a.y[i] = static_cast<uint8_t *>(out[i]);
    a.in_row[i] = rows[i] * size;
    a.out_row[i] = (long long)H[i] * D * size;
    a.H[i] = H[i];
    a.first[i + 1] = a.first[i] + (i == 2 && !v ? 0 : across ? 1 : (H[i] + heads - 1) / heads);
  }
  const long long items = (long long)n * a.first[3];
  if (items > 0x7fffffffLL) return HSA_ERR_UNSUPPORTED;
  a.weight[0] = q_weight;
  a.weight[1] = k_weight;
  a.table = table;
  a.tidx = table_idx;
  a.kidx = k_idx;
  a.err = device_error_word();
  if (!a.err) return HSA_ERR_CUDA;
  a.units = make_divider((unsigned)a.first[3]);
  a.items = (unsigned)items;
  a.D = D;
  a.table_rows = table_rows;
  a.k_rows = k_rows;
  a.eps = eps;
  a.inv = 1.f / (float)D;
  cudaStream_t s = (cudaStream_t)stream;
  const bool f32 = dtype == HSA_F32;
  count_launches(1);
  if (!across) {
    const long long need = (items + kThreads / 32 - 1) / (kThreads / 32);
    const long long cap = (long long)sm_count() * kHeadBlocks;
    const int known = D == 64 ? 3 : D == 128 ? 4 : -1;
    launch_pdl(f32 ? (known == 3   ? norm_heads_kernel<true, 3>
                      : known == 4 ? norm_heads_kernel<true, 4>
                                   : norm_heads_kernel<true, -1>)
                   : (known == 3   ? norm_heads_kernel<false, 3>
                      : known == 4 ? norm_heads_kernel<false, 4>
                                   : norm_heads_kernel<false, -1>),
               dim3((unsigned)(need < cap ? need : cap)), dim3(kThreads), 0, s, a);
  } else if (!(f32 ? launch_ring<true>(a, n, v != nullptr, s)
                   : launch_ring<false>(a, n, v != nullptr, s))) {
    int t = 32;
    while (t * kVectors < most * (D / 8)) t *= 2;
    if (f32) launch_row<true>(a, t, s);
    else launch_row<false>(a, t, s);
  }
  return launch_status();
}

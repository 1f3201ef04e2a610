// What the kernels of attention over paged caches share: fragments and copies, the cut of all
// sequences' key tiles into equal runs, and the join of what several blocks made of a unit.
// hsa_paged_attention.cu tells how they work together.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hsa_internal.cuh"
#include "hsa_ptx.cuh"

namespace hsa {

// What the join has to know of a unit that several blocks shared, from the block that
// ended it: how many, the first, and that one's slot; parts = 0: that block ended none.
struct CutUnit {
  int parts, first, slot, b, unit, pad[3];
};

struct PagedArgs {
  CutUnit *cuts;                   // [blocks]
  const __nv_bfloat16 *q;
  const uint8_t *k, *v;            // pages [n_pages][page][Hkv][D]
  const uint8_t *ks, *vs;          // [n_pages][page][Hkv]
  const int32_t *table, *lens;
  __nv_bfloat16 *out;
  float *ws;
  unsigned *err;
  int batch, n_new, Hq, Hkv, rows, row_tiles;   // rows = n_new G
  Divider group;                                // by G = Hq / Hkv
  int n_pages, page_log2, max_pages, sms;
  int side;                        // units that run side by side (4 bits), or 1
  int inject_stall;                // test hook (hsa_test.h)
  float scale_log2, scale_digits, scale_power;   // the first is the others' product
};

// The 4-bit cache's kernels (hsa_paged_attention4.cu) over checked arguments.
int launch_paged4(PagedArgs &a, int D, void *workspace, cudaStream_t stream);

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kMostRows = 32;         // query rows of a unit at most
constexpr int kMaxPerSm = 4;          // CTAs per SM that the workspace is sized for
constexpr float kLowest = -3.0e38f;   // running maximum before the first key
constexpr float kPShift = 14.f;       // fp16 probabilities are 2^(u - M + 14)
constexpr float kFar = 0x1p64f;       // a lane's weights' sum above it takes a new R

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// d += a b, 16 rows x 8 columns x 16.
template <bool kF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                    uint32_t b1) {
  if (kF16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
        "{%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// An 8 x 8 block of 16-bit values, a pair per lane, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t w) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(w));
  return r;
}

// 16 bytes into shared memory, zeros where !ok.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src),
               "r"(ok ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void wait_all_but() {
  asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// A part of a unit in the workspace: its rows' sums, then of each row M, l (and with codes R).
__host__ __device__ constexpr int part_stats(bool code) { return code ? 4 : 2; }
__host__ __device__ constexpr int part_floats(int D, bool code, int rows) {
  return rows * (D + part_stats(code));
}

// What every block of a launch derives from the lengths: the key tiles of all units, cut
// into `ctas` runs of `base` or base + 1 tiles.  A tile per block up to one block per SM,
// then at least two, which overlap (one token against 4001 keys of 8 heads 10.3 us, 11.7
// with 456 blocks of one or two).
struct Plan {
  int total, ctas, base, more;     // more: how many runs have one tile more, the first ones
};
__device__ __forceinline__ Plan plan_of(int total, int grid, int sms) {
  Plan p;
  p.total = total;
  p.ctas = max(1, min(grid, max(min(total, sms), total / 2)));
  p.base = total / p.ctas;
  p.more = total - p.base * p.ctas;
  return p;
}
__device__ __forceinline__ int first_tile(const Plan &p, int cta) {
  return cta * p.base + min(cta, p.more);
}
__device__ __forceinline__ int cta_of(const Plan &p, int tile) {
  const int longer = p.more * (p.base + 1);
  return tile < longer ? tile / (p.base + 1) : p.more + (tile - longer) / p.base;
}

// len_b, checked: negative, or more than the table's pages hold.
__device__ __forceinline__ int length(const PagedArgs &a, int b) {
  const int n = __ldg(a.lens + b);
  const long long most = (long long)a.max_pages << a.page_log2;
  if (n < 0 || n > most) {
    set_error(a.err, kErrIndex);
    return n < 0 ? 0 : (int)most;
  }
  return n;
}

// A place in the row of key tiles.
struct Cursor {
  int b, unit, tile, tiles, len;   // unit: head * row_tiles + row tile
};
__device__ __forceinline__ void step(const PagedArgs &a, Cursor &c, int tile, int side = 1) {
  if (++c.tile < c.tiles) return;
  c.tile = 0;
  if (side == 1) {
    if (++c.unit < a.Hkv * a.row_tiles) return;
    c.unit = 0;
  }
  do {
    if (++c.b >= a.batch) return;   // past the end: not used any more
    c.len = length(a, c.b);
    c.tiles = (c.len + tile - 1) / tile;
  } while (c.tiles == 0);
}

// Zeros for the rows of sequences without keys; the blocks share the sequences out.
template <int D>
__device__ __forceinline__ void clear_empty(const PagedArgs &a) {
  for (int b = blockIdx.x; b < a.batch; b += gridDim.x) {
    if (length(a, b) != 0) continue;
    const long long n = (long long)a.n_new * a.Hq * (D / 8);
    uint4 *dst = reinterpret_cast<uint4 *>(a.out) + b * n;
    for (long long i = threadIdx.x; i < n; i += kThreads) dst[i] = make_uint4(0u, 0u, 0u, 0u);
  }
}

__device__ __forceinline__ uint64_t both(float lo, float hi) {
  return pack2(__float_as_uint(lo), __float_as_uint(hi));
}

// Codes: the products of two rows with one key times the query rows' power of two (where it
// is below 1) and the key's, w = (kf, kf, vs, vs).  Only the key's factor holds digits, the
// scale's, so that a score is rounded here and the powers of two after it are exact: R, one of
// the scores, and the scores inside the FMA that subtracts it are the same numbers.  (A product
// rounded as it is subtracted would differ from itself, by a half step of it.)
__device__ __forceinline__ uint64_t code_product(const float (&y)[4], int n, const float (&before)[2],
                                             const uint4 &w) {
  return mul2(mul2(both(y[2 * n], y[2 * n + 1]), both(before[0], before[1])), pack2(w.x, w.y));
}

template <int D, int kNR>
struct CodeTile {
  uint2 q[D / 16][kNR];
  float before[kNR][2], after[kNR][2];
  int limit[kNR][2];                            // keys of the tile that a row sees
  float ref[kNR][2], l[kNR][2], m[kNR][2];      // those before the tile; then the new R, l with
  float s[2][kNR][4], mx[kNR][2];               // the tile's, the old m relative to R, u
};

// The end of a row's sums: x 2^h / l, by factors that are in range wherever the result is.  h may
// lie beyond the exponents that 2^h has alone, where scores far from R meet values near the ends
// of their range (l then has scores of that size too): l's exponent goes into it first, and what
// is left in two halves.  Else the usual 2^h, and 1 / l.
template <bool kCode>
struct RowEnd {
  float inv, up = 1.f, rest = 1.f;
  __device__ __forceinline__ RowEnd(float l, float h) {
    inv = l > 0.f ? 1.f / l : l == 0.f ? 0.f : l;
    if (!kCode) return;
    if (fabsf(h) > 100.f && l > 0.f) {
      const uint32_t w = __float_as_uint(l);
      inv = 1.f / __uint_as_float((w & 0x7fffffu) | 0x3f800000u);
      up = rest = fast_exp2(0.5f * (h - (float)((int)(w >> 23) - 127)));
    } else {
      up = fast_exp2(h);
    }
  }
  __device__ __forceinline__ float operator()(float x) const { return x * inv * up * rest; }
};

// Joins a row's parts where several blocks shared its unit: one block for each block of
// the kernel before and each row, and most of them find that theirs ended no such unit.
// A part takes D/4 lanes, four dimensions each; bound by the round trips to L2, so each
// lane group loads eight parts at once, and statistics with sums.  With codes, with a third
// statistic, four: with eight it fits an SM three blocks or spills (48 ragged sequences 9.4
// against 6.6 us, 12 heads x 64 of 16 sequences 8.4 against 6.4).
constexpr int kJoinThreads = 256;

template <int D, bool kCode, int kNR>
__global__ void __launch_bounds__(kJoinThreads, 4)
paged_join_kernel(const PagedArgs a) {
  constexpr int kRows = 8 * kNR, kStat = part_stats(kCode), kPart = part_floats(D, kCode, kRows);
  constexpr int kL = D / 4, kGroups = kJoinThreads / kL;
  constexpr int kAtOnce = kCode ? 4 : 8;
  __shared__ float4 sh_o[kJoinThreads];
  __shared__ float4 sh_stat[kGroups];    // M, l, R
  pdl_wait();
  pdl_trigger();
  const CutUnit u = a.cuts[blockIdx.x];
  if (u.parts == 0) return;
  const int h = u.unit / a.row_tiles, rr = blockIdx.y, r = (u.unit - h * a.row_tiles) * kRows + rr;
  if (r >= a.rows) return;
  const int sub = threadIdx.x % kL, group = threadIdx.x / kL;
  // in 8 bits L and M are relative to R
  float M = kLowest, R = kLowest, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto level = [&](const float4 &w) { return kCode ? w.z - R + w.x : w.x; };
  auto refer = [&](float to_r) {   // R rises
    if (!kCode) return;
    L *= fast_exp2(R - to_r);
    M = fmaxf(M + (R - to_r), kLowest);
    R = to_r;
  };
  auto add = [&](const float4 &w, const float4 &x) {
    const float f = fast_exp2(level(w) - M);
    L = fmaf(kCode ? fast_exp2(w.z - R) : f, w.y, L);
    acc.x = fmaf(f, x.x, acc.x);
    acc.y = fmaf(f, x.y, acc.y);
    acc.z = fmaf(f, x.z, acc.z);
    acc.w = fmaf(f, x.w, acc.w);
  };
  for (int p0 = group; p0 < u.parts; p0 += kAtOnce * kGroups) {
    float4 w[kAtOnce], x[kAtOnce];
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) {
      const int p = p0 + y * kGroups;
      w[y] = make_float4(kLowest, 0.f, kLowest, 0.f);
      x[y] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (p < u.parts) {
        const float *part = a.ws + (size_t)(p ? 2 * (u.first + p * a.side) : u.slot) * kPart;
        const float *stat = part + kRows * D + kStat * rr;
        if constexpr (kCode) {
          w[y] = *reinterpret_cast<const float4 *>(stat);
        } else {
          const float2 z = *reinterpret_cast<const float2 *>(stat);
          w[y].x = z.x, w[y].y = z.y;
        }
        x[y] = *reinterpret_cast<const float4 *>(part + rr * D + 4 * sub);
      }
    }
    float to_r = R;
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) to_r = fmaxf(to_r, w[y].z);
    refer(to_r);
    float to = M;
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) to = fmaxf(to, level(w[y]));
    const float f0 = fast_exp2(M - to);
    M = to;
    if (!kCode) L *= f0;
    acc.x *= f0, acc.y *= f0, acc.z *= f0, acc.w *= f0;
#pragma unroll
    for (int y = 0; y < kAtOnce; ++y) add(w[y], x[y]);
  }
  sh_o[threadIdx.x] = acc;
  if (sub == 0) sh_stat[group] = make_float4(M, L, R, 0.f);
  __syncthreads();
  if (group) return;
#pragma unroll
  for (int y = 0; y < kGroups; ++y) R = fmaxf(R, sh_stat[y].z);
  M = kLowest;
#pragma unroll
  for (int y = 0; y < kGroups; ++y) M = fmaxf(M, level(sh_stat[y]));
  L = 0.f;
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int y = 0; y < kGroups; ++y) add(sh_stat[y], sh_o[y * kL + sub]);
  const RowEnd<kCode> end(L, M - kPShift);
  const int i = quotient(r, a.group);
  reinterpret_cast<uint2 *>(a.out + ((size_t)((size_t)u.b * a.n_new + i) * a.Hq +
                                     h * (int)a.group.d +
                                     (r - i * (int)a.group.d)) * D)[sub] =
      make_uint2(pack_bf16(end(acc.x), end(acc.y)), pack_bf16(end(acc.z), end(acc.w)));
}

size_t workspace_bytes(int D) {
  return (size_t)sm_count() * kMaxPerSm * (sizeof(CutUnit) + 2 * kMostRows * ((size_t)D + 4) * 4);
}

}  // namespace
}  // namespace hsa

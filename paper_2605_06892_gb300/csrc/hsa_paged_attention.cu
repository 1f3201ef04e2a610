// Attention of a few new tokens per sequence over a paged KV cache, bf16 or 8-bit:
//   o[b, i, h] = sum_j softmax_j(scale <q[b,i,h], k_j>) v_j,  j < len_b - n_new + i + 1,
// with k, v of the head that h's group shares.  A few FLOPs per byte of cache, so what
// bounds it is reading the cache once.
//
// Work split.  A unit is (sequence, K/V head, 16 query rows); its rows are the group's
// heads of all new tokens, row r = i G + g, so that one pass over the keys serves the
// whole group.  The units' key tiles, laid end to end, are cut into equal runs, one per
// CTA and as many CTAs as are resident: sequences of any mix of lengths keep every SM
// busy to the end.  A run that holds a whole unit stores its rows; the others leave
// (M, l, O) in the workspace and the join kernel merges them.
//
// In a CTA each of four warps takes its own kKW keys of a tile, with its own running
// maximum, its own ring of cp.async stages and no CTA barrier until the unit's end; the
// ring runs on across units.  The products are m16n8k16 MMAs: 16 rows are all there is,
// an eighth of the 128-row tile of the tcgen05 form, and the tensor pipe idles most of
// the time at these rows (the attention over whole prompts uses tcgen05).  The fragments
// come straight from 16-byte shared loads: the order of the head's dimensions inside a
// product and of the keys inside a tile is free, so each lane multiplies what lies
// together (column orders below), without transposing loads.
//
// 8-bit cache.  A key's e4m3 codes are exact in fp16, and so is a bf16 query row after
// scaling by a power of two (its values below 2^-39 of the largest aside), so the
// products are exact and the key's 2^ks multiplies the score.  The value's 2^vs goes into
// the probability: with t_j the score in log2 units, u_j = t_j + vs_j and M = max u_j,
//   o = sum_j 2^(u_j - M) code_j / sum_j 2^(t_j - M),
// where no factor 2^(u_j - M) exceeds 1 and the sum of the second lies within 2^-120 and
// 2^100 n because vs does within [-100, 120].
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "hsa_internal.cuh"
#include "hsa_ptx.cuh"

namespace hsa {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 16;             // query rows of a unit
constexpr int kMaxPerSm = 4;          // CTAs per SM that the workspace is sized for
constexpr float kLowest = -3.0e38f;   // running maximum before the first key
constexpr float kPShift = 14.f;       // fp16 probabilities are 2^(u - M + 14)

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

__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint32_t codes16) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes16));
  return h;
}

// d += a b, 16 rows x 8 columns x 16.
template <bool kF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
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

// 16 bytes into shared memory, zeros where !ok.
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0)
               : "memory");
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

template <int D, bool kF8>
struct Cfg {
  static constexpr int kRowBytes = D * (kF8 ? 1 : 2);
  static constexpr int kChunks = kRowBytes / 16;               // 16-byte chunks per row
  static constexpr int kKW = kRowBytes == 256 ? 16 : 32;       // keys per warp and tile
  static constexpr int kTile = kWarps * kKW;                   // keys per tile
  static constexpr int kStages = kRowBytes == 64 ? 4 : 3;
  static constexpr int kHalf = kKW * kRowBytes;                // K (or V) bytes of a stage
  static constexpr int kScales = kF8 ? kKW * 8 : 0;            // (2^ks, vs) per key
  static constexpr int kStage = 2 * kHalf + kScales;
  static constexpr int kMergeO = kRows * D * 4;                // O of one warp
  static constexpr int kSmem = kWarps * kStages * kStage + kMergeO;
};

// The key (row of an 8-key block) of MMA column n.  A lane quad's 16-byte loads of K
// (keys of columns 2x, 2x+1; four chunks) and of V (keys of columns 0, 2, 4, 6 or 1, 3,
// 5, 7; two chunks) then fall into distinct banks under the swizzles below.
template <int kChunks>
__device__ __forceinline__ int key_of(int n) {
  return kChunks == 4 ? n ^ ((n >> 1) & 1) : (n >> 1) | ((n & 1) << 2);
}
template <int kChunks>
__device__ __forceinline__ int k_chunk(int c, int row) {
  return kChunks == 4 ? c : c ^ (row & 7);
}
template <int kChunks>
__device__ __forceinline__ int v_chunk(int c, int row) {
  return kChunks == 4 ? c ^ (((row >> 2) & 1) << 1) : c ^ ((row & 3) << 1);
}

struct Args {
  const __nv_bfloat16 *q;
  const uint8_t *k, *v;            // pages [n_pages][page][Hkv][D]
  const uint8_t *ks, *vs;          // [n_pages][page][Hkv]
  const int32_t *table, *lens;
  __nv_bfloat16 *out;
  float *ws;
  unsigned *err;
  int batch, n_new, Hq, Hkv, G, rows, row_tiles;   // rows = n_new G
  int n_pages, page_log2, max_pages;
  float scale_log2;
};

// What every block of a launch derives from the lengths: the number of tiles, and this
// tile's (or sequence's) place among them.
struct Plan {
  long long total;     // key tiles of all units
  int ctas;            // blocks with work: min(gridDim, total)
};
__device__ __forceinline__ long long first_tile(const Plan &p, int cta) {
  return (long long)cta * p.total / p.ctas;
}
__device__ __forceinline__ int cta_of(const Plan &p, long long tile) {
  return (int)(((tile + 1) * p.ctas - 1) / p.total);
}

// len_b, checked: negative, or more than the table's pages hold.
__device__ __forceinline__ int length(const Args &a, int b) {
  const int n = __ldg(a.lens + b);
  const long long most = (long long)a.max_pages << a.page_log2;
  if (n < 0 || n > most) {
    set_error(a.err, kErrIndex);
    return n < 0 ? 0 : (int)most;
  }
  return n;
}

// Sums the sequences' tiles over the block: `before` is what comes before this thread's
// own run of sequences [b0, b1), `total` all of them.  kN threads; two barriers.
template <int kN>
__device__ __forceinline__ void scan_tiles(const Args &a, int tile, int &b0, int &b1, long long &before,
                                           long long &mine, long long &total, long long *sh) {
  const int per = (a.batch + kN - 1) / kN;
  b0 = min(a.batch, (int)threadIdx.x * per);
  b1 = min(a.batch, b0 + per);
  mine = 0;
  for (int b = b0; b < b1; ++b) mine += (length(a, b) + tile - 1) / tile;
  mine *= (long long)a.Hkv * a.row_tiles;
  long long x = mine;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) sh[warp] = x;
  __syncthreads();
  before = x - mine;
  total = 0;
#pragma unroll
  for (int w = 0; w < kN / 32; ++w) {
    if (w < warp) before += sh[w];
    total += sh[w];
  }
  __syncthreads();
}

// A place in the row of key tiles.
struct Cursor {
  int b, unit, tile, tiles, len;   // unit: head * row_tiles + row tile
};
__device__ __forceinline__ void step(const Args &a, Cursor &c, int tile) {
  if (++c.tile < c.tiles) return;
  c.tile = 0;
  if (++c.unit < a.Hkv * a.row_tiles) return;
  c.unit = 0;
  do {
    if (++c.b >= a.batch) return;   // past the end: not used any more
    c.len = length(a, c.b);
    c.tiles = (c.len + tile - 1) / tile;
  } while (c.tiles == 0);
}

template <int D, bool kF8>
__global__ void __launch_bounds__(kThreads)
paged_attention_kernel(const Args a) {
  using C = Cfg<D, kF8>;
  constexpr int kCh = C::kChunks, kNB = C::kKW / 16, kSteps = D / 16, kNT = D / 8;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long sh_sum[kWarps];
  __shared__ int sh_b;
  __shared__ long long sh_off;
  __shared__ float sh_m[kWarps][kRows], sh_l[kWarps][kRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint8_t *ring = smem + warp * (C::kStages * C::kStage);
  float *merge = reinterpret_cast<float *>(smem + kWarps * C::kStages * C::kStage);
  pdl_wait();
  pdl_trigger();   // the join's blocks wait beside this kernel's, which are all resident by then

  // ---- this block's run of tiles
  Plan plan;
  {
    int b0, b1;
    long long before, mine;
    scan_tiles<kThreads>(a, C::kTile, b0, b1, before, mine, plan.total, sh_sum);
    plan.ctas = (int)min((long long)gridDim.x, plan.total);
    if ((int)blockIdx.x >= plan.ctas) return;
    const long long at = first_tile(plan, blockIdx.x);
    if (at >= before && at < before + mine) {
      const long long per_tile = (long long)a.Hkv * a.row_tiles;
      for (int b = b0; b < b1; ++b) {
        const long long n = (long long)((length(a, b) + C::kTile - 1) / C::kTile) * per_tile;
        if (at < before + n) {
          sh_b = b;
          sh_off = at - before;
          break;
        }
        before += n;
      }
    }
    __syncthreads();
  }
  const int n_tiles = (int)(first_tile(plan, blockIdx.x + 1) - first_tile(plan, blockIdx.x));
  Cursor cur;
  cur.b = sh_b;
  cur.len = length(a, cur.b);
  cur.tiles = (cur.len + C::kTile - 1) / C::kTile;
  cur.unit = (int)(sh_off / cur.tiles);
  cur.tile = (int)(sh_off % cur.tiles);

  // ---- the ring: `ahead` is the next tile to load; the page of this lane's key in it is
  // read one tile before its use
  Cursor ahead = cur;
  int loaded = 0;
  const int krow = lane & (C::kKW - 1);
  auto page_of = [&](const Cursor &c) -> int {
    const int key = c.tile * C::kTile + warp * C::kKW + krow;
    if (key >= c.len) return -1;
    const int p = __ldg(a.table + (size_t)c.b * a.max_pages + (key >> a.page_log2));
    if (p < 0 || p >= a.n_pages) {
      set_error(a.err, kErrIndex);
      return -1;
    }
    return p;
  };
  int page = page_of(ahead);
  unsigned ks_byte = 127, vs_byte = 127;   // of the tile loaded last, not yet in its stage
  auto put_scales = [&]() {
    if (kF8 && loaded > 0 && lane < C::kKW) {
      *reinterpret_cast<float2 *>(ring + ((loaded - 1) % C::kStages) * C::kStage + 2 * C::kHalf +
                                  8 * lane) =
          make_float2(__uint_as_float(ks_byte ? ks_byte << 23 : 0x00400000u),
                      (float)((int)vs_byte - 127));
    }
  };
  auto load_tile = [&]() {
    put_scales();
    if (loaded < n_tiles) {
      const int key = ahead.tile * C::kTile + warp * C::kKW + krow;
      const int slot = page < 0 ? -1 : (page << a.page_log2) + (key & ((1 << a.page_log2) - 1));
      const int h = ahead.unit / a.row_tiles;
      const uint32_t dst = smem_addr(ring + (loaded % C::kStages) * C::kStage);
      if (kF8) {
        ks_byte = vs_byte = 127;
        if (slot >= 0 && lane < C::kKW) {
          ks_byte = a.ks[(size_t)slot * a.Hkv + h];
          vs_byte = a.vs[(size_t)slot * a.Hkv + h];
        }
      }
#pragma unroll
      for (int i = 0; i < C::kKW * kCh / 32; ++i) {
        const int e = 32 * i + lane, row = e / kCh, c = e % kCh;
        const int s = __shfl_sync(0xffffffffu, slot, row);
        const size_t at = ((size_t)max(s, 0) * a.Hkv + h) * C::kRowBytes + 16 * c;
        copy16(dst + row * C::kRowBytes + 16 * k_chunk<kCh>(c, row), a.k + at, s >= 0);
        copy16(dst + C::kHalf + row * C::kRowBytes + 16 * v_chunk<kCh>(c, row), a.v + at, s >= 0);
      }
      ++loaded;
      if (loaded < n_tiles) {
        step(a, ahead, C::kTile);
        page = page_of(ahead);
      }
    } else if (kF8) {
      loaded = -1;   // the last tile's scales are in place
    }
    commit();
  };
#pragma unroll
  for (int s = 0; s < C::kStages - 1; ++s)
    if (loaded >= 0) load_tile();
    else commit();

  // ---- per unit state
  uint32_t qf[kSteps][4];
  float o[kNT][4], m[2], l[2], c2[2];
  int limit[2];          // keys that rows g and g + 8 see
  int unit_tile0 = 0;    // the unit's tile that this run of it starts with
  bool fresh = true;
  bool first_unit = true;

  for (int it = 0; it < n_tiles; ++it) {
    if (fresh) {
      fresh = false;
      unit_tile0 = cur.tile;
      const int h = cur.unit / a.row_tiles, r0 = (cur.unit % a.row_tiles) * kRows;
      float big[2] = {0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        // dimensions of K = 16 step s that this lane's K fragments hold
        const int d = kF8 ? 16 * (t + 4 * (s / 4)) + 4 * (s % 4) : 8 * (t + 4 * (s / 2)) + 4 * (s % 2);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = r0 + g + 8 * e;
          uint2 w = make_uint2(0u, 0u);
          if (r < a.rows) {
            const int i = r / a.G, head = h * a.G + r % a.G;
            w = __ldg(reinterpret_cast<const uint2 *>(
                a.q + ((size_t)((size_t)cur.b * a.n_new + i) * a.Hq + head) * D + d));
          }
          qf[s][e] = w.x;
          qf[s][2 + e] = w.y;
          if (kF8)
            big[e] = fmaxf(fmaxf(big[e], fmaxf(fabsf(lo_bf16(w.x)), fabsf(hi_bf16(w.x)))),
                           fmaxf(fabsf(lo_bf16(w.y)), fabsf(hi_bf16(w.y))));
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = r0 + g + 8 * e;
        limit[e] = r < a.rows ? cur.len - a.n_new + r / a.G + 1 : 0;
        m[e] = kLowest;
        l[e] = 0.f;
        c2[e] = a.scale_log2;
        if (kF8) {
          // the row times 2^(14 - E), its largest magnitude in [2^14, 2^15)
          big[e] = fmaxf(big[e], __shfl_xor_sync(0xffffffffu, big[e], 1));
          big[e] = fmaxf(big[e], __shfl_xor_sync(0xffffffffu, big[e], 2));
          const unsigned E = max(__float_as_uint(big[e]) >> 23, 20u);   // biased
          const float f = __uint_as_float((268u - E) << 23);
          c2[e] *= __uint_as_float((E - 14u) << 23);
#pragma unroll
          for (int s = 0; s < kSteps; ++s) {
            qf[s][e] = pack_f16(lo_bf16(qf[s][e]) * f, hi_bf16(qf[s][e]) * f);
            qf[s][2 + e] = pack_f16(lo_bf16(qf[s][2 + e]) * f, hi_bf16(qf[s][2 + e]) * f);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < kNT; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    }

    wait_all_but<C::kStages - 2>();
    __syncwarp();
    if (loaded >= 0) load_tile();
    else commit();

    const int key0 = cur.tile * C::kTile + warp * C::kKW;
    if (key0 < cur.len) {
      const uint32_t sk = smem_addr(ring + (it % C::kStages) * C::kStage);
      const uint32_t sv = sk + C::kHalf;
      const float2 *scales = reinterpret_cast<const float2 *>(ring + (it % C::kStages) * C::kStage +
                                                              2 * C::kHalf);
      // ---- scores: column n of block q is key 8 q + key_of(n)
      float s[2 * kNB][4];
#pragma unroll
      for (int q = 0; q < 2 * kNB; ++q) {
        s[q][0] = s[q][1] = s[q][2] = s[q][3] = 0.f;
        const int row = 8 * q + key_of<kCh>(g);
#pragma unroll
        for (int i = 0; i < kCh / 4; ++i) {
          const uint4 w = lds128(sk + row * C::kRowBytes + 16 * k_chunk<kCh>(t + 4 * i, row));
          if (kF8) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              mma<true>(s[q], qf[(4 * i + e) % kSteps], f16x2_of_e4m3x2(word(w, e)),
                        f16x2_of_e4m3x2(word(w, e) >> 16));
          } else {
            mma<false>(s[q], qf[(2 * i) % kSteps], w.x, w.y);
            mma<false>(s[q], qf[(2 * i + 1) % kSteps], w.z, w.w);
          }
        }
      }
      // ---- log2 units, the mask, the running maximum
      float vinv[2 * kNB][2], mx[2] = {m[0], m[1]};
      const bool ragged = key0 + C::kKW > cur.len - a.n_new + 1;
#pragma unroll
      for (int q = 0; q < 2 * kNB; ++q) {
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int row = 8 * q + key_of<kCh>(2 * t + n);
          float kf = 1.f, ve = 0.f;
          if (kF8) {
            const float2 f = scales[row];
            kf = f.x, ve = f.y, vinv[q][n] = fast_exp2(-ve);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float &x = s[q][2 * e + n];
            x = kF8 ? fmaf(x * kf, c2[e], ve) : x * c2[e];
            if (ragged && key0 + row >= limit[e]) x = -INFINITY;
            mx[e] = fmaxf(mx[e], x);
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
        mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
      }
      if (__any_sync(0xffffffffu, mx[0] != m[0] || mx[1] != m[1])) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float f = fast_exp2(m[e] - mx[e]);
          m[e] = mx[e];
          l[e] *= f;
#pragma unroll
          for (int n = 0; n < kNT; ++n) o[n][2 * e] *= f, o[n][2 * e + 1] *= f;
        }
      }
      // ---- probabilities, in place
      const float shift[2] = {kF8 ? m[0] - kPShift : m[0], kF8 ? m[1] - kPShift : m[1]};
#pragma unroll
      for (int q = 0; q < 2 * kNB; ++q)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            float &x = s[q][2 * e + n];
            x = fast_exp2(x - shift[e]);
            l[e] = kF8 ? fmaf(x, vinv[q][n], l[e]) : l[e] + x;
          }
      // ---- O += P V, 16 keys at a time
#pragma unroll
      for (int blk = 0; blk < kNB; ++blk) {
        uint32_t p[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          p[e] = kF8 ? pack_f16(s[2 * blk][2 * e], s[2 * blk][2 * e + 1])
                     : pack_bf16(s[2 * blk][2 * e], s[2 * blk][2 * e + 1]);
          p[2 + e] = kF8 ? pack_f16(s[2 * blk + 1][2 * e], s[2 * blk + 1][2 * e + 1])
                         : pack_bf16(s[2 * blk + 1][2 * e], s[2 * blk + 1][2 * e + 1]);
        }
        // This lane's V rows: the keys of MMA rows 2t, 2t+1, 2t+8, 2t+9.  vf[n] holds
        // dimension E g + n (+ 64 for n >= 8 in bf16) of them, E = kNT or 8.
        uint32_t vf[kNT][2];
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const int ra = 16 * blk + 8 * hi + key_of<kCh>(2 * t);
          const int rb = 16 * blk + 8 * hi + key_of<kCh>(2 * t + 1);
          const uint32_t pa = sv + ra * C::kRowBytes, pb = sv + rb * C::kRowBytes;
          if (kF8) {
            uint32_t wa[4] = {0, 0, 0, 0}, wb[4] = {0, 0, 0, 0};
            if (D == 128) {
              const uint4 x = lds128(pa + 16 * v_chunk<kCh>(g, ra)), y = lds128(pb + 16 * v_chunk<kCh>(g, rb));
              wa[0] = x.x, wa[1] = x.y, wa[2] = x.z, wa[3] = x.w;
              wb[0] = y.x, wb[1] = y.y, wb[2] = y.z, wb[3] = y.w;
            } else {
              const uint2 x = lds64(pa + 16 * v_chunk<kCh>(g >> 1, ra) + 8 * (g & 1));
              const uint2 y = lds64(pb + 16 * v_chunk<kCh>(g >> 1, rb) + 8 * (g & 1));
              wa[0] = x.x, wa[1] = x.y, wb[0] = y.x, wb[1] = y.y;
            }
#pragma unroll
            for (int w = 0; w < kNT / 4; ++w) {
              const uint32_t u = __byte_perm(wa[w], wb[w], 0x5140), v = __byte_perm(wa[w], wb[w], 0x7362);
              vf[4 * w][hi] = f16x2_of_e4m3x2(u);
              vf[4 * w + 1][hi] = f16x2_of_e4m3x2(u >> 16);
              vf[4 * w + 2][hi] = f16x2_of_e4m3x2(v);
              vf[4 * w + 3][hi] = f16x2_of_e4m3x2(v >> 16);
            }
          } else {
#pragma unroll
            for (int half = 0; half < kNT / 8; ++half) {
              const uint4 x = lds128(pa + 16 * v_chunk<kCh>(g + 8 * half, ra));
              const uint4 y = lds128(pb + 16 * v_chunk<kCh>(g + 8 * half, rb));
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                vf[8 * half + 2 * w][hi] = __byte_perm(word(x, w), word(y, w), 0x5410);
                vf[8 * half + 2 * w + 1][hi] = __byte_perm(word(x, w), word(y, w), 0x7632);
              }
            }
          }
        }
        // A key that some of the rows may not see must not reach them by 0 * NaN: where a
        // value among the newest keys is not finite, each token's rows take the product
        // with the keys behind their own as zeros.
        bool apart = false;
        if (ragged && a.n_new > 1) {
          bool odd = false;
          constexpr uint32_t kExp = kF8 ? 0x7c00u : 0x7f80u;
#pragma unroll
          for (int n = 0; n < kNT; ++n)
#pragma unroll
            for (int hi = 0; hi < 2; ++hi)
              odd |= (vf[n][hi] & kExp) == kExp || (vf[n][hi] >> 16 & kExp) == kExp;
          apart = __any_sync(0xffffffffu, odd);
        }
        if (!apart) {
#pragma unroll
          for (int n = 0; n < kNT; ++n) mma<kF8>(o[n], p, vf[n][0], vf[n][1]);
        } else {
          const int r0 = (cur.unit % a.row_tiles) * kRows;
          const int i1 = (min(a.rows, r0 + kRows) - 1) / a.G;
          for (int i = r0 / a.G; i <= i1; ++i) {
            const int lim = cur.len - a.n_new + i + 1;
            uint32_t pi[4];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const bool mine = limit[e] == lim && r0 + g + 8 * e < a.rows;
              pi[e] = mine ? p[e] : 0u;
              pi[2 + e] = mine ? p[2 + e] : 0u;
            }
            uint32_t keep[2];
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
              const int k = key0 + 16 * blk + 8 * hi;
              keep[hi] = (k + key_of<kCh>(2 * t) < lim ? 0xffffu : 0u) |
                         (k + key_of<kCh>(2 * t + 1) < lim ? 0xffff0000u : 0u);
            }
            // rows of the other tokens take nothing, not 0 * NaN: their sums stand aside
#pragma unroll
            for (int n = 0; n < kNT; ++n) {
              float x[4] = {0.f, 0.f, 0.f, 0.f};
              mma<kF8>(x, pi, vf[n][0] & keep[0], vf[n][1] & keep[1]);
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (limit[e] == lim && r0 + g + 8 * e < a.rows) {
                  o[n][2 * e] += x[2 * e];
                  o[n][2 * e + 1] += x[2 * e + 1];
                }
            }
          }
        }
      }
    }

    const bool unit_done = cur.tile + 1 == cur.tiles;
    if (unit_done || it + 1 == n_tiles) {
      // ---- the unit's end, or the run's: the four warps' parts become one in warp 0
      const int r0 = (cur.unit % a.row_tiles) * kRows, h = cur.unit / a.row_tiles;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 1);
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
        if (t == 0) {
          sh_m[warp][g + 8 * e] = m[e];
          sh_l[warp][g + 8 * e] = l[e];
        }
      }
      __syncthreads();
      float M[2], sum[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        M[e] = sh_m[0][g + 8 * e];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) M[e] = fmaxf(M[e], sh_m[w][g + 8 * e]);
        sum[e] = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w)
          sum[e] += sh_l[w][g + 8 * e] * fast_exp2(sh_m[w][g + 8 * e] - M[e]);
        const float f = fast_exp2(m[e] - M[e]);
#pragma unroll
        for (int n = 0; n < kNT; ++n) o[n][2 * e] *= f, o[n][2 * e + 1] *= f;
      }
      // lane-major: each lane adds the same lane's sums of another warp; the buffer holds
      // one warp's O, or halves of two
      auto at = [&](int n) { return reinterpret_cast<float4 *>(merge) + n * 32 + lane; };
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int base = (warp & 1) * (kNT / 2);
        if (warp >= 2) {
#pragma unroll
          for (int n = 0; n < kNT / 2; ++n) {
            const float(&x)[4] = o[half * (kNT / 2) + n];
            *at(base + n) = make_float4(x[0], x[1], x[2], x[3]);
          }
        }
        __syncthreads();
        if (warp < 2) {
#pragma unroll
          for (int n = 0; n < kNT / 2; ++n) {
            const float4 x = *at(base + n);
            float(&y)[4] = o[half * (kNT / 2) + n];
            y[0] += x.x, y[1] += x.y, y[2] += x.z, y[3] += x.w;
          }
        }
        __syncthreads();
      }
      if (warp == 1) {
#pragma unroll
        for (int n = 0; n < kNT; ++n) *at(n) = make_float4(o[n][0], o[n][1], o[n][2], o[n][3]);
      }
      __syncthreads();
      if (warp == 0) {
#pragma unroll
        for (int n = 0; n < kNT; ++n) {
          const float4 x = *at(n);
          o[n][0] += x.x, o[n][1] += x.y, o[n][2] += x.z, o[n][3] += x.w;
        }
        const bool whole = unit_tile0 == 0 && unit_done;
        float *part = a.ws + (size_t)(2 * blockIdx.x + (first_unit ? 0 : 1)) * (kRows * (D + 2));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int rr = g + 8 * e, r = r0 + rr;
          if (r >= a.rows) continue;
          const float inv = sum[e] > 0.f ? 1.f / sum[e] : sum[e] == 0.f ? 0.f : sum[e];
          __nv_bfloat16 *dst = a.out + ((size_t)((size_t)cur.b * a.n_new + r / a.G) * a.Hq + h * a.G + r % a.G) * D;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            // columns 2t + j of all n: neighbouring dimensions
            constexpr int kE = kF8 ? kNT : 8;
#pragma unroll
            for (int n0 = 0; n0 < kNT; n0 += 8) {
              const int d = kE * (2 * t + j) + (kE == 8 ? 8 * n0 : n0);
              if (whole) {
                uint4 w;
                w.x = pack_bf16(o[n0][2 * e + j] * inv, o[n0 + 1][2 * e + j] * inv);
                w.y = pack_bf16(o[n0 + 2][2 * e + j] * inv, o[n0 + 3][2 * e + j] * inv);
                w.z = pack_bf16(o[n0 + 4][2 * e + j] * inv, o[n0 + 5][2 * e + j] * inv);
                w.w = pack_bf16(o[n0 + 6][2 * e + j] * inv, o[n0 + 7][2 * e + j] * inv);
                *reinterpret_cast<uint4 *>(dst + d) = w;
              } else {
                float4 *f = reinterpret_cast<float4 *>(part + rr * D + d);
                f[0] = make_float4(o[n0][2 * e + j], o[n0 + 1][2 * e + j], o[n0 + 2][2 * e + j], o[n0 + 3][2 * e + j]);
                f[1] = make_float4(o[n0 + 4][2 * e + j], o[n0 + 5][2 * e + j], o[n0 + 6][2 * e + j], o[n0 + 7][2 * e + j]);
              }
            }
          }
          if (!whole && t == 0) {
            part[kRows * D + 2 * rr] = M[e];
            part[kRows * D + 2 * rr + 1] = sum[e];
          }
        }
      }
      first_unit = false;
      fresh = true;
    }
    if (it + 1 < n_tiles) step(a, cur, C::kTile);
  }
  wait_all_but<0>();
}

// Joins the parts of each output row whose unit several blocks shared, and stores zeros
// for sequences without keys.  One block per (sequence, K/V head, row); a warp takes
// every eighth part, D/4 lanes a part's four-dimension vectors.
constexpr int kJoinThreads = 256;
constexpr int kJoinWarps = kJoinThreads / 32;

template <int D>
__global__ void __launch_bounds__(kJoinThreads)
paged_join_kernel(const Args a, int tile, int grid) {
  __shared__ long long sh_sum[kJoinWarps];
  __shared__ long long sh_before;
  __shared__ float sh_red[kJoinWarps];
  __shared__ float4 sh_o[kJoinThreads];
  __shared__ float sh_l[kJoinThreads / (D / 4)];
  pdl_wait();
  pdl_trigger();
  const int r = blockIdx.x % a.rows, h = blockIdx.x / a.rows % a.Hkv;
  const int b = blockIdx.x / a.rows / a.Hkv;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Plan plan;
  {
    int b0, b1;
    long long before, mine;
    scan_tiles<kJoinThreads>(a, tile, b0, b1, before, mine, plan.total, sh_sum);
    if (b >= b0 && b < b1) {
      for (int x = b0; x < b; ++x)
        before += (long long)((length(a, x) + tile - 1) / tile) * a.Hkv * a.row_tiles;
      sh_before = before;
    }
    __syncthreads();
  }
  plan.ctas = (int)min((long long)grid, plan.total);
  const int tiles = (length(a, b) + tile - 1) / tile;
  __nv_bfloat16 *dst =
      a.out + ((size_t)((size_t)b * a.n_new + r / a.G) * a.Hq + h * a.G + r % a.G) * D;
  if (tiles == 0) {
    if (threadIdx.x < D / 8) reinterpret_cast<uint4 *>(dst)[threadIdx.x] = make_uint4(0, 0, 0, 0);
    return;
  }
  const long long t0 = sh_before + (long long)(h * a.row_tiles + r / kRows) * tiles;
  const int c0 = cta_of(plan, t0), c1 = cta_of(plan, t0 + tiles - 1);
  if (c0 == c1) return;   // stored by its block
  const int parts = c1 - c0 + 1, rr = r % kRows;
  const int slot0 = first_tile(plan, c0) == t0 ? 2 * c0 : 2 * c0 + 1;
  auto part = [&](int p) {
    return a.ws + (size_t)(p ? 2 * (c0 + p) : slot0) * (kRows * (D + 2));
  };
  float M = kLowest;
  for (int p = threadIdx.x; p < parts; p += kJoinThreads) M = fmaxf(M, part(p)[kRows * D + 2 * rr]);
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (lane == 0) sh_red[warp] = M;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) M = fmaxf(M, sh_red[w]);
  constexpr int kL = D / 4;                 // lanes per part
  const int sub = threadIdx.x % kL, at = threadIdx.x / kL;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
#pragma unroll 4
  for (int p = at; p < parts; p += kJoinThreads / kL) {
    const float *w = part(p);
    const float2 ml = *reinterpret_cast<const float2 *>(w + kRows * D + 2 * rr);
    const float4 x = *reinterpret_cast<const float4 *>(w + rr * D + 4 * sub);
    const float f = fast_exp2(ml.x - M);
    sum = fmaf(f, ml.y, sum);
    acc.x = fmaf(f, x.x, acc.x);
    acc.y = fmaf(f, x.y, acc.y);
    acc.z = fmaf(f, x.z, acc.z);
    acc.w = fmaf(f, x.w, acc.w);
  }
  sh_o[threadIdx.x] = acc;
  if (sub == 0) sh_l[at] = sum;
  __syncthreads();
  if (threadIdx.x < kL) {
    float total = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kJoinThreads / kL; ++i) {
      const float4 x = sh_o[i * kL + threadIdx.x];
      acc.x += x.x, acc.y += x.y, acc.z += x.z, acc.w += x.w;
      total += sh_l[i];
    }
    const float inv = total > 0.f ? 1.f / total : total == 0.f ? 0.f : total;
    reinterpret_cast<uint2 *>(dst)[threadIdx.x] =
        make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  }
}

// -------------------------------------------------------------- host side

template <int D, bool kF8>
int launch(const Args &a, size_t ws_bytes, cudaStream_t stream) {
  using C = Cfg<D, kF8>;
  auto kernel = paged_attention_kernel<D, kF8>;
  static std::atomic<int> per_sm[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return HSA_ERR_CUDA;
  int nb = per_sm[dev].load(std::memory_order_acquire);
  if (nb <= 0) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) !=
            cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&nb, kernel, kThreads, C::kSmem) !=
            cudaSuccess ||
        nb < 1)
      return HSA_ERR_CUDA;
    nb = std::min(nb, kMaxPerSm);
    per_sm[dev].store(nb, std::memory_order_release);
  }
  const long long units = (long long)a.batch * a.Hkv * a.row_tiles;
  const long long most = units * ((((long long)a.max_pages << a.page_log2) + C::kTile - 1) / C::kTile);
  const int grid = (int)std::min<long long>((long long)nb * sm_count(), std::max(1LL, most));
  if ((size_t)grid * 2 * kRows * (D + 2) * 4 > ws_bytes) return HSA_ERR_WORKSPACE;
  count_launches(2);
  launch_pdl(kernel, dim3((unsigned)grid), dim3(kThreads), C::kSmem, stream, a);
  if (cudaGetLastError() != cudaSuccess) return HSA_ERR_CUDA;
  launch_pdl(paged_join_kernel<D>, dim3((unsigned)(a.batch * a.Hkv * a.rows)), dim3(kJoinThreads), 0,
             stream, a, (int)C::kTile, grid);
  return launch_status();
}

}  // namespace
}  // namespace hsa

using namespace hsa;

extern "C" size_t hsa_paged_attention_workspace_bytes(int batch, int n_new, int Hq, int Hkv, int D) {
  if (batch <= 0 || n_new <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv || (D != 64 && D != 128)) return 0;
  return (size_t)sm_count() * kMaxPerSm * 2 * kRows * (D + 2) * 4;
}

extern "C" int hsa_paged_attention(const void *q, int batch, int n_new, int Hq, const void *k_pages,
                                   const void *v_pages, const uint8_t *k_scale,
                                   const uint8_t *v_scale, int n_pages, int page_size, int Hkv, int D,
                                   hsa_dtype cache_dtype, const int32_t *page_table, int max_pages,
                                   const int32_t *seq_lens, float scale, void *out, void *workspace,
                                   size_t workspace_bytes, hsa_stream_t stream) {
  if (batch < 0 || n_new < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv || n_pages < 0 || max_pages < 0 ||
      page_size < 1)
    return HSA_ERR_INVALID_ARG;
  if (cache_dtype != HSA_BF16 && cache_dtype != HSA_F32 && cache_dtype != HSA_E4M3)
    return HSA_ERR_INVALID_ARG;
  if (cache_dtype == HSA_F32 || (D != 64 && D != 128) || (page_size & (page_size - 1)))
    return HSA_ERR_UNSUPPORTED;
  const long long rows = (long long)n_new * (Hq / Hkv);
  if ((long long)n_pages * page_size > 0x7fffffffLL || (long long)max_pages * page_size > 0x7fffff00LL ||
      Hq > 65535 || rows > 0x7fffffffLL || (long long)batch * Hkv * rows > 0x7fffffffLL)
    return HSA_ERR_UNSUPPORTED;
  if (batch == 0 || n_new == 0) return HSA_OK;
  if (!q || !out || !seq_lens || !aligned16(q) || !aligned16(out)) return HSA_ERR_INVALID_ARG;
  const bool f8 = cache_dtype == HSA_E4M3;
  if (n_pages > 0 && max_pages > 0 &&
      (!k_pages || !v_pages || !page_table || (f8 && (!k_scale || !v_scale)) ||
       !aligned16(k_pages) || !aligned16(v_pages)))
    return HSA_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace)) return HSA_ERR_WORKSPACE;
  if (!(scale > 0.f) || !std::isfinite(scale)) scale = 1.f / std::sqrt((float)D);
  Args a;
  a.q = static_cast<const __nv_bfloat16 *>(q);
  a.k = static_cast<const uint8_t *>(k_pages);
  a.v = static_cast<const uint8_t *>(v_pages);
  a.ks = k_scale;
  a.vs = v_scale;
  a.table = page_table;
  a.lens = seq_lens;
  a.out = static_cast<__nv_bfloat16 *>(out);
  a.ws = static_cast<float *>(workspace);
  a.err = device_error_word();
  if (!a.err) return HSA_ERR_CUDA;
  a.batch = batch;
  a.n_new = n_new;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = Hq / Hkv;
  a.rows = (int)rows;
  a.row_tiles = (int)((rows + kRows - 1) / kRows);
  a.n_pages = n_pages;
  a.max_pages = n_pages > 0 ? max_pages : 0;
  a.page_log2 = 0;
  while ((1 << a.page_log2) < page_size) ++a.page_log2;
  a.scale_log2 = scale * 1.4426950408889634f;
  cudaStream_t s = (cudaStream_t)stream;
  if (f8) return D == 128 ? launch<128, true>(a, workspace_bytes, s) : launch<64, true>(a, workspace_bytes, s);
  return D == 128 ? launch<128, false>(a, workspace_bytes, s) : launch<64, false>(a, workspace_bytes, s);
}

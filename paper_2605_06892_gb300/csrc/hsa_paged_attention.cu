// Attention of a few new tokens per sequence over a paged KV cache, bf16 or 8-bit:
//   o[b, i, h] = sum_j softmax_j(scale <q[b,i,h], k_j>) v_j,  j < len_b - n_new + i + 1,
// with k, v of the head that h's group shares.  A few FLOPs per byte of cache, so what
// bounds it is reading the cache once.
//
// Work split.  A unit is (sequence, K/V head, up to 8 kNR query rows); its rows are the
// group's heads of all new tokens, row r = i G + g, so that one pass over the keys serves
// the whole group.  The units' key tiles, laid end to end, are cut into equal runs, one per
// CTA and as many CTAs as are resident: sequences of any mix of lengths keep every SM busy
// to the end.  A run that holds a whole unit stores its rows; the others leave (M, l, O) in
// the workspace and the join kernel merges them.
//
// In a CTA each of four warps takes its own kKW keys of a tile, with its own running
// maximum, its own ring of cp.async stages and no CTA barrier until the unit's end; the
// ring runs on across units.  The products are m16n8k16 MMAs with the keys (and the head's
// dimensions) as the 16 rows and the query rows as the 8 columns: S^T = K Q^T and O^T = V^T
// P^T.  Eight rows are what one token of a group has, a sixteenth of the 128-row tile of
// the tcgen05 form, so nothing is computed for rows that are not there; more rows take kNR
// column blocks that share the K and V fragments.  The fragments come straight from 16-byte
// shared loads: the order of the head's dimensions inside a product and of the keys inside
// a tile is free, so each lane multiplies what lies together (column orders below), without
// transposing loads; P^T is transposed on its way by movmatrix.
//
// 8-bit cache.  A key's e4m3 codes are exact in fp16, and so is a bf16 query row after
// scaling by a power of two (its values below 2^-31 of the largest aside: those are rounded,
// by 2^-39 of the largest at most), so the products are exact and the key's 2^ks multiplies
// the score.  The value's 2^vs goes into the probability: with t_j the score in log2 units, R
// within 64 of max t_j, u_j = t_j - R + vs_j and M = max u_j,
//   o = 2^M sum_j 2^(u_j - M) code_j / sum_j 2^(t_j - R).
// No factor 2^(u_j - M) exceeds 1.  The weights' sum has a reference of its own: relative to
// that of the other sum it would lie between 2^-120 and 2^100 n, since vs does within
// [-100, 120] (-127 in rows of fresh memory), and long stretches of zero rows would overflow
// it.  All else is relative to R, so that scores of any size lose nothing beside vs.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "hsa_paged.cuh"

namespace hsa {
namespace {

__device__ __forceinline__ uint32_t f16x2_of_e4m3x2(uint32_t codes16) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes16));
  return h;
}

template <int D, bool kF8, int kNR>
struct Cfg {
  static constexpr int kRows = 8 * kNR;                        // query rows of a unit
  static constexpr int kRowBytes = D * (kF8 ? 1 : 2);
  static constexpr int kChunks = kRowBytes / 16;               // 16-byte chunks per row
  // Four column blocks at D = 128 leave no registers for the query rows, which are then
  // read from shared memory at each product.
  static constexpr bool kLean = D == 128 && kNR == 4;
  static_assert(!(kLean && kF8), "the rows in shared memory are bf16");
  static constexpr int kKW = kRowBytes == 256 ? 16 : 32;       // keys per warp and tile
  static constexpr int kTile = kWarps * kKW;                   // keys per tile
  static constexpr int kStages = 2;
  static constexpr int kBlocks = kNR == 1 ? (D == 64 ? 4 : 3) : 2;   // per SM: registers
  static constexpr int kHalf = kKW * kRowBytes;                // K (or V) bytes of a stage
  static constexpr int kScales = kF8 ? kKW * 16 : 0;           // per key four words
  static constexpr int kStage = 2 * kHalf + kScales;
  static constexpr int kQ = kRows * D * 2;                     // a unit's query rows
  static constexpr int kStat = part_stats(kF8);
  static constexpr int kPart = part_floats(D, kF8, kRows);
  static constexpr int kSmem = kWarps * kStages * kStage + kStages * kQ;
};

// The key (row of an 8-key block) of MMA index n.  The 16-byte loads of K (a quarter-warp:
// keys of n = 2x, 2x+1; four chunks) and of V (keys of n = 0, 2, 4, 6 or 1, 3, 5, 7; two
// chunks) then fall into distinct banks under the swizzles below.
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

// Where a query row's dimensions of K = 16 step s lie in shared memory that lane t of a
// quad multiplies: those that its K fragments hold (chunk c of row r lies at c ^ (r & 7)).
template <int D, bool kF8>
__device__ __forceinline__ int query_place(int r, int s, int t) {
  const int d = kF8 ? 16 * (t + 4 * (s / 4)) + 4 * (s % 4) : 8 * (t + 4 * (s / 2)) + 4 * (s % 2);
  return r * (2 * D) + 16 * ((d / 8) ^ (r & 7)) + (d & 4) * 2;
}

// The products of a warp's keys of a tile at sk with the query rows: MMA row n (n + 8) of block
// b is key 16 b + key_of(n) (+ 8).  rows(step, x): this lane's part of column block x.
template <int D, bool kF8, int kNR, typename Rows>
__device__ __forceinline__ void score_tile(uint32_t sk, int g, int t,
                                           float (&s)[Cfg<D, kF8, kNR>::kKW / 16][kNR][4],
                                           Rows &&rows) {
  using C = Cfg<D, kF8, kNR>;
  constexpr int kCh = C::kChunks;
#pragma unroll
  for (int b = 0; b < C::kKW / 16; ++b) {
#pragma unroll
    for (int x = 0; x < kNR; ++x) s[b][x][0] = s[b][x][1] = s[b][x][2] = s[b][x][3] = 0.f;
    const int row = 16 * b + key_of<kCh>(g);
#pragma unroll
    for (int i = 0; i < kCh / 4; ++i) {
      const uint32_t at = 16 * k_chunk<kCh>(t + 4 * i, row);   // the same for row + 8
      const uint4 w0 = lds128(sk + row * C::kRowBytes + at);
      const uint4 w1 = lds128(sk + (row + 8) * C::kRowBytes + at);
#pragma unroll
      for (int e = 0; e < (kF8 ? 4 : 2); ++e) {
        uint32_t k[4];
        if (kF8) {
          k[0] = f16x2_of_e4m3x2(word(w0, e)), k[2] = f16x2_of_e4m3x2(word(w0, e) >> 16);
          k[1] = f16x2_of_e4m3x2(word(w1, e)), k[3] = f16x2_of_e4m3x2(word(w1, e) >> 16);
        } else {
          k[0] = word(w0, 2 * e), k[2] = word(w0, 2 * e + 1);
          k[1] = word(w1, 2 * e), k[3] = word(w1, 2 * e + 1);
        }
#pragma unroll
        for (int x = 0; x < kNR; ++x) {
          const uint2 q = rows((kF8 ? 4 : 2) * i + e, x);
          mma<kF8>(s[b][x], k, q.x, q.y);
        }
      }
    }
  }
}

// 8 bits: R is zero to begin with.  Where scores are beyond +-64 of it, so that a lane's sum
// leaves the range that holds all that counts, the warp takes the tile again, here, against the
// largest score so far.
template <int D, int kNR>
__device__ __noinline__ void take_again(CodeTile<D, kNR> &z, uint32_t sk, const uint4 *scales,
                                        bool first) {
  using C = Cfg<D, true, kNR>;
  constexpr int kCh = C::kChunks;
  static_assert(C::kKW == 32, "two blocks of 16 keys");
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  score_tile<D, true, kNR>(sk, g, t, z.s, [&](int step, int x) { return z.q[step][x]; });
#pragma unroll 1
  for (int x = 0; x < kNR; ++x) {
    uint64_t score[4];
    float top[2], l[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)   // at least the sum so far, which is then 1 at most
      top[j] = first ? kLowest : fmaxf(z.ref[x][j], z.ref[x][j] + __log2f(z.l[x][j]));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + key_of<kCh>(g);
      score[i] = mul2(code_product(z.s[i >> 1][x], i & 1, z.before[x], scales[row]),
                      both(z.after[x][0], z.after[x][1]));
      if (row < z.limit[x][0]) top[0] = fmaxf(top[0], lo_f(score[i]));
      if (row < z.limit[x][1]) top[1] = fmaxf(top[1], hi_f(score[i]));
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int d = 4; d < 32; d <<= 1)
        top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], d));
      const float down = z.ref[x][j] - top[j];
      l[j] = first ? 0.f : z.l[x][j] * fast_exp2(down);
      z.m[x][j] = first ? kLowest : fmaxf(z.m[x][j] + down, kLowest);
      z.mx[x][j] = z.m[x][j];
      z.ref[x][j] = top[j];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + key_of<kCh>(g);
      const float ve = __uint_as_float(scales[row].z);
      const float d[2] = {lo_f(score[i]) - top[0], hi_f(score[i]) - top[1]};
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const bool seen = row < z.limit[x][j];
        const float u = seen ? d[j] + ve : -INFINITY;
        if (seen) l[j] += fast_exp2(d[j]);
        z.s[i >> 1][x][2 * (i & 1) + j] = u;
        z.mx[x][j] = fmaxf(z.mx[x][j], u);
      }
    }
    z.l[x][0] = l[0], z.l[x][1] = l[1];
  }
}

template <int D, bool kF8, int kNR>
__global__ void __launch_bounds__(kThreads, (Cfg<D, kF8, kNR>::kBlocks))
paged_attention_kernel(const PagedArgs a) {
  using C = Cfg<D, kF8, kNR>;
  constexpr int kCh = C::kChunks, kNB = C::kKW / 16, kSteps = D / 16, kNT = D / 8, kMT = D / 16;
  constexpr int kRows = C::kRows;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int sh_sum[kWarps], sh_at[3];
  __shared__ float sh_m[kWarps][kRows], sh_l[kWarps][kRows], sh_r[kF8 ? kWarps : 1][kRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint8_t *ring = smem + warp * (C::kStages * C::kStage);
  pdl_wait();
  pdl_trigger();   // the join's blocks wait beside this kernel's, which are all resident by then

  // ---- this block's run of tiles: thread x counts those of a run of sequences, and the
  // one whose sequences the block's first tile falls into says where
  Plan plan;
  {
    const int per = (a.batch + kThreads - 1) / kThreads;
    const int b0 = min(a.batch, (int)threadIdx.x * per), b1 = min(a.batch, b0 + per);
    const int per_tile = a.Hkv * a.row_tiles;
    int first_len = 0, mine = 0;
    for (int b = b0; b < b1; ++b) {
      const int n = length(a, b);
      if (b == b0) first_len = n;
      mine += (n + C::kTile - 1) / C::kTile * per_tile;
    }
    int end = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, end, o);
      if (lane >= o) end += y;
    }
    if (lane == 31) sh_sum[warp] = end;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) end += sh_sum[w];
      total += sh_sum[w];
    }
    plan = plan_of(total, gridDim.x, a.sms);
    if (total == 0 || (int)blockIdx.x >= plan.ctas) {
      if (threadIdx.x == 0) a.cuts[blockIdx.x].parts = 0;
      clear_empty<D>(a);
      return;
    }
    const int at = first_tile(plan, blockIdx.x);
    if (at >= end - mine && at < end) {
      int before = end - mine, len = first_len;
      for (int b = b0;; len = length(a, ++b)) {
        const int n = (len + C::kTile - 1) / C::kTile * per_tile;
        if (at < before + n) {
          sh_at[0] = b;
          sh_at[1] = len;
          sh_at[2] = at - before;
          break;
        }
        before += n;
      }
    }
    __syncthreads();
  }
  const int n_tiles = first_tile(plan, blockIdx.x + 1) - first_tile(plan, blockIdx.x);
  Cursor cur;
  cur.b = sh_at[0];
  cur.len = sh_at[1];
  cur.tiles = (cur.len + C::kTile - 1) / C::kTile;
  cur.unit = sh_at[2] / cur.tiles;
  cur.tile = sh_at[2] - cur.unit * cur.tiles;
  CutUnit cut = {};

  // ---- the ring: `ahead` is the next tile to load; the pages of this lane's keys in it are
  // read one tile before their use, and looked at only then
  Cursor ahead = cur;
  int left = n_tiles;                       // tiles to load
  uint32_t fill = 0;                        // where the next one goes: offset of its stage
  constexpr int kStep = 32 / kCh;           // rows that a warp copies at a time
  const int krow = lane & (C::kKW - 1);
  const uint32_t ring_s = smem_addr(ring);
  const unsigned row_stride = a.Hkv * C::kRowBytes;
  // this lane's chunk of rows lane / kCh + kStep i, in K's order and in V's; the swizzles
  // repeat after eight rows
  uint32_t to_k[kStep < 8 ? 8 / kStep : 1], to_v[kStep < 8 ? 8 / kStep : 1];
#pragma unroll
  for (int i = 0; i < (kStep < 8 ? 8 / kStep : 1); ++i) {
    const int row = lane / kCh + kStep * i;
    to_k[i] = row * C::kRowBytes + 16 * k_chunk<kCh>(lane % kCh, row);
    to_v[i] = row * C::kRowBytes + 16 * v_chunk<kCh>(lane % kCh, row) + C::kHalf;
  }
  int page;
  auto look_up = [&]() {
    const int key = ahead.tile * C::kTile + warp * C::kKW + krow;
    page = -1;
    if (key < ahead.len)
      page = __ldg(a.table + (size_t)ahead.b * a.max_pages + (key >> a.page_log2));
  };
  look_up();
  int q_fill = 0, q_now = 0;                // buffers of the next unit's rows, and of this one's
  uint8_t *sq = smem + kWarps * C::kStages * C::kStage;
  auto load_tile = [&]() {
    if (left > 0) {
      const int h = ahead.unit / a.row_tiles;
      if (ahead.tile == 0 || left == n_tiles) {
        // The unit's query rows come with its first tile here, a chunk or more per thread:
        // rows past the last are zeros.  Chunk c of row r lies at c ^ (r & 7).
        const int r0 = (ahead.unit - h * a.row_tiles) * kRows;
        const uint32_t to = smem_addr(sq + q_fill * C::kQ);
#pragma unroll
        for (int e0 = 0; e0 < kRows * (D / 8); e0 += kThreads) {
          const int e = e0 + threadIdx.x, r = e / (D / 8), c = e % (D / 8);
          if (kRows * (D / 8) % kThreads != 0 && e >= kRows * (D / 8)) break;
          const bool ok = r0 + r < a.rows;
          const int i = ok ? quotient(r0 + r, a.group) : 0;
          const int head = h * (int)a.group.d + (ok ? r0 + r - i * (int)a.group.d : 0);
          copy16(to + r * (2 * D) + 16 * (c ^ (r & 7)),
                 a.q + (((size_t)ahead.b * a.n_new + i) * a.Hq + head) * D + 8 * c, ok);
        }
        q_fill = q_fill + 1 == C::kStages ? 0 : q_fill + 1;
      }
      const int key = ahead.tile * C::kTile + warp * C::kKW + krow;
      const bool ok = page >= 0 && page < a.n_pages;
      if (!ok && key < ahead.len) set_error(a.err, kErrIndex);
      const int slot = ok ? (page << a.page_log2) + (key & ((1 << a.page_log2) - 1)) : 0;
      const unsigned have = __ballot_sync(0xffffffffu, ok);   // rows that there are
      if (kF8 && lane < C::kKW) {
        // The aligned words around the key's scale bytes, and the bytes' place in them: the
        // bytes need not be waited for here.  A word that holds a byte of the scales can be
        // read whole, whatever the other three are.  No page: a row of zeros, times one.
        const size_t at = (size_t)slot * a.Hkv + h;
        const uintptr_t ks = (uintptr_t)(a.ks + at), vs = (uintptr_t)(a.vs + at);
        uint32_t *to = reinterpret_cast<uint32_t *>(ring + fill + 2 * C::kHalf) + 4 * lane;
        if (ok) {
          copy4(smem_addr(to), (const void *)(ks & ~(uintptr_t)3));
          copy4(smem_addr(to + 1), (const void *)(vs & ~(uintptr_t)3));
        } else {
          to[0] = to[1] = 0x7f7f7f7fu;
        }
        to[2] = (uint32_t)(ks & 3) * 8 + ((uint32_t)(vs & 3) * 8 << 16);
      }
      const uint8_t *kb = a.k + (size_t)h * C::kRowBytes + 16 * (lane % kCh);
      const uint8_t *vb = a.v + (size_t)h * C::kRowBytes + 16 * (lane % kCh);
#pragma unroll
      for (int i = 0; i < C::kKW / kStep; ++i) {
        constexpr int kCycle = kStep < 8 ? 8 / kStep : 1;
        const int row = lane / kCh + kStep * i;
        const unsigned at = __shfl_sync(0xffffffffu, slot, row);
        const bool there = have >> row & 1;
        const uint32_t dst = ring_s + fill + (i / kCycle) * (kCycle * kStep * C::kRowBytes);
        copy16(dst + to_k[i % kCycle], kb + (uint64_t)at * row_stride, there);
        copy16(dst + to_v[i % kCycle], vb + (uint64_t)at * row_stride, there);
      }
      fill = fill + C::kStage == C::kStages * C::kStage ? 0 : fill + C::kStage;
      if (--left > 0) {
        step(a, ahead, C::kTile);
        look_up();
      }
    }
    commit();
  };
#pragma unroll
  for (int s = 0; s < C::kStages - 1; ++s) load_tile();

  // ---- per unit state; column block x of the MMAs holds rows 8 x .. 8 x + 7, and this
  // lane row 8 x + g of Q^T and P^T, rows 8 x + 2 t + j of S^T and O^T
  constexpr bool kLean = C::kLean;
  uint32_t qf[kLean ? 1 : kSteps][kNR][2];
  float o[kMT][kNR][4], m[kNR][2], l[kNR][2];
  // 8 bits: a query row's power of two times the scale's, in two factors, and its R; rows 2 t
  // and 2 t + 1 go together through packed instructions
  float before[kF8 ? kNR : 1][2], after[kF8 ? kNR : 1][2], ref[kF8 ? kNR : 1][2];
  uint32_t sq_now = 0;   // kLean: the unit's rows
  int unit_tile0 = 0;    // the unit's tile that this run of it starts with
  bool fresh = true, first_unit = true;
  bool first = true;     // this warp has none of the unit's keys yet
  uint32_t now = 0;      // the stage of tile `it`

  for (int it = 0; it < n_tiles; ++it) {
    wait_all_but<C::kStages - 2>();
    if (fresh) __syncthreads();   // the query rows are every thread's copies
    else __syncwarp();
    load_tile();

    if (fresh) {
      fresh = false;
      first = true;
      unit_tile0 = cur.tile;
      const uint32_t from = smem_addr(sq + q_now * C::kQ);
      q_now = q_now + 1 == C::kStages ? 0 : q_now + 1;
      sq_now = from;
      // 8 bits: a row times 2^(14 - E), its largest magnitude in [2^14, 2^15); `big` over the
      // lanes that hold the row
      auto scales_of = [&](float big, float &f) {
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const unsigned E = max(__float_as_uint(big) >> 23, 20u);   // biased
        f = __uint_as_float((268u - E) << 23);
        return __uint_as_float((E - 14u) << 23);
      };
      auto larger = [](float big, uint32_t w) {
        return fmaxf(big, fmaxf(fabsf(lo_bf16(w)), fabsf(hi_bf16(w))));
      };
      auto scaled = [](uint32_t w, float f) { return pack_f16(lo_bf16(w) * f, hi_bf16(w) * f); };
#pragma unroll
      for (int x = 0; x < kNR; ++x) {
        float scale = 0.f;
        if constexpr (!kLean) {
          const int r = 8 * x + g;
          float big = 0.f, f;
#pragma unroll
          for (int s = 0; s < kSteps; ++s) {
            const uint2 w = lds64(from + query_place<D, kF8>(r, s, t));
            qf[s][x][0] = w.x;
            qf[s][x][1] = w.y;
            if (kF8) big = larger(larger(big, w.x), w.y);
          }
          if (kF8) {
            scale = scales_of(big, f);
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
              for (int y = 0; y < 2; ++y) qf[s][x][y] = scaled(qf[s][x][y], f);
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (kF8) {
            // A product y stands for y 2^ks c, c a power of two: multiplied in this order, with
            // c first where it is below 1 and last else, it overflows only where the product of
            // query and key does, whatever their sizes.
            const float c = __shfl_sync(0xffffffffu, scale, 4 * (2 * t + j));
            before[kF8 ? x : 0][j] = fminf(c, 1.f);
            after[kF8 ? x : 0][j] = fminf(fmaxf(c, 1.f) * a.scale_power, 0x1p127f);
            ref[kF8 ? x : 0][j] = 0.f;
          }
          m[x][j] = kLowest;
          l[x][j] = 0.f;
        }
#pragma unroll
        for (int n = 0; n < kMT; ++n) o[n][x][0] = o[n][x][1] = o[n][x][2] = o[n][x][3] = 0.f;
      }
    }

    const int key0 = cur.tile * C::kTile + warp * C::kKW;
    if (key0 < cur.len) {
      const uint32_t sk = ring_s + now, sv = sk + C::kHalf;
      uint4 *scales = reinterpret_cast<uint4 *>(ring + now + 2 * C::kHalf);
      if (kF8) {
        // each lane makes 2^ks, times the scale's digits, and vs of its key's scale bytes
        // (within [27, 247], or 0), each twice
        if (lane < C::kKW) {
          const uint4 w = scales[lane];
          const uint32_t ks = w.x >> (w.z & 0xffffu) & 255u, vs = w.y >> (w.z >> 16) & 255u;
          const uint32_t ve = __float_as_uint((float)((int)vs - 127));
          const uint32_t kf = __float_as_uint(__uint_as_float(ks << 23) * a.scale_digits);
          scales[lane] = make_uint4(kf, kf, ve, ve);
        }
        __syncwarp();
      }
      const bool ragged = key0 + C::kKW > cur.len - a.n_new + 1;
      // keys that row 8 x + 2 t + j sees, where that matters
      auto limit = [&](int x, int j) {
        return cur.len - a.n_new + 1 +
               (int)quotient((cur.unit % a.row_tiles) * kRows + 8 * x + 2 * t + j, a.group);
      };
      float s[kNB][kNR][4], mx[kNR][2], sum[kF8 ? kNR : 1][2];
      if constexpr (kLean)
        score_tile<D, kF8, kNR>(sk, g, t, s, [&](int step, int x) {
          return lds64(sq_now + query_place<D, kF8>(8 * x + g, step, t));
        });
      else
        score_tile<D, kF8, kNR>(sk, g, t, s, [&](int step, int x) {
          return make_uint2(qf[step][x][0], qf[step][x][1]);
        });
      // ---- log2 units, the mask, the running maximum; in 8 bits the weights' sum as well
#pragma unroll
      for (int x = 0; x < kNR; ++x) {
        mx[x][0] = m[x][0], mx[x][1] = m[x][1];
        if constexpr (kF8) sum[x][0] = l[x][0], sum[x][1] = l[x][1];
      }
      auto weigh = [&](auto masked) {
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const int row = 16 * b + 8 * n + key_of<kCh>(g);
            if constexpr (kF8) {
              const uint4 w = scales[row];
#pragma unroll
              for (int x = 0; x < kNR; ++x) {
                const uint64_t z =
                    fma2(code_product(s[b][x], n, before[x], w), both(after[x][0], after[x][1]),
                         both(-ref[x][0], -ref[x][1]));
                const uint64_t u = add2(z, pack2(w.z, w.w));
                float &y0 = s[b][x][2 * n], &y1 = s[b][x][2 * n + 1];
                float e0 = fast_exp2(lo_f(z)), e1 = fast_exp2(hi_f(z));
                y0 = lo_f(u), y1 = hi_f(u);
                if (decltype(masked)::value) {
                  if (key0 + row >= limit(x, 0)) y0 = -INFINITY, e0 = 0.f;
                  if (key0 + row >= limit(x, 1)) y1 = -INFINITY, e1 = 0.f;
                }
                const uint64_t w2 = add2(both(sum[x][0], sum[x][1]), both(e0, e1));
                sum[x][0] = lo_f(w2), sum[x][1] = hi_f(w2);
                mx[x][0] = fmaxf(mx[x][0], y0), mx[x][1] = fmaxf(mx[x][1], y1);
              }
            } else {
#pragma unroll
              for (int x = 0; x < kNR; ++x)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                  const bool seen = !decltype(masked)::value || key0 + row < limit(x, j);
                  float &y = s[b][x][2 * n + j];
                  y = seen ? __fmul_rn(y, a.scale_log2) : -INFINITY;
                  mx[x][j] = fmaxf(mx[x][j], y);
                }
            }
          }
      };
      if (!ragged) weigh(std::false_type());
      else weigh(std::true_type());
      if constexpr (kF8) {
        // Out of line, so that what is rare costs the usual path no registers.
        float most = 0.f;
#pragma unroll
        for (int x = 0; x < kNR; ++x) most = max3f(most, sum[x][0], sum[x][1]);
        bool far = most > kFar;
        if (first) {
#pragma unroll
          for (int x = 0; x < kNR; ++x)
#pragma unroll
            for (int j = 0; j < 2; ++j) far |= sum[x][j] < 1.f / kFar && mx[x][j] > kLowest;
        }
        if (__any_sync(0xffffffffu, far)) {
          CodeTile<D, kNR> z;
#pragma unroll
          for (int x = 0; x < kNR; ++x) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
              z.q[i][x] = make_uint2(qf[kLean ? 0 : i][x][0], qf[kLean ? 0 : i][x][1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              z.before[x][j] = before[x][j], z.after[x][j] = after[x][j];
              z.limit[x][j] = ragged ? limit(x, j) - key0 : C::kKW;
              z.ref[x][j] = ref[x][j], z.l[x][j] = l[x][j], z.m[x][j] = m[x][j];
            }
          }
          take_again<D, kNR>(z, sk, scales, first);
#pragma unroll
          for (int x = 0; x < kNR; ++x) {
#pragma unroll
            for (int b = 0; b < kNB; ++b)
#pragma unroll
              for (int i = 0; i < 4; ++i) s[b][x][i] = z.s[b][x][i];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              ref[x][j] = z.ref[x][j], sum[x][j] = z.l[x][j];
              m[x][j] = z.m[x][j], mx[x][j] = z.mx[x][j];
            }
          }
        }
        first = false;
      }
      bool moved = false;
#pragma unroll
      for (int x = 0; x < kNR; ++x)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1)
            mx[x][j] = fmaxf(mx[x][j], __shfl_xor_sync(0xffffffffu, mx[x][j], d));
          moved |= mx[x][j] != m[x][j];
        }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int x = 0; x < kNR; ++x)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float f = fast_exp2(m[x][j] - mx[x][j]);
            m[x][j] = mx[x][j];
            if (!kF8) l[x][j] *= f;
#pragma unroll
            for (int n = 0; n < kMT; ++n) o[n][x][j] *= f, o[n][x][2 + j] *= f;
          }
      }
      if constexpr (kF8) {
#pragma unroll
        for (int x = 0; x < kNR; ++x) l[x][0] = sum[x][0], l[x][1] = sum[x][1];
      }
      // ---- probabilities, as the 16 x 8 B operand of O^T += V^T P^T.  They are rounded to the
      // 16 bits that the MMA takes: bf16 beside bf16 values, and fp16 beside 8-bit ones, which
      // are exact in it and leave the probabilities three bits more.  Each is off by half a
      // step at most (2^-8 or 2^-11 of itself), up or down, and an output by no more than that
      // of its row's sum of |p v|; the sum l takes them unrounded, which adds nothing to it.
      // In fp16 those with u more than 28 below M lose further bits, and more than 39 below
      // they are zero.
      uint32_t p[kNB][kNR][2];
#pragma unroll
      for (int b = 0; b < kNB; ++b)
#pragma unroll
        for (int x = 0; x < kNR; ++x)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            float y[2];
            if constexpr (kF8) {
              const uint64_t z = add2(both(s[b][x][2 * n], s[b][x][2 * n + 1]),
                                      both(kPShift - m[x][0], kPShift - m[x][1]));
              y[0] = fast_exp2(lo_f(z)), y[1] = fast_exp2(hi_f(z));
            } else {
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                y[j] = fast_exp2(s[b][x][2 * n + j] - m[x][j]);
                l[x][j] += y[j];
              }
            }
            p[b][x][n] = transposed(kF8 ? pack_f16(y[0], y[1]) : pack_bf16(y[0], y[1]));
          }
      // ---- O^T += V^T P^T, 16 keys at a time
#pragma unroll
      for (int b = 0; b < kNB; ++b) {
        // This lane's V rows: the keys of MMA indices 2t, 2t+1 (+ 8).  vf[n][hi] holds their
        // values of dimension E g + n (bf16: + 56 for n >= 8), E = kNT in 8 bits, else 8.
        uint32_t vf[kNT][2];
#pragma unroll
        for (int hi = 0; hi < 2; ++hi) {
          const int ra = 16 * b + 8 * hi + key_of<kCh>(2 * t);
          const int rb = 16 * b + 8 * hi + key_of<kCh>(2 * t + 1);
          const uint32_t pa = sv + ra * C::kRowBytes, pb = sv + rb * C::kRowBytes;
          if (kF8) {
            uint32_t wa[4] = {0, 0, 0, 0}, wb[4] = {0, 0, 0, 0};
            if (D == 128) {
              const uint4 y = lds128(pa + 16 * v_chunk<kCh>(g, ra));
              const uint4 z = lds128(pb + 16 * v_chunk<kCh>(g, rb));
              wa[0] = y.x, wa[1] = y.y, wa[2] = y.z, wa[3] = y.w;
              wb[0] = z.x, wb[1] = z.y, wb[2] = z.z, wb[3] = z.w;
            } else {
              const uint2 y = lds64(pa + 16 * v_chunk<kCh>(g >> 1, ra) + 8 * (g & 1));
              const uint2 z = lds64(pb + 16 * v_chunk<kCh>(g >> 1, rb) + 8 * (g & 1));
              wa[0] = y.x, wa[1] = y.y, wb[0] = z.x, wb[1] = z.y;
            }
#pragma unroll
            for (int w = 0; w < kNT / 4; ++w) {
              const uint32_t y = __byte_perm(wa[w], wb[w], 0x5140);
              const uint32_t z = __byte_perm(wa[w], wb[w], 0x7362);
              vf[4 * w][hi] = f16x2_of_e4m3x2(y);
              vf[4 * w + 1][hi] = f16x2_of_e4m3x2(y >> 16);
              vf[4 * w + 2][hi] = f16x2_of_e4m3x2(z);
              vf[4 * w + 3][hi] = f16x2_of_e4m3x2(z >> 16);
            }
          } else {
#pragma unroll
            for (int half = 0; half < kNT / 8; ++half) {
              const uint4 y = lds128(pa + 16 * v_chunk<kCh>(g + 8 * half, ra));
              const uint4 z = lds128(pb + 16 * v_chunk<kCh>(g + 8 * half, rb));
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                vf[8 * half + 2 * w][hi] = __byte_perm(word(y, w), word(z, w), 0x5410);
                vf[8 * half + 2 * w + 1][hi] = __byte_perm(word(y, w), word(z, w), 0x7632);
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
          for (int n = 0; n < kMT; ++n) {
            const uint32_t v[4] = {vf[2 * n][0], vf[2 * n + 1][0], vf[2 * n][1], vf[2 * n + 1][1]};
#pragma unroll
            for (int x = 0; x < kNR; ++x) mma<kF8>(o[n][x], v, p[b][x][0], p[b][x][1]);
          }
        } else {
          const int r0 = (cur.unit % a.row_tiles) * kRows;
          const int i1 = (min(a.rows, r0 + kRows) - 1) / (int)a.group.d;
          for (int i = r0 / (int)a.group.d; i <= i1; ++i) {
            const int lim = cur.len - a.n_new + i + 1;
            uint32_t keep[2];
#pragma unroll
            for (int hi = 0; hi < 2; ++hi) {
              const int k = key0 + 16 * b + 8 * hi;
              keep[hi] = (k + key_of<kCh>(2 * t) < lim ? 0xffffu : 0u) |
                         (k + key_of<kCh>(2 * t + 1) < lim ? 0xffff0000u : 0u);
            }
            // the other tokens' sums stand aside: they take nothing, not 0 * NaN
#pragma unroll
            for (int n = 0; n < kMT; ++n) {
              const uint32_t v[4] = {vf[2 * n][0] & keep[0], vf[2 * n + 1][0] & keep[0],
                                     vf[2 * n][1] & keep[1], vf[2 * n + 1][1] & keep[1]};
#pragma unroll
              for (int x = 0; x < kNR; ++x) {
                float y[4] = {0.f, 0.f, 0.f, 0.f};
                mma<kF8>(y, v, p[b][x][0], p[b][x][1]);
#pragma unroll
                for (int j = 0; j < 2; ++j)
                  if (limit(x, j) == lim && r0 + 8 * x + 2 * t + j < a.rows) {
                    o[n][x][j] += y[j];
                    o[n][x][2 + j] += y[2 + j];
                  }
              }
            }
          }
        }
      }
    }

    const bool unit_done = cur.tile + 1 == cur.tiles;
    if (unit_done || it + 1 == n_tiles) {
      // ---- the unit's end, or the run's: the four warps' parts become one.  Each leaves its
      // sums in the stage that it has just read, lane by lane, and takes a quarter of the
      // dimensions of all four.  The stage is filled again only after the barrier that
      // starts the next unit.
      const int h = cur.unit / a.row_tiles, r0 = (cur.unit - h * a.row_tiles) * kRows;
#pragma unroll
      for (int x = 0; x < kNR; ++x)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[x][j] += __shfl_xor_sync(0xffffffffu, l[x][j], d);
          if (g == 0) {
            sh_m[warp][8 * x + 2 * t + j] = m[x][j];
            sh_l[warp][8 * x + 2 * t + j] = l[x][j];
            if constexpr (kF8) sh_r[warp][8 * x + 2 * t + j] = l[x][j] == 0.f ? kLowest : ref[x][j];
          }
        }
      __syncwarp();   // every lane has read the stage
      constexpr int kQuarter = kMT / kWarps;                // MMA blocks of 16 dimensions
      constexpr int kFit = C::kStage / (kMT * 512);         // column blocks whose sums fit
      constexpr int kAt = kFit < 1 ? 0 : kFit < kNR ? kFit : kNR;
      static_assert(kAt > 0 && kNR % kAt == 0, "a stage takes the sums of a column block");
      const bool whole = unit_tile0 == 0 && unit_done;
      float *part = a.ws + (size_t)(2 * blockIdx.x + (first_unit ? 0 : 1)) * C::kPart;
#pragma unroll
      for (int x0 = 0; x0 < kNR; x0 += kAt) {
        if (x0) __syncthreads();
#pragma unroll
        for (int n = 0; n < kMT; ++n)
#pragma unroll
          for (int x = 0; x < kAt; ++x) {
            const float(&y)[4] = o[n][x0 + x];
            reinterpret_cast<float4 *>(ring + now)[(n * kAt + x) * 32 + lane] =
                make_float4(y[0], y[1], y[2], y[3]);
          }
        __syncthreads();
#pragma unroll
        for (int x = x0; x < x0 + kAt; ++x) {
          float f[2][kWarps], M[2], R[2], sum[2];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int r = 8 * x + 2 * t + j;
            // 8 bits: the warps' M relative to the largest R
            R[j] = 0.f;
            if constexpr (kF8) {
              R[j] = sh_r[0][r];
#pragma unroll
              for (int w = 1; w < kWarps; ++w) R[j] = fmaxf(R[j], sh_r[w][r]);
            }
            auto level = [&](int w) {
              return kF8 ? sh_r[kF8 ? w : 0][r] - R[j] + sh_m[w][r] : sh_m[w][r];
            };
            M[j] = level(0);
#pragma unroll
            for (int w = 1; w < kWarps; ++w) M[j] = fmaxf(M[j], level(w));
            sum[j] = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
              f[j][w] = fast_exp2(level(w) - M[j]);
              sum[j] = fmaf(sh_l[w][r], kF8 ? fast_exp2(sh_r[kF8 ? w : 0][r] - R[j]) : f[j][w],
                            sum[j]);
            }
          }
          float y[kQuarter][4];
#pragma unroll
          for (int n = 0; n < kQuarter; ++n) {
            y[n][0] = y[n][1] = y[n][2] = y[n][3] = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
              const float4 z =
                  reinterpret_cast<const float4 *>(smem + w * (C::kStages * C::kStage) + now)
                      [((warp * kQuarter + n) * kAt + x - x0) * 32 + lane];
              y[n][0] = fmaf(z.x, f[0][w], y[n][0]), y[n][1] = fmaf(z.y, f[1][w], y[n][1]);
              y[n][2] = fmaf(z.z, f[0][w], y[n][2]), y[n][3] = fmaf(z.w, f[1][w], y[n][3]);
            }
          }
          // block n holds dimensions E g + 2 n and the next (bf16: + 56 from n = 4 on)
          constexpr int kE = kF8 ? kNT : 8;
          const int n0 = warp * kQuarter;
          const int d = kE * g + (kE == 8 ? (n0 / 4) * 64 + 2 * (n0 % 4) : 2 * n0);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int rr = 8 * x + 2 * t + j, r = r0 + rr;
            if (r >= a.rows) continue;
            if (whole) {
              const RowEnd<kF8> end(sum[j], M[j] - kPShift);
              const int i = quotient(r, a.group);
              __nv_bfloat16 *dst = a.out + ((size_t)((size_t)cur.b * a.n_new + i) * a.Hq +
                                            h * (int)a.group.d + (r - i * (int)a.group.d)) * D + d;
              uint32_t w[kQuarter];
#pragma unroll
              for (int n = 0; n < kQuarter; ++n)
                w[n] = pack_bf16(end(y[n][j]), end(y[n][2 + j]));
              if constexpr (kQuarter == 2)
                *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[kQuarter - 1]);
              else
                *reinterpret_cast<uint32_t *>(dst) = w[0];
            } else {
#pragma unroll
              for (int n = 0; n < kQuarter; ++n)
                *reinterpret_cast<float2 *>(part + rr * D + d + 2 * n) =
                    make_float2(y[n][j], y[n][2 + j]);
              if (warp == 0 && g == 0) {
                float *stat = part + kRows * D + C::kStat * rr;
                stat[0] = M[j];
                stat[1] = sum[j];
                if (kF8) stat[2] = R[j];
              }
            }
          }
        }
      }
      if (unit_done && !whole) {   // a run ends one such unit at most: its first
        const int t0 = first_tile(plan, blockIdx.x) - unit_tile0;
        const int c0 = cta_of(plan, t0);
        cut.parts = blockIdx.x - c0 + 1;
        cut.first = c0;
        cut.slot = first_tile(plan, c0) == t0 ? 2 * c0 : 2 * c0 + 1;
        cut.b = cur.b;
        cut.unit = cur.unit;
      }
      first_unit = false;
      fresh = true;
    }
    now = now + C::kStage == C::kStages * C::kStage ? 0 : now + C::kStage;
    if (it + 1 < n_tiles) step(a, cur, C::kTile);
  }
  wait_all_but<0>();
  if (threadIdx.x == 0) a.cuts[blockIdx.x] = cut;
  clear_empty<D>(a);
}

// -------------------------------------------------------------- host side

template <int D, bool kF8, int kNR>
int launch(PagedArgs &a, void *workspace, cudaStream_t stream) {
  using C = Cfg<D, kF8, kNR>;
  auto kernel = paged_attention_kernel<D, kF8, kNR>;
  static std::atomic<int> per_sm[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return HSA_ERR_CUDA;
  int nb = per_sm[dev].load(std::memory_order_acquire);
  if (nb <= 0) {
    // Both kernels ask for the same split between L1 and shared memory: a call that starts
    // beside the join of the call before would otherwise find the join's, with room for
    // half of its blocks, until the SM is empty (its blocks then start in two rounds).
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) !=
            cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout,
                             cudaSharedmemCarveoutMaxShared) != cudaSuccess ||
        cudaFuncSetAttribute(paged_join_kernel<D, kF8, kNR>,
                             cudaFuncAttributePreferredSharedMemoryCarveout,
                             cudaSharedmemCarveoutMaxShared) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&nb, kernel, kThreads, C::kSmem) !=
            cudaSuccess ||
        nb < 1)
      return HSA_ERR_CUDA;
    nb = std::min(nb, kMaxPerSm);
    per_sm[dev].store(nb, std::memory_order_release);
  }
  a.row_tiles = (a.rows + C::kRows - 1) / C::kRows;
  const long long units = (long long)a.batch * a.Hkv * a.row_tiles;
  const long long tiles = (((long long)a.max_pages << a.page_log2) + C::kTile - 1) / C::kTile;
  if (units * tiles > 0x7fffffffLL) return HSA_ERR_UNSUPPORTED;   // tiles are counted in 32 bits
  const int blocks = nb * sm_count();
  const int grid = (int)std::min<long long>(blocks, tiles ? units * tiles : a.batch);
  a.cuts = static_cast<CutUnit *>(workspace);
  a.ws = reinterpret_cast<float *>(a.cuts + (size_t)sm_count() * kMaxPerSm);
  count_launches(2);
  launch_pdl(kernel, dim3((unsigned)grid), dim3(kThreads), C::kSmem, stream, a);
  if (cudaGetLastError() != cudaSuccess) return HSA_ERR_CUDA;
  launch_pdl(paged_join_kernel<D, kF8, kNR>,
             dim3((unsigned)grid, (unsigned)std::min(a.rows, C::kRows)), dim3(kJoinThreads), 0,
             stream, a);
  return launch_status();
}

// Column blocks of eight rows per unit: one or two where the rows fit, else two or four.
// Further units read the keys again, from L2, and by then the products bound the time: a
// unit of four blocks takes 1.6 to 1.7 times one of two (4 sequences of 9000 to 30000 keys,
// 8 K/V heads: 24 rows 48 against 57 us at D = 64, 82 against 99 at D = 128; 40 rows 77
// against 75, 143 against 135; 24 rows at D = 64 in 8 bits 55 against 66).  8-bit keys at
// D = 128 leave it too few registers (24 rows, with the sum of the weights relative to the
// probabilities' maximum, 84 against 73 us).
template <int D, bool kF8>
int launch_rows(PagedArgs &a, void *workspace, cudaStream_t stream) {
  if (a.rows <= 8) return launch<D, kF8, 1>(a, workspace, stream);
  if constexpr (!(kF8 && D == 128))
    if (5 * ((a.rows + 31) / 32) < 3 * ((a.rows + 15) / 16))
      return launch<D, kF8, 4>(a, workspace, stream);
  return launch<D, kF8, 2>(a, workspace, stream);
}

}  // namespace
}  // namespace hsa

using namespace hsa;

extern "C" size_t hsa_paged_attention_workspace_bytes(int batch, int n_new, int Hq, int Hkv,
                                                      int D) {
  if (batch <= 0 || n_new <= 0 || Hq <= 0 || Hkv <= 0 || Hq % Hkv) return 0;
  if (D != 64 && D != 128) return 0;
  return workspace_bytes(D);
}

extern "C" int hsa_paged_attention(const void *q, int batch, int n_new, int Hq, const void *k_pages,
                                   const void *v_pages, const uint8_t *k_scale,
                                   const uint8_t *v_scale, int n_pages, int page_size, int Hkv,
                                   int D, hsa_dtype cache_dtype, const int32_t *page_table,
                                   int max_pages, const int32_t *seq_lens, float scale, void *out,
                                   void *workspace, size_t size, hsa_stream_t stream) {
  if (batch < 0 || n_new < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv || n_pages < 0 || max_pages < 0 ||
      page_size < 1)
    return HSA_ERR_INVALID_ARG;
  if (cache_dtype != HSA_BF16 && cache_dtype != HSA_F32 && cache_dtype != HSA_E4M3 &&
      cache_dtype != HSA_E2M1)
    return HSA_ERR_INVALID_ARG;
  if (cache_dtype == HSA_F32 || (D != 64 && D != 128) || (page_size & (page_size - 1)))
    return HSA_ERR_UNSUPPORTED;
  const long long rows = (long long)n_new * (Hq / Hkv);
  if ((long long)n_pages * page_size > 0x7fffffffLL ||
      (long long)max_pages * page_size > 0x7fffff00LL ||
      Hq > 65535 || rows > 0x7fffffffLL || (long long)batch * Hkv * rows > 0x7fffff00LL)
    return HSA_ERR_UNSUPPORTED;
  if (batch == 0 || n_new == 0) return HSA_OK;
  if (!q || !out || !seq_lens || !aligned16(q) || !aligned16(out)) return HSA_ERR_INVALID_ARG;
  const bool f8 = cache_dtype == HSA_E4M3, f4 = cache_dtype == HSA_E2M1;
  if (n_pages > 0 && max_pages > 0 &&
      (!k_pages || !v_pages || !page_table || ((f8 || f4) && (!k_scale || !v_scale)) ||
       !aligned16(k_pages) || !aligned16(v_pages) ||
       (f4 && ((reinterpret_cast<uintptr_t>(k_scale) | reinterpret_cast<uintptr_t>(v_scale)) & 3))))
    return HSA_ERR_INVALID_ARG;
  if (!workspace || !aligned16(workspace) || size < workspace_bytes(D)) return HSA_ERR_WORKSPACE;
  if (!(scale > 0.f) || !std::isfinite(scale)) scale = 1.f / std::sqrt((float)D);
  PagedArgs a;
  a.q = static_cast<const __nv_bfloat16 *>(q);
  a.k = static_cast<const uint8_t *>(k_pages);
  a.v = static_cast<const uint8_t *>(v_pages);
  a.ks = k_scale;
  a.vs = v_scale;
  a.table = page_table;
  a.lens = seq_lens;
  a.out = static_cast<__nv_bfloat16 *>(out);
  a.err = device_error_word();
  if (!a.err) return HSA_ERR_CUDA;
  a.batch = batch;
  a.n_new = n_new;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.group = make_divider((unsigned)(Hq / Hkv));
  a.rows = (int)rows;
  a.row_tiles = 0;
  a.cuts = nullptr;
  a.ws = nullptr;
  a.n_pages = n_pages;
  a.max_pages = n_pages > 0 ? max_pages : 0;
  a.sms = sm_count();
  a.side = 1;
  a.inject_stall = attention_stall();
  a.page_log2 = 0;
  while ((1 << a.page_log2) < page_size) ++a.page_log2;
  a.scale_log2 = scale * 1.4426950408889634f;
  int power = 0;
  a.scale_digits = 2.f * std::frexp(std::min(a.scale_log2, 3.4e38f), &power);   // in [1, 2)
  a.scale_power = std::ldexp(1.f, power - 1);
  cudaStream_t s = (cudaStream_t)stream;
  if (f4) return launch_paged4(a, D, workspace, s);
  if (f8)
    return D == 128 ? launch_rows<128, true>(a, workspace, s)
                    : launch_rows<64, true>(a, workspace, s);
  return D == 128 ? launch_rows<128, false>(a, workspace, s)
                  : launch_rows<64, false>(a, workspace, s);
}

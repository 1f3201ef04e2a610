// Attention of a few new tokens per sequence over a paged 4-bit KV cache.  The work's split, the
// MMAs' roles, the references R and M of the weights' two sums and the join are those of the
// 8-bit kernel (hsa_paged_attention.cu); what a row is (hsa_kv4.cu) makes the rest.
//
// A key row is D e2m1 codes with a factor m_g of six bits for each of four groups of its
// dimensions and a power of two, so a score is
//   2^ks sum_g m_g <q_g, code_g>,
// sums of exact fp16 products over one group each, times the factors in 32 bits.  A value's
// factors go into the probabilities, one group of dimensions after the other: P in fp16 is
// 2^(u - M + 6), at most 2^10 * 63 with a factor (u is 4 above M at most), and its product with
// one is rounded to fp16 again (2^-11 of itself).  Codes and factors are always finite; where a
// row is held as NaN its power is NaN, and so become the scores, or the weights, of the query
// rows that see it and of no others.
//
// The groups interleave (dimension d is of group (d / (D/32)) mod 4): the 16 (D = 64: 8) bytes
// of a key that a lane of a quad multiplies, and the 8 (4) bytes of a value, hold all four in
// equal parts, and MMAs over one group only.
//
// What bounds it is latency.  68 bytes a key and head leave 370 issue slots of an SM's quarter for
// 16 keys of one head at the memory's rate, and decoding (64 conversions and shuffles of bits), 16
// MMAs and the softmax take 292 of them; but three warps a quarter, which is what the registers
// allow, issue once in about five cycles each, and so use half of the slots: what counts is a
// warp's own chain of loads, wait, words, products and softmax.  So what does not grow with the
// bytes is kept small: the tiles come by TMA, a box of a page's rows each, a warp holds 64 keys of a
// tile and takes them 32 at a time, their words wait in registers, and the blocks of a key's heads
// run side by side: their rows and words lie together, and what one block leaves of a line or sector
// the others find in L2 (4 sequences of 95000 keys: 134 -> 112 us).  32 query heads over 8 of D =
// 128: 4 sequences of 95000 keys 90 us, 4.6 TB/s, 0.67 of HBM's measured rate (tiles of 32 keys a
// warp took 8 us more, the two parts of a tile in a loop 4); 48 of 4500 61 us, 0.56; one of 4001
// 10.9 us.
#include <algorithm>
#include <atomic>
#include <cstring>
#include <type_traits>

#include "hsa_paged.cuh"
#include "hsa_tma.cuh"

namespace hsa {
namespace {

constexpr int kKW = 32;                        // keys that a warp takes at a time
constexpr int kParts = 2;                      // parts of a tile's keys of one warp, kKW each
constexpr int kHold = kParts * kKW;
constexpr int kTile = kWarps * kHold;
constexpr float kShift = 6.f;                  // probabilities are 2^(u - M + 6)
constexpr float kSlack = 4.f;                  // u - M at most; then M rises

template <int D, int kNR>
struct Cfg4 {
  static constexpr int kRows = 8 * kNR;        // query rows of a unit
  static constexpr int kRowBytes = D / 2;
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kStages = 2;
  static constexpr int kBlocks = kNR == 1 ? (D == 64 ? 4 : 3) : 2;   // per SM: registers
  static constexpr int kHalf = kHold * kRowBytes;                      // K (or V) bytes of a stage
  static constexpr int kStage = 2 * kHalf;
  static constexpr int kMade = kKW * 40;                             // what kKW keys' words make
  static constexpr int kQ = kRows * D * 2;                           // a unit's query rows
  static constexpr int kPart = part_floats(D, true, kRows);
  static constexpr int kAlign = 512;                                 // the swizzle's period
  static constexpr int kSmem =
      kAlign + kWarps * (kStages * kStage + kMade) + kStages * kQ;
};

// The key (row of an 8-key block) of MMA index n: the pairs 2t, 2t+1 are neighbours, and the
// loads of K (16 bytes of keys 2x, 2x+1 at D = 128; 8 bytes of n = 0 .. 3 or 4 .. 7 at D = 64)
// and of V (8 bytes of n = 0, 2, 4, 6 or 1, 3, 5, 7; 4 bytes) fall into distinct banks.
template <int D>
__device__ __forceinline__ int key_of(int n) {
  return D == 128 ? n ^ (n >> 1 & 1) : n ^ (n >> 2 & 1);
}
// Whether the key in a row has an even MMA index.
template <int D>
__device__ __forceinline__ bool is_even(int row) {
  return (row & 1) == (row >> (D == 128 ? 1 : 2) & 1);
}
// Where chunk c (16 bytes) of row r lies: the 64-byte swizzle of TMA, or as it is.
template <int D>
__device__ __forceinline__ int place(int r, int c) {
  return D == 128 ? r * 64 + 16 * (c ^ (r >> 1 & 3)) : r * 32 + 16 * c;
}

// The values of eight e2m1 codes, in pairs.
__device__ __forceinline__ void f16_of_e2m1x8(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n.reg .b8 a, b, c, e;\n"
      "mov.b32 {a, b, c, e}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n"
      "cvt.rn.f16x2.e2m1x2 %3, e;\n}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
}
// d = a b, 16 rows x 8 columns x 16, fp16.
__device__ __forceinline__ void mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                          uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ void bulk16(uint32_t dst, const void *src, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], 16, [%2];" ::
          "r"(dst), "l"(src), "r"(bar)
      : "memory");
}
// The four dimensions of a query row that lane t of a quad multiplies at step s of K = 16, in
// the order of its K fragments (chunk c of row r lies at c ^ (r & 7)).  A step stays within a
// group: two steps to one at D = 128; at D = 64 it takes two pairs eight dimensions apart.
template <int D>
__device__ __forceinline__ uint2 query_at(uint32_t rows, int r, int s, int t) {
  const int d = D / 4 * t + (D == 128 ? 4 * (s / 2) + 16 * (s % 2) : 2 * s);
  const uint32_t at = rows + r * (2 * D) + 16 * ((d / 8) ^ (r & 7)) + (d & 6) * 2;
  if constexpr (D == 64)
    return make_uint2(lds32(at), lds32(at ^ 16));
  else
    return lds64(at);
}

// The products of a warp's keys of a tile at sk with the query rows: MMA row n (n + 8) of block
// b is key 16 b + key_of(n) (+ 8).  m: the keys' factors, four each.  rows(step, x): this lane's
// part of column block x.
template <int D, int kNR, typename Rows>
__device__ __forceinline__ void score_tile(uint32_t sk, const uint4 *m, int g, int t,
                                           float (&s)[kKW / 16][kNR][4], Rows &&rows) {
#pragma unroll
  for (int b = 0; b < kKW / 16; ++b) {
#pragma unroll
    for (int x = 0; x < kNR; ++x) s[b][x][0] = s[b][x][1] = s[b][x][2] = s[b][x][3] = 0.f;
    const int row = 16 * b + key_of<D>(g);
    const uint4 m0 = m[row], m1 = m[row + 8];
    // words w and w + kW of the lane's part hold the same groups, D / 64 each
    constexpr int kW = D / 64;
    uint32_t k0[2 * kW], k1[2 * kW];
    if constexpr (D == 128) {
      const uint4 y = lds128(sk + place<D>(row, t)), z = lds128(sk + place<D>(row + 8, t));
      k0[0] = y.x, k0[1] = y.y, k0[2 * kW - 2] = y.z, k0[2 * kW - 1] = y.w;
      k1[0] = z.x, k1[1] = z.y, k1[2 * kW - 2] = z.z, k1[2 * kW - 1] = z.w;
    } else {
      const uint2 y = lds64(sk + place<D>(row, 0) + 8 * t);
      const uint2 z = lds64(sk + place<D>(row + 8, 0) + 8 * t);
      k0[0] = y.x, k0[1] = y.y, k1[0] = z.x, k1[1] = z.y;
    }
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      uint32_t h0[2][4], h1[2][4];   // [first or second half of the part][pair]
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        f16_of_e2m1x8(k0[w + kW * half], h0[half]);
        f16_of_e2m1x8(k1[w + kW * half], h1[half]);
      }
#pragma unroll
      for (int e = 0; e < 4 / kW; ++e) {
        const int group = 4 / kW * w + e;
        const float f0 = __uint_as_float(word(m0, group)), f1 = __uint_as_float(word(m1, group));
        float y[kNR][4];
#pragma unroll
        for (int j = 0; j < kW; ++j) {
          // D = 128: the group's four dimensions of one half; D = 64: two of each
          const uint32_t k[4] = {D == 128 ? h0[j][2 * e % 4] : h0[0][e],
                                 D == 128 ? h1[j][2 * e % 4] : h1[0][e],
                                 D == 128 ? h0[j][(2 * e + 1) % 4] : h0[1][e],
                                 D == 128 ? h1[j][(2 * e + 1) % 4] : h1[1][e]};
#pragma unroll
          for (int x = 0; x < kNR; ++x) {
            const uint2 q = rows(kW * group + j, x);
            if (j == 0) mma_first(y[x], k, q.x, q.y);
            else mma<true>(y[x], k, q.x, q.y);
          }
        }
#pragma unroll
        for (int x = 0; x < kNR; ++x) {
          float(&z)[4] = s[b][x];
          z[0] = fmaf(y[x][0], f0, z[0]), z[1] = fmaf(y[x][1], f0, z[1]);
          z[2] = fmaf(y[x][2], f1, z[2]), z[3] = fmaf(y[x][3], f1, z[3]);
        }
      }
    }
  }
}

// O^T += V^T P^T over 16 keys, block b of a tile at sv, with the keys' factors for each group in
// the probabilities (factors: four pairs for each two keys).
template <int D, int kNR>
__device__ __forceinline__ void add_values(float (&o)[D / 16][kNR][4],
                                           const uint32_t (&p)[kNR][2], uint32_t sv,
                                           const uint4 *factors, int b, int g, int t) {
  constexpr int kW = D / 64;   // words of a lane's part of a row
  // A byte holds two dimensions of a key: the low halves of both keys' bytes make a pair of one
  // dimension, the high halves of the next.
  constexpr uint32_t kLow = 0x0f0f0f0fu;
  uint32_t wa[2][kW], wb[2][kW], factor[2][4];
#pragma unroll
  for (int hi = 0; hi < 2; ++hi) {
    const int ra = 16 * b + 8 * hi + key_of<D>(2 * t);
    const int rb = 16 * b + 8 * hi + key_of<D>(2 * t + 1);
    if constexpr (kW == 2) {
      const uint2 y = lds64(sv + place<D>(ra, g >> 1) + 8 * (g & 1));
      const uint2 z = lds64(sv + place<D>(rb, g >> 1) + 8 * (g & 1));
      wa[hi][0] = y.x, wa[hi][1] = y.y, wb[hi][0] = z.x, wb[hi][1] = z.y;
    } else {
      wa[hi][0] = lds32(sv + place<D>(ra, 0) + 4 * g);
      wb[hi][0] = lds32(sv + place<D>(rb, 0) + 4 * g);
    }
    const uint4 f = factors[8 * b + 4 * hi + t];
#pragma unroll
    for (int i = 0; i < 4; ++i) factor[hi][i] = word(f, i);
  }
#pragma unroll
  for (int w = 0; w < kW; ++w) {   // a word: four MMA blocks of 16 dimensions
    uint32_t even[2][4], odd[2][4];
#pragma unroll
    for (int hi = 0; hi < 2; ++hi) {
      f16_of_e2m1x8((wa[hi][w] & kLow) | (wb[hi][w] << 4 & ~kLow), even[hi]);
      f16_of_e2m1x8((wa[hi][w] >> 4 & kLow) | (wb[hi][w] & ~kLow), odd[hi]);
    }
#pragma unroll
    for (int x = 0; x < kNR; ++x) {
      uint32_t y[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i % kW == 0) {   // a group has kW blocks
#pragma unroll
          for (int hi = 0; hi < 2; ++hi) {
            const __half2 z =
                __hmul2(*reinterpret_cast<const __half2 *>(&p[x][hi]),
                        *reinterpret_cast<const __half2 *>(&factor[hi][(4 * w + i) / kW]));
            y[hi] = *reinterpret_cast<const uint32_t *>(&z);
          }
        }
        const uint32_t v[4] = {even[0][i], odd[0][i], even[1][i], odd[1][i]};
        mma<true>(o[4 * w + i][x], v, y[0], y[1]);
      }
    }
  }
}

// A tile taken again, out of line, against the largest score so far, where scores are beyond
// +-64 of R: as in 8 bits.
template <int D, int kNR>
__device__ __noinline__ void take_again(CodeTile<D, kNR> &z, uint32_t sk, const uint4 *made,
                                        bool first) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  score_tile<D, kNR>(sk, made + kKW, g, t, z.s, [&](int step, int x) { return z.q[step][x]; });
#pragma unroll 1
  for (int x = 0; x < kNR; ++x) {
    uint64_t score[4];
    float top[2], l[2];
#pragma unroll
    for (int j = 0; j < 2; ++j)   // at least the sum so far, which is then 1 at most
      top[j] = first ? kLowest : fmaxf(z.ref[x][j], z.ref[x][j] + __log2f(z.l[x][j]));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 8 * i + key_of<D>(g);
      score[i] = mul2(code_product(z.s[i >> 1][x], i & 1, z.before[x], made[row]),
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
      const int row = 8 * i + key_of<D>(g);
      const float ve = __uint_as_float(made[row].z);
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

struct Maps {
  CUtensorMap k, v;
};

// A place in the row of key tiles, with its unit's head and first query row.
struct Place {
  Cursor c;
  int head, row0;
};
__device__ __forceinline__ void set_unit(const PagedArgs &a, Place &p, int rows) {
  p.head = p.c.unit / a.row_tiles;
  p.row0 = (p.c.unit - p.head * a.row_tiles) * rows;
}
__device__ __forceinline__ void advance(const PagedArgs &a, Place &p, int side, int rows) {
  const int unit = p.c.unit;
  step(a, p.c, kTile, side);
  if (p.c.unit != unit) set_unit(a, p, rows);
}

template <int D, int kNR>
__global__ void __launch_bounds__(kThreads, (Cfg4<D, kNR>::kBlocks))
paged_attention4_kernel(const __grid_constant__ Maps maps, const PagedArgs a) {
  using C = Cfg4<D, kNR>;
  constexpr int kNB = kKW / 16, kSteps = D / 16, kMT = D / 16, kRows = C::kRows;
  extern __shared__ uint8_t dyn[];
  __shared__ uint64_t full[kWarps][C::kStages];
  __shared__ int sh_sum[kWarps], sh_at[3], abort_flag;
  __shared__ float sh_m[kWarps][kRows], sh_l[kWarps][kRows], sh_r[kWarps][kRows];
  uint8_t *smem = dyn + (-smem_addr(dyn) & (C::kAlign - 1));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint8_t *ring = smem + warp * (C::kStages * C::kStage);
  uint4 *made = reinterpret_cast<uint4 *>(smem + kWarps * C::kStages * C::kStage +
                                          warp * C::kMade);         // of the present keys
  uint8_t *sq = smem + kWarps * (C::kStages * C::kStage + C::kMade);
  if (lane == 0)
    for (int s = 0; s < C::kStages; ++s) mbar_init(&full[warp][s], 1);
  if (threadIdx.x == 0) abort_flag = 0;
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  // `side` neighbouring blocks take the same run of tiles, each for a unit of its own
  const int side = a.side, run = blockIdx.x / side;
  pdl_wait();
  pdl_trigger();   // the join's blocks wait beside this kernel's, which are all resident by then

  // ---- this block's run of tiles: thread x counts those of a run of sequences, and the
  // one whose sequences the block's first tile falls into says where
  Plan plan;
  {
    const int per = (a.batch + kThreads - 1) / kThreads;
    const int b0 = min(a.batch, (int)threadIdx.x * per), b1 = min(a.batch, b0 + per);
    const int per_tile = side > 1 ? 1 : a.Hkv * a.row_tiles;
    int first_len = 0, mine = 0;
    for (int b = b0; b < b1; ++b) {
      const int n = length(a, b);
      if (b == b0) first_len = n;
      mine += (n + kTile - 1) / kTile * per_tile;
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
    plan = plan_of(total, gridDim.x / side, a.sms);
    if (total == 0 || run >= plan.ctas) {
      if (threadIdx.x == 0) a.cuts[blockIdx.x].parts = 0;
      clear_empty<D>(a);
      return;
    }
    const int at = first_tile(plan, run);
    if (at >= end - mine && at < end) {
      int before = end - mine, len = first_len;
      for (int b = b0;; len = length(a, ++b)) {
        const int n = (len + kTile - 1) / kTile * per_tile;
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
  const int n_tiles = first_tile(plan, run + 1) - first_tile(plan, run);
  Cursor cur;
  cur.b = sh_at[0];
  cur.len = sh_at[1];
  cur.tiles = (cur.len + kTile - 1) / kTile;
  cur.unit = sh_at[2] / cur.tiles;
  cur.tile = sh_at[2] - cur.unit * cur.tiles;
  if (side > 1) cur.unit = blockIdx.x - run * side;   // from 0, of one unit
  if (threadIdx.x == 0) a.cuts[blockIdx.x].parts = 0;

  // ---- the ring: `ahead` is the next tile to load; the pages of this lane's keys in it are read
  // one tile before, and looked at only then
  Place next = {cur, 0, 0};
  Cursor &ahead = next.c;
  set_unit(a, next, kRows);
  int left = n_tiles, loaded = 0;           // tiles to load, and loaded
  int fill = 0;                             // the stage of the next one
  const uint32_t ring_s = smem_addr(ring), bars = smem_addr(&full[warp][0]);
  // a box is a page's rows, or kHold; boxes below 128 bytes go row by row instead
  const int box = min(kHold, 1 << a.page_log2);
  const bool boxes = box * C::kRowBytes >= 128;
  int page[kParts];
  uint32_t wk[kParts], wv[kParts];          // the keys' words, loaded a tile before they are used
  auto look_up = [&]() {
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int key = ahead.tile * kTile + warp * kHold + i * kKW + lane;
      page[i] = -1;
      if (key < ahead.len)
        page[i] = __ldg(a.table + (size_t)ahead.b * a.max_pages + (key >> a.page_log2));
    }
  };
  look_up();
  int q_fill = 0, q_now = 0;                // buffers of the next unit's rows, and of this one's
  auto load_tile = [&]() {
    if (left <= 0) return;
    const int h = next.head;
    if (ahead.tile == 0 || left == n_tiles) {
      // The unit's query rows come with its first tile here, a chunk or more per thread:
      // rows past the last are zeros.  Chunk c of row r lies at c ^ (r & 7).
      const int r0 = next.row0;
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
      commit();   // every thread: the unit's start waits for its own copies
      q_fill = q_fill + 1 == C::kStages ? 0 : q_fill + 1;
    }
    const uint32_t bar = bars + 8 * fill;
    int slot[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int key = ahead.tile * kTile + warp * kHold + i * kKW + lane;
      const bool ok = page[i] >= 0 && page[i] < a.n_pages;
      if (!ok && key < ahead.len) set_error(a.err, kErrIndex);
      // a row that there is not lies past the last: TMA fills it with zeros
      slot[i] = ok ? (page[i] << a.page_log2) + (key & ((1 << a.page_log2) - 1))
                   : a.n_pages << a.page_log2;
      wk[i] = wv[i] = 0u;   // factors of zero
      if (ok) {
        const size_t at = (size_t)slot[i] * a.Hkv + h;
        wk[i] = __ldg(reinterpret_cast<const uint32_t *>(a.ks) + at);
        wv[i] = __ldg(reinterpret_cast<const uint32_t *>(a.vs) + at);
      }
    }
    const bool withheld = a.inject_stall == 1 && loaded == 0;   // test hook: V never loads
    if (boxes) {
      uint8_t *dst = ring + fill * C::kStage;
      const bool leads = elect_one();
      if (leads) mbar_expect_tx(&full[warp][fill], C::kStage);
      for (int i = 0; i < kHold; i += box) {
        const int y = __shfl_sync(0xffffffffu, i < kKW ? slot[0] : slot[kParts - 1], i % kKW);
        if (leads) {
          tma_load_2d(dst + i * C::kRowBytes, &maps.k, &full[warp][fill], h * C::kRowBytes, y);
          if (!withheld)
            tma_load_2d(dst + C::kHalf + i * C::kRowBytes, &maps.v, &full[warp][fill],
                        h * C::kRowBytes, y);
        }
      }
    } else {
      const int none = a.n_pages << a.page_log2;
      unsigned have = 0;
#pragma unroll
      for (int i = 0; i < kParts; ++i) have += __popc(__ballot_sync(0xffffffffu, slot[i] < none));
      if (lane == 0) mbar_expect_tx(&full[warp][fill], have * 2 * C::kRowBytes);
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kParts; ++i) {
        if (slot[i] >= none) continue;   // what the stage held is finite, and its factors are zero
        const uint32_t dst = ring_s + fill * C::kStage;
        const size_t at = ((size_t)slot[i] * a.Hkv + h) * C::kRowBytes;
#pragma unroll
        for (int c = 0; c < C::kChunks; ++c) {
          const uint32_t to = dst + place<D>(i * kKW + lane, c);
          bulk16(to, a.k + at + 16 * c, bar);
          if (!withheld) bulk16(to + C::kHalf, a.v + at + 16 * c, bar);
        }
      }
    }
    fill = fill + 1 == C::kStages ? 0 : fill + 1;
    ++loaded;
    if (--left > 0) {
      advance(a, next, side, kRows);
      look_up();
    }
  };
#pragma unroll
  for (int s = 0; s < C::kStages - 1; ++s) load_tile();

  // ---- per unit state; column block x of the MMAs holds rows 8 x .. 8 x + 7, and this
  // lane row 8 x + g of Q^T and P^T, rows 8 x + 2 t + j of S^T and O^T
  uint32_t qf[kSteps][kNR][2];
  float o[kMT][kNR][4], l[kNR][2];
  // a query row's power of two times the scale's, in two factors, -R, and kShift - M; rows 2 t
  // and 2 t + 1 go together through packed instructions
  float before[kNR][2], after[kNR][2], down[kNR][2], up[kNR][2];
  int unit_tile0 = 0;    // the unit's tile that this run of it starts with
  bool fresh = true, first_unit = true;
  bool first = true;     // this warp has none of the unit's keys yet
  bool live = true;      // no wait has run out
  int now = 0;           // the stage of tile `it`
  auto row0 = [&]() { return cur.unit % a.row_tiles * kRows; };   // the unit's first row
  uint32_t phase = 0;

  for (int it = 0; it < n_tiles; ++it) {
    if (live)
      live = __all_sync(0xffffffffu, mbar_wait(&full[warp][now], phase, &abort_flag, a.err));
    if (fresh) {   // the query rows are every thread's copies
      wait_all_but<0>();
      __syncthreads();
    } else {
      __syncwarp();
    }
    uint32_t wk_now[kParts], wv_now[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) wk_now[i] = wk[i], wv_now[i] = wv[i];
    if (live) load_tile();

    if (fresh) {
      fresh = false;
      first = true;
      unit_tile0 = cur.tile;
      const uint32_t from = smem_addr(sq + q_now * C::kQ);
      q_now = q_now + 1 == C::kStages ? 0 : q_now + 1;
      // a row times 2^(14 - E), its largest magnitude in [2^14, 2^15); `big` over the lanes
      // that hold the row
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
#pragma unroll
      for (int x = 0; x < kNR; ++x) {
        float big = 0.f, f;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const uint2 w = query_at<D>(from, 8 * x + g, s, t);
          qf[s][x][0] = w.x;
          qf[s][x][1] = w.y;
          big = larger(larger(big, w.x), w.y);
        }
        const float scale = scales_of(big, f);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t w = qf[s][x][y];
            qf[s][x][y] = pack_f16(lo_bf16(w) * f, hi_bf16(w) * f);
          }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          // A product y stands for y 2^ks c, c a power of two: multiplied in this order, with
          // c first where it is below 1 and last else, it overflows only where the product of
          // query and key does, whatever their sizes.
          const float c = __shfl_sync(0xffffffffu, scale, 4 * (2 * t + j));
          before[x][j] = fminf(c, 1.f);
          after[x][j] = fminf(fmaxf(c, 1.f) * a.scale_power, 0x1p127f);
          down[x][j] = 0.f;
          up[x][j] = 0.f;   // until the first tile's largest u is known
          l[x][j] = 0.f;
        }
#pragma unroll
        for (int n = 0; n < kMT; ++n) o[n][x][0] = o[n][x][1] = o[n][x][2] = o[n][x][3] = 0.f;
      }
    }

#pragma unroll
    for (int i = 0; i < kParts; ++i) {
      const int key0 = cur.tile * kTile + warp * kHold + i * kKW;
      if (key0 >= cur.len) break;
      const uint32_t sk = ring_s + now * C::kStage + i * (C::kHalf / kParts), sv = sk + C::kHalf;
      if (i) __syncwarp();   // the keys before have been taken
      {
        // A lane's key: (kf, kf, ve, ve) with kf = 2^ks times the scale's digits and ve = vs;
        // K's factors; V's in fp16, beside those of the pair's other key: this lane makes two
        // groups' of both, the key of the even MMA index low.  A row of NaN has s = 255: its kf,
        // or ve, is NaN.
        const uint2 w = i == 0 ? make_uint2(wk_now[0], wv_now[0])
                               : make_uint2(wk_now[kParts - 1], wv_now[kParts - 1]);
        const uint32_t ks = w.x >> 24, vs = w.y >> 24;
        const uint32_t kf =
            ks == 255u ? 0x7fffffffu : __float_as_uint(__uint_as_float(ks << 23) * a.scale_digits);
        const uint32_t ve =
            vs == 255u ? 0x7fffffffu
                       : __float_as_uint(__uint_as_float(0x4b000000u | vs) - (0x1p23f + 127.f));
        made[lane] = make_uint4(kf, kf, ve, ve);
        auto factor = [&](int i) {
          return __float_as_uint(__uint_as_float(0x4b000000u | (w.x >> (6 * i) & 63u)) - 0x1p23f);
        };
        made[kKW + lane] = make_uint4(factor(0), factor(1), factor(2), factor(3));
        const uint32_t other = __shfl_xor_sync(0xffffffffu, w.y, 1);
        const bool even = is_even<D>(lane & 7);
        const uint32_t lo = even ? w.y : other, hi = even ? other : w.y;
        auto pair = [&](int i) {
          __half2 z;
          *reinterpret_cast<uint32_t *>(&z) =
              0x64006400u | (lo >> (6 * i) & 63u) | (hi >> (6 * i) & 63u) << 16;
          z = __hsub2(z, __float2half2_rn(1024.f));
          return *reinterpret_cast<uint32_t *>(&z);
        };
        const int two = even ? 0 : 2;
        reinterpret_cast<uint2 *>(made + 2 * kKW)[2 * (lane >> 1) + (even ? 0 : 1)] =
            make_uint2(pair(two), pair(two + 1));
        __syncwarp();
      }
      const bool ragged = key0 + kKW > cur.len - a.n_new + 1;
      // keys that row 8 x + 2 t + j sees, where that matters
      auto limit = [&](int x, int j) {
        return cur.len - a.n_new + 1 +
               (int)quotient(row0() + 8 * x + 2 * t + j, a.group);
      };
      float s[kNB][kNR][4], mx[kNR][2], sum[kNR][2];
      score_tile<D, kNR>(sk, made + kKW, g, t, s, [&](int step, int x) {
        return make_uint2(qf[step][x][0], qf[step][x][1]);
      });
      // ---- log2 units above R, the weights' sum, and u - M + kShift, of which no one may be
      // above kShift + kSlack
#pragma unroll
      for (int x = 0; x < kNR; ++x) {
        mx[x][0] = mx[x][1] = -INFINITY;
        sum[x][0] = l[x][0], sum[x][1] = l[x][1];
      }
      // (without masks first: one piece of code with the products, in which the two blocks overlap)
      float e[kNB][kNR][4];
#pragma unroll
      for (int b = 0; b < kNB; ++b)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const uint4 w = made[16 * b + 8 * n + key_of<D>(g)];
#pragma unroll
          for (int x = 0; x < kNR; ++x) {
            const uint64_t z =
                fma2(code_product(s[b][x], n, before[x], w), both(after[x][0], after[x][1]),
                     both(down[x][0], down[x][1]));
            const uint64_t u = add2(add2(z, pack2(w.z, w.w)), both(up[x][0], up[x][1]));
            e[b][x][2 * n] = fast_exp2(lo_f(z)), e[b][x][2 * n + 1] = fast_exp2(hi_f(z));
            s[b][x][2 * n] = lo_f(u), s[b][x][2 * n + 1] = hi_f(u);
          }
        }
      if (ragged) {
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int x = 0; x < kNR; ++x)
#pragma unroll
              for (int j = 0; j < 2; ++j)
                if (key0 + 16 * b + 8 * n + key_of<D>(g) >= limit(x, j))
                  s[b][x][2 * n + j] = -INFINITY, e[b][x][2 * n + j] = 0.f;
      }
#pragma unroll
      for (int x = 0; x < kNR; ++x)
#pragma unroll
        for (int b = 0; b < kNB; ++b)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            const uint64_t w2 = add2(both(sum[x][0], sum[x][1]),
                                     both(e[b][x][2 * n], e[b][x][2 * n + 1]));
            sum[x][0] = lo_f(w2), sum[x][1] = hi_f(w2);
            mx[x][0] = fmaxf(mx[x][0], s[b][x][2 * n]);
            mx[x][1] = fmaxf(mx[x][1], s[b][x][2 * n + 1]);
          }
      // Rare: the first tile, sums far from R, or a u further above M than fp16 has room for.  M
      // is a largest u, but rises only then: a new largest is in two thirds of the first 20
      // tiles, and O would be scaled each time.
      float most = 0.f, above = -INFINITY;
#pragma unroll
      for (int x = 0; x < kNR; ++x) {
        most = max3f(most, sum[x][0], sum[x][1]);
        above = max3f(above, mx[x][0], mx[x][1]);
      }
      if (first || __any_sync(0xffffffffu, most > kFar || above > kShift + kSlack)) {
        bool far = most > kFar;
        if (first) {
#pragma unroll
          for (int x = 0; x < kNR; ++x)
#pragma unroll
            for (int j = 0; j < 2; ++j) far |= sum[x][j] < 1.f / kFar && mx[x][j] > -INFINITY;
        }
        far = __any_sync(0xffffffffu, far);
        float old[kNR][2];   // M, and mx, relative to R
#pragma unroll
        for (int x = 0; x < kNR; ++x)
#pragma unroll
          for (int j = 0; j < 2; ++j) old[x][j] = kShift - up[x][j], mx[x][j] -= up[x][j];
        if (far) {
          // out of line, so that it costs the usual path no registers
          CodeTile<D, kNR> z;
#pragma unroll
          for (int x = 0; x < kNR; ++x) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) z.q[i][x] = make_uint2(qf[i][x][0], qf[i][x][1]);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              z.before[x][j] = before[x][j], z.after[x][j] = after[x][j];
              z.limit[x][j] = ragged ? limit(x, j) - key0 : kKW;
              z.ref[x][j] = -down[x][j], z.l[x][j] = l[x][j], z.m[x][j] = old[x][j];
            }
          }
          take_again<D, kNR>(z, sk, made, first);
#pragma unroll
          for (int x = 0; x < kNR; ++x)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              down[x][j] = -z.ref[x][j], sum[x][j] = z.l[x][j];
              old[x][j] = z.m[x][j], mx[x][j] = z.mx[x][j];
#pragma unroll
              for (int b = 0; b < kNB; ++b) {
                s[b][x][j] = z.s[b][x][j], s[b][x][2 + j] = z.s[b][x][2 + j];   // u
              }
            }
        }
#pragma unroll
        for (int x = 0; x < kNR; ++x)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1)
              mx[x][j] = fmaxf(mx[x][j], __shfl_xor_sync(0xffffffffu, mx[x][j], d));
            // a row that sees no key of the first tile sees none here at all
            const float M = !first                ? fmaxf(mx[x][j], old[x][j])
                            : mx[x][j] > kLowest ? mx[x][j]
                                                 : 0.f;
            const float f = first ? 1.f : fast_exp2(old[x][j] - M);
            const float by = kShift - M - (far ? 0.f : up[x][j]);
            up[x][j] = kShift - M;
#pragma unroll
            for (int b = 0; b < kNB; ++b) s[b][x][j] += by, s[b][x][2 + j] += by;
#pragma unroll
            for (int n = 0; n < kMT; ++n) o[n][x][j] *= f, o[n][x][2 + j] *= f;
          }
      }
      first = false;
#pragma unroll
      for (int x = 0; x < kNR; ++x) l[x][0] = sum[x][0], l[x][1] = sum[x][1];
      // ---- probabilities in fp16, as the 16 x 8 B operand of O^T += V^T P^T: off by half a
      // step at most (2^-11 of themselves, and 2^-11 again with a factor); the sum l takes
      // them unrounded.  Those with u more than 20 below M lose further bits, and more than
      // 31 below they are zero.
#pragma unroll
      for (int b = 0; b < kNB; ++b) {
        uint32_t p[kNR][2];
#pragma unroll
        for (int x = 0; x < kNR; ++x)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            p[x][n] = transposed(
                pack_f16(fast_exp2(s[b][x][2 * n]), fast_exp2(s[b][x][2 * n + 1])));
          }
        add_values<D, kNR>(o, p, sv, made + 2 * kKW, b, g, t);
      }
    }

    const bool unit_done = cur.tile + 1 == cur.tiles;
    if (unit_done || it + 1 == n_tiles) {
      // ---- the unit's end, or the run's: the four warps' parts become one.  Each leaves its
      // sums in the stage that it has just read, lane by lane, and takes a quarter of the
      // dimensions of all four.  TMA fills the stage again only after the barrier that starts
      // the next unit.
      const int h = cur.unit / a.row_tiles, r0 = row0();
#pragma unroll
      for (int x = 0; x < kNR; ++x)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[x][j] += __shfl_xor_sync(0xffffffffu, l[x][j], d);
          if (g == 0) {
            sh_m[warp][8 * x + 2 * t + j] = kShift - up[x][j];
            sh_l[warp][8 * x + 2 * t + j] = l[x][j];
            sh_r[warp][8 * x + 2 * t + j] = l[x][j] == 0.f ? kLowest : -down[x][j];
          }
        }
      __syncwarp();   // every lane has read the stage
      constexpr int kQuarter = kMT / kWarps;                // MMA blocks of 16 dimensions
      static_assert(C::kStage >= kMT * 512, "a stage takes the sums of a column block");
      const bool whole = unit_tile0 == 0 && unit_done;
      float *part = a.ws + (size_t)(2 * blockIdx.x + (first_unit ? 0 : 1)) * C::kPart;
#pragma unroll
      for (int x = 0; x < kNR; ++x) {
        if (x) __syncthreads();
#pragma unroll
        for (int n = 0; n < kMT; ++n) {
          const float(&y)[4] = o[n][x];
          reinterpret_cast<float4 *>(ring + now * C::kStage)[n * 32 + lane] =
              make_float4(y[0], y[1], y[2], y[3]);
        }
        __syncthreads();
        float f[2][kWarps], M[2], R[2], sum[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int r = 8 * x + 2 * t + j;
          R[j] = sh_r[0][r];   // the warps' M relative to the largest R
#pragma unroll
          for (int w = 1; w < kWarps; ++w) R[j] = fmaxf(R[j], sh_r[w][r]);
          auto level = [&](int w) { return sh_r[w][r] - R[j] + sh_m[w][r]; };
          M[j] = level(0);
#pragma unroll
          for (int w = 1; w < kWarps; ++w) M[j] = fmaxf(M[j], level(w));
          sum[j] = 0.f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            f[j][w] = fast_exp2(level(w) - M[j]);
            sum[j] = fmaf(sh_l[w][r], fast_exp2(sh_r[w][r] - R[j]), sum[j]);
          }
        }
        float y[kQuarter][4];
#pragma unroll
        for (int n = 0; n < kQuarter; ++n) {
          y[n][0] = y[n][1] = y[n][2] = y[n][3] = 0.f;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float4 z = reinterpret_cast<const float4 *>(
                smem + (w * C::kStages + now) * C::kStage)[(warp * kQuarter + n) * 32 + lane];
            y[n][0] = fmaf(z.x, f[0][w], y[n][0]), y[n][1] = fmaf(z.y, f[1][w], y[n][1]);
            y[n][2] = fmaf(z.z, f[0][w], y[n][2]), y[n][3] = fmaf(z.w, f[1][w], y[n][3]);
          }
        }
        const int d = D / 8 * g + 2 * warp * kQuarter;   // block n: dimensions D/8 g + 2 n, + 1
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int rr = 8 * x + 2 * t + j, r = r0 + rr;
          if (r >= a.rows) continue;
          if (whole) {
            const RowEnd<true> end(sum[j], M[j] - kShift);
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
              float *stat = part + kRows * D + part_stats(true) * rr;
              stat[0] = M[j] + (kPShift - kShift);   // the join's probabilities have kPShift
              stat[1] = sum[j];
              stat[2] = R[j];
            }
          }
        }
      }
      // what was written to the stage here comes before what TMA writes there
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      if (unit_done && !whole) {   // a run ends one such unit at most: its first
        const int t0 = first_tile(plan, run) - unit_tile0;
        const int c0 = cta_of(plan, t0);
        const int first_block = blockIdx.x - (run - c0) * side;
        if (threadIdx.x == 0)
          a.cuts[blockIdx.x] = {run - c0 + 1, first_block,
                                2 * first_block + (first_tile(plan, c0) == t0 ? 0 : 1), cur.b,
                                cur.unit};
      }
      first_unit = false;
      fresh = true;
    }
    if (++now == C::kStages) now = 0, phase ^= 1;
    if (it + 1 < n_tiles) step(a, cur, kTile, side);
  }
  wait_all_but<0>();
  if (!live) {
    // copies that a wait gave up on, or was not made for, land before the block ends
    for (int i = max(0, loaded - C::kStages); i < loaded; ++i)
      mbar_wait(&full[warp][i % C::kStages], i / C::kStages & 1, &abort_flag, a.err, false);
  }
  clear_empty<D>(a);
}

// -------------------------------------------------------------- host side

// A cache of n rows of all heads, as rows of bytes; a box is `rows` of one head's.
bool make_map(CUtensorMap &map, const void *base, long long n, int heads, int row_bytes, int rows) {
  auto enc = encode_fn();
  const cuuint64_t dims[2] = {(cuuint64_t)heads * row_bytes, (cuuint64_t)n};
  const cuuint64_t strides[1] = {(cuuint64_t)heads * row_bytes};
  const cuuint32_t box[2] = {(cuuint32_t)row_bytes, (cuuint32_t)rows};
  const cuuint32_t ones[2] = {1, 1};
  return enc && enc(&map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides,
                    box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    row_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE,
                    CU_TENSOR_MAP_L2_PROMOTION_NONE,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int kNR>
int launch(PagedArgs &a, void *workspace, cudaStream_t stream) {
  using C = Cfg4<D, kNR>;
  auto kernel = paged_attention4_kernel<D, kNR>;
  static std::atomic<int> per_sm[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return HSA_ERR_CUDA;
  int nb = per_sm[dev].load(std::memory_order_acquire);
  if (nb <= 0) {
    // both kernels ask for the same split between L1 and shared memory (see the 8-bit one)
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem) !=
            cudaSuccess ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout,
                             cudaSharedmemCarveoutMaxShared) != cudaSuccess ||
        cudaFuncSetAttribute(paged_join_kernel<D, true, kNR>,
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
  const long long heads = (long long)a.Hkv * a.row_tiles, units = a.batch * heads;
  const long long tiles = (((long long)a.max_pages << a.page_log2) + kTile - 1) / kTile;
  if (units * tiles > 0x7fffffffLL) return HSA_ERR_UNSUPPORTED;   // tiles are counted in 32 bits
  Maps maps;
  std::memset(&maps, 0, sizeof maps);
  if (tiles) {
    const long long rows = (long long)a.n_pages << a.page_log2;
    const int box = std::min(kHold, 1 << a.page_log2);
    if (!make_map(maps.k, a.k, rows, a.Hkv, C::kRowBytes, box) ||
        !make_map(maps.v, a.v, rows, a.Hkv, C::kRowBytes, box))
      return HSA_ERR_CUDA;
  }
  int grid = (int)std::min<long long>(nb * sm_count(), tiles ? units * tiles : a.batch);
  // A key's rows of all heads lie together, of 32 or 64 bytes and a word each: where the heads'
  // blocks read the same keys at the same time, the halves of lines and the seven eighths of
  // sectors that one does not need are the others' from L2.  Not where the blocks that are left
  // over outweigh that.
  const long long runs = heads <= grid ? grid / heads : 0;
  if (heads > 1 && 16 * runs * heads >= 15 * (long long)grid) {
    a.side = (int)heads;
    grid = (int)(runs * heads);
    a.sms = std::max(1, a.sms / a.side);
  }
  a.cuts = static_cast<CutUnit *>(workspace);
  a.ws = reinterpret_cast<float *>(a.cuts + (size_t)sm_count() * kMaxPerSm);
  count_launches(2);
  launch_pdl(kernel, dim3((unsigned)grid), dim3(kThreads), C::kSmem, stream, maps, a);
  if (cudaGetLastError() != cudaSuccess) return HSA_ERR_CUDA;
  launch_pdl(paged_join_kernel<D, true, kNR>,
             dim3((unsigned)grid, (unsigned)std::min(a.rows, C::kRows)), dim3(kJoinThreads), 0,
             stream, a);
  return launch_status();
}

}  // namespace

// Column blocks of eight query rows per unit: one, or two that share the keys' fragments.  48
// sequences of 4500 keys, 8 K/V heads, D = 128 (64): 4 and 8 rows a head 61 and 65 us (49); 16 rows
// 97 (74), with units of eight rows, which decode the keys twice, 113 (86); 24 rows 161 (120)
// against 153 (119), 32 rows 162 (121) against 203 (147).  More than two do not fit the registers.
int launch_paged4(PagedArgs &a, int D, void *workspace, cudaStream_t stream) {
  if (D == 128)
    return a.rows <= 8 ? launch<128, 1>(a, workspace, stream)
                       : launch<128, 2>(a, workspace, stream);
  return a.rows <= 8 ? launch<64, 1>(a, workspace, stream)
                     : launch<64, 2>(a, workspace, stream);
}

}  // namespace hsa

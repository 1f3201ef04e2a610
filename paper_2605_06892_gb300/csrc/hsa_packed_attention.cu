// Attention over whole prompts: several sequences packed one behind the other, query
// heads in groups that share a K/V head, bidirectional or causal by frames of F tokens
// (F = 1: plainly causal).  Query i of a sequence of Lq queries and Lk keys stands at
// p = i + Lk - Lq and sees the keys below
//   limit_i = Lk, or min(Lk, (floor(p / F) + 1) F) with a mask (none where that is <= 0).
// 4 D FLOPs per query head and visible pair: bound by the tensor pipe.
//
// The pipeline of a CTA (256 query rows in two Q tiles, 128-key tiles through a TMA ring,
// scores and O in TMEM, named-barrier hand-offs) is the active attention's (hsa_tc.cuh,
// hsa_attention.cu).  What differs:
//  - Rows.  A unit's rows are (token, head of the group) pairs, row R = i G + g of a
//    sequence and K/V head.  One pass over the keys serves the whole group: K and V are
//    read 1/G as often, short sequences fill the 256 rows G times sooner, and the rows of
//    a unit span only 256 / G tokens, so fewer of its key tiles cross the mask's edge.
//  - Units.  The lengths are on the device, so every block works out its units from them:
//    sequence by sequence, head by head, each head's query blocks from the last (under a
//    mask the longest) to the first, so that a head's K/V are read by blocks that run
//    together and the last units to start are short.  A block goes on to further units.
//  - Mask.  A unit's key tiles end at its last row's limit; a row's own limit is applied
//    to its scores in the tiles that some row of its warp does not see whole.
//  - Few units.  With a workspace the units of the last, partly filled wave (all of them
//    where there are fewer units than SMs) are cut along the keys and joined afterwards;
//    under a mask only the latter, since the last units to start are short already.
//  - Rows without keys come out as zeros.
//  - Values that a row does not see must not reach it by 0 * NaN.  The rows of V behind a
//    sequence's end are zeroed in shared memory before they are multiplied.  Under a mask,
//    a row whose result is not finite looks through the values it should not have met in
//    its unit's tiles; if one of those is not finite the row is formed again without them
//    on the CUDA cores, once the block has ended its units.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "hsa_internal.cuh"
#include "hsa_ptx.cuh"
#include "hsa_tc.cuh"

namespace hsa {
namespace {

struct Cuts;

constexpr int kUnitRows = kQT * kBM;
constexpr float kLowest = -3.0e38f;   // running maximum of a row that has seen no key

struct PackedArgs {
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16 *out;
  const int32_t *cu_q, *cu_k;
  unsigned *err;
  int batch, total_q, total_k, Hq, Hkv, mask;
  Divider group, frame;            // by G = Hq / Hkv and by the mask
  long long q_row, k_row, v_row;   // elements from a token to the next
  float scale_log2;
  int sms, most;                   // most: pieces that a cut may make, 0: none
  int bound;                       // units that the host allowed for
  int q_map, o_map;                // the query rows come, the output rows go by TMA
  int inject_stall;                // test hook (hsa_test.h)
  float *ws_o, *ws_ml;             // [piece][sum_place], [piece][kUnitRows][2]
  Cuts *cuts;                      // what the join reads
};

struct Sequence {
  int q0, lq, k0, lk;
};

__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, uint64_t *bar,
                                            int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_addr(dst)),
      "l"(map), "r"(smem_addr(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, const void *src, int x, int y,
                                             int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map),
      "r"(smem_addr(src)), "r"(x), "r"(y), "r"(z)
      : "memory");
}

__device__ __forceinline__ void bulk_store(void *dst, const void *src, int bytes) {
  asm volatile(
      "cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;\n"
      "cp.async.bulk.commit_group;" ::"l"(dst), "r"(smem_addr(src)), "r"(bytes)
      : "memory");
}

// Sequence b's rows and keys; ends that run backwards or past the tensors are moved
// inside and reported.
__device__ __forceinline__ Sequence sequence(const PackedArgs &a, int b) {
  const int q0 = __ldg(a.cu_q + b), q1 = __ldg(a.cu_q + b + 1);
  const int k0 = __ldg(a.cu_k + b), k1 = __ldg(a.cu_k + b + 1);
  Sequence s;
  s.q0 = min(max(q0, 0), a.total_q);
  s.k0 = min(max(k0, 0), a.total_k);
  const int qe = min(max(q1, s.q0), a.total_q), ke = min(max(k1, s.k0), a.total_k);
  if (s.q0 != q0 || s.k0 != k0 || qe != q1 || ke != k1) set_error(a.err, kErrIndex);
  s.lq = qe - s.q0;
  s.lk = ke - s.k0;
  return s;
}

__device__ __forceinline__ int query_blocks(const PackedArgs &a, const Sequence &s) {
  return (int)(((long long)s.lq * a.group.d + kUnitRows - 1) / kUnitRows);
}

// Keys that query i of a sequence sees.
__device__ __forceinline__ int key_limit(const PackedArgs &a, const Sequence &s, int i) {
  if (!a.mask) return s.lk;
  const int p = i + s.lk - s.lq;
  if (p < 0) return 0;
  return (int)min((long long)s.lk, ((long long)quotient(p, a.frame) + 1) * a.mask);
}

// What all blocks of a launch share.  Units below n_whole are whole.  The others are cut:
// all of them (n_whole = 0) into parts of `longest` key tiles of their sequence, or, with
// longest = 0, the last units into `pieces` each.
struct Plan {
  int units, n_whole, pieces, longest;
};

// One unit, or one part of one.
struct Unit {
  Sequence seq;
  int head, row0, rows;  // row0: its first row among the sequence's lq G
  int j0, nT;            // key tiles: j0 .. j0 + nT - 1
  int part, parts;       // parts = 1: whole; 0: there is no unit
  int slot;              // of its first part in the workspace
  int cut;               // its place among the cut units, or -1
};

// A part of a cut unit has four key tiles at least (two are no faster: 26 tokens after 19095
// 25.3 against 25.9 us, eight slower, 28.5), and the join costs what seven tiles take: 64
// tokens after 900, eight tiles, take 15.1 us whole and 18.5 in two.
constexpr int kLeastTiles = 4, kJoinTiles = 7;

__device__ __forceinline__ int parts_of(const Sequence &s, int longest) {
  const int tiles = (s.lk + kBN - 1) / kBN;
  return longest && tiles > longest ? (tiles + longest - 1) / longest : 1;
}

// The sequences b0 .. b0 + 31, one per lane, and how many units (with `longest` also parts)
// come before them.  A block's ids rise, so it goes through the sequences once.
struct Window {
  Sequence seq;
  int blocks, b0, ids, units;
};
__device__ __forceinline__ void look_at(const PackedArgs &a, Window &w, int b0, int ids,
                                        int units) {
  const int b = b0 + (threadIdx.x & 31);
  w.seq = {};
  if (b < a.batch) w.seq = sequence(a, b);
  w.blocks = query_blocks(a, w.seq);
  w.b0 = b0;
  w.ids = ids;
  w.units = units;
}

// The plan; called by a whole warp, `first` its window on the first sequences.
__device__ __forceinline__ void plan_units(const PackedArgs &a, const Window &first, Plan &p) {
  const int lane = threadIdx.x & 31;
  // f(sequence, its query blocks) for this lane's sequences
  auto each = [&](auto &&f) {
    f(first.seq, first.blocks);
    for (int b = lane + 32; b < a.batch; b += 32) {
      const Sequence s = sequence(a, b);
      f(s, query_blocks(a, s));
    }
  };
  // offsets that overlap may make more units than there are ids: those go without
  unsigned mine = 0;
  each([&](const Sequence &, int blocks) { mine = min(mine + blocks, 1u << 26); });
  const long long units_all = (long long)__reduce_add_sync(0xffffffffu, mine) * a.Hkv;
  p.units = (int)min(units_all, 0x7fffffffLL);
  p.n_whole = p.units;
  p.pieces = 1;
  p.longest = 0;
  auto longest = [&]() {   // key tiles of a unit at most
    int keys = 0;
    each([&](const Sequence &s, int blocks) {
      if (blocks) keys = max(keys, s.lk);
    });
    return (__reduce_max_sync(0xffffffffu, keys) + kBN - 1) / kBN;
  };
  const bool may = a.most && p.units > 0 && p.units <= a.bound;   // more: offsets that overlap
  if (may && p.units < a.sms) {
    // Fewer units than SMs: the shortest part length that makes no more parts than SMs, or
    // than two waves of them; a part costs its tiles and about 5 tiles' time more.
    unsigned work = 0;   // < 2^24 tiles of fewer units than SMs
    each([&](const Sequence &s, int blocks) {
      work += (unsigned)blocks * ((s.lk + kBN - 1) / kBN);
    });
    const int far = longest();
    work = __reduce_add_sync(0xffffffffu, work) * a.Hkv;
    auto shortest = [&](int most) {
      // n parts of L tiles: work / L <= n < work / L + units
      int lo = max(kLeastTiles, (int)(work / most));
      int hi = most > p.units ? min(far, (int)(work / (most - p.units)) + 1) : far;
      hi = max(hi, lo);
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        int n = 0;
        each([&](const Sequence &s, int blocks) { n += blocks * parts_of(s, mid); });
        if (__reduce_add_sync(0xffffffffu, n) * a.Hkv <= most) hi = mid;
        else lo = mid + 1;
      }
      return lo;
    };
    // (no search where even parts of one length would not pay: each takes a microsecond)
    if ((int)(work / a.sms) + kJoinTiles < far) {
      int len = shortest(a.sms);
      if (a.most > a.sms && 2 * ((int)(work / (2 * a.sms)) + 5) < len + 5) {
        const int two = shortest(2 * a.sms);
        if (2 * (two + 5) < len + 5) len = two;
      }
      if (len + kJoinTiles < far) {
        p.n_whole = 0;
        p.longest = len;
      }
    }
  } else if (may && a.most >= 2 * a.sms && !a.mask && p.units % a.sms) {
    // More units than SMs: under a mask the last ones to start are short already.  Without,
    // the rem units of the last wave in P pieces each take ceil(rem P / sms) waves of 1/P
    // unit, and each piece 0.005 unit more; at most two waves.
    const int rem = p.units % a.sms;
    float best = 1.005f;
    for (int p0 = 2; p0 <= 2 * a.sms / rem; p0 += 32) {
      const int n = p0 + lane;
      float cost =
          n <= 2 * a.sms / rem ? (float)((rem * n + a.sms - 1) / a.sms) / n + 0.005f * n : INFINITY;
      int at = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const float c = __shfl_xor_sync(0xffffffffu, cost, o);
        const int x = __shfl_xor_sync(0xffffffffu, at, o);
        if (c < cost || (c == cost && x < at)) cost = c, at = x;
      }
      if (cost < best) best = cost, p.pieces = at;
    }
    if (p.pieces > 1 && (1.f - best) * longest() > kJoinTiles) p.n_whole = p.units - rem;
    else p.pieces = 1;
  }
}

// The unit and part of block `id` (which counts units, or with `longest` parts); false: it
// has none.  Called by a whole warp.
__device__ __forceinline__ bool unit_of(const PackedArgs &a, int id, const Plan &p, Window &w,
                                        Unit &u) {
  const int lane = threadIdx.x & 31;
  u.part = u.slot = 0;
  u.cut = -1;
  int pieces = 1;
  if (!p.longest && id >= p.n_whole) {
    const int i = id - p.n_whole;
    pieces = p.pieces;
    u.cut = i / pieces;
    u.part = i - u.cut * pieces;
    u.slot = u.cut * pieces;
    id = p.n_whole + u.cut;
    if (id >= p.units) return false;
  }
  if (id < w.ids) look_at(a, w, 0, 0, 0);   // ids that do not rise
  while (true) {
    const int parts = parts_of(w.seq, p.longest);
    const int n = w.blocks * a.Hkv * parts;
    int end = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, end, o);
      if (lane >= o) end += x;
    }
    end += w.ids;
    const unsigned here = __ballot_sync(0xffffffffu, id >= end - n && id < end);
    if (here) {
      const int src = __ffs(here) - 1;
      u.seq.q0 = __shfl_sync(0xffffffffu, w.seq.q0, src);
      u.seq.lq = __shfl_sync(0xffffffffu, w.seq.lq, src);
      u.seq.k0 = __shfl_sync(0xffffffffu, w.seq.k0, src);
      u.seq.lk = __shfl_sync(0xffffffffu, w.seq.lk, src);
      int at = id - __shfl_sync(0xffffffffu, end - n, src);
      if (p.longest) {
        pieces = __shfl_sync(0xffffffffu, parts, src);
        const int before = __reduce_add_sync(0xffffffffu, lane < src ? w.blocks * a.Hkv : 0);
        const int x = at / pieces;
        u.part = at - x * pieces;
        u.slot = id - u.part;
        u.cut = w.units + before + x;
        at = x;
      }
      const int blocks = __shfl_sync(0xffffffffu, w.blocks, src);
      u.head = at / blocks;
      u.row0 = (blocks - 1 - (at - u.head * blocks)) * kUnitRows;
      const long long rows = (long long)u.seq.lq * a.group.d;
      u.rows = (int)min(rows - u.row0, (long long)kUnitRows);
      const int tiles =
          (key_limit(a, u.seq, quotient(u.row0 + u.rows - 1, a.group)) + kBN - 1) / kBN;
      u.parts = max(1, min(pieces, tiles / kLeastTiles));
      // parts of one length, the first ones a tile longer
      u.nT = tiles / u.parts;
      const int more = tiles - u.nT * u.parts;
      u.j0 = u.part * u.nT + min(u.part, more);
      u.nT += u.part < more;
      return u.part < u.parts;
    }
    if (w.b0 + 32 >= a.batch) return false;
    const int units = w.units + __reduce_add_sync(0xffffffffu, w.blocks * a.Hkv);
    look_at(a, w, w.b0 + 32, __shfl_sync(0xffffffffu, end, 31), units);
  }
}

// What the join has to know, written by the kernel before it: how many units were cut, and
// of each its first part's slot and parts, its rows and where they go.
struct CutUnit {
  int parts, slot, rows, row0, q0, head, pad[2];
};
struct Cuts {
  int n, pad[7];
  CutUnit unit[1];   // one per SM at most
};

// Address of output row R of a K/V head and the sequence whose first row is q0.
template <int D>
__device__ __forceinline__ __nv_bfloat16 *out_row(const PackedArgs &a, int q0, int head, int R) {
  const int i = quotient(R, a.group);
  return a.out + ((size_t)(q0 + i) * a.Hq + head * (int)a.group.d + (R - i * (int)a.group.d)) * D;
}

// Where a piece's workspace holds the sums of dimensions 4 x .. 4 x + 3 of row r, in vectors:
// half of the dimensions of 32 rows lie together, as they leave shared memory.
template <int D>
__device__ __forceinline__ int sum_place(int r, int x) {
  constexpr int kV = D / 8;
  const int y = x % kV;
  return (((r >> 5) * 2 + x / kV) * 32 + (r & 31)) * kV + ((y & ~7) | ((y ^ r) & 7));
}

// A row of V's elements that are not finite (kNan: that are NaN), a bit each.
template <int D, bool kNan>
__device__ __forceinline__ void odd_elements(const __nv_bfloat16 *v, uint32_t (&bits)[D / 32]) {
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint4 w = __ldg(reinterpret_cast<const uint4 *>(v + 32 * c + 8 * i));
      const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lo = x[e] << 16 & 0x7fff0000u, hi = x[e] & 0x7fff0000u;
        constexpr uint32_t kFrom = kNan ? 0x7f810000u : 0x7f800000u;
        bits[c] |= (uint32_t)(lo >= kFrom) << (8 * i + 2 * e);
        bits[c] |= (uint32_t)(hi >= kFrom) << (8 * i + 2 * e + 1);
      }
    }
}

// Forms and stores those of this warp's rows again (r: this lane's) whose sums took in a
// masked value that is not finite: the softmax over the row's own keys of the unit or piece,
// on the CUDA cores, 32 keys at a time by way of `st`, 64 D bytes of the warp's own.  Rare and
// slow (4 us a key); out of line so that it costs the usual path no registers.  A row stays as
// it is where one of its own last keys has NaN in each dimension that a masked value spoils:
// it is NaN there in any case, and so values that are NaN throughout cost no more than a look.
template <int D>
__device__ __noinline__ void form_again(const PackedArgs &a, const Unit &u, int r, uint4 *st) {
  const int lane = threadIdx.x & 31;
  const int piece = u.parts > 1 ? u.slot + u.part : -1;
  const int k0 = u.j0 * kBN, k1 = min(u.seq.lk, k0 + u.nT * kBN), R = u.row0 + r;
  const bool valid = r < u.rows;
  const __nv_bfloat16 *K = a.k + (size_t)u.seq.k0 * a.k_row + (size_t)u.head * D;
  const __nv_bfloat16 *V = a.v + (size_t)u.seq.k0 * a.v_row + (size_t)u.head * D;
  const int tok = valid ? quotient(R, a.group) : 0;
  const int limit = valid ? key_limit(a, u.seq, tok) : 0;
  const __nv_bfloat16 *Q = a.q + (size_t)(u.seq.q0 + tok) * a.q_row +
                           (u.head * (int)a.group.d + (valid ? R - tok * (int)a.group.d : 0)) * D;
  bool bad = false;
  if (valid) {
    uint32_t spoilt[D / 32] = {}, own[D / 32] = {};
    auto left = [&]() {
      uint32_t any = 0;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) any |= spoilt[c] & ~own[c];
      return any != 0;
    };
    for (int j = max(limit, k0); j < k1; ++j)
      odd_elements<D, false>(V + (size_t)j * a.v_row, spoilt);
    bad = left();
    for (int j = min(limit, k1) - 1, n = 0; j >= k0 && n < 32 && bad; --j, ++n) {
      odd_elements<D, true>(V + (size_t)j * a.v_row, own);
      bad = left();
    }
  }
  const int end = bad ? min(limit, k1) : 0;
  const int most = __reduce_max_sync(0xffffffffu, end);
  if (!__any_sync(0xffffffffu, bad)) return;
  uint4 q[D / 8];
#pragma unroll
  for (int v = 0; v < D / 8; ++v)
    q[v] = bad ? __ldg(reinterpret_cast<const uint4 *>(Q) + v) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
  for (int c = 0; c < D / 32; ++c) {
    float acc[32], m = kLowest, l = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i] = 0.f;
#pragma unroll 1
    for (int j0 = k0; j0 < most; j0 += 32) {
      auto bring = [&](const __nv_bfloat16 *rows, long long row, int vectors) {
        __syncwarp();
        for (int e = lane; e < 32 * vectors; e += 32) {
          const int j = j0 + e / vectors;
          st[e] = j < most ? __ldg(reinterpret_cast<const uint4 *>(rows + (size_t)j * row) +
                                   e % vectors)
                           : make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
      };
      float p[32], top = m;
      bring(K, a.k_row, D / 8);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < D / 8; ++v) {
          const uint4 kw = st[i * (D / 8) + v];
          const uint32_t x[4] = {q[v].x, q[v].y, q[v].z, q[v].w}, y[4] = {kw.x, kw.y, kw.z, kw.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[e] = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), s[e]);
            s[e] = fmaf(__uint_as_float(x[e] & 0xffff0000u), __uint_as_float(y[e] & 0xffff0000u),
                        s[e]);
          }
        }
        p[i] = ((s[0] + s[1]) + (s[2] + s[3])) * a.scale_log2;
        if (j0 + i < end) top = fmaxf(top, p[i]);
      }
      const float f = fast_exp2(m - top);
      m = top;
      l *= f;
#pragma unroll
      for (int i = 0; i < 32; ++i) acc[i] *= f;
      bring(V + 32 * c, a.v_row, 4);
#pragma unroll
      for (int i = 0; i < 32; ++i) {
        if (j0 + i >= end) continue;
        const float w = fast_exp2(p[i] - m);
        l += w;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const uint4 x4 = st[i * 4 + v];
          const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            acc[8 * v + 2 * e] = fmaf(w, __uint_as_float(x[e] << 16), acc[8 * v + 2 * e]);
            acc[8 * v + 2 * e + 1] =
                fmaf(w, __uint_as_float(x[e] & 0xffff0000u), acc[8 * v + 2 * e + 1]);
          }
        }
      }
    }
    if (bad && piece >= 0) {
      float4 *to = reinterpret_cast<float4 *>(a.ws_o) + (size_t)piece * (kUnitRows * D / 4);
#pragma unroll
      for (int v = 0; v < 8; ++v)
        to[sum_place<D>(r, 8 * c + v)] =
            make_float4(acc[4 * v], acc[4 * v + 1], acc[4 * v + 2], acc[4 * v + 3]);
      reinterpret_cast<float2 *>(a.ws_ml)[(size_t)piece * kUnitRows + r] = make_float2(m, l);
    } else if (bad) {
      const float f = l > 0.f ? 1.f / l : l;
      uint4 *to = reinterpret_cast<uint4 *>(out_row<D>(a, u.seq.q0, u.head, R) + 32 * c);
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        uint32_t pk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          pk[i] = pack_bf16(acc[8 * v + 2 * i] * f, acc[8 * v + 2 * i + 1] * f);
        to[v] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
      }
    }
  }
}

// Stores a warp's 32 rows (r0 ..) of a unit or a piece by way of `stage`, 64 D bytes of
// the warp's own (see the active attention's store: neighbouring lanes store neighbouring
// vectors).  True: the sums are not all finite.  `stage` is free again once lane 0 has
// waited for its bulk copies' reads.  Where the 32 rows are whole tokens, all the sequence's,
// TMA stores them as a box: by the lanes' own stores 128 dimensions took 4800 clocks.
template <int D>
__device__ __forceinline__ bool store_rows(const PackedArgs &a, const CUtensorMap *tm_o,
                                           const Unit &u, int piece, int r0, int lane, uint32_t tO,
                                           float m_run, float l_run, uint8_t *stage) {
  uint4 *st = reinterpret_cast<uint4 *>(stage);
  constexpr int kV = D / 8;
  if (piece >= 0) {
    float worst[4] = {0.f, 0.f, 0.f, 0.f};   // NaN where a sum is not finite
    // fp32, half of the dimensions at a time
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        uint32_t o[32];
        tmem_ld32(tO + half * (D / 2) + 32 * c, o);
        tmem_wait_ld();
#pragma unroll
        for (int v = 0; v < 8; ++v)
          st[lane * kV + (8 * c + (v ^ (lane & 7)))] =
              make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
#pragma unroll
        for (int i = 0; i < 32; ++i) worst[i & 3] = fmaf(__uint_as_float(o[i]), 0.f, worst[i & 3]);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        bulk_store(reinterpret_cast<uint4 *>(a.ws_o) + (size_t)piece * (kUnitRows * D / 4) +
                       (r0 / 32 * 2 + half) * (32 * kV),
                   st, 32 * kV * 16);
        if (half == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      }
      __syncwarp();
    }
    reinterpret_cast<float2 *>(a.ws_ml)[(size_t)piece * kUnitRows + r0 + lane] =
        make_float2(m_run, l_run);
    return __any_sync(0xffffffffu, (worst[0] + worst[1]) + (worst[2] + worst[3]) != 0.f) != 0;
  }
  const float inv = l_run > 0.f ? 1.f / l_run : l_run == 0.f ? 0.f : l_run;   // no keys: zeros
  const bool box = a.o_map && u.rows - r0 >= 32;
  // vector x of this lane's row: in a box 64 dimensions of all rows lie together
  auto place_of = [&](int x) {
    const int y = (x & ~7) | ((x & 7) ^ (lane & 7));
    return box ? (x >> 3) * 256 + lane * 8 + (y & 7) : lane * kV + y;
  };
  const uint64_t inv2 = pack2(__float_as_uint(inv), __float_as_uint(inv));
  const uint64_t minus0 = 0x8000000080000000ull;
  uint32_t odd2 = 0u;   // bf16 pair: NaN where a value is not finite
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    uint32_t o[64];
    tmem_ld32(tO + 64 * c, *reinterpret_cast<uint32_t(*)[32]>(&o[0]));
    tmem_ld32(tO + 64 * c + 32, *reinterpret_cast<uint32_t(*)[32]>(&o[32]));
    tmem_wait_ld();
#pragma unroll
    for (int v = 0; v < 8; ++v) {
      uint32_t pk[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t x = fma2(pack2(o[8 * v + 2 * i], o[8 * v + 2 * i + 1]), inv2, minus0);
        pk[i] = pack_bf16(lo_f(x), hi_f(x));
        asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(odd2) : "r"(pk[i]), "r"(0u));
      }
      st[place_of(8 * c + v)] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
    }
  }
  const bool odd = __any_sync(0xffffffffu, odd2 & 0x7fff7fffu) != 0;
  if (box) {
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
      const int tok = u.seq.q0 + (int)quotient(u.row0 + r0, a.group);
#pragma unroll
      for (int c = 0; c < D / 64; ++c)
        tma_store_3d(tm_o, stage + c * 4096, c * 64, u.head * (int)a.group.d, tok);
      asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
    return odd;
  }
  __syncwarp();
  // a lane works out the place of its own row, from the unit's first, in vectors
  const int rows = u.rows - r0;
  const int tok0 = quotient(u.row0, a.group), R = u.row0 + r0 + lane, tok = quotient(R, a.group);
  const int place = ((tok - tok0) * a.Hq + R - tok * (int)a.group.d) * (D / 8);
  uint4 *base = reinterpret_cast<uint4 *>(a.out) +
                ((size_t)(u.seq.q0 + tok0) * a.Hq + u.head * (int)a.group.d) * (D / 8);
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int e = 32 * i + lane, row = e / kV, v = e % kV;
    const int at = __shfl_sync(0xffffffffu, place, row);
    const uint4 x = st[row * kV + ((v & ~7) | ((v & 7) ^ (row & 7)))];
    if (row < rows) base[at + v] = x;
  }
  return odd;
}

// Sequences times K/V heads of a call at most.  Those without rows have ids all the same, and
// a block that passes over many of them, or over many sequences, keeps its other warps
// waiting for a unit: their waits are bounded (about a second, hsa_tc.cuh).
constexpr long long kMaxSequences = 1LL << 23;

// Asks for the id of a block that has not started, which then never does (cluster launch
// control); by one thread.
__device__ __forceinline__ void ask_block(uint4 *answer, uint64_t *bar) {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the last answer was read
  mbar_expect_tx(bar, 16);
  asm volatile(
      "clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128"
      " [%0], [%1];" ::"r"(smem_addr(answer)), "r"(smem_addr(bar))
      : "memory");
}
// The id once the answer is there, or -1 where no block is left: then it is not to be asked
// again.
__device__ __forceinline__ int block_of(const uint4 *answer) {
  int id;
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 lo, hi;\n .reg .b128 h;\n .reg .b32 x;\n"
      " ld.shared.v2.b64 {lo, hi}, [%1];\n mov.b128 h, {lo, hi};\n"
      " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n mov.b32 x, -1;\n"
      " @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 x, h;\n"
      " mov.b32 %0, x;\n}\n"
      : "=r"(id)
      : "r"(smem_addr(answer))
      : "memory");
  return id;
}

// Named barriers of this kernel: the start of the block; the query rows of a unit are in
// shared memory (softmax and issuing warps); the rows of Q tile t have left shared memory.
constexpr int kBarStart = 7, kBarQ = 8, kBarStored = 9;   // kBarStored + t

// A block that is one of more than two per SM (kChain) takes one unit after another: its
// own, then those of blocks that have not started yet (ask_block), so that the roles run on
// from unit to unit and the tensor pipe does not wait through a block's end and the next
// one's start.  Warp 0 works out the next unit while the present one's last tiles are
// multiplied and loads its first tiles into the slots that fall free, its query rows as soon
// as the last S no longer needs the present ones; its first S is computed beside the present
// one's store.  Units are handed over through unit_sh: bar_unit says that unit n is there,
// bar_taken that all other warps have read on to it and so are done with unit n - 1, whose
// place unit n + 1 takes.  Against a block per unit: six prompts of 503 to 5200 tokens, 32
// heads x 128 on 8, 311 -> 283 us; two of 16 frames of 384, 32 x 64, 277 -> 264; 64 prompts of
// 200 tokens, 32 x 128 on 8, 130 -> 104; 1024 of 20, 920 -> 270, mostly since a block goes
// through the sequences once.
template <int D, bool kChain>
__global__ void __launch_bounds__(kTcThreads, 1)
packed_attention_kernel(const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v,
                        const __grid_constant__ CUtensorMap tm_q,
                        const __grid_constant__ CUtensorMap tm_o,
                        const __grid_constant__ PackedArgs a) {
  using C = TcCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                            ~(uintptr_t)1023);
  uint8_t *sQ = sm;
  uint8_t *sKV = sm + kQT * C::kTileBytes;
  __shared__ __align__(8) uint64_t bar_full[C::kStages], bar_empty[C::kStages];
  __shared__ __align__(8) uint64_t bar_s[kQT * C::kSBars], bar_o[kQT];
  __shared__ __align__(8) uint64_t bar_unit, bar_taken, bar_q, bar_answer;
  __shared__ __align__(16) uint4 answer;
  __shared__ uint32_t tmem_base_sh;
  __shared__ volatile int abort_flag;
  __shared__ Unit unit_sh[2], odd_sh[2];
  __shared__ volatile int odd_flag;
  const TcPipe pipe = {bar_full, bar_empty, bar_s, bar_o, &abort_flag, a.err};

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  if (threadIdx.x == 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_v) : "memory");
    if (a.q_map) asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_q) : "memory");
    if (a.o_map) asm volatile("prefetch.tensormap [%0];" ::"l"(&tm_o) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&bar_full[s], 1);
      mbar_init(&bar_empty[s], 1);
    }
    for (int t = 0; t < kQT * C::kSBars; ++t) mbar_init(&bar_s[t], 1);
    for (int t = 0; t < kQT; ++t) mbar_init(&bar_o[t], 1);
    mbar_init(&bar_unit, 1);
    mbar_init(&bar_taken, kTcThreads / 32 - 1);
    mbar_init(&bar_q, 1);
    mbar_init(&bar_answer, 1);
    abort_flag = 0;
    odd_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  pdl_wait();

  // Unit n, once it is there; false: there is none.  All waits of warp 0 are bounded, so it
  // comes, also after a failure.
  auto take = [&](int n) {
    if (!kChain) return n == 0 && unit_sh[0].parts > 0;
    bool there = __all_sync(0xffffffffu, mbar_wait(&bar_unit, n & 1, &abort_flag, a.err, false));
    there = there && unit_sh[n & 1].parts > 0;
    __syncwarp();
    if (there && lane == 0) mbar_arrive(&bar_taken);
    return there;
  };
  TcSpan w = {0, 0, 0};
  int done = 0;   // units with keys so far

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLow));
    if (warp == 0) {
      const int withheld = a.inject_stall == 1 ? 1 : -1;
      int id = blockIdx.x, asked = 0, issued = 0;
      bool live = true;
      auto answered = [&]() -> int {   // the id that was asked for
        const bool ok = __all_sync(
            0xffffffffu, mbar_wait(&bar_answer, asked++ & 1, &abort_flag, a.err, false));
        const int x = ok ? block_of(&answer) : -1;
        return __shfl_sync(0xffffffffu, x, 0);
      };
      Window window;
      look_at(a, window, 0, 0, 0);
      Plan plan;
      plan_units(a, window, plan);
      // The unit of `id` or of a later block; parts = 0: there is none.
      auto find = [&]() {
        Unit u = {};
        while (live && id >= 0) {
          const bool busy = unit_of(a, id, plan, window, u);
          if (lane == 0 && a.most) {
            if (id == 0) a.cuts->n = plan.units - plan.n_whole;
            if (busy && u.cut >= 0 && u.part == 0)
              a.cuts->unit[u.cut] = {u.parts, u.slot, u.rows, u.row0, u.seq.q0, u.head, {0, 0}};
          }
          if (busy) break;
          u.parts = 0;
          if (!kChain) break;
          if (lane == 0) ask_block(&answer, &bar_answer);
          id = answered();
        }
        if (u.parts == 0) u.nT = 0;
        return u;
      };
      auto publish = [&](int n, const Unit &u) {   // unit n - 1 has been taken by all warps
        if (lane == 0) {
          unit_sh[n & 1] = u;
          if (kChain) mbar_arrive(&bar_unit);
        }
        __syncwarp();
      };
      Unit u;
      int from = 0;   // the unit's next load
      // The query rows: where G divides a tile's 128 rows a box of 128 / G tokens, G heads
      // and 64 dimensions is a tile's column chunk as the MMA wants it, and arrives on the
      // first K tile's barrier; rows past the sequence's last are another sequence's or
      // zeros, and are never stored.  Else the softmax warps load row by row.
      auto load_kv = [&](int L, int slot) {
        mbar_expect_tx(&bar_full[slot], C::kTileBytes * (L == 0 && a.q_map ? 1 + kQT : 1));
        uint8_t *dst = sKV + slot * C::kTileBytes;
#pragma unroll
        for (int c = 0; c < C::kChunks; ++c)
          tma_load_2d(dst + c * (kBN * 128), (L & 1) ? &tm_v : &tm_k, &bar_full[slot],
                      u.head * D + c * 64, u.seq.k0 + (u.j0 + (L >> 1)) * kBN);
      };
      auto load_q = [&]() {
        const int G = a.group.d, tok = u.seq.q0 + (int)quotient(u.row0, a.group);
        uint64_t *bar = &bar_full[w.L % C::kStages];
#pragma unroll
        for (int t = 0; t < kQT; ++t)
#pragma unroll
          for (int c = 0; c < C::kChunks; ++c)
            tma_load_3d(sQ + t * C::kTileBytes + c * (kBM * 128), &tm_q, bar, c * 64, u.head * G,
                        tok + t * (int)quotient(kBM, a.group));
      };
      auto load_to = [&](int to) {
        to = max(from, min(to, 2 * w.nT));
        if (lane == 0) live = live && tc_load<D>(pipe, w, from, to, withheld, issued, load_kv);
        from = to;
      };
      // What the unit's first S needs, before the other warps hear of the unit.
      auto begin = [&]() {
        w.nT = u.nT;
        from = 0;
        if (!done) {
          if (lane == 0 && a.q_map && w.nT) load_q();   // K_0's barrier still waits for K_0
          load_to(3);
          return;
        }
        load_to(1);
        // K_0 is on its way, so its barrier waits for the rows too: they are loaded even if
        // the wait fails
        if (lane == 0 && a.q_map && issued > w.L) {
          live = mbar_wait(&bar_q, (done - 1) & 1, &abort_flag, a.err) && live;
          load_q();
        }
      };
      u = find();
      begin();
      publish(0, u);
      named_barrier_sync(kBarStart, kTcThreads);
      for (int n = 0; u.parts; ++n) {
        if (!kChain) {
          load_to(2 * w.nT);
          break;
        }
        // The next id is asked for before the last loads, which wait for their slots, and
        // when the softmax warps have begun this unit: not sooner, since a block that took
        // units ahead would leave others without at the end (64 prompts of 200 tokens, 32
        // heads x 128 on 8: 114 -> 104 us).
        load_to(max(3, 2 * w.nT - 3));
        mbar_wait(&bar_taken, n & 1, &abort_flag, a.err, false);
        __syncwarp();
        // else the block ends: it has rows to form again
        const bool ask = __shfl_sync(0xffffffffu, odd_flag, 0) == 0;
        if (ask && lane == 0) ask_block(&answer, &bar_answer);
        load_to(2 * w.nT);
        live = __shfl_sync(0xffffffffu, live, 0);
        id = ask ? answered() : -1;
        // No block is left: the next kernel may start.  TMEM is taken by now, as in the
        // active attention.
        if (ask && id < 0) pdl_trigger();
        if (w.nT) {
          tc_pass<D>(w);
          ++done;
        }
        u = find();
        if (u.parts) begin();
        publish(n + 1, u);
      }
      if (lane == 0) tc_drain<D>(pipe, issued, withheld);
      __syncwarp();
    } else {
      if (warp == 1) {
        // TMEM after the wait and before the trigger, as in the active attention
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                         smem_addr(&tmem_base_sh)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        if (!kChain) pdl_trigger();
      }
      fence_before();
      named_barrier_sync(kBarStart, kTcThreads);
      fence_after();
      const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_sh, 0);
      for (int n = 0; take(n); ++n) {
        const Unit &u = unit_sh[n & 1];
        w.nT = __shfl_sync(0xffffffffu, u.nT, 0);
        if (w.nT == 0) continue;
        if (warp == 1) {
          if (!a.q_map) {
            named_barrier_sync(kBarQ, 256 + 32);
            fence_after();
          }
          tc_issue<D, true>(pipe, tmem, smem_addr(sQ), smem_addr(sKV), w);
        } else if (warp == 2) {
          // V rows behind the sequence's last key (another sequence's, or what lies behind
          // the last) become zeros before the issuer hears of the tile.
          const int keys = u.seq.lk - u.j0 * kBN;
          tc_watch_kv<D, true>(pipe, lane, w, [&](int j) {
            const int have = keys - j * kBN;
            if (have >= kBN) return;
            uint8_t *tile = sKV + ((w.L + 2 * j + 1) % C::kStages) * C::kTileBytes;
            for (int i = have * 8 + lane; i < kBN * 8; i += 32)
#pragma unroll
              for (int c = 0; c < C::kChunks; ++c)
                *reinterpret_cast<uint4 *>(tile + c * (kBN * 128) + 16 * i) =
                    make_uint4(0u, 0u, 0u, 0u);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          });
        } else {
          tc_watch_s<D>(pipe, w);
          if (lane == 0) mbar_arrive(&bar_q);   // the last S has read the query rows
        }
        tc_pass<D>(w);
        ++done;
      }
      // TMEM is quiet before it is freed, also after a failure
      if (warp == 1 && done) mbar_wait(&bar_o[1], (done - 1) & 1, &abort_flag, a.err, false);
      __syncwarp();
    }
    fence_before();
    named_barrier_sync(kBarTeardown, kTcThreads);
    if (warp == 1) {
      fence_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base_sh),
                   "r"(kTmemCols)
                   : "memory");
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsHigh));
    fence_before();
    named_barrier_sync(kBarStart, kTcThreads);
    fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_sh, 0);
    const int t = (warp - 4) >> 2;
    const int wq = warp & 3;
    const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
    const uint32_t tO = tmem + lane_off + C::kOCol0 + D * t;
    const float sl2 = a.scale_log2;
    unsigned odd = 0;   // bit n & 1: rows of unit n are to be formed again
    for (int n = 0; take(n); ++n) {
      // Read where it is needed: held in registers over the key loop it would spill, to an
      // L1 that the tiles have left no room in.
      const Unit &u = unit_sh[n & 1];
      w.nT = __shfl_sync(0xffffffffu, u.nT, 0);
      if (w.nT == 0) {   // no row has keys
        for (int i = threadIdx.x - 128; i < u.rows * (D / 8); i += 256)
          *reinterpret_cast<uint4 *>(out_row<D>(a, u.seq.q0, u.head, u.row0 + i / (D / 8)) +
                                     8 * (i % (D / 8))) =
              make_uint4(0u, 0u, 0u, 0u);
        continue;
      }
      if (!a.q_map) {
        // These warps have stored the unit before, so its products are done.  The addresses
        // first, then the loads together, in two halves.
        constexpr int kVecPerRow = D / 8, kPer = kUnitRows * kVecPerRow / 256 / 2;
        const int G = a.group.d;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint4 *src[kPer];
          uint4 v[kPer];
          const int i0 = threadIdx.x - 128 + half * (kPer * 256);
#pragma unroll
          for (int x = 0; x < kPer; ++x) {
            const int i = i0 + x * 256, R = u.row0 + i / kVecPerRow, tok = quotient(R, a.group);
            src[x] = reinterpret_cast<const uint4 *>(a.q + (size_t)(u.seq.q0 + tok) * a.q_row +
                                                     (u.head * G + (R - tok * G)) * D) +
                     i % kVecPerRow;
          }
#pragma unroll
          for (int x = 0; x < kPer; ++x) {
            v[x] = make_uint4(0u, 0u, 0u, 0u);
            if ((i0 + x * 256) / kVecPerRow < u.rows)
              asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                           : "=r"(v[x].x), "=r"(v[x].y), "=r"(v[x].z), "=r"(v[x].w)
                           : "l"(src[x]));
          }
#pragma unroll
          for (int x = 0; x < kPer; ++x) {
            const int i = i0 + x * 256, row = i / kVecPerRow, c = i % kVecPerRow;
            const int rr = row % kBM;
            *reinterpret_cast<uint4 *>(sQ + (row / kBM) * C::kTileBytes + (c >> 3) * (kBM * 128) +
                                       rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) = v[x];
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        fence_before();
        named_barrier_sync(kBarQ, 256 + 32);
      }
      float m_run = kLowest, l_run = 0.f;
      // Keys from the next tile on that this thread's row sees; rows past the sequence's last
      // take no mask.  The warp's first row sees fewest.
      const int r = t * kBM + wq * 32 + lane;
      int limit = (r < u.rows ? key_limit(a, u.seq, quotient(u.row0 + r, a.group)) : u.seq.lk) -
                  u.j0 * kBN;
      int all_see = __shfl_sync(0xffffffffu, limit, 0);
      const int end = w.J + w.nT;
      for (int j = w.J; j < end; ++j) {
        named_barrier_sync(kBarS0 + t, kMeetS);
        fence_after();
        const uint32_t tSj = tmem + lane_off + 128 * (C::kThreeS ? (2 * j + t) % 3 : t);
        auto o_idle = [&]() -> bool {   // as in the active attention
          if constexpr (!C::kThreeS) return true;
          uint64_t *b = t == 0 ? &bar_s[2 + (j & 1)] : &bar_s[(j + 1) & 1];
          const uint32_t par = t == 0 ? (j >> 1) & 1 : ((j + 1) >> 1) & 1;
          const bool idle = __all_sync(0xffffffffu, mbar_wait(b, par, &abort_flag, a.err));
          fence_after();
          return idle;
        };
        if (all_see >= kBN)
          softmax_tile<D, false>(tSj, tO, kBN, j == w.J, sl2, m_run, l_run, o_idle);
        else
          softmax_tile<D, true>(tSj, tO, limit, j == w.J, sl2, m_run, l_run, o_idle);
        limit -= kBN;
        all_see -= kBN;
        tmem_wait_st();
        fence_before();
        named_barrier_sync(kBarP0 + t, kMeetP);
      }
      bool ok = __all_sync(0xffffffffu, mbar_wait(&bar_o[t], done & 1, &abort_flag, a.err));
      ok = !__any_sync(0xffffffffu, abort_flag != 0) && ok;
      // by way of the unit's last K (t = 0) or V slot, which this group then gives back
      const int slot = (w.L + 2 * w.nT - 2 + t) % C::kStages;
      if (ok) {
        fence_after();
        const int piece = u.parts > 1 ? u.slot + u.part : -1;
        if (store_rows<D>(a, &tm_o, u, piece, t * kBM + wq * 32, lane, tO, m_run, l_run,
                          sKV + slot * C::kTileBytes + wq * (C::kTileBytes / 4)) &&
            a.mask) {
          // Forming rows again may take longer than the other roles wait for one another, so
          // it is left until they have ended.  The unit after this one may have been handed
          // over already, no other follows.
          odd |= 1u << (n & 1);
          if (lane == 0) {
            odd_sh[n & 1] = u;
            odd_flag = 1;
          }
          __syncwarp();
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        fence_before();
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
      }
      if (kChain) {
        named_barrier_sync(kBarStored + t, kBM);
        if (ok && wq == 0 && lane == 0) mbar_arrive(&bar_empty[slot]);
      }
      tc_pass<D>(w);
      ++done;
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    if (a.mask) {
      named_barrier_sync(kBarQ, 256);   // all stores have left shared memory
      if (odd) {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
#pragma unroll 1
        for (int i = 0; i < 2; ++i)
          if (odd >> i & 1)
            form_again<D>(a, odd_sh[i], t * kBM + wq * 32 + lane,
                          reinterpret_cast<uint4 *>(sKV + (warp - 4) * (C::kTileBytes / 4)));
      }
    }
    fence_before();
    named_barrier_sync(kBarTeardown, kTcThreads);
  }
}

// Joins the parts of the units that were cut.  A row takes D/4 lanes, four dimensions
// each, and where there are many parts all lane groups of the block share a row: bound by
// the round trips to L2, each group loads four parts at once.  The blocks divide the cut
// units' rows into runs.
constexpr int kJoinThreads = 256;

template <int D>
__global__ void __launch_bounds__(kJoinThreads)
packed_join_kernel(const PackedArgs a) {
  constexpr int kL = D / 4, kGroups = kJoinThreads / kL;
  __shared__ float4 sh_o[kJoinThreads];
  __shared__ float2 sh_ml[kGroups];
  pdl_wait();
  pdl_trigger();
  const int n = a.cuts->n * kUnitRows;
  const int i0 = (int)((long long)n * blockIdx.x / gridDim.x);
  const int i1 = (int)((long long)n * (blockIdx.x + 1) / gridDim.x);
  const int sub = threadIdx.x % kL, group = threadIdx.x / kL;
  for (int i = i0; i < i1;) {
    const int tail = i / kUnitRows, end = min(i1, (tail + 1) * kUnitRows);
    const CutUnit u = a.cuts->unit[tail];
    int r = i - tail * kUnitRows;
    const int r1 = u.parts > 1 ? min(end - tail * kUnitRows, u.rows) : 0;
    i = end;
    const bool wide = u.parts > 8;                 // the block's groups share a row
    for (; r < r1; r += wide ? 1 : kGroups) {
      const int row = wide ? r : r + group;
      float M = kLowest, L = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row < r1) {
        const size_t at = (size_t)u.slot * kUnitRows + row;
        const float2 *ml = reinterpret_cast<const float2 *>(a.ws_ml) + at;
        const float4 *o = reinterpret_cast<const float4 *>(a.ws_o) +
                          (size_t)u.slot * (kUnitRows * kL) + sum_place<D>(row, sub);
        const int step = wide ? kGroups : 1;
        for (int p0 = wide ? group : 0; p0 < u.parts; p0 += 4 * step) {
          float2 w[4];
          float4 x[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int p = p0 + y * step;
            w[y] = make_float2(kLowest, 0.f);
            x[y] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (p < u.parts) {
              w[y] = ml[(size_t)p * kUnitRows];
              x[y] = o[(size_t)p * kUnitRows * kL];
            }
          }
          const float to = fmaxf(fmaxf(fmaxf(w[0].x, w[1].x), fmaxf(w[2].x, w[3].x)), M);
          const float f0 = fast_exp2(M - to);
          M = to;
          L *= f0, acc.x *= f0, acc.y *= f0, acc.z *= f0, acc.w *= f0;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const float f = fast_exp2(w[y].x - M);
            L = fmaf(f, w[y].y, L);
            acc.x = fmaf(f, x[y].x, acc.x);
            acc.y = fmaf(f, x[y].y, acc.y);
            acc.z = fmaf(f, x[y].z, acc.z);
            acc.w = fmaf(f, x[y].w, acc.w);
          }
        }
      }
      if (wide) {                                  // the same in the whole block
        sh_o[threadIdx.x] = acc;
        if (sub == 0) sh_ml[group] = make_float2(M, L);
        __syncthreads();
        if (group == 0) {
#pragma unroll
          for (int y = 0; y < kGroups; ++y) M = fmaxf(M, sh_ml[y].x);
          L = 0.f;
          acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int y = 0; y < kGroups; ++y) {
            const float2 w = sh_ml[y];
            const float4 x = sh_o[y * kL + sub];
            const float f = fast_exp2(w.x - M);
            L = fmaf(f, w.y, L);
            acc.x = fmaf(f, x.x, acc.x);
            acc.y = fmaf(f, x.y, acc.y);
            acc.z = fmaf(f, x.z, acc.z);
            acc.w = fmaf(f, x.w, acc.w);
          }
        }
        __syncthreads();
      }
      if (row < r1 && (!wide || group == 0)) {
        const float inv = L > 0.f ? 1.f / L : L == 0.f ? 0.f : L;
        reinterpret_cast<uint2 *>(out_row<D>(a, u.q0, u.head, u.row0 + row))[sub] =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
      }
    }
  }
}

// -------------------------------------------------------------- host side

// 3-D map over N tokens of H heads x D bf16 values, the tokens `row` elements apart: boxes
// of `tokens` x `heads` x 64 dimensions, 128-byte swizzle, tokens past N read as zero.
bool make_rows_map(CUtensorMap *map, const void *base, int N, int H, int D, long long row,
                   int heads, int tokens) {
  auto enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)H, (cuuint64_t)N};
  const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)row * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)tokens};
  const cuuint32_t estride[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box,
             estride, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool kChain>
int configure(int dev) {
  static std::atomic<int> configured[64];
  if (configured[dev].load()) return HSA_OK;
  auto kernel = packed_attention_kernel<D, kChain>;
  // the register hand-over assumes exactly kLaunchRegs registers at launch
  cudaFuncAttributes fa;
  if (cudaFuncGetAttributes(&fa, kernel) != cudaSuccess) return HSA_ERR_CUDA;
  if (fa.numRegs != kLaunchRegs || fa.maxThreadsPerBlock < kTcThreads) return HSA_ERR_UNSUPPORTED;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, TcCfg<D>::kSmem) !=
      cudaSuccess)
    return HSA_ERR_CUDA;
  configured[dev].store(1);
  return HSA_OK;
}

template <int D>
int launch(PackedArgs &a, const void *any, cudaStream_t stream) {
  using C = TcCfg<D>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return HSA_ERR_CUDA;
  CUtensorMap mk, mv, mq, mo;
  // without keys no tile is loaded: any valid map serves
  const int keys = std::max(a.total_k, 1);
  if (!make_kv_map(&mk, a.total_k ? a.k : any, keys, a.Hkv * D,
                   a.total_k ? a.k_row : (long long)a.Hkv * D) ||
      !make_kv_map(&mv, a.total_k ? a.v : any, keys, a.Hkv * D,
                   a.total_k ? a.v_row : (long long)a.Hkv * D))
    return HSA_ERR_CUDA;
  // A box of the query tensor [total_q, Hq, D] is a Q tile where G divides its rows.
  const int G = (int)a.group.d;
  a.q_map = kBM % G == 0;
  if (a.q_map && !make_rows_map(&mq, a.q, a.total_q, a.Hq, D, a.q_row, G, kBM / G))
    return HSA_ERR_CUDA;
  if (!a.q_map) mq = mk;
  // and a warp's 32 rows are a box of the output
  a.o_map = 32 % G == 0;
  if (a.o_map &&
      !make_rows_map(&mo, a.out, a.total_q, a.Hq, D, (long long)a.Hq * D, G, 32 / G))
    return HSA_ERR_CUDA;
  if (!a.o_map) mo = mk;
  // Units at most: every sequence has at most one partly filled block.  How many there are
  // is on the device, so the grid holds what a cut may make of them: a block too many costs
  // about a microsecond of an SM.  Fewer units than SMs become at most sms parts, or 2 sms
  // where they are too many for a part each; without a mask pieces of the last wave's
  // units come on top of the others.  Too few keys for a cut to pay: no join.
  const long long units = ((long long)a.total_q * a.group.d / kUnitRows + a.batch) * a.Hkv;
  if (a.total_k <= (kLeastTiles + kJoinTiles) * kBN) a.most = 0;
  if (a.most) a.most = 2 * units <= a.sms || (a.mask && units >= a.sms) ? a.sms : 2 * a.sms;
  const long long grid =
      a.mask || units < a.sms ? std::max<long long>(units, a.most) : units + a.most;
  if (grid > 0x7fffffffLL) return HSA_ERR_UNSUPPORTED;
  a.bound = (int)units;
  // Two waves of blocks of one unit are as fast as a chain of two units, and a block that
  // takes no other starts 0.6 us sooner (two prompts of 3000 to 6000 tokens, 8 heads x 128 on
  // 2: 78 against 79 us; 2000 tokens, 16 x 128 on 2: 30 against 32).
  const bool chain = grid > 2LL * a.sms;
  const int st = chain ? configure<D, true>(dev) : configure<D, false>(dev);
  if (st != HSA_OK) return st;
  count_launches(a.most ? 2 : 1);
  launch_pdl(chain ? packed_attention_kernel<D, true> : packed_attention_kernel<D, false>,
             dim3((unsigned)grid), dim3(kTcThreads), C::kSmem, stream, mk, mv, mq, mo,
             a);
  if (cudaGetLastError() != cudaSuccess) return HSA_ERR_CUDA;
  if (a.most)
    launch_pdl(packed_join_kernel<D>, dim3((unsigned)(8 * a.sms)), dim3(kJoinThreads), 0, stream,
               a);
  return launch_status();
}

size_t workspace_bytes(int D) {
  return 2 * (size_t)sm_count() * kUnitRows * ((size_t)D * 4 + 8) +
         ((size_t)sm_count() + 1) * sizeof(CutUnit);
}

}  // namespace
}  // namespace hsa

using namespace hsa;

extern "C" size_t hsa_packed_attention_workspace_bytes(int Hq, int Hkv, int D) {
  if (Hq <= 0 || Hkv <= 0 || Hq % Hkv || (D != 64 && D != 128)) return 0;
  return workspace_bytes(D);
}

extern "C" int hsa_packed_attention(const void *q, long long q_row, const void *k, long long k_row,
                                    const void *v, long long v_row, const int32_t *cu_q,
                                    const int32_t *cu_k, int batch, int total_q, int total_k,
                                    int Hq, int Hkv, int D, int mask, float scale, void *out,
                                    hsa_dtype dtype, void *workspace, size_t workspace_size,
                                    hsa_stream_t stream) {
  if (batch < 0 || total_q < 0 || total_k < 0 || Hq < 1 || Hkv < 1 || Hq % Hkv || mask < 0)
    return HSA_ERR_INVALID_ARG;
  if (dtype != HSA_BF16 && dtype != HSA_F32) return HSA_ERR_INVALID_ARG;
  if (dtype == HSA_F32 || (D != 64 && D != 128) || (long long)Hq * D > (1LL << 24))
    return HSA_ERR_UNSUPPORTED;
  if ((long long)batch * Hkv > kMaxSequences || total_k > 0x7fffff00 ||
      (long long)total_q * (Hq / Hkv) > 0x7fffff00LL)
    return HSA_ERR_UNSUPPORTED;
  if (q_row < (long long)Hq * D || k_row < (long long)Hkv * D || v_row < (long long)Hkv * D ||
      (q_row & 7) || (k_row & 7) || (v_row & 7) || q_row > (1LL << 31) || k_row > (1LL << 31) ||
      v_row > (1LL << 31))
    return HSA_ERR_INVALID_ARG;
  if (batch == 0 || total_q == 0) return HSA_OK;
  if (!q || !out || !cu_q || !cu_k || !aligned16(q) || !aligned16(out)) return HSA_ERR_INVALID_ARG;
  if (total_k > 0 && (!k || !v || !aligned16(k) || !aligned16(v))) return HSA_ERR_INVALID_ARG;
  PackedArgs a;
  a.sms = sm_count();
  a.most = 0;
  a.ws_o = a.ws_ml = nullptr;
  a.cuts = nullptr;
  if (workspace) {
    if (workspace_size < workspace_bytes(D) || !aligned16(workspace)) return HSA_ERR_WORKSPACE;
    a.most = 1;
    a.ws_o = static_cast<float *>(workspace);
    a.ws_ml = a.ws_o + 2 * (size_t)a.sms * kUnitRows * D;
    a.cuts = reinterpret_cast<Cuts *>(a.ws_ml + 2 * (size_t)a.sms * kUnitRows * 2);
  }
  if (!(scale > 0.f) || !std::isfinite(scale)) scale = 1.f / std::sqrt((float)D);
  a.q = static_cast<const __nv_bfloat16 *>(q);
  a.k = static_cast<const __nv_bfloat16 *>(k);
  a.v = static_cast<const __nv_bfloat16 *>(v);
  a.out = static_cast<__nv_bfloat16 *>(out);
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  a.err = device_error_word();
  if (!a.err) return HSA_ERR_CUDA;
  a.batch = batch;
  a.total_q = total_q;
  a.total_k = total_k;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.group = make_divider((unsigned)(Hq / Hkv));
  a.frame = make_divider((unsigned)std::max(mask, 1));
  a.mask = mask;
  a.q_row = q_row;
  a.k_row = k_row;
  a.v_row = v_row;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.inject_stall = attention_stall();
  cudaStream_t s = (cudaStream_t)stream;
  return D == 128 ? launch<128>(a, q, s) : launch<64>(a, q, s);
}

// Active-query full-context attention (Sec. 2.3, step 3): the |A_i| active
// queries attend to all N rows of the layer's KV cache, O(|A_i| N) work.
//
// bf16 path: one CTA owns 256 active query rows (two 128-row Q tiles) of one
// head and streams every 128-key tile of that head's keys through shared
// memory.  The keys are the rows of up to two sources read in order: the KV
// cache, then (token reordering, Sec. 2.5) the fresh K/V of the baseline
// group, which is active at every iteration and so needs no cache.  Warp roles:
//   warp 0      TMA producer: K and V tiles of the head, 128-byte swizzled,
//               into a ring of shared-memory slots (rows >= N are zero-filled).
//   warp 1      tensor-core issuer (one lane issues, the warp walks the
//               schedule): S_t = Q_t K^T into TMEM and O_t += P_t V from TMEM
//               P and shared V, tcgen05.mma kind::f16.
//   warp 2      K/V watcher: waits for the K/V tiles to land, hands them to
//               the issuer at the P meetings, and gives ring slots back to
//               the producer.
//   warp 3      S watcher: waits for each S tile to complete and meets its
//               softmax group.
//   warps 4-7   softmax of Q tile 0, warps 8-11 softmax of Q tile 1: each
//               thread owns one query row (its TMEM lane; a warp may only
//               reach the lane quarter warp%4), reads its S row,
//               keeps the running maximum and sum, writes P as bf16 back into
//               the S columns, and at the end normalises O and stores it.
//   all warps   load the 256 query rows once, by index, into swizzled smem.
// The two Q tiles ping-pong: while one softmax group works on its scores the
// tensor core runs the other tile's MMAs.  At D = 64 the TMEM also has room for
// a third S buffer, so each Q tile's next scores are computed while its softmax
// still works on the current ones.  The issuer waits only on hardware
// named barriers, two per key tile (P of a tile, with the K/V tiles the next
// MMAs read), where the other roles meet it; an mbarrier test on its path
// would idle the tensor core.  Units of odd waves walk their keys backwards
// (so they start on the tiles the previous wave of the head read last, still
// in L2), and the query and output rows, read and written once, are marked
// for early L2 eviction.  After the
// first key tile the probabilities are formed against the running reference
// maximum without computing the tile's maximum; only if a row sum would pass
// 2^32 is the tile redone with its exact maximum (and O rescaled in TMEM).
// The final division by the running sum makes the result exact whatever
// reference was used.
// Registers: the block launches at 168 per thread; the first warpgroup then
// gives registers back (setmaxnreg.dec to 96) and the two softmax warpgroups
// take them (setmaxnreg.inc to 200): 128*96 + 256*200 <= 384*168.
// Every mbarrier wait is bounded in time; on a timeout the kernel records
// HSA_ERR_TIMEOUT, stops loading K/V tiles and waiting for them, lets the MMA
// schedule run out over whatever the buffers hold, drains its own copies and
// MMAs, frees TMEM and returns.
//
// fp32 calls go to hsa_attention_f32.cu.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cmath>

#include "hsa_internal.cuh"
#include "hsa_ptx.cuh"
#include "hsa_tc.cuh"
#include "hsa_test.h"

namespace hsa {
namespace {

struct TcArgs {
  const __nv_bfloat16 *q;
  const int32_t *q_idx;
  __nv_bfloat16 *out;
  unsigned *err;
  int n_active, N, H, q_rows, n_kv_tiles;
  int rows1, rows2, tiles1;   // key sources: rows1 cache rows, then rows2 rows
  float scale_log2;
  int inject_stall;   // test hook (hsa_test.h): 1 = the first V tile is never loaded
  // Work split.  CTA b < n_whole owns unit b (head b / n_qblocks, query block
  // b % n_qblocks) over all key tiles.  Every later CTA owns one of `pieces`
  // key ranges of a tail unit and writes its unnormalised O, running maximum
  // and sum to ws_o / ws_ml for the combine kernel.
  int n_qblocks, n_whole, pieces;
  int wave;           // CTAs resident at once (one per SM): the length of a wave
  float *ws_o;        // [piece CTA][kQT*kBM rows][D] fp32
  float *ws_ml;       // [piece CTA][kQT*kBM rows][2] fp32: m (log2 units), l
};

// Key-tile range [j0, j1) and unit of CTA b.
struct CtaWork {
  int head, row0, j0, j1, piece;   // piece = -1 for a whole unit
};

__host__ __device__ inline CtaWork cta_work(int b, int n_qblocks, int n_whole, int pieces,
                                            int n_kv_tiles) {
  CtaWork w;
  int unit;
  if (b < n_whole) {
    unit = b;
    w.j0 = 0;
    w.j1 = n_kv_tiles;
    w.piece = -1;
  } else {
    const int pi = b - n_whole;
    unit = n_whole + pi / pieces;
    const int k = pi % pieces;
    w.j0 = (int)((long long)n_kv_tiles * k / pieces);
    w.j1 = (int)((long long)n_kv_tiles * (k + 1) / pieces);
    w.piece = pi;
  }
  w.head = unit / n_qblocks;
  w.row0 = (unit % n_qblocks) * (kBM * kQT);
  return w;
}

// Stores 32 finished rows of a unit (r0 .. r0+31 of its kQT*kBM; this lane holds
// row r0 + lane in TMEM columns tO ..), or of a piece of a split unit
// (unnormalised O, maximum and sum, for the combine), by way of `stage`, 32 * D
// floats of the warp's own.  A lane's row there is a run of 16-byte vectors, their
// order turned by the row so that the 8 lanes of a quarter-warp use distinct banks.
// A lane that stores its own row touches 32 lines per instruction: 2000 clocks per
// unit at D = 64, 4000 for a piece or at D = 128, on the one path to the L1.
template <int D>
__device__ __forceinline__ void store_rows(const TcArgs &a, const CtaWork &wk, int r0, int lane,
                                           uint32_t tO, float m_run, float l_run,
                                           uint8_t *stage) {
  const bool piece = wk.piece >= 0;
  const float inv = 1.f / l_run;
  uint4 *st = reinterpret_cast<uint4 *>(stage);
  if (piece) {
    constexpr int kV = D / 4;                      // vectors per row
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tmem_ld32(tO + 32 * c, o);
      tmem_wait_ld();
#pragma unroll
      for (int v = 0; v < 8; ++v)
        st[lane * kV + (8 * c + (v ^ (lane & 7)))] =
            make_uint4(o[4 * v], o[4 * v + 1], o[4 * v + 2], o[4 * v + 3]);
    }
    __syncwarp();
    uint4 *dst = reinterpret_cast<uint4 *>(a.ws_o) +
                 ((size_t)wk.piece * (kQT * kBM) + r0) * kV;
#pragma unroll 8
    for (int i = 0; i < kV; ++i) {
      const int e = 32 * i + lane, row = e / kV, v = e % kV;
      dst[e] = st[row * kV + ((v & ~7) | ((v & 7) ^ (row & 7)))];
    }
    reinterpret_cast<float2 *>(a.ws_ml)[(size_t)wk.piece * (kQT * kBM) + r0 + lane] =
        make_float2(m_run, l_run);
    return;
  }
  constexpr int kV = D / 8;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    uint32_t o[32];
    tmem_ld32(tO + 32 * c, o);
    tmem_wait_ld();
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      uint32_t pk[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        pk[i] = pack_bf16(__uint_as_float(o[8 * v + 2 * i]) * inv,
                          __uint_as_float(o[8 * v + 2 * i + 1]) * inv);
      const int u = 4 * c + v;                     // vector of the row
      st[lane * kV + ((u & ~7) | ((u & 7) ^ (lane & 7)))] = make_uint4(pk[0], pk[1], pk[2], pk[3]);
    }
  }
  __syncwarp();
  uint64_t pol;                 // the output rows are written once: evict first
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int e = 32 * i + lane, row = e / kV, v = e % kV;
    const int grow = wk.row0 + r0 + row;
    const uint4 x = st[row * kV + ((v & ~7) | ((v & 7) ^ (row & 7)))];
    if (grow < a.n_active)
      asm volatile("st.global.L2::cache_hint.v4.u32 [%0], {%1,%2,%3,%4}, %5;" ::"l"(
                       a.out + ((size_t)grow * a.H + wk.head) * D + 8 * v),
                   "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w), "l"(pol)
                   : "memory");
  }
}

template <int D>
__global__ void __launch_bounds__(kTcThreads, 1)
attn_tc_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
               const __grid_constant__ CUtensorMap tm_k2, const __grid_constant__ CUtensorMap tm_v2,
               const TcArgs a) {
  using C = TcCfg<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                            ~(uintptr_t)1023);
  uint8_t *sQ = sm;
  uint8_t *sKV = sm + kQT * C::kTileBytes;
  __shared__ __align__(8) uint64_t bar_full[C::kStages], bar_empty[C::kStages];
  __shared__ __align__(8) uint64_t bar_s[kQT * C::kSBars], bar_o;
  __shared__ uint32_t tmem_base_sh;
  __shared__ volatile int abort_flag;
  const TcPipe pipe = {bar_full, bar_empty, bar_s, &bar_o, &abort_flag, a.err};

  // the same in every lane, and read from one: branches on it and what is
  // computed under them stay uniform for the compiler
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const CtaWork wk = cta_work(blockIdx.x, a.n_qblocks, a.n_whole, a.pieces, a.n_kv_tiles);
  const int h = wk.head;
  const int row0 = wk.row0;
  const int j0 = wk.j0;
  const int nT = wk.j1 - wk.j0;        // key tiles of this CTA (local index j = 0..nT-1)
  // Key order of the unit.  Whole units of odd "waves" (blocks [k*sms,
  // (k+1)*sms) for odd k) walk the keys backwards, so they start on the key
  // tiles the previous wave's units of the same head read last, which are
  // still in L2.  The order of the keys does not change the result (up to
  // rounding): the softmax is accumulated online.
  const bool rev = wk.piece < 0 && ((blockIdx.x / a.wave) & 1);
  auto key_tile = [&](int j) { return rev ? wk.j1 - 1 - j : j0 + j; };

  // K or V tile L/2 of this unit's key range (L even: K, odd: V) into its
  // ring slot, completing on bar_full.  Issued by thread 0, the producer.
  auto load_kv = [&](int L) {
    const int slot = L % C::kStages;
    mbar_expect_tx(&bar_full[slot], C::kTileBytes);
    const int jg = key_tile(L >> 1);                // global key tile
    const bool second = jg >= a.tiles1;
    const CUtensorMap *map = second ? ((L & 1) ? &tm_v2 : &tm_k2) : ((L & 1) ? &tm_v : &tm_k);
    const int y = (second ? jg - a.tiles1 : jg) * kBN;
    uint8_t *dst = sKV + slot * C::kTileBytes;
#pragma unroll
    for (int c = 0; c < C::kChunks; ++c)
      tma_load_2d(dst + c * (kBN * 128), map, &bar_full[slot], h * D + c * 64, y);
  };
  const int withheld = a.inject_stall == 1 ? 1 : -1;   // test hook: V of tile 0 never loads
  const int n_pre = min(3, 2 * nT);                   // loads issued before the Q tile: K_0 V_0 K_1
  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&bar_full[s], 1);
      mbar_init(&bar_empty[s], 1);
    }
    for (int t = 0; t < kQT * C::kSBars; ++t) mbar_init(&bar_s[t], 1);
    mbar_init(&bar_o, 1);
    abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // Launched with programmatic dependent launch: up to here the block touches
  // only its own shared memory, and runs beside the end of the kernel before it;
  // wait for that kernel and those before it (the KV scatter writes the keys read
  // below).  TMEM is taken after the wait, never before: a block that held it while
  // waiting could keep it from a block of that kernel (another library's, which lets
  // its dependents start before it allocates) on the same SM, and each would wait
  // for the other.  For the same reason the next kernel may start only once this
  // block has its own.  The blocks of the last wave let it start launching onto the
  // SMs they free; no block of this grid is still waiting for an SM by then.
  pdl_wait();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_addr(&tmem_base_sh)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    if (blockIdx.x + (unsigned)a.wave >= gridDim.x) pdl_trigger();
  }
  // The first key tiles load while the CTA loads its query rows below, and no
  // more than the first MMAs need: a whole ring's worth on every SM at once held
  // the query rows up for 2000 clocks.
  if (threadIdx.x == 0)
    for (int L = 0; L < n_pre; ++L)
      if (L != withheld) load_kv(L);

  // ---- query rows, by index, into the two swizzled Q tiles (all threads)
  // Each thread first reads the indices of all its rows, then issues all its
  // 16-byte loads, then stores them: two dependent round trips to memory in
  // all rather than two per vector.
  {
    constexpr int kVecPerRow = D / 8;                        // 16-byte vectors per row
    constexpr int kVecs = kBM * kQT * kVecPerRow;
    constexpr int kPer = (kVecs + kTcThreads - 1) / kTcThreads;
    const size_t row_stride = (size_t)a.H * D;
    int src[kPer];
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = threadIdx.x + u * kTcThreads;
      const int grow = row0 + i / kVecPerRow;
      src[u] = -1;
      if (i < kVecs && grow < a.n_active) src[u] = a.q_idx ? __ldg(a.q_idx + grow) : grow;
    }
    uint4 v[kPer];
    uint64_t pol;                       // the query rows are read once: evict first
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = threadIdx.x + u * kTcThreads;
      v[u] = make_uint4(0u, 0u, 0u, 0u);
      if (src[u] >= 0 && src[u] < a.q_rows) {
        const uint4 *p = reinterpret_cast<const uint4 *>(a.q + (size_t)src[u] * row_stride +
                                                         (size_t)h * D) + i % kVecPerRow;
        asm volatile("ld.global.nc.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;"
                     : "=r"(v[u].x), "=r"(v[u].y), "=r"(v[u].z), "=r"(v[u].w)
                     : "l"(p), "l"(pol));
      }
      else if (i < kVecs && row0 + i / kVecPerRow < a.n_active && i % kVecPerRow == 0)
        set_error(a.err, kErrIndex);
    }
#pragma unroll
    for (int u = 0; u < kPer; ++u) {
      const int i = threadIdx.x + u * kTcThreads;
      if (i < kVecs) {
        const int row = i / kVecPerRow, c = i % kVecPerRow;
        const int t = row / kBM, rr = row % kBM;
        uint8_t *dst = sQ + t * C::kTileBytes + (c >> 3) * (kBM * 128) + rr * 128 +
                       (((c & 7) ^ (rr & 7)) << 4);
        *reinterpret_cast<uint4 *>(dst) = v[u];
      }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_base_sh, 0);

  // The warpgroups' code paths never rejoin below: each ends with its own
  // teardown on named barrier 1, so each path is compiled for its own
  // register budget.

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsLow));
    if (warp == 0) {
      tc_produce<D>(pipe, lane, nT, n_pre, withheld, load_kv);
    } else if (warp == 1) {
      tc_issue<D>(pipe, tmem, smem_addr(sQ), smem_addr(sKV), {0, 0, nT});
    } else if (warp == 2) {
      tc_watch_kv<D>(pipe, lane, {0, 0, nT}, [](int) {});
    } else if (warp == 3) {
      tc_watch_s<D>(pipe, {0, 0, nT});
    }
    fence_before();
    named_barrier_sync(kBarTeardown, kTcThreads);
    if (warp == 1) {
      fence_after();
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                   "r"(kTmemCols)
                   : "memory");
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsHigh));
    // ------------------------------------------------ softmax / epilogue
    const int t = (warp - 4) >> 2;
    const int wq = warp & 3;                       // TMEM lane quarter of this warp
    const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
    const uint32_t tS = tmem + lane_off + 128 * t;
    const uint32_t tO = tmem + lane_off + C::kOCol0 + D * t;
    const float sl2 = a.scale_log2;
    float m_run = -INFINITY, l_run = 0.f;
    // The S watcher and the issuer are met for every key tile whatever happens,
    // so all their syncs complete: after a failed wait the tiles are formed from
    // whatever TMEM holds, and the abort flag, read before the rows are stored,
    // keeps them from being written.  Meeting the issuer (rather than arriving)
    // costs nothing: S_t(j+1) is issued only after the issuer has passed this
    // meeting for P_t(j).
    for (int j = 0; j < nT; ++j) {
      named_barrier_sync(kBarS0 + t, kMeetS);      // S_t(j) is complete
      fence_after();
      const int jg = key_tile(j);                // keys of this tile that exist
      const int valid = jg < a.tiles1 ? a.rows1 - jg * kBN : a.rows2 - (jg - a.tiles1) * kBN;
      // three S buffers (D = 64): S_t(j) is the (2j + t)-th S MMA
      const uint32_t tSj = C::kThreeS ? tmem + lane_off + 128 * ((2 * j + t) % 3) : tS;
      // O_t(j-1) has completed once an MMA issued after it has.  With two
      // S buffers that is S_t(j), complete already.  With three, S_t(j) is
      // issued before O_t(j-1): wait for S_1(j) (Q tile 0) or S_0(j+1) (Q
      // tile 1; at the last key tile the issuer commits that barrier with
      // no MMA).  Neither barrier can complete again before this warp's
      // next meeting.  Needed only on the exact path's rescale, so rare.
      auto o_idle = [&]() -> bool {
        if constexpr (!C::kThreeS) return true;
        uint64_t *b = t == 0 ? &bar_s[2 + (j & 1)] : &bar_s[(j + 1) & 1];
        const uint32_t par = t == 0 ? (j >> 1) & 1 : ((j + 1) >> 1) & 1;
        const bool idle = __all_sync(0xffffffffu, mbar_wait(b, par, &abort_flag, a.err));
        fence_after();
        return idle;
      };
      if (valid >= kBN)
        softmax_tile<D, false>(tSj, tO, valid, j == 0, sl2, m_run, l_run, o_idle);
      else
        softmax_tile<D, true>(tSj, tO, valid, j == 0, sl2, m_run, l_run, o_idle);
      tmem_wait_st();
      fence_before();
      named_barrier_sync(kBarP0 + t, kMeetP);
    }
    // warp-uniform: the loads below span the warp
    bool ok = __all_sync(0xffffffffu, mbar_wait(&bar_o, 0, &abort_flag, a.err));
    ok = !__any_sync(0xffffffffu, abort_flag != 0) && ok;
    // Every MMA has completed, so the ring's memory is free: each warp turns its
    // 32 rows around in its own part of it, so that neighbouring lanes store
    // neighbouring 16-byte vectors.
    if (ok) {
      fence_after();
      store_rows<D>(a, wk, t * kBM + wq * 32, lane, tO, m_run, l_run,
                    sKV + (warp - 4) * (32 * D * 4));
    }
    fence_before();
    named_barrier_sync(kBarTeardown, kTcThreads);
  }
}

// ------------------------------------------------------ split-unit combine
//
// D/4 lanes per (tail unit, row), four dimensions each: merge the unit's
// key-range pieces, O = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p with M =
// max_p m_p, and store the bf16 row.  Bound by latency (the pieces are in L2), so
// lane p of the row loads (m, l) of piece p and the weights go around by
// shuffles, then all pieces' vectors load at once: two round trips to memory.
template <int D>
__global__ void __launch_bounds__(256)
attn_combine_kernel(const float *__restrict__ ws_o, const float *__restrict__ ws_ml, int n_tail,
                    int n_whole, int pieces, int n_qblocks, int n_active, int H,
                    __nv_bfloat16 *__restrict__ out) {
  pdl_wait();
  pdl_trigger();
  constexpr int kRows = kQT * kBM, kL = D / 4;     // lanes per row
  const int wid = (int)((blockIdx.x * blockDim.x + threadIdx.x) / kL);
  const int sub = threadIdx.x % kL;
  const int u = wid / kRows, row = wid % kRows;
  if (u >= n_tail) return;                         // whole warps: kRows rows are whole warps
  const int unit = n_whole + u;
  const int head = unit / n_qblocks;
  const int grow = (unit % n_qblocks) * kRows + row;
  const float2 *ml = reinterpret_cast<const float2 *>(ws_ml) + (size_t)u * pieces * kRows + row;
  const float4 *o = reinterpret_cast<const float4 *>(ws_o) +
                    ((size_t)u * pieces * kRows + row) * kL + sub;
  float M = -INFINITY;
  for (int p = sub; p < pieces; p += kL) M = fmaxf(M, ml[(size_t)p * kRows].x);
#pragma unroll
  for (int x = 1; x < kL; x <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, x));
  float L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0; p0 < pieces; p0 += kL) {
    float2 v = make_float2(-INFINITY, 0.f);
    if (p0 + sub < pieces) v = ml[(size_t)(p0 + sub) * kRows];
    const float wl = exp2f(v.x - M);
    const int np = min(kL, pieces - p0);
#pragma unroll 8
    for (int p = 0; p < np; ++p) {
      const float4 x = o[(size_t)(p0 + p) * kRows * kL];
      const float w = __shfl_sync(0xffffffffu, wl, p, kL);
      L = fmaf(w, __shfl_sync(0xffffffffu, v.y, p, kL), L);
      acc.x = fmaf(w, x.x, acc.x);
      acc.y = fmaf(w, x.y, acc.y);
      acc.z = fmaf(w, x.z, acc.z);
      acc.w = fmaf(w, x.w, acc.w);
    }
  }
  if (grow >= n_active) return;
  const float inv = 1.f / L;
  *reinterpret_cast<uint2 *>(out + ((size_t)grow * H + head) * D + 4 * sub) =
      make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
}

// -------------------------------------------------------------- host side

std::atomic<int> g_inject_stall{0};   // test hook (hsa_test.h)

// Bytes of split-unit workspace for head dimension D: at most two pieces per
// SM, kQT*kBM rows each, D fp32 of O plus (m, l).
size_t split_workspace_bytes(int D) {
  return 2 * (size_t)sm_count() * (kQT * kBM) * ((size_t)D * 4 + 8) + 512;
}

// Pieces per tail unit.  The rem units of the last wave, cut into P key
// ranges each, occupy ceil(rem*P / sms) waves of 1/P unit: minimise that,
// plus 0.005 unit per piece for its extra prologue, partial write and merge,
// with at most two waves of pieces and at least one key tile per piece.
int tail_pieces(int rem, int sms, int n_kv_tiles) {
  if (rem <= 0) return 1;
  int best = 1;
  double best_cost = 1.0 + 0.005;
  const int pmax = std::min(n_kv_tiles, (2 * sms) / rem);
  for (int p = 2; p <= pmax; ++p) {
    const double cost = (double)((rem * p + sms - 1) / sms) / p + 0.005 * p;
    if (cost < best_cost - 1e-12) {
      best_cost = cost;
      best = p;
    }
  }
  return best;
}

template <int D>
int launch_tc(const void *q, const int32_t *q_idx, int n_active, const void *k_cache,
              const void *v_cache, int rows1, const void *k_base, const void *v_base, int rows2,
              int H, float scale, void *out, void *ws, size_t ws_bytes, cudaStream_t stream,
              unsigned *err) {
  const int N = rows1 + rows2;
  using C = TcCfg<D>;
  static std::atomic<int> configured[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return HSA_ERR_CUDA;
  if (!configured[dev].load()) {
    // The register hand-over inside the kernel assumes exactly kLaunchRegs
    // registers per thread at launch; any other count could leave the
    // softmax warps waiting for registers, so refuse to launch.
    cudaFuncAttributes fa;
    if (cudaFuncGetAttributes(&fa, attn_tc_kernel<D>) != cudaSuccess) return HSA_ERR_CUDA;
    if (fa.numRegs != kLaunchRegs || fa.maxThreadsPerBlock < kTcThreads) return HSA_ERR_UNSUPPORTED;
    if (cudaFuncSetAttribute(attn_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             C::kSmem) != cudaSuccess)
      return HSA_ERR_CUDA;
    configured[dev].store(1);
  }
  CUtensorMap mk, mv, mk2, mv2;
  if (rows1 > 0 && (!make_kv_map(&mk, k_cache, rows1, H * D, (long long)H * D) ||
                    !make_kv_map(&mv, v_cache, rows1, H * D, (long long)H * D)))
    return HSA_ERR_CUDA;
  if (rows2 > 0 && (!make_kv_map(&mk2, k_base, rows2, H * D, (long long)H * D) ||
                    !make_kv_map(&mv2, v_base, rows2, H * D, (long long)H * D)))
    return HSA_ERR_CUDA;
  if (rows1 == 0) mk = mk2, mv = mv2;   // unused source: any valid map
  if (rows2 == 0) mk2 = mk, mv2 = mv;
  TcArgs a;
  a.q = static_cast<const __nv_bfloat16 *>(q);
  a.q_idx = q_idx;
  a.out = static_cast<__nv_bfloat16 *>(out);
  a.err = err;
  a.n_active = n_active;
  a.N = N;
  a.H = H;
  a.q_rows = q_idx ? N : n_active;
  a.rows1 = rows1;
  a.rows2 = rows2;
  a.tiles1 = (rows1 + kBN - 1) / kBN;
  a.n_kv_tiles = a.tiles1 + (rows2 + kBN - 1) / kBN;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.inject_stall = attention_stall();
  // Work plan: one CTA per SM at a time, so U units take ceil(U / sms) waves.
  // With a workspace, the rem = U mod sms units of the last wave are split
  // along the keys into `pieces` ranges (tail_pieces) that shorten that wave,
  // then combined.
  a.n_qblocks = (n_active + kQT * kBM - 1) / (kQT * kBM);
  const long long units = (long long)a.n_qblocks * H;
  if (units > 0x7fffffffLL) return HSA_ERR_UNSUPPORTED;
  const int sms = sm_count();
  a.wave = sms;
  const int rem = (int)(units % sms);
  int pieces = 1;
  if (ws && rem > 0) {
    pieces = tail_pieces(rem, sms, a.n_kv_tiles);
    const size_t need = (size_t)rem * pieces * (kQT * kBM) * ((size_t)D * 4 + 8);
    if (pieces < 2 || need > ws_bytes || (reinterpret_cast<uintptr_t>(ws) & 15)) pieces = 1;
  }
  a.pieces = pieces;
  a.n_whole = pieces > 1 ? (int)(units - rem) : (int)units;
  a.ws_o = pieces > 1 ? static_cast<float *>(ws) : nullptr;
  a.ws_ml = pieces > 1 ? a.ws_o + (size_t)rem * pieces * (kQT * kBM) * D : nullptr;
  const long long grid = (long long)a.n_whole + (pieces > 1 ? (long long)rem * pieces : 0);
  count_launches(1);
  launch_pdl(attn_tc_kernel<D>, dim3((unsigned)grid), dim3(kTcThreads), C::kSmem, stream, mk, mv,
             mk2, mv2, a);
  if (cudaGetLastError() != cudaSuccess) return HSA_ERR_CUDA;
  if (pieces > 1) {
    const long long threads = (long long)rem * (kQT * kBM) * (D / 4);
    count_launches(1);
    launch_pdl(attn_combine_kernel<D>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0,
               stream, (const float *)a.ws_o, (const float *)a.ws_ml, (int)rem, a.n_whole,
               pieces, a.n_qblocks, n_active, H, a.out);
  }
  return launch_status();
}

}  // namespace

int attention_stall() { return g_inject_stall.load(std::memory_order_relaxed); }

}  // namespace hsa

using namespace hsa;

extern "C" size_t hsa_active_attention_workspace_bytes(int n_active, int N, int H, int D,
                                                      hsa_dtype dtype) {
  if (dtype != HSA_BF16 || (D != 64 && D != 128) || n_active <= 0 || N <= 0 || H <= 0) return 0;
  return split_workspace_bytes(D);
}

namespace {

int attention_two_sources(const void *q, const int32_t *q_idx, int n_active, const void *k_cache,
                          const void *v_cache, int rows1, const void *k_base,
                          const void *v_base, int rows2, int H, int D, float scale, void *out,
                          hsa_dtype dtype, void *workspace, size_t workspace_bytes,
                          hsa_stream_t stream) {
  const long long N = (long long)rows1 + rows2;
  if (n_active < 0 || rows1 < 0 || rows2 < 0 || N < 1 || N > 0x7fffffffLL || H < 1)
    return HSA_ERR_INVALID_ARG;
  if (dtype != HSA_BF16 && dtype != HSA_F32) return HSA_ERR_INVALID_ARG;
  if (D != 64 && D != 128) return HSA_ERR_UNSUPPORTED;
  if ((long long)H * D > (1LL << 24)) return HSA_ERR_UNSUPPORTED;
  if (!q_idx && n_active > N) return HSA_ERR_INVALID_ARG;
  if (n_active == 0) return HSA_OK;
  if (!q || !out || (rows1 > 0 && (!k_cache || !v_cache)) || (rows2 > 0 && (!k_base || !v_base)))
    return HSA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || (rows1 > 0 && (!aligned16(k_cache) || !aligned16(v_cache))) ||
      (rows2 > 0 && (!aligned16(k_base) || !aligned16(v_base))))
    return HSA_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale)) scale = 1.f / std::sqrt((float)D);
  unsigned *err = device_error_word();
  if (!err) return HSA_ERR_CUDA;
  cudaStream_t s = (cudaStream_t)stream;
  if (H > 65535) return HSA_ERR_UNSUPPORTED;
  if (dtype == HSA_BF16)
    return D == 128 ? launch_tc<128>(q, q_idx, n_active, k_cache, v_cache, rows1, k_base, v_base,
                                     rows2, H, scale, out, workspace, workspace_bytes, s, err)
                    : launch_tc<64>(q, q_idx, n_active, k_cache, v_cache, rows1, k_base, v_base,
                                    rows2, H, scale, out, workspace, workspace_bytes, s, err);
  return launch_attention_f32(q, q_idx, n_active, k_cache, v_cache, rows1, k_base, v_base, rows2,
                              H, D, scale, out, s, err);
}

}  // namespace

extern "C" int hsa_active_attention(const void *q, const int32_t *q_idx, int n_active,
                                    const void *k_cache, const void *v_cache, int N, int H,
                                    int D, float scale, void *out, hsa_dtype dtype,
                                    void *workspace, size_t workspace_bytes,
                                    hsa_stream_t stream) {
  if (N < 1) return HSA_ERR_INVALID_ARG;
  return attention_two_sources(q, q_idx, n_active, k_cache, v_cache, N, nullptr, nullptr, 0, H,
                               D, scale, out, dtype, workspace, workspace_bytes, stream);
}

extern "C" int hsa_active_attention_prefix(const void *q, const int32_t *q_idx, int n_active,
                                           const void *k_cache, const void *v_cache, int M,
                                           const void *k_base, const void *v_base, int B, int H,
                                           int D, float scale, void *out, hsa_dtype dtype,
                                           void *workspace, size_t workspace_bytes,
                                           hsa_stream_t stream) {
  return attention_two_sources(q, q_idx, n_active, k_cache, v_cache, M, k_base, v_base, B, H, D,
                               scale, out, dtype, workspace, workspace_bytes, stream);
}

extern "C" int hsa_test_inject_attention_stall(int mode) {
  if (mode != 0 && mode != 1) return HSA_ERR_INVALID_ARG;
  return g_inject_stall.exchange(mode);
}

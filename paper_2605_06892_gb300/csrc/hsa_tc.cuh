// The tensor-core attention pipeline that the two bf16 kernels share: PTX wrappers,
// tile constants, the softmax of a key tile, and the roles of the first warpgroup (the
// softmax warpgroups' loops are the kernels' own).  hsa_attention.cu tells how the roles
// work together.
#pragma once

#include <cuda_bf16.h>

#include <atomic>

#include "hsa_internal.cuh"
#include "hsa_ptx.cuh"
#include "hsa_tma.cuh"

namespace hsa {
namespace {

// ----------------------------------------------------------- PTX wrappers

__device__ __forceinline__ void fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// Shared-memory matrix descriptor (tcgen05), 128-byte swizzle.  For a
// K-major operand only the stride between 8-row groups (sbo) matters; for an
// MN-major operand lbo is the stride between 64-element column chunks.
__device__ __forceinline__ uint64_t sdesc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((saddr >> 4) & 0x3FFF) | ((uint64_t)((lbo >> 4) & 0x3FFF) << 16) |
         ((uint64_t)((sbo >> 4) & 0x3FFF) << 32) | (1ull << 46) | (2ull << 61);
}

// Instruction descriptor of kind::f16 with bf16 A/B, fp32 accumulator.
__host__ __device__ constexpr uint32_t idesc_bf16(int M, int N, int b_mn_major) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)b_mn_major << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// The MMAs and commits are issued by the lane with lead != 0, but every lane of
// the issuing warp runs the code around them (see the issuer).
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id,
                                       uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
      "l"(a), "l"(b), "r"(id), "r"(acc), "r"(lead)
      : "memory");
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t id,
                                       uint32_t acc, uint32_t lead) {
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
      " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d),
      "r"(a_tmem), "l"(b), "r"(id), "r"(acc), "r"(lead)
      : "memory");
}

__device__ __forceinline__ void mma_commit(uint64_t *b, uint32_t lead) {
  asm volatile(
      "{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n"
      " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(
          smem_addr(b)),
      "r"(lead)
      : "memory");
}

// 32 consecutive TMEM columns of this thread's lane.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
      "%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,"
      "%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
      "%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,"
      "%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void tmem_wait_ld() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void named_barrier_sync(int id, int threads) {
  asm volatile("barrier.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}


__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t *>(&v);
}

// ------------------------------------------------------ tile constants

constexpr int kBM = 128;         // query rows per Q tile (= TMEM lanes)
constexpr int kQT = 2;           // Q tiles per CTA
constexpr int kBN = 128;         // keys per K/V tile
constexpr int kTcThreads = 384;  // 12 warps = 3 warpgroups
constexpr int kLaunchRegs = 168;         // registers per thread at launch
constexpr int kRegsLow = 96;             // producer / MMA warpgroup
constexpr int kRegsHigh = 200;           // softmax warpgroups
static_assert(128 * kRegsLow + 256 * kRegsHigh <= kTcThreads * kLaunchRegs,
              "register split exceeds the launch allocation");
constexpr int kTmemCols = 512;
// Named barriers (hardware, not in shared memory): 1 = teardown of the whole
// CTA; kBarK0 = the first K tile has landed (the K/V watcher and the issuing
// warp meet once); kBarP0 + t = P of Q tile t is in TMEM, for key tile j (its
// 128 softmax threads, the issuing warp and the K/V watcher meet; at the
// meeting for P_0(j) the watcher has seen V_j and K_(j+1) land).  Every party
// syncs (a rendezvous, never a lone arrive) once per hand-off in the same
// order, so no party can run a whole round ahead and the barrier instances
// always pair up, also after a failed wait.
constexpr int kBarTeardown = 1;
constexpr int kBarP0 = 2;
constexpr int kBarK0 = 4;
constexpr int kMeetP = kBM + 64;   // threads at a P meeting
// kBarS0 + t: S of Q tile t is complete, for key tile j (its 128 softmax threads
// and the S watcher meet).
constexpr int kBarS0 = 5;
constexpr int kMeetS = kBM + 32;

template <int D>
struct TcCfg {
  static constexpr int kTileBytes = kBM * D * 2;            // one Q, K or V tile
  static constexpr int kChunks = D / 64;                    // 128-byte column chunks
  static constexpr int kStages = D == 128 ? 5 : 8;          // K/V ring slots
  static constexpr int kSmem = (kQT + kStages) * kTileBytes + 1024;
  // D = 64: three S buffers in TMEM (384 columns) and O_t at 384 + 64t, so that
  // each Q tile's next S is computed while its softmax still works on the
  // current one.  D = 128: S_t in columns 128t, O_t at 256 + 128t.
  static constexpr bool kThreeS = D == 64;
  static constexpr int kOCol0 = kThreeS ? 384 : 256;        // O_t at kOCol0 + t*D
  static constexpr int kSBars = kThreeS ? 2 : 1;            // S barriers per Q tile
};

// P = 2^(s*scale*log2e - m) for this thread's 128 scores, as bf16 pairs
// written over the first 64 S columns (all scores are in registers, so P may
// overwrite S); returns the row sum of the fp32 values.  bf16 is what the MMA
// takes beside bf16 values, and its range lets P stand far above 1 (the fast
// path below).  Each P is off by 2^-8 of itself at most, up or down, and an
// output by no more than that of its row's sum of |p v|; the sum takes P
// unrounded, which adds nothing to it.  The product is exact and m rounded, so
// a row's P are all off by one factor, 2^(half a step of m), which the division
// by their sum takes out: for |m| below 2^31 it is 2^64 at most.
__device__ __forceinline__ float exp_store_tile(uint32_t tS, const uint32_t (&r)[128],
                                                float sl2, float m) {
  // x = s*scale*log2e - m for a pair of scores in one packed FMA; p = 2^x.
  const uint64_t scale2 = pack2(__float_as_uint(sl2), __float_as_uint(sl2));
  const uint64_t negm2 = pack2(__float_as_uint(-m), __float_as_uint(-m));
  uint64_t ps[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t pk[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const uint64_t x = fma2(pack2(r[64 * h + 2 * i], r[64 * h + 2 * i + 1]), scale2, negm2);
      const float p0 = fast_exp2(lo_f(x));
      const float p1 = fast_exp2(hi_f(x));
      ps[i & 3] = add2(ps[i & 3], pack2(__float_as_uint(p0), __float_as_uint(p1)));
      pk[i] = pack_bf16(p0, p1);
    }
    tmem_st32(tS + 32 * h, pk);
  }
  const uint64_t s01 = add2(ps[0], ps[1]), s23 = add2(ps[2], ps[3]);
  const uint64_t st = add2(s01, s23);
  return lo_f(st) + hi_f(st);
}

// One 128-key tile of this thread's row.  softmax(s) V = sum 2^(c s - m) v /
// sum 2^(c s - m) holds for any reference m as long as nothing overflows, and
// m_run (a maximum of earlier tiles) never exceeds the row's true maximum, so
// after the first tile P is formed against m_run without looking at this
// tile's maximum (fast path).  If a row's sum then exceeds 2^32 (or is not
// finite) the warp redoes the tile on the exact path: the row maximum of the
// scores (still in registers) becomes the new reference, O (in TMEM) and the
// running sum take the factor 2^(m_old - m_new), and P is formed again.  O is
// rescaled only once o_idle() has returned true: the previous O += P V has
// then completed (false: a wait failed, O is left alone).  The first tile
// always takes the exact path.  kTail masks keys >= valid (the last, ragged
// tile); full tiles take no per-key test.
template <int D, bool kTail, typename OIdle>
__device__ __forceinline__ void softmax_tile(uint32_t tS, uint32_t tO, int valid, bool first,
                                             float sl2, float &m_run, float &l_run,
                                             OIdle &&o_idle) {
  // The second half of S is read while the first half is masked.
  uint32_t r[128];
  tmem_ld32(tS, *reinterpret_cast<uint32_t(*)[32]>(&r[0]));
  tmem_ld32(tS + 32, *reinterpret_cast<uint32_t(*)[32]>(&r[32]));
  tmem_wait_ld();
  tmem_ld32(tS + 64, *reinterpret_cast<uint32_t(*)[32]>(&r[64]));
  tmem_ld32(tS + 96, *reinterpret_cast<uint32_t(*)[32]>(&r[96]));
  if (kTail) {
#pragma unroll
    for (int i = 0; i < 64; ++i)
      if (i >= valid) r[i] = __float_as_uint(-INFINITY);
  }
  tmem_wait_ld();
  if (kTail) {
#pragma unroll
    for (int i = 64; i < 128; ++i)
      if (i >= valid) r[i] = __float_as_uint(-INFINITY);
  }
  if (!first) {
    const float rs = exp_store_tile(tS, r, sl2, m_run);
    const bool bad = !(rs <= 4294967296.0f);
    if (!__any_sync(0xffffffffu, bad)) {
      l_run += rs;
      return;
    }
    tmem_wait_st();   // the exact path rewrites the same P columns
  }
  // Exact path.  pm[p] = maximum of scores 16p .. 16p+15: seven
  // three-input steps cover 16p+1 .. 16p+14, the last step adds 16p+15.
  float pm[8];
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    float m = __uint_as_float(r[16 * p]);
#pragma unroll
    for (int i = 1; i < 15; i += 2)
      m = max3f(m, __uint_as_float(r[16 * p + i]), __uint_as_float(r[16 * p + i + 1]));
    pm[p] = fmaxf(m, __uint_as_float(r[16 * p + 15]));
  }
  const float mx = fmaxf(max3f(pm[0], pm[1], pm[2]),
                         fmaxf(max3f(pm[3], pm[4], pm[5]), fmaxf(pm[6], pm[7])));
  const float m_new = fmaxf(m_run, mx * sl2);
  const float alpha = (!first && m_new > m_run) ? fast_exp2(m_run - m_new) : 1.f;
  l_run = first ? 0.f : l_run * alpha;
  m_run = m_new;
  if (!first && __any_sync(0xffffffffu, alpha != 1.f) && o_idle()) {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      uint32_t o[16];
      tmem_ld16(tO + 16 * c, o);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
      tmem_st16(tO + 16 * c, o);
    }
  }
  l_run += exp_store_tile(tS, r, sl2, m_run);
}

// ------------------------------------------------------------ warp roles

// A unit's place in its CTA's pipeline: its nT key tiles are the tiles J .. of the S
// barriers and buffers and fill the ring from load L on.  A CTA of one unit starts at 0
// (constants, which cost nothing); in a chain of units each starts where the one before
// ended.
struct TcSpan {
  int J, L, nT;
};
// Moves past a span: three S buffers close a chained one with a round of S barriers of its
// own (see the issuer).
template <int D>
__device__ __forceinline__ void tc_pass(TcSpan &w) {
  w.J += w.nT + TcCfg<D>::kThreeS;
  w.L += 2 * w.nT;
}

// The barriers of a CTA's pipeline, in its shared memory.
struct TcPipe {
  uint64_t *full, *empty;   // ring slots, kStages each
  uint64_t *s, *o;          // kQT * kSBars; one, or in a chain one per Q tile
  volatile int *abort_flag;
  unsigned *err;
};

// TMA producer (one lane): loads [from, to) of a unit's 2 nT; load_kv(L, slot) issues the
// copy of its tile L/2 (L even: K, odd: V).  `withheld`: a load that a test leaves out, or
// -1.  False: a wait failed; `issued` is the load after the last one issued.
template <int D, typename Load>
__device__ __forceinline__ bool tc_load(const TcPipe &p, const TcSpan &w, int from, int to,
                                        int withheld, int &issued, Load &&load_kv) {
  using C = TcCfg<D>;
  for (int L = from; L < to; ++L) {
    const int slot = (w.L + L) % C::kStages, use = (w.L + L) / C::kStages;
    if (use > 0 && !mbar_wait(&p.empty[slot], (use - 1) & 1, p.abort_flag, p.err)) return false;
    if (w.L + L == withheld) continue;
    load_kv(L, slot);
    issued = w.L + L + 1;
  }
  return true;
}
// Every issued copy has landed before the CTA may exit.  A slot is only refilled once its
// previous tile was consumed, so the copies in flight are among the last kStages issued.
template <int D>
__device__ __forceinline__ void tc_drain(const TcPipe &p, int issued, int withheld) {
  using C = TcCfg<D>;
  for (int L = issued > C::kStages ? issued - C::kStages : 0; L < issued; ++L)
    if (L != withheld)
      mbar_wait(&p.full[L % C::kStages], (L / C::kStages) & 1, p.abort_flag, p.err, false);
}
// The producer warp of a CTA of one unit, from load n_pre on; load_kv(L) finds the slot.
template <int D, typename Load>
__device__ __forceinline__ void tc_produce(const TcPipe &p, int lane, int nT, int n_pre,
                                           int withheld, Load &&load_kv) {
  if (lane == 0) {
    int issued = n_pre;
    tc_load<D>(p, {0, 0, nT}, n_pre, 2 * nT, withheld, issued,
               [&](int L, int) { load_kv(L); });
    tc_drain<D>(p, issued, withheld);
  }
  __syncwarp();
}

// MMA issuer (one warp).  The whole warp walks the schedule so that it can take part in the
// named-barrier hand-offs; one lane issues the MMAs and commits.  The
// tensor pipe takes a new MMA only about when it starts it, so every
// pause of the issuing thread between MMAs idles the tensor core.  An
// mbarrier test on this path costs about a hundred clocks while an S
// group's operand reads fill the shared-memory bandwidth; a named
// barrier whose other parties have already arrived costs far less.
// So the issuer waits on named barriers only, two per key tile:
// kBarP0 + t, where the softmax of Q tile t has stored P and the K/V
// watcher has seen the tiles the next MMAs read land (once, before the
// loop, kBarK0 for the first K tile).  Every party meets it exactly once
// per hand-off whatever happens, so each sync completes.  The issuer
// reads no shared memory on this path either: a load waits behind the
// MMAs' operand reads (a probe measured about 165 clocks of tensor time
// per load of the abort flag), so after an abort it keeps issuing, over
// whatever the ring and the TMEM hold, until the schedule ends; the
// kernel then returns with the error recorded.
// Every lane computes the addresses and descriptors of the MMAs, in code
// without divergence, and only the instruction itself is predicated to
// one lane.  The values are then uniform to the compiler; under a branch
// on the lane each MMA first had to move its operands there, in issue
// slots that two softmax warps of the same scheduler compete for, and the
// tensor core waited for them: D = 64, whose MMAs are half as long, went
// from 1269 to 1505 TFLOP/s (24 heads, N = 32760), the LTX layer from 980
// to 1132.  D = 128 is bound by the MMAs (1990 -> 1995).
// kChain: more units may follow.  p.o[t] then tells the softmax warps of Q tile t that this
// one's O_t is complete, and the barriers of three S buffers all complete once for the tile
// after the last, so that their phases stay in step.
template <int D, bool kChain = false>
__device__ __forceinline__ void tc_issue(const TcPipe &p, uint32_t tmem, uint32_t q_base,
                                         uint32_t kv_base, const TcSpan &w) {
  using C = TcCfg<D>;
  const uint32_t lead = elect_one();
  const int nT = w.nT;
  constexpr uint32_t kIdS = idesc_bf16(kBM, kBN, 0);
  constexpr uint32_t kIdO = idesc_bf16(kBM, D, 1);
  // Descriptors differ only in their start-address field (bits 0-13,
  // address >> 4), so each MMA adds a constant to a base descriptor.
  const uint64_t dq0 = sdesc(q_base, 16, 1024);
  const uint64_t dk0 = sdesc(kv_base, 16, 1024);
  const uint64_t dv0 = sdesc(kv_base, kBN * 128, 1024);
  constexpr uint32_t kTile16 = C::kTileBytes >> 4;
  // S_t = Q_t K^T: K = D in steps of 16 (32 bytes inside a 128-byte chunk).
  auto issue_s = [&](int t, int L) {
    const uint64_t dq = dq0 + t * kTile16;
    const uint64_t dk = dk0 + ((w.L + L) % C::kStages) * kTile16;
    const uint32_t ts = tmem + 128 * t;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      const uint32_t off = ((k >> 2) * (kBM * 128) + (k & 3) * 32) >> 4;
      mma_ss(ts, dq + off, dk + off, kIdS, k > 0, lead);
    }
  };
  // O_t += P_t V: P in TMEM (bf16 pairs in the S_t columns), V MN-major.
  auto issue_o = [&](int t, int L, bool acc) {
    const uint64_t dv = dv0 + ((w.L + L) % C::kStages) * kTile16;
    const uint32_t to = tmem + C::kOCol0 + D * t, tp = tmem + 128 * t;
#pragma unroll
    for (int k = 0; k < kBN / 16; ++k)
      mma_ts(to, tp + 8 * k, dv + ((k * 2048) >> 4), kIdO, (acc || k > 0) ? 1u : 0u, lead);
  };
  auto p_ready = [&](int t) {
    named_barrier_sync(kBarP0 + t, kMeetP);
    fence_after();
  };
  if constexpr (!C::kThreeS) {
    named_barrier_sync(kBarK0, 64);             // K_0 has landed
    fence_after();
    issue_s(0, 0);
    mma_commit(&p.s[0], lead);
    issue_s(1, 0);
    mma_commit(&p.s[1], lead);
    for (int j = 0; j < nT; ++j) {
      const int Lv = 2 * j + 1, Lk = 2 * j + 2;
      const bool more = j + 1 < nT;
      p_ready(0);                               // P_0(j); V_j and K_(j+1) landed
      issue_o(0, Lv, j > 0);
      if (more) {
        issue_s(0, Lk);
        mma_commit(&p.s[0], lead);
      } else if (kChain) {
        mma_commit(&p.o[0], lead);
      }
      p_ready(1);
      issue_o(1, Lv, j > 0);
      if (more) {
        issue_s(1, Lk);
        mma_commit(&p.s[1], lead);
      }
    }
  } else {
    // Three S buffers.  The s-th S MMA in issue order (S_t(j) is number
    // 2j + t) writes buffer s mod 3, so S_0(j+2) and S_1(j+1) reuse the
    // buffers whose P the O MMAs just issued have read (the tensor core
    // runs its MMAs in order).  Each Q tile's S is computed one or two key
    // tiles ahead of its softmax.  S_t(j) completes on bar_s[2t + j%2];
    // alternating two barriers per Q tile means no waiter can be overtaken
    // by two completions of the barrier it waits on.
    auto issue_s3 = [&](int t, int j) {
      const uint64_t dq = dq0 + t * kTile16;
      const uint64_t dk = dk0 + ((w.L + 2 * j) % C::kStages) * kTile16;
      const uint32_t ts = tmem + 128 * ((2 * (w.J + j) + t) % 3);
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
        const uint32_t off = ((k >> 2) * (kBM * 128) + (k & 3) * 32) >> 4;
        mma_ss(ts, dq + off, dk + off, kIdS, k > 0, lead);
      }
      mma_commit(&p.s[2 * t + ((w.J + j) & 1)], lead);
    };
    auto issue_o3 = [&](int t, int j) {
      const uint64_t dv = dv0 + ((w.L + 2 * j + 1) % C::kStages) * kTile16;
      const uint32_t to = tmem + C::kOCol0 + D * t;
      const uint32_t tp = tmem + 128 * ((2 * (w.J + j) + t) % 3);
#pragma unroll
      for (int k = 0; k < kBN / 16; ++k)
        mma_ts(to, tp + 8 * k, dv + ((k * 2048) >> 4), kIdO, (j > 0 || k > 0) ? 1u : 0u, lead);
    };
    named_barrier_sync(kBarK0, 64);             // K_0 (and K_1) have landed
    fence_after();
    issue_s3(0, 0);
    issue_s3(1, 0);
    if (nT > 1) issue_s3(0, 1);
    for (int j = 0; j < nT; ++j) {
      p_ready(0);                               // P_0(j); V_j and K_(j+1) landed
      issue_o3(0, j);
      if (j + 1 < nT) issue_s3(1, j + 1);
      else if (kChain) mma_commit(&p.o[0], lead);
      p_ready(1);                               // P_1(j); K_(j+2) landed
      issue_o3(1, j);
      if (j + 2 < nT)
        issue_s3(0, j + 2);
      else if (j + 2 == nT)
        mma_commit(&p.s[(w.J + j + 2) & 1], lead);  // O_1(j) done, for the last tile's rescale
    }
    if constexpr (kChain) {
      if (nT == 1) mma_commit(&p.s[(w.J + 1) & 1], lead);
      mma_commit(&p.s[2 + ((w.J + nT) & 1)], lead);
    }
  }
  // Completes once every MMA issued above has finished (also on abort), so
  // TMEM is quiet before it is freed.
  mma_commit(&p.o[kChain], lead);
  if constexpr (!kChain) mbar_wait(p.o, 0, p.abort_flag, p.err, false);
  __syncwarp();
}

// K/V watcher (one warp).  Waits (bounded) for the K/V tiles to land and hands them to the
// issuer at the P meetings: V_j and K_(j+1) before P_0(j) (K_0 alone,
// before the loop).  It also gives ring slots back to the producer, so
// the issuer commits nothing for them: once S_1 of key tile j has
// completed (the tensor core runs its MMAs in order), K_j and V_(j-1)
// have been read by every MMA that uses them.  It waits for that between
// the meetings for P_0(j) and P_1(j); S_1 of key tile j+1 is issued only
// after the meeting for P_1(j), so the phase it waits for is never
// overtaken.  It meets the issuer at every meeting even after a failed
// wait, so the issuer never waits forever, and after a failure it gives
// nothing back, so no slot is refilled while a copy into it may still be
// in flight.
// v_landed(j) is called once V_j is in its slot, before the issuer is told.
// kChain: all slots are given back but the last K's and V's, which the softmax warps give
// back when they have stored the unit's rows by way of them.
template <int D, bool kChain = false, typename Landed>
__device__ __forceinline__ void tc_watch_kv(const TcPipe &p, int lane, const TcSpan &w,
                                            Landed &&v_landed) {
  using C = TcCfg<D>;
  bool live = true;
  const int nT = w.nT;
  auto landed = [&](int L) {
    const int at = w.L + L;
    if (live)
      live = __all_sync(0xffffffffu, mbar_wait(&p.full[at % C::kStages], (at / C::kStages) & 1,
                                               p.abort_flag, p.err));
  };
  auto give_back = [&](int L) {
    if (lane == 0) mbar_arrive(&p.empty[(w.L + L) % C::kStages]);
  };
  if constexpr (!C::kThreeS) {
    landed(0);
    named_barrier_sync(kBarK0, 64);
    for (int j = 0; j < nT; ++j) {
      landed(2 * j + 1);                       // V_j
      if (live) v_landed(j);
      if (j + 1 < nT) landed(2 * j + 2);       // K_(j+1)
      named_barrier_sync(kBarP0, kMeetP);
      if (live) {
        live = __all_sync(0xffffffffu, mbar_wait(&p.s[1], (w.J + j) & 1, p.abort_flag, p.err));
        if (live) {
          if (!kChain || j + 1 < nT) give_back(2 * j);   // K_j
          if (j > 0) give_back(2 * j - 1);     // V_(j-1)
        }
      }
      named_barrier_sync(kBarP0 + 1, kMeetP);
    }
  } else {
    // Three S buffers: K_(j+2) is needed at the meeting for P_1(j) (the
    // issuer then issues S_0(j+2)).  S_0(j+1) is issued after O_1(j-1), so
    // once it has completed K_j and V_(j-1) have been read by every MMA
    // that uses them; it waits for that between the meetings for P_0(j) and
    // P_1(j).  The next completion of the same barrier, S_0(j+3), is issued
    // only after the meeting for P_1(j+1).
    landed(0);                                 // K_0
    if (nT > 1) landed(2);                     // K_1
    named_barrier_sync(kBarK0, 64);
    for (int j = 0; j < nT; ++j) {
      landed(2 * j + 1);                       // V_j
      if (live) v_landed(j);
      named_barrier_sync(kBarP0, kMeetP);
      // chained: after the last tile, the barrier's extra round
      if (live && (j + 1 < nT || (kChain && nT > 1))) {
        const int i = w.J + j + 1;
        live = __all_sync(0xffffffffu, mbar_wait(&p.s[i & 1], (i >> 1) & 1, p.abort_flag, p.err));
        if (live) {
          if (!kChain || j + 1 < nT) give_back(2 * j);   // K_j
          if (j > 0) give_back(2 * j - 1);     // V_(j-1)
        }
      }
      if (j + 2 < nT) landed(2 * j + 4);       // K_(j+2)
      named_barrier_sync(kBarP0 + 1, kMeetP);
    }
  }
}

// S watcher (one warp).  An mbarrier test by a softmax warp takes about 300 clocks while the S
// groups' operand reads fill the shared-memory bandwidth, on a completed
// phase too; a named barrier takes a tenth of that.  So this warp makes
// the (bounded) test, ahead of need where the scores are computed ahead,
// and meets the softmax group.  It meets even after a failed wait.  24 x
// 64, N = 32760: 1508 -> 1595 TFLOP/s; D = 128 within its spread.
template <int D>
__device__ __forceinline__ void tc_watch_s(const TcPipe &p, const TcSpan &w) {
  using C = TcCfg<D>;
  bool live = true;
  for (int j = w.J; j < w.J + w.nT; ++j) {
#pragma unroll
    for (int t = 0; t < kQT; ++t) {
      uint64_t *b = C::kThreeS ? &p.s[2 * t + (j & 1)] : &p.s[t];
      const uint32_t par = C::kThreeS ? (j >> 1) & 1 : j & 1;
      if (live) live = __all_sync(0xffffffffu, mbar_wait(b, par, p.abort_flag, p.err));
      fence_before();
      named_barrier_sync(kBarS0 + t, kMeetS);
    }
  }
}

// -------------------------------------------------------------- host side

// 2-D map over N rows of `cols` bf16 values, `row` elements apart: boxes of 64 columns x
// 128 rows, 128-byte swizzle, rows past N read as zero.
inline bool make_kv_map(CUtensorMap *map, const void *base, int N, int cols, long long row) {
  auto enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)N};
  const cuuint64_t strides[1] = {(cuuint64_t)row * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)kBN};
  const cuuint32_t estride[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims, strides,
             box, estride, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace hsa

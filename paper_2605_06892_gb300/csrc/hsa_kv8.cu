// The 8-bit KV cache: quantising fresh K/V rows as they are written into it, and
// reading rows back.
//
// A row of D values of one token and head is held as D e4m3 codes and one power of
// two, 2^e: e is the least integer with max|x| 2^-e <= 448 (the largest e4m3), at
// least -100, and the codes are x 2^-e rounded to nearest even.  With max|x| =
// 1.f 2^E that is e = E - 8, or E - 7 where 1.f > 1.75, an integer addition on the bits
// of the maximum.  Scaling by a power of two is exact, so the only rounding is that of
// the code, and code 2^e (four significant bits, 2^-109 to 1.75 2^127) is exact in bf16:
// what is read back as bf16 is the cache's value, and the tensor cores can take it.
//
// Both kernels are bound by HBM: 3 bytes move per element of a bf16 tensor.  The lanes of a
// group (a power of two) hold vectors of eight elements of a head's row, of K and of V, so
// that a row's maximum takes a few shuffles and all loads and stores are coalesced.  When
// quantising, what is done per row and not per element would fill the issue slots, so a
// lane holds two vectors, c and c + L (LTX-like layer, three quarters of the rows rotated
// and in: 19.5 us with one vector a lane).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hsa_internal.cuh"

namespace hsa {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxD = 256;             // 32 vectors of 8 elements
constexpr unsigned kLeastScale = 27;   // e >= -100: every value is a normal fp32 and bf16

__device__ __forceinline__ uint4 ld_stream(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint2 ld_codes(const void *p) {
  uint2 v;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
  return v;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Two e4m3 codes (lo in the low byte).
__device__ __forceinline__ uint32_t codes2(float lo, float hi) {
  uint16_t c;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(hi), "f"(lo));
  return c;
}
__device__ __forceinline__ float2 values2(uint32_t codes16) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)codes16));
  return __half22float2(*reinterpret_cast<__half2 *>(&h));
}

// Eight neighbouring elements of a row as they are stored.
template <bool kF32>
struct Eight {
  uint4 w[kF32 ? 2 : 1];
};
template <bool kF32>
__device__ __forceinline__ Eight<kF32> load8(const void *base, size_t elem) {
  Eight<kF32> v;
  if (kF32) {
    const float *p = static_cast<const float *>(base) + elem;
    v.w[0] = ld_stream(p);
    v.w[kF32 ? 1 : 0] = ld_stream(p + 4);
  } else {
    v.w[0] = ld_stream(static_cast<const __nv_bfloat16 *>(base) + elem);
  }
  return v;
}

// Pairs (x0, x1) of a bf16 row turned by the table's (cos, sin): fma(x0, c, -(x1 s)),
// fma(x0, s, x1 c) in fp32, rounded to bf16: what the bf16 cache would hold.
__device__ __forceinline__ uint32_t rotate2(uint32_t w, float c, float s) {
  const float a = lo_bf16(w), b = hi_bf16(w);
  return pack_bf16(__fmaf_rn(a, c, -__fmul_rn(b, s)), __fmaf_rn(a, s, __fmul_rn(b, c)));
}

// The scale byte e + 127 for the bits of a row's largest magnitude.
__device__ __forceinline__ unsigned scale_byte(uint32_t bits) {
  const unsigned t = (bits + 0x1fffffu) >> 23;   // exponent, plus one where 1.f > 1.75
  return max(t, kLeastScale + 8u) - 8u;
}

// The largest magnitude's bits among eight elements.
template <bool kF32>
__device__ __forceinline__ uint32_t largest(const Eight<kF32> &v) {
  if (kF32) {
    const uint4 &p = v.w[0], &q = v.w[kF32 ? 1 : 0];
    constexpr uint32_t kM = 0x7fffffffu;
    return max(max(max(p.x & kM, p.y & kM), max(p.z & kM, p.w & kM)),
               max(max(q.x & kM, q.y & kM), max(q.z & kM, q.w & kM)));
  }
  // magnitudes of bf16 are ordered as their bits: two at a time
  const uint4 &q = v.w[0];
  constexpr uint32_t kM = 0x7fff7fffu;
  const uint32_t m = __vmaxu2(__vmaxu2(q.x & kM, q.y & kM), __vmaxu2(q.z & kM, q.w & kM));
  return max(m << 16, m & 0xffff0000u);
}
template <bool kF32>
__device__ __forceinline__ void unpack8(const Eight<kF32> &v, float (&x)[8]) {
  const uint4 &p = v.w[0], &q = v.w[kF32 ? 1 : 0];
  if (kF32) {
    x[0] = __uint_as_float(p.x), x[1] = __uint_as_float(p.y), x[2] = __uint_as_float(p.z);
    x[3] = __uint_as_float(p.w), x[4] = __uint_as_float(q.x), x[5] = __uint_as_float(q.y);
    x[6] = __uint_as_float(q.z), x[7] = __uint_as_float(q.w);
  } else {
    x[0] = lo_bf16(p.x), x[1] = hi_bf16(p.x), x[2] = lo_bf16(p.y), x[3] = hi_bf16(p.y);
    x[4] = lo_bf16(p.z), x[5] = hi_bf16(p.z), x[6] = lo_bf16(p.w), x[7] = hi_bf16(p.w);
  }
}

constexpr uint32_t kTop = 0x7f700000u;   // 1.875 2^127: the next code would stand for 2^128

// The codes of a row's eight elements, twice (all lanes of the warp call it together: a
// shuffle over fewer costs a synchronisation of its own), and the row's scale byte.  `bad` is set
// where an element is not finite: its code is NaN and the others go by the largest finite
// magnitude.  Finite magnitudes above kTop count as that.
template <bool kF32>
__device__ __forceinline__ void quantise(const Eight<kF32> (&v)[2], int L, uint2 (&c)[2],
                                         unsigned &scale, bool &bad) {
  uint32_t m = max(largest(v[0]), largest(v[1]));
  for (int o = 1; o < L; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  const bool odd = __any_sync(0xffffffffu, m > kTop);   // rare
  if (odd) {
    m = 0;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      float x[8];
      unpack8(v[y], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
        if (b >= 0x7f800000u) bad = true;
        else m = max(m, min(b, kTop));
      }
    }
    for (int o = 1; o < L; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  scale = scale_byte(m);
  const float f = __uint_as_float((254u - scale) << 23);   // 2^-e, a normal number
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    float x[8];
    unpack8(v[y], x);
    if (odd) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(x[i]) & 0x7fffffffu;
        if (b >= 0x7f800000u) x[i] = __uint_as_float(0x7fffffffu);
        else if (b > kTop) x[i] = copysignf(__uint_as_float(kTop), x[i]);
      }
    }
    c[y].x = codes2(x[0] * f, x[1] * f) | codes2(x[2] * f, x[3] * f) << 16;
    c[y].y = codes2(x[4] * f, x[5] * f) | codes2(x[6] * f, x[7] * f) << 16;
  }
}

struct QuantArgs {
  uint8_t *kc, *vc, *ks, *vs;
  const void *kf, *vf;
  const int32_t *idx, *tidx;
  const float *table;
  unsigned *err;
  Divider heads;
  unsigned items;   // n H
  int N, D, table_rows, lpr_log2;
};

// Blocks per SM, all resident at once: 6 hold more loads in flight than 5 (720p layer, a
// quarter of the rows 116 -> 104 us), and a single wave of them beats 32 that follow one
// another (LTX-like layer 13.7 -> 12.5).
constexpr int kQuantBlocks = 6;

// One item is a (token, head) of the fresh rows, K and V.
template <bool kF32, bool kRope>
__global__ void __launch_bounds__(kThreads, kF32 ? 4 : kQuantBlocks)
kv_quant_scatter_kernel(const QuantArgs a) {
  pdl_wait();
  const int L = 1 << a.lpr_log2, lane = threadIdx.x & 31, c = lane & (L - 1);
  const bool in[2] = {8 * c < a.D, 8 * (c + L) < a.D};
  const unsigned step = (gridDim.x * (unsigned)kThreads) >> a.lpr_log2;
  const unsigned first = (blockIdx.x * (unsigned)kThreads + threadIdx.x) >> a.lpr_log2;
  // all lanes of a warp run as often as its first
  for (unsigned long long i = first; i - (lane >> a.lpr_log2) < a.items; i += step) {
    const bool there = i < a.items;
    const unsigned j = quotient((unsigned)i, a.heads), h = (unsigned)i - j * a.heads.d;
    int slot = 0, trow = 0;
    Eight<kF32> k[2] = {}, v[2] = {};
    if (there) {
      slot = __ldg(a.idx + j);
      trow = !kRope ? 0 : a.tidx ? __ldg(a.tidx + j) : slot;
      const size_t at = (size_t)i * a.D + 8 * c;
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (in[y]) {
          k[y] = load8<kF32>(a.kf, at + 8 * L * y);
          v[y] = load8<kF32>(a.vf, at + 8 * L * y);
        }
    }
    const bool ok = there && slot >= 0 && slot < a.N &&
                    (!kRope || (trow >= 0 && trow < a.table_rows));
    if (there && !ok) set_error(a.err, kErrIndex);
    if (kRope && ok) {
      const float4 *t = reinterpret_cast<const float4 *>(a.table + (size_t)trow * a.D) + 2 * c;
#pragma unroll
      for (int y = 0; y < 2; ++y)
        if (in[y]) {
          const float4 t0 = __ldg(t + 2 * L * y), t1 = __ldg(t + 2 * L * y + 1);
          uint4 &w = k[y].w[0];
          w.x = rotate2(w.x, t0.x, t0.y);
          w.y = rotate2(w.y, t0.z, t0.w);
          w.z = rotate2(w.z, t1.x, t1.y);
          w.w = rotate2(w.w, t1.z, t1.w);
        }
    }
    bool bad = false;
    unsigned sk, sv;
    uint2 ck[2], cv[2];
    quantise<kF32>(k, L, ck, sk, bad);
    quantise<kF32>(v, L, cv, sv, bad);
    if (!ok) continue;
    if (bad) set_error(a.err, kErrNonfinite);
    const size_t row = (size_t)slot * a.heads.d + h, to = row * a.D + 8 * c;
#pragma unroll
    for (int y = 0; y < 2; ++y)
      if (in[y]) {
        *reinterpret_cast<uint2 *>(a.kc + to + 8 * L * y) = ck[y];
        *reinterpret_cast<uint2 *>(a.vc + to + 8 * L * y) = cv[y];
      }
    if (c == 0) {
      a.ks[row] = (uint8_t)sk;
      a.vs[row] = (uint8_t)sv;
    }
  }
}

struct DequantArgs {
  const uint8_t *kc, *vc, *ks, *vs;
  void *ko, *vo;
  const int32_t *idx;
  unsigned *err;
  Divider heads;
  unsigned items;   // n H
  int N, D, lpr_log2;
};

// 2^(byte - 127)
__device__ __forceinline__ float scale_of(unsigned byte) {
  return __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

template <bool kF32>
__device__ __forceinline__ void store_values(void *base, size_t elem, uint2 code, float f) {
  float2 x[4] = {values2(code.x), values2(code.x >> 16), values2(code.y), values2(code.y >> 16)};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i].x *= f, x[i].y *= f;
  if (kF32) {
    float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + elem);
    p[0] = make_float4(x[0].x, x[0].y, x[1].x, x[1].y);
    p[1] = make_float4(x[2].x, x[2].y, x[3].x, x[3].y);
  } else {
    *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(base) + elem) =
        make_uint4(pack_bf16(x[0].x, x[0].y), pack_bf16(x[1].x, x[1].y),
                   pack_bf16(x[2].x, x[2].y), pack_bf16(x[3].x, x[3].y));
  }
}

template <bool kF32, int kU>
__global__ void __launch_bounds__(kThreads)
kv_dequant_gather_kernel(const DequantArgs a) {
  pdl_wait();
  const int L = 1 << a.lpr_log2, c = threadIdx.x & (L - 1);
  if (8 * c >= a.D) return;
  const unsigned step = (gridDim.x * (unsigned)kThreads) >> a.lpr_log2;
  const unsigned first = (blockIdx.x * (unsigned)kThreads + threadIdx.x) >> a.lpr_log2;
  for (unsigned long long i0 = first; i0 < a.items; i0 += (unsigned long long)step * kU) {
    uint2 k[kU], v[kU];
    unsigned sk[kU], sv[kU];
    bool ok[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const unsigned long long i = i0 + (unsigned long long)u * step;
      ok[u] = i < a.items;
      if (ok[u]) {
        size_t row = (size_t)i;
        if (a.idx) {
          const unsigned j = quotient((unsigned)i, a.heads);
          const int r = __ldg(a.idx + j);
          ok[u] = r >= 0 && r < a.N;
          if (!ok[u]) set_error(a.err, kErrIndex);
          row = (size_t)r * a.heads.d + ((unsigned)i - j * a.heads.d);
        }
        if (ok[u]) {
          k[u] = ld_codes(a.kc + row * a.D + 8 * c);
          v[u] = ld_codes(a.vc + row * a.D + 8 * c);
          sk[u] = a.ks[row];
          sv[u] = a.vs[row];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (!ok[u]) continue;
      const size_t at = (size_t)(i0 + (unsigned long long)u * step) * a.D + 8 * c;
      store_values<kF32>(a.ko, at, k[u], scale_of(sk[u]));
      store_values<kF32>(a.vo, at, v[u], scale_of(sv[u]));
    }
  }
}

int log2i(int x) {
  int l = 0;
  while ((1 << l) < x) ++l;
  return l;
}

// Blocks for `items` items of lane groups of L, kU at a time.
unsigned grid_for(unsigned items, int lpr_log2, int kU, int per_sm) {
  const long long groups = kThreads >> lpr_log2;
  const long long need = ((long long)items + groups * kU - 1) / (groups * kU);
  const long long cap = (long long)sm_count() * per_sm;
  return (unsigned)(need < 1 ? 1 : need < cap ? need : cap);
}

constexpr int kU = 2;        // items of a lane at a time, reading back
constexpr int kBlocks = 32;

// Sizes that both calls take; 1 where there is nothing to do.
int check_sizes(int n, int N, int H, int D, int dtype) {
  if (n < 0 || N < 0 || H < 1 || D < 8 || (D & 7)) return HSA_ERR_INVALID_ARG;
  if (dtype != HSA_BF16 && dtype != HSA_F32) return HSA_ERR_INVALID_ARG;
  if (D > kMaxD || (long long)n * H > 0x7fffffffLL || H > (1 << 24)) return HSA_ERR_UNSUPPORTED;
  return n == 0;
}

}  // namespace
}  // namespace hsa

using namespace hsa;

extern "C" int hsa_kv_quant_scatter(void *k_cache, void *v_cache, uint8_t *k_scale,
                                    uint8_t *v_scale, const void *k_fresh, const void *v_fresh,
                                    const int32_t *idx, int n_active, int N, int H, int D,
                                    hsa_dtype dtype, const float *table,
                                    const int32_t *table_idx, int table_rows,
                                    hsa_stream_t stream) {
  const int st = check_sizes(n_active, N, H, D, dtype);
  if (st < 0) return st;
  if (table ? table_rows < 1 : table_idx != nullptr) return HSA_ERR_INVALID_ARG;
  if (table && dtype != HSA_BF16) return HSA_ERR_UNSUPPORTED;
  if (st) return HSA_OK;
  if (!k_cache || !v_cache || !k_scale || !v_scale || !k_fresh || !v_fresh || !idx)
    return HSA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_fresh) || !aligned16(v_fresh) ||
      !aligned16(table))
    return HSA_ERR_INVALID_ARG;
  QuantArgs a;
  a.kc = static_cast<uint8_t *>(k_cache);
  a.vc = static_cast<uint8_t *>(v_cache);
  a.ks = k_scale;
  a.vs = v_scale;
  a.kf = k_fresh;
  a.vf = v_fresh;
  a.idx = idx;
  a.tidx = table_idx;
  a.table = table;
  a.err = device_error_word();
  if (!a.err) return HSA_ERR_CUDA;
  a.heads = make_divider((unsigned)H);
  a.items = (unsigned)n_active * (unsigned)H;
  a.N = N;
  a.D = D;
  a.table_rows = table_rows;
  a.lpr_log2 = log2i((D / 8 + 1) / 2);
  count_launches(1);
  launch_pdl(dtype == HSA_F32 ? kv_quant_scatter_kernel<true, false>
             : table          ? kv_quant_scatter_kernel<false, true>
                              : kv_quant_scatter_kernel<false, false>,
             dim3(grid_for(a.items, a.lpr_log2, 1, dtype == HSA_F32 ? 4 : kQuantBlocks)),
             dim3(kThreads), 0, (cudaStream_t)stream, a);
  return launch_status();
}

extern "C" int hsa_kv_dequant_gather(const void *k_cache, const void *v_cache,
                                     const uint8_t *k_scale, const uint8_t *v_scale,
                                     const int32_t *idx, int n, int N, int H, int D, void *k_out,
                                     void *v_out, hsa_dtype dtype, hsa_stream_t stream) {
  const int st = check_sizes(n, N, H, D, dtype);
  if (st < 0) return st;
  if (!idx && n > N) return HSA_ERR_INVALID_ARG;
  if (st) return HSA_OK;
  if (!k_cache || !v_cache || !k_scale || !v_scale || !k_out || !v_out) return HSA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_out) || !aligned16(v_out))
    return HSA_ERR_INVALID_ARG;
  DequantArgs a;
  a.kc = static_cast<const uint8_t *>(k_cache);
  a.vc = static_cast<const uint8_t *>(v_cache);
  a.ks = k_scale;
  a.vs = v_scale;
  a.ko = k_out;
  a.vo = v_out;
  a.idx = idx;
  a.err = device_error_word();
  if (!a.err) return HSA_ERR_CUDA;
  a.heads = make_divider((unsigned)H);
  a.items = (unsigned)n * (unsigned)H;
  a.N = N;
  a.D = D;
  a.lpr_log2 = log2i(D / 8);
  count_launches(1);
  launch_pdl(dtype == HSA_F32 ? kv_dequant_gather_kernel<true, kU>
                              : kv_dequant_gather_kernel<false, kU>,
             dim3(grid_for(a.items, a.lpr_log2, kU, kBlocks)), dim3(kThreads), 0,
             (cudaStream_t)stream, a);
  return launch_status();
}

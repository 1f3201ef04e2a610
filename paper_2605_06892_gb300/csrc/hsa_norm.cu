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

#include <cmath>

#include "hsa_internal.cuh"

namespace hsa {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxD = 256;
constexpr int kHeads = 4;        // heads of a lane group at a time
constexpr float kDown = 0x1p-80f;

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
template <bool kF32>
__device__ __forceinline__ void unpack8(const Eight<kF32> &v, float (&x)[8]) {
  const uint32_t w[4] = {v.w[0].x, v.w[0].y, v.w[0].z, v.w[0].w};
  if (kF32) {
    const uint4 &q = v.w[kF32 ? 1 : 0];
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]), x[4 + i] = __uint_as_float(u[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <bool kF32>
__device__ __forceinline__ Eight<kF32> pack8(const float (&x)[8]) {
  Eight<kF32> v;
  if (kF32) {
    v.w[0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                        __float_as_uint(x[3]));
    v.w[kF32 ? 1 : 0] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]),
                                   __float_as_uint(x[6]), __float_as_uint(x[7]));
  } else {
    v.w[0] = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                        pack_bf16(x[6], x[7]));
  }
  return v;
}

template <bool kF32>
__device__ __forceinline__ float squares(const Eight<kF32> &v, float f) {
  float x[8], s = 0.f;
  unpack8<kF32>(v, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = x[i] * f;
    s = fmaf(y, y, s);
  }
  return s;
}

// What a lane keeps of the weights and of the table's row for its eight dimensions.
struct Turn {
  float w[8], cs[8];   // cs: (cos, sin) of the four pairs
};
__device__ __forceinline__ void read8(const float *p, float (&x)[8]) {
  const float4 a = __ldg(reinterpret_cast<const float4 *>(p));
  const float4 b = __ldg(reinterpret_cast<const float4 *>(p) + 1);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
  x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// x times r (1 / the root), times the weights, turned.  `down`: the row's squares overflow in
// 32 bits, and r is for x 2^-80.
template <bool kF32>
__device__ __forceinline__ Eight<kF32> normed(const Eight<kF32> &v, float r, bool down,
                                              const Turn &t, bool turn) {
  float x[8];
  unpack8<kF32>(v, x);
  if (down) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] *= kDown;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = x[i] * r * t.w[i];
  if (turn) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const float a = x[i], b = x[i + 1], c = t.cs[i], s = t.cs[i + 1];
      x[i] = fmaf(a, c, -(b * s));
      x[i + 1] = fmaf(a, s, b * c);
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

// A unit is the kHeads lane groups' heads of one token and tensor.
template <bool kF32>
__global__ void __launch_bounds__(kThreads) norm_heads_kernel(const Args a) {
  pdl_wait();
  pdl_trigger();
  constexpr int kVec = kF32 ? 32 : 16;
  const int L = 1 << a.lpr_log2, lane = threadIdx.x & 31, c = lane & (L - 1);
  const int group = lane >> a.lpr_log2, groups = 32 >> a.lpr_log2;
  const bool in = 8 * c < a.D;
  const unsigned warps = gridDim.x * (kThreads / 32);
  for (unsigned long long i = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); i < a.items;
       i += warps) {
    const unsigned j = quotient((unsigned)i, a.units);
    const int u = (unsigned)i - j * a.units.d;
    const int of = u < a.first[1] ? 0 : u < a.first[2] ? 1 : 2;
    const int h0 = (u - a.first[of]) * groups * kHeads + group;
    const Place p = place_of(a, of, j);
    if (p.to < 0) continue;
    Eight<kF32> v[kHeads] = {};
    const uint8_t *src = a.x[of] + (long long)j * a.in_row[of] + c * kVec;
    uint8_t *dst = a.y[of] + p.to * a.out_row[of] + c * kVec;
#pragma unroll
    for (int y = 0; y < kHeads; ++y)
      if (in && h0 + y * groups < a.H[of])
        v[y] = load8<kF32>(src + (size_t)(h0 + y * groups) * (a.D / 8) * kVec);
    if (of < 2) {
      Turn t;
#pragma unroll
      for (int e = 0; e < 8; ++e) t.w[e] = 1.f;
      if (in && a.weight[of]) read8(a.weight[of] + 8 * c, t.w);
      if (in && a.table) read8(a.table + (size_t)p.trow * a.D + 8 * c, t.cs);
      float s[kHeads];
#pragma unroll
      for (int y = 0; y < kHeads; ++y) s[y] = squares<kF32>(v[y], 1.f);
      for (int o = 1; o < L; o <<= 1)
#pragma unroll
        for (int y = 0; y < kHeads; ++y) s[y] += __shfl_xor_sync(0xffffffffu, s[y], o);
#pragma unroll
      for (int y = 0; y < kHeads; ++y) {
        const bool down = s[y] == INFINITY;
        float r = __frsqrt_rn(fmaf(s[y], a.inv, a.eps));
        if (__any_sync(0xffffffffu, down)) {   // rare
          float z = squares<kF32>(v[y], kDown);
          for (int o = 1; o < L; o <<= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
          if (down) r = __frsqrt_rn(z * a.inv);
        }
        v[y] = normed<kF32>(v[y], r, down, t, a.table != nullptr);
      }
    }
#pragma unroll
    for (int y = 0; y < kHeads; ++y)
      if (in && h0 + y * groups < a.H[of])
        store8<kF32>(dst + (size_t)(h0 + y * groups) * (a.D / 8) * kVec, v[y]);
  }
}

// A unit is one token's row of one tensor, taken by kT threads of a block.
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
  float r = 0.f;
  bool down = false;
  auto total = [&](float f, float (&part)[kBlock / 32]) {
    float s = 0.f;
#pragma unroll
    for (int y = 0; y < kVectors; ++y) s += squares<kF32>(v[y], f);
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
  const float s = total(1.f, sh[0]);
  r = __frsqrt_rn(fmaf(s, inv, a.eps));
  down = s == INFINITY;
  if (__syncthreads_or(down)) {   // rare
    const float z = total(kDown, sh[1]);
    if (down) r = __frsqrt_rn(z * inv);
  }
  uint8_t *dst = a.y[of] + p.to * a.out_row[of];
#pragma unroll
  for (int y = 0; y < kVectors; ++y) {
    const int at = sub + y * kT;
    if (at >= vecs) continue;
    if (of < 2) {
      Turn t;
#pragma unroll
      for (int e = 0; e < 8; ++e) t.w[e] = 1.f;
      if (a.weight[of]) read8(a.weight[of] + 8 * at, t.w);
      if (a.table) read8(a.table + (size_t)p.trow * a.D + 8 * (at % vecs8), t.cs);
      v[y] = normed<kF32>(v[y], r, down, t, a.table != nullptr);
    }
    store8<kF32>(dst + (size_t)at * kVec, v[y]);
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
  count_launches(1);
  if (!across) {
    const long long need = (items + kThreads / 32 - 1) / (kThreads / 32);
    const long long cap = (long long)sm_count() * 32;
    launch_pdl(dtype == HSA_F32 ? norm_heads_kernel<true> : norm_heads_kernel<false>,
               dim3((unsigned)(need < cap ? need : cap)), dim3(kThreads), 0, s, a);
  } else {
    int t = 32;
    while (t * kVectors < most * (D / 8)) t *= 2;
    if (dtype == HSA_F32) launch_row<true>(a, t, s);
    else launch_row<false>(a, t, s);
  }
  return launch_status();
}

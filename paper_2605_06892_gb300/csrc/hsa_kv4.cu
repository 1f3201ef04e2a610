// The 4-bit KV cache: quantising fresh K/V rows as they are written into it, and reading rows
// back.
//
// A row of D values of one token and head is held as D e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6
// and their negatives), the even dimension of a pair in a byte's low half, and a word: factors
// m_0 .. m_3 of six bits each from the lowest bit on, and a byte s above them.  Dimension d is
// of group (d / (D/32)) mod 4, and its code stands for code * m_group * 2^(s - 127).  With a_g
// the largest magnitude of group g and A that of the row, e is the least integer with
// A <= 378 2^e (378 = 6 * 63), at least -100; s = e + 127 and m_g = ceil(a_g / (6 2^e)), so
// that no value lies beyond the codes; codes are x / (m_g 2^e) rounded to nearest even.  A code
// has two significant bits and a factor six, so a value is exact in fp16 (before its power of
// two), bf16 and fp32.
//
// The groups interleave so that whoever takes every fourth, or every eighth, of a row in one
// load holds as many dimensions of each: the attention's lanes then apply the factors to sums
// over one group instead of to values.
//
// Borders are decided exactly.  A bf16 value has eight bits and a border, m_g times 0.25 .. 5,
// at most nine, so x / m_g is at a border or at least 2^-10 from it: formed within 2^-20 and
// rounded to multiples of 2^-14 it falls on the right side.  In fp32 x / m_g, formed within
// 2^-22 of itself and so within 2^-19, falls on the right side where it is 2^-18 or more from
// each multiple of 1/4, which all borders are; nearer values (zeros too) are compared with the
// borders m_g 0.25 .. m_g 5 themselves, which are exact.
//
// Both kernels are bound by HBM: 2.5 bytes move per element of a bf16 tensor, so there are few
// issue slots for each.  A lane group (a power of two) holds a head's row, of K and of V: four
// vectors of eight elements a lane when quantising (two in fp32), one when reading back.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hsa_internal.cuh"
#include "hsa_ptx.cuh"

namespace hsa {
namespace {

constexpr int kThreads = 256;
constexpr unsigned kLeastScale = 27;     // e >= -100
constexpr uint32_t kTop = 0x7f7c0000u;   // 252 2^120: what is above counts as that
constexpr uint32_t kNanRow = 0xff000000u;

__device__ __forceinline__ uint4 ld_stream(const void *p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void prefetch_l2(const void *p) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
}
__device__ __forceinline__ uint32_t ld_codes(const void *p) {
  uint32_t v;
  asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(v) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint64_t twice(float f) {
  return pack2(__float_as_uint(f), __float_as_uint(f));
}
__device__ __forceinline__ float lo_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Eight e2m1 codes, the first lowest.
__device__ __forceinline__ uint32_t codes8(const float (&x)[8]) {
  uint32_t d;
  asm("{\n.reg .b8 a, b, c, e;\n"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 e, %8, %7;\n"
      "mov.b32 %0, {a, b, c, e};\n}"
      : "=r"(d)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return d;
}
// The values of eight codes, in pairs.
__device__ __forceinline__ void values8(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n.reg .b8 a, b, c, e;\n"
      "mov.b32 {a, b, c, e}, %4;\n"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n"
      "cvt.rn.f16x2.e2m1x2 %3, e;\n}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
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

// Pairs (x0, x1) of a bf16 row turned by the table's (cos, sin) in fp32, rounded to bf16: what
// the bf16 cache would hold.
__device__ __forceinline__ uint32_t rotate2(uint32_t w, float c, float s) {
  const float a = lo_bf16(w), b = hi_bf16(w);
  return pack_bf16(__fmaf_rn(a, c, -__fmul_rn(b, s)), __fmaf_rn(a, s, __fmul_rn(b, c)));
}

// A lane's vectors are c, c + L, .. of a row's D / 8, kN of them (what is done per row and not
// per element is a third of the work with two).  A vector holds, at D = 128, four dimensions of
// group 0 and four of 1 (c even), or of 2 and of 3 (c odd); at D = 64 two of each group.  kG groups
// a lane.
template <int D, bool kF32>
struct Lay {
  static constexpr int kN = kF32 ? 2 : 4, kL = D / 8 / kN, kG = D == 128 ? 2 : 4, kRun = 8 / kG;
};

// The largest magnitudes of the lane's groups over the row, as bits of fp32.
template <int D, bool kF32, typename Y = Lay<D, kF32>>
__device__ __forceinline__ void largest(const Eight<kF32> (&v)[Y::kN], uint32_t (&m)[Y::kG]) {
  constexpr int kG = Y::kG, kL = Y::kL, kN = Y::kN;
  if (kF32) {
#pragma unroll
    for (int i = 0; i < kG; ++i) m[i] = 0;
#pragma unroll
    for (int y = 0; y < kN; ++y) {
      float x[8];
      unpack8(v[y], x);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        m[i / Y::kRun] = max(m[i / Y::kRun], __float_as_uint(x[i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = kG == 2 ? 2 : 1; o < kL; o <<= 1)
#pragma unroll
      for (int i = 0; i < kG; ++i) m[i] = max(m[i], __shfl_xor_sync(0xffffffffu, m[i], o));
  } else {
    // magnitudes of bf16 are ordered as their bits: two groups to a word
    constexpr uint32_t kM = 0x7fff7fffu;
    uint32_t w[4] = {};
#pragma unroll
    for (int y = 0; y < kN; ++y) {
      const uint4 &p = v[y].w[0];
      w[0] = __vmaxu2(w[0], p.x & kM), w[1] = __vmaxu2(w[1], p.y & kM);
      w[2] = __vmaxu2(w[2], p.z & kM), w[3] = __vmaxu2(w[3], p.w & kM);
    }
    auto across = [](uint32_t a, uint32_t b) {   // (largest half of a, of b)
      return __vmaxu2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
    };
    uint32_t r[kG / 2];
    if (kG == 2) {
      r[0] = across(__vmaxu2(w[0], w[1]), __vmaxu2(w[2], w[3]));
    } else {
      r[0] = across(w[0], w[1]);
      r[kG / 2 - 1] = across(w[2], w[3]);
    }
#pragma unroll
    for (int o = kG == 2 ? 2 : 1; o < kL; o <<= 1)
#pragma unroll
      for (int i = 0; i < kG / 2; ++i) r[i] = __vmaxu2(r[i], __shfl_xor_sync(0xffffffffu, r[i], o));
#pragma unroll
    for (int i = 0; i < kG / 2; ++i) m[2 * i] = r[i] << 16, m[2 * i + 1] = r[i] & 0xffff0000u;
  }
}

// The codes of a lane's vectors and the row's word, all lanes of the warp together.  `bad` is set
// where the row holds what is not finite: it is then NaN throughout.
template <int D, bool kF32, typename Y = Lay<D, kF32>>
__device__ __forceinline__ void quantise(Eight<kF32> (&v)[Y::kN], uint32_t (&code)[Y::kN],
                                         uint32_t &word, bool &bad) {
  constexpr int kG = Y::kG, kRun = Y::kRun, kN = Y::kN;
  uint32_t m[kG];
  largest<D, kF32>(v, m);
  uint32_t top = max(m[0], m[1]);
  if (kG == 4) top = max(top, max(m[kG - 2], m[kG - 1]));
  if (kG == 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  const bool odd = top >= 0x7f800000u;
  if (top > kTop) {   // rare
    top = kTop;
#pragma unroll
    for (int i = 0; i < kG; ++i) m[i] = min(m[i], kTop);
#pragma unroll
    for (int y = 0; y < kN; ++y)
#pragma unroll
      for (int i = 0; i < (kF32 ? 2 : 1); ++i) {
        uint32_t w[4] = {v[y].w[i].x, v[y].w[i].y, v[y].w[i].z, v[y].w[i].w};
#pragma unroll
        for (int z = 0; z < 4; ++z) {
          w[z] = kF32 ? min(w[z] & 0x7fffffffu, kTop) | (w[z] & 0x80000000u)
                      : __vminu2(w[z] & 0x7fff7fffu, kTop | kTop >> 16) | (w[z] & 0x80008000u);
          if (odd) w[z] = 0;
        }
        v[y].w[i] = make_uint4(w[0], w[1], w[2], w[3]);
      }
  }
  bad |= odd;
  // e of the bits 1.f 2^E: E - 8, or E - 7 where 1.f is above 1.4765625 = 378 / 256
  const unsigned t = (top + (0x7fffffu - 0x3d0000u)) >> 23;
  const unsigned s = max(t, kLeastScale + 8u) - 8u;
  const float f = __uint_as_float((254u - s) << 23);   // 2^-e
  uint32_t factors = 0;
  float unit[kG], per[kG];
#pragma unroll
  for (int i = 0; i < kG; ++i) {
    // at most 378, and exact, but for groups so far below the row that their factor is 1
    const float a = __uint_as_float(m[i]) * f;
    // ceil(a / 6): a times a little less than 1/6, rounded up to a whole number as it joins
    // 2^23.  Of bf16 values a is 6 n or above it by 2^-8 of itself and so well above a little
    // less; of fp32 ones it may be one too few.
    float n = __fadd_ru(a * __uint_as_float(0x3e2aaaa8u), 0x1p23f);
    if (kF32 && (n - 0x1p23f) * 6.f < a) n += 1.f;
    // a, or a sixth of it, may have vanished in 32 bits where the group is not zero
    if (m[i]) n = fmaxf(n, 0x1p23f + 1.f);
    factors |= (__float_as_uint(n) & 63u) << (6 * i);
    unit[i] = n - 0x1p23f;
    float inverse;   // within 2^-23; of a group of zeros any will do
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inverse) : "f"(fmaxf(unit[i], 1.f)));
    per[i] = f * inverse;
  }
  if (kG == 2) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, factors, 1);
    const bool high = threadIdx.x & 1;
    factors = high ? other | factors << 12 : factors | other << 12;
  }
  word = odd ? kNanRow : s << 24 | factors;
#pragma unroll
  for (int y = 0; y < kN; ++y) {
    float x[8];
    unpack8(v[y], x);
    if (kF32) {
      float r[8], near = 1.f;   // x / m_g, and how far the closest is from a multiple of 1/4
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uint64_t z = mul2(pack2(__float_as_uint(x[i]), __float_as_uint(x[i + 1])),
                                twice(per[i / kRun]));
        const uint64_t quarters = add2(add2(z, twice(0x1.8p21f)), twice(-0x1.8p21f));
        const uint64_t off = fma2(quarters, twice(-1.f), z);   // exact
        near = fminf(near, fminf(fabsf(lo_f(off)), fabsf(hi_f(off))));
        r[i] = lo_f(z), r[i + 1] = hi_f(z);
      }
      if (near >= 0x1p-18f) {
        code[y] = codes8(r);
        continue;
      }
      uint32_t c = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float z = fabsf(x[i]) * f, u = unit[i / kRun];
        uint32_t k = (z > 0.25f * u) + (z >= 0.75f * u) + (z > 1.25f * u) + (z >= 1.75f * u) +
                     (z > 2.5f * u) + (z >= 3.5f * u) + (z > 5.f * u);
        if (u == 0.f) k = 0;
        c |= (k | __float_as_uint(x[i]) >> 31 << 3) << (4 * i);
      }
      code[y] = c;
    } else {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const uint64_t z = add2(fma2(pack2(__float_as_uint(x[i]), __float_as_uint(x[i + 1])),
                                     twice(per[i / kRun]), twice(768.f)), twice(-768.f));
        x[i] = lo_f(z), x[i + 1] = hi_f(z);
      }
      code[y] = codes8(x);
    }
  }
}

struct QuantArgs {
  uint8_t *kc, *vc;
  uint32_t *ks, *vs;
  const void *kf, *vf;
  const int32_t *idx, *tidx;
  const float *table;
  unsigned *err;
  Divider heads;
  long long k_row, v_row;   // elements from a token's fresh row to the next
  unsigned items;           // n H
  int N, table_rows;
};

constexpr int kQuantBlocks = 3;   // per SM, all resident at once

// One item is a (token, head) of the fresh rows, K and V.  18900 tokens of 40 heads of D = 128,
// turned: 85 us, 0.87 of HBM's measured rate, and fp32 141, 0.92; 37800 of D = 64 100 us, 0.74, for
// what is done per row is done twice as often.  At D = 128 rows are asked for one item ahead (3 us
// less; at D = 64, where issue slots bind, 2 us more).  Four blocks of 64 registers 85 (D = 64 104).
template <int D, bool kF32, bool kRope>
__global__ void __launch_bounds__(kThreads, kQuantBlocks)
kv4_quant_scatter_kernel(const QuantArgs a) {
  pdl_wait();
  using Y = Lay<D, kF32>;
  constexpr int kL = Y::kL, kN = Y::kN;
  const int lane = threadIdx.x & 31, c = lane & (kL - 1);
  const unsigned step = gridDim.x * (unsigned)(kThreads / kL);
  const unsigned first = (blockIdx.x * (unsigned)kThreads + threadIdx.x) / kL;
  // all lanes of a warp run as often as its first
  for (unsigned long long i = first; i - lane / kL < a.items; i += step) {
    const bool there = i < a.items;
    if (D == 128 && i + step < a.items) {   // a line of the lane group's next rows, into L2
      static_assert(D * (kF32 ? 4 : 2) / 128 * 2 == kL, "the lanes' lines are the rows'");
      const unsigned n = (unsigned)i + step, nj = quotient(n, a.heads);
      const bool of_k = c < kL / 2;
      const size_t at = (size_t)nj * (of_k ? a.k_row : a.v_row) +
                        (size_t)(n - nj * a.heads.d) * D + c % (kL / 2) * (kF32 ? 32 : 64);
      prefetch_l2(static_cast<const uint8_t *>(of_k ? a.kf : a.vf) + at * (kF32 ? 4 : 2));
    }
    const unsigned j = quotient((unsigned)i, a.heads), h = (unsigned)i - j * a.heads.d;
    int slot = -1, trow = 0;
    Eight<kF32> k[kN] = {}, v[kN] = {};
    if (there) {
      slot = __ldg(a.idx + j);
      trow = !kRope ? 0 : a.tidx ? __ldg(a.tidx + j) : slot;
      const size_t in_row = (size_t)h * D + 8 * c;
#pragma unroll
      for (int y = 0; y < kN; ++y) {
        k[y] = load8<kF32>(a.kf, (size_t)j * a.k_row + in_row + 8 * kL * y);
        v[y] = load8<kF32>(a.vf, (size_t)j * a.v_row + in_row + 8 * kL * y);
      }
    }
    const bool ok = slot >= 0 && slot < a.N && (!kRope || (trow >= 0 && trow < a.table_rows));
    if (there && !ok && slot != -1) set_error(a.err, kErrIndex);
    if (kRope && ok) {
      const float4 *t = reinterpret_cast<const float4 *>(a.table + (size_t)trow * D) + 2 * c;
#pragma unroll
      for (int y = 0; y < kN; ++y) {
        const float4 t0 = __ldg(t + 2 * kL * y), t1 = __ldg(t + 2 * kL * y + 1);
        uint4 &w = k[y].w[0];
        w.x = rotate2(w.x, t0.x, t0.y);
        w.y = rotate2(w.y, t0.z, t0.w);
        w.z = rotate2(w.z, t1.x, t1.y);
        w.w = rotate2(w.w, t1.z, t1.w);
      }
    }
    const size_t row = (size_t)slot * a.heads.d + h, to = row * (D / 2) + 4 * c;
    uint8_t *codes = a.kc;
    uint32_t *words = a.ks;
#pragma unroll 1
    for (int of = 0; of < 2; ++of) {   // K, then V: one code for both (84.7 us; two 87.8)
      bool bad = false;
      uint32_t word, code[kN];
      quantise<D, kF32>(k, code, word, bad);
      if (ok) {
        if (bad) set_error(a.err, kErrNonfinite);
#pragma unroll
        for (int y = 0; y < kN; ++y)
          *reinterpret_cast<uint32_t *>(codes + to + 4 * kL * y) = code[y];
        if (c == 0) words[row] = word;
      }
#pragma unroll
      for (int y = 0; y < kN; ++y) k[y] = v[y];
      codes = a.vc;
      words = a.vs;
    }
  }
}

struct DequantArgs {
  const uint8_t *kc, *vc;
  const uint32_t *ks, *vs;
  void *ko, *vo;
  const int32_t *idx;
  unsigned *err;
  Divider heads;
  unsigned items;   // n H
  int N;
};

// Vector c (eight dimensions) of a row with this word.
template <int D, bool kF32>
__device__ __forceinline__ void store_values(void *base, size_t elem, int c, uint32_t code,
                                             uint32_t word) {
  uint32_t h[4];
  values8(code, h);
  float x[8];
  // 2^(s - 127); s is at least 27 where a factor is not zero, and 255 in rows of NaN
  const unsigned s = word >> 24;
  const float f = s == 255 ? __uint_as_float(0x7fffffffu) : __uint_as_float(s << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int group = D == 128 ? 2 * (c & 1) + i / 2 : i;
    const __half m = __ushort2half_rn(word >> (6 * group) & 63u);
    const float2 y =
        __half22float2(__hmul2(*reinterpret_cast<__half2 *>(&h[i]), __half2half2(m)));   // exact
    x[2 * i] = y.x * f, x[2 * i + 1] = y.y * f;
  }
  if (kF32) {
    float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + elem);
    p[0] = make_float4(x[0], x[1], x[2], x[3]);
    p[1] = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(base) + elem) =
        make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]),
                   pack_bf16(x[6], x[7]));
  }
}

// Reading back, an item is a (token, head) of the cache, K and V, a vector of eight a lane.  75600
// tokens of 40 heads of D = 128, bf16: 308 us, 0.94 of HBM's measured rate; D = 64 158, 0.92.  fp32
// 778 us, 0.66 (each of a lane's two 16-byte stores fills half of a sector, which may be why).
constexpr int kU = 2;        // items of a lane at a time, reading back
constexpr int kBlocks = 32;  // blocks per SM at most

template <int D, bool kF32>
__global__ void __launch_bounds__(kThreads)
kv4_dequant_gather_kernel(const DequantArgs a) {
  pdl_wait();
  constexpr int kL = D / 8;
  const int c = threadIdx.x & (kL - 1);
  const unsigned step = gridDim.x * (unsigned)(kThreads / kL);
  const unsigned first = (blockIdx.x * (unsigned)kThreads + threadIdx.x) / kL;
  for (unsigned long long i0 = first; i0 < a.items; i0 += (unsigned long long)step * kU) {
    uint32_t k[kU], v[kU], wk[kU], wv[kU];
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
          if (!ok[u] && r != -1) set_error(a.err, kErrIndex);
          row = (size_t)r * a.heads.d + ((unsigned)i - j * a.heads.d);
        }
        if (ok[u]) {
          k[u] = ld_codes(a.kc + row * (D / 2) + 4 * c);
          v[u] = ld_codes(a.vc + row * (D / 2) + 4 * c);
          wk[u] = a.ks[row];
          wv[u] = a.vs[row];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (!ok[u]) continue;
      const size_t at = (size_t)(i0 + (unsigned long long)u * step) * D + 8 * c;
      store_values<D, kF32>(a.ko, at, c, k[u], wk[u]);
      store_values<D, kF32>(a.vo, at, c, v[u], wv[u]);
    }
  }
}

// Blocks for `items` items of lane groups of L, n at a time.
unsigned grid_for(unsigned items, int L, int n, int per_sm) {
  const long long at_once = (long long)(kThreads / L) * n;
  const long long need = (items + at_once - 1) / at_once, cap = (long long)sm_count() * per_sm;
  return (unsigned)(need < 1 ? 1 : need < cap ? need : cap);
}

// Sizes that both calls take; 1 where there is nothing to do.
int check_sizes(int n, int N, int H, int D, int dtype) {
  if (n < 0 || N < 0 || H < 1 || D < 1) return HSA_ERR_INVALID_ARG;
  if (dtype != HSA_BF16 && dtype != HSA_F32) return HSA_ERR_INVALID_ARG;
  if ((D != 64 && D != 128) || (long long)n * H > 0x7fffffffLL || H > (1 << 24))
    return HSA_ERR_UNSUPPORTED;
  return n == 0;
}

bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace
}  // namespace hsa

using namespace hsa;

extern "C" int hsa_kv4_quant_scatter(void *k_cache, void *v_cache, uint32_t *k_scale,
                                     uint32_t *v_scale, const void *k_fresh, long long k_row,
                                     const void *v_fresh, long long v_row, const int32_t *idx,
                                     int n_active, int N, int H, int D, hsa_dtype dtype,
                                     const float *table, const int32_t *table_idx, int table_rows,
                                     hsa_stream_t stream) {
  const int st = check_sizes(n_active, N, H, D, dtype);
  if (st < 0) return st;
  if (table ? table_rows < 1 : table_idx != nullptr) return HSA_ERR_INVALID_ARG;
  if (table && dtype != HSA_BF16) return HSA_ERR_UNSUPPORTED;
  const int step = dtype == HSA_F32 ? 4 : 8;
  for (const long long row : {k_row, v_row})
    if (row < (long long)H * D || row % step || row > (1LL << 31)) return HSA_ERR_INVALID_ARG;
  if (st) return HSA_OK;
  if (!k_cache || !v_cache || !k_scale || !v_scale || !k_fresh || !v_fresh || !idx)
    return HSA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_fresh) || !aligned16(v_fresh) ||
      !aligned16(table) || !aligned4(k_scale) || !aligned4(v_scale))
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
  a.k_row = k_row;
  a.v_row = v_row;
  a.items = (unsigned)n_active * (unsigned)H;
  a.N = N;
  a.table_rows = table_rows;
  const int lanes = D / 8 / (dtype == HSA_F32 ? 2 : 4);
  auto go = [&](auto kernel) {
    launch_pdl(kernel, dim3(grid_for(a.items, lanes, 1, kQuantBlocks)), dim3(kThreads), 0,
               (cudaStream_t)stream, a);
  };
  count_launches(1);
  if (D == 128) {
    if (dtype == HSA_F32) go(kv4_quant_scatter_kernel<128, true, false>);
    else if (table) go(kv4_quant_scatter_kernel<128, false, true>);
    else go(kv4_quant_scatter_kernel<128, false, false>);
  } else {
    if (dtype == HSA_F32) go(kv4_quant_scatter_kernel<64, true, false>);
    else if (table) go(kv4_quant_scatter_kernel<64, false, true>);
    else go(kv4_quant_scatter_kernel<64, false, false>);
  }
  return launch_status();
}

extern "C" int hsa_kv4_dequant_gather(const void *k_cache, const void *v_cache,
                                      const uint32_t *k_scale, const uint32_t *v_scale,
                                      const int32_t *idx, int n, int N, int H, int D, void *k_out,
                                      void *v_out, hsa_dtype dtype, hsa_stream_t stream) {
  const int st = check_sizes(n, N, H, D, dtype);
  if (st < 0) return st;
  if (!idx && n > N) return HSA_ERR_INVALID_ARG;
  if (st) return HSA_OK;
  if (!k_cache || !v_cache || !k_scale || !v_scale || !k_out || !v_out) return HSA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_out) || !aligned16(v_out) ||
      !aligned4(k_scale) || !aligned4(v_scale))
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
  auto go = [&](auto kernel) {
    launch_pdl(kernel, dim3(grid_for(a.items, D / 8, kU, kBlocks)), dim3(kThreads), 0,
               (cudaStream_t)stream, a);
  };
  count_launches(1);
  if (D == 128) {
    if (dtype == HSA_F32) go(kv4_dequant_gather_kernel<128, true>);
    else go(kv4_dequant_gather_kernel<128, false>);
  } else {
    if (dtype == HSA_F32) go(kv4_dequant_gather_kernel<64, true>);
    else go(kv4_dequant_gather_kernel<64, false>);
  }
  return launch_status();
}

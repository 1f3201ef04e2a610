// The bookkeeping of a paged KV cache before a server's step: pages taken and given back,
// the rows that new tokens go to, their positions, and the packed batch's offsets.
//
// For sequence b with l = lens[b], w = want[b] and pages of P rows, H = ceil(l/P) and
// W = ceil(w/P): max(0, H - W) pages go back onto the stack, max(0, W - H) come from its top,
// max(0, w - l) tokens are new.  All places follow from sums over the sequences before b, so
// the step is a few prefix sums and, between them, the moves.  A few kilobytes move: what
// bounds it is the chain of loads, sums and barriers, and the launch.
//
// One block does the sums and moves the pages: of up to 512 or 1024 sequences, a thread each,
// with one exchange of all four sums, or of 1024 at a time.  The sums saturate at 2^31 - 1,
// where min(a + b, 2^31 - 1) is still associative, so 32 bits serve whatever the lengths are.
// The rows of tokens and keys are filled by the same block where they are few, else by a second
// grid.
#include "hsa_internal.cuh"

namespace hsa {
namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
// Threads for as many sequences or fewer.  Replayed from a graph (an empty one takes 4.1 us), 64
// sequences, a token each / six of them ended besides, with 750 pages given back: 256 threads
// 4.1 / 8.2 us, 512 4.1 / 6.2, 1024 6.2 / 6.2.
constexpr int kFew = 512;
constexpr unsigned kMost = 0x7fffffffu;

struct Args {
  const int32_t *lens, *want, *n_free;      // may be lens_out, n_free_out
  int32_t *table, *free_pages, *n_free_out, *lens_out, *cu_q, *cu_k, *slots, *positions, *key_rows;
  unsigned *err;
  int batch, page_log2, max_pages, n_pages, max_new, max_keys;
};

__device__ __forceinline__ unsigned add_up(unsigned a, unsigned b) { return min(a + b, kMost); }

// Inclusive prefix sums of kN numbers per thread over the block, and the totals.
template <int kN, int kW>
__device__ __forceinline__ void block_scan(unsigned (&x)[kN], unsigned (&total)[kN],
                                           unsigned (&sh)[kN][kW]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned y = __shfl_up_sync(0xffffffffu, x[i], o);
      if (lane >= o) x[i] = add_up(x[i], y);
    }
    if (lane == 31) sh[i][warp] = x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    unsigned s = lane < kW ? sh[i][lane] : 0;
#pragma unroll
    for (int o = 1; o < kW; o <<= 1) {
      const unsigned y = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s = add_up(s, y);
    }
    total[i] = __shfl_sync(0xffffffffu, s, kW - 1);
    const unsigned before = __shfl_sync(0xffffffffu, s, (warp + 31) & 31);
    if (warp) x[i] = add_up(x[i], before);
  }
  __syncthreads();
}

// The first of n ascending numbers that is above v.
template <typename Get>
__device__ __forceinline__ int first_above(int n, unsigned v, Get &&get) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (get(mid) > v) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// Cache rows of elements i .. i + 3 of the batch: element i of sequence b, cu[b] <= i <
// cu[b + 1], is its (i - cu[b])th key, or the like of its newest tokens.  Those from cu[batch]
// on get -1.
__device__ __forceinline__ void fill4(const Args &a, const int32_t *cu, const int32_t *lens, int i,
                                      int n, int32_t *rows, int32_t *positions) {
  int b = first_above(a.batch, (unsigned)i, [&](int m) { return (unsigned)cu[m + 1]; });
  int begin = 0, end = 0, first = 0;
  auto look = [&]() {
    if (b >= a.batch) return;
    begin = cu[b];
    end = cu[b + 1];
    first = positions ? lens[b] - (end - begin) : 0;
  };
  look();
#pragma unroll
  for (int u = 0; u < 4; ++u, ++i) {
    if (i >= n) return;
    while (b < a.batch && i >= end) {
      ++b;
      look();
    }
    int row = -1, at = -1;
    if (b < a.batch) {
      at = first + (i - begin);
      const int id = a.table[(size_t)b * a.max_pages + (at >> a.page_log2)];
      if (id >= 0 && id < a.n_pages) row = (id << a.page_log2) + (at & ((1 << a.page_log2) - 1));
      else set_error(a.err, kErrIndex);
    }
    rows[i] = row;
    if (positions) positions[i] = at;
  }
}

// Elements of slots, then of key_rows, four a thread, with the offsets and lengths at cu_q, cu_k
// and lens.
__device__ __forceinline__ void fill_rows(const Args &a, const int32_t *cu_q, const int32_t *cu_k,
                                          const int32_t *lens, unsigned first, unsigned step) {
  const unsigned tokens = ((unsigned)a.max_new + 3) / 4;
  const unsigned all = tokens + (a.key_rows ? ((unsigned)a.max_keys + 3) / 4 : 0);
  for (unsigned e = first; e < all; e += step) {
    if (e < tokens) fill4(a, cu_q, lens, 4 * e, a.max_new, a.slots, a.positions);
    else fill4(a, cu_k, lens, 4 * (e - tokens), a.max_keys, a.key_rows, nullptr);
  }
}

__device__ __forceinline__ int pages_of(const Args &a, int n) {
  return (n >> a.page_log2) + ((n & ((1 << a.page_log2) - 1)) != 0);
}
// A length, checked.
__device__ __forceinline__ int checked(const Args &a, int n) {
  const long long most = (long long)a.max_pages << a.page_log2;
  if (n >= 0 && n <= most) return n;
  set_error(a.err, kErrIndex);
  return n < 0 ? 0 : (int)most;
}
__device__ __forceinline__ int checked_stack(const Args &a, int n) {
  if (n >= 0 && n <= a.n_pages) return n;
  if (threadIdx.x == 0) set_error(a.err, kErrIndex);
  return n < 0 ? 0 : a.n_pages;
}
// Page e of those given back goes onto the stack at `at`.
__device__ __forceinline__ void push(const Args &a, long long at, const int32_t *from) {
  const int id = *from;
  if (at < a.n_pages) a.free_pages[at] = id;
  if (at >= a.n_pages || id < 0 || id >= a.n_pages) set_error(a.err, kErrIndex);
}
__device__ __forceinline__ int pop(const Args &a, unsigned at, int32_t *to) {
  const int id = a.free_pages[at];
  if (id < 0 || id >= a.n_pages) set_error(a.err, kErrIndex);
  return *to = id;
}

// Up to kT sequences, a thread each.
template <int kT, bool kFill>
__global__ void __launch_bounds__(kT) page_plan_one_kernel(const Args a) {
  __shared__ unsigned sh_sum[4][kT / 32];
  __shared__ unsigned sh_back[kT], sh_get[kT];     // pages moved, up to and with each sequence
  __shared__ int sh_to[kT], sh_from[kT];           // first page that moves
  __shared__ int32_t sh_cu[2][kFill ? kT + 1 : 1], sh_len[kFill ? kT : 1];
  pdl_wait();
  pdl_trigger();
  const int b = threadIdx.x, P1 = (1 << a.page_log2) - 1;
  int l = 0, w = 0;
  if (b < a.batch) {
    l = a.lens[b];
    w = a.want[b];
  }
  int n_free = *a.n_free;
  l = checked(a, l);
  w = checked(a, w);
  n_free = checked_stack(a, n_free);
  int32_t *row = a.table + (size_t)b * a.max_pages;
  const int from = pages_of(a, l), to = pages_of(a, w), fresh = max(0, w - l);
  // the page that the first new token goes to, where the sequence holds it already
  int held = -1;
  if (fresh && (l & P1)) held = row[l >> a.page_log2];
  const unsigned back = max(0, from - to), get = max(0, to - from);
  unsigned x[4] = {back, get, (unsigned)fresh, (unsigned)w}, total[4];
  block_scan(x, total, sh_sum);
  const unsigned back_total = total[0], back_end = x[0];
  const unsigned count = min((unsigned)n_free + back_total, (unsigned)a.n_pages);
  // a sequence grows where its pages and its tokens' places last for it and all that ask
  // before it, whether they got theirs or not
  const bool ok = fresh == 0 || ((get == 0 || x[1] <= count) && x[2] <= (unsigned)a.max_new);
  sh_back[b] = back_end;
  sh_to[b] = to;
  if (__syncthreads_or(!ok)) {   // rare: the sums again, without those
    x[1] = ok ? get : 0;
    x[2] = ok ? fresh : 0;
    x[3] = ok ? w : l;
    block_scan(x, total, sh_sum);
  }
  const int len = ok ? w : l, mine = ok ? fresh : 0;
  if (b < a.batch) {
    a.lens_out[b] = len;
    a.cu_q[b + 1] = (int)x[2];
    if (a.cu_k) a.cu_k[b + 1] = (int)x[3];
  }
  if (b == 0) {
    a.cu_q[0] = 0;
    if (a.cu_k) a.cu_k[0] = 0;
    *a.n_free_out = (int)(count - total[1]);
    if (a.key_rows && total[3] > (unsigned)a.max_keys) set_error(a.err, kErrIndex);
  }
  // ---- pages given back, in the order of the sequences, then those taken from the top
  for (unsigned e = b; e < back_total; e += kT) {
    const int s = first_above(kT, e, [&](int m) { return sh_back[m]; });
    const unsigned j = e - (s ? sh_back[s - 1] : 0);
    push(a, (long long)n_free + e, a.table + (size_t)s * a.max_pages + sh_to[s] + j);
  }
  sh_get[b] = x[1];
  sh_from[b] = from;
  if (kFill) {
    sh_cu[0][b + 1] = (int)x[2];
    sh_cu[1][b + 1] = (int)x[3];
    sh_len[b] = len;
    if (b == 0) sh_cu[0][0] = sh_cu[1][0] = 0;
  }
  // a token each at most, as in a decoder's step: its sequence's thread does it all
  if (!__syncthreads_or(mine > 1) && kFill && !a.key_rows) {
    if (mine) {
      const int id = ok && get ? pop(a, count - x[1], row + from) : held;
      int at = -1;
      if (id >= 0 && id < a.n_pages) at = (id << a.page_log2) + (l & P1);
      else set_error(a.err, kErrIndex);
      a.slots[x[2] - 1] = at;
      a.positions[x[2] - 1] = l;
    }
    for (unsigned i = total[2] + b; i < (unsigned)a.max_new; i += kT)
      a.slots[i] = a.positions[i] = -1;
    return;
  }
  for (unsigned e = b; e < total[1]; e += kT) {
    const int s = first_above(kT, e, [&](int m) { return sh_get[m]; });
    const unsigned j = e - (s ? sh_get[s - 1] : 0);
    pop(a, count - 1 - e, a.table + (size_t)s * a.max_pages + sh_from[s] + j);
  }
  if (kFill) {
    __syncthreads();
    fill_rows(a, sh_cu[0], sh_cu[1], sh_len, b, kT);
  }
}

// Any number of sequences, kThreads at a time.
__global__ void __launch_bounds__(kThreads) page_plan_kernel(const Args a) {
  __shared__ unsigned sh_sum[3][kWarps];
  __shared__ unsigned sh_end[kThreads];   // pages moved, up to and with each sequence
  __shared__ int sh_page[kThreads];       // first page that moves
  auto &sh_one = *reinterpret_cast<unsigned(*)[1][kWarps]>(&sh_sum[0]);
  pdl_wait();
  pdl_trigger();
  auto pages = [&](int n) { return pages_of(a, n); };
  int l = 0, w = 0;
  auto read = [&](int b) {
    l = w = 0;
    if (b >= a.batch) return;
    l = checked(a, a.lens[b]);
    w = checked(a, a.want[b]);
  };
  const int n_free = checked_stack(a, *a.n_free);

  // ---- pages given back, in the order of the sequences
  unsigned back_total = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    read(b);
    const int to = pages(w);
    unsigned x[1] = {(unsigned)max(0, pages(l) - to)}, total[1];
    block_scan(x, total, sh_one);
    if (total[0]) {
      sh_end[threadIdx.x] = x[0];
      sh_page[threadIdx.x] = to;
      __syncthreads();
      for (unsigned e = threadIdx.x; e < total[0]; e += kThreads) {
        const int s = first_above(kThreads, e, [&](int m) { return sh_end[m]; });
        const unsigned j = e - (s ? sh_end[s - 1] : 0);
        push(a, (long long)n_free + back_total + e,
             a.table + (size_t)(b0 + s) * a.max_pages + sh_page[s] + j);
      }
      __syncthreads();
    }
    back_total = add_up(back_total, total[0]);
  }
  const unsigned count = min((unsigned)n_free + back_total, (unsigned)a.n_pages);

  // ---- growth: a sequence grows where its pages and its tokens' places last for it and all
  // that ask before it, whether they got theirs or not
  unsigned asked_pages = 0, asked = 0;          // of the sequences before these
  unsigned got = 0, sum_q = 0, sum_k = 0;       // granted to them
  if (threadIdx.x == 0) {
    a.cu_q[0] = 0;
    if (a.cu_k) a.cu_k[0] = 0;
  }
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    read(b);
    const int from = pages(l);
    const unsigned get = max(0, pages(w) - from), fresh = max(0, w - l);
    unsigned x[3] = {get, fresh, (unsigned)w}, total[3];
    block_scan(x, total, sh_sum);
    const bool ok = fresh == 0 || ((get == 0 || add_up(asked_pages, x[0]) <= count) &&
                                   add_up(asked, x[1]) <= (unsigned)a.max_new);
    const unsigned want_pages = total[0], want_total = total[1];
    if (__syncthreads_or(!ok)) {   // rare: the sums again, without those
      x[0] = ok ? get : 0;
      x[1] = ok ? fresh : 0;
      x[2] = ok ? w : l;
      block_scan(x, total, sh_sum);
    }
    if (b < a.batch) {
      a.lens_out[b] = ok ? w : l;
      a.cu_q[b + 1] = (int)add_up(sum_q, x[1]);
      if (a.cu_k) a.cu_k[b + 1] = (int)add_up(sum_k, x[2]);
    }
    if (total[0]) {
      sh_end[threadIdx.x] = x[0];
      sh_page[threadIdx.x] = from;
      __syncthreads();
      for (unsigned e = threadIdx.x; e < total[0]; e += kThreads) {
        const int s = first_above(kThreads, e, [&](int m) { return sh_end[m]; });
        const unsigned j = e - (s ? sh_end[s - 1] : 0);
        pop(a, count - 1 - got - e, a.table + (size_t)(b0 + s) * a.max_pages + sh_page[s] + j);
      }
      __syncthreads();
    }
    got += total[0];   // at most count
    asked_pages = add_up(asked_pages, want_pages);
    asked = add_up(asked, want_total);
    sum_q = add_up(sum_q, total[1]);
    sum_k = add_up(sum_k, total[2]);
  }
  if (threadIdx.x == 0) {
    *a.n_free_out = (int)(count - got);
    if (a.key_rows && sum_k > (unsigned)a.max_keys) set_error(a.err, kErrIndex);
  }
}

// The rows by a grid of their own; the offsets come to shared memory, where a search takes a
// tenth of the time, as long as they fit.
constexpr int kFillThreads = 256, kFillBatch = 1024;
__global__ void __launch_bounds__(kFillThreads) page_rows_kernel(const Args a) {
  __shared__ int32_t sh_cu[2][kFillBatch + 1], sh_len[kFillBatch];
  pdl_wait();
  pdl_trigger();
  const unsigned first = blockIdx.x * kFillThreads + threadIdx.x;
  if (a.batch <= kFillBatch) {
    for (int i = threadIdx.x; i <= a.batch; i += kFillThreads) {
      sh_cu[0][i] = __ldg(a.cu_q + i);
      if (a.key_rows) sh_cu[1][i] = __ldg(a.cu_k + i);
      if (i < a.batch) sh_len[i] = __ldg(a.lens_out + i);
    }
    __syncthreads();
    fill_rows(a, sh_cu[0], sh_cu[1], sh_len, first, gridDim.x * kFillThreads);
  } else {
    fill_rows(a, a.cu_q, a.cu_k, a.lens_out, first, gridDim.x * kFillThreads);
  }
}

// Rows that the planning block fills itself.
constexpr long long kOwnRows = 8192;

}  // namespace
}  // namespace hsa

using namespace hsa;

extern "C" int hsa_page_plan(const int32_t *lens, const int32_t *want, int batch, int page_size,
                             int32_t *page_table, int max_pages, int32_t *free_pages, int n_pages,
                             const int32_t *n_free, int32_t *n_free_out, int32_t *lens_out,
                             int32_t *cu_q, int32_t *slots, int32_t *positions, int max_new,
                             int32_t *cu_k, int32_t *key_rows, int max_keys,
                             hsa_stream_t stream) {
  if (batch < 0 || page_size < 1 || max_pages < 0 || n_pages < 0 || max_new < 0 || max_keys < 0)
    return HSA_ERR_INVALID_ARG;
  if (page_size & (page_size - 1)) return HSA_ERR_UNSUPPORTED;
  if ((long long)n_pages * page_size > 0x7fffffffLL ||
      (long long)max_pages * page_size > 0x7fffff00LL || max_new > 0x7fffff00 ||
      max_keys > 0x7fffff00)
    return HSA_ERR_UNSUPPORTED;
  if (!n_free || !n_free_out || !cu_q || (batch && (!lens || !want || !lens_out)) ||
      (batch && max_pages && !page_table) || (n_pages && !free_pages) ||
      (max_new && (!slots || !positions)) || (key_rows && !cu_k))
    return HSA_ERR_INVALID_ARG;
  Args a;
  a.lens = lens;
  a.want = want;
  a.n_free = n_free;
  a.table = page_table;
  a.free_pages = free_pages;
  a.n_free_out = n_free_out;
  a.lens_out = lens_out;
  a.cu_q = cu_q;
  a.cu_k = cu_k;
  a.slots = slots;
  a.positions = positions;
  a.key_rows = max_keys ? key_rows : nullptr;
  a.err = device_error_word();
  if (!a.err) return HSA_ERR_CUDA;
  a.batch = batch;
  a.page_log2 = 0;
  while ((1 << a.page_log2) < page_size) ++a.page_log2;
  a.max_pages = max_pages;
  a.n_pages = n_pages;
  a.max_new = max_new;
  a.max_keys = a.key_rows ? max_keys : 0;
  cudaStream_t s = (cudaStream_t)stream;
  const long long rows = (long long)max_new + a.max_keys;
  const bool own = rows <= kOwnRows && batch <= kThreads;
  count_launches(own ? 1 : 2);
  if (batch > kThreads)
    launch_pdl(page_plan_kernel, dim3(1), dim3(kThreads), 0, s, a);
  else if (batch > kFew || (own && rows > 4 * kFew))
    launch_pdl(own ? page_plan_one_kernel<kThreads, true> : page_plan_one_kernel<kThreads, false>,
               dim3(1), dim3(kThreads), 0, s, a);
  else
    launch_pdl(own ? page_plan_one_kernel<kFew, true> : page_plan_one_kernel<kFew, false>, dim3(1),
               dim3(kFew), 0, s, a);
  if (own) return launch_status();
  if (cudaGetLastError() != cudaSuccess) return HSA_ERR_CUDA;
  const long long need = (rows / 4 + 2 + kFillThreads - 1) / kFillThreads;
  const long long cap = (long long)sm_count() * 8;
  launch_pdl(page_rows_kernel, dim3((unsigned)(need < cap ? need : cap)), dim3(kFillThreads), 0, s,
             a);
  return launch_status();
}

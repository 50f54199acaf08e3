// Append of new K/V rows into pages of 8-bit values with a power-of-two scale a
// page, head and tensor.
//
//   e    = max(least e with max |x| <= 448 2^e, the page's e if it goes on, -40)
//   y    = e4m3(x 2^-e)            new rows, to nearest even
//   held = e4m3(held 2^(e_old-e))  the page's earlier rows, when e grew
//
// A power of two keeps the old rows' bits when the scale moves (a product with
// 2^-k is exact until an entry falls below 2^-6, where it is rounded once), and
// lets the attention take a scale into an exponent.
//
// A run is the new rows of one page: a warp takes a run of one head and tensor, half a
// warp a row, eight entries a lane, all of the run's rows (at most 16) in registers, so
// that the maximum and the rounding read a row once.  A warp looks at a group of
// consecutive new rows, a lane each, and works through the runs that start there; the
// group's rows are on their way to L2 while the request and the page are looked up.
//
// What bounds it: the launch and four dependent loads for a step's rows (128 requests of one
// row, 8 heads: 4.8 us; 64 spans of 1 to 16 rows, 4 heads: 5.5 us); for prompts two waves of such
// chains (12 of 200 to 2,000 rows, 4 heads: 13.1 us, 0.50 of a copy's rate; 24 warps an SM at 80
// registers, 14.7 us at 111 and 16 warps, 14.3 at 64 with spills).
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "common.cuh"
#include "e4m3.cuh"

IPD_DECLARE_ERROR_WORD(g_kv8_err);
// whether this process has launched (or captured) a kernel that may set the word:
// a program without these calls does not pay for reading it
static std::atomic<bool> g_kv8_used{false};

namespace {

constexpr int kThreads = 128;
constexpr int kLeast = 87;  // scale byte of e = -40

struct AppendDev {
  ipd_kv8_append_desc d;
  int group;        // new rows a warp looks at: 1 .. 16
  int groups;       // ... and how many such groups there are
};

struct AppendParams {
  AppendDev a[IPD_MAX_BATCHES];
  long long end[IPD_MAX_BATCHES];  // warps up to and with each append
  int n;
};

// A request with cu_new[r] <= tok, the last one where offsets are in order; 32 probes a
// round (for a whole warp).
IPD_DEVINL int request_before(const ipd_kv8_append_desc &D, int tok, int lane) {
  int from = 0, end = D.num_reqs;
  while (end - from > 1) {
    const int step = (end - from + 31) / 32, at = from + lane * step;
    const uint32_t in = __ballot_sync(0xffffffffu, at < end && D.cu_new[at] <= tok);
    if (in != 0) from += (31 - __clz(in)) * step;
    end = min(end, from + step);
  }
  return from;
}

// The run that starts with new row `tok`: its page (< 0: none starts here, or it
// is at fault), first slot and number of rows.  Its request is `lo` or a later one.
IPD_DEVINL int find_run(const ipd_kv8_append_desc &D, int lo, int tok, int *slot, int *rows) {
  if (tok < D.cu_new[0] || tok >= D.cu_new[D.num_reqs]) {
    ipd_set_error(&g_kv8_err, IPD_DEVERR_SPAN);
    return -1;
  }
  int hi = tok < D.cu_new[lo + 1] ? lo : D.num_reqs - 1;  // the last request with cu_new[r] <= tok
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (D.cu_new[mid] <= tok) lo = mid;
    else hi = mid - 1;
  }
  const int c0 = D.cu_new[lo], c1 = min(D.cu_new[lo + 1], D.total_new), len = D.seq_len[lo];
  if (c1 <= tok) {  // offsets out of order
    ipd_set_error(&g_kv8_err, IPD_DEVERR_SPAN);
    return -1;
  }
  const long long p = (long long)len - (D.cu_new[lo + 1] - c0) + (tok - c0);
  if (p < 0 || p >= len || (p >> 4) >= D.max_pages) {
    ipd_set_error(&g_kv8_err, IPD_DEVERR_SEQ_LEN);
    return -1;
  }
  *slot = (int)(p & 15);
  if (*slot != 0 && tok != c0) return -1;  // its page's run started before it
  const int page = D.page_table[(size_t)lo * D.max_pages + (size_t)(p >> 4)];
  if (page < 0 || page >= D.cache.num_pages) {
    ipd_set_error(&g_kv8_err, IPD_DEVERR_PAGE_ID);
    return -1;
  }
  *rows = min(16 - *slot, c1 - tok);
  return page;
}

IPD_DEVINL uint32_t max_abs2(uint32_t m, const uint4 &v) {
  return __vmaxu2(__vmaxu2(m, __vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu)),
                  __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
}
// largest |entry| among the finite of eight bf16, as bits of a non-negative bf16
IPD_DEVINL uint32_t finite_max(const uint4 &v) {
  uint32_t m = 0;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = w[i] & 0x7fffu, hi = w[i] >> 16 & 0x7fffu;
    m = max(m, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
  }
  return m;
}

// the least scale byte that brings the bf16 of bits m to 448 or below
IPD_DEVINL int byte_of(uint32_t m) {
  if (m == 0) return kLeast;
  const uint32_t f = __float_as_uint(bf16f((uint16_t)m));
  if (f < 0x00800000u) return kLeast;  // a subnormal
  // f = 2^(E - 127) (1 + frac), 448 = 2^8 * 1.75
  const int E = (int)(f >> 23);
  return max(kLeast, E - 8 + ((f & 0x7fffffu) > 0x600000u ? 1 : 0));
}

// four values times s as e4m3
IPD_DEVINL uint32_t four(const float *x, float s) {
  const unsigned long long ss = f2_pack(s, s);
  float y[4];
  f2_unpack(f2_mul(f2_pack(x[0], x[1]), ss), y[0], y[1]);
  f2_unpack(f2_mul(f2_pack(x[2], x[3]), ss), y[2], y[3]);
  return e4m3x2(y[0], y[1]) | e4m3x2(y[2], y[3]) << 16;
}
// eight entries, none of them an infinity, times s as e4m3
IPD_DEVINL uint2 quantise(const uint4 &v, float s) {
  const float x[8] = {bf16lo(v.x), bf16hi(v.x), bf16lo(v.y), bf16hi(v.y), bf16lo(v.z), bf16hi(v.z), bf16lo(v.w), bf16hi(v.w)};
  return make_uint2(four(x, s), four(x + 4, s));
}

// ... with NaN for infinities (the conversion would take them for 448)
IPD_DEVINL uint4 without_infinities(uint4 v) {
  uint32_t *w = &v.x;
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] |= __vcmpeq2(w[e], 0x7f807f80u) | __vcmpeq2(w[e], 0xff80ff80u);
  return v;
}
IPD_DEVINL void prefetch_l2(const void *p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }

__global__ void __launch_bounds__(kThreads, 6) kv8_append_kernel(
    const __grid_constant__ AppendParams P) {
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * (kThreads / 32);
  for (long long u = (long long)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < P.end[P.n - 1];
       u += warps) {
    int di = 0;
    while (di + 1 < P.n && u >= P.end[di]) ++di;
    const AppendDev &A = P.a[di];
    const ipd_kv8_append_desc &D = A.d;
    const int hkv = D.cache.num_kv_heads;
    const long long w = u - (di > 0 ? P.end[di - 1] : 0);
    const int g = (int)(w / (2 * hkv)), th = (int)(w % (2 * hkv));
    const bool is_v = th >= hkv;
    const int h = is_v ? th - hkv : th;
    const uint16_t *src = is_v ? D.v_new : D.k_new;
    const long long stride = is_v ? D.v_stride : D.k_stride;
    uint8_t *pages = is_v ? D.cache.v_pages : D.cache.k_pages;
    uint8_t *scales = is_v ? D.cache.v_scale : D.cache.k_scale;
    int page = -1, slot = 0, rows = 0;
    const int tok = g * A.group + lane;
    {  // the group's rows on their way to L2, while their places are looked up
      const int row = g * A.group + (lane >> 1);
      if (lane < 2 * A.group && row < D.total_new) prefetch_l2(src + row * stride + h * 128 + (lane & 1) * 64);
    }
    const int lo = request_before(D, g * A.group, lane);
    if (lane < A.group && tok < D.total_new) page = find_run(D, lo, tok, &slot, &rows);
    uint32_t left = __ballot_sync(0xffffffffu, page >= 0);
    while (left) {
      const int from = __ffs(left) - 1;
      left &= left - 1;
      const int pg = __shfl_sync(0xffffffffu, page, from), s0 = __shfl_sync(0xffffffffu, slot, from),
                n = __shfl_sync(0xffffffffu, rows, from);
      // half a warp a row, eight entries a lane
      const int half = lane >> 4, part = lane & 15;
      const uint16_t *x = src + (long long)(g * A.group + from + half) * stride + h * 128 + part * 8;
      uint8_t *scale = scales + (size_t)pg * hkv + h;
      uint2 *dst = reinterpret_cast<uint2 *>(pages + ((size_t)pg * hkv + h) * 2048) + half * 16 + part;
      uint4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        v[i] = 2 * i + half < n ? *reinterpret_cast<const uint4 *>(x + 2 * i * stride) : make_uint4(0u, 0u, 0u, 0u);
      const int was = s0 > 0 ? *scale : 0;
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max_abs2(m, v[i]);
      m = __reduce_max_sync(0xffffffffu, max(m & 0xffffu, m >> 16));
      const bool finite = m < 0x7f80u;  // (all of the run's rows)
      if (!finite) {
        m = 0;
#pragma unroll 1
        for (int i = half; i < n; i += 2)  // (read again: what is kept for this are registers of every call's)
          m = max(m, finite_max(*reinterpret_cast<const uint4 *>(x + (i - half) * stride)));
        m = __reduce_max_sync(0xffffffffu, m);
      }
      const int b = max(byte_of(m), was);
      if (s0 > 0 && b != was) {
        const float f = pow2i(was - b);  // b is not 255 where it grew
#pragma unroll 2
        for (int i = half; i < s0; i += 2) {
          uint2 &w = dst[(i - half) * 16];
          float y[4], z[4];
          e4m3x4_to_floats(w.x, y), e4m3x4_to_floats(w.y, z);
          w = make_uint2(four(y, f), four(z, f));
        }
      }
      const float f = b == 255 ? __uint_as_float(0x7fc00000u) : pow2i(127 - b);
      dst += s0 * 16;
      if (finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (2 * i + half < n) dst[i * 32] = quantise(v[i], f);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (2 * i + half < n) dst[i * 32] = quantise(without_infinities(v[i]), f);
      }
      __syncwarp();  // every lane has read the page's present scale
      if (lane == 0) *scale = (uint8_t)b;
    }
  }
}

int check(const ipd_kv8_append_desc &a) {
  const ipd_kv8_cache &c = a.cache;
  if (a.num_reqs < 0 || a.total_new < 0 || c.num_pages < 0 || c.num_kv_heads < 1 || a.max_pages < 1)
    return IPD_ERR_INVALID_ARG;
  if (c.page_size != 16 || c.head_dim != 128 || c.num_kv_heads > 64) return IPD_ERR_UNSUPPORTED;
  if (a.total_new == 0) return IPD_OK;
  if (a.num_reqs == 0 || !c.k_pages || !c.v_pages || !c.k_scale || !c.v_scale || !a.k_new ||
      !a.v_new || !a.cu_new || !a.seq_len || !a.page_table)
    return IPD_ERR_INVALID_ARG;
  const int64_t row = (int64_t)c.num_kv_heads * 128;
  if (a.k_stride < row || a.v_stride < row || (a.k_stride | a.v_stride) & 7) return IPD_ERR_INVALID_ARG;
  if (((uintptr_t)c.k_pages | (uintptr_t)c.v_pages | (uintptr_t)a.k_new | (uintptr_t)a.v_new) & 15)
    return IPD_ERR_INVALID_ARG;
  return IPD_OK;
}

}  // namespace

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_kv8_error() {
  if (!g_kv8_used.load(std::memory_order_relaxed)) return 0u;
  unsigned int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_kv8_err, sizeof(v)) != cudaSuccess) return 0xffffffffu;
  if (cudaMemcpyToSymbol(g_kv8_err, &z, sizeof(z)) != cudaSuccess) return 0xffffffffu;
  return v;
}

extern "C" int ipd_kv8_append(const ipd_kv8_append_desc *appends, int n, ipd_stream_t stream) {
  if (n < 0 || n > IPD_MAX_BATCHES || (n > 0 && !appends)) return IPD_ERR_INVALID_ARG;
  AppendParams P;
  memset(&P, 0, sizeof(P));
  long long total = 0;
  for (int i = 0; i < n; ++i) {
    const ipd_kv8_append_desc &a = appends[i];
    const int st = check(a);
    if (st != IPD_OK) return st;
    if (a.total_new == 0) continue;  // nothing to write: not part of the launch
    AppendDev &A = P.a[P.n];
    A.d = a;
    // Rows a warp looks at: 1 where most start a run, 4 for spans, 16 for many (128 single rows: 4.8 us at 1,
    // 5.6 at 2; 64 spans of 1 to 16: 6.2 at 1, 5.5 at 2 and 4, 6.2 at 8, 10.3 at 16; 13,000 rows of
    // prompts: 44 at 1, 17.1 at 8, 13.1 at 16).
    A.group = a.total_new >= 4LL * a.num_reqs && a.total_new > 2048 ? 16 : a.total_new > 2LL * a.num_reqs ? 4 : 1;
    A.groups = (a.total_new + A.group - 1) / A.group;
    total += (long long)A.groups * 2 * a.cache.num_kv_heads;
    P.end[P.n++] = total;
  }
  if (P.n == 0) return IPD_OK;
  const long long blocks = (total + kThreads / 32 - 1) / (kThreads / 32);
  g_kv8_used.store(true, std::memory_order_relaxed);
  kv8_append_kernel<<<(int)(blocks < 65536 ? blocks : 65536), kThreads, 0,
                      reinterpret_cast<cudaStream_t>(stream)>>>(P);
  return cudaGetLastError() == cudaSuccess ? IPD_OK : IPD_ERR_CUDA;
}

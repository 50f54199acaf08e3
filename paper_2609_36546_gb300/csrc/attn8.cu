// Span-verify and decode attention over a paged cache held in 8 bits.
//
//   o_i = sum_j p_ij 2^ev_j v_j / sum_j p_ij,  p_ij = exp(scale 2^ek_j q_i.k_j - m_i)
//
// k_j, v_j e4m3 values, ek, ev the scales of their page and head, key j seen by
// query i of a span of n where j <= L - n + i.
//
// The plainest form: a CTA takes 16 rows (query, head of the group) of one request
// and KV head over all its keys, 32 at a time, with the running maximum and sum.
#include <cuda_runtime.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "common.cuh"
#include "e4m3.cuh"

IPD_DECLARE_ERROR_WORD(g_attn8_err);
// whether this process has launched (or captured) a kernel that may set the word:
// a program without these calls does not pay for reading it
static std::atomic<bool> g_attn8_used{false};

namespace {

constexpr int kD = 128;
constexpr int kPage = 16;
constexpr int kRows = 16;
constexpr int kKeys = 32;
constexpr int kMaxGroup = 128;

struct BatchDev {
  const uint8_t *k, *v, *ks, *vs;
  const uint16_t *q;
  uint16_t *out;
  const int *cu_q, *seq_len, *page_table;
  int num_reqs, hq, hkv, group, max_pages, max_q_len, max_seq_len, total_q, blocks, num_pages;
};
struct Params {
  BatchDev b[IPD_MAX_BATCHES];
  int end[IPD_MAX_BATCHES];  // CTAs up to and with each batch
  int n;
  float scale_log2;
};

__global__ void __launch_bounds__(128) attn8_kernel(const __grid_constant__ Params P) {
  __shared__ float q[kRows][kD], k[kKeys][kD + 1], v[kKeys][kD], s[kRows][kKeys], m[kRows], l[kRows],
      alpha[kRows];
  int bi = 0;
  while (bi + 1 < P.n && (int)blockIdx.x >= P.end[bi]) ++bi;
  const BatchDev &B = P.b[bi];
  int u = blockIdx.x - (bi ? P.end[bi - 1] : 0);
  const int rb = u % B.blocks, h = u / B.blocks % B.hkv, r = u / B.blocks / B.hkv;
  const int c0 = B.cu_q[r], n = B.cu_q[r + 1] - c0, L = B.seq_len[r];
  const int tid = threadIdx.x;
  if (n < 0 || c0 < 0 || c0 + n > B.total_q) {
    if (tid == 0) ipd_set_error(&g_attn8_err, IPD_DEVERR_SPAN);
    return;
  }
  if (n > B.max_q_len || L < n || L > B.max_seq_len) {
    if (tid == 0) ipd_set_error(&g_attn8_err, IPD_DEVERR_SEQ_LEN);
    return;
  }
  const int rows = min(kRows, n * B.group - rb * kRows);
  if (rows <= 0) return;
  auto at = [&](int i) {  // row i's place in q and out
    const int row = rb * kRows + i;
    return ((size_t)(c0 + row / B.group) * B.hq + h * B.group + row % B.group) * kD;
  };
  for (int i = 0; i < kRows; ++i) q[i][tid] = i < rows ? bf16f(B.q[at(i) + tid]) * P.scale_log2 : 0.f;
  if (tid < kRows) m[tid] = -INFINITY, l[tid] = 0.f;
  float o[kRows] = {};
  for (int j0 = 0; j0 < L; j0 += kKeys) {
    __syncthreads();
    for (int j = 0; j < kKeys; ++j) {
      const int key = j0 + j;
      float kk = 0.f, vv = 0.f;
      if (key < L) {
        const int page = B.page_table[(size_t)r * B.max_pages + key / kPage];
        if (page < 0 || page >= B.num_pages) {
          if (tid == 0) ipd_set_error(&g_attn8_err, IPD_DEVERR_PAGE_ID);
          kk = __uint_as_float(0xff800000u);  // marks the key
        } else {
          const size_t g = (size_t)page * B.hkv + h;
          float f[4];
          e4m3x4_to_floats(B.k[(g * kPage + key % kPage) * kD + tid], f);
          kk = f[0] * e8m0(B.ks[g]);
          e4m3x4_to_floats(B.v[(g * kPage + key % kPage) * kD + tid], f);
          vv = f[0] * e8m0(B.vs[g]);
        }
      }
      k[j][tid] = kk;
      v[j][tid] = vv;
    }
    __syncthreads();
    for (int e = tid; e < kRows * kKeys; e += 128) {
      const int i = e / kKeys, j = e % kKeys, query = (rb * kRows + i) / B.group;
      float a = 0.f;
      for (int d = 0; d < kD; ++d) a = fmaf(q[i][d], k[j][d], a);
      const bool seen = i < rows && j0 + j <= L - n + query && __float_as_uint(k[j][0]) != 0xff800000u;
      s[i][j] = seen ? a : -INFINITY;
    }
    __syncthreads();
    if (tid < kRows) {
      float top = m[tid];
      for (int j = 0; j < kKeys; ++j) top = fmaxf(top, s[tid][j]);
      const float ref = top == -INFINITY ? 0.f : top;
      float sum = 0.f;
      for (int j = 0; j < kKeys; ++j) sum += exp2f(s[tid][j] - ref);
      alpha[tid] = exp2f(m[tid] - ref);
      for (int j = 0; j < kKeys; ++j) s[tid][j] = s[tid][j] == -INFINITY ? -INFINITY : exp2f(s[tid][j] - ref);
      l[tid] = l[tid] * alpha[tid] + sum;
      m[tid] = top;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      float a = o[i] * alpha[i];
      for (int j = 0; j < kKeys; ++j)
        if (s[i][j] != -INFINITY) a = fmaf(s[i][j], v[j][tid], a);
      o[i] = a;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    if (i < rows) B.out[at(i) + tid] = f2bf16(l[i] == 0.f ? 0.f : o[i] / l[i]);
}

int validate(const ipd_attn8_batch *b) {
  if (!b || !b->cache) return IPD_ERR_INVALID_ARG;
  const ipd_kv8_cache *c = b->cache;
  if (c->page_size != kPage || c->head_dim != kD) return IPD_ERR_UNSUPPORTED;
  if (c->num_kv_heads < 1 || c->num_kv_heads > 64) return IPD_ERR_UNSUPPORTED;
  if (b->num_q_heads < 1 || b->num_q_heads % c->num_kv_heads) return IPD_ERR_INVALID_ARG;
  if (b->num_q_heads / c->num_kv_heads > kMaxGroup) return IPD_ERR_UNSUPPORTED;
  if (b->num_reqs < 0 || b->total_q < 0 || b->max_q_len < 0 || b->max_seq_len < 0)
    return IPD_ERR_INVALID_ARG;
  if (b->num_reqs == 0 || b->total_q == 0) return IPD_OK;
  if (b->max_q_len < 1 || b->max_seq_len < b->max_q_len) return IPD_ERR_INVALID_ARG;
  if ((long long)b->max_pages * kPage < b->max_seq_len) return IPD_ERR_INVALID_ARG;
  if (c->num_pages < 1) return IPD_ERR_INVALID_ARG;
  if (c->num_pages >= (1LL << 27) || c->num_pages * c->num_kv_heads >= (1LL << 27))
    return IPD_ERR_UNSUPPORTED;
  if (!b->q || !b->out || !b->cu_q || !b->seq_len || !b->page_table || !c->k_pages || !c->v_pages ||
      !c->k_scale || !c->v_scale)
    return IPD_ERR_INVALID_ARG;
  if (((uintptr_t)b->q | (uintptr_t)b->out | (uintptr_t)c->k_pages | (uintptr_t)c->v_pages) & 15)
    return IPD_ERR_INVALID_ARG;
  return IPD_OK;
}

int collect(const ipd_attn8_batch *verify, int nv, const ipd_attn8_batch *decode, int nd,
            const ipd_attn8_batch **out) {
  if (nv < 0 || nd < 0 || nv > IPD_MAX_BATCHES || nd > IPD_MAX_BATCHES - nv) return IPD_ERR_INVALID_ARG;
  if ((nv && !verify) || (nd && !decode)) return IPD_ERR_INVALID_ARG;
  int n = 0;
  for (int i = 0; i < nv; ++i) out[n++] = &verify[i];
  for (int i = 0; i < nd; ++i) out[n++] = &decode[i];
  for (int i = 0; i < n; ++i) {
    const int st = validate(out[i]);
    if (st != IPD_OK) return st;
  }
  return IPD_OK;
}

}  // namespace

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_attn8_error() {
  if (!g_attn8_used.load(std::memory_order_relaxed)) return 0u;
  unsigned int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_attn8_err, sizeof(v)) != cudaSuccess) return 0xffffffffu;
  if (cudaMemcpyToSymbol(g_attn8_err, &z, sizeof(z)) != cudaSuccess) return 0xffffffffu;
  return v;
}

extern "C" size_t ipd_attn8_workspace_size(const ipd_attn8_batch *verify, int n_verify,
                                           const ipd_attn8_batch *decode, int n_decode) {
  const ipd_attn8_batch *bs[IPD_MAX_BATCHES];
  return collect(verify, n_verify, decode, n_decode, bs) == IPD_OK ? 256 : 0;
}

extern "C" int ipd_verify_attn8(const ipd_attn8_batch *verify, int n_verify,
                                const ipd_attn8_batch *decode, int n_decode, float softmax_scale,
                                void *workspace, size_t workspace_bytes, ipd_stream_t stream) {
  const ipd_attn8_batch *bs[IPD_MAX_BATCHES];
  const int st = collect(verify, n_verify, decode, n_decode, bs);
  if (st != IPD_OK) return st;
  if (!(softmax_scale > 0.f) || !(softmax_scale - softmax_scale == 0.f)) return IPD_ERR_INVALID_ARG;
  Params P;
  memset(&P, 0, sizeof(P));
  P.scale_log2 = softmax_scale * kLog2e;
  long long ctas = 0;
  for (int i = 0; i < n_verify + n_decode; ++i) {
    const ipd_attn8_batch &b = *bs[i];
    if (b.num_reqs == 0 || b.total_q == 0) continue;
    const ipd_kv8_cache &c = *b.cache;
    const int group = b.num_q_heads / c.num_kv_heads;
    const int blocks = (b.max_q_len * group + kRows - 1) / kRows;
    P.b[P.n] = BatchDev{c.k_pages, c.v_pages, c.k_scale, c.v_scale, b.q, b.out, b.cu_q, b.seq_len,
                        b.page_table, b.num_reqs, b.num_q_heads, c.num_kv_heads, group, b.max_pages,
                        b.max_q_len, b.max_seq_len, b.total_q, blocks, (int)c.num_pages};
    ctas += (long long)b.num_reqs * c.num_kv_heads * blocks;
    P.end[P.n++] = (int)ctas;
  }
  if (P.n == 0) return IPD_OK;
  if (!workspace || workspace_bytes < 256 || ((uintptr_t)workspace & 255)) return IPD_ERR_WORKSPACE;
  if (ctas > 0x7fffffffLL) return IPD_ERR_UNSUPPORTED;
  g_attn8_used.store(true, std::memory_order_relaxed);
  attn8_kernel<<<(int)ctas, 128, 0, reinterpret_cast<cudaStream_t>(stream)>>>(P);
  return cudaGetLastError() == cudaSuccess ? IPD_OK : IPD_ERR_CUDA;
}

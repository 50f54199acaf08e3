// Verification of drafted tokens by rejection, from given uniform numbers.
//
// With whole-number weights w_v = floor(2^30 2^x_v + 1/2), x_v = fl(fl(l_v - max l) c),
// c = fl(log2 e / temperature), and their sums Z (below 2^48: exact, in any order):
//   accepted   u w_q(x) Z_p < w_p(x) Z_q        (fp64, one rounding a product)
//   residual   r_v = max(0, w_p(v) - (w_q(v) m >> s)),  m 2^-s = Z_p / Z_q in 31 bits
//   token      the entry in which floor(u' S) falls in the running sum of r, by id
// so a verdict is a fixed function of (rows, settings, u): no sum depends on an order.
//
// Two launches.  Rows: every drafted position's two rows, the maximum and the weights' sum:
// long pieces in one look, through a histogram of their values, short ones in two.
// Verdicts: a cluster of CTAs a request finds the first rejected draft and goes through that
// one position's two rows (or the bonus row), each CTA a piece: sums of tiles of 256
// entries, then the tile, then the entry that holds the drawn position.
//
// What bounds it: a small call the two kernels' chains of dependent steps (one request, 4 drafts
// over 151,936 entries: 18.5 us, 6 and 12); a large one the atomics of the row pass (64
// requests of 1 to 16 over 151,936: 121 us, 2.7 TB/s, of which the row pass 92).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>

#include "cluster.cuh"
#include "common.cuh"
#include "weights.cuh"

IPD_DECLARE_ERROR_WORD(g_draft_err);
// whether this process has launched (or captured) a kernel that may set the word:
// a program without these calls does not pay for reading it
static std::atomic<bool> g_draft_used{false};

namespace {

constexpr int kThreads = 512;  // of a verdict's CTA
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;   // CTAs of a row in the row pass
constexpr int kMaxVerdict = 16;  // ... of a request's verdict (as many as one may ask for)
constexpr int kTile = 256;  // entries a warp sums at once: 8 a lane
constexpr int kTiles = (IPD_TRUNC_MAX_VOCAB + 8) / kTile + 1;

// What the row pass leaves of a row.
struct Row {
  u64 z[kMaxCluster];  // sums of the weights of its pieces
  float top;           // largest logit (-inf: the row has no entry)
  uint32_t w;          // the drafted token's weight
  float x;             // ... and x (-inf: the row's entry there is none)
  int owner;           // the request that it was weighed for
  IPD_DEVINL u64 sum(int pieces) const {
    u64 s = 0;
#pragma unroll
    for (int i = 0; i < kMaxCluster; ++i)
      if (i < pieces) s += z[i];
    return s;
  }
};

struct Params {
  ipd_draft_args a;
  Row *rows;     // [2 total]: target and draft row of every position
  int piece;     // 8-entry vectors a CTA takes of a row (verdicts: a multiple of 32)
  int pieces;    // CTAs of a row in the row pass
  float one;     // 1: see pow2_weight2
};

IPD_DEVINL uint32_t max2(uint32_t a, uint32_t b) {  // of two bf16 each; NaN loses
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&a),
                                   *reinterpret_cast<__nv_bfloat162 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&m);
}

// A row as whole 16-byte vectors: it may start and end inside one.
struct RowView {
  const uint4 *base;
  int before, entries, n_vec;  // entries of the first vector that are not the row's
  IPD_DEVINL RowView(const uint16_t *p, int vocab) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    base = reinterpret_cast<const uint4 *>(a & ~(uintptr_t)15);
    before = (int)(a & 15) / 2;
    entries = vocab;
    n_vec = (before + vocab + 7) / 8;
  }
  // vector i with -inf in place of what is not the row's
  IPD_DEVINL uint4 get(int i) const {
    uint4 v = ldg_stream(base + i);
    if (i == 0 || i == n_vec - 1) {
      uint32_t *w = &v.x;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int at = i * 8 + e - before;
        if (at < 0 || at >= entries) w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | 0xff800000u : (w[e >> 1] & 0xffff0000u) | 0xff80u;
      }
    }
    return v;
  }
};

// Weights of a row's entries.  How entries far below the top are kept out of the
// procedure's range: kNear, by a bf16 value of weight 0 that takes the place of all
// below it (and of NaN); kCoarse, where no bf16 value lies between weight 0 and that
// range, by a bound on x; kInf, the top is +inf and only its equals have a weight;
// kNone, the row has no entry.
enum { kNear, kCoarse, kInf, kNone };
struct Weigher {
  float top, c, one;
  uint32_t least2;
  int mode;
  IPD_DEVINL Weigher(float t, float cc, float o) : top(t), c(cc), one(o), least2(0xff80ff80u), mode(kCoarse) {
    if (t == INFINITY) mode = kInf;
    else if (t == -INFINITY) mode = kNone;
    else {
      // as a bf16 value, rounded away from the top
      const float least = t - 34.f / cc;
      const uint32_t b = __float_as_uint(least);
      const uint32_t h = (b >> 16) + ((b >> 31) && (b & 0xffffu) ? 1u : 0u);
      const float at = x(bf16f((uint16_t)h));
      if (at < -32.f && at > -90.f) least2 = h | h << 16, mode = kNear;
    }
  }
  template <int kMode>
  IPD_DEVINL void two(uint32_t w, uint32_t &w0, uint32_t &w1) const {
    if (kMode == kInf || kMode == kNone) {
      w0 = kMode == kInf && (w & 0xffffu) == 0x7f80u ? 1u << 30 : 0u;
      w1 = kMode == kInf && w >> 16 == 0x7f80u ? 1u << 30 : 0u;
      return;
    }
    if (kMode == kNear) w = max2(w, least2);
    u64 y = f2_mul(f2_sub(f2_pack(bf16lo(w), bf16hi(w)), f2_pack(top, top)), f2_pack(c, c));
    if (kMode == kCoarse) {
      float a, b;
      f2_unpack(y, a, b);
      y = f2_pack(fmaxf(a, -64.f), fmaxf(b, -64.f));  // (fmaxf drops a NaN)
    }
    pow2_weight2(y, w0, w1, f2_pack(one, one));
  }
  IPD_DEVINL void any_two(uint32_t w, uint32_t &w0, uint32_t &w1) const {
    if (mode == kNear) two<kNear>(w, w0, w1);
    else if (mode == kCoarse) two<kCoarse>(w, w0, w1);
    else if (mode == kInf) two<kInf>(w, w0, w1);
    else w0 = w1 = 0;
  }
  template <int kMode>
  IPD_DEVINL void eight(const uint4 &v, uint32_t (&r)[8]) const {
    two<kMode>(v.x, r[0], r[1]);
    two<kMode>(v.y, r[2], r[3]);
    two<kMode>(v.z, r[4], r[5]);
    two<kMode>(v.w, r[6], r[7]);
  }
  IPD_DEVINL float x(float l) const { return l == top ? 0.f : __fmul_rn(__fsub_rn(l, top), c); }
};

IPD_DEVINL float scale_of(const float *inv_temp, int r) {
  return __fmul_rn(kLog2e, inv_temp ? inv_temp[r] : 1.f);
}
IPD_DEVINL bool valid(float c) { return c > 0.f && c < INFINITY; }

IPD_DEVINL u64 warp_sum64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// ... of values below 2^40: two sums of parts
IPD_DEVINL u64 warp_sum40(u64 v) {
  return (u64)__reduce_add_sync(0xffffffffu, (uint32_t)v & 0xffffffu) +
         ((u64)__reduce_add_sync(0xffffffffu, (uint32_t)(v >> 24)) << 24);
}

IPD_DEVINL u64 remote_ld64(const void *p, uint32_t rank) {
  const uint32_t a = remote(p, rank);
  return (u64)remote_ld(a) | (u64)remote_ld(a + 4) << 32;
}

// The block's sum / maximum, in every thread (red: kWarps words of its own use).
IPD_DEVINL u64 block_sum(u64 v, u64 *red) {
  v = warp_sum64(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  u64 s = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) s += red[i];
  return s;
}
IPD_DEVINL float block_max(float v, float *red) {
  v = warp_max(v);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) v = fmaxf(v, red[i]);
  return v;
}

// Largest entry of vectors [from, to) of a row.
IPD_DEVINL float piece_max(const RowView &R, int from, int to) {
  uint32_t m = 0xff80ff80u;
  for (int i = from + threadIdx.x; i < to; i += kThreads) {
    const uint4 v = R.get(i);
    m = max2(m, max2(max2(v.x, v.y), max2(v.z, v.w)));
  }
  return fmaxf(bf16lo(m), bf16hi(m));
}

// Whether request r's drafts hold position t.
IPD_DEVINL bool holds(const ipd_draft_args &a, int r, int t) {
  const int c0 = a.cu_draft[r], c1 = a.cu_draft[r + 1];
  return c0 >= 0 && c0 <= t && t < c1 && c1 <= a.total;
}
// The request whose drafts hold position t where the offsets are in order, or -1: none, or they are not.
IPD_DEVINL int request_of(const ipd_draft_args &a, int t) {
  int lo = 0, hi = a.num_reqs - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.cu_draft[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  return holds(a, lo, t) ? lo : -1;
}

// ---- rows ------------------------------------------------------------------
// A row's maximum and the sum of its weights.  bf16 logits have few values, and entries of
// one value have one weight: a long piece of a row is read once into a histogram of its
// values (an integer atomic in shared memory an entry), and the sum is taken from the bins.
// 2^-19 <= |l| < 2^12 is 31 binades of 128 values a sign, whose low 12 bits and sign are the
// bin.  What is nearer to 0 goes to a list (zeros are counted); -inf, NaN and what is not
// above -2^12 have no weight next to such a maximum and go to a bin that no value has.  A
// row that does not fit this (a maximum outside, a full list, so high a temperature that
// -2^12 matters) and short pieces are read twice: for the maximum, then, from L2, entry by
// entry.
constexpr int kBins = 8192;
constexpr uint32_t kLowBits = 0x3600;   // bf16 bits of 2^-19
constexpr uint32_t kHighBits = 0x4580;  // ... of 2^12
constexpr int kList = 256;
constexpr int kHistThreads = 512, kPlainThreads = 512;
// Pieces from here on take a histogram; pieces of rows that are split, which are those of small calls, from
// kHistPiece on: clearing and adding up the bins is a fixed time.  Two looks against a histogram, us a
// call: 64 requests of 16 drafts, 16,001 entries 48.5 and 45.2, 32,000 67 and 60, 100,003 162 and
// 131; one request of 4, 151,936 entries in pieces of 18,992, 17.8 and 20.6.
constexpr int kHistRow = 8 * 1024, kHistPiece = 24 * 1024;

// The byte offsets of two entries' bins.
IPD_DEVINL uint32_t bins2(uint32_t w) { return ((w << 2) & 0x3ffc3ffcu) | ((w >> 1) & 0x40004000u); }
// The bf16 bits of a bin's value.
IPD_DEVINL uint32_t bin_bits(uint32_t bin) {
  const uint32_t low = bin & 0xfffu;
  return (bin >> 12) << 15 | (low >= (kLowBits & 0xfffu) ? 0x3000u : 0x4000u) | low;
}
IPD_DEVINL uint32_t min_abs2(uint32_t a, uint32_t w) {
  const __nv_bfloat162 m = __hmin2(*reinterpret_cast<__nv_bfloat162 *>(&a), __habs2(*reinterpret_cast<__nv_bfloat162 *>(&w)));
  return *reinterpret_cast<const uint32_t *>(&m);
}
IPD_DEVINL void shared_add(uint32_t addr, uint32_t v) {
  asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

template <int kT>
struct RowShared {
  u64 red[kT / 32];
  float fred[kT / 32], top;
  float cp, cq;           // the request's scales
  int r;                  // ... and itself (-1: not found, INT_MAX: the position is none's)
  uint32_t zeros, listed;
  uint16_t list[kList];
};

// Sum of a thread's weights in a piece, entry by entry.
template <int kMode, int kT>
IPD_DEVINL u64 piece_sum(const Weigher &W, const RowView &R, int from, int to) {
  u64 z = 0;
  for (int i = from + threadIdx.x; i < to; i += kT) {
    uint32_t w[8];
    W.eight<kMode>(R.get(i), w);
#pragma unroll
    for (int k = 0; k < 8; k += 2) z += w[k] + w[k + 1];
  }
  return z;
}

template <bool kHist>
__global__ void __launch_bounds__(kHist ? kHistThreads : kPlainThreads, kHist ? 4 : 3)
    draft_rows_kernel(const __grid_constant__ Params P) {
  constexpr int kT = kHist ? kHistThreads : kPlainThreads;
  extern __shared__ uint4 hist4[];
  __shared__ RowShared<kT> S;
  const ipd_draft_args &a = P.a;
  const uint32_t csize = cluster_size(), rank = cluster_rank();
  const int row = blockIdx.x / csize, t = row >> 1, tid = threadIdx.x, lane = tid & 31;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const bool draft = row & 1;
  if (tid == kT - 1) {  // beside the first loads
    const int r = request_of(a, t);
    S.r = r;
    S.cp = scale_of(a.inv_temp_target, max(r, 0)), S.cq = scale_of(a.inv_temp_draft, max(r, 0));
  }
  const uint16_t *p = draft ? a.logits_draft + (long long)t * a.draft_stride
                            : a.logits_target + (long long)t * a.target_stride;
  // the drafted token's entry
  int tok = 0;
  uint16_t entry = 0xff80;
  if (rank == 0 && tid == 0) {
    tok = a.tokens[t];
    if (tok >= 0 && tok < a.vocab) entry = p[tok];
  }
  const RowView R(p, a.vocab);
  const int from = min((int)rank * P.piece, R.n_vec), to = min(from + P.piece, R.n_vec);
  uint32_t m = 0xff80ff80u;
  if (kHist) {
    for (int i = tid; i < kBins / 4; i += kT) hist4[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) S.zeros = S.listed = 0u;
    __syncthreads();
    const uint32_t hist = smem_u32(hist4);
    constexpr uint32_t kLowest2 = (0x8000u | kHighBits) * 0x10001u;
    constexpr int kAhead = 2;
    for (int i0 = from + tid; i0 < to; i0 += kAhead * kT) {
      uint4 v[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        v[k] = i0 + k * kT < to ? R.get(i0 + k * kT) : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
      uint32_t least = 0x7f807f80u;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint32_t w[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          m = max2(m, w[e]);
          least = min_abs2(least, w[e]);
          const uint32_t b = bins2(max2(w[e], kLowest2));
          shared_add(hist + (b & 0xffffu), 1u);
          shared_add(hist + (b >> 16), 1u);
        }
      }
      if (min(least & 0xffffu, least >> 16) < kLowBits) {
        // entries near 0 were counted in another's bin
#pragma unroll 1
        for (int k = 0; k < 8 * kAhead; ++k) {
          uint32_t w = 0;
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            const uint32_t x[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (k >> 1 == 4 * j + e) w = x[e];
          }
          w = k & 1 ? w >> 16 : w & 0xffffu;
          if ((w & 0x7fffu) >= kLowBits) continue;
          shared_add(hist + (bins2(w) & 0xffffu), 0xffffffffu);
          if ((w & 0x7fffu) == 0) {
            atomicAdd(&S.zeros, 1u);
          } else {
            const uint32_t n = atomicAdd(&S.listed, 1u);
            if (n < (uint32_t)kList) S.list[n] = (uint16_t)w;
          }
        }
      }
    }
  } else {
#pragma unroll 4
    for (int i = from + tid; i < to; i += kT) {
      const uint4 v = R.get(i);
      m = max2(m, max2(max2(v.x, v.y), max2(v.z, v.w)));
    }
  }
  float top = warp_max(fmaxf(bf16lo(m), bf16hi(m)));
  if (lane == 0) S.fred[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kT / 32; ++i) top = fmaxf(top, S.fred[i]);
  if (S.r < 0) {
    // A position behind the last request, or offsets out of order, among which it may be
    // anyone's: all are looked through, and the first that holds it has it.
    __syncthreads();
    if (tid == 0) S.r = INT_MAX;
    __syncthreads();
    for (int r = tid; r < a.num_reqs; r += kT)
      if (holds(a, r, t)) atomicMin(&S.r, r);
    __syncthreads();
    if (tid == 0 && S.r != INT_MAX) S.cp = scale_of(a.inv_temp_target, S.r), S.cq = scale_of(a.inv_temp_draft, S.r);
    __syncthreads();
  }
  if (csize > 1) {
    if (tid == 0) S.top = top;
    cluster_sync();
    if (lane < (int)csize) top = __uint_as_float(remote_ld(remote(&S.top, lane)));
    top = warp_max(top);
    cluster_arrive();  // (waited for at the end: no CTA leaves while its maximum is read)
  }
  const Weigher W(top, draft ? S.cq : S.cp, P.one);
  u64 z = 0;
  if (kHist && W.mode != kNone && top < 4096.f && W.x(-4096.f) < -32.f && S.listed <= (uint32_t)kList) {
    const uint32_t *hist = reinterpret_cast<const uint32_t *>(hist4);
#pragma unroll 2
    for (int k = 2 * tid; k < kBins; k += 2 * kT) {
      const uint32_t n0 = hist[k], n1 = hist[k + 1];
      if ((n0 | n1) == 0u || (k & 0xf80) == (kHighBits & 0xf80)) continue;  // (the bin of no value)
      uint32_t w0, w1;
      W.two<kCoarse>(bin_bits(k) | bin_bits(k + 1) << 16, w0, w1);
      z += (u64)n0 * w0 + (u64)n1 * w1;
    }
    for (int k = tid; k <= (int)S.listed; k += kT) {  // the list, and the zeros
      const bool zero = k == (int)S.listed;
      uint32_t w0, w1;
      W.two<kCoarse>((zero ? 0u : S.list[k]) | 0xff800000u, w0, w1);
      z += (u64)w0 * (zero ? S.zeros : 1u);
    }
  } else if (W.mode == kNear) {
    z = piece_sum<kNear, kT>(W, R, from, to);
  } else if (W.mode == kCoarse) {
    z = piece_sum<kCoarse, kT>(W, R, from, to);
  } else if (W.mode == kInf) {
    z = piece_sum<kInf, kT>(W, R, from, to);
  }
  z = warp_sum64(z);
  if (lane == 0) S.red[tid >> 5] = z;
  __syncthreads();
  if (tid == 0 && S.r != INT_MAX) {
    z = 0;
    for (int i = 0; i < kT / 32; ++i) z += S.red[i];
    Row &O = P.rows[row];
    O.z[rank] = z;
    if (rank == 0) {
      uint32_t w0, w1;
      W.any_two(entry | 0xff800000u, w0, w1);
      const float l = bf16f(entry);
      O.top = top, O.w = w0, O.x = l != l ? -INFINITY : W.x(l), O.owner = S.r;
    }
  }
  if (csize > 1) cluster_wait();
}

// ---- verdicts ----------------------------------------------------------------
struct Verdict {
  u64 tile[kTiles];  // sums of the tiles of this CTA's piece
  u64 red[kWarps];
  float fred[kWarps];
  u64 sum;           // ... of the piece
  u64 m;             // Residual's
  int s;
  float top;
  int n;             // accepted drafts
};

IPD_DEVINL bool accepted(const Params &P, int t) {
  const int tok = P.a.tokens[t];
  if (tok < 0 || tok >= P.a.vocab) return false;
  const Row &p = P.rows[2 * t], &q = P.rows[2 * t + 1];
  return __dmul_rn(__dmul_rn((double)P.a.u_accept[t], (double)q.w), (double)p.sum(P.pieces)) <
         __dmul_rn((double)p.w, (double)q.sum(P.pieces));
}

// Log-probability of a drafted token.  (The sum in fp32 is off by 2^-24 of itself, log2f by
// an ulp of a number no larger than the result.)
IPD_DEVINL float logp_of(const Params &P, int row) {
  const int tok = P.a.tokens[row >> 1];
  if (tok < 0 || tok >= P.a.vocab) {
    ipd_set_error(&g_draft_err, IPD_DEVERR_TOKEN);
    return __uint_as_float(0x7fc00000u);
  }
  const Row &R = P.rows[row];
  const u64 z = R.sum(P.pieces);
  return z == 0 ? -INFINITY : (R.x - log2f((float)z * 0x1p-30f)) * kLn2;
}

__device__ __noinline__ void logps(const Params &P, int t) {
  const float lp = logp_of(P, 2 * t), lq = logp_of(P, 2 * t + 1);
  if (P.a.logp_target) P.a.logp_target[t] = lp;
  if (P.a.logp_draft) P.a.logp_draft[t] = lq;
}

// What a residual is taken from: the target's row and the draft's, and their ratio.
struct Residual {
  RowView p, q;
  Weigher wp, wq;
  u64 m;       // 0: nothing is taken off
  int s, off;  // off: the draft row's entries lie this much further on in its vectors

  // target vector i, and the draft row's entries of the same ids
  IPD_DEVINL void load(int i, uint4 &v, uint4 &o) const {
    v = p.get(i);
    o = v;
    if (m != 0) {
      if (off == 0) {
        o = q.get(i);
      } else {  // rows of different alignment: entry by entry
        const uint16_t *l = reinterpret_cast<const uint16_t *>(q.base) + q.before;
        uint32_t *w = &o.x;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const int at = i * 8 + e - p.before;
          const uint32_t lo = at >= 0 && at < p.entries ? l[at] : 0xff80u,
                         hi = at + 1 >= 0 && at + 1 < p.entries ? l[at + 1] : 0xff80u;
          w[e >> 1] = lo | hi << 16;
        }
      }
    }
  }
  // their weights
  IPD_DEVINL void eight(const uint4 &v, const uint4 &o, uint32_t (&r)[8]) const {
    if (wp.mode == kNear && wq.mode == kNear) {
      wp.eight<kNear>(v, r);
      if (m != 0) {
        uint32_t g[8];
        wq.eight<kNear>(o, g);
        take(r, g);
      }
    } else {
      const uint32_t vw[4] = {v.x, v.y, v.z, v.w}, ow[4] = {o.x, o.y, o.z, o.w};
      uint32_t g[8] = {};
#pragma unroll 1
      for (int k = 0; k < 4; ++k) {
        uint32_t a, b, c, d;
        wp.any_two(vw[k], a, b);
        wq.any_two(ow[k], c, d);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (j == k) r[2 * j] = a, r[2 * j + 1] = b, g[2 * j] = c, g[2 * j + 1] = d;
      }
      if (m != 0) take(r, g);
    }
  }
  IPD_DEVINL void take(uint32_t (&r)[8], const uint32_t (&g)[8]) const {
    const uint32_t mm = (uint32_t)m;
    if (s >= 32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t less = __umulhi(g[e], mm) >> (s - 32);
        r[e] = max(r[e], less) - less;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const u64 p = (u64)g[e] * mm;
        const uint32_t hi = (uint32_t)(p >> 32), less = hi >> s ? 0xffffffffu : __funnelshift_r((uint32_t)p, hi, s);
        r[e] = max(r[e], less) - less;
      }
    }
  }
};

__global__ void __launch_bounds__(kThreads, 2) draft_verdict_kernel(const __grid_constant__ Params P) {
  __shared__ Verdict S;
  const ipd_draft_args &a = P.a;
  const uint32_t csize = cluster_size(), rank = cluster_rank();
  const int r = blockIdx.x / csize, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int c0 = a.cu_draft[r], c1 = a.cu_draft[r + 1];
  const float cp = scale_of(a.inv_temp_target, r), cq = scale_of(a.inv_temp_draft, r);
  const bool spans = c0 >= 0 && c1 >= c0 && c1 <= a.total;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // what the row pass wrote
  const auto refuse = [&](unsigned int code) {
    if (rank == 0 && threadIdx.x == 0) {
      ipd_set_error(&g_draft_err, code);
      a.n_accept[r] = 0;
      a.next_token[r] = -1;
    }
  };
  if (!spans || !valid(cp) || !valid(cq)) {
    refuse(spans ? IPD_DEVERR_SETTING : IPD_DEVERR_SPAN);
    if (spans && rank == 0)
      for (int t = c0 + threadIdx.x; t < c1; t += kThreads) {
        if (P.rows[2 * t].owner != r) continue;
        if (a.logp_target) a.logp_target[t] = __uint_as_float(0x7fc00000u);
        if (a.logp_draft) a.logp_draft[t] = __uint_as_float(0x7fc00000u);
      }
    return;
  }
  // The log-probabilities come last, from warps that the search for the token leaves.
  const auto report = [&]() {
    if (rank == csize - 1)
      for (int t = c0 + threadIdx.x; t < c1; t += kThreads) logps(P, t);
  };
  if (threadIdx.x == 0) S.n = c1 - c0;
  __syncthreads();
  // (offsets out of order can give a position to two requests: its rows are weighed for one)
  for (int t = c0 + threadIdx.x; t < c1; t += kThreads) {
    const int owner = P.rows[2 * t].owner;
    const bool ok = accepted(P, t);
    if (owner != r || !ok) atomicMin(&S.n, owner != r ? -1 : t - c0);
  }
  __syncthreads();
  if (S.n < 0) return refuse(IPD_DEVERR_SPAN);
  const int n = S.n;
  const bool full = n == c1 - c0;
  if (rank == 0 && threadIdx.x == 0) a.n_accept[r] = n;
  const int at = c0 + n;
  float top = 0.f, top_q = 0.f;
  if (!full) {
    const Row &p = P.rows[2 * at], &q = P.rows[2 * at + 1];
    top = p.top, top_q = q.top;
    if (threadIdx.x == 0) {  // (the fp64 unit is narrow: once)
      const u64 zp = p.sum(P.pieces), zq = q.sum(P.pieces);
      S.m = 0, S.s = 0;
      if (zp != 0 && zq != 0) {  // (the quotient's leading 31 bits)
        const u64 f = (u64)__double_as_longlong(__ddiv_rn((double)zp, (double)zq));
        S.m = (f & 0xfffffffffffffull | 1ull << 52) >> 22;
        S.s = 31 + 1022 - (int)(f >> 52);  // 13 .. 49
      }
    }
  }
  if (full ? !a.logits_bonus : top == -INFINITY) {
    if (rank == 0 && threadIdx.x == 0) a.next_token[r] = -1;
    return report();
  }
  const uint16_t *pp = full ? a.logits_bonus + (long long)r * a.bonus_stride
                            : a.logits_target + (long long)at * a.target_stride;
  const uint16_t *pq = full ? pp : a.logits_draft + (long long)at * a.draft_stride;
  const RowView vp(pp, a.vocab), vq(pq, a.vocab);
  const int from = min((int)rank * P.piece, vp.n_vec), to = min(from + P.piece, vp.n_vec);
  if (full) {
    top = block_max(piece_max(vp, from, to), S.fred);
    if (csize > 1) {
      if (threadIdx.x == 0) S.top = top;
      cluster_sync();
      if (lane < (int)csize) top = __uint_as_float(remote_ld(remote(&S.top, lane)));
      top = warp_max(top);
    }
  }
  __syncthreads();
  Residual D{vp, vq, Weigher(top, cp, P.one), Weigher(top_q, cq, P.one), full ? 0ull : S.m, full ? 0 : S.s, vq.before - vp.before};
  // Sums of the tiles.  A second time with the target's weights alone where
  // nothing is left of them.
  const int tiles = (to - from + 31) / 32;
  u64 total = 0, before = 0;
  for (int round = 0; round < 2; ++round) {
    if (round && csize > 1) cluster_wait();  // (the others have read S.sum)
    u64 mine = 0;
    uint4 v, o;  // the next tile's, under way
    if (from + warp * 32 + lane < to) D.load(from + warp * 32 + lane, v, o);
    for (int k = warp; k < tiles; k += kWarps) {
      const int i = from + k * 32 + lane, ahead = i + kWarps * 32;
      const uint4 v0 = v, o0 = o;
      if (ahead < to) D.load(ahead, v, o);
      u64 s = 0;
      if (i < to) {
        uint32_t w[8];
        D.eight(v0, o0, w);
        // (a weight is at most 2^30)
        s = (u64)(w[0] + w[1] + w[2]) + (u64)(w[3] + w[4] + w[5]) + (u64)(w[6] + w[7]);
      }
      s = warp_sum40(s);
      if (lane == 0) S.tile[k] = s, mine += s;
    }
    __syncthreads();  // (S.red is read by the round before)
    const u64 sum = block_sum(mine, S.red);
    total = sum, before = 0;
    if (csize > 1) {
      if (threadIdx.x == 0) S.sum = sum;
      cluster_sync();
      const u64 part = lane < (int)csize ? remote_ld64(&S.sum, lane) : 0ull;
      total = warp_sum64(part);
      before = warp_sum64(lane < (int)rank ? part : 0ull);
      cluster_arrive();  // (waited for before S.sum changes, and at the end)
    }
    if (total != 0 || D.m == 0) break;
    D.m = 0;
  }
  if (csize > 1) cluster_wait();
  if (total == 0 || warp != 0) {
    if (total == 0 && rank == 0 && threadIdx.x == 0) a.next_token[r] = -1;  // (a bonus row without an entry)
    return report();
  }
  report();
  const float u = a.u_next[r];
  const double d = u > 0.f ? floor(__dmul_rn((double)u, (double)total)) : 0.0;
  const u64 pos = d < (double)total ? (u64)d : total - 1;
  if (pos < before) return;
  u64 left = pos - before;
  // the tile: 32 at a time
  int k0 = 0;
  u64 sum = 0, v = 0;
  for (;; k0 += 32) {
    if (k0 >= tiles) return;  // in a later CTA's piece
    v = k0 + lane < tiles ? S.tile[k0 + lane] : 0;
    sum = warp_sum64(v);
    if (left < sum) break;
    left -= sum;
  }
  auto scan = [&](u64 x) {  // inclusive, over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    return x;
  };
  u64 up = scan(v);
  int who = __ffs(__ballot_sync(0xffffffffu, left < up)) - 1;
  left -= __shfl_sync(0xffffffffu, up - v, who);
  const int i = from + (k0 + who) * 32 + lane;
  uint32_t w[8] = {};
  if (i < to) {
    uint4 x, y;
    D.load(i, x, y);
    D.eight(x, y, w);
  }
  v = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) v += w[e];
  up = scan(v);
  who = __ffs(__ballot_sync(0xffffffffu, left < up)) - 1;
  if (lane != who) return;
  left -= up - v;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if (left < w[e]) {
      a.next_token[r] = i * 8 + e - vp.before;
      return;
    }
    left -= w[e];
  }
}

int g_sms[64];

int launch(void (*kernel)(Params), int grid, int csize, int threads, int shared, bool follows, const Params &P,
           cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid * csize);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)shared;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = csize;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = follows ? 2 : 1;  // begins as the kernel before ends, and waits for what that wrote
  if (cudaLaunchKernelEx(&cfg, kernel, P) != cudaSuccess) {
    (void)cudaGetLastError();
    return IPD_ERR_CUDA;
  }
  return IPD_OK;
}

}  // namespace

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_draft_error() {
  if (!g_draft_used.load(std::memory_order_relaxed)) return 0u;
  unsigned int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_draft_err, sizeof(v)) != cudaSuccess) return 0xffffffffu;
  if (cudaMemcpyToSymbol(g_draft_err, &z, sizeof(z)) != cudaSuccess) return 0xffffffffu;
  return v;
}

extern "C" size_t ipd_verify_draft_workspace_size(int num_reqs, int total, int vocab) {
  if (num_reqs < 0 || total < 0 || vocab < 1) return 0;
  return (2 * (size_t)total * sizeof(Row) + 255) / 256 * 256;
}

extern "C" int ipd_verify_draft(const ipd_draft_args *args, void *workspace,
                                size_t workspace_bytes, ipd_stream_t stream) {
  if (!args) return IPD_ERR_INVALID_ARG;
  const ipd_draft_args &a = *args;
  if (a.num_reqs < 0 || a.total < 0 || a.vocab < 1) return IPD_ERR_INVALID_ARG;
  if (a.vocab > IPD_TRUNC_MAX_VOCAB || a.total > (1 << 26) || a.num_reqs > (1 << 26))
    return IPD_ERR_UNSUPPORTED;
  if (a.num_reqs == 0) return IPD_OK;
  if (!a.cu_draft || !a.u_next || !a.n_accept || !a.next_token) return IPD_ERR_INVALID_ARG;
  if (a.total > 0 && (!a.logits_target || !a.logits_draft || !a.tokens || !a.u_accept))
    return IPD_ERR_INVALID_ARG;
  if (((uintptr_t)a.logits_target | (uintptr_t)a.logits_draft | (uintptr_t)a.logits_bonus) & 1)
    return IPD_ERR_INVALID_ARG;
  if (a.target_stride < 0 || a.draft_stride < 0 || a.bonus_stride < 0) return IPD_ERR_INVALID_ARG;
  const size_t need = ipd_verify_draft_workspace_size(a.num_reqs, a.total, a.vocab);
  if (need && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 15)))
    return IPD_ERR_WORKSPACE;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return IPD_ERR_CUDA;
  if (g_sms[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return IPD_ERR_CUDA;
    if (cudaFuncSetAttribute(draft_verdict_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
      return IPD_ERR_CUDA;
    g_sms[dev] = n;
  }
  const int sms = g_sms[dev];
  Params P;
  memset(&P, 0, sizeof(P));
  P.a = a;
  P.rows = static_cast<Row *>(workspace);
  P.one = 1.f;
  const int vecs = (a.vocab + 14) / 8;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  g_draft_used.store(true, std::memory_order_relaxed);
  if (a.total > 0) {
    // CTAs of a row: as many (1, 2, 4, 8) as leave every CTA a quarter of an SM (32 requests of up to 6
    // drafts over 151,936 entries: row pass 30.6 us at 2, 34.6 at 1)
    int c = kMaxCluster;
    while (c > 1 && (2LL * a.total * c > 4LL * sms || vecs < c * 512)) c /= 2;
    P.piece = (vecs + c - 1) / c;
    P.pieces = c;
    const bool hist = P.piece * 8 >= (c > 1 ? kHistPiece : kHistRow);
    if (launch(hist ? draft_rows_kernel<true> : draft_rows_kernel<false>, 2 * a.total, c, hist ? kHistThreads : kPlainThreads,
               hist ? kBins * 4 : 0, false, P, st) != IPD_OK)
      return IPD_ERR_CUDA;
  }
  // CTAs of a verdict: as many (to 16) as leave every CTA half an SM (one request over 151,936
  // entries: 22.6 us at 4, 18.5 at 8, 17.8 at 16)
  int c = kMaxVerdict;
  while (c > 1 && ((long long)a.num_reqs * c > 2LL * sms || vecs < c * 512)) c /= 2;
  P.piece = (vecs + 32 * c - 1) / (32 * c) * 32;
  return launch(draft_verdict_kernel, a.num_reqs, c, kThreads, 0, a.total > 0, P, st);
}

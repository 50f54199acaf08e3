// One token per row from the softmax at a temperature, cut by top-k, min-p and
// top-p, from a given uniform number: one launch, each logit read once.
//
// The draw is a fixed function of (row, settings, u), the same on any device,
// because its sums are of whole numbers and so depend on no order:
//   c   = fl(fp32(log2 e) * inv_temperature)
//   x_v = fl(fl(l_v - l_max) c)                          (0 for l_v == l_max)
//   w_v = floor(2^30 2^x_v + 1/2), 2^x by the fp32 procedure below (weight2)
// with the entries in the order of falling logit, lower id first:
//   top-k   the first k entries
//   min-p   of those, the ones with w_v >= ceil(2^30 min_p)
//   top-p   of those, the shortest prefix with a mass of at least
//           ceil(top_p M), M the mass (sum of w) of what is left
//   token   the entry in which floor(u S) falls, S the mass of what is kept
//   logp    ln 2 (x_token - log2(2^-30 S))
// A sum is below 2^48, so the two products in fp64 see exact sums.
//
// What bounds it: a row's bytes are read once (HBM), and then everything
// happens in shared memory: a cluster of 1 to 8 CTAs holds a row, an equal
// piece each.  The three cuts and the draw are the same question, "which entry
// holds position t of the running sum of counts (or weights) from the largest
// logit down", answered in two steps: a histogram over the top 12 bits of the
// logits' order (4,096 bins, integer atomics in shared memory) finds the bin,
// and a count of the bin's 16 logit values finds the value; entries of one
// value have one weight, so the rest is a division, and the rank that is left
// is looked up in index order.  bf16 logits make this exact without sorting:
// equal logits are the only ties, and there are 16 values to a bin.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

IPD_DECLARE_ERROR_WORD(g_trunc_err);

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 4096;             // order key >> 4
constexpr int kValues = 16;             // order keys in a bin
constexpr int kMaxCluster = 8;          // portable cluster size
constexpr int kMaxPiece = 32768;        // entries of one CTA: 2^15 * 2^16 fits the histogram words
static_assert(IPD_TRUNC_MAX_VOCAB + 7 <= kMaxPiece * kMaxCluster, "a row fits one cluster");
constexpr float kMagic = 12582912.f;    // 1.5 * 2^23: x + kMagic rounds x to a whole number

typedef unsigned long long u64;

struct Settings {
  const float *inv_t, *top_p, *min_p;
  const int32_t *top_k;
};

struct Params {
  const uint16_t *logits;
  long long stride;
  const float *u;
  Settings set;
  int32_t *tokens, *kept;
  float *logp;
  int vocab, piece;  // piece: entries a CTA holds (a multiple of 8)
};

struct Shared {
  uint32_t lo[kBins], hi[kBins];  // per bin: sums of the weights' low and high 16 bits, or counts
  u64 slice[kMaxCluster];         // mass of each CTA's slice of bins
  u64 win_before;                 // the bin a search found, and the mass above it
  uint32_t win_bin;
  uint32_t count[kMaxCluster][kValues + 1];  // per CTA: entries of each value of a bin, and of kept
  uint32_t mine[kValues + 1];
  uint32_t max_key[kMaxCluster];
  u64 scan[kWarps];
  uint32_t warp_count[kWarps];
  u64 found_before;
  uint32_t found_key;
  uint32_t top;
};
// the CTA's entries follow, as bf16 (0x8000 and NaN do not occur in them)

// ---- cluster ---------------------------------------------------------------
IPD_DEVINL uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
IPD_DEVINL uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
IPD_DEVINL void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
IPD_DEVINL void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
IPD_DEVINL void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
IPD_DEVINL uint32_t remote(const void *p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
IPD_DEVINL uint32_t remote_ld(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
IPD_DEVINL void remote_st(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
IPD_DEVINL void remote_st64(uint32_t addr, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

// ---- order keys --------------------------------------------------------------
// bf16 bits -> a 16-bit key that rises with the value, for two entries at once
IPD_DEVINL uint32_t order2(uint32_t w) {
  const uint32_t neg = ((w >> 15) & 0x00010001u) * 0xffffu;
  return w ^ (neg | 0x80008000u);
}
IPD_DEVINL float key_value(uint32_t key) {
  return bf16f((uint16_t)((key & 0x8000u) ? key ^ 0x8000u : ~key));
}
constexpr uint32_t kKeyMinusInf = 0x007fu;

// NaN -> -inf, -0 -> +0 (two entries)
IPD_DEVINL uint32_t clean2(uint32_t w) {
  __nv_bfloat162 v = *reinterpret_cast<__nv_bfloat162 *>(&w);
  const uint32_t ninf = 0xff80ff80u, zero = 0u;
  v = __hmax2(v, *reinterpret_cast<const __nv_bfloat162 *>(&ninf));
  v = __hadd2(v, *reinterpret_cast<const __nv_bfloat162 *>(&zero));
  return *reinterpret_cast<uint32_t *>(&v);
}
IPD_DEVINL uint32_t max2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&a),
                                   *reinterpret_cast<__nv_bfloat162 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&m);
}

// ---- weights -------------------------------------------------------------------
IPD_DEVINL u64 f2_mul(u64 a, u64 b) {
  u64 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

struct Scale {
  float top, c;     // l_max and fl(log2 e * inv_temperature)
  bool inf;         // l_max is +inf: its entries have weight 2^30, the others 0
  uint32_t min_w;   // smallest weight that counts (min-p; at least 1)
};

// w of two entries: 2^x = 2^i P(f), i = x rounded, f = x - i in [-1/2, 1/2], P
// by Horner's rule, every product and sum rounded to fp32 on its own; P is a
// least-squares fit of 2^f on Chebyshev nodes with constant term 1 (relative
// error below 1.9e-7 with its rounding).
IPD_DEVINL void weight2(const Scale &S, float l0, float l1, uint32_t &w0, uint32_t &w1) {
  if (S.inf) {
    w0 = l0 == S.top ? 1u << 30 : 0u;
    w1 = l1 == S.top ? 1u << 30 : 0u;
  } else {
    float a, b;
    f2_unpack(f2_mul(f2_sub(f2_pack(l0, l1), f2_pack(S.top, S.top)), f2_pack(S.c, S.c)), a, b);
    const u64 x = f2_pack(fmaxf(a, -64.f), fmaxf(b, -64.f));
    const u64 r = f2_add(x, f2_pack(kMagic, kMagic));
    const u64 f = f2_sub(x, f2_sub(r, f2_pack(kMagic, kMagic)));
    const float c1 = __uint_as_float(0x3f317213u), c2 = __uint_as_float(0x3e75fcdbu),
                c3 = __uint_as_float(0x3d635d55u), c4 = __uint_as_float(0x3c1e760bu),
                c5 = __uint_as_float(0x3aad4281u);
    u64 p = f2_pack(c5, c5);
    p = f2_add(f2_mul(p, f), f2_pack(c4, c4));
    p = f2_add(f2_mul(p, f), f2_pack(c3, c3));
    p = f2_add(f2_mul(p, f), f2_pack(c2, c2));
    p = f2_add(f2_mul(p, f), f2_pack(c1, c1));
    p = f2_add(f2_mul(p, f), f2_pack(1.f, 1.f));
    float r0, r1, p0, p1;
    f2_unpack(r, r0, r1);
    f2_unpack(p, p0, p1);
    // 2^31 2^x: i and 31 into the exponent; truncated, then halved upwards
    const float y0 = __uint_as_float(__float_as_uint(p0) + (__float_as_uint(r0) << 23) + (31u << 23));
    const float y1 = __uint_as_float(__float_as_uint(p1) + (__float_as_uint(r1) << 23) + (31u << 23));
    w0 = (__float2uint_rz(y0) + 1u) >> 1;
    w1 = (__float2uint_rz(y1) + 1u) >> 1;
  }
  if (w0 < S.min_w) w0 = 0u;
  if (w1 < S.min_w) w1 = 0u;
}
IPD_DEVINL uint32_t weight_of_key(const Scale &S, uint32_t key) {
  uint32_t a, b;
  const float l = key_value(key);
  weight2(S, l, l, a, b);
  return a;
}

// ---- searches --------------------------------------------------------------------
// The cluster's histogram, cut into one slice of bins per CTA (slice 0 holds
// the highest bins) and a run of bins per thread, with the mass above each.
struct Slices {
  u64 above;   // mass of the bins above this thread's run, within its slice
  u64 run;     // mass of the run
  u64 before;  // mass of the slices above
  u64 total;
};

IPD_DEVINL uint32_t bin_at(uint32_t rank, uint32_t csize, int i) {
  return kBins - 1 - (rank * (kBins / csize) + i);
}
IPD_DEVINL u64 bin_mass(const Shared &S, uint32_t csize, uint32_t bin) {
  u64 v = 0;
  for (uint32_t p = 0; p < csize; ++p)
    v += (u64)remote_ld(remote(&S.lo[bin], p)) + ((u64)remote_ld(remote(&S.hi[bin], p)) << 16);
  return v;
}

// After the histograms are written: two cluster barriers.
__device__ Slices reduce_histogram(Shared &S, uint32_t rank, uint32_t csize) {
  cluster_sync();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = kBins / (int)csize / kThreads;  // bins of a thread's run: 8 / csize
  Slices R;
  R.run = 0;
  for (int b = 0; b < per; ++b) R.run += bin_mass(S, csize, bin_at(rank, csize, tid * per + b));
  u64 inc = R.run;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  if (lane == 31) S.scan[warp] = inc;
  __syncthreads();
  u64 base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const u64 t = S.scan[w];
    if (w < warp) base += t;
    sum += t;
  }
  R.above = base + inc - R.run;
  if (tid < (int)csize) remote_st64(remote(&S.slice[rank], tid), sum);
  cluster_sync();
  R.before = 0;
  R.total = 0;
  for (uint32_t p = 0; p < csize; ++p) {
    const u64 t = S.slice[p];
    if (p < rank) R.before += t;
    R.total += t;
  }
  return R;
}

// The bin holding position t (0 <= t < total) of the running sum: every CTA
// has it in S.win_bin / S.win_before afterwards.  One cluster barrier.
__device__ void find_bin(Shared &S, const Slices &R, uint32_t rank, uint32_t csize, u64 t) {
  const u64 at = R.before + R.above;
  if (t >= at && t - at < R.run) {
    const int per = kBins / (int)csize / kThreads;
    u64 before = at;
    uint32_t bin = bin_at(rank, csize, threadIdx.x * per);
    for (int b = 0; b + 1 < per; ++b) {
      const u64 v = bin_mass(S, csize, bin);
      if (t - before < v) break;
      before += v;
      --bin;
    }
    for (uint32_t p = 0; p < csize; ++p) {
      remote_st(remote(&S.win_bin, p), bin);
      remote_st64(remote(&S.win_before, p), before);
    }
  }
  cluster_sync();
}

// Counts this CTA's entries of each value of a bin (and whatever `also`
// counts), and gives every CTA all the counts.  One cluster barrier.
template <typename Also>
__device__ void count_values(Shared &S, const uint32_t *data, int words, uint32_t rank,
                             uint32_t csize, uint32_t bin, Also also) {
  const int tid = threadIdx.x;
  if (tid <= kValues) S.mine[tid] = 0;
  __syncthreads();
  uint32_t extra = 0;
  for (int i = tid; i < words; i += kThreads) {
    const uint32_t w = data[i], k = order2(w);
    if (((k >> 4) & 0xfffu) == bin) atomicAdd(&S.mine[k & 15u], 1u);
    if ((k >> 20) == bin) atomicAdd(&S.mine[(k >> 16) & 15u], 1u);
    extra += also(w, k);
  }
  extra = __reduce_add_sync(0xffffffffu, extra);
  if ((tid & 31) == 0 && extra) atomicAdd(&S.mine[kValues], extra);
  __syncthreads();
  for (int i = tid; i < (kValues + 1) * (int)csize; i += kThreads)
    remote_st(remote(&S.count[rank][i % (kValues + 1)], i / (kValues + 1)), S.mine[i % (kValues + 1)]);
  cluster_sync();
}

// The value of bin `win` holding position t, the mass above it, from the
// counts; weight(key, n) is the weight of an entry and limits n.  All threads.
template <typename Weight>
__device__ void find_value(Shared &S, uint32_t csize, u64 t, Weight weight, uint32_t &key,
                           u64 &before) {
  if (threadIdx.x < 32) {
    const int v = threadIdx.x & 15;
    uint32_t n = 0;
    for (uint32_t p = 0; p < csize; ++p) n += S.count[p][v];
    const uint32_t k = S.win_bin * kValues + v;
    const uint32_t w = weight(k, n);
    const u64 mass = (u64)w * n;
    u64 b = S.win_before;
    int at = 0;
    for (int i = kValues - 1; i >= 0; --i) {
      const u64 m = __shfl_sync(0xffffffffu, mass, i);
      at = i;
      if (t - b < m) break;
      if (i > 0) b += m;
    }
    if (threadIdx.x == 0) {
      S.found_key = S.win_bin * kValues + at;
      S.found_before = b;
    }
  }
  __syncthreads();
  key = S.found_key;
  before = S.found_before;
}

__global__ void __launch_bounds__(kThreads, 2) sample_trunc_kernel(const __grid_constant__ Params P) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Shared &S = *reinterpret_cast<Shared *>(smem_raw);
  uint32_t *data = reinterpret_cast<uint32_t *>(smem_raw + ((sizeof(Shared) + 15) & ~15ull));
  const uint32_t rank = cluster_rank(), csize = cluster_size();
  const int row = blockIdx.x / csize;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float inv_t = P.set.inv_t ? P.set.inv_t[row] : 1.f;
  const float top_p = P.set.top_p ? P.set.top_p[row] : 1.f;
  const float min_p = P.set.min_p ? P.set.min_p[row] : 0.f;
  const int top_k = P.set.top_k ? P.set.top_k[row] : 0;
  cluster_arrive();  // (waited for below: no CTA's memory is written before it runs)
  Scale C;
  C.c = __fmul_rn(kLog2e, inv_t);
  const bool good = C.c > 0.f && C.c - C.c == 0.f && top_p == top_p && min_p >= 0.f && min_p <= 1.f;
  if (!good && rank == 0 && tid == 0) ipd_set_error(&g_trunc_err, IPD_DEVERR_SETTING);

  // ---- the CTA's piece of the row, and the largest logit ----
  // pieces are cut at 16-byte boundaries: entry i of the row sits at i + shift
  const uint16_t *src = P.logits + (long long)row * P.stride;
  const int shift = (int)(((uintptr_t)src & 15) >> 1);
  const uint16_t *base = src - shift;
  const int i0 = (int)rank * P.piece;  // in shifted entries
  const int n_vec = P.piece / 8;
  const int end = P.vocab + shift;
  uint32_t mx = 0xff80ff80u;
#pragma unroll 4
  for (int v = tid; v < n_vec; v += kThreads) {
    const int i = i0 + 8 * v;
    uint4 w = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
    if (i >= shift && i + 8 <= end) {
      w = ldg_stream(base + i);
    } else {
      uint16_t e[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = i + k >= shift && i + k < end ? base[i + k] : 0xff80u;
      w.x = e[0] | (uint32_t)e[1] << 16, w.y = e[2] | (uint32_t)e[3] << 16;
      w.z = e[4] | (uint32_t)e[5] << 16, w.w = e[6] | (uint32_t)e[7] << 16;
    }
    w = make_uint4(clean2(w.x), clean2(w.y), clean2(w.z), clean2(w.w));
    reinterpret_cast<uint4 *>(data)[v] = w;
    mx = max2(max2(max2(mx, w.x), max2(w.y, w.z)), w.w);
  }
  for (int i = tid; i < kBins; i += kThreads) S.lo[i] = 0, S.hi[i] = 0;
  if (tid == 0) S.top = 0;
  __syncthreads();
  {
    const uint32_t k = order2(mx);
    const uint32_t m = __reduce_max_sync(0xffffffffu, max(k & 0xffffu, k >> 16));
    if (lane == 0) atomicMax(&S.top, m);
  }
  __syncthreads();
  cluster_wait();
  if (tid < (int)csize) remote_st(remote(&S.max_key[rank], tid), S.top);
  cluster_sync();
  uint32_t top_key = 0;
  for (uint32_t p = 0; p < csize; ++p) top_key = max(top_key, S.max_key[p]);
  // a row with nothing but -inf and NaN, or bad settings: no token
  if (!good || top_key <= kKeyMinusInf) {
    if (rank == 0 && tid == 0) {
      P.tokens[row] = -1;
      if (P.logp) P.logp[row] = -INFINITY;
      if (P.kept) P.kept[row] = 0;
    }
    return;  // the whole cluster
  }
  C.top = key_value(top_key);
  C.inf = top_key == 0xff80u;
  const double thr = ceil((double)min_p * 1073741824.0);
  C.min_w = thr > 1.0 ? (uint32_t)thr : 1u;
  // entries below this have x < -32 and so weight 0
  const float least = C.inf ? C.top : C.top - 33.f / C.c;
  const int words = P.piece / 2;

  // ---- top-k: its last value, and how many entries of that value are in ----
  uint32_t key_k = 0, in_k = 0;  // entries with a greater key, and in_k of key_k
  if (top_k > 0 && top_k < P.vocab) {
    for (int i = tid; i < words; i += kThreads) {
      const uint32_t w = data[i], k = order2(w);
      if (bf16lo(w) >= least) atomicAdd(&S.lo[(k >> 4) & 0xfffu], 1u);
      if (bf16hi(w) >= least) atomicAdd(&S.lo[k >> 20], 1u);
    }
    const Slices R = reduce_histogram(S, rank, csize);
    if (R.total > (u64)top_k) {
      find_bin(S, R, rank, csize, (u64)top_k - 1);
      // the bin's values counted under the same bound as the histogram
      count_values(S, data, words, rank, csize, S.win_bin,
                   [](uint32_t, uint32_t) { return 0u; });
      u64 before;
      find_value(S, csize, (u64)top_k - 1, [](uint32_t, uint32_t) { return 1u; }, key_k, before);
      in_k = (uint32_t)((u64)top_k - before);
    }
    __syncthreads();
    for (int i = tid; i < kBins; i += kThreads) S.lo[i] = 0;
    __syncthreads();
  }
  // the first in_k entries of key_k in index order: this CTA's share
  uint32_t share = 0;
  if (key_k) {
    uint32_t before = 0;
    for (uint32_t p = 0; p < rank; ++p) before += S.count[p][key_k & 15u];
    const uint32_t here = S.count[rank][key_k & 15u];
    share = in_k > before ? min(in_k - before, here) : 0u;
  }

  // ---- the masses of the bins ----
  for (int i = tid; i < words; i += kThreads) {
    const uint32_t w = data[i], k = order2(w);
    const float l0 = bf16lo(w), l1 = bf16hi(w);
    if (l0 < least && l1 < least) continue;
    const uint32_t k0 = k & 0xffffu, k1 = k >> 16;
    uint32_t w0, w1;
    weight2(C, l0, l1, w0, w1);
    if (k0 <= key_k) w0 = 0;
    if (k1 <= key_k) w1 = 0;
    if (w0) {
      atomicAdd(&S.lo[k0 >> 4], w0 & 0xffffu);
      if (w0 >> 16) atomicAdd(&S.hi[k0 >> 4], w0 >> 16);
    }
    if (w1) {
      atomicAdd(&S.lo[k1 >> 4], w1 & 0xffffu);
      if (w1 >> 16) atomicAdd(&S.hi[k1 >> 4], w1 >> 16);
    }
  }
  if (share && tid == 0) {
    const uint32_t w = weight_of_key(C, key_k);
    atomicAdd(&S.lo[key_k >> 4], share * (w & 0xffffu));
    atomicAdd(&S.hi[key_k >> 4], share * (w >> 16));
  }
  const Slices R = reduce_histogram(S, rank, csize);
  // an entry's weight in the sums, with the number of entries of its value that
  // are in the top k
  const auto weight = [&](uint32_t key, uint32_t &n) -> uint32_t {
    if (key < key_k) n = 0;
    else if (key == key_k) n = min(n, in_k);
    return n ? weight_of_key(C, key) : 0u;
  };
  // R.total >= 1: the largest logit has weight 2^30 >= min_w and rank 0

  // ---- top-p: its last value, and the mass that is kept ----
  uint32_t key_p = 0, in_p = 0;  // entries with a greater key, and in_p of key_p
  u64 kept_mass = R.total;
  {
    double need = ceil((double)top_p * (double)R.total);
    need = need < 1.0 ? 1.0 : need;
    if (need < (double)R.total) {
      const u64 last = (u64)need - 1;  // position of the last unit of mass that is needed
      find_bin(S, R, rank, csize, last);
      count_values(S, data, words, rank, csize, S.win_bin,
                   [](uint32_t, uint32_t) { return 0u; });
      u64 before;
      find_value(S, csize, last, [&](uint32_t k, uint32_t &n) { return weight(k, n); }, key_p,
                 before);
      const uint32_t w = weight_of_key(C, key_p);
      in_p = (uint32_t)((last - before) / w) + 1;
      kept_mass = before + (u64)in_p * w;
    }
  }

  // ---- the draw ----
  const float uf = P.u[row];
  u64 t = 0;
  if (uf > 0.f) {
    const double d = floor((double)uf * (double)kept_mass);
    t = d < (double)kept_mass ? (u64)d : kept_mass - 1;
  }
  find_bin(S, R, rank, csize, t);
  // with the values of the bin, the entries that are kept besides in_p (or, when
  // all of the top k is, in_k): greater keys with a weight.  The exponent x
  // decides wherever it is more than 0.01 from the smallest weight that counts
  // (w >= min_w at 2^30 2^x >= min_w - 1/2); between, the weight itself.
  const uint32_t edge = key_p ? key_p : key_k;
  const float x_in = log2f((float)C.min_w) - 29.99f, x_out = log2f((float)C.min_w - 0.5f) - 30.01f;
  count_values(S, data, words, rank, csize, S.win_bin, [&](uint32_t w, uint32_t k) {
    const bool a = (k & 0xffffu) > edge, b = (k >> 16) > edge;
    if (!a && !b) return 0u;
    const float l0 = bf16lo(w), l1 = bf16hi(w);
    const float x0 = __fmul_rn(__fsub_rn(l0, C.top), C.c), x1 = __fmul_rn(__fsub_rn(l1, C.top), C.c);
    uint32_t w0 = x0 >= x_in, w1 = x1 >= x_in;
    if (C.inf || (!w0 && x0 >= x_out) || (!w1 && x1 >= x_out)) weight2(C, l0, l1, w0, w1);
    return (uint32_t)(a && w0) + (uint32_t)(b && w1);
  });
  uint32_t key_d;
  u64 before;
  find_value(S, csize, t, [&](uint32_t k, uint32_t &n) { return weight(k, n); }, key_d, before);
  uint32_t j = (uint32_t)((t - before) / weight_of_key(C, key_d));  // rank among the value's entries
  if (rank == 0 && tid == 0 && P.kept) {
    uint32_t n = key_p ? in_p : 0u;
    if (!key_p && key_k && weight_of_key(C, key_k)) n = in_k;
    for (uint32_t p = 0; p < csize; ++p) n += S.count[p][kValues];
    P.kept[row] = (int32_t)n;
  }
  // ---- the j-th entry of key_d, in the CTA and warp that hold it ----
  for (uint32_t p = 0; p < rank; ++p) {
    const uint32_t n = S.count[p][key_d & 15u];
    if (j < n) return;  // an earlier CTA's
    j -= n;
  }
  if (j >= S.count[rank][key_d & 15u]) return;  // a later CTA's
  const int seg = (words + kWarps - 1) / kWarps;
  const int a0 = warp * seg, a1 = min(words, a0 + seg);
  uint32_t mine = 0;
  for (int i = a0 + lane; i < a1; i += 32) {
    const uint32_t k = order2(data[i]);
    mine += ((k & 0xffffu) == key_d) + ((k >> 16) == key_d);
  }
  mine = __reduce_add_sync(0xffffffffu, mine);
  if (lane == 0) S.warp_count[warp] = mine;
  __syncthreads();
  for (int w = 0; w < warp; ++w) {
    const uint32_t n = S.warp_count[w];
    if (j < n) return;
    j -= n;
  }
  if (j >= mine) return;
  for (int i = a0; i < a1; i += 32) {
    const uint32_t k = i + lane < a1 ? order2(data[i + lane]) : 0u;
    const uint32_t e0 = __ballot_sync(0xffffffffu, (k & 0xffffu) == key_d);
    const uint32_t e1 = __ballot_sync(0xffffffffu, (k >> 16) == key_d);
    const uint32_t n = __popc(e0) + __popc(e1);
    if (j >= n) {
      j -= n;
      continue;
    }
    const uint32_t below = (1u << lane) - 1u;
    const uint32_t first = __popc(e0 & below) + __popc(e1 & below);
    const uint32_t is0 = (e0 >> lane) & 1u, is1 = (e1 >> lane) & 1u;
    int hit = -1;
    if (is0 && first == j) hit = 0;
    else if (is1 && first + is0 == j) hit = 1;
    if (hit >= 0) {
      P.tokens[row] = i0 + 2 * (i + lane) + hit - shift;
      if (P.logp) {
        const float x = key_d == top_key ? 0.f : __fmul_rn(__fsub_rn(key_value(key_d), C.top), C.c);
        P.logp[row] = (x - log2f((float)kept_mass * 0x1p-30f)) * kLn2;
      }
    }
    return;
  }
}

struct DevInfo {
  int sms = 0;
};
DevInfo g_trunc_dev[64];

size_t shared_bytes(int piece) { return ((sizeof(Shared) + 15) & ~(size_t)15) + 2 * (size_t)piece; }
constexpr size_t kMaxShared = ((sizeof(Shared) + 15) & ~(size_t)15) + 2 * (size_t)kMaxPiece;

}  // namespace

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_trunc_error() {
  unsigned int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_trunc_err, sizeof(v)) != cudaSuccess) return 0xffffffffu;
  if (cudaMemcpyToSymbol(g_trunc_err, &z, sizeof(z)) != cudaSuccess) return 0xffffffffu;
  return v;
}

extern "C" int ipd_sample_trunc(const uint16_t *logits, int64_t row_stride, int n_rows, int vocab,
                                const float *u, const float *inv_temperature, const int32_t *top_k,
                                const float *top_p, const float *min_p, int32_t *tokens,
                                float *logp, int32_t *n_kept, ipd_stream_t stream) {
  if (n_rows < 0 || vocab < 1 || row_stride < 0) return IPD_ERR_INVALID_ARG;
  if (vocab > IPD_TRUNC_MAX_VOCAB) return IPD_ERR_UNSUPPORTED;
  if (n_rows == 0) return IPD_OK;
  if (!logits || !u || !tokens || ((uintptr_t)logits & 1)) return IPD_ERR_INVALID_ARG;
  if (n_rows > (1 << 27)) return IPD_ERR_UNSUPPORTED;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return IPD_ERR_CUDA;
  DevInfo &D = g_trunc_dev[dev];
  if (D.sms == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaFuncSetAttribute(sample_trunc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)kMaxShared) != cudaSuccess)
      return IPD_ERR_CUDA;
    D.sms = n;
  }
  // CTAs of a row: as many as its entries need, and more while SMs are idle and
  // a piece is more than a few loads a thread
  int csize = 1;
  const long long span = (long long)vocab + 7;  // a row may start inside a 16-byte piece
  while (csize < kMaxCluster &&
         ((span + csize - 1) / csize > kMaxPiece - 7 ||
          ((long long)n_rows * csize < D.sms && span / csize > 2048)))
    csize *= 2;
  Params P;
  P.logits = logits;
  P.stride = row_stride;
  P.u = u;
  P.set = Settings{inv_temperature, top_p, min_p, top_k};
  P.tokens = tokens;
  P.kept = n_kept;
  P.logp = logp;
  P.vocab = vocab;
  P.piece = (int)(((span + csize - 1) / csize + 7) / 8 * 8);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_rows * csize);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = shared_bytes(P.piece);
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = csize;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, sample_trunc_kernel, P) != cudaSuccess) {
    (void)cudaGetLastError();
    return IPD_ERR_CUDA;
  }
  return IPD_OK;
}

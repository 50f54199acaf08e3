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
// piece each.  Two ways from there:
//
// Head: the entries from a threshold up (a value that at least max(top_k, 256)
// entries reach, taken from the threads' own maxima) are gathered in the
// cluster's first CTA, sorted, and summed along; every cut and the draw is then
// a comparison.  Right whenever the answers lie in the head: with a top-k that
// the head holds, always; without, when the mass that top-p needs, or the
// draw's position, is at most the head's (all weights are summed for that).
//
// Histogram: the three cuts and the draw are the same question, "which entry
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

#include <type_traits>

#include "common.cuh"

IPD_DECLARE_ERROR_WORD(g_trunc_err);

namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 4096;             // order key >> 4
constexpr int kValues = 16;             // order keys in a bin
constexpr int kGroupBins = 64, kGroups = kBins / kGroupBins;
constexpr int kMaxCluster = 8;          // portable cluster size
constexpr int kMaxPiece = 32768;        // entries of one CTA: 2^15 * 2^16 fits the histogram words
static_assert(IPD_TRUNC_MAX_VOCAB + 7 <= kMaxPiece * kMaxCluster, "a row fits one cluster");
constexpr int kHead = 2048;             // entries the head holds (sorted by 512 threads, 4 each)
constexpr int kMaxima = kThreads / 2;   // maxima of thread pairs, for the head's threshold
static_assert(kWarps == 16, "the threshold's search tries 4 bits a round");
constexpr int kHeadAim = 256;           // entries aimed at where top-k asks for none
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
  int id_bits;       // vocab <= 2^id_bits, id_bits >= 1
};

struct Shared {
  union {
    struct {
      uint32_t lo[kBins], hi[kBins];  // per bin: sums of the weights' low and high 16 bits, or counts
    };
    struct {
      uint32_t head[kHead];  // first CTA: the cluster's head entries, kHead / size a CTA (pack_entry)
      uint32_t sorted[kHead];
      uint32_t maxima[kMaxima];
    };
  };
  u64 group[kMaxCluster][kGroups];  // per CTA: sums of its groups of bins
  u64 group_before[kGroups + 1];    // the cluster's sum above each group, highest first
  u64 part[kThreads];
  int win_group;
  u64 all_mass[kMaxCluster], head_mass[kMaxCluster];  // per CTA: weights of its entries
  uint32_t all_n[kMaxCluster], head_n[kMaxCluster];   // ... and how many have one, and are in the head
  uint32_t max_key[kMaxCluster], floor_key[kMaxCluster];
  u64 win_before;                 // the bin a search found, and the mass above it
  uint32_t win_bin;
  uint32_t count[kMaxCluster][kValues + 1];  // per CTA: entries of each value of a bin, and of kept
  uint32_t mine[kValues + 1];
  u64 scan[kWarps], scan2[kWarps];
  uint32_t warp_count[kWarps];
  u64 found_before, word;
  uint32_t found_key, list_n;
  uint8_t reached[4][kWarps];
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
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
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
constexpr uint32_t kKeyMinusInf = 0x007fu, kKeyInf = 0xff80u;

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

// 0xffff in each half where the entry of w is >= that of v
IPD_DEVINL uint32_t ge2(uint32_t w, uint32_t v) {
  return __hge2_mask(*reinterpret_cast<__nv_bfloat162 *>(&w), *reinterpret_cast<__nv_bfloat162 *>(&v));
}
// a key's bf16 bits in both halves
IPD_DEVINL uint32_t key_bits2(uint32_t key) {
  const uint32_t b = (key & 0x8000u) ? key ^ 0x8000u : ~key & 0xffffu;
  return b | b << 16;
}

// ---- weights -------------------------------------------------------------------
IPD_DEVINL u64 f2_mul(u64 a, u64 b) {
  u64 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

struct Scale {
  float top, c;     // l_max (finite) and fl(log2 e * inv_temperature)
  uint32_t least2;  // a bf16 value (twice) of weight 0 from which on weights are 0
  bool coarse;      // ... whose x is far below -64: bf16 is coarse at l_max
  uint32_t min_w;   // smallest weight that counts (min-p; at least 1)
};

// w of two entries: 2^x = 2^i P(f), i = x rounded, f = x - i in [-1/2, 1/2], P
// by Horner's rule, every product and sum rounded to fp32 on its own; P is a
// least-squares fit of 2^f on Chebyshev nodes with constant term 1 (relative
// error below 1.9e-7 with its rounding).
template <bool MINW>
IPD_DEVINL void weight2(const Scale &S, uint32_t w, uint32_t &w0, uint32_t &w1) {
  w = max2(w, S.least2);
  u64 x = f2_mul(f2_sub(f2_pack(bf16lo(w), bf16hi(w)), f2_pack(S.top, S.top)), f2_pack(S.c, S.c));
  if (S.coarse) {
    float a, b;
    f2_unpack(x, a, b);
    x = f2_pack(fmaxf(a, -64.f), fmaxf(b, -64.f));
  }
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
  // 2^x: i into the exponent; times 2^31 (exact), truncated, halved upwards
  const u64 y = f2_mul(f2_pack(__uint_as_float(__float_as_uint(p0) + (__float_as_uint(r0) << 23)),
                               __uint_as_float(__float_as_uint(p1) + (__float_as_uint(r1) << 23))),
                       f2_pack(0x1p31f, 0x1p31f));
  float y0, y1;
  f2_unpack(y, y0, y1);
  w0 = (__float2uint_rz(y0) + 1u) >> 1;
  w1 = (__float2uint_rz(y1) + 1u) >> 1;
  if (MINW) {
    if (w0 < S.min_w) w0 = 0u;
    if (w1 < S.min_w) w1 = 0u;
  }
}
IPD_DEVINL uint32_t weight_of_key(const Scale &S, uint32_t key) {
  uint32_t a, b;
  weight2<true>(S, key_bits2(key), a, b);
  return a;
}
// x of an entry, as weight2 has it before any bound
IPD_DEVINL float exponent(const Scale &S, float l) {
  return __fmul_rn(__fsub_rn(l, S.top), S.c);
}

// ---- sums over the CTA -----------------------------------------------------------
IPD_DEVINL u64 warp_sum64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// sum of v over the threads before this one, and over all (two CTA barriers)
__device__ u64 scan_cta(Shared &S, u64 v, u64 &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  if (lane == 31) S.scan[warp] = inc;
  __syncthreads();
  u64 base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const u64 t = S.scan[w];
    if (w < warp) base += t;
    total += t;
  }
  __syncthreads();
  return base + inc - v;
}

// ---- searches --------------------------------------------------------------------
// The cluster's histogram is searched from groups of 64 bins: each CTA sums its
// groups and gives the sums to all, one barrier; every CTA then finds the group
// for itself, reads the group's bins from all and finds the bin.
IPD_DEVINL uint32_t remote_ld(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
IPD_DEVINL u64 bin_sum(const Shared &S, int bin) { return S.lo[bin] + ((u64)S.hi[bin] << 16); }

// After the histograms are written.  One cluster barrier; the histograms must
// then stay until the next.  The cluster's sum of all bins.
__device__ u64 share_groups(Shared &S, uint32_t rank, uint32_t csize) {
  __syncthreads();
  constexpr int kEach = kBins / kThreads;  // 8 bins a thread, 8 threads a group
  static_assert(kEach * 8 == kGroupBins && kMaxCluster <= 8, "a group's threads each serve one CTA");
  const int tid = threadIdx.x;
  u64 v = 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) v += bin_sum(S, kEach * tid + i);
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((tid & 7) < (int)csize) remote_st64(remote(&S.group[rank][tid >> 3], tid & 7), v);
  cluster_sync();
  u64 total = 0;
  if (tid < kGroups) {
#pragma unroll
    for (uint32_t p = 0; p < kMaxCluster; ++p)
      if (p < csize) total += S.group[p][kGroups - 1 - tid];  // highest group first
  }
  u64 sum;
  const u64 before = scan_cta(S, total, sum);
  if (tid < kGroups) S.group_before[tid] = before;
  if (tid == 0) S.group_before[kGroups] = sum;
  __syncthreads();
  return sum;
}

// The bin holding position t (0 <= t < the sum) of the running sum, into
// S.win_bin / S.win_before of this CTA.
__device__ void find_bin(Shared &S, uint32_t csize, u64 t) {
  const int tid = threadIdx.x;
  if (tid < kGroups && t >= S.group_before[tid] && t < S.group_before[tid + 1]) S.win_group = tid;
  __syncthreads();
  const int g = S.win_group, first = (kGroups - g) * kGroupBins - 1;  // the group's highest bin
  // thread: CTA tid / 64, bin tid % 64 from the top
  u64 v = 0;
  const uint32_t p = tid / kGroupBins;
  if (p < csize) {
    const int bin = first - tid % kGroupBins;
    v = remote_ld(remote(&S.lo[bin], p)) + ((u64)remote_ld(remote(&S.hi[bin], p)) << 16);
  }
  S.part[tid] = v;
  __syncthreads();
  if (tid < 32) {  // two bins a lane
    u64 a = 0, b = 0;
#pragma unroll
    for (uint32_t q = 0; q < kMaxCluster; ++q) {
      if (q < csize) a += S.part[q * kGroupBins + 2 * tid], b += S.part[q * kGroupBins + 2 * tid + 1];
    }
    u64 inc = a + b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const u64 x = __shfl_up_sync(0xffffffffu, inc, o);
      if (tid >= o) inc += x;
    }
    const u64 at = S.group_before[g] + inc - a - b;
    if (t >= at && t < at + a) S.win_bin = first - 2 * tid, S.win_before = at;
    if (t >= at + a && t < at + a + b) S.win_bin = first - 2 * tid - 1, S.win_before = at + a;
  }
  __syncthreads();
}

// Counts this CTA's entries of each value of a bin (and whatever `also`
// counts), and gives every CTA all the counts.  One cluster barrier.
template <typename Also>
__device__ void count_values(Shared &S, const uint4 *data, int vecs, uint32_t rank, uint32_t csize,
                             uint32_t bin, Also also) {
  const int tid = threadIdx.x;
  if (tid <= kValues) S.mine[tid] = 0;
  __syncthreads();
  // entries between the bin's smallest and largest value; the key decides (a
  // comparison takes -0, which ends a bin, for +0, which begins the next)
  const uint32_t lo = key_bits2(max(bin * kValues, kKeyMinusInf));
  const uint32_t hi = key_bits2(min(bin * kValues + kValues - 1, kKeyInf));
  uint32_t extra = 0;
  u64 hits = 0;  // as in gather_head
  int shift = 0;
  for (int i = tid; i < vecs; i += kThreads, shift += 8) {
    const uint4 v = data[i];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      extra += also(w[e]);
      m |= ge2(w[e], lo) & ge2(hi, w[e]) & (0x00020001u << (2 * e));
    }
    hits |= (u64)((m | m >> 16) & 0xffu) << shift;
  }
  for (; hits; hits &= hits - 1) {
    const int bit = __ffsll((long long)hits) - 1;
    const uint32_t b =
        reinterpret_cast<const uint16_t *>(data)[8 * (tid + (bit >> 3) * kThreads) + (bit & 7)];
    const uint32_t k = order2(b) & 0xffffu;
    if (k >> 4 == bin) atomicAdd(&S.mine[k & 15u], 1u);
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
    const int lane = threadIdx.x;
    const int v = kValues - 1 - (lane & 15);  // lane 0 holds the largest value
    uint32_t c[kMaxCluster], n = 0;
#pragma unroll
    for (uint32_t p = 0; p < kMaxCluster; ++p) c[p] = p < csize ? S.count[p][v] : 0u;
#pragma unroll
    for (uint32_t p = 0; p < kMaxCluster; ++p) n += c[p];
    const uint32_t k = S.win_bin * kValues + v;
    const uint32_t w = weight(k, n);
    const u64 mass = (u64)w * n;
    u64 inc = mass;
#pragma unroll
    for (int o = 1; o < kValues; o <<= 1) {
      const u64 below = __shfl_up_sync(0xffffffffu, inc, o, kValues);
      if ((lane & 15) >= o) inc += below;
    }
    const u64 end = S.win_before + inc;
    if (lane < kValues && t >= end - mass && t < end) {
      S.found_key = k;
      S.found_before = end - mass;
    }
  }
  __syncthreads();
  key = S.found_key;
  before = S.found_before;
}

// The mass top-p needs of a mass m, and the draw's position in a mass m: one
// thread's fp64, as both are CTA-wide values.
IPD_DEVINL u64 needed(float top_p, u64 m) {
  const double need = ceil((double)top_p * (double)m);
  return need < 1.0 ? 1ull : (need < (double)m ? (u64)need : m);
}
IPD_DEVINL u64 position(float u, u64 m) {
  if (!(u > 0.f)) return 0ull;
  const double d = floor((double)u * (double)m);
  return d < (double)m ? (u64)d : m - 1;
}
// a / w for a quotient below 2^20: an fp32 estimate, off by one at most
IPD_DEVINL uint32_t quotient(u64 a, uint32_t w) {
  uint32_t q = (uint32_t)((float)a / (float)w);
  if ((u64)q * w > a) --q;
  else if ((u64)(q + 1) * w <= a) ++q;
  return q;
}
// f evaluated by one thread for all
template <typename F>
__device__ u64 once(Shared &S, F f) {
  if (threadIdx.x == 0) S.word = f();
  __syncthreads();
  const u64 v = S.word;
  __syncthreads();
  return v;
}

// A head entry as one word that rises with (logit, then falling id): the key
// above the head's threshold over the id's complement.
IPD_DEVINL uint32_t pack_entry(uint32_t key, int id, int id_bits) {
  return key << id_bits | (~(uint32_t)id & ((1u << id_bits) - 1u));
}

constexpr int kHeadEach = kHead / kThreads;  // sorted entries a thread takes

IPD_DEVINL void order_pair(uint32_t &a, uint32_t &b, bool down) {
  const uint32_t hi = max(a, b), lo = min(a, b);
  a = down ? hi : lo;
  b = down ? lo : hi;
}

// Sorts the n entries that S.head holds in pieces (piece p, S.head_n[p] long,
// at p * kHead / csize) downwards into e: thread t holds entries 4t .. 4t + 3.  A
// bitonic network, unrolled (its steps depend on each other, so a loop's own
// latency would count 66 times) and left at the first power of two that holds
// n: strides 1 and 2 inside a thread, up to 64 between lanes by shuffles,
// longer ones through shared memory.
__device__ void sort_head(Shared &S, uint32_t csize, int n, uint32_t (&e)[kHeadEach]) {
  const int tid = threadIdx.x, at = kHeadEach * tid;
#pragma unroll
  for (int i = 0; i < kHeadEach; ++i) {
    int g = at + i;
    e[i] = 0u;  // past the end: sorts last
    if (g < n) {
      uint32_t p = 0;
      while ((uint32_t)g >= S.head_n[p]) g -= S.head_n[p++];
      e[i] = S.head[p * (kHead / csize) + g];
    }
  }
  const bool live = (at & ~127) < n;  // by whole warps
#pragma unroll
  for (int k = 2; k <= kHead; k <<= 1) {
    if (k / 2 >= n && k > 2) break;  // sorted: k / 2 is a power of two >= n
#pragma unroll
    for (int j = k >> 1; j >= 1; j >>= 1) {
      if (j >= 128) {  // partners in another warp; dead warps hold zeros
        __syncthreads();
        *reinterpret_cast<uint4 *>(&S.sorted[at]) = make_uint4(e[0], e[1], e[2], e[3]);
        __syncthreads();
        const uint4 o = *reinterpret_cast<const uint4 *>(&S.sorted[at ^ j]);
        const bool big = ((at & j) == 0) == ((at & k) == 0);
        e[0] = big ? max(e[0], o.x) : min(e[0], o.x);
        e[1] = big ? max(e[1], o.y) : min(e[1], o.y);
        e[2] = big ? max(e[2], o.z) : min(e[2], o.z);
        e[3] = big ? max(e[3], o.w) : min(e[3], o.w);
      } else if (j >= kHeadEach) {
        if (k > 128 || live) {
          const bool big = ((at & j) == 0) == ((at & k) == 0);
#pragma unroll
          for (int i = 0; i < kHeadEach; ++i) {
            const uint32_t o = __shfl_xor_sync(0xffffffffu, e[i], j / kHeadEach);
            e[i] = big ? max(e[i], o) : min(e[i], o);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < kHeadEach; ++i)
          if ((i & j) == 0) order_pair(e[i], e[i + j], ((at + i) & k) == 0);
      }
    }
  }
}

// The same for at most kThreads entries: an entry's place is the number of
// greater ones, counted against all of them (little code, and few entries).
__device__ void sort_small_head(Shared &S, uint32_t csize, int n, uint32_t (&e)[kHeadEach]) {
  const int tid = threadIdx.x;
  uint32_t x = 0u;
  if (tid < n) {
    int g = tid;
    uint32_t p = 0;
    while ((uint32_t)g >= S.head_n[p]) g -= S.head_n[p++];
    x = S.head[p * (kHead / csize) + g];
  }
  __syncthreads();
  S.sorted[tid] = x;  // zeros past the end: greater than nothing
  __syncthreads();
  int at = 0;
  if (tid < n) {
    int c[4] = {0, 0, 0, 0};
    for (int i = 0; i < n; i += 16) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint4 v = *reinterpret_cast<const uint4 *>(&S.sorted[i + 4 * k]);
        c[k] += (v.x > x) + (v.y > x) + (v.z > x) + (v.w > x);
      }
    }
    at = c[0] + c[1] + c[2] + c[3];
  }
  __syncthreads();
  if (tid < n) S.sorted[at] = x;
  __syncthreads();
  const uint4 v = *reinterpret_cast<const uint4 *>(&S.sorted[kHeadEach * tid]);
  e[0] = v.x, e[1] = v.y, e[2] = v.z, e[3] = v.w;  // (what lies past n is not read)
}

struct Masses {
  u64 all, head;   // sums of weights over the CTA's entries, and over those in the head
  uint32_t all_n;  // entries with a weight
};

// One pass over the CTA's entries: those at or above the threshold go to the
// first CTA's head; MASS: the weights are summed (COUNT: and counted).
template <bool MASS, bool COUNT, bool MINW>
__device__ Masses gather_head(Shared &S, const Scale &C, const uint4 *vecs, int n_vec, int id0,
                              uint32_t floor_key, int id_bits, uint32_t slots, uint32_t at0) {
  Masses M = {0ull, 0ull, 0u};
  const uint32_t floor2 = key_bits2(floor_key);
  // a thread's hits, 8 bits a vector: gathered after the pass, so that its
  // warps do not diverge at every vector
  u64 hits = 0;
  static_assert(kMaxPiece / 8 / kThreads <= 8, "a thread's vectors fit its hit mask");
  int k = 0;
  for (int i = threadIdx.x; i < n_vec; i += kThreads, k += 8) {
    const uint4 v = vecs[i];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (MASS) {
        uint32_t w0, w1;
        weight2<MINW>(C, w[e], w0, w1);
        M.all += w0 + w1;  // at most 2^31
        if (COUNT) M.all_n += min(w0, 1u) + min(w1, 1u);
      }
      m |= ge2(w[e], floor2) & (0x00020001u << (2 * e));
    }
    hits |= (u64)((m | m >> 16) & 0xffu) << k;
  }
  if (hits) {
    uint32_t at = atomicAdd(&S.list_n, (uint32_t)__popcll(hits));
    do {
      const int bit = __ffsll((long long)hits) - 1;
      hits &= hits - 1;
      const int entry = 8 * ((int)threadIdx.x + (bit >> 3) * kThreads) + (bit & 7);
      const uint32_t b = reinterpret_cast<const uint16_t *>(vecs)[entry];
      if (MASS) {
        uint32_t w0, w1;
        weight2<MINW>(C, b, w0, w1);
        M.head += w0;
      }
      if (at < slots)
        remote_st(at0 + 4 * at, pack_entry((order2(b) & 0xffffu) - floor_key, id0 + entry, id_bits));
      ++at;
    } while (hits);
  }
  return M;
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
  constexpr int kBatch = 8;  // 16-byte loads in flight a thread: a whole piece
  for (int vb = tid; vb < n_vec; vb += kBatch * kThreads) {
    uint4 w[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int i = i0 + 8 * (vb + k * kThreads);
      w[k] = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
      if (vb + k * kThreads < n_vec && i >= shift && i + 8 <= end) w[k] = ldg_stream(base + i);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int v = vb + k * kThreads, i = i0 + 8 * v;
      if (v >= n_vec) break;
      if (i < shift || i + 8 > end) {  // a vector the row covers in part, or not at all
        uint16_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = i + j >= shift && i + j < end ? base[i + j] : 0xff80u;
        w[k].x = e[0] | (uint32_t)e[1] << 16, w[k].y = e[2] | (uint32_t)e[3] << 16;
        w[k].z = e[4] | (uint32_t)e[5] << 16, w[k].w = e[6] | (uint32_t)e[7] << 16;
      }
      w[k] = make_uint4(clean2(w[k].x), clean2(w[k].y), clean2(w[k].z), clean2(w[k].w));
      reinterpret_cast<uint4 *>(data)[v] = w[k];
      mx = max2(max2(max2(mx, w[k].x), max2(w[k].y, w[k].z)), w[k].w);
    }
  }
  {
    const uint32_t k = order2(mx);
    uint32_t m = max(k & 0xffffu, k >> 16);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    if (!(lane & 1)) S.maxima[tid >> 1] = m;
  }
  if (tid == 0) S.list_n = 0;
  __syncthreads();
  // the head's threshold: the largest key that this CTA's share of the aim is
  // reached by among its thread pairs' maxima; the lowest of the cluster's.
  // Four bits a round, each of the 16 warps tries one value of them.
  const bool cut_k = top_k > 0 && top_k < P.vocab;
  uint32_t floor_key = 0;
  {
    const int aim = ((cut_k ? top_k : kHeadAim) + (int)csize - 1) / (int)csize;
    uint32_t m[kMaxima / 32], top = 0;
#pragma unroll
    for (int i = 0; i < kMaxima / 32; ++i) m[i] = S.maxima[32 * i + lane], top = max(top, m[i]);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint32_t c = floor_key | (uint32_t)warp << (12 - 4 * r);
      int n = 0;
#pragma unroll
      for (int i = 0; i < kMaxima / 32; ++i) n += m[i] >= c;
      n = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0) S.reached[r][warp] = n >= aim;
      __syncthreads();
      const uint32_t yes = __ballot_sync(0xffffffffu, lane < kWarps && S.reached[r][lane & 15]);
      if (yes) floor_key |= (uint32_t)(31 - __clz(yes)) << (12 - 4 * r);
    }
    cluster_wait();
    if (warp == 0) {
      top = __reduce_max_sync(0xffffffffu, top);
      if (lane < (int)csize) {
        remote_st(remote(&S.max_key[rank], lane), top);
        remote_st(remote(&S.floor_key[rank], lane), floor_key);
      }
    }
  }
  cluster_sync();
  floor_key = 0xffffu;
  uint32_t top_key = 0;
#pragma unroll
  for (uint32_t p = 0; p < kMaxCluster; ++p) {
    if (p < csize) {
      top_key = max(top_key, S.max_key[p]);
      floor_key = min(floor_key, S.floor_key[p]);
    }
  }
  // a row with nothing but -inf and NaN, or bad settings: no token
  if (!good || top_key <= kKeyMinusInf) {
    if (rank == 0 && tid == 0) {
      P.tokens[row] = -1;
      if (P.logp) P.logp[row] = -INFINITY;
      if (P.kept) P.kept[row] = 0;
    }
    return;  // the whole cluster
  }
  if (top_key == kKeyInf) {  // +inf: 0 in its place, and -inf for everything else
    for (int i = tid; i < P.piece / 2; i += kThreads) {
      const uint32_t is = ge2(data[i], 0x7f807f80u);
      data[i] = ~is & 0xff80ff80u;
    }
    __syncthreads();
    top_key = 0x8000u;
    floor_key = 0u;
  }
  // the head is all there is (a row of one CTA fits it)
  const bool whole = floor_key <= kKeyMinusInf + 1 || csize == 1;
  if (whole) floor_key = kKeyMinusInf + 1;
  C.top = key_value(top_key);
  {
    // entries below top - 33 / c have x < -32 and so weight 0; as a bf16 value,
    // rounded down (-inf where no finite one is as low)
    const float least = C.top - 33.f / C.c;
    const uint32_t b = __float_as_uint(least);
    const uint32_t up = (b >> 31) && (b & 0xffffu) ? 1u : 0u;  // away from 0 is down
    uint32_t h = (b >> 16) + up;
    if ((h & 0x7fffu) >= 0x7f80u) h = 0xff80u;
    // (top so large that 33 / c is lost in it: its bf16 neighbour is far below)
    if (exponent(C, bf16f((uint16_t)h)) > -32.f) h += (h & 0x8000u) ? 1u : 0xffffffffu;
    C.least2 = h | h << 16;
    C.coarse = !(exponent(C, bf16f((uint16_t)h)) > -100.f);
  }
  C.min_w = max(1u, (uint32_t)ceilf(min_p * 0x1p30f));  // exact: a power of two times min_p
  const uint4 *vecs = reinterpret_cast<const uint4 *>(data);
  const int words = P.piece / 2;
  const float uf = P.u[row];

  // ---- the head's entries, and without top-k the masses of head and row ----
  const uint32_t slots = kHead / csize;
  Masses M;
  {
    const uint32_t at0 = remote(&S.head[rank * slots], 0);
    const auto gather = [&](auto mass, auto count, auto minw) {
      return gather_head<decltype(mass)::value, decltype(count)::value, decltype(minw)::value>(
          S, C, vecs, n_vec, i0 - shift, floor_key, P.id_bits, slots, at0);
    };
    const std::true_type yes;
    const std::false_type no;
    if (cut_k) M = gather(no, no, no);
    else if (C.min_w > 1u) M = gather(yes, yes, yes);
    else if (P.kept && top_p >= 1.f) M = gather(yes, yes, no);
    else M = gather(yes, no, no);
  }
  if (!cut_k) {
    M.all = warp_sum64(M.all);
    M.head = warp_sum64(M.head);
    M.all_n = __reduce_add_sync(0xffffffffu, M.all_n);
    if (lane == 0) S.scan[warp] = M.all, S.scan2[warp] = M.head, S.warp_count[warp] = M.all_n;
  }
  __syncthreads();
  if (warp == 0) {
    if (!cut_k) {
      M.all = warp_sum64(lane < kWarps ? S.scan[lane] : 0ull);
      M.head = warp_sum64(lane < kWarps ? S.scan2[lane] : 0ull);
      M.all_n = __reduce_add_sync(0xffffffffu, lane < kWarps ? S.warp_count[lane] : 0u);
    }
    if (lane < (int)csize) {
      remote_st64(remote(&S.all_mass[rank], lane), M.all);
      remote_st64(remote(&S.head_mass[rank], lane), M.head);
      remote_st(remote(&S.all_n[rank], lane), M.all_n);
      remote_st(remote(&S.head_n[rank], lane), S.list_n);
    }
  }
  cluster_sync();
  uint32_t head_n = 0, all_n = 0;
  u64 all_mass = 0, head_mass = 0;
  // (a head over so wide a range of values that an entry does not pack is left)
  bool in_head = ((top_key - floor_key) >> (32 - P.id_bits)) == 0;
#pragma unroll
  for (uint32_t p = 0; p < kMaxCluster; ++p) {
    if (p < csize) {
      in_head = in_head && S.head_n[p] <= slots;
      head_n += S.head_n[p];
      all_mass += S.all_mass[p];
      head_mass += S.head_mass[p];
      all_n += S.all_n[p];
    }
  }
  u64 need = 0, t = 0;
  if (cut_k) {
    in_head = in_head && (whole || head_n >= (uint32_t)top_k);
  } else {
    // (all_mass >= 2^30: the largest entry's weight is never below min_w)
    need = once(S, [&] { return needed(top_p, all_mass); });
    if (need < all_mass) {
      in_head = in_head && need <= head_mass;
    } else {
      t = once(S, [&] { return position(uf, all_mass); });
      in_head = in_head && t < head_mass;
    }
  }
  if (in_head) {
    if (rank != 0) return;
    uint32_t e[kHeadEach], w[kHeadEach];
    if (head_n <= kThreads) sort_small_head(S, csize, (int)head_n, e);
    else sort_head(S, csize, (int)head_n, e);
    // entries e[0], e[1], ... in falling order over the CTA's threads; their
    // weights within top-k and min-p, and the running sum
    const int at = kHeadEach * tid;
    const int limit = cut_k ? min(top_k, (int)head_n) : (int)head_n;
    u64 cum[kHeadEach + 1], mine = 0;
#pragma unroll
    for (int i = 0; i < kHeadEach; i += 2) {
      w[i] = w[i + 1] = 0u;
      if (at + i < limit) {
        const uint32_t next = at + i + 1 < limit ? e[i + 1] : e[i];
        weight2<true>(C, (key_bits2((e[i] >> P.id_bits) + floor_key) & 0xffffu) |
                             (key_bits2((next >> P.id_bits) + floor_key) << 16),
                      w[i], w[i + 1]);
        if (at + i + 1 >= limit) w[i + 1] = 0u;
      }
      mine += (u64)w[i] + w[i + 1];
    }
    u64 head_sum;
    cum[0] = scan_cta(S, mine, head_sum);
#pragma unroll
    for (int i = 0; i < kHeadEach; ++i) cum[i + 1] = cum[i] + w[i];
    if (cut_k) need = once(S, [&] { return needed(top_p, head_sum); });
    u64 kept_mass = cut_k ? head_sum : all_mass;
    const bool cut_p = need < kept_mass;
    if (cut_p) {  // the entry that completes the mass top-p needs is the last
#pragma unroll
      for (int i = 0; i < kHeadEach; ++i) {
        if (cum[i] < need && need <= cum[i + 1]) S.found_before = cum[i + 1];
        if (cum[i] >= need) w[i] = 0u;
      }
      __syncthreads();
      kept_mass = S.found_before;
    }
    if (cut_k || cut_p) t = once(S, [&] { return position(uf, kept_mass); });
    if (P.kept) {
      uint32_t kept = all_n;
      if (cut_k || cut_p) {
        uint32_t n = 0;
#pragma unroll
        for (int i = 0; i < kHeadEach; ++i) n += w[i] != 0u;
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) S.warp_count[warp] = n;
        __syncthreads();
        kept = __reduce_add_sync(0xffffffffu, lane < kWarps ? S.warp_count[lane] : 0u);
      }
      if (tid == 0) P.kept[row] = (int32_t)kept;
    }
#pragma unroll
    for (int i = 0; i < kHeadEach; ++i) {
      if (t >= cum[i] && t < cum[i] + w[i]) {
        const uint32_t key = (e[i] >> P.id_bits) + floor_key;
        P.tokens[row] = (int32_t)(~e[i] & ((1u << P.id_bits) - 1u));
        if (P.logp) {
          P.logp[row] = (exponent(C, key_value(key)) - log2f((float)kept_mass * 0x1p-30f)) * kLn2;
        }
      }
    }
    return;
  }
  // ---- not in the head: the histogram (over the head's memory) ----
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads) S.lo[i] = 0, S.hi[i] = 0;
  __syncthreads();

  // ---- top-k: its last value, and how many entries of that value are in ----
  uint32_t key_k = 0, in_k = 0;  // entries with a greater key, and in_k of key_k
  if (cut_k) {
    for (int i = tid; i < words; i += kThreads) {
      const uint32_t w = data[i], in = ge2(w, C.least2), k = order2(w);
      if (in & 0xffffu) atomicAdd(&S.lo[(k >> 4) & 0xfffu], 1u);
      if (in >> 16) atomicAdd(&S.lo[k >> 20], 1u);
    }
    if (share_groups(S, rank, csize) > (u64)top_k) {
      find_bin(S, csize, (u64)top_k - 1);
      // the bin's values counted under the same bound as the histogram
      count_values(S, vecs, n_vec, rank, csize, S.win_bin, [](uint32_t) { return 0u; });
      u64 before;
      find_value(S, csize, (u64)top_k - 1, [](uint32_t, uint32_t) { return 1u; }, key_k, before);
      in_k = (uint32_t)((u64)top_k - before);
    }
    cluster_sync();  // no CTA reads these counts any more
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
  for (int i = tid; i < n_vec; i += kThreads) {
    const uint4 v = vecs[i];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m[8], k[4];  // all weights first: the atomics then wait for none of them
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      weight2<true>(C, w[e], m[2 * e], m[2 * e + 1]);
      k[e] = order2(w[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t key = e & 1 ? k[e / 2] >> 16 : k[e / 2] & 0xffffu;
      if (m[e] && key > key_k) {
        atomicAdd(&S.lo[key >> 4], m[e] & 0xffffu);
        if (m[e] >> 16) atomicAdd(&S.hi[key >> 4], m[e] >> 16);
      }
    }
  }
  if (share && tid == 0) {
    const uint32_t w = weight_of_key(C, key_k);
    atomicAdd(&S.lo[key_k >> 4], share * (w & 0xffffu));
    atomicAdd(&S.hi[key_k >> 4], share * (w >> 16));
  }
  const u64 total = share_groups(S, rank, csize);
  // an entry's weight in the sums, with the number of entries of its value that
  // are in the top k
  const auto weight = [&](uint32_t key, uint32_t &n) -> uint32_t {
    if (key < key_k) n = 0;
    else if (key == key_k) n = min(n, in_k);
    return n ? weight_of_key(C, key) : 0u;
  };
  // total >= 1: the largest logit has weight 2^30 >= min_w and rank 0

  // ---- top-p: its last value, and the mass that is kept ----
  uint32_t key_p = 0, in_p = 0;  // entries with a greater key, and in_p of key_p
  u64 kept_mass = total;
  {
    double need = ceil((double)top_p * (double)total);
    need = need < 1.0 ? 1.0 : need;
    if (need < (double)total) {
      const u64 last = (u64)need - 1;  // position of the last unit of mass that is needed
      find_bin(S, csize, last);
      count_values(S, vecs, n_vec, rank, csize, S.win_bin, [](uint32_t) { return 0u; });
      u64 before;
      find_value(S, csize, last, [&](uint32_t k, uint32_t &n) { return weight(k, n); }, key_p,
                 before);
      const uint32_t w = weight_of_key(C, key_p);
      in_p = quotient(last - before, w) + 1;
      kept_mass = before + (u64)in_p * w;
    }
  }

  // ---- the draw ----
  t = once(S, [&] { return position(uf, kept_mass); });
  find_bin(S, csize, t);
  // with the values of the bin, the entries that are kept besides in_p (or, when
  // all of the top k is, in_k): greater keys with a weight.  The exponent x
  // decides wherever it is more than 0.01 from the smallest weight that counts
  // (w >= min_w at 2^30 2^x >= min_w - 1/2); between, the weight itself.
  const uint32_t edge = key_p ? key_p : key_k;
  const float x_in = log2f((float)C.min_w) - 29.99f, x_out = log2f((float)C.min_w - 0.5f) - 30.01f;
  const uint32_t edge2 = key_bits2(max(edge, kKeyMinusInf));
  count_values(S, vecs, n_vec, rank, csize, S.win_bin, [&](uint32_t w) {
    const uint32_t above = ~ge2(edge2, w);
    const bool a = above & 0xffffu, b = above >> 16;
    if (!a && !b) return 0u;
    const float x0 = exponent(C, bf16lo(w)), x1 = exponent(C, bf16hi(w));
    uint32_t w0 = x0 >= x_in, w1 = x1 >= x_in;
    if ((!w0 && x0 >= x_out) || (!w1 && x1 >= x_out)) weight2<true>(C, w, w0, w1);
    return (uint32_t)(a && w0) + (uint32_t)(b && w1);
  });
  uint32_t key_d;
  u64 before;
  find_value(S, csize, t, [&](uint32_t k, uint32_t &n) { return weight(k, n); }, key_d, before);
  const uint32_t weight_d = weight_of_key(C, key_d);
  uint32_t j = quotient(t - before, weight_d);  // rank among the value's entries
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
      if (P.logp)
        P.logp[row] = (exponent(C, key_value(key_d)) - log2f((float)kept_mass * 0x1p-30f)) * kLn2;
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
  // CTAs of a row: one where the head holds all of it, else as many as its
  // entries need, and more while SMs are idle and a piece is more than a few
  // loads a thread
  int csize = vocab <= kHead ? 1 : 2;
  const long long span = (long long)vocab + 7;  // a row may start inside a 16-byte piece
  while (vocab > kHead && csize < kMaxCluster &&
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
  P.id_bits = 1;
  while ((1 << P.id_bits) < vocab) ++P.id_bits;
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

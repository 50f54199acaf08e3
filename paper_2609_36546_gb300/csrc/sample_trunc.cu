// One token per row from the softmax at a temperature, cut by top-k, min-p and
// top-p, from a given uniform number, in one launch.
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
// bf16 logits have few values, and entries of one value have one weight.  So a
// row is read once into a histogram of its values, one integer atomic in shared
// memory for an entry, and all the rest happens on the bins: weights, the three
// cuts and the draw, which are the same question, "which bin holds position t
// of the running sum of counts (or weights) from the largest logit down".  What
// is left of t in the bin, divided by the bin's weight, is the entry's rank
// among its equals, which is looked up in index order in a second look at a
// part of the row (in L2).  No sorting, no order of summation, and no entry's
// weight is computed on its own.
//
// Bins: 2^-19 <= |l| < 2^12 is 31 binades of 128 values a sign, one bin each.
// What is nearer to 0 is rare (zeros apart, which are counted) and goes to a
// list, which takes the bins between the signs in the order of its values.
// -inf, NaN and what is below -2^12 have no weight next to such a maximum.  A
// row that does not fit this (a maximum outside, +inf, a full list, so high a
// temperature that -2^12 matters) is worked through by its first CTA in windows
// of 2^13 bins over all 2^16 values, a pass over the row for each.
//
// What bounds it (GB300, device time).  Many rows: the pass over the entries.  512
// rows of 151,936 take 70.5 us (2.2 TB/s).  All are in flight at once: the pass takes
// about 32 us of a row's life (half of that without its atomics: random words put
// three to four of a warp's 32 on one bank), the searches 8, the look-up up to 20 for
// an entry far down the row; the last rows' searches and look-ups have nothing left
// to hide behind.  Entries near 0 and below the range are kept out of the
// common path: it has no branch for an entry, and one for a thread's batch of 32 (is
// one of them near 0).  Few rows: a chain of barriers.  One
// row of 151,936 takes 14.1 us: reading it 2.2, the cluster's barriers and the sum
// of its histograms 3, the bins' weights and sums 2.1, the searches 3, the look-up 2;
// 64 rows take 21.2 us, 33 rows of 50,021 12.9 (13.8, 20.8, 12.5 and 70.1 for the 512 with
// contracted weights, which are not the defined ones).  A sorted head of the row with the
// searches as the exception took 20.5 us for one row and 174 for 512.  Rows outside
// the bins' range: 70 to 80 us with a maximum there, 210 with all of it near 0.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "cluster.cuh"
#include "common.cuh"
#include "weights.cuh"

IPD_DECLARE_ERROR_WORD(g_trunc_err);
// whether this process has launched (or captured) a kernel that may set the word:
// a program without these calls does not pay for reading it
static std::atomic<bool> g_trunc_used{false};

namespace {

constexpr int kMaxCluster = 8;          // portable cluster size
constexpr int kSplitRow = 48 * 1024, kMinPiece = 12 * 1024;  // entries: see ipd_sample_trunc
constexpr int kBins = 8192;
constexpr int kBatch = 4;               // 16-byte vectors in flight a thread
constexpr uint32_t kLowBits = 0x3600;   // bf16 bits of 2^-19
constexpr int kSide = 31 * 128;         // bins of a sign; up to the bits of 2^12
constexpr int kMid = kBins - 2 * kSide;  // bins between the signs
constexpr int kRound = 8;               // see look_up

struct Params {
  const uint16_t *logits;
  long long stride;
  const float *u;
  const float *inv_t, *top_p, *min_p;
  const int32_t *top_k;
  int32_t *tokens, *kept;
  float *logp;
  int vocab, piece;  // piece: entries a CTA counts (a multiple of 8)
  float one;         // 1: see pow2_weight2
};

struct Scale {
  float top, c;     // l_max and fl(log2 e * inv_temperature)
  bool inf;         // l_max is +inf: only its equals have a weight, x = 0
  bool coarse;      // the x of least2 is far below -64: bf16 is coarse at l_max
  uint32_t least2;  // a bf16 value (twice) of weight 0 from which on weights are 0
  uint32_t min_w;   // smallest weight that counts (min-p; at least 1)
  float one;        // 1: see pow2_weight2
};

// ---- order keys --------------------------------------------------------------
// A 16-bit key rises with the bf16 value; NaN counts as -inf, -0 as 0.
constexpr uint32_t kKeyMinusInf = 0x007fu, kKeyZero = 0x8000u, kKeyInf = 0xff80u;
IPD_DEVINL uint32_t order_key(uint32_t b) {
  const uint32_t a = b & 0x7fffu;
  if (a > 0x7f80u) return kKeyMinusInf;
  if (a == 0u) return kKeyZero;
  return (b & 0x8000u) ? ~b & 0xffffu : b | 0x8000u;
}
IPD_DEVINL uint32_t key_bits(uint32_t key) {
  return (key & 0x8000u) ? key ^ 0x8000u : ~key & 0xffffu;
}
IPD_DEVINL float key_value(uint32_t key) { return bf16f((uint16_t)key_bits(key)); }
IPD_DEVINL uint32_t max2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<__nv_bfloat162 *>(&a),
                                   *reinterpret_cast<__nv_bfloat162 *>(&b));
  return *reinterpret_cast<const uint32_t *>(&m);
}

// ---- weights -------------------------------------------------------------------
// w of two entries (pow2_weight2 of their x).
IPD_DEVINL void weight2(const Scale &S, uint32_t w, uint32_t &w0, uint32_t &w1) {
  w = max2(w, S.least2);
  u64 x = f2_mul(f2_sub(f2_pack(bf16lo(w), bf16hi(w)), f2_pack(S.top, S.top)), f2_pack(S.c, S.c));
  if (S.coarse) {
    float a, b;
    f2_unpack(x, a, b);
    x = f2_pack(fmaxf(a, -64.f), fmaxf(b, -64.f));
  }
  pow2_weight2(x, w0, w1, f2_pack(S.one, S.one));
  if (w0 < S.min_w) w0 = 0u;
  if (w1 < S.min_w) w1 = 0u;
}
// x of an entry, as weight2 has it before any bound
IPD_DEVINL float exponent(const Scale &S, float l) {
  return S.inf ? 0.f : __fmul_rn(__fsub_rn(l, S.top), S.c);
}
IPD_DEVINL void weights(const Scale &S, uint32_t w, uint32_t &w0, uint32_t &w1) {
  if (S.inf) {
    w0 = (w & 0xffffu) == 0x7f80u ? 1u << 30 : 0u;
    w1 = w >> 16 == 0x7f80u ? 1u << 30 : 0u;
  } else {
    weight2(S, w, w0, w1);
  }
}
IPD_DEVINL uint32_t weight_floor(float min_p) {
  return max(1u, (uint32_t)ceilf(min_p * 0x1p30f));  // exact: a power of two times min_p
}
IPD_DEVINL Scale make_scale(float c, float min_p, uint32_t top_key, float one) {
  Scale C;
  C.one = one;
  C.c = c;
  C.inf = top_key == kKeyInf;
  C.top = key_value(top_key);
  C.min_w = weight_floor(min_p);
  // entries from 33 - log2(min_w) binades of weight below the top on have none (x
  // < log2(min_w) - 32); as a bf16 value, rounded down (-inf where no finite one
  // is as low)
  const float bits = log2f((float)C.min_w);
  const float least = C.top - (33.f - bits) / C.c;
  const uint32_t b = __float_as_uint(least);
  const uint32_t up = (b >> 31) && (b & 0xffffu) ? 1u : 0u;  // away from 0 is down
  uint32_t h = (b >> 16) + up;
  if ((h & 0x7fffu) >= 0x7f80u) h = 0xff80u;
  // (top so large that the distance is lost in it: its bf16 neighbour is far below)
  if (exponent(C, bf16f((uint16_t)h)) > bits - 32.f) h += (h & 0x8000u) ? 1u : 0xffffffffu;
  C.least2 = h | h << 16;
  C.coarse = !(exponent(C, bf16f((uint16_t)h)) > -100.f);
  return C;
}

// The mass top-p needs of a mass m, and the draw's position in a mass m.
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
// ---- the row -----------------------------------------------------------------
// A row may start anywhere: it is read as 16-byte vectors from the boundary
// before it, entry i of the row at i + shift of those.
struct Row {
  const uint16_t *base;
  int shift, end;  // entries shift .. end - 1 of base are the row's
  IPD_DEVINL bool has(int i) const { return i >= shift && i < end; }
  IPD_DEVINL bool cut(int v) const { return 8 * v < shift || 8 * v + 8 > end; }
  // vector v if it is the row's as a whole and below last, else -inf
  IPD_DEVINL uint4 load(int v, int last) const {
    if (v < last && !cut(v))
      return __ldg(reinterpret_cast<const uint4 *>(base + 8ll * v));
    return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
  }
  // for thread i < 16: an entry of the first or last vector, if the row has only a
  // part of that vector, it has the entry, and the vector is in first .. last - 1;
  // else -1
  IPD_DEVINL int edge_entry(int i, int first, int last) const {
    const int v = i < 8 ? 0 : end / 8, e = 8 * v + (i & 7);
    if (i >= 16 || v < first || v >= last || !has(e)) return -1;
    if (!cut(v)) return -1;
    if (i >= 8 && v == 0) return -1;  // the same vector
    return e;
  }
};

// ---- bins --------------------------------------------------------------------
constexpr int kFreeWord = (kLowBits + kSide) & (kBins / 2 - 1);  // of each half, to the next value's
static_assert(kBins / 2 - kSide == kMid / 2 && (kLowBits & (kBins / 2 - 1)) == kFreeWord + kMid / 2, "");
// The bins in the order of falling values, p = 0 .. kBins - 1, of a row's one
// histogram (window < 0) or of a window of keys.
IPD_DEVINL int word_at(int window, int p) {
  if (window >= 0) return kBins - 1 - p;
  // a value's word: its sign, and the low 12 of its other bits (3,968 values in a
  // row differ in those); the bins between the signs take the 128 words that
  // this leaves of each half
  if (p < kSide) return (int)(kLowBits + kSide - 1 - p) & (kBins / 2 - 1);
  if (p >= kSide + kMid) return kBins / 2 + ((int)(kLowBits + p - kSide - kMid) & (kBins / 2 - 1));
  return (kFreeWord + ((p - kSide) & (kMid / 2 - 1))) + (p - kSide < kMid / 2 ? 0 : kBins / 2);
}
// What a row takes by blocks of kThreads.
template <int kThreads>
struct Sampler {
static constexpr int kWarps = kThreads / 32;
static constexpr int kEach = kBins / kThreads;  // bins a thread sums
static_assert(kEach >= 16 && kEach <= 32, "a thread's bins are searched by one warp");

struct Shared {
  uint32_t hist[kBins];
  u64 before[kThreads + 1];       // sums of the bins before a thread's, and of all
  uint32_t n_before[kThreads + 1];
  uint16_t near_key[kMid];  // keys of this CTA's entries near 0
  uint16_t mid_key[kMid];   // first CTA: keys of the bins between the signs
  uint32_t near_n, zeros, largest;  // entries near 0, zeros, and the piece's largest key
  uint32_t all_near[kMaxCluster], all_zeros[kMaxCluster], all_largest[kMaxCluster];
  Scale scale;
  int window;                     // the bins' keys: see key_at
  u64 scan[kWarps];
  uint32_t scan_n[kWarps];
  u64 found_before, word;
  uint32_t found_key, found_weight, found_n, found_count;
  uint16_t block[2][kWarps * kRound];  // entries of the drawn value in each block of a round
};

// f evaluated by one thread for all (fp64 is slow)
template <typename F>
static IPD_DEVINL u64 once(Shared &S, F f) {
  __syncthreads();
  if (threadIdx.x == 0) S.word = f();
  __syncthreads();
  return S.word;
}

static IPD_DEVINL uint32_t key_at(const Shared &S, int window, int p) {
  if (window >= 0) return (uint32_t)window * kBins + kBins - 1 - p;
  if (p < kSide) return 0x8000u + kLowBits + kSide - 1 - p;
  if (p >= kSide + kMid) return 0x7fffu - kLowBits - (p - kSide - kMid);
  return S.mid_key[p - kSide];
}
static_assert(kSide % kEach == 0 && kMid % (2 * kEach) == 0, "a thread's bins are contiguous words");
static constexpr uint32_t kKeyHigh = 0x8000u + kLowBits + kSide;        // 2^12
static constexpr uint32_t kKeyLow = 0x7fffu - kLowBits - kSide;         // -2^12

static IPD_DEVINL void shared_add(uint32_t addr, uint32_t v) {
  asm volatile("red.shared.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
// the byte offsets of two entries' words
static IPD_DEVINL uint32_t words2(uint32_t w) {
  return ((w << 2) & 0x3ffc3ffcu) | ((w >> 1) & 0x40004000u);
}
static IPD_DEVINL uint32_t eq2(uint32_t a, uint32_t b) {  // 0xffff in each half where they are equal
  return __heq2_mask(*reinterpret_cast<__nv_bfloat162 *>(&a), *reinterpret_cast<__nv_bfloat162 *>(&b));
}
// 0xffff in each half where the entry is near 0, without a bin of its own
static IPD_DEVINL uint32_t near2(uint32_t w) {
  const __nv_bfloat162 a = __habs2(*reinterpret_cast<__nv_bfloat162 *>(&w));
  const uint32_t low = kLowBits * 0x00010001u;
  return __hlt2_mask(a, *reinterpret_cast<const __nv_bfloat162 *>(&low));
}
static IPD_DEVINL uint32_t min_abs2(uint32_t a, uint32_t w) {
  const __nv_bfloat162 m = __hmin2(*reinterpret_cast<__nv_bfloat162 *>(&a),
                                   __habs2(*reinterpret_cast<__nv_bfloat162 *>(&w)));
  return *reinterpret_cast<const uint32_t *>(&m);
}
static constexpr uint32_t kLowest2 = (0x8000u | (kLowBits + kSide)) * 0x00010001u;  // -2^12, twice
// Two entries into the histogram.  What is not above -2^12, and NaN, counts as
// -2^12, whose word is no value's here and is emptied later; what is from 2^12 up
// shows in the maximum; what is near 0 is taken out again.
static IPD_DEVINL void count2(uint32_t hist, uint32_t w) {
  const uint32_t z = words2(max2(w, kLowest2));
  shared_add(hist + (z & 0xffffu), 1u);
  shared_add(hist + (z >> 16), 1u);
}
// An entry that was counted, if it is near 0 but not 0, into the list instead.
static __device__ __noinline__ void list_near(Shared &S, uint32_t b) {
  const uint32_t a = b & 0x7fffu;
  if (a >= kLowBits || a == 0u) return;
  shared_add(smem_u32(S.hist) + (words2(b) & 0xffffu), 0xffffffffu);
  const uint32_t n = atomicAdd(&S.near_n, 1u);
  if (n < (uint32_t)kMid) S.near_key[n] = (uint16_t)order_key(b);
}

// Sums over the bins before each thread's, and over all, of the masses into
// S.before and of the entries with a weight into S.n_before.
static __device__ __noinline__ void sum_bins(Shared &S) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, window = S.window;
  u64 mass = 0;
  uint32_t n = 0;
  const Scale C = S.scale;
  // the thread's words, from the lowest on, and the bf16 bits of their values, which
  // follow one another, but between the signs
  const int p0 = kEach * tid;
  const bool mids = window < 0 && p0 >= kSide && p0 < kSide + kMid;
  const int wa = word_at(window, p0), wb = word_at(window, p0 + kEach - 1), word0 = min(wa, wb);
  const uint32_t bits0 = key_bits(key_at(S, window, wa < wb ? p0 : p0 + kEach - 1));
  const uint32_t step = window >= 0 && (bits0 & 0x8000u) ? 0xffffffffu : 1u;
#pragma unroll 1
  for (int q = 0; q < kEach / 4; ++q) {
    // four bins, in an order that spreads a warp's over the banks
    const int o = 4 * ((q + lane / (32 / kEach)) & (kEach / 4 - 1));
    const uint4 c = *reinterpret_cast<const uint4 *>(&S.hist[word0 + o]);
    if (!(c.x | c.y | c.z | c.w)) continue;
    uint32_t v01 = (bits0 + step * o) * 0x00010001u + (step << 16), v23 = v01 + step * 0x00020002u;
    if (mids) {
      const uint16_t *k = &S.mid_key[p0 - kSide + o];
      v01 = key_bits(k[0]) | key_bits(k[1]) << 16;
      v23 = key_bits(k[2]) | key_bits(k[3]) << 16;
    }
    uint32_t w0, w1, w2, w3;
    weights(C, v01, w0, w1);
    weights(C, v23, w2, w3);
    mass += (u64)w0 * c.x + (u64)w1 * c.y + (u64)w2 * c.z + (u64)w3 * c.w;
    n += (w0 ? c.x : 0u) + (w1 ? c.y : 0u) + (w2 ? c.z : 0u) + (w3 ? c.w : 0u);
  }
  u64 im = mass;
  uint32_t in = n;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const u64 x = __shfl_up_sync(0xffffffffu, im, o);
    const uint32_t y = __shfl_up_sync(0xffffffffu, in, o);
    if (lane >= o) im += x, in += y;
  }
  if (lane == 31) S.scan[warp] = im, S.scan_n[warp] = in;
  __syncthreads();
  // the warps before this one: their sums, below 2^48, in two halves of 24 bits
  const bool is = lane < warp;
  const u64 x = is ? S.scan[lane] : 0ull;
  const u64 bm = im - mass + __reduce_add_sync(0xffffffffu, (uint32_t)x & 0xffffffu) +
                 ((u64)__reduce_add_sync(0xffffffffu, (uint32_t)(x >> 24)) << 24);
  const uint32_t bn = in - n + __reduce_add_sync(0xffffffffu, is ? S.scan_n[lane] : 0u);
  S.before[tid] = bm, S.n_before[tid] = bn;
  if (tid == kThreads - 1) S.before[kThreads] = bm + mass, S.n_before[kThreads] = bn + n;
  __syncthreads();
}

// The bin that holds position t, which lies in the sums, of the running sum of
// the entries (`ranks`) or of their masses: into S.found_* its key, its entries
// and their weight, and the sum and the number of entries above it.
static __device__ __noinline__ void find_bin(Shared &S, bool ranks, u64 t) {
  const int tid = threadIdx.x, lane = tid & 31, window = S.window;
  const u64 lo = ranks ? S.n_before[tid] : S.before[tid];
  const u64 hi = ranks ? S.n_before[tid + 1] : S.before[tid + 1];
  const uint32_t here = __ballot_sync(0xffffffffu, t >= lo && t < hi);
  if (here) {  // one warp, for one of its threads
    const int win = tid - lane + __ffs(here) - 1, p = kEach * win + (lane & (kEach - 1));
    const uint32_t key = key_at(S, window, p), count = S.hist[word_at(window, p)];
    uint32_t w, w1;
    weights(S.scale, key_bits(key), w, w1);
    const uint32_t n = w ? count : 0u;
    const u64 mass = (u64)n * w;
    u64 im = mass;
    uint32_t in = n;
#pragma unroll
    for (int o = 1; o < kEach; o <<= 1) {
      const u64 x = __shfl_up_sync(0xffffffffu, im, o, kEach);
      const uint32_t y = __shfl_up_sync(0xffffffffu, in, o, kEach);
      if ((lane & (kEach - 1)) >= o) im += x, in += y;
    }
    const u64 above = S.before[win] + im - mass, first = ranks ? S.n_before[win] + in - n : above;
    if (lane < kEach && t >= first && t - first < (ranks ? n : mass)) {
      S.found_key = key;
      S.found_weight = w;
      S.found_before = above;
      S.found_n = S.n_before[win] + in - n;
      S.found_count = count;
    }
  }
  __syncthreads();
}

// A vector that the row has a part of.
static __device__ __noinline__ uint4 edge_vector(const uint16_t *base, int v, int shift, int end) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int a = 8 * v + 2 * i;
    w[i] = (a >= shift && a < end ? base[a] : 0xff80u) |
           (a + 1 >= shift && a + 1 < end ? base[a + 1] : 0xff80u) << 16;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A window's histogram, from the whole row.
static __device__ __noinline__ void count_window(Shared &S, const Row R, int n_vec, int window) {
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads) S.hist[i] = 0u;
  if (threadIdx.x == 0) S.window = window;
  __syncthreads();
#pragma unroll 2
  for (int v = threadIdx.x; v < n_vec; v += kThreads) {
    uint4 x = R.load(v, n_vec);
    if (R.cut(v)) x = edge_vector(R.base, v, R.shift, R.end);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t k = order_key(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu);
      if ((int)(k / kBins) == window && k > kKeyMinusInf)
        shared_add(smem_u32(&S.hist[k % kBins]), 1u);
    }
  }
  __syncthreads();
}

// The row's id of entry `rank` (in index order, from vector `first` on) of
// those with this key: in rounds of kRound blocks a warp, 32 vectors a block,
// counted and then looked up in the block, by the thread that finds it.
static IPD_DEVINL void look_up(Shared &S, const Row &R, int first, int last, uint32_t key, uint32_t rank,
                        int32_t *token) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t want = key_bits(key) * 0x00010001u;
  const auto match = [&](const uint4 &v) {  // a bit for each of the vector's entries (-0 is 0)
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m |= eq2(w[i], want) & (0x00020001u << (2 * i));
    return (m | m >> 16) & 0xffu;
  };
  const auto cut = [&](int v) { return v < last && R.cut(v); };
  constexpr int kMine = kWarps * kRound / 32;  // blocks a lane sums
  static_assert(kWarps * kRound % 32 == 0, "whole lanes of blocks");
  int round = 0;
#pragma unroll 1
  for (int v1 = first; v1 < last; v1 += kWarps * kRound * 32, round ^= 1) {
    uint4 part[kRound];  // all in flight at once
    const int v0 = v1 + warp * kRound * 32 + lane;
#pragma unroll
    for (int b = 0; b < kRound; ++b) part[b] = R.load(v0 + 32 * b, last);
#pragma unroll
    for (int b = 0; b < kRound; ++b) {
      if (cut(v0 + 32 * b)) part[b] = edge_vector(R.base, v0 + 32 * b, R.shift, R.end);
      __syncwarp();
      const uint32_t n = __reduce_add_sync(0xffffffffu, __popc(match(part[b])));
      if (lane == 0) S.block[round][warp * kRound + b] = (uint16_t)n;
    }
    __syncthreads();
    // every warp finds the block for itself
    uint32_t mine[kMine], n = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) n += mine[i] = S.block[round][kMine * lane + i];
    uint32_t in = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, in, o);
      if (lane >= o) in += y;
    }
    const uint32_t all = __shfl_sync(0xffffffffu, in, 31);
    if (rank >= all) {
      rank -= all;
      continue;
    }
    if (warp != 0) return;
    uint32_t before = in - n, at = 0, left = 0;
    bool here = false;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      if (rank >= before && rank - before < mine[i]) here = true, at = kMine * lane + i, left = rank - before;
      before += mine[i];
    }
    const int from = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
    at = __shfl_sync(0xffffffffu, at, from);
    left = __shfl_sync(0xffffffffu, left, from);
    const int v = v1 + (int)at * 32 + lane;
    uint4 x = R.load(v, last);
    if (cut(v)) x = edge_vector(R.base, v, R.shift, R.end);
    __syncwarp();
    uint32_t hits = match(x);
    n = __popc(hits);
    in = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(0xffffffffu, in, o);
      if (lane >= o) in += y;
    }
    if (left >= in - n && left < in) {
      for (left -= in - n; left; --left) hits &= hits - 1;
      *token = 8 * v + __ffs(hits) - 1 - R.shift;
    }
    return;
  }
}

static IPD_DEVINL void run(const Params &P) {
  extern __shared__ __align__(16) uint8_t smem_raw[];
  Shared &S = *reinterpret_cast<Shared *>(smem_raw);
  const uint32_t rank = cluster_rank(), csize = cluster_size();
  const int row = blockIdx.x / csize;
  const int tid = threadIdx.x, lane = tid & 31;
  const float inv_t = P.inv_t ? P.inv_t[row] : 1.f;
  const float top_p = P.top_p ? P.top_p[row] : 1.f;
  const float min_p = P.min_p ? P.min_p[row] : 0.f;
  const int top_k = P.top_k ? P.top_k[row] : 0;
  const bool cut_k = top_k > 0 && top_k < P.vocab;
  const float uf = P.u[row];
  const float c = __fmul_rn(kLog2e, inv_t);
  const bool good = c > 0.f && c - c == 0.f && top_p == top_p && min_p >= 0.f && min_p <= 1.f;
  const uint16_t *src = P.logits + (long long)row * P.stride;
  Row R;
  R.shift = (int)(((uintptr_t)src & 15) >> 1);
  R.base = src - R.shift;
  R.end = P.vocab + R.shift;
  const int n_vec = (R.end + 7) / 8, piece = P.piece / 8;

  // ---- the piece's histogram ----
#pragma unroll
  for (int i = 0; i < kBins / 4 / kThreads; ++i)
    reinterpret_cast<uint4 *>(S.hist)[tid + i * kThreads] = make_uint4(0, 0, 0, 0);
  if (tid == 0) {
    S.near_n = S.zeros = S.largest = 0;
    S.window = -1;
  }
  __syncthreads();
  {
    uint32_t zeros[2] = {0u, 0u}, largest = 0xff80ff80u;  // (by sign)
    const uint32_t hist = smem_u32(S.hist);
    const int v0 = (int)rank * piece, v1 = min(v0 + piece, n_vec);
    const int e = R.edge_entry(tid, v0, v1);
    if (e >= 0) {
      const uint32_t b = R.base[e];
      largest = max2(largest, b | 0xff800000u);
      count2(hist, b | 0xff800000u);
      if (b & 0x7fffu) list_near(S, b);
      else ++zeros[b >> 15];
    }
#pragma unroll 1
    for (int vb = v0 + tid; vb < v1; vb += kBatch * kThreads) {
      uint4 x[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) x[k] = R.load(vb + k * kThreads, v1);
      uint32_t nearest = 0x7f807f80u;  // to 0
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          largest = max2(largest, w[i]);
          nearest = min_abs2(nearest, w[i]);
          count2(hist, w[i]);
        }
      }
      if (!near2(nearest)) continue;
      uint32_t tiny = 0;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t is0 = eq2(w[i], 0u);
          zeros[0] += __popc(is0 & ~w[i] & 0x80008000u);
          zeros[1] += __popc(is0 & w[i] & 0x80008000u);
          tiny |= near2(w[i]) & ~is0 & (0x00010001u << k);
        }
      }
      for (tiny = (tiny | tiny >> 16) & 0xffffu; tiny; tiny &= tiny - 1) {
        const uint4 v = R.load(vb + (__ffs(tiny) - 1) * kThreads, v1);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (near2(w[i])) list_near(S, w[i] & 0xffffu), list_near(S, w[i] >> 16);
        }
      }
    }
    zeros[0] = __reduce_add_sync(0xffffffffu, zeros[0]);
    zeros[1] = __reduce_add_sync(0xffffffffu, zeros[1]);
    const uint32_t m = __reduce_max_sync(
        0xffffffffu, max(order_key(largest & 0xffffu), order_key(largest >> 16)));
    if (lane == 0) {
      if (zeros[0] | zeros[1]) {  // out of the words they were counted in
        shared_add(hist + (words2(0x0000u) & 0xffffu), 0u - zeros[0]);
        shared_add(hist + (words2(0x8000u) & 0xffffu), 0u - zeros[1]);
        atomicAdd(&S.zeros, zeros[0] + zeros[1]);
      }
      atomicMax(&S.largest, m);
    }
  }
  if (csize > 1) {
    // each CTA sums its share of the bins over all, in place in the first one's
    cluster_sync();
    if (tid == 0) {
      remote_st(remote(&S.all_near[rank], 0), S.near_n);
      remote_st(remote(&S.all_zeros[rank], 0), S.zeros);
      remote_st(remote(&S.all_largest[rank], 0), S.largest);
    }
    const int share = kBins / 4 / (int)csize;
#pragma unroll 1
    for (int i = (int)rank * share + tid; i < ((int)rank + 1) * share; i += kThreads) {
      uint4 v[kMaxCluster], a = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (uint32_t p = 0; p < kMaxCluster; ++p)
        v[p] = p < csize ? remote_ld4(remote(S.hist, p) + 16 * i) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (uint32_t p = 0; p < kMaxCluster; ++p)
        a.x += v[p].x, a.y += v[p].y, a.z += v[p].z, a.w += v[p].w;
      remote_st4(remote(S.hist, 0) + 16 * i, a);
    }
    cluster_sync();
    if (rank != 0) {
      cluster_sync();  // the first CTA has read what it needs
      return;
    }
  } else {
    __syncthreads();
    if (tid == 0) S.all_near[0] = S.near_n, S.all_zeros[0] = S.zeros, S.all_largest[0] = S.largest;
    __syncthreads();
  }
  uint32_t near = 0, zeros = 0, top_key = kKeyMinusInf;
  for (uint32_t p = 0; p < csize; ++p) {
    near += S.all_near[p];
    zeros += S.all_zeros[p];
    top_key = max(top_key, S.all_largest[p]);
  }
  // a row with nothing but -inf and NaN, or bad settings: no token
  if (!good || top_key <= kKeyMinusInf) {
    if (tid == 0) {
      if (!good) ipd_set_error(&g_trunc_err, IPD_DEVERR_SETTING);
      P.tokens[row] = -1;
      if (P.logp) P.logp[row] = -INFINITY;
      if (P.kept) P.kept[row] = 0;
    }
    if (csize > 1) cluster_sync();
    return;
  }
  const Scale C = make_scale(c, min_p, top_key, P.one);
  if (tid == 0) {
    S.scale = C;
    S.hist[kBins / 2 + kFreeWord] = 0;  // what counted as -2^12
  }
  const uint32_t least_key = C.inf ? kKeyInf : order_key(C.least2 & 0xffffu);
  const uint32_t mid = near + (zeros != 0);
  const bool windows = top_key <= kKeyLow || top_key >= kKeyHigh || mid > (uint32_t)kMid ||
                       least_key < kKeyLow;

  // ---- the bins between the signs: an entry's place is the number of greater ones ----
  if (mid && !windows) {
    uint32_t key = kKeyZero, mult = zeros;
    if (tid < (int)near) {
      uint32_t i = tid, p = 0;
      while (i >= S.all_near[p]) i -= S.all_near[p++];
      const uint32_t pair = remote_ld(remote(&S.near_key[i & ~1u], p));
      key = pair >> (16 * (i & 1)) & 0xffffu;
      mult = 0;
    }
    uint32_t *list = S.n_before;  // (not in use yet)
    if (tid < (int)mid) list[tid] = key;
    if (tid < kMid) S.mid_key[tid] = kKeyZero;
    __syncthreads();
    if (tid < (int)mid) {
      uint32_t greater = 0, first = 1;
#pragma unroll 1
      for (int i = 0; i < (int)mid; ++i) {
        const uint32_t k = list[i];
        greater += k > key;
        if (k == key && i < tid) first = 0;
        if (key != kKeyZero) mult += k == key;
      }
      if (first) {
        S.mid_key[greater] = (uint16_t)key;
        S.hist[word_at(-1, kSide + greater)] = mult;
      }
    }
  }
  __syncthreads();

  // ---- the cuts and the draw: positions in the running sums ----
  // 0 the sums of all, 1 the last entry of top-k, 2 the last unit of mass that
  // top-p needs, 3 the drawn one
  const int w_first = windows ? (int)(top_key / kBins) : 0;
  const int w_last = windows ? (int)(least_key / kBins) : 0;
  u64 t = 0, kept_mass = 0, above = 0;
  uint32_t kept_n = 0;
#pragma unroll 1
  for (int what = 0; what < 4; ++what) {
    above = 0;
    uint32_t above_n = 0;
#pragma unroll 1
    for (int w = w_first; w >= w_last; --w) {
      if (windows) count_window(S, R, n_vec, w);
      if (windows || what == 0) sum_bins(S);
      const u64 mass = S.before[kThreads];
      const uint32_t n = S.n_before[kThreads];
      if (what == 1 ? t - above_n < n : what > 1 && t - above < mass) {
        find_bin(S, what == 1, what == 1 ? t - above_n : t - above);
        break;
      }
      above += mass;
      above_n += n;
    }
    if (what == 0) {  // (at least 2^30: the largest logit is in)
      kept_mass = above;
      kept_n = above_n;
      t = (u64)(top_k - 1);
      if (!cut_k || (uint32_t)top_k >= kept_n) ++what;
    } else {
      above += S.found_before;
      if (what < 3) {  // the last entry that is in, one of its equals
        above_n += S.found_n;
        const uint32_t n = what == 1 ? (uint32_t)t - above_n : quotient(t - above, S.found_weight);
        kept_mass = above + (u64)(n + 1) * S.found_weight;
        kept_n = above_n + n + 1;
      }
    }
    if (what == 1) {
      const u64 need = once(S, [&] { return needed(top_p, kept_mass); });
      t = need - 1;
      if (need == kept_mass) ++what;
    }
    if (what == 2) t = once(S, [&] { return position(uf, kept_mass); });
  }
  const uint32_t key = S.found_key;
  uint32_t j = quotient(t - above, S.found_weight);  // rank among its equals
  if (tid == 0) {
    if (P.kept) P.kept[row] = (int32_t)kept_n;
    if (P.logp)
      P.logp[row] = (exponent(C, key_value(key)) - log2f((float)kept_mass * 0x1p-30f)) * kLn2;
  }
  // the piece that holds it, if the pieces' histograms tell
  int first = 0, last = n_vec;
  if (csize > 1) {
    const uint32_t bits = key_bits(key);
    if (!windows && (bits & 0x7fffu) - kLowBits < (uint32_t)kSide) {
      uint32_t n = 0;
      if (lane > 0 && lane < (int)csize)
        n = remote_ld(remote(S.hist, lane) + (words2(bits) & 0xffffu));
      const uint32_t others = __reduce_add_sync(0xffffffffu, n);
      if (lane == 0) n = S.found_count - others;
      uint32_t p = 0;
      for (; p + 1 < csize; ++p) {
        const uint32_t m = __shfl_sync(0xffffffffu, n, p);
        if (j < m) break;
        j -= m;
      }
      first = (int)p * piece;
      last = min(first + piece, n_vec);
    }
    cluster_arrive();
  }
  look_up(S, R, first, last, key, j, &P.tokens[row]);
  if (csize > 1) cluster_wait();
}
};

template <int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
    sample_trunc_kernel(const __grid_constant__ Params P) {
  Sampler<kThreads>::run(P);
}

struct DevInfo {
  int sms = 0;
};
DevInfo g_trunc_dev[64];

}  // namespace

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_trunc_error() {
  if (!g_trunc_used.load(std::memory_order_relaxed)) return 0u;
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
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
      return IPD_ERR_CUDA;
    D.sms = n;
  }
  // CTAs of a row.  A cluster's barriers and the sum of its histograms cost about
  // 3 us, a CTA alone 0.1 us per 1,024 entries: clusters are for long rows, and while
  // every CTA has an SM (clusters of 8 do not fill the SMs evenly).  Measured on rows
  // of mixed settings with 1 / 2 / 4 / 8 CTAs, in us, 151,936 entries: 1 row 23.1 / 18.6
  // / 14.9 / 14.0, 16 rows 25.0 / 19.9 / 15.6 / 18.1, 48 rows 24.8 / 20.0 / 20.7 / 29.3, 64
  // rows 25.1 / 20.3 / 21.5 / 33.0, 77 rows 24.9 / 26.0 / 28.8 / 40.3 (two CTAs an SM gain
  // nothing), 152 rows 28.7 / 29.2 / 46.8 / 72.4; 50,021: 1 row 12.7 / 13.2 / 12.5 / 12.6, 77
  // rows 14.3 / 17.9 / 23.4 / 35.5; 32,000: 1 row 10.8 / 12.3 / 12.3 / 12.4.
  const int span = vocab + 7;  // a row may start inside a 16-byte vector
  int csize = kMaxCluster;
  while (csize > 1 && (span < kSplitRow || span < csize * kMinPiece ||
                       (long long)n_rows * csize > (csize == 8 ? D.sms * 3 / 4 : D.sms)))
    csize /= 2;
  Params P;
  P.logits = logits;
  P.stride = row_stride;
  P.u = u;
  P.inv_t = inv_temperature;
  P.top_p = top_p;
  P.min_p = min_p;
  P.top_k = top_k;
  P.tokens = tokens;
  P.kept = n_kept;
  P.logp = logp;
  P.vocab = vocab;
  P.one = 1.f;
  P.piece = (int)(((span + csize - 1) / csize + 7) / 8 * 8);
  // Threads of a CTA: 512, two CTAs an SM, or 256 and four once there are rows for
  // them, whose searches overlap more.  512 / 256 threads: 512 rows of 151,936 72.1 /
  // 69.9 us, of 50,021 38.8 / 32.2, of 4,096 22.7 / 15.3; 400 rows 66.9 / 58.2, 34.4 / 26.6,
  // 19.4 / 12.8; 304 rows 41.6 / 47.1, 20.7 / 21.1, 12.9 / 11.2.
  const bool narrow = n_rows > 2 * D.sms;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)n_rows * csize);
  cfg.blockDim = dim3(narrow ? 256 : 512);
  cfg.dynamicSmemBytes = narrow ? sizeof(Sampler<256>::Shared) : sizeof(Sampler<512>::Shared);
  cfg.stream = reinterpret_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = csize;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  g_trunc_used.store(true, std::memory_order_relaxed);
  if (cudaLaunchKernelEx(&cfg, narrow ? sample_trunc_kernel<256> : sample_trunc_kernel<512>, P) !=
      cudaSuccess) {
    (void)cudaGetLastError();
    return IPD_ERR_CUDA;
  }
  return IPD_OK;
}

// Span-verify and decode attention over a paged cache held in 8 bits.
//
//   o_i = sum_j p_ij 2^ev_j v_j / sum_j p_ij,  p_ij = exp(scale 2^ek_j q_i.k_j - m_i)
//
// k_j, v_j e4m3 values, ek, ev the scales of their page and head, key j seen by
// query i of a span of n where j <= L - n + i.
//
// What bounds it: 256 bytes a key and KV head against 512 flop a row, so HBM; a
// tile of 128 keys (32 KB) is about 1,400 cycles of an SM's share, which is what
// everything else has to stay below.  The tensor cores take the cache's bytes as
// they are (kind::f8f6f4), nothing is unpacked:
//   S^T = K Q^T   keys are the 128 rows of the product, the rows (query, head of
//                 the group) its columns; q as two e4m3 terms of its row's scale
//   O^T = V^T P^T dims are the rows; V and P in the order they lie in, keys last
// The transposed form makes the cost follow the number of rows (16, 32 or 64
// columns) and gives every thread one key: a key's scales are two numbers of its
// thread.  P goes into the second product as two e4m3 terms, the second times 32,
// side by side as columns; O's two halves are added at the end.
//
// Softmax.  p = 2^(s ck ar + dE - ref): ck holds the softmax scale and K's, ar q's
// row scale, dE V's exponent relative to that of the item's first pages.  ref is the
// row's largest in that tile, less 4; it rises (and O and the sums are rescaled) only
// when a weight would leave 2^8, so most tiles need no maximum across threads.  The
// reference includes V's scale, since it is the product that has to fit e4m3.
// The terms end at 2^-15: 12 to 14 nats below one large weight that V answers with next to
// nothing, all other keys of a long sequence would be lost.  So references fall too, to a
// tile's maximum less 4, where all of a row's weights there lie below 2^-5.  This is looked
// for in a part's second tile, in the tile after a fall or a rise by more than 2^8, and 64
// tiles after the last move; with every far rise the wait behind the next one doubles, to 32
// tiles, so that heads whose tiles differ that much do not swing all the time (64 spans of 1 to
// 16 over 256 to 16,384 keys, K scales of pages 2^3 apart: 128 us, 129 where references do
// not fall; a look in every tile 209 before the code was shortened).
//
// Work.  All (request, KV head, block of 128 rows, tile) in one line, cut into parts of
// equal cost, a CTA each: nothing is claimed, the cut depends on the lengths alone.
// A task cut between CTAs leaves normalised partial rows; the CTA that finishes last
// joins them in order.  Within a CTA up to four tasks (of up to 32 rows; two of up to 64)
// run side by side, a warpgroup each, and get a tile each in turn, so that one's first
// maximum and last rows pass behind the others' tiles.
//
// Warps: 0-15 softmax, four warpgroups of up to 32 rows, 16 loads, 17 issues the first
// product, 18 the second, 19 finds the items, 20 puts their tiles in order and fetches page
// ids and scales.
//
// Measured (bytes of the visible keys and of the rows, at 6,784 GB/s for a copy): 19 requests
// of one query over 32,768 keys, 8 KV heads, 199 us, 0.94 of a copy's rate; 128 over 256 to
// 16,384 keys 174 us, 0.88.  With 128 rows a key: 271 us for 19 x 16 queries over 32,768 keys of
// 4 heads, 602 TFLOP/s; no unit is full there (issue slots half busy), the softmax warps wait for
// TMEM and at the barrier of their warpgroup's tile.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>
#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "e4m3.cuh"

IPD_DECLARE_ERROR_WORD(g_attn8_err);
// whether this process has launched (or captured) a kernel that may set the word:
// a program without these calls does not pay for reading it
static std::atomic<bool> g_attn8_used{false};

namespace {

typedef unsigned long long u64;

constexpr int kD = 128;
constexpr int kPage = 16;
constexpr int kKeys = 128;                // keys of a tile
constexpr int kPages = kKeys / kPage;     // its pages
constexpr int kTileBytes = kKeys * kD;    // 16 KB of K or V
constexpr int kPageBytes = kPage * kD;
constexpr int kMaxGroup = 128;
constexpr int kBlockRows = 128;           // rows of a task
constexpr int kGroups = 4;                // softmax warpgroups
constexpr int kRows = 32;                 // ... and the rows of one
constexpr int kKStages = 4, kVStages = 5;
// Tiles handed out whose product is not complete, and items.  (128 requests of 256 to 16,384 keys /
// 1,000 of 300, us: 195 / 249 with 8 tiles, 172 / 271 with 11, 173 / 294 with 16, 174 / 315 with 32;
// with 11 and 16 items in place of 8 170 / 255, with 4 175 / 330.)
constexpr int kTiles = 11;
constexpr int kScales = 16;               // of a warpgroup's tiles, scales handed out that it has not read
constexpr int kBatch = 4;                 // ... fetched at once
constexpr int kSlots = 16;
constexpr int kSoftmaxWarps = 4 * kGroups;
constexpr int kLoadWarp = kSoftmaxWarps, kQkWarp = kLoadWarp + 1, kPvWarp = kLoadWarp + 2, kItemWarp = kLoadWarp + 3;
// (the fifth orders tiles; with two for loads and two that converted queries ahead of their turn
// 1,000 requests of 300 keys took 411 us in place of 322)
constexpr int kThreads = 32 * (kSoftmaxWarps + 5);
constexpr int kItemReaders = kSoftmaxWarps + 1;
static_assert(kBatch * kPages == 32, "a lane a page");

// TMEM columns of a warpgroup: scores, O (two terms), and every thread's own sums
constexpr uint32_t kTmemCols = 512;
__host__ __device__ constexpr uint32_t col_s(uint32_t g) { return 32u * g; }
__host__ __device__ constexpr uint32_t col_o(uint32_t g) { return 128u + 64u * g; }
__host__ __device__ constexpr uint32_t col_l(uint32_t g) { return 384u + 32u * g; }

constexpr float kBase = 4.f;      // a row's reference is its largest exponent less this
constexpr float kLimit = 8.f;     // weights stay below 2^8 (e4m3 ends at 448, and their second term too: 8 kLoScale)
constexpr float kLoScale = 32.f;
// When references fall: see the head of this file.
constexpr float kLow = -5.f;      // a tile of lower exponents makes a row's reference fall
constexpr float kDeep = 64.f;     // ... but no lower than this below its highest: sums and O stay far from fp32's ends
constexpr float kFarRise = 8.f;   // after a rise by more the next tile is looked through
// Tiles from a move to the next look; at most, after far rises.  (19 x 16 queries / 38 x 8 over 32,768 keys of
// 4 heads, us: 278 / 354 at 32 and 32, 271 / 339 at 64 and 32, 262 / 326 where references do not fall.)
constexpr int kIdle = 64, kMostWait = 32;
constexpr int kShort = 4 * kKeys; // sequences up to here: references do not fall
constexpr int kFar = 80;       // V scales further than 2^80 from that of the first tile count as that far
// What a tile of a task with up to 16, 32, 64 and 128 rows costs, and a task beside its tiles (up to
// 32, 64, 128 rows): the line is cut into equal costs.  In cycles a tile takes about 1,480, 2,170,
// 3,200 and 3,750 where a CTA has one task alone, 1,450, 1,600, 2,400 and 3,700 where it has several.
constexpr int kTileH = 4, kTile1 = 5, kTile2 = 7, kTile4 = 12;
constexpr int kTask1 = 20, kTask2 = 40, kTask4 = 60;
constexpr int kNoPage = 1 << 20;  // in place of an exponent: no such page

struct BatchDev {
  const uint8_t *ks, *vs;
  const uint16_t *q;
  uint16_t *out;
  const int *cu_q, *seq_len, *page_table;
  int num_reqs, hq, hkv, group, max_pages, max_q_len, max_seq_len, total_q, num_pages;
  int rows_end;  // a pool row that is not there: loads as zeros
};

struct Params {
  CUtensorMap k[IPD_MAX_BATCHES], v[IPD_MAX_BATCHES];
  BatchDev b[IPD_MAX_BATCHES];
  int req_base[IPD_MAX_BATCHES + 1];
  int n, total_reqs;
  float scale_log2;
  long long *prefix;  // [total_reqs + 1] cost of the requests before each, and the dearest tile's
  int4 *info;         // [total_reqs] length, queries, first row, tiles
  int *done;          // [CTAs][kGroups] parts done of the task that starts in this CTA and goes on, by row group
  float *part;        // [2 CTAs] partial rows: part_rows x 128, then part_rows log-sums
  int part_rows;
};

struct Item {
  int valid, b, c0, n, L, h;
  int row0, rows;       // first row of the task among the request's, and number
  int nr, ng, wg;       // rows of a warpgroup (16 or 32); its warpgroups (1, 2 or 4) and their first
  int t0, t1;           // tiles
  int masked;           // the first key that some row of the task does not see
  int r, n_pages;       // request of the batch, its pages
  int part;             // partial slot (-1: the whole task is here)
  int cta0, ctab, cta1; // the CTAs of the task: cta0, then ctab .. cta1
  int bad;              // a key with NaN in V was hidden from some of its rows (see mend)
};

// A tile on its way through the loading and issuing warps.
enum { kFirst = 1, kLast = 2, kHides = 4, kEnd = 8 };
struct Tile {
  alignas(16) int y[kPages];  // first pool rows of its pages
  uint32_t what;  // the rest in one word, which one warp-wide move makes uniform:
  // its item's first, last; it holds hidden keys; there is none after the one before (4 bits);
  // warpgroups (3), the first of them (2), 32 rows each or 16 (1), the item's place
  // in this CTA's order (5: slot and turn), batch (3)
};
static_assert(2 * kSlots == 32 && kGroups == 4 && IPD_MAX_BATCHES <= 8, "the fields of Tile::what");
struct What {
  uint32_t w;
  IPD_DEVINL bool is(int flag) const { return w & flag; }
  IPD_DEVINL int ng() const { return w >> 4 & 7u; }
  IPD_DEVINL int wg() const { return w >> 7 & 3u; }
  IPD_DEVINL int nr() const { return 16u << (w >> 9 & 1u); }
  IPD_DEVINL uint32_t item() const { return w >> 10 & 31u; }
  IPD_DEVINL int b() const { return w >> 15 & 7u; }
};
// ... and what a warpgroup has to know of it.
struct Scales {
  float ck[kPages];  // K's scale times the softmax scale, in log2
  int ev[kPages];    // V's exponent (128: NaN), or kNoPage
  int gap, v;        // a page that is not there lies among the keys; V's stage
};

struct Shared {
  alignas(1024) uint8_t k[kKStages][kTileBytes];
  alignas(1024) uint8_t v[kVStages][kTileBytes];
  alignas(1024) uint8_t q[2][kGroups][kRows * kD];     // the two terms of the queries
  alignas(1024) uint8_t p[kGroups][kKeys * 2 * kRows]; // a warpgroup's P
  alignas(16) float4 state[kGroups][kRows / 2];        // a pair of rows: ar, ar', -ref, -ref'
  alignas(16) float alpha[kGroups][kRows];
  alignas(16) float red[kGroups][4][kRows];
  uint32_t unseen[kGroups];                            // rows that have not seen a key of their item
  uint32_t below[kGroups][4];                          // rows that a warp's keys have below kLow
  uint32_t moved[kGroups], deep[kGroups];              // rows whose sums are rescaled; rows at their floor
  float floor[kGroups][kRows];                         // how low a row's reference may fall
  int look[kGroups], gap[kGroups];                     // tiles to the next look for rows that fall; after a far rise
  // first key of a span with a NaN in this dim of V (by an item's first warpgroup)
  int nan_key[kGroups][kD];
  int last[kGroups], abort;
  uint32_t tmem;
  Tile tile[kTiles];
  Scales scales[kGroups][kScales];
  Item item[kSlots];
  uint64_t k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
  uint64_t tile_full[kTiles], tile_empty[kTiles];
  uint64_t sc_full[kGroups][kScales], sc_empty[kGroups][kScales];
  uint64_t q_full[kSlots], s_full[kGroups], s_empty[kGroups], p_full[kGroups], pv_done[kGroups];
  uint64_t v_ready[kGroups];  // a tile with hidden keys has landed
  uint64_t item_full[kSlots], item_taken[kSlots], item_empty[kSlots], pair[2], all, drain[2];
};
constexpr int kSharedBytes = (int)sizeof(Shared) + 1024;  // the base is aligned by hand
static_assert(kSharedBytes <= 232448, "shared memory of one CTA");

// ---- PTX ---------------------------------------------------------------------
IPD_DEVINL void tma_load_2d(void *dst, const CUtensorMap *map, int x, int y, uint64_t *bar, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3}], [%4], %5;" ::"r"(smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(smem_u32(bar)), "l"(policy)
      : "memory");
}
// D[tmem] (+)= A[smem] B[smem], e4m3 operands, fp32 accumulation (one thread).
IPD_DEVINL void tc_mma_f8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Instruction descriptor: e4m3 A and B, fp32 D; transposed operands are MN-major.
__host__ __device__ constexpr uint32_t idesc_f8(int n, int transposed) {
  return (1u << 4) | (uint32_t)transposed << 15 | (uint32_t)transposed << 16 | (uint32_t)(n >> 3) << 17 |
         (128u >> 4) << 24;
}
// Shared-memory descriptor with 8-row groups of `row` bytes a row, swizzled over
// the row (128, 64 or 32 bytes).
IPD_DEVINL uint64_t sdesc(uint32_t saddr, int row) {
  const uint64_t layout = row == 128 ? 2 : row == 64 ? 4 : 6;
  return (uint64_t)((saddr & 0x3ffffu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(8 * row >> 4) << 32 | 1ull << 46 |
         layout << 61;
}
IPD_DEVINL bool bar_or(int id, int threads, bool x) {
  uint32_t r;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %3, 0;\n\t"
      "barrier.cta.red.or.pred.aligned p, %1, %2, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"(id), "r"(threads), "r"((uint32_t)x)
      : "memory");
  return r != 0;
}
IPD_DEVINL void tc_st_32x32b_x16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
IPD_DEVINL void tc_ld_32x32b_x8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
IPD_DEVINL void tc_ld_x1(uint32_t taddr, uint32_t &r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(taddr) : "memory");
}
IPD_DEVINL void tc_st_x1(uint32_t taddr, uint32_t r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(r) : "memory");
}
IPD_DEVINL uint32_t half2_of(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
IPD_DEVINL uint32_t half2_sub(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
IPD_DEVINL uint32_t half2_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Four fp16 values as e4m3, and back.
IPD_DEVINL uint32_t e4m3x4_h(uint32_t h01, uint32_t h23) {
  uint32_t d;
  asm("{\n\t.reg .b16 a, b;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 a, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 b, %2;\n\t"
      "mov.b32 %0, {a, b};\n\t}"
      : "=r"(d)
      : "r"(h01), "r"(h23));
  return d;
}
IPD_DEVINL void h_from_e4m3x4(uint32_t v, uint32_t &h01, uint32_t &h23) {
  asm("{\n\t.reg .b16 a, b;\n\t"
      "mov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
      "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(h01), "=r"(h23)
      : "r"(v));
}
IPD_DEVINL void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
IPD_DEVINL void grid_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// ---- waits ---------------------------------------------------------------------
// For a whole warp, with one answer.  Gives up after about a second, or as soon as
// another warp of the CTA has given up.  Warps that poll take issue slots from those
// that work (without a pause they were half of all instructions), so those that run
// ahead sleep `pause` ns between two looks.  (A call: code that every warp comes by often has
// to be short, for the instruction cache's sake; inlined, 1,000 requests of 300 keys took
// 328 us, now 292.)
__device__ __noinline__ bool wait_slow(uint64_t *bar, uint32_t parity, volatile int *abort, uint32_t pause) {
  const long long t0 = clock64();
  bool ok;
#pragma unroll 1
  while (!(ok = mbar_try_wait(bar, parity)) && !*abort) {
    if (pause) __nanosleep(pause);
    if (clock64() - t0 > kWaitLimitCycles) {
      ipd_set_error(&g_attn8_err, IPD_DEVERR_WAIT);
      *abort = 1;
    }
  }
  return __all_sync(0xffffffffu, ok) != 0;
}
IPD_DEVINL bool wait(uint64_t *bar, uint32_t parity, volatile int *abort, uint32_t pause = 200) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return wait_slow(bar, parity, abort, pause);
}
// One lane of a converged warp issues; every other value is the whole warp's, so that
// operands stay in uniform registers (issued from a branch of one lane, a product
// or a copy takes hundreds of cycles).
IPD_DEVINL bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
IPD_DEVINL int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
// The n-th use (0, 1, ...) of a barrier of a ring of `ring`: a consumer waits for it
// with full(n), a producer for the release of its slot with free(n).
IPD_DEVINL uint32_t full(uint32_t n, uint32_t ring) { return n / ring & 1u; }
IPD_DEVINL uint32_t free_(uint32_t n, uint32_t ring) { return (n / ring & 1u) ^ 1u; }
IPD_DEVINL void arrive_warp(uint64_t *bar, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(bar);
}

// ---- plan ------------------------------------------------------------------------
IPD_DEVINL int batch_of(const Params &P, int g) {
  int b = 0;
  while (b + 1 < P.n && g >= P.req_base[b + 1]) ++b;
  return b;
}

IPD_DEVINL int tile_cost(int rows) { return rows > 64 ? kTile4 : rows > 32 ? kTile2 : rows > 16 ? kTile1 : kTileH; }
IPD_DEVINL int item_cost(int rows) { return rows > 64 ? kTask4 : rows > 32 ? kTask2 : kTask1; }
IPD_DEVINL long long task_cost(int rows, int tiles) { return item_cost(rows) + (long long)tiles * tile_cost(rows); }

// Checks the requests and adds up their costs; one block.
__global__ void __launch_bounds__(1024) attn8_plan_kernel(const __grid_constant__ Params P, int ctas) {
  __shared__ long long warp_units[32];
  grid_launch();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  for (int i = tid; i < ctas * kGroups; i += blockDim.x) P.done[i] = 0;
  long long carry = 0;
  int dearest = 1;
  for (int base = 0; base < P.total_reqs; base += blockDim.x) {
    const int g = base + tid;
    long long units = 0;
    if (g < P.total_reqs) {
      const int b = batch_of(P, g), r = g - P.req_base[b];
      const BatchDev &B = P.b[b];
      const int c0 = B.cu_q[r], c1 = B.cu_q[r + 1], L = B.seq_len[r];
      const int n = c1 - c0;
      int tiles = 0;
      if (c0 < 0 || c1 < c0 || c1 > B.total_q) {
        ipd_set_error(&g_attn8_err, IPD_DEVERR_SPAN);
      } else if (n > B.max_q_len || L < n || L > B.max_seq_len) {
        ipd_set_error(&g_attn8_err, IPD_DEVERR_SEQ_LEN);
      } else if (n > 0) {
        tiles = (L + kKeys - 1) / kKeys;
        const int rows = n * B.group, blocks = (rows + kBlockRows - 1) / kBlockRows;
        dearest = max(dearest, tile_cost(min(rows, kBlockRows)));
        units = (long long)B.hkv *
                ((blocks - 1) * task_cost(kBlockRows, tiles) + task_cost(rows - (blocks - 1) * kBlockRows, tiles));
      }
      P.info[g] = make_int4(L, n, c0, tiles);
    }
    long long up = units;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, up, o);
      if (lane >= o) up += x;
    }
    if (lane == 31) warp_units[warp] = up;
    __syncthreads();
    long long before = carry, all = 0;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += warp_units[w];
      all += warp_units[w];
    }
    if (g < P.total_reqs) P.prefix[g] = before + up - units;
    carry += all;
    __syncthreads();
  }
  dearest = __reduce_max_sync(0xffffffffu, dearest);
  if (lane == 0) warp_units[warp] = dearest;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < warps; ++w) warp_units[0] = max(warp_units[0], warp_units[w]);
    P.prefix[P.total_reqs] = carry, P.prefix[P.total_reqs + 1] = warp_units[0];
  }
}

// ---- items (one warp) ----------------------------------------------------------------
// A task's place in the line: its first tile begins at 0, tile t at `item` + t w, and
// it ends at `item` + tiles w, w the cost of one of its tiles.
// the first tile that begins at `off` or later
IPD_DEVINL int tile_at(long long off, int item, int w, int tiles) {
  if (off <= 0) return 0;
  const long long t = (off - item + w - 1) / w;
  return (int)max(1LL, min((long long)tiles, t));
}

__device__ void item_warp(const Params &P, Shared &S, int lane) {
  grid_wait();  // what the plan wrote
  const long long W = P.prefix[P.total_reqs];
  // (a part is no shorter than a tile, so that none between a task's ends has no tile)
  const long long C = max(1LL, min((long long)gridDim.x, W / P.prefix[P.total_reqs + 1]));
  uint32_t n = 0;
  const long long lo = blockIdx.x < C ? blockIdx.x * W / C : W, hi = blockIdx.x < C ? (blockIdx.x + 1) * W / C : W;
  int g = 0;
  if (lo < hi) {
    // the last request that begins at lo or before: 32 probes a round
    int from = 0, end = P.total_reqs;  // prefix[from] <= lo < prefix[end]
    while (end - from > 1) {
      const int step = (end - from + 31) / 32;
      const int at = from + lane * step;
      const uint32_t in = __ballot_sync(0xffffffffu, at < end && P.prefix[at] <= lo);
      const int k = 31 - __clz(in);
      from += k * step;
      end = min(end, from + step);
    }
    g = from;
  }
  long long pos = lo;  // where the next task to look at begins, or this CTA's part
  while (pos < hi) {
    const long long first = P.prefix[g], next = P.prefix[g + 1];
    if (next <= pos) {  // nothing to do for this request
      ++g;
      continue;
    }
    const int b = batch_of(P, g);
    const int group = P.b[b].group;
    const int4 info = P.info[g];
    const int L = info.x, tiles = info.w, rows_all = info.y * group;
    // (a request's blocks are alike but for the last, which may have fewer rows)
    const int blocks = (rows_all + kBlockRows - 1) / kBlockRows, last_rows = rows_all - (blocks - 1) * kBlockRows;
    const long long c_full = task_cost(kBlockRows, tiles), c_last = task_cost(last_rows, tiles);
    const long long c_head = (blocks - 1) * c_full + c_last;
    int h = (int)((pos - first) / c_head);
    long long in_head = pos - first - h * c_head;
    int block = (int)min((long long)blocks - 1, in_head / c_full);
    long long at = first + h * c_head + block * c_full;  // the task's beginning
    while (at < hi && at < next) {
      const int like = block == blocks - 1 ? last_rows : kBlockRows, w = tile_cost(like), item = item_cost(like);
      const long long cost = block == blocks - 1 ? c_last : c_full;
      const int t0 = tile_at(lo - at, item, w, tiles), t1 = hi - at >= cost ? tiles : tile_at(hi - at, item, w, tiles);
      if (t0 < t1) {
        const int slot = n % kSlots;
        if (!wait(&S.item_empty[slot], free_(n, kSlots), &S.abort)) return;
        const int row0 = block * kBlockRows, rows = min(kBlockRows, rows_all - row0);
        const int ng = rows > 64 ? 4 : rows > 32 ? 2 : 1;
        if (lane == 0) {
          Item &I = S.item[slot];
          I.valid = 1, I.b = b, I.c0 = info.z, I.n = info.y, I.L = L, I.h = h;
          I.row0 = row0, I.rows = rows, I.nr = rows > 16 ? 32 : 16, I.ng = ng;
          I.t0 = t0, I.t1 = t1, I.bad = 0;
          I.masked = L - info.y + 1 + row0 / group;
          I.r = g - P.req_base[b], I.n_pages = (L + kPage - 1) / kPage;
          I.part = t1 - t0 == tiles ? -1 : t0 > 0 ? 2 * (int)blockIdx.x : 2 * (int)blockIdx.x + 1;
          if (I.part >= 0) {
            // CTA i begins at floor(i W / C): the last one that begins at p or before
            const auto cta = [&](int t) {
              const long long p = at + (t > 0 ? item + (long long)t * w : 0);
              return (int)(((p + 1) * C - 1) / W);
            };
            I.cta0 = cta(0), I.ctab = max(I.cta0 + 1, cta(1)), I.cta1 = cta(tiles - 1);
          }
          mbar_arrive(&S.item_full[slot]);
        }
        __syncwarp();
        ++n;
      }
      at += cost;
      if (++block == blocks) block = 0, ++h;
    }
    pos = min(hi, next);
  }
  const int slot = n % kSlots;
  if (!wait(&S.item_empty[slot], free_(n, kSlots), &S.abort)) return;
  if (lane == 0) {
    S.item[slot].valid = 0;
    mbar_arrive(&S.item_full[slot]);
  }
}

// ---- the order of tiles, page ids and scales (one warp) -------------------------------
// Items are taken in order, each as soon as there is a warpgroup for it (two, four) that has
// been given all its tiles, and the items under way get a tile each in turn: up to four
// softmaxes run side by side, and one item's end is hidden behind the others' tiles.
// Tiles go out four at a time, a lane a page: while a batch's scales are under way, so are
// the next one's page ids.
IPD_DEVINL bool mbar_test(uint64_t *bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

__device__ void page_warp(const Params &P, Shared &S, int lane) {
  const int mine = lane / kPages, place = lane % kPages;  // a lane's tile of a batch, and page
  uint32_t n = 0, it = 0;    // items taken; tiles handed out
  int known = 0;             // warpgroups that item n wants (0: it has not been looked at)
  bool ended = false, given_up = false;
  int last_g = kGroups - 1;
  // lane g < 4: what warpgroup g has been given: the item, its next tile and its end, the
  // first of its warpgroups; how many tiles the warpgroup has had
  int w_item = 0, w_t = 0, w_t1 = 0, w_first = 0;
  uint32_t w_tiles = 0;
  // the batch whose ids are under way: a lane's item, tile, first warpgroup, how many tiles
  // before it are that item's; w_tiles before the batch
  int e_item = 0, e_t = 0, e_g = 0, e_q = 0, id = -1, left = 0;
  uint32_t e_tiles = 0;

  // The next batch: left = 0 where there is none, or none yet.  May wait for an item only where
  // `block`: with tiles in hand that have not gone out, the item could be waiting for theirs to end.
  const auto fetch = [&](bool block) {
    left = 0, id = -1;
    uint32_t act;  // first warpgroups of the items under way
    while (true) {
      const bool active = lane < kGroups && w_t < w_t1;
      const uint32_t busy = __ballot_sync(0xffffffffu, active);
      act = __ballot_sync(0xffffffffu, active && w_first == lane);
      if (ended) break;
      const int slot = n % kSlots;
      if (known == 0) {
        // (items under way go on while the next one is not there yet)
        if (act || !block) {
          if (!__all_sync(0xffffffffu, mbar_test(&S.item_full[slot], full(n, kSlots)))) break;
        } else if (!wait(&S.item_full[slot], full(n, kSlots), &S.abort, 20)) {
          given_up = true;
          return;
        }
        if (!S.item[slot].valid) {
          ended = true;
          break;
        }
        known = S.item[slot].ng;
      }
      int g = -1;
#pragma unroll
      for (int k = kGroups; k >= 1; --k) {  // the next after the one that had a tile last
        const int at = (last_g + k) & (kGroups - known);
        if ((busy >> at & ((1u << known) - 1u)) == 0) g = at;
      }
      if (g < 0) break;
      if (lane == 0) {
        S.item[slot].wg = g;
        mbar_arrive(&S.item_taken[slot]);
      }
      if (lane >= g && lane < g + known)
        w_item = (int)n, w_t = S.item[slot].t0, w_t1 = S.item[slot].t1, w_first = g;
      ++n;
      known = 0;
    }
    if (act == 0) return;
    // the items under way in turn, a tile each, and again
    const int some = __popc(act), turn = mine % some;
    uint32_t bits = (act | act << kGroups) >> (last_g + 1) & ((1u << kGroups) - 1u);
    for (int i = 0; i < turn; ++i) bits &= bits - 1;
    int g = (last_g + __ffs(bits)) & (kGroups - 1), q = mine / some;
    int t = __shfl_sync(0xffffffffu, w_t, g) + q;
    const uint32_t past = __ballot_sync(0xffffffffu, t >= __shfl_sync(0xffffffffu, w_t1, g));
    left = past ? (__ffs(past) - 1) / kPages : kBatch;
    // (the lanes of tiles past an end do as the last one's do)
    const int from = min(mine, left - 1) * kPages + place;
    e_g = __shfl_sync(0xffffffffu, g, from), e_t = __shfl_sync(0xffffffffu, t, from), e_q = __shfl_sync(0xffffffffu, q, from);
    e_item = __shfl_sync(0xffffffffu, w_item, e_g);
    e_tiles = w_tiles;
    last_g = __shfl_sync(0xffffffffu, e_g, 31);
    int given = 0;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) given += i < left && __shfl_sync(0xffffffffu, e_g, i * kPages) == w_first;
    if (lane < kGroups && w_t < w_t1) w_t += given, w_tiles += given;
    const Item &I = S.item[e_item % kSlots];
    const BatchDev &B = P.b[I.b];
    const int page = e_t * kPages + place;
    if (page < I.n_pages) {
      id = B.page_table[(size_t)I.r * B.max_pages + page];
      if (id < 0 || id >= B.num_pages) {
        ipd_set_error(&g_attn8_err, IPD_DEVERR_PAGE_ID);
        id = -2;
      }
    }
  };
  while (true) {
    if (left == 0) {
      fetch(true);
      if (left == 0) break;
    }
    const int now = left, item = e_item, t = e_t, g = e_g, q = e_q;
    const uint32_t tiles = e_tiles, at = it + min(mine, now - 1);
    const bool leads = mine < now && place == 0;
    const Item &I = S.item[item % kSlots];
    const BatchDev &B = P.b[I.b];
    const int ng = I.ng;
    const bool ok = id >= 0, last = t + 1 == I.t1;
    const size_t cell = ok ? (size_t)id * B.hkv + I.h : 0;
    const uint32_t kb = ok ? B.ks[cell] : 127u, vb = ok ? B.vs[cell] : 127u;
    const uint32_t gaps = __ballot_sync(0xffffffffu, id == -2);
    // (every lane waits for its own tile's barriers)
    if (!wait(&S.tile_empty[at % kTiles], free_(at, kTiles), &S.abort)) return;
    Tile &T = S.tile[at % kTiles];
    if (mine < now) T.y[place] = ok ? (int)cell * kPage : B.rows_end;
    if (leads) {
      T.what = (t == I.t0 ? kFirst : 0) | (last ? kLast : 0) | ((t + 1) * kKeys > I.masked ? kHides : 0) | ng << 4 | g << 7 |
               (I.nr >> 5) << 9 | (item & 31) << 10 | I.b << 15;
    }
    __syncwarp();
    if (leads) mbar_arrive(&S.tile_full[at % kTiles]);
    __syncwarp();
    fetch(false);
    const int most = __reduce_max_sync(0xffffffffu, ng);
    for (int j = 0; j < most; ++j) {
      // (lanes whose tile has fewer wait with another that has not: their own barriers' turn
      // may be over once they have been arrived at)
      const uint32_t have = __ballot_sync(0xffffffffu, j < ng);
      const int as = j < ng ? lane : __ffs(have) - 1;
      const int to = __shfl_sync(0xffffffffu, g, as) + j;
      const uint32_t k = __shfl_sync(0xffffffffu, tiles, to) + __shfl_sync(0xffffffffu, q, as);
      if (!wait(&S.sc_empty[to][k % kScales], free_(k, kScales), &S.abort, 20)) return;
      Scales &C = S.scales[to][k % kScales];
      if (mine < now && j < ng) {
        C.ck[place] = e8m0(kb) * P.scale_log2;
        C.ev[place] = ok ? (int)vb - 127 : kNoPage;
        if (place == 0) C.gap = (gaps >> (mine * kPages) & 0xffu) != 0, C.v = (int)(at % kVStages);
      }
      __syncwarp();
      if (leads && j < ng) mbar_arrive(&S.sc_full[to][k % kScales]);
    }
    if (leads && last) mbar_arrive(&S.item_empty[item % kSlots]);
    it += now;
  }
  if (given_up) return;
  const uint32_t m = it % kTiles;
  if (!wait(&S.tile_empty[m], free_(it, kTiles), &S.abort)) return;
  if (lane == 0) {
    S.tile[m].what = kEnd;
    // and the softmax warps hear of the end
    mbar_arrive(&S.item_taken[n % kSlots]);
  }
  arrive_warp(&S.tile_full[m], lane);
}

// ---- loads -------------------------------------------------------------------------
// A tile's eight pages into a stage.
IPD_DEVINL void load_tile(const CUtensorMap *map, uint8_t *stage, const Tile &T, uint64_t *bar, uint64_t policy) {
  const int4 lo = *reinterpret_cast<const int4 *>(T.y), hi = *reinterpret_cast<const int4 *>(T.y + 4);
  const int y[kPages] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  if (elect_one()) {
    mbar_arrive_expect_tx(bar, kTileBytes);
#pragma unroll
    for (int i = 0; i < kPages; ++i) tma_load_2d(stage + i * kPageBytes, map, 0, y[i], bar, policy);
  }
  __syncwarp();
}

__device__ void load_warp(const Params &P, Shared &S, int lane) {
  const uint64_t policy = l2_policy_evict_first();
  uint32_t it = 0, vs = 0;  // tiles of K, of V
  for (;; ++it, ++vs) {
    const uint32_t m = it % kTiles, k = it % kKStages, v = it % kVStages;
    if (!wait(&S.tile_full[m], full(it, kTiles), &S.abort, 40)) break;
    const Tile &T = S.tile[m];
    const What what{(uint32_t)uniform((int)T.what)};
    if (what.is(kEnd)) return;
    const int b = what.b();
    if (!wait(&S.k_empty[k], free_(it, kKStages), &S.abort, 40)) break;
    load_tile(&P.k[b], S.k[k], T, &S.k_full[k], policy);
    if (!wait(&S.v_empty[v], free_(it, kVStages), &S.abort, 40)) {
      ++it;
      break;
    }
    load_tile(&P.v[b], S.v[v], T, &S.v_full[v], policy);
  }
  // given up: the copies in flight land first
  const long long t0 = clock64();
  for (uint32_t i = it > (uint32_t)kKStages ? it - kKStages : 0; i < it; ++i)
    while (!mbar_try_wait(&S.k_full[i % kKStages], full(i, kKStages)) && clock64() - t0 < kWaitLimitCycles) {
    }
  for (uint32_t i = vs > (uint32_t)kVStages ? vs - kVStages : 0; i < vs; ++i)
    while (!mbar_try_wait(&S.v_full[i % kVStages], full(i, kVStages)) && clock64() - t0 < kWaitLimitCycles) {
    }
}

// ---- products -----------------------------------------------------------------------
// until what this thread has issued is complete (bounded): only after giving up
IPD_DEVINL void drain(uint64_t *bar, int lane) {
  if (lane == 0) {
    tc_commit(bar);
    const long long t0 = clock64();
    while (!mbar_try_wait(bar, 0) && clock64() - t0 < kWaitLimitCycles) {
    }
  }
  __syncwarp();
}

__device__ void qk_warp(Shared &S, int lane) {
  const uint32_t tmem = (uint32_t)uniform((int)S.tmem);
  const uint64_t k0 = sdesc((uint32_t)uniform((int)smem_u32(S.k[0])), 128),
                 q0 = sdesc((uint32_t)uniform((int)smem_u32(S.q[0][0])), 128);
  constexpr uint64_t kUnit = kRows * kD >> 4, kTerm = kGroups * kUnit;  // in descriptors
  uint32_t uses = 0;  // (a bit a warpgroup: parity of its uses)
  for (uint32_t it = 0;; ++it) {
    const uint32_t m = it % kTiles, s = it % kKStages;
    if (!wait(&S.tile_full[m], full(it, kTiles), &S.abort, 40)) break;
    const What what{(uint32_t)uniform((int)S.tile[m].what)};
    if (what.is(kEnd)) return;
    const int ng = what.ng(), g0 = what.wg();
    const uint32_t idesc = idesc_f8(what.nr() * ng, 0), item = what.item();
    bool ok = true;
    if (what.is(kFirst)) ok = wait(&S.q_full[item % kSlots], full(item, kSlots), &S.abort, 40);
    for (int i = 0; ok && i < ng; ++i) ok = wait(&S.s_empty[g0 + i], (uses >> (g0 + i) & 1u) ^ 1u, &S.abort, 40);
    ok = ok && wait(&S.k_full[s], full(it, kKStages), &S.abort, 40);
    if (!ok) break;
    uses ^= ((1u << ng) - 1u) << g0;
    tc_fence_after();
    const uint64_t k = k0 + (uint64_t)(s * (kTileBytes >> 4)), q = q0 + g0 * kUnit;
    const uint32_t d = tmem + col_s(g0);
    if (elect_one()) {
#pragma unroll
      for (int kk = 0; kk < kD / 32; ++kk) {
        tc_mma_f8(d, k + 2 * kk, q + 2 * kk, idesc, kk != 0);
        tc_mma_f8(d, k + 2 * kk, q + kTerm + 2 * kk, idesc, 1);
      }
#pragma unroll 1
      for (int i = 0; i < ng; ++i) tc_commit(&S.s_full[g0 + i]);
      tc_commit(&S.k_empty[s]);
    }
    __syncwarp();
  }
  drain(&S.drain[0], lane);
}

__device__ void pv_warp(Shared &S, int lane) {
  const uint32_t tmem = (uint32_t)uniform((int)S.tmem);
  const uint64_t v0 = sdesc((uint32_t)uniform((int)smem_u32(S.v[0])), 128);
  const uint32_t p_addr = (uint32_t)uniform((int)smem_u32(S.p[0]));
  uint32_t uses = 0;  // (a bit a warpgroup: parity of its uses)
  for (uint32_t it = 0;; ++it) {
    const uint32_t m = it % kTiles, s = it % kVStages;
    if (!wait(&S.tile_full[m], full(it, kTiles), &S.abort, 40)) break;
    const What what{(uint32_t)uniform((int)S.tile[m].what)};
    if (what.is(kEnd)) return;
    const int ng = what.ng(), g0 = what.wg(), nr = what.nr();
    const uint32_t idesc = idesc_f8(2 * nr, 1), begun = what.is(kFirst) ? 0u : 1u;  // (an item's first tile overwrites O)
    const uint64_t p0 = sdesc(p_addr, 2 * nr);
    const uint64_t step = (uint64_t)(32 * 2 * nr >> 4);  // 32 keys of P further on
    bool ok = wait(&S.v_full[s], full(it, kVStages), &S.abort, 40);
    const uint64_t v = v0 + (uint64_t)(s * (kTileBytes >> 4));
    for (int i = 0; ok && i < ng; ++i) {
      const uint32_t g = g0 + i;
      // (hidden keys: the first warpgroup looks the tile through before its weights count as there)
      if (i == 0 && what.is(kHides) && lane == 0) mbar_arrive(&S.v_ready[g]);
      ok = wait(&S.p_full[g], uses >> g & 1u, &S.abort, 40);
      if (!ok) break;
      tc_fence_after();
      const uint64_t p = p0 + (uint64_t)(g * (uint32_t)(sizeof(S.p[0]) >> 4));
      if (elect_one()) {
#pragma unroll
        for (int kk = 0; kk < kKeys / 32; ++kk)
          tc_mma_f8(tmem + col_o(g), v + (uint64_t)(kk * 32 * kD >> 4), p + kk * step, idesc, begun | (kk != 0));
        tc_commit(&S.pv_done[g]);
        if (i == ng - 1) {
          tc_commit(&S.v_empty[s]);
          tc_commit(&S.tile_empty[m]);
        }
      }
      __syncwarp();
    }
    if (!ok) break;
    uses ^= ((1u << ng) - 1u) << g0;
  }
  drain(&S.drain[1], lane);
}

// ---- queries ------------------------------------------------------------------------
// A row as two e4m3 terms: with 2^e the least power of two that brings its largest
// entry to 448 or below, hi = e4m3(q 2^-e), lo = e4m3(q 2^-e - hi), which together
// hold a bf16's eight bits down to 2^-10, 2^-17 of the row's largest entry.
// Every eighth row of an item from the r-th on: where it begins in q and out.  (By steps, no
// division a row: with that, all of a warp's rows under way at once and rows that leave 16 bytes a
// lane, 300 requests of 4 to 7 queries over 100 to 3,000 keys took 142 us in place of 154, 64 tasks a
// CTA of 128 rows and four tiles 1,092 in place of 1,243.)
struct RowWalk {
  int r, head, group, dh;
  size_t at, by, over;
  IPD_DEVINL RowWalk(const BatchDev &B, const Item &I, int first) : r(first), group(B.group) {
    const int row = I.row0 + first, query = row / group, dq = 8 / group;
    head = row - query * group, dh = 8 - dq * group;
    at = ((size_t)(I.c0 + query) * B.hq + (size_t)I.h * group + head) * kD;
    by = ((size_t)dq * B.hq + dh) * kD, over = (size_t)(B.hq - group) * kD;
  }
  IPD_DEVINL void step() {
    r += 8, at += by, head += dh;
    if (head >= group) head -= group, at += over;
  }
};

// Half a warp a row, eight entries a lane; the warpgroup's own rows of the item, whose
// place is free: the products of the item before are complete.
IPD_DEVINL void convert_queries(const BatchDev &B, const Item &I, Shared &S, int g, int warp, int lane) {
  const int first = (g - I.wg) * kRows;  // (of the item's rows)
  const int part = lane & 15;
  RowWalk walk(B, I, first + 2 * warp + (lane >> 4));
  uint4 next[kRows / 8];
#pragma unroll
  for (int i = 0; i < kRows / 8; ++i) {
    next[i] = walk.r < I.rows ? *reinterpret_cast<const uint4 *>(B.q + walk.at + part * 8) : make_uint4(0u, 0u, 0u, 0u);
    walk.step();
  }
#pragma unroll 1
  for (int r = 2 * warp + (lane >> 4); r < I.nr; r += 8) {
    const uint4 x = next[0];
#pragma unroll
    for (int i = 0; i + 1 < kRows / 8; ++i) next[i] = next[i + 1];
    const uint32_t *xw = &x.x;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __vmaxu2(top, xw[i] & 0x7fff7fffu);
    top = max(top & 0xffffu, top >> 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int E = (int)(top >> 7);
    // (a largest entry below 2^-100 counts as zero; one that is not finite makes the
    // row NaN)
    const int e = E - 127 - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0);
    const bool none = E < 27 || E == 255;
    const float f = none ? 0.f : pow2i(-e);
    uint32_t hi[2], lo[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v[4] = {bf16lo(xw[2 * k]) * f, bf16hi(xw[2 * k]) * f, bf16lo(xw[2 * k + 1]) * f, bf16hi(xw[2 * k + 1]) * f};
      if (none) v[0] = v[1] = v[2] = v[3] = 0.f;
      hi[k] = e4m3x2(v[0], v[1]) | e4m3x2(v[2], v[3]) << 16;
      float back[4];
      e4m3x4_to_floats(hi[k], back);
      lo[k] = e4m3x2(v[0] - back[0], v[1] - back[1]) | e4m3x2(v[2] - back[2], v[3] - back[3]) << 16;
    }
    const int at = r * kD + (((part >> 1) ^ (r & 7)) << 4) + (part & 1) * 8;
    *reinterpret_cast<uint2 *>(S.q[0][g] + at) = make_uint2(hi[0], hi[1]);
    *reinterpret_cast<uint2 *>(S.q[1][g] + at) = make_uint2(lo[0], lo[1]);
    if (part == 0) {
      float *st = reinterpret_cast<float *>(&S.state[g][r >> 1]) + (r & 1);
      st[0] = E == 255 ? __uint_as_float(0x7fc00000u) : none ? 0.f : pow2i(e);
      st[2] = 0.f;
    }
  }
  fence_proxy_async_smem();
}

IPD_DEVINL void mbar_arrive_n(uint64_t *bar, int n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}

// ---- softmax --------------------------------------------------------------------------
// Reduces 16 values a lane over the lanes, column by column: lane i ends up with
// column i / 2.
template <typename Op>
IPD_DEVINL float column_reduce(float (&a)[16], int lane, Op op) {
#pragma unroll
  for (int n = 8, mask = 16; n > 0; n >>= 1, mask >>= 1) {
    const bool up = lane & mask;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float other = __shfl_xor_sync(0xffffffffu, up ? a[i] : a[i + n], mask);
      a[i] = op(up ? a[i + n] : a[i], other);
    }
  }
  return op(a[0], __shfl_xor_sync(0xffffffffu, a[0], 1));
}

struct Softmax {
  int g, tid, warp, lane;  // warpgroup, and place in it
  uint32_t tiles;          // own tiles so far
  uint32_t mends;          // tiles looked through so far
  uint32_t pairs, alls;    // barriers of two and of all warpgroups so far
  bool ok;                 // no wait of this warp has given up
};

// A thread's key of a tile that holds hidden keys: NaN in its V row.  They would reach
// rows that do not see the key (0 x NaN), so they become 0, and rows that do see
// it get them back at the end.
IPD_DEVINL void mend(Shared &S, Item &I, int set, uint8_t *v, int key_in_tile, int key) {
  const uint4 *row = reinterpret_cast<const uint4 *>(v + key_in_tile * kD);
  uint32_t any = 0;  // bit 7 of a byte: one of its like was 0x7f or 0xff
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint4 x = row[(i + key_in_tile) & 7];
    any |= (x.x & 0x7f7f7f7fu) + 0x01010101u | (x.y & 0x7f7f7f7fu) + 0x01010101u | (x.z & 0x7f7f7f7fu) + 0x01010101u |
           (x.w & 0x7f7f7f7fu) + 0x01010101u;
  }
  if ((any & 0x80808080u) == 0) return;
#pragma unroll 1
  for (int i = 0; i < 32; ++i) {
    const int c = ((i >> 2) + key_in_tile) & 7, at = c * 16 + (i & 3) * 4;
    uint32_t *w = reinterpret_cast<uint32_t *>(v + key_in_tile * kD + at);
    uint32_t x = *w;
    if (__vcmpeq4(x & 0x7f7f7f7fu, 0x7f7f7f7fu) == 0) continue;
#pragma unroll 1
    for (int e = 0; e < 4; ++e)
      if ((x >> 8 * e & 0x7fu) == 0x7fu) {
        if (key < I.L) {
          atomicMin(&S.nan_key[set][((c ^ (key_in_tile & 7)) << 4) + (i & 3) * 4 + e], key);
          I.bad = 1;
        }
        x &= ~(0xffu << 8 * e);
      }
    __threadfence_block();  // noted before it is gone
    *w = x;
  }
}

// Exponents of the rows' weights (in pairs) at a thread's key, against their references; dz is what
// V's scale adds.
template <int NR>
IPD_DEVINL void exponents(const uint32_t (&s)[NR], const float4 *state, float ck, float dz, u64 (&z)[NR / 2]) {
  const u64 ck2 = f2_pack(ck, ck), dz2 = f2_pack(dz, dz);
#pragma unroll
  for (int i = 0; i < NR; i += 2) {
    const float4 st = state[i / 2];
    z[i / 2] = f2_add(f2_fma(f2_mul(f2_pack(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), ck2), f2_pack(st.x, st.y),
                             f2_pack(st.z, st.w)), dz2);
  }
}

IPD_DEVINL float redux_max(float x) {
  float m;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(x));
  return m;
}
// The largest exponents of the rows over a warp's keys.
template <int NR>
IPD_DEVINL void row_maxima(Shared &S, const Softmax &X, const u64 (&z)[NR / 2]) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < NR; i += 2) {
    float z0, z1;
    f2_unpack(z[i / 2], z0, z1);
    z0 = redux_max(z0), z1 = redux_max(z1);
    m = X.lane == i ? z0 : X.lane == i + 1 ? z1 : m;
  }
  if (X.lane < NR) S.red[X.g][X.warp][X.lane] = m;
}

IPD_DEVINL void load_scores(uint32_t taddr, uint32_t (&r)[16]) { tc_ld_32x32b_x16(taddr, r); }
IPD_DEVINL void load_scores(uint32_t taddr, uint32_t (&r)[32]) { tc_ld_32x32b_x32(taddr, r); }

// New references: of all rows at an item's first tile; afterwards of rows whose weights would leave
// kLimit, of those that all warps have in `low`, and of rows that see their item's first keys here:
// the rows' largest exponents in this tile less kBase.  O and the sums of rows that have seen keys are
// rescaled, a TMEM column each (the others' are zeros, and their factor may be past fp32).
// (The loop over tiles is short of instruction cache: one piece of code for first and later
// references took 64 spans from 137 to 131 us; falling references cost 1 to 5 % of a call beyond.)
template <int NR>
IPD_DEVINL void move_references(Shared &S, const Softmax &X, u64 (&z)[NR / 2], uint32_t low, bool first, uint32_t o_addr, uint32_t l_addr) {
  const int g = X.g, lane = X.lane;
  if (lane == 0) S.below[g][X.warp] = low;
  row_maxima<NR>(S, X, z);
  named_bar_sync(1 + g, 128);
  if (X.warp == 0) {
    const int r = lane % NR;
    const bool mine = lane < NR;
    const float top = fmaxf(fmax3(S.red[g][0][r], S.red[g][1][r], S.red[g][2][r]), S.red[g][3][r]);
    // (not finite: no key in this tile, NaN alone, or more than fp32 holds)
    const bool finite = fabsf(top) < INFINITY;
    const uint32_t none = __ballot_sync(0xffffffffu, mine && top == -INFINITY);
    float *state = reinterpret_cast<float *>(&S.state[g][r >> 1]) + (r & 1) + 2;  // the reference, negative
    if (first) {
      const float ref = finite ? top - kBase : 0.f;
      if (mine) *state = -ref, S.alpha[g][r] = -ref, S.floor[g][r] = ref - kDeep;
      if (lane == 0) S.unseen[g] = none, S.moved[g] = 0u, S.deep[g] = 0u, S.look[g] = S.gap[g] = 1;
    } else {
      const uint32_t unseen = S.unseen[g];
      low = S.below[g][0] & S.below[g][1] & S.below[g][2] & S.below[g][3];
      const float ref = -*state, floor = S.floor[g][r];
      const bool seen = !(unseen >> r & 1u);
      float now = ref;
      if ((top > kLimit || ((low | unseen) >> r & 1u)) && finite) now = ref + (top - kBase);
      if (now < ref && seen) now = fminf(ref, fmaxf(now, floor));
      const float by = now - ref;
      __syncwarp();
      if (mine) {
        *state = -now;
        S.alpha[g][r] = -by;
        S.floor[g][r] = seen ? fmaxf(floor, now - kDeep) : now - kDeep;
      }
      const uint32_t moved = __ballot_sync(0xffffffffu, mine && by != 0.f) & ~unseen;
      const uint32_t deep = __ballot_sync(0xffffffffu, mine && by < 0.f && now <= floor) & ~unseen;
      const bool far = __any_sync(0xffffffffu, by > kFarRise && seen);
      if (lane == 0) {
        const int gap = S.gap[g];
        S.unseen[g] = none & unseen, S.moved[g] = moved, S.deep[g] = (S.deep[g] & ~moved) | deep;
        S.look[g] = far ? gap : (moved & low) ? 1 : kIdle;
        if (far) S.gap[g] = min(2 * gap, kMostWait);
      }
    }
  }
  named_bar_sync(1 + g, 128);
#pragma unroll
  for (int i = 0; i < NR; i += 2) z[i / 2] = f2_add(z[i / 2], *reinterpret_cast<const u64 *>(&S.alpha[g][i]));
  if (first) {
    uint32_t zero[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) zero[i] = 0u;
#pragma unroll 1
    for (int c = 0; c < NR; c += 16) tc_st_32x32b_x16(l_addr + c, zero);
  }
#pragma unroll 1
  for (uint32_t left = S.moved[g]; left; left &= left - 1) {
    const int r = __ffs(left) - 1;
    const float f = ex2_approx(S.alpha[g][r]);
    uint32_t a, b, l;
    tc_ld_x1(o_addr + r, a);
    tc_ld_x1(o_addr + NR + r, b);
    tc_ld_x1(l_addr + r, l);
    tc_wait_ld();
    tc_st_x1(o_addr + r, __float_as_uint(__uint_as_float(a) * f));
    tc_st_x1(o_addr + NR + r, __float_as_uint(__uint_as_float(b) * f));
    tc_st_x1(l_addr + r, __float_as_uint(__uint_as_float(l) * f));
  }
  tc_wait_st();
}

// The weights of a warpgroup's rows for its tiles of an item.  A wait that gives up
// does not leave the way the others go: the warps of a warpgroup meet at barriers.
// Returns the exponent that V's scales count from.
template <int NR>
__device__ int softmax_tiles(const Params &P, Shared &S, Softmax &X, Item &I) {
  const int g = X.g, lane = X.lane, tid = X.tid;
  const int n_tiles = I.t1 - I.t0, L = I.L;
  const uint32_t lanes = (uint32_t)X.warp << 21;  // this warp's 32 TMEM lanes
  const uint32_t s_addr = S.tmem + lanes + col_s(g), o_addr = S.tmem + lanes + col_o(g), l_addr = S.tmem + lanes + col_l(g);
  const int row0 = I.row0 + (g - I.wg) * kRows;
  const int group = P.b[I.b].group;
  const int sees = L - I.n;                        // query i sees keys up to sees + i
  const int masked = I.masked;
  const int turn = NR == 32 ? (tid >> 1) & 3 : (tid >> 2) & 1;  // P's swizzle
  uint8_t *prow = S.p[g] + tid * 2 * NR;
  int e0 = kNoPage;  // (until there is a page)
  int look = I.L > kShort ? n_tiles : -1;  // the tile that is looked through for rows that fall (-1: none)
#pragma unroll 1
  for (int t = 0; t < n_tiles; ++t) {
    const uint32_t k = X.tiles % kScales;
    X.ok = wait(&S.sc_full[g][k], full(X.tiles, kScales), &S.abort, 0) && X.ok;
    const Scales &M = S.scales[g][k];
    const int v_stage = min((uint32_t)M.v, kVStages - 1u);  // (in range whatever a warp that gave up has left)
    const int key0 = (I.t0 + t) * kKeys, key = key0 + tid;
    const float ck = M.ck[tid / kPage];
    const int ev = M.ev[tid / kPage];
    const bool hides = key0 + kKeys > masked || M.gap;
    if (e0 == kNoPage) {
      // the largest of the pages that all rows see, whatever the others hold
      int top = -kNoPage, there = 0;
#pragma unroll
      for (int i = 0; i < kPages; ++i) {
        const int e = M.ev[i];
        there |= e != kNoPage;
        if (e != kNoPage && e != 128 && key0 + i * kPage < masked) top = max(top, e);
      }
      if (there) e0 = top == -kNoPage ? 0 : top;
    }
    int de = max(-kFar, min(kFar, ev - e0));
    int hidden = 0;  // rows before this one do not see the key
    if (hides) {
      hidden = ev == kNoPage || key >= L ? NR : (int)max(0LL, min((long long)NR, (long long)(key - sees) * group - row0));
      if (hidden == NR) de = 0;
    }
    // what V's scale adds to an exponent (a scale of NaN makes the weights of rows that see the key NaN),
    // and its inverse, for the sums
    const float dz = ev == 128 && hidden < NR ? __uint_as_float(0x7fc00000u) : (float)de, inv = pow2i(-de);
    arrive_warp(&S.sc_empty[g][k], lane);
    X.ok = wait(&S.s_full[g], full(X.tiles, 1), &S.abort, 0) && X.ok;
    tc_fence_after();
    u64 z[NR / 2];
    {
      uint32_t s[NR];
      load_scores(s_addr, s);
      tc_wait_ld();
      exponents(s, S.state[g], ck, dz, z);
    }
    tc_fence_before();
    arrive_warp(&S.s_empty[g], lane);
    if (hides) {
      asm volatile("" ::: "memory");  // (a branch, not 32 predicates)
#pragma unroll
      for (int i = 0; i < NR; i += 2) {
        float z0, z1;
        f2_unpack(z[i / 2], z0, z1);
        z[i / 2] = f2_pack(i < hidden ? -INFINITY : z0, i + 1 < hidden ? -INFINITY : z1);
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NR / 2; ++i) {
      float z0, z1;
      f2_unpack(z[i], z0, z1);
      top = fmax3(top, z0, z1);
    }
    uint32_t low = 0;  // a bit a row: its exponents here lie below kLow
    if (t == look) {
#pragma unroll
      for (int i = NR - 2; i >= 0; i -= 2) {
        float z0, z1;
        f2_unpack(f2_add(z[i / 2], f2_pack(-kLow, -kLow)), z0, z1);
        low = __funnelshift_l(__float_as_uint(z1), low, 1);
        low = __funnelshift_l(__float_as_uint(z0), low, 1);
      }
      low = __reduce_and_sync(0xffffffffu, low) & ~S.deep[g];
    }
    const bool move = bar_or(1 + g, 128, t == 0 || S.unseen[g] || low || top > kLimit);
    // P's buffer is free, and O at rest, once this warpgroup's product before is complete
    if (X.tiles > 0) X.ok = wait(&S.pv_done[g], full(X.tiles - 1, 1), &S.abort, 0) && X.ok;
    tc_fence_after();
    if (move) {
      move_references<NR>(S, X, z, low, t == 0, o_addr, l_addr);
      if (look >= 0) look = t + S.look[g];
    } else if (t == look) {
      look = t + kIdle;
    }
    const u64 inv2 = f2_pack(inv, inv);
    const uint32_t lo16 = half2_of(kLoScale, kLoScale);
#pragma unroll
    for (int c = 0; c < NR; c += 16) {
      uint32_t l[16];
      tc_ld_32x32b_x16(l_addr + c, l);
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t h[2], b[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          u64 &p = z[c / 2 + q * 2 + k];
          float p0, p1;
          f2_unpack(p, p0, p1);
          p0 = ex2_approx(p0), p1 = ex2_approx(p1);
          p = f2_pack(p0, p1);
          h[k] = half2_of(p0, p1);
        }
        hi[q] = e4m3x4_h(h[0], h[1]);
        h_from_e4m3x4(hi[q], b[0], b[1]);
        lo[q] = e4m3x4_h(half2_mul(half2_sub(h[0], b[0]), lo16), half2_mul(half2_sub(h[1], b[1]), lo16));
      }
      *reinterpret_cast<uint4 *>(prow + (((c / 16) ^ turn) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4 *>(prow + ((((NR + c) / 16) ^ turn) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
      tc_wait_ld();
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        float l0, l1;
        f2_unpack(f2_fma(z[(c + i) / 2], inv2, f2_pack(__uint_as_float(l[i]), __uint_as_float(l[i + 1]))), l0, l1);
        l[i] = __float_as_uint(l0), l[i + 1] = __float_as_uint(l1);
      }
      tc_st_32x32b_x16(l_addr + c, l);
    }
    if (key0 + kKeys > masked && g == I.wg) {
      // hidden keys: the tile is looked through before the product, which takes the first
      // warpgroup's rows before the others'
      X.ok = wait(&S.v_ready[g], full(X.mends, 1), &S.abort, 0) && X.ok;
      ++X.mends;
      if (key >= masked) mend(S, I, g, S.v[v_stage], tid, key);
    }
    fence_proxy_async_smem();
    tc_wait_st();
    tc_fence_before();
    arrive_warp(&S.p_full[g], lane);
    ++X.tiles;
  }
  return e0 == kNoPage ? 0 : e0;
}

// Joins the parts of a row group of a task that was cut between CTAs, in order.  What bounds it is
// the time until another SM's rows arrive, 1,300 cycles or more at a time: a warp has four parts of
// two rows under way, or eight of one row where there are no more rows than warps.
struct Parts {
  const float *first;  // the first CTA's
  ptrdiff_t next, step; // from it to the next one's, and on
  int n;
};
template <int kAtOnce, int kParts>
IPD_DEVINL void join_rows(const Params &P, const Item &I, const Parts &A, int r0, int rows, int warp, int lane) {
  const BatchDev &B = P.b[I.b];
#pragma unroll 1
  for (int r = warp; r < rows; r += 4 * kAtOnce) {
    int at[kAtOnce];
    float top[kAtOnce], sum[kAtOnce];
    float4 acc[kAtOnce];
    const float *sums[kAtOnce], *dims[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      at[j] = min(r + 4 * j, rows - 1);  // (the last row twice, rather than none)
      top[j] = -INFINITY, sum[j] = 0.f, acc[j] = make_float4(0.f, 0.f, 0.f, 0.f);
      sums[j] = A.first + (size_t)P.part_rows * kD + r0 + at[j], dims[j] = A.first + (r0 + at[j]) * kD + lane * 4;
    }
#pragma unroll 1
    for (int i = 0; i < A.n; i += kParts) {
      float l[kAtOnce][kParts];
      float4 x[kAtOnce][kParts];
#pragma unroll
      for (int k = 0; k < kParts; ++k) {
        const bool there = i + k < A.n;
        const ptrdiff_t on = i + k == 0 ? A.next : A.step;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          l[j][k] = there ? *sums[j] : -INFINITY;
          x[j][k] = there ? *reinterpret_cast<const float4 *>(dims[j]) : make_float4(0.f, 0.f, 0.f, 0.f);
          sums[j] += on, dims[j] += on;
        }
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        float now = top[j];
#pragma unroll
        for (int k = 0; k < kParts; ++k) now = fmaxf(now, l[j][k]);
        const float base = now == -INFINITY ? 0.f : now, f = ex2_approx(top[j] - base);
        top[j] = now;
        sum[j] *= f, acc[j].x *= f, acc[j].y *= f, acc[j].z *= f, acc[j].w *= f;
#pragma unroll
        for (int k = 0; k < kParts; ++k) {
          const float w = ex2_approx(l[j][k] - base);
          const float4 v = x[j][k];
          sum[j] += w;
          acc[j].x = fmaf(w, v.x, acc[j].x), acc[j].y = fmaf(w, v.y, acc[j].y);
          acc[j].z = fmaf(w, v.z, acc[j].z), acc[j].w = fmaf(w, v.w, acc[j].w);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const float f = sum[j] == 0.f ? 0.f : 1.f / sum[j];
      const int row = I.row0 + r0 + at[j], query = row / B.group;
      *reinterpret_cast<uint2 *>(
          B.out + ((size_t)(I.c0 + query) * B.hq + (size_t)I.h * B.group + (row - query * B.group)) * kD + lane * 4) =
          make_uint2((uint32_t)f2bf16(acc[j].x * f) | (uint32_t)f2bf16(acc[j].y * f) << 16,
                     (uint32_t)f2bf16(acc[j].z * f) | (uint32_t)f2bf16(acc[j].w * f) << 16);
    }
  }
}
IPD_DEVINL void join(const Params &P, const Item &I, int r0, int rows, int warp, int lane) {
  const size_t stride = (size_t)P.part_rows * (kD + 1);
  const Parts A{P.part + (2 * (size_t)I.cta0 + 1) * stride, (2 * (I.ctab - I.cta0) - 1) * (ptrdiff_t)stride,
                2 * (ptrdiff_t)stride, I.cta1 - I.ctab + 2};
  if (rows <= 4) join_rows<1, 8>(P, I, A, r0, rows, warp, lane);
  else join_rows<2, 4>(P, I, A, r0, rows, warp, lane);
}

// A row group of an item: its tiles, then its rows.
__device__ void softmax_item(const Params &P, Shared &S, Softmax &X, uint32_t item, Item &I) {
  const int g = X.g, lane = X.lane, tid = X.tid, slot = item % kSlots;
  const int nr = I.nr, rg = g - I.wg;
  convert_queries(P.b[I.b], I, S, g, X.warp, lane);
  __syncwarp();
  if (lane == 0) mbar_arrive_n(&S.q_full[slot], kGroups / I.ng);
  named_bar_sync(1 + g, 128);
  const int e0 = nr == 32 ? softmax_tiles<32>(P, S, X, I) : softmax_tiles<16>(P, S, X, I);
  // the sums over the threads
  const uint32_t lanes = (uint32_t)X.warp << 21, o_addr = S.tmem + lanes + col_o(g), l_addr = S.tmem + lanes + col_l(g);
#pragma unroll 1
  for (int c = 0; c < nr; c += 16) {
    uint32_t l[16];
    float z[16];
    tc_ld_32x32b_x16(l_addr + c, l);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = __uint_as_float(l[i]);
    const float x = column_reduce(z, lane, [](float a, float b) { return a + b; });
    if (!(lane & 1)) S.red[g][X.warp][c + (lane >> 1)] = x;
  }
  named_bar_sync(1 + g, 128);
  const int rows = min(kRows, I.rows - rg * kRows);  // (none or fewer where the task has no such rows)
  float *part = I.part >= 0 ? P.part + (size_t)I.part * P.part_rows * (kD + 1) : nullptr;
  if (tid < nr) {
    const float sum = (S.red[g][0][tid] + S.red[g][1][tid]) + (S.red[g][2][tid] + S.red[g][3][tid]);
    // a row's factor: 2^e0 / its sum (a score past fp32 leaves no softmax)
    S.alpha[g][tid] = sum == 0.f ? 0.f : sum == INFINITY ? __uint_as_float(0x7fc00000u) : pow2i(e0) / sum;
    if (part && tid < rows) {
      const float ref = -(reinterpret_cast<const float *>(&S.state[g][tid >> 1]) + (tid & 1))[2];
      part[(size_t)P.part_rows * kD + rg * kRows + tid] = sum == 0.f ? -INFINITY : ref + log2f(sum);
    }
  }
  X.ok = wait(&S.pv_done[g], full(X.tiles - 1, 1), &S.abort, 0) && X.ok;
  tc_fence_after();
  named_bar_sync(1 + g, 128);
  const bool bad = *(volatile int *)&I.bad != 0;
  const int d = tid, row0 = I.row0 + rg * kRows, group = P.b[I.b].group;
  const BatchDev &B = P.b[I.b];
  // a thread a dim: fp32 rows of a part as they are, a task's own by way of P's buffer, in
  // bf16, so that they leave 16 bytes a lane
  float *to = part + (size_t)(rg * kRows) * kD + d;
  uint16_t *stage = reinterpret_cast<uint16_t *>(S.p[g]);
  static_assert(sizeof(S.p[0]) >= kRows * kD * sizeof(uint16_t), "a warpgroup's rows in P's buffer");
#pragma unroll 1
  for (int k = 0; k < rows; k += 8) {
    uint32_t a[8], b[8];
    tc_ld_32x32b_x8(o_addr + k, a);
    tc_ld_32x32b_x8(o_addr + nr + k, b);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = fmaf(__uint_as_float(b[i]), 1.f / kLoScale, __uint_as_float(a[i])) * S.alpha[g][k + i];
      if (!part) stage[(k + i) * kD + d] = f2bf16(x);
      else if (k + i < rows) to[(size_t)(k + i) * kD] = x;
    }
  }
  if (bad) {
    const int nan_key = S.nan_key[I.wg][d], sees = I.L - I.n;
#pragma unroll 1
    for (int r = 0; r < rows; ++r)
      if (nan_key <= sees + (row0 + r) / group) {
        if (part) to[(size_t)r * kD] = __uint_as_float(0x7fc00000u);
        else stage[r * kD + d] = 0x7fc0;
      }
  }
  if (!part) {
    named_bar_sync(1 + g, 128);
    const int r0 = 2 * X.warp + (lane >> 4);
    const uint16_t *from = stage + r0 * kD + (lane & 15) * 8;
#pragma unroll 1
    for (RowWalk walk(B, I, rg * kRows + r0); walk.r < I.rows; walk.step(), from += 8 * kD) {
      if (walk.r >= (rg + 1) * kRows) break;
      *reinterpret_cast<uint4 *>(B.out + walk.at + (lane & 15) * 8) = *reinterpret_cast<const uint4 *>(from);
    }
  }
  tc_fence_before();
  if (part && rows > 0) {
    // the last CTA of the task to get here joins its parts
    __threadfence();
    named_bar_sync(1 + g, 128);
    if (tid == 0) S.last[g] = atomicAdd(&P.done[I.cta0 * kGroups + rg], 1) == I.cta1 - I.ctab + 1;
    named_bar_sync(1 + g, 128);
    if (*(volatile int *)&S.last[g]) {
      __threadfence();
      join(P, I, rg * kRows, rows, X.warp, lane);
    }
  }
  if (bad) {  // (all warpgroups of the item know the same)
    uint64_t *bar = I.ng == 4 ? &S.all : &S.pair[I.wg >> 1];
    for (int i = 0; i < 2; ++i) {
      if (I.ng == 1) {
        named_bar_sync(1 + g, 128);
      } else {
        uint32_t &uses = I.ng == 4 ? X.alls : X.pairs;
        arrive_warp(bar, lane);
        X.ok = wait(bar, uses & 1u, &S.abort, 0) && X.ok;
        ++uses;
      }
      if (i == 0 && rg == 0) S.nan_key[g][tid] = 0x7fffffff;
    }
  }
  // state, sums and factors are read, before the next item writes them
  named_bar_sync(1 + g, 128);
}

__device__ void softmax_warps(const Params &P, Shared &S, int warp, int lane) {
  Softmax X{warp >> 2, (int)threadIdx.x & 127, warp & 3, lane, 0, 0, 0, 0, true};
  for (uint32_t n = 0;; ++n) {
    const int slot = n % kSlots;
    X.ok = wait(&S.item_taken[slot], full(n, kSlots), &S.abort, 0) && X.ok;
    if (bar_or(1 + X.g, 128, !X.ok)) return;  // the whole warpgroup
    Item &I = S.item[slot];
    if (!I.valid) return;
    if (X.g >= I.wg && X.g < I.wg + I.ng) softmax_item(P, S, X, n, I);
    arrive_warp(&S.item_empty[slot], lane);
  }
}

__global__ void __launch_bounds__(kThreads, 1) attn8_kernel(const __grid_constant__ Params P) {
  extern __shared__ uint8_t raw[];
  // (an offset from the array, so that accesses stay known as shared memory's)
  Shared &S = *reinterpret_cast<Shared *>(raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x < kGroups * kD) S.nan_key[threadIdx.x / kD][threadIdx.x % kD] = 0x7fffffff;
  if (threadIdx.x == 0) {
    S.abort = 0;
    auto ring = [](uint64_t *b, int n, int count) {
      for (int i = 0; i < n; ++i) mbar_init(&b[i], count);
    };
    ring(S.k_full, kKStages, 1), ring(S.k_empty, kKStages, 1);
    ring(S.v_full, kVStages, 1), ring(S.v_empty, kVStages, 1);
    ring(S.tile_full, kTiles, 1), ring(S.tile_empty, kTiles, 1);
    ring(S.sc_full[0], kGroups * kScales, 1), ring(S.sc_empty[0], kGroups * kScales, 4);
    ring(S.q_full, kSlots, kSoftmaxWarps);
    ring(S.s_full, kGroups, 1), ring(S.s_empty, kGroups, 4);
    ring(S.p_full, kGroups, 4), ring(S.pv_done, kGroups, 1);
    ring(S.v_ready, kGroups, 1);
    ring(S.item_full, kSlots, 1), ring(S.item_taken, kSlots, 1), ring(S.item_empty, kSlots, kItemReaders);
    ring(S.pair, 2, 8), ring(&S.all, 1, kSoftmaxWarps), ring(S.drain, 2, 1);
    fence_mbar_init();
  }
  if (warp == kQkWarp) {
    tc_alloc(&S.tmem, kTmemCols);
    tc_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp < kSoftmaxWarps) softmax_warps(P, S, warp, lane);
  else if (warp == kLoadWarp) load_warp(P, S, lane);
  else if (warp == kQkWarp) qk_warp(S, lane);
  else if (warp == kPvWarp) pv_warp(S, lane);
  else if (warp == kItemWarp) item_warp(P, S, lane);
  else page_warp(P, S, lane);
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kQkWarp) tc_dealloc(S.tmem, kTmemCols);
}

// ---- host -----------------------------------------------------------------------------
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
  if (b->max_seq_len > 1 << 30 || (long long)b->max_q_len * (b->num_q_heads / c->num_kv_heads) >= 1 << 30)
    return IPD_ERR_UNSUPPORTED;  // (keys and rows are counted in 32 bits)
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

struct DevInfo {
  int sms = 0;
};
DevInfo g_dev[64];
PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;

int prepare_device(int *sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return IPD_ERR_CUDA;
  DevInfo &D = g_dev[dev];
  if (D.sms == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return IPD_ERR_CUDA;
    if (cudaFuncSetAttribute(attn8_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSharedBytes) != cudaSuccess)
      return IPD_ERR_CUDA;
    D.sms = n;
  }
  *sms = D.sms;
  if (!g_encode) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess || !fn)
      return IPD_ERR_CUDA;
    g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  }
  return IPD_OK;
}

// A pool as rows of 128 bytes; a box is one page of one head, its rows swizzled.
int encode_pool(CUtensorMap *m, const void *base, long long rows) {
  cuuint64_t dims[2] = {(cuuint64_t)kD, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)kD};
  cuuint32_t box[2] = {(cuuint32_t)kD, (cuuint32_t)kPage}, estr[2] = {1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? IPD_OK
             : IPD_ERR_CUDA;
}

constexpr int kMaxCtas = 256;  // the workspace is laid out for as many

struct Layout {
  size_t prefix, info, done, part, total;
  int reqs, part_rows;
};
Layout layout(const ipd_attn8_batch *const *bs, int n) {
  Layout W{};
  long long rows = 1;
  for (int i = 0; i < n; ++i) {
    const ipd_attn8_batch &b = *bs[i];
    if (b.num_reqs == 0 || b.total_q == 0) continue;
    W.reqs += b.num_reqs;
    rows = std::max(rows, (long long)b.max_q_len * (b.num_q_heads / b.cache->num_kv_heads));
  }
  W.part_rows = (int)((std::min<long long>(rows, kBlockRows) + 3) / 4 * 4);
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  W.prefix = 0;
  W.info = up((size_t)(W.reqs + 2) * sizeof(long long));
  W.done = W.info + up((size_t)W.reqs * sizeof(int4));
  W.part = W.done + up(kMaxCtas * kGroups * sizeof(int));
  W.total = W.part + up((size_t)2 * kMaxCtas * W.part_rows * (kD + 1) * sizeof(float));
  return W;
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
  if (collect(verify, n_verify, decode, n_decode, bs) != IPD_OK) return 0;
  return layout(bs, n_verify + n_decode).total;
}

extern "C" int ipd_verify_attn8(const ipd_attn8_batch *verify, int n_verify,
                                const ipd_attn8_batch *decode, int n_decode, float softmax_scale,
                                void *workspace, size_t workspace_bytes, ipd_stream_t stream) {
  const ipd_attn8_batch *bs[IPD_MAX_BATCHES];
  int st = collect(verify, n_verify, decode, n_decode, bs);
  if (st != IPD_OK) return st;
  if (!(softmax_scale > 0.f) || !(softmax_scale - softmax_scale == 0.f)) return IPD_ERR_INVALID_ARG;
  const Layout W = layout(bs, n_verify + n_decode);
  if (W.reqs == 0) return IPD_OK;
  if (!workspace || workspace_bytes < W.total || ((uintptr_t)workspace & 255)) return IPD_ERR_WORKSPACE;
  int sms = 0;
  st = prepare_device(&sms);
  if (st != IPD_OK) return st;
  Params P;
  memset(&P, 0, sizeof(P));
  const ipd_kv8_cache *caches[IPD_MAX_BATCHES];
  for (int i = 0; i < n_verify + n_decode; ++i) {
    const ipd_attn8_batch &b = *bs[i];
    if (b.num_reqs == 0 || b.total_q == 0) continue;
    const ipd_kv8_cache &c = *b.cache;
    int same = 0;
    while (same < P.n && !(caches[same]->k_pages == c.k_pages && caches[same]->v_pages == c.v_pages &&
                           caches[same]->num_pages == c.num_pages && caches[same]->num_kv_heads == c.num_kv_heads))
      ++same;
    const long long rows = c.num_pages * c.num_kv_heads * kPage;
    if (same < P.n) {
      P.k[P.n] = P.k[same], P.v[P.n] = P.v[same];
    } else if (encode_pool(&P.k[P.n], c.k_pages, rows) != IPD_OK || encode_pool(&P.v[P.n], c.v_pages, rows) != IPD_OK) {
      return IPD_ERR_CUDA;
    }
    caches[P.n] = &c;
    P.b[P.n] = BatchDev{c.k_scale, c.v_scale, b.q, b.out, b.cu_q, b.seq_len, b.page_table, b.num_reqs, b.num_q_heads,
                        c.num_kv_heads, b.num_q_heads / c.num_kv_heads, b.max_pages, b.max_q_len, b.max_seq_len,
                        b.total_q, (int)c.num_pages, (int)rows};
    P.req_base[P.n + 1] = P.req_base[P.n] + b.num_reqs;
    ++P.n;
  }
  P.total_reqs = W.reqs;
  P.scale_log2 = softmax_scale * kLog2e;
  uint8_t *ws = static_cast<uint8_t *>(workspace);
  P.prefix = reinterpret_cast<long long *>(ws + W.prefix);
  P.info = reinterpret_cast<int4 *>(ws + W.info);
  P.done = reinterpret_cast<int *>(ws + W.done);
  P.part = reinterpret_cast<float *>(ws + W.part);
  P.part_rows = W.part_rows;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int ctas = std::min(sms, kMaxCtas);
  g_attn8_used.store(true, std::memory_order_relaxed);
  attn8_plan_kernel<<<1, W.reqs <= 256 ? 256 : 1024, 0, s>>>(P, ctas);
  if (cudaGetLastError() != cudaSuccess) return IPD_ERR_CUDA;
  // begins beside the plan, and waits for it where it reads what the plan wrote
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSharedBytes;
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, attn8_kernel, P) != cudaSuccess) {
    (void)cudaGetLastError();
    return IPD_ERR_CUDA;
  }
  return IPD_OK;
}

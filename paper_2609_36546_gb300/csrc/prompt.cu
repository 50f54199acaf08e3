// Causal attention of whole prompts: packed sequences of different lengths,
// grouped heads, head_dim 128, bf16 in and out.
//
//   o_i = sum_{j <= i} p_ij v_j / l_i,  p_ij = exp(scale q_i.k_j - m_i),
//   l_i = sum_{j <= i} p_ij,            lse_i = m_i + ln l_i
//
// one pass over the keys with the running maximum m and sum l in fp32.
//
// What bounds it: 4 * 128 flop a head and visible key against 512 bytes of K
// and V that every query tile shares, so the tensor cores from a few hundred
// tokens on, and launch and pipeline latency below.
//
// Work item: one sequence, one KV head, two tiles of 128 query rows.  A row is
// (position, query head of the group), so that the group's heads share every
// K / V tile and a short prompt still fills its rows; a tile is floor(128 / G)
// positions x G heads, loaded by one TMA box per 64-dim half.  Per 128 keys
// and tile t:
//   S_t = Q_t K^T          tcgen05, both operands in shared memory, fp32 in TMEM
//   P_t = 2^(S_t c - m c)  one thread a row; bf16 back into S_t's TMEM columns
//   O_t += P_t V           tcgen05, P from TMEM, V from shared memory
// While one warpgroup exponentiates its tile, the tensor cores work on the
// other's products.  P is rounded to bf16 (to nearest) for the second product,
// the operand type of V: a relative error of at most 2^-8 a term, the size of
// the output's own rounding; sums (of P before that rounding), maxima and O stay
// in fp32.  O is rescaled only
// when a row's maximum has grown by more than 2^8 since the last time (the
// running maximum only has to keep the exponentials in range).
//
// Warps: 0-3 and 4-7 one tile each (softmax, rescale, output), 8 loads, 9
// issues the products, 10 finds the items and sends the outputs off, 11 looks
// through V tiles that hold keys which some row of the item must not see (the
// diagonal, the sequence's end): their P is 0, but 0 x inf and 0 x NaN would
// leak a broken value into rows that come before it or belong to another
// sequence.  What is not finite there is set to 0 in shared memory, and rows
// that do see it get it back at the end.
//
// Why this shape: two query tiles an item are what TMEM holds (S and O twice, 512
// columns) and what gives the tensor cores one tile's products during the other's
// softmax; tiles of 128 keys keep a row's scores in the registers of one thread
// (200 of them: with 224 / 56 for the third warpgroup 364 us instead of 340, with
// 192 / 120 347; measured on one sequence of 8,192 with 32 / 4 heads).  Four K / V
// stages (three: 436 us where four took 377; a fifth gained nothing), one CTA an SM.
// Items go out by a fixed order, longest first, back and forth over the CTAs;
// claiming them as CTAs come free gained nothing.
//
// Measured (GB300, device time): one sequence of 8,192, 32 / 4 heads, 550 GFLOP: 337 to
// 341 us in runs of some 20 to 100 calls (1,632 to 1,612 TFLOP/s, 85 % of the measured
// bf16 GEMM rate), 361 to 363 in runs of seconds, where the power cap holds the clock
// at 1,935 MHz (1,515 TFLOP/s, 88 % of the sustained GEMM rate), up to 373 in a run of
// three calls; tensor pipe busy 69 % of cycles, the rest the hand-over of scores and
// P.  24 sequences of 0 to 900, 16 /
// 8 heads, 22.7 GFLOP: 40 us, 561 TFLOP/s; there an item is two or three key tiles,
// and a tile's end (its last product, the output, the way back to the first scores,
// about 3,000 cycles with instruction misses) is not all hidden.  One sequence of
// 29: 7.4 to 7.6 us, launch and one pass through the pipeline.
#include <cuda.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "common.cuh"

IPD_DECLARE_ERROR_WORD(g_prompt_err);
// whether this process has launched (or captured) a kernel that may set the word:
// a program without these calls does not pay for reading it
static std::atomic<bool> g_prompt_used{false};

namespace {

constexpr int kD = 128;
constexpr int kRows = 128;                   // rows of a query tile (M)
constexpr int kKeys = 128;                   // keys of a K / V tile (N)
constexpr int kTileBytes = kRows * kD * 2;   // 32 KB: a Q, K or V tile
constexpr int kHalfBytes = kTileBytes / 2;   // its 64-dim halves, 128-byte swizzled rows
constexpr int kStages = 4;                   // K and V tiles in flight (a fifth gained nothing)
constexpr int kSlots = 3;                    // items handed from the item warp to the others
constexpr int kMendSlots = 4;               // more than the V tiles that can be in flight
constexpr int kThreads = 384;
constexpr int kLoadWarp = 8, kMmaWarp = 9, kItemWarp = 10, kMendWarp = 11;
constexpr uint32_t kTmemCols = 512;          // S_0, S_1, O_0, O_1 of 128 fp32 columns
__host__ __device__ constexpr uint32_t col_s(int t) { return 128u * (uint32_t)t; }
__host__ __device__ constexpr uint32_t col_o(int t) { return 256u + 128u * (uint32_t)t; }
// Registers: launched with 168 a thread; the third warpgroup gives back what
// the softmax warpgroups need to hold a row's 128 scores.
constexpr int kRegsLaunch = 168, kRegsAux = 104, kRegsSoftmax = 200;
static_assert(kMendSlots > (kStages + 1) / 2, "a slot is reused only after its tile was consumed");
static_assert(256 * kRegsSoftmax + 128 * kRegsAux <= kThreads * kRegsLaunch,
              "the register split must fit the registers the block was launched with");
constexpr float kRescaleLog2 = 8.0f;         // growth of the maximum that rescales O
constexpr int kItemReaders = 8 + 3;          // softmax warps, loader, issuer, mender

struct Item {
  int start, len;   // the sequence's first token and length
  int pos;          // first query position
  int kvh;
  int nk[2];        // K / V tiles of each query tile (0: the tile has no rows)
  int first_masked; // first K / V tile in which some row sees only part of the keys
  int valid;
  int bad;          // a visible non-finite value was taken out of a diagonal V tile
};

struct Shared {
  alignas(1024) uint8_t q[2][kTileBytes];
  alignas(1024) uint8_t kv[kStages][kTileBytes];
  alignas(1024) uint8_t out[2][kHalfBytes];  // a tile's output on its way, as its 64-dim halves
  uint64_t q_full, q_empty, kv_full[kStages], kv_empty[kStages], s_full[2], p_full[2][2], o_full[2],
      o_empty[2], out_full[2], out_free[2], v_landed[kMendSlots], item_full[kSlots], item_empty[kSlots], drain;
  Item item[kSlots];
  uint32_t tmem;
  int abort;
};
constexpr int kSharedBytes = (int)sizeof(Shared) + 1024;  // the base is aligned by hand
static_assert(kSharedBytes <= 232448, "shared memory of one CTA");

struct Params {
  CUtensorMap q, k, v, out_map;
  const uint16_t *v_ptr;
  long long v_stride, out_stride;
  uint16_t *out;
  float *lse;
  const int32_t *cu;
  int num_seqs, total, max_len;
  int hkv, group;
  int tile_pos;  // positions of one query tile: floor(128 / group)
  uint32_t pos_mul, pos_shift;  // n / (2 tile_pos) = (n * mul >> 32) >> shift, n < 2^31
  float scale_log2;
};

// 3-D tiled TMA load (dims, heads, tokens).
IPD_DEVINL void tma_load_3d(void *dst, const CUtensorMap *map, int x, int y, int z, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
      : "memory");
}

// 3-D tiled TMA store, in a bulk group of the thread.
IPD_DEVINL void tma_store_3d(const CUtensorMap *map, int x, int y, int z, const void *src) {
  asm volatile(
      "cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map),
      "r"(x), "r"(y), "r"(z), "r"(smem_u32(src))
      : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// until the thread's bulk stores have read their shared memory
IPD_DEVINL void tma_store_wait() {
  asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
}

// A wait that gives up after about a second, or as soon as another warp of the
// CTA has given up.  Each try suspends the thread for a while in hardware; the
// clock and the flag are looked at every few tries only, so that waiting warps
// leave the issue slots to the others.
IPD_DEVINL bool wait_slow(uint64_t *bar, uint32_t parity, volatile int *abort) {
  const long long t0 = clock64();
  while (true) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort) return false;
    if (clock64() - t0 > kWaitLimitCycles) {
      ipd_set_error(&g_prompt_err, IPD_DEVERR_WAIT);
      *abort = 1;
      return false;
    }
  }
}
IPD_DEVINL bool wait(uint64_t *bar, uint32_t parity, volatile int *abort) {
  return mbar_try_wait(bar, parity) || wait_slow(bar, parity, abort);
}
// the same for a whole warp, with one answer
IPD_DEVINL bool wait_warp(uint64_t *bar, uint32_t parity, volatile int *abort) {
  return __all_sync(0xffffffffu, wait(bar, parity, abort)) != 0;
}

// Phase of the n-th use (0, 1, ...) of a barrier: a consumer waits for it with
// parity n & 1, a producer for the release of its slot with the other.
IPD_DEVINL uint32_t full_parity(uint32_t n) { return n & 1u; }
IPD_DEVINL uint32_t empty_parity(uint32_t n) { return (n & 1u) ^ 1u; }

// --------------------------------------------------------------------------
// items
// --------------------------------------------------------------------------
// Length of sequence r; 0 (recorded once) where the offsets are out of order
// or past the tensors, or the length is over the caller's bound.
IPD_DEVINL int seq_len(const Params &P, int r, int *start) {
  const int a = P.cu[r], b = P.cu[r + 1];
  *start = a;
  if (a < 0 || b < a || b > P.total) {
    ipd_set_error(&g_prompt_err, IPD_DEVERR_SPAN);
    return 0;
  }
  if (b - a > P.max_len) {
    ipd_set_error(&g_prompt_err, IPD_DEVERR_SEQ_LEN);
    return 0;
  }
  return b - a;
}

// Items in order of falling cost: level by level from the longest (an item's
// level is its place along its sequence, which is what it costs), the
// sequences that reach a level in order, KV heads innermost.  The CTAs take
// them round by round, every other round backwards, so that the rounds'
// differences cancel.
//
// Up to 32 sequences stay in the warp's registers.  With more, each item is
// looked for from sequence 0 on, two offsets read again for each, so that the
// search grows with the square of their number and is what bounds a call of
// hundreds of short ones: 32 / 33 / 333 / 1,024 / 4,000 sequences of 1 to 40, 16 / 8
// heads, take 12.0 / 12.6 / 76 / 332 / 3,838 us, 512 / 1,024 of 20 to 300 305 / 763.
struct ItemFinder {
  int level;          // items below `before` lie at higher levels
  long long before;
  int here;           // (sequence, tile) pairs at `level`
  int start, len;     // sequence `lane`, when there are at most 32 (else read again)

  int mine;           // ... and its tiles

  static IPD_DEVINL int tiles_of(const Params &P, int len) {
    return len > 0 ? (int)(__umulhi((uint32_t)len - 1u, P.pos_mul) >> P.pos_shift) + 1 : 0;
  }
  __device__ int tiles(const Params &P, int r) {
    int a;
    if (P.num_seqs <= 32) return mine;
    return r < P.num_seqs ? tiles_of(P, seq_len(P, r, &a)) : 0;
  }
  __device__ void count(const Params &P, int lane) {
    int n = 0;
    for (int r = lane; r < P.num_seqs; r += 32) n += tiles(P, r) > level ? 1 : 0;
    here = __reduce_add_sync(0xffffffffu, n);
  }
  __device__ void init(const Params &P, int lane) {
    start = len = 0;
    if (P.num_seqs <= 32 && lane < P.num_seqs) len = seq_len(P, lane, &start);
    mine = tiles_of(P, len);
    before = 0;
    int top = 0;
    for (int r = lane; r < P.num_seqs; r += 32) top = max(top, tiles(P, r));
    level = __reduce_max_sync(0xffffffffu, top) - 1;  // the highest that has a sequence
    here = 0;
    if (level >= 0) count(P, lane);
  }
  // the s-th (sequence, tile) pair: its tile (< 0: there is none), and the
  // sequence's place; pairs are asked for in rising order
  __device__ int find(const Params &P, int lane, long long s, int *at, int *n) {
    while (level >= 0 && s >= before + here) {
      before += here;
      --level;
      if (level >= 0) count(P, lane);
    }
    if (level < 0) return -1;
    int rank = (int)(s - before);
    for (int r0 = 0; r0 < P.num_seqs; r0 += 32) {
      const uint32_t in = __ballot_sync(0xffffffffu, tiles(P, r0 + lane) > level);
      const int c = __popc(in);
      if (rank < c) {
        const uint32_t hit = __ballot_sync(
            0xffffffffu, ((in >> lane) & 1u) && __popc(in & ((1u << lane) - 1u)) == rank);
        const int src = __ffs(hit) - 1;
        if (P.num_seqs <= 32) {
          *at = __shfl_sync(0xffffffffu, start, src);
          *n = __shfl_sync(0xffffffffu, len, src);
        } else {
          *n = seq_len(P, r0 + src, at);
        }
        return level;
      }
      rank -= c;
    }
    return -1;
  }
};

// A tile whose rows all belong to the sequence leaves through shared memory.
IPD_DEVINL bool leaves(const Params &P, const Item &I, int tile) {
  return I.pos + (tile + 1) * P.tile_pos <= I.len;
}

// Sends the output tiles of item n off, tile 0 then tile 1.  The two share one
// buffer, handed over once an item each way whether or not a tile leaves: every
// phase of every barrier is then waited for, and none can be mistaken.
IPD_DEVINL bool send_outputs(const Params &P, Shared &S, uint32_t n, int lane) {
  const Item &I = S.item[n % kSlots];
#pragma unroll 1
  for (int t = 0; t < 2; ++t) {
    if (!wait_warp(&S.out_full[t], full_parity(n), &S.abort)) return false;
    if (lane == 0) {
      if (leaves(P, I, t)) {
        for (int h = 0; h < 2; ++h)
          tma_store_3d(&P.out_map, 64 * h, I.kvh * P.group, I.start + I.pos + t * P.tile_pos,
                       S.out[h]);
        if (I.bad) {  // rows will be read back: until the stores are complete
          asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
          __threadfence();
        }
        tma_store_wait();
      }
      mbar_arrive(&S.out_free[1 - t]);
    }
    __syncwarp();
  }
  return true;
}

__device__ void item_warp(const Params &P, Shared &S, int lane) {
  const int pt = 2 * P.tile_pos;
  ItemFinder F;
  F.init(P, lane);
  // this CTA's place in the order, n * gridDim.x + blockIdx.x (or the CTAs from
  // behind, every other round), as a pair and its KV head; the steps to the
  // next one of an even and an odd round
  const uint32_t hkv = P.hkv, step0 = 2 * (gridDim.x - blockIdx.x) - 1, step1 = 2 * blockIdx.x + 1;
  const uint32_t pairs0 = step0 / hkv, pairs1 = step1 / hkv;
  long long pair = blockIdx.x / hkv;
  uint32_t head = blockIdx.x % hkv;
  uint32_t n = 0;
  for (;; ++n) {
    const int slot = n % kSlots;
    const uint32_t use = n / kSlots;
    int start = 0, len = 0;
    const int tile = F.find(P, lane, pair, &start, &len);
    const uint32_t kvh = head;
    pair += n & 1 ? pairs1 : pairs0;
    head += n & 1 ? step1 - pairs1 * hkv : step0 - pairs0 * hkv;
    if (head >= hkv) head -= hkv, ++pair;
    const bool ok = tile >= 0;
    // the item that had the slot before
    if (use > 0 && !send_outputs(P, S, n - kSlots, lane)) return;
    if (!wait_warp(&S.item_empty[slot], empty_parity(use), &S.abort)) return;
    if (lane == 0) {
      Item &I = S.item[slot];
      I.valid = ok;
      I.bad = 0;
      if (ok) {
        I.start = start;
        I.len = len;
        I.pos = tile * pt;
        I.kvh = (int)kvh;
        for (int t = 0; t < 2; ++t) {
          const int p0 = I.pos + t * P.tile_pos, p1 = min(I.len, p0 + P.tile_pos);
          I.nk[t] = p0 < I.len ? (p1 + kKeys - 1) / kKeys : 0;
        }
        // tile k is seen whole by every row when its last key is at or before
        // the item's first position
        I.first_masked = (I.pos + 1) / kKeys;
      }
      mbar_arrive(&S.item_full[slot]);
    }
    __syncwarp();
    if (!ok) break;
  }
  // the items still out: the last kSlots - 1 before the end
  for (uint32_t m = n > kSlots - 1 ? n - (kSlots - 1) : 0; m < n; ++m)
    if (!send_outputs(P, S, m, lane)) return;
}

// --------------------------------------------------------------------------
// loads
// --------------------------------------------------------------------------
__device__ void load_warp(const Params &P, Shared &S) {
  uint32_t ring = 0, n_q = 0, n_mend = 0;
  const uint32_t q_bytes = (uint32_t)(P.group * P.tile_pos) * kD * 2;
  for (uint32_t n = 0;; ++n) {
    const int slot = n % kSlots;
    if (!wait(&S.item_full[slot], full_parity(n / kSlots), &S.abort)) break;
    const Item I = S.item[slot];
    mbar_arrive(&S.item_empty[slot]);
    if (!I.valid) break;
    if (!wait(&S.q_empty, empty_parity(n), &S.abort)) break;
    const int tiles = I.nk[1] > 0 ? 2 : 1;
    mbar_arrive_expect_tx(&S.q_full, q_bytes * tiles);
    for (int t = 0; t < tiles; ++t)
      for (int h = 0; h < 2; ++h)
        tma_load_3d(S.q[t] + h * kHalfBytes, &P.q, 64 * h, I.kvh * P.group,
                    I.start + I.pos + t * P.tile_pos, &S.q_full);
    ++n_q;
    const int nk = max(I.nk[0], I.nk[1]);
    bool ok = true;
    for (int j = 0; j < 2 * nk && ok; ++j, ++ring) {
      const int st = ring % kStages;
      ok = wait(&S.kv_empty[st], empty_parity(ring / kStages), &S.abort);
      if (!ok) break;
      // a V tile with hidden keys lands at the mending warp, which then fills the stage
      uint64_t *landed = &S.kv_full[st];
      if ((j & 1) && (j >> 1) >= I.first_masked) landed = &S.v_landed[n_mend++ % kMendSlots];
      mbar_arrive_expect_tx(landed, kTileBytes);
      for (int h = 0; h < 2; ++h)
        tma_load_3d(S.kv[st] + h * kHalfBytes, (j & 1) ? &P.v : &P.k, 64 * h, I.kvh,
                    I.start + (j >> 1) * kKeys, landed);
    }
    if (!ok) break;
  }
  if (*(volatile int *)&S.abort) {
    // the CTA gives up: its copies in flight land first (bounded)
    if (n_q > 0) mbar_wait_bounded(&S.q_full, full_parity(n_q - 1));
    for (uint32_t s = 0; s < (uint32_t)kStages && s < ring; ++s) {
      const uint32_t last = ring - 1 - s;
      mbar_wait_bounded(&S.kv_full[last % kStages], full_parity(last / kStages));
    }
    for (uint32_t s = 0; s < (uint32_t)kMendSlots && s < n_mend; ++s) {
      const uint32_t last = n_mend - 1 - s;
      mbar_wait_bounded(&S.v_landed[last % kMendSlots], full_parity(last / kMendSlots));
    }
  }
}

// --------------------------------------------------------------------------
// products
// --------------------------------------------------------------------------
// The warp's elected lane issues; every other value is the whole warp's, so that
// the operands stay in uniform registers (issued from a branch of one lane,
// each product cost its own time again in register moves).
IPD_DEVINL uint32_t elect_one() {
  uint32_t e;
  asm volatile(
      "{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(e));
  return e;
}
IPD_DEVINL int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }

__device__ void mma_warp(const Params &P, Shared &S, int lane) {
  constexpr uint32_t idesc_s = idesc_bf16_f32(kRows, kKeys, 0);
  constexpr uint32_t idesc_o = idesc_bf16_f32(kRows, kD, 1);
  constexpr uint64_t kTileStep = kTileBytes >> 4, kHalfStep = kHalfBytes >> 4;
  const uint32_t tmem = (uint32_t)uniform((int)S.tmem);
  // descriptors of the first Q tile and stage; V is N-major: 64-dim halves
  // kHalfBytes apart, 8-key groups 1024 apart
  const uint64_t q0 = sdesc_sw128((uint32_t)uniform((int)smem_u32(S.q[0])), 16, 1024);
  const uint64_t k0 = sdesc_sw128((uint32_t)uniform((int)smem_u32(S.kv[0])), 16, 1024);
  const uint64_t v0 = sdesc_sw128((uint32_t)uniform((int)smem_u32(S.kv[0])), kHalfBytes, 1024);
  uint32_t ring = 0, n_p[2] = {0, 0}, n_o[2] = {0, 0};
  const auto issue_s = [&](int t, int stage) {
    const uint64_t a = q0 + t * kTileStep, b = k0 + stage * kTileStep;
    if (elect_one()) {
#pragma unroll
      for (int kk = 0; kk < kD / 16; ++kk) {
        const uint64_t off = (kk >> 2) * kHalfStep + (uint64_t)(32 * (kk & 3) >> 4);
        tc_mma_bf16(tmem + col_s(t), a + off, b + off, idesc_s, kk > 0);
      }
      tc_commit(&S.s_full[t]);
    }
    __syncwarp();
  };
  // keys 64 half .. 64 half + 63
  const auto issue_o = [&](int t, int stage, int half, bool accumulate) {
    const uint64_t b = v0 + stage * kTileStep + (uint64_t)(half * 8192 >> 4);
    const uint32_t a = tmem + col_s(t) + 32 * half;
    if (elect_one()) {
#pragma unroll
      for (int kk = 0; kk < 4; ++kk)
        tc_mma_bf16_ta(tmem + col_o(t), a + 8 * kk, b + (uint64_t)(2048 * kk >> 4), idesc_o,
                       accumulate || kk > 0);
    }
    __syncwarp();
  };
  const auto commit = [&](uint64_t *bar) {
    if (elect_one()) tc_commit(bar);
    __syncwarp();
  };
  // The products run on from item to item: where a tile's last O product is
  // issued, the first scores of its next item follow.
  uint32_t n = 0;              // items taken
  int nk0 = 0, nk1 = 0;        // this item's tiles
  int next0 = 0, next1 = 0;    // the next one's (none: 0, 0)
  const auto take = [&]() {
    const int slot = n % kSlots;
    if (!wait_warp(&S.item_full[slot], full_parity(n / kSlots), &S.abort)) return false;
    const Item &I = S.item[slot];
    const int valid = uniform(I.valid), a = uniform(I.nk[0]), b = uniform(I.nk[1]);
    next0 = valid ? a : 0;
    next1 = valid ? b : 0;
    __syncwarp();
    if (lane == 0) mbar_arrive(&S.item_empty[slot]);
    ++n;
    return true;
  };
  // O_t += P_t V_j
  const auto add_o = [&](int t, int stage, int j) {
    if (j == 0) {  // O_t of the item before has been read
      if (!wait_warp(&S.o_empty[t], empty_parity(n_o[t]), &S.abort)) return false;
      ++n_o[t];
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      if (!wait_warp(&S.p_full[t][half], full_parity(n_p[t]), &S.abort)) return false;
      tc_fence_after();
      issue_o(t, stage, half, j + half > 0);
    }
    ++n_p[t];
    return true;
  };
  bool ok = take();
  int j = -1;
  while (ok) {
    // all but the item's last K tile: S_t's columns hold P_t until the products
    // before have read them; the tensor core takes this thread's instructions
    // in order
    const int nk = max(nk0, nk1);
#pragma unroll 1
    for (; j >= 0 && j + 1 < nk; ++j) {
      const int vs = ring % kStages, ks = (ring + 1) % kStages;
      if (!(ok = wait_warp(&S.kv_full[vs], full_parity(ring / kStages), &S.abort))) break;
      ++ring;
      if (!(ok = wait_warp(&S.kv_full[ks], full_parity(ring / kStages), &S.abort))) break;
      ++ring;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int mine = t ? nk1 : nk0;
        if (j >= mine) continue;
        if (!(ok = add_o(t, vs, j))) break;
        if (j + 1 < mine) issue_s(t, ks);
        else commit(&S.o_full[t]);
      }
      if (!ok) break;
      commit(&S.kv_empty[vs]);
      commit(&S.kv_empty[ks]);
      if (j + 2 == nk) commit(&S.q_empty);  // the item's last scores are issued
    }
    if (!ok) break;
    // the last one, and the next item's first scores
    int vs = 0;
    if (j >= 0) {
      vs = ring % kStages;
      if (!(ok = wait_warp(&S.kv_full[vs], full_parity(ring / kStages), &S.abort))) break;
      ++ring;
      if (!(ok = take())) break;
    }
    const int ks = ring % kStages;
    bool waited = false;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (j >= 0 && j + 1 == (t ? nk1 : nk0)) {
        if (!(ok = add_o(t, vs, j))) break;
        commit(&S.o_full[t]);
      }
      if ((t ? next1 : next0) > 0) {
        if (!waited) {
          ok = wait_warp(&S.q_full, full_parity(n - 1), &S.abort) &&
               wait_warp(&S.kv_full[ks], full_parity(ring / kStages), &S.abort);
          if (!ok) break;
          tc_fence_after();
          waited = true;
        }
        issue_s(t, ks);
      }
    }
    if (!ok) break;
    if (j >= 0) commit(&S.kv_empty[vs]);
    if (next0 == 0) break;  // (a tile 1 without a tile 0 does not occur)
    commit(&S.kv_empty[ks]);
    ++ring;
    nk0 = next0, nk1 = next1;
    j = 0;
    if (max(nk0, nk1) == 1) commit(&S.q_empty);
  }
  if (!ok) {  // the CTA gives up: products in flight end before TMEM is freed
    commit(&S.drain);
    mbar_wait_bounded(&S.drain, 0);
  }
}

// --------------------------------------------------------------------------
// V tiles with hidden keys
// --------------------------------------------------------------------------
IPD_DEVINL uint32_t not_finite2(uint32_t w) {  // bit 15 of each half: its exponent is all ones
  return ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
IPD_DEVINL uint32_t fma0_bf16x2(uint32_t v, uint32_t acc) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(v), "r"(0u), "r"(acc));
  return d;
}
// Whether rows row0 .. 127 of a V tile hold anything that is not finite: 0 x v
// summed is NaN then, and 0 otherwise.
IPD_DEVINL bool any_not_finite(const uint8_t *tile, int row0, int lane) {
  uint32_t a[4] = {0u, 0u, 0u, 0u};
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    const uint4 *v = reinterpret_cast<const uint4 *>(tile + h * kHalfBytes);
#pragma unroll 8
    for (int i = row0 * 8 + lane; i < kKeys * 8; i += 32) {
      const uint4 w = v[i];
      a[0] = fma0_bf16x2(w.x, a[0]);
      a[1] = fma0_bf16x2(w.y, a[1]);
      a[2] = fma0_bf16x2(w.z, a[2]);
      a[3] = fma0_bf16x2(w.w, a[3]);
    }
  }
  return __any_sync(0xffffffffu, ((a[0] | a[1] | a[2] | a[3]) & 0x7fff7fffu) != 0u) != 0;
}
// Sets them to 0; true if one belonged to a row below row_end.
IPD_DEVINL bool drop_not_finite(uint8_t *tile, int row0, int row_end, int lane) {
  bool seen = false;
#pragma unroll 1
  for (int i = lane; i < 2 * kKeys * 8; i += 32) {
    const int r = (i >> 3) & (kKeys - 1);
    if (r < row0) continue;
    uint4 *v = reinterpret_cast<uint4 *>(tile) + i;
    const uint4 w = *v;
    if (not_finite2(w.x) | not_finite2(w.y) | not_finite2(w.z) | not_finite2(w.w)) {
      const auto clear = [](uint32_t x) {
        const uint32_t bad = not_finite2(x) >> 15;
        return x & ~(bad * 0xffffu);
      };
      *v = make_uint4(clear(w.x), clear(w.y), clear(w.z), clear(w.w));
      seen = seen || r < row_end;
    }
  }
  fence_proxy_async_smem();
  return __any_sync(0xffffffffu, seen) != 0;
}

__device__ void mend_warp(const Params &P, Shared &S, int lane) {
  uint32_t ring = 0, n_mend = 0;
  for (uint32_t n = 0;; ++n) {
    const int slot = n % kSlots;
    if (!wait_warp(&S.item_full[slot], full_parity(n / kSlots), &S.abort)) return;
    const Item I = S.item[slot];
    const int nk = I.valid ? max(I.nk[0], I.nk[1]) : 0;
    for (int j = I.valid ? min(I.first_masked, nk) : 0; j < nk; ++j, ++n_mend) {
      if (!wait_warp(&S.v_landed[n_mend % kMendSlots], full_parity(n_mend / kMendSlots), &S.abort))
        return;
      const int st = (ring + 2 * j + 1) % kStages;  // V tile j's stage
      const int row0 = max(0, I.pos + 1 - j * kKeys);
      if (any_not_finite(S.kv[st], row0, lane)) {
        const bool seen = drop_not_finite(S.kv[st], row0, I.len - j * kKeys, lane);
        if (seen && lane == 0) S.item[slot].bad = 1;
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.kv_full[st]);
    }
    ring += 2 * nk;
    __syncwarp();
    if (lane == 0) mbar_arrive(&S.item_empty[slot]);
    if (!I.valid) return;
  }
}

// --------------------------------------------------------------------------
// softmax and output of one query tile
// --------------------------------------------------------------------------
// O's row in TMEM times f (all warps of the tile, 128 columns).
IPD_DEVINL void scale_o(uint32_t o, float f) {
#pragma unroll 1
  for (int c = 0; c < kD; c += 32) {
    uint32_t r[32];
    tc_ld_32x32b_x32(o + c, r);
    tc_wait_ld();
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
    tc_st_32x32b_x32(o + c, r);
  }
  tc_wait_st();
}

// The non-finite values of the keys after the item's first position that were
// taken out of the V tiles, added back to the stored output of a row at `pos`
// that sees them: any weight of theirs leaves an infinity infinite and a NaN a
// NaN, so the finite part's rounding does not matter.
IPD_DEVINL void add_not_finite(const Params &P, const Item &I, int pos, uint16_t *out) {
#pragma unroll 1
  for (int d = 0; d < kD; d += 2) {
    uint32_t *at = reinterpret_cast<uint32_t *>(out + d);
    float lo = bf16lo(*at), hi = bf16hi(*at);
#pragma unroll 1
    for (int key = I.pos + 1; key <= pos; ++key) {
      const uint32_t w = *reinterpret_cast<const uint32_t *>(
          P.v_ptr + (long long)(I.start + key) * P.v_stride + (long long)I.kvh * kD + d);
      if ((w & 0x00007f80u) == 0x00007f80u) lo += bf16lo(w);
      if ((w & 0x7f800000u) == 0x7f800000u) hi += bf16hi(w);
    }
    *at = pack_bf16x2(lo, hi);
  }
}

// Largest of 64 scores and m; MASKED: keys past `lim` count as -inf.
template <bool MASKED>
IPD_DEVINL float max_of(uint32_t *s, int lim, float m) {
  if (MASKED) {
#pragma unroll
    for (int i = 0; i < 64; ++i)
      if (i > lim) s[i] = 0xff800000u;
  }
  float a[4] = {m, __uint_as_float(s[0]), __uint_as_float(s[1]), __uint_as_float(s[2])};
#pragma unroll
  for (int i = 3; i < 59; i += 8)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      a[k] = fmax3(a[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
  a[0] = fmax3(a[0], __uint_as_float(s[59]), __uint_as_float(s[60]));
  a[1] = fmax3(a[1], __uint_as_float(s[61]), __uint_as_float(s[62]));
  return fmax3(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]), __uint_as_float(s[63]));
}

__device__ void softmax_warps(const Params &P, Shared &S, int t, int warp, int lane) {
  const int row = (warp & 3) * 32 + lane;
  const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t s_col = S.tmem + lanes + col_s(t), o_col = S.tmem + lanes + col_o(t);
  const int row_pos = row / P.group, row_head = row % P.group;
  const float c = P.scale_log2;
  const unsigned long long c2 = f2_pack(c, c);
  uint32_t n_s = 0, n_o = 0;
  for (uint32_t n = 0;; ++n) {
    const int slot = n % kSlots;
    if (!wait_warp(&S.item_full[slot], full_parity(n / kSlots), &S.abort)) return;
    const Item &I = S.item[slot];  // (there until this warp's release)
    // tile 0 has the output buffer first, and again when tile 1's has left
    const uint32_t free_parity = t == 0 ? empty_parity(n) : full_parity(n);
    const int nk = I.valid ? I.nk[t] : 0;
    if (nk > 0) {
      const int pos = I.pos + t * P.tile_pos + row_pos;
      const bool live = row_pos < P.tile_pos && pos < I.len;
      const int last = min(pos, I.len - 1);  // a row without a query follows the last one
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < nk; ++j) {
        if (!wait_warp(&S.s_full[t], full_parity(n_s), &S.abort)) return;
        ++n_s;
        tc_fence_after();
        // the second half of the scores is on its way while the first is looked at
        uint32_t s[kKeys];
        const auto load = [&](int k) {
          tc_ld_32x32b_x32(s_col + k, reinterpret_cast<uint32_t(&)[32]>(s[k]));
        };
        load(0);
        load(32);
        tc_wait_ld();
        load(64);
        load(96);
        float mx;
        if (j >= I.first_masked) {
          mx = max_of<true>(s, last - j * kKeys, -INFINITY);
          tc_wait_ld();
          mx = max_of<true>(s + 64, last - j * kKeys - 64, mx);
        } else {
          mx = max_of<false>(s, 0, -INFINITY);
          tc_wait_ld();
          mx = max_of<false>(s + 64, 0, mx);
        }
        if (j == 0) {
          m = mx;
        } else {
          // m is -inf while every visible score has been: the first finite
          // one then rescales (a sum of zeros)
          const bool grow = (mx - m) * c > kRescaleLog2;
          if (__any_sync(0xffffffffu, grow)) {
            float f = 1.f;
            if (grow) {
              f = m == -INFINITY ? 0.f : ex2_approx((m - mx) * c);
              m = mx;
            }
            l *= f;
            // s_full counted the products before S_t's too: O_t is complete
            scale_o(o_col, f);
          }
        }
        const float off = m == -INFINITY ? 0.f : -m * c;
        const unsigned long long off2 = f2_pack(off, off);
        unsigned long long sum[2] = {0ull, 0ull};
#pragma unroll
        for (int hb = 0; hb < 2; ++hb) {
          uint32_t p[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const int e = hb * 64 + 2 * i;
            float x0, x1;
            f2_unpack(f2_fma(f2_pack(__uint_as_float(s[e]), __uint_as_float(s[e + 1])), c2, off2),
                      x0, x1);
            x0 = ex2_approx(x0);
            x1 = ex2_approx(x1);
            sum[i & 1] = f2_add(sum[i & 1], f2_pack(x0, x1));
            p[i] = pack_bf16x2(x0, x1);
          }
          tc_st_32x32b_x32(s_col + 32 * hb, p);
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&S.p_full[t][hb]);  // half of the product may start
        }
        float a, b;
        f2_unpack(f2_add(sum[0], sum[1]), a, b);
        l += a + b;
      }
      // while the last product runs
      const float inv = 1.f / l;
      if (live && P.lse)
        P.lse[(long long)(I.kvh * P.group + row_head) * P.total + I.start + pos] =
            (m == -INFINITY ? -INFINITY : (m * c + log2f(l)) * kLn2);
      if (!wait_warp(&S.o_full[t], full_parity(n_o), &S.abort)) return;
      ++n_o;
      tc_fence_after();
      const bool bad = *(volatile int *)&S.item[slot].bad != 0;
      uint16_t *out = P.out + (long long)(I.start + pos) * P.out_stride +
                      (long long)(I.kvh * P.group + row_head) * kD;
      uint32_t w[64];
#pragma unroll
      for (int k = 0; k < 4; k += 2) {
        uint32_t o[64];
        tc_ld_32x32b_x32(o_col + 32 * k, reinterpret_cast<uint32_t(&)[32]>(o[0]));
        tc_ld_32x32b_x32(o_col + 32 * k + 32, reinterpret_cast<uint32_t(&)[32]>(o[32]));
        tc_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i)
          w[16 * k + i] =
              pack_bf16x2(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&S.o_empty[t]);  // O_t is read: the next item may write it
      if (leaves(P, I, t)) {
        // through shared memory and TMA (16-byte stores of 32 rows each would
        // hold up the SM's other warps)
        if (!wait_warp(&S.out_free[t], free_parity, &S.abort)) return;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          *reinterpret_cast<uint4 *>(S.out[i >> 3] + row * 128 + (((i & 7) ^ (row & 7)) << 4)) =
              make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&S.out_full[t]);
        // (the buffer's next hand-over follows the store)
        if (bad && !wait_warp(&S.out_free[1 - t], full_parity(n), &S.abort)) return;
      } else if (live) {
#pragma unroll
        for (int i = 0; i < 16; ++i)
          *reinterpret_cast<uint4 *>(out + 8 * i) =
              make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
      }
      if (bad && live) add_not_finite(P, I, pos, out);
    }
    const bool last_item = !I.valid;
    if (!last_item && !leaves(P, I, t)) {  // the buffer passes by
      if (!wait_warp(&S.out_free[t], free_parity, &S.abort)) return;
      if (lane == 0) mbar_arrive(&S.out_full[t]);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&S.item_empty[slot]);
    if (last_item) return;
  }
}

__global__ void __launch_bounds__(kThreads, 1) prompt_attn_kernel(const __grid_constant__ Params P) {
  extern __shared__ uint8_t smem_raw[];
  Shared &S = *reinterpret_cast<Shared *>(
      smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 32 * kLoadWarp) {
    for (const CUtensorMap *m : {&P.q, &P.k, &P.v, &P.out_map})
      asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
  }
  if (threadIdx.x == 0) {
    mbar_init(&S.q_full, 1);
    mbar_init(&S.q_empty, 1);
    for (int i = 0; i < kStages; ++i) mbar_init(&S.kv_full[i], 1), mbar_init(&S.kv_empty[i], 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&S.s_full[t], 1);
      mbar_init(&S.p_full[t][0], 4);
      mbar_init(&S.p_full[t][1], 4);
      mbar_init(&S.o_full[t], 1);
      mbar_init(&S.o_empty[t], 4);
      mbar_init(&S.out_full[t], 4);
      mbar_init(&S.out_free[t], 1);
    }
    for (int i = 0; i < kMendSlots; ++i) mbar_init(&S.v_landed[i], 1);
    mbar_init(&S.drain, 1);
    for (int i = 0; i < kSlots; ++i)
      mbar_init(&S.item_full[i], 1), mbar_init(&S.item_empty[i], kItemReaders);
    S.abort = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) {
    tc_alloc(&S.tmem, kTmemCols);
    tc_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(kRegsAux));
    if (warp == kItemWarp) item_warp(P, S, lane);
    else if (warp == kMmaWarp) mma_warp(P, S, lane);
    else if (warp == kMendWarp) mend_warp(P, S, lane);
    else if (lane == 0) load_warp(P, S);
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(kRegsSoftmax));
    softmax_warps(P, S, warp >> 2, warp, lane);
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tc_dealloc(S.tmem, kTmemCols);
}

// --------------------------------------------------------------------------
struct DevInfo {
  int sms = 0;
};
DevInfo g_prompt_dev[64];
PFN_cuTensorMapEncodeTiled_v12000 g_prompt_encode = nullptr;

int prepare_device(int *sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return IPD_ERR_CUDA;
  if (!g_prompt_encode) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault,
                                         &q) != cudaSuccess ||
        q != cudaDriverEntryPointSuccess || !fn)
      return IPD_ERR_CUDA;
    g_prompt_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  }
  DevInfo &D = g_prompt_dev[dev];
  if (D.sms == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
        cudaFuncSetAttribute(prompt_attn_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             kSharedBytes) != cudaSuccess)
      return IPD_ERR_CUDA;
    D.sms = n;
  }
  *sms = D.sms;
  return IPD_OK;
}

// [tokens][heads][128] bf16, tokens `stride` entries apart; a box is 64 dims x
// `heads` heads x `tokens` tokens: rows (token, head) of 128 swizzled bytes.
int encode(CUtensorMap *m, const void *base, int heads, int tokens, long long stride, int box_heads,
           int box_tokens) {
  const cuuint64_t dims[3] = {kD, (cuuint64_t)heads, (cuuint64_t)tokens};
  const cuuint64_t strides[2] = {kD * 2, (cuuint64_t)stride * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_tokens};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r =
      g_prompt_encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims,
                      strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                      CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? IPD_OK : IPD_ERR_CUDA;
}

}  // namespace

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_prompt_error() {
  if (!g_prompt_used.load(std::memory_order_relaxed)) return 0u;
  unsigned int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_prompt_err, sizeof(v)) != cudaSuccess) return 0xffffffffu;
  if (cudaMemcpyToSymbol(g_prompt_err, &z, sizeof(z)) != cudaSuccess) return 0xffffffffu;
  return v;
}

extern "C" int ipd_prompt_attn(const ipd_prompt_args *args, ipd_stream_t stream) {
  if (!args) return IPD_ERR_INVALID_ARG;
  const ipd_prompt_args &a = *args;
  if (a.num_seqs < 0 || a.total < 0 || a.max_len < 0 || a.num_kv_heads < 1 || a.num_q_heads < 1 ||
      a.num_q_heads % a.num_kv_heads || !(a.softmax_scale > 0.f) ||
      !(a.softmax_scale - a.softmax_scale == 0.f))
    return IPD_ERR_INVALID_ARG;
  const int group = a.num_q_heads / a.num_kv_heads;
  if (a.head_dim != kD || group > kRows || a.num_q_heads > 65536) return IPD_ERR_UNSUPPORTED;
  if (a.total == 0 || a.num_seqs == 0 || a.max_len == 0) return IPD_OK;
  const long long qrow = (long long)a.num_q_heads * kD, krow = (long long)a.num_kv_heads * kD;
  if (!a.q || !a.k || !a.v || !a.out || !a.cu_seq) return IPD_ERR_INVALID_ARG;
  if (a.q_stride < qrow || a.out_stride < qrow || a.k_stride < krow || a.v_stride < krow)
    return IPD_ERR_INVALID_ARG;
  const uintptr_t align = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.out |
                          (uintptr_t)(2 * a.q_stride) | (uintptr_t)(2 * a.k_stride) |
                          (uintptr_t)(2 * a.v_stride) | (uintptr_t)(2 * a.out_stride);
  if (align & 15) return IPD_ERR_INVALID_ARG;
  // the tensor maps hold strides below 2^40 bytes
  if ((a.q_stride | a.k_stride | a.v_stride | a.out_stride) >> 38) return IPD_ERR_UNSUPPORTED;
  int sms = 0;
  int st = prepare_device(&sms);
  if (st != IPD_OK) return st;
  Params P;
  memset(&P, 0, sizeof(P));
  P.tile_pos = kRows / group;
  {
    const uint32_t d = 2u * (uint32_t)P.tile_pos;  // 2 .. 256
    uint32_t k = 1;
    while ((1u << k) < d) ++k;
    P.pos_mul = (uint32_t)((((uint64_t)1 << (31 + k)) + d - 1) / d);
    P.pos_shift = k - 1;
  }
  if (encode(&P.q, a.q, a.num_q_heads, a.total, a.q_stride, group, P.tile_pos) != IPD_OK ||
      encode(&P.k, a.k, a.num_kv_heads, a.total, a.k_stride, 1, kKeys) != IPD_OK ||
      encode(&P.v, a.v, a.num_kv_heads, a.total, a.v_stride, 1, kKeys) != IPD_OK ||
      encode(&P.out_map, a.out, a.num_q_heads, a.total, a.out_stride, group, P.tile_pos) != IPD_OK)
    return IPD_ERR_CUDA;
  P.v_ptr = a.v;
  P.v_stride = a.v_stride;
  P.out = a.out;
  P.out_stride = a.out_stride;
  P.lse = a.lse;
  P.cu = a.cu_seq;
  P.num_seqs = a.num_seqs;
  P.total = a.total;
  P.max_len = a.max_len;
  P.hkv = a.num_kv_heads;
  P.group = group;
  P.scale_log2 = a.softmax_scale * kLog2e;
  // at most one CTA per SM and per item (a sequence's last item may be partial)
  const long long pt = 2 * P.tile_pos;
  const long long items = ((long long)a.total / pt + a.num_seqs) * a.num_kv_heads;
  const int grid = (int)(items < sms ? items : sms);
  g_prompt_used.store(true, std::memory_order_relaxed);
  prompt_attn_kernel<<<grid, kThreads, kSharedBytes, reinterpret_cast<cudaStream_t>(stream)>>>(P);
  return cudaGetLastError() == cudaSuccess ? IPD_OK : IPD_ERR_CUDA;
}

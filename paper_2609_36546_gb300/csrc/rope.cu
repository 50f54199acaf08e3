// Rotary positions: the cos / sin table, the rotation of a tensor's heads (and
// its transpose, which is its gradient), and the rotation of a step's new
// queries and keys fused with the write of the K/V rows into a paged cache.
//
// A pair (a, b) of a head's entries at position p turns by the angle p f_i:
//   y_a = a c - b s,  y_b = b c + a s,  (c, s) = table[p][i] = m (cos, sin)(p f_i)
// in fp32 from the stored inputs, rounded once to the output's type.  The
// transposed rotation takes -s.
//
// What bounds it: the rows are read and written once (3 flop for each 4 bytes),
// so HBM at thousands of tokens and the launch and a chain of five loads (the
// request, its length, its page, the angles, the rows) at a few.  A warp takes
// one token (or a share of its heads when tokens are few): lane = one unit of
// 2 x 16 bytes of a head (entries i.. and their partners) times a few heads at
// once, so that each lane reads its cos / sin once into registers and then walks
// over the heads with independent 16-byte loads.  Small blocks: a block's
// registers are free again when its two tokens are done.
//
// Measured (GB300, device time): the append of 14,599 prompt tokens of 32 / 4
// heads, 317 MB, in 50.9 us, 6.24 TB/s (blocks of 128 threads 51.3, of 256 57.0);
// 553 span tokens of 32 / 4 heads in 4.1 us; 128 single tokens of 16 / 8 heads in
// 3.0 us; 8,191 x 16 fp32 heads turned in 22.6 us, 6.1 TB/s.  Reading the rows
// before the position is known gains nothing at a few tokens and costs the
// registers of 15 % at many.
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>
#include <string.h>

#include <atomic>

#include "common.cuh"

IPD_DECLARE_ERROR_WORD(g_rope_err);
// whether this process has launched (or captured) a kernel that may set the word:
// a program without these calls does not pay for reading it
static std::atomic<bool> g_rope_used{false};

namespace {

constexpr int kRopeThreads = 64;
constexpr int kRopeWarps = kRopeThreads / 32;
constexpr int kUnroll = 4;        // heads in flight per lane
constexpr int kMaxFreqs = 128;    // rot_dim <= 256
// warps below which a token's heads are split over several: 8 for each SM of a GB300
constexpr int kTargetWarps = 152 * 8;

__host__ __device__ constexpr int ceil_div(int a, int b) { return (a + b - 1) / b; }

// 16 bytes of T as fp32 values and back
template <typename T>
struct Vec;
template <>
struct Vec<uint16_t> {
  static constexpr int N = 8;
  static IPD_DEVINL void unpack(const uint4 &r, float (&f)[8]) {
    f[0] = bf16lo(r.x), f[1] = bf16hi(r.x), f[2] = bf16lo(r.y), f[3] = bf16hi(r.y);
    f[4] = bf16lo(r.z), f[5] = bf16hi(r.z), f[6] = bf16lo(r.w), f[7] = bf16hi(r.w);
  }
  static IPD_DEVINL uint4 pack(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                      pack_bf16x2(f[6], f[7]));
  }
  static IPD_DEVINL float get(const uint16_t *p) { return bf16f(*p); }
  static IPD_DEVINL void put(uint16_t *p, float v) { *p = (uint16_t)pack_bf16x2(v, v); }
};
template <>
struct Vec<float> {
  static constexpr int N = 4;
  static IPD_DEVINL void unpack(const uint4 &r, float (&f)[4]) {
    f[0] = __uint_as_float(r.x), f[1] = __uint_as_float(r.y);
    f[2] = __uint_as_float(r.z), f[3] = __uint_as_float(r.w);
  }
  static IPD_DEVINL uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  }
  static IPD_DEVINL float get(const float *p) { return *p; }
  static IPD_DEVINL void put(float *p, float v) { *p = v; }
};

struct Rot {
  const float2 *table;  // [max_pos][rot / 2] (cos, sin)
  int max_pos, rot, layout;
  float sign;  // -1: the transposed rotation
};

// Rotates (or copies, where `turn` is false) one token's heads h0, h0 + step,
// ... < n_heads of head_dim D.  io(h) gives a head's source, destination, an
// optional second destination and whether it turns.  VEC: 16-byte units;
// otherwise one entry pair a time, for rotated parts that do not divide into
// units and for unaligned rows.
template <typename T, bool VEC, typename IO>
IPD_DEVINL void rotate_heads(const Rot &R, int pos, int D, int n_heads, int h0, int step, int unit,
                             int n_units, IO io) {
  constexpr int N = Vec<T>::N;
  const float2 *cs = R.table + (size_t)pos * (R.rot / 2);
  if constexpr (VEC) {
    const bool rot_unit = unit < R.rot / (2 * N);
    const bool half = R.layout == IPD_ROPE_HALF && rot_unit;
    const int oa = half ? unit * N : unit * 2 * N;
    const int ob = half ? R.rot / 2 + unit * N : oa + N;
    float c[N], s[N];
    if (rot_unit) {
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float4 t = __ldg(reinterpret_cast<const float4 *>(cs + unit * N + i));
        c[i] = t.x, s[i] = R.sign * t.y, c[i + 1] = t.z, s[i + 1] = R.sign * t.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) c[i] = 1.f, s[i] = 0.f;
    }
    for (int hb = h0; hb < n_heads; hb += step * kUnroll) {
      uint4 a[kUnroll], b[kUnroll];
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int h = hb + k * step;
        if (h < n_heads) {
          const T *src = io(h).src;
          a[k] = *reinterpret_cast<const uint4 *>(src + oa);
          b[k] = *reinterpret_cast<const uint4 *>(src + ob);
        }
      }
#pragma unroll
      for (int k = 0; k < kUnroll; ++k) {
        const int h = hb + k * step;
        if (h >= n_heads) break;
        const auto d = io(h);
        if (rot_unit && d.turn) {
          float x[2][N], y[2][N];
          Vec<T>::unpack(a[k], x[0]);
          Vec<T>::unpack(b[k], x[1]);
          if (half) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
              y[0][i] = x[0][i] * c[i] - x[1][i] * s[i];
              y[1][i] = x[1][i] * c[i] + x[0][i] * s[i];
            }
          } else {  // pair i: entries 2i and 2i + 1 of the unit's 2N
#pragma unroll
            for (int i = 0; i < N; ++i) {
              const float p = x[(2 * i) / N][(2 * i) % N], q = x[(2 * i + 1) / N][(2 * i + 1) % N];
              y[(2 * i) / N][(2 * i) % N] = p * c[i] - q * s[i];
              y[(2 * i + 1) / N][(2 * i + 1) % N] = q * c[i] + p * s[i];
            }
          }
          a[k] = Vec<T>::pack(y[0]);
          b[k] = Vec<T>::pack(y[1]);
        }
        *reinterpret_cast<uint4 *>(d.dst + oa) = a[k];
        *reinterpret_cast<uint4 *>(d.dst + ob) = b[k];
        if (d.dst2) {
          *reinterpret_cast<uint4 *>(d.dst2 + oa) = a[k];
          *reinterpret_cast<uint4 *>(d.dst2 + ob) = b[k];
        }
      }
    }
  } else {
    // pairs of a head: the rotated ones, then the entries left as they are two
    // at a time (an odd head_dim's last entry is its own pair)
    const int n_rot = R.rot / 2, n_pairs = n_rot + ceil_div(D - R.rot, 2);
    for (int h = h0; h < n_heads; h += step) {
      const auto d = io(h);
      for (int i = unit; i < n_pairs; i += n_units) {
        if (i < n_rot) {
          const int oa = R.layout == IPD_ROPE_HALF ? i : 2 * i;
          const int ob = R.layout == IPD_ROPE_HALF ? i + n_rot : 2 * i + 1;
          const T ra = d.src[oa], rb = d.src[ob];
          T wa = ra, wb = rb;
          if (d.turn) {
            const float2 t = __ldg(cs + i);
            const float sn = R.sign * t.y, p = Vec<T>::get(&ra), q = Vec<T>::get(&rb);
            Vec<T>::put(&wa, p * t.x - q * sn);
            Vec<T>::put(&wb, q * t.x + p * sn);
          }
          d.dst[oa] = wa;
          d.dst[ob] = wb;
          if (d.dst2) d.dst2[oa] = wa, d.dst2[ob] = wb;
        } else {
          const int o = R.rot + 2 * (i - n_rot);
          for (int e = o; e < o + 2 && e < D; ++e) {
            const T v = d.src[e];
            d.dst[e] = v;
            if (d.dst2) d.dst2[e] = v;
          }
        }
      }
    }
  }
}

template <typename T>
struct HeadIO {
  const T *src;
  T *dst, *dst2;
  bool turn;
};

template <typename T>
struct RopeParams {
  const T *x;
  T *y;
  long long x_stride, y_stride;
  const int32_t *pos;
  Rot rot;
  int n, heads, D, split;  // split: warps per token
  int units, hsplit;       // lanes: units x hsplit heads at once
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const RopeParams<T> P) {
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
  const long long tok = w / P.split;
  if (tok >= P.n) return;
  const int part = (int)(w % P.split);
  const int pos = P.pos[tok];
  if (pos < 0 || pos >= P.rot.max_pos) {
    if (lane == 0) ipd_set_error(&g_rope_err, IPD_DEVERR_POSITION);
    return;
  }
  const int unit = lane % P.units, hs = lane / P.units;
  if (hs >= P.hsplit) return;
  const T *x = P.x + tok * P.x_stride;
  T *y = P.y + tok * P.y_stride;
  const int D = P.D;
  rotate_heads<T, VEC>(P.rot, pos, D, P.heads, part * P.hsplit + hs, P.hsplit * P.split, unit,
                       P.units, [&](int h) {
                         return HeadIO<T>{x + (long long)h * D, y + (long long)h * D, nullptr, true};
                       });
}

struct AppendParams {
  ipd_rope_append_desc d;
  Rot rot;
  int split;
};

// Heads of a token in the order q, k, v; each goes to its place: q_out, the
// cache's page slot (and k_out), the page slot.
template <bool VEC>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(
    const __grid_constant__ AppendParams P) {
  constexpr int D = 128, kUnits = VEC ? 8 : 32, kHs = 32 / kUnits;
  const ipd_rope_append_desc &A = P.d;
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
  const long long tok = w / P.split;
  if (tok >= A.total_new) return;
  const int part = (int)(w % P.split);
  // the request holding the row: the last r with cu_new[r] <= tok, by a
  // 32-way search of the whole warp (two rounds for up to 1024 requests)
  int r = 0, n = A.num_reqs;
  bool covered = true;
  while (true) {
    const int step = ceil_div(n, 32), i = r + lane * step;
    const bool le = lane * step < n && A.cu_new[i] <= tok;
    const int cnt = __popc(__ballot_sync(0xffffffffu, le));
    if (cnt == 0) {
      covered = false;
      break;
    }
    r += (cnt - 1) * step;
    n = min(step, n - (cnt - 1) * step);
    if (step == 1) break;
  }
  int c0 = 0, c1 = 0;
  if (covered) c0 = A.cu_new[r], c1 = A.cu_new[r + 1];
  if (!covered || tok < c0 || tok >= c1) {  // a row that no request's offsets cover
    if (lane == 0) ipd_set_error(&g_rope_err, IPD_DEVERR_SPAN);
    return;
  }
  const int len = A.seq_len[r];
  const long long p = (long long)len - c1 + tok;  // its position
  if (p < 0 || (p >> 4) >= A.max_pages) {
    if (lane == 0) ipd_set_error(&g_rope_err, IPD_DEVERR_SEQ_LEN);
    return;
  }
  if (p >= P.rot.max_pos) {
    if (lane == 0) ipd_set_error(&g_rope_err, IPD_DEVERR_POSITION);
    return;
  }
  const int page = A.page_table[(size_t)r * A.max_pages + (p >> 4)];
  if (page < 0 || page >= A.num_pages) {
    if (lane == 0) ipd_set_error(&g_rope_err, IPD_DEVERR_PAGE_ID);
    return;
  }
  const uint16_t *q = A.q + tok * A.q_stride;
  const uint16_t *k = A.k + tok * A.k_stride;
  const uint16_t *v = A.v + tok * A.v_stride;
  uint16_t *qo = A.q_out + tok * A.q_out_stride;
  uint16_t *ko = A.k_out ? A.k_out + tok * A.k_out_stride : nullptr;
  const int hq = A.num_q_heads, hkv = A.num_kv_heads;
  const size_t slot = ((size_t)page * hkv * 16 + (p & 15)) * D;
  rotate_heads<uint16_t, VEC>(
      P.rot, (int)p, D, hq + 2 * hkv, part * kHs + lane / kUnits, kHs * P.split, lane % kUnits,
      kUnits, [&](int h) {
        if (h < hq) return HeadIO<uint16_t>{q + h * D, qo + h * D, nullptr, true};
        if (h < hq + hkv) {
          const int j = h - hq;
          return HeadIO<uint16_t>{k + j * D, A.k_pages + slot + (size_t)j * 16 * D,
                                  ko ? ko + j * D : nullptr, true};
        }
        const int j = h - hq - hkv;
        return HeadIO<uint16_t>{v + j * D, A.v_pages + slot + (size_t)j * 16 * D, nullptr, false};
      });
}

struct TableParams {
  double freq[kMaxFreqs];
  double mag;
  float2 *table;
  long long total;
  int half;
};

// The angle is formed and reduced in 64 bits: a position in the hundred
// thousands times a frequency near 1 leaves an fp32 angle no correct digits
// after the second decimal.
__global__ void __launch_bounds__(256) rope_table_kernel(const __grid_constant__ TableParams P) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < P.total;
       i += (long long)gridDim.x * 256) {
    double s, c;
    sincos((double)(i / P.half) * P.freq[i % P.half], &s, &c);
    P.table[i] = make_float2((float)(c * P.mag), (float)(s * P.mag));
  }
}

// Warps that share a token's heads: one where tokens alone give every SM some
// warps, else as many as do, at most one per group of heads a warp takes at
// once.  Aiming at 24 warps an SM instead of 8 makes 553 tokens of 40 heads take
// 5.7 us for 4.1 (each warp repeats the search), and aiming at 4 gains nothing.
int head_split(long long tokens, int heads, int hsplit) {
  const long long want = (kTargetWarps + tokens - 1) / tokens;
  const int most = ceil_div(heads, hsplit);
  return (int)(want < 1 ? 1 : (want < most ? want : most));
}

int check_rot(const float *table, int max_pos, int rot_dim, int layout, int head_dim) {
  if (max_pos < 1 || rot_dim < 2 || rot_dim > head_dim || rot_dim % 2 ||
      (layout != IPD_ROPE_HALF && layout != IPD_ROPE_INTERLEAVED))
    return IPD_ERR_INVALID_ARG;
  return table && !((uintptr_t)table & 15) ? IPD_OK : IPD_ERR_INVALID_ARG;
}

template <typename T>
int launch_rope(const ipd_rope_args &a, cudaStream_t st) {
  constexpr int N = Vec<T>::N;
  const uintptr_t bases = (uintptr_t)a.x | (uintptr_t)a.y;
  if (bases & (sizeof(T) - 1)) return IPD_ERR_INVALID_ARG;
  // 16-byte units need aligned rows and heads, a head of whole units and a
  // rotated part of whole units; and a table row that starts on 16 bytes
  const bool vec = !(bases & 15) && a.x_stride % N == 0 && a.y_stride % N == 0 &&
                   a.head_dim % (2 * N) == 0 && a.rot_dim % (2 * N) == 0;
  RopeParams<T> P;
  P.x = static_cast<const T *>(a.x);
  P.y = static_cast<T *>(a.y);
  P.x_stride = a.x_stride;
  P.y_stride = a.y_stride;
  P.pos = a.pos;
  P.rot = Rot{reinterpret_cast<const float2 *>(a.table), a.max_pos, a.rot_dim, a.layout,
              a.inverse ? -1.f : 1.f};
  P.n = a.n_tokens;
  P.heads = a.n_heads;
  P.D = a.head_dim;
  P.units = vec ? a.head_dim / (2 * N) : 32;
  P.hsplit = vec ? 32 / P.units : 1;
  P.split = head_split(a.n_tokens, a.n_heads, P.hsplit);
  const long long warps = (long long)a.n_tokens * P.split;
  const unsigned grid = (unsigned)((warps + kRopeWarps - 1) / kRopeWarps);
  g_rope_used.store(true, std::memory_order_relaxed);
  if (vec) rope_kernel<T, true><<<grid, kRopeThreads, 0, st>>>(P);
  else rope_kernel<T, false><<<grid, kRopeThreads, 0, st>>>(P);
  return cudaGetLastError() == cudaSuccess ? IPD_OK : IPD_ERR_CUDA;
}

}  // namespace

extern "C" __attribute__((visibility("hidden"))) unsigned int ipd_internal_take_rope_error() {
  if (!g_rope_used.load(std::memory_order_relaxed)) return 0u;
  unsigned int v = 0, z = 0;
  if (cudaMemcpyFromSymbol(&v, g_rope_err, sizeof(v)) != cudaSuccess) return 0xffffffffu;
  if (cudaMemcpyToSymbol(g_rope_err, &z, sizeof(z)) != cudaSuccess) return 0xffffffffu;
  return v;
}

extern "C" int ipd_rope_table(float *table, int max_pos, int rot_dim,
                              const ipd_rope_scaling *scaling, ipd_stream_t stream) {
  if (max_pos < 1 || rot_dim < 2 || rot_dim % 2 || !scaling || !table ||
      ((uintptr_t)table & 15))
    return IPD_ERR_INVALID_ARG;
  if (rot_dim > 2 * kMaxFreqs) return IPD_ERR_UNSUPPORTED;
  const ipd_rope_scaling &s = *scaling;
  if (!(s.base > 1.0) || !isfinite(s.base)) return IPD_ERR_INVALID_ARG;
  if (s.kind < IPD_ROPE_SCALE_NONE || s.kind > IPD_ROPE_SCALE_YARN) return IPD_ERR_INVALID_ARG;
  if (s.kind != IPD_ROPE_SCALE_NONE && (!(s.factor >= 1.0) || !isfinite(s.factor)))
    return IPD_ERR_INVALID_ARG;
  if (s.kind == IPD_ROPE_SCALE_NTK && rot_dim <= 2) return IPD_ERR_INVALID_ARG;
  if (s.kind == IPD_ROPE_SCALE_YARN &&
      (!(s.trained_len > 0.0) || !isfinite(s.trained_len) || !(s.beta_slow > 0.0) ||
       !(s.beta_fast >= s.beta_slow) || !isfinite(s.beta_fast)))
    return IPD_ERR_INVALID_ARG;
  TableParams P;
  memset(&P, 0, sizeof(P));
  const int half = rot_dim / 2;
  const double rot = rot_dim;
  double base = s.base;
  if (s.kind == IPD_ROPE_SCALE_NTK) base *= pow(s.factor, rot / (rot - 2.0));
  for (int i = 0; i < half; ++i) P.freq[i] = pow(base, -2.0 * i / rot);
  P.mag = 1.0;
  if (s.kind == IPD_ROPE_SCALE_LINEAR)
    for (int i = 0; i < half; ++i) P.freq[i] /= s.factor;
  if (s.kind == IPD_ROPE_SCALE_YARN) {
    // the index whose frequency turns `beta` times over the trained length
    const double two_pi = 6.283185307179586, ln_base = log(base);
    const auto at = [&](double beta) {
      return rot * log(s.trained_len / (beta * two_pi)) / (2.0 * ln_base);
    };
    const double lo = fmax(floor(at(s.beta_fast)), 0.0),
                 hi = fmin(ceil(at(s.beta_slow)), rot - 1.0), width = fmax(hi - lo, 1e-3);
    for (int i = 0; i < half; ++i) {
      const double ramp = fmin(fmax((i - lo) / width, 0.0), 1.0);
      P.freq[i] = P.freq[i] / s.factor * ramp + P.freq[i] * (1.0 - ramp);
    }
    P.mag = 0.1 * log(s.factor) + 1.0;
  }
  P.table = reinterpret_cast<float2 *>(table);
  P.half = half;
  P.total = (long long)max_pos * half;
  const long long blocks = (P.total + 255) / 256;
  rope_table_kernel<<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0,
                      reinterpret_cast<cudaStream_t>(stream)>>>(P);
  return cudaGetLastError() == cudaSuccess ? IPD_OK : IPD_ERR_CUDA;
}

extern "C" int ipd_rope(const ipd_rope_args *args, ipd_stream_t stream) {
  if (!args) return IPD_ERR_INVALID_ARG;
  const ipd_rope_args &a = *args;
  if (a.n_tokens < 0 || a.n_heads < 1 || a.head_dim < 2 ||
      (a.dtype != IPD_DTYPE_F32 && a.dtype != IPD_DTYPE_BF16))
    return IPD_ERR_INVALID_ARG;
  if (a.head_dim > 256 || a.n_heads > 65536) return IPD_ERR_UNSUPPORTED;
  if (a.n_tokens == 0) return IPD_OK;
  const int st = check_rot(a.table, a.max_pos, a.rot_dim, a.layout, a.head_dim);
  if (st != IPD_OK) return st;
  const long long row = (long long)a.n_heads * a.head_dim;
  if (!a.x || !a.y || !a.pos || a.x_stride < row || a.y_stride < row) return IPD_ERR_INVALID_ARG;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return a.dtype == IPD_DTYPE_BF16 ? launch_rope<uint16_t>(a, s) : launch_rope<float>(a, s);
}

extern "C" int ipd_rope_append(const ipd_rope_append_desc *desc, ipd_stream_t stream) {
  if (!desc) return IPD_ERR_INVALID_ARG;
  const ipd_rope_append_desc &a = *desc;
  if (a.num_reqs < 0 || a.total_new < 0 || a.num_pages < 0 || a.num_kv_heads < 1 ||
      a.num_q_heads < 0 || a.max_pages < 1)
    return IPD_ERR_INVALID_ARG;
  if (a.page_size != 16 || a.head_dim != 128) return IPD_ERR_UNSUPPORTED;
  if (a.num_q_heads > 65536 || a.num_kv_heads > 65536) return IPD_ERR_UNSUPPORTED;
  if (a.total_new == 0) return IPD_OK;
  const int st = check_rot(a.table, a.max_pos, a.rot_dim, a.layout, a.head_dim);
  if (st != IPD_OK) return st;
  const long long qrow = 128ll * a.num_q_heads, krow = 128ll * a.num_kv_heads;
  const bool has_q = a.num_q_heads > 0;
  if (a.num_reqs == 0 || !a.k || !a.v || !a.k_pages || !a.v_pages || !a.cu_new || !a.seq_len ||
      !a.page_table || (has_q && (!a.q || !a.q_out)))
    return IPD_ERR_INVALID_ARG;
  if (a.k_stride < krow || a.v_stride < krow || (a.k_out && a.k_out_stride < krow) ||
      (has_q && (a.q_stride < qrow || a.q_out_stride < qrow)))
    return IPD_ERR_INVALID_ARG;
  uintptr_t align = (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.k_pages | (uintptr_t)a.v_pages |
                    (uintptr_t)a.k_out | (uintptr_t)(2 * a.k_stride) | (uintptr_t)(2 * a.v_stride);
  if (has_q)
    align |= (uintptr_t)a.q | (uintptr_t)a.q_out | (uintptr_t)(2 * a.q_stride) |
             (uintptr_t)(2 * a.q_out_stride);
  if (a.k_out) align |= (uintptr_t)(2 * a.k_out_stride);
  if (align & 15) return IPD_ERR_INVALID_ARG;
  AppendParams P;
  P.d = a;
  if (!has_q) P.d.q_stride = P.d.q_out_stride = 0;
  P.rot = Rot{reinterpret_cast<const float2 *>(a.table), a.max_pos, a.rot_dim, a.layout, 1.f};
  const bool vec = a.rot_dim % 16 == 0;
  P.split = head_split(a.total_new, a.num_q_heads + 2 * a.num_kv_heads, vec ? 4 : 1);
  const long long warps = (long long)a.total_new * P.split;
  const unsigned grid = (unsigned)((warps + kRopeWarps - 1) / kRopeWarps);
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  g_rope_used.store(true, std::memory_order_relaxed);
  if (vec) rope_append_kernel<true><<<grid, kRopeThreads, 0, s>>>(P);
  else rope_append_kernel<false><<<grid, kRopeThreads, 0, s>>>(P);
  return cudaGetLastError() == cudaSuccess ? IPD_OK : IPD_ERR_CUDA;
}

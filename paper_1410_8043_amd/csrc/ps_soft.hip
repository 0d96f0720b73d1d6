// Operators over a whole item table (include/ps_soft.h): softmax cross entropy and distillation
// with the gradients of both tables, and each row's k best items.
//
// The mathematics.  With s_ij = x_i . w_j, both losses need, per row i, lse_i and the mean
// o_i = sum_j p_ij w_j of the items under the row's softmax, and, per item j, the sum
// c_j = sum_i a_i p_ij x_i with a_i the row's share of the gradient.  The targets add sparse
// terms: their scores for the loss, coef w_j to dX_i and coef x_i to dW_j.  So there are two dense
// passes of one shape (k_pass): an OWN table whose rows stay in registers, a STREAM table that goes
// by in tiles of 32 rows; a tile's scores come from matrix instructions, the weights p' = 2^(score -
// reference) stay in the registers where the next matrix instruction wants them, and that one
// adds p' times the tile's rows to the own rows' sums.  Rows over items carry the running sum
// of p' (the softmax's), items over rows know each row's lse already and multiply by a_i.
//
// Numbers.  Matrix instructions of 16-bit floats with 32-bit sums: a table is scaled by a power of two
// so that its largest number lies in [2^13, 2^14) and is held as one plane of fp16 (bf16 and
// f16 tables: exact for all numbers above 2^-28 of the largest) or as two, h = fp16(x), l =
// fp16(x - h) (f32 tables: 22 bits, to 2^-38 of the largest below that), and products drop l*l
// (2^-22).  The weights p' are held in two planes too.  Sums over items and rows, running maxima and log-sum-exps
// are fp32.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <new>
#include <string>
#include <type_traits>
#include <vector>

#include "../../include/ps_soft.h"
#include "soft_plan.h"

namespace {

using namespace pssoft;

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kPackBlocks = 8;  // blocks of 32 numbers that packing holds in LDS at once
constexpr float kNone = -3e38f; // reference before the first tile: below all scores, and finite, so that 2^(-inf - kNone) is 0
// p' = 2^(score - reference + kShift), and the reference follows the maximum when it is exceeded by more than
// kLag: p' stays below 2^15, and a weight of 2^-17 of the largest keeps 22 bits
constexpr float kShift = 7.f, kLag = 8.f;
constexpr float kFar = -120.f;  // least reference of an item with targets: 2^(kShift - reference) is a finite number

// A launch holds less than 2^32 threads in a dimension: workgroups beyond 2^22 go to the second
constexpr int kGridBits = 22;
__device__ inline int32_t block_index() { return static_cast<int32_t>(blockIdx.y << kGridBits | blockIdx.x); }

// ------------------------------------------------------------------ element types
struct bf16_t { uint16_t u; };
struct f16_t { _Float16 h; };
__device__ inline float to_f(float v) { return v; }
__device__ inline float to_f(bf16_t v) { return __uint_as_float(static_cast<uint32_t>(v.u) << 16); }
__device__ inline float to_f(f16_t v) { return static_cast<float>(v.h); }
__device__ inline void from_f(float v, float &o) { o = v; }
__device__ inline void from_f(float v, bf16_t &o) {
  const uint32_t u = __float_as_uint(v);
  o.u = v != v ? 0x7fc0 : static_cast<uint16_t>((u + 0x7fff + ((u >> 16) & 1)) >> 16);  // to nearest, ties to even
}
__device__ inline void from_f(float v, f16_t &o) { o.h = static_cast<_Float16>(v); }

// K numbers k0 .. k0+3 of a row as floats, zeros behind K; vec: the row starts at a multiple of 4 elements' bytes
template <class T>
__device__ inline f32x4 load4(const T *row, int k0, int K, bool vec) {
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  if (vec && k0 + 4 <= K) {
    if constexpr (sizeof(T) == 4) {
      o = *reinterpret_cast<const f32x4 *>(row + k0);
    } else {
      const u16x4 v = *reinterpret_cast<const u16x4 *>(row + k0);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        T t;
        __builtin_memcpy(&t, reinterpret_cast<const char *>(&v) + 2 * q, 2);
        o[q] = to_f(t);
      }
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (k0 + q < K) o[q] = to_f(row[k0 + q]);
  }
  return o;
}
template <class T>
__device__ inline void store4(T *row, int k0, int K, bool vec, f32x4 v) {
  T t[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) from_f(v[q], t[q]);
  if (vec && k0 + 4 <= K) {
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<f32x4 *>(row + k0) = v;
    } else {
      u16x4 o;
      __builtin_memcpy(&o, t, 8);
      *reinterpret_cast<u16x4 *>(row + k0) = o;
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (k0 + q < K) row[k0 + q] = t[q];
  }
}

__device__ inline float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ inline float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}
__device__ inline float block_max(float v, float *sh) {  // kThreads threads; sh: 4 floats
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  return fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
}

// ------------------------------------------------------------------ targets
// A call's rows and targets before the passes.  Where dW is wanted, each entry of the lists also becomes a record for
// the pass over rows: key, the tile of 32 items that its item lies in (or `dead`, one behind the last), and a
// payload of row * 32 + item mod 32 and its share weight tau coef of the gradients.
struct Targets {
  int64_t n, entries;
  int32_t items, k, dead;    // k: entries per row without row_ptr
  const int64_t *row_ptr;
  const int32_t *item;
  const float *value;        // xent
  const float *score, *tlse; // distill
  int64_t ldt;
  float tau;
  double per_tau;            // 1 / tau
  const float *weight;
  int32_t *key;              // NULL: no dW
  uint2 *pay;
  int32_t *act;                             // [n] 0: masked
  float *total, *extra, *share, *gw;        // [n] sum of coef; sum q log q (NaN: a bad row); gw total; weight tau
  double *logz;                             // [n] the teacher's log-sum-exp
  float *part;                              // [gridDim.x] largest |gw| sum |coef|
};

// log q of a teacher's score, z the log-sum-exp over tau.  In 64 bits: both may be far larger than their difference (scores
// of 3000 in fp32 put q off by 1e-4)
__device__ inline float log_q(const Targets &a, float score, double z) { return static_cast<float>(fma(static_cast<double>(score), a.per_tau, -z)); }

__device__ inline bool row_range(const int64_t *row_ptr, int64_t entries, int32_t k, int64_t i, int64_t &b, int64_t &e) {
  if (!row_ptr) {
    b = i * k;
    e = b + k;
    return true;
  }
  b = row_ptr[i];
  e = row_ptr[i + 1];
  if (b < 0 || e < b || e > entries) {
    b = e = 0;
    return false;
  }
  return true;
}

__global__ __launch_bounds__(kThreads) void k_fill_keys(int32_t *key, int64_t entries, int32_t dead) {
  for (int64_t e = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; e < entries; e += static_cast<int64_t>(gridDim.x) * kThreads)
    key[e] = dead;
}

// One wavefront per row.  Bound by the reads of the lists and the writes of the records (16,384 rows, 3.4M entries: 27 us,
// 2.5 TB/s).
template <bool Distill>
__global__ __launch_bounds__(kThreads) void k_targets(Targets a) {
  __shared__ float sh[4];
  const int lane = threadIdx.x & 63;
  const int64_t step = static_cast<int64_t>(gridDim.x) * 4;
  const float inf = __builtin_inff();
  float most = 0.f;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6); i < a.n; i += step) {
    int64_t b, e;
    bool bad = !row_range(a.row_ptr, a.entries, a.k, i, b, e);
    const int64_t src = Distill ? i * a.ldt - b : 0;  // the lists' stride
    const float w = a.weight ? a.weight[i] : 1.f;
    double z = 0.0;  // log of the teacher's sum
    if constexpr (Distill) {
      bool some = false;
      float top = -inf;
      for (int64_t x = b + lane; x < e; x += 64) {
        const int32_t j = a.item[x + src];
        const float t = j >= 0 && j < a.items ? a.score[x + src] : -inf;
        if (!(t == -inf)) {
          some = true;
          top = t != t ? t : fmaxf(top, t);
        }
      }
      if (__any(some)) {
        if (a.tlse) {
          z = a.tlse[i];
        } else {
          top = wave_max(top);
          float den = 0.f;
          for (int64_t x = b + lane; x < e; x += 64) {
            const int32_t j = a.item[x + src];
            const float t = j >= 0 && j < a.items ? a.score[x + src] : -inf;
            if (!(t == -inf)) den += expf(log_q(a, t, top * a.per_tau));
          }
          z = top * a.per_tau + log(static_cast<double>(wave_sum(den)));
        }
      }
    }
    bool live = false;
    float total = 0.f, size = 0.f, extra = 0.f;
    float gw = w * a.tau;
    for (int64_t x = b + lane; x < e; x += 64) {
      const int32_t j = a.item[x + src];
      bad = bad || j >= a.items;
      bool here = j >= 0 && j < a.items;
      float c = 0.f;
      if (here) {
        if constexpr (Distill) {
          const float t = a.score[x + src];
          here = !(t == -inf);
          const float lq = log_q(a, t, z);
          c = here ? expf(lq) : 0.f;
          extra += c == 0.f ? 0.f : c * lq;
        } else {
          c = a.value ? a.value[x] : 1.f;
        }
      }
      live = live || here;
      if (a.key) {
        a.key[x] = here && w != 0.f ? j >> 5 : a.dead;
        a.pay[x] = make_uint2(static_cast<uint32_t>(i) << 5 | (j & 31), __float_as_uint(gw * c));
      }
      total += c;
      size += fabsf(c);
    }
    const bool act = __any(live) && w != 0.f;
    bad = __any(bad);
    if (!act) gw = total = size = extra = 0.f;
    total = wave_sum(total);
    extra = wave_sum(extra);
    size = fabsf(gw) * wave_sum(size);
    most = fmaxf(most, size < inf ? size : 0.f);
    if (lane == 0) {
      a.act[i] = act;
      a.total[i] = total;
      a.extra[i] = bad ? __builtin_nanf("") : extra;
      a.share[i] = gw * total;
      a.gw[i] = gw;
      if constexpr (Distill) a.logz[i] = z;
    }
  }
  most = block_max(most, sh);
  if (threadIdx.x == 0) a.part[blockIdx.x] = most;
}

// ------------------------------------------------------------------ packing
template <class T>
struct Table {
  const T *p;
  int64_t ld, rows;
  bool vec;
  const int32_t *act;  // rows that are read (NULL: all)
};

// Largest finite magnitude of each table, kParts partial maxima each.  A row's numbers by as many lanes as its float4s,
// rounded up to a power of two; bound by memory and by latency (55 MB in 20 us, 2.7 TB/s; with a
// division per float4 it was 0.9).
constexpr int kScanThreads = 1024;
template <class T>
__global__ __launch_bounds__(kScanThreads) void k_absmax(Table<T> x, Table<T> w, int32_t K, int32_t lanes, float *part) {
  __shared__ float sh[kScanThreads / 64];
  const bool second = blockIdx.x >= kParts;
  const Table<T> t = second ? w : x;
  const int blk = blockIdx.x - (second ? kParts : 0);
  const int k0 = (threadIdx.x & (lanes - 1)) * 4, rows = kScanThreads / lanes;
  const int64_t step = static_cast<int64_t>(kParts) * rows;
  const float inf = __builtin_inff();
  float most = 0.f;
  if (k0 < K) {
#pragma unroll 4
    for (int64_t r = static_cast<int64_t>(blk) * rows + threadIdx.x / lanes; r < t.rows; r += step) {
      if (t.act && !t.act[r]) continue;
      const f32x4 v = load4(t.p + r * t.ld, k0, K, t.vec);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float m = fabsf(v[c]);
        most = fmaxf(most, m < inf ? m : 0.f);
      }
    }
  }
  most = wave_max(most);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = most;
  __syncthreads();
  if (threadIdx.x < 64) {
    most = wave_max(threadIdx.x < kScanThreads / 64 ? sh[threadIdx.x] : 0.f);
    if (threadIdx.x == 0) part[blockIdx.x] = most;
  }
}

__device__ inline int scale_exp(float most) {
  if (!(most > 0.f)) return 0;
  int e;
  (void)frexpf(most, &e);  // most in [2^(e-1), 2^e)
  return 14 - e;
}

// Scalars that the kernels share
struct Scal {
  int32_t ex, ew;  // x~ = x 2^ex, w~ = w 2^ew
  float amax;      // a power of two >= 2 |gw| sum |coef| of every row (1 where all are 0): shares and targets are taken by it
  float pad;
};
static_assert(sizeof(Scal) == kScalBytes, "the workspace's plan");

// log2 of the weights per unit of the packed tables' scores; scale: log2(e) / tau.  Not 0, so that -inf stays
__device__ inline float unit_of(const Scal *scal, float scale) { return fmaxf(ldexpf(scale, -(scal->ex + scal->ew)), 0x1p-126f); }

struct PackSide {
  _Float16 *out;
  int64_t stride;  // halves per tile
  int32_t tiles;
  bool turned;     // the turned fragments too
};

// A tile of 32 rows as fragments: for the scores, chunk c of 16 numbers, lane l holds row l%32, numbers
// 16c + 8(l/32) ..+7; and turned, for the sums, rows 16q ..+15 and numbers 32b ..+31: lane l holds
// number 32b + l%32 of the rows that the score instruction leaves in this lane's registers
// 8q .. 8q+7, 16q + {4h ..+3, 8 + 4h ..+3} with h = l/32: so weights go from one matrix instruction to
// the next without a move.  One workgroup per tile; bound by memory (8192 + 100,000 rows, K = 256 bf16: 165 MB in 32 us,
// 5.2 TB/s).
template <class T, int NP>
__global__ __launch_bounds__(kThreads) void k_pack(Table<T> x, Table<T> w, PackSide px, PackSide pw, int32_t K, int32_t k16,
                                                   int32_t kd, const float *part, const float *row_part, int32_t row_parts,
                                                   Scal *scal) {
  extern __shared__ float tile[];  // [32][32 min(kd, kPackBlocks) + 1]
  __shared__ float sh[4];
  const int32_t block = block_index();
  const bool second = block >= px.tiles;
  const Table<T> t = second ? w : x;
  const PackSide ps = second ? pw : px;
  const int64_t at = static_cast<int64_t>(block) - (second ? px.tiles : 0);
  if (at >= ps.tiles) return;
  const float most = block_max(part[(second ? kParts : 0) + threadIdx.x], sh);
  const int ex = scale_exp(most);
  if (at == 0) {
    if (threadIdx.x == 0) (second ? scal->ew : scal->ex) = ex;
    if (!second) {
      float m = 0.f;
      for (int q = threadIdx.x; q < row_parts; q += kThreads) m = fmaxf(m, row_part[q]);
      __syncthreads();
      m = block_max(m, sh);
      if (threadIdx.x == 0) scal->amax = m > 0.f ? ldexpf(1.f, min(max(15 - scale_exp(m), -100), 126)) : 1.f;
    }
  }
  _Float16 *out = ps.out + at * ps.stride;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
  const int wide = min(kd, kPackBlocks), ld = wide * 32 + 1;
  for (int b0 = 0; b0 < kd; b0 += wide) {  // 256 numbers at a time: 33 KB of LDS
    const int nb = min(wide, kd - b0), per = nb * 8;  // float4s per row
    __syncthreads();
    for (int q = threadIdx.x; q < kTile * per; q += kThreads) {
      const int r = q / per, k0 = (q - r * per) * 4;
      const int64_t row = at * kTile + r;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      if (row < t.rows && b0 * 32 + k0 < K && (!t.act || t.act[row])) v = load4(t.p + row * t.ld, b0 * 32 + k0, K, t.vec);
#pragma unroll
      for (int c = 0; c < 4; ++c) tile[r * ld + k0 + c] = ldexpf(v[c], ex);
    }
    __syncthreads();
    for (int c = 2 * b0 + wave; c < min(2 * (b0 + nb), k16); c += 4) {
      h8 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = tile[l32 * ld + (c - 2 * b0) * 16 + half * 8 + i];
        hi[i] = static_cast<_Float16>(v);
        lo[i] = static_cast<_Float16>(v - static_cast<float>(hi[i]));
      }
      *reinterpret_cast<h8 *>(out + (c * NP) * kFrag + lane * 8) = hi;
      if constexpr (NP == 2) *reinterpret_cast<h8 *>(out + (c * NP + 1) * kFrag + lane * 8) = lo;
    }
    if (!ps.turned) continue;
    for (int f = wave; f < 2 * nb; f += 4) {
      const int q = f / nb, b = f - q * nb;
      h8 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = tile[(q * 16 + (i >> 2) * 8 + half * 4 + (i & 3)) * ld + b * 32 + l32];
        hi[i] = static_cast<_Float16>(v);
        lo[i] = static_cast<_Float16>(v - static_cast<float>(hi[i]));
      }
      _Float16 *to = out + (k16 + q * kd + b0 + b) * NP * kFrag + lane * 8;
      *reinterpret_cast<h8 *>(to) = hi;
      if constexpr (NP == 2) *reinterpret_cast<h8 *>(to + kFrag) = lo;
    }
  }
}

// ------------------------------------------------------------------ the dense passes
struct PassArgs {
  const _Float16 *own, *str;
  int64_t own_stride, str_stride;  // halves per tile
  int64_t own_tiles, str_rows;
  int32_t d0;                      // the first block of 32 numbers summed here
  int32_t splits;                  // pieces of the stream
  const float *rowvec;             // COL: per tile of 32 stream rows, 32 powers of two and 32 factors (see k_row_finish)
  const Scal *scal;
  float scale;                     // log2(e) / tau
  int64_t tiles_per_split;
  const int64_t *first;            // COL: where the records of each own tile start ([own tiles + 1], NULL: none)
  const uint2 *pay;                // sorted by own tile, then row
  float *m, *l, *o;                // [splits][own rows padded]: reference (COL: in powers of two; else a packed tables' score), sum of p', sums [..][32 kd]
};

__device__ inline f32x16 mfma(h8 a, h8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

// From memory to LDS without registers: lane l's 16 (4) bytes at `from` go to `to` + 16 (4) l; `to` is the wavefront's
typedef const __attribute__((address_space(1))) uint32_t *global_ptr;
typedef __attribute__((address_space(3))) uint32_t *lds_ptr;
__device__ inline void to_lds16(const void *from, void *to) {
  __builtin_amdgcn_global_load_lds(reinterpret_cast<global_ptr>(reinterpret_cast<uintptr_t>(from)), (lds_ptr)to, 16, 0, 0);
}
__device__ inline void to_lds4(const void *from, void *to) {
  __builtin_amdgcn_global_load_lds(reinterpret_cast<global_ptr>(reinterpret_cast<uintptr_t>(from)), (lds_ptr)to, 4, 0, 0);
}

// The rest of a number behind a half of `h`, p - h (one instruction: the half is read as it is).  On the rounded fp16
// number itself: a product and its rounding, fused at one of two uses, once gave a rest of another
// fp16 number (2^-11 off in a weight of a thousand)
__device__ inline float rest_low(uint32_t h, float p) {
  float r;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(p));
  return r;
}
__device__ inline float rest_high(uint32_t h, float p) {
  float r;
  asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(p));
  return r;
}
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t to_halves(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, h2));
}
// Both planes of two weights
__device__ inline void planes(float a, float b, uint32_t &h, uint32_t &l) {
  h = to_halves(a, b);
  l = to_halves(rest_low(h, a), rest_high(h, b));
}
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ inline h8 halves(u32x4 v) { return __builtin_bit_cast(h8, v); }

constexpr int kLds = 160 * 1024;
constexpr int kHalfTile = kTile * 16;  // floats of half a tile's targets

// LDS of a pass, in halves: tiles' fragments for the scores (one or two tiles), the turned ones (two), the row values of a
// pass over rows (four) and its wavefronts' targets
struct Stage {
  int scores, turned;   // fragments: for the scores, and the turned ones of each half of the tile's rows
  int score_tiles;      // tiles of score fragments
  int at_turned, at_rows, at_targets, halves;
};
__host__ __device__ constexpr Stage stage_of(int np, int kc, int db, bool col) {
  Stage s{};
  s.scores = kc * np;
  s.turned = db * np;
  const int rest = 2 * 2 * s.turned * kFrag + (col ? 4 * 128 + kWaves * kHalfTile * 2 : 0);
  s.score_tiles = (2 * s.scores * kFrag + rest) * 2 <= kLds ? 2 : 1;
  s.at_turned = s.score_tiles * s.scores * kFrag;
  s.at_rows = s.at_turned + 2 * 2 * s.turned * kFrag;
  s.at_targets = s.at_rows + (col ? 4 * 128 : 0);
  s.halves = s.at_turned + rest;
  return s;
}

// The sorted target records of one own tile, in windows of 64, one per lane, the next one read ahead
struct Window {
  const uint2 *pay;
  int left, pos;  // records from the lane's on (up to 2^31, so that a place and 64 more would not do)
  uint32_t due;   // the next record's row
  uint2 now, next;
  // a record behind the last: a row above all
  __device__ uint2 get(int lane, int ahead) const { return ahead < left ? pay[lane + ahead] : make_uint2(0xffffffffu, 0u); }
  __device__ void open(const uint2 *p, int64_t b, int64_t e, int lane) {
    pay = p + b;
    left = static_cast<int>(e - b) - lane;
    pos = 0;
    now = get(lane, 0);
    next = get(lane, 64);
    due = __builtin_amdgcn_readfirstlane(now.x) >> 5;
  }
  __device__ void step(int lane) {
    pay += 64;
    left -= 64;
    pos = 0;
    now = next;
    next = get(lane, 64);
  }
  __device__ void skip(int n, int lane) {  // n records are done
    pos += n;
    if (pos == 64) step(lane);
    due = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(now.x), pos)) >> 5;
  }
};

// The first of records [b, e) whose row is at least `row` (rows ascend): all lanes probe at once
__device__ inline int64_t first_of_row(const uint2 *pay, int64_t b, int64_t e, uint32_t row, int lane) {
  while (e - b > 0) {
    const int64_t step = (e - b + 63) / 64;
    const int64_t at = b + lane * step;
    const bool below = at < e && (pay[at].x >> 5) < row;
    const int n = __popcll(__ballot(below));  // lanes 0 .. n-1 are below
    if (n == 0) return b;
    const int64_t lo = b + (n - 1) * step + 1;
    e = min(b + n * step, e);
    b = lo;
  }
  return b;
}

// What targets are multiplied by for their place beside weights of that reference; any finite number where there are none
__device__ inline float up_to(float ref) { return __builtin_amdgcn_exp2f(fminf(kShift - ref, kShift - kFar)); }

// The largest of the two lanes that hold an own row
__device__ inline float of_both_halves(float v) {
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}

// Wavefronts per SIMD that the registers are cut for
constexpr int waves_per_simd(int np, int kc, int db) {
  const int need = 4 * kc * np + 16 * db;  // own rows and sums; a tile's scores, weights and fragments take 60 to 110 more
  return need <= 64 ? 3 : need <= 192 && np * kc < 24 ? 2 : 1;
}

// Rows over items (COL = false) or items over rows (COL = true).  A wavefront owns 32 rows; the stream's tiles go
// through LDS, shared by the workgroup, loaded one step ahead of their use.
// Score instruction: stream rows x own rows, so a lane holds one own row (l%32) and 16 stream rows
// 8(r/4) + 4h + r%4 of each tile.
// The weights have two planes whatever the tables' type: with one, 2^-11 of each weight, 6 of 100 numbers of a bf16
// gradient are rounded to the neighbour of the nearest.
// The matrix instructions bound rows over items (1.12 PFLOP/s of them at K = 128 fp32, 1.08 at K = 256 bf16; a large
// library product reaches 1.2), so the loop keeps them fed: the next tile's scores are made beside the exponentials of this one's,
// the sums beside the rounding.  Items over rows have the records and the factors besides (16,384 rows x 17,770 items, K = 128
// fp32, 400 / 557 us; 4096 x 100,000, K = 128 bf16, 337 / 388).  The tiles' way from L2 is a seventh to a fifth of it.  With items' weights of
// one plane (331 / 316 us then) were tried: 8 wavefronts a workgroup, which halve that way, 320 / 360; two own tiles a wavefront, which halve
// the reads of LDS too and leave one wavefront a SIMD, 421 / 458; reading further ahead the same.
template <int NP, int KC, int DB, bool COL>
__global__ __launch_bounds__(64 * kWaves, waves_per_simd(NP, KC, DB)) void k_pass(PassArgs a) {
  constexpr Stage sg = stage_of(NP, KC, DB, COL);
  constexpr int KD = KC / 2;
  extern __shared__ _Float16 buf[];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t block = block_index();
  const int split = block % a.splits;
  const int64_t own_tile = static_cast<int64_t>(block / a.splits) * kWaves + wave;
  if (own_tile - wave >= a.own_tiles) return;
  const int64_t tiles = (a.str_rows + kTile - 1) / kTile;
  const int t0 = static_cast<int>(split * a.tiles_per_split);
  const int t1 = static_cast<int>(min(t0 + a.tiles_per_split, tiles));
  const float sc = unit_of(a.scal, a.scale);
  const bool live = own_tile < a.own_tiles;  // the last workgroup's wavefronts behind the last row only help loading
  auto fetch_scores = [&](int t) {
    const _Float16 *src = a.str + t * a.str_stride + lane * 8;
    _Float16 *to = buf + (sg.score_tiles == 2 ? (t & 1) * sg.scores * kFrag : 0);
#pragma unroll
    for (int f0 = 0; f0 < sg.scores; f0 += kWaves) {
      const int f = f0 + wave;
      if (sg.scores % kWaves != 0 && f >= sg.scores) break;
      to_lds16(src + f * kFrag, to + f * kFrag);
    }
  };
  auto fetch_turned = [&](int t) {
    const _Float16 *src = a.str + t * a.str_stride + (sg.scores + a.d0 * NP) * kFrag + lane * 8;
    _Float16 *to = buf + sg.at_turned + (t & 1) * 2 * sg.turned * kFrag;
#pragma unroll
    for (int f0 = 0; f0 < 2 * sg.turned; f0 += kWaves) {
      const int f = f0 + wave;
      if (2 * sg.turned % kWaves != 0 && f >= 2 * sg.turned) break;
      to_lds16(src + (f + (f >= sg.turned ? (KD - DB) * NP : 0)) * kFrag, to + f * kFrag);
    }
  };
  auto fetch_rows = [&](int t) {
    if (COL && wave == 0) to_lds4(a.rowvec + static_cast<int64_t>(t) * 64 + lane, buf + sg.at_rows + (t & 3) * 128);
  };
  // The reference of each own row follows the largest of its own weights, and an item's starts where all of its targets in this
  // piece together are 2^14 at most: so an item of small weights keeps 22 bits of them, whatever its neighbours' or the rows' shares
  // are.  (Asking each half tile's targets for their largest instead took 4 to 18% of a call.)
  float ref = kNone, sum = 0.f, lost = 0.f, unit = 0.f;
  bool targets = false;
  Window win;
  float *y = nullptr;
  if constexpr (COL) {
    y = reinterpret_cast<float *>(buf + sg.at_targets) + wave * kHalfTile;
#pragma unroll
    for (int r = 0; r < kHalfTile / 64; ++r) y[r * 64 + lane] = 0.f;
    if (a.first && live) {
      const int64_t b = first_of_row(a.pay, a.first[own_tile], a.first[own_tile + 1], static_cast<uint32_t>(t0) * kTile, lane);
      const int64_t e = a.first[own_tile + 1];
      win.open(a.pay, b, e, lane);
      targets = win.due < static_cast<uint32_t>(t1) * kTile;
    }
    if (targets) {
      unit = 1.f / a.scal->amax;
      // by item, 16 sums each so that few lanes meet at one
      const int64_t e = a.first[own_tile + 1];
      bool more = true;
      for (int64_t at = win.pay - a.pay + lane; more; at += 256) {
        uint2 r[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) r[u] = at + 64 * u < e ? a.pay[at + 64 * u] : make_uint2(0xffffffffu, 0u);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          more = (r[u].x >> 5) < static_cast<uint32_t>(t1) * kTile;
          if (more) atomicAdd(y + (r[u].x & 31) * 16 + (lane & 15), fabsf(__uint_as_float(r[u].y)) * unit);
        }
        more = __any(more);
      }
      __builtin_amdgcn_wave_barrier();
      f32x4 *const mine = reinterpret_cast<f32x4 *>(y + (lane & 31) * 16);
      const f32x4 v = (mine[0] + mine[1]) + (mine[2] + mine[3]);
      __builtin_amdgcn_wave_barrier();
      mine[0] = mine[1] = mine[2] = mine[3] = f32x4{0.f, 0.f, 0.f, 0.f};
      __builtin_amdgcn_wave_barrier();
      const float all = (v[0] + v[1]) + (v[2] + v[3]);
      if (all > 0.f) ref = fmaxf(__builtin_amdgcn_logf(all) - (14.f - kShift), kFar);
    }
  }
  h8 q[KC][NP];
  const _Float16 *own = a.own + own_tile * a.own_stride;
#pragma unroll
  for (int c = 0; c < KC; ++c)
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      q[c][p] = h8{0, 0, 0, 0, 0, 0, 0, 0};
      if (live) q[c][p] = *reinterpret_cast<const h8 *>(own + (c * NP + p) * kFrag + lane * 8);
    }
  f32x16 o[DB > 0 ? DB : 1];
#pragma unroll
  for (int b = 0; b < DB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[b][r] = 0.f;
  // Chunk c of a tile's score fragments, and step i of its turned ones (half i / DB, block i % DB)
  auto read_scores = [&](h8 (&f)[NP], int t, int c) {
    const _Float16 *from = buf + (sg.score_tiles == 2 ? (t & 1) * sg.scores * kFrag : 0) + c * NP * kFrag + lane * 8;
#pragma unroll
    for (int p = 0; p < NP; ++p) f[p] = *reinterpret_cast<const h8 *>(from + p * kFrag);
  };
  auto read_turned = [&](h8 (&f)[NP], int t, int i) {
    const _Float16 *from = buf + sg.at_turned + ((t & 1) * 2 * sg.turned + i * NP) * kFrag + lane * 8;
#pragma unroll
    for (int p = 0; p < NP; ++p) f[p] = *reinterpret_cast<const h8 *>(from + p * kFrag);
  };
  // An item's and a row's planes in the same order in both passes, so a score has equal bits in them: a weight that is nearly 1 in
  // the row's sum is that in the item's difference to its target
  auto add_scores = [&](f32x16 s, const h8 (&f)[NP], int c) {
    s = mfma(f[0], q[c][0], s);
    if constexpr (NP == 2) {
      s = mfma(f[COL], q[c][!COL], s);
      s = mfma(f[!COL], q[c][COL], s);
    }
    return s;
  };
  // Rows over items: the scores as they are, and the reference one of them, so that what the exponential gets is rounded at the
  // size of their difference (scaled scores rounded at their own size left weights near 1 2^-25 |score| off, and with them
  // the items' differences to their targets).  Items over rows: log2 weights, the score's and the row's power of two.  That is
  // added here: as the matrix instruction's first value, every one of its roundings would be at the size of the log-sum-exp
  auto row_values = [&](int t, int g, int which) {  // rows 8g + 4h ..+3: the powers of two, or the factors
    return *reinterpret_cast<const f32x4 *>(reinterpret_cast<const float *>(buf + sg.at_rows + (t & 3) * 128) + which * 32 + g * 8 + half * 4);
  };
  fetch_scores(t0);
  if constexpr (DB > 0) fetch_turned(t0);
  fetch_rows(t0);
  if (t0 + 1 < t1) {
    if (sg.score_tiles == 2) fetch_scores(t0 + 1);
    fetch_rows(t0 + 1);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  float p[16], top;
  const float lag = COL ? kLag : kLag / sc;
  auto weigh = [&](const f32x16 &s, int t) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 v = COL ? row_values(t, g, 0) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) p[4 * g + i] = COL ? fmaf(s[4 * g + i], sc, v[i]) : s[4 * g + i];
    }
    top = p[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, p[r]);
  };
  {
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      h8 f[NP];
      read_scores(f, t0, c);
      s = add_scores(s, f, c);
    }
    weigh(s, t0);
  }
  __syncthreads();  // all have read the first tile: the loop's first step loads over it
  if (sg.score_tiles == 1 && t0 + 1 < t1) {
    fetch_scores(t0 + 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  // Steps of matrix instructions whose fragments are read ahead, about 6 instructions (192 cycles)
  // (fewer where 256 numbers of one plane leave no registers)
  constexpr int SA = NP == 2 || KC >= 16 ? 2 : 4, TA = NP == 2 || KC >= 16 ? 2 : 3;
  for (int t = t0; t < t1; ++t) {
    if (t + 2 < t1) {
      if (sg.score_tiles == 2) fetch_scores(t + 2);
      fetch_rows(t + 2);
    }
    if (DB > 0 && t + 1 < t1) fetch_turned(t + 1);
    h8 f[KC + SA][NP];
#pragma unroll
    for (int c = 0; c < SA && c < KC; ++c) read_scores(f[c], t + 1, c);
    if (!COL && (t + 1) * static_cast<int64_t>(kTile) > a.str_rows) {  // items behind the last
      const int left = static_cast<int>(a.str_rows - t * static_cast<int64_t>(kTile)) - 4 * half;
      top = -__builtin_inff();
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (8 * (r >> 2) + (r & 3) >= left) p[r] = -__builtin_inff();
        top = fmaxf(top, p[r]);
      }
    }
    top = of_both_halves(top);
    if (__any(top > ref + lag)) {
      const float to = top > ref + lag ? top : ref;
      const float down = __builtin_amdgcn_exp2f(COL ? ref - to : (ref - to) * sc);
      ref = to;
      sum *= down;
      lost *= down;
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[b][r] *= down;
    }
    const float shift = kShift - ref;
    float w[4] = {0.f, 0.f, 0.f, 0.f};
    f32x4 factor[4];  // each read a step ahead of its use
    if constexpr (COL) factor[0] = row_values(t, 0, 1);
    // the next tile's scores beside this one's weights (behind the last tile: what lies in LDS, and not used)
    f32x16 next;
#pragma unroll
    for (int r = 0; r < 16; ++r) next[r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      if (c + SA < KC) read_scores(f[c + SA], t + 1, c + SA);
      if constexpr (COL) {
#pragma unroll
        for (int g = 4 * c / KC + 1; g <= 4 * (c + 1) / KC && g < 4; ++g) factor[g] = row_values(t, g, 1);
      }
      next = add_scores(next, f[c], c);
#pragma unroll
      for (int r = 16 * c / KC; r < 16 * (c + 1) / KC; ++r) {
        p[r] = __builtin_amdgcn_exp2f(COL ? p[r] + shift : fmaf(p[r] - ref, sc, kShift));
        if constexpr (COL) p[r] *= factor[r >> 2][r & 3];
        else w[r & 3] += p[r];
        asm volatile("" : "+v"(p[r]));  // here, beside the matrix instructions
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (!COL) {
      // the tile's sum first, and what each addition loses kept: one by one, thousands of small weights were rounded
      // away against the sum (6e-6 of it over 17,770 items)
      const float add = ((w[0] + w[1]) + (w[2] + w[3])) - lost;
      const float now = sum + add;
      lost = (now - sum) - add;
      sum = now;
    }
    if (sg.score_tiles == 1 && t + 2 < t1) {
      __syncthreads();
      fetch_scores(t + 2);
    }
    if constexpr (DB > 0) {
      if (COL && targets && win.due < static_cast<uint32_t>(t + 1) * kTile) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          // this half tile's records, through the wavefront's own table of 32 items x 16 rows in LDS, zero between uses.  A
          // row that lists an item twice adds twice: one wavefront's LDS additions come in the order of its
          // instructions and, within one, in an order that its addresses alone decide.
          const uint32_t limit = static_cast<uint32_t>(t * kTile + 16 * k + 16);
          bool some = false;
          while (win.due < limit) {
            const bool mine = lane >= win.pos && (win.now.x >> 5) < limit;
            const int n = __popcll(__ballot(mine));
            some = true;
            if (mine) {
              const uint32_t r = (win.now.x >> 5) & 15, c = win.now.x & 31;
              atomicAdd(y + c * 16 + (((r >> 2) ^ ((c >> 2) & 3)) << 2) + (r & 3), __uint_as_float(win.now.y) * unit);
            }
            win.skip(n, lane);
          }
          if (some) {
            __builtin_amdgcn_wave_barrier();
            const int col = lane & 31, turn = (col >> 2) & 3;
            f32x4 *const y0 = reinterpret_cast<f32x4 *>(y + col * 16 + ((half ^ turn) << 2));
            f32x4 *const y1 = reinterpret_cast<f32x4 *>(y + col * 16 + (((2 + half) ^ turn) << 2));
            const f32x4 v0 = *y0, v1 = *y1;
            __builtin_amdgcn_wave_barrier();
            *y0 = *y1 = f32x4{0.f, 0.f, 0.f, 0.f};
            __builtin_amdgcn_wave_barrier();
            const float up = up_to(ref);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              p[8 * k + i] = fmaf(-up, v0[i], p[8 * k + i]);
              p[8 * k + 4 + i] = fmaf(-up, v1[i], p[8 * k + 4 + i]);
            }
          }
        }
      }
      // the sums beside the next tile's log2 weights
      h8 g[2 * DB + TA][NP];
#pragma unroll
      for (int i = 0; i < TA && i < 2 * DB; ++i) read_turned(g[i], t, i);
      u32x4 ph[2], pl[2];
      auto make_planes = [&](int k, int i) {
        uint32_t h, l;
        planes(p[8 * k + 2 * i], p[8 * k + 2 * i + 1], h, l);
        ph[k][i] = h;
        pl[k][i] = l;
      };
#pragma unroll
      for (int i = 0; i < 4; ++i) make_planes(0, i);
      float n[16], m[2] = {-__builtin_inff(), -__builtin_inff()};
      f32x4 v[4];
      if constexpr (COL) v[0] = row_values(t + 1, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < 2 * DB; ++i) {
        const int k = i / DB, b = i % DB;
        if (i + TA < 2 * DB) read_turned(g[i + TA], t, i + TA);
        if constexpr (COL) {
#pragma unroll
          for (int z = 2 * i / DB + 1; z <= 2 * (i + 1) / DB && z < 4; ++z) v[z] = row_values(t + 1, z, 0);
        }
        o[b] = mfma(g[i][0], halves(ph[k]), o[b]);
        o[b] = mfma(g[i][0], halves(pl[k]), o[b]);
        if constexpr (NP == 2) o[b] = mfma(g[i][1], halves(ph[k]), o[b]);
        if (k == 0) {
#pragma unroll
          for (int z = 4 * b / DB; z < 4 * (b + 1) / DB; ++z) make_planes(1, z);
        }
#pragma unroll
        for (int r = 16 * i / (2 * DB); r < 16 * (i + 1) / (2 * DB); ++r) {
          n[r] = COL ? fmaf(next[r], sc, v[r >> 2][r & 3]) : next[r];
          m[r & 1] = fmaxf(m[r & 1], n[r]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) p[r] = n[r];
      top = fmaxf(m[0], m[1]);
    } else {
      weigh(next, t + 1);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  if (!live) return;
  const int64_t row = split * (a.own_tiles * kTile) + own_tile * kTile + (lane & 31);
  if (a.d0 == 0) {
    sum += __shfl_xor(sum, 32);
    if (half == 0) {
      a.m[row] = ref;
      if constexpr (!COL) a.l[row] = sum;
    }
  }
  if constexpr (DB > 0) {
    float *to = a.o + row * (KD * 32) + a.d0 * 32 + half * 4;
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4 *>(to + b * 32 + g * 8) = f32x4{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]};
  }
}

// ------------------------------------------------------------------ rows: join, targets, loss, dX
// Lanes of a group hold a row: number k = v 4G + 4g + q at lane g, vector v, element q
template <class T, int G, int V>
__device__ inline void load_row(f32x4 (&x)[V], const T *row, int g, int K, bool vec) {
#pragma unroll
  for (int v = 0; v < V; ++v) x[v] = load4(row, v * 4 * G + 4 * g, K, vec);
}

template <class T>
struct RowArgs {
  Targets t;
  int64_t own_pad;
  int32_t K, ldo, splits;
  Table<T> x, w;
  const Scal *scal;
  float scale;             // log2(e) / tau; 0: the references are powers of two (k_few's)
  const float *m, *l, *o;
  float *loss, *lse;
  T *dX;
  int64_t lddx;
  bool vec_out;
  float *rowvec;  // NULL: no pass over rows follows
};

// TW wavefronts per row (more for few rows).  The targets' part is c_i = sum coef w_j: dX_i needs it, and the loss
// too, since sum coef s_ij = x_i . c_i: one product per row instead of one per target.  Gathers of w rows bound it
// (16,384 rows of 208 items, K = 128 fp32: 1.75 GB in 212 us, 8.3 TB/s, 58% of it from L2).
template <class T, int G, int V, int TW>
__global__ __launch_bounds__(TW == 16 ? 1024 : kThreads) void k_row_finish(RowArgs<T> a) {
  constexpr int NG = TW * 64 / G;      // groups per row
  constexpr int RF = V == 1 ? 8 : 4;   // rows in flight per group
  constexpr int RB = TW == 16 ? 1 : 4 / TW;  // rows per workgroup
  __shared__ f32x4 part[TW > 1 ? TW : 1][TW > 1 ? 2 * V * G : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane & (G - 1);
  const int grp = (TW > 1 ? wave * (64 / G) : 0) + lane / G;
  const int64_t i = static_cast<int64_t>(block_index()) * RB + (TW == 1 ? wave : 0);
  const int64_t row_end = (a.t.n + kTile - 1) / kTile * kTile;
  if (i >= a.t.n) {  // rows behind the last, to the end of its tile: no weight in the pass over rows
    if (a.rowvec && i < row_end && lane == 0 && (TW == 1 || wave == 0)) {
      a.rowvec[(i >> 5) * 64 + (i & 31)] = -__builtin_inff();
      a.rowvec[(i >> 5) * 64 + 32 + (i & 31)] = 0.f;
    }
    return;
  }
  const bool act = a.t.act[i];
  const float unit = a.scale > 0.f ? unit_of(a.scal, a.scale) : 1.f;
  float top = kNone, den = 0.f;
#pragma unroll 4
  for (int s = lane; s < a.splits; s += 64) {
    const float m = a.m[s * a.own_pad + i], l = a.l[s * a.own_pad + i];
    const float now = fmaxf(top, m);
    den = den * __builtin_amdgcn_exp2f((top - now) * unit) + l * __builtin_amdgcn_exp2f((m - now) * unit);
    top = now;
  }
  const float mine = top;
  top = wave_max(top);
  den = wave_sum(den * __builtin_amdgcn_exp2f((mine - top) * unit));
  // in 64 bits: the loss is what is left of total lse - x . c, and a log2-sum-exp in 32 would be off by 5e-7 at 8 .. 16
  const double lse64 = static_cast<double>(top) * unit - static_cast<double>(kShift) + log2(static_cast<double>(den)), lse = lse64 * 0.69314718055994530942;
  f32x4 acc[V], o[V];
#pragma unroll
  for (int v = 0; v < V; ++v) acc[v] = o[v] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (act) {
    int64_t b, e;
    row_range(a.t.row_ptr, a.t.entries, a.t.k, i, b, e);
    const int64_t src = a.t.score ? i * a.t.ldt - b : 0;
    const double z = a.t.score ? a.t.logz[i] : 0.0;
    int32_t key[RF], coming[RF];
    float c[RF], soon[RF];
    auto read_list = [&](int64_t q) {  // a round ahead: its items' rows wait for it
#pragma unroll
      for (int f = 0; f < RF; ++f) {
        const int64_t at = q + f * NG;
        coming[f] = at < e ? a.t.item[at + src] : -1;
        soon[f] = at < e ? a.t.score ? a.t.score[at + src] : a.t.value ? a.t.value[at] : 1.f : 0.f;
      }
    };
    read_list(b + grp);
    for (int64_t q = b + grp; q < e; q += NG * RF) {
      f32x4 w[RF][V];
#pragma unroll
      for (int f = 0; f < RF; ++f) {
        key[f] = coming[f] < a.t.items ? coming[f] : -1;
        c[f] = key[f] >= 0 ? soon[f] : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) w[f][v] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (key[f] >= 0) load_row<T, G, V>(w[f], a.w.p + key[f] * a.w.ld, g, a.K, a.w.vec);
      }
      read_list(q + NG * RF);
#pragma unroll
      for (int f = 0; f < RF; ++f) {
        if (a.t.score) {
          c[f] = key[f] >= 0 ? expf(log_q(a.t, c[f], z)) : 0.f;
          if (c[f] == 0.f) continue;  // no entry: what its item holds does not count
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[v][u] = fmaf(c[f], w[f][v][u], acc[v][u]);
      }
    }
    if (a.dX)
      for (int s = grp; s < a.splits; s += NG) {
        const float f = __builtin_amdgcn_exp2f((a.m[s * a.own_pad + i] - top) * unit);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int k0 = v * 4 * G + 4 * g;
          if (k0 >= a.ldo) continue;
          const f32x4 u = *reinterpret_cast<const f32x4 *>(a.o + (s * a.own_pad + i) * a.ldo + k0);
#pragma unroll
          for (int q = 0; q < 4; ++q) o[v][q] = fmaf(u[q], f, o[v][q]);
        }
      }
#pragma unroll
    for (int s = G; s < 64; s <<= 1)
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          acc[v][u] += __shfl_xor(acc[v][u], s);
          o[v][u] += __shfl_xor(o[v][u], s);
        }
  }
  if constexpr (TW > 1) {
    if (lane < G) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        part[wave][2 * v * G + g] = acc[v];
        part[wave][(2 * v + 1) * G + g] = o[v];
      }
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      acc[v] = part[0][2 * v * G + g];
      o[v] = part[0][(2 * v + 1) * G + g];
      for (int w = 1; w < TW; ++w) {
        acc[v] += part[w][2 * v * G + g];
        o[v] += part[w][(2 * v + 1) * G + g];
      }
    }
  }
  double d = 0.0;  // x . c
  if (act) {
    f32x4 x[V];
    load_row<T, G, V>(x, a.x.p + i * a.x.ld, g, a.K, a.x.vec);
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int u = 0; u < 4; ++u) d = fma(static_cast<double>(x[v][u]), static_cast<double>(acc[v][u]), d);
#pragma unroll
    for (int s = G / 2; s > 0; s >>= 1) d += __shfl_xor(d, s);
  }
  if (lane == 0) {
    if (a.loss)
      a.loss[i] = act || a.t.extra[i] != 0.f ? static_cast<float>(static_cast<double>(a.t.tau) * a.t.tau * (a.t.extra[i] + (a.t.total[i] * lse - d / a.t.tau))) : 0.f;
    if (a.lse) a.lse[i] = static_cast<float>(lse);
    if (a.rowvec) {
      // a p_ij = 2^(score + v) f with the share a = 2^e m: v = e - log2-sum-exp, so that the items' references see the share
      // too, and f = m 2^r makes up for the rounding of v by r (at most 2^-19 at 16 .. 32)
      int e;
      const float m = frexpf(act ? a.t.share[i] / a.scal->amax : 0.f, &e);
      const double v = (m == 0.f ? -__builtin_inf() : static_cast<double>(e)) - lse64;
      const float v32 = static_cast<float>(v);
      a.rowvec[(i >> 5) * 64 + (i & 31)] = act ? v32 : -__builtin_inff();
      const double rest = (v - v32) * 0.69314718055994530942;  // below 2^-9 for scores below 2^15, and 2^-3 below 2^21
      const double back = 1.0 + rest * (1.0 + rest * (1.0 / 2 + rest * (1.0 / 6 + rest * (1.0 / 24))));
      a.rowvec[(i >> 5) * 64 + 32 + (i & 31)] = m == 0.f ? 0.f : m * static_cast<float>(back);
    }
  }
  if (a.dX && lane < G) {
    const float gw = a.t.gw[i], mean = a.t.total[i] / den;
    const int ew = a.scal->ew;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k0 = v * 4 * G + 4 * g;
      if (k0 >= a.K) continue;
      f32x4 out;
#pragma unroll
      for (int u = 0; u < 4; ++u) out[u] = act ? gw * (ldexpf(mean * o[v][u], -ew) - acc[v][u]) : 0.f;
      store4(a.dX + i * a.lddx, k0, a.K, a.vec_out, out);
    }
  }
}

// ------------------------------------------------------------------ scores in 64 bits
//
// A score in 64 bits: products of the tables' numbers are exact, and the sum has one order everywhere: 8 lanes of 4
// numbers each take every eighth 4, then the lanes are added in pairs.
constexpr int kDotLanes = 8;
template <int Move>
__device__ inline double moved(double v) {  // of another lane of the 8: 0xb1 of the pair, 0x4e of the other pair, 0x141 of the other four
  const unsigned long long u = __double_as_longlong(v);
  const int lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(u), Move, 0xf, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(u >> 32), Move, 0xf, 0xf, false);
  return __longlong_as_double(static_cast<long long>(static_cast<unsigned long long>(static_cast<uint32_t>(hi)) << 32 | static_cast<uint32_t>(lo)));
}
__device__ inline double sum8(double s) {
  s += moved<0xb1>(s);
  s += moved<0x4e>(s);
  return s + moved<0x141>(s);
}
// Of lane l ^ 4: two moves, each for half of the lanes
__device__ inline int far4(int v) {
  const int up = __builtin_amdgcn_update_dpp(0, v, 0x104, 0xf, 0x5, false);  // lanes 0..3 and 8..11 of 16 take l + 4
  return __builtin_amdgcn_update_dpp(up, v, 0x114, 0xf, 0xa, false);         // the others l - 4
}
__device__ inline double far4(double v) {
  const unsigned long long u = __double_as_longlong(v);
  const uint32_t lo = static_cast<uint32_t>(far4(static_cast<int>(u))), hi = static_cast<uint32_t>(far4(static_cast<int>(u >> 32)));
  return __longlong_as_double(static_cast<long long>(static_cast<unsigned long long>(hi) << 32 | lo));
}
// The sums of R numbers over 8 lanes, sum8's order: lane l gets number spread_of<R>(l), 8 / R lanes each.  Each step halves
// what a lane holds, so 8 numbers take 7 additions instead of 24
template <int R>
__device__ inline int spread_of(int l) {
  return R == 8 ? (l & 1) << 2 | (l & 2) | l >> 2 : R == 4 ? (l & 1) << 1 | (l >> 1 & 1) : 0;
}
template <int R>
__device__ inline double spread8(double (&s)[R], int l) {
  static_assert(R == 1 || R == 4 || R == 8, "1, 4 or 8 numbers");
  if constexpr (R == 1) {
    return sum8(s[0]);
  } else {
    double a[R / 2], b[R / 4];
    const bool odd = l & 1, second = l & 2, far = l & 4;
#pragma unroll
    for (int i = 0; i < R / 2; ++i) {
      const double keep = odd ? s[R / 2 + i] : s[i], give = odd ? s[i] : s[R / 2 + i];
      a[i] = keep + moved<0xb1>(give);
    }
#pragma unroll
    for (int i = 0; i < R / 4; ++i) {
      const double keep = second ? a[R / 4 + i] : a[i], give = second ? a[i] : a[R / 4 + i];
      b[i] = keep + moved<0x4e>(give);
    }
    if constexpr (R == 4) return b[0] + far4(b[0]);
    else return (far ? b[1] : b[0]) + far4(far ? b[0] : b[1]);
  }
}
template <class T>
__device__ inline double dot64(const double *x, const T *w, int l, int K, bool vec) {
  double s = 0.0;
#pragma unroll 4
  for (int k = 4 * l; k < K; k += 4 * kDotLanes) {
    const f32x4 v = load4(w, k, K, vec);
#pragma unroll
    for (int z = 0; z < 4; ++z) s = fma(x[k + z], static_cast<double>(v[z]), s);
  }
  return sum8(s);
}

// ------------------------------------------------------------------ few rows, the loss alone
//
// Log-sum-exps of R rows over pieces of the items: scores in 64 bits from the tables as they are (ps_soft_top's), the sums
// in fp32 with the maximum of what a lane has seen.  Reads W once for R rows; nothing is packed.  Bound by that
// read and by latency (one row, 9.1 MB: 4.6 us, 2 TB/s).
struct FewArgs {
  int64_t n, own_pad;
  int32_t items, K;
  int64_t per;       // items of a piece, a multiple of 32
  const int32_t *act;
  float scale;       // log2(e) / tau
  float *m, *l;      // [pieces][own_pad]
};
template <class T, int R>
__global__ __launch_bounds__(kThreads) void k_few(FewArgs a, Table<T> xt, Table<T> wt) {
  __shared__ double x[R][kMaxK];
  __shared__ float part[2][kThreads / 64][R];
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * R;
  const int l = threadIdx.x & (kDotLanes - 1), g = threadIdx.x / kDotLanes;
  for (int q = threadIdx.x; q < R * a.K; q += kThreads) {
    const int r = q / a.K, k = q - r * a.K;
    x[r][k] = r0 + r < a.n && a.act[r0 + r] ? static_cast<double>(to_f(xt.p[(r0 + r) * xt.ld + k])) : 0.0;
  }
  for (int q = threadIdx.x; q < R * ((4 - a.K % 4) % 4); q += kThreads) x[q % R][a.K + q / R] = 0.0;  // up to a whole float4
  __syncthreads();
  const int row = spread_of<R>(l);
  const int64_t j0 = blockIdx.x * a.per, j1 = min(j0 + a.per, static_cast<int64_t>(a.items));
  float top = kNone, sum = 0.f;
  for (int64_t j = j0 + g; j < j0 + a.per; j += kThreads / kDotLanes) {
    double s[R];
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = 0.0;
    if (j < j1) {
      const T *w = wt.p + j * wt.ld;
#pragma unroll(R == 8 ? 2 : 4)
      for (int k = 4 * l; k < a.K; k += 4 * kDotLanes) {
        const f32x4 v = load4(w, k, a.K, wt.vec);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int z = 0; z < 4; ++z) s[r] = fma(x[r][k + z], static_cast<double>(v[z]), s[r]);
      }
    }
    const float s2 = j < j1 ? static_cast<float>(spread8<R>(s, l) * a.scale) : (static_cast<void>(spread8<R>(s, l)), -__builtin_inff());
    const float now = fmaxf(top, s2);
    sum = sum * __builtin_amdgcn_exp2f(top - now) + __builtin_amdgcn_exp2f(s2 - now);
    top = now;
  }
  auto join = [&](float m, float v) {
    const float now = fmaxf(top, m);
    sum = sum * __builtin_amdgcn_exp2f(top - now) + v * __builtin_amdgcn_exp2f(m - now);
    top = now;
  };
#pragma unroll
  for (int o = kDotLanes; o < 64; o <<= 1) join(__shfl_xor(top, o), __shfl_xor(sum, o));
  if ((threadIdx.x & 63) < R) {
    part[0][threadIdx.x >> 6][row] = top;
    part[1][threadIdx.x >> 6][row] = sum;
  }
  __syncthreads();
  if (threadIdx.x < R && r0 + threadIdx.x < a.n) {
    top = part[0][0][threadIdx.x];
    sum = part[1][0][threadIdx.x];
    for (int w = 1; w < kThreads / 64; ++w) join(part[0][w][threadIdx.x], part[1][w][threadIdx.x]);
    a.m[blockIdx.x * a.own_pad + r0 + threadIdx.x] = top;
    a.l[blockIdx.x * a.own_pad + r0 + threadIdx.x] = sum * 0x1p7f;  // as the passes' sums: 2^(score - reference + kShift)
  }
}
static_assert(kShift == 7.f, "k_few's sums");

// ------------------------------------------------------------------ the targets by tiles of items
// A stable sort of the records by their key, up to 10 bits a pass (one pass up to 32,736 items): records of a tile stay
// in row order, which the pass over rows relies on, and nothing depends on the order of atomics.  A workgroup
// takes 4096 records, a wavefront 1024 of them in order; the rank of a record among its wavefront's
// equal digits comes from the lanes' ballots.  Bound by the scattered writes of the payloads (3.4M records: 47 us, and 19
// for the counts).
constexpr int kSortThreads = 512, kSortWaves = kSortThreads / 64;

__global__ __launch_bounds__(kThreads) void k_sort_count(const int32_t *key, int64_t n, int shift, int bins, int32_t *hist, int32_t blocks) {
  __shared__ int32_t cnt[kBins];
  for (int b = threadIdx.x; b < bins; b += kThreads) cnt[b] = 0;
  __syncthreads();
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kSortTile;
#pragma unroll 4
  for (int q = threadIdx.x; q < kSortTile; q += kThreads)
    if (base + q < n) atomicAdd(&cnt[(key[base + q] >> shift) & (bins - 1)], 1);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kThreads) hist[static_cast<int64_t>(b) * blocks + blockIdx.x] = cnt[b];
}

// Exclusive sums of each digit's counts over the workgroups, and the digit's total
__global__ __launch_bounds__(kThreads) void k_sort_scan(int32_t *hist, int32_t blocks, int32_t *total) {
  __shared__ int32_t sh[4], carry;
  int32_t *h = hist + static_cast<int64_t>(blockIdx.x) * blocks;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) carry = 0;
  for (int base = 0; base < blocks; base += kThreads) {
    const int at = base + threadIdx.x;
    const int32_t v = at < blocks ? h[at] : 0;
    int32_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int32_t u = __shfl_up(s, o);
      if (lane >= o) s += u;
    }
    if (lane == 63) sh[wave] = s;
    __syncthreads();
    int32_t before = carry;
    for (int w = 0; w < wave; ++w) before += sh[w];
    if (at < blocks) h[at] = before + s - v;
    __syncthreads();
    if (threadIdx.x == kThreads - 1) carry = before + s;
    __syncthreads();
  }
  if (threadIdx.x == 0) total[blockIdx.x] = carry;
}

struct Records {
  int32_t *key;
  uint2 *pay;
};
// first: where the digits start, for the one pass whose digits are the whole keys (NULL otherwise).  A lane's keys and
// payloads are read at once: in turn, each round waited for its own (24 us for 4096 records a workgroup, however few)
__global__ __launch_bounds__(kSortThreads) void k_sort_move(Records in, Records out, int64_t n, int shift, int bits, const int32_t *hist,
                                                        int32_t blocks, const int32_t *total, int64_t *first, int32_t firsts) {
  constexpr int kOwn = kSortTile / kSortThreads, kDigits = kBins / kSortThreads;  // records and digits of a thread
  __shared__ int32_t cnt[kSortWaves][kBins], sh[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << bits;
  const int64_t base = static_cast<int64_t>(blockIdx.x) * kSortTile + wave * (kSortTile / kSortWaves) + lane;
  int32_t key[kOwn];
  uint2 pay[kOwn];
#pragma unroll
  for (int q = 0; q < kOwn; ++q) key[q] = base + 64 * q < n ? in.key[base + 64 * q] : -1;  // keys are not negative
#pragma unroll
  for (int q = 0; q < kOwn; ++q) pay[q] = base + 64 * q < n ? in.pay[base + 64 * q] : make_uint2(0u, 0u);
  for (int b = threadIdx.x; b < kSortWaves * kBins; b += kSortThreads) (&cnt[0][0])[b] = 0;
  __syncthreads();
#pragma unroll
  for (int q = 0; q < kOwn; ++q)
    if (key[q] >= 0) atomicAdd(&cnt[wave][(key[q] >> shift) & (bins - 1)], 1);
  // where each digit starts: the digits before it
  const int b0 = kDigits * threadIdx.x;
  int32_t v[kDigits], at[kDigits], s = 0;
  if (blocks == 1) {  // one workgroup's counts are the totals
    __syncthreads();
#pragma unroll
    for (int z = 0; z < kDigits; ++z) {
      v[z] = at[z] = 0;
      for (int w = 0; w < kSortWaves && b0 + z < bins; ++w) v[z] += cnt[w][b0 + z];
      s += v[z];
    }
  } else {
#pragma unroll
    for (int z = 0; z < kDigits; ++z) {
      v[z] = b0 + z < bins ? total[b0 + z] : 0;
      at[z] = b0 + z < bins ? hist[static_cast<int64_t>(b0 + z) * blocks + blockIdx.x] : 0;
      s += v[z];
    }
  }
  const int32_t own = s;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t u = __shfl_up(s, o);
    if (lane >= o) s += u;
  }
  if (lane == 63) sh[wave] = s;
  __syncthreads();
  int32_t before = s - own;
  for (int w = 0; w < wave; ++w) before += sh[w];
#pragma unroll
  for (int z = 0; z < kDigits; ++z) {
    if (b0 + z < bins) {
      if (first && blockIdx.x == 0 && b0 + z < firsts) first[b0 + z] = before;
      int32_t to = before + at[z];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const int32_t c = cnt[w][b0 + z];
        cnt[w][b0 + z] = to;
        to += c;
      }
    }
    before += v[z];
  }
  __syncthreads();
  volatile int32_t *mine = cnt[wave];
#pragma unroll
  for (int q = 0; q < kOwn; ++q) {
    const bool there = key[q] >= 0;
    const int d = (key[q] >> shift) & (bins - 1);
    unsigned long long same = __ballot(there);
    for (int bit = 0; bit < bits; ++bit) {
      const unsigned long long set = __ballot((d >> bit) & 1);
      same &= (d >> bit) & 1 ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (there) {
      const int32_t to = mine[d] + rank;
      if (!first) out.key[to] = key[q];
      out.pay[to] = pay[q];
    }
    __builtin_amdgcn_wave_barrier();
    if (there && rank == 0) mine[d] += __popcll(same);
    __builtin_amdgcn_wave_barrier();
  }
}

// Where the records of each tile start, after more than one sorting pass
__global__ __launch_bounds__(kThreads) void k_first(const int32_t *key, int64_t n, int64_t *first, int32_t firsts) {
  const int32_t t = blockIdx.x * kThreads + threadIdx.x;
  if (t >= firsts) return;
  int64_t lo = 0, hi = n;
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (key[mid] < t) lo = mid + 1; else hi = mid;
  }
  first[t] = lo;
}

template <class T>
struct ItemArgs {
  int64_t own_pad;
  int32_t items, K, ldo, splits;
  const Scal *scal;
  const float *m, *o;
  T *dW;
  int64_t lddw;
  bool vec_out;
};

// dW_j: the passes' pieces joined.  Bound by memory (100,000 items in 4 pieces, K = 256 bf16: 461 MB in 98 us, 4.7 TB/s).
template <class T, int G, int V>
__global__ __launch_bounds__(kThreads) void k_item_finish(ItemArgs<T> a) {
  const int g = threadIdx.x & (G - 1);
  const int64_t j = static_cast<int64_t>(block_index()) * (kThreads / G) + threadIdx.x / G;
  if (j >= a.items) return;
  const float back = a.splits ? ldexpf(a.scal->amax, -a.scal->ex) : 0.f;
  f32x4 o[V];
#pragma unroll
  for (int v = 0; v < V; ++v) o[v] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < a.splits; ++s) {
    const float f = __builtin_amdgcn_exp2f(a.m[s * a.own_pad + j] - kShift);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int k0 = v * 4 * G + 4 * g;
      if (k0 >= a.ldo) continue;
      const f32x4 u = *reinterpret_cast<const f32x4 *>(a.o + (s * a.own_pad + j) * a.ldo + k0);
#pragma unroll
      for (int z = 0; z < 4; ++z) o[v][z] = fmaf(u[z], f, o[v][z]);
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int k0 = v * 4 * G + 4 * g;
    if (k0 >= a.K) continue;
    f32x4 d;
#pragma unroll
    for (int z = 0; z < 4; ++z) d[z] = o[v][z] * back;
    store4(a.dW + j * a.lddw, k0, a.K, a.vec_out, d);
  }
}

// ------------------------------------------------------------------ the best items
// Scores in 64 bits, as keys whose unsigned order is that of the numbers; a workgroup keeps the best of what
// it has seen in LDS: what beats the k-th best so far is put behind, and when the room is full it is
// sorted and cut to k again.
constexpr int kTopRoom = 2048;

__device__ inline uint64_t order_key(double v) {
  if (v != v) return ~0ull;  // NaN above all
  const uint64_t u = static_cast<uint64_t>(__double_as_longlong(v + 0.0));  // -0 as 0
  return u >> 63 ? ~u : u | (1ull << 63);
}
__device__ inline double key_value(uint64_t k) {
  return __longlong_as_double(static_cast<long long>(k >> 63 ? k & ~(1ull << 63) : ~k));
}

struct Best {
  uint64_t *key;  // [kTopRoom]
  int32_t *item;  // [kTopRoom]
  int32_t *count;
};
__device__ inline bool before(uint64_t ka, int32_t ia, uint64_t kb, int32_t ib) { return ka > kb || (ka == kb && ia < ib); }

// The room's first `count` entries in order, all threads; at most k of them stay.  Returns the k-th key (0: fewer).
__device__ inline uint64_t best_cut(Best b, int k) {
  __syncthreads();
  const int n = *b.count;
  int size = 2;
  while (size < n) size <<= 1;
  for (int q = n + threadIdx.x; q < size; q += kThreads) {
    b.key[q] = 0;
    b.item[q] = 0x7fffffff;
  }
  __syncthreads();
  for (int len = 2; len <= size; len <<= 1)
    for (int d = len >> 1; d > 0; d >>= 1) {
      for (int q = threadIdx.x; q < size / 2; q += kThreads) {
        const int lo = ((q & ~(d - 1)) << 1) | (q & (d - 1)), hi = lo | d;
        const bool up = (lo & len) == 0;
        const uint64_t ka = b.key[lo], kb = b.key[hi];
        const int32_t ia = b.item[lo], ib = b.item[hi];
        if (before(kb, ib, ka, ia) == up) {
          b.key[lo] = kb; b.key[hi] = ka;
          b.item[lo] = ib; b.item[hi] = ia;
        }
      }
      __syncthreads();
    }
  if (threadIdx.x == 0) *b.count = min(n, k);
  __syncthreads();
  return n >= k ? b.key[k - 1] : 0;
}

// Every thread may bring one entry; entries come with increasing items or all differ
__device__ inline void best_add(Best b, int k, bool want, uint64_t key, int32_t item, uint64_t &least) {
  if (want && key >= least) {
    const int at = atomicAdd(b.count, 1);
    b.key[at] = key;
    b.item[at] = item;
  }
  __syncthreads();
  if (*b.count > kTopRoom - kThreads) {
    const uint64_t now = best_cut(b, k);
    least = now > least ? now : least;
  }
  __syncthreads();
}

template <class T>
struct TopArgs {
  int64_t row0, n;  // rows of this launch
  int32_t items, K, k, words;
  Table<T> x, w;
  const uint32_t *excluded;  // [n][words] bits (NULL: none)
  const int64_t *row_ptr;    // the lists themselves
  const int32_t *list;
  int64_t entries;
  // few rows: keys of the scores and the groups' largest
  int32_t groups;
  uint64_t *key, *most;      // [n][groups 64], [n][groups]
  // many: candidates
  const int32_t *found, *count;  // [n][room], [n]: more than room: all items
  int32_t room;
  int32_t *out_item;
  float *out_score;
  int64_t ldo;
};

// Up to 256 scores, an item per thread: 8 lanes make 8 items' in turn, the 32 groups of lanes neighbouring ones (80
// candidates take 3 turns).  item_of(q): the q-th of n, or -1
template <class T, class F>
__device__ inline void top_batch(const TopArgs<T> &a, const double *x, Best b, uint64_t &least, int n, F item_of) {
  const int l = threadIdx.x & (kDotLanes - 1), g = threadIdx.x / kDotLanes;
  int32_t mine = -1;
  uint64_t key = 0;
#pragma unroll 4
  for (int q = 0; q < kDotLanes; ++q) {
    const int at = q * (kThreads / kDotLanes) + g;
    const int32_t j = at < n ? item_of(at) : -1;
    if (j < 0) continue;  // the same for the 8 lanes
    const double s = dot64(x, a.w.p + j * a.w.ld, l, a.K, a.w.vec);
    if (l == q) {
      mine = j;
      key = order_key(s);
    }
  }
  best_add(b, a.k, mine >= 0, key, mine, least);
}

template <class T>
__device__ inline void top_row(const TopArgs<T> &a, int64_t r, double *x, int32_t *count) {
  const T *xr = a.x.p + (a.row0 + r) * a.x.ld;
  for (int k = threadIdx.x; k < kMaxK; k += kThreads) x[k] = k < a.K ? static_cast<double>(to_f(xr[k])) : 0.0;
  if (threadIdx.x == 0) *count = 0;
  __syncthreads();
}

template <class T>
__device__ inline void top_all(const TopArgs<T> &a, int64_t r, const double *x, Best b, int64_t j0, int64_t j1) {
  uint64_t least = 0;
  for (int64_t base = j0; base < j1; base += kThreads)
    top_batch(a, x, b, least, kThreads, [&](int q) {
      const int64_t j = base + q;
      if (j >= j1 || (a.excluded && ((a.excluded[r * a.words + (j >> 5)] >> (j & 31)) & 1))) return -1;
      return static_cast<int32_t>(j);
    });
  best_cut(b, a.k);
}

template <class T>
__device__ inline void top_out(const TopArgs<T> &a, int64_t r, Best b) {
  const int64_t to = (a.row0 + r) * a.ldo;
  for (int q = threadIdx.x; q < a.k; q += kThreads) {
    const bool there = q < *b.count;
    a.out_item[to + q] = there ? b.item[q] : -1;
    a.out_score[to + q] = there ? static_cast<float>(key_value(b.key[q])) : -__builtin_inff();
  }
}

// ---- few rows
//
// Scores of R rows with groups of 64 items, as keys, and each row's largest key of the group.  A row's k best lie in
// the groups whose largest key is among the k largest of these (equal ones too), so the second kernel looks at few
// more than k groups.  A workgroup takes `per` groups, so that many rows load their numbers and lists less often.
// Bound by the reads of the items' rows, once for R rows, and by latency for few rows (one, 9.1 MB: 5.5 us), else by the
// products in 64 bits (64 rows x 20,000 items, K = 64: 20 us).
constexpr int kTopGroups = 8;  // most groups of a workgroup
template <class T, int R>
__global__ __launch_bounds__(kThreads) void k_top_scores(TopArgs<T> a, int per) {
  __shared__ double x[R][kMaxK];
  __shared__ uint64_t most[2][4][R];
  __shared__ uint64_t out[R][kTopGroups];
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * R;
  const int l = threadIdx.x & (kDotLanes - 1), g = threadIdx.x / kDotLanes;
  const int g0 = blockIdx.x * per, g1 = min(g0 + per, a.groups);
  for (int q = threadIdx.x; q < R * a.K; q += kThreads) {
    const int r = q / a.K, k = q - r * a.K;
    if (r0 + r < a.n) x[r][k] = static_cast<double>(to_f(a.x.p[(a.row0 + r0 + r) * a.x.ld + k]));
  }
  for (int q = threadIdx.x; q < R * ((4 - a.K % 4) % 4); q += kThreads) x[q % R][a.K + q / R] = 0.0;  // up to a whole float4
  if (threadIdx.x < R * kTopGroups) out[threadIdx.x / kTopGroups][threadIdx.x % kTopGroups] = 0;
  __syncthreads();
  if (a.row_ptr) {  // the groups' excluded items, a bit each
    constexpr int W = R < 4 ? R : 4, L = kThreads / W;  // rows at a time, threads each
    for (int r = threadIdx.x / L; r < R; r += W) {
      if (r0 + r >= a.n) continue;
      int64_t b, e;
      row_range(a.row_ptr, a.entries, 0, a.row0 + r0 + r, b, e);
#pragma unroll 4
      for (int64_t q = b + threadIdx.x % L; q < e; q += L) {
        const int64_t d = a.list[q] - static_cast<int64_t>(g0) * kTopGroup;
        if (d >= 0 && d < per * kTopGroup) atomicOr(reinterpret_cast<unsigned long long *>(&out[r][d / kTopGroup]), 1ull << (d % kTopGroup));
      }
    }
    __syncthreads();
  }
  const int row = spread_of<R>(l);  // whose scores this lane ends up with
  for (int at = g0; at < g1; ++at) {
    const int64_t j0 = static_cast<int64_t>(at) * kTopGroup;
    uint64_t best = 0;
#pragma unroll 1
    for (int q = 0; q < kTopGroup * kDotLanes / kThreads; ++q) {
      const int d = q * (kThreads / kDotLanes) + g;
      const int64_t j = j0 + d;
      double s[R];
#pragma unroll
      for (int r = 0; r < R; ++r) s[r] = 0.0;
      if (j < a.items) {
        const T *w = a.w.p + j * a.w.ld;
#pragma unroll(R == 8 ? 2 : 4)
        for (int k = 4 * l; k < a.K; k += 4 * kDotLanes) {
          const f32x4 v = load4(w, k, a.K, a.w.vec);
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int z = 0; z < 4; ++z) s[r] = fma(x[r][k + z], static_cast<double>(v[z]), s[r]);
        }
      }
      const double sum = spread8<R>(s, l);
      const uint64_t key = j < a.items && !((out[row][at - g0] >> d) & 1) ? max(order_key(sum), static_cast<uint64_t>(1)) : 0;  // 0: no item
      best = max(best, key);
      if (l < (R == 8 ? 8 : R) && j < a.items && r0 + row < a.n) a.key[(r0 + row) * a.groups * kTopGroup + j] = key;
    }
    uint64_t(*const m)[R] = most[at & 1];
#pragma unroll
    for (int o = kDotLanes; o < 64; o <<= 1) best = max(best, static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(best), o)));
    if ((threadIdx.x & 63) < R) m[threadIdx.x >> 6][row] = best;
    __syncthreads();
    if (threadIdx.x < R && r0 + threadIdx.x < a.n) {
      const int r = threadIdx.x;
      a.most[(r0 + r) * a.groups + at] = max(max(m[0][r], m[1][r]), max(m[2][r], m[3][r]));
    }
  }
}

// The k-th largest of n keys' upper 32 bits, rounded down to their upper 22 (two histograms of 11 bits); 0 for fewer
// than k.  value(q): the q-th.  kThreads threads
template <class F>
__device__ inline uint32_t kth_largest(int64_t n, int k, int32_t *hist, int32_t *sh, F value) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t prefix = 0;
  int need = k;
  for (int round = 0; round < 2; ++round) {
    const int shift = round ? 10 : 21;
    for (int b = threadIdx.x; b < 2048; b += kThreads) hist[b] = 0;
    __syncthreads();
#pragma unroll 4
    for (int64_t q = threadIdx.x; q < n; q += kThreads) {
      const uint32_t u = value(q);
      if (round == 0 || u >> 21 == prefix) atomicAdd(&hist[(u >> shift) & 2047], 1);
    }
    __syncthreads();
    // digits from the largest down: thread i holds 2047 - 8i .. 2040 - 8i
    int own = 0;
    for (int z = 0; z < 8; ++z) own += hist[2047 - 8 * threadIdx.x - z];
    int s = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(s, o);
      if (lane >= o) s += u;
    }
    if (lane == 63) sh[wave] = s;
    if (threadIdx.x == 0) sh[4] = -1;
    __syncthreads();
    int above = s - own;
    for (int w = 0; w < wave; ++w) above += sh[w];
    if (above < need && above + own >= need) {
      for (int z = 0; z < 8; ++z) {
        const int b = 2047 - 8 * threadIdx.x - z;
        if (above + hist[b] >= need) {
          sh[4] = b;
          sh[5] = need - above;
          break;
        }
        above += hist[b];
      }
    }
    __syncthreads();
    if (sh[4] < 0) return 0;
    prefix = round ? prefix << 11 | sh[4] : sh[4];
    need = sh[5];
    __syncthreads();
  }
  return prefix << 10;
}

// The k best of a row from its groups' keys
template <class T>
__global__ __launch_bounds__(kThreads) void k_top_pick(TopArgs<T> a) {
  __shared__ uint64_t keys[kTopRoom];
  __shared__ int32_t items[kTopRoom], count, groups, hist[2048], sh[6];
  const int64_t r = blockIdx.x;
  const uint64_t *most = a.most + r * a.groups;
  if (threadIdx.x == 0) count = groups = 0;
  const uint32_t least32 = max(kth_largest(a.groups, a.k, hist, sh, [&](int64_t q) { return static_cast<uint32_t>(most[q] >> 32); }), 1u);
  const Best b{keys, items, &count};
  // room for the numbers of 2048 groups at a time
  uint64_t least = static_cast<uint64_t>(least32) << 32;
  for (int64_t g0 = 0; g0 < a.groups; g0 += 2048) {
    const int64_t g1 = min(g0 + 2048, static_cast<int64_t>(a.groups));
    __syncthreads();
    if (threadIdx.x == 0) groups = 0;
    __syncthreads();
    for (int64_t q = g0 + threadIdx.x; q < g1; q += kThreads)
      if (most[q] >= least) hist[atomicAdd(&groups, 1)] = static_cast<int32_t>(q);
    __syncthreads();
    const int n = groups;
    for (int q = 0; q < n; q += kThreads / kTopGroup) {
      const int at = q + threadIdx.x / kTopGroup;
      const int64_t j = at < n ? static_cast<int64_t>(hist[at]) * kTopGroup + threadIdx.x % kTopGroup : a.items;
      const uint64_t key = j < a.items ? a.key[r * a.groups * kTopGroup + j] : 0;
      best_add(b, a.k, key > 0, key, static_cast<int32_t>(j), least);
    }
  }
  best_cut(b, a.k);
  top_out(a, r, b);
}

// ---- many rows: candidates by matrix instructions
//
// Scores of fp16 numbers (one plane) are off by at most e_ij = c (|x_i| + 1)(|w_j| + 1) of the scaled tables, and
// that product is one more number of each row: with |w| there and -|x| here the score comes out as a lower
// bound of the true one, with +|x| as an upper bound.  A first pass keeps the largest lower bound of every 16
// items; the k-th largest of those, T, is below at least k true scores.  A second pass finds the items whose
// upper bound is not below T: all of the k best are among them, and few others (about 1.2 k of 17,770 normal
// scores at K = 128).  These are then scored in 64 bits and put in order.  A row with more candidates
// than its room (far more equal scores than that, rows of zeros, numbers that are not finite) looks at
// all items in 64 bits.
//
// c: with x' = fp16(x): |x' - x| <= 2^-11 |x| + 2^-25, so products add up to at most (2^-10 + 2^-22) |x||w| (nothing
// for tables of 16 bits) + 2^-24 sqrt(K) (|x| + |w|), and the instruction's sums of 2 KC groups, counted at
// 2^-22 each, to (2 KC + 16) 2^-22 |x||w|.
constexpr int row_room(int kc) { return kc > 25 ? 16 : 32; }  // candidates of a row that a workgroup keeps in LDS

template <class T>
__global__ __launch_bounds__(kThreads) void k_top_pack(Table<T> x, Table<T> w, int64_t row0, int64_t rows, int32_t xt, _Float16 *px, _Float16 *pw,
                                                       int32_t K, int32_t kc, float c, const float *part, int32_t *count) {
  extern __shared__ float tile[];
  __shared__ float sh[4], norm[kTile];
  const int32_t block = block_index();
  const bool second = block >= xt;
  const Table<T> t = second ? w : x;
  const int64_t at = static_cast<int64_t>(block) - (second ? xt : 0);
  if (second && at * kTile >= w.rows) return;
  int ex = 0;
  if constexpr (!std::is_same<T, f16_t>::value) ex = scale_exp(block_max(part[(second ? kParts : 0) + threadIdx.x], sh));
  const int64_t begin = second ? 0 : row0, end = second ? t.rows : row0 + rows;
  // a tile: kc fragments, and one more of rows' tiles, the last number's chunk with that number negated
  _Float16 *out = second ? pw + at * kc * kFrag : px + at * (kc + 1) * kFrag;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, l32 = lane & 31;
  const int kd = (K + 31) / 32, wide = min(kd, kPackBlocks), ld = wide * 32 + 1;
  const int last = K / 16;  // the chunk of the bound's number
  float sum = 0.f;
  int b0 = 0;
  for (;; b0 += wide) {
    const int nb = min(wide, kd - b0), per = nb * 8;
    __syncthreads();
    for (int q = threadIdx.x; q < kTile * per; q += kThreads) {
      const int r = q / per, k0 = (q - r * per) * 4;
      const int64_t row = begin + at * kTile + r;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      if (row < end && b0 * 32 + k0 < K) v = load4(t.p + row * t.ld, b0 * 32 + k0, K, t.vec);
#pragma unroll
      for (int z = 0; z < 4; ++z) tile[r * ld + k0 + z] = ldexpf(v[z], ex);
    }
    __syncthreads();
    for (int k = threadIdx.x & 7; k < nb * 32; k += 8) {
      const float v = tile[(threadIdx.x >> 3) * ld + k];
      sum = fmaf(v, v, sum);
    }
    for (int f = 2 * b0 + wave; f < min(2 * (b0 + nb), last); f += 4) {
      h8 hi;
#pragma unroll
      for (int i = 0; i < 8; ++i) hi[i] = static_cast<_Float16>(tile[l32 * ld + (f - 2 * b0) * 16 + half * 8 + i]);
      *reinterpret_cast<h8 *>(out + f * kFrag + lane * 8) = hi;
    }
    if (b0 + nb >= kd) break;
  }
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 7) == 0) {
    const int r = threadIdx.x >> 3;
    // rounded up: 2^-9 for the sum, the root and fp16
    norm[r] = (sqrtf(sum) + 1.f) * (1.f + 0x1p-9f) * (second ? c * 64.f : 1.f / 64.f);
    const int64_t row = at * kTile + r;
    if (!second && row < rows) count[row] = sum < __builtin_inff() ? 0 : 1 << 30;
  }
  __syncthreads();
  for (int f = last + wave; f <= kc; f += 4) {
    if (f == kc && second) break;
    const int from = f == kc ? last : f;
    h8 hi;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = from * 16 + half * 8 + i;
      float v = k < K ? tile[l32 * ld + k - 32 * b0] : 0.f;
      if (k == K) v = f == kc ? -norm[l32] : norm[l32];
      hi[i] = static_cast<_Float16>(v);
    }
    *reinterpret_cast<h8 *>(out + f * kFrag + lane * 8) = hi;
  }
}

struct ScoreArgs {
  const _Float16 *own, *str;
  int64_t rows, own_tiles, tiles, steps_per_split;
  int32_t items, splits, words, last;  // last: the chunk of the bound's number
  const uint32_t *excluded;
  float *most;        // [rows][per_row] first pass: largest lower bounds, 4 per step
  int64_t per_row;
  int64_t steps;
  const float *least; // [rows] second pass: T
  int32_t *found, *count;
};

// First pass (Find = false) or second.  A wavefront owns 64 rows; the matrix instructions' rate bounds both (8192 rows x
// 17,770 items, K = 128: 46 us, 0.9 PFLOP/s, and 62 with the tests and lists).
template <int KC, bool Find>
__global__ __launch_bounds__(kThreads, 2) void k_score(ScoreArgs a) {
  constexpr int kStage = kScoreTiles * KC * kFrag, kRowRoom = row_room(KC);
  __shared__ _Float16 buf[2 * kStage];
  __shared__ int32_t list[Find ? kWaves * 64 * kRowRoom : 1], have[Find ? kWaves * 64 : 1];
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x % a.splits;
  const int64_t own_tile = (static_cast<int64_t>(blockIdx.x / a.splits) * kWaves + wave) * 2;
  const int64_t s0 = split * a.steps_per_split, s1 = min(s0 + a.steps_per_split, a.steps);
  auto fetch = [&](int64_t step, int at) {
    const _Float16 *src = a.str + step * kStage;
    const int n = static_cast<int>(min(static_cast<int64_t>(kScoreTiles), a.tiles - step * kScoreTiles)) * KC;
    for (int f = wave; f < n; f += kWaves)
      to_lds16(src + f * kFrag + lane * 8, buf + at * kStage + f * kFrag);
  };
  h8 q[KC][2];
  int64_t row[2];
  float least[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const bool live = own_tile + u < a.own_tiles;
    const _Float16 *own = a.own + (own_tile + u) * (KC + 1) * kFrag;
#pragma unroll
    for (int c = 0; c < KC; ++c) {
      q[c][u] = h8{0, 0, 0, 0, 0, 0, 0, 0};
      if (live) q[c][u] = *reinterpret_cast<const h8 *>(own + (!Find && c == a.last ? KC : c) * kFrag + lane * 8);
    }
    row[u] = (own_tile + u) * kTile + (lane & 31);
    if (row[u] >= a.rows) row[u] = -1;
    least[u] = __builtin_inff();
    if (Find && row[u] >= 0) least[u] = a.least[row[u]];
  }
  if constexpr (Find) {
    have[threadIdx.x] = 0;
  }
  // the rows' excluded bits of a step's tiles, read a step ahead
  uint32_t bits[2][kScoreTiles], coming[2][kScoreTiles];
  auto read_bits = [&](uint32_t (&to)[2][kScoreTiles], int64_t step) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int z = 0; z < kScoreTiles; ++z) {
        const int64_t t = step * kScoreTiles + z;
        to[u][z] = a.excluded && row[u] >= 0 && t < a.words ? a.excluded[row[u] * a.words + t] : 0u;
      }
  };
  float even[2][kScoreTiles];  // an even step's bounds (pieces start at even steps)
  if (s0 < s1) {
    fetch(s0, 0);
    read_bits(coming, s0);
  }
  for (int64_t st = s0; st < s1; ++st) {
    const int at = static_cast<int>(st - s0) & 1;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int z = 0; z < kScoreTiles; ++z) bits[u][z] = coming[u][z];
    if (st + 1 < s1) {
      fetch(st + 1, at ^ 1);
      read_bits(coming, st + 1);
    }
    float most[2][kScoreTiles];
#pragma unroll
    for (int z = 0; z < kScoreTiles; ++z) {
      const int64_t t = st * kScoreTiles + z;
      most[0][z] = most[1][z] = -__builtin_inff();
      if (t >= a.tiles) continue;
      const uint32_t out[2] = {bits[0][z] >> (4 * half), bits[1][z] >> (4 * half)};
      f32x16 s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
      const _Float16 *f = buf + at * kStage + z * KC * kFrag + lane * 8;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const h8 h = *reinterpret_cast<const h8 *>(f + c * kFrag);
        s[0] = mfma(h, q[c][0], s[0]);
        s[1] = mfma(h, q[c][1], s[1]);
      }
      const bool part = (t + 1) * kTile > a.items;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if constexpr (!Find) {
          if (__any(out[u])) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int bit = 8 * (r >> 2) + (r & 3);
              if ((out[u] >> bit) & 1) s[u][r] = -__builtin_inff();
            }
          }
          if (part) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (t * kTile + 8 * (r >> 2) + 4 * half + (r & 3) >= a.items) s[u][r] = -__builtin_inff();
          }
          float m = s[u][0];
#pragma unroll
          for (int r = 1; r < 16; ++r) m = fmaxf(m, s[u][r]);
          most[u][z] = m;
        } else {
          uint32_t hits = 0;
#pragma unroll
          for (int r = 15; r >= 0; --r) hits = hits * 2 + (s[u][r] < least[u] ? 0u : 1u);  // NaN is a candidate
          if (row[u] < 0) hits = 0;
          if (__any(hits != 0)) {
            // the excluded, and in the last tile what lies behind the items
            hits &= ~((out[u] & 15) | ((out[u] >> 4) & 0xf0) | ((out[u] >> 8) & 0xf00) | ((out[u] >> 12) & 0xf000));
            if (part)
              for (int r = 0; r < 16; ++r)
                if (t * kTile + 8 * (r >> 2) + 4 * half + (r & 3) >= a.items) hits &= ~(1u << r);
            if (hits) {
              const int mine = wave * 64 + u * 32 + (lane & 31);
              int to = atomicAdd(&have[mine], __popc(hits));
              while (hits) {
                const int r = __ffs(hits) - 1;
                hits &= hits - 1;
                const int32_t j = static_cast<int32_t>(t * kTile) + 8 * (r >> 2) + 4 * half + (r & 3);
                if (to < kRowRoom) {
                  list[mine * kRowRoom + to] = j;
                } else {
                  const int g = atomicAdd(&a.count[row[u]], 1);
                  if (g < kCandidates) a.found[row[u] * kCandidates + g] = j;
                }
                ++to;
              }
            }
          }
        }
      }
    }
    if constexpr (!Find) {
      // two steps' bounds in one store: the rows lie far apart, each store is a line of its own
      static_assert(kScoreTiles == 2, "stored as two pairs");
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (!(st & 1)) {
          even[u][0] = most[u][0];
          even[u][1] = most[u][1];
        }
        if (row[u] >= 0 && ((st & 1) || st + 1 == s1)) {
          const float none = -__builtin_inff();
          *reinterpret_cast<f32x4 *>(a.most + row[u] * a.per_row + (st >> 1) * 8 + half * 4) =
              f32x4{even[u][0], even[u][1], st & 1 ? most[u][0] : none, st & 1 ? most[u][1] : none};
        }
      }
    }
  }
  if constexpr (Find) {
    __syncthreads();
    // a row's list behind the others' of its row, a lane per row (a row in turn waited for its counter 64 times)
    const int mine = wave * 64 + lane;
    const int64_t r = own_tile * kTile + lane;
    const int n = r < a.rows ? min(have[mine], kRowRoom) : 0;
    if (n > 0) {
      const int to = atomicAdd(&a.count[r], n);
      for (int q = 0; q < n && to + q < kCandidates; ++q) a.found[r * kCandidates + to + q] = list[mine * kRowRoom + q];
    }
  }
}

__device__ inline uint32_t order_bits(float v) {
  const uint32_t u = __float_as_uint(v);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ inline float bits_value(uint32_t u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }

// T of each row: the k-th largest of its bounds, rounded down.  One workgroup per row; bound by the reads of the bounds
// (8192 rows of 1112: 28 us).
__global__ __launch_bounds__(kThreads) void k_top_least(const float *most, int64_t per_row, int32_t k, float *least) {
  __shared__ int32_t hist[2048], sh[6];
  const float *row = most + blockIdx.x * per_row;
  const uint32_t u = kth_largest(per_row, k, hist, sh, [&](int64_t q) { return order_bits(row[q]); });
  if (threadIdx.x == 0) least[blockIdx.x] = u ? bits_value(u) : -__builtin_inff();
}

// The candidates of a row (or all items) in order.  Gathers of w rows bound it, and the sort (8192 rows, about 80 candidates:
// 80 us)
template <class T>
__global__ __launch_bounds__(kThreads) void k_top_rank(TopArgs<T> a) {
  __shared__ double x[kMaxK];
  __shared__ uint64_t keys[kTopRoom];
  __shared__ int32_t items[kTopRoom], count;
  const int64_t r = blockIdx.x;
  const Best b{keys, items, &count};
  top_row(a, r, x, &count);
  const int n = a.count[r];
  if (n > a.room) {
    top_all(a, r, x, b, 0, a.items);
  } else {
    uint64_t least = 0;
    for (int base = 0; base < n; base += kThreads)
      top_batch(a, x, b, least, n - base, [&](int q) { return a.found[r * a.room + base + q]; });
    best_cut(b, a.k);
  }
  top_out(a, r, b);
}

__global__ __launch_bounds__(kThreads) void k_clear(uint32_t *p, int64_t n) {
  for (int64_t q = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x; q < n; q += static_cast<int64_t>(gridDim.x) * kThreads)
    p[q] = 0;
}
// a bit per excluded item; one wavefront per row
__global__ __launch_bounds__(kThreads) void k_exclude(const int64_t *row_ptr, const int32_t *item, int64_t entries, int64_t row0,
                                                      int64_t n, int32_t items, int32_t words, uint32_t *bits) {
  const int64_t r = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (r >= n) return;
  int64_t b, e;
  row_range(row_ptr, entries, 0, row0 + r, b, e);
  for (int64_t q = b + (threadIdx.x & 63); q < e; q += 64) {
    const int32_t j = item[q];
    if (j >= 0 && j < items) atomicOr(&bits[r * words + (j >> 5)], 1u << (j & 31));
  }
}

}  // namespace

// ------------------------------------------------------------------ the handle
struct ps_soft : pssoft::Shape {
  int device = -1;
  bool opened = false;
  hipStream_t stream = nullptr;  // NULL: HIP's null stream
  hipEvent_t moved = nullptr;
  char *work = nullptr;
  int64_t work_bytes = 0;
  bool captured = false;
  std::vector<void *> kept;  // workspaces that a captured graph may hold
  std::string err;
};

namespace {

int fail(ps_soft_t *h, int code, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  try {
    h->err = buf;
  } catch (const std::bad_alloc &) {
  }
  return code;
}

#define SOFT_TRY(h, expr)                                                                                      \
  do {                                                                                                        \
    const hipError_t e_ = (expr);                                                                             \
    if (e_ != hipSuccess) {                                                                                   \
      (void)hipGetLastError();                                                                                \
      return fail(h, e_ == hipErrorOutOfMemory ? PS_SOFT_ENOMEM : PS_SOFT_EDEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
    }                                                                                                         \
  } while (0)

// The caller's device comes back when the call returns
struct DeviceGuard {
  int before = -1;
  ~DeviceGuard() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

int open(ps_soft_t *h, DeviceGuard &guard) {
  int dev = 0;
  SOFT_TRY(h, hipGetDevice(&dev));
  if (h->device < 0) h->device = dev;
  if (h->device != dev) {
    const hipError_t e = hipSetDevice(h->device);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      return fail(h, PS_SOFT_EDEVICE, "hipSetDevice(%d): %s", h->device, hipGetErrorString(e));
    }
    guard.before = dev;
  }
  h->opened = true;
  return PS_SOFT_OK;
}

int capturing(ps_soft_t *h, hipStream_t s, bool *out) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (s) SOFT_TRY(h, hipStreamIsCapturing(s, &st));  // the null stream is never captured
  *out = st == hipStreamCaptureStatusActive;
  return PS_SOFT_OK;
}

int grow(ps_soft_t *h, int64_t bytes) {
  bool cap = false;
  const int rc = capturing(h, h->stream, &cap);
  if (rc) return rc;
  if (cap && bytes > h->work_bytes)
    return fail(h, PS_SOFT_ESTATE, "the workspace has %lld of %lld bytes and cannot grow while the stream is captured: ps_soft_reserve, or the call itself, before",
                (long long)h->work_bytes, (long long)bytes);
  h->captured = h->captured || cap;
  if (bytes <= h->work_bytes) return PS_SOFT_OK;
  SOFT_TRY(h, hipStreamSynchronize(h->stream));
  if (h->work) {
    if (h->captured) {
      try {
        h->kept.push_back(h->work);
      } catch (const std::bad_alloc &) {
        return fail(h, PS_SOFT_ENOMEM, "host memory");
      }
    } else {
      (void)hipFree(h->work);
    }
    h->work = nullptr;
    h->work_bytes = 0;
  }
  void *p = nullptr;
  const hipError_t e = hipMalloc(&p, static_cast<size_t>(bytes));
  if (e != hipSuccess) {
    (void)hipGetLastError();
    return fail(h, e == hipErrorOutOfMemory ? PS_SOFT_ENOMEM : PS_SOFT_EDEVICE, "workspace of %lld bytes: %s", (long long)bytes, hipGetErrorString(e));
  }
  h->work = static_cast<char *>(p);
  h->work_bytes = bytes;
  return PS_SOFT_OK;
}

unsigned blocks_for(int64_t n, int64_t per, int64_t most) {
  return static_cast<unsigned>(std::max<int64_t>(1, std::min(up(n, per), most)));
}

dim3 grid_of(int64_t blocks) {  // for kernels that use block_index(); the last dimension's surplus returns at once
  const int64_t most = 1LL << kGridBits;
  return dim3(static_cast<unsigned>(std::min(blocks, most)), static_cast<unsigned>(up(blocks, most)));
}

int32_t row_lanes(int32_t K) {  // lanes of 4 numbers for a row, a power of two
  int32_t n = 1;
  while (4 * n < K) n *= 2;
  return n;
}

template <class T>
bool aligned4(const T *p, int64_t ld) {
  return (reinterpret_cast<uintptr_t>(p) % (4 * sizeof(T))) == 0 && ld % 4 == 0;
}

void hip_launch(void (*f)(PassArgs), dim3 grid, unsigned lds, const PassArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(f, grid, dim3(64 * kWaves), lds, s, a);
}

template <int NP, int KC, int DB>
void launch_pass(const PassArgs &a, bool col, hipStream_t s) {
  const dim3 grid = grid_of(up(a.own_tiles, kWaves) * a.splits);
  const unsigned lds = static_cast<unsigned>(stage_of(NP, KC, DB, col).halves * 2);
  if (!col) {
    hip_launch((k_pass<NP, KC, DB, false>), grid, lds, a, s);
  } else if constexpr (DB > 0) {
    hip_launch((k_pass<NP, KC, DB, true>), grid, lds, a, s);
  }
}

template <int NP, int KC>
void run_pass_of(PassArgs a, bool col, bool sums, hipStream_t s) {
  constexpr int KD = KC / 2, DB = std::min(KD, 8);
  a.d0 = 0;
  if (!sums) launch_pass<NP, KC, 0>(a, false, s);
  else
    for (; a.d0 < KD; a.d0 += DB) launch_pass<NP, KC, DB>(a, col, s);
}
template <int NP>
void run_pass(const PassArgs &a, int k16, bool col, bool sums, hipStream_t s) {
  switch (k16) {
    case 2: return run_pass_of<NP, 2>(a, col, sums, s);
    case 4: return run_pass_of<NP, 4>(a, col, sums, s);
    case 6: return run_pass_of<NP, 6>(a, col, sums, s);
    case 8: return run_pass_of<NP, 8>(a, col, sums, s);
    case 12: return run_pass_of<NP, 12>(a, col, sums, s);
    case 16: return run_pass_of<NP, 16>(a, col, sums, s);
    default: return run_pass_of<NP, 32>(a, col, sums, s);
  }
}

template <class T, int G, int V>
void run_rows(const RowArgs<T> &a, hipStream_t s) {
  const int64_t rows = a.rowvec ? up(a.t.n, kTile) * kTile : a.t.n;
  // wavefronts per row: all that 256 CUs hold, for lists long enough
  if (a.t.n <= 256) hipLaunchKernelGGL((k_row_finish<T, G, V, 16>), dim3(static_cast<unsigned>(rows)), dim3(1024), 0, s, a);
  else if (a.t.n <= 2048) hipLaunchKernelGGL((k_row_finish<T, G, V, 4>), dim3(static_cast<unsigned>(rows)), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((k_row_finish<T, G, V, 1>), grid_of(up(rows, 4)), dim3(kThreads), 0, s, a);
}

// Lanes per row: 4 numbers each, 8 above 256
template <class F>
void by_k(int K, F f) {
  if (K <= 16) f(std::integral_constant<int, 4>{}, std::integral_constant<int, 1>{});
  else if (K <= 32) f(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
  else if (K <= 64) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 1>{});
  else if (K <= 128) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 1>{});
  else if (K <= 256) f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{});
  else f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
}

// One loss with its gradients; `t` holds the caller's lists
template <class T, bool Distill>
int soft_loss(ps_soft_t *h, Targets t, const T *X, int64_t ldx, const T *W, int64_t ldw, float *loss, float *lse, T *dX,
              int64_t lddx, T *dW, int64_t lddw) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;
  const bool dx = dX != nullptr, dw = dW != nullptr;
  const Plan p = plan(h, t.n, t.entries, dx, dw);
  int rc = grow(h, p.bytes);
  if (rc) return rc;
  char *const base = h->work;
  auto at_f = [&](int64_t o) { return reinterpret_cast<float *>(base + o); };
  auto at_i = [&](int64_t o) { return reinterpret_cast<int32_t *>(base + o); };
  hipStream_t s = h->stream;
  Scal *scal = reinterpret_cast<Scal *>(base + p.scal);
  t.items = static_cast<int32_t>(h->items);
  t.dead = static_cast<int32_t>(p.wt);
  t.key = dw ? at_i(p.key[0]) : nullptr;
  t.pay = reinterpret_cast<uint2 *>(base + p.pay[0]);
  t.act = at_i(p.act);
  t.total = at_f(p.total);
  t.extra = at_f(p.extra);
  t.share = at_f(p.share);
  t.gw = at_f(p.gw);
  t.logz = reinterpret_cast<double *>(base + p.logz);
  t.part = at_f(p.row_part);
  Table<T> x{X, ldx, t.n, aligned4(X, ldx), t.act}, w{W, ldw, h->items, aligned4(W, ldw), nullptr};
  _Float16 *px = reinterpret_cast<_Float16 *>(base + p.px), *pw = reinterpret_cast<_Float16 *>(base + p.pw);
  const float scale = 1.44269504088896340736f / t.tau;
  if (t.n > 0) {
    if (t.row_ptr && dw && t.entries > 0)
      hipLaunchKernelGGL(k_fill_keys, dim3(blocks_for(t.entries, kThreads * 4, 4096)), dim3(kThreads), 0, s, t.key, t.entries, t.dead);
    const unsigned row_blocks = blocks_for(t.n, 4, kRowParts);
    hipLaunchKernelGGL((k_targets<Distill>), dim3(row_blocks), dim3(kThreads), 0, s, t);
    PassArgs a{};
    a.m = at_f(p.m);
    a.l = at_f(p.l);
    a.o = at_f(p.o);
    if (p.few) {
      const FewArgs f{t.n, p.xt * kTile, t.items, h->K, p.few_items, t.act, scale, a.m, a.l};
      const int64_t at_once = few_rows(t.n);
      const dim3 grid(static_cast<unsigned>(p.rsplits), static_cast<unsigned>(up(t.n, at_once)));
      if (at_once == 8) hipLaunchKernelGGL((k_few<T, 8>), grid, dim3(kThreads), 0, s, f, x, w);
      else if (at_once == 4) hipLaunchKernelGGL((k_few<T, 4>), grid, dim3(kThreads), 0, s, f, x, w);
      else hipLaunchKernelGGL((k_few<T, 1>), grid, dim3(kThreads), 0, s, f, x, w);
    } else {
      hipLaunchKernelGGL((k_absmax<T>), dim3(2 * kParts), dim3(kScanThreads), 0, s, x, w, h->K, row_lanes(h->K), at_f(p.part));
      const PackSide sx{px, p.x_stride, static_cast<int32_t>(p.xt), dw}, sw{pw, p.w_stride, static_cast<int32_t>(p.wt), dx};
      hipLaunchKernelGGL((k_pack<T, NP>), grid_of(p.xt + p.wt), dim3(kThreads),
                         static_cast<unsigned>(kTile * (std::min(p.kd, kPackBlocks) * 32 + 1) * 4), s, x, w, sx, sw, h->K, p.k16, p.kd, at_f(p.part),
                         at_f(p.row_part), static_cast<int32_t>(row_blocks), scal);
      a.own = px;
      a.own_stride = p.x_stride;
      a.own_tiles = p.xt;
      a.splits = p.rsplits;
      a.str = pw;
      a.str_stride = p.w_stride;
      a.str_rows = h->items;
      a.scal = scal;
      a.scale = scale;
      a.tiles_per_split = p.rper;
      run_pass<NP>(a, p.k16, false, dx, s);
    }
    RowArgs<T> r{};
    r.t = t;
    r.own_pad = p.xt * kTile;
    r.K = h->K;
    r.ldo = p.kd * 32;
    r.splits = p.rsplits;
    r.x = x;
    r.w = w;
    r.scal = scal;
    r.scale = p.few ? 0.f : scale;
    r.m = a.m;
    r.l = a.l;
    r.o = a.o;
    r.loss = loss;
    r.lse = lse;
    r.dX = dX;
    r.lddx = lddx;
    r.vec_out = dx && aligned4(dX, lddx);
    r.rowvec = dw ? at_f(p.rowvec) : nullptr;
    by_k(h->K, [&](auto g, auto v) { run_rows<T, g(), v()>(r, s); });
    if (dw) {
      Records rec[2];
      for (int q = 0; q < 2; ++q) rec[q] = Records{at_i(p.key[q]), reinterpret_cast<uint2 *>(base + p.pay[q])};
      int64_t *first = reinterpret_cast<int64_t *>(base + p.first);
      const int32_t firsts = static_cast<int32_t>(p.wt + 1);
      int from = 0;
      if (t.entries > 0) {
        for (int q = 0; q < p.passes; ++q, from ^= 1) {
          const dim3 blocks(static_cast<unsigned>(p.sort_blocks));
          if (p.sort_blocks > 1) {
            hipLaunchKernelGGL(k_sort_count, blocks, dim3(kThreads), 0, s, rec[from].key, t.entries, q * p.bits, 1 << p.bits, at_i(p.hist),
                               p.sort_blocks);
            hipLaunchKernelGGL(k_sort_scan, dim3(1 << p.bits), dim3(kThreads), 0, s, at_i(p.hist), p.sort_blocks, at_i(p.bins));
          }
          hipLaunchKernelGGL(k_sort_move, blocks, dim3(kSortThreads), 0, s, rec[from], rec[from ^ 1], t.entries, q * p.bits, p.bits,
                             at_i(p.hist), p.sort_blocks, at_i(p.bins), p.passes == 1 ? first : nullptr, firsts);
        }
        if (p.passes > 1)
          hipLaunchKernelGGL(k_first, dim3(static_cast<unsigned>(up(firsts, kThreads))), dim3(kThreads), 0, s, rec[from].key, t.entries, first,
                             firsts);
      }
      a.own = pw;
      a.own_stride = p.w_stride;
      a.own_tiles = p.wt;
      a.splits = p.csplits;
      a.str = px;
      a.str_stride = p.x_stride;
      a.str_rows = t.n;
      a.rowvec = at_f(p.rowvec);
      a.tiles_per_split = p.cper;
      a.first = t.entries > 0 ? first : nullptr;
      a.pay = rec[from].pay;
      run_pass<NP>(a, p.k16, true, true, s);
    }
  }
  if (dw) {
    ItemArgs<T> a{};
    a.own_pad = p.wt * kTile;
    a.items = t.items;
    a.K = h->K;
    a.ldo = p.kd * 32;
    a.splits = t.n > 0 ? p.csplits : 0;
    a.scal = scal;
    a.m = at_f(p.m);
    a.o = at_f(p.o);
    a.dW = dW;
    a.lddw = lddw;
    a.vec_out = aligned4(dW, lddw);
    by_k(h->K, [&](auto g, auto v) {
      hipLaunchKernelGGL((k_item_finish<T, g(), v()>), grid_of(up(h->items, kThreads / g())), dim3(kThreads), 0, s, a);
    });
  }
  SOFT_TRY(h, hipGetLastError());
  return PS_SOFT_OK;
}

template <int KC, bool Find>
void run_score_of(const ScoreArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((k_score<KC, Find>), dim3(static_cast<unsigned>(up(a.own_tiles, 2 * kWaves) * a.splits)), dim3(kThreads), 0, s, a);
}
template <bool Find>
void run_score(const ScoreArgs &a, int32_t kc, hipStream_t s) {
  switch (kc) {
    case 2: return run_score_of<2, Find>(a, s);
    case 3: return run_score_of<3, Find>(a, s);
    case 5: return run_score_of<5, Find>(a, s);
    case 7: return run_score_of<7, Find>(a, s);
    case 9: return run_score_of<9, Find>(a, s);
    case 13: return run_score_of<13, Find>(a, s);
    case 17: return run_score_of<17, Find>(a, s);
    case 25: return run_score_of<25, Find>(a, s);
    default: return run_score_of<33, Find>(a, s);
  }
}

template <class T>
int soft_top(ps_soft_t *h, int64_t n, const T *X, int64_t ldx, const T *W, int64_t ldw, int32_t k, const int64_t *row_ptr,
             const int32_t *item, int64_t entries, int32_t *top_item, float *top_score, int64_t ldo) {
  const TopPlan p = top_plan(h, n, k, row_ptr != nullptr, h->search);
  const int rc = grow(h, p.bytes);
  if (rc) return rc;
  char *const base = h->work;
  hipStream_t s = h->stream;
  TopArgs<T> a{};
  a.items = static_cast<int32_t>(h->items);
  a.K = h->K;
  a.k = k;
  a.words = p.words;
  a.x = Table<T>{X, ldx, n, aligned4(X, ldx), nullptr};
  a.w = Table<T>{W, ldw, h->items, aligned4(W, ldw), nullptr};
  uint32_t *bits = reinterpret_cast<uint32_t *>(base + p.bits);
  a.excluded = row_ptr ? bits : nullptr;
  a.row_ptr = row_ptr;
  a.list = item;
  a.entries = entries;
  a.groups = p.groups;
  a.key = reinterpret_cast<uint64_t *>(base + p.key);
  a.most = reinterpret_cast<uint64_t *>(base + p.maxima);
  a.found = reinterpret_cast<int32_t *>(base + p.found);
  a.count = reinterpret_cast<int32_t *>(base + p.count);
  a.room = kCandidates;
  a.out_item = top_item;
  a.out_score = top_score;
  a.ldo = ldo;
  float *part = reinterpret_cast<float *>(base + p.part);
  if (p.filter && h->type != PS_SOFT_F16)
    hipLaunchKernelGGL((k_absmax<T>), dim3(2 * kParts), dim3(kScanThreads), 0, s, a.x, a.w, h->K, row_lanes(h->K), part);
  for (a.row0 = 0; a.row0 < n; a.row0 += p.rows) {
    a.n = std::min(p.rows, n - a.row0);
    const unsigned rows = static_cast<unsigned>(a.n);
    if (!p.filter) {
      const int64_t at_once = a.n >= 8 ? 8 : a.n >= 3 ? 4 : 1, blocks = up(a.n, at_once);
      const int32_t per = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(kTopGroups, p.groups * blocks / 768)));
      const dim3 grid(static_cast<unsigned>(up(p.groups, per)), static_cast<unsigned>(blocks));
      if (at_once == 8) hipLaunchKernelGGL((k_top_scores<T, 8>), grid, dim3(kThreads), 0, s, a, per);
      else if (at_once == 4) hipLaunchKernelGGL((k_top_scores<T, 4>), grid, dim3(kThreads), 0, s, a, per);
      else hipLaunchKernelGGL((k_top_scores<T, 1>), grid, dim3(kThreads), 0, s, a, per);
      hipLaunchKernelGGL((k_top_pick<T>), dim3(rows), dim3(kThreads), 0, s, a);
      continue;
    }
    if (row_ptr) {
      hipLaunchKernelGGL(k_clear, dim3(blocks_for(a.n * p.words, kThreads * 4, 8192)), dim3(kThreads), 0, s, bits, a.n * p.words);
      hipLaunchKernelGGL(k_exclude, dim3(static_cast<unsigned>(up(a.n, 4))), dim3(kThreads), 0, s, row_ptr, item, entries, a.row0,
                         a.n, a.items, p.words, bits);
    }
    ScoreArgs q{};
    _Float16 *px = reinterpret_cast<_Float16 *>(base + p.px), *pw = reinterpret_cast<_Float16 *>(base + p.pw);
    int32_t *count = reinterpret_cast<int32_t *>(base + p.count);
    const int64_t xt = up(a.n, kTile);
    const float c = (h->type == PS_SOFT_F32 ? 0x1p-10f + 0x1p-22f : 0.f) + (2 * p.kc + 16) * 0x1p-22f + std::sqrt(static_cast<float>(h->K)) * 0x1p-24f;
    const int kd = std::min((h->K + 31) / 32, kPackBlocks);
    hipLaunchKernelGGL((k_top_pack<T>), grid_of(xt + (a.row0 ? 0 : p.wt)), dim3(kThreads),
                       static_cast<unsigned>(kTile * (kd * 32 + 1) * 4), s, a.x, a.w, a.row0, a.n, static_cast<int32_t>(xt), px, pw, h->K,
                       p.kc, c, part, count);
    q.own = px;
    q.str = pw;
    q.rows = a.n;
    q.own_tiles = xt;
    q.tiles = p.wt;
    q.steps_per_split = p.per_split;
    q.items = a.items;
    q.splits = p.splits;
    q.words = p.words;
    q.last = h->K / 16;
    q.excluded = a.excluded;
    q.most = reinterpret_cast<float *>(base + p.most);
    q.steps = p.steps;
    q.per_row = p.per_row;
    float *least = reinterpret_cast<float *>(base + p.least);
    q.least = least;
    q.found = reinterpret_cast<int32_t *>(base + p.found);
    q.count = count;
    run_score<false>(q, p.kc, s);
    hipLaunchKernelGGL(k_top_least, dim3(rows), dim3(kThreads), 0, s, q.most, p.per_row, k, least);
    run_score<true>(q, p.kc, s);
    hipLaunchKernelGGL((k_top_rank<T>), dim3(rows), dim3(kThreads), 0, s, a);
  }
  SOFT_TRY(h, hipGetLastError());
  return PS_SOFT_OK;
}

int check_tables(ps_soft_t *h, int64_t n, const void *X, int64_t ldx, const void *W, int64_t ldw) {
  if (n < 0 || n > kMaxRows) return fail(h, PS_SOFT_EINVAL, "rows must be in [0, 2^26], not %lld", (long long)n);
  if ((n > 0 && !X) || !W) return fail(h, PS_SOFT_EINVAL, "null table");
  if (ldx < h->K || ldw < h->K) return fail(h, PS_SOFT_EINVAL, "row strides must be at least K = %d", h->K);
  return PS_SOFT_OK;
}

int check_outputs(ps_soft_t *h, const void *dX, int64_t lddx, const void *dW, int64_t lddw, int64_t entries) {
  if ((dX && lddx < h->K) || (dW && lddw < h->K)) return fail(h, PS_SOFT_EINVAL, "gradients' row strides must be at least K = %d", h->K);
  if (entries < 0 || entries > kMaxEntries) return fail(h, PS_SOFT_EINVAL, "entries must be in [0, 2^31 - 65], not %lld", (long long)entries);
  return PS_SOFT_OK;
}

template <bool Distill>
int any_loss(ps_soft_t *h, const Targets &t, const void *X, int64_t ldx, const void *W, int64_t ldw, float *loss, float *lse, void *dX,
             int64_t lddx, void *dW, int64_t lddw) {
  DeviceGuard guard;
  const int rc = open(h, guard);
  if (rc) return rc;
  switch (h->type) {
    case PS_SOFT_F32:
      return soft_loss<float, Distill>(h, t, static_cast<const float *>(X), ldx, static_cast<const float *>(W), ldw, loss, lse,
                                       static_cast<float *>(dX), lddx, static_cast<float *>(dW), lddw);
    case PS_SOFT_BF16:
      return soft_loss<bf16_t, Distill>(h, t, static_cast<const bf16_t *>(X), ldx, static_cast<const bf16_t *>(W), ldw, loss, lse,
                                        static_cast<bf16_t *>(dX), lddx, static_cast<bf16_t *>(dW), lddw);
    default:
      return soft_loss<f16_t, Distill>(h, t, static_cast<const f16_t *>(X), ldx, static_cast<const f16_t *>(W), ldw, loss, lse,
                                       static_cast<f16_t *>(dX), lddx, static_cast<f16_t *>(dW), lddw);
  }
}

}  // namespace

extern "C" {

int ps_soft_create(int64_t items, int32_t K, int32_t type, ps_soft_t **out) {
  if (!out) return PS_SOFT_EINVAL;
  *out = nullptr;
  if (items < 1 || items > kMaxItems || K < 1 || K > kMaxK || type < PS_SOFT_F32 || type > PS_SOFT_F16) return PS_SOFT_EINVAL;
  ps_soft_t *h = new (std::nothrow) ps_soft_t();
  if (!h) return PS_SOFT_ENOMEM;
  h->items = items;
  h->K = K;
  h->type = type;
  *out = h;
  return PS_SOFT_OK;
}

int ps_soft_set_option(ps_soft_t *h, int32_t key, int64_t value) {
  if (!h) return PS_SOFT_EINVAL;
  switch (key) {
    case PS_SOFT_OPT_DEVICE:
      if (value < -1 || value > 4095) return fail(h, PS_SOFT_EINVAL, "device ordinal must be in [-1, 4095]");
      if (h->opened) return fail(h, PS_SOFT_ESTATE, "the device is already in use");
      h->device = static_cast<int>(value);
      return PS_SOFT_OK;
    case PS_SOFT_OPT_SPLITS:
      if (value < 0 || value > 1024) return fail(h, PS_SOFT_EINVAL, "pieces must be in [0, 1024]");
      h->splits = static_cast<int32_t>(value);
      return PS_SOFT_OK;
    case PS_SOFT_OPT_SEARCH:
      if (value < -1 || value > 1) return fail(h, PS_SOFT_EINVAL, "the search's form must be in [-1, 1]");
      h->search = static_cast<int32_t>(value);
      return PS_SOFT_OK;
    default:
      return fail(h, PS_SOFT_EINVAL, "unknown option key %d", key);
  }
}

int ps_soft_set_stream(ps_soft_t *h, void *hip_stream) {
  if (!h) return PS_SOFT_EINVAL;
  hipStream_t to = static_cast<hipStream_t>(hip_stream);
  if (h->stream == to || !h->opened) {
    h->stream = to;
    return PS_SOFT_OK;
  }
  DeviceGuard guard;
  int rc = open(h, guard);
  if (rc) return rc;
  bool from_cap = false, to_cap = false;
  if ((rc = capturing(h, h->stream, &from_cap)) || (rc = capturing(h, to, &to_cap))) return rc;
  if (!from_cap && !to_cap) {
    if (!h->moved) SOFT_TRY(h, hipEventCreateWithFlags(&h->moved, hipEventDisableTiming));
    SOFT_TRY(h, hipEventRecord(h->moved, h->stream));
    SOFT_TRY(h, hipStreamWaitEvent(to, h->moved, 0));
  }
  h->stream = to;
  return PS_SOFT_OK;
}

int ps_soft_reserve(ps_soft_t *h, int64_t n, int64_t entries, int32_t top) {
  if (!h) return PS_SOFT_EINVAL;
  if (n < 0 || n > kMaxRows || entries < 0 || entries > kMaxEntries || top < 0 || top > kMaxTop)
    return fail(h, PS_SOFT_EINVAL, "rows must be in [0, 2^26], entries in [0, 2^31 - 65], top in [0, %d]", kMaxTop);
  DeviceGuard guard;
  const int rc = open(h, guard);
  if (rc) return rc;
  return grow(h, reserved_bytes(h, n, entries, top));
}

int ps_soft_xent(ps_soft_t *h, int64_t n, const void *X, int64_t ldx, const void *W, int64_t ldw, const int64_t *row_ptr,
                 const int32_t *item, const float *value, int64_t entries, const float *weight, float *loss, float *lse, void *dX,
                 int64_t lddx, void *dW, int64_t lddw) {
  if (!h) return PS_SOFT_EINVAL;
  int rc = check_tables(h, n, X, ldx, W, ldw);
  if (rc || (rc = check_outputs(h, dX, lddx, dW, lddw, entries))) return rc;
  if (!row_ptr && entries != n) return fail(h, PS_SOFT_EINVAL, "one target per row takes entries = n");
  if (entries > 0 && !item) return fail(h, PS_SOFT_EINVAL, "null item list");
  Targets t{};
  t.n = n;
  t.entries = entries;
  t.k = 1;
  t.row_ptr = row_ptr;
  t.item = item;
  t.value = value;
  t.tau = 1.f;
  t.per_tau = 1.0;
  t.weight = weight;
  return any_loss<false>(h, t, X, ldx, W, ldw, loss, lse, dX, lddx, dW, lddw);
}

int ps_soft_distill(ps_soft_t *h, int64_t n, const void *X, int64_t ldx, const void *W, int64_t ldw, int32_t k, const int32_t *item,
                    const float *score, int64_t ldt, float tau, const float *tlse, const float *weight, float *loss, float *lse,
                    void *dX, int64_t lddx, void *dW, int64_t lddw) {
  if (!h) return PS_SOFT_EINVAL;
  int rc = check_tables(h, n, X, ldx, W, ldw);
  if (rc) return rc;
  if (k < 1 || ldt < k) return fail(h, PS_SOFT_EINVAL, "teacher's lists: k = %d, stride %lld", k, (long long)ldt);
  if (!(tau > 0) || !std::isfinite(tau)) return fail(h, PS_SOFT_EINVAL, "tau must be positive and finite");
  if (n > 0 && (!item || !score)) return fail(h, PS_SOFT_EINVAL, "null teacher's lists");
  if ((rc = check_outputs(h, dX, lddx, dW, lddw, n * k))) return rc;
  Targets t{};
  t.n = n;
  t.entries = n * k;
  t.k = k;
  t.item = item;
  t.score = score;
  t.tlse = tlse;
  t.ldt = ldt;
  t.tau = tau;
  t.per_tau = 1.0 / tau;
  t.weight = weight;
  return any_loss<true>(h, t, X, ldx, W, ldw, loss, lse, dX, lddx, dW, lddw);
}

int ps_soft_top(ps_soft_t *h, int64_t n, const void *X, int64_t ldx, const void *W, int64_t ldw, int32_t k, const int64_t *row_ptr,
                const int32_t *item, int64_t entries, int32_t *top_item, float *top_score, int64_t ldo) {
  if (!h) return PS_SOFT_EINVAL;
  int rc = check_tables(h, n, X, ldx, W, ldw);
  if (rc) return rc;
  if (k < 1 || k > kMaxTop || ldo < k) return fail(h, PS_SOFT_EINVAL, "k must be in [1, %d] and the outputs' stride at least k", kMaxTop);
  if (entries < 0 || entries > kMaxEntries) return fail(h, PS_SOFT_EINVAL, "entries must be in [0, 2^31 - 65], not %lld", (long long)entries);
  if (row_ptr && entries > 0 && !item) return fail(h, PS_SOFT_EINVAL, "null item list");
  if (n > 0 && (!top_item || !top_score)) return fail(h, PS_SOFT_EINVAL, "null outputs");
  if (n == 0) return PS_SOFT_OK;
  DeviceGuard guard;
  if ((rc = open(h, guard))) return rc;
  switch (h->type) {
    case PS_SOFT_F32:
      return soft_top<float>(h, n, static_cast<const float *>(X), ldx, static_cast<const float *>(W), ldw, k, row_ptr, item, entries,
                             top_item, top_score, ldo);
    case PS_SOFT_BF16:
      return soft_top<bf16_t>(h, n, static_cast<const bf16_t *>(X), ldx, static_cast<const bf16_t *>(W), ldw, k, row_ptr, item, entries,
                              top_item, top_score, ldo);
    default:
      return soft_top<f16_t>(h, n, static_cast<const f16_t *>(X), ldx, static_cast<const f16_t *>(W), ldw, k, row_ptr, item, entries,
                             top_item, top_score, ldo);
  }
}

const char *ps_soft_last_error(const ps_soft_t *h) {
  return h ? h->err.c_str() : "";
}

void ps_soft_destroy(ps_soft_t *h) {
  if (!h) return;
  if (h->opened) {
    DeviceGuard guard;
    int dev = 0;
    if (hipGetDevice(&dev) == hipSuccess && dev != h->device && hipSetDevice(h->device) == hipSuccess) guard.before = dev;
    (void)hipStreamSynchronize(h->stream);
    if (h->work) (void)hipFree(h->work);
    for (void *p : h->kept) (void)hipFree(p);
    if (h->moved) (void)hipEventDestroy(h->moved);
    (void)hipGetLastError();
  }
  delete h;
}

}  // extern "C"

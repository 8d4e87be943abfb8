// Linear attention in bfloat16 and float16: the sweeps of linattn.hip on the 16-bit
// matrix instructions (sixteen times the rate of the 32-bit ones), in chunks of
// 64 positions, 32 columns a wave and the scores shared by the workgroup.
//
// What bounds a sweep here is what surrounds the matrix unit: operands out of
// LDS, 32-bit factors taken apart, waits.  So a wave's block is as large as its
// registers hold (32 columns: each operand read from LDS meets 32 of them),
// each 32 x 32 block of the scores is formed once (the waves take them in
// turn, put them into LDS as the operand that the product with the values
// reads, and do the state's products before the barrier that the scores
// need), the next chunk's tiles are fetched into registers meanwhile, and
// loops that need not be unrolled are not: the first chunk of a launch waits for its
// instructions too (0.5 us a KB of them).
//
// Measured: 100,003 positions of 8 heads, 64 x 64 states, 92 us for 410 MB
// (4.5 TB/s) after 41 us of segment states; 4 x 4,096 positions of 16 heads, 128 x 128
// states, 85 us for 268 MB in eight segments, and 290 to 335 us for the three gradients
// in one segment, 192 workgroups of which each has a compute unit to itself:
// 4.5 to 5.2 us a chunk, of which the vector, the matrix and the LDS units are busy 68%,
// 42% and 42%, in turn.
//
// A lane's eight elements of a contraction are those that a result gives it
// (32 x 32: rows 4 h + r and 8 + 4 h + r of each 16, h = lane / 32).  The
// transposed operands (K^T for the state, V^T) are read from the row-major
// tiles by the transposing LDS load: sixteen lanes read 4 rows x 16 columns
// and each gets its column of them.
//
// q.k products of 16-bit factors are exact in the matrix unit.  The other
// products have one 32-bit factor (the scores, the entering state, the weighted
// values), taken in three 16-bit parts, which keep its 24 bits: a state of 2^23 and
// one of a unit less still differ by that unit in an output.  (Two parts, 16 bits, would
// do for outputs that do not cancel, in four fifths of the time.)  What is left of an infinity is
// NaN: an infinite input, score or state gives NaN where the sum would be infinite.
//
// A float16 input is taken apart into two bfloat16 parts as it enters LDS, which is
// exact (8 and 3 bits): bfloat16's range, whatever the states and scores grow to.  Of
// a 32-bit factor the lowest part times an input's low one is left out (2^-25 of a
// term).  It costs two thirds as many products again (of the scores four times as many) and
// twice the LDS, so dimensions to 128; 4 x 4,096 positions of 16 heads, 128 x 128: forward and
// gradients in 610 us, 1,360 on the 32-bit instructions.
#include "linattn.hpp"

namespace fstc {
namespace {

using b16x2 = bf16 __attribute__((ext_vector_type(2)));
using b16x4 = bf16 __attribute__((ext_vector_type(4)));
using b16x8 = bf16 __attribute__((ext_vector_type(8)));
using s16x4 = short __attribute__((ext_vector_type(4)));
using f32x2 = float __attribute__((ext_vector_type(2)));
using f32x16 = float __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16 mfma32(b16x8 a, b16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Column lane % 16 of 4 rows: `p` is the lane's quad, row (lane % 16) / 4 of
// them and columns 4 * (lane % 4) .. + 3.
__device__ __forceinline__ b16x4 read_transposed(const bf16 *p) {
  return __builtin_bit_cast(b16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                       (__attribute__((address_space(3))) s16x4 *)p));
}

__device__ __forceinline__ b16x8 both(b16x4 a, b16x4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ b16x8 read_both(const bf16 *a, const bf16 *b) {
  return both(*reinterpret_cast<const b16x4 *>(a), *reinterpret_cast<const b16x4 *>(b));
}

// Lanes l and l + 32 hold columns 0-3 and 4-7 of one eight (x) and of the next
// (y), 16 bits each: eight of `x` to the lower lane, eight of `y` to the upper.
using u32x2 = u32 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u32x4 exchange(u32x2 x, u32x2 y) {
  const auto p = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false);
  const auto q = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
  return u32x4{p[0], q[0], p[1], q[1]};
}

// The nearest 16-bit values of N numbers, which keep what is left.
template <int N>
__device__ __forceinline__ void take_part(float (&x)[N], bf16 (&part)[N]) {
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    const b16x2 y = __builtin_convertvector((f32x2{x[e], x[e + 1]}), b16x2);
    const u32 w = __builtin_bit_cast(u32, y);
    part[e] = y[0];
    part[e + 1] = y[1];
    x[e] -= __builtin_bit_cast(float, w << 16);
    x[e + 1] -= __builtin_bit_cast(float, w & 0xffff0000u);
  }
}
template <class T = bf16, int N>
__device__ __forceinline__ auto round_all(const float (&x)[N]) {
  using V = T __attribute__((ext_vector_type(N)));
  using V2 = T __attribute__((ext_vector_type(2)));
  V y;
#pragma unroll
  for (int e = 0; e < N; e += 2) {
    const V2 z = __builtin_convertvector((f32x2{x[e], x[e + 1]}), V2);
    y[e] = z[0];
    y[e + 1] = z[1];
  }
  return y;
}
template <int N>
__device__ __forceinline__ auto as_vector(const bf16 (&x)[N]) {
  using V = bf16 __attribute__((ext_vector_type(N)));
  V y;
#pragma unroll
  for (int e = 0; e < N; ++e) y[e] = x[e];
  return y;
}

// A number in 16-bit parts, which sum to it but for what N of them cannot hold.
template <int N>
__device__ __forceinline__ void parts_of(float (&x)[8], b16x8 (&part)[N]) {
#pragma unroll
  for (int i = 0; i < N - 1; ++i) {
    bf16 y[8];
    take_part(x, y);
    part[i] = as_vector(y);
  }
  part[N - 1] = round_all(x);
}

// Eight 16-bit elements without the first n, which may be 8 and more; zeros follow.
__device__ __forceinline__ u32x4 without_first(u32x4 x, u32 n) {
  const u64 lo = x[0] | (u64)x[1] << 32, hi = x[2] | (u64)x[3] << 32;
  const u32 s = n % 4 * 16;
  const u64 both = n < 4 ? lo >> s | (s ? hi << (64 - s) : 0) : n < 8 ? hi >> s : 0, top = n < 4 ? hi >> s : 0;
  return u32x4{(u32)both, (u32)(both >> 32), (u32)top, (u32)(top >> 32)};
}

// 64 rows of up to COLS elements on their way into LDS: zeros beyond n rows and
// `cols` columns.  fetch() starts the loads and put() ends them, so that the
// next chunk's are in flight while one is worked on.  FAST: rows of whole
// 16-byte units less than 2^24 bytes apart; a chunk's addresses are a uniform
// base and 32-bit offsets, clamped into the tile instead of branched on (a
// branch a unit would wait for each load in turn).  Of other rows the last
// unit is read as the row's last eight elements and shifted into place.
template <class T, int LD, int COLS, int NT, bool FAST>
struct Tile16 {
  static constexpr u32 kUnits = kChunk16 * (COLS / 8) / NT, kRows = NT / (COLS / 8);
  u32x4 x[kUnits];

  // rows p = first .. first + n - 1, at position p, or len - 1 - p in reverse
  __device__ __forceinline__ void fetch(const T *src, int64_t pos, u32 cols, u32 n, u32 first, u32 len,
                                        bool reverse) {
    const u32 row0 = threadIdx.x / (COLS / 8), c = threadIdx.x % (COLS / 8) * 8;
    const u32 low = reverse ? len - first - n : first;  // the lowest position
    if (FAST) {
      const char *base = reinterpret_cast<const char *>(src + (int64_t)low * pos);
      const u32 step = (u32)pos * 2, at = (c < cols ? c : 0) * 2;
#pragma unroll
      for (u32 u = 0; u < kUnits; ++u) {
        const u32 row = min(row0 + u * kRows, n - 1);
        x[u] = __builtin_bit_cast(
            u32x4, load_wide(reinterpret_cast<const T *>(base + (__umul24(reverse ? n - 1 - row : row, step) + at))));
      }
    } else {
#pragma unroll
      for (u32 u = 0; u < kUnits; ++u) {
        const u32 row = row0 + u * kRows;
        const T *s = src + (int64_t)(low + (reverse ? n - 1 - min(row, n - 1) : min(row, n - 1))) * pos;
        if (cols >= 8) {
          x[u] = __builtin_bit_cast(u32x4, load_wide(s + min(c, cols - 8)));
        } else {
          Vec<T, 8> y;
#pragma unroll
          for (u32 e = 0; e < 8; ++e) y.v[e] = c + e < cols ? s[c + e] : (T)0.f;
          x[u] = __builtin_bit_cast(u32x4, y);
        }
      }
    }
  }
  // `dst`: the tile, and kPlane elements on that of the second parts
  __device__ __forceinline__ void put(bf16 *dst, u32 cols, u32 n) const {
    const u32 row0 = threadIdx.x / (COLS / 8), c = threadIdx.x % (COLS / 8) * 8;
    bf16 *d = dst + row0 * LD + c;
    const bool whole = n == kChunk16 && (FAST ? cols >= COLS : false);
    const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
    for (u32 u = 0; u < kUnits; ++u) {
      u32x4 y = x[u];
      if (!FAST && cols >= 8 && c + 8 > cols) y = without_first(y, c + 8 - cols);
      y = whole || (row0 + u * kRows < n && c < cols) ? y : zero;
      if constexpr (std::is_same<T, bf16>::value) {
        *reinterpret_cast<u32x4 *>(d + u * kRows * LD) = y;
      } else {
        const auto h = __builtin_bit_cast(Vec<T, 8>, y);
        float z[8];
#pragma unroll
        for (u32 e = 0; e < 8; ++e) z[e] = (float)h.v[e];
        bf16 hi[8];
        take_part(z, hi);
        *reinterpret_cast<b16x8 *>(d + u * kRows * LD) = as_vector(hi);
        *reinterpret_cast<b16x8 *>(d + kPlane + u * kRows * LD) = round_all(z);
      }
    }
  }
  static constexpr int kPlane = kChunk16 * LD;
};

using f32x4u = float __attribute__((ext_vector_type(4), aligned(4)));

// A wave's block of a state, by strides: element r of block t is row
// 32 t + 8 (r / 4) + 4 half + r % 4, column `col`.  States have whole blocks
// (padded_dim).
template <int AB, bool LOAD>
__device__ __forceinline__ void move_state(f32x16 (&st)[AB], float *p, const States &s, u32 half, u32 col) {
  if (s.a == 1) {
    float *q = p + (u64)col * s.w + half * 4;
#pragma unroll
    for (int t = 0; t < AB; ++t)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        f32x4u *m = reinterpret_cast<f32x4u *>(q + t * 32 + y * 8);
        f32x4u x;
        if (LOAD) {
          x = *m;
#pragma unroll
          for (int e = 0; e < 4; ++e) st[t][y * 4 + e] = x[e];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = st[t][y * 4 + e];
          *m = x;
        }
      }
  } else {
    float *q = p + (u64)(half * 4) * s.a + col;
    const u32 a = (u32)s.a;
#pragma unroll
    for (int t = 0; t < AB; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        float *m = q + (t * 32 + r / 4 * 8 + r % 4) * a;
        if (LOAD) st[t][r] = *m;
        else *m = st[t][r];
      }
  }
}

// AB: blocks of 32 that hold the contraction's A elements; NW: blocks of 32 columns.
// P: waves of a block of columns, each with its share of the state's rows.  Of
// two, each forms its rows' part of all 64 outputs, hands the other 32 queries'
// to its partner through LDS, and finishes its own 32.
constexpr u32 kNone = 32;  // keys after the query, at most 31 in a block of 32
constexpr int kParts = 3;   // 16-bit parts of a 32-bit factor
template <class T, int AB, int NW, int P, bool OUT, bool FAST>
__global__ __launch_bounds__(P * NW * kWave, AB <= 4 ? 2 : 1) void k_attend16(AttendJobs jobs) {
  // Rows of the tiles are kPad elements apart more: 24 halve the bank conflicts of 8
  // (15.8 for 16.0 us a chunk of four workgroups of 128 x 128 states); of 64 x 64 states four
  // workgroups share a compute unit's LDS with 8, three with 24 (6.2, 8.9 us).
  constexpr int kPad = AB == 2 && NW == 2 ? 8 : 24;
  constexpr int SB = AB / P, kThreads = P * NW * kWave, kTile = NW * 32, kA = AB * 32, kLdA = kA + kPad, kLdV = kTile + kPad;
  constexpr int kIn = std::is_same<T, bf16>::value ? 1 : 2;  // of an input
  constexpr int kPlaneA = kChunk16 * kLdA, kPlaneV = kChunk16 * kLdV;
  __shared__ __align__(16) bf16 s_q[OUT ? kIn * kPlaneA : 8], s_k[kIn * kPlaneA], s_v[kIn * kPlaneV];
  // scores as operands of 32 queries: key blocks 0 and 1 of the first 32, 0 to 3 of the others
  // (32 bits a score, which each wave takes apart: three parts would be 6 bytes, and leave room
  // for three workgroups of 64 x 64 states on a compute unit, not four: 8.0 us a chunk, not 6.2)
  __shared__ __align__(16) float s_p[OUT ? 6 * kWave * 8 : 8];
  __shared__ f32x4 s_part[P == 2 ? P * NW * 4 * kWave : 1];  // outputs for the partner
  __shared__ float s_pow[kChunk16 + 1];                // g^n
  __shared__ float s_factor[OUT ? kNone + kChunk16 : 1];  // of a score, by query - key + kNone
  __shared__ __align__(16) float s_add[kChunk16];  // a row's weight in the state after the chunk
  const Part at = part_of(jobs);
  if (!at.any) return;
  const AttendArgs &a = jobs.j[at.job];
  const u32 seg = at.seg, bh = at.bh, b = bh / jobs.heads, h = bh % jobs.heads;
  const u32 len = row_length(jobs.lengths, b, jobs.length);
  const u32 p0 = seg * jobs.segment;
  const u32 rows = min(jobs.segment, jobs.length - min(p0, jobs.length));
  const u32 live = len > p0 ? min(jobs.segment, len - p0) : 0;
  const bool reverse = a.lead == 0;
  const u32 lane = lane_id(), l32 = lane & 31, half = lane / 32, li = lane & 15;
  const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const u32 block = wave % NW, part = P == 2 ? wave / NW : 0;  // of the columns, of the state's rows
  const u32 col0 = at.tile * kTile, cols = a.W - col0;

  const T *q = static_cast<const T *>(a.q.p) + b * a.q.batch + h * a.q.head;
  const T *k = static_cast<const T *>(a.k.p) + b * a.k.batch + h * a.k.head;
  const T *v = static_cast<const T *>(a.v.p) + b * a.v.batch + h * a.v.head + col0;
  T *out = OUT ? static_cast<T *>(a.out) + ((u64)b * jobs.length * jobs.heads + h) * a.W + col0 : nullptr;
  const u64 out_pos = (u64)jobs.heads * a.W;
  Tile16<T, kLdA, kA, kThreads, FAST> tq, tk;
  Tile16<T, kLdV, kTile, kThreads, FAST> tv;
  auto fetch = [&](u32 c) {
    const u32 n = min(kChunk16, live - c);
    if (OUT) tq.fetch(q, a.q.pos, a.A, n, p0 + c, len, reverse);
    tk.fetch(k, a.k.pos, a.A, n, p0 + c, len, reverse);
    tv.fetch(v, a.v.pos, cols, n, p0 + c, len, reverse);
  };
  f32x16 st[SB];
#pragma unroll
  for (int t = 0; t < SB; ++t) st[t] = f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
  if (OUT && a.start.p)
    move_state<SB, true>(st, a.start.p + bh * a.start.bh + seg * a.start.seg + part * (kA / P) * a.start.a, a.start, half,
                         col0 + block * 32 + l32);
  if (live) fetch(0);
  for (u32 i = threadIdx.x; i <= kChunk16; i += kThreads) {
    const float x = decay_power(jobs.log_decay, h, i);
    s_pow[i] = x;
    if (OUT && i < kChunk16) s_factor[kNone + i] = a.within * x;
    if (OUT && i < kNone) s_factor[i] = 0.f;
  }
  __syncthreads();
  // where a lane's quad of the transposed tiles is
  const bf16 *v_quad = s_v + (half * 4 + li / 4) * kLdV + block * 32 + (l32 / 16) * 16 + (li & 3) * 4;
  const bf16 *k_quad = s_k + (half * 4 + li / 4) * kLdA + part * (kA / P) + (l32 / 16) * 16 + (li & 3) * 4;
  // 16 rows of this wave's 32 columns of the values' part i
  auto values = [&](u32 jb, int i) {
    const bf16 *s = v_quad + i * kPlaneV + jb * 16 * kLdV;
    return both(read_transposed(s), read_transposed(s + 8 * kLdV));
  };

#pragma unroll 1
  for (u32 c = 0; c < live; c += kChunk16) {
    const u32 n = min(kChunk16, live - c);
    if (c) __syncthreads();
    if (OUT) tq.put(s_q, a.A, n);
    tk.put(s_k, a.A, n);
    tv.put(s_v, cols, n);
    if ((c == 0 || n < kChunk16) && threadIdx.x < kChunk16)
      s_add[threadIdx.x] = threadIdx.x < n ? a.add * s_pow[n - a.lead - threadIdx.x] : 0.f;
    __syncthreads();
    constexpr int kOwn = P == 2 ? 1 : 2;  // blocks of 32 queries that the wave finishes, from `part` on
    f32x16 o[2];
    if (OUT) {
      // 32 x 32 blocks of the scores (queries it, keys jt): (1, 0), (0, 0), (1, 1) in
      // turn.  Of two waves the second forms its last one again, so that no branch
      // keeps one block's loads from the other's products; of four one has none.
#pragma unroll
      for (u32 x = 0; x < (kThreads == 2 * kWave ? 2 : 1); ++x) {
        const u32 t = min(wave + x * 2, 2u);
        if (kThreads > 2 * kWave && wave > 2) break;
        const u32 it = t != 1, jt = t == 2;
        const bf16 *sq = s_q + (it * 32 + l32) * kLdA + half * 8, *sk = s_k + (jt * 32 + l32) * kLdA + half * 8;
        f32x16 p = f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int m = 0; m < 2 * AB; ++m) {
          const b16x8 x0 = *reinterpret_cast<const b16x8 *>(sk + m * 16), y0 = *reinterpret_cast<const b16x8 *>(sq + m * 16);
          p = mfma32(x0, y0, p);
          if constexpr (kIn == 2) {
            const b16x8 x1 = *reinterpret_cast<const b16x8 *>(sk + kPlaneA + m * 16);
            p = mfma32(x1, y0, p);
            const b16x8 y1 = *reinterpret_cast<const b16x8 *>(sq + kPlaneA + m * 16);
            p = mfma32(x0, y1, p);
            p = mfma32(x1, y1, p);
          }
        }
        // query l32, key 8 (r / 4) + 4 half + r % 4: decayed, 0 for keys after the query
        const float *f = s_factor + kNone + 32 * (it - jt) + l32 - half * 4 - 27;
        float z[2][8];
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r / 8][r % 8] = p[r] * f[27 - r / 4 * 8 - r % 4];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const u32 at = ((it * 2 + jt * 2 + y) * kWave + lane) * 8;
          *reinterpret_cast<f32x4 *>(s_p + at) = f32x4{z[y][0], z[y][1], z[y][2], z[y][3]};
          *reinterpret_cast<f32x4 *>(s_p + at + 4) = f32x4{z[y][4], z[y][5], z[y][6], z[y][7]};
        }
      }
      // the entering state's part of the outputs
      o[0] = o[1] = f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int m = 0; m < 2 * SB; ++m) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = st[m / 2][m % 2 * 8 + e];
        b16x8 w[kParts];
        parts_of(x, w);
        const bf16 *s = s_q + l32 * kLdA + part * (kA / P) + m * 16 + half * 4;
        const b16x8 q0 = read_both(s, s + 8), q1 = read_both(s + 32 * kLdA, s + 32 * kLdA + 8);
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
          o[0] = mfma32(w[i], q0, o[0]);
          o[1] = mfma32(w[i], q1, o[1]);
        }
        if constexpr (kIn == 2) {
          const bf16 *r = s + kPlaneA;
          const b16x8 r0 = read_both(r, r + 8), r1 = read_both(r + 32 * kLdA, r + 32 * kLdA + 8);
#pragma unroll
          for (int i = 0; i < kParts - 1; ++i) {
            o[0] = mfma32(w[i], r0, o[0]);
            o[1] = mfma32(w[i], r1, o[1]);
          }
        }
      }
      if constexpr (P == 1) {
#pragma unroll
        for (int it = 0; it < 2; ++it) o[it] *= a.across * s_pow[it * 32 + l32 + a.lead];
      } else {
        const f32x16 x = part ? o[0] : o[1];
        if (part) o[0] = o[1];
#pragma unroll
        for (u32 y = 0; y < 4; ++y)
          s_part[(wave * 4 + y) * kWave + lane] = f32x4{x[y * 4], x[y * 4 + 1], x[y * 4 + 2], x[y * 4 + 3]};
      }
    }
    // (here, and not earlier: the registers are free by now)
    if (c + kChunk16 < live) fetch(c + kChunk16);
    // the state after the chunk
    const float left = s_pow[n];
#pragma unroll
    for (int t = 0; t < SB; ++t) st[t] *= left;
#pragma unroll
    for (u32 jb = 0; jb < 4; ++jb) {
      b16x8 vq[kIn];
#pragma unroll
      for (int i = 0; i < kIn; ++i) vq[i] = values(jb, i);
      const f32x4 w0 = *reinterpret_cast<const f32x4 *>(s_add + jb * 16 + half * 4),
                  w1 = *reinterpret_cast<const f32x4 *>(s_add + jb * 16 + 8 + half * 4);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y = kIn == 2 ? (float)vq[0][e] + (float)vq[kIn - 1][e] : (float)vq[0][e];
        x[e] = y * (e < 4 ? w0[e & 3] : w1[e & 3]);
      }
      b16x8 w[kParts];
      parts_of(x, w);
#pragma unroll
      for (int z = 0; z < kIn; ++z) {
        b16x8 kt[SB];
#pragma unroll
        for (int t = 0; t < SB; ++t) {
          const bf16 *s = k_quad + z * kPlaneA + jb * 16 * kLdA + t * 32;
          kt[t] = both(read_transposed(s), read_transposed(s + 8 * kLdA));
        }
#pragma unroll
        for (int i = 0; i < kParts - z; ++i)  // (a product of a block waits for the one before)
#pragma unroll
          for (int t = 0; t < SB; ++t) st[t] = mfma32(kt[t], w[i], st[t]);
      }
    }
    if (OUT) {
      __syncthreads();  // the scores, and the partner's outputs
      if constexpr (P == 2) {
        const u32 partner = block + (1 - part) * NW;
#pragma unroll
        for (u32 y = 0; y < 4; ++y) {
          const f32x4 x = s_part[(partner * 4 + y) * kWave + lane];
#pragma unroll
          for (u32 e = 0; e < 4; ++e) o[0][y * 4 + e] += x[e];
        }
        o[0] *= a.across * s_pow[part * 32 + l32 + a.lead];
      }
#pragma unroll
      for (u32 jb = 0; jb < 4; ++jb) {
        if (P == 2 && jb >= 2 + 2 * part) break;
        b16x8 vq[kIn];
#pragma unroll
        for (int z = 0; z < kIn; ++z) vq[z] = values(jb, z);
#pragma unroll
        for (u32 x = P == 2 ? 0 : jb / 2; x < kOwn; ++x) {
          const f32x4 *p = reinterpret_cast<const f32x4 *>(s_p + (((part + x) * 2 + jb) * kWave + lane) * 8);
          const f32x4 p0 = p[0], p1 = p[1];
          float y[8] = {p0[0], p0[1], p0[2], p0[3], p1[0], p1[1], p1[2], p1[3]};
          b16x8 w[kParts];
          parts_of(y, w);
#pragma unroll
          for (int z = 0; z < kIn; ++z)
#pragma unroll
            for (int i = 0; i < kParts - z; ++i) o[x] = mfma32(vq[z], w[i], o[x]);
        }
      }
      // lane (l32, half): a query, columns 8 y + 4 half .. + 3 of the block's 32
#pragma unroll
      for (u32 it = 0; it < kOwn; ++it) {
        const u32 i = (part + it) * 32 + l32;
        const u32 p = p0 + c + i, t = reverse ? len - 1 - p : p;
        using T4 = T __attribute__((ext_vector_type(4)));
        T4 w[4];
#pragma unroll
        for (u32 y = 0; y < 4; ++y) {
          const float z[4] = {o[it][y * 4], o[it][y * 4 + 1], o[it][y * 4 + 2], o[it][y * 4 + 3]};
          w[y] = round_all<T>(z);
        }
        // halves exchanged: columns 16 y + 8 half .. + 7
        const u32 col = block * 32 + half * 8;
        T *dst = out + t * out_pos + col;
#pragma unroll
        for (u32 y = 0; y < 2; ++y) {
          const u32x4 x = exchange(__builtin_bit_cast(u32x2, w[2 * y]), __builtin_bit_cast(u32x2, w[2 * y + 1]));
          if (i < n && col + y * 16 + (FAST ? 0 : 7) < cols) {
            *reinterpret_cast<typename WideBits<T>::type *>(dst + y * 16) = x;
          } else if (!FAST && i < n) {
            const auto z = __builtin_bit_cast(Vec<T, 8>, x);
#pragma unroll
            for (u32 e = 0; e < 8; ++e)
              if (col + y * 16 + e < cols) dst[y * 16 + e] = z.v[e];
          }
        }
      }
    }
  }
  if (a.end.p)
    move_state<SB, false>(st, a.end.p + bh * a.end.bh + seg * a.end.seg + part * (kA / P) * a.end.a, a.end, half,
                          col0 + block * 32 + l32);
  if (OUT) {
    // rows beyond the length
    const u32 wide = min(cols, (u32)kTile);
    for (u32 i = live + threadIdx.x / kTile; i < rows; i += kThreads / kTile)
      if (threadIdx.x % kTile < wide) out[(p0 + i) * out_pos + threadIdx.x % kTile] = (T)0.f;
  }
}

template <class T, int AB, int NW, int P, bool OUT>
void launch(const AttendJobs &l, bool fast, hipStream_t s) {
  if (fast) hipLaunchKernelGGL((k_attend16<T, AB, NW, P, OUT, true>), grid_of(l), dim3(P * NW * kWave), 0, s, l);
  else hipLaunchKernelGGL((k_attend16<T, AB, NW, P, OUT, false>), grid_of(l), dim3(P * NW * kWave), 0, s, l);
}

// Two waves for each block of columns shorten a chunk but take the weighted values apart
// twice: they are for workgroups that have a compute unit to themselves, because
// there are few or because no two fit its LDS (float16 with more than 64 rows or
// columns), for two on one (64 x 64, bfloat16), and for 64 columns with 128 or 256 rows,
// whose registers leave a lane no other wave.  In us a chunk of 64, one wave and two:
//   workgroups for each compute unit    1           2           3           4
//   bfloat16  64 x 64                3.3, 2.7    4.8, 3.9    5.1, 5.7    6.0, 7.1
//            128 x 64                5.1, 3.2    5.5, 4.9   10.0, 7.7   10.4, 9.8
//            256 x 64               12.8, 5.6   29.0, 10.9
//             64 x 128               3.3, 3.3    5.5, 6.8    8.3, 9.5   10.4, 13.4
//            128 x 128               4.3, 4.3    7.8, 8.5   11.8, 12.6  15.2, 16.6
//   float16   64 x 64                5.4, 3.9    5.7, 7.6   11.1, 11.4  11.1, 15.2
//            128 x 64                8.1, 5.4
//             64 x 128               5.4, 4.7
//            128 x 128               7.3, 6.7
// (The three gradients of 128 x 128 states, 192 workgroups: 410 us with training's
// other launches, 403 with two waves.)
template <class T, int AB, int NW>
void launch(const AttendJobs &l, bool out, bool fast, hipStream_t s) {
  constexpr bool kHalf = std::is_same<T, f16>::value, kAll = AB >= 4 && NW == 2 || kHalf && (AB == 4 || NW == 4);
  if (!out) return launch<T, AB, NW, 1, false>(l, fast, s);
  if constexpr (AB <= 4 || kAll)
    if (kAll || grid_of(l).x <= (!kHalf && NW == 2 ? 2 : 1) * (u32)compute_units())
      return launch<T, AB, NW, 2, true>(l, fast, s);
  if constexpr (!kAll) launch<T, AB, NW, 1, true>(l, fast, s);
}

bool fast_view(const View &v) { return v.vec == 8 && v.pos >= 0 && v.pos < (1 << 23); }

template <class T>
void attend_all(const AttendJobs &jobs, bool out, hipStream_t s) {
  constexpr bool kWide = std::is_same<T, bf16>::value;  // (float16: dimensions to 128)
  // (sweeps of another kernel, or with other needs, have launches of their own)
  auto kind = [&](const AttendArgs &a) {
    const bool fast = (!out || (fast_view(a.q) && a.W % 8 == 0)) && fast_view(a.k) && fast_view(a.v);
    return padded_dim(a.A) * 4 + (a.W <= 64 ? 0 : 2) + (fast ? 1 : 0);
  };
  auto tiles = [](const AttendArgs &a) { return (u32)ceil_div(a.W, columns16(a.W)); };
  for (u32 i = 0; i < jobs.jobs;) {
    AttendJobs l = jobs;
    const u32 first = kind(jobs.j[i]);
    l.col_tiles = tiles(jobs.j[i]);
    l.jobs = 0;
    for (; i < jobs.jobs && kind(jobs.j[i]) == first && tiles(jobs.j[i]) == l.col_tiles; ++i)
      l.j[l.jobs++] = jobs.j[i];
    const bool fast = first & 1;
    const u32 A = first / 4;
    if (first & 2) {
      if (A == 64) launch<T, 2, 4>(l, out, fast, s);
      else if (A == 128) launch<T, 4, 4>(l, out, fast, s);
      else if constexpr (kWide) launch<T, 8, 4>(l, out, fast, s);
    } else {
      if (A == 64) launch<T, 2, 2>(l, out, fast, s);
      else if (A == 128) launch<T, 4, 2>(l, out, fast, s);
      else if constexpr (kWide) launch<T, 8, 2>(l, out, fast, s);
    }
  }
}

}  // namespace

void attend16(const AttendJobs &jobs, int dtype, bool out, hipStream_t s) {
  if (dtype == FSTC_BF16) attend_all<bf16>(jobs, out, s);
  else attend_all<f16>(jobs, out, s);
}

}  // namespace fstc

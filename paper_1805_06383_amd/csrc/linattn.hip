// Linear attention with a decay for each head (fstc_linattn, fstc_linattn_grad,
// fstc_linattn_step).
//
// For head h with decay g = exp(log_decay[h]) and scale c, over the positions
// t = 0 .. len - 1 of a batch row:
//   S_t = g S_{t-1} + k_t v_t^T        (S_{-1}: the initial state, dim_k x dim_v)
//   o_t = c S_t^T q_t = c (sum_{j<=t} g^(t-j) (q_t.k_j) v_j + g^(t+1) S_{-1}^T q_t)
// and with P_t = dL/dS before position t (P_len: the final state's gradient),
//   P_t = g (c q_t do_t^T + P_{t+1}),
//   dq_t = c S_t do_t,  dk_t = (c q_t do_t^T + P_{t+1}) v_t,
//   dv_t = (c q_t do_t^T + P_{t+1})^T k_t.
// So dq, dk and dv are each a decayed attention with other roles, (do, v, k),
// (v, do, q) and (k, q, do), the last two from the last position to the
// first, and one kernel computes all four.  In reverse the state enters a
// position before the position's own factor g: `lead` is 1 forward and 0 in
// reverse, the state's weight in row i of a chunk is g^(i+lead) and a row's
// weight in the state after n rows g^(n-lead-i).
//
// k_attend takes chunks of kChunk positions.  Inside a chunk the scores'
// chunk x chunk product, masked and decayed, times the values; between chunks
// the state.  A workgroup of four waves owns 64 columns of v (16 a wave) and
// walks a segment of the positions in order with its columns of the state in
// registers.  Every product is laid out so that no result has to change
// lanes: with the score matrix computed as K Q^T its registers (row = key
// position 4 * (lane / 16) + r, column = query position lane % 16) are the
// B operand of V^T P^T with the contraction index permuted the same way in
// both operands, and the state's (row = its k index, column = its v index)
// are the A operand of S^T Q^T.  Each 16 x 16 block of the scores is formed by
// one wave and read by all from LDS, after the state's products; the next
// chunk's rows are on their way meanwhile.
//
// A long text or a small batch has too few (row, head, column tile) workgroups for
// the chip, so the positions are cut into segments: k_attend without output
// sums each segment's own state, k_join_few or k_join_many turns those into the states
// at the segments' starts (and the final state), and k_attend with output
// runs every segment at once.
//
// Sums, scores and states are held in 32 bits.  These kernels take float32, and float16
// of dimensions above 128.  Measured: a chunk of 64 positions with 64 x 64
// states of float32 takes 6.5 us on a compute unit of its own, 4.1 where three share it
// (the matrix instructions 2.3, memory 3.3): what bounds it is a chunk's
// chain of loads, scores, products and barriers.
#include "linattn.hpp"

namespace fstc {
namespace {

constexpr int kNT = 256;
constexpr int kChunk = 32;
constexpr int kCols = 64;       // value columns of a workgroup
constexpr u32 kMaxDim = 256;    // of dim_k and dim_v

// Four elements as one access at any element.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Quad {
  T v[4];
};

// kChunk rows of one head on their way into LDS as 32-bit values: zeros beyond n
// rows and beyond `cols` columns.  fetch() starts the loads and put() ends them, so
// that the next chunk's are in flight while one is worked on.  FAST: rows of
// whole quads, every address clamped into the tile and read (a branch a quad
// would wait for each load in turn).
template <class T, int LD, int COLS, bool FAST>
struct Tile {
  static constexpr u32 kUnits = kChunk * (COLS / 4) / kNT, kRows = kNT / (COLS / 4);
  Quad<T> x[kUnits];

  __device__ __forceinline__ void fetch(const T *src, int64_t pos, u32 cols, u32 n, u32 first, u32 len,
                                        bool reverse) {
    const u32 row0 = threadIdx.x / (COLS / 4), c = threadIdx.x % (COLS / 4) * 4;
#pragma unroll
    for (u32 u = 0; u < kUnits; ++u) {
      const u32 p = first + min(row0 + u * kRows, n - 1), t = reverse ? len - 1 - p : p;
      const T *s = src + (int64_t)t * pos;
      if (FAST) {
        x[u] = *reinterpret_cast<const Quad<T> *>(s + (c < cols ? c : 0));
      } else {
#pragma unroll
        for (u32 e = 0; e < 4; ++e) x[u].v[e] = s[c + e < cols ? c + e : 0];
      }
    }
  }
  __device__ __forceinline__ void put(float *dst, u32 cols, u32 n) const {
    const u32 row0 = threadIdx.x / (COLS / 4), c = threadIdx.x % (COLS / 4) * 4;
#pragma unroll
    for (u32 u = 0; u < kUnits; ++u) {
      const u32 row = row0 + u * kRows;
      f32x4 y;
#pragma unroll
      for (u32 e = 0; e < 4; ++e) y[e] = row < n && c + e < cols ? to_f32(x[u].v[e]) : 0.f;
      *reinterpret_cast<f32x4 *>(dst + row * LD + c) = y;
    }
  }
};

__device__ __forceinline__ f32x4 mfma(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// AB: blocks of 16 that hold the contraction's A elements.
template <class T, int AB, bool OUT, bool FAST>
__global__ __launch_bounds__(kNT) void k_attend(AttendJobs jobs) {
  constexpr int kA = AB * 16, kLdA = kA + 4, kLdV = kCols + 4;
  __shared__ __align__(16) float s_q[OUT ? kChunk * kLdA : 4], s_k[kChunk * kLdA], s_v[kChunk * kLdV];
  // 16 x 16 blocks of the scores (key block, query block): (0, 0), (0, 1), (1, 1)
  __shared__ f32x4 s_p[OUT ? 3 * kWave : 1];
  __shared__ float s_pow[kChunk + 1];
  const Part part = part_of(jobs);
  if (!part.any) return;
  const AttendArgs &a = jobs.j[part.job];
  const u32 seg = part.seg, tile = part.tile, bh = part.bh, b = bh / jobs.heads, h = bh % jobs.heads;
  const u32 len = row_length(jobs.lengths, b, jobs.length);
  const u32 p0 = seg * jobs.segment;
  const u32 rows = min(jobs.segment, jobs.length - min(p0, jobs.length));
  const u32 live = len > p0 ? min(jobs.segment, len - p0) : 0;
  const bool reverse = a.lead == 0;
  const u32 lane = lane_id(), li = lane & 15, g = lane / 16;
  const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const u32 col0 = tile * kCols;  // of the workgroup
  const u32 wcol = col0 + wave * 16 + li;  // this lane's column of the state

  const T *q = static_cast<const T *>(a.q.p) + b * a.q.batch + h * a.q.head;
  const T *k = static_cast<const T *>(a.k.p) + b * a.k.batch + h * a.k.head;
  const T *v = static_cast<const T *>(a.v.p) + b * a.v.batch + h * a.v.head + col0;
  T *out = OUT ? static_cast<T *>(a.out) + ((u64)b * jobs.length * jobs.heads + h) * a.W + col0 : nullptr;
  const u64 out_pos = (u64)jobs.heads * a.W;
  const u32 cols = a.W - col0;  // this tile's columns and those to its right
  Tile<T, kLdA, kA, FAST> tq, tk;
  Tile<T, kLdV, kCols, FAST> tv;
  auto fetch = [&](u32 c) {
    const u32 n = min((u32)kChunk, live - c);
    if (OUT) tq.fetch(q, a.q.pos, a.A, n, p0 + c, len, reverse);
    tk.fetch(k, a.k.pos, a.A, n, p0 + c, len, reverse);
    tv.fetch(v, a.v.pos, cols, n, p0 + c, len, reverse);
  };
  if (live) fetch(0);
  if (threadIdx.x <= kChunk) s_pow[threadIdx.x] = decay_power(jobs.log_decay, h, threadIdx.x);

  f32x4 st[AB];
#pragma unroll
  for (int ab = 0; ab < AB; ++ab)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const u32 ka = ab * 16 + g * 4 + r;
      st[ab][r] = 0.f;
      if (OUT && a.start.p && ka < a.A && wcol < a.W)
        st[ab][r] = a.start.p[bh * a.start.bh + seg * a.start.seg + ka * a.start.a + wcol * a.start.w];
    }
  __syncthreads();

#pragma unroll 1
  for (u32 c = 0; c < live; c += kChunk) {
    const u32 n = min((u32)kChunk, live - c);
    if (c) __syncthreads();
    if (OUT) tq.put(s_q, a.A, n);
    tk.put(s_k, a.A, n);
    tv.put(s_v, cols, n);
    if (c + kChunk < live) fetch(c + kChunk);
    __syncthreads();
    float vv[2][4];
#pragma unroll
    for (int jb = 0; jb < 2; ++jb)
#pragma unroll
      for (int r = 0; r < 4; ++r) vv[jb][r] = s_v[(jb * 16 + g * 4 + r) * kLdV + wave * 16 + li];
    f32x4 o0 = {0, 0, 0, 0}, o1 = o0;
    if (OUT) {
      if (wave < 3) {
        const u32 jb = wave / 2, ib = (wave + 1) / 2;
        f32x4 p = {0, 0, 0, 0};
#pragma unroll
        for (int ab = 0; ab < AB; ++ab) {
          const f32x4 x = *reinterpret_cast<const f32x4 *>(s_k + (jb * 16 + li) * kLdA + ab * 16 + g * 4);
          const f32x4 y = *reinterpret_cast<const f32x4 *>(s_q + (ib * 16 + li) * kLdA + ab * 16 + g * 4);
#pragma unroll
          for (int r = 0; r < 4; ++r) p = mfma(x[r], y[r], p);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          // (selected, not multiplied by 0: a score may be infinite)
          const int gap = (int)(ib * 16 + li) - (int)(jb * 16 + g * 4 + r);
          p[r] = gap >= 0 ? p[r] * (a.within * s_pow[gap < 0 ? 0 : gap]) : 0.f;
        }
        s_p[wave * kWave + lane] = p;
      }
      // the entering state's part of the outputs
#pragma unroll
      for (int ab = 0; ab < AB; ++ab) {
        const u32 at = ab * 16 + g * 4;
        const f32x4 q0 = *reinterpret_cast<const f32x4 *>(s_q + li * kLdA + at);
        const f32x4 q1 = *reinterpret_cast<const f32x4 *>(s_q + (16 + li) * kLdA + at);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          o0 = mfma(st[ab][r], q0[r], o0);
          o1 = mfma(st[ab][r], q1[r], o1);
        }
      }
      o0 *= a.across * s_pow[li + a.lead];
      o1 *= a.across * s_pow[16 + li + a.lead];
    }
    // the state after the chunk
    const float left = s_pow[n];
#pragma unroll
    for (int ab = 0; ab < AB; ++ab) st[ab] *= left;
#pragma unroll
    for (int jb = 0; jb < 2; ++jb)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 j = jb * 16 + g * 4 + r;
        const float x = j < n ? vv[jb][r] * (a.add * s_pow[n - a.lead - j]) : 0.f;
#pragma unroll
        for (int ab = 0; ab < AB; ++ab) st[ab] = mfma(s_k[j * kLdA + ab * 16 + li], x, st[ab]);
      }
    if (OUT) {
      __syncthreads();  // the scores
      const f32x4 p00 = s_p[lane], p01 = s_p[kWave + lane], p11 = s_p[2 * kWave + lane];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        o0 = mfma(vv[0][r], p00[r], o0);
        o1 = mfma(vv[0][r], p01[r], o1);
        o1 = mfma(vv[1][r], p11[r], o1);
      }
      // lane (li, g): position li of the block, columns 4 g .. 4 g + 3 of the wave's 16
#pragma unroll
      for (int ib = 0; ib < 2; ++ib) {
        const u32 i = ib * 16 + li, wc = wave * 16 + g * 4;
        if (i >= n) continue;
        const u32 p = p0 + c + i, t = reverse ? len - 1 - p : p;
        T *dst = out + t * out_pos + wc;
        const f32x4 o = ib ? o1 : o0;
        if (a.W % 4 == 0) {
          if (wc < cols) {
            Quad<T> y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y.v[e] = from_f32<T>(o[e]);
            *reinterpret_cast<Quad<T> *>(dst) = y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (wc + e < cols) dst[e] = from_f32<T>(o[e]);
        }
      }
    }
  }
  if (a.end.p) {
#pragma unroll
    for (int ab = 0; ab < AB; ++ab)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const u32 ka = ab * 16 + g * 4 + r;
        if (ka < a.A && wcol < a.W)
          a.end.p[bh * a.end.bh + seg * a.end.seg + ka * a.end.a + wcol * a.end.w] = st[ab][r];
      }
  }
  // rows beyond the length
  if (OUT) {
    const u32 wide = min(cols, (u32)kCols);
    for (u32 i = live + threadIdx.x / 64; i < rows; i += kNT / 64)
      if ((threadIdx.x & 63) < wide) out[(p0 + i) * out_pos + (threadIdx.x & 63)] = from_f32<T>(0.f);
  }
}

// Segments' own states -> the states at their starts, in place; the state
// after the last one to `final` (may be NULL).  In the workspace a state has
// rows x cols elements, outside A x W.
struct JoinArgs {
  float *state;
  const float *init;
  float *final;
};
struct JoinJobs {
  JoinArgs j[2];
  u32 segments, segment, rows, cols, A, W;
  u32 heads, length, blocks_per;  // workgroups' parts of a batch row's head, and of all
  u32 blocks;
  const float *log_decay;
  const int32_t *lengths;
};
// The decays of a whole segment and of the one that the length ends in, taken by one
// wave of the workgroup.
__device__ __forceinline__ float2 segment_decays(const JoinJobs &a, u32 h, u32 len) {
  __shared__ float s_decay[2];
  if (threadIdx.x < 2) s_decay[threadIdx.x] = decay_power(a.log_decay, h, threadIdx.x ? len % a.segment : a.segment);
  __syncthreads();
  return make_float2(s_decay[0], s_decay[1]);
}

// A thread an element: kFew segments' are on their way before the first is added.
// (One segment of padded states may have 2^20 states of 256 workgroups' parts: more threads than a
// launch holds, so the parts are walked by the grid.)
constexpr u32 kFew = 8;
__global__ __launch_bounds__(kNT) void k_join_few(JoinJobs a) {
  const JoinArgs &job = a.j[blockIdx.y];
  for (u32 block = blockIdx.x; block < a.blocks; block += gridDim.x) {
    const u32 bh = block / a.blocks_per, cells = a.rows * a.cols;
    const u32 i = block % a.blocks_per * kNT + threadIdx.x;
    const u32 len = row_length(a.lengths, bh / a.heads, a.length);
    const float2 decay = segment_decays(a, bh % a.heads, len);
    const float whole = decay.x, last = decay.y;
    __syncthreads();  // (the next part's decays go where these were)
    if (i >= cells) continue;
    const u32 ka = i / a.cols, w = i % a.cols;
    const bool in = ka < a.A && w < a.W;
    const u64 outside = (u64)bh * a.A * a.W + ka * a.W + w;
    float s = in && job.init ? job.init[outside] : 0.f;
    float *p = job.state + (u64)bh * a.segments * cells + i;
    for (u32 k0 = 0; k0 < a.segments; k0 += kFew) {
      float own[kFew];
#pragma unroll
      for (u32 j = 0; j < kFew; ++j) own[j] = p[(u64)min(k0 + j, a.segments - 1) * cells];
#pragma unroll
      for (u32 j = 0; j < kFew; ++j) {
        const u32 k = k0 + j;
        if (k >= a.segments) break;
        p[(u64)k * cells] = s;
        const u32 ends = len / a.segment;
        s = fmaf(k < ends ? whole : k == ends ? last : 1.f, s, own[j]);
      }
    }
    if (in && job.final) job.final[outside] = s;
  }
}

// Of many segments: a workgroup owns 64 elements, and its waves take kAhead segments
// each at once, all loads on their way before the first is added.  A wave first
// joins its own, which maps what enters, s, to factor * s + sum; those maps,
// through LDS, give each wave what enters it.  125 segments of 8 states of 64 x 64:
// 11 us, a thread an element 16; 4 segments of 64 of 128 x 128: 29 and 12.5.
constexpr u32 kMany = 2 * kFew;
__global__ __launch_bounds__(kNT) void k_join_many(JoinJobs a) {
  constexpr u32 kAhead = 32;
  constexpr u32 kWaves = kNT / kWave;
  __shared__ float s_factor[2][kWaves], s_sum[2][kWaves][kWave];
  const JoinArgs &job = a.j[blockIdx.y];
  const u32 bh = blockIdx.x / a.blocks_per, cells = a.rows * a.cols;
  const u32 lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const u32 i = blockIdx.x % a.blocks_per * kWave + lane;
  const bool mine = i < cells;
  const u32 len = row_length(a.lengths, bh / a.heads, a.length);
  const float2 decay = segment_decays(a, bh % a.heads, len);
  const float whole = decay.x, last = decay.y;
  const u32 ends = len / a.segment;
  const u32 ka = i / a.cols, w = i % a.cols;
  const bool in = mine && ka < a.A && w < a.W;
  const u64 outside = (u64)bh * a.A * a.W + ka * a.W + w;
  float carry = in && job.init ? job.init[outside] : 0.f;
  float *p = job.state + (u64)bh * a.segments * cells + (mine ? i : 0);
  for (u32 k0 = 0, x = 0; k0 < a.segments; k0 += kAhead * kWaves, x ^= 1) {
    const u32 k1 = k0 + wave * kAhead;
    float own[kAhead], factor = 1.f, sum = 0.f;
#pragma unroll
    for (u32 j = 0; j < kAhead; ++j) own[j] = p[(u64)min(k1 + j, a.segments - 1) * cells];
#pragma unroll
    for (u32 j = 0; j < kAhead; ++j) {
      const u32 k = k1 + j;
      const float f = k < ends ? whole : k == ends ? last : 1.f;
      sum = fmaf(f, sum, k < a.segments ? own[j] : 0.f);
      factor *= f;
    }
    s_sum[x][wave][lane] = sum;
    if (lane == 0) s_factor[x][wave] = factor;
    __syncthreads();
    float s = carry;
#pragma unroll
    for (u32 v = 0; v < kWaves; ++v) {
      if (v == wave) s = carry;
      carry = fmaf(s_factor[x][v], carry, s_sum[x][v][lane]);
    }
#pragma unroll
    for (u32 j = 0; j < kAhead; ++j) {
      const u32 k = k1 + j;
      if (k >= a.segments) break;
      if (mine) p[(u64)k * cells] = s;
      s = fmaf(k < ends ? whole : k == ends ? last : 1.f, s, own[j]);
    }
  }
  if (wave == 0 && in && job.final) job.final[outside] = carry;
}

// One position of each row: a workgroup owns `cols` columns of one state,
// reads them, updates them, writes them, and sums q_a S[a, :] over the rows.
// Bound: HBM, 8 bytes a state element (1,024 rows of 16 states of 128 x 128: 390 us,
// 5.5 TB/s); for a few rows the launch (8 rows of 8 states of 64 x 64: 4 us).
struct StepArgs {
  const void *q, *k, *v;
  int64_t q_batch, q_head, k_batch, k_head, v_batch, v_head;
  const float *log_decay;
  const float *in;
  const int32_t *parents;  // may be NULL
  u32 in_rows;
  float *state;
  void *out;  // [batch, heads, W]
  u32 heads, A, W, cols, tiles;
  float scale;
};

template <class T, int N>
__global__ __launch_bounds__(kNT) void k_step(StepArgs a) {
  constexpr int kAhead = 8;
  __shared__ float s_q[kMaxDim], s_k[kMaxDim];
  __shared__ float s_o[kNT / kWave][kMaxDim];
  const u32 tile = blockIdx.x % a.tiles, bh = blockIdx.x / a.tiles, b = bh / a.heads, h = bh % a.heads;
  const T *q = static_cast<const T *>(a.q) + b * a.q_batch + h * a.q_head;
  const T *k = static_cast<const T *>(a.k) + b * a.k_batch + h * a.k_head;
  const T *v = static_cast<const T *>(a.v) + b * a.v_batch + h * a.v_head;
  const int64_t from = a.parents ? (int64_t)a.parents[b] : (int64_t)b;
  const bool known = (u64)from < a.in_rows;  // else a new hypothesis: a zero state
  const u64 cells = (u64)a.A * a.W;
  const u32 across = a.cols / N;  // threads over the columns (a power of two, at most 64)
  const u32 x = threadIdx.x & (across - 1), y = threadIdx.x / across, ys = kNT / across;
  const u32 w = tile * a.cols + x * N;
  const float *src = a.in + ((u64)(known ? from : 0) * a.heads + h) * cells + w;
  float *dst = a.state + (u64)bh * cells + w;
  const bool in = w < a.W;  // (N divides W)
  if (threadIdx.x < a.A) {
    s_q[threadIdx.x] = to_f32(q[threadIdx.x]);
    s_k[threadIdx.x] = to_f32(k[threadIdx.x]);
  }
  const float decay = expf(a.log_decay[h]);
  Vec<float, N> vv;
#pragma unroll
  for (int e = 0; e < N; ++e) vv.v[e] = in ? to_f32(v[w + e]) : 0.f;
  float o[N];
#pragma unroll
  for (int e = 0; e < N; ++e) o[e] = 0.f;
  __syncthreads();
  if (in)
    for (u32 r = y; r < a.A; r += ys * kAhead) {
      Vec<float, N> s[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const u32 row = r + j * ys;
        if (known && row < a.A) s[j] = *reinterpret_cast<const Vec<float, N> *>(src + (u64)row * a.W);
        else
#pragma unroll
          for (int e = 0; e < N; ++e) s[j].v[e] = 0.f;
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const u32 row = r + j * ys;
        if (row >= a.A) break;
        const float kk = s_k[row], qq = s_q[row];
#pragma unroll
        for (int e = 0; e < N; ++e) {
          s[j].v[e] = fmaf(decay, s[j].v[e], kk * vv.v[e]);
          o[e] = fmaf(qq, s[j].v[e], o[e]);
        }
        *reinterpret_cast<Vec<float, N> *>(dst + (u64)row * a.W) = s[j];
      }
    }
  // over the rows: lanes of a wave that share the columns, then the waves
  for (u32 d = across; d < (u32)kWave; d <<= 1)
#pragma unroll
    for (int e = 0; e < N; ++e) o[e] += __shfl_xor(o[e], d);
  const u32 wave = threadIdx.x / kWave;
  if (lane_id() < across)
#pragma unroll
    for (int e = 0; e < N; ++e) s_o[wave][x * N + e] = o[e];
  __syncthreads();
  const u32 c = threadIdx.x;
  if (c < a.cols && tile * a.cols + c < a.W) {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kNT / kWave; ++i) t += s_o[i][c];
    static_cast<T *>(a.out)[(u64)bh * a.W + tile * a.cols + c] = from_f32<T>(a.scale * t);
  }
}

// ---------------------------------------------------------------------------
// Segments of the positions, and the shape of a state in the workspace.
//
// More segments fill the chip sooner; each of them costs its states (written,
// joined, read), and any at all a pass over the keys and values before the
// sweep proper.  The plan is the cheapest by a model of the time in
// chunk times of a compute unit: k workgroups on a compute unit take
// kAlone + kEach k a chunk while at most kResident of them are there at once.
// The figures are measured, in us a chunk of 64 (16 bits: linattn16.hip, at the
// launches; 32-bit instructions, 64 columns of 64 x 64 states 6.5, 9.2, 12.3 for 1
// to 3, of 128 x 128 ones 9.4 and 14.5, of 256 x 256 ones 17.5).
struct Plan {
  u32 segments, segment, rows, cols;
  bool direct;  // one segment whose states are read and written where the caller has them
  u64 state_bytes = 0;  // of one array of segment states; 0 when direct

  Plan(const fstc_linattn_args &a, u32 sweeps) {
    const u32 wide = std::max(a.dim_k, a.dim_v);
    const bool half = takes16(a.dtype, wide);
    rows = half ? padded_dim(a.dim_k) : a.dim_k;
    cols = half ? padded_dim(a.dim_v) : a.dim_v;
    const u32 large = (a.dim_k > 64) + (a.dim_v > 64);
    double alone = 4.0, each = 2.7 * wide / 64;
    u32 resident = wide > 128 ? 1 : wide > 64 ? 2 : 3;
    if (half && a.dtype == FSTC_F16) {
      alone = large ? 0.0 : 2.2;
      each = large == 2 ? 6.7 : large ? 5.1 : 1.75;
      resident = large ? 1 : 2;
    } else if (half) {
      alone = large == 2 ? 0.8 : 1.3;
      each = large == 2 ? 3.5 : large ? 1.95 : 1.2;
      resident = large ? 2 : 4;
    }
    auto chunk_time = [&](u64 groups) {
      const u64 k = ceil_div(groups, kComputeUnits), left = k % resident;
      return double(k / resident) * (alone + each * resident) + (left ? alone + each * double(left) : 0.0);
    };
    const bool exact_shape = rows == a.dim_k && cols == a.dim_v;
    const u64 bh = std::max<u64>(1, (u64)a.batch * a.heads), tiles = ceil_div(wide, half ? columns16(wide) : kCols);
    const u64 chunks = std::max<u64>(1, ceil_div(a.length, kChunk16));
    const double state_time = 12.0 * rows * cols / 65536.0 * double(bh) / kComputeUnits;  // of one segment's
    // (chunks a segment: every number up to 16, then in steps of an eighth)
    double best = 0;
    u64 per = chunks;
    for (u64 p = chunks;;) {
      const u64 n = ceil_div(chunks, p);
      if (n > 1 && bh * tiles * n > kMostGroups) break;
      double t = chunk_time(bh * tiles * n * sweeps) * double(p + 1);  // (1: before the first)
      if (n > 1 || !exact_shape) {
        const u64 states = sweeps > 1 ? 2 : 1;
        t += kStatePass * chunk_time(bh * tiles * n * states) * double(p + 1) +
             state_time * double(n * states) + kLaunches;
      }
      if (n == 1 || t < best) {
        best = t;
        per = p;
      }
      if (p == 1) break;
      p -= p > 16 ? p / 8 : 1;
    }
    segment = (u32)(per * kChunk16);
    segments = (u32)ceil_div(chunks, per);
    direct = segments == 1 && exact_shape;
    if (!direct) state_bytes = ((u64)a.batch * a.heads * segments * rows * cols * sizeof(float) + 255) & ~255ull;
  }

  static constexpr u64 kComputeUnits = 256;  // (not asked for: a workspace's size needs no device)
  static constexpr u64 kMostGroups = 8 * kComputeUnits;
  static constexpr double kStatePass = 0.45;  // of the sweep proper's time
  static constexpr double kLaunches = 14;     // of two more launches, us
};
constexpr u32 kForwardSweeps = 1, kBackwardSweeps = 3;

size_t workspace_bytes_for(const fstc_linattn_args &a, bool grad) {
  return grad ? 2 * Plan(a, kBackwardSweeps).state_bytes : Plan(a, kForwardSweeps).state_bytes;
}

View view_of(const void *p, const int64_t *stride, u32 cols) {
  return {p, stride[0], stride[1], stride[2], cols % 8 == 0 ? 8 : cols % 4 == 0 ? 4 : 1};
}

template <class T, bool OUT>
void attend(AttendJobs jobs, hipStream_t s) {
  constexpr int dtype = std::is_same<T, bf16>::value ? FSTC_BF16 : std::is_same<T, f16>::value ? FSTC_F16 : FSTC_F32;
  u32 widest = 0;
  for (u32 i = 0; i < jobs.jobs; ++i) widest = std::max({widest, jobs.j[i].A, jobs.j[i].W});
  if (takes16(dtype, widest)) return attend16(jobs, dtype, OUT, s);
  if constexpr (dtype != FSTC_BF16) {
    // (sweeps of another kernel have launches of their own; rows in whole quads, or
    // element by element)
    auto blocks = [](const AttendArgs &a) { return a.A <= 32 ? 32u : padded_dim(a.A); };
    auto whole = [](const AttendArgs &a) { return (!OUT || a.q.vec >= 4) && a.k.vec >= 4 && a.v.vec >= 4; };
    for (u32 i = 0; i < jobs.jobs;) {
      AttendJobs l = jobs;
      l.jobs = 0;
      l.col_tiles = (u32)ceil_div(jobs.j[i].W, kCols);
      const u32 A = blocks(jobs.j[i]);
      const bool fast = whole(jobs.j[i]);
      for (; i < jobs.jobs && blocks(jobs.j[i]) == A && whole(jobs.j[i]) == fast &&
             ceil_div(jobs.j[i].W, kCols) == l.col_tiles;
           ++i)
        l.j[l.jobs++] = jobs.j[i];
      const dim3 grid = grid_of(l);
      if (!fast && A <= 64) hipLaunchKernelGGL((k_attend<T, 4, OUT, false>), grid, dim3(kNT), 0, s, l);
      else if (!fast && A <= 128) hipLaunchKernelGGL((k_attend<T, 8, OUT, false>), grid, dim3(kNT), 0, s, l);
      else if (!fast) hipLaunchKernelGGL((k_attend<T, 16, OUT, false>), grid, dim3(kNT), 0, s, l);
      else if (A <= 32) hipLaunchKernelGGL((k_attend<T, 2, OUT, true>), grid, dim3(kNT), 0, s, l);
      else if (A <= 64) hipLaunchKernelGGL((k_attend<T, 4, OUT, true>), grid, dim3(kNT), 0, s, l);
      else if (A <= 128) hipLaunchKernelGGL((k_attend<T, 8, OUT, true>), grid, dim3(kNT), 0, s, l);
      else hipLaunchKernelGGL((k_attend<T, 16, OUT, true>), grid, dim3(kNT), 0, s, l);
    }
  }
}

int check_linattn(const fstc_linattn_args *a) {
  if (!a) return report_failure(FSTC_ERR_INVALID_ARG, "args is NULL");
  if (!element_bytes(a->dtype)) return report_failure(FSTC_ERR_INVALID_ARG, "unknown element type");
  if (a->heads == 0 || a->dim_k == 0 || a->dim_v == 0)
    return report_failure(FSTC_ERR_INVALID_ARG, "heads, dim_k and dim_v must be positive");
  if (a->dim_k > kMaxDim || a->dim_v > kMaxDim)
    return report_failure(FSTC_ERR_RANGE, "dim_k and dim_v must be at most 256");
  if (!a->log_decay) return report_failure(FSTC_ERR_INVALID_ARG, "log_decay is NULL");
  if (a->batch && a->length && (!a->q || !a->k || !a->v))
    return report_failure(FSTC_ERR_INVALID_ARG, "q, k or v is NULL");
  const size_t e = element_bytes(a->dtype);
  if (!aligned_to(a->q, e) || !aligned_to(a->k, e) || !aligned_to(a->v, e))
    return report_failure(FSTC_ERR_INVALID_ARG, "q, k or v is not aligned to its elements");
  const u64 bh = (u64)a->batch * a->heads;
  if (a->length >= (1u << 31) || bh >= (1u << 20))
    return report_failure(FSTC_ERR_RANGE, "length must be below 2^31 and batch * heads below 2^20");
  return FSTC_OK;
}

AttendJobs jobs_of(const fstc_linattn_args &a, const Plan &pl) {
  AttendJobs r{};
  r.log_decay = a.log_decay;
  r.lengths = a.lengths;
  r.length = a.length;
  r.heads = a.heads;
  r.batch_heads = a.batch * a.heads;
  r.segments = pl.segments;
  r.segment = pl.segment;
  return r;
}

void join_segments(const fstc_linattn_args &a, const Plan &pl, const JoinArgs *j, u32 n, hipStream_t s) {
  JoinJobs r{};
  for (u32 i = 0; i < n; ++i) r.j[i] = j[i];
  r.segments = pl.segments;
  r.segment = pl.segment;
  r.rows = pl.rows;
  r.cols = pl.cols;
  r.A = a.dim_k;
  r.W = a.dim_v;
  r.heads = a.heads;
  r.length = a.length;
  r.log_decay = a.log_decay;
  r.lengths = a.lengths;
  const bool many = pl.segments > kMany;
  r.blocks_per = (u32)ceil_div(pl.rows * pl.cols, many ? kWave : kNT);
  r.blocks = a.batch * a.heads * r.blocks_per;  // below 2^28
  // (k_join_many does not walk: where there are many segments, there are fewer states than kMostGroups)
  const dim3 grid(std::min<u32>(r.blocks, (u32)kMaxGrid), n);
  if (many) hipLaunchKernelGGL(k_join_many, grid, dim3(kNT), 0, s, r);
  else hipLaunchKernelGGL(k_join_few, grid, dim3(kNT), 0, s, r);
}

// States [bh][segment][rows][cols], or their transposes.
States states_of(float *p, const Plan &pl, bool transposed) {
  const int64_t cells = (int64_t)pl.rows * pl.cols;
  return {p, cells * pl.segments, cells, transposed ? 1 : (int64_t)pl.cols, transposed ? (int64_t)pl.cols : 1};
}

template <class T>
void forward(const fstc_linattn_args &a, void *out, float *final, char *ws, hipStream_t s) {
  const Plan pl(a, kForwardSweeps);
  AttendJobs jobs = jobs_of(a, pl);
  jobs.jobs = 1;
  AttendArgs &f = jobs.j[0];
  f.q = view_of(a.q, a.q_stride, a.dim_k);
  f.k = view_of(a.k, a.k_stride, a.dim_k);
  f.v = view_of(a.v, a.v_stride, a.dim_v);
  f.A = a.dim_k;
  f.W = a.dim_v;
  f.lead = 1;
  f.within = f.across = a.scale;
  f.add = 1.f;
  f.out = out;
  if (pl.direct) {
    f.start = states_of(const_cast<float *>(a.init), pl, false);
    f.end = states_of(final, pl, false);
  } else {
    float *seg = reinterpret_cast<float *>(ws);
    f.end = states_of(seg, pl, false);
    attend<T, false>(jobs, s);
    const JoinArgs j{seg, a.init, final};
    join_segments(a, pl, &j, 1, s);
    f.start = f.end;
    f.end.p = nullptr;
  }
  attend<T, true>(jobs, s);
}

template <class T>
void backward(const fstc_linattn_args &a, const void *dout, const int64_t *dout_stride, const float *dfinal,
              void *dq, void *dk, void *dv, float *dinit, char *ws, hipStream_t s) {
  const Plan pl(a, kBackwardSweeps);
  const View q = view_of(a.q, a.q_stride, a.dim_k), k = view_of(a.k, a.k_stride, a.dim_k),
             v = view_of(a.v, a.v_stride, a.dim_v), o = view_of(dout, dout_stride, a.dim_v);
  float *fs = const_cast<float *>(a.init), *bs = const_cast<float *>(dfinal);
  if (!pl.direct) {
    fs = reinterpret_cast<float *>(ws);
    bs = reinterpret_cast<float *>(ws + pl.state_bytes);
    AttendJobs jobs = jobs_of(a, pl);
    jobs.jobs = 2;
    AttendArgs &f = jobs.j[0], &b = jobs.j[1];
    f.k = k;  // S: keys k, values v
    f.v = v;
    f.A = a.dim_k;
    f.W = a.dim_v;
    f.lead = 1;
    f.add = 1.f;
    f.end = states_of(fs, pl, false);
    b = f;  // P: keys c q, values do, from the end
    b.k = q;
    b.v = o;
    b.lead = 0;
    b.add = a.scale;
    b.end = states_of(bs, pl, false);
    attend<T, false>(jobs, s);
    const JoinArgs j[2] = {{fs, a.init, nullptr}, {bs, dfinal, dinit}};
    join_segments(a, pl, j, 2, s);
  }
  AttendJobs jobs = jobs_of(a, pl);
  jobs.jobs = 3;
  AttendArgs &f = jobs.j[0], &g = jobs.j[1], &h = jobs.j[2];
  f.q = o;  // dq
  f.k = v;
  f.v = k;
  f.A = a.dim_v;
  f.W = a.dim_k;
  f.lead = 1;
  f.within = f.across = a.scale;
  f.add = 1.f;
  f.start = states_of(fs, pl, true);
  f.out = dq;
  g.q = v;  // dk
  g.k = o;
  g.v = q;
  g.A = a.dim_v;
  g.W = a.dim_k;
  g.lead = 0;
  g.within = g.add = a.scale;
  g.across = 1.f;
  g.start = states_of(bs, pl, true);
  g.out = dk;
  h = g;  // dv
  h.q = k;
  h.k = q;
  h.v = o;
  h.A = a.dim_k;
  h.W = a.dim_v;
  h.start = states_of(bs, pl, false);
  h.out = dv;
  if (pl.direct) h.end = states_of(dinit, pl, false);
  attend<T, true>(jobs, s);
}

bool overlap(const void *a, u64 na, const void *b, u64 nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

}  // namespace
}  // namespace fstc

using namespace fstc;

extern "C" {

size_t fstc_linattn_workspace(const fstc_linattn_args *args, int grad) {
  return args && check_linattn(args) == FSTC_OK ? workspace_bytes_for(*args, grad != 0) : 0;
}

int fstc_linattn(const fstc_linattn_args *args, void *out, float *final_state, void *workspace,
                 size_t workspace_bytes, hipStream_t stream) {
  const int rc = check_linattn(args);
  if (rc) return rc;
  if (args->batch == 0) return FSTC_OK;
  if (args->length && !out) return report_failure(FSTC_ERR_INVALID_ARG, "out is NULL");
  const size_t need = workspace_bytes_for(*args, false);
  if (workspace_bytes < need || (need && !workspace))
    return report_failure(FSTC_ERR_INVALID_ARG, "the workspace is smaller than fstc_linattn_workspace says");
  return run_reported("fstc_linattn", stream, [&] {
    with_dtype(args->dtype, [&](auto t) {
      forward<decltype(t)>(*args, out, final_state, static_cast<char *>(workspace), stream);
    });
    FSTC_HIP(hipGetLastError());
  });
}

int fstc_linattn_grad(const fstc_linattn_args *args, const void *dout, const int64_t dout_stride[3],
                      const float *dfinal_state, void *dq, void *dk, void *dv, float *dinit,
                      void *workspace, size_t workspace_bytes, hipStream_t stream) {
  const int rc = check_linattn(args);
  if (rc) return rc;
  if (args->batch == 0) return FSTC_OK;
  if (!dout_stride || (args->length && (!dout || !dq || !dk || !dv)))
    return report_failure(FSTC_ERR_INVALID_ARG, "dout, dq, dk or dv is NULL");
  if (!aligned_to(dout, element_bytes(args->dtype)))
    return report_failure(FSTC_ERR_INVALID_ARG, "dout is not aligned to its elements");
  const size_t need = workspace_bytes_for(*args, true);
  if (workspace_bytes < need || (need && !workspace))
    return report_failure(FSTC_ERR_INVALID_ARG, "the workspace is smaller than fstc_linattn_workspace says");
  return run_reported("fstc_linattn_grad", stream, [&] {
    with_dtype(args->dtype, [&](auto t) {
      backward<decltype(t)>(*args, dout, dout_stride, dfinal_state, dq, dk, dv, dinit,
                            static_cast<char *>(workspace), stream);
    });
    FSTC_HIP(hipGetLastError());
  });
}

int fstc_linattn_step(const fstc_linattn_args *args, const int32_t *parents, uint32_t state_rows,
                      float *state, void *out, hipStream_t stream) {
  const int rc = check_linattn(args);
  if (rc) return rc;
  if (args->length != 1) return report_failure(FSTC_ERR_INVALID_ARG, "a step has length 1");
  if (args->lengths) return report_failure(FSTC_ERR_INVALID_ARG, "a step takes no lengths");
  if (args->batch == 0) return FSTC_OK;
  if ((state_rows && !args->init) || !state || !out)
    return report_failure(FSTC_ERR_INVALID_ARG, "init, state or out is NULL");
  if (state_rows >= (1u << 31)) return report_failure(FSTC_ERR_RANGE, "state_rows must be below 2^31");
  const u64 row = (u64)args->heads * args->dim_k * args->dim_v * sizeof(float);
  if (!parents && state_rows != args->batch)
    return report_failure(FSTC_ERR_INVALID_ARG, "without parents there is one entering state a row");
  if (overlap(args->init, state_rows * row, state, args->batch * row) && (parents || args->init != state))
    return report_failure(FSTC_ERR_INVALID_ARG,
                          "state overlaps init (only a step without parents may update in place)");
  return run_reported("fstc_linattn_step", stream, [&] {
    StepArgs a{};
    a.q = args->q;
    a.k = args->k;
    a.v = args->v;
    a.q_batch = args->q_stride[0];
    a.q_head = args->q_stride[2];
    a.k_batch = args->k_stride[0];
    a.k_head = args->k_stride[2];
    a.v_batch = args->v_stride[0];
    a.v_head = args->v_stride[2];
    a.log_decay = args->log_decay;
    a.in = args->init;
    a.parents = parents;
    a.in_rows = state_rows;
    a.state = state;
    a.out = out;
    a.heads = args->heads;
    a.A = args->dim_k;
    a.W = args->dim_v;
    a.scale = args->scale;
    const bool wide = a.W % 4 == 0 && aligned_to(a.in, 16) && aligned_to(a.state, 16);
    const u64 bh = (u64)args->batch * args->heads;
    // all columns of a state in one workgroup (at most 64 threads across);
    // fewer columns each while that leaves compute units idle
    a.cols = std::min<u32>(pow2_at_least(a.W), wide ? 256u : 64u);
    while (a.cols > 16 && bh * ceil_div(a.W, a.cols) < 512) a.cols /= 2;
    if (wide) a.cols = std::max(a.cols, 4u);
    a.tiles = (u32)ceil_div(a.W, a.cols);
    with_dtype(args->dtype, [&](auto t) {
      using T = decltype(t);
      const dim3 grid((u32)(bh * a.tiles));
      if (wide) hipLaunchKernelGGL((k_step<T, 4>), grid, dim3(kNT), 0, stream, a);
      else hipLaunchKernelGGL((k_step<T, 1>), grid, dim3(kNT), 0, stream, a);
    });
    FSTC_HIP(hipGetLastError());
  });
}

}  // extern "C"

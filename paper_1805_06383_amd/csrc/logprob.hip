// Log-probabilities of given labels, their gradient, and the preference loss
// of pairs of label sequences (fstc_label_logprob, fstc_label_logprob_grad,
// fstc_preference_loss).
//
//   lp_i = x[i, y_i] - log sum_v exp(x[i, v])
//   dx[i, v] = w_i (1[v = y_i] - exp(x[i, v]) / sum_u exp(x[i, u]))
//
// A row whose label is outside [0, vocab) has lp = 0 and a zero gradient and
// is not read.  A row of nothing but -inf has lp = -inf and a zero gradient.
//
// A workgroup takes a row in one pass with the running maximum and sum of the
// softmax in 32-bit registers: a thread takes kBatch vectors, their maximum,
// rescales its sum once and adds their exponentials.  Threads, waves and the
// workgroup join their (maximum, sum) pairs at the end.  The gradient takes
// the row's maximum and 1 / sum from the forward pass, so it reads each logit
// once more and writes it once.  Bound: HBM in both; the forward's
// exponentials (a quarter of the vector rate) come next.  Measured in bfloat16:
// 4,096 x 25,179 logits, a tenth of them padding, forward 35 us (5.4 TB/s),
// gradient 62 us (the logits still in cache, 6.3 TB/s in all); 8,192 x 50,000, half
// of them padding, 70 us (5.8 TB/s) and 240 us (5.1 TB/s).
#include "scoring.hpp"

namespace fstc {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eLow = 1.4426950408889634 - kLog2e;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kBatch = 4;  // vectors a thread has in flight

// e^x of x <= 0 by one rounded product: |x| 2^-24 of e^x off.  In a row's sum the
// terms of weight have |x| of at most about log(vocab) on average, so the logarithm of the
// sum is off by less than its own rounding; of a 16-bit gradient it is at most a hundredth of a unit.
__device__ __forceinline__ float exp_below(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// The same for each element of a gradient.  In 32 bits a probability far below the row's largest
// keeps its digits: 2^h (1 + l) with l what the rounded h lacks, three units of 2^-24 (those below
// 2^-126 are 0).
template <class T>
__device__ __forceinline__ float exp_of(float x) {
  if constexpr (!std::is_same<T, float>::value) return exp_below(x);
  const float h = x * kLog2e, e = __builtin_amdgcn_exp2f(h);
  const float l = fmaf(x, kLog2eLow * kLn2, fmaf(x, kLog2e, -h) * kLn2);
  return e == 0.f ? e : fmaf(e, l, e);  // (x of -inf has no l)
}

// A running maximum and the sum of exp(x - maximum) of what was seen.
struct MaxSum {
  float m, s;
};
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b) {
  const float m = fmaxf(a.m, b.m);
  // (no -inf - -inf where nothing finite was seen)
  const float at = m == -INFINITY ? 0.f : m;
  return {m, a.s * exp_below(a.m - at) + b.s * exp_below(b.m - at)};
}

struct RowArgs {
  u64 rows;
  u32 vocab;
  int64_t stride;
  Labels labels;
};

template <class T, int NT>
__global__ __launch_bounds__(NT) void k_label_logprob(RowArgs a, const T *logits, float *lp, float2 *stats) {
  constexpr int N = 16 / sizeof(T);
  __shared__ MaxSum s_part[NT / kWave];
  for (u64 row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t y = a.labels.at(row);
    if ((u64)y >= a.vocab) {
      if (threadIdx.x == 0) {
        lp[row] = 0.f;
        stats[row] = make_float2(0.f, 0.f);
      }
      continue;
    }
    const T *x = logits + (int64_t)row * a.stride;
    const u32 vectors = a.vocab / N, tail = vectors * N;
    MaxSum r{-INFINITY, 0.f};
    auto add = [&](float v) { r = join(r, MaxSum{v, 1.f}); };
    if (tail + threadIdx.x < a.vocab) add(to_f32(x[tail + threadIdx.x]));
    for (u32 c = threadIdx.x; c < vectors; c += NT * kBatch) {
      Wide<T> v[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) v[j] = load_wide(x + (u64)min(c + j * NT, vectors - 1) * N);
      float m = r.m;
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) m = fmaxf(m, to_f32(v[j].v[e]));
      const float at = m == -INFINITY ? 0.f : m;
      float s = r.s * exp_below(r.m - at);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        float t = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) t += exp_below(to_f32(v[j].v[e]) - at);
        s += c + j * NT < vectors ? t : 0.f;
      }
      r = {m, s};
    }
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) r = join(r, MaxSum{__shfl_xor(r.m, d), __shfl_xor(r.s, d)});
    if (lane_id() == 0) s_part[threadIdx.x / kWave] = r;
    __syncthreads();
    if (threadIdx.x == 0) {
      for (int w = 1; w < NT / kWave; ++w) r = join(r, s_part[w]);
      const bool none = r.m == -INFINITY && r.s == 0.f;
      // (in 64 bits, so that difference and logarithm are rounded once, together)
      lp[row] = none ? -INFINITY : (float)(((double)to_f32(x[y]) - (double)r.m) - log((double)r.s));
      stats[row] = make_float2(none ? 0.f : r.m, none ? 0.f : 1.f / r.s);
    }
    __syncthreads();  // (s_part is read)
  }
}

// Row i's weight is weight[i / per] times *factor (1 without it).  Rows are
// taken from the last to the first: those that the forward pass read last may
// still be in the 256 MB cache.
template <class T, int NT>
__global__ __launch_bounds__(NT) void k_label_logprob_grad(RowArgs a, const T *logits, const float2 *stats,
                                                           const float *weight, u64 per,
                                                           const float *factor, T *dlogits) {
  constexpr int N = 16 / sizeof(T);
  for (u64 i = blockIdx.x; i < a.rows; i += gridDim.x) {
    const u64 row = a.rows - 1 - i;
    const int64_t y = a.labels.at(row);
    const T *x = logits + (int64_t)row * a.stride;
    T *d = dlogits + row * a.vocab;
    const bool live = (u64)y < a.vocab;
    const float w = live ? weight[row / per] * (factor ? *factor : 1.f) : 0.f;
    const float2 st = live ? stats[row] : make_float2(0.f, 0.f);
    const bool zero = !live || st.y == 0.f;
    const float c = -w * st.y;
    auto grad = [&](float v, u32 at) {
      const float p = c * exp_of<T>(v - st.x);
      return zero ? 0.f : at == (u32)y ? p + w : p;
    };
    // elements before the first 16-byte boundary of the output, whole pieces, the rest
    const u32 head = min((u32)((16 - ((uintptr_t)d & 15)) & 15) / (u32)sizeof(T), a.vocab);
    const u32 vectors = (a.vocab - head) / N, tail = head + vectors * N;
    if (threadIdx.x < head)
      d[threadIdx.x] = from_f32<T>(grad(zero ? 0.f : to_f32(x[threadIdx.x]), threadIdx.x));
    for (u32 e = tail + threadIdx.x; e < a.vocab; e += NT)
      d[e] = from_f32<T>(grad(zero ? 0.f : to_f32(x[e]), e));
    for (u32 b = threadIdx.x; b < vectors; b += NT * kBatch) {
      Wide<T> v[kBatch];
      if (!zero) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) v[j] = load_wide(x + head + (u64)min(b + j * NT, vectors - 1) * N);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const u32 k = b + j * NT;
        if (k >= vectors) break;
        Wide<T> o;
#pragma unroll
        for (int e = 0; e < N; ++e) o.v[e] = from_f32<T>(grad(zero ? 0.f : to_f32(v[j].v[e]), head + k * N + e));
        store_out(d + head + (u64)k * N, o);
      }
    }
  }
}

// Sums of each sequence's log-probabilities, then every pair's margin, loss and
// weights, and the mean loss, in one workgroup.  Everything after the
// log-probabilities is in 64 bits and rounded once where it is returned: a sum
// of hundreds of labels is in the thousands, its reference within a few units of it, and
// their difference would keep four digits of 32-bit sums (16 pairs of up to 256 labels, 50,000 logits:
// margins 1.4e-5 of their norm from the definition with sums in 32 bits, 1.5e-6 with these).
constexpr int kPrefNT = 1024;
__global__ __launch_bounds__(kPrefNT) void k_preference(const float *lp, u64 pairs, u64 positions,
                                                        const float *ref, float beta, float smoothing,
                                                        float *loss, float *seq_lp, float *margin,
                                                        float *seq_weight) {
  __shared__ double s_sum[kPrefNT / kWave];
  const u32 lane = lane_id(), wave = threadIdx.x / kWave;
  double total = 0;
  for (u64 p = wave; p < pairs; p += kPrefNT / kWave) {
    double side[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const u64 s = p + (k ? pairs : 0);
      double t = 0;
      for (u64 i = lane * 4; i < positions; i += 4 * kWave) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = i + e < positions ? lp[s * positions + i + e] : 0.f;
        t += ((double)x[0] + x[1]) + ((double)x[2] + x[3]);
      }
      side[k] = wave_sum(t);
      if (lane == 0) seq_lp[s] = (float)side[k];
    }
    if (lane == 0) {
      const double apart = (side[0] - (double)ref[p]) - (side[1] - (double)ref[pairs + p]);
      // no number, though all of its terms are: infinities that cancel
      const bool none = isnan(apart) && !isnan(side[0]) && !isnan(side[1]) && !isnan(ref[p]) && !isnan(ref[pairs + p]);
      const double z = beta == 0.f && !isnan(apart) ? 0.0 : (double)beta * apart;  // (0 times an infinity)
      const double eps = smoothing;
      // -log sigmoid(z) = max(-z, 0) + log(1 + exp(-|z|))
      const double soft = log1p(exp(-fabs(z)));
      double term = (1 - eps) * (fmax(-z, 0.0) + soft);
      if (eps != 0) term += eps * (fmax(z, 0.0) + soft);  // (not 0 times an infinity)
      if (!none) total += term;
      const double g = none ? 0.0 : (eps - 1 / (1 + exp(z))) * (double)beta / (double)pairs;
      margin[p] = (float)z;
      seq_weight[p] = (float)g;
      seq_weight[pairs + p] = (float)-g;
    }
  }
  if (lane == 0) s_sum[wave] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0;
    for (int w = 0; w < kPrefNT / kWave; ++w) t += s_sum[w];
    *loss = (float)(t / (double)pairs);
  }
}

// Threads a row: rows that fill the chip take 256; few rows take 1,024, which
// halves a row's time when it has a compute unit to itself.
inline bool wide_rows(u64 rows) { return rows < 2 * (u64)compute_units(); }

int check_rows(const void *logits, int dtype, u64 rows, u32 vocab, int64_t stride, const void *labels,
               int label_bytes) {
  if (!element_bytes(dtype)) return report_failure(FSTC_ERR_INVALID_ARG, "unknown element type");
  if (label_bytes != 4 && label_bytes != 8)
    return report_failure(FSTC_ERR_INVALID_ARG, "labels are 4- or 8-byte integers");
  if (vocab == 0) return report_failure(FSTC_ERR_INVALID_ARG, "vocab is 0");
  if (stride < (int64_t)vocab) return report_failure(FSTC_ERR_INVALID_ARG, "row stride below vocab");
  if (rows && (!logits || !labels)) return report_failure(FSTC_ERR_INVALID_ARG, "logits or labels is NULL");
  if (!aligned_to(logits, element_bytes(dtype)))
    return report_failure(FSTC_ERR_INVALID_ARG, "logits are not aligned to their elements");
  if (rows >= (1ull << 31) || vocab >= (1u << 31) - (1u << 16))
    return report_failure(FSTC_ERR_RANGE, "rows and vocab must be below 2^31");
  return FSTC_OK;
}

}  // namespace
}  // namespace fstc

using namespace fstc;

extern "C" {

int fstc_label_logprob(const void *logits, int dtype, uint64_t rows, uint32_t vocab, int64_t row_stride,
                       const void *labels, int label_bytes, float *logprob, float *row_stats,
                       hipStream_t stream) {
  const int rc = check_rows(logits, dtype, rows, vocab, row_stride, labels, label_bytes);
  if (rc) return rc;
  if (rows && (!logprob || !row_stats))
    return report_failure(FSTC_ERR_INVALID_ARG, "logprob or row_stats is NULL");
  if (rows == 0) return FSTC_OK;
  return run_reported("fstc_label_logprob", stream, [&] {
    const RowArgs a{rows, vocab, row_stride, Labels{labels, label_bytes}};
    const u32 grid = (u32)std::min(rows, kMaxGrid);
    with_dtype(dtype, [&](auto t) {
      using T = decltype(t);
      const T *x = static_cast<const T *>(logits);
      float2 *st = reinterpret_cast<float2 *>(row_stats);
      if (wide_rows(rows))
        hipLaunchKernelGGL((k_label_logprob<T, 1024>), dim3(grid), dim3(1024), 0, stream, a, x, logprob, st);
      else
        hipLaunchKernelGGL((k_label_logprob<T, 256>), dim3(grid), dim3(256), 0, stream, a, x, logprob, st);
    });
    FSTC_HIP(hipGetLastError());
  });
}

int fstc_label_logprob_grad(const void *logits, int dtype, uint64_t rows, uint32_t vocab,
                            int64_t row_stride, const void *labels, int label_bytes,
                            const float *row_stats, const float *weight, uint64_t rows_per_weight,
                            const float *factor, void *dlogits, hipStream_t stream) {
  const int rc = check_rows(logits, dtype, rows, vocab, row_stride, labels, label_bytes);
  if (rc) return rc;
  if (rows && (!row_stats || !weight || !dlogits))
    return report_failure(FSTC_ERR_INVALID_ARG, "row_stats, weight or dlogits is NULL");
  if (rows_per_weight == 0) return report_failure(FSTC_ERR_INVALID_ARG, "rows_per_weight is 0");
  if (rows == 0) return FSTC_OK;
  return run_reported("fstc_label_logprob_grad", stream, [&] {
    const RowArgs a{rows, vocab, row_stride, Labels{labels, label_bytes}};
    const u32 grid = (u32)std::min(rows, kMaxGrid);
    with_dtype(dtype, [&](auto t) {
      using T = decltype(t);
      const T *x = static_cast<const T *>(logits);
      const float2 *st = reinterpret_cast<const float2 *>(row_stats);
      T *d = static_cast<T *>(dlogits);
      if (wide_rows(rows))
        hipLaunchKernelGGL((k_label_logprob_grad<T, 1024>), dim3(grid), dim3(1024), 0, stream, a, x, st,
                           weight, rows_per_weight, factor, d);
      else
        hipLaunchKernelGGL((k_label_logprob_grad<T, 256>), dim3(grid), dim3(256), 0, stream, a, x, st,
                           weight, rows_per_weight, factor, d);
    });
    FSTC_HIP(hipGetLastError());
  });
}

int fstc_preference_loss(const float *logprob, uint64_t pairs, uint64_t positions, const float *ref,
                         float beta, float label_smoothing, float *loss, float *seq_logprob,
                         float *margin, float *seq_weight, hipStream_t stream) {
  if (pairs == 0) return report_failure(FSTC_ERR_INVALID_ARG, "no pairs");
  if ((positions && !logprob) || !ref || !loss || !seq_logprob || !margin || !seq_weight)
    return report_failure(FSTC_ERR_INVALID_ARG, "an array is NULL");
  if (!(label_smoothing >= 0.f && label_smoothing < 0.5f))
    return report_failure(FSTC_ERR_INVALID_ARG, "label_smoothing must be in [0, 0.5)");
  if (pairs >= (1ull << 31) || positions >= (1ull << 31))
    return report_failure(FSTC_ERR_RANGE, "pairs and positions must be below 2^31");
  return run_reported("fstc_preference_loss", stream, [&] {
    hipLaunchKernelGGL(k_preference, dim3(1), dim3(kPrefNT), 0, stream, logprob, pairs, positions, ref,
                       beta, label_smoothing, loss, seq_logprob, margin, seq_weight);
    FSTC_HIP(hipGetLastError());
  });
}

}  // extern "C"

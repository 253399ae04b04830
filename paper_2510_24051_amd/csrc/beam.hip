// Selection over beams and vocabulary: per group of rows (the beams of one search) the candidates of largest score
//   score(r, v) = s_r + z_rv / T - log sum_u exp(z_ru / T)
// ordered by descending score, then by beam, then by token.  A logit of -inf or NaN is no candidate, +inf counts as the
// largest finite value of its type, a row with s_r = -inf or NaN has no candidates, a finished row has exactly one.
//
// Scores are compared in 64 bits: candidates of different beams lie within 1e-3 of one another in every step, and one unit in
// the last place of a 32-bit score (1e-6 at 10) reorders them now and then.
#include "internal.h"

namespace {
// One logit as the selection sees it.
template <typename T>
__device__ __forceinline__ float beam_logit(T x);
template <>
__device__ __forceinline__ float beam_logit<float>(float x) {
  return x != x ? -INFINITY : fminf(x, 3.402823466e38f);
}
template <>
__device__ __forceinline__ float beam_logit<bf16_t>(bf16_t x) {
  const float f = (float)x;
  return f != f ? -INFINITY : fminf(f, 3.3895313892515355e38f);
}
template <>
__device__ __forceinline__ float beam_logit<_Float16>(_Float16 x) {
  const float f = (float)x;
  return f != f ? -INFINITY : fminf(f, 65504.f);
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}

#define BR_THREADS 256
// base[row] = (b, m) with m the largest logit and score = b + (z - m) / T: b = s_r - log sum exp((z - m) / T), -inf where the row has
// no candidates.  (Not s_r - (m / T + log sum ..): beside a logit of 1e38 the logarithm would be lost, 64 bits or not.)
template <typename T>
__global__ __launch_bounds__(BR_THREADS) void beam_row_kernel(const T* __restrict__ logits, int64_t stride, int V, double inv_temp,
                                                              const float* __restrict__ scores, const uint8_t* __restrict__ finished,
                                                              double2* __restrict__ base) {
  __shared__ float smax[BR_THREADS / 64];
  __shared__ double ssum[BR_THREADS / 64];
  const int row = blockIdx.x, tid = threadIdx.x;
  const T* z = logits + (int64_t)row * stride;
  float s = scores ? scores[row] : 0.f;
  s = s != s ? -INFINITY : fminf(s, 3.402823466e38f);
  if (finished && finished[row]) {
    if (tid == 0) base[row] = make_double2((double)s, 0.0);
    return;
  }
  float m = -INFINITY;
  for (int i = tid; i < V; i += BR_THREADS) m = fmaxf(m, beam_logit(z[i]));
  m = wave_max(m);
  if ((tid & 63) == 0) smax[tid >> 6] = m;
  __syncthreads();
  for (int w = 0; w < BR_THREADS / 64; ++w) m = fmaxf(m, smax[w]);
  if (m == -INFINITY || s == -INFINITY) {
    if (tid == 0) base[row] = make_double2(-INFINITY, 0.0);
    return;
  }
  double sum = 0;
  for (int i = tid; i < V; i += BR_THREADS) sum += exp(((double)beam_logit(z[i]) - (double)m) * inv_temp);
  sum = wave_sum_f64(sum);
  if ((tid & 63) == 0) ssum[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0) {
    sum = 0;
    for (int w = 0; w < BR_THREADS / 64; ++w) sum += ssum[w];
    base[row] = make_double2((double)s - log(sum), (double)m);
  }
}

struct BeamGroups { int32_t row0[BEAM_GROUPS_BY_VALUE + 1]; };

#define BG_THREADS 1024
// n_out rounds, each taking the first candidate behind the last one taken
template <typename T>
__global__ __launch_bounds__(BG_THREADS) void beam_group_kernel(const T* __restrict__ logits, int64_t stride, int V, double inv_temp,
                                                                const uint8_t* __restrict__ finished, int eos, BeamGroups groups, int n_out,
                                                                const double2* __restrict__ base, int32_t* __restrict__ out_beams,
                                                                int32_t* __restrict__ out_tokens, float* __restrict__ out_scores) {
  __shared__ double skey[BG_THREADS / 64];
  __shared__ int sidx[BG_THREADS / 64];
  const int g = blockIdx.x, tid = threadIdx.x;
  const int row0 = groups.row0[g], rows = groups.row0[g + 1] - row0;
  double last = INFINITY;
  int last_idx = -1;
  for (int k = 0; k < n_out; ++k) {
    double best = -INFINITY;
    int best_idx = 0x7FFFFFFF;
    for (int r = 0; r < rows; ++r) {
      const double2 b = base[row0 + r];
      if (b.x == -INFINITY) continue;
      const bool done = finished && finished[row0 + r];
      const T* z = logits + (int64_t)(row0 + r) * stride;
      for (int v = tid; v < V; v += BG_THREADS) {
        double key = b.x + (done ? 0.0 : ((double)beam_logit(z[v]) - b.y) * inv_temp);
        if (done && v != eos) key = -INFINITY;
        const int idx = r * V + v;
        const bool after = key < last || (key == last && idx > last_idx);
        if (after && key > best) { best = key; best_idx = idx; }  // (indices ascend)
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const double k2 = __shfl_xor(best, o);
      const int i2 = __shfl_xor(best_idx, o);
      if (k2 > best || (k2 == best && i2 < best_idx)) { best = k2; best_idx = i2; }
    }
    __syncthreads();
    if ((tid & 63) == 0) { skey[tid >> 6] = best; sidx[tid >> 6] = best_idx; }
    __syncthreads();
    for (int w = 0; w < BG_THREADS / 64; ++w)
      if (skey[w] > best || (skey[w] == best && sidx[w] < best_idx)) { best = skey[w]; best_idx = sidx[w]; }
    const bool none = best == -INFINITY;
    if (tid == 0) {
      out_beams[(int64_t)g * n_out + k] = none ? -1 : best_idx / V;
      out_tokens[(int64_t)g * n_out + k] = none ? -1 : best_idx % V;
      out_scores[(int64_t)g * n_out + k] = none ? -INFINITY : (float)best;
    }
    last = best;
    last_idx = best_idx;
  }
}

template <typename T>
hipError_t beam_select(const BeamArgs& a, hipStream_t s) {
  const T* z = reinterpret_cast<const T*>(a.logits);
  const int n = a.group_indptr[a.n_groups];
  if (n > 0) beam_row_kernel<T><<<dim3((unsigned)n), dim3(BR_THREADS), 0, s>>>(z, a.stride, a.V, a.inv_temp, a.scores, a.finished, reinterpret_cast<double2*>(a.ws));
  for (int g0 = 0; g0 < a.n_groups; g0 += BEAM_GROUPS_BY_VALUE) {
    const int ng = a.n_groups - g0 < BEAM_GROUPS_BY_VALUE ? a.n_groups - g0 : BEAM_GROUPS_BY_VALUE;
    BeamGroups groups{};
    for (int g = 0; g <= ng; ++g) groups.row0[g] = a.group_indptr[g0 + g];
    beam_group_kernel<T><<<dim3((unsigned)ng), dim3(BG_THREADS), 0, s>>>(z, a.stride, a.V, a.inv_temp, a.finished, a.eos, groups, a.n_out, reinterpret_cast<double2*>(a.ws),
                                                                         a.out_beams + (int64_t)g0 * a.n_out, a.out_tokens + (int64_t)g0 * a.n_out,
                                                                         a.out_scores + (int64_t)g0 * a.n_out);
  }
  return hipGetLastError();
}
}  // namespace

size_t beam_ws_doubles(int rows, int vocab) {
  (void)vocab;
  return 2 * (size_t)rows;
}

hipError_t launch_beam_select(const BeamArgs& a, hipStream_t s) {
  if (a.dtype == PIE_BF16) return beam_select<bf16_t>(a, s);
  if (a.dtype == PIE_F16) return beam_select<_Float16>(a, s);
  return beam_select<float>(a, s);
}

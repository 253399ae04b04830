// Selection over beams and vocabulary: per group of rows (the beams of one search) the candidates of largest score
//   score(r, v) = s_r + (z_rv - m_r) / T - log sum_u exp((z_ru - m_r) / T),  m_r = max_u z_ru
// ordered by descending score, then by beam, then by token.  A logit of -inf or NaN is no candidate, +inf counts as the
// largest finite value of its type, a row with s_r = -inf or NaN has no candidates, a finished row has exactly one.
//
// Scores are compared in 64 bits: candidates of different beams lie within 1e-3 of one another in every step, and one unit in
// the last place of a 32-bit score (1e-6 at 10) reorders them now and then.  The exponentials are taken in 32 bits, each off
// by its argument's three roundings and a step, and summed in 64 (in 32, small terms beside a large one are lost: 1e-7 to 1e-6 on the
// logarithm of a peaked row).  2.4e-6 on the logarithm at most, a few 1e-8 on a language model's rows, 1e-9 where one token has nearly all
// of the probability.  512 rows of 128256 with sums in 64 bits and in 32: fp32 53.8 and 53.1 us a call, 16 bits 41.7 and 39.5.
//
// Two kernels.  beam_tiles reads every logit once and leaves, per segment (what a wave loads at once), the largest, and per tile of
// eight segments the largest and the sum of exponentials.  beam_pick, one workgroup per group, turns the segments' maxima into scores
// and keeps the n_out best segments by (score, beam, place): no other segment can hold one of the n_out best candidates, as
// each of those n_out has one that comes before all of its own.  Only these are read again.  Where groups are small beam_pick does
// the tiles as well.
#include "internal.h"

namespace {
// One logit as the selection sees it.
__device__ __forceinline__ float beam_logit(float x) { return x != x ? -INFINITY : fminf(x, 3.402823466e38f); }
__device__ __forceinline__ float beam_logit(bf16_t x) {
  const float f = (float)x;
  return f != f ? -INFINITY : fminf(f, 3.3895313892515355e38f);
}
__device__ __forceinline__ float beam_logit(_Float16 x) {
  const float f = (float)x;
  return f != f ? -INFINITY : fminf(f, 65504.f);
}
__device__ __forceinline__ float beam_score(const float* scores, int row) {  // -inf: the row has no candidates
  const float s = scores ? scores[row] : 0.f;
  return s != s ? -INFINITY : fminf(s, 3.402823466e38f);
}

#define BT_SEGS 8  // segments of a tile
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
// A row cut into segments by its tokens, wherever it lies in memory: equal rows then have equal sums, bit for bit, and so
// equal scores.  (Cut at 16-byte addresses instead, two beams with the same logits differed in the last bits of 64.)  Loads of 16
// bytes from rows that are aligned to their elements only are ordinary on this chip; they touch a line more now and then.
template <typename T>
struct BeamRow {
  static constexpr int VEC = 16 / sizeof(T), SEG = 64 * VEC, TILE = BT_SEGS * SEG;
  const T* z;
  int V;
  __device__ BeamRow(const T* logits, int64_t stride, int row, int V_) : z(logits + (int64_t)row * stride), V(V_) {}
  // the VEC logits from token p on, -inf in place of what is behind the row
  __device__ __forceinline__ void load(int p, float (&x)[VEC]) const {
    if (p + VEC <= V) {
      unpack(*reinterpret_cast<const u32x4_at2*>(z + p), x);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) x[i] = p + i < V ? beam_logit(z[p + i]) : -INFINITY;
    }
  }
  __device__ __forceinline__ u32x4 stream(int p) const { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_at2*>(z + p)); }
  static __device__ __forceinline__ void unpack(u32x4 u, float (&x)[VEC]) {
    union { u32x4 u; T e[VEC]; } w;
    w.u = u;
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = beam_logit(w.e[i]);
  }
};
template <typename T>
constexpr int beam_tiles_of(int V) { return (V + BeamRow<T>::TILE - 1) / BeamRow<T>::TILE; }

// Wave-wide maxima of eight values at once: each exchange halves how many a lane carries on, 4 + 2 + 1 + 3 instead of 8 x 6.  Lane l
// returns the maximum of value l / 8.
__device__ __forceinline__ float wave_max8(const float (&v)[8], int lane) {
  float a[4], b[2], c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // lanes below 32 go on with values 0 .. 3
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 4]), false, false);
    a[i] = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a[i]), __float_as_uint(a[i + 2]), false, false);
    b[i] = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  const bool up = lane & 8;
  const float mine = up ? b[1] : b[0], other = up ? b[0] : b[1];
  c = fmaxf(mine, __shfl_xor(other, 8));
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) c = fmaxf(c, __shfl_xor(c, o));
  return c;
}

// One tile of a row: lane l returns the maximum of segment l / 8, *stats (maximum, sum of exponentials) of the tile.
// exp((x - m) / T) = exp2((x - m) (c_hi + c_lo)), c = log2(e) / T in two parts; x_min keeps infinities out (exp2 is 0 there).
struct BeamScale { float c_hi, c_lo, x_min; };
struct __attribute__((aligned(16))) TileStats { double sum; float m; };
template <typename T>
__device__ __forceinline__ float beam_tile(const BeamRow<T>& z, int tile, const BeamScale& scale, int lane, TileStats* stats) {
  constexpr int VEC = BeamRow<T>::VEC, SEG = BeamRow<T>::SEG;
  float x[BT_SEGS][VEC], top[BT_SEGS];
  const int p0 = tile * BT_SEGS * SEG + lane * VEC;
  if ((tile + 1) * BT_SEGS * SEG <= z.V) {  // (uniform: all eight loads go out at once)
    u32x4 raw[BT_SEGS];
#pragma unroll
    for (int j = 0; j < BT_SEGS; ++j) raw[j] = z.stream(p0 + j * SEG);
#pragma unroll
    for (int j = 0; j < BT_SEGS; ++j) BeamRow<T>::unpack(raw[j], x[j]);
  } else {
#pragma unroll
    for (int j = 0; j < BT_SEGS; ++j) z.load(p0 + j * SEG, x[j]);
  }
#pragma unroll
  for (int j = 0; j < BT_SEGS; ++j) {
    top[j] = x[j][0];
#pragma unroll
    for (int i = 1; i < VEC; ++i) top[j] = fmaxf(top[j], x[j][i]);
  }
  const float seg = wave_max8(top, lane);
  float m = seg;
#pragma unroll
  for (int o = 32; o >= 8; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  double sum = 0;
  if (m != -INFINITY) {
#pragma unroll
    for (int j = 0; j < BT_SEGS; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const float d = fmaxf(x[j][i] - m, scale.x_min);
        sum += (double)__builtin_amdgcn_exp2f(__builtin_fmaf(d, scale.c_lo, d * scale.c_hi));
      }
  }
  *stats = TileStats{wave_sum_f64(sum), m};
  return seg;
}

// A wave per tile.  Bound by HBM: 262 MB of logits (512 rows of 128256) in 41 to 43 us, 6.1 to 6.4 TB/s, the rate of a streaming read.
#define BT_WAVES 4
template <typename T>
__global__ __launch_bounds__(64 * BT_WAVES) void beam_tiles_kernel(const T* __restrict__ logits, int64_t stride, int V, int n_tiles, BeamScale scale,
                                                                   const float* __restrict__ scores, const uint8_t* __restrict__ finished,
                                                                   float* __restrict__ seg_max, TileStats* __restrict__ tile_stats, int64_t total) {
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)blockIdx.x * BT_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int row = (int)(at / n_tiles), tile = (int)(at % n_tiles);
  if ((finished && finished[row]) || beam_score(scores, row) == -INFINITY) return;  // (nothing of theirs is looked at)
  TileStats stats;
  const float seg = beam_tile(BeamRow<T>(logits, stride, row, V), tile, scale, lane, &stats);
  if ((lane & 7) == 0) seg_max[at * BT_SEGS + (lane >> 3)] = seg;
  if (lane == 0) tile_stats[at] = stats;
}

// ---------------------------------------------------------------------------------------------
// picking
// ---------------------------------------------------------------------------------------------
typedef unsigned long long u64;
// Order-preserving integer of a score; 0 stands for no candidate.
__device__ __forceinline__ u64 score_key(double s) {
  if (s == -INFINITY) return 0;
  const u64 u = __double_as_longlong(s + 0.0);  // (-0 and 0 are one score)
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double key_score(u64 k) { return __longlong_as_double(k >> 63 ? k & ~(1ull << 63) : ~k); }

#define BP_THREADS 1024
#define BP_SEGS 576   // segments kept for reading again: at most 2 n_out + 64
#define BP_CANDS 512  // candidates that are put in order
#define BP_COUNTED 192  // of which so many by counting
#define BP_CACHED 8192  // maxima of segments kept in LDS
#define BP_WHOLE 16     // tiles of a group that is read by its one workgroup
template <int N>
struct BeamGroups { int32_t row0[N + 1]; };  // (a short list has a small block: calls back to back 3.4 us of the host's time each, 6.4 with the large one)
#define BP_HELD (BP_CACHED / BP_THREADS)
struct PickShared {
  double2 row[BEAM_MAX_ROWS];  // (b, m): score = b + (z - m) / T; b = -inf: no candidates
  u64 cand_key[BP_CANDS];
  int cand_idx[BP_CANDS];
  int segs[BP_SEGS], segs_sorted[BP_SEGS];
  uint32_t hist[1024];
  float maxima[BP_CACHED];
  TileStats stats[BP_WHOLE];
  u64 red_lo[BP_THREADS / 64], red_hi[BP_THREADS / 64];
  uint32_t red_n[BP_THREADS / 64];
  uint32_t count, n_cand, bin, below, upto;
  uint8_t done[BEAM_MAX_ROWS];
};

// A bound `lo` that at least `need` of the n keys reach (all valid ones, where there are fewer) and at most `cap` do, if there is one
// (ties at lo otherwise: then `ties` of those equal to lo, in order, belong to the first `need`).  Keys are counted in 1024 bins of
// the range they span, and the range narrows to the bin of the need-th: one pass where the scores are spread, seven at most.
struct Bound { u64 lo; uint32_t n; uint32_t ties; bool tied; };
template <typename F>
__device__ Bound pick_bound(PickShared& sh, int n, uint32_t need, uint32_t cap, F key) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  u64 lo = ~0ull, hi = 0;
  uint32_t valid = 0;
  for (int i = tid; i < n; i += BP_THREADS) {
    const u64 k = key(i);
    if (k) { lo = k < lo ? k : lo; hi = k > hi ? k : hi; ++valid; }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const u64 l = __shfl_xor(lo, o), h = __shfl_xor(hi, o);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
    valid += __shfl_xor(valid, o);
  }
  __syncthreads();
  if (lane == 0) { sh.red_lo[wave] = lo; sh.red_hi[wave] = hi; sh.red_n[wave] = valid; }
  __syncthreads();
  valid = 0;
#pragma unroll
  for (int w = 0; w < BP_THREADS / 64; ++w) {
    lo = sh.red_lo[w] < lo ? sh.red_lo[w] : lo;
    hi = sh.red_hi[w] > hi ? sh.red_hi[w] : hi;
    valid += sh.red_n[w];
  }
  if (valid <= need || valid <= cap) return Bound{valid ? lo : 1ull, valid, 0, false};
  uint32_t above = 0;  // keys above the range
  for (;;) {
    const u64 span = hi - lo;
    const int bits = span ? 64 - __clzll((long long)span) : 0, shift = bits > 10 ? bits - 10 : 0;
    sh.hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += BP_THREADS) {
      const u64 k = key(i);
      if (k >= lo && k <= hi) atomicAdd(&sh.hist[(uint32_t)((k - lo) >> shift)], 1u);
    }
    __syncthreads();
    const uint32_t c = sh.hist[BP_THREADS - 1 - tid];  // from the top down
    uint32_t incl = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t t = __shfl_up(incl, o);
      if (lane >= o) incl += t;
    }
    if (lane == 63) sh.red_n[wave] = incl;
    __syncthreads();
    uint32_t before = above;
    for (int w = 0; w < wave; ++w) before += sh.red_n[w];
    incl += before;
    if (incl >= need && incl - c < need) { sh.bin = BP_THREADS - 1 - tid; sh.below = incl - c; sh.upto = incl; }
    __syncthreads();
    const uint32_t bin = sh.bin, excl = sh.below, upto = sh.upto;
    lo += (u64)bin << shift;
    if (upto <= cap) return Bound{lo, upto, 0, false};
    if (shift == 0) return Bound{lo, upto, need - excl, true};
    above = excl;
    const u64 end = lo + ((1ull << shift) - 1);
    hi = end < hi ? end : hi;
    __syncthreads();
  }
}

// put(i) for every i whose key reaches the bound, of those that tie for the last places the first ones; any order, whole
// workgroup.  Returns how many there are.
template <typename F, typename P>
__device__ uint32_t pick_collect(PickShared& sh, int n, const Bound& b, F key, P put) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  __syncthreads();
  if (tid == 0) sh.count = 0;
  __syncthreads();
  const u64 from = b.tied ? b.lo + 1 : b.lo;
  for (int i = tid; i < n; i += BP_THREADS) {
    const u64 k = key(i);
    if (k && k >= from) put(atomicAdd(&sh.count, 1u), i, k);
  }
  __syncthreads();
  uint32_t have = sh.count;
  if (b.tied) {
    uint32_t left = b.ties;
    for (int i0 = 0; i0 < n && left; i0 += BP_THREADS) {  // (uniform)
      const bool mine = i0 + tid < n && key(i0 + tid) == b.lo;
      const u64 votes = __ballot(mine);
      __syncthreads();
      if (lane == 0) sh.red_n[wave] = __popcll(votes);
      __syncthreads();
      uint32_t at = __popcll(votes & ((1ull << lane) - 1)), all = 0;
      for (int w = 0; w < BP_THREADS / 64; ++w) {
        if (w < wave) at += sh.red_n[w];
        all += sh.red_n[w];
      }
      if (mine && at < left) put(have + at, i0 + tid, b.lo);
      const uint32_t took = all < left ? all : left;
      have += took;
      left -= took;
    }
  }
  __syncthreads();
  return have;
}

// How far a score is behind the best of the group, as a bin: 64 to an octave from half a nat on (a bin is 0.008 wide at the front,
// then 1/64 to 1/128 of the distance), up to 32767 nats.  Distances are sums of two terms of one sign in fp32, off by 1e-6 of
// themselves: whoever takes one bin more than needed misses nobody.
#define BP_BINS 1024
__device__ __forceinline__ uint32_t far_bin(float d) { return min((__float_as_uint(d + 0.5f) >> 17) - (__float_as_uint(0.5f) >> 17), (uint32_t)BP_BINS - 1u); }

template <typename T>
struct Picker {
  static constexpr int VEC = BeamRow<T>::VEC, SEG = BeamRow<T>::SEG;
  PickShared& sh;
  const T* logits;
  int64_t stride;
  int V, n_segs, n, n_out, row0, rows, eos;
  double inv_temp;
  float per;             // 1 / n_segs
  const float* maxima;   // of the group's segments, in LDS or not
  int tid, lane, wave;

  __device__ int row_of(int i) const { return (int)(((float)i + 0.5f) * per); }  // (i < 256 x 512: off by 5e-5, half a segment is 1e-3)
  __device__ u64 key_of(int r, float z) const {
    const double2 b = sh.row[r];
    return b.x == -INFINITY || z == -INFINITY ? 0ull : score_key(b.x + ((double)z - b.y) * inv_temp);
  }

  // The usual call: the group's candidates by their distances in fp32, one pass over the segments' maxima (in registers) and one over
  // the logits of those kept.  Returns how many candidates it left in sh, or -1 where that does not serve: candidates further
  // apart than the bins reach or more of them in a bin than there is room for.
  template <typename H>
  __device__ int quick(const H& held, bool cached) {
    double best = -INFINITY;
    for (int r = lane; r < rows; r += 64) best = fmax(best, sh.row[r].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) best = fmax(best, __shfl_xor(best, o));
    if (best == -INFINITY) return 0;  // (uniform over the workgroup)
    // One step of a 64-bit score at 2^40 is 2^-12, a thirtieth of the narrowest bin.  Far beyond, scores swallow what tells their
    // logits apart, and candidates that are bins apart here are equal there and go by beam and token.
    if (fabs(best) > 1099511627776.0) return -1;
    const float c = (float)inv_temp;
    // (behind, m): a row's best score behind the group's and its largest logit; z is far_bin(behind + (m - z) c) away, -inf infinitely
    auto row_at = [&](int r) { return make_float2((float)(best - sh.row[r].x), (float)sh.row[r].y); };
    auto seg_bin = [&](int i, float z) {  // BP_BINS - 1: not counted
      const int r = row_of(i);
      const float2 at = row_at(r);
      if (sh.done[r]) return i == r * n_segs ? far_bin(at.x) : BP_BINS - 1u;
      return far_bin(at.x + (at.y - z) * c);
    };
    uint32_t bins[BP_HELD];
    if (cached) {
#pragma unroll
      for (int j = 0; j < BP_HELD; ++j) {
        const int i = tid + j * BP_THREADS;
        bins[j] = i < n ? seg_bin(i, held[j]) : BP_BINS - 1;
        if (bins[j] < BP_BINS - 1) atomicAdd(&sh.hist[bins[j]], 1u);
      }
    } else {
      for (int i = tid; i < n; i += BP_THREADS) {
        const uint32_t b = seg_bin(i, maxima[i]);
        if (b < BP_BINS - 1) atomicAdd(&sh.hist[b], 1u);
      }
    }
    __syncthreads();
    // one bin more than the n_out-th segment's (see far_bin); all, where there are fewer segments
    int bin = cut_bin();
    bool by_logit = bin < 0;
    if (by_logit) {
      if (n > BP_SEGS) return -1;
      bin = BP_BINS - 2;
    }
    auto keep = [&](int i) {
      const uint32_t k = atomicAdd(&sh.count, 1u);
      if (k < BP_SEGS) sh.segs[k] = i;
    };
    if (cached) {
#pragma unroll
      for (int j = 0; j < BP_HELD; ++j)
        if ((int)bins[j] <= bin) keep(tid + j * BP_THREADS);
    } else {
      for (int i = tid; i < n; i += BP_THREADS)
        if ((int)seg_bin(i, maxima[i]) <= bin) keep(i);
    }
    __syncthreads();
    const int kept = (int)sh.count;
    if (kept > BP_SEGS) return -1;
    // the kept segments' logits, 8 of a thread at a time (16 bits: four of these spill): take(bin, row, token, logit)
    auto each = [&](auto take) {
      constexpr int U = 8 / VEC;
      for (int e0 = tid * VEC; e0 < kept * SEG; e0 += U * BP_THREADS * VEC) {
        float x[U][VEC];
        int row[U], p[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int e = e0 + u * BP_THREADS * VEC;
          row[u] = -1;
          if (e >= kept * SEG) continue;
          const int i = sh.segs[e / SEG], r = row_of(i);
          p[u] = (i - r * n_segs) * SEG + e % SEG;
          row[u] = r;
          if (!sh.done[r]) BeamRow<T>(logits, stride, row0 + r, V).load(p[u], x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int r = row[u];
          if (r < 0) continue;
          const float2 at = row_at(r);
          if (sh.done[r]) {
            if (p[u] == 0) take((int)far_bin(at.x), r, eos, 0.f);  // (its one candidate stands in its first segment)
            continue;
          }
#pragma unroll
          for (int k = 0; k < VEC; ++k) take((int)far_bin(at.x + (at.y - x[u][k]) * c), r, p[u] + k, x[u][k]);
        }
      }
    };
    auto collect = [&](int b, int r, int v, float z) {
      if (b <= bin) put(sh.done[r] ? score_key(sh.row[r].x) : key_of(r, z), r * V + v);
    };
    if (!by_logit) {
      each(collect);
      __syncthreads();
      if (sh.n_cand <= BP_CANDS) return (int)sh.n_cand;
      __syncthreads();
    }
    // fewer segments than candidates asked for, or many candidates in them: the bins of the logits themselves
    sh.hist[tid] = 0;
    if (tid == 0) sh.n_cand = 0;
    __syncthreads();
    each([&](int b, int, int, float) { if (b <= bin) atomicAdd(&sh.hist[b], 1u); });
    __syncthreads();
    bin = cut_bin();
    if (bin < 0) return -1;
    each(collect);
    __syncthreads();
    return sh.n_cand <= BP_CANDS ? (int)sh.n_cand : -1;
  }
  // One bin more than that of the n_out-th counted in sh.hist, -1 where fewer are; every wave finds it for itself, 16 bins to a lane.
  __device__ int cut_bin() const {
    uint32_t h[16], mine = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) { h[k] = sh.hist[lane * 16 + k]; mine += h[k]; }
    uint32_t incl = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(incl, o);
      if (lane >= o) incl += up;
    }
    const u64 reached = __ballot(incl >= (uint32_t)n_out);
    if (!reached) return -1;
    uint32_t run = incl - mine;
    int bin = BP_BINS;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      run += h[k];
      if (bin == BP_BINS && run >= (uint32_t)n_out) bin = lane * 16 + k;
    }
    bin = __shfl(bin, __ffsll((long long)reached) - 1) + 1;
    return bin < BP_BINS - 1 ? bin : -1;
  }
  __device__ void put(u64 key, int idx) {
    const uint32_t at = atomicAdd(&sh.n_cand, 1u);
    if (at < BP_CANDS) { sh.cand_key[at] = key; sh.cand_idx[at] = idx; }
  }

  // Any group: the same choice by exact bounds, twice.
  __device__ int exactly() {
    // a finished row's one candidate stands in its first segment
    auto seg_key = [&](int i) {
      const int r = row_of(i);
      if (sh.done[r]) return i == r * n_segs && sh.row[r].x != -INFINITY ? score_key(sh.row[r].x) : 0ull;
      return key_of(r, maxima[i]);
    };
    const Bound segs = pick_bound(sh, n, (uint32_t)n_out, (uint32_t)(2 * n_out + 64), seg_key);
    const int kept = (int)pick_collect(sh, n, segs, seg_key, [&](uint32_t at, int i, u64) { sh.segs[at] = i; });
    for (int i = tid; i < kept; i += BP_THREADS) {  // in order of their places
      const int mine = sh.segs[i];
      int at = 0;
      for (int k = 0; k < kept; ++k) at += sh.segs[k] < mine;
      sh.segs_sorted[at] = mine;
    }
    __syncthreads();
    // candidates: the kept segments' logits that reach the bound (all, where there are fewer segments than candidates asked for)
    const u64 floor_key = segs.n < (uint32_t)n_out ? 1ull : segs.lo;
    auto place = [&](int e, int& r, int& p) {
      const int i = sh.segs_sorted[e / SEG];
      r = row_of(i);
      p = (i - r * n_segs) * SEG + e % SEG;
    };
    auto elem_key = [&](int e) {
      int r, p;
      place(e, r, p);
      if (sh.done[r]) return e % SEG == 0 ? score_key(sh.row[r].x) : 0ull;
      if (p >= V) return 0ull;
      const u64 k = key_of(r, beam_logit(logits[(int64_t)(row0 + r) * stride + p]));
      return k >= floor_key ? k : 0ull;
    };
    const Bound best = pick_bound(sh, kept * SEG, (uint32_t)n_out, (uint32_t)BP_CANDS, elem_key);
    return (int)pick_collect(sh, kept * SEG, best, elem_key, [&](uint32_t at, int e, u64 key) {
      int r, p;
      place(e, r, p);
      sh.cand_key[at] = key;
      sh.cand_idx[at] = r * V + (sh.done[r] ? eos : p);
    });
  }
};

// One workgroup per group.  Bound by its chain of latencies: 9 us for eight rows of 128256 (the tiles' results and the rows'
// logarithms 2.0, bins 1.9, cutting and keeping 1.7, the kept segments' logits 1 to 2, ranks and outputs 1).
// WHOLE: groups of at most BP_WHOLE tiles, which the workgroup reads itself, in one launch instead of two (groups of four rows of
// 1024, 4096 and 8192, 4, 8 and 16 tiles: 12.4 -> 11.6, 11.3 -> 10.0, 11.7 -> 11.1 us a call, 64 of them 14.5 -> 12.2, 12.6 ->
// 11.2, 12.6 -> 12.0; at 32 tiles, two to a wave, 14.6 against 12).
template <typename T, bool WHOLE, int N>
__global__ __launch_bounds__(BP_THREADS) void beam_pick_kernel(const T* __restrict__ logits, int64_t stride, int V, int n_tiles, double inv_temp,
                                                               BeamScale scale, const float* __restrict__ scores,
                                                               const uint8_t* __restrict__ finished, int eos, BeamGroups<N> groups, int n_out,
                                                               const float* __restrict__ seg_max, const TileStats* __restrict__ tile_stats,
                                                               int32_t* __restrict__ out_beams, int32_t* __restrict__ out_tokens,
                                                               float* __restrict__ out_scores) {
  __shared__ PickShared sh;
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row0 = groups.row0[g], rows = groups.row0[g + 1] - row0;
  const int n_segs = n_tiles * BT_SEGS, n = rows * n_segs;
  const float* maxima = WHOLE ? sh.maxima : seg_max + (int64_t)row0 * n_segs;
  const TileStats* stats = WHOLE ? sh.stats : tile_stats + (int64_t)row0 * n_tiles;
  if (WHOLE) {
    for (int q = wave; q < rows * n_tiles; q += BP_THREADS / 64) {
      const int r = q / n_tiles;
      if ((finished && finished[row0 + r]) || beam_score(scores, row0 + r) == -INFINITY) continue;
      TileStats st;
      const float seg = beam_tile(BeamRow<T>(logits, stride, row0 + r, V), q % n_tiles, scale, lane, &st);
      if ((lane & 7) == 0) sh.maxima[q * BT_SEGS + (lane >> 3)] = seg;
      if (lane == 0) sh.stats[q] = st;
    }
    __syncthreads();
  }
  const bool cached = n <= BP_CACHED;
  float held[BP_HELD];
#pragma unroll
  for (int j = 0; j < BP_HELD; ++j) held[j] = cached && tid + j * BP_THREADS < n ? maxima[tid + j * BP_THREADS] : 0.f;

  for (int r = wave; r < rows; r += BP_THREADS / 64) {  // a wave per row: its tiles' sums
    const float s = beam_score(scores, row0 + r);
    const bool done = finished && finished[row0 + r];
    double b = -INFINITY, m = 0;
    if (done) b = s;
    else if (s != -INFINITY) {
      const TileStats st = lane < n_tiles ? stats[r * n_tiles + lane] : TileStats{0, -INFINITY};  // (64 at most)
      const float top = wave_max(st.m);
      if (top != -INFINITY) {
        const double sum = wave_sum_f64(st.m == -INFINITY ? 0.0 : st.sum * exp(((double)st.m - (double)top) * inv_temp));
        m = top;
        b = (double)s - log(sum);
      }
    }
    if (lane == 0) { sh.row[r] = make_double2(b, m); sh.done[r] = done; }
  }
  if (cached && !WHOLE) {
#pragma unroll
    for (int j = 0; j < BP_HELD; ++j)
      if (tid + j * BP_THREADS < n) sh.maxima[tid + j * BP_THREADS] = held[j];
  }
  sh.hist[tid] = 0;
  if (tid == 0) sh.count = sh.n_cand = 0;
  __syncthreads();

  Picker<T> pick{sh, logits, stride, V, n_segs, n, n_out, row0, rows, eos, inv_temp, 1.0f / (float)n_segs, cached ? sh.maxima : maxima, tid, lane, wave};
  int n_cand = pick.quick(held, cached);
  if (n_cand < 0) n_cand = pick.exactly();  // (uniform)

  const int64_t o = (int64_t)g * n_out;
  auto tell = [&](int at, u64 key, int idx) {
    if (at >= n_out) return;
    const int r = idx / V;
    out_beams[o + at] = r;
    out_tokens[o + at] = idx - r * V;
    out_scores[o + at] = (float)key_score(key);
  };
  if (n_cand <= BP_COUNTED) {  // ranks: each candidate is compared with all by a group of lanes
    int share = 64;  // lanes to a candidate
    while (share * n_cand > BP_THREADS) share >>= 1;
    const int c = tid / share;
    if (c < n_cand) {
      const u64 key = sh.cand_key[c];
      const int idx = sh.cand_idx[c];
      int at = 0;
      for (int k = tid % share; k < n_cand; k += share) {
        const u64 k2 = sh.cand_key[k];
        at += k2 > key || (k2 == key && sh.cand_idx[k] < idx);
      }
      for (int d = share >> 1; d > 0; d >>= 1) at += __shfl_xor(at, d);
      if (tid % share == 0) tell(at, key, idx);
    }
  } else {  // sorted (400 candidates: 3 us for 15)
    for (int i = n_cand + tid; i < BP_CANDS; i += BP_THREADS) { sh.cand_key[i] = 0; sh.cand_idx[i] = 0x7FFFFFFF; }
    for (int size = 2; size <= BP_CANDS; size <<= 1)
      for (int d = size >> 1; d > 0; d >>= 1) {
        __syncthreads();
        if (tid < BP_CANDS / 2) {
          const int a = (tid & ~(d - 1)) * 2 + (tid & (d - 1)), b = a + d;
          const u64 ka = sh.cand_key[a], kb = sh.cand_key[b];
          const int ia = sh.cand_idx[a], ib = sh.cand_idx[b];
          const bool b_first = kb > ka || (kb == ka && ib < ia);
          if (b_first == ((a & size) == 0)) {
            sh.cand_key[a] = kb; sh.cand_key[b] = ka;
            sh.cand_idx[a] = ib; sh.cand_idx[b] = ia;
          }
        }
      }
    __syncthreads();
    for (int i = tid; i < n_cand; i += BP_THREADS) tell(i, sh.cand_key[i], sh.cand_idx[i]);
  }
  for (int i = n_cand + tid; i < n_out; i += BP_THREADS) {
    out_beams[o + i] = -1;
    out_tokens[o + i] = -1;
    out_scores[o + i] = -INFINITY;
  }
}

template <typename T>
hipError_t beam_select(const BeamArgs& a, hipStream_t s) {
  const T* z = reinterpret_cast<const T*>(a.logits);
  const int rows = a.group_indptr[a.n_groups], n_tiles = beam_tiles_of<T>(a.V);
  const int64_t total = (int64_t)rows * n_tiles;
  TileStats* stats = reinterpret_cast<TileStats*>(a.ws);
  float* maxima = reinterpret_cast<float*>(stats + total);
  const double c = 1.4426950408889634074 * a.inv_temp;
  const float c_hi = (float)c;
  const BeamScale scale{c_hi, (float)(c - (double)c_hi), (float)(-256.0 / c)};
  int most = 0;  // rows of a group
  for (int g = 0; g < a.n_groups; ++g) most = most > a.group_indptr[g + 1] - a.group_indptr[g] ? most : a.group_indptr[g + 1] - a.group_indptr[g];
  const bool whole = most * n_tiles <= BP_WHOLE;
  if (!whole)
    beam_tiles_kernel<T><<<dim3((unsigned)((total + BT_WAVES - 1) / BT_WAVES)), dim3(64 * BT_WAVES), 0, s>>>(
        z, a.stride, a.V, n_tiles, scale, a.scores, a.finished, maxima, stats, total);
  for (int g0 = 0; g0 < a.n_groups; g0 += BEAM_GROUPS_BY_VALUE) {
    const int ng = a.n_groups - g0 < BEAM_GROUPS_BY_VALUE ? a.n_groups - g0 : BEAM_GROUPS_BY_VALUE;
    const int64_t o = (int64_t)g0 * a.n_out;
    auto go = [&](auto groups) {
      constexpr int N = sizeof(groups) / sizeof(int32_t) - 1;
      for (int g = 0; g <= ng; ++g) groups.row0[g] = a.group_indptr[g0 + g];
      auto* pick = whole ? beam_pick_kernel<T, true, N> : beam_pick_kernel<T, false, N>;
      pick<<<dim3((unsigned)ng), dim3(BP_THREADS), 0, s>>>(z, a.stride, a.V, n_tiles, a.inv_temp, scale, a.scores, a.finished, a.eos, groups, a.n_out,
                                                           maxima, stats, a.out_beams + o, a.out_tokens + o, a.out_scores + o);
    };
    if (ng <= 16) go(BeamGroups<16>{});
    else go(BeamGroups<BEAM_GROUPS_BY_VALUE>{});
  }
  return hipGetLastError();
}
}  // namespace

size_t beam_ws_doubles(int rows, int vocab) {  // per tile: its maximum and sum, and its segments' maxima; fp32 rows have the most tiles
  return (size_t)rows * beam_tiles_of<float>(vocab) * (sizeof(TileStats) / sizeof(double) + BT_SEGS / 2);
}

hipError_t launch_beam_select(const BeamArgs& a, hipStream_t s) {
  if (a.dtype == PIE_BF16) return beam_select<bf16_t>(a, s);
  if (a.dtype == PIE_F16) return beam_select<_Float16>(a, s);
  return beam_select<float>(a, s);
}

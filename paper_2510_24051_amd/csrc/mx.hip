// Microscaled rows (blocks of 32 values, a power of two as scale, elements E4M3 or E2M1): quantisation, the norm that adds the residual
// and writes them, the layout of 4-bit weights, and the products of both on the scaled matrix instructions.
#include <algorithm>
#include <iterator>
#include <type_traits>

#include "internal.h"

typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------------------------------------
// A block's scale and elements
// ---------------------------------------------------------------------------------------------
// Magnitudes are compared as the bits they are: finite < infinity < NaN.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
// floor(log2 max) - EMAX + 127, at least 0.  (A denormal maximum has exponent field 0 and a scale of 2^-127, as its logarithm asks for.)
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  constexpr int EMAX = FMT == PIE_MXFP8 ? 8 : 2;
  return most >= 0x7f800000u ? 255u : (uint32_t)max((int)(most >> 23) - EMAX, 0);
}
// 2^(127 - byte), by which elements are multiplied (exactly: what becomes denormal rounds to 0 in either format).
__device__ __forceinline__ float unscale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Four values -> four E4M3, nearest even.  (The conversion itself saturates up to 464 and then gives NaN, so it is fed at most 448.)
__device__ __forceinline__ uint32_t to_fp8x4(float a, float b, float c, float d) {
  auto sat = [](float v) { return __builtin_amdgcn_fmed3f(v, 448.f, -448.f); };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(sat(a), sat(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(sat(c), sat(d), r, true);
}
// Eight values -> eight E2M1, nearest even, saturating (the conversion does).
__device__ __forceinline__ uint32_t to_fp4x8(const float (&v)[8]) {
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], 1.f, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], 1.f, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], 1.f, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], 1.f, 3);
  return r;
}

// Eight values of a lane, four neighbouring lanes to a block: elements and, by the first of the four, the scale.
template <int FMT>
__device__ __forceinline__ void put_eight(const float (&v)[8], uint8_t* elements, uint8_t* scales, int c) {
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = max(most, magnitude(v[e]));
  most = max(most, (uint32_t)__shfl_xor((int)most, 1));
  most = max(most, (uint32_t)__shfl_xor((int)most, 2));
  const uint32_t byte = scale_byte<FMT>(most);
  const uint32_t held = byte == 255u ? 0u : ~0u;  // (a NaN block's elements are 0)
  const float un = unscale(byte);
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] = v[e] * un;
  if (FMT == PIE_MXFP8) {
    const u32x2 r = {to_fp8x4(s[0], s[1], s[2], s[3]) & held, to_fp8x4(s[4], s[5], s[6], s[7]) & held};
    *reinterpret_cast<u32x2*>(elements + c) = r;
  } else {
    *reinterpret_cast<uint32_t*>(elements + (c >> 1)) = to_fp4x8(s) & held;
  }
  if ((c & 31) == 0) scales[c >> 5] = (uint8_t)byte;
}
// The bytes behind a row's last scale, up to a multiple of four.
__device__ __forceinline__ void pad_scales(uint8_t* scales, int k) {
  for (int b = k >> 5; b & 3; ++b) scales[b] = 0;
}

// ---------------------------------------------------------------------------------------------
// Rows of plain values
// ---------------------------------------------------------------------------------------------
RowsView mx_view(const void* p, int dtype, int64_t stride) { return RowsView{p, stride, dtype}; }
static RowsView rows_behind(RowsView r, int64_t rows) {
  if (r.p) r.p = reinterpret_cast<const uint8_t*>(r.p) + rows * r.stride * (r.dtype == PIE_F32 ? 4 : 2);
  return r;
}
// (Vector accesses at addresses that are aligned to the elements only are ordinary on this chip; they touch a line more now and then.)
typedef f32x4 f32x4_at4 __attribute__((aligned(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
__device__ __forceinline__ void load8(const RowsView& r, int64_t row, int c, float (&v)[8]) {
  const int64_t at = row * r.stride + c;
  if (r.dtype == PIE_F32) {
    const float* p = reinterpret_cast<const float*>(r.p) + at;
    const f32x4 a = *reinterpret_cast<const f32x4_at4*>(p), b = *reinterpret_cast<const f32x4_at4*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
    return;
  }
  Pack16 k;
  k.u = *reinterpret_cast<const u32x4_at2*>(reinterpret_cast<const uint16_t*>(r.p) + at);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = r.dtype == PIE_BF16 ? bf16_bits_to_f32(k.s[e]) : (float)__builtin_bit_cast(_Float16, k.s[e]);
}
// Rounds v to r's type (v becomes what is stored) and, where r.p is given, stores it.  ONCE: past the caches, for results that they would not hold;
// 16-bit ones only, of which a lane stores 16 bytes in a row.
template <bool ONCE = false>
__device__ __forceinline__ void store8(const RowsView& r, int64_t row, int c, float (&v)[8]) {
  const int64_t at = row * r.stride + c;
  void* to = const_cast<void*>(r.p);
  if (r.dtype == PIE_F32) {
    if (to == nullptr) return;
    float* p = reinterpret_cast<float*>(to) + at;
    *reinterpret_cast<f32x4_at4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f32x4_at4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    return;
  }
  Pack16 k;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    k.s[e] = r.dtype == PIE_BF16 ? __builtin_bit_cast(uint16_t, f32_to_bf16(v[e])) : __builtin_bit_cast(uint16_t, (_Float16)v[e]);
    v[e] = r.dtype == PIE_BF16 ? bf16_bits_to_f32(k.s[e]) : (float)__builtin_bit_cast(_Float16, k.s[e]);
  }
  if (to == nullptr) return;
  u32x4_at2* p = reinterpret_cast<u32x4_at2*>(reinterpret_cast<uint16_t*>(to) + at);
  if (ONCE) __builtin_nontemporal_store((u32x4_at2)k.u, p);
  else *p = k.u;
}

// Eight columns of split sums, `stride` apart, in their order; up to four splits' loads go out together.
__device__ __forceinline__ void add_splits(const float* p, int64_t stride, int splits, float (&v)[8]) {
  f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
  int i = 0;
  for (; i + 4 <= splits; i += 4) {
    f32x4 x[4], y[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      x[u] = *reinterpret_cast<const f32x4*>(p + (i + u) * stride);
      y[u] = *reinterpret_cast<const f32x4*>(p + (i + u) * stride + 4);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) { a += x[u]; b += y[u]; }
  }
  if (i + 2 <= splits) {
    f32x4 x[2], y[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      x[u] = *reinterpret_cast<const f32x4*>(p + (i + u) * stride);
      y[u] = *reinterpret_cast<const f32x4*>(p + (i + u) * stride + 4);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) { a += x[u]; b += y[u]; }
    i += 2;
  }
  if (i < splits) {
    a += *reinterpret_cast<const f32x4*>(p + i * stride);
    b += *reinterpret_cast<const f32x4*>(p + i * stride + 4);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
}

// ---------------------------------------------------------------------------------------------
// Quantisation and its inverse: eight values a lane and piece, MX_PIECES pieces of a thread requested together.  Bound by HBM; back to back in a graph: 28672 x 4096
// of bf16 to 4 bits 58 us (5.1 TB/s), with one piece a thread and 64-bit divisions 75; 64 x 4096 to 8 bits 2.4 us, a launch.  Back from 4 bits 53 us, 60 where
// its stores went through the caches; both in turn, where these are then written back underneath the other, 103 and 120.  (Loads past the caches gain
// nothing here, and lose what they hold of a smaller input: 8320 x 4096 to 8 bits 21.5 us, 23.4.  fp32's halves of 32 bytes stored past them: 28.5, 52.)
// ---------------------------------------------------------------------------------------------
constexpr int MX_PIECES = 4;
// Row and column of piece i of rows of k values; SMALL: pieces fit 32 bits, where a division is a few instructions.
template <bool SMALL>
__device__ __forceinline__ void piece_at(int64_t i, int per_row, int64_t& row, int& c) {
  if (SMALL) {
    const uint32_t r = (uint32_t)i / (uint32_t)per_row;
    row = r;
    c = (int)((uint32_t)i - r * (uint32_t)per_row) * 8;
  } else {
    row = i / per_row;
    c = (int)(i - row * per_row) * 8;
  }
}

template <int FMT, bool SMALL, int P>
__global__ __launch_bounds__(256) void mx_quantise_kernel(RowsView x, int64_t pieces, int k, MxRowsView out) {
  const int64_t first = (int64_t)blockIdx.x * (256 * P) + threadIdx.x;
  float v[P][8];
  int64_t row[P];
  int c[P];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (first + j * 256 >= pieces) break;  // (a row's pieces are a multiple of four: the lanes of a block stay together)
    piece_at<SMALL>(first + j * 256, k >> 3, row[j], c[j]);
    load8(x, row[j], c[j], v[j]);
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (first + j * 256 >= pieces) break;
    uint8_t* scales = out.scales + row[j] * out.scale_bytes;
    put_eight<FMT>(v[j], out.elements + row[j] * out.row_bytes, scales, c[j]);
    if (c[j] == 0) pad_scales(scales, k);
  }
}

template <bool SMALL, int P>
__global__ __launch_bounds__(256) void mx_dequantise_kernel(MxRowsView a, int fmt, int64_t pieces, int k, RowsView out) {
  const int64_t first = (int64_t)blockIdx.x * (256 * P) + threadIdx.x;
  int64_t row[P];
  int c[P];
  u32x2 e[P];
  uint32_t byte[P];
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (first + j * 256 >= pieces) break;
    piece_at<SMALL>(first + j * 256, k >> 3, row[j], c[j]);
    byte[j] = a.scales[row[j] * a.scale_bytes + (c[j] >> 5)];
    const uint8_t* p = a.elements + row[j] * a.row_bytes;
    if (fmt == PIE_MXFP8) e[j] = *reinterpret_cast<const u32x2*>(p + c[j]);
    else e[j][0] = *reinterpret_cast<const uint32_t*>(p + (c[j] >> 1));
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    if (first + j * 256 >= pieces) break;
    // 2^(byte - 127): a denormal for byte 0
    const float scale = byte[j] == 255u ? __uint_as_float(0x7fc00000u) : byte[j] == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(byte[j] << 23);
    float v[8];
    if (fmt == PIE_MXFP8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)e[j][i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)e[j][i], true);
        v[4 * i] = lo[0] * scale; v[4 * i + 1] = lo[1] * scale; v[4 * i + 2] = hi[0] * scale; v[4 * i + 3] = hi[1] * scale;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t n = e[j][0] >> (4 * i), m = n & 7;  // 0, 1/2, then 1.f * 2^(e - 1): the exponent and fraction bits moved into place
        const float f = m < 2 ? 0.5f * (float)m : __uint_as_float((m << 22) + (126u << 23));
        v[i] = (n & 8 ? -f : f) * scale;
      }
    }
    store8<(P > 1)>(out, row[j], c[j], v);
  }
}

static dim3 pieces_grid(int64_t pieces) { return dim3((unsigned)((pieces + 255) / 256)); }

// One piece a thread while that leaves fewer than eight workgroups to a compute unit.
template <typename F>
static void with_pieces(int64_t pieces, F&& go) {
  using std::integral_constant;
  if (pieces < 256 * 2048) go(std::true_type{}, integral_constant<int, 1>{});
  else if (pieces < INT32_MAX) go(std::true_type{}, integral_constant<int, MX_PIECES>{});
  else go(std::false_type{}, integral_constant<int, MX_PIECES>{});
}

hipError_t launch_mx_quantise(const RowsView& x, int rows, int k, int format, const MxRowsView& out, hipStream_t s) {
  const int64_t pieces = (int64_t)rows * (k / 8);
  if (pieces <= 0) return hipSuccess;
  with_pieces(pieces, [&](auto small_c, auto p_c) {
    constexpr bool SMALL = decltype(small_c)::value;
    constexpr int P = decltype(p_c)::value;
    const dim3 grid = pieces_grid((pieces + P - 1) / P);
    if (format == PIE_MXFP8) mx_quantise_kernel<PIE_MXFP8, SMALL, P><<<grid, dim3(256), 0, s>>>(x, pieces, k, out);
    else mx_quantise_kernel<PIE_MXFP4, SMALL, P><<<grid, dim3(256), 0, s>>>(x, pieces, k, out);
  });
  return hipGetLastError();
}

hipError_t launch_mx_dequantise(const MxRowsView& a, int format, int rows, int k, const RowsView& out, hipStream_t s) {
  const int64_t pieces = (int64_t)rows * (k / 8);
  if (pieces <= 0) return hipSuccess;
  with_pieces(pieces, [&](auto small_c, auto p_c) {
    constexpr bool SMALL = decltype(small_c)::value;
    constexpr int P = decltype(p_c)::value;
    mx_dequantise_kernel<SMALL, P><<<pieces_grid((pieces + P - 1) / P), dim3(256), 0, s>>>(a, format, pieces, k, out);
  });
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Norm: a workgroup per row, eight columns a thread (as rmsnorm_row in elementwise.hip).  Bound by HBM for many rows, by latency for few.
// An element that rounds the other way is off by a step, an eighth of it, so the normalised values are off by their last rounding to fp32 alone:
// squares are summed in 64 bits, and gain over root enters as a pair of fp32.  (8320 x 4096 of bf16 30.0 us; the first eight squares of a thread in
// fp32 29.6, and rows that its columns dominate two units off; root and quotient in 64 bits by every wave 42: the root is the fp32 reciprocal one and a
// step of Newton's method in 64 bits, good to 2^-44.  Several rows to a workgroup, the next one's values requested ahead, gained nothing.  8320 x 4096 of
// fp32 with the residual's addition, 444 MB: 78 us, 5.7 TB/s; one row 3.1 us.  All back to back in a graph.)
// ---------------------------------------------------------------------------------------------
template <int FMT, int THREADS, bool SUMS>
__global__ __launch_bounds__(THREADS) void mx_norm_kernel(MxNormArgs a, double inv_k, int k, MxRowsView out) {
  __shared__ double red[THREADS / 64];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, c = tid * 8;
  const bool in = c < k;  // (k is a multiple of 32: the four lanes of a block go the same way)
  float v[8];
  double ss = 0.0;
  Pack16 g;
  if (in) {
    g.u = *reinterpret_cast<const u32x4_at2*>(reinterpret_cast<const uint16_t*>(a.gain) + c);
    load8(a.x, a.ids ? a.ids[row] : row, c, v);
    if (a.delta.p) {
      float d[8];
      load8(a.delta, row, c, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += d[e];
    }
    if constexpr (SUMS) {  // partial sums of the product before, in their order, then what they are added to
      float d[8];
      add_splits(a.part + row * a.part_stride + c, a.split_stride, a.splits, d);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += d[e];
    }
    store8(a.h, row, c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fma((double)v[e], (double)v[e], ss);
  }
  ss = wave_sum_f64(ss);
  if constexpr (THREADS > 64) {
    if ((tid & 63) == 0) red[tid >> 6] = ss;
    __syncthreads();
    ss = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) ss += red[w];
  }
  const double m = ss * inv_k + (double)a.eps;
  if (in) {
    if (m > 1e-30 && m < 1e30) {  // (uniform)
      double r = (double)__builtin_amdgcn_rsqf((float)m);
      r = r * (1.5 - 0.5 * m * r * r);
      const float rh = (float)r, rl = (float)(r - (double)rh);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float ge = bf16_to_f32(g.h[e]), hi = rh * ge, lo = __builtin_fmaf(rh, ge, -hi) + rl * ge;
        v[e] = __builtin_fmaf(v[e], hi, v[e] * lo);
      }
    } else {  // a root that 32 bits hold as a denormal or not at all; an infinity or a NaN in the row
      const double r = m == INFINITY ? 0.0 : 1.0 / sqrt(m);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)((double)v[e] * (r * (double)bf16_to_f32(g.h[e])));
    }
    uint8_t* scales = out.scales + row * out.scale_bytes;
    put_eight<FMT>(v, out.elements + row * out.row_bytes, scales, c);
    if (c == 0) pad_scales(scales, k);
  }
}

hipError_t launch_mx_norm(const MxNormArgs& a, int rows, int k, int format, const MxRowsView& out, hipStream_t s) {
  if (rows <= 0) return hipSuccess;
  if (k > 8192) return hipErrorInvalidValue;
  auto go = [&](auto threads_c) {
    constexpr int T = decltype(threads_c)::value;
    if (a.splits > 0) {  // (a layer's)
      mx_norm_kernel<PIE_MXFP8, T, true><<<dim3(rows), dim3(T), 0, s>>>(a, 1.0 / k, k, out);
      return hipGetLastError();
    }
    constexpr int MOST = 1 << 21;  // rows of a launch, which may have fewer than 2^32 threads
    MxNormArgs p = a;
    MxRowsView o = out;
    for (int left = rows; left > 0; left -= MOST) {
      const dim3 grid(std::min(left, MOST));
      if (format == PIE_MXFP8) mx_norm_kernel<PIE_MXFP8, T, false><<<grid, dim3(T), 0, s>>>(p, 1.0 / k, k, o);
      else mx_norm_kernel<PIE_MXFP4, T, false><<<grid, dim3(T), 0, s>>>(p, 1.0 / k, k, o);
      p.x = rows_behind(p.x, MOST); p.delta = rows_behind(p.delta, MOST); p.h = rows_behind(p.h, MOST);
      if (p.ids) p.ids += MOST;
      o.elements += MOST * o.row_bytes;
      o.scales += MOST * o.scale_bytes;
    }
    return hipGetLastError();
  };
  using std::integral_constant;
  if (k <= 512) return go(integral_constant<int, 64>{});
  if (k <= 2048) return go(integral_constant<int, 256>{});
  if (k <= 4096) return go(integral_constant<int, 512>{});
  return go(integral_constant<int, 1024>{});
}

// ---------------------------------------------------------------------------------------------
// Weights: tiles of 32 rows x 64 inputs, 1 KiB each, stored [N/32][K/64]; lane l = h * 32 + n of a tile holds the 32 elements of row n
// and block h (16 bytes): the operand of mfma_scale 32x32x64.  Their scales: [N/32][K/256][64] dwords, byte t of lane l's dword being the
// scale of its block in tile 4 q + t: one load for four steps, of which the instruction picks the byte.  What is behind the last row
// or block is 0.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void mx_pack_kernel(MxRowsView src, int rows, int k, int first, int interleave, MxTiles w, int64_t from) {
  const int64_t i = from + (int64_t)blockIdx.x * 256 + threadIdx.x;  // one per (32-row block of the part, k step, lane)
  const int KT = w.KT;
  const int64_t total = (int64_t)((rows + 31) / 32) * KT * 64;
  if (i >= total) return;
  const int lane = (int)(i & 63), kt = (int)((i >> 6) % KT), sb = (int)((i >> 6) / KT);
  const int r = sb * 32 + (lane & 31), b = kt * 2 + (lane >> 5);
  if (r >= rows) return;
  const int n = interleave ? (2 * sb + first) * 32 + (lane & 31) : first + r;  // row of the stacked (or interleaved) weight
  const int nb = n >> 5, l = (lane & 32) + (n & 31);
  const bool real = b < k / 32;
  u32x4 e = {0, 0, 0, 0};
  if (real) e = *reinterpret_cast<const u32x4*>(src.elements + r * src.row_bytes + b * 16);
  *reinterpret_cast<u32x4*>(w.data + (((int64_t)nb * KT + kt) * 64 + l) * 16) = e;
  reinterpret_cast<uint8_t*>(w.scales)[(((int64_t)nb * w.KQ + (kt >> 2)) * 64 + l) * 4 + (kt & 3)] = real ? src.scales[r * src.scale_bytes + b] : 0;
}

hipError_t launch_mx_pack(const MxRowsView& src, int rows, int k, int first, int interleave, const MxPacked& w, hipStream_t s) {
  const int64_t total = (int64_t)((rows + 31) / 32) * w.KT * 64;
  constexpr int64_t MOST = 1ll << 31;  // (a launch has fewer than 2^32 threads)
  for (int64_t from = 0; from < total; from += MOST)
    mx_pack_kernel<<<pieces_grid(std::min(total - from, MOST)), dim3(256), 0, s>>>(src, rows, k, first, interleave, w, from);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Epilogues.  An accumulator tile has a token per lane (l % 32) and weight rows in its registers: v is row (v / 4) * 8 + (l / 32) * 4 + v % 4
// of the 32, so a lane's four groups are four consecutive columns of its token's row.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {  // lower lanes: a, a of lane + 32; upper: b of lane - 32, b
  const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
  a = r[0];
  b = r[1];
}

// Gate and up columns [n0, n0 + 32) of token m (n0: the gate block's packed column) -> 32 columns of activations.
template <int FMT>
__device__ __forceinline__ void mx_gated_columns(const MxEpi& e, const f32x16& gate, const f32x16& up, int64_t m, int M, int n0, int lane) {
  const int h = lane >> 5;
  float v[16];
  uint32_t most = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    v[i] = silu_f(gate[i]) * up[i];
    most = max(most, magnitude(v[i]));
  }
  const auto both = __builtin_amdgcn_permlane32_swap(most, most, false, false);
  const uint32_t byte = scale_byte<FMT>(max((uint32_t)both[0], (uint32_t)both[1]));
  const uint32_t held = byte == 255u ? 0u : ~0u;
  const float un = unscale(byte);
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] *= un;
  const int c = n0 >> 1;
  uint8_t* row = reinterpret_cast<uint8_t*>(e.out) + m * e.ldo;
  if (FMT == PIE_MXFP8) {
    uint32_t g[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = to_fp8x4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]) & held;
    swap_halves(g[0], g[2]);
    swap_halves(g[1], g[3]);
    if (m < M) *reinterpret_cast<u32x4*>(row + c + h * 16) = u32x4{g[0], g[2], g[1], g[3]};
  } else {
    const float a[8] = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]}, b[8] = {v[8], v[9], v[10], v[11], v[12], v[13], v[14], v[15]};
    uint32_t p = to_fp4x8(a) & held, q = to_fp4x8(b) & held;
    swap_halves(p, q);
    if (m < M) *reinterpret_cast<u32x2*>(row + (c >> 1) + h * 8) = u32x2{(p & 0xffffu) | (q << 16), (p >> 16) | (q & 0xffff0000u)};
  }
  if (m < M && h == 0) {
    uint8_t* scales = e.scales + m * e.lds;
    scales[c >> 5] = (uint8_t)byte;
    if (c + 32 >= e.N) pad_scales(scales, e.N);
  }
}
__device__ __forceinline__ void mx_gated_epilogue(const MxEpi& e, const f32x16& gate, const f32x16& up, int64_t m, int M, int n0, int lane) {
  if (e.mode == MX_SWIGLU8) mx_gated_columns<PIE_MXFP8>(e, gate, up, m, M, n0, lane);
  else mx_gated_columns<PIE_MXFP4>(e, gate, up, m, M, n0, lane);
}

// Columns [n0, n0 + 32) of token m of a product that is not gated: a residual or none, then bf16 or fp32 (uniform; rows of residuals are whole blocks).
__device__ __forceinline__ void mx_plain_epilogue(const MxEpi& e, const f32x16& acc, int64_t m, int M, int n0, int lane) {
  const int h = lane >> 5;
  if (m >= M) return;  // (lanes l and l + 32 have the same token)
  float y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = acc[i];
  if (e.mode == MX_RESID_EMBED && !e.resid) {
    const bf16_t* r = e.embeds + (int64_t)e.ids[m] * e.H + n0 + h * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16x4 v = *reinterpret_cast<const bf16x4*>(r + 8 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[4 * i + j] += bf16_to_f32(v[j]);
    }
  } else if (e.mode == MX_RESID_EMBED || e.mode == MX_RESID_OUT) {
    const float* r = e.resid + m * e.H + n0 + h * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 v = *reinterpret_cast<const f32x4*>(r + 8 * i);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[4 * i + j] += v[j];
    }
  }
  const bool to_embed = e.mode == MX_RESID_OUT && !e.out, whole = n0 + 32 <= e.N;
  if (e.mode == MX_BF16 || to_embed) {
    const int64_t id = to_embed ? e.ids[m] : m;
    if (id < 0) return;
    uint16_t* row = reinterpret_cast<uint16_t*>(to_embed ? e.embeds : e.out) + id * (to_embed ? e.H : e.ldo) + n0;
    uint32_t g[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bf16x2 b = {f32_to_bf16(y[2 * i]), f32_to_bf16(y[2 * i + 1])};
      g[i] = __builtin_bit_cast(uint32_t, b);
    }
    if (whole) {
#pragma unroll
      for (int i = 0; i < 4; ++i) swap_halves(g[i], g[i + 4]);
      *reinterpret_cast<u32x4_at2*>(row + h * 16) = u32x4{g[0], g[1], g[4], g[5]};
      *reinterpret_cast<u32x4_at2*>(row + h * 16 + 8) = u32x4{g[2], g[3], g[6], g[7]};
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int n = (i >> 2) * 8 + h * 4 + (i & 3);
        if (n0 + n < e.N) row[n] = (uint16_t)(g[i >> 1] >> (16 * (i & 1)));
      }
    }
  } else {
    float* row = reinterpret_cast<float*>(e.out) + m * e.ldo + n0;
    if (whole) {
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4_at4*>(row + 8 * i + h * 4) = f32x4{y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]};
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int n = (i >> 2) * 8 + h * 4 + (i & 3);
        if (n0 + n < e.N) row[n] = y[i];
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Products.  D[weight row][token] = W x A^T on v_mfma_scale_f32_32x32x64_f8f6f4: a lane of the weight operand has 32 elements of one block; a
// lane of an MXFP8 operand has bytes [16 h, 16 h + 16) and [32 + 16 h, 48 + 16 h) of its row's 64, and in either case the scale of block
// h of its row.  Sums are fp32, and whole in between: the instruction adds eight neighbouring products aligned to the largest sum of two operands'
// exponents, E, and drops what is below 2^(E - 13) (found with all pairs of elements, and eight at a time at random).  Products of two E2M1 elements are multiples of 2^-2
// with E at most 4 and lose nothing.  Those of E4M3 with E2M1 are multiples of 2^-10 with E up to 10, so MXFP8 rows are multiplied in two parts: elements of at
// least 2, multiples of 2^-2, whose products are multiples of 2^-3 = 2^(10 - 13), and the smaller ones, whose products have E at most 2.  Each sum of eight is
// then exact, and is added to the fp32 sum.  That costs a second instruction: 8192 rows of 14336 onto 4096 take 600 us, with one 350, at sums that are 1.5e-5 of their
// size off where channels differ as a model's do; the parts themselves take 5 to 10% of it.  (bf16 operands have the rate of two such instructions.)
// Up to 16 rows have their parts side by side instead, as columns c and 16 + c of one instruction, added behind the contraction: SwiGLU of one row, 4096 onto
// 2 x 14336, 18.2 us for 19.1, 16 rows of 14336 onto 4096 14.9 for 15.4.
// ---------------------------------------------------------------------------------------------
// ---------------------------------------------------------------------------------------------
// Tiles of 256 tokens x 256 weight rows: many rows, bound by the matrix cores.
// Eight waves, two along the tokens and four along the weight rows, of 4 x 2 accumulator tiles each.  Activations go to LDS by direct copies, 128 bytes of
// a row (SK steps of 64) a stage, four stages, and every fourth stage the scales of four; weights go from memory to registers, each set refilled for the next
// stage right behind the instructions that used it (as in gemm_large_async_kernel, whose order of requests, waits and barriers this is).
// The 16-byte pieces of a row are swizzled by its number: piece c of row r is stored at c ^ (r / 2 % 8), so that the 32 rows of an operand
// read from all banks.  What is behind K is read from the row's first piece instead: its weights are 0, and so is its scale.
// 8192 rows of 14336 onto 4096 take 620 us with 8-bit rows, on zeros, which the power limit does not hold back, 507; 4-bit rows 217 and 164.  SwiGLU of 4096 onto
// 2 x 14336: 1290 and 1080, 510 and 400.
// A row's scales of a stage are 4 or 8 bytes of a cache line of their own, and the lines that a copy touches are what it costs: with the scales copied every
// stage 8192 rows of 14336 onto 4096 took 370 us, with four stages' at a time 342, when 8-bit rows were multiplied in one part (on zeros 295 and 267).
// (Weights requested up to two stages earlier, copies two or three stages ahead: the same.)
// ---------------------------------------------------------------------------------------------
constexpr int MX_TM = 256, MX_TN = 256;

// Byte offset of a tile's row for its copies.  Rows past the matrix are out of the descriptor's range: nothing is fetched for them, and
// what their lanes compute is not stored.
__device__ __forceinline__ int mx_row_offset(int r, int rows, int64_t stride) { return r < rows ? (int)(r * stride) : 0x7f000000; }
#if __HIP_DEVICE_COMPILE__
// One step of a stage: step S takes byte S of the weights' scales, and byte 0 or 2 of the rows'.
template <int FMT, int S>
__device__ __forceinline__ f32x16 mx_mfma(const i32x8& w, const i32x8& a, const f32x16& c, int ws, int as) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w, a, c, 4, FMT == PIE_MXFP8 ? 0 : 4, S, ws, S % 2 * 2, as);
}
// Ones in the bytes of E4M3 codes whose value is at least 2 (bit 6).
__device__ __forceinline__ uint32_t mx_large(uint32_t codes) { return __builtin_amdgcn_perm(codes << 1, codes << 9, 0x0B090A08u); }
// acc[first + i][j] += weights j times rows i of a unit, step s of a stage (known at compile time: the bytes of the scales are part of the instruction).
// flip: with PAIRS, ones in the lanes that have the smaller elements' turn.
template <int FMT, bool PAIRS, int UI, int NJ, int MI, int SD>
__device__ __forceinline__ void mx_multiply(f32x16 (&acc)[MI][NJ], const u32x4 (&w)[NJ], const i32x8 (&a)[UI], int first, int s, const int (&xs)[NJ], const int (&sc)[SD][MI],
                                            uint32_t flip) {
  constexpr int PARTS = FMT == PIE_MXFP8 && !PAIRS ? 2 : 1;
#pragma unroll
  for (int i = 0; i < UI; ++i) {
    i32x8 part[2] = {a[i], a[i]};
    if constexpr (FMT == PIE_MXFP8) {
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        const uint32_t u = (uint32_t)a[i][d], large = mx_large(u);
        part[0][d] = (int)(u & (PAIRS ? large ^ flip : large));
        part[1][d] = (int)(u & ~large);
      }
    }
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const i32x8 wo = {(int)w[j][0], (int)w[j][1], (int)w[j][2], (int)w[j][3], 0, 0, 0, 0};
        f32x16& c = acc[first + i][j];
        const int as = sc[s / 2][first + i];
        if (s == 0) c = mx_mfma<FMT, 0>(wo, part[p], c, xs[j], as);
        if (s == 1) c = mx_mfma<FMT, 1>(wo, part[p], c, xs[j], as);
        if (s == 2) c = mx_mfma<FMT, 2>(wo, part[p], c, xs[j], as);
        if (s == 3) c = mx_mfma<FMT, 3>(wo, part[p], c, xs[j], as);
      }
  }
}
#endif
#if __HIP_DEVICE_COMPILE__
// Copy piece p of a tile of rows: 1 KiB, rows 8 p .. 8 p + 7, lane -> row lane / 8 of them, stored piece lane % 8.  Byte of its row's 128 that a
// lane brings:
__device__ __forceinline__ int mx_piece_byte(int p, int lane) { return (((lane & 7) ^ (lane >> 4)) * 16) ^ (p & 1) * 64; }
// How far the bytes of the last stage that are behind a row's end are moved, for pieces of p's parity: to the stage's first bytes.
__device__ __forceinline__ int mx_piece_back(int p, int lane, int row_len) {
  const int byte = mx_piece_byte(p, lane), held = row_len & 127;
  return held && byte >= held ? byte : 0;
}
// From stage k to `to`; off: byte offset of the lane's row plus mx_piece_byte.  (Without a branch: one around the last stage's copies made the compiler
// wait for weights at every step: 9% of 8192 rows of 14336 onto 4096, multiplied in one part.)
__device__ __forceinline__ void mx_copy_piece(__amdgpu_buffer_rsrc_t rsrc, int off, uint8_t* to, int k, int back, bool last) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)to, 16, off - (back & (last ? -1 : 0)), k * 128, 0, 0);
}
#endif

template <bool GATED, int FMT>
__global__ __launch_bounds__(512, 2) void mx_tiles_kernel(MxRowsView a, int M, MxTiles w, MxEpi epi, int tiles_m, int tiles_n) {
  constexpr int SK = FMT == PIE_MXFP8 ? 2 : 4;  // steps of 64 a stage
  constexpr int SD = SK / 2;                    // dwords of scales a row and stage
  constexpr int MI = 4, NJ = 2;
  [[maybe_unused]] constexpr int UI = 2, UN = MI / UI;  // accumulator blocks whose operands are read at a time, and such units of a step
  [[maybe_unused]] __shared__ __align__(16) uint8_t As0[MX_TM * 128], As1[MX_TM * 128], As2[MX_TM * 128], As3[MX_TM * 128];
  [[maybe_unused]] __shared__ __align__(16) uint8_t Ss[2][MX_TM * SD * 16], spare[SD == 1 ? 1024 : 16];  // scales of four stages: 16 SD bytes a row
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  [[maybe_unused]] const int h = lane >> 5;
  const int wm = wave >> 2, wn = wave & 3;
  int tm, tn;
  tile_at(xcd_range(blockIdx.x, tiles_m, tiles_n), tiles_m, tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * MX_TM;
  const int nb0 = tn * (MX_TN / 32) + wn * NJ;
  f32x16 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  {
#if __HIP_DEVICE_COMPILE__  // (buffer descriptors: see gemm_large_async_kernel)
    constexpr int RSRC_FLAGS = 0x00020000;
    const int rows = (int)(M - m0 < MX_TM ? M - m0 : MX_TM);
    const int row_len = FMT == PIE_MXFP8 ? w.K : w.K / 2, NS = (row_len + 127) / 128;
    const __amdgpu_buffer_rsrc_t rsrc_a = __builtin_amdgcn_make_buffer_rsrc(a.elements + m0 * a.row_bytes, 0, (int)((rows - 1) * a.row_bytes) + row_len, RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t rsrc_s =
        __builtin_amdgcn_make_buffer_rsrc(a.scales + m0 * a.scale_bytes, 0, (int)((rows - 1) * a.scale_bytes) + (w.K / 32 + 3) / 4 * 4, RSRC_FLAGS);
    // blocks past the matrix are out of the descriptors' range: nothing is fetched for them, and their results are dropped
    // (readfirstlane: the compiler takes their number for a lane's own, and rebuilt the descriptors at every load: 7% of the kernel's time)
    const int held_w = __builtin_amdgcn_readfirstlane(max(0, min(NJ, w.NB - nb0))), nbw = held_w > 0 ? nb0 : 0;
    const __amdgpu_buffer_rsrc_t rsrc_w = __builtin_amdgcn_make_buffer_rsrc(w.data + (int64_t)nbw * w.KT * 1024, 0, held_w * w.KT * 1024, RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t rsrc_x = __builtin_amdgcn_make_buffer_rsrc(w.scales + (int64_t)nbw * w.KQ * 64, 0, held_w * w.KQ * 256, RSRC_FLAGS);
    const int back[2] = {mx_piece_back(0, lane, row_len), mx_piece_back(1, lane, row_len)};
    int aoff[MI];  // (a wave copies pieces wave * MI .. wave * MI + MI - 1)
#pragma unroll
    for (int jj = 0; jj < MI; ++jj)
      aoff[jj] = mx_row_offset((wave * MI + jj) * 8 + (lane >> 3), rows, a.row_bytes) + mx_piece_byte(jj, lane);
    // scales: SD lanes a row; with MXFP8 four waves copy them all, the others nothing, elsewhere (so that all count the same copies)
    const bool scopies = wave < 4 * SD;
    const int soff = scopies ? mx_row_offset(wave * (64 / SD) + lane / SD, rows, a.scale_bytes) + lane % SD * 16 : 0x7f000000;
    int woff[NJ], xoff[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      woff[j] = j * w.KT * 1024 + lane * 16;
      xoff[j] = j * w.KQ * 256 + lane * 4;
    }
    // scales of stages 4 g .. 4 g + 3 (behind the last one of a row: others, or out of range, which is checked by the dword; masked when they are read)
    auto issue_s = [&](int g) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_s, (__attribute__((address_space(3))) void*)(scopies ? &Ss[g & 1][wave * 1024] : spare), 16, soff, g * SD * 16, 0, 0);
    };
    auto issue_a = [&](uint8_t* As, int kt) {
      const int k = kt < NS ? kt : NS - 1;  // past the end: a copy nobody reads, so that the wait counts stay uniform
#pragma unroll
      for (int jj = 0; jj < MI; ++jj) mx_copy_piece(rsrc_a, aoff[jj], As + (wave * MI + jj) * 1024, k, back[jj & 1], k == NS - 1);
    };
    u32x4 wreg[SK][NJ];
    int xreg[2][NJ];  // the weights' scales, a dword for four steps
    auto load_w = [&](int kt, int s) {
      const int k = kt < NS ? kt : NS - 1;
#pragma unroll
      for (int j = 0; j < NJ; ++j) wreg[s][j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc_w, woff[j], (k * SK + s) * 1024, 0);
    };
    auto load_x = [&](int kt, int slot) {
      const int k = kt < NS ? kt : NS - 1;
#pragma unroll
      for (int j = 0; j < NJ; ++j) xreg[slot][j] = __builtin_amdgcn_raw_buffer_load_b32(rsrc_x, xoff[j], (k * SK >> 2) * 256, 0);
    };
    auto load_a = [&](const uint8_t* As, int unit, i32x8 (&af)[UI]) {
      const int s = unit / UN;
#pragma unroll
      for (int i = 0; i < UI; ++i) {
        const int r = wm * (MX_TM / 2) + (unit % UN * UI + i) * 32 + (lane & 31), z = (r >> 1) & 7;
        const uint8_t* row = As + r * 128;
        if (FMT == PIE_MXFP8) {
          const u32x4 lo = *reinterpret_cast<const u32x4*>(row + (((s * 4 + h) ^ z) << 4)), hi = *reinterpret_cast<const u32x4*>(row + (((s * 4 + 2 + h) ^ z) << 4));
          af[i] = i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
        } else {
          const u32x4 lo = *reinterpret_cast<const u32x4*>(row + (((s * 2 + h) ^ z) << 4));
          af[i] = i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], 0, 0, 0, 0};
        }
      }
    };
    auto load_s = [&](int kt, int at, int (&sc)[SD][MI]) {  // (at: kt % 4)
      const uint32_t* group = reinterpret_cast<const uint32_t*>(&Ss[(kt >> 2) & 1][(wm * (MX_TM / 2) + (lane & 31)) * SD * 16]);
#pragma unroll
      for (int d = 0; d < SD; ++d) {
        const int left = w.K / 32 - (kt * SD + d) * 4;  // blocks from here on
        const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
        for (int i = 0; i < MI; ++i) sc[d][i] = (int)((group[i * 32 * SD * 4 + at * SD + d] & mask) >> (8 * h));
      }
    };
    i32x8 af[2][UI];
    int sc[SD][MI];
    auto step = [&](auto at_c, const uint8_t* Acur, const uint8_t* Anext, uint8_t* Afill, int kt) {
      constexpr int AT = decltype(at_c)::value;  // kt % 4
      constexpr int GROUP = (AT + 3) % 4 == 0;
      if constexpr (GROUP) issue_s((kt + 3) >> 2);
      issue_a(Afill, kt + 3);
      __builtin_amdgcn_sched_barrier(0);
      load_x(kt + 1, 1);
      const int shift = FMT == PIE_MXFP8 ? (kt & 1) * 16 : 0;
      int xs[NJ], nsc[SD][MI];
#pragma unroll
      for (int j = 0; j < NJ; ++j) xs[j] = (int)((uint32_t)xreg[0][j] >> shift);
#pragma unroll
      for (int u = 0; u < SK * UN; ++u) {
        const int s = u / UN;
        if (u + 1 < SK * UN) {
          load_a(Acur, u + 1, af[(u + 1) & 1]);
        } else {
          PIE_S_WAIT_LGKMCNT0();  // this wave's last reads of Acur have returned
          // all but the copies, scales and weights requested in this stage: the copies of stage kt + 1 are older, and of the others all is needed by now
          PIE_S_WAIT_VMCNT(GROUP + MI + NJ + (SK - 1) * NJ);
          wg_barrier();
          load_a(Anext, 0, af[(u + 1) & 1]);
          load_s(kt + 1, (AT + 1) % 4, nsc);
        }
        mx_multiply<FMT, false>(acc, wreg[s], af[u & 1], u % UN * UI, s, xs, sc, 0);
        if (u % UN == UN - 1) load_w(kt + 1, s);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) xreg[0][j] = xreg[1][j];
#pragma unroll
      for (int d = 0; d < SD; ++d)
#pragma unroll
        for (int i = 0; i < MI; ++i) sc[d][i] = nsc[d][i];
    };
    issue_s(0);
    issue_a(As0, 0);
    issue_a(As1, 1);
    issue_a(As2, 2);
    __builtin_amdgcn_sched_barrier(0);
    load_x(0, 0);
#pragma unroll
    for (int s = 0; s < SK; ++s) load_w(0, s);
    __builtin_amdgcn_sched_barrier(0);
    PIE_S_WAIT_VMCNT(2 * MI + NJ + SK * NJ);  // the first stage has arrived
    wg_barrier();
    load_a(As0, 0, af[0]);
    load_s(0, 0, sc);
    using std::integral_constant;
    for (int kt = 0;;) {
      step(integral_constant<int, 0>{}, As0, As1, As3, kt);
      if (++kt >= NS) break;
      step(integral_constant<int, 1>{}, As1, As2, As0, kt);
      if (++kt >= NS) break;
      step(integral_constant<int, 2>{}, As2, As3, As1, kt);
      if (++kt >= NS) break;
      step(integral_constant<int, 3>{}, As3, As0, As2, kt);
      if (++kt >= NS) break;
    }
    PIE_S_WAIT_VMCNT(0);  // the surplus copies of the last steps land before the workgroup gives up its LDS
#endif
  }
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int64_t m = m0 + wm * (MX_TM / 2) + i * 32 + (lane & 31);
    if constexpr (GATED) {
      if (nb0 < w.NB) mx_gated_epilogue(epi, acc[i][0], acc[i][1], m, M, nb0 * 32, lane);
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        if (nb0 + j < w.NB) mx_plain_epilogue(epi, acc[i][j], m, M, (nb0 + j) * 32, lane);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Few rows: bound by the stream of weights, or by its latency.
// Eight waves; KS slices of the contraction (or parts of them, where the product is split over workgroups as well) with 8 / KS waves each, a
// wave with MB x NJ accumulator tiles: 32 weight rows (SwiGLU: a gate and an up block) by 32 MB tokens.  Each wave keeps SW stages of
// weights in registers (stages as in mx_tiles_kernel, requested non-temporally), each slice SA stages of its activations in LDS, and the
// scales of SG stages at a time (one stage's by themselves cost as much as its activations: 333 rows of 4 bits, 4096 onto 6144, 14.8 us for 13.4).  A slice's
// stages are NS p / parts .. NS (p + 1) / parts; all walk as many as the longest has, the others doing nothing in the last.  The slices'
// sums meet in LDS, in their order.
// ---------------------------------------------------------------------------------------------
constexpr int mx_stages_a(int mb, int ks) { return mb * ks <= 8 ? 4 : mb * ks <= 12 ? 3 : 2; }
// weights in flight: 64 to 128 KiB of a compute unit, less where the registers hold accumulators
constexpr int mx_stages_w(int fmt, int nj, int mb, int ks) {
  const int room = mb == 1 ? 128 : mb == 2 ? 64 : 48, stage = (fmt == PIE_MXFP8 ? 8 : 16) * nj;  // registers
  const int fit = room / stage;
  return mx_stages_a(mb, ks) == 3 ? (fit >= 6 ? 6 : fit >= 3 ? 3 : fit >= 2 ? 2 : 1) : fit >= 8 ? 8 : fit >= 4 ? 4 : fit >= 2 ? 2 : 1;
}

template <bool GATED, int FMT, int MB, int KS, int NJ, bool PAIRS>
__global__ __launch_bounds__(512, 2) void mx_stream_kernel(MxRowsView a, int M, MxTiles w, MxEpi epi, int tiles_m, int tiles_n, int splits, float* part) {
  static_assert(!GATED || NJ == 2, "a gate and an up block");
  static_assert(!PAIRS || (MB == 1 && FMT == PIE_MXFP8), "two lanes' columns to a row");
  constexpr int WN = 8 / KS, BM = 32 * MB;
  [[maybe_unused]] constexpr int SK = FMT == PIE_MXFP8 ? 2 : 4, SD = SK / 2;
  constexpr int SA = mx_stages_a(MB, KS);
  [[maybe_unused]] constexpr int SW = mx_stages_w(FMT, NJ, MB, KS), RS = SA > SW ? SA : SW;  // (RS: steps of a round of both rings)
  [[maybe_unused]] constexpr int SG = SA == 4 ? 4 : SA == 3 && SD == 1 ? 3 : 1, SL = SG == 1 ? 4 : 16, SROW = SD * SL;  // stages whose scales are copied together (as LDS has room), a lane's bytes of a copy, a row's
  [[maybe_unused]] constexpr int SB = SG == 1 ? SA : 2;  // such groups held
  [[maybe_unused]] constexpr int UI = FMT == PIE_MXFP8 && MB > 2 ? 1 : MB == 4 ? 2 : MB, UN = MB / UI;  // (see mx_tiles_kernel; three blocks at a time do not fit the registers beside their halves)
  constexpr int STAGE = KS * BM * 128;
  [[maybe_unused]] constexpr int PIECES = STAGE / 1024, CP = (PIECES + 7) / 8;              // copy instructions of a stage, and of a wave
  [[maybe_unused]] constexpr int SPIECES = (KS * BM * SD + 63) / 64, SP = (SPIECES + 7) / 8;  // the same of SG stages' scales
  __shared__ __align__(16) uint8_t As[SA][STAGE];
  [[maybe_unused]] __shared__ __align__(16) uint8_t Ss[SB][SPIECES * 64 * SL];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  [[maybe_unused]] const int h = lane >> 5;
  const int ks = wave / WN;
  int tm, tn;
  tile_at(xcd_range(blockIdx.x, tiles_m, tiles_n), tiles_m, tiles_n, tm, tn);
  const int64_t m0 = (int64_t)tm * BM;
  const int nb0 = (tn * WN + wave % WN) * NJ;
  f32x16 acc[MB][NJ];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
  {
#if __HIP_DEVICE_COMPILE__
    constexpr int RSRC_FLAGS = 0x00020000;
    const int rows = (int)(M - m0 < BM ? M - m0 : BM);
    const int row_len = FMT == PIE_MXFP8 ? w.K : w.K / 2, NS = (row_len + 127) / 128;
    const int parts = KS * splits;
    auto first_of = [&](int sl) { return (int)((int64_t)NS * ((int)blockIdx.y * KS + sl) / parts); };
    const int first = first_of(ks), n = first_of(ks + 1) - first;  // this slice's stages
    const int nmax = (NS + parts - 1) / parts;
    const __amdgpu_buffer_rsrc_t rsrc_a = __builtin_amdgcn_make_buffer_rsrc(a.elements + m0 * a.row_bytes, 0, (int)((rows - 1) * a.row_bytes) + row_len, RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t rsrc_s =
        __builtin_amdgcn_make_buffer_rsrc(a.scales + m0 * a.scale_bytes, 0, (int)((rows - 1) * a.scale_bytes) + (w.K / 32 + 3) / 4 * 4, RSRC_FLAGS);
    // blocks past the matrix are out of the descriptors' range: nothing is fetched for them, and their results are dropped
    const int held = __builtin_amdgcn_readfirstlane(max(0, min(NJ, w.NB - nb0))), nbw = held > 0 ? nb0 : 0;  // (see mx_tiles_kernel)
    const __amdgpu_buffer_rsrc_t rsrc_w = __builtin_amdgcn_make_buffer_rsrc(w.data + (int64_t)nbw * w.KT * 1024, 0, held * w.KT * 1024, RSRC_FLAGS);
    const __amdgpu_buffer_rsrc_t rsrc_x = __builtin_amdgcn_make_buffer_rsrc(w.scales + (int64_t)nbw * w.KQ * 64, 0, held * w.KQ * 256, RSRC_FLAGS);
    // a wave copies pieces wave * CP .. of the slices' tiles one after the other; past the last one it copies that one again (same bytes)
    const int back[2] = {mx_piece_back(0, lane, row_len), mx_piece_back(1, lane, row_len)};
    int aoff[CP], afirst[CP], soff[SP];
#pragma unroll
    for (int jj = 0; jj < CP; ++jj) {
      const int p = min(wave * CP + jj, PIECES - 1);
      aoff[jj] = mx_row_offset(p % (BM / 8) * 8 + (lane >> 3), rows, a.row_bytes) + mx_piece_byte(p, lane);
      afirst[jj] = first_of(p / (BM / 8));
    }
    // scales: SG stages of a row lie together, SD lanes' copies; row r of slice sl is row sl * BM + r of them
#pragma unroll
    for (int jj = 0; jj < SP; ++jj) {
      const int p = min(wave * SP + jj, SPIECES - 1), at = min(p * 64 + lane, KS * BM * SD - 1), sl = at / (BM * SD), r = at / SD % BM;
      soff[jj] = mx_row_offset(r, rows, a.scale_bytes) + first_of(sl) * SD * 4 + at % SD * SL;
    }
    // stages g SG .. of every slice (behind the last scale of a row: others, or out of range, by the dword; masked when they are read)
    auto issue_s = [&](int g, int buf) {
#pragma unroll
      for (int jj = 0; jj < SP; ++jj) {
        const int p = min(wave * SP + jj, SPIECES - 1);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_s, (__attribute__((address_space(3))) void*)(&Ss[buf][p * 64 * SL]), SL, soff[jj], g * SG * SD * 4, 0, 0);
      }
    };
    auto issue_a = [&](int st, int kt) {
      const int k = min(kt, nmax - 1);  // past the end: a copy nobody reads, so that the wait counts stay uniform
#pragma unroll
      for (int jj = 0; jj < CP; ++jj) {
        const int p = min(wave * CP + jj, PIECES - 1), at = afirst[jj] + k;  // (at NS, in a shorter slice: never read)
        mx_copy_piece(rsrc_a, aoff[jj], &As[st][p * 1024], at, back[p & 1], at == NS - 1);
      }
    };
    u32x4 wreg[SW][SK][NJ];
    int xreg[SW][NJ];
    const int stage_last = min(first + max(n, 1), NS) - 1;
    auto load_x = [&](int slot, int kt) {
      const int k = min(first + kt, stage_last);
#pragma unroll
      for (int j = 0; j < NJ; ++j) xreg[slot][j] = __builtin_amdgcn_raw_buffer_load_b32(rsrc_x, j * w.KQ * 256 + lane * 4, (k * SK >> 2) * 256, 0);
    };
    auto load_w = [&](int slot, int kt, int s) {
      const int k = min(first + kt, stage_last);
#pragma unroll
      for (int j = 0; j < NJ; ++j) wreg[slot][s][j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc_w, j * w.KT * 1024 + lane * 16, (k * SK + s) * 1024, 2);  // (2: non-temporal)
    };
    auto load_a = [&](int st, int unit, i32x8 (&af)[UI]) {
      const int s = unit / UN;
#pragma unroll
      for (int i = 0; i < UI; ++i) {
        const int r = (unit % UN * UI + i) * 32 + (lane & (PAIRS ? 15 : 31)), z = (r >> 1) & 7;
        const uint8_t* row = &As[st][(ks * BM + r) * 128];
        if (FMT == PIE_MXFP8) {
          const u32x4 lo = *reinterpret_cast<const u32x4*>(row + (((s * 4 + h) ^ z) << 4)), hi = *reinterpret_cast<const u32x4*>(row + (((s * 4 + 2 + h) ^ z) << 4));
          af[i] = i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
        } else {
          const u32x4 lo = *reinterpret_cast<const u32x4*>(row + (((s * 2 + h) ^ z) << 4));
          af[i] = i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], 0, 0, 0, 0};
        }
      }
    };
    auto load_s = [&](int at, int kt, int buf, int (&sc)[SD][MB]) {  // (at: kt % SG)
      const uint32_t* group = reinterpret_cast<const uint32_t*>(&Ss[buf][(ks * BM + (lane & (PAIRS ? 15 : 31))) * SROW]) + at * SD;
#pragma unroll
      for (int d = 0; d < SD; ++d) {
        const int left = w.K / 32 - ((first + kt) * SD + d) * 4;  // blocks from here on
        const uint32_t mask = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
        for (int i = 0; i < MB; ++i) sc[d][i] = (int)((group[i * 32 * SROW / 4 + d] & mask) >> (8 * h));
      }
    };
    i32x8 af[2][UI];
    int sc[SD][MB];
    const uint32_t flip = PAIRS && (lane & 16) ? ~0u : 0u;
    // Step kt from weight slot `slot` and activation stage slot % SA; the order of requests and waits is that of mx_tiles_kernel, with the copies
    // SA - 1 steps ahead and the weights SW.  TAIL: no weights are requested any more, and only the copies are counted.
    auto step = [&](auto tail_c, auto slot_c, int kt) {
      constexpr int SLOT = decltype(slot_c)::value % SW, AT = decltype(slot_c)::value, CUR = AT % SA, NEXT = (AT + 1) % SA, FILL = (AT + SA - 1) % SA;
      constexpr bool TAIL = decltype(tail_c)::value;
      issue_a(FILL, kt + SA - 1);
      if constexpr ((AT + SA - 1) % SG == 0) issue_s((kt + SA - 1) / SG, SG == 1 ? FILL : (kt + SA - 1) / SG % SB);  // (behind them: in front 8% slower, SwiGLU of 128 rows)
      __builtin_amdgcn_sched_barrier(0);
      const int shift = FMT == PIE_MXFP8 ? ((first + kt) & 1) * 16 : 0;
      int xs[NJ], nsc[SD][MB];
#pragma unroll
      for (int j = 0; j < NJ; ++j) xs[j] = (int)((uint32_t)xreg[SLOT][j] >> shift);
      if constexpr (!TAIL) load_x(SLOT, kt + SW);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int u = 0; u < SK * UN; ++u) {
        const int s = u / UN;
        if (u + 1 < SK * UN) {
          load_a(CUR, u + 1, af[(u + 1) & 1]);
        } else {
          PIE_S_WAIT_LGKMCNT0();  // this wave's last reads of the stage have returned
          // newer than the copies of stage kt + 1: those of stages kt + 2 .. kt + SA - 1, the scales that went out with them, and weights
          constexpr int COPIES = (SA - 2) * CP + ((SA > 2 && (AT + 2) % SG == 0) + (SA > 3 && (AT + 3) % SG == 0)) * SP;
          if constexpr (TAIL) PIE_S_WAIT_VMCNT(COPIES);
          else PIE_S_WAIT_VMCNT(COPIES + (SW < SA - 2 ? SW : SA - 2) * (SK + 1) * NJ + SK * NJ);  // (the prologue has SW steps' weights)
          wg_barrier();
          load_a(NEXT, 0, af[(u + 1) & 1]);
          load_s((AT + 1) % SG, kt + 1, SG == 1 ? NEXT : (kt + 1) / SG % SB, nsc);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (kt < n) {  // (uniform; a slice that is one stage shorter than the longest)
          mx_multiply<FMT, PAIRS>(acc, wreg[SLOT][s], af[u & 1], u % UN * UI, s, xs, sc, flip);
        }
        if constexpr (!TAIL)
          if (u % UN == UN - 1) load_w(SLOT, kt + SW, s);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int d = 0; d < SD; ++d)
#pragma unroll
        for (int i = 0; i < MB; ++i) sc[d][i] = nsc[d][i];
    };
    // Prologue: the first scales, copies of stages 0 .. SA - 2, then the weights of SW steps.
#pragma unroll
    for (int g = 0; g * SG <= SA - 2; ++g) issue_s(g, g);
#pragma unroll
    for (int j = 0; j < SA - 1; ++j) issue_a(j, j);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < SW; ++j) {
      load_x(j, j);
#pragma unroll
      for (int s = 0; s < SK; ++s) load_w(j, j, s);
      __builtin_amdgcn_sched_barrier(0);
    }
    constexpr int NEWER = (SA - 2) * CP + SW * (SK + 1) * NJ;
    PIE_S_WAIT_VMCNT(NEWER < 63 ? NEWER : 63);  // the first stage has arrived
    wg_barrier();
    load_a(0, 0, af[0]);
    load_s(0, 0, 0, sc);
    int kt = 0;
    using std::integral_constant;
    // a round, or its first `left` steps, which request no weights
    auto round = [&](auto tail_c, int left) {
      constexpr bool TAIL = decltype(tail_c)::value;
      auto one = [&](auto slot_c) {
        constexpr int AT = decltype(slot_c)::value;
        if constexpr (AT < (TAIL ? SW : RS)) {
          if (!TAIL || AT < left) step(tail_c, slot_c, kt + AT);
        }
      };
      one(integral_constant<int, 0>{}); one(integral_constant<int, 1>{}); one(integral_constant<int, 2>{}); one(integral_constant<int, 3>{});
      one(integral_constant<int, 4>{}); one(integral_constant<int, 5>{}); one(integral_constant<int, 6>{}); one(integral_constant<int, 7>{});
    };
    static_assert(RS <= 8 && RS % SA == 0 && RS % SW == 0 && RS % SG == 0, "a round is written out");
    for (; kt + SW < nmax; kt += RS) round(std::false_type{}, RS);  // (steps past the last do nothing)
    round(std::true_type{}, nmax - kt);
    PIE_S_WAIT_VMCNT(0);  // the surplus copies of the last steps land before the stages are used for anything else
#endif
  }
  // The slices' sums meet one row of token blocks at a time: wave (ks, column) of block i's turn adds those of the others to its own, in
  // slice order, and finishes it.
  auto finish = [&](int i) {
    const int64_t m = m0 + i * 32 + (lane & 31);
    if constexpr (PAIRS) {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[i][j][v] = sum_xor16(acc[i][j][v]);
    }
    if (part != nullptr) {
      if (m >= M) return;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (nb0 + j >= w.NB) continue;
        float* p = part + (((int64_t)blockIdx.y * M + m) * w.NB + nb0 + j) * 32 + (lane >> 5) * 4;
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4*>(p + 8 * g) = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
      }
    } else if constexpr (GATED) {
      if (nb0 < w.NB) mx_gated_epilogue(epi, acc[i][0], acc[i][1], m, M, nb0 * 32, lane);
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        if (nb0 + j < w.NB) mx_plain_epilogue(epi, acc[i][j], m, M, (nb0 + j) * 32, lane);
    }
  };
  static_assert(KS > 1, "slices whose sums meet");
  constexpr int OTHERS = (KS - 1) * WN;  // waves whose sums a block's owners read
  constexpr int FIT = SA * STAGE / (OTHERS * NJ * 4096), ROUND = FIT < MB ? FIT : MB;  // token blocks whose sums fit the stages
  static_assert(ROUND >= 1, "a block of every wave fits the stages");
  auto sums_of = [&](int i, int sl, int j) {  // of slice sl (not the owner i % KS), block i of a round
    const int other = sl < i % KS ? sl : sl - 1;
    return reinterpret_cast<float*>(&As[0][0]) + ((i % ROUND * OTHERS + other * WN + wave % WN) * NJ + j) * 1024 + lane * 4;
  };
#pragma unroll
  for (int i0 = 0; i0 < MB; i0 += ROUND) {
    __syncthreads();
#pragma unroll
    for (int i = i0; i < (i0 + ROUND < MB ? i0 + ROUND : MB); ++i)
      if (i % KS != ks) {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int v = 0; v < 16; v += 4)
            *reinterpret_cast<f32x4*>(sums_of(i, ks, j) + v * 64) = f32x4{acc[i][j][v], acc[i][j][v + 1], acc[i][j][v + 2], acc[i][j][v + 3]};
      }
    __syncthreads();
#pragma unroll
    for (int i = i0; i < (i0 + ROUND < MB ? i0 + ROUND : MB); ++i)
      if (i % KS == ks) {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          f32x16 t;
#pragma unroll
          for (int v = 0; v < 16; ++v) t[v] = 0.f;
#pragma unroll
          for (int sl = 0; sl < KS; ++sl) {
            if (sl == ks) {
              t += acc[i][j];
            } else {
#pragma unroll
              for (int v = 0; v < 16; v += 4) {
                const f32x4 o = *reinterpret_cast<const f32x4*>(sums_of(i, sl, j) + v * 64);
#pragma unroll
                for (int u = 0; u < 4; ++u) t[v + u] += o[u];
              }
            }
          }
          acc[i][j] = t;
        }
        finish(i);
      }
  }
}

// ---------------------------------------------------------------------------------------------
// Joins the sums [splits][M][NB * 32] of a product that was split over workgroups, in their order: eight columns a lane.
// ---------------------------------------------------------------------------------------------
template <bool GATED>
__global__ __launch_bounds__(256) void mx_join_kernel(const float* __restrict__ part, int splits, int M, int NB, MxEpi e) {
  const int cols8 = GATED ? NB * 2 : NB * 4;  // pieces of eight columns (of the result) a row
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (int64_t)M * cols8) return;
  const int64_t m = at / cols8;
  const int c = (int)(at % cols8) * 8;
  const int64_t stride = (int64_t)M * NB * 32;
  auto total = [&](int n, float (&v)[8]) { add_splits(part + m * NB * 32 + n, stride, splits, v); };
  float v[8];
  if constexpr (GATED) {
    const int n = (c >> 5) * 64 + (c & 31);
    float u[8];
    total(n, v);
    total(n + 32, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = silu_f(v[i]) * u[i];
    uint8_t* row = reinterpret_cast<uint8_t*>(e.out) + m * e.ldo;
    uint8_t* scales = e.scales + m * e.lds;
    if (e.mode == MX_SWIGLU8) put_eight<PIE_MXFP8>(v, row, scales, c);
    else put_eight<PIE_MXFP4>(v, row, scales, c);
    if (c == 0) pad_scales(scales, e.N);
    return;
  }
  if (c >= e.N) return;
  total(c, v);
  if (e.mode == MX_RESID_EMBED || e.mode == MX_RESID_OUT) {
    float r[8];
    if (e.mode == MX_RESID_EMBED && !e.resid) load8(RowsView{e.embeds, e.H, PIE_BF16}, e.ids[m], c, r);
    else load8(RowsView{e.resid, e.H, PIE_F32}, m, c, r);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += r[i];
    if (e.mode == MX_RESID_OUT && !e.out) {
      const int id = e.ids[m];
      if (id >= 0) store8(RowsView{e.embeds, e.H, PIE_BF16}, id, c, v);
      return;
    }
  }
  const RowsView out{e.out, e.ldo, e.mode == MX_BF16 ? PIE_BF16 : PIE_F32};
  if (c + 8 <= e.N) {
    store8(out, m, c, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (c + i >= e.N) break;
      if (e.mode == MX_BF16) reinterpret_cast<bf16_t*>(e.out)[m * e.ldo + c + i] = f32_to_bf16(v[i]);
      else reinterpret_cast<float*>(e.out)[m * e.ldo + c + i] = v[i];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// dispatch
// ---------------------------------------------------------------------------------------------
// How a product is taken: tiles of 256 x 256 (mb 0), or mx_stream_kernel of mb token blocks, ks slices and nj weight blocks a wave, split over
// `splits` workgroups along K; of the leading `rows` rows, the rest being a product of its own.
struct MxForm { int mb, ks, nj; };
struct MxPlan { MxForm form; int splits, rows; double us; };
static constexpr MxForm MX_TILES = {0, 1, 2};
// The forms that a sweep of 1 to 4 blocks and 1 to 8 slices needed to come within 1% of its best.
static constexpr MxForm MX_PLAIN[] = {{1, 2, 1}, {1, 4, 1}, {1, 8, 1}, {2, 4, 1}, {2, 8, 1}, {3, 2, 1}, {3, 4, 1}, {1, 4, 2}, {2, 4, 2}, {3, 2, 2}, {4, 2, 2}, {4, 4, 2}};
static constexpr MxForm MX_GATED[] = {{1, 2, 2}, {1, 4, 2}, {2, 2, 2}, {2, 4, 2}, {3, 2, 2}, {3, 4, 2}, {4, 2, 2}, {4, 4, 2}};

// Estimated microseconds.  Workgroups go in rounds of one to a compute unit; a round costs its start (first requests, the slices' sums, the epilogue) and its
// stages, a stage the longest of its matrix instructions, of what it fetches and of its reads of LDS.  The constants are fitted to every form and
// split of 207 products of 1 to 2500 rows (weights from HBM, calls in a graph): what this picks takes 1.1% more time than the best form with 8-bit
// rows on average, 1.9% with 4-bit ones, 2.2% on 35 products outside the fit, and 16% at most (40 rows of 608 onto 4874: 8.1 us, 7.0).
// Examples, its choice and the next best, 8-bit rows: SwiGLU of 4096 onto 2 x 14336 at one row (1, 4, 2) 18.7 us, (1, 2, 2) in 2 splits 20.7; at 64 rows (2, 4, 2)
// 24.1, (1, 2, 2) 27.6; at 333 (3, 2, 2) 78.9, tiles 91; at 2100 tiles 369, (3, 2, 2) 408.  14336 onto 4096 at 64 rows (2, 4, 2) in 7 splits 22.8, the best (1, 4, 2) in
// 4 20.1; at 900 (4, 4, 2) 105, (4, 2, 2) in 2 105.
struct MxCosts {
  double round, stage, busy;               // tiles: a round, a stage, and what that costs more on all compute units
  double mma, bandwidth, reads, step;      // others, a stage: matrix instructions of an accumulator tile, KiB a us, reads of a block of rows; what comes on top
  double start, tile, join, sums;          // a round, and that of an accumulator tile; a split product's join, GB/ms of its sums
};
static constexpr MxCosts MX_COSTS8 = {7.48, 2.06, 0.43, 0.35, 32.2, 0.48, 0.091, 3.59, 0.27, 3.34, 3.2}, MX_COSTS4 = {5.83, 0.93, 1.05, 0.27, 53.6, 0.058, 0.015, 5.77, 0.03, 2.14, 1.75};
static double mx_tiles_us(int M, int NB, int NS, bool fp8, int n_cus) {
  const MxCosts& c = fp8 ? MX_COSTS8 : MX_COSTS4;
  const int64_t wgs = (int64_t)((M + MX_TM - 1) / MX_TM) * ((NB + MX_TN / 32 - 1) / (MX_TN / 32));
  auto round = [&](int64_t busy) { return c.round + NS * (c.stage + c.busy * (double)busy / n_cus); };
  return 0.9 + (double)(wgs / n_cus) * round(n_cus) + (wgs % n_cus ? round(wgs % n_cus) : 0.0);
}
static double mx_stream_us(const MxForm& f, int splits, int M, int NB, int NS, bool fp8, bool defer, int n_cus) {
  const MxCosts& c = fp8 ? MX_COSTS8 : MX_COSTS4;
  const int WN = 8 / f.ks, tiles_m = (M + 32 * f.mb - 1) / (32 * f.mb), tiles_n = (NB + f.nj * WN - 1) / (f.nj * WN);
  const int64_t wgs = (int64_t)tiles_m * tiles_n * splits, rounds = (wgs + n_cus - 1) / n_cus;
  const int steps = (NS + f.ks * splits - 1) / (f.ks * splits);
  const double kib = f.ks * std::min(32 * f.mb, M) / 8.0 + (fp8 ? 16 : 32) * f.nj;
  const double stage = std::max({c.mma * f.mb * f.nj, kib / c.bandwidth, c.reads * f.mb}) + c.step;
  const double t = 0.9 + (double)rounds * (c.start + c.tile * f.mb * f.nj + steps * stage);
  return t + (splits > 1 ? (defer ? 0.5 : c.join) + (double)splits * M * NB * 32 * 8e-6 / c.sums : 0.0);
}
// The best of one form for all rows, and of tiles for whole rounds with another form behind them (8320 rows of 14336 onto 4096 in 4 bits: 33 x 16 tiles
// take 285 us, 32 x 16 and the last 128 rows in another form 239; SwiGLU of 8320 rows of 8 bits 1392 and 1348).
static MxPlan mx_plan_whole(int M, const MxPacked& w, bool gated, bool fp8, bool defer, int n_cus) {
  const int row = fp8 ? w.K : w.K / 2, NS = (row + 127) / 128;
  MxPlan best{MX_TILES, 1, M, M > 128 ? mx_tiles_us(M, w.NB, NS, fp8, n_cus) : 1e30};  // (the sweep has no product of up to 128 rows for them)
  auto look = [&](const MxForm& f) {
    for (int splits = 1; splits <= 8; ++splits) {
      if (splits > 1 && ((size_t)splits * M * w.NB * 32 > MX_WS_FLOATS || f.ks * splits * 2 > NS)) break;
      const double us = mx_stream_us(f, splits, M, w.NB, NS, fp8, defer, n_cus);
      if (us < best.us) best = MxPlan{f, splits, M, us};
    }
  };
  if (gated) for (const MxForm& f : MX_GATED) look(f);
  else for (const MxForm& f : MX_PLAIN) look(f);
  return best;
}
static MxPlan mx_plan(int M, const MxPacked& w, bool gated, bool fp8, bool defer, int n_cus) {
  MxPlan best = mx_plan_whole(M, w, gated, fp8, defer, n_cus);
  const int tiles_m = (M + MX_TM - 1) / MX_TM, NS = ((fp8 ? w.K : w.K / 2) + 127) / 128;
  for (int cut = tiles_m - 1; cut >= 1 && cut >= tiles_m - 4; --cut) {
    const int rows = cut * MX_TM;
    const double us = mx_tiles_us(rows, w.NB, NS, fp8, n_cus) + mx_plan_whole(M - rows, w, gated, fp8, false, n_cus).us;
    if (us < best.us) best = MxPlan{MX_TILES, 1, rows, us};
  }
  return best;
}

template <bool GATED, int FMT, int MB, int KS, int NJ>
static hipError_t run_stream_form(const MxRowsView& a, int M, const MxPacked& w, const MxEpi& e, int splits, bool defer, float* ws, hipStream_t s) {
  constexpr int WN = 8 / KS;
  const int tiles_m = (M + MB * 32 - 1) / (MB * 32), tiles_n = (w.NB + NJ * WN - 1) / (NJ * WN);
  auto go = [&](auto pairs_c) {
    mx_stream_kernel<GATED, FMT, MB, KS, NJ, decltype(pairs_c)::value>
        <<<dim3(tiles_m * tiles_n, splits), dim3(512), 0, s>>>(a, M, w, e, tiles_m, tiles_n, splits, splits > 1 ? ws : nullptr);
  };
  if (FMT == PIE_MXFP8 && MB == 1 && M <= 16) go(std::integral_constant<bool, FMT == PIE_MXFP8 && MB == 1>{});
  else go(std::false_type{});
  if (splits > 1 && !defer) {
    const int64_t pieces = (int64_t)M * w.NB * (GATED ? 2 : 4);
    mx_join_kernel<GATED><<<pieces_grid(pieces), dim3(256), 0, s>>>(ws, splits, M, w.NB, e);
  }
  return hipGetLastError();
}

template <bool GATED, int FMT>
static hipError_t run_product(const MxRowsView& a, int M, const MxPacked& w, const MxEpi& e, const MxPlan& p, bool defer, float* ws, hipStream_t s) {
  const MxForm& f = p.form;
  if (f.mb == 0) {
    const int tiles_m = (M + MX_TM - 1) / MX_TM, tiles_n = (w.NB + MX_TN / 32 - 1) / (MX_TN / 32);
    mx_tiles_kernel<GATED, FMT><<<dim3(tiles_m * tiles_n), dim3(512), 0, s>>>(a, M, w, e, tiles_m, tiles_n);
    return hipGetLastError();
  }
#define MX_FORM(MB, KS, NJ) \
  if (f.mb == MB && f.ks == KS && f.nj == NJ) return run_stream_form<GATED, FMT, MB, KS, NJ>(a, M, w, e, p.splits, defer, ws, s);
  MX_FORM(1, 4, 2) MX_FORM(2, 4, 2) MX_FORM(3, 2, 2) MX_FORM(4, 2, 2) MX_FORM(4, 4, 2)
  if constexpr (GATED) {
    MX_FORM(1, 2, 2) MX_FORM(2, 2, 2) MX_FORM(3, 4, 2)
  } else {
    MX_FORM(1, 2, 1) MX_FORM(1, 4, 1) MX_FORM(1, 8, 1) MX_FORM(2, 4, 1) MX_FORM(2, 8, 1) MX_FORM(3, 2, 1) MX_FORM(3, 4, 1)
  }
#undef MX_FORM
  return hipErrorInvalidValue;
}

// Rows of one launch, which has fewer than 2^32 threads: at most 2^22 tiles, were they of 32 x 32.
static int mx_rows_at_once(const MxPacked& w) { return std::max((1 << 27) / w.NB / MX_TM * MX_TM, MX_TM); }

hipError_t launch_mx_product(const MxRowsView& a, int format, int M, const MxPacked& w, const MxEpi& e, float* ws, int n_cus, hipStream_t s, int* deferred) {
  if (deferred) *deferred = 0;
  if (M <= 0) return hipSuccess;
  const bool gated = e.mode == MX_SWIGLU8 || e.mode == MX_SWIGLU4, fp8 = format == PIE_MXFP8;
  auto behind = [&](int rows) {  // the product of the rows from `rows` on
    MxRowsView rest = a;
    rest.elements += rows * a.row_bytes;
    rest.scales += rows * a.scale_bytes;
    MxEpi r = e;
    if (e.out) r.out = reinterpret_cast<uint8_t*>(e.out) + rows * e.ldo * (gated ? 1 : e.mode == MX_BF16 ? 2 : 4);
    if (e.scales) r.scales = e.scales + rows * e.lds;
    if (e.ids) r.ids = e.ids + rows;
    if (e.resid) r.resid = e.resid + (int64_t)rows * e.H;
    return launch_mx_product(rest, format, M - rows, w, r, ws, n_cus, s);
  };
  if (const int most = mx_rows_at_once(w); M > most) {
    const hipError_t err = launch_mx_product(a, format, most, w, e, ws, n_cus, s);
    return err != hipSuccess ? err : behind(most);
  }
  const bool defer = deferred != nullptr;
  const int key = 4 * M + 2 * defer + fp8;  // (gated or not, and the number of compute units, do not change from call to call)
  const MxPacked::Plan* kept = std::find_if(std::begin(w.plans), std::end(w.plans), [&](const MxPacked::Plan& x) { return x.key == key; });
  if (kept == std::end(w.plans)) {
    const MxPlan q = mx_plan(M, w, gated, fp8, defer, n_cus);
    MxPacked::Plan& slot = w.plans[w.oldest++ % std::size(w.plans)];
    slot = MxPacked::Plan{key, q.form.mb, q.form.ks, q.form.nj, q.splits, q.rows};
    kept = &slot;
  }
  const MxPlan p{{kept->mb, kept->ks, kept->nj}, kept->splits, kept->rows, 0.0};
  const hipError_t err = gated ? (fp8 ? run_product<true, PIE_MXFP8>(a, p.rows, w, e, p, defer, ws, s) : run_product<true, PIE_MXFP4>(a, p.rows, w, e, p, defer, ws, s))
                               : (fp8 ? run_product<false, PIE_MXFP8>(a, p.rows, w, e, p, defer, ws, s) : run_product<false, PIE_MXFP4>(a, p.rows, w, e, p, defer, ws, s));
  if (deferred && p.splits > 1) *deferred = p.splits;
  return err != hipSuccess || p.rows == M ? err : behind(p.rows);
}

void mx_product_plan(int M, const MxPacked& w, bool gated, int format, int n_cus, int64_t out[5]) {
  const MxPlan p = mx_plan(std::min(M, mx_rows_at_once(w)), w, gated, format == PIE_MXFP8, false, n_cus);
  out[0] = p.form.mb ? 32 * p.form.mb : MX_TM;
  out[1] = p.form.mb ? 32 * p.form.nj * (8 / p.form.ks) : MX_TN;
  out[2] = p.form.ks;
  out[3] = p.splits;
  out[4] = p.rows;
}

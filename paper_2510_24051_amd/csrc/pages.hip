// Whole KvPages: forked (copied onto other pages, permuted in place), compacted (the visible tokens of a request moved to the front
// of its pages), saved into a caller's buffer and restored from it.  Everything here moves bytes; what bounds it is HBM, and for
// small calls the launch.
#include "internal.h"

namespace {
// ---------------------------------------------------------------------------------------------
// fork
// ---------------------------------------------------------------------------------------------
// A thread owns the same 16 bytes of every page of its layer and walks the moves of one run in order.  The host orders them so that
// a page is written only after every move that reads it, so within a thread each load comes before the store that replaces what it
// reads, and no other thread touches those bytes: any graph of moves, permutations included, needs no second buffer and no
// synchronisation.  A run with a cycle starts by keeping the page that the cycle's last move reads (PageRun::keep; the
// order: page_plans.h).
// Bound by HBM: 200 pages (64 KiB in each of 16 layers, 210 MB) read and written in 65 us by themselves, 6.4 TB/s, 73 behind a
// kernel that has left its output in the caches; a small call by its launch (one page seven times, 32 layers: 6 us).  Sources are read
// non-temporally, pages stored plainly, as what forks them soon reads them (stored non-temporally: 200 pages and their
// save 151 -> 160 us a pass).
#define FORK_THREADS 256
#define FORK_AHEAD 8  // moves whose sources are read before the first of them is stored: a read only ever comes too late, never too early
template <int N>
struct ForkMoves {
  PageMove moves[N];
  PageRun runs[N];
};
template <int N>
__global__ __launch_bounds__(FORK_THREADS) void fork_kernel(unsigned char* __restrict__ kv, int64_t layer_bytes, int64_t page_bytes, int slices,
                                                            ForkMoves<N> plan) {
  const int run = blockIdx.x / slices, slice = blockIdx.x % slices;
  unsigned char* base = kv + (int64_t)blockIdx.y * layer_bytes + ((int64_t)slice * FORK_THREADS + threadIdx.x) * 16;
  const PageRun r = plan.runs[run];
  u32x4 kept = {0, 0, 0, 0}, now = {0, 0, 0, 0};
  if (r.keep >= 0) kept = *reinterpret_cast<const u32x4*>(base + r.keep * page_bytes);
  const int end = r.first + r.n;
  int before = -1;  // source of the move in front
  for (int i = r.first; i < end; i += FORK_AHEAD) {
    u32x4 v[FORK_AHEAD];
    int last = before;
#pragma unroll
    for (int q = 0; q < FORK_AHEAD; ++q) {
      if (i + q >= end) break;
      const int src = plan.moves[i + q].src;
      if (src >= 0 && src != last) v[q] = load_nt(reinterpret_cast<const u32x4*>(base + src * page_bytes));
      last = src;
    }
#pragma unroll
    for (int q = 0; q < FORK_AHEAD; ++q) {
      if (i + q >= end) break;
      const PageMove m = plan.moves[i + q];
      if (m.src < 0) now = kept;
      else if (m.src != before) now = v[q];
      before = m.src;
      *reinterpret_cast<u32x4*>(base + m.dst * page_bytes) = now;
    }
  }
}

// ---------------------------------------------------------------------------------------------
// save and restore
// ---------------------------------------------------------------------------------------------
// (Kernel arguments cost the host time, here and above, so short lists have a small block of their own.  Calls back to back, the host's
// time for each with the large block and with the small one: two pages saved 3.35 and 3.20 us, a fork with the call's checks 4.7 and 4.4,
// a fork after an append 15.1 and 11.1.  A short compaction's plan, 13.1 and 12.9, has one block.)
template <int N>
struct PageIds { int32_t v[N]; };

// The pool keeps V as 8 tokens of one dim next to each other, tokens' rows have 8 dims of one token next to each other: eight lanes
// turn the one into the other among themselves.  Lane i of eight stands for row label(i) before and after; with
// label(i) = i ^ (i >> 2) * 3 the three exchanges (labels that differ in bit 2, 1, 0) are a half mirror and two quad permutations.
__device__ __forceinline__ int octet_label(int i) { return i ^ ((i >> 2 & 1) * 3); }
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true); }
__device__ __forceinline__ u32x4 transpose8(u32x4 w, int label) {
  const bool b2 = label & 4, b1 = label & 2, b0 = label & 1;
  // rows i and i ^ 4: this lane goes on with columns 4 b2 .. 4 b2 + 3 of both
  const uint32_t k0 = b2 ? w[2] : w[0], k1 = b2 ? w[3] : w[1], g0 = dpp<0x141>(b2 ? w[0] : w[2]), g1 = dpp<0x141>(b2 ? w[1] : w[3]);
  const uint32_t a0 = b2 ? g0 : k0, a1 = b2 ? g1 : k1, c0 = b2 ? k0 : g0, c1 = b2 ? k1 : g1;  // row i & 3, row i | 4
  // rows that differ in bit 1: two columns of each
  const uint32_t ka = b1 ? a1 : a0, kc = b1 ? c1 : c0, ga = dpp<0x4E>(b1 ? a0 : a1), gc = dpp<0x4E>(b1 ? c0 : c1);
  const uint32_t r0 = b1 ? ga : ka, r2 = b1 ? ka : ga, r4 = b1 ? gc : kc, r6 = b1 ? kc : gc;
  // rows that differ in bit 0: one column of each, the two rows side by side
  const uint32_t pick = b0 ? 0x03020706u : 0x05040100u;  // high half of the neighbour's and of this row's, or both low halves
  u32x4 out;
  out[0] = __builtin_amdgcn_perm(dpp<0xB1>(r0), r0, pick);
  out[1] = __builtin_amdgcn_perm(dpp<0xB1>(r2), r2, pick);
  out[2] = __builtin_amdgcn_perm(dpp<0xB1>(r4), r4, pick);
  out[3] = __builtin_amdgcn_perm(dpp<0xB1>(r6), r6, pick);
  return out;
}

// The image is [page][layer][K or V][slot][kv head][dim].  A wave takes one head of one 16-token block.  An access covers 8 tokens and 64
// dims, so that both sides move whole lines: 128 bytes of each token in the image; in the pool, where 16-byte pieces hold 8 dims of a
// token (K) or 8 tokens of a dim (V), 128 bytes of each octet of dims.  (16 tokens and 32 dims, a KiB of the pool and 64 bytes of a
// token: lines of the image that are read past the caches come twice, 64 pages of an 8B-shaped model restored in 54 us for 49, saved in
// 50 for 47.)  Bound by HBM: those are 134 MB each way, 5.6 TB/s.  One thread per 8 dims of a token, V gathered 2 bytes at a time, took
// 262 and 102.
// Written plainly.  Read so where the image is less than a quarter of the 256 MB cache in front of the memory, which then often holds the
// pages, and non-temporally (ONCE) from there on.  Three sets of pages and images in turn, plain and non-temporal: 16.8 MB 6.5 and 7.6 us,
// 33.6 MB 10.7 and 12.8, 46 MB 16 both, 57 MB 22 and 18, 67 MB 27 and 21, 134 MB 51 and 47; three sets of pages into one image 57 MB 16
// and 18, 67 MB 21 both, 134 MB 36 and 35, 188 MB 70 and 47.
#define IMAGE_WAVES 4
#define IMAGE_ONCE ((int64_t)64 << 20)
template <int D, bool TO_POOL, int IDS, bool ONCE>
__global__ __launch_bounds__(64 * IMAGE_WAVES) void page_image_kernel(bf16_t* __restrict__ kv, int64_t layer_elems, int n_layers, PageIds<IDS> ids, int total,
                                                                      int F, int Hkv, uint16_t* __restrict__ image) {
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 63, layer = blockIdx.y;
  const int at = blockIdx.x * IMAGE_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int h = at % Hkv, f = at / Hkv % F, p = at / (Hkv * F);
  uint16_t* blk = reinterpret_cast<uint16_t*>(kv) + layer * layer_elems + (((int64_t)ids.v[p] * F + f) * Hkv + h) * (2 * PAGE * D);
  const int64_t row = (int64_t)Hkv * D, part = (int64_t)F * PAGE * row;
  uint16_t* img = image + (((int64_t)p * n_layers + layer) * 2) * part + (int64_t)f * PAGE * row + h * D;
  const int label = octet_label(lane & 7);
  const int octet = lane >> 3;  // of the 64 dims that an access covers
  uint16_t* pk = blk + octet * 128 + (lane & 7) * 8;
  uint16_t* pv = blk + PAGE * D + (octet >> 2) * 512 + (octet & 3) * 64 + label * 8;
  uint16_t* ik = img + swap23(lane & 7) * row + octet * 8;  // (swap23 of a slot and of that slot 8 further on: 4 apart)
  uint16_t* iv = img + part + label * row + octet * 8;
  u32x4 k[N], v[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {  // 64 dims j / 2, half j % 2 of the tokens
    const u32x4* from_k = reinterpret_cast<const u32x4*>(TO_POOL ? ik + (j & 1) * 4 * row + (j >> 1) * 64 : pk + (j >> 1) * 1024 + (j & 1) * 64);
    const u32x4* from_v = reinterpret_cast<const u32x4*>(TO_POOL ? iv + (j & 1) * 8 * row + (j >> 1) * 64 : pv + (j >> 1) * 1024 + (j & 1) * 256);
    k[j] = ONCE ? load_nt(from_k) : *from_k;
    v[j] = ONCE ? load_nt(from_v) : *from_v;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    *reinterpret_cast<u32x4*>(TO_POOL ? pk + (j >> 1) * 1024 + (j & 1) * 64 : ik + (j & 1) * 4 * row + (j >> 1) * 64) = k[j];
    *reinterpret_cast<u32x4*>(TO_POOL ? pv + (j >> 1) * 1024 + (j & 1) * 256 : iv + (j & 1) * 8 * row + (j >> 1) * 64) = transpose8(v[j], label);
  }
}

// ---------------------------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------------------------
// A wave owns 64 dims of one head of one layer, of K or of V, and walks a chain: it reads the source blocks that hold kept tokens one
// after the other, each once and in whole KiB, puts the kept tokens' rows of 8 dims (16 bytes) behind each other into a ring of 32
// tokens in LDS, and stores a destination block whenever 16 are there.  V is turned into rows on the way in and back on the way
// out (transpose8).  A wave of K takes 32 dims and those D/2 above, which the rotation pairs them with.
// In place: a kept token moves towards the front, so when a destination block is stored every token at or before its last one has
// been read, and what the chain reads later lies behind it; no other wave touches these dims.  The reads run COMPACT_AHEAD
// blocks in front of the stores, which only makes them earlier.
// Bound by HBM where there are waves enough: 4 x 1021 of 3600 tokens of an 8B-shaped model in place with rotated keys (0.54 GB each
// way) 231 us, 4.6 TB/s, where a copy of 1 GiB reaches 4.7; half of 4830 tokens of 16 layers into other pages 46 us, 5.5 TB/s of whole
// source blocks and what is written.  With few, by the chain: 0.45 us a block.  Two blocks ahead instead of four: 337 -> 385 us (8000
// tokens, 32 layers, in order); six or eight: the same.  Non-temporal stores: 456 -> 437 us for the first with its save, 82 -> 88
// for the second, so plain ones.
#define COMPACT_WAVES 4
#define COMPACT_AHEAD 4
template <int D, bool IS_K>
__device__ __forceinline__ void compact_walk(const uint16_t* src, uint16_t* dst, int64_t block_elems, int part, CompactChain chain, u32x4* ring,
                                             const CompactEntry* __restrict__ entries, const int32_t* __restrict__ tiles,
                                             const int32_t* __restrict__ turn, const float* __restrict__ angles) {
  const int lane = threadIdx.x & 63;
  // this lane's token of a block and its place in the two KiB of it: K holds rows of 8 dims, V is taken by dims and turned
  const int label = octet_label(lane & 7);
  const int t = IS_K ? swap23(lane & 15) : (lane >> 5) * 8 + label;
  const int piece = IS_K ? lane >> 4 : lane >> 3 & 3;  // dims 8 piece .. of the first KiB; pieces 4 .. 7 are the second's
  const int o0 = IS_K ? part * 512 + lane * 8 : PAGE * D + part * 1024 + (lane & ~7) * 8 + label * 8, o1 = o0 + (IS_K ? D * 8 : 512);
  const uint32_t before = (1u << t) - 1u;
  auto slot_at = [&](int slot, int q) { return (slot & 31) * 8 + (q ^ (slot & 7)); };  // (rows a bank apart, whatever the slots)

  int count = 0, stored = 0;  // tokens put into the ring, blocks stored
  auto store = [&](int n) {  // the next 16 tokens of the ring, of which n are there
    uint16_t* to = dst + tiles[chain.tile0 + stored] * block_elems;
    u32x4 a = ring[slot_at(stored * PAGE + t, piece)], b = ring[slot_at(stored * PAGE + t, piece + 4)];
    ++stored;
    if (IS_K) {
      if (t >= n) return;
    } else {
      a = transpose8(a, label);
      b = transpose8(b, label);
      const int here = n - (lane >> 5) * 8;  // tokens of this lane's octet that are there
      if (here <= 0) return;
      if (here < 8) {  // the others stay as they are
        Pack16 x, y, p, q;
        x.u = a; y.u = b;
        p.u = *reinterpret_cast<const u32x4*>(to + o0);
        q.u = *reinterpret_cast<const u32x4*>(to + o1);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= here) { x.s[e] = p.s[e]; y.s[e] = q.s[e]; }
        a = x.u;
        b = y.u;
      }
    }
    *reinterpret_cast<u32x4*>(to + o0) = a;
    *reinterpret_cast<u32x4*>(to + o1) = b;
  };

  u32x4 raw[COMPACT_AHEAD][2];
  int rows[COMPACT_AHEAD] = {};  // of the table, where a block's tokens turn differently
  auto request = [&](int i, u32x4 (&r)[2], int& row) {  // (the last block again behind the end: nothing depends on a branch)
    const CompactEntry e = entries[min(i, chain.entry1 - 1)];
    const uint16_t* from = src + e.block * block_elems;
    r[0] = load_nt(reinterpret_cast<const u32x4*>(from + o0));
    r[1] = load_nt(reinterpret_cast<const u32x4*>(from + o1));
    if (IS_K && e.turn == COMPACT_MIXED) row = turn[e.first + min(__popc(e.mask & before), __popc(e.mask) - 1)];
  };
  // K: the angles of a block are asked for one block ahead, so that waiting for them does not empty the queue of reads; two sets,
  // which blocks that turn by one row share until another row comes
  float cs[2][8], sn[2][8];
  int held[2] = {COMPACT_STILL, COMPACT_STILL};
  auto take = [&](int i, int row, float (&c)[8], float (&s)[8], int& held_row) {
    const int by = entries[min(i, chain.entry1 - 1)].turn;
    if (by == COMPACT_STILL || (by != COMPACT_MIXED && by == held_row)) return;
    held_row = by;
    if (by != COMPACT_MIXED) row = by;
    const float* a = angles + (int64_t)max(row, 0) * D + part * 32 + piece * 8;  // of 8 dims; those D/2 above turn with them
#pragma unroll
    for (int e = 0; e < 8; ++e) { c[e] = a[e]; s[e] = a[D / 2 + e]; }
  };
#pragma unroll
  for (int q = 0; q < COMPACT_AHEAD; ++q) request(chain.entry0 + q, raw[q], rows[q]);
  if (IS_K) take(chain.entry0, rows[0], cs[0], sn[0], held[0]);
  for (int i0 = chain.entry0; i0 < chain.entry1; i0 += COMPACT_AHEAD) {
#pragma unroll
    for (int q = 0; q < COMPACT_AHEAD; ++q) {
      if (i0 + q >= chain.entry1) break;
      const CompactEntry e = entries[i0 + q];
      const int slot = count + __popc(e.mask & before);
      Pack16 a, b;
      a.u = raw[q][0];
      b.u = raw[q][1];
      const int row = e.turn == COMPACT_MIXED ? rows[q] : e.turn;
      if (IS_K) take(i0 + q + 1, rows[(q + 1) % COMPACT_AHEAD], cs[(q + 1) & 1], sn[(q + 1) & 1], held[(q + 1) & 1]);
      request(i0 + q + COMPACT_AHEAD, raw[q], rows[q]);
      if (IS_K) {
        if (e.turn != COMPACT_STILL) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float x = (float)a.h[k], y = (float)b.h[k], c = cs[q & 1][k], s = sn[q & 1][k];
            const bf16_t u = f32_to_bf16(x * c - y * s), v = f32_to_bf16(y * c + x * s);
            if (row >= 0) { a.h[k] = u; b.h[k] = v; }  // (else: the bits as they are)
          }
        }
      } else {
        a.u = transpose8(a.u, label);
        b.u = transpose8(b.u, label);
      }
      if (e.mask >> t & 1) {
        ring[slot_at(slot, piece)] = a.u;
        ring[slot_at(slot, piece + 4)] = b.u;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // (one wave: its LDS accesses take effect in the order they have here)
      count += __popc(e.mask);
      if (count >= (stored + 1) * PAGE) {
        store(PAGE);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
    }
  }
  if (count > stored * PAGE) store(count - stored * PAGE);
}

template <int D>
__global__ __launch_bounds__(64 * COMPACT_WAVES) void compact_kernel(const bf16_t* src, int64_t src_layer, bf16_t* dst, int64_t dst_layer, int Hkv, int total,
                                                                     const CompactChain* __restrict__ chains,
                                                                     const CompactEntry* __restrict__ entries, const int32_t* __restrict__ tiles,
                                                                     const int32_t* __restrict__ turn, const float* __restrict__ angles) {
  constexpr int PARTS = 2 * (D / 64);  // waves of a head: K, then V
  __shared__ u32x4 rings[COMPACT_WAVES][32 * 8];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int at = blockIdx.x * COMPACT_WAVES + wave;
  if (at >= total) return;
  const int part = at % PARTS, h = at / PARTS % Hkv;
  const CompactChain chain = chains[at / (PARTS * Hkv)];
  const uint16_t* from = reinterpret_cast<const uint16_t*>(src) + (int64_t)blockIdx.y * src_layer + (int64_t)h * (2 * PAGE * D);  // (in place: the same)
  uint16_t* to = reinterpret_cast<uint16_t*>(dst) + (int64_t)blockIdx.y * dst_layer + (int64_t)h * (2 * PAGE * D);
  const int64_t block_elems = (int64_t)Hkv * (2 * PAGE * D);
  if (part < PARTS / 2) compact_walk<D, true>(from, to, block_elems, part, chain, rings[wave], entries, tiles, turn, angles);
  else compact_walk<D, false>(from, to, block_elems, part - PARTS / 2, chain, rings[wave], entries, tiles, turn, angles);
}

// A small plan, as kernel arguments, into device memory, and the angles of its shifts (64 bits, rounded once: a shift may be long).
struct PlanBytes { uint32_t w[PLAN_BY_VALUE / 4]; };
__global__ void put_plan_kernel(PlanBytes plan, int words, uint32_t* __restrict__ dev, int turn0, int n_turns, const double* __restrict__ inv_freq,
                                int D, float* __restrict__ angles) {
  const int idx = blockIdx.x * blockDim.x + threadIdx.x, half = D / 2;
  if (idx < words) dev[idx] = plan.w[idx];
  if (idx >= n_turns * half) return;
  const int r = idx / half, i = idx % half;
  double sn, cs;
  sincos((double)(int32_t)plan.w[turn0 + r] * inv_freq[i], &sn, &cs);
  angles[(int64_t)r * D + i] = (float)cs;
  angles[(int64_t)r * D + half + i] = (float)sn;
}
}  // namespace

hipError_t launch_fork(bf16_t* kv, size_t layer_elems, int n_layers, size_t page_elems, const PageMove* moves, int n_moves, const PageRun* runs,
                       int n_runs, hipStream_t s) {
  if (n_moves > FORK_MOVES || n_runs > FORK_MOVES) return hipErrorInvalidValue;
  if (n_runs <= 0) return hipSuccess;
  const int slices = (int)(page_elems * sizeof(bf16_t) / (FORK_THREADS * 16));  // (a page has a multiple of 4 KiB in a layer)
  auto go = [&](auto plan) {
    for (int i = 0; i < n_moves; ++i) plan.moves[i] = moves[i];
    for (int i = 0; i < n_runs; ++i) plan.runs[i] = runs[i];
    fork_kernel<<<dim3((unsigned)(n_runs * slices), (unsigned)n_layers), dim3(FORK_THREADS), 0, s>>>(
        reinterpret_cast<unsigned char*>(kv), layer_elems * 2, page_elems * 2, slices, plan);
  };
  if (n_moves <= 16) go(ForkMoves<16>());  // (a run has a move at least)
  else go(ForkMoves<FORK_MOVES>());
  return hipGetLastError();
}

hipError_t launch_page_image(bf16_t* kv, size_t layer_elems, int n_layers, const int32_t* host_ids, int n, int F, int Hkv, int D, bf16_t* image,
                             bool to_pool, hipStream_t s) {
  const int64_t page_image = (int64_t)n_layers * 2 * F * PAGE * Hkv * D;
  for (int p0 = 0; p0 < n; p0 += IDS_BY_VALUE) {
    const int m = n - p0 < IDS_BY_VALUE ? n - p0 : IDS_BY_VALUE;
    const int total = m * F * Hkv;
    const dim3 grid((unsigned)((total + IMAGE_WAVES - 1) / IMAGE_WAVES), (unsigned)n_layers), block(64 * IMAGE_WAVES);
    uint16_t* img = reinterpret_cast<uint16_t*>(image) + p0 * page_image;
    auto go = [&](auto ids, auto once) {
      constexpr int N = sizeof(ids) / sizeof(int32_t);
      constexpr bool ONCE = decltype(once)::value;
      for (int i = 0; i < m; ++i) ids.v[i] = host_ids[p0 + i];
      auto* kernel = D == 128 ? (to_pool ? page_image_kernel<128, true, N, ONCE> : page_image_kernel<128, false, N, ONCE>)
                              : (to_pool ? page_image_kernel<64, true, N, ONCE> : page_image_kernel<64, false, N, ONCE>);
      kernel<<<grid, block, 0, s>>>(kv, layer_elems, n_layers, ids, total, F, Hkv, img);
    };
    if (n * page_image * (int64_t)sizeof(bf16_t) >= IMAGE_ONCE) go(PageIds<IDS_BY_VALUE>(), std::true_type());
    else if (m <= 64) go(PageIds<64>(), std::false_type());
    else go(PageIds<IDS_BY_VALUE>(), std::false_type());
  }
  return hipGetLastError();
}

hipError_t launch_put_plan(const unsigned char* plan, size_t size, unsigned char* dev, size_t turns, int n_turns, const double* inv_freq, int D,
                           float* angles, hipStream_t s) {
  if (size > PLAN_BY_VALUE || size % 4 || turns % 4 || turns + (size_t)n_turns * 4 > size) return hipErrorInvalidValue;
  const int words = (int)(size / 4), threads = words > n_turns * (D / 2) ? words : n_turns * (D / 2);
  PlanBytes bytes;
  __builtin_memcpy(bytes.w, plan, size);
  put_plan_kernel<<<dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s>>>(bytes, words, reinterpret_cast<uint32_t*>(dev), (int)(turns / 4), n_turns,
                                                                                inv_freq, D, angles);
  return hipGetLastError();
}

hipError_t launch_compact(const CompactPlan& p, int n_chains, int n_layers, int Hkv, int D, hipStream_t s) {
  if (n_chains <= 0) return hipSuccess;
  const int total = n_chains * Hkv * 2 * (D / 64);
  const dim3 grid((unsigned)((total + COMPACT_WAVES - 1) / COMPACT_WAVES), (unsigned)n_layers), block(64 * COMPACT_WAVES);
  auto* kernel = D == 128 ? compact_kernel<128> : compact_kernel<64>;
  kernel<<<grid, block, 0, s>>>(p.src, (int64_t)p.src_layer, p.dst, (int64_t)p.dst_layer, Hkv, total, p.chains, p.entries, p.tiles, p.turn, p.angles);
  return hipGetLastError();
}

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
// synchronisation.  A run with a cycle starts by keeping the page that the cycle's last move reads (PageRun::keep).
#define FORK_THREADS 256
template <typename Plan>
__global__ __launch_bounds__(FORK_THREADS) void fork_kernel(unsigned char* __restrict__ kv, int64_t layer_bytes, int64_t page_bytes, int slices,
                                                            Plan plan) {
  const int run = blockIdx.x / slices, slice = blockIdx.x % slices;
  unsigned char* base = kv + (int64_t)blockIdx.y * layer_bytes + ((int64_t)slice * FORK_THREADS + threadIdx.x) * 16;
  const PageRun r = plan.run(run);
  u32x4 kept = {0, 0, 0, 0}, v = {0, 0, 0, 0};
  if (r.keep >= 0) kept = *reinterpret_cast<const u32x4*>(base + r.keep * page_bytes);
  int last = -1;
  for (int i = r.first; i < r.first + r.n; ++i) {
    const PageMove m = plan.move(i);
    if (m.src < 0) v = kept;
    else if (m.src != last) v = *reinterpret_cast<const u32x4*>(base + m.src * page_bytes);
    last = m.src;
    *reinterpret_cast<u32x4*>(base + m.dst * page_bytes) = v;
  }
}

struct ForkByValue {
  PageMove moves[FORK_BY_VALUE];
  PageRun runs[FORK_BY_VALUE];
  __device__ PageRun run(int i) const { return runs[i]; }
  __device__ PageMove move(int i) const { return moves[i]; }
};
struct ForkByPointer {
  const PageMove* moves;
  const PageRun* runs;
  __device__ PageRun run(int i) const { return runs[i]; }
  __device__ PageMove move(int i) const { return moves[i]; }
};

// ---------------------------------------------------------------------------------------------
// save and restore
// ---------------------------------------------------------------------------------------------
struct PageIds { int32_t v[IDS_BY_VALUE]; };

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

// The image is [page][layer][K or V][slot][kv head][dim].  A wave takes one head of one 16-token block: D/32 times 1 KiB of K, which in
// the pool are 16-byte pieces of 8 dims of a token already, and as much of V.  On the pool's side every access is 1 KiB
// in one piece, on the image's 16 tokens of 64 bytes.
#define IMAGE_WAVES 4
template <int D, bool TO_POOL>
__global__ __launch_bounds__(64 * IMAGE_WAVES) void page_image_kernel(bf16_t* __restrict__ kv, int64_t layer_elems, int n_layers, PageIds ids, int total,
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
  uint16_t* pk = blk + lane * 8;
  uint16_t* pv = blk + PAGE * D + (lane & ~7) * 8 + label * 8;
  uint16_t* ik = img + swap23(lane & 15) * row + (lane >> 4) * 8;
  uint16_t* iv = img + part + ((lane >> 5) * 8 + label) * row + (lane >> 3 & 3) * 8;
  u32x4 k[N], v[N];
#pragma unroll
  for (int j = 0; j < N; ++j) {
    k[j] = load_nt(reinterpret_cast<const u32x4*>(TO_POOL ? ik + j * 32 : pk + j * 512));
    v[j] = load_nt(reinterpret_cast<const u32x4*>(TO_POOL ? iv + j * 32 : pv + j * 512));
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    *reinterpret_cast<u32x4*>(TO_POOL ? pk + j * 512 : ik + j * 32) = k[j];
    *reinterpret_cast<u32x4*>(TO_POOL ? pv + j * 512 : iv + j * 32) = transpose8(v[j], label);
  }
}

// ---------------------------------------------------------------------------------------------
// compact
// ---------------------------------------------------------------------------------------------
// A wave owns some dims of one head of one layer and walks the tiles (16-token destination blocks) of a chain in order.  Kept tokens
// move towards the front, so a tile's sources lie at or behind its own tokens, and every later tile's behind all of them: in place,
// a wave's stores only ever replace tokens that it has loaded already, and no other wave touches its dims.
//   K: waves 0 .. D/64 - 1, lane (token, 8 dims i .. i+7) with the dims D/2 above them, which the rotation pairs them with;
//   V: waves D/64 .. 2 D/64 - 1, lane = dim, the two octets of a tile's tokens one after the other.
template <int D>
__global__ __launch_bounds__(2 * D) void compact_kernel(bf16_t* __restrict__ kv, int64_t layer_elems, int Hkv, CompactPlan plan) {
  constexpr int KW = D / 64;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int chain = blockIdx.x / Hkv, h = blockIdx.x % Hkv;
  uint16_t* pool = reinterpret_cast<uint16_t*>(kv) + (int64_t)blockIdx.y * layer_elems;
  auto block_of = [&](int b) { return pool + ((int64_t)b * Hkv + h) * (2 * PAGE * D); };
  const int2 tiles = plan.chains[chain];
  for (int i = tiles.x; i < tiles.y; ++i) {
    const CompactTile tile = plan.tiles[i];
    uint16_t* dst = block_of(tile.dst_block);
    if (wave < KW) {
      const int t = lane & 15, c = wave * 4 + (lane >> 4);  // dims 8c .. 8c + 7 and D/2 above
      if (t < tile.n) {
        const int src = plan.src[tile.first + t], turn = plan.turn ? plan.turn[tile.first + t] : -1;
        const uint16_t* from = block_of(src / PAGE);
        Pack16 a, b;
        a.u = *reinterpret_cast<const u32x4*>(from + k_elem_offset(src % PAGE, 8 * c));
        b.u = *reinterpret_cast<const u32x4*>(from + k_elem_offset(src % PAGE, 8 * c + D / 2));
        if (turn >= 0) {
          const float* angles = plan.angles + (int64_t)turn * D + 8 * c;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = (float)a.h[e], y = (float)b.h[e], cs = angles[e], sn = angles[D / 2 + e];
            a.h[e] = f32_to_bf16(x * cs - y * sn);
            b.h[e] = f32_to_bf16(y * cs + x * sn);
          }
        }
        *reinterpret_cast<u32x4*>(dst + k_elem_offset(t, 8 * c)) = a.u;
        *reinterpret_cast<u32x4*>(dst + k_elem_offset(t, 8 * c + D / 2)) = b.u;
      }
    } else {
      const int d = (wave - KW) * 64 + lane;
      for (int o = 0; o * 8 < tile.n; ++o) {
        Pack16 out;
        out.u = *reinterpret_cast<const u32x4*>(dst + v_elem_offset(8 * o, d, D));
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (8 * o + e < tile.n) {
            const int src = plan.src[tile.first + 8 * o + e];
            out.s[e] = block_of(src / PAGE)[v_elem_offset(src % PAGE, d, D)];
          }
        *reinterpret_cast<u32x4*>(dst + v_elem_offset(8 * o, d, D)) = out.u;
      }
    }
  }
}
}  // namespace

hipError_t launch_fork(bf16_t* kv, size_t layer_elems, int n_layers, size_t page_elems, const PageMove* moves, int n_moves, const PageRun* runs,
                       int n_runs, bool on_device, hipStream_t s) {
  if (n_runs <= 0) return hipSuccess;
  const int slices = (int)(page_elems * sizeof(bf16_t) / (FORK_THREADS * 16));  // (a page has a multiple of 4 KiB in a layer)
  const dim3 grid((unsigned)(n_runs * slices), (unsigned)n_layers), block(FORK_THREADS);
  unsigned char* p = reinterpret_cast<unsigned char*>(kv);
  if (on_device) {
    fork_kernel<ForkByPointer><<<grid, block, 0, s>>>(p, layer_elems * 2, page_elems * 2, slices, ForkByPointer{moves, runs});
    return hipGetLastError();
  }
  if (n_moves > FORK_BY_VALUE || n_runs > FORK_BY_VALUE) return hipErrorInvalidValue;
  ForkByValue plan;
  for (int i = 0; i < n_moves; ++i) plan.moves[i] = moves[i];
  for (int i = 0; i < n_runs; ++i) plan.runs[i] = runs[i];
  fork_kernel<ForkByValue><<<grid, block, 0, s>>>(p, layer_elems * 2, page_elems * 2, slices, plan);
  return hipGetLastError();
}

hipError_t launch_page_image(bf16_t* kv, size_t layer_elems, int n_layers, const int32_t* host_ids, int n, int F, int Hkv, int D, bf16_t* image,
                             bool to_pool, hipStream_t s) {
  const int64_t page_image = (int64_t)n_layers * 2 * F * PAGE * Hkv * D;
  for (int p0 = 0; p0 < n; p0 += IDS_BY_VALUE) {
    const int m = n - p0 < IDS_BY_VALUE ? n - p0 : IDS_BY_VALUE;
    PageIds ids;
    for (int i = 0; i < m; ++i) ids.v[i] = host_ids[p0 + i];
    const int total = m * F * Hkv;
    const dim3 grid((unsigned)((total + IMAGE_WAVES - 1) / IMAGE_WAVES), (unsigned)n_layers), block(64 * IMAGE_WAVES);
    uint16_t* img = reinterpret_cast<uint16_t*>(image) + p0 * page_image;
    if (D == 128 && to_pool) page_image_kernel<128, true><<<grid, block, 0, s>>>(kv, layer_elems, n_layers, ids, total, F, Hkv, img);
    else if (D == 128) page_image_kernel<128, false><<<grid, block, 0, s>>>(kv, layer_elems, n_layers, ids, total, F, Hkv, img);
    else if (to_pool) page_image_kernel<64, true><<<grid, block, 0, s>>>(kv, layer_elems, n_layers, ids, total, F, Hkv, img);
    else page_image_kernel<64, false><<<grid, block, 0, s>>>(kv, layer_elems, n_layers, ids, total, F, Hkv, img);
  }
  return hipGetLastError();
}

hipError_t launch_compact(bf16_t* kv, size_t layer_elems, int n_layers, int Hkv, int D, const CompactPlan& plan, int n_chains, hipStream_t s) {
  if (n_chains <= 0) return hipSuccess;
  const dim3 grid((unsigned)(n_chains * Hkv), (unsigned)n_layers);
  if (D == 128) compact_kernel<128><<<grid, dim3(256), 0, s>>>(kv, layer_elems, Hkv, plan);
  else compact_kernel<64><<<grid, dim3(128), 0, s>>>(kv, layer_elems, Hkv, plan);
  return hipGetLastError();
}

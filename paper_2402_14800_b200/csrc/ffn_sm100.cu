// Dense gated feed-forward block on the caller's own weights, forward and backward.
//
//   forward   g = x W1^T,  u = x W3^T,  a = silu(g) * u            (one launch)
//             y = a W2^T [+ residual]
//   backward  da = dy W2,  dg = da * u * silu'(g),  du = da * silu(g)
//             dx = dg W1 + du W3,   dW1 = dg^T x,  dW3 = du^T x,  dW2 = dy^T a
//
// One persistent warp-specialised GEMM does all of it, D[m][n] = sum_k A[m][k] B[n][k], stored as
// out[n][m]: m is always the contiguous index of the output, so a warp's 32 tensor-memory lanes write
// neighbouring elements.  What differs between the launches is where A and B come from, how they lie in
// memory (contiguous in k, or in m / n: the tensor cores take either from a 128-byte swizzled tile), and the
// epilogue.
//
// A pair of CTAs (cluster of two, cta_group::2) computes an item of 4 R x n_tile: two accumulators of M = 256
// (each CTA holds 128 rows of each, R of them in use) by up to 256 columns, half of them staged by either CTA.
// In the gate/up launch the accumulators are g and u of the same 2 R features, so a thread holds both and the
// activation needs no exchange.  The tile follows from the sizes (choose_plan): large problems take 512 x 256
// per pair, which halves the traffic from L2 that a 256 x 128 tile per CTA would need and that bounds the tensor
// pipe; a few tokens take as many weight rows a CTA as give every SM the same number of weight bytes, since then
// HBM is all that counts; and where rows alone do not fill the machine the contraction is split, the partial
// sums go to fp32 planes and a small kernel adds them in a fixed order.
//
// The forward pass saves what the backward pass makes of g and u: p = u * silu'(g) and q = silu(g), so that
// dg = da * p and du = da * q, and a itself for dW2.  It has the sigmoid at hand; a second evaluation behind the da
// products would keep the accumulators from the tensor cores for a quarter of their time.
//
// Rounding: sums and everything in an epilogue are fp32.  a, dg and du are rounded to the tensors' type, because the
// tensor cores take them as 16-bit operands; p and q are saved in fp32, since rounding them as well would cost the
// gradients as much again as those operands' roundings do.
//
// Waits are bounded and end in the status word of moe_operators_status.
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

#include "ffn.h"
#include "moe_test_hooks.h"
#include "sm100.h"

namespace moe {

namespace {

__device__ int g_status;  // set when a bounded wait of this file's kernels expired

enum Kind { kGateUp, kGateUpSave, kPlain, kDact, kGrads };

// Launches of at most 64 columns, or 128 with a contraction of at most 16 k-blocks, run a slim form of the kernel, half
// an SM each in shared memory, registers and tensor memory: with few tokens what counts is the gap between two launches,
// and the next launch's CTAs set up and fetch their first weights beside the last ones of this launch.  Forward pass in
// us, full form / slim form, tokens 64 and 128: (h 512, f 1024) 18.6 / 16.3, 18.1 / 16.8; (2048, 4096) 31.7 / 29.8, 32.9 /
// 33.9; (4096, 4096) 48.8 / 46.5, 50.6 / 63.9; (4096, 14336) 76.6 / 75.8, 78.9 / 90.9.  Up to 32 columns a matrix of 96 MB and
// more streams longer than the gap costs, and the full form has more of it in flight: 8 tokens of (4096, 14336), 117 MB,
// 67.2 / 69.9, of (4096, 8192), 67 MB, 50.0 / 49.7; where between the two the line lies was not measured.
template <bool SLIM> struct Form {
  static constexpr int kEpiWarps = SLIM ? 4 : 16;
  static constexpr int kThreads = 96 + 32 * kEpiWarps;
  static constexpr int kAccCols = SLIM ? 128 : 256;            // columns of an accumulator, of which there are two
  static constexpr int kChunks = kAccCols / 4 / kEpiWarps;     // chunks of 16 columns a warp reads of an accumulator
  static constexpr int kSmem = SLIM ? 114688 : 230400;         // dynamic shared memory at most
};
constexpr int kAccRows = 128;           // rows of an accumulator in one CTA
constexpr int kMaxStages = 8;           // size of the barrier block
constexpr int kBandTiles = 16;          // n tiles that sweep the m tiles together

// A operand contiguous in m (W2 of da, W1 and W3 of dx, x and a of the weights' gradients)
constexpr __host__ __device__ bool a_mn(int kind) { return kind == kDact || kind == kGrads; }
constexpr __host__ __device__ bool gate_up(int kind) { return kind == kGateUp || kind == kGateUpSave; }

struct Problem {
  int M, N;       // m and n range
  int mt, nt;     // tiles
  void* out;      // [N][M]
  int KB, segKB;  // k-blocks of 64; of one segment (dx: two segments, else segKB = KB)
  int S, kbs;     // k-splits, k-blocks of each
  int R, n_tile;  // rows of A a CTA and accumulator loads, columns of an item
  int a0, b0;     // tensor maps of the first segment
  int bmn;        // B contiguous in n (weights' gradients)
  float* planes;  // S > 1: [S][N][M] partial sums
};

struct Args {
  Problem p[4];               // kGrads: dx, dW1, dW3, dW2
  int np;
  int first, skip;            // kGrads: the dx items, one a pair, count as `skip` rounds of the others
  int stages, slot_a, stage, tail;  // pipeline stages, bytes of an accumulator's A tile, of a stage, behind the last one
  int fp16;
  const void* residual;       // kPlain
  float2* saved;              // [N][M] (p, q): written by kGateUpSave, read by kDact
  void* du;                   // kDact, beside out = dg
  int early;                  // A is no earlier launch of this call's output: its first stages may be read ahead
};

struct Maps {
  CUtensorMap a[5], b[5];
};

__device__ __forceinline__ uint32_t pack16(float a, float b, int fp16) {
  if (fp16) {
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
  return pack_bf16(a, b);
}
__device__ __forceinline__ float2 unpack16(uint32_t v, int fp16) {
  if (fp16) return __half22float2(*reinterpret_cast<const __half2*>(&v));
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

// Descriptor of a tile that is contiguous in m (or n): boxes of 64 elements x 64 k, each 64 rows of 128 bytes;
// groups of 8 k are 1024 bytes apart (stride offset), boxes 8192 (leading offset).
__device__ __forceinline__ uint64_t smem_desc_mn128(uint32_t saddr) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3ffffu) >> 4);
  d |= (uint64_t)(8192 >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(taddr)
               : "memory");
}
// copies of 16 bytes through L2 to shared memory (bytes = 0: zeros), in groups; all groups but the newest
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_wait_but_one() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
__device__ __forceinline__ void copy_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float2 load8_shared(uint32_t addr) {
  float2 v;
  asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void prefetch_tensor_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
constexpr uint32_t kMnBoxBytes = 64 * 128;
constexpr uint32_t kStepK = 32 >> 4;            // 16 k further, in descriptor units: 32 bytes along a row
constexpr uint32_t kStepMn = (16 * 128) >> 4;   // or 16 rows of k

// Both operands of one type, fp16 or bf16 (never mixed), fp32 accumulation; bits 15 and 16: A, B contiguous in m, n.
__device__ __forceinline__ uint32_t idesc16(int M, int N, int fp16, bool amn, bool bmn) {
  const uint32_t t = fp16 ? 0u : 1u;
  return (1u << 4) | (t << 7) | (t << 10) | ((amn ? 1u : 0u) << 15) | ((bmn ? 1u : 0u) << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

struct Item {
  int prob, m0, n0, ks, kb0, kb1;  // m0: first row of the pair's item
  int valid;                       // columns that exist
};

// The k-th item of a pair, past the last one when there is none.  Items are dealt in rounds; where dx shares a launch
// with the weights' gradients the pairs that got one of its long items join the rounds of short ones late.
template <int KIND> __host__ __device__ __forceinline__ int item_of(const Args& a, int k, int pair, int n_pairs) {
  if (KIND != kGrads || a.first == 0) return pair + k * n_pairs;
  const int rest = n_pairs - a.first;
  if (pair < a.first) return k == 0 ? pair : a.first + a.skip * rest + (k - 1) * n_pairs + pair;
  return a.first + (k < a.skip ? k * rest + pair - a.first : a.skip * rest + (k - a.skip) * n_pairs + pair);
}

// The item of which a pair may read A ahead of the wait, -1 for none.  There are at least as many items as pairs, but a
// pair can have none all the same: without a round that is left out (skip 0) the pairs of dx take part in the first round
// of the others, and the last pairs find it empty.  What such a pair loaded would still be under way when its CTAs end.
template <int KIND> __host__ __device__ __forceinline__ int item_ahead(const Args& a, int pair, int n_pairs, int n_items) {
  const int item = item_of<KIND>(a, 0, pair, n_pairs);
  return a.early && item < n_items ? item : -1;
}

// Items of a problem: k-split -> band of at most kBandTiles n tiles -> m tile -> n tile, so that the items in
// flight share few tiles of either operand in L2.
template <int KIND> __device__ __forceinline__ Item decode_item(const Args& a, int item) {
  Item t;
  t.prob = 0;
  if (KIND == kGrads) {
    while (t.prob + 1 < a.np && item >= a.p[t.prob].mt * a.p[t.prob].nt * a.p[t.prob].S) {
      item -= a.p[t.prob].mt * a.p[t.prob].nt * a.p[t.prob].S;
      ++t.prob;
    }
  }
  const Problem& p = a.p[t.prob];
  t.ks = gate_up(KIND) ? 0 : item / (p.mt * p.nt);
  item -= t.ks * p.mt * p.nt;
  const int bands = (p.nt + kBandTiles - 1) / kBandTiles;
  const int per_band = (p.nt + bands - 1) / bands;
  const int band = item / (per_band * p.mt);
  const int rem = item - band * per_band * p.mt;
  const int band_tiles = min(per_band, p.nt - band * per_band);
  const int m = rem / band_tiles;
  t.m0 = m * (gate_up(KIND) ? 2 : 4) * p.R;
  t.n0 = (band * per_band + rem - m * band_tiles) * p.n_tile;
  t.valid = min(p.n_tile, p.N - t.n0);
  t.kb0 = t.ks * p.kbs;
  t.kb1 = min(p.KB, t.kb0 + p.kbs);
  return t;
}

// Stores 2 PAIRS columns n (from col0 of the item on) of the warp's 32 neighbouring m, given as packed pairs of
// columns per lane: even lanes take the even columns of two neighbouring m, odd lanes the odd ones.
// `out` points at (n of col0, m of lane 0); in_m: this lane's pair of m exists.
template <int PAIRS>
__device__ __forceinline__ void store_cols(const uint32_t* v, uint16_t* out, long long ld, int col0, int valid, bool in_m,
                                           int lane) {
  const bool odd = lane & 1;
  uint16_t* o = out + (lane & 30) + (odd ? ld : 0);
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    const uint32_t other = __shfl_xor_sync(0xffffffffu, v[i], 1);
    const uint32_t w = odd ? __byte_perm(other, v[i], 0x7632) : __byte_perm(v[i], other, 0x5410);
    if (in_m && col0 + 2 * i + (lane & 1) < valid) *reinterpret_cast<uint32_t*>(o) = w;
    o += 2 * ld;
  }
}

template <int KIND, bool SLIM>
__global__ void __launch_bounds__(Form<SLIM>::kThreads, SLIM ? 2 : 1)
ffn_gemm_kernel(const __grid_constant__ Maps maps, const Args args) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ Bars bars;
  constexpr bool AMN = a_mn(KIND), GU = gate_up(KIND);
  constexpr int kEpiWarps = Form<SLIM>::kEpiWarps, kAccCols = Form<SLIM>::kAccCols, kChunks = Form<SLIM>::kChunks;
  constexpr int kStride = kEpiWarps / 4;  // of a warp's chunks
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();  // 0 = leader of the pair
  const int pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;

  setup_barriers<kMaxStages>(bars, 2 * kEpiWarps, 2);
  if (warp == 1) {
    tmem_alloc_pair(smem_u32(&bars.tmem_base), 2 * kAccCols);
    tmem_relinquish_pair();
  }
  constexpr int kMapsA = KIND == kGrads ? 5 : GU ? 2 : 1, kMapsB = KIND == kGrads ? 5 : 1;
  if (warp == 0 && lane < kMapsA) prefetch_tensor_map(&maps.a[lane]);
  if (warp == 0 && lane >= 8 && lane < 8 + kMapsB) prefetch_tensor_map(&maps.b[lane - 8]);
  __syncwarp();
  tc_fence_before();
  cluster_sync_all();  // both CTAs' barriers exist before anything is signalled across the pair
  tc_fence_after();
  const uint32_t tmem_base = *(volatile uint32_t*)&bars.tmem_base;
  volatile int* abort_flag = &bars.abort_flag;

  const uint32_t ns = (uint32_t)args.stages, stage_bytes = (uint32_t)args.stage, slot_a = (uint32_t)args.slot_a;
  int n_items = 0;
  for (int i = 0; i < (KIND == kGrads ? args.np : 1); ++i) n_items += args.p[i].mt * args.p[i].nt * args.p[i].S;
  uint32_t issued = 0;

  if (warp == 0) {
    // ---- TMA producer of this CTA's rows of A and its half of the columns; the bytes of both CTAs are counted on
    // the leader's barrier
    uint32_t s = 0, ph = 0;
    bool ok = true;
    auto load_a = [&](const Item& t, int kb, uint32_t stage) {  // and what the stage's barrier expects
      const Problem& p = args.p[t.prob];
      const int half = p.n_tile >> 1;  // a multiple of 8
      const uint32_t a_bytes = AMN ? (uint32_t)((p.R + 63) >> 6) * kMnBoxBytes : (uint32_t)p.R * 128u;
      const uint32_t b_bytes = KIND == kGrads && p.bmn ? (uint32_t)((half + 63) >> 6) * kMnBoxBytes : (uint32_t)half * 128u;
      const uint32_t full = map_to_cta(smem_u32(&bars.full[stage]), 0), sa = smem_base + stage * stage_bytes;
      if (rank == 0) mbar_expect_tx(smem_u32(&bars.full[stage]), 2u * (2u * a_bytes + b_bytes));
      const int seg = KIND == kGrads && kb >= p.segKB ? 1 : 0;
      const int k0 = (kb - seg * p.segKB) * BK, row0 = t.m0 + p.R * (int)rank;
#pragma unroll
      for (int acc = 0; acc < 2; ++acc) {
        const CUtensorMap* map = &maps.a[GU ? acc : p.a0 + seg];
        const int row = GU ? row0 : row0 + 2 * p.R * acc;
        if (AMN) {
          for (int j = 0; j < p.R; j += 64) tma_load_2d_pair(sa + acc * slot_a + j * 128, map, row + j, k0, full);
        } else {
          tma_load_2d_pair(sa + acc * slot_a, map, k0, row, full);
        }
      }
    };
    auto load_b = [&](const Item& t, int kb, uint32_t stage) {
      const Problem& p = args.p[t.prob];
      const int half = p.n_tile >> 1, col0 = t.n0 + half * (int)rank;
      const uint32_t full = map_to_cta(smem_u32(&bars.full[stage]), 0), sb = smem_base + stage * stage_bytes + 2 * slot_a;
      const int seg = KIND == kGrads && kb >= p.segKB ? 1 : 0, k0 = (kb - seg * p.segKB) * BK;
      const CUtensorMap* map = &maps.b[p.b0 + seg];
      if (KIND == kGrads && p.bmn) {
        for (int j = 0; j < half; j += 64) tma_load_2d_pair(sb + j * 128, map, col0 + j, k0, full);
      } else {
        tma_load_2d_pair(sb, map, k0, col0, full);
      }
    };
    // The launch before this one let it start after its own wait (below), so everything older than that launch is
    // complete, the weights among it: the first ring of stages of A may come before the wait.
    uint32_t ahead = 0;
    const int early = item_ahead<KIND>(args, pair, n_pairs, n_items);
    if (early >= 0) {
      const Item t = decode_item<KIND>(args, early);
      ahead = min(ns, (uint32_t)(t.kb1 - t.kb0));
      if (lane == 0)
        for (uint32_t i = 0; i < ahead; ++i) load_a(t, t.kb0 + (int)i, i);
      __syncwarp();
    }
    pdl_wait();
    pdl_launch_dependents();
    for (int k = 0, item; ok && (item = item_of<KIND>(args, k, pair, n_pairs)) < n_items; ++k) {
      const Item t = decode_item<KIND>(args, item);
      for (int kb = t.kb0; kb < t.kb1; ++kb, ++issued) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars.empty[s]), ph ^ 1u, abort_flag));
        if (!ok) break;
        if (lane == 0) {
          if (issued >= ahead) load_a(t, kb, s);
          load_b(t, kb, s);
        }
        if (++s == ns) { s = 0; ph ^= 1u; }
        __syncwarp();
      }
    }
    issued = max(issued, ahead);
  } else if (warp <= 2) {
    // ---- MMA issuers of the leader, one warp per accumulator.  No stage is full before the producers have passed the
    // wait; these warps pass it too, so that the limit of their first wait counts this launch's time and not what is left
    // of a launch in front that let this one start at once.
    if (rank == 0) {
      pdl_wait();
      const uint32_t acc = (uint32_t)warp - 1u;
      const uint32_t d_tmem = tmem_base + (uint32_t)kAccCols * acc;
      const uint32_t tmem_full = smem_u32(&bars.tmem_full[acc]), tmem_empty = smem_u32(&bars.tmem_empty[acc]);
      constexpr uint32_t sa_k = AMN ? kStepMn : kStepK;
      uint32_t s = 0, ph = 0, nu = 0;  // nu: items so far
      bool ok = true;
      for (int item; ok && (item = item_of<KIND>(args, (int)nu, pair, n_pairs)) < n_items; ++nu) {
        const Item t = decode_item<KIND>(args, item);
        const bool bmn = KIND == kGrads && args.p[t.prob].bmn;
        const uint32_t idesc = idesc16(256, args.p[t.prob].n_tile, args.fp16, AMN, bmn);
        const uint32_t sb_k = bmn ? kStepMn : kStepK;
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          bool ready = mbar_wait(smem_u32(&bars.full[s]), ph, abort_flag);
          if (kb == t.kb0) ready = ready && mbar_wait(tmem_empty, (nu & 1u) ^ 1u, abort_flag);
          ok = __all_sync(0xffffffffu, ready);
          if (!ok) break;
          tc_fence_after();
          if (lane == 0) {
            const uint32_t sa = smem_base + s * stage_bytes + acc * slot_a, sb = smem_base + s * stage_bytes + 2 * slot_a;
            const uint64_t adesc = AMN ? smem_desc_mn128(sa) : smem_desc_k128(sa);
            const uint64_t bdesc = bmn ? smem_desc_mn128(sb) : smem_desc_k128(sb);
            umma_bf16_pair(d_tmem, adesc, bdesc, idesc, kb > t.kb0 ? 1u : 0u);
            umma_bf16_pair(d_tmem, adesc + sa_k, bdesc + sb_k, idesc, 1u);
            umma_bf16_pair(d_tmem, adesc + 2 * sa_k, bdesc + 2 * sb_k, idesc, 1u);
            umma_bf16_pair(d_tmem, adesc + 3 * sa_k, bdesc + 3 * sb_k, idesc, 1u);
            umma_commit_pair(smem_u32(&bars.empty[s]));
            if (kb == t.kb1 - 1) umma_commit_pair(tmem_full);
          }
          if (++s == ns) { s = 0; ph ^= 1u; }
          __syncwarp();
        }
      }
    }
  } else {
    pdl_wait();
    // ---- epilogue: warp w reads tensor-memory lanes 32 (w % 4) .. + 31, and of the chunks of 16 columns every kStride-th
    const int wq = warp & 3, group = (warp - 3) >> 2;
    const int row = 32 * wq + lane;  // row of this thread in its CTA's part of an accumulator
    const uint32_t empty0 = map_to_cta(smem_u32(&bars.tmem_empty[0]), 0);
    const uint32_t empty1 = map_to_cta(smem_u32(&bars.tmem_empty[1]), 0);
    const uint32_t taddr0 = tmem_base + ((uint32_t)(32 * wq) << 16);
    const int fp16 = args.fp16;
    uint32_t nu = 0;
    bool ok = true;
    for (int item; ok && (item = item_of<KIND>(args, (int)nu, pair, n_pairs)) < n_items; ++nu) {
      const Item t = decode_item<KIND>(args, item);
      const Problem& p = args.p[t.prob];
      const long long ld = p.M;
      const int R = p.R;
      if constexpr (GU) {
        ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars.tmem_full[0]), nu & 1u, abort_flag) &&
                                         mbar_wait(smem_u32(&bars.tmem_full[1]), nu & 1u, abort_flag));
        if (!ok) break;
        tc_fence_after();
        const int m0 = t.m0 + R * (int)rank + 32 * wq;  // of lane 0
        const bool in_m = row < R && m0 + lane < p.M;
        auto store_act = [&](const uint32_t* act, int c0) {  // R and M are even: both m of a lane's pair exist or neither
          store_cols<8>(act, reinterpret_cast<uint16_t*>(p.out) + (long long)(t.n0 + c0) * ld + m0, ld, c0, t.valid, in_m, lane);
        };
        // with rounds of items to come the accumulators go back to the MMAs before the stores; slim launches have one, and
        // there the loop stays a loop: instructions are fetched once a launch (1-4 % of the smallest calls)
        uint32_t act[SLIM ? 1 : kChunks][8];
#pragma unroll(SLIM ? 1 : kChunks)
        for (int i = 0; i < kChunks; ++i) {
          const int c0 = 16 * (group + kStride * i);
          if (c0 >= t.valid) continue;
          uint32_t g[16], u[16];
          tmem_ld16(taddr0 + c0, g);
          tmem_ld16(taddr0 + kAccCols + c0, u);
          tmem_ld_wait();
          float2* o = args.saved + (long long)(t.n0 + c0) * ld + m0 + lane;
#pragma unroll
          for (int c = 0; c < 16; ++c) {
            const float gc = __uint_as_float(g[c]), uc = __uint_as_float(u[c]);
            const float sg = ffn_sigmoid(gc), q = gc * sg;
            g[c] = __float_as_uint(q * uc);
            if constexpr (KIND == kGateUpSave) {
              if (in_m && c0 + c < t.valid) *o = make_float2(uc * fmaf(q, 1.0f - sg, sg), q);
              o += ld;
            }
          }
#pragma unroll
          for (int c = 0; c < 8; ++c)
            act[SLIM ? 0 : i][c] = pack16(__uint_as_float(g[2 * c]), __uint_as_float(g[2 * c + 1]), fp16);
          if (SLIM) store_act(act[0], c0);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive_cluster(empty0);
          mbar_arrive_cluster(empty1);
        }
        if (!SLIM) {
#pragma unroll
          for (int i = 0; i < kChunks; ++i) {
            const int c0 = 16 * (group + kStride * i);
            if (c0 < t.valid) store_act(act[SLIM ? 0 : i], c0);
          }
        }
      } else {
        if constexpr (!SLIM && KIND != kDact) {
          // The usual case: both accumulators are read, rounded and handed back before the first store, so that the
          // next item's MMAs run beside the stores.
          if (p.S == 1 && !(KIND == kPlain && args.residual)) {
            uint32_t w[2][kChunks][8];
#pragma unroll
            for (int acc = 0; acc < 2; ++acc) {
              ok = ok && __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars.tmem_full[acc]), nu & 1u, abort_flag));
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int i = 0; i < kChunks; ++i) {
                uint32_t v[16];
                tmem_ld16(taddr0 + kAccCols * acc + 16 * (group + kStride * i), v);
                tmem_ld_wait();
#pragma unroll
                for (int c = 0; c < 8; ++c)
                  w[acc][i][c] = pack16(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]), fp16);
              }
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive_cluster(acc ? empty1 : empty0);
            }
            if (!ok) break;
#pragma unroll
            for (int acc = 0; acc < 2; ++acc) {
              const int m0 = t.m0 + R * (2 * acc + (int)rank) + 32 * wq;
              const bool in_m = row < R && m0 + lane < p.M;
#pragma unroll
              for (int i = 0; i < kChunks; ++i) {
                const int c0 = 16 * (group + kStride * i);
                if (c0 < t.valid)
                  store_cols<8>(w[acc][i], reinterpret_cast<uint16_t*>(p.out) + (long long)(t.n0 + c0) * ld + m0, ld, c0,
                                t.valid, in_m, lane);
              }
            }
            continue;
          }
        }
        if constexpr (KIND == kDact) {
          if (p.S == 1) {
            // Units of 8 columns, accumulator 0 and then 1.  What this epilogue waits for is the saved values, 235 MB at
            // 2048 tokens (h 4096, f 14336), most of them from HBM.  A warp copies its values of two units ahead to shared
            // memory, since before the accumulators are complete: of each two columns the even lanes one and the odd lanes
            // the other, for two neighbouring rows (16 bytes).  Against one unit ahead in registers: a training step of 100
            // tokens of (128, 448) 36.4 -> 33.8 us, 8000 of (64, 2000) 177 -> 172, 2048 of (4096, 14336) the same.
            // (Three stages of operands are as fast as four.  Fetching all of it to L2 during the MMAs was 20 % slower: it
            // was evicted again, and 649 MB came from HBM instead of 436.)
            const uint32_t mine = smem_base + ns * stage_bytes + args.tail + ((warp - 3) * 32 + lane) * 8;
            const int odd = lane & 1;
            constexpr uint32_t kCol = kEpiWarps * 32 * 8;  // bytes of a column
            int units = 0;  // of an accumulator
            while (units < 2 * kChunks && 16 * (group + kStride * (units >> 1)) + 8 * (units & 1) < t.valid) ++units;
            auto col_of = [&](int u) { return 16 * (group + kStride * (u >> 1)) + 8 * (u & 1); };
            auto copy_unit = [&](int u) {
              const int acc = u >= units, c0 = col_of(u - acc * units);
              const int m = t.m0 + R * (2 * acc + (int)rank) + row - odd;  // even, and so are R and M
              const bool in_m = row < R && m < p.M;
              const float2* sp = args.saved + (long long)(t.n0 + c0 + odd) * ld + m;
#pragma unroll
              for (int c = 0; c < 8; c += 2) {
                const bool in = in_m && c0 + c + odd < t.valid;
                copy16_async(mine - 8 * odd + (8 * (u & 1) + c + odd) * kCol, in ? sp : args.saved, in ? 16 : 0);
                sp += 2 * ld;
              }
            };
            if (units) copy_unit(0);
            copy_commit();
            if (units) copy_unit(1);
            copy_commit();
#pragma unroll 1
            for (int u = 0; u < max(2 * units, 2); ++u) {
              const int acc = units ? u >= units : u, i = u - acc * units;
              if (i == 0 || !units) {
                ok = ok && __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars.tmem_full[acc]), nu & 1u, abort_flag));
                if (!ok) break;
                tc_fence_after();
              }
              uint32_t v[8], wg[4], wu[4];
              const int c0 = units ? col_of(i) : 0;
              if (units) {
                copy_wait_but_one();
                __syncwarp();  // the neighbours' copies too
                tmem_ld8(taddr0 + kAccCols * acc + c0, v);
                tmem_ld_wait();
              }
              if (!units || i == units - 1) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(acc ? empty1 : empty0);
              }
              if (!units) continue;
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                const float2 a = load8_shared(mine + (8 * (u & 1) + 2 * c) * kCol);
                const float2 b = load8_shared(mine + (8 * (u & 1) + 2 * c + 1) * kCol);
                const float d0 = __uint_as_float(v[2 * c]), d1 = __uint_as_float(v[2 * c + 1]);
                wg[c] = pack16(d0 * a.x, d1 * b.x, fp16);
                wu[c] = pack16(d0 * a.y, d1 * b.y, fp16);
              }
              __syncwarp();  // all lanes have read what is written over
              if (u + 2 < 2 * units) copy_unit(u + 2);
              copy_commit();  // an empty group keeps the count
              const int m0 = t.m0 + R * (2 * acc + (int)rank) + 32 * wq;
              const bool in_m = row < R && m0 + lane < p.M;
              const long long at = (long long)(t.n0 + c0) * ld + m0;
              store_cols<4>(wg, reinterpret_cast<uint16_t*>(p.out) + at, ld, c0, t.valid, in_m, lane);
              store_cols<4>(wu, reinterpret_cast<uint16_t*>(args.du) + at, ld, c0, t.valid, in_m, lane);
            }
            copy_wait_all();  // nothing in flight when the CTA gives up
            if (!ok) break;
            continue;
          }
        }
#pragma unroll 1
        for (int acc = 0; acc < 2; ++acc) {
          ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bars.tmem_full[acc]), nu & 1u, abort_flag));
          if (!ok) break;
          tc_fence_after();
          const uint32_t taddr = taddr0 + kAccCols * acc;
          const int m0 = t.m0 + R * (2 * acc + (int)rank) + 32 * wq;
          const bool in_m = row < R && m0 + lane < p.M;
          // everything this warp wants of the accumulator goes to registers, and the accumulator back to the
          // MMAs, before the stores
#pragma unroll 1
          for (int j = 0; j < kChunks; j += 4) {
            uint32_t v[4][16];
#pragma unroll
            for (int i = 0; i < 4; ++i) tmem_ld16(taddr + 16 * (group + kStride * (j + i)), v[i]);
            tmem_ld_wait();
            if (j + 4 >= kChunks) {
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive_cluster(acc ? empty1 : empty0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int c0 = 16 * (group + kStride * (j + i));
              if (c0 >= t.valid) continue;
              const long long at = (long long)(t.n0 + c0) * ld + m0;
              if (p.S > 1) {
                float* o = p.planes + (long long)t.ks * p.N * ld + at + lane;
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                  if (in_m && c0 + c < t.valid) *o = __uint_as_float(v[i][c]);
                  o += ld;
                }
              } else {
                if (KIND == kPlain && args.residual) {  // y itself, maybe: a store carries only what was added before
                  const uint16_t* r = reinterpret_cast<const uint16_t*>(args.residual) + at + lane;
#pragma unroll
                  for (int c = 0; c < 16; ++c) {
                    if (in_m && c0 + c < t.valid)
                      v[i][c] = __float_as_uint(__uint_as_float(v[i][c]) + unpack16(__ldcg(r), fp16).x);
                    r += ld;
                  }
                }
                uint32_t w[8];
#pragma unroll
                for (int c = 0; c < 8; ++c)
                  w[c] = pack16(__uint_as_float(v[i][2 * c]), __uint_as_float(v[i][2 * c + 1]), fp16);
                store_cols<8>(w, reinterpret_cast<uint16_t*>(p.out) + at, ld, c0, t.valid, in_m, lane);
              }
            }
          }
        }
      }
    }
  }

  teardown_pair(bars, tmem_base, 2 * kAccCols, issued, ns, rank, &g_status);
}

// Lets its successor start at once and takes `ns` itself (moe_test_hold).
__global__ void hold_kernel(unsigned long long ns) {
  pdl_launch_dependents();
  for (const unsigned long long t0 = gtimer(); gtimer() - t0 < ns;) __nanosleep(1000);
}

// Sum of the S planes of a split launch in their order, and what the epilogue would have done with it: four
// neighbouring m a thread, a problem of the launch for each blockIdx.y.
struct Join {
  const float* planes[4];
  long long n[4];  // outputs of a problem
  int S[4];        // 1: nothing to do
  void* out[4];
  const void* residual;
  const float2* saved;  // da: the problem's outputs are dg and du
  void* du;
  int fp16;
};

__device__ __forceinline__ float4 sum_planes(const float* planes, int S, long long n, long long i) {
  float4 v = ld_l2(reinterpret_cast<const float4*>(planes + i));
  for (int s = 1; s < S; ++s) {
    const float4 w = ld_l2(reinterpret_cast<const float4*>(planes + (long long)s * n + i));
    v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
  }
  return v;
}

template <bool DACT> __global__ void __launch_bounds__(256) ffn_join_kernel(const __grid_constant__ Join a) {
  pdl_wait();
  pdl_launch_dependents();  // behind the wait: the launch that follows may read the weights ahead
  const int p = DACT ? 0 : blockIdx.y, fp16 = a.fp16;
  const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= a.n[p] || a.S[p] == 1) return;
  float4 v = sum_planes(a.planes[p], a.S[p], a.n[p], i);
  uint16_t* out = reinterpret_cast<uint16_t*>(a.out[p]) + i;
  if constexpr (!DACT) {
    if (a.residual) {
      const uint2 r = __ldcg(reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(a.residual) + i));
      const float2 r0 = unpack16(r.x, fp16), r1 = unpack16(r.y, fp16);
      v.x += r0.x; v.y += r0.y; v.z += r1.x; v.w += r1.y;
    }
    *reinterpret_cast<uint2*>(out) = make_uint2(pack16(v.x, v.y, fp16), pack16(v.z, v.w, fp16));
  } else {
    const float4 s0 = ld_l2(reinterpret_cast<const float4*>(a.saved + i)), s1 = ld_l2(reinterpret_cast<const float4*>(a.saved + i) + 1);
    *reinterpret_cast<uint2*>(out) = make_uint2(pack16(v.x * s0.x, v.y * s0.z, fp16), pack16(v.z * s1.x, v.w * s1.z, fp16));
    *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.du) + i) =
        make_uint2(pack16(v.x * s0.y, v.y * s0.w, fp16), pack16(v.z * s1.y, v.w * s1.w, fp16));
  }
}

// ------------------------------------------------------------------------------ host

struct Plan {
  int R, n_tile, S, mt, nt;
  bool slim;
};

// The kernel counts items in 32 bits, those of up to four problems together.  The largest sizes that the calls take, 2^24
// tokens of 2^20 by 2^20, are 2^28 items of the largest tile; small tiles of them would be 2^32 and more.
constexpr long long kMostItems = 1 << 29;

// Pipeline of a tile: bytes of an accumulator's rows of A and of a stage, and the stages that fit.
struct Ring {
  int slot_a, stage, tail, stages;
};


// Shared memory of the epilogue of the da launch: two units of 8 columns, 8 bytes a value.
int saved_bytes(int kind, bool slim) { return kind == kDact ? 2 * 8 * 8 * 32 * (slim ? Form<true>::kEpiWarps : Form<false>::kEpiWarps) : 0; }

Ring ring_of(int kind, int R, int n_tile, bool slim) {
  Ring r;
  if (kind == kGrads) {  // what the weights' gradients need, which is the most
    r.slot_a = kAccRows / 64 * (int)kMnBoxBytes;
    r.stage = 2 * r.slot_a + Form<false>::kAccCols / (slim ? 4 : 2) / 64 * (int)kMnBoxBytes;
  } else {
    r.slot_a = a_mn(kind) ? (R + 63) / 64 * (int)kMnBoxBytes : (R + 7) / 8 * 1024;
    r.stage = 2 * r.slot_a + n_tile / 2 * 128;
  }
  // an MMA reads 128 rows of A whatever was loaded: up to 16 KB behind the last slot
  r.tail = std::max(0, kAccRows * 128 - r.slot_a);
  const int smem = slim ? Form<true>::kSmem : Form<false>::kSmem;
  r.stages = std::min(kMaxStages, (smem - 1024 - r.tail - saved_bytes(kind, slim)) / r.stage);
  return r;
}

// Tile and split of a launch of M x N outputs and KB k-blocks, by a model in SM cycles.  A k-block of an item takes
// the largest of
//   4.6 n_tile          the tensor pipe: eight MMAs of n_tile / 2 cycles, which the ring of stages keeps 88 % busy (an MMA of
//                       M = 256 takes about 90 cycles at least, 720 a k-block, which the model knows of the weights'
//                       gradients only: items of few columns and of fewer than 128 rows are reckoned too short),
//   bytes / 7600        what all running pairs draw from L2, 128 bytes for each row of A and column of B
//   bytes / 3800        what they draw from HBM: rows of A that no other running item shares,
//   bytes / 110         what a pair by itself can draw,
//   4500 / stages       the latency of memory, for stages of few bytes
// and an item a fixed part and an epilogue besides; items are dealt to the pairs in rounds, and in the last round
// fewer pairs share the memory.  A split launch writes its planes and the join reads them.  Measured, gate/up launch
// of 4096 tokens (h 4096, f 14336, R 128; cycles per k-block of an item with its epilogue's share, and TB/s from L2):
// n_tile 256 1271, 8.4; 192 969, 11.0; 128 842, 11.4; 64 778, 12.3; 32 746, 12.2.  Rows that are no multiple of 8 leave
// a swizzle atom in part empty and cost 18 % (R 98 against 112, n_tile 256).
bool is_slim(int kind, int M, int N, int KB) {
  if (kind == kGrads) return N <= Form<true>::kAccCols && (long long)M * KB * 32 <= (1 << 19);  // KB: of two segments
  if (N <= 32 && (long long)M * KB * BK * 2 >= ((long long)96 << 20)) return false;
  return N <= 64 || (N <= Form<true>::kAccCols && KB <= 16);
}

Plan search_plan(int kind, int M, int N, int KB, bool may_split, int pairs) {
  const int unit = gate_up(kind) ? 2 : 4;
  Plan best = {};
  double best_cost = 1e300;
  const bool slim = is_slim(kind, M, N, KB);
  const int mt_min = (M + unit * kAccRows - 1) / (unit * kAccRows);
  for (int cols = slim ? Form<true>::kAccCols : 256; cols >= 16; cols -= 16) {
    const int nt = (N + cols - 1) / cols;
    const int n_tile = ((N + nt - 1) / nt + 15) / 16 * 16;
    if (n_tile != cols) continue;  // the same tiles with fewer columns come later
    for (int S = 1; S <= 16 && (S == 1 || (may_split && KB / S >= 4 && (long long)(S - 1) * nt * mt_min < 2 * pairs)); ++S) {
      const int kbs = (KB + S - 1) / S;
      if ((KB + kbs - 1) / kbs != S) continue;
      const long long least = ((long long)mt_min * nt * S + pairs - 1) / pairs;  // rounds
      for (int fill = 0; fill < 2; ++fill) {  // whole tiles, or as many rows as fill the rounds
        int R = kAccRows;
        if (fill) {
          if (a_mn(kind)) {
            R = 64;
          } else {
            const long long most = least * pairs / (nt * S);
            R = (int)((M + unit * most - 1) / (unit * most) + 7) / 8 * 8;
          }
          if (R >= kAccRows) continue;
        }
        const int mt = (M + unit * R - 1) / (unit * R);
        const long long items = (long long)mt * nt * S, full = items / pairs;
        const int rest = (int)(items - full * pairs);
        if (items > kMostItems) continue;
        const int stages = ring_of(kind, R, n_tile, slim).stages;
        auto round = [&](int active) {
          const double l2 = active * (4.0 * R + n_tile) * 128 / 7600.0;
          const double hbm = active * 4.0 * R * 128 / (active < nt ? active : nt) / 3800.0;
          const double own = std::max((4.0 * R + n_tile) * 128 / 110.0, 4500.0 / stages);
          return kbs * std::max(std::max(4.6 * n_tile, own), std::max(l2, hbm)) + 1500.0 + (gate_up(kind) ? 16.0 : 6.0) * n_tile;
        };
        double cost = full * (full ? round(pairs) : 0.0) + (rest ? round(rest) : 0.0);
        if (S > 1) cost += 4500.0 + (double)S * N * M * 8 / 7000.0;
        if (cost < best_cost) {
          best_cost = cost;
          best = {R, n_tile, S, mt, nt, slim};
        }
      }
    }
  }
  return best;
}

// The weights' gradients, three problems of one tile: 512 x 256 where they fill the machine, smaller tiles and splits
// over the tokens where h and f are small and the tokens many.  8192 tokens of (h 128, f 448) in 512 x 256 tiles are five
// items of 128 k-blocks.
Plan search_weights_plan(int T, int h, int f, int pairs, bool slim) {
  const int KB = (T + BK - 1) / BK;
  Plan best = {};
  double best_cost = 1e300;
  for (int n = slim ? Form<true>::kAccCols : Form<false>::kAccCols; n >= 32; n >>= 1)
    for (int R = kAccRows; R >= 64; R -= 64)
      for (int S = 1; S <= 16 && (S == 1 || KB / S >= 2); ++S) {
        const int kbs = (KB + S - 1) / S;
        if ((KB + kbs - 1) / kbs != S) continue;
        auto tiles = [&](int M, int N) { return (long long)((M + 4 * R - 1) / (4 * R)) * ((N + n - 1) / n); };
        const long long items = S * (2 * tiles(h, f) + tiles(f, h));
        if ((S > 1 && items > 4 * pairs) || items > kMostItems) break;
        double cost = (double)((items + pairs - 1) / pairs) * (kbs * std::max(800.0, 4.6 * n) + 2000.0 + 8.0 * n);
        if (S > 1) cost += 4500.0 + 3.0 * S * h * f * 8 / 7000.0;
        if (cost < best_cost) {
          best_cost = cost;
          best = {R, n, S, 0, 0, slim};
        }
      }
  return best;
}

// The same, remembered for the sizes that this thread asked about last: a search takes 1 to 8 us of the host, and a call
// needs each plan two or three times.  Kind -1, -2: the weights' gradients, -2 in the slim form (M: h, N: tokens, KB: f).
Plan choose_plan(int kind, int M, int N, int KB, bool may_split, int pairs) {
  struct Known {
    int kind, M, N, KB, pairs;
    Plan plan;
  };
  static thread_local Known known[32] = {};
  const unsigned hash = (unsigned)M * 0x9e3779b1u ^ (unsigned)N * 0x85ebca6bu ^ (unsigned)KB * 0xc2b2ae35u ^ (unsigned)kind * 0x27d4eb2fu;
  Known& k = known[(hash >> 16) & 31u];
  if (k.kind != kind || k.M != M || k.N != N || k.KB != KB || k.pairs != pairs)
    k = {kind, M, N, KB, pairs, kind < 0 ? search_weights_plan(N, M, KB, pairs, may_split) : search_plan(kind, M, N, KB, may_split, pairs)};
  return k.plan;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Splits the contractions and deals the items; returns how many there are.
int deal_items(int kind, Args& a, int pairs) {
  int items = 0;
  for (int i = 0; i < a.np; ++i) {
    Problem& p = a.p[i];
    p.kbs = (p.KB + p.S - 1) / p.S;
    items += p.mt * p.nt * p.S;
  }
  if (kind == kGrads) {
    // an item of dx against one of the weights' gradients, in cycles: the tensor pipe, or what a pair draws of weights
    // (600 a k-block) and stores (9000 an item)
    const Problem &x = a.p[0], &w = a.p[1];
    const int n = x.mt * x.nt * x.S, grid = std::min(items, pairs);
    a.first = n < grid ? n : 0;
    a.skip = a.first ? (int)(x.kbs * std::max(4.6 * x.n_tile, 600.0) / std::max(std::max(4.6 * w.n_tile, 800.0) * w.kbs + 4000.0, 9000.0)) : 0;
  }
  return items;
}

template <int KIND, bool SLIM> cudaError_t launch_form(const Maps& maps, Args& a, int pairs, cudaStream_t st) {
  const Ring ring = ring_of(KIND, a.p[0].R, a.p[0].n_tile, SLIM);
  a.slot_a = ring.slot_a;
  a.stage = ring.stage;
  a.tail = ring.tail;
  const int items = deal_items(KIND, a, pairs);
  int kbs = 2;
  for (int i = 0; i < a.np; ++i) kbs = std::max(kbs, a.p[i].kbs);
  a.stages = std::min(ring.stages, kbs);
  static std::atomic<unsigned long long> set{0};  // devices on which the kernel may use its shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !(set.load() >> dev & 1)) {
    e = cudaFuncSetAttribute(ffn_gemm_kernel<KIND, SLIM>, cudaFuncAttributeMaxDynamicSharedMemorySize, Form<SLIM>::kSmem);
    if (e != cudaSuccess) return e;
    if (dev < 64) set.fetch_or(1ull << dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * std::min(items, pairs));
  cfg.blockDim = dim3(Form<SLIM>::kThreads);
  cfg.dynamicSmemBytes = 1024 + (size_t)a.stages * a.stage + ring.tail + saved_bytes(KIND, SLIM);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = g_pdl_enabled ? 1 : 0;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, ffn_gemm_kernel<KIND, SLIM>, maps, a);
}

template <int KIND> cudaError_t launch_gemm(const Maps& maps, Args& a, bool slim, int pairs, cudaStream_t st) {
  if (slim) return launch_form<KIND, true>(maps, a, pairs, st);
  return launch_form<KIND, false>(maps, a, pairs, st);
}

// nothing to do where no problem of the launch was split
cudaError_t launch_join(bool dact, const Args& a, cudaStream_t st) {
  Join j = {};
  long long most = 0;
  for (int i = 0; i < a.np; ++i) {
    const Problem& p = a.p[i];
    j.planes[i] = p.planes;
    j.n[i] = (long long)p.M * p.N;
    j.S[i] = p.S;
    j.out[i] = p.out;
    if (p.S > 1) most = std::max(most, j.n[i]);
  }
  if (!most) return cudaSuccess;
  j.residual = a.residual;
  j.saved = a.saved;
  j.du = a.du;
  j.fp16 = a.fp16;
  const dim3 grid((unsigned)((most / 4 + 255) / 256), (unsigned)a.np);
  return dact ? launch_pdl(ffn_join_kernel<true>, grid, dim3(256), 0, st, j) : launch_pdl(ffn_join_kernel<false>, grid, dim3(256), 0, st, j);
}

Problem problem_of(const Plan& p, int M, int N, int KB, void* out) {
  return {M, N, p.mt, p.nt, out, KB, KB, p.S, 0, p.R, p.n_tile, 0, 0, 0, nullptr};
}

Args args_of(const Problem& p, int dtype) {
  Args a = {};
  a.p[0] = p;
  a.np = 1;
  a.fp16 = dtype == MOE_FP16;
  return a;
}

// gradient of a weight matrix [N][M], summed over KB blocks of tokens
Problem weight_gradient(const Plan& p, int M, int N, int KB, void* out, int map) {
  return {M, N, (M + 4 * p.R - 1) / (4 * p.R), (N + p.n_tile - 1) / p.n_tile, out, KB, KB, p.S, 0, p.R, p.n_tile, map, map, 1, nullptr};
}

// Tensor map of one operand: contiguous in k ([rows][K]), boxes of 64 k x box rows, or in m / n ([K][rows]), boxes of
// 64 rows x 64 k.
int map_k(CUtensorMap* m, const void* base, int K, int rows, int box) { return make_map_2d(m, base, K, rows, box); }
int map_mn(CUtensorMap* m, const void* base, int rows, int K) { return make_map_2d(m, base, rows, K, BK); }

int kblocks(int K) { return (K + BK - 1) / BK; }

Plan gu_plan(int T, int h, int f, int pairs) { return choose_plan(kGateUp, f, T, kblocks(h), false, pairs); }
Plan down_plan(int T, int h, int f, int pairs) { return choose_plan(kPlain, h, T, kblocks(f), true, pairs); }
Plan dact_plan(int T, int h, int f, int pairs) { return choose_plan(kDact, f, T, kblocks(h), true, pairs); }
Plan dx_plan(int T, int h, int f, int pairs) { return choose_plan(kGrads, h, T, 2 * kblocks(f), true, pairs); }
Plan weights_plan(int T, int h, int f, int pairs) {
  const bool slim = dx_plan(T, h, f, pairs).slim;  // one launch, one form
  return choose_plan(slim ? -2 : -1, h, T, f, slim, pairs);
}

// The gradients' launch but for its operands and outputs.
Args grads_args(int T, int h, int f, int dtype, int pairs) {
  Args a = args_of(problem_of(dx_plan(T, h, f, pairs), h, T, 2 * kblocks(f), nullptr), dtype);
  a.p[0].segKB = kblocks(f);
  const Plan wp = weights_plan(T, h, f, pairs);
  a.p[1] = weight_gradient(wp, h, f, kblocks(T), nullptr, 2);
  a.p[2] = weight_gradient(wp, h, f, kblocks(T), nullptr, 3);
  a.p[3] = weight_gradient(wp, f, h, kblocks(T), nullptr, 4);
  a.np = 4;
  a.early = 1;
  return a;
}

// the saved buffer: (p, q), then a
size_t pq_bytes(int T, int f) { return round256((size_t)T * f * sizeof(float2)); }

size_t plane_bytes(const Plan& p, int N, int M) { return p.S > 1 ? round256((size_t)p.S * N * M * sizeof(float)) : 0; }

int check_block(int T, int h, int f, int dtype) {
  if (dtype != MOE_BF16 && dtype != MOE_FP16)
    return set_error(MOE_ERR_INVALID_ARG, "dtype = %d is neither MOE_BF16 nor MOE_FP16", dtype);
  if (T < 0 || T > kMaxOperatorTokens) return set_error(MOE_ERR_INVALID_ARG, "T = %d outside 0..%d", T, kMaxOperatorTokens);
  if (h < 8 || f < 8 || h % 8 || f % 8 || h > (1 << 20) || f > (1 << 20))
    return set_error(MOE_ERR_UNSUPPORTED_SHAPE, "h = %d and f = %d must be multiples of 8 in 8..%d", h, f, 1 << 20);
  return MOE_OK;
}

// once per device: the current device can run the kernels, the driver's encoder is there
int check_device() {
  static std::atomic<unsigned long long> good{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return set_error(MOE_ERR_CUDA, "cudaGetDevice: %s", cudaGetErrorString(e));
  if (dev < 64 && (good.load() >> dev & 1)) return MOE_OK;
  int major = 0;
  e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  if (e != cudaSuccess) return set_error(MOE_ERR_CUDA, "cudaDeviceGetAttribute: %s", cudaGetErrorString(e));
  if (major != 10) return set_error(MOE_ERR_ARCH, "device has compute capability %d.x, sm_100 is required", major);
  if (gemm_init_driver_api()) return set_error(MOE_ERR_CUDA, "cuTensorMapEncodeTiled not available");
  if (dev < 64) good.fetch_or(1ull << dev);
  return MOE_OK;
}

#define FFN_TRY(what, expr)                                                                             \
  do {                                                                                                  \
    const cudaError_t e_ = (expr);                                                                      \
    if (e_ != cudaSuccess) return set_error(MOE_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e_));      \
  } while (0)
#define FFN_MAP(expr)                                                                    \
  do {                                                                                   \
    if (expr) return set_error(MOE_ERR_CUDA, "building a tensor map failed: " #expr);    \
  } while (0)

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" {

size_t moe_ffn_saved_bytes(int T, int f) {
  if (T < 1 || T > kMaxOperatorTokens || f < 8 || f % 8 || f > (1 << 20)) return 0;
  return pq_bytes(T, f) + (size_t)T * f * 2;
}

size_t moe_ffn_forward_workspace(int T, int h, int f) {
  if (T < 1 || check_block(T, h, f, MOE_BF16)) return 0;
  return round256((size_t)T * f * 2) + plane_bytes(down_plan(T, h, f, sm_count() / 2), T, h);
}

size_t moe_ffn_backward_workspace(int T, int h, int f) {
  if (T < 1 || check_block(T, h, f, MOE_BF16)) return 0;
  const int pairs = sm_count() / 2;
  return 2 * round256((size_t)T * f * 2) +
         std::max(plane_bytes(dact_plan(T, h, f, pairs), T, f),
                  plane_bytes(dx_plan(T, h, f, pairs), T, h) + 3 * plane_bytes(weights_plan(T, h, f, pairs), f, h));
}

int moe_ffn_forward(const void* x, const void* W1, const void* W3, const void* W2, const void* residual, int T, int h, int f,
                    int dtype, void* y, void* saved, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  int rc = check_block(T, h, f, dtype);
  if (rc) return rc;
  if (T == 0) return MOE_OK;
  if (!x || !W1 || !W3 || !W2 || !y) return set_error(MOE_ERR_INVALID_ARG, "x, W1, W3, W2 or y is NULL");
  if (!aligned16(x) || !aligned16(W1) || !aligned16(W3) || !aligned16(W2) || !aligned16(residual) || !aligned16(y) ||
      !aligned16(saved) || !aligned16(workspace))
    return set_error(MOE_ERR_INVALID_ARG, "every tensor must be 16-byte aligned");
  const size_t n = (size_t)T * h * 2, w = (size_t)h * f * 2, n_saved = moe_ffn_saved_bytes(T, f);
  if (overlap(y, n, x, n) || overlap(y, n, W1, w) || overlap(y, n, W3, w) || overlap(y, n, W2, w) ||
      overlap(y, n, saved, n_saved) || (residual != y && overlap(y, n, residual, n)))
    return set_error(MOE_ERR_INVALID_ARG, "y overlaps another tensor (only the residual itself is allowed)");
  const void* ins[5] = {x, W1, W3, W2, residual};
  const size_t in_bytes[5] = {n, w, w, w, n};
  for (int i = 0; i < 5; ++i)
    if (overlap(ins[i], in_bytes[i], saved, n_saved)) return set_error(MOE_ERR_INVALID_ARG, "saved overlaps an input");
  const size_t need = moe_ffn_forward_workspace(T, h, f);
  if (!workspace || workspace_bytes < need)
    return set_error(MOE_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need);
  for (int i = 0; i < 5; ++i)
    if (overlap(ins[i], in_bytes[i], workspace, need)) return set_error(MOE_ERR_INVALID_ARG, "the workspace overlaps a tensor");
  if (overlap(y, n, workspace, need) || overlap(saved, n_saved, workspace, need))
    return set_error(MOE_ERR_INVALID_ARG, "the workspace overlaps a tensor");
  if ((rc = check_device())) return rc;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int pairs = sm_count() / 2;
  char* ws = static_cast<char*>(workspace);
  void* act = saved ? static_cast<char*>(saved) + pq_bytes(T, f) : ws;
  if (!saved && ffn_few_fits(T, h, f)) {
    FFN_TRY("launch for few tokens", launch_ffn_few(x, W1, W3, W2, residual, T, h, f, dtype, act, y, st));
    return MOE_OK;
  }
  Plan p = gu_plan(T, h, f, pairs);
  Args a = args_of(problem_of(p, f, T, kblocks(h), act), dtype);
  a.saved = static_cast<float2*>(saved);
  Maps maps = {};
  FFN_MAP(map_k(&maps.a[0], W1, h, f, p.R));
  FFN_MAP(map_k(&maps.a[1], W3, h, f, p.R));
  FFN_MAP(map_k(&maps.b[0], x, h, T, p.n_tile / 2));
  FFN_TRY("gate/up launch", saved ? launch_gemm<kGateUpSave>(maps, a, p.slim, pairs, st) : launch_gemm<kGateUp>(maps, a, p.slim, pairs, st));
  p = down_plan(T, h, f, pairs);
  a = args_of(problem_of(p, h, T, kblocks(f), y), dtype);
  a.residual = residual;
  a.early = 1;
  a.p[0].planes = reinterpret_cast<float*>(ws + round256((size_t)T * f * 2));
  FFN_MAP(map_k(&maps.a[0], W2, f, h, p.R));
  FFN_MAP(map_k(&maps.b[0], act, f, T, p.n_tile / 2));
  FFN_TRY("down launch", launch_gemm<kPlain>(maps, a, p.slim, pairs, st));
  FFN_TRY("join launch", launch_join(false, a, st));
  return MOE_OK;
}

int moe_ffn_backward(const void* dy, const void* x, const void* W1, const void* W3, const void* W2, const void* saved, int T,
                     int h, int f, int dtype, void* dx, void* dW1, void* dW3, void* dW2, void* workspace,
                     size_t workspace_bytes, void* cuda_stream) {
  int rc = check_block(T, h, f, dtype);
  if (rc) return rc;
  const size_t n = (size_t)T * h * 2, w = (size_t)h * f * 2;
  if (!dW1 || !dW3 || !dW2) return set_error(MOE_ERR_INVALID_ARG, "dW1, dW3 or dW2 is NULL");
  if (!aligned16(dW1) || !aligned16(dW3) || !aligned16(dW2))
    return set_error(MOE_ERR_INVALID_ARG, "every tensor must be 16-byte aligned");
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  void* outs[4] = {dW1, dW3, dW2, dx};
  const size_t out_bytes[4] = {w, w, w, n};
  const void* ins[6] = {dy, x, W1, W3, W2, saved};
  const size_t in_bytes[6] = {n, n, w, w, w, moe_ffn_saved_bytes(T, f)};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 6; ++j)
      if (overlap(outs[i], out_bytes[i], ins[j], in_bytes[j]))
        return set_error(MOE_ERR_INVALID_ARG, "a gradient overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], out_bytes[i], outs[j], out_bytes[j]))
        return set_error(MOE_ERR_INVALID_ARG, "two gradients overlap");
  }
  if (T == 0) {  // sums of nothing
    for (int i = 0; i < 3; ++i) FFN_TRY("clearing a gradient", cudaMemsetAsync(outs[i], 0, w, st));
    return MOE_OK;
  }
  if (!dy || !x || !W1 || !W3 || !W2 || !saved || !dx)
    return set_error(MOE_ERR_INVALID_ARG, "dy, x, W1, W3, W2, saved or dx is NULL");
  if (!aligned16(dy) || !aligned16(x) || !aligned16(W1) || !aligned16(W3) || !aligned16(W2) || !aligned16(saved) ||
      !aligned16(dx) || !aligned16(workspace))
    return set_error(MOE_ERR_INVALID_ARG, "every tensor must be 16-byte aligned");
  const size_t need = moe_ffn_backward_workspace(T, h, f);
  if (!workspace || workspace_bytes < need)
    return set_error(MOE_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0, need);
  for (int i = 0; i < 6; ++i)
    if (overlap(ins[i], in_bytes[i], workspace, need) || (i < 4 && overlap(outs[i], out_bytes[i], workspace, need)))
      return set_error(MOE_ERR_INVALID_ARG, "the workspace overlaps a tensor");
  if ((rc = check_device())) return rc;
  const int pairs = sm_count() / 2;
  char* ws = static_cast<char*>(workspace);
  const size_t part = round256((size_t)T * f * 2);
  const void* act = static_cast<const char*>(saved) + pq_bytes(T, f);
  void *dg = ws, *du = ws + part;
  char* planes = ws + 2 * part;
  Maps maps = {};
  // da = dy W2, and dg, du
  Plan p = dact_plan(T, h, f, pairs);
  Args a = args_of(problem_of(p, f, T, kblocks(h), dg), dtype);
  a.saved = static_cast<float2*>(const_cast<void*>(saved));
  a.du = du;
  a.p[0].planes = reinterpret_cast<float*>(planes);
  FFN_MAP(map_mn(&maps.a[0], W2, f, h));
  FFN_MAP(map_k(&maps.b[0], dy, h, T, p.n_tile / 2));
  FFN_TRY("da launch", launch_gemm<kDact>(maps, a, p.slim, pairs, st));
  FFN_TRY("join launch", launch_join(true, a, st));
  // dx = dg W1 + du W3; dW1 = dg^T x, dW3 = du^T x (rows f, contiguous h), dW2 = dy^T a (rows h, contiguous f)
  p = dx_plan(T, h, f, pairs);
  a = grads_args(T, h, f, dtype, pairs);
  void* grads[4] = {dx, dW1, dW3, dW2};
  for (int i = 0; i < 4; ++i) {
    a.p[i].out = grads[i];
    a.p[i].planes = reinterpret_cast<float*>(planes);
    planes += i ? plane_bytes(weights_plan(T, h, f, pairs), f, h) : plane_bytes(p, T, h);
  }
  FFN_MAP(map_mn(&maps.a[0], W1, h, f));
  FFN_MAP(map_mn(&maps.a[1], W3, h, f));
  FFN_MAP(map_mn(&maps.a[2], x, h, T));
  maps.a[3] = maps.a[2];
  FFN_MAP(map_mn(&maps.a[4], act, f, T));
  FFN_MAP(map_k(&maps.b[0], dg, f, T, p.n_tile / 2));
  FFN_MAP(map_k(&maps.b[1], du, f, T, p.n_tile / 2));
  FFN_MAP(map_mn(&maps.b[2], dg, f, T));
  FFN_MAP(map_mn(&maps.b[3], du, f, T));
  FFN_MAP(map_mn(&maps.b[4], dy, h, T));
  FFN_TRY("gradients launch", launch_gemm<kGrads>(maps, a, p.slim, pairs, st));
  FFN_TRY("join launch", launch_join(false, a, st));
  return MOE_OK;
}

int moe_test_ffn_plan(int launch, int T, int h, int f, int pairs, int plan[6]) {
  if (T < 1 || pairs < 1 || !plan || launch < 0 || launch > 4 || check_block(T, h, f, MOE_BF16))
    return set_error(MOE_ERR_INVALID_ARG, "bad launch, sizes or pairs");
  const Plan p = launch == 0   ? gu_plan(T, h, f, pairs)
                 : launch == 1 ? down_plan(T, h, f, pairs)
                 : launch == 2 ? dact_plan(T, h, f, pairs)
                 : launch == 3 ? dx_plan(T, h, f, pairs)
                               : weights_plan(T, h, f, pairs);
  const int kb = launch == 4 ? kblocks(T) : launch == 0 || launch == 2 ? kblocks(h) : kblocks(f) * (launch == 3 ? 2 : 1);
  const int v[6] = {p.R, p.n_tile, p.S, p.mt, p.nt, kb};
  for (int i = 0; i < 6; ++i) plan[i] = v[i];
  return MOE_OK;
}

int moe_test_ffn_deal(int T, int h, int f, int pairs, int pair, int* items, int most, int deal[3]) {
  if (T < 1 || pairs < 1 || !items || !deal || most < 0 || check_block(T, h, f, MOE_BF16))
    return set_error(MOE_ERR_INVALID_ARG, "bad sizes or pairs");
  Args a = grads_args(T, h, f, MOE_BF16, pairs);
  const int total = deal_items(kGrads, a, pairs), grid = std::min(total, pairs);
  if (pair < 0 || pair >= grid) return set_error(MOE_ERR_INVALID_ARG, "pair = %d of %d", pair, grid);
  int n = 0;
  for (int item; (item = item_of<kGrads>(a, n, pair, grid)) < total; ++n)
    if (n < most) items[n] = item;
  deal[0] = total;
  deal[1] = n;
  deal[2] = item_ahead<kGrads>(a, pair, grid, total);
  return MOE_OK;
}

int moe_test_operators_expiry(unsigned limit_us, void* cuda_stream) {
  if (limit_us < 1 || limit_us > 100000) return set_error(MOE_ERR_INVALID_ARG, "limit_us = %u outside 1..100000", limit_us);
  int rc = check_device();
  if (rc) return rc;
  void* status = nullptr;
  FFN_TRY("the status word's address", cudaGetSymbolAddress(&status, g_status));
  FFN_TRY("launch", launch_wait_expiry_pair(static_cast<int*>(status), (unsigned long long)limit_us * 1000ull, 0,
                                            static_cast<cudaStream_t>(cuda_stream)));
  return MOE_OK;
}

int moe_test_hold(unsigned ms, void* cuda_stream) {
  if (ms < 1 || ms > 6000) return set_error(MOE_ERR_INVALID_ARG, "ms = %u outside 1..6000", ms);
  FFN_TRY("launch", launch_plain(hold_kernel, dim3(1), dim3(1), 0, static_cast<cudaStream_t>(cuda_stream), ms * 1000000ull));
  return MOE_OK;
}

int moe_operators_status(void) {
  int v = 0, zero = 0;
  FFN_TRY("waiting for the device", cudaDeviceSynchronize());
  FFN_TRY("reading the status", cudaMemcpyFromSymbol(&v, g_status, sizeof(v)));
  if (!v) return MOE_OK;
  FFN_TRY("clearing the status", cudaMemcpyToSymbol(g_status, &zero, sizeof(zero)));
  return set_error(MOE_ERR_DEVICE_TIMEOUT, "a bounded wait inside a kernel expired");
}

}  // extern "C"

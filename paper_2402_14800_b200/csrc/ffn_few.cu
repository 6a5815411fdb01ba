// The dense feed-forward block for few tokens, without pipelines to set up: one and two tokens on the CUDA cores, up
// to 32 on the warp-level matrix instructions.
//
//   a = silu(x W1^T) * (x W3^T),  y = a W2^T [+ residual]
//
// With few tokens the weights' way from HBM is all that counts, or on small layers the latency of two launches.  So
// these kernels only keep plain 16-byte loads in flight, eight a lane; they take no tensor memory, no TMA and leave
// no partial sums, which is what costs the tensor-core launches of ffn_sm100.cu a fifth of their time at one token
// and most of it on a small layer.  The down launch starts while the gate/up launch drains and has its first weights
// in registers before it waits for a.  Sums are fp32 in a fixed order, a is rounded to the tensors' type.
//
//   ffn_gemv_*    a warp takes a feature (its rows of W1 and W3) or an output (a row of W2); rows are dealt over the
//                 SMs in turn, and the warps of a block follow from the rows an SM gets, so that the last round is full.
//   ffn_mma_*     a block takes a run of rows, a warp 16 of them (8 features: rows of W1 and the same of W3) and a
//                 part of the contraction; the parts are added up in shared memory in their order.  A lane's 16 bytes
//                 are 8 neighbouring k of one row.  Which k an instruction's slots mean is free as long as both
//                 operands agree, so they go into the fragments as they lie in memory, and the tokens' likewise.
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

#include "ffn.h"

namespace moe {

namespace {

constexpr int kGemvTokens = 2;  // with more the CUDA cores' instructions bound the streaming (4 tokens 72 us, 2 tokens 56)
constexpr int kMostWarps = 28;
constexpr int kLeastWarps = 16;
// Tokens' rows in shared memory at most.  What they take is L1's loss, and the loads in flight, 114 KB with 28 warps,
// live in L1: 7 tokens of 14336 columns (200 KB) took 96 us, on the tensor cores 68.
constexpr int kMostSmem = 100 * 1024;

template <typename T> __device__ __forceinline__ float2 pair_of(uint32_t v);
template <> __device__ __forceinline__ float2 pair_of<__nv_bfloat16>(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 pair_of<__half>(uint32_t v) {
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
template <typename T> __device__ __forceinline__ T round_to(float v);
template <> __device__ __forceinline__ __nv_bfloat16 round_to(float v) { return __float2bfloat16(v); }
template <> __device__ __forceinline__ __half round_to(float v) { return __float2half(v); }

// acc += the products of 8 elements, in their order
template <typename T> __device__ __forceinline__ float dot8(const uint4& a, const uint4& w, float acc) {
  const uint32_t av[4] = {a.x, a.y, a.z, a.w}, wv[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = pair_of<T>(av[i]), q = pair_of<T>(wv[i]);
    acc = fmaf(p.x, q.x, acc);
    acc = fmaf(p.y, q.y, acc);
  }
  return acc;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}

// rows of n 16-byte vectors to shared memory, zeros for tokens that do not exist
template <int NT> __device__ __forceinline__ void stage_rows(uint4* s, const void* rows, int tokens, int nvec) {
  for (int v = threadIdx.x; v < NT * nvec; v += blockDim.x)
    s[v] = v < tokens * nvec ? ld_l2(reinterpret_cast<const uint4*>(rows) + v) : make_uint4(0, 0, 0, 0);
  __syncthreads();
}

template <typename T, int NT>
__global__ void __launch_bounds__(32 * kMostWarps, 1)
ffn_gemv_gate_up_kernel(const void* x, const uint4* W1, const uint4* W3, int tokens, int h, int f, T* act) {
  extern __shared__ uint4 s_x[];
  pdl_wait();
  pdl_launch_dependents();  // behind the wait: the down launch may read its weights ahead
  const int nvec = h >> 3, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int step = gridDim.x * (blockDim.x >> 5);
  stage_rows<NT>(s_x, x, tokens, nvec);
  for (int j = blockIdx.x + gridDim.x * warp; j < f; j += step) {
    const uint4 *g = W1 + (size_t)j * nvec, *u = W3 + (size_t)j * nvec;
    float ag[NT] = {}, au[NT] = {};
    int v = lane;
    for (; v + 96 < nvec; v += 128) {
      uint4 wg[4], wu[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        wg[k] = __ldcg(g + v + 32 * k);
        wu[k] = __ldcg(u + v + 32 * k);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const uint4 xv = s_x[t * nvec + v + 32 * k];
          ag[t] = dot8<T>(xv, wg[k], ag[t]);
          au[t] = dot8<T>(xv, wu[k], au[t]);
        }
      }
    }
    for (; v < nvec; v += 32) {
      const uint4 wg = __ldcg(g + v), wu = __ldcg(u + v);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        ag[t] = dot8<T>(s_x[t * nvec + v], wg, ag[t]);
        au[t] = dot8<T>(s_x[t * nvec + v], wu, au[t]);
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const float gt = warp_sum(ag[t]), ut = warp_sum(au[t]);
      if (lane == 0 && t < tokens) act[(size_t)t * f + j] = round_to<T>(gt * ffn_sigmoid(gt) * ut);
    }
  }
}

template <typename T, int NT>
__global__ void __launch_bounds__(32 * kMostWarps, 1)
ffn_gemv_down_kernel(const T* act, const uint4* W2, const T* residual, int tokens, int h, int f, T* y) {
  extern __shared__ uint4 s_a[];
  const int nvec = f >> 3, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int step = gridDim.x * (blockDim.x >> 5);
  int n = blockIdx.x + gridDim.x * warp;
  uint4 w[8];
  if (n < h) {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (lane + 32 * k < nvec) w[k] = __ldcg(W2 + (size_t)n * nvec + lane + 32 * k);
  }
  pdl_wait();
  pdl_launch_dependents();
  stage_rows<NT>(s_a, act, tokens, nvec);
  for (bool first = true; n < h; n += step, first = false) {
    const uint4* row = W2 + (size_t)n * nvec;
    float acc[NT] = {};
    for (int v = lane; v < nvec; v += 256) {
      if (!first || v != lane) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (v + 32 * k < nvec) w[k] = __ldcg(row + v + 32 * k);
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (v + 32 * k < nvec) {
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[t] = dot8<T>(s_a[t * nvec + v + 32 * k], w[k], acc[t]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float z = warp_sum(acc[t]);
      if (lane == 0 && t < tokens) {
        const size_t at = (size_t)t * h + n;
        if (residual) {
          const uint32_t r = __ldcg(reinterpret_cast<const unsigned short*>(residual) + at);
          z += pair_of<T>(r).x;
        }
        y[at] = round_to<T>(z);
      }
    }
  }
}

// Warps of a block: of those that deal `rows` rows of an SM in full rounds, the most.
int warps_for(int rows) {
  if (rows <= kMostWarps) return std::max(rows, kLeastWarps);
  int best = kMostWarps, least = 1 << 30;
  for (int w = kMostWarps; w >= kLeastWarps; --w) {
    const int dealt = (rows + w - 1) / w * w;
    if (dealt < least) {
      least = dealt;
      best = w;
    }
  }
  return best;
}

template <typename T, int NT>
cudaError_t launch_as(const void* x, const void* W1, const void* W3, const void* W2, const void* residual, int tokens, int h,
                      int f, void* act, void* y, cudaStream_t st) {
  static std::atomic<unsigned long long> set{0};  // devices on which the kernels may use their shared memory
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !(set.load() >> dev & 1)) {
    e = cudaFuncSetAttribute(ffn_gemv_gate_up_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(ffn_gemv_down_kernel<T, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
    if (e != cudaSuccess) return e;
    if (dev < 64) set.fetch_or(1ull << dev);
  }
  const int sms = sm_count();
  const int gu = warps_for((f + sms - 1) / sms), dn = warps_for((h + sms - 1) / sms);
  e = launch_pdl(ffn_gemv_gate_up_kernel<T, NT>, dim3(std::min(sms, f)), dim3(32 * gu), (size_t)NT * h * 2, st, x,
                 (const uint4*)W1, (const uint4*)W3, tokens, h, f, (T*)act);
  if (e != cudaSuccess) return e;
  return launch_pdl(ffn_gemv_down_kernel<T, NT>, dim3(std::min(sms, h)), dim3(32 * dn), (size_t)NT * f * 2, st, (const T*)act,
                    (const uint4*)W2, (const T*)residual, tokens, h, f, (T*)y);
}

// ------------------------------------------------------------------- matrix instructions

template <typename T>
__device__ __forceinline__ void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
#define FFN_MMA(TYPE, NAME)                                                                                        \
  template <>                                                                                                      \
  __device__ __forceinline__ void mma16816<TYPE>(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,     \
                                                 uint32_t b0, uint32_t b1) {                                       \
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32." NAME "." NAME ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "      \
                 "{%8,%9}, {%0,%1,%2,%3};"                                                                         \
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])                                                  \
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));                                          \
  }
FFN_MMA(__nv_bfloat16, "bf16")
FFN_MMA(__half, "f16")
#undef FFN_MMA

// Bytes of a token's row in shared memory: 64 more than a multiple of 128, so that the eight lanes that a 16-byte
// load serves at once, two tokens of four vectors, lie in different banks.
__host__ __device__ inline int mma_pitch(int K) { return (K * 2 + 127) / 128 * 128 + 64; }

struct MmaArgs {
  const void* x;               // [tokens][K]
  const uint4 *A0, *A1;        // rows of W1 and W3, or W2 twice
  const void* residual;
  void* out;                   // [tokens][M]
  int tokens, M, K, splits;    // parts of the contraction
};

// GATE_UP: tiles of 8 features, else of 16 rows.
template <typename T, int NB, bool GATE_UP>
__global__ void __launch_bounds__(32 * kMostWarps, 1) ffn_mma_kernel(const MmaArgs a) {
  extern __shared__ uint4 s_x[];
  constexpr int kRows = GATE_UP ? 8 : 16;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int r = lane >> 2, kq = lane & 3;
  const int nvec = a.K >> 3, units = (a.K + 31) >> 5, pitch = mma_pitch(a.K) / 16;
  const int lo = (int)((long long)a.M * blockIdx.x / gridDim.x), hi = (int)((long long)a.M * (blockIdx.x + 1) / gridDim.x);
  const int tiles = (hi - lo + kRows - 1) / kRows;
  const int part = warp % a.splits, tile0 = warp / a.splits, tile_step = warps / a.splits;
  const int u0 = (int)((long long)units * part / a.splits), u1 = (int)((long long)units * (part + 1) / a.splits);
  // four units of 32 k: two rows of 16 bytes each
  auto fetch = [&](uint4 (&w)[8], int tile, int u) {
    const int m0 = lo + tile * kRows + r, m1 = GATE_UP ? m0 : m0 + 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int v = (u + i) * 4 + kq;
      const bool in = u + i < u1 && v < nvec;
      w[2 * i] = in && m0 < hi ? __ldcg(a.A0 + (size_t)m0 * nvec + v) : make_uint4(0, 0, 0, 0);
      w[2 * i + 1] = in && m1 < hi ? __ldcg(a.A1 + (size_t)m1 * nvec + v) : make_uint4(0, 0, 0, 0);
    }
  };
  uint4 w[8];
  if (!GATE_UP) fetch(w, tile0, u0);  // weights: nothing that the launch before this one writes
  pdl_wait();
  pdl_launch_dependents();  // behind the wait: the down launch may read its weights ahead
  if (GATE_UP) fetch(w, tile0, u0);
  for (int i = threadIdx.x; i < a.tokens * pitch; i += blockDim.x) {
    const int t = i / pitch, v = i - t * pitch;
    s_x[i] = v < nvec ? ld_l2(reinterpret_cast<const uint4*>(a.x) + (size_t)t * nvec + v) : make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  // More than one round only without splits.  With them every warp goes through the one round and its barriers: a block
  // of fewer tiles than the largest has warps whose rows all lie behind its last, which load and store nothing.
  for (int tile = tile0; a.splits > 1 ? tile == tile0 : tile < tiles; tile += tile_step) {
    float d[NB][4] = {};
    for (int u = u0; u < u1; u += 4) {
      if (u != u0 || tile != tile0) fetch(w, tile, u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (u + i >= u1) break;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const int t = min(8 * b + r, a.tokens - 1);  // a token behind the last is one more column that is not stored
          const uint4 xv = s_x[t * pitch + (u + i) * 4 + kq];
          mma16816<T>(d[b], w[2 * i].x, w[2 * i + 1].x, w[2 * i].y, w[2 * i + 1].y, xv.x, xv.y);
          mma16816<T>(d[b], w[2 * i].z, w[2 * i + 1].z, w[2 * i].w, w[2 * i + 1].w, xv.z, xv.w);
        }
      }
    }
    if (a.splits > 1) {  // a single round: the tokens' rows have been read, their place takes the sums
      float* sums = reinterpret_cast<float*>(s_x);
      __syncthreads();
#pragma unroll
      for (int b = 0; b < NB; ++b)
        *reinterpret_cast<float4*>(sums + ((size_t)(warp * NB + b) * 32 + lane) * 4) = make_float4(d[b][0], d[b][1], d[b][2], d[b][3]);
      __syncthreads();
      if (part) break;
      for (int p = 1; p < a.splits; ++p)
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const float4 o = *reinterpret_cast<const float4*>(sums + ((size_t)((warp + p) * NB + b) * 32 + lane) * 4);
          d[b][0] += o.x; d[b][1] += o.y; d[b][2] += o.z; d[b][3] += o.w;
        }
    }
    // d[b]: row r for tokens 8 b + 2 kq and the next, row r + 8 for the same
    const int m0 = lo + tile * kRows + r;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int t = 8 * b + 2 * kq + j;
        if (t >= a.tokens) continue;
        T* out = reinterpret_cast<T*>(a.out) + (size_t)t * a.M;
        if (GATE_UP) {
          const float g = d[b][j];
          if (m0 < hi) out[m0] = round_to<T>(g * ffn_sigmoid(g) * d[b][2 + j]);
        } else {
          const unsigned short* res = reinterpret_cast<const unsigned short*>(a.residual) + (size_t)t * a.M;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int m = m0 + 8 * q;
            if (m >= hi) continue;
            float z = d[b][2 * q + j];
            if (a.residual) z += pair_of<T>(__ldcg(res + m)).x;
            out[m] = round_to<T>(z);
          }
        }
      }
    }
  }
}

template <typename T, int NB, bool GATE_UP> cudaError_t launch_mma(MmaArgs a, cudaStream_t st) {
  static std::atomic<unsigned long long> set{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 64 || !(set.load() >> dev & 1)) {
    e = cudaFuncSetAttribute(ffn_mma_kernel<T, NB, GATE_UP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostSmem);
    if (e != cudaSuccess) return e;
    if (dev < 64) set.fetch_or(1ull << dev);
  }
  constexpr int kRows = GATE_UP ? 8 : 16;
  const int grid = std::min(sm_count(), (a.M + kRows - 1) / kRows);
  const int tiles = ((a.M + grid - 1) / grid + kRows - 1) / kRows;  // of the largest block
  a.splits = std::max(1, std::min(kMostWarps / tiles, (a.K + 31) / 32));
  const int warps = std::min(kMostWarps, tiles * a.splits);
  const size_t smem = std::max((size_t)a.tokens * mma_pitch(a.K), a.splits > 1 ? (size_t)warps * NB * 512 : 0);
  return launch_pdl(ffn_mma_kernel<T, NB, GATE_UP>, dim3(grid), dim3(32 * warps), smem, st, a);
}

template <typename T, bool GATE_UP> cudaError_t launch_mma_for(const MmaArgs& a, cudaStream_t st) {
  if (a.tokens <= 8) return launch_mma<T, 1, GATE_UP>(a, st);
  if (a.tokens <= 16) return launch_mma<T, 2, GATE_UP>(a, st);
  return launch_mma<T, 4, GATE_UP>(a, st);
}

template <typename T>
cudaError_t launch_type(const void* x, const void* W1, const void* W3, const void* W2, const void* residual, int tokens, int h,
                        int f, void* act, void* y, cudaStream_t st) {
  if (tokens == 1) return launch_as<T, 1>(x, W1, W3, W2, residual, tokens, h, f, act, y, st);
  if (tokens <= kGemvTokens) return launch_as<T, 2>(x, W1, W3, W2, residual, tokens, h, f, act, y, st);
  const cudaError_t e =
      launch_mma_for<T, true>({x, (const uint4*)W1, (const uint4*)W3, nullptr, act, tokens, f, h, 0}, st);
  if (e != cudaSuccess) return e;
  return launch_mma_for<T, false>({act, (const uint4*)W2, (const uint4*)W2, residual, y, tokens, h, f, 0}, st);
}

}  // namespace

bool ffn_few_fits(int tokens, int h, int f) {
  if (tokens <= kGemvTokens) return (size_t)tokens * std::max(h, f) * 2 <= kMostSmem;
  return tokens <= kFfnFewTokens && (size_t)tokens * mma_pitch(std::max(h, f)) <= kMostSmem;
}

cudaError_t launch_ffn_few(const void* x, const void* W1, const void* W3, const void* W2, const void* residual, int tokens,
                           int h, int f, int dtype, void* act, void* y, cudaStream_t st) {
  return dtype == MOE_FP16 ? launch_type<__half>(x, W1, W3, W2, residual, tokens, h, f, act, y, st)
                           : launch_type<__nv_bfloat16>(x, W1, W3, W2, residual, tokens, h, f, act, y, st);
}

}  // namespace moe

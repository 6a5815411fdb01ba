// Residual addition with RMS norm: forward, forward with an 8-bit output, backward.
//
//   s   = T(x + r)                      the residual stream, held in the tensors' type T
//   out = s * rstd * gain,              rstd = 1 / sqrt(mean(s^2) + eps)
//   q   = e4m3(v / scale), v = (s * gain) * rstd in fp32, scale = max |v| / 448 over a row or 128 columns of it
//   dx  = d_s + rstd * (g - hat * mean(g * hat)),   hat = s * rstd,  g = d_out * gain
//   dgain = sum over rows of d_out * hat
//
// The norm is taken of s as it is held, so that the backward pass and the next layer, which read s from
// memory, see the value that was normalised.  Sums, rstd, the gradient of the gain and everything between
// load and store are fp32; each output is rounded once.
//
// All of it is bound by HBM: one row is read once into registers, reduced, and written.  A group of TPR
// threads owns a row and keeps NV 16-byte vectors of each operand a thread; blocks are persistent, so the
// gain stays in registers over all rows of a block (a gain that is read through L2 for every row adds half
// of the operands' traffic: under the rule of launch_pdl it may not come from L1), and the next row's loads
// are issued before the current row is reduced.  Rows that 16 bytes do not divide take the same kernels with
// one element a vector; rows beyond what the registers hold (NV = 0) are read a second time, from s.
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "moe_test_hooks.h"
#include "operators.h"

namespace moe {

namespace {

constexpr float kE4m3Max = 448.f;
constexpr float kMinScale = 1.17549435e-38f;  // smallest normal number: a group of zeros has a scale that divides

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float to_f(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_f(float v) { return __float2bfloat16(v); }
template <> __device__ __forceinline__ __half from_f(float v) { return __float2half(v); }
template <> __device__ __forceinline__ float from_f(float v) { return v; }

template <int BYTES> struct Raw;
template <> struct Raw<16> { typedef uint4 type; };
template <> struct Raw<4> { typedef uint32_t type; };
template <> struct Raw<2> { typedef unsigned short type; };

// E elements as they travel: one load or store
template <typename T, int E> struct Vec {
  typename Raw<E * (int)sizeof(T)>::type raw;
  __device__ __forceinline__ float get(int i) const { return to_f(reinterpret_cast<const T*>(&raw)[i]); }
  __device__ __forceinline__ void set(int i, float v) { reinterpret_cast<T*>(&raw)[i] = from_f<T>(v); }
  __device__ __forceinline__ void load(const T* p) {  // L2: the rule of launch_pdl
    raw = __ldcg(reinterpret_cast<const decltype(raw)*>(p));
  }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<decltype(raw)*>(p) = raw; }
};

// Sum (or maximum of non-negative values) over the TPR threads of a row; every thread gets the same bits.
// `part` holds one float per warp; the caller alternates two of them, so that the barrier of one reduction
// stands between the reads of the one before it and the writes of the one behind it.
template <int TPR, bool MAX> __device__ __forceinline__ float row_reduce(float v, float* part) {
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    const float o = __shfl_xor_sync(0xffffffffu, v, s);
    v = MAX ? fmaxf(v, o) : v + o;
  }
  if (TPR == 32) return v;
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  constexpr int kWarps = TPR / 32;
  float t = part[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) t = MAX ? fmaxf(t, part[w]) : t + part[w];
  return t;
}

// Both at once, behind one barrier: the sum and the maximum (of non-negative values) of a row.
template <int TPR> __device__ __forceinline__ void row_reduce_both(float& sum, float& most, float* part, float* part_most) {
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, s);
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
  }
  if (TPR == 32) return;
  if ((threadIdx.x & 31) == 0) {
    part[threadIdx.x >> 5] = sum;
    part_most[threadIdx.x >> 5] = most;
  }
  __syncthreads();
  sum = part[0];
  most = part_most[0];
#pragma unroll
  for (int w = 1; w < TPR / 32; ++w) {
    sum += part[w];
    most = fmaxf(most, part_most[w]);
  }
}

struct NormArgs {
  const void* x;
  const void* r;     // or null
  const void* gain;  // or null: 1
  void* out;         // T, or e4m3
  void* s;           // null where r is
  float* rstd;       // or null
  float* scales;     // e4m3
  int T, h, group;   // group: 0 = one scale a row, else 128
  float eps;
};

// Rows per block: 256 / 32 with a warp a row, else one.
template <int TPR> struct Shape {
  static constexpr int kThreads = TPR == 32 ? 256 : TPR;
  static constexpr int kRows = kThreads / TPR;
};

// amax of the group a vector belongs to; lanes whose vector lies behind the row pass 0.
// A group of 128 columns is 128 / E neighbouring vectors, 16 or 32 lanes of a warp.
template <int E> __device__ __forceinline__ float group_max(float v) {
#pragma unroll
  for (int s = 64 / E; s > 0; s >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, s));
  return v;
}

// Scale of a group and the factor that takes p = s * gain to q.  rstd cancels in v / scale: with m = max |p| it is
// p * (448 / m), two roundings where v / scale has five (of 16-bit types p is exact in fp32), and one division a
// group.  Groups whose scale is at its lower limit, whose 448 / m is no number, or whose rstd is none (a NaN in the
// row) take v / scale itself: factor 0.  With s * gain beyond fp32 v is infinite although rstd might bring it back;
// taking the maximum of s * rstd * gain for such groups alone cost all others 2-16 % in registers (8000 x 2048 fp16 in
// groups of 128 20.4 -> 22.4 us, 30000 x 1536 bf16 a scale a row 72.7 -> 81.0).
__device__ __forceinline__ float2 scale_of(float m, float rstd) {
  const float scale = fmaxf(m * rstd / kE4m3Max, kMinScale), f = kE4m3Max / m;
  return make_float2(scale, scale > kMinScale && f < 3.0e38f ? f : 0.f);
}

template <int E> __device__ __forceinline__ void store_e4m3(uint8_t* q, float* p, float2 sc, float rstd) {
  if (sc.y > 0.f) {
#pragma unroll
    for (int i = 0; i < E; ++i) p[i] *= sc.y;
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) p[i] = p[i] * rstd / sc.x;
  }
  if constexpr (E == 1) {
    *q = (uint8_t)__nv_cvt_float_to_fp8(p[0], __NV_SATFINITE, __NV_E4M3);
  } else {
    uint32_t w[E / 4] = {};
#pragma unroll
    for (int i = 0; i < E; i += 2)
      w[i / 4] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(p[i], p[i + 1]), __NV_SATFINITE, __NV_E4M3) << (8 * (i & 3));
    if constexpr (E == 8) *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(q) = w[0];
  }
}

template <typename T, int E, int TPR, int NV, bool Q>
__global__ void __launch_bounds__(Shape<TPR>::kThreads) add_rmsnorm_kernel(const NormArgs a) {
  typedef Vec<T, E> V;
  __shared__ float part[2][32], most[2][32];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x % TPR;
  const int h = a.h, nvec = h / E;
  const T* gp = reinterpret_cast<const T*>(a.gain);
  const bool add = a.r != nullptr;
  int row = blockIdx.x * Shape<TPR>::kRows + threadIdx.x / TPR;
  const int step = gridDim.x * Shape<TPR>::kRows;

  if constexpr (NV > 0) {
    V gain[NV], x[NV], r[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = i * TPR + lane;
      if (gp && v < nvec) {
        gain[i].load(gp + v * E);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) gain[i].set(k, 1.f);
      }
    }
    auto fetch = [&](int t) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int v = i * TPR + lane;
        if (t < a.T && v < nvec) {
          const size_t o = (size_t)t * h + (size_t)v * E;
          x[i].load(reinterpret_cast<const T*>(a.x) + o);
          if (add) r[i].load(reinterpret_cast<const T*>(a.r) + o);
        }
      }
    };
    fetch(row);
    int odd = 0;
    // the rows of a block end together: a row behind the last one is reduced with the others and left out
    for (int base = blockIdx.x * Shape<TPR>::kRows; base < a.T; base += step, row += step, odd ^= 1) {
      const bool live = row < a.T;
      V s[NV];
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (add) {
#pragma unroll
          for (int k = 0; k < E; ++k) s[i].set(k, x[i].get(k) + r[i].get(k));
        } else {
          s[i] = x[i];
        }
        if (live && i * TPR + lane < nvec) {
#pragma unroll
          for (int k = 0; k < E; ++k) ss = fmaf(s[i].get(k), s[i].get(k), ss);
        }
      }
      fetch(row + step);
      // the largest |s * gain| needs no rstd: one reduction for both
      float mx[Q ? NV : 1], all = 0.f;
      if constexpr (Q) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          mx[i] = 0.f;
          if (live && i * TPR + lane < nvec) {
#pragma unroll
            for (int k = 0; k < E; ++k) mx[i] = fmaxf(mx[i], fabsf(s[i].get(k) * gain[i].get(k)));
          }
          if constexpr (E > 1) {
            if (a.group) mx[i] = group_max<E>(mx[i]);
          }
          all = fmaxf(all, mx[i]);
        }
      }
      if (Q && !a.group) row_reduce_both<TPR>(ss, all, part[odd], most[odd]);
      else ss = row_reduce<TPR, false>(ss, part[odd]);
      const float rstd = 1.0f / sqrtf(ss / (float)h + a.eps);
      if (live && lane == 0 && a.rstd) a.rstd[row] = rstd;
      if constexpr (!Q) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int v = i * TPR + lane;
          if (!live || v >= nvec) continue;
          const size_t o = (size_t)row * h + (size_t)v * E;
          if (add) s[i].store(reinterpret_cast<T*>(a.s) + o);
          V y;
#pragma unroll
          for (int k = 0; k < E; ++k) y.set(k, s[i].get(k) * rstd * gain[i].get(k));
          y.store(reinterpret_cast<T*>(a.out) + o);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          const int v = i * TPR + lane;
          if (!live || v >= nvec) continue;
          const size_t o = (size_t)row * h + (size_t)v * E;
          if (add) s[i].store(reinterpret_cast<T*>(a.s) + o);
          const float2 sc = scale_of(a.group ? mx[i] : all, rstd);
          float p[E];
#pragma unroll
          for (int k = 0; k < E; ++k) p[k] = s[i].get(k) * gain[i].get(k);
          store_e4m3<E>(reinterpret_cast<uint8_t*>(a.out) + o, p, sc, rstd);
          if (a.group) {
            if (v % (128 / E) == 0) a.scales[(size_t)row * (h / 128) + v / (128 / E)] = sc.x;
          } else if (v == 0) {
            a.scales[row] = sc.x;
          }
        }
      }
    }
  } else {
    // rows of any length: the sum is written in the first pass and read back by the thread that wrote it
    for (; row < a.T; row += step) {
      const T* xp = reinterpret_cast<const T*>(a.x) + (size_t)row * h;
      const T* rp = reinterpret_cast<const T*>(a.r) + (size_t)row * h;
      T* sp = reinterpret_cast<T*>(a.s) + (size_t)row * h;
      float ss = 0.f;
      for (int v = lane; v < nvec; v += TPR) {
        V x, r;
        x.load(xp + (size_t)v * E);
        if (add) {
          r.load(rp + (size_t)v * E);
#pragma unroll
          for (int k = 0; k < E; ++k) x.set(k, x.get(k) + r.get(k));
          x.store(sp + (size_t)v * E);
        }
#pragma unroll
        for (int k = 0; k < E; ++k) ss = fmaf(x.get(k), x.get(k), ss);
      }
      ss = row_reduce<TPR, false>(ss, part[0]);
      const float rstd = 1.0f / sqrtf(ss / (float)h + a.eps);
      if (lane == 0 && a.rstd) a.rstd[row] = rstd;
      const T* hp = add ? sp : xp;
      auto value = [&](int v, float* y) {
        V s, g;
        s.load(hp + (size_t)v * E);
        if (gp) g.load(gp + (size_t)v * E);
#pragma unroll
        for (int k = 0; k < E; ++k) y[k] = (Q ? s.get(k) : s.get(k) * rstd) * (gp ? g.get(k) : 1.f);
      };
      float all = 0.f;
      if (Q && !a.group) {
        for (int v = lane; v < nvec; v += TPR) {
          float y[E];
          value(v, y);
#pragma unroll
          for (int k = 0; k < E; ++k) all = fmaxf(all, fabsf(y[k]));
        }
        all = row_reduce<TPR, true>(all, most[0]);
      }
      const int padded = (nvec + TPR - 1) / TPR * TPR;  // whole warps reach the shuffles
      for (int v = lane; v < padded; v += TPR) {
        float y[E];
        float mx = 0.f;
        if (v < nvec) {
          value(v, y);
#pragma unroll
          for (int k = 0; k < E; ++k) mx = fmaxf(mx, fabsf(y[k]));
        }
        if constexpr (Q && E > 1) {
          if (a.group) mx = group_max<E>(mx);
        }
        if (v >= nvec) continue;
        const size_t o = (size_t)row * h + (size_t)v * E;
        if (Q) {
          const float2 sc = scale_of(a.group ? mx : all, rstd);
          store_e4m3<E>(reinterpret_cast<uint8_t*>(a.out) + o, y, sc, rstd);
          if (a.group) {
            if (v % (128 / E) == 0) a.scales[(size_t)row * (h / 128) + v / (128 / E)] = sc.x;
          } else if (v == 0) {
            a.scales[row] = sc.x;
          }
        } else {
          V w;
#pragma unroll
          for (int k = 0; k < E; ++k) w.set(k, y[k]);
          w.store(reinterpret_cast<T*>(a.out) + o);
        }
      }
      __syncthreads();
    }
  }
}

struct NormBwdArgs {
  const void *d_out, *d_s, *s, *gain;  // d_s, gain: or null
  const float* rstd;
  void* dx;
  float* partial;  // [gridDim.x][h], or null: no gradient of the gain
  int T, h;
};

template <typename T, int E, int TPR, int NV>
__global__ void __launch_bounds__(Shape<TPR>::kThreads) add_rmsnorm_backward_kernel(const NormBwdArgs a) {
  typedef Vec<T, E> V;
  constexpr int kRows = Shape<TPR>::kRows;
  __shared__ float part[2][32];
  pdl_launch_dependents();
  pdl_wait();
  const int lane = threadIdx.x % TPR;
  const int h = a.h, nvec = h / E;
  const T* gp = reinterpret_cast<const T*>(a.gain);
  const T* dp = reinterpret_cast<const T*>(a.d_out);
  const T* ep = reinterpret_cast<const T*>(a.d_s);
  const T* sp = reinterpret_cast<const T*>(a.s);
  int row = blockIdx.x * kRows + threadIdx.x / TPR;
  const int step = gridDim.x * kRows;
  const float inv_h = 1.0f / (float)h;

  if constexpr (NV > 0) {
    V gain[NV], d[NV], s[NV], e[NV];
    float acc[NV][E];
    float rstd = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = i * TPR + lane;
      if (gp && v < nvec) {
        gain[i].load(gp + v * E);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) gain[i].set(k, 1.f);
      }
#pragma unroll
      for (int k = 0; k < E; ++k) acc[i][k] = 0.f;
    }
    auto fetch = [&](int t) {
      if (t < a.T) rstd = ld_l2(a.rstd + t);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int v = i * TPR + lane;
        if (t < a.T && v < nvec) {
          const size_t o = (size_t)t * h + (size_t)v * E;
          d[i].load(dp + o);
          s[i].load(sp + o);
          if (ep) e[i].load(ep + o);
        }
      }
    };
    int odd = 0;
    fetch(row);
    for (int base = blockIdx.x * kRows; base < a.T; base += step, row += step, odd ^= 1) {
      const bool live = row < a.T;
      V d0[NV], s0[NV], e0[NV];
      const float rstd0 = rstd;
      float c = 0.f;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        d0[i] = d[i];
        s0[i] = s[i];
        if (ep) e0[i] = e[i];
      }
      fetch(row + step);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        if (!live || i * TPR + lane >= nvec) continue;
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const float dh = d0[i].get(k) * (s0[i].get(k) * rstd0);
          acc[i][k] += dh;
          c = fmaf(dh, gain[i].get(k), c);
        }
      }
      c = row_reduce<TPR, false>(c, part[odd]) * inv_h;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int v = i * TPR + lane;
        if (!live || v >= nvec) continue;
        V y;
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const float g = d0[i].get(k) * gain[i].get(k), hat = s0[i].get(k) * rstd0;
          y.set(k, fmaf(rstd0, g - hat * c, ep ? e0[i].get(k) : 0.f));
        }
        y.store(reinterpret_cast<T*>(a.dx) + (size_t)row * h + (size_t)v * E);
      }
    }
    if (!a.partial) return;
    float* out = a.partial + (size_t)blockIdx.x * h;
    if constexpr (kRows == 1) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int v = i * TPR + lane;
        if (v < nvec) {
#pragma unroll
          for (int k = 0; k < E; ++k) out[(size_t)v * E + k] = acc[i][k];
        }
      }
    } else {
      // the warps of a block add up in their order, one vector column at a time
      __shared__ float sum[kRows][32 * E];
#pragma unroll
      for (int i = 0; i < NV; ++i) {
#pragma unroll
        for (int k = 0; k < E; ++k) sum[threadIdx.x / 32][lane * E + k] = acc[i][k];
        __syncthreads();
        for (int c = threadIdx.x; c < 32 * E; c += Shape<TPR>::kThreads) {
          float t = 0.f;
#pragma unroll
          for (int w = 0; w < kRows; ++w) t += sum[w][c];
          if (i * 32 * E + c < h) out[i * 32 * E + c] = t;
        }
        __syncthreads();
      }
    }
  } else {
    for (; row < a.T; row += step) {
      const float rstd = ld_l2(a.rstd + row);
      const size_t o = (size_t)row * h;
      float c = 0.f;
      for (int v = lane; v < nvec; v += TPR) {
        V d, s, g;
        d.load(dp + o + (size_t)v * E);
        s.load(sp + o + (size_t)v * E);
        if (gp) g.load(gp + (size_t)v * E);
#pragma unroll
        for (int k = 0; k < E; ++k) c = fmaf(d.get(k) * (s.get(k) * rstd), gp ? g.get(k) : 1.f, c);
      }
      c = row_reduce<TPR, false>(c, part[0]) * inv_h;
      for (int v = lane; v < nvec; v += TPR) {
        V d, s, g, e, y;
        d.load(dp + o + (size_t)v * E);
        s.load(sp + o + (size_t)v * E);
        if (gp) g.load(gp + (size_t)v * E);
        if (ep) e.load(ep + o + (size_t)v * E);
#pragma unroll
        for (int k = 0; k < E; ++k)
          y.set(k, fmaf(rstd, d.get(k) * (gp ? g.get(k) : 1.f) - s.get(k) * rstd * c, ep ? e.get(k) : 0.f));
        y.store(reinterpret_cast<T*>(a.dx) + o + (size_t)v * E);
      }
      __syncthreads();
    }
  }
}

// Gradient of the gain of rows too long for the registers: block (x, y) adds up the columns 256 x .. of every
// gridDim.y-th row from y on.
template <typename T>
__global__ void __launch_bounds__(256) dgain_columns_kernel(const T* d_out, const T* s, const float* rstd, int rows, int h,
                                                            float* partial) {
  pdl_launch_dependents();
  pdl_wait();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= h) return;
  float acc = 0.f;
  for (int t = blockIdx.y; t < rows; t += gridDim.y) {
    Vec<T, 1> d, v;
    d.load(d_out + (size_t)t * h + c);
    v.load(s + (size_t)t * h + c);
    acc = fmaf(d.get(0), v.get(0) * ld_l2(rstd + t), acc);
  }
  partial[(size_t)blockIdx.y * h + c] = acc;
}

// dgain = the partial sums of `n` blocks, 32 columns a block: 32 threads a column add every 32nd partial in order,
// then a fixed tree over the 32.
template <typename T>
__global__ void __launch_bounds__(1024) dgain_reduce_kernel(const float* partial, int n, int h, T* dgain) {
  __shared__ float sum[32][33];
  pdl_launch_dependents();
  pdl_wait();
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + tx;
  float acc = 0.f;
  if (c < h)
    for (int p = ty; p < n; p += 32) acc += ld_l2(partial + (size_t)p * h + c);
  sum[ty][tx] = acc;
  __syncthreads();
  acc = sum[tx][ty];
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, s);
  if (tx == 0 && blockIdx.x * 32 + ty < h) dgain[blockIdx.x * 32 + ty] = from_f<T>(acc);
}

// How a row is cut: threads a row and vectors a thread.  In the forward pass rows that 128 threads of two vectors fill to
// three quarters and more take those: more rows are under way on an SM, and what a row waits for is its reduction.  256
// threads of one vector / 128 of two, us, columns 1544 / 1792 / 2048 of bf16: e4m3 of 8000 rows 22.7 / 19.6, 22.9 / 19.9,
// 24.0 / 20.9, of 30000 rows 76.7 / 65.9, 76.6 / 65.3, 79.5 / 68.5; norm of 8000 rows 18.1 / 17.9, 20.1 / 20.1, 22.6 / 22.8,
// of 30000 rows 59.8 / 59.4, 72.9 / 74.5, 85.5 / 83.6.  fp32 of 772 to 1024 columns: e4m3 of 8000 rows 2-11 % faster, of
// 30000 x 1024 61.1 / 64.3, norm within 2 %.  Single elements, 30000 x 193 to 255: norm 30 / 21, e4m3 48 / 33.  Below, 30000 x
// 1536, it is slower: 57.0 / 61.  Three vectors a thread were 4-10 % slower than the next cut (1536 to 6144 columns).
struct Cut { int tpr, nv; };
Cut cut_of(int h, int E, bool forward) {
  const int n = h / E;
  if (n <= 32) return {32, 1};
  if (n <= 64) return {32, 2};
  if (n <= 128) return {32, 4};
  if (forward && n > 192 && n <= 256) return {128, 2};
  if (n <= 256) return {256, 1};
  if (n <= 512) return {256, 2};
  if (n <= 1024) return {256, 4};
  if (E == 1 && n <= 8192) return {1024, 8};
  return {256, 0};
}

std::atomic<int> g_fail_occupancy{0};  // moe_test_fail_occupancy

// Blocks of a persistent launch: what is resident at once, so that every block walks about as many rows.  A kernel's
// blocks per SM are asked for once a device and remembered when there was an answer.
constexpr int kBlocksPerSm = 8;  // of the backward pass at most: partial sums of the gain's gradient are sized for it
struct Resident {
  std::atomic<int> blocks[64];
};
template <typename... KArgs>
cudaError_t grid_of(void (*kernel)(KArgs...), int T, const Cut& c, int most_blocks, Resident& known, int* grid) {
  const int threads = c.tpr == 32 ? 256 : c.tpr, rows = threads / c.tpr;
  int dev = 0, n = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64) n = known.blocks[dev].load(std::memory_order_relaxed);
  if (!n) {
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0);
    if (g_fail_occupancy.load(std::memory_order_relaxed) > 0) {
      g_fail_occupancy.fetch_sub(1);
      e = cudaErrorUnknown;
    }
    if (e != cudaSuccess) return e;
    if (n < 1) return cudaErrorInvalidConfiguration;
    n = n < most_blocks ? n : most_blocks;
    if (dev < 64) known.blocks[dev].store(n, std::memory_order_relaxed);
  }
  const int need = (T + rows - 1) / rows, most = sm_count() * n;
  *grid = need < most ? need : most;
  return cudaSuccess;
}

#define MOE_NORM_CUTS(CASE) CASE(32, 1) CASE(32, 2) CASE(32, 4) CASE(256, 1) CASE(256, 2) CASE(256, 4)

template <typename T, int E, int TPR, int NV, bool Q> cudaError_t launch_norm_cut(const NormArgs& a, cudaStream_t st) {
  static Resident known = {};
  int grid = 0;
  const cudaError_t e = grid_of(add_rmsnorm_kernel<T, E, TPR, NV, Q>, a.T, {TPR, NV}, 16, known, &grid);
  if (e != cudaSuccess) return e;
  return launch_pdl(add_rmsnorm_kernel<T, E, TPR, NV, Q>, dim3(grid), dim3(Shape<TPR>::kThreads), 0, st, a);
}

template <typename T, int E, bool Q> cudaError_t launch_norm_as(const NormArgs& a, cudaStream_t st) {
  const Cut c = cut_of(a.h, E, true);
#define CASE(TPR, NV) if (c.tpr == TPR && c.nv == NV) return launch_norm_cut<T, E, TPR, NV, Q>(a, st);
  MOE_NORM_CUTS(CASE)
  CASE(128, 2)
  if constexpr (E == 1) { CASE(1024, 8) }
#undef CASE
  return launch_norm_cut<T, E, 256, 0, Q>(a, st);
}

template <typename T> cudaError_t launch_norm_type(const NormArgs& a, bool q, cudaStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  if (a.h % E == 0) return q ? launch_norm_as<T, E, true>(a, st) : launch_norm_as<T, E, false>(a, st);
  return q ? launch_norm_as<T, 1, true>(a, st) : launch_norm_as<T, 1, false>(a, st);
}

template <typename T, int E, int TPR, int NV> cudaError_t launch_bwd_cut(const NormBwdArgs& a, int* grid, cudaStream_t st) {
  static Resident known = {};
  const cudaError_t e = grid_of(add_rmsnorm_backward_kernel<T, E, TPR, NV>, a.T, {TPR, NV}, kBlocksPerSm, known, grid);
  if (e != cudaSuccess) return e;
  return launch_pdl(add_rmsnorm_backward_kernel<T, E, TPR, NV>, dim3(*grid), dim3(Shape<TPR>::kThreads), 0, st, a);
}

template <typename T, int E> cudaError_t launch_bwd_as(const NormBwdArgs& a, const Cut& c, int* grid, cudaStream_t st) {
#define CASE(TPR, NV) if (c.tpr == TPR && c.nv == NV) return launch_bwd_cut<T, E, TPR, NV>(a, grid, st);
  MOE_NORM_CUTS(CASE)
  if constexpr (E == 1) { CASE(1024, 8) }
#undef CASE
  return launch_bwd_cut<T, E, 256, 0>(a, grid, st);
}

int dgain_rows(int T) { return T < 256 ? T : 256; }  // row chunks of dgain_columns_kernel

template <typename T> cudaError_t launch_bwd_type(NormBwdArgs a, void* dgain, float* partial, cudaStream_t st) {
  constexpr int E = 16 / (int)sizeof(T);
  const bool wide = a.h % E == 0;
  const Cut c = cut_of(a.h, wide ? E : 1, false);
  int grid = 0;
  const bool columns = dgain && c.nv == 0;
  a.partial = dgain && !columns ? partial : nullptr;
  cudaError_t e = wide ? launch_bwd_as<T, E>(a, c, &grid, st) : launch_bwd_as<T, 1>(a, c, &grid, st);
  if (e != cudaSuccess || !dgain) return e;
  int n = grid;
  if (columns) {
    n = dgain_rows(a.T);
    e = launch_pdl(dgain_columns_kernel<T>, dim3((a.h + 255) / 256, n), dim3(256), 0, st, (const T*)a.d_out, (const T*)a.s,
                   a.rstd, a.T, a.h, partial);
    if (e != cudaSuccess) return e;
  }
  return launch_pdl(dgain_reduce_kernel<T>, dim3((a.h + 31) / 32), dim3(1024), 0, st, (const float*)partial, n, a.h, (T*)dgain);
}

constexpr int kMaxH = 1 << 20;

int check_sizes(int T, int h, int dtype) {
  if (!element_size(dtype)) return set_error(MOE_ERR_INVALID_ARG, "dtype = %d is none of MOE_BF16, MOE_FP16, MOE_FP32", dtype);
  if (T < 0 || T > kMaxOperatorTokens) return set_error(MOE_ERR_INVALID_ARG, "T = %d outside 0..%d", T, kMaxOperatorTokens);
  if (h < 1 || h > kMaxH) return set_error(MOE_ERR_UNSUPPORTED_SHAPE, "h = %d outside 1..%d", h, kMaxH);
  return MOE_OK;
}

int forward(const void* x, const void* residual, const void* gain, int T, int h, float eps, int dtype, int group, void* out,
            float* scales, void* s, float* rstd, bool q, cudaStream_t st) {
  int rc = check_sizes(T, h, dtype);
  if (rc) return rc;
  if (!(eps >= 0.f)) return set_error(MOE_ERR_INVALID_ARG, "eps = %g must not be negative", (double)eps);
  if (q && group != 0 && group != 128) return set_error(MOE_ERR_INVALID_ARG, "group = %d: 0 (a row) or 128", group);
  if (q && group && h % group) return set_error(MOE_ERR_UNSUPPORTED_SHAPE, "h = %d is not a multiple of the group of %d", h, group);
  if (T == 0) return MOE_OK;
  if (!x || !out) return set_error(MOE_ERR_INVALID_ARG, "x or the output is NULL");
  if (q && !scales) return set_error(MOE_ERR_INVALID_ARG, "scales is NULL");
  if ((residual == nullptr) != (s == nullptr))
    return set_error(MOE_ERR_INVALID_ARG, "residual and s go together: both or neither");
  if (!aligned16(x) || !aligned16(residual) || !aligned16(gain) || !aligned16(out) || !aligned16(s))
    return set_error(MOE_ERR_INVALID_ARG, "every tensor must be 16-byte aligned");
  if (!aligned4(rstd) || !aligned4(scales)) return set_error(MOE_ERR_INVALID_ARG, "rstd or scales is not aligned to its fp32 values");
  const size_t e = (size_t)element_size(dtype), n = (size_t)T * h * e;
  const size_t n_out = q ? (size_t)T * h : n;
  // an output may be an input of the same place and type (its row is read before it is written), nothing in between
  const void* in[2] = {x, residual};
  for (const void* p : in) {
    if (p && s && p != s && overlap(p, n, s, n)) return set_error(MOE_ERR_INVALID_ARG, "s overlaps an input in part");
    if (p && (q || p != out) && overlap(p, n, out, n_out))
      return set_error(MOE_ERR_INVALID_ARG, "the output overlaps an input");
  }
  const size_t n_scales = q ? (size_t)T * (group ? h / group : 1) * sizeof(float) : 0, n_rstd = (size_t)T * sizeof(float);
  const void* whole[5] = {x, residual, out, s, gain};
  const size_t bytes[5] = {n, n, n_out, n, h * e};
  for (int i = 0; i < 5; ++i)
    if (overlap(whole[i], bytes[i], rstd, n_rstd) || overlap(whole[i], bytes[i], scales, n_scales))
      return set_error(MOE_ERR_INVALID_ARG, "rstd or scales overlaps another tensor");
  if (overlap(s, n, out, n_out)) return set_error(MOE_ERR_INVALID_ARG, "s and the output overlap");
  if (overlap(gain, h * e, out, n_out) || overlap(gain, h * e, s, n))
    return set_error(MOE_ERR_INVALID_ARG, "the gain overlaps an output");
  NormArgs a = {x, residual, gain, out, s, rstd, scales, T, h, group, eps};
  const cudaError_t err = dtype == MOE_BF16 ? launch_norm_type<__nv_bfloat16>(a, q, st)
                          : dtype == MOE_FP16 ? launch_norm_type<__half>(a, q, st) : launch_norm_type<float>(a, q, st);
  if (err != cudaSuccess) return set_error(MOE_ERR_CUDA, "add_rmsnorm launch: %s", cudaGetErrorString(err));
  return MOE_OK;
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" {

int moe_add_rmsnorm(const void* x, const void* residual, const void* gain, int T, int h, float eps, int dtype, void* out,
                    void* s, float* rstd, void* cuda_stream) {
  return forward(x, residual, gain, T, h, eps, dtype, 0, out, nullptr, s, rstd, false, static_cast<cudaStream_t>(cuda_stream));
}

int moe_add_rmsnorm_e4m3(const void* x, const void* residual, const void* gain, int T, int h, float eps, int dtype, int group,
                         void* q, float* scales, void* s, void* cuda_stream) {
  return forward(x, residual, gain, T, h, eps, dtype, group, q, scales, s, nullptr, true, static_cast<cudaStream_t>(cuda_stream));
}

size_t moe_add_rmsnorm_backward_workspace(int T, int h) {
  if (T < 1 || T > kMaxOperatorTokens || h < 1 || h > kMaxH) return 0;
  const int blocks = sm_count() * kBlocksPerSm;
  const int n = T < blocks ? T : blocks;
  return (size_t)(n > dgain_rows(T) ? n : dgain_rows(T)) * h * sizeof(float);
}

int moe_add_rmsnorm_backward(const void* d_out, const void* d_s, const void* s, const float* rstd, const void* gain, int T,
                             int h, int dtype, void* dx, void* dgain, void* workspace, size_t workspace_bytes,
                             void* cuda_stream) {
  int rc = check_sizes(T, h, dtype);
  if (rc) return rc;
  const size_t e = (size_t)element_size(dtype), n = (size_t)T * h * e;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (!aligned16(dgain) || !aligned16(workspace)) return set_error(MOE_ERR_INVALID_ARG, "every tensor must be 16-byte aligned");
  if (T == 0) {  // no rows: the gradient of the gain is a sum of nothing
    if (dgain) {
      const cudaError_t err = cudaMemsetAsync(dgain, 0, h * e, st);
      if (err != cudaSuccess) return set_error(MOE_ERR_CUDA, "clearing dgain: %s", cudaGetErrorString(err));
    }
    return MOE_OK;
  }
  if (!d_out || !s || !rstd || !dx) return set_error(MOE_ERR_INVALID_ARG, "d_out, s, rstd or dx is NULL");
  if (!aligned16(d_out) || !aligned16(d_s) || !aligned16(s) || !aligned16(gain) || !aligned16(dx))
    return set_error(MOE_ERR_INVALID_ARG, "every tensor must be 16-byte aligned");
  if (!aligned4(rstd)) return set_error(MOE_ERR_INVALID_ARG, "rstd is not aligned to its fp32 values");
  if (dgain && (!workspace || workspace_bytes < moe_add_rmsnorm_backward_workspace(T, h)))
    return set_error(MOE_ERR_INVALID_ARG, "workspace of %zu bytes, %zu are needed", workspace ? workspace_bytes : (size_t)0,
                     moe_add_rmsnorm_backward_workspace(T, h));
  // dx may be d_s (each element is read before it is written), but the other operands are read again: d_out and s by the
  // gain's sums, the gain by blocks that start later and for every row that the registers do not hold
  if (overlap(dx, n, d_out, n) || overlap(dx, n, s, n) || overlap(dx, n, gain, h * e) || (dx != d_s && overlap(dx, n, d_s, n)))
    return set_error(MOE_ERR_INVALID_ARG, "dx overlaps an input (only d_s itself is allowed)");
  if (overlap(dgain, h * e, d_out, n) || overlap(dgain, h * e, s, n) || overlap(dgain, h * e, dx, n) ||
      overlap(dgain, h * e, gain, h * e) || overlap(dgain, h * e, d_s, n))
    return set_error(MOE_ERR_INVALID_ARG, "dgain overlaps another tensor");
  const size_t n_ws = dgain ? moe_add_rmsnorm_backward_workspace(T, h) : 0, n_rstd = (size_t)T * sizeof(float);
  const void* whole[7] = {d_out, d_s, s, gain, rstd, dx, dgain};
  const size_t bytes[7] = {n, n, n, h * e, n_rstd, n, h * e};
  for (int i = 0; i < 7; ++i)
    if ((n_ws && overlap(whole[i], bytes[i], workspace, n_ws)) || (i > 4 && overlap(whole[i], bytes[i], rstd, n_rstd)))
      return set_error(MOE_ERR_INVALID_ARG, "the workspace overlaps a tensor, or a gradient rstd");
  NormBwdArgs a = {d_out, d_s, s, gain, rstd, dx, nullptr, T, h};
  float* partial = static_cast<float*>(workspace);
  const cudaError_t err = dtype == MOE_BF16   ? launch_bwd_type<__nv_bfloat16>(a, dgain, partial, st)
                          : dtype == MOE_FP16 ? launch_bwd_type<__half>(a, dgain, partial, st)
                                              : launch_bwd_type<float>(a, dgain, partial, st);
  if (err != cudaSuccess) return set_error(MOE_ERR_CUDA, "add_rmsnorm_backward launch: %s", cudaGetErrorString(err));
  return MOE_OK;
}

int moe_test_fail_occupancy(int times) {
  if (times < 0) return set_error(MOE_ERR_INVALID_ARG, "times = %d", times);
  g_fail_occupancy.store(times);
  return MOE_OK;
}

}  // extern "C"

// HIP kernels of the operators of a transformer block around its matrix
// products and its attention (gfx950; fp32 or bf16 storage, fp32 arithmetic):
// rotary positions, layer norm and dropout, forward and backward.  None of
// them multiplies matrices: each reads its inputs and writes its outputs once,
// and HBM bounds it where there are many rows, the launch where there are few.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "device.h"
#include "internal.h"

namespace erase {

namespace {

// hipLaunchKernel's own result (not the last error of any earlier call).
template <typename A>
hipError_t launch1(void (*kernel)(A), int64_t grid, int block, const A& a, hipStream_t s) {
  A copy = a;
  void* args[] = {&copy};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((uint32_t)grid), dim3((uint32_t)block), args, 0, s);
}

// sine and cosine of a 64-bit fraction of a turn: the quadrant from the top
// bits, then the Taylor polynomials on [-pi/4, pi/4] (next terms 1.8e-9 and
// 1.2e-10, below a quarter of an fp32 rounding of 1)
__device__ __forceinline__ void sincos_turn(uint64_t turn, float& s, float& c) {
  const uint32_t t = (uint32_t)(turn >> 32) + 0x20000000u;  // + 1/8: quadrants centred on multiples of 1/4
  const int32_t r = (int32_t)(t & 0x3fffffffu) - 0x20000000;
  const float x = (float)r * 1.4629180792671596e-9f;  // 2 pi / 2^32
  const float z = x * x;
  const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -0.16666667f), x);
  const float cs =
      fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
  const uint32_t q = t >> 30;
  const float a = q & 1 ? cs : sn, b = q & 1 ? sn : cs;
  s = q & 2 ? -a : a;                   // sn, cs, -sn, -cs
  c = (q == 1 || q == 2) ? -b : b;      // cs, -sn, -cs, sn
}

__device__ __forceinline__ int64_t rope_position(const RopeArgs& a, int b, int t) {
  return a.positions ? (int64_t)a.positions[b * a.pos_b + t * a.pos_t] : a.start + a.start_t * t;
}

}  // namespace

// ---------------------------------------------------------------------------
// rotary positions
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kRopeFill) void ops_rope_fill(RopeFillArgs a) {
  if ((int)threadIdx.x < a.n) a.table[threadIdx.x] = a.v[threadIdx.x];
}

hipError_t launch_rope_fill(const RopeFillArgs& a, hipStream_t s) { return launch1(ops_rope_fill, 1, kRopeFill, a, s); }

// One token per workgroup; a thread takes pairs and passed columns in turn.
template <typename T>
__global__ __launch_bounds__(256) void ops_rope(RopeArgs a) {
  const int half = a.rot / 2, units = a.dim - half;  // pairs, then columns that pass
  const float amp = __uint_as_float((uint32_t)a.table[half]);
  for (int64_t n = blockIdx.x; n < (int64_t)a.batch * a.seq; n += gridDim.x) {
    const int b = (int)(n / a.seq), t = (int)(n % a.seq);
    const int64_t p = rope_position(a, b, t);
    for (int u = threadIdx.x; u < (a.heads[0] + a.heads[1]) * units; u += 256) {
      int h = u / units;
      const int i = u % units, w = h >= a.heads[0];
      if (w) h -= a.heads[0];
      const T* x = static_cast<const T*>(a.x[w]) + b * a.xs[w][0] + t * a.xs[w][1] + h * a.xs[w][2];
      T* y = static_cast<T*>(a.y[w]) + b * a.ys[w][0] + t * a.ys[w][1] + h * a.ys[w][2];
      if (i >= half) {
        y[half + i] = x[half + i];
        continue;
      }
      float s, c;
      sincos_turn((uint64_t)p * a.table[i], s, c);
      s *= a.inverse ? -amp : amp;
      c *= amp;
      const int i1 = a.interleaved ? 2 * i : i, i2 = a.interleaved ? 2 * i + 1 : half + i;
      const float x1 = ldf(x + i1), x2 = ldf(x + i2);
      y[i1] = cvt<T>(fmaf(x1, c, -(x2 * s)));
      y[i2] = cvt<T>(fmaf(x2, c, x1 * s));
    }
  }
}

hipError_t launch_rope(int bf16, const RopeArgs& a, hipStream_t s) {
  const int64_t n = std::min<int64_t>((int64_t)a.batch * a.seq, 1 << 20);
  return launch1(bf16 ? ops_rope<uint16_t> : ops_rope<float>, n, 256, a, s);
}

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------
namespace {

// Sums of two values over a workgroup of 256 threads, in every thread.
__device__ __forceinline__ void block_sum2(float& u, float& v) {
  __shared__ float part[2][4];
  const int wave = threadIdx.x >> 6;
  u = wave_sum(u);
  v = wave_sum(v);
  __syncthreads();  // the last call's sums have been read
  if ((threadIdx.x & 63) == 0) {
    part[0][wave] = u;
    part[1][wave] = v;
  }
  __syncthreads();
  u = part[0][0] + part[0][1] + part[0][2] + part[0][3];
  v = part[1][0] + part[1][1] + part[1][2] + part[1][3];
}

}  // namespace

// One row per workgroup.
template <typename T>
__global__ __launch_bounds__(256) void ops_norm(NormArgs a) {
  for (int64_t n = blockIdx.x; n < a.rows; n += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + n * a.ldx;
    T* y = static_cast<T*>(a.y) + n * a.ldy;
    float s = 0.f, q = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) s += ldf(x + c);
    block_sum2(s, q);
    const float mean = s / (float)a.cols;
    q = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) {
      const float d = ldf(x + c) - mean;
      q = fmaf(d, d, q);
    }
    s = 0.f;
    block_sum2(s, q);
    const float r = 1.f / sqrtf(q / (float)a.cols + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[n] = mean;
      if (a.rstd) a.rstd[n] = r;
    }
    for (int c = threadIdx.x; c < a.cols; c += 256) {
      const float h = (ldf(x + c) - mean) * r;
      y[c] = cvt<T>(fmaf(h, a.w ? a.w[c] : 1.f, a.b ? a.b[c] : 0.f));
    }
  }
}

hipError_t launch_norm(int bf16, const NormArgs& a, hipStream_t s) {
  return launch1(bf16 ? ops_norm<uint16_t> : ops_norm<float>, std::min<int64_t>(a.rows, 1 << 20), 256, a, s);
}

// Workgroup g takes rows g, g + nparts, ...; its weight gradients pass through
// its slice of `part`, every column by one thread.
template <typename T>
__global__ __launch_bounds__(256) void ops_norm_bwd(NormBwdArgs a) {
  float* pw = a.part ? a.part + (int64_t)blockIdx.x * 2 * a.ldpart : nullptr;
  float* pb = a.part ? pw + a.ldpart : nullptr;
  if (pw)
    for (int c = threadIdx.x; c < a.cols; c += 256) pw[c] = pb[c] = 0.f;
  for (int64_t n = blockIdx.x; n < a.rows; n += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + n * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + n * a.lddy;
    const T* res = a.res ? static_cast<const T*>(a.res) + n * a.ldres : nullptr;
    T* dx = a.dx ? static_cast<T*>(a.dx) + n * a.lddx : nullptr;
    const float mean = a.mean[n], r = a.rstd[n];
    float sg = 0.f, sgh = 0.f;
    for (int c = threadIdx.x; c < a.cols; c += 256) {
      const float d = ldf(dy + c), h = (ldf(x + c) - mean) * r, g = d * (a.w ? a.w[c] : 1.f);
      sg += g;
      sgh = fmaf(g, h, sgh);
      if (pw) {
        pw[c] = fmaf(d, h, pw[c]);
        pb[c] += d;
      }
    }
    block_sum2(sg, sgh);
    if (!dx) continue;
    const float mg = sg / (float)a.cols, mgh = sgh / (float)a.cols;
    for (int c = threadIdx.x; c < a.cols; c += 256) {
      const float h = (ldf(x + c) - mean) * r, g = ldf(dy + c) * (a.w ? a.w[c] : 1.f);
      dx[c] = cvt<T>(fmaf(r, g - mg - h * mgh, res ? ldf(res + c) : 0.f));
    }
  }
}

int norm_bwd_parts(int, int64_t rows, int) { return (int)std::max<int64_t>(1, std::min<int64_t>(rows, 1024)); }

hipError_t launch_norm_bwd(int bf16, const NormBwdArgs& a, hipStream_t s) {
  return launch1(bf16 ? ops_norm_bwd<uint16_t> : ops_norm_bwd<float>, a.nparts, 256, a, s);
}

struct NormSumArgs {
  const float* part;
  int64_t ldpart;
  int nparts, cols;
  float *dw, *db;
};
__global__ __launch_bounds__(256) void ops_norm_sum(NormSumArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  float w = 0.f, b = 0.f;
  for (int g = 0; g < a.nparts; ++g) {
    const float* p = a.part + (int64_t)g * 2 * a.ldpart + c;
    w += p[0];
    b += p[a.ldpart];
  }
  if (a.dw) a.dw[c] = w;
  if (a.db) a.db[c] = b;
}

hipError_t launch_norm_sum(const float* part, int64_t ldpart, int nparts, int cols, float* dw, float* db, hipStream_t s) {
  const NormSumArgs a{part, ldpart, nparts, cols, dw, db};
  return launch1(ops_norm_sum, (cols + 255) / 256, 256, a, s);
}

// ---------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------
namespace {

// Philox4x32-10 (Salmon et al. 2011): ten rounds of two 32 x 32 -> 64 bit
// products; the key advances by the Weyl constants.
__device__ __forceinline__ void philox(uint32_t x[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int i = 0; i < 10; ++i) {
    const uint64_t p = (uint64_t)x[0] * 0xD2511F53u, q = (uint64_t)x[2] * 0xCD9E8D57u;
    x[0] = (uint32_t)(q >> 32) ^ x[1] ^ k0;
    x[1] = (uint32_t)q;
    x[2] = (uint32_t)(p >> 32) ^ x[3] ^ k1;
    x[3] = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}

}  // namespace

// A thread takes groups of eight columns of a row.
template <typename T>
__global__ __launch_bounds__(256) void ops_dropout(DropArgs a) {
  const uint64_t off = a.offset + (a.step ? *a.step : 0);
  const int groups = (a.cols + 7) / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.rows * groups; i += (int64_t)gridDim.x * 256) {
    const int64_t n = i / groups;
    const int g = (int)(i % groups);
    uint32_t bits[4] = {(uint32_t)g, (uint32_t)(a.row0 + n), (uint32_t)off, (uint32_t)(off >> 32)};
    philox(bits, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
    const T* x = static_cast<const T*>(a.x) + n * a.ldx;
    const T* res = a.res ? static_cast<const T*>(a.res) + n * a.ldres : nullptr;
    T* y = static_cast<T*>(a.y) + n * a.ldy;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = 8 * g + k;
      if (c >= a.cols) break;
      const uint32_t u = (bits[k >> 1] >> (16 * (k & 1))) & 0xffffu;
      const float v = u >= a.limit ? ldf(x + c) * a.scale : 0.f;
      y[c] = cvt<T>(res ? v + ldf(res + c) : v);
    }
  }
}

hipError_t launch_dropout(int bf16, const DropArgs& a, hipStream_t s) {
  const int64_t n = (a.rows * ((a.cols + 7) / 8) + 255) / 256;
  return launch1(bf16 ? ops_dropout<uint16_t> : ops_dropout<float>, std::min<int64_t>(n, 1 << 20), 256, a, s);
}

}  // namespace erase

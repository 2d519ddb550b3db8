// HIP kernels of the operators of a transformer block around its matrix
// products and its attention (gfx950; fp32 or bf16 storage, fp32 arithmetic):
// rotary positions, layer norm and dropout, forward and backward.  None of
// them multiplies matrices: each reads its inputs and writes its outputs once,
// and HBM bounds it where there are many rows, the launch where there are few.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "device.h"
#include "ops.h"

namespace erase {

namespace {

// hipLaunchKernel's own result (not the last error of any earlier call, and none
// left behind for a later one).
template <typename A>
hipError_t launch1(void (*kernel)(A), int64_t grid, int block, const A& a, hipStream_t s, uint32_t grid_y = 1) {
  A copy = a;
  void* args[] = {&copy};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((uint32_t)grid, grid_y),
                                       dim3((uint32_t)block), args, 0, s);
  if (e != hipSuccess) (void)hipGetLastError();
  return e;
}

// Eight bf16 or four fp32 consecutive elements, moved by one 16-byte access from
// any element's address (the hardware splits what straddles a line).  Where
// fewer are left they move in accesses of 8, 4 and 2 bytes, one for each binary
// digit of their number: three independent loads instead of up to seven that
// wait for one another.  Elements past the end are zero.
typedef uint32_t u32x4_at2_t __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_at4_t __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_at2_t __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x2_at4_t __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32_at2_t __attribute__((aligned(2)));
template <typename T>
struct Chunk {
  static constexpr int V = 16 / sizeof(T);
  typedef std::conditional_t<sizeof(T) == 2, u32x4_at2_t, u32x4_at4_t> mem_t;
  typedef std::conditional_t<sizeof(T) == 2, u32x2_at2_t, u32x2_at4_t> mem2_t;
  u32x4_t r;
  __device__ __forceinline__ float operator[](int k) const {
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(r[k]);
    else
      return __uint_as_float(k & 1 ? r[k >> 1] & 0xffff0000u : r[k >> 1] << 16);
  }
};
template <typename T>
__device__ __forceinline__ Chunk<T> ld_chunk(const T* p, int n) {
  Chunk<T> c;
  if (n >= Chunk<T>::V) {
    c.r = *reinterpret_cast<const typename Chunk<T>::mem_t*>(p);
  } else {
    c.r = u32x4_t{0u, 0u, 0u, 0u};
    if (n > 0) {
      constexpr int E = 8 / sizeof(T);  // elements of 8 bytes
      typename Chunk<T>::mem2_t two = {0u, 0u};
      uint32_t one = 0u, half = 0u;
      if (n & E) two = *reinterpret_cast<const typename Chunk<T>::mem2_t*>(p);
      if constexpr (sizeof(T) == 4) {
        if (n & 1) one = __float_as_uint(p[n & 2]);
      } else {
        if (n & 2) one = *reinterpret_cast<const u32_at2_t*>(p + (n & 4));
        if (n & 1) half = p[n & 6];
      }
      const bool front = !(n & E);  // the 4-byte word comes first
      c.r[0] = front ? one : two[0];
      c.r[1] = front ? 0u : two[1];
      c.r[2] = front ? 0u : one;
      if constexpr (sizeof(T) == 2) {
        const int w = (n & 6) >> 1;
#pragma unroll
        for (int k = 0; k < 4; ++k) c.r[k] |= k == w ? half : 0u;
      }
    }
  }
  return c;
}
template <typename T>
__device__ __forceinline__ Chunk<T> pack_chunk(const float v[Chunk<T>::V]) {
  Chunk<T> c;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(T) == 4)
      c.r[k] = __float_as_uint(v[k]);
    else
      c.r[k] = (uint32_t)f2bf(v[2 * k]) | ((uint32_t)f2bf(v[2 * k + 1]) << 16);
  }
  return c;
}
template <typename T>
__device__ __forceinline__ void st_raw(T* p, int n, const Chunk<T>& c) {
  if (n >= Chunk<T>::V) {
    *reinterpret_cast<typename Chunk<T>::mem_t*>(p) = c.r;
  } else if (n > 0) {
    constexpr int E = 8 / sizeof(T);
    if (n & E) *reinterpret_cast<typename Chunk<T>::mem2_t*>(p) = typename Chunk<T>::mem2_t{c.r[0], c.r[1]};
    const uint32_t one = n & E ? c.r[2] : c.r[0];
    if constexpr (sizeof(T) == 4) {
      if (n & 1) p[n & 2] = __uint_as_float(one);
    } else {
      if (n & 2) *reinterpret_cast<u32_at2_t*>(p + (n & 4)) = one;
      const uint32_t next = n & E ? c.r[3] : c.r[1];
      if (n & 1) p[n & 6] = (T)(n & 2 ? next : one);
    }
  }
}
template <typename T>
__device__ __forceinline__ void st_chunk(T* p, int n, const float v[Chunk<T>::V]) {
  st_raw(p, n, pack_chunk<T>(v));
}

// Sum over groups of L = 4, 8, 16, 32 or 64 lanes, the same bits in every lane:
// within 16 lanes by lane permutations in the add itself (xor 1, xor 2, mirrored
// halves, mirrored rows), beyond by exchanging rows and halves.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int L>
__device__ __forceinline__ float lane_sum(float v) {
  v += dpp<0xb1>(v);
  v += dpp<0x4e>(v);
  if constexpr (L >= 8) v += dpp<0x141>(v);
  if constexpr (L >= 16) v += dpp<0x140>(v);
  if constexpr (L >= 32) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  }
  if constexpr (L >= 64) {
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
  }
  return v;
}

// sine and cosine of a 64-bit fraction of a turn (its low half, less than 1.5e-9
// radians, is dropped): the quadrant from the top bits, then the Taylor polynomials on [-pi/4, pi/4] (next terms 1.8e-9 and
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

// A workgroup takes `tokens` consecutive positions of a batch row: it computes
// their sines and cosines once into LDS, then its threads take units of those
// tokens' heads, 32 bytes each: V pairs (two 16-byte chunks) or 2 V columns that
// pass.  HBM bounds it: 671 MB read and written (32768 tokens of 40 heads of 128,
// half of each turned) take 129 us, 5.2 TB/s.  Columns that pass in units of one
// chunk, on a path of their own, took 163 us; several units' loads issued before
// the sines 162 to 224 (the registers cost more waves than the loads hide).
constexpr int kRopePairs = 2048;  // pairs of a workgroup's tokens (16 KB of LDS)
struct RopePlan {
  RopeArgs a;
  FastDiv per_token, per_head, pairs;  // units of a token, of a head; pairs of a head
  int turn;                            // units of a head that turn (the others pass)
  int tokens;
  uint32_t row_groups, groups;         // groups of tokens in a batch row, in all
  int whole;  // the last unit ends with the columns it is for, overlapping the one before (not in place)
};

namespace {

__device__ __forceinline__ uint32_t quotient(uint32_t n, const FastDiv& d) {
  const uint32_t t = __umulhi(d.m, n);
  return (t + ((n - t) >> d.s1)) >> d.s2;
}

}  // namespace

template <typename T, bool INTER>
__global__ __launch_bounds__(256) void ops_rope(RopePlan p) {
  constexpr int V = Chunk<T>::V;
  __shared__ float2 cs[kRopePairs + V];  // read to the end of a chunk
  const RopeArgs& a = p.a;
  const int half = a.rot / 2;
  const float amp = __uint_as_float((uint32_t)a.table[half]);
  for (uint32_t g = blockIdx.x; g < p.groups; g += gridDim.x) {
    const int b = (int)(g / p.row_groups), t0 = (int)(g % p.row_groups) * p.tokens;
    const int tokens = min(p.tokens, a.seq - t0);
    const uint32_t units = (uint32_t)tokens * p.per_token.d;
    if (g != blockIdx.x) __syncthreads();  // the last group's sines have been read
    for (uint32_t j = threadIdx.x; j < (uint32_t)(tokens * half); j += 256) {
      const uint32_t tok = quotient(j, p.pairs);
      const int64_t pos = rope_position(a, b, t0 + (int)tok);
      float s, c;
      sincos_turn((uint64_t)pos * a.table[j - tok * half], s, c);
      cs[j] = make_float2(c * amp, a.inverse ? -(s * amp) : s * amp);
    }
    __syncthreads();
    for (uint32_t id = blockIdx.y * 256 + threadIdx.x; id < units; id += 256 * gridDim.y) {
      const uint32_t tok = quotient(id, p.per_token), in_tok = id - tok * p.per_token.d;
      const uint32_t hh = quotient(in_tok, p.per_head), c = in_tok - hh * p.per_head.d;
      const int w = hh >= (uint32_t)a.heads[0], h = (int)hh - (w ? a.heads[0] : 0);
      const int64_t t = t0 + (int64_t)tok;
      const T* x = static_cast<const T*>(w ? a.x[1] : a.x[0]) + b * (w ? a.xs[1][0] : a.xs[0][0]) +
                   t * (w ? a.xs[1][1] : a.xs[0][1]) + h * (w ? a.xs[1][2] : a.xs[0][2]);
      T* y = static_cast<T*>(w ? a.y[1] : a.y[0]) + b * (w ? a.ys[1][0] : a.ys[0][0]) +
             t * (w ? a.ys[1][1] : a.ys[0][1]) + h * (w ? a.ys[1][2] : a.ys[0][2]);
      const bool turns = (int)c < p.turn;
      // 2 V columns of a head: V pairs, or columns behind rot
      const int end = turns ? a.rot : a.dim - a.rot;
      int i = (turns ? (int)c : (int)c - p.turn) * 2 * V;
      if (p.whole && end >= 2 * V) i = min(i, end - 2 * V);
      const int left = min(2 * V, end - i);
      int n1 = min(V, left), n2 = left - n1, second = V, at = (turns ? 0 : a.rot) + i;
      if (!INTER && turns) {
        n1 = n2 = left / 2;
        second = half;
        at = i / 2;
      }
      x += at;
      y += at;
      // whole chunks are loaded where the head has the columns, the unit's own are
      // stored (24673 tokens of 12 heads of 80, 14 columns turned: 34.5 us, 42.7 with
      // the loads in pieces too)
      const int room = a.dim - at;
      Chunk<T> x1 = ld_chunk(x, room >= V ? V : n1), x2 = ld_chunk(x + second, room - second >= V ? V : n2);
      if (turns) {
        const float2* q = cs + (int)tok * half + i / 2;
        float o1[V], o2[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          if constexpr (INTER) {  // pair k is columns 2 k, 2 k + 1 of the two chunks in a row
            const float v1 = 2 * k < V ? x1[2 * k] : x2[2 * k - V];
            const float v2 = 2 * k < V ? x1[2 * k + 1] : x2[2 * k + 1 - V];
            const float w1 = fmaf(v1, q[k].x, -(v2 * q[k].y)), w2 = fmaf(v2, q[k].x, v1 * q[k].y);
            (2 * k < V ? o1[2 * k] : o2[2 * k - V]) = w1;
            (2 * k < V ? o1[2 * k + 1] : o2[2 * k + 1 - V]) = w2;
          } else {
            o1[k] = fmaf(x1[k], q[k].x, -(x2[k] * q[k].y));
            o2[k] = fmaf(x2[k], q[k].x, x1[k] * q[k].y);
          }
        }
        x1 = pack_chunk<T>(o1);
        x2 = pack_chunk<T>(o2);
      }
      st_raw(y, n1, x1);
      st_raw(y + second, n2, x2);
    }
  }
}

hipError_t launch_rope(int bf16, const RopeArgs& args, hipStream_t s) {
  RopePlan p{};
  RopeArgs& a = p.a = args;
  if (a.seq == 1) {  // one token a row: the rows are the positions
    a.seq = a.batch;
    a.batch = 1;
    for (int w = 0; w < 2; ++w) {
      a.xs[w][1] = a.xs[w][0];
      a.ys[w][1] = a.ys[w][0];
    }
    a.pos_t = a.pos_b;
    a.start_t = 0;
  }
  const int V = bf16 ? 8 : 4, half = a.rot / 2;
  const bool in_place = a.x[0] == a.y[0] || (a.heads[1] && a.x[1] == a.y[1]);
  const bool all_in_place = a.x[0] == a.y[0] && (!a.heads[1] || a.x[1] == a.y[1]);
  p.whole = !in_place;
  p.turn = (half + V - 1) / V;
  const int per_head = p.turn + (all_in_place ? 0 : (a.dim - a.rot + 2 * V - 1) / (2 * V));
  const int per_token = per_head * (a.heads[0] + a.heads[1]);
  p.per_head = fast_div((uint32_t)per_head);
  p.per_token = fast_div((uint32_t)per_token);
  p.pairs = fast_div((uint32_t)half);
  // as many tokens as give every thread one unit, or two where that leaves fewer
  // threads without any (57274 tokens of 144 units: 107 us with three tokens in
  // two rounds, 129 to 137 with one token on 144 of 256 threads; more rounds hide
  // less latency: tokens of 320 units 82 us in two rounds of one, 92 in five of four;
  // the second round is taken where it uses at least a twentieth of the threads more:
  // 100000 tokens of 24 units, 10 of them a round, 35.3 us, 21 in two rounds 36.3);
  // fewer where that leaves less than two workgroups a compute unit
  int best = 1;
  double used = 0.0;  // share of the threads' rounds
  for (int n = 1; n <= 2; ++n) {
    const int t = 256 * n / per_token;
    if (t >= 1 && double(t) * per_token / (256 * n) > used + 0.05) {
      best = t;
      used = double(t) * per_token / (256 * n);
    }
  }
  p.tokens = std::max(1, std::min({best, kRopePairs / half, a.seq}));
  auto row_groups = [&] { return ((int64_t)a.seq + p.tokens - 1) / p.tokens; };
  while (p.tokens > 1 && a.batch * row_groups() < 512) p.tokens = (p.tokens + 1) / 2;
  p.row_groups = (uint32_t)row_groups();
  p.groups = (uint32_t)a.batch * p.row_groups;
  const uint32_t grid = std::min<uint32_t>(p.groups, 1 << 20);
  const uint32_t splits = (uint32_t)((per_token + 1023) / 1024);  // of one token's heads, beyond four units a thread
  if (bf16) return launch1(a.interleaved ? ops_rope<uint16_t, true> : ops_rope<uint16_t, false>, grid, 256, p, s, splits);
  return launch1(a.interleaved ? ops_rope<float, true> : ops_rope<float, false>, grid, 256, p, s, splits);
}

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------
// Layouts of the row kernels: a row is held by `lanes` threads (4 to 64 of a wave,
// or W waves), K chunks of 16 bytes each; a workgroup of the forward takes
// `groups` rows, one of the backward as many as 1024 threads hold.
template <typename E, int Lanes, int Waves, int Chunks, bool Narrow = false>
struct RowShape {
  typedef E T;
  static constexpr int L = Lanes, W = Waves, K = Chunks;
  static constexpr bool narrow = Narrow;  // rows of less than a chunk
  static constexpr int lanes = L * W, cols = lanes * K * Chunk<T>::V;
  static constexpr int groups = lanes < 256 ? 256 / lanes : 1, threads = lanes * groups;
  static constexpr int bwd_groups = 1024 / lanes;
};

namespace {

// Calls f with the shape that holds a row of `cols` elements in the forward, and
// in the backward (whose workgroups have 1024 threads).  Narrow rows share a wave
// (1196284 x 26 bf16: 32 us with 4 lanes a row, 89 with 16; 161542 x 201: 34 with 32,
// 57 with 64).  The forward takes the fewest waves that hold the row with weight
// and bias: rows of a wave need no barrier (16000 x 1500: 21.5 us with 3 chunks a
// lane, 25.6 with 4 waves), and several rows of a compute unit are in flight (3605
// x 4160: 17.3 us with 4 waves of 3 chunks, 25.5 with 16 of 1).  The backward holds
// three times as much a column and takes one chunk a lane while it can.
template <typename T, typename F>
auto with_norm_shape(int cols, F&& f) {
  constexpr int V = Chunk<T>::V;
  if (cols < V) return f(RowShape<T, 4, 1, 1, true>());
  if (cols <= 4 * V) return f(RowShape<T, 4, 1, 1>());
  if (cols <= 8 * V) return f(RowShape<T, 8, 1, 1>());
  if (cols <= 16 * V) return f(RowShape<T, 16, 1, 1>());
  if (cols <= 32 * V) return f(RowShape<T, 32, 1, 1>());
  if (cols <= 64 * V) return f(RowShape<T, 64, 1, 1>());
  if (cols <= 128 * V) return f(RowShape<T, 64, 1, 2>());
  if (cols <= 192 * V) return f(RowShape<T, 64, 1, 3>());
  if (cols <= 256 * V) return f(RowShape<T, 64, 4, 1>());
  if (cols <= 512 * V) return f(RowShape<T, 64, 4, 2>());
  if (cols <= 768 * V) return f(RowShape<T, 64, 4, 3>());
  if (cols <= 1024 * V) return f(RowShape<T, 64, 4, 4>());
  if constexpr (V == 4)
    if (cols > 2048 * V) return f(RowShape<T, 64, 16, 4>());
  return f(RowShape<T, 64, 16, 2>());
}
template <typename T, typename F>
auto with_norm_bwd_shape(int cols, F&& f) {
  constexpr int V = Chunk<T>::V;
  if (cols < V) return f(RowShape<T, 4, 1, 1, true>());
  if (cols <= 4 * V) return f(RowShape<T, 4, 1, 1>());
  if (cols <= 8 * V) return f(RowShape<T, 8, 1, 1>());
  if (cols <= 16 * V) return f(RowShape<T, 16, 1, 1>());
  if (cols <= 32 * V) return f(RowShape<T, 32, 1, 1>());
  if (cols <= 64 * V) return f(RowShape<T, 64, 1, 1>());
  if (cols <= 128 * V) return f(RowShape<T, 64, 2, 1>());
  if (cols <= 256 * V) return f(RowShape<T, 64, 4, 1>());
  if (cols <= 512 * V) return f(RowShape<T, 64, 8, 1>());
  if (cols <= 1024 * V) return f(RowShape<T, 64, 16, 1>());
  if constexpr (V == 4)
    if (cols > 2048 * V) return f(RowShape<T, 64, 16, 4>());
  return f(RowShape<T, 64, 16, 2>());
}

// The V columns that a thread's chunk i covers: [at, at + V), of which the first
// `skip` belong to the chunk before.  A row's last chunk ends with the row, so
// that every load is a whole one and none waits in a branch for the row's last
// columns (0 to 7 of them); a thread behind the row skips all V.  The first
// `Whole` chunks are known to have nothing to skip.
struct Window {
  int at, skip;
};
template <typename S, int Whole = 0>
__device__ __forceinline__ Window window(int pos, int i, int cols) {
  constexpr int V = Chunk<typename S::T>::V;
  const int c = (pos + i * S::lanes) * V, at = min(c, cols - V);
  return i < Whole ? Window{c, 0} : Window{at, min(c - at, V)};
}
// Chunk i of every thread lies within the row: nothing to skip.
template <typename S, int Whole = 0>
__device__ __forceinline__ bool whole(int i, int cols) {
  return i < Whole || (i + 1) * S::lanes * Chunk<typename S::T>::V <= cols;
}
// The V elements of a window (rows narrower than V: one by one).
template <typename S, typename T>
__device__ __forceinline__ Chunk<T> ld_window(const T* p, const Window& w) {
  constexpr int V = Chunk<T>::V;
  Chunk<T> c;
  if constexpr (!S::narrow) {
    c.r = *reinterpret_cast<const typename Chunk<T>::mem_t*>(p + w.at);
  } else {
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = k >= w.skip ? ldf(p + w.at + k) : 0.f;
    c = pack_chunk<T>(v);
  }
  return c;
}
// Zeros in the first `skip` elements.
template <typename T>
__device__ __forceinline__ void clear_front(Chunk<T>& c, int skip) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if constexpr (sizeof(T) == 4)
      c.r[k] = k >= skip ? c.r[k] : 0u;
    else
      c.r[k] &= 2 * k >= skip ? 0xffffffffu : 2 * k + 1 >= skip ? 0xffff0000u : 0u;
  }
}
// V elements of an fp32 vector (none: `empty`).
template <typename S, int V>
__device__ __forceinline__ void ld_weights(const float* p, const Window& w, float empty, float (&v)[V]) {
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = empty;
  if (!p) return;
  if constexpr (!S::narrow) {
#pragma unroll
    for (int j = 0; j < V / 4; ++j) {
      const u32x4_t t = *reinterpret_cast<const u32x4_at4_t*>(p + w.at + 4 * j);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[4 * j + k] = __uint_as_float(t[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= w.skip) v[k] = p[w.at + k];
  }
}
// Stores a window's own columns: all V, or the last ones by the binary digits of
// their number.
template <typename T>
__device__ __forceinline__ void st_window(T* p, const Window& w, const float v[Chunk<T>::V]) {
  constexpr int V = Chunk<T>::V, E = 8 / sizeof(T);
  const Chunk<T> c = pack_chunk<T>(v);
  const int n = V - w.skip;
  T* end = p + w.at + V;
  if (n == V) {
    *reinterpret_cast<typename Chunk<T>::mem_t*>(end - V) = c.r;
  } else if (n > 0) {
    if (n & E) *reinterpret_cast<typename Chunk<T>::mem2_t*>(end - E) = typename Chunk<T>::mem2_t{c.r[2], c.r[3]};
    const uint32_t one = n & E ? c.r[1] : c.r[3];
    if constexpr (sizeof(T) == 4) {
      if (n & 1) end[-(n & 2) - 1] = __uint_as_float(one);
    } else {
      if (n & 2) *reinterpret_cast<u32_at2_t*>(end - (n & 4) - 2) = one;
      const uint32_t next = n & E ? c.r[0] : c.r[2];
      if (n & 1) end[-(n & 6) - 1] = (T)((n & 2 ? next : one) >> 16);
    }
  }
}

}  // namespace

constexpr int kNormGroups = 2048;  // workgroups of the forward, eight a compute unit

// Forward: a row is read once into registers; the mean, then the sums of the
// centred row and of its squares, two reductions that wait for one another.  The
// rounded mean m leaves c = mean(x - m), which is taken off the row and its square
// off the mean of squares: rows of one value are centred to zero, and rows far from
// zero are off by the rounding of c, not of m (700 columns of 30000.3: y was -0.53).
// The second sum, its correction and r as one rsqrt (within 1 ulp, twice a correctly
// rounded quotient's error) take what the quotients by cols and of the square root
// took: 16384 x 512 8.7 us, 9.2 with a square root and a quotient for r, 9.6 with all
// quotients.  A workgroup takes many
// rows, so that weight and bias (twice the bytes of a bf16 row each) are read
// once per thread, not per row: 8000 x 4096 bf16 takes 27.4 us (4.7 TB/s), 34.9
// with weight and bias read again for every row.
// HEAD: also the target logit of the stored row.
template <typename S, bool HEAD>
__global__ __launch_bounds__(S::threads) void ops_norm(NormArgs a) {
  typedef typename S::T T;
  constexpr int V = Chunk<T>::V, L = S::L, W = S::W, K = S::K;
  __shared__ float sums[HEAD ? 2 : 1][S::groups][W];
  __shared__ float2 sums2[S::groups][W];
  const int grp = threadIdx.x / S::lanes, pos = threadIdx.x % S::lanes;
  const float cols = (float)a.cols, inv = 1.f / cols;
  // v / cols, rounded once: with 1 / cols rounded, the remainder of v * inv (exact in
  // an fma) corrects it to the nearest (Markstein 1990), so that equal numbers have
  // their own mean
  auto over_cols = [&](float v) {
    const float q = v * inv;
    return fmaf(fmaf(-q, cols, v), inv, q);
  };
  float w[K][V], b[K][V];
  Window at[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    at[i] = window<S>(pos, i, a.cols);
    ld_weights<S>(a.w, at[i], 1.f, w[i]);
    ld_weights<S>(a.b, at[i], 0.f, b[i]);
  }
  auto total = [&](float v, int which) {
    v = lane_sum<L>(v);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) sums[which][grp][pos >> 6] = v;
      __syncthreads();
      v = 0.f;
#pragma unroll
      for (int j = 0; j < W; ++j) v += sums[which][grp][j];
    }
    return v;
  };
  auto total2 = [&](float2 v) {
    v = make_float2(lane_sum<L>(v.x), lane_sum<L>(v.y));
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) sums2[grp][pos >> 6] = v;
      __syncthreads();
      v = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        v.x += sums2[grp][j].x;
        v.y += sums2[grp][j].y;
      }
    }
    return v;
  };
  // the same number of rounds for every row group of the workgroup
  for (int64_t n0 = (int64_t)blockIdx.x * S::groups; n0 < a.rows; n0 += (int64_t)gridDim.x * S::groups) {
    const bool row = n0 + grp < a.rows;
    const int64_t n = row ? n0 + grp : n0;  // (behind the last row: an existing one, not stored)
    Chunk<T> x[K];
#pragma unroll
    for (int i = 0; i < K; ++i) x[i] = ld_window<S>(static_cast<const T*>(a.x) + n * a.ldx, at[i]);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      if (whole<S>(i, a.cols)) {
#pragma unroll
        for (int k = 0; k < V; ++k) s += x[i][k];
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) s += k >= at[i].skip ? x[i][k] : 0.f;
      }
    }
    s = total(s, 0);
    const float mean = isinf(s) ? s : over_cols(s);
    float2 dq = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < K; ++i) {
      if (whole<S>(i, a.cols)) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float d = x[i][k] - mean;
          dq.x += d;
          dq.y = fmaf(d, d, dq.y);
        }
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float d = k >= at[i].skip ? x[i][k] - mean : 0.f;
          dq.x += d;
          dq.y = fmaf(d, d, dq.y);
        }
      }
    }
    dq = total2(dq);
    // (apart from the mean: mean + left rounds again)
    const float left = over_cols(dq.x), v = fmaf(-left, left, dq.y * inv);
    const float r = rsqrtf((v < 0.f ? 0.f : v) + a.eps);  // (a NaN stays one)
    if (!HEAD && !row) continue;
    if (row && pos == 0) {
      if (a.mean) a.mean[n] = isinf(mean) ? mean : mean + left;
      if (a.rstd) a.rstd[n] = r;
    }
    const int32_t target = HEAD ? a.target[n] : -1;
    float logit = 0.f;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = fmaf((x[i][k] - mean - left) * r, w[i][k], b[i][k]);
      if (row) st_window(static_cast<T*>(a.y) + n * a.ldy, at[i], o);
      if constexpr (HEAD) {
        if (target >= 0) {  // (whole chunks: cols is a multiple of V)
          const Chunk<T> c = pack_chunk<T>(o), hw = ld_window<S>(a.hw + (int64_t)target * a.ldhw, at[i]);
#pragma unroll
          for (int k = 0; k < V; ++k) logit = fmaf(at[i].skip ? 0.f : c[k], hw[k], logit);
        }
      }
    }
    if constexpr (HEAD) {
      logit = total(logit, 1);
      if (row && pos == 0) a.xref[n] = logit;
    }
  }
}

hipError_t launch_norm(int bf16, const NormArgs& a, hipStream_t s) {
  auto grid = [&](auto sh) { return std::min<int64_t>((a.rows + sh.groups - 1) / sh.groups, kNormGroups); };
  if (a.hw) {
    if (!bf16 || a.cols % 64 || a.cols > 4096) return hipErrorInvalidValue;
    auto run = [&](auto sh) {
      typedef decltype(sh) S;
      if constexpr (S::cols >= 64 && S::cols <= 4096) return launch1(ops_norm<S, true>, grid(sh), sh.threads, a, s);
      return hipErrorInvalidValue;
    };
    return with_norm_shape<uint16_t>(a.cols, run);
  }
  auto run = [&](auto sh) { return launch1(ops_norm<decltype(sh), false>, grid(sh), sh.threads, a, s); };
  return bf16 ? with_norm_shape<uint16_t>(a.cols, run) : with_norm_shape<float>(a.cols, run);
}

namespace {

// A workgroup's sums of its rows' columns into `part` (NULL: not wanted), its
// row groups added in order in LDS, in two stages where few threads have a column
// (425494 x 32 bf16: 22.9 us, 32.1 in one).
template <typename S, typename A>
__device__ __forceinline__ void st_norm_part(const A& acc, const Window* at, float* comb, int grp, int cols, float* part) {
  constexpr int V = Chunk<typename S::T>::V;
  if (!part) return;
#pragma unroll
  for (int i = 0; i < S::K; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k)
      if (k >= at[i].skip) (S::bwd_groups > 1 ? comb + grp * S::cols : part)[at[i].at + k] = acc[i][k];
  if constexpr (S::bwd_groups > 1 && S::cols > 256) {
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += 1024) {
      float v = comb[c];
#pragma unroll 4
      for (int g = 1; g < S::bwd_groups; ++g) v += comb[g * S::cols + c];
      part[c] = v;
    }
  } else if constexpr (S::bwd_groups > 1) {  // many groups of few columns: slices of them, then the slices
    constexpr int slices = 1024 / S::cols, per = S::bwd_groups / slices;
    const int c = threadIdx.x % S::cols, slice = threadIdx.x / S::cols;
    __syncthreads();
    float v = 0.f;
    if (c < cols)
#pragma unroll
      for (int g = 0; g < per; ++g) v += comb[(slice * per + g) * S::cols + c];
    __syncthreads();
    comb[threadIdx.x] = v;
    __syncthreads();
    if (slice == 0 && c < cols) {
      v = 0.f;
#pragma unroll 8
      for (int g = 0; g < slices; ++g) v += comb[g * S::cols + c];
      part[c] = v;
    }
  }
}

// What the backward takes and gives: PLAIN is the public operator; HEAD takes a
// row scale and, where there are slices, their sum as dy; F32 stores dx in fp32.
enum NormMode { PLAIN, HEAD, F32 };

// Elements in fp32 with a Chunk's reading.
template <int V>
struct Floats {
  float v[V];
  __device__ __forceinline__ float operator[](int k) const { return v[k]; }
};
template <int V>
__device__ __forceinline__ void clear_front(Floats<V>& c, int skip) {
#pragma unroll
  for (int k = 0; k < V; ++k) c.v[k] = k >= skip ? c.v[k] : 0.f;
}

// A thread's part of x and dy of row n, and the row's statistics.
template <typename S, NormMode M>
struct NormRow {
  typedef Chunk<typename S::T> C;
  C x[S::K];
  std::conditional_t<M == HEAD, Floats<C::V>, C> d[S::K];
  float mean, r;
};
template <typename S, NormMode M>
__device__ __forceinline__ NormRow<S, M> ld_norm_row(const NormBwdArgs& a, const Window* at, int64_t n) {
  typedef typename S::T T;
  constexpr int V = Chunk<T>::V;
  NormRow<S, M> v;
  v.mean = a.mean[n];
  v.r = a.rstd[n];
#pragma unroll
  for (int i = 0; i < S::K; ++i) {
    v.x[i] = ld_window<S>(static_cast<const T*>(a.x) + n * a.ldx, at[i]);
    if constexpr (M == HEAD) {
      float(&d)[V] = v.d[i].v;
      if (a.nslice > 0) {
#pragma unroll
        for (int k = 0; k < V; ++k) d[k] = 0.f;
        const float* p = a.slice + n * a.ldslice + at[i].at;
        for (int z = 0; z < a.nslice; ++z, p += a.zslice)  // added in order
#pragma unroll
          for (int j = 0; j < V; j += 4) {
            const float4 t = *reinterpret_cast<const float4*>(p + j);
            d[j] += t.x, d[j + 1] += t.y, d[j + 2] += t.z, d[j + 3] += t.w;
          }
      } else {
        const Chunk<T> c = ld_window<S>(static_cast<const T*>(a.dy) + n * a.lddy, at[i]);
#pragma unroll
        for (int k = 0; k < V; ++k) d[k] = c[k];
      }
      const float scale = a.dyscale[n];
#pragma unroll
      for (int k = 0; k < V; ++k) d[k] *= scale;
    } else {
      v.d[i] = ld_window<S>(static_cast<const T*>(a.dy) + n * a.lddy, at[i]);
    }
  }
  return v;
}

// dw and db of 16 chunks of columns over all rows, 64 rows at a time: they need
// the forward's statistics but none of dx's sums, so with few rows these
// workgroups run beside those of dx and no launch adds partial rows up.
template <typename S>
__device__ __forceinline__ void norm_strip(const NormBwdArgs& a, int strip, float* comb) {
  typedef typename S::T T;
  constexpr int V = Chunk<T>::V;
  typedef RowShape<T, 16, 1, 1, S::narrow> C;
  const int grp = threadIdx.x >> 4, pos = threadIdx.x & 15;
  const Window at = window<C>(strip * 16 + pos, 0, a.cols);
  float aw[V] = {}, ab[V] = {};
#pragma unroll 4
  for (int64_t n = grp; n < a.rows; n += 64) {
    const NormRow<C, PLAIN> v = ld_norm_row<C, PLAIN>(a, &at, n);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      aw[k] = fmaf(v.d[0][k], (v.x[0][k] - v.mean) * v.r, aw[k]);
      ab[k] += v.d[0][k];
    }
  }
  const int c0 = strip * 16 * V;
  for (int which = 0; which < 2; ++which) {
    float* out = which ? a.db : a.dw;
    if (!out) continue;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < V; ++k) comb[(grp * 16 + pos) * V + k] = which ? ab[k] : aw[k];
    __syncthreads();
    // column c of the strip: the window slot that holds it as its own
    const int c = c0 + (int)threadIdx.x;
    if ((int)threadIdx.x < 16 * V && c < a.cols) {
      const int l = (int)threadIdx.x / V, s = c - window<C>(strip * 16 + l, 0, a.cols).at;
      float v = 0.f;
#pragma unroll 8
      for (int g = 0; g < 64; ++g) v += comb[(g * 16 + l) * V + s];
      out[c] = v;
    }
  }
}

}  // namespace

// Backward.  A thread keeps its columns' weights and its partial sums of dw and
// db in registers over all its rows.  With 16 columns a thread (rows of more than
// 8192) the sums stand in LDS, in places that no other thread uses, since all of
// it spills in registers: 2500 x 16384 bf16 with res takes 86 us (117 with spills,
// 93 with the weights in LDS, 88 with the next row loaded ahead as well), fp32 148
// (189, 160, 164).  At the end the workgroup's row groups are added in order
// through LDS and one partial row per workgroup is stored (a single workgroup
// stores dw and db themselves).  Workgroups of 1024 threads, one a compute unit,
// keep the partial rows few: 16384 x 512 bf16 with res takes 16.8 us and the launch
// that adds them up 3.9 (in all 23 with 512 of 256 threads, 31 with 256 of 256: too
// few rows in flight).  16384 x 4096 takes 79.9 and 4.9 us, 5.0 TB/s.  The next
// row's loads are issued ahead where a row's waves meet at a barrier (17495 x 1083:
// 42.9 us, 47.0 without; rows of one wave lose up to a tenth by it).
template <typename S, NormMode M>
__global__ __launch_bounds__(1024) void ops_norm_bwd(NormBwdArgs a) {
  typedef typename S::T T;
  constexpr int V = Chunk<T>::V, G = S::bwd_groups, L = S::L, W = S::W, K = S::K;
  __shared__ float2 sums[2][G][W];
  constexpr bool kFew = K * V <= 8;  // elements a thread holds
  // the row groups' sums at the end, or (not few) every thread's own sums
  constexpr int kSums = !kFew ? 2 * S::cols : G > 1 ? G * S::cols : M == PLAIN ? 1024 * V : 4;
  __shared__ float4 lds[kSums / 4];
  float* comb = reinterpret_cast<float*>(lds);
  if constexpr (M == PLAIN)
    if ((int)blockIdx.x >= a.nparts) {
      norm_strip<S>(a, (int)blockIdx.x - a.nparts, comb);
      return;
    }
  // (a wave's one row group in a scalar register: so are its rows' addresses and
  // statistics; 17495 x 1083: 49.4 us, 50.8 without)
  const int grp = L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / S::lanes) : threadIdx.x / S::lanes;
  const int pos = threadIdx.x % S::lanes;
  constexpr int H = K / 2;  // chunks that are whole: else a shape of fewer is taken
  float w[K][V], aw[kFew ? K : 1][V], ab[kFew ? K : 1][V];
  Window at[K];
#pragma unroll
  for (int i = 0; i < K; ++i) {
    at[i] = window<S, H>(pos, i, a.cols);
    ld_weights<S>(a.w, at[i], 1.f, w[i]);
#pragma unroll
    for (int k = 0; k < V; ++k) {
      if constexpr (kFew)
        aw[i][k] = ab[i][k] = 0.f;
      else if (k % 4 == 0)
        lds[(i * V + k) / 4 * 2048 + threadIdx.x] = lds[(i * V + k) / 4 * 2048 + 1024 + threadIdx.x] =
            make_float4(0.f, 0.f, 0.f, 0.f);
    }
  }
  const float inv = 1.f / (float)a.cols;
  int buf = 0;
  const int64_t first = (int64_t)blockIdx.x * G;
  NormRow<S, M> cur, next;
  constexpr bool kAhead = W > 1 && kFew;
  if constexpr (kAhead) next = ld_norm_row<S, M>(a, at, first + grp < a.rows ? first + grp : first);
  // the same number of rounds for every row group of the workgroup
  for (int64_t n0 = first; n0 < a.rows; n0 += (int64_t)a.nparts * G) {
    const bool row = n0 + grp < a.rows;  // (behind the last row: an existing one)
    const int64_t n = row ? n0 + grp : n0, ahead = n0 + (int64_t)a.nparts * G;
    if constexpr (kAhead) {
      cur = next;
      if (ahead < a.rows) next = ld_norm_row<S, M>(a, at, ahead + grp < a.rows ? ahead + grp : ahead);
    } else {
      cur = ld_norm_row<S, M>(a, at, n);
    }
    auto &x = cur.x;
    auto &d = cur.d;
    const float mean = cur.mean, r = cur.r;
    // what is not the thread's adds nothing: columns of the chunk before, rows behind the last
#pragma unroll
    for (int i = 0; i < K; ++i)
      if (!whole<S, H>(i, a.cols)) {
        clear_front(x[i], at[i].skip);
        clear_front(d[i], at[i].skip);
      }
    if (!row) {
#pragma unroll
      for (int i = 0; i < K; ++i) clear_front(d[i], V);
    }
    float sg = 0.f, sgh = 0.f;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      float h[V];
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float dv = d[i][k], g = dv * w[i][k];
        h[k] = (x[i][k] - mean) * r;
        sg += g;
        sgh = fmaf(g, h[k], sgh);
        if constexpr (kFew) {
          aw[i][k] = fmaf(dv, h[k], aw[i][k]);
          ab[i][k] += dv;
        }
      }
      if constexpr (!kFew) {
#pragma unroll
        for (int k = 0; k < V; k += 4) {
          float4 *p = lds + (i * V + k) / 4 * 2048 + threadIdx.x, *q = p + 1024, sw = *p, sb = *q;
          sw.x = fmaf(d[i][k], h[k], sw.x), sb.x += d[i][k];
          sw.y = fmaf(d[i][k + 1], h[k + 1], sw.y), sb.y += d[i][k + 1];
          sw.z = fmaf(d[i][k + 2], h[k + 2], sw.z), sb.z += d[i][k + 2];
          sw.w = fmaf(d[i][k + 3], h[k + 3], sw.w), sb.w += d[i][k + 3];
          *p = sw;
          *q = sb;
        }
      }
    }
    if (M == F32 ? !a.dx32 : !a.dx) continue;
    Chunk<T> res[K];  // asked for before the sums are known
#pragma unroll
    for (int i = 0; i < K; ++i) {
      res[i].r = u32x4_t{0u, 0u, 0u, 0u};
      if (a.res) res[i] = ld_window<S>(static_cast<const T*>(a.res) + n * a.ldres, at[i]);
    }
    sg = lane_sum<L>(sg);
    sgh = lane_sum<L>(sgh);
    if constexpr (W > 1) {
      if ((threadIdx.x & 63) == 0) sums[buf][grp][pos >> 6] = make_float2(sg, sgh);
      __syncthreads();
      sg = sgh = 0.f;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        sg += sums[buf][grp][j].x;
        sgh += sums[buf][grp][j].y;
      }
      buf ^= 1;  // one barrier a round: the round after next writes this buffer again
    }
    if (!row) continue;
    const float mg = sg * inv, mgh = sgh * inv;
#pragma unroll
    for (int i = 0; i < K; ++i) {
      // g and h are unpacked again: held over the reduction they cost 2 K V registers
      asm volatile("" : "+v"(x[i].r));
      if constexpr (M != HEAD) asm volatile("" : "+v"(d[i].r));
      float o[V];
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = fmaf(r, d[i][k] * w[i][k] - mg - (x[i][k] - mean) * r * mgh, res[i][k]);
      if constexpr (M == F32) {
        float* p = a.dx32 + n * a.lddx32 + at[i].at;
        if (at[i].skip == 0)  // (whole chunks: cols is a multiple of V)
#pragma unroll
          for (int k = 0; k < V; k += 4) *reinterpret_cast<float4*>(p + k) = make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
      } else {
        st_window(static_cast<T*>(a.dx) + n * a.lddx, at[i], o);
      }
    }
  }
  if (!a.part) return;
  const bool alone = a.nparts == 1;
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.ldpart;
  if constexpr (kFew) {
    st_norm_part<S>(aw, at, comb, grp, a.cols, alone ? a.dw : part);
    if constexpr (G > 1) __syncthreads();
    st_norm_part<S>(ab, at, comb, grp, a.cols, alone ? a.db : part + a.ldpart);
  } else {
    for (int which = 0; which < 2; ++which) {
      float* to = alone ? (which ? a.db : a.dw) : part + which * a.ldpart;
      if (!to) continue;
#pragma unroll
      for (int i = 0; i < K; ++i)
#pragma unroll
        for (int k = 0; k < V; ++k)
          if (k >= at[i].skip)
            to[at[i].at + k] = comb[(((i * V + k) / 4 * 2 + which) * 1024 + (int)threadIdx.x) * 4 + k % 4];
    }
  }
}

// Partial rows: one per workgroup, a workgroup per compute unit; a single one
// (and no second launch) while it takes at most two rounds of rows.
int norm_bwd_parts(int bf16, int64_t rows, int cols) {
  auto parts = [&](auto sh) {
    constexpr int g = decltype(sh)::bwd_groups;
    return rows <= 2 * g ? 1 : (int)std::min<int64_t>((rows + g - 1) / g, 256);
  };
  return bf16 ? with_norm_bwd_shape<uint16_t>(cols, parts) : with_norm_bwd_shape<float>(cols, parts);
}

// Strips read x and dy once more, and take a round for every 64 rows: 270 x 512
// bf16 in 8.6 us (host time) against 11.3 with two launches, 700 x 8192 16.0 / 26.7;
// from 1000 rows on no faster (1000 x 2048 13.1 / 11.3).
bool norm_bwd_strips(int64_t rows) { return rows <= 768; }

hipError_t launch_norm_bwd(int bf16, const NormBwdArgs& args, hipStream_t s) {
  NormBwdArgs a = args;
  if (a.dyscale || a.dx32) {
    if (!bf16 || a.cols % 64 || a.cols > 4096 || a.strips) return hipErrorInvalidValue;
    auto run = [&](auto sh) {
      typedef decltype(sh) S;
      if constexpr (S::cols >= 64 && S::cols <= 4096)
        return launch1(a.dyscale ? ops_norm_bwd<S, HEAD> : ops_norm_bwd<S, F32>, a.nparts, 1024, a, s);
      return hipErrorInvalidValue;
    };
    return with_norm_bwd_shape<uint16_t>(a.cols, run);
  }
  auto run = [&](auto sh) {
    typedef decltype(sh) S;
    const int strip = 16 * Chunk<typename S::T>::V;
    const int strips = a.strips ? (a.cols + strip - 1) / strip : 0;
    if (a.strips) {
      a.part = nullptr;  // the first workgroups give dx alone
      a.nparts = a.dx ? (int)((a.rows + S::bwd_groups - 1) / S::bwd_groups) : 0;
    }
    return launch1(ops_norm_bwd<S, PLAIN>, a.nparts + strips, 1024, a, s);
  };
  return bf16 ? with_norm_bwd_shape<uint16_t>(a.cols, run) : with_norm_bwd_shape<float>(a.cols, run);
}

// dw and db from the partial rows ([slice][dw | db][ldpart]): 16 columns a
// workgroup, 64 threads down the slices for each 4 of them, then a tree in LDS.
struct NormSumArgs {
  const float* part;
  int64_t ldpart;
  int nparts, cols;
  float *dw, *db;
};
__global__ __launch_bounds__(256) void ops_norm_sum(NormSumArgs a) {
  __shared__ float4 sum[64][4];
  const int64_t c = (int64_t)blockIdx.x * 16 + (threadIdx.x & 3) * 4;  // of dw | db, a multiple of 4
  const int slice = threadIdx.x >> 2;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < 2 * a.ldpart)
#pragma unroll 4
    for (int g = slice; g < a.nparts; g += 64) {
      const float4 p = *reinterpret_cast<const float4*>(a.part + (int64_t)g * 2 * a.ldpart + c);
      v.x += p.x, v.y += p.y, v.z += p.z, v.w += p.w;
    }
  sum[slice][threadIdx.x & 3] = v;
#pragma unroll
  for (int n = 32; n >= 1; n >>= 1) {
    __syncthreads();
    if (slice < n) {
      const float4 p = sum[slice + n][threadIdx.x & 3];
      v.x += p.x, v.y += p.y, v.z += p.z, v.w += p.w;
      sum[slice][threadIdx.x & 3] = v;
    }
  }
  if (slice || c >= 2 * a.ldpart) return;
  float* out = c < a.ldpart ? a.dw : a.db;
  if (!out) return;
  const int c0 = (int)(c < a.ldpart ? c : c - a.ldpart);
  const float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (c0 + k < a.cols) out[c0 + k] = o[k];
}

hipError_t launch_norm_sum(const float* part, int64_t ldpart, int nparts, int cols, float* dw, float* db, hipStream_t s) {
  const NormSumArgs a{part, ldpart, nparts, cols, dw, db};
  return launch1(ops_norm_sum, (2 * ldpart + 15) / 16, 256, a, s);
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

// A thread takes eight columns of a row: one counter, one or two chunks.  The
// ten rounds are 20 products of 32 x 32 bits, which issue at a quarter of the
// rate of an addition: 16 bits an element (rather than 32) keep them below the
// time HBM needs.  16384 x 4096 bf16 takes 45.7 us for 268 MB read and written.
struct DropPlan {
  DropArgs a;
  FastDiv groups;  // eights of a row
  uint32_t total;
};
template <typename T>
__global__ __launch_bounds__(256) void ops_dropout(DropPlan p) {
  const DropArgs& a = p.a;
  constexpr int V = Chunk<T>::V;
  const uint32_t id = blockIdx.x * 256 + threadIdx.x;
  if (id >= p.total) return;
  const uint32_t n = quotient(id, p.groups), g = id - n * p.groups.d;
  const int c = (int)(8 * g), left = a.cols - c;
  const T* x = static_cast<const T*>(a.x) + n * a.ldx + c;
  const T* res = a.res ? static_cast<const T*>(a.res) + n * a.ldres + c : nullptr;
  T* y = static_cast<T*>(a.y) + n * a.ldy + c;
  Chunk<T> xv[8 / V], rv[8 / V];
#pragma unroll
  for (int j = 0; j < 8 / V; ++j) {
    xv[j] = ld_chunk(x + j * V, left - j * V);
    rv[j].r = u32x4_t{0u, 0u, 0u, 0u};
    if (res) rv[j] = ld_chunk(res + j * V, left - j * V);
  }
  const uint64_t off = a.offset + (a.step ? *a.step : 0);
  uint32_t bits[4] = {g, (uint32_t)a.row0 + n, (uint32_t)off, (uint32_t)(off >> 32)};
  philox(bits, (uint32_t)a.seed, (uint32_t)(a.seed >> 32));
#pragma unroll
  for (int j = 0; j < 8 / V; ++j) {
    float o[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const int e = j * V + k;
      const uint32_t u = e & 1 ? bits[e >> 1] >> 16 : bits[e >> 1] & 0xffffu;
      o[k] = u >= a.limit ? xv[j][k] * a.scale : 0.f;
      if (res) o[k] += rv[j][k];
    }
    st_chunk(y + j * V, left - j * V, o);
  }
}

hipError_t launch_dropout(int bf16, const DropArgs& args, hipStream_t s) {
  DropPlan p{};
  p.a = args;
  p.groups = fast_div((uint32_t)(((int64_t)args.cols + 7) / 8));
  // threads are numbered in 32 bits: that many rows a launch
  const int64_t slab = std::max<int64_t>(1, (int64_t(1) << 31) / p.groups.d);
  for (int64_t r = 0; r < args.rows; r += slab) {
    const size_t size = bf16 ? 2 : 4;
    p.a.row0 = args.row0 + r;
    p.a.rows = std::min(slab, args.rows - r);
    p.a.x = static_cast<const char*>(args.x) + size * r * args.ldx;
    if (args.res) p.a.res = static_cast<const char*>(args.res) + size * r * args.ldres;
    p.a.y = static_cast<char*>(args.y) + size * r * args.ldy;
    p.total = (uint32_t)p.a.rows * p.groups.d;
    const hipError_t e = launch1(bf16 ? ops_dropout<uint16_t> : ops_dropout<float>, (p.total + 255) / 256, 256, p, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace erase

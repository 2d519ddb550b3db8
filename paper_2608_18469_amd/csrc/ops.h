// Internal interface between the host side (ops_api.cpp, tf_api.cpp) and the
// kernels of the operators of a transformer block (ops.hip); pointers of element
// type fp32 or, with bf16 set, bf16.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace erase {

// Division of 32-bit numbers by a number fixed per launch (Granlund and
// Montgomery 1994, "Division by invariant integers using multiplication"):
// with l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1 and t = high word of
// m n, n / d = (t + ((n - t) >> min(l, 1))) >> max(l - 1, 0) for every n.
struct FastDiv {
  uint32_t d, m, s1, s2;
};
inline FastDiv fast_div(uint32_t d) {
  uint32_t l = 0;
  while (l < 32 && (uint64_t(1) << l) < d) ++l;
  return {d, uint32_t(((uint64_t(1) << 32) * ((uint64_t(1) << l) - d)) / d + 1), l < 1 ? l : 1u, l > 1 ? l - 1 : 0u};
}

// Rotary positions of q and k ([batch][seq][heads][head_dim] by strides);
// table: rot / 2 turn fractions, then the amplitude (bits of a float in the low
// word).  inverse: by the negative angle.  positions NULL: start + start_t t.
struct RopeArgs {
  const void* x[2]; void* y[2];          // q and k
  int64_t xs[2][3], ys[2][3];            // batch, position, head
  int heads[2];
  int batch, seq, dim, rot;
  const int32_t* positions; int64_t pos_b, pos_t;
  int64_t start, start_t;
  const uint64_t* table;
  int interleaved, inverse;
};
constexpr int kRopeFill = 128;  // table entries of one launch
struct RopeFillArgs {
  uint64_t* table;
  int n;
  uint64_t v[kRopeFill];
};
hipError_t launch_rope_fill(const RopeFillArgs& a, hipStream_t s);
hipError_t launch_rope(int bf16, const RopeArgs& a, hipStream_t s);

// Layer norm; w, b, mean and rstd as in the C ABI (nullable).  With hw set (the
// vocabulary head's bf16 weight [V][ldhw]; bf16 rows of a multiple of 64 columns,
// 4096 at most) also the target logit xref[n] = y[n] . hw[target[n]] of the stored
// row (0 where the target is invalid).
struct NormArgs {
  const void* x; int64_t ldx;
  const float* w; const float* b;
  void* y; int64_t ldy;
  float* mean; float* rstd;
  int64_t rows;
  int cols;
  float eps;
  const uint16_t* hw; int64_t ldhw;
  const int32_t* target;
  float* xref;
};
hipError_t launch_norm(int bf16, const NormArgs& a, hipStream_t s);

// Its backward: dx (nullable) and, over norm_bwd_parts() slices of the rows,
// partial sums part[slice][0: dw, 1: db][ldpart] (part nullable: no sums
// wanted), which launch_norm_sum adds in order into dw and db (each nullable).  A
// single slice goes into dw and db at once; so do strips of columns where
// norm_bwd_strips() says that they pay.
struct NormBwdArgs {
  const void* x; int64_t ldx;
  const void* dy; int64_t lddy;
  const float* w; const float* mean; const float* rstd;
  const void* res; int64_t ldres;
  void* dx; int64_t lddx;
  float* part; int64_t ldpart; int nparts;
  float* dw; float* db;
  int strips;  // dw and db by workgroups of their own, beside dx (which may not be dy then)
  int64_t rows;
  int cols;
  // bf16 rows of a multiple of 64 columns, 4096 at most: with dyscale set the
  // gradient is dyscale[n] dy[n], dy the sum of nslice fp32 slices
  // slice[z][n][ldslice] where nslice > 0; with dx32 set dx is stored in fp32 there
  const float* dyscale;
  const float* slice; int64_t ldslice, zslice; int nslice;
  float* dx32; int64_t lddx32;
};
int norm_bwd_parts(int bf16, int64_t rows, int cols);
bool norm_bwd_strips(int64_t rows);
inline int64_t norm_part_pitch(int cols) { return (cols + 3) / 4 * 4; }
hipError_t launch_norm_bwd(int bf16, const NormBwdArgs& a, hipStream_t s);
hipError_t launch_norm_sum(const float* part, int64_t ldpart, int nparts, int cols, float* dw, float* db, hipStream_t s);

// Dropout (+ residual, nullable): element (row0 + r, c) is kept where its 16
// random bits are at least `limit`, and scaled.
struct DropArgs {
  const void* x; int64_t ldx;
  const void* res; int64_t ldres;
  void* y; int64_t ldy;
  int64_t rows, row0;
  int cols;
  uint64_t seed, offset;
  const uint64_t* step;  // nullable: added to offset
  uint32_t limit;
  float scale;
};
hipError_t launch_dropout(int bf16, const DropArgs& a, hipStream_t s);
// `limit` and `scale` of a probability: steps of 2^-16, the scale exact for the step.
inline void drop_rate(double p, DropArgs* a) {
  a->limit = uint32_t(p * 65536.0 + 0.5);
  a->scale = a->limit < 65536 ? float(65536.0 / (65536 - a->limit)) : 0.f;
}

}  // namespace erase

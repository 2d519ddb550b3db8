// C-ABI entry points of the operators of a transformer block: host checks and
// launches (include/erase_ops.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "erase_ops.h"
#include "ops.h"

namespace {

using namespace erase;

bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }
size_t elem(int32_t dtype) { return dtype == ERASE_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == ERASE_F32 || dtype == ERASE_BF16; }

// elements an array may span, far beyond any memory: products of sizes and
// pitches stay within 64 bits
constexpr int64_t kSpan = int64_t(1) << 48;
constexpr int64_t kRows = int64_t(1) << 31;
constexpr int32_t kNormCols = 16384;

bool pitch_ok(int64_t rows, int64_t cols, int64_t ld) {
  return rows <= 1 || (ld >= cols && static_cast<__int128>(rows) * ld < kSpan);
}
// one buffer in two roles: element for element
bool same_or_apart(const void* out, int64_t ldo, const void* in, int64_t ldi, int64_t rows) {
  return out != in || ldo == ldi || rows <= 1;
}

erase_status done(hipError_t e) { return e == hipSuccess ? ERASE_OK : ERASE_ERR_HIP; }

// ---------------------------------------------------------------------------
// rotary positions
// ---------------------------------------------------------------------------
constexpr long double kTau = 6.283185307179586476925286766559006L;

erase_status check_spec(const erase_rope_spec* p) {
  if (!p) return ERASE_ERR_INVALID_ARG;
  if (p->rot_dim < 2 || p->rot_dim > 1024 || p->rot_dim % 2) return ERASE_ERR_SHAPE;
  if (p->scaling < ERASE_ROPE_NONE || p->scaling > ERASE_ROPE_BY_PARTS) return ERASE_ERR_INVALID_ARG;
  if (!(p->base >= 1) || !std::isfinite(p->base)) return ERASE_ERR_INVALID_ARG;
  if (p->scaling != ERASE_ROPE_NONE && (!(p->factor >= 1) || !std::isfinite(p->factor))) return ERASE_ERR_INVALID_ARG;
  if (p->scaling == ERASE_ROPE_BY_PARTS &&
      (!(p->original_length > 0) || !std::isfinite(p->original_length) || !(p->slow >= 0) || !(p->fast > p->slow) ||
       !std::isfinite(p->fast)))
    return ERASE_ERR_INVALID_ARG;
  return ERASE_OK;
}

double amplitude_of(const erase_rope_spec& p) {
  return p.scaling == ERASE_ROPE_BY_PARTS ? 0.1 * std::log(p.factor) + 1.0 : 1.0;
}

// f_i in 64 significant bits: a table's angles are products with positions, which
// multiply its rounding (a double's reached 2^-57 turns a position).
long double frequency(const erase_rope_spec& p, int i) {
  const long double r = p.rot_dim, s = p.factor;
  long double base = p.base;
  if (p.scaling == ERASE_ROPE_NTK && p.rot_dim > 2) base *= std::pow(s, r / (r - 2));  // one pair: f = 1 for any base
  const long double g = std::pow(base, -2.0L * i / r);
  if (p.scaling == ERASE_ROPE_LINEAR) return g / s;
  if (p.scaling != ERASE_ROPE_BY_PARTS) return g;
  const long double turns = p.original_length * g / kTau, ramp = (turns - p.slow) / ((long double)p.fast - p.slow);
  const long double keep = std::min(1.0L, std::max(0.0L, ramp));
  return g * (keep + (1.0L - keep) / s);
}

// f / (2 pi) modulo 1 as a 64-bit fraction, to the nearest.
uint64_t turn_fraction(long double f) {
  return static_cast<uint64_t>(std::floor(std::ldexp(f / kTau, 64) + 0.5L));
}

// The elements of an output [n0][n1][n2][dim] do not coincide: sorted by
// stride, each dimension steps over the extent of those before.
bool distinct(const int64_t n[3], const int64_t stride[3], int64_t dim) {
  int order[3] = {0, 1, 2};
  std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
  __int128 extent = dim;
  for (int d : order) {
    if (n[d] <= 1) continue;
    if (stride[d] < extent) return false;
    extent += static_cast<__int128>(stride[d]) * (n[d] - 1);
  }
  return true;
}
bool span_ok(const int64_t n[3], const int64_t stride[3], int64_t dim) {
  __int128 span = dim;
  for (int d = 0; d < 3; ++d) {
    if (stride[d] < 0) return false;
    if (n[d] > 1) span += static_cast<__int128>(stride[d]) * (n[d] - 1);
  }
  return span < kSpan;
}

erase_status rope(const erase_rope_config* cfg, const void* q, const void* k, void* qo, void* ko,
                  const int32_t* positions, const void* table, void* stream, int inverse) {
  if (!cfg) return ERASE_ERR_INVALID_ARG;
  const erase_rope_config& c = *cfg;
  if (!known(c.dtype) || c.layout < ERASE_ROPE_HALF || c.layout > ERASE_ROPE_INTERLEAVED) return ERASE_ERR_INVALID_ARG;
  if (c.batch < 0 || c.seq < 0 || int64_t(c.batch) * c.seq >= kRows || c.q_heads < 1 || c.q_heads > 4096 ||
      c.k_heads < 0 || c.k_heads > 4096 || c.head_dim > 1024 || c.rot_dim < 2 || c.rot_dim % 2 ||
      c.rot_dim > c.head_dim || c.pos_stride < 0 ||
      (c.batch > 1 && static_cast<__int128>(c.batch) * c.pos_stride >= kSpan))
    return ERASE_ERR_SHAPE;
  if (c.start < -(int64_t(1) << 40) || c.start > (int64_t(1) << 40)) return ERASE_ERR_INVALID_ARG;
  const int64_t nq[3] = {c.batch, c.seq, c.q_heads}, nk[3] = {c.batch, c.seq, c.k_heads};
  if (!span_ok(nq, c.q_stride, c.head_dim) || !span_ok(nq, c.qo_stride, c.head_dim) ||
      !distinct(nq, c.qo_stride, c.head_dim))
    return ERASE_ERR_SHAPE;
  if (c.k_heads > 0 && (!span_ok(nk, c.k_stride, c.head_dim) || !span_ok(nk, c.ko_stride, c.head_dim) ||
                        !distinct(nk, c.ko_stride, c.head_dim)))
    return ERASE_ERR_SHAPE;
  if (c.batch == 0 || c.seq == 0) return ERASE_OK;
  const size_t es = elem(c.dtype);
  if (!q || !qo || misaligned(q, es) || misaligned(qo, es) || !table || misaligned(table, 8) ||
      misaligned(positions, 4))
    return ERASE_ERR_INVALID_ARG;
  if (c.k_heads > 0 && (!k || !ko || misaligned(k, es) || misaligned(ko, es) || qo == ko || qo == k || ko == q))
    return ERASE_ERR_INVALID_ARG;
  auto in_place = [](const void* x, const void* y, const int64_t n[3], const int64_t xs[3], const int64_t ys[3]) {
    if (x != y) return true;
    for (int d = 0; d < 3; ++d)
      if (n[d] > 1 && xs[d] != ys[d]) return false;
    return true;
  };
  if (!in_place(q, qo, nq, c.q_stride, c.qo_stride) ||
      (c.k_heads > 0 && !in_place(k, ko, nk, c.k_stride, c.ko_stride)))
    return ERASE_ERR_INVALID_ARG;
  RopeArgs a{};
  a.x[0] = q;
  a.x[1] = k;
  a.y[0] = qo;
  a.y[1] = ko;
  for (int d = 0; d < 3; ++d) {
    a.xs[0][d] = c.q_stride[d];
    a.xs[1][d] = c.k_stride[d];
    a.ys[0][d] = c.qo_stride[d];
    a.ys[1][d] = c.ko_stride[d];
  }
  a.heads[0] = c.q_heads;
  a.heads[1] = c.k_heads;
  a.batch = c.batch;
  a.seq = c.seq;
  a.dim = c.head_dim;
  a.rot = c.rot_dim;
  a.positions = positions;
  a.pos_b = c.pos_stride;
  a.pos_t = 1;
  a.start = c.start;
  a.start_t = 1;
  a.table = static_cast<const uint64_t*>(table);
  a.interleaved = c.layout == ERASE_ROPE_INTERLEAVED;
  a.inverse = inverse;
  return done(launch_rope(c.dtype == ERASE_BF16, a, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// layer norm
// ---------------------------------------------------------------------------
erase_status check_norm(const erase_norm_config* cfg) {
  if (!cfg || !known(cfg->dtype)) return ERASE_ERR_INVALID_ARG;
  if (cfg->rows < 0 || cfg->rows >= kRows || cfg->cols < 1 || cfg->cols > kNormCols) return ERASE_ERR_SHAPE;
  return ERASE_OK;
}

// ---------------------------------------------------------------------------
// dropout
// ---------------------------------------------------------------------------
erase_status dropout(const erase_dropout_config* cfg, const void* x, const void* res, void* y, const uint64_t* step,
                     void* stream) {
  if (!cfg) return ERASE_ERR_INVALID_ARG;
  const erase_dropout_config& c = *cfg;
  if (!known(c.dtype) || !(c.p >= 0 && c.p <= 1)) return ERASE_ERR_INVALID_ARG;
  if (c.rows < 0 || c.rows >= kRows || c.cols < 0 || c.cols >= kRows ||
      static_cast<__int128>(c.rows) * c.cols >= kSpan || !pitch_ok(c.rows, c.cols, c.x_ld) ||
      !pitch_ok(c.rows, c.cols, c.y_ld) || (res && !pitch_ok(c.rows, c.cols, c.res_ld)))
    return ERASE_ERR_SHAPE;
  const size_t es = elem(c.dtype);
  if (misaligned(step, 8)) return ERASE_ERR_INVALID_ARG;
  if (c.rows == 0 || c.cols == 0) return ERASE_OK;
  if (!x || !y || misaligned(x, es) || misaligned(res, es) || misaligned(y, es) ||
      !same_or_apart(y, c.y_ld, x, c.x_ld, c.rows) || (res && !same_or_apart(y, c.y_ld, res, c.res_ld, c.rows)))
    return ERASE_ERR_INVALID_ARG;
  DropArgs a{};
  a.x = x;
  a.ldx = c.x_ld;
  a.res = res;
  a.ldres = c.res_ld;
  a.y = y;
  a.ldy = c.y_ld;
  a.rows = c.rows;
  a.cols = (int)c.cols;
  a.seed = c.seed;
  a.offset = c.offset;
  a.step = step;
  drop_rate(c.p, &a);
  return done(launch_dropout(c.dtype == ERASE_BF16, a, static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

erase_status erase_rope_frequencies(const erase_rope_spec* spec, double* freq, double* amplitude) {
  if (erase_status st = check_spec(spec); st != ERASE_OK) return st;
  if (!freq || !amplitude) return ERASE_ERR_INVALID_ARG;
  for (int i = 0; i < spec->rot_dim / 2; ++i) freq[i] = static_cast<double>(frequency(*spec, i));
  *amplitude = amplitude_of(*spec);
  return ERASE_OK;
}

erase_status erase_rope_table_bytes(const erase_rope_spec* spec, size_t* bytes) {
  if (erase_status st = check_spec(spec); st != ERASE_OK) return st;
  if (!bytes) return ERASE_ERR_INVALID_ARG;
  *bytes = 8 * (size_t(spec->rot_dim) / 2 + 1);
  return ERASE_OK;
}

erase_status erase_rope_table(const erase_rope_spec* spec, void* table, void* stream) {
  if (erase_status st = check_spec(spec); st != ERASE_OK) return st;
  if (!table || misaligned(table, 8)) return ERASE_ERR_INVALID_ARG;
  const int half = spec->rot_dim / 2;
  for (int i0 = 0; i0 <= half; i0 += kRopeFill) {
    RopeFillArgs a{};
    a.table = static_cast<uint64_t*>(table) + i0;
    a.n = std::min(kRopeFill, half + 1 - i0);
    for (int i = 0; i < a.n; ++i) {
      if (i0 + i < half) {
        a.v[i] = turn_fraction(frequency(*spec, i0 + i));
      } else {
        const float amp = (float)amplitude_of(*spec);
        uint32_t bits;
        std::memcpy(&bits, &amp, 4);
        a.v[i] = bits;
      }
    }
    if (launch_rope_fill(a, static_cast<hipStream_t>(stream)) != hipSuccess) return ERASE_ERR_HIP;
  }
  return ERASE_OK;
}

erase_status erase_rope(const erase_rope_config* cfg, const void* q, const void* k, void* q_out, void* k_out,
                        const int32_t* positions, const void* table, void* stream) {
  return rope(cfg, q, k, q_out, k_out, positions, table, stream, 0);
}

erase_status erase_rope_backward(const erase_rope_config* cfg, const void* dq_out, const void* dk_out, void* dq,
                                 void* dk, const int32_t* positions, const void* table, void* stream) {
  return rope(cfg, dq_out, dk_out, dq, dk, positions, table, stream, 1);
}

erase_status erase_layer_norm(const erase_norm_config* cfg, const void* x, const float* w, const float* b, void* y,
                              float* mean, float* rstd, void* stream) {
  if (erase_status st = check_norm(cfg); st != ERASE_OK) return st;
  const erase_norm_config& c = *cfg;
  if (!(c.eps >= 0) || !std::isfinite(c.eps)) return ERASE_ERR_INVALID_ARG;
  if (!pitch_ok(c.rows, c.cols, c.x_ld) || !pitch_ok(c.rows, c.cols, c.y_ld)) return ERASE_ERR_SHAPE;
  if (misaligned(w, 4) || misaligned(b, 4) || misaligned(mean, 4) || misaligned(rstd, 4)) return ERASE_ERR_INVALID_ARG;
  if (c.rows == 0) return ERASE_OK;
  const size_t es = elem(c.dtype);
  if (!x || !y || misaligned(x, es) || misaligned(y, es) || !same_or_apart(y, c.y_ld, x, c.x_ld, c.rows) ||
      (mean && mean == rstd))
    return ERASE_ERR_INVALID_ARG;
  NormArgs a{};
  a.x = x;
  a.ldx = c.x_ld;
  a.w = w;
  a.b = b;
  a.y = y;
  a.ldy = c.y_ld;
  a.mean = mean;
  a.rstd = rstd;
  a.rows = c.rows;
  a.cols = c.cols;
  a.eps = c.eps;
  return done(launch_norm(c.dtype == ERASE_BF16, a, static_cast<hipStream_t>(stream)));
}

erase_status erase_layer_norm_backward_scratch_bytes(const erase_norm_config* cfg, size_t* bytes) {
  if (erase_status st = check_norm(cfg); st != ERASE_OK) return st;
  if (!bytes) return ERASE_ERR_INVALID_ARG;
  *bytes = size_t(8) * size_t(norm_bwd_parts(cfg->dtype == ERASE_BF16, cfg->rows, cfg->cols)) *
           size_t(norm_part_pitch(cfg->cols));
  return ERASE_OK;
}

erase_status erase_layer_norm_backward(const erase_norm_config* cfg, const void* x, const void* dy, const float* w,
                                       const float* mean, const float* rstd, const void* res, void* dx, float* dw,
                                       float* db, void* scratch, size_t scratch_bytes, void* stream) {
  size_t need = 0;
  if (erase_status st = erase_layer_norm_backward_scratch_bytes(cfg, &need); st != ERASE_OK) return st;
  const erase_norm_config& c = *cfg;
  if (!pitch_ok(c.rows, c.cols, c.x_ld) || !pitch_ok(c.rows, c.cols, c.dy_ld) ||
      (dx && !pitch_ok(c.rows, c.cols, c.dx_ld)) || (res && !pitch_ok(c.rows, c.cols, c.res_ld)))
    return ERASE_ERR_SHAPE;
  const size_t es = elem(c.dtype);
  if (misaligned(x, es) || misaligned(dy, es) || misaligned(res, es) || misaligned(dx, es) || misaligned(w, 4) ||
      misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(dw, 4) || misaligned(db, 4) || (dw && dw == db))
    return ERASE_ERR_INVALID_ARG;
  if (c.rows > 0) {
    if (!x || !dy || !mean || !rstd) return ERASE_ERR_INVALID_ARG;
    // dx may be dy or res, never x: other rows' sums may still read it
    if (dx && (dx == x || !same_or_apart(dx, c.dx_ld, dy, c.dy_ld, c.rows) ||
               (res && !same_or_apart(dx, c.dx_ld, res, c.res_ld, c.rows))))
      return ERASE_ERR_INVALID_ARG;
  }
  const bool sums = dw || db;
  if (sums && (!scratch || misaligned(scratch, 16) || scratch_bytes < need)) return ERASE_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int bf16 = c.dtype == ERASE_BF16;
  const int64_t ldp = norm_part_pitch(c.cols);
  float* part = sums ? static_cast<float*>(scratch) : nullptr;
  const int nparts = c.rows > 0 ? norm_bwd_parts(bf16, c.rows, c.cols) : 0;
  const bool strips = sums && nparts > 1 && dx != dy && norm_bwd_strips(c.rows);
  if (c.rows > 0 && (dx || sums)) {
    NormBwdArgs a{};
    a.x = x;
    a.ldx = c.x_ld;
    a.dy = dy;
    a.lddy = c.dy_ld;
    a.w = w;
    a.mean = mean;
    a.rstd = rstd;
    a.res = res;
    a.ldres = c.res_ld;
    a.dx = dx;
    a.lddx = c.dx_ld;
    a.part = part;
    a.ldpart = ldp;
    a.nparts = nparts;
    a.strips = strips;
    a.dw = dw;
    a.db = db;
    a.rows = c.rows;
    a.cols = c.cols;
    if (launch_norm_bwd(bf16, a, s) != hipSuccess) return ERASE_ERR_HIP;
  }
  return sums && nparts != 1 && !strips ? done(launch_norm_sum(part, ldp, nparts, c.cols, dw, db, s)) : ERASE_OK;
}

erase_status erase_dropout(const erase_dropout_config* cfg, const void* x, const void* res, void* y,
                           const uint64_t* step, void* stream) {
  return dropout(cfg, x, res, y, step, stream);
}

erase_status erase_dropout_backward(const erase_dropout_config* cfg, const void* dy, void* dx, const uint64_t* step,
                                    void* stream) {
  return dropout(cfg, dy, nullptr, dx, step, stream);
}

}  // extern "C"

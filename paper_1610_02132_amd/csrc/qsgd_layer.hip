// C ABI of the operators of a layer in 8 bits (see include/qsgd.h): checks of arguments, workspace
// layout, kernel launches.  Everything is checked before anything is queued.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "qsgd.h"
#include "qsgd_kernels.hpp"
#include "qsgd_layer.hpp"

namespace {

using namespace qsgd;

bool aligned(const void* p, uint64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

uint64_t size_of(uint32_t type) { return type == QSGD_TYPE_F32 ? 4 : type == QSGD_TYPE_I8 ? 1 : 2; }

uint64_t padded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// A matrix as the header describes it: of levels (I8) or of values.
bool sound(const qsgd_matrix* m, bool levels) {
  if (!m || m->reserved || m->rows >= 1ull << 31 || m->cols >= 1ull << 31 || m->ld < m->cols || m->ld >= 1ull << 46 ||
      (levels ? m->type != QSGD_TYPE_I8 : m->type > QSGD_TYPE_F16))
    return false;
  if (m->rows && m->ld >= (1ull << 46) / m->rows) return false;
  if (m->rows == 0 || m->cols == 0) return true;
  return m->data_dev && aligned(m->data_dev, levels ? 16 : size_of(m->type)) && !(levels && m->ld % 16);
}

bool shaped(const qsgd_matrix* m, uint64_t rows, uint64_t cols) { return m->rows == rows && m->cols == cols; }

// Bytes [from, to) that something covers.
struct Span { uintptr_t from, to; };
Span span(const qsgd_matrix* m) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(m->data_dev);
  if (!m->rows || !m->cols) return {p, p};
  return {p, p + ((m->rows - 1) * m->ld + m->cols) * size_of(m->type)};
}
bool meet(const Span& a, const Span& b) { return a.from < a.to && b.from < b.to && a.from < b.to && b.from < a.to; }
// Whether two matrices share an element.  Column ranges of one larger matrix (rows equally far apart) do not where the
// ranges are apart; other matrices whose extents meet count as overlapping.
bool overlap(const qsgd_matrix* x, const qsgd_matrix* y) {
  const Span a = span(x), b = span(y);
  if (!meet(a, b)) return false;
  const uint64_t ld = x->ld * size_of(x->type);
  if (ld != y->ld * size_of(y->type)) return true;
  const uint64_t wx = x->cols * size_of(x->type), wy = y->cols * size_of(y->type);
  const uint64_t d = a.from <= b.from ? (b.from - a.from) % ld : (ld - (a.from - b.from) % ld) % ld;
  return d < wx || d + wy > ld;
}
bool same_place(const qsgd_matrix* x, const qsgd_matrix* y) {
  return x->data_dev == y->data_dev && (x->ld == y->ld || x->rows <= 1);
}
// Whether n floats at p share a byte with a matrix.
bool overlap(const float* p, uint64_t n, const qsgd_matrix* m) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return p && m && meet({at, at + 4 * n}, span(m));
}
bool overlap(const float* p, uint64_t n, const float* q, uint64_t m) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p && q && meet({a, a + 4 * n}, {b, b + 4 * m});
}

// Whether the word that is added to the iteration lies in an output, which would be written while it is read.
bool iteration_in(const qsgd_draws* d, const qsgd_matrix* m) {
  if (!d || !d->iteration_dev || !m || !m->rows || !m->cols) return false;
  const uintptr_t at = reinterpret_cast<uintptr_t>(d->iteration_dev);
  const Span to = span(m);
  if (!meet({at, at + 4}, to)) return false;
  const uint64_t size = size_of(m->type), ld = m->ld * size;
  const uint64_t in_row = at < to.from ? 0 : (at - to.from) % ld;   // (between two rows it is in neither)
  return in_row < m->cols * size || in_row + 4 > ld;
}
bool iteration_in(const qsgd_draws* d, const float* p, uint64_t n) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  const uintptr_t word = d ? reinterpret_cast<uintptr_t>(d->iteration_dev) : 0;
  return p && word && meet({word, word + 4}, {at, at + 4 * n});
}

bool floats(const float* p, uint64_t n) { return n == 0 || (p && aligned(p, 4)); }

int draw_args(const qsgd_draws* d, uint64_t rows, DrawArgs& a) {
  if (!d || d->reserved || d->row_base + rows > 1ull << 32 || !aligned(d->iteration_dev, 4)) return QSGD_ERR_INVALID_ARG;
  a = {(uint32_t)d->seed, (uint32_t)(d->seed >> 32), d->stream_id, d->iteration, d->row_base, d->iteration_dev};
  return QSGD_OK;
}

constexpr uint64_t kMostThreads = 0xFFFF0000ull;   // of a launch: they are counted in 32 bits

int status(hipError_t e) { return e == hipSuccess ? QSGD_OK : QSGD_ERR_HIP; }

int dropout(const qsgd_draws* draws, float p, const qsgd_matrix* x, const qsgd_matrix* residual, const qsgd_matrix* y,
            const char* name, hipStream_t st) {
  if (!(p >= 0.0f && p <= 1.0f) || !sound(x, false) || !sound(y, false) || (residual && !sound(residual, false)))
    return QSGD_ERR_INVALID_ARG;
  if (!shaped(y, x->rows, x->cols) || y->type != x->type) return QSGD_ERR_INVALID_ARG;
  if (residual && (!shaped(residual, x->rows, x->cols) || residual->type != x->type)) return QSGD_ERR_INVALID_ARG;
  if (overlap(x, y) && !same_place(x, y)) return QSGD_ERR_INVALID_ARG;
  if (residual && overlap(residual, y) && !same_place(residual, y)) return QSGD_ERR_INVALID_ARG;
  if (iteration_in(draws, y)) return QSGD_ERR_INVALID_ARG;
  DropoutArgs a = {};
  if (int rc = draw_args(draws, x->rows, a.draws)) return rc;
  if (x->rows * ((x->cols + 7) / 8) >= kMostThreads) return QSGD_ERR_UNSUPPORTED;
  if (x->rows == 0 || x->cols == 0) return QSGD_OK;
  a.x = x->data_dev; a.x_ld = x->ld;
  a.y = y->data_dev; a.y_ld = y->ld;
  if (residual) { a.residual = residual->data_dev; a.residual_ld = residual->ld; }
  a.rows = (uint32_t)x->rows; a.cols = (uint32_t)x->cols;
  a.drop = (uint32_t)std::nearbyint(65536.0 * (double)p);
  a.scale = a.drop == 65536 ? 0.0f : 65536.0f / (float)(65536 - a.drop);
  ScopedTiming tm(name, st);
  return status(launch_dropout(a, x->type, st));
}

// ---- quantizer -------------------------------------------------------------------

// Workspace of a column form.
struct ColumnSpace {
  uint32_t strip_lanes, chunks, chunk_rows;
  uint64_t max_at, sum_at, bytes;
};
ColumnSpace column_space(uint64_t rows, uint64_t cols) {
  ColumnSpace s = {};
  plan_columns((uint32_t)rows, (uint32_t)cols, s.strip_lanes, s.chunks, s.chunk_rows);
  s.sum_at = padded(4 * cols * s.chunks);
  s.bytes = 2 * s.sum_at;
  return s;
}
// What is enough for it and for every smaller matrix's: its own bytes go up and down with the columns.
uint64_t most_column_bytes(uint64_t rows, uint64_t cols) { return 2 * padded(4 * column_numbers(rows, cols)); }

QuantizeArgs job(const qsgd_matrix* x, const DrawArgs& draws) {
  QuantizeArgs q = {};
  q.x = x->data_dev; q.ld = x->ld;
  q.rows = (uint32_t)x->rows; q.cols = (uint32_t)x->cols;
  q.draws = draws;
  return q;
}
void want_rows(QuantizeArgs& q, int8_t* levels, uint64_t ld, float* scale) {
  q.q_rows = levels; q.q_rows_ld = ld; q.row_scale = scale;
}
// scale: or null, where only the sums are wanted
void want_columns(QuantizeArgs& q, uint8_t* ws, int8_t* levels, uint64_t ld, float* scale, float* sum) {
  const ColumnSpace s = column_space(q.rows, q.cols);
  q.q_cols = levels; q.q_cols_ld = ld; q.col_scale = scale;
  q.strip_lanes = s.strip_lanes; q.chunks = s.chunks; q.chunk_rows = s.chunk_rows;
  // (without rows there is no workspace either, and nothing is read there)
  q.part_max = scale ? reinterpret_cast<uint32_t*>(s.bytes ? ws + s.max_at : reinterpret_cast<uint8_t*>(scale)) : nullptr;
  q.part_sum = sum ? reinterpret_cast<float*>(s.bytes ? ws + s.sum_at : reinterpret_cast<uint8_t*>(sum)) : nullptr;
  q.col_sum = sum;
}

int quantize(QuantizeJobs& jobs, uint32_t type, uint32_t rounding, hipStream_t st) {
  const bool stochastic = rounding == QSGD_ROUND_STOCHASTIC;
  if (plan_quantize(jobs, type) * 256 >= kMostThreads) return QSGD_ERR_UNSUPPORTED;
  {
    ScopedTiming tm("quantize_rows", st);
    if (int rc = status(launch_quantize(jobs, type, stochastic, st, false))) return rc;
  }
  bool columns = false;
  for (uint32_t j = 0; j < jobs.count; ++j) columns |= jobs.job[j].part_max || jobs.job[j].part_sum;
  if (!columns) return QSGD_OK;
  ScopedTiming tm("quantize_columns", st);
  return status(launch_quantize(jobs, type, stochastic, st, true));
}

// ---- product ---------------------------------------------------------------------

constexpr uint64_t kMostLd = 1ull << 23;
constexpr uint64_t kMostRows = 1ull << 26;      // of an operand
constexpr uint64_t kMostResults = 1ull << 38;   // of one product: workgroups are counted in 31 bits
bool too_many(uint64_t M, uint64_t N) { return M >= kMostRows || N >= kMostRows || (N && M >= kMostResults / N); }

int product(ProductArgs& p, const ProductPlan& plan, uint8_t* ws, hipStream_t st) {
  p.splits = plan.splits; p.split_k = plan.split_k;
  p.part = plan.bytes ? reinterpret_cast<int32_t*>(ws) : nullptr;
  {
    ScopedTiming tm("product", st);
    if (int rc = status(launch_products({{p}, 1, 0}, plan.kind, st))) return rc;
  }
  if (!p.part) return QSGD_OK;
  ScopedTiming tm("product_join", st);
  return status(launch_product_join(p, st));
}

// Two products whose plans are alike, each in one piece, can share a launch: plans[0] is the pair's then.  The tiles of 64
// count as one kind, with four stages where all of them run at once.
bool plan_pair(ProductPair& pair, ProductPlan (&plans)[2]) {
  auto small = [](uint32_t kind) { return kind == kProductTile64 || kind == kProductTile64Deep; };
  if (plans[0].splits != 1 || plans[1].splits != 1) return false;
  if (small(plans[0].kind) && small(plans[1].kind)) {
    uint64_t tiles = 0;
    for (const ProductArgs& p : pair.of) tiles += (uint64_t)((p.M + 63) / 64) * ((p.N + 63) / 64);
    plans[0].kind = tiles <= 512 ? kProductTile64Deep : kProductTile64;
  } else if (plans[0].kind != plans[1].kind || plans[0].kind == kProductFew) {
    return false;
  }
  for (ProductArgs& p : pair.of) { p.splits = 1; p.split_k = plans[0].split_k; }
  return true;
}


// Rows of the workspace's levels start at cache lines (8192 x 8192 x 8000: 440 us per 8192 of k with them, 493 without).
uint64_t levels_ld(uint64_t k) { return (k + 127) / 128 * 128; }

bool in_range(uint64_t a, uint64_t b, uint64_t c) { return a < 1ull << 31 && b < 1ull << 31 && c < 1ull << 31; }

ProductPlan product_plan(uint64_t M, uint64_t N, uint64_t K) {
  if (!M || !N || too_many(M, N) || K >= kMostLd) return {};   // (nothing to do, or refused)
  return plan_product((uint32_t)M, (uint32_t)N, (uint32_t)K);
}
// What is enough for it and for every smaller one: a plan's own bytes go up and down, as small products are summed in pieces.
uint64_t most_product_bytes(uint64_t M, uint64_t N, uint64_t K) {
  return !M || !N || too_many(M, N) || K >= kMostLd ? 0 : product_space(M, N, K);
}

bool room(const void* ws, size_t have, uint64_t need) { return need == 0 || (ws && aligned(ws, 16) && have >= need); }

// Why a workspace is refused.
int no_room(const void* ws, uint64_t need) { return need && (!ws || !aligned(ws, 16)) ? QSGD_ERR_INVALID_ARG : QSGD_ERR_CAPACITY; }

// Workspace of the layer: x's levels and scales, then what the product needs.  bytes: of this call; most: of this and every smaller one.
struct ForwardSpace {
  ProductPlan plan;
  uint64_t scale, rest, bytes, most;
};
ForwardSpace forward_space(uint64_t M, uint64_t N, uint64_t K) {
  ForwardSpace s = {};
  s.plan = product_plan(M, N, K);
  s.scale = padded(M * levels_ld(K));
  s.rest = s.scale + padded(4 * M);
  s.bytes = s.rest + s.plan.bytes;
  s.most = s.rest + most_product_bytes(M, N, K);
  return s;
}

// Workspace of the layer's gradients: levels and scales of its operands, the columns' maxima and sums, and what the
// products need, one after the other.
struct BackwardSpace {
  uint64_t dy_rows, dy_row_scale, w_cols, w_scale, dy_cols, dy_col_scale, x_cols, x_scale;
  uint64_t dy_space, w_space, x_space, rest, bytes, most;
  ProductPlan dx, dw;
};
BackwardSpace backward_space(uint64_t M, uint64_t N, uint64_t K) {
  BackwardSpace s = {};
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) { const uint64_t p = at; at += padded(bytes); return p; };
  s.dy_rows = take(M * levels_ld(N)); s.dy_row_scale = take(4 * M);
  s.w_cols = take(K * levels_ld(N)); s.w_scale = take(4 * K);
  s.dy_cols = take(N * levels_ld(M)); s.dy_col_scale = take(4 * N);
  s.x_cols = take(K * levels_ld(M)); s.x_scale = take(4 * K);
  const uint64_t operands = at;
  s.dy_space = take(column_space(M, N).bytes);
  s.w_space = take(column_space(N, K).bytes);
  s.x_space = take(column_space(M, K).bytes);
  s.dx = product_plan(M, K, N);
  s.dw = product_plan(N, K, M);
  s.rest = take(std::max(s.dx.bytes, s.dw.bytes));
  s.bytes = at;
  s.most = operands + most_column_bytes(M, N) + most_column_bytes(N, K) + most_column_bytes(M, K) +
           padded(std::max(most_product_bytes(M, K, N), most_product_bytes(N, K, M)));
  return s;
}

}  // namespace

extern "C" {

int qsgd_dropout(const qsgd_draws* draws, float p, const qsgd_matrix* x, const qsgd_matrix* residual, const qsgd_matrix* y,
                 void* hip_stream) {
  return dropout(draws, p, x, residual, y, "dropout", reinterpret_cast<hipStream_t>(hip_stream));
}

int qsgd_dropout_backward(const qsgd_draws* draws, float p, const qsgd_matrix* dy, const qsgd_matrix* dx, void* hip_stream) {
  return dropout(draws, p, dy, nullptr, dx, "dropout_backward", reinterpret_cast<hipStream_t>(hip_stream));
}

size_t qsgd_quantize_workspace_bytes(uint64_t rows, uint64_t cols) {
  return in_range(rows, cols, 0) && cols ? most_column_bytes(rows, cols) : 0;
}

int qsgd_quantize(const qsgd_draws* draws, uint32_t rounding, const qsgd_matrix* x, const qsgd_matrix* rows,
                  float* row_scale_dev, const qsgd_matrix* columns, float* column_scale_dev, void* workspace_dev,
                  size_t workspace_bytes, void* hip_stream) {
  if (rounding > QSGD_ROUND_STOCHASTIC || !sound(x, false) || (!rows && !columns)) return QSGD_ERR_INVALID_ARG;
  if (rows && (!sound(rows, true) || !shaped(rows, x->rows, x->cols) || !floats(row_scale_dev, x->rows) || overlap(x, rows)))
    return QSGD_ERR_INVALID_ARG;
  if (columns && (!sound(columns, true) || !shaped(columns, x->cols, x->rows) || !floats(column_scale_dev, x->cols) ||
                  overlap(x, columns) || (rows && overlap(rows, columns))))
    return QSGD_ERR_INVALID_ARG;
  const float *rs = rows ? row_scale_dev : nullptr, *cs = columns ? column_scale_dev : nullptr;
  if (overlap(rs, x->rows, cs, x->cols)) return QSGD_ERR_INVALID_ARG;
  for (const qsgd_matrix* m : {x, rows, columns})
    if (overlap(rs, x->rows, m) || overlap(cs, x->cols, m)) return QSGD_ERR_INVALID_ARG;
  if (iteration_in(draws, rows) || iteration_in(draws, columns) || iteration_in(draws, rs, x->rows) || iteration_in(draws, cs, x->cols))
    return QSGD_ERR_INVALID_ARG;
  DrawArgs d = {};
  if (rounding == QSGD_ROUND_STOCHASTIC || draws)
    if (int rc = draw_args(draws, x->rows, d)) return rc;
  const uint64_t need = columns && x->cols ? column_space(x->rows, x->cols).bytes : 0;
  if (!room(workspace_dev, workspace_bytes, need)) return no_room(workspace_dev, need);
  QuantizeJobs jobs = {1, {}, {job(x, d)}};
  if (rows && x->rows) want_rows(jobs.job[0], reinterpret_cast<int8_t*>(rows->data_dev), rows->ld, row_scale_dev);
  if (columns && x->cols)
    want_columns(jobs.job[0], reinterpret_cast<uint8_t*>(workspace_dev), reinterpret_cast<int8_t*>(columns->data_dev),
                 columns->ld, column_scale_dev, nullptr);
  return quantize(jobs, x->type, rounding, reinterpret_cast<hipStream_t>(hip_stream));
}

size_t qsgd_int_matmul_workspace_bytes(uint64_t M, uint64_t N, uint64_t K) {
  return in_range(M, N, K) ? most_product_bytes(M, N, K) : 0;
}

int qsgd_int_matmul(const qsgd_matrix* a, const float* a_scale_dev, const qsgd_matrix* b, const float* b_scale_dev,
                    const float* bias_dev, const qsgd_matrix* y, void* workspace_dev, size_t workspace_bytes,
                    void* hip_stream) {
  if (!sound(a, true) || !sound(b, true) || !sound(y, false) || a->cols != b->cols || !shaped(y, a->rows, b->rows) ||
      !floats(a_scale_dev, a->rows) || !floats(b_scale_dev, b->rows) || !aligned(bias_dev, 4) || overlap(a, y) || overlap(b, y) ||
      overlap(a_scale_dev, a->rows, y) || overlap(b_scale_dev, b->rows, y) || overlap(bias_dev, b->rows, y))
    return QSGD_ERR_INVALID_ARG;
  if (a->ld >= kMostLd || b->ld >= kMostLd || too_many(y->rows, y->cols)) return QSGD_ERR_UNSUPPORTED;
  if (y->rows == 0 || y->cols == 0) return QSGD_OK;
  const ProductPlan plan = product_plan(a->rows, b->rows, a->cols);
  const uint64_t need = plan.bytes;
  if (!room(workspace_dev, workspace_bytes, need)) return no_room(workspace_dev, need);
  ProductArgs p = {};
  p.a = reinterpret_cast<const int8_t*>(a->data_dev); p.a_ld = a->ld;
  p.b = reinterpret_cast<const int8_t*>(b->data_dev); p.b_ld = b->ld;
  p.M = (uint32_t)a->rows; p.N = (uint32_t)b->rows; p.K = (uint32_t)a->cols;
  p.a_scale = a_scale_dev; p.b_scale = b_scale_dev; p.bias = bias_dev;
  p.y = y->data_dev; p.y_ld = y->ld; p.type = y->type;
  return product(p, plan, reinterpret_cast<uint8_t*>(workspace_dev), reinterpret_cast<hipStream_t>(hip_stream));
}

size_t qsgd_linear_forward_workspace_bytes(uint64_t tokens, uint64_t outputs, uint64_t inputs) {
  return in_range(tokens, outputs, inputs) ? forward_space(tokens, outputs, inputs).most : 0;
}

int qsgd_linear_forward(const qsgd_draws* draws, uint32_t rounding, const qsgd_matrix* x, const qsgd_matrix* w,
                        const float* w_scale_dev, const float* bias_dev, const qsgd_matrix* y, void* workspace_dev,
                        size_t workspace_bytes, void* hip_stream) {
  if (rounding > QSGD_ROUND_STOCHASTIC || !sound(x, false) || !sound(w, true) || !sound(y, false) || x->cols != w->cols ||
      !shaped(y, x->rows, w->rows) || y->type != x->type || !floats(w_scale_dev, w->rows) || !aligned(bias_dev, 4) ||
      overlap(x, y) || overlap(w, y) || overlap(w_scale_dev, w->rows, y) || overlap(bias_dev, w->rows, y) || iteration_in(draws, y))
    return QSGD_ERR_INVALID_ARG;
  if (w->ld >= kMostLd || levels_ld(x->cols) >= kMostLd || too_many(y->rows, y->cols)) return QSGD_ERR_UNSUPPORTED;
  DrawArgs d = {};
  if (rounding == QSGD_ROUND_STOCHASTIC || draws)
    if (int rc = draw_args(draws, x->rows, d)) return rc;
  if (y->rows == 0 || y->cols == 0) return QSGD_OK;
  const ForwardSpace s = forward_space(x->rows, w->rows, x->cols);
  if (!room(workspace_dev, workspace_bytes, s.bytes)) return no_room(workspace_dev, s.bytes);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  uint8_t* ws = reinterpret_cast<uint8_t*>(workspace_dev);
  ProductArgs p = {};
  p.b = reinterpret_cast<const int8_t*>(w->data_dev); p.b_ld = w->ld;
  p.M = (uint32_t)x->rows; p.N = (uint32_t)w->rows; p.K = (uint32_t)x->cols;
  p.b_scale = w_scale_dev; p.bias = bias_dev;
  p.y = y->data_dev; p.y_ld = y->ld; p.type = y->type;
  if (linear_few_fits(p.M, p.N, p.K)) {
    ScopedTiming tm("linear_few", st);
    return status(launch_linear_few({p, x->data_dev, x->ld, d}, x->type, rounding == QSGD_ROUND_STOCHASTIC, st));
  }
  const uint64_t ld = levels_ld(x->cols);
  QuantizeJobs jobs = {1, {}, {job(x, d)}};
  QuantizeArgs& q = jobs.job[0];
  want_rows(q, reinterpret_cast<int8_t*>(ws), ld, reinterpret_cast<float*>(ws + s.scale));
  if (int rc = quantize(jobs, x->type, rounding, st)) return rc;
  p.a = q.q_rows; p.a_ld = ld;
  p.a_scale = q.row_scale;
  return product(p, s.plan, ws + s.rest, st);
}

size_t qsgd_linear_backward_workspace_bytes(uint64_t tokens, uint64_t outputs, uint64_t inputs) {
  if (!in_range(tokens, outputs, inputs) || tokens >= kMostLd || outputs >= kMostLd) return 0;
  return backward_space(tokens, outputs, inputs).most;
}

int qsgd_linear_backward(const qsgd_draws* draws, uint32_t rounding, const qsgd_matrix* x, const qsgd_matrix* w,
                         const qsgd_matrix* dy, const qsgd_matrix* dx, const qsgd_matrix* dw, float* db_dev,
                         void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
  if (rounding > QSGD_ROUND_STOCHASTIC || !sound(x, false) || !sound(w, false) || !sound(dy, false) || x->cols != w->cols ||
      !shaped(dy, x->rows, w->rows) || w->type != x->type || dy->type != x->type || (!dx && !dw && !db_dev) ||
      !aligned(db_dev, 4))
    return QSGD_ERR_INVALID_ARG;
  const qsgd_matrix *in[3] = {x, w, dy}, *out[2] = {dx, dw};
  if (dx && (!sound(dx, false) || !shaped(dx, x->rows, x->cols) || dx->type != x->type)) return QSGD_ERR_INVALID_ARG;
  if (dw && (!sound(dw, false) || !shaped(dw, w->rows, w->cols) || dw->type != QSGD_TYPE_F32)) return QSGD_ERR_INVALID_ARG;
  for (const auto* o : out)
    for (const auto* i : in)
      if (o && overlap(o, i)) return QSGD_ERR_INVALID_ARG;
  if (dx && dw && overlap(dx, dw)) return QSGD_ERR_INVALID_ARG;
  for (const qsgd_matrix* m : {x, w, dy, dx, dw})
    if (overlap(db_dev, w->rows, m)) return QSGD_ERR_INVALID_ARG;
  if (iteration_in(draws, dx) || iteration_in(draws, dw) || iteration_in(draws, db_dev, w->rows)) return QSGD_ERR_INVALID_ARG;
  const uint64_t M = x->rows, N = w->rows, K = x->cols;
  if (levels_ld(N) >= kMostLd || levels_ld(M) >= kMostLd || too_many(M, K) || too_many(N, K)) return QSGD_ERR_UNSUPPORTED;
  DrawArgs d = {};
  if (rounding == QSGD_ROUND_STOCHASTIC || draws) {
    if (int rc = draw_args(draws, M, d)) return rc;
  }
  const BackwardSpace s = backward_space(M, N, K);
  if (!room(workspace_dev, workspace_bytes, s.bytes)) return no_room(workspace_dev, s.bytes);
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  uint8_t* ws = reinterpret_cast<uint8_t*>(workspace_dev);
  auto levels = [&](uint64_t at) { return reinterpret_cast<int8_t*>(ws + at); };
  auto scales = [&](uint64_t at) { return reinterpret_cast<float*>(ws + at); };
  DrawArgs draws_w = d, draws_x = d;
  draws_w.stream_id += 1; draws_w.row_base = 0;
  draws_x.stream_id += 2;
  const bool want_dx = dx && M && K, want_dw = dw && N && K, want_db = db_dev && N;
  QuantizeJobs jobs = {};
  {
    QuantizeArgs& q = jobs.job[jobs.count++] = job(dy, d);
    if (want_dx) want_rows(q, levels(s.dy_rows), levels_ld(N), scales(s.dy_row_scale));
    if (want_dw || want_db)
      want_columns(q, ws + s.dy_space, levels(s.dy_cols), levels_ld(M), want_dw ? scales(s.dy_col_scale) : nullptr,
                   want_db ? db_dev : nullptr);
  }
  if (want_dx) {
    QuantizeArgs& q = jobs.job[jobs.count++] = job(w, draws_w);
    want_columns(q, ws + s.w_space, levels(s.w_cols), levels_ld(N), scales(s.w_scale), nullptr);
  }
  if (want_dw) {
    QuantizeArgs& q = jobs.job[jobs.count++] = job(x, draws_x);
    want_columns(q, ws + s.x_space, levels(s.x_cols), levels_ld(M), scales(s.x_scale), nullptr);
  }
  if (int rc = quantize(jobs, x->type, rounding, st)) return rc;
  ProductPair pair = {};
  ProductPlan plans[2];
  if (want_dw) {
    ProductArgs& p = pair.of[pair.count];
    p.a = levels(s.dy_cols); p.b = levels(s.x_cols); p.a_ld = p.b_ld = levels_ld(M);
    p.M = (uint32_t)N; p.N = (uint32_t)K; p.K = (uint32_t)M;
    p.a_scale = scales(s.dy_col_scale); p.b_scale = scales(s.x_scale);
    p.y = dw->data_dev; p.y_ld = dw->ld; p.type = QSGD_TYPE_F32;
    plans[pair.count++] = s.dw;
  }
  if (want_dx) {
    ProductArgs& p = pair.of[pair.count];
    p.a = levels(s.dy_rows); p.b = levels(s.w_cols); p.a_ld = p.b_ld = levels_ld(N);
    p.M = (uint32_t)M; p.N = (uint32_t)K; p.K = (uint32_t)N;
    p.a_scale = scales(s.dy_row_scale); p.b_scale = scales(s.w_scale);
    p.y = dx->data_dev; p.y_ld = dx->ld; p.type = dx->type;
    plans[pair.count++] = s.dx;
  }
  if (pair.count == 2 && plan_pair(pair, plans)) {   // both in one launch
    ScopedTiming tm("product", st);
    return status(launch_products(pair, plans[0].kind, st));
  }
  for (uint32_t i = 0; i < pair.count; ++i)
    if (int rc = product(pair.of[i], plans[i], ws + s.rest, st)) return rc;
  return QSGD_OK;
}

}  // extern "C"

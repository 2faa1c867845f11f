// C-ABI entry points of 4-bit and 8-bit buffers, grouped products and the order of groups: argument checks and kernel dispatch.
#include "api_checks.h"
#include "grouped.h"
#include "mx8.h"

using namespace poetx;

namespace {

int check_desc(const poetx_grouped_desc* d) {
  if (!d || d->d_in <= 0 || d->d_out <= 0 || d->groups <= 0 || d->rows < 0 || !dtype_ok(d->dtype) || d->reserved != 0) return POETX_ERR_INVALID_ARG;
  if ((d->flags & ~(POETX_GROUPED_W_MX4 | POETX_GROUPED_X_MX4 | POETX_GROUPED_X_MX8)) != 0) return POETX_ERR_INVALID_ARG;
  if ((d->flags & POETX_GROUPED_X_MX4) && (d->flags & POETX_GROUPED_X_MX8)) return POETX_ERR_INVALID_ARG;
  if ((d->flags & POETX_GROUPED_X_MX4) && !(d->flags & POETX_GROUPED_W_MX4)) return POETX_ERR_INVALID_ARG;
  if ((d->flags & POETX_GROUPED_W_MX4) && d->dtype != POETX_BF16) return POETX_ERR_UNSUPPORTED;
  const i64 wide = d->d_in > d->d_out ? d->d_in : d->d_out;
  if (wide >= (1 << 24) || d->rows >= (1ll << 30) || (i64)d->groups * d->d_out >= (1ll << 31) || d->rows * wide >= kMostElements ||
      (i64)d->groups * d->d_out * d->d_in >= kMostElements)
    return POETX_ERR_UNSUPPORTED;
  return POETX_OK;
}

size_t weight_bytes(const poetx_grouped_desc* d) {
  const i64 rows = (i64)d->groups * d->d_out;
  return d->flags & POETX_GROUPED_W_MX4 ? mx4::bytes(rows, d->d_in) : (size_t)rows * d->d_in * esize(d->dtype);
}
// the weight's values
size_t dequantised_bytes(const poetx_grouped_desc* d) { return align256((size_t)d->groups * d->d_out * d->d_in * 2); }

// X in four bits, as values
size_t rounded_bytes(const poetx_grouped_desc* d) { return align256((size_t)d->rows * d->d_in * 2) + align256(mx4::bytes(d->rows, d->d_in)); }

// fp32 sums of contractions that are split among workgroups, where the tensors allow the streaming kernels
size_t parts_bytes(const poetx_grouped_desc* d) {
  size_t most = 0;
  for (const grouped::Dir dir : {grouped::FWD, grouped::INPUT}) {
    if (grouped::few_supported(d->dtype, dir, d->rows, d->d_in, d->d_out, d->groups, grouped::DENSE_WEIGHT)) continue;
    grouped::Call c = {};
    c.rows = d->rows;
    c.m = d->d_in;
    c.n = d->d_out;
    c.groups = d->groups;
    if (!grouped::stream_supported(d->dtype, dir, c)) continue;
    const size_t p = grouped::plan(d->dtype, dir, c, true, ~(size_t)0).parts;
    most = p > most ? p : most;
  }
  return align256(most);
}

// What the 4-bit forms of the operands take; parts of the products follow.
size_t operand_bytes(const poetx_grouped_desc* d) {
  if (!(d->flags & POETX_GROUPED_W_MX4) || d->rows == 0) return 0;
  if (!(d->flags & POETX_GROUPED_X_MX4)) return dequantised_bytes(d);
  const size_t codes = align256(grouped::codes_workspace_bytes(d)), values = dequantised_bytes(d) + rounded_bytes(d);
  return codes > values ? codes : values;
}
// Weight gradient of an 8-bit X.  The workspace: X's values, in rows of whole vectors; dZ again in such rows, where its own have another length; then fp32 sums of a contraction that is
// split among workgroups, or of gradients whose rows are no whole vectors.
struct Held {
  i64 ldx, lddz;      // lddz: 0 where dZ is taken as it is
  size_t x, dz, sums;
};
grouped::Call held_call(const poetx_grouped_desc* d, const Held& h) {
  grouped::Call c = {};
  c.rows = d->rows;
  c.m = d->d_in;
  c.n = d->d_out;
  c.groups = d->groups;
  c.ld_in = h.ldx;
  c.ld_in2 = h.lddz;
  c.ld_out = d->d_in;
  c.row_in = (int)h.ldx;
  c.row_in2 = (int)h.lddz;
  return c;
}
Held held_of(const poetx_grouped_desc* d) {
  const size_t es = esize(d->dtype);
  const i64 v = 16 / (i64)es;
  Held h;
  h.ldx = (d->d_in + v - 1) / v * v;
  h.lddz = d->d_out % v ? (d->d_out + v - 1) / v * v : 0;
  h.x = align256((size_t)d->rows * h.ldx * es);
  h.dz = align256((size_t)d->rows * h.lddz * es);
  const grouped::Call c = held_call(d, h);
  h.sums = grouped::weight_stream_supported(d->dtype, c) ? align256(grouped::plan(d->dtype, grouped::WEIGHT, c, true, ~(size_t)0).parts) : 0;
  return h;
}
size_t workspace_bytes(const poetx_grouped_desc* d) {
  if (d->rows == 0) return 0;
  if (!(d->flags & POETX_GROUPED_X_MX8)) return operand_bytes(d) + parts_bytes(d);
  const Held h = held_of(d);
  return h.x + h.dz + h.sums;
}

// A 4-bit weight's values, made in the workspace, for the products that do not decode it themselves.
const void* dense_weight(const poetx_grouped_desc* d, const void* W, const int32_t* offsets, void* ws, hipStream_t st) {
  if (!(d->flags & POETX_GROUPED_W_MX4)) return W;
  StageTimer tm(POETX_STAGE_DEQUANT, st);
  mx4_dequantize_groups_launch(W, d->groups, d->d_out, d->d_in, offsets, d->rows, ws, st);
  return ws;
}

// scratch: for the parts of a split contraction, behind what the operands take of the workspace
void product(const poetx_grouped_desc* d, grouped::Dir dir, const grouped::Call& c, void* ws, size_t ws_bytes, hipStream_t st) {
  StageTimer tm(POETX_STAGE_DENSE, st);
  const int dtype = d->dtype;
  if (grouped::few_supported(dtype, dir, c.rows, c.m, c.n, c.groups, grouped::DENSE_WEIGHT)) return grouped::few_dense(dtype, c, st);
  const size_t before = operand_bytes(d);
  const size_t scratch = ws && ((uintptr_t)ws & 15) == 0 && ws_bytes > before ? ws_bytes - before : 0;
  const grouped::Plan p = grouped::plan(dtype, dir, c, grouped::stream_supported(dtype, dir, c), scratch);
  if (p.kernel >= grouped::STREAM_256) grouped::stream_launch(dtype, dir, p, c, (char*)ws + before, st);
  else grouped::edge_launch(dtype, dir, p.kernel, c, st);
}

inline bool enough(const poetx_grouped_desc* d, const void* ws, size_t ws_bytes) { return ws && ((uintptr_t)ws & 15) == 0 && ws_bytes >= workspace_bytes(d); }

// Forward and input gradient: in is rows x d_i, out rows x d_o.  needs_ws: the call cannot do without its scratch.
int check_rows_call(const poetx_grouped_desc* d, const void* in, i64 ld_in, int d_i, const void* W, const int32_t* offsets, const void* out, i64 ld_out,
                    int d_o, bool needs_ws, const void* ws, size_t ws_bytes) {
  const int rc = check_desc(d);
  if (rc != POETX_OK) return rc;
  if (d->flags & POETX_GROUPED_X_MX8) return POETX_ERR_UNSUPPORTED;
  if (!W || !offsets || (d->rows > 0 && (!in || !out))) return POETX_ERR_INVALID_ARG;
  if (ld_in < d_i || ld_out < d_o) return POETX_ERR_BAD_SHAPE;
  if (d->rows > 0 && (ld_in >= kMostElements / d->rows || ld_out >= kMostElements / d->rows)) return POETX_ERR_UNSUPPORTED;
  const size_t es = esize(d->dtype), ob = span(d->rows, d_o, ld_out, es);
  if ((d->flags & POETX_GROUPED_W_MX4) && ((uintptr_t)W & 15)) return POETX_ERR_INVALID_ARG;
  if (overlap(out, ob, in, span(d->rows, d_i, ld_in, es)) || overlap(out, ob, W, weight_bytes(d)) || overlap(out, ob, offsets, 4 * ((size_t)d->groups + 1)))
    return POETX_ERR_INVALID_ARG;
  if (needs_ws && d->rows > 0 && !enough(d, ws, ws_bytes)) return POETX_ERR_WORKSPACE;
  return POETX_OK;
}

}  // namespace

extern "C" {

size_t poetx_mx4_bytes(int64_t rows, int32_t cols) {
  if (rows <= 0 || cols <= 0 || rows >= kMostElements / cols) return 0;
  return mx4::bytes(rows, cols);
}

int poetx_mx4_quantize(const void* X, int32_t dtype, int64_t rows, int32_t cols, int64_t ld, void* Q, void* stream) {
  const int rc = check_matrix(X, dtype, rows, cols, ld);
  if (rc != POETX_OK) return rc;
  if (!Q || ((uintptr_t)Q & 15) || overlap(X, span(rows, cols, ld, esize(dtype)), Q, mx4::bytes(rows, cols))) return POETX_ERR_INVALID_ARG;
  StageTimer tm(POETX_STAGE_DEQUANT, (hipStream_t)stream);
  mx4_quantize_launch(dtype, X, rows, cols, ld, Q, (hipStream_t)stream);
  return launch_status();
}

int poetx_mx4_dequantize(const void* Q, int64_t rows, int32_t cols, int32_t dtype, void* out, int64_t ld, void* stream) {
  const int rc = check_matrix(out, dtype, rows, cols, ld);
  if (rc != POETX_OK) return rc;
  if (!Q || ((uintptr_t)Q & 15) || overlap(out, span(rows, cols, ld, esize(dtype)), Q, mx4::bytes(rows, cols))) return POETX_ERR_INVALID_ARG;
  StageTimer tm(POETX_STAGE_DEQUANT, (hipStream_t)stream);
  mx4_dequantize_launch(Q, rows, cols, dtype, out, ld, (hipStream_t)stream);
  return launch_status();
}

size_t poetx_grouped_workspace_bytes(const poetx_grouped_desc* desc) { return check_desc(desc) == POETX_OK ? workspace_bytes(desc) : 0; }

int poetx_grouped_fwd(const poetx_grouped_desc* d, const void* X, int64_t ldx, const void* W, const int32_t* offsets, void* Z, int64_t ldz, void* ws,
                      size_t ws_bytes, void* stream) {
  // dense weights do without scratch, and so does a 4-bit one: it can always be decoded on the way (see the header)
  const int rc = check_rows_call(d, X, ldx, d ? d->d_in : 0, W, offsets, Z, ldz, d ? d->d_out : 0, d && (d->flags & POETX_GROUPED_X_MX4), ws, ws_bytes);
  if (rc != POETX_OK || d->rows == 0) return rc;
  hipStream_t st = (hipStream_t)stream;
  const bool mx4 = d->flags & POETX_GROUPED_W_MX4, both = d->flags & POETX_GROUPED_X_MX4, whole = mx4 && enough(d, ws, ws_bytes);
  const bool values = mx4 && !both && grouped::values_supported(d, X, ldx, Z, ldz);
  const bool few = mx4 && grouped::few_supported(d->dtype, grouped::FWD, d->rows, d->d_in, d->d_out, d->groups, both ? grouped::CODES_MX4 : values ? grouped::VALUES_STREAMED_MX4 : grouped::VALUES_MX4);
  if (both && few) {
    {
      StageTimer tm(POETX_STAGE_DEQUANT, st);
      mx4_quantize_launch(POETX_BF16, X, d->rows, d->d_in, ldx, ws, st, offsets, d->groups);
    }
    StageTimer tm(POETX_STAGE_DENSE, st);
    grouped::few_codes(d, ws, W, offsets, Z, ldz, st);
    return launch_status();
  }
  if (both && grouped::codes_supported(d, Z, ldz)) {
    grouped::codes_launch(d, X, ldx, W, offsets, Z, ldz, ws, st);
    return launch_status();
  }
  if (values) {
    const size_t sums = whole ? workspace_bytes(d) : ws && ((uintptr_t)ws & 15) == 0 ? ws_bytes : 0;
    if (grouped::values_launch(d, X, ldx, W, offsets, Z, ldz, few, whole, ws, sums, parts_bytes(d), st)) return launch_status();
  }
  if (mx4 && !both && (few || !whole)) {
    StageTimer tm(POETX_STAGE_DENSE, st);
    grouped::few_values(d, X, ldx, W, offsets, Z, ldz, st);
    return launch_status();
  }
  const void* w = dense_weight(d, W, offsets, ws, st);
  if (d->flags & POETX_GROUPED_X_MX4) {
    char* values = (char*)ws + dequantised_bytes(d);
    char* codes = values + align256((size_t)d->rows * d->d_in * 2);
    StageTimer tm(POETX_STAGE_DEQUANT, st);
    mx4_quantize_launch(POETX_BF16, X, d->rows, d->d_in, ldx, codes, st, offsets, d->groups);
    mx4_dequantize_launch(codes, d->rows, d->d_in, POETX_BF16, values, d->d_in, st);
    X = values;
    ldx = d->d_in;
  }
  product(d, grouped::FWD, grouped::Call{X, nullptr, w, Z, ldx, 0, ldz, offsets, d->rows, d->d_in, d->d_out, d->groups, 0}, ws, ws_bytes, st);
  return launch_status();
}

int poetx_grouped_bwd_input(const poetx_grouped_desc* d, const void* dZ, int64_t lddz, const void* W, const int32_t* offsets, void* dX, int64_t lddx,
                            void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_rows_call(d, dZ, lddz, d ? d->d_out : 0, W, offsets, dX, lddx, d ? d->d_in : 0, d && (d->flags & POETX_GROUPED_W_MX4), ws, ws_bytes);
  if (rc != POETX_OK || d->rows == 0) return rc;
  hipStream_t st = (hipStream_t)stream;
  const void* w = dense_weight(d, W, offsets, ws, st);
  product(d, grouped::INPUT, grouped::Call{dZ, nullptr, w, dX, lddz, 0, lddx, offsets, d->rows, d->d_in, d->d_out, d->groups, 0}, ws, ws_bytes, st);
  return launch_status();
}

int poetx_grouped_bwd_weight(const poetx_grouped_desc* d, const void* X, int64_t ldx, const void* dZ, int64_t lddz, const int32_t* offsets, float* dW,
                             int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_desc(d);
  if (rc != POETX_OK) return rc;
  if (!offsets || !dW || (d->rows > 0 && (!X || !dZ))) return POETX_ERR_INVALID_ARG;
  if (d->flags & POETX_GROUPED_W_MX4) return POETX_ERR_UNSUPPORTED;
  const bool mx8 = d->flags & POETX_GROUPED_X_MX8;
  if (mx8) ldx = d->d_in;      // of its values
  if (ldx < d->d_in || lddz < d->d_out) return POETX_ERR_BAD_SHAPE;
  if (d->rows > 0 && (ldx >= kMostElements / d->rows || lddz >= kMostElements / d->rows)) return POETX_ERR_UNSUPPORTED;
  const size_t es = esize(d->dtype), ob = (size_t)d->groups * d->d_out * d->d_in * sizeof(float);
  const size_t xb = mx8 && d->rows > 0 ? mx8::bytes(d->rows, d->d_in) : span(d->rows, d->d_in, ldx, es), zb = span(d->rows, d->d_out, lddz, es);
  if (mx8 && ((uintptr_t)X & 15)) return POETX_ERR_INVALID_ARG;
  if (overlap(dW, ob, X, xb) || overlap(dW, ob, dZ, zb) || overlap(dW, ob, offsets, 4 * ((size_t)d->groups + 1))) return POETX_ERR_INVALID_ARG;
  hipStream_t st = (hipStream_t)stream;
  if (mx8 && d->rows > 0) {
    if (!enough(d, ws, ws_bytes)) return POETX_ERR_WORKSPACE;
    const size_t wb = workspace_bytes(d);
    if (overlap(ws, wb, X, xb) || overlap(ws, wb, dZ, zb) || overlap(ws, wb, dW, ob) || overlap(ws, wb, offsets, 4 * ((size_t)d->groups + 1))) return POETX_ERR_INVALID_ARG;
    const Held h = held_of(d);
    grouped::Call c = held_call(d, h);
    c.in = ws;
    c.in2 = dZ;
    c.out = dW;
    c.offsets = offsets;
    c.accumulate = accumulate != 0;
    const bool whole = ((uintptr_t)dZ & 15) == 0 && lddz % (16 / (i64)es) == 0;      // as its rows are, that is
    {
      StageTimer tm(POETX_STAGE_DEQUANT, st);
      mx8_dequantize_launch(X, d->rows, d->d_in, d->dtype, ws, h.ldx, st, offsets, d->groups);
      if (h.lddz) {
        c.in2 = (char*)ws + h.x;
        relay_rows_launch(d->dtype, dZ, d->rows, d->d_out, lddz, (char*)ws + h.x, h.lddz, st, offsets, d->groups, true);
      } else {
        c.ld_in2 = lddz;
      }
    }
    StageTimer tm(POETX_STAGE_DENSE, st);
    const bool streams = (h.lddz || whole) && grouped::weight_stream_supported(d->dtype, c) && ((uintptr_t)dW & 15) == 0;
    const grouped::Plan p = grouped::plan(d->dtype, grouped::WEIGHT, c, streams, h.sums);
    if (p.kernel >= grouped::STREAM_256) grouped::stream_launch(d->dtype, grouped::WEIGHT, p, c, (char*)ws + h.x + h.dz, st);
    else grouped::edge_launch(d->dtype, grouped::WEIGHT, p.kernel, c, st);
    return launch_status();
  }
  product(d, grouped::WEIGHT, grouped::Call{X, dZ, nullptr, dW, ldx, lddz, d->d_in, offsets, d->rows, d->d_in, d->d_out, d->groups, accumulate != 0}, nullptr, 0, st);
  return launch_status();
}

size_t poetx_mx8_bytes(int64_t rows, int32_t cols) {
  if (rows <= 0 || cols <= 0 || rows >= kMostElements / cols) return 0;
  return mx8::bytes(rows, cols);
}

int poetx_mx8_quantize(const void* X, int32_t dtype, int64_t rows, int32_t cols, int64_t ld, void* Q, void* stream) {
  const int rc = check_matrix(X, dtype, rows, cols, ld);
  if (rc != POETX_OK) return rc;
  if (!Q || ((uintptr_t)Q & 15) || overlap(X, span(rows, cols, ld, esize(dtype)), Q, mx8::bytes(rows, cols))) return POETX_ERR_INVALID_ARG;
  StageTimer tm(POETX_STAGE_DEQUANT, (hipStream_t)stream);
  mx8_quantize_launch(dtype, X, rows, cols, ld, Q, (hipStream_t)stream);
  return launch_status();
}

int poetx_mx8_dequantize(const void* Q, int64_t rows, int32_t cols, int32_t dtype, void* out, int64_t ld, void* stream) {
  const int rc = check_matrix(out, dtype, rows, cols, ld);
  if (rc != POETX_OK) return rc;
  if (!Q || ((uintptr_t)Q & 15) || overlap(out, span(rows, cols, ld, esize(dtype)), Q, mx8::bytes(rows, cols))) return POETX_ERR_INVALID_ARG;
  StageTimer tm(POETX_STAGE_DEQUANT, (hipStream_t)stream);
  mx8_dequantize_launch(Q, rows, cols, dtype, out, ld, (hipStream_t)stream);
  return launch_status();
}

size_t poetx_group_order_workspace_bytes(int64_t n, int32_t groups) {
  return n < 0 || n >= (1ll << 31) || groups <= 0 || groups > POETX_GROUP_ORDER_MAX ? 0 : group_order_workspace_bytes(n, groups);
}

int poetx_group_order(const int32_t* ids, int64_t n, int32_t groups, int32_t* offsets, int32_t* order, void* ws, size_t ws_bytes, void* stream) {
  if (!offsets || n < 0 || groups <= 0 || (n > 0 && (!ids || !order))) return POETX_ERR_INVALID_ARG;
  if (groups > POETX_GROUP_ORDER_MAX || n >= (1ll << 31)) return POETX_ERR_UNSUPPORTED;
  const size_t ib = 4 * (size_t)n, ob = 4 * ((size_t)groups + 1);
  if (overlap(ids, ib, order, ib) || overlap(ids, ib, offsets, ob) || overlap(order, ib, offsets, ob)) return POETX_ERR_INVALID_ARG;
  const size_t need = group_order_workspace_bytes(n, groups);
  if (need > 0) {
    if (!ws || ((uintptr_t)ws & 3) || ws_bytes < need) return POETX_ERR_WORKSPACE;
    if (overlap(ws, need, ids, ib) || overlap(ws, need, order, ib) || overlap(ws, need, offsets, ob)) return POETX_ERR_INVALID_ARG;
  }
  StageTimer tm(POETX_STAGE_LAYOUT, (hipStream_t)stream);
  group_order_launch(ids, n, groups, offsets, order, ws, (hipStream_t)stream);
  return launch_status();
}

}  // extern "C"

// C-ABI entry points of the gated feed-forward block: argument checks and kernel dispatch.
#include "api_checks.h"
#include "gated.h"

using namespace poetx;

namespace {

int check_desc(const poetx_gated_desc* d) {
  if (!d || d->d_in <= 0 || d->d_hidden <= 0 || d->groups <= 0 || d->rows < 0 || !dtype_ok(d->dtype)) return POETX_ERR_INVALID_ARG;
  if ((d->flags & ~(POETX_GATED_W_MX4 | POETX_GATED_HELD_MX8)) != 0 || (d->activation != POETX_GATED_SILU && d->activation != POETX_GATED_GELU)) return POETX_ERR_INVALID_ARG;
  if ((d->flags & POETX_GATED_W_MX4) && d->dtype != POETX_BF16) return POETX_ERR_UNSUPPORTED;
  const i64 out = 2 * (i64)d->d_hidden, wide = d->d_in > out ? d->d_in : out;
  if (wide >= (1 << 24) || d->rows >= (1ll << 30) || d->groups * out >= (1ll << 31) || d->rows * wide >= kMostElements || d->groups * out * d->d_in >= kMostElements)
    return POETX_ERR_UNSUPPORTED;
  return POETX_OK;
}

size_t weight_bytes(const poetx_gated_desc* d) {
  const i64 rows = 2 * (i64)d->groups * d->d_hidden;
  return d->flags & POETX_GATED_W_MX4 ? mx4::bytes(rows, d->d_in) : (size_t)rows * d->d_in * esize(d->dtype);
}

// A tensor of a call: `bytes` from its first element to its last one's end.
struct Area {
  const void* p;
  size_t bytes;
};
bool apart(const Area* outs, int no, const Area* ins, int ni) {
  for (int i = 0; i < no; ++i) {
    if (!outs[i].p) continue;
    for (int j = 0; j < ni; ++j)
      if (ins[j].p && overlap(outs[i].p, outs[i].bytes, ins[j].p, ins[j].bytes)) return false;
  }
  return true;
}
// Do two matrices of one leading dimension share an element?  They may lie between each other's rows.
bool pair_apart(const void* a, const void* b, i64 rows, i64 cols, i64 ld, size_t es) {
  if (!overlap(a, span(rows, cols, ld, es), b, span(rows, cols, ld, es))) return true;
  const i64 pitch = ld * (i64)es, d = (i64)((uintptr_t)b - (uintptr_t)a) % pitch, off = d < 0 ? d + pitch : d;
  return off >= cols * (i64)es && pitch - off >= cols * (i64)es;
}

bool ld_fits(i64 rows, i64 ld) { return rows == 0 || ld < kMostElements / rows; }

// G | U as one product of 2n columns: what the choice of kernels goes by
grouped::Call product_of(const poetx_gated_desc* d, const void* X, i64 ldx, const void* W, const int32_t* offsets) {
  return grouped::Call{X, nullptr, W, nullptr, ldx, 0, 2 * (i64)d->d_hidden, offsets, d->rows, d->d_in, 2 * d->d_hidden, d->groups, 0};
}
bool few(const poetx_gated_desc* d, grouped::Weight w) { return grouped::few_supported(d->dtype, grouped::FWD, d->rows, d->d_in, 2 * d->d_hidden, d->groups, w); }
// fp32 sums of contractions that are split among workgroups, where the tensors allow the streaming kernels
size_t stream_sums_bytes(const poetx_gated_desc* d) {
  const grouped::Call c = product_of(d, nullptr, d->d_in, nullptr, nullptr);
  const gated::Call q{nullptr, nullptr, d->d_in, nullptr, d->rows, d->d_in, d->d_hidden, d->groups, gated::FWD, {}};
  return d->d_hidden % 2 == 0 && gated::stream_supported(d->dtype, q) ? align256(grouped::plan(d->dtype, grouped::FWD, c, true, ~(size_t)0).parts) : 0;
}
// Where a row of X is no whole 16-byte vectors, by its length alone: are X and a dense W laid anew in rows that are, zeros behind their columns, for the streams?  A model of the times with and without
// says so; a 4-bit weight, whose rows are whole anyway, leaves only X.  us, without / with: 11484 rows, 916 -> 2 x 6560 in four bits 897 / 366; 309 rows, 3366 -> 2 x 416 in four bits 37.5 / 19.5; 2048
// rows, 4001 -> 2 x 4000 398 / 154; 4000 rows over 8 groups, 1001 -> 2 x 2000 116 / 100; fp32 1405 rows, 1014 -> 2 x 544 59.9 / 54.5.
bool relaid(const poetx_gated_desc* d, poetx_gated_desc* as) {
  const i64 es = (i64)esize(d->dtype), v = 16 / es;
  const bool four = d->flags & POETX_GATED_W_MX4;
  if (d->d_in % v == 0 || few(d, four ? grouped::VALUES_MX4 : grouped::DENSE_WEIGHT)) return false;
  *as = *d;
  as->d_in = (int)((d->d_in + v - 1) / v * v);
  if (four) return true;
  const gated::Call q{nullptr, nullptr, as->d_in, nullptr, d->rows, as->d_in, d->d_hidden, d->groups, gated::FWD, {}};
  if (!gated::stream_supported(d->dtype, q)) return false;
  const double copies = 6 + ((double)d->rows + 2. * d->groups * d->d_hidden) * (d->d_in + as->d_in) * es / 4.5e6;
  const grouped::Call c = product_of(d, nullptr, d->d_in, nullptr, nullptr), w = product_of(as, nullptr, as->d_in, nullptr, nullptr);
  return copies + grouped::plan(d->dtype, grouped::FWD, w, true, 0).us < grouped::plan(d->dtype, grouped::FWD, c, false, 0).us;
}

// The workspace: X again, where it is laid anew; a 4-bit weight's values, where a call may need them (which of two kernels for a handful of rows takes one depends on its tensors), or a dense one laid
// anew; then sums.
struct Scratch {
  size_t x, weight, sums;
};
Scratch scratch_of(const poetx_gated_desc* d) {
  Scratch s{0, 0, 0};
  if (d->rows == 0) return s;
  poetx_gated_desc as;
  if (relaid(d, &as)) {
    s = scratch_of(&as);
    s.x = align256((size_t)d->rows * as.d_in * esize(d->dtype));
    if (!(d->flags & POETX_GATED_W_MX4)) s.weight = align256((size_t)d->groups * 2 * d->d_hidden * as.d_in * esize(d->dtype));
    return s;
  }
  if (!(d->flags & POETX_GATED_W_MX4)) {
    s.sums = few(d, grouped::DENSE_WEIGHT) ? 0 : stream_sums_bytes(d);
    return s;
  }
  const bool streamed = few(d, grouped::VALUES_STREAMED_MX4);
  if (!streamed || !few(d, grouped::VALUES_MX4)) {
    s.weight = align256((size_t)d->groups * 2 * d->d_hidden * d->d_in * 2);
    s.sums = stream_sums_bytes(d);
  }
  const size_t v = align256(gated::values_parts_bytes(d->d_in, d->d_hidden, d->groups, d->rows, streamed, s.sums));
  s.sums = v > s.sums ? v : s.sums;
  return s;
}
size_t workspace_bytes(const poetx_gated_desc* d) {
  const Scratch s = scratch_of(d);
  return s.x + s.weight + s.sums;
}

// The tile of the streams for bf16 groups whose rows are fewer than the largest one's: what the choice for plain products goes by leaves out that such groups read the weights at the rate of the
// memory, for which smaller tiles divide the work more evenly, and that a tile ends with the activation.  Forward that keeps G and U, groups of uneven sizes, us on tiles of
// 256 x 256 / 256 x 128 / 128 x 128, by rows per group: 64 of 2 x 1376 x 2048 (7 without any), 89 rows 218 / 198 / 178, 127 221 / 220 / 200, 160 220 / 227 / 226, 191 269 / 256 / 254,
// 228 273 / 287 / 285; 8 of 2 x 8192 x 4096, 100 rows 290 / 266 / 247, 143 297 / 279 / 286, 180 385 / 334 / 338, 215 366 / 351 / 420, 256 368 / 395 / 490; 3 of 2 x 11008 x 4096, 143 rows
// 241 / 195 / 174; 24 of 2 x 704 x 1024, 143 rows 43 / 47 / 33, 200 44 / 48 / 44.
grouped::Kernel tile_for_groups(const poetx_gated_desc* d, grouped::Kernel k) {
  const i64 live = d->rows < d->groups ? d->rows : d->groups, mean = d->rows / live;
  const bool large = k == grouped::STREAM_256, wide = k == grouped::STREAM_256x128;
  if (d->groups == 1 || mean > 220 || !(large || wide)) return k;
  return mean <= 150 ? grouped::STREAM_128 : grouped::STREAM_256x128;
}

// weight, sums: the workspace's parts
void products_of(const poetx_gated_desc* d, const void* X, i64 ldx, const void* W, const int32_t* offsets, gated::Mode mode, const gated::Out& out, char* weight, char* sums, size_t sums_bytes,
                 hipStream_t st) {
  gated::Call q{X, W, ldx, offsets, d->rows, d->d_in, d->d_hidden, d->groups, mode, out};
  const bool four = d->flags & POETX_GATED_W_MX4, streamed = four && gated::values_supported(q);
  const bool handful = few(d, !four ? grouped::DENSE_WEIGHT : streamed ? grouped::VALUES_STREAMED_MX4 : grouped::VALUES_MX4);
  if (streamed && gated::values_launch(q, handful, sums, sums_bytes, sums_bytes, st)) return;
  if (handful) {
    StageTimer tm(POETX_STAGE_DENSE, st);
    return gated::few_launch(d->dtype, four, q, st);
  }
  if (four) {
    StageTimer tm(POETX_STAGE_DEQUANT, st);
    mx4_dequantize_groups_launch(W, d->groups, 2 * d->d_hidden, d->d_in, offsets, d->rows, weight, st);
    q.W = weight;
  }
  StageTimer tm(POETX_STAGE_DENSE, st);
  const grouped::Call c = product_of(d, X, ldx, q.W, offsets);
  const grouped::Plan p = grouped::plan(d->dtype, grouped::FWD, c, gated::stream_supported(d->dtype, q), d->d_hidden % 2 == 0 ? sums_bytes : 0);      // sums are stored in whole vectors
  if (p.kernel < grouped::STREAM_256) return gated::edge_launch(d->dtype, p.kernel, q, st);
  if (p.splits == 1) return gated::stream_launch(d->dtype, tile_for_groups(d, p.kernel), q, st);
  grouped::stream_sums(d->dtype, p, c, sums, st);
  gated::rows_launch(d->dtype, gated::SUMS, gated::In{sums, nullptr, 0, p.splits}, offsets, d->groups, d->rows, d->d_hidden, mode, out, st);
}

void products(const poetx_gated_desc* d, const void* X, i64 ldx, const void* W, const int32_t* offsets, gated::Mode mode, const gated::Out& out, void* ws, hipStream_t st) {
  const Scratch s = scratch_of(d);
  char *x = (char*)ws, *weight = x + s.x, *sums = weight + s.weight;
  poetx_gated_desc as;
  if (!relaid(d, &as)) return products_of(d, X, ldx, W, offsets, mode, out, weight, sums, s.sums, st);
  {
    StageTimer tm(POETX_STAGE_LAYOUT, st);
    relay_rows_launch(d->dtype, X, d->rows, d->d_in, ldx, x, as.d_in, st, offsets, d->groups);
    if (!(d->flags & POETX_GATED_W_MX4)) {
      relay_rows_launch(d->dtype, W, 2 * (i64)d->groups * d->d_hidden, d->d_in, d->d_in, weight, as.d_in, st);
      W = weight;
    }
  }
  products_of(&as, x, as.d_in, W, offsets, mode, out, weight, sums, s.sums, st);
}

}  // namespace

extern "C" {

size_t poetx_gated_workspace_bytes(const poetx_gated_desc* desc) { return check_desc(desc) == POETX_OK ? workspace_bytes(desc) : 0; }

int poetx_gated_fwd(const poetx_gated_desc* d, const void* X, int64_t ldx, const void* W, const int32_t* offsets, void* H, int64_t ldh, void* G, void* U,
                    int64_t ldgu, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_desc(d);
  if (rc != POETX_OK) return rc;
  if (!W || !offsets || !G != !U || (d->rows > 0 && (!X || !H))) return POETX_ERR_INVALID_ARG;
  const bool mx8 = G && (d->flags & POETX_GATED_HELD_MX8);
  const i64 rows = d->rows, n = d->d_hidden;
  if (ldx < d->d_in || ldh < n || (G && !mx8 && ldgu < n)) return POETX_ERR_BAD_SHAPE;
  if (!ld_fits(rows, ldx) || !ld_fits(rows, ldh) || (G && !mx8 && !ld_fits(rows, ldgu))) return POETX_ERR_UNSUPPORTED;
  const size_t es = esize(d->dtype), kept = rows == 0 ? 0 : mx8 ? mx8::bytes(rows, (int)n) : span(rows, n, ldgu, es);
  if (((d->flags & POETX_GATED_W_MX4) && ((uintptr_t)W & 15)) || (mx8 && (((uintptr_t)G | (uintptr_t)U) & 15))) return POETX_ERR_INVALID_ARG;
  const Area outs[] = {{H, span(rows, n, ldh, es)}, {G, kept}, {U, kept}};
  const Area ins[] = {{X, span(rows, d->d_in, ldx, es)}, {W, weight_bytes(d)}, {offsets, 4 * ((size_t)d->groups + 1)}};
  if (!apart(outs, 3, ins, 3) || !apart(outs, 1, outs + 1, 2) || (G && rows > 0 && (mx8 ? overlap(G, kept, U, kept) : !pair_apart(G, U, rows, n, ldgu, es))))
    return POETX_ERR_INVALID_ARG;
  if (rows == 0) return POETX_OK;
  const size_t need = workspace_bytes(d);
  if (need > 0) {
    if (!ws || ((uintptr_t)ws & 15) || ws_bytes < need) return POETX_ERR_WORKSPACE;
    const Area scratch[] = {{ws, need}};
    if (!apart(scratch, 1, ins, 3) || !apart(scratch, 1, outs, 3)) return POETX_ERR_INVALID_ARG;
  }
  const gated::Out out{H, G, U, nullptr, ldh, G && !mx8 ? ldgu : 0, 0, gated::act_of(d->activation)};      // a stride of nothing chooses no kernel
  products(d, X, ldx, W, offsets, !G ? gated::FWD : mx8 ? gated::HOLD_MX8 : gated::HOLD, out, ws, (hipStream_t)stream);
  return launch_status();
}

int poetx_gated_bwd(const poetx_gated_desc* d, const void* dH, int64_t lddh, const void* G, const void* U, int64_t ldgu, const int32_t* offsets, void* dG, void* dU,
                    int64_t lddgu, void* H, int64_t ldh, void* stream) {
  const int rc = check_desc(d);
  if (rc != POETX_OK) return rc;
  const i64 rows = d->rows, n = d->d_hidden;
  if (!offsets || (rows > 0 && (!dH || !G || !U || !dG || !dU))) return POETX_ERR_INVALID_ARG;
  const bool mx8 = d->flags & POETX_GATED_HELD_MX8;
  if (lddh < n || (!mx8 && ldgu < n) || lddgu < n || (H && ldh < n)) return POETX_ERR_BAD_SHAPE;
  if (!ld_fits(rows, lddh) || (!mx8 && !ld_fits(rows, ldgu)) || !ld_fits(rows, lddgu) || (H && !ld_fits(rows, ldh))) return POETX_ERR_UNSUPPORTED;
  if (mx8 && (((uintptr_t)G | (uintptr_t)U) & 15)) return POETX_ERR_INVALID_ARG;
  const size_t es = esize(d->dtype), kept = rows == 0 ? 0 : mx8 ? mx8::bytes(rows, (int)n) : span(rows, n, ldgu, es), grads = span(rows, n, lddgu, es);
  const Area outs[] = {{H, H ? span(rows, n, ldh, es) : 0}, {dG, grads}, {dU, grads}};
  const Area ins[] = {{dH, span(rows, n, lddh, es)}, {G, kept}, {U, kept}, {offsets, 4 * ((size_t)d->groups + 1)}};
  if (!apart(outs, 3, ins, 4) || !apart(outs, 1, outs + 1, 2) || (rows > 0 && !pair_apart(dG, dU, rows, n, lddgu, es))) return POETX_ERR_INVALID_ARG;
  if (rows == 0) return POETX_OK;
  StageTimer tm(POETX_STAGE_LAYOUT, (hipStream_t)stream);
  const gated::Out out{H, dG, dU, dH, H ? ldh : 0, lddgu, lddh, gated::act_of(d->activation)};
  gated::rows_launch(d->dtype, mx8 ? gated::MX8 : gated::SAME, gated::In{G, U, ldgu, 1}, offsets, d->groups, rows, d->d_hidden, gated::BWD, out, (hipStream_t)stream);
  return launch_status();
}

int poetx_gated_bwd_recompute(const poetx_gated_desc* d, const void* dH, int64_t lddh, const void* X, int64_t ldx, const void* W, const int32_t* offsets, void* dG,
                              void* dU, int64_t lddgu, void* H, int64_t ldh, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_desc(d);
  if (rc != POETX_OK) return rc;
  const i64 rows = d->rows, n = d->d_hidden;
  if (!W || !offsets || (rows > 0 && (!dH || !X || !dG || !dU))) return POETX_ERR_INVALID_ARG;
  if (lddh < n || ldx < d->d_in || lddgu < n || (H && ldh < n)) return POETX_ERR_BAD_SHAPE;
  if (!ld_fits(rows, lddh) || !ld_fits(rows, ldx) || !ld_fits(rows, lddgu) || (H && !ld_fits(rows, ldh))) return POETX_ERR_UNSUPPORTED;
  if ((d->flags & POETX_GATED_W_MX4) && ((uintptr_t)W & 15)) return POETX_ERR_INVALID_ARG;
  const size_t es = esize(d->dtype), grads = span(rows, n, lddgu, es);
  const Area outs[] = {{H, H ? span(rows, n, ldh, es) : 0}, {dG, grads}, {dU, grads}};
  const Area ins[] = {{dH, span(rows, n, lddh, es)}, {X, span(rows, d->d_in, ldx, es)}, {W, weight_bytes(d)}, {offsets, 4 * ((size_t)d->groups + 1)}};
  if (!apart(outs, 3, ins, 4) || !apart(outs, 1, outs + 1, 2) || (rows > 0 && !pair_apart(dG, dU, rows, n, lddgu, es))) return POETX_ERR_INVALID_ARG;
  if (rows == 0) return POETX_OK;
  const size_t need = workspace_bytes(d);
  if (need > 0) {
    if (!ws || ((uintptr_t)ws & 15) || ws_bytes < need) return POETX_ERR_WORKSPACE;
    const Area scratch[] = {{ws, need}};
    if (!apart(scratch, 1, ins, 4) || !apart(scratch, 1, outs, 3)) return POETX_ERR_INVALID_ARG;
  }
  const gated::Out out{H, dG, dU, dH, H ? ldh : 0, lddgu, lddh, gated::act_of(d->activation)};
  products(d, X, ldx, W, offsets, gated::BWD, out, ws, (hipStream_t)stream);
  return launch_status();
}

}  // extern "C"

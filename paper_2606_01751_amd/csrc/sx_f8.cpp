// Host side of the 8-bit layer body (include/sx_f8.h): argument validation and dispatch.
#include "sx_f8.h"

#include <cmath>

#include "sx_args.h"
#include "sx_f8k.h"

#ifndef SX_DEVICE_CHECKS
#define SX_DEVICE_CHECKS 0
#endif

namespace {

using sx::aligned16;
using sx::overlap;
using sx::reportf;

constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - ((int64_t)1 << 16);   // of a one-dimensional launch
constexpr int kMaxRequests = 65535;

struct Arg {
  const void* p;
  int64_t bytes;
  const char* name;
};

// Outputs `out` must not overlap each other or the inputs `in`; but out[0] may be in[in_place] itself (-1: none may).
template <int NO, int NI>
sx_status apart(const char* who, const Arg (&out)[NO], const Arg (&in)[NI], int in_place = -1) {
  for (int i = 0; i < NO; ++i) {
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes))
        return reportf(SX_EINVAL, "%s: %s and %s overlap", who, out[j].name, out[i].name);
    for (int j = 0; j < NI; ++j) {
      if (i == 0 && j == in_place && out[i].p == in[j].p) continue;
      if (overlap(out[i].p, out[i].bytes, in[j].p, in[j].bytes))
        return reportf(SX_EINVAL, "%s: %s overlaps %s", who, out[i].name, in[j].name);
    }
  }
  return SX_OK;
}

template <int N>
sx_status aligned(const char* who, const Arg (&args)[N]) {
  for (const Arg& a : args)
    if (!aligned16(a.p)) return reportf(SX_EINVAL, "%s: %s is not 16-byte aligned", who, a.name);
  return SX_OK;
}

sx_status width_ok(const char* who, const char* name, int64_t n, int64_t most) {
  if (n <= 0 || n % sx::kF8Group != 0)
    return reportf(SX_EUNSUPPORTED, "%s needs %s a positive multiple of %d (%lld)", who, name, sx::kF8Group, (long long)n);
  if (n > most) return reportf(SX_EUNSUPPORTED, "%s: %s %lld above %lld", who, name, (long long)n, (long long)most);
  return SX_OK;
}

sx_status verdict(const char* who, hipError_t e, const int v[4]) {
  if (e != hipSuccess) return reportf(SX_EHIP, "%s: device check: %s", who, hipGetErrorString(e));
  if (v[0] != 0) return reportf(SX_EDEVICE, "%s: an index array is invalid (entry %d, value %d)", who, v[2], v[3]);
  return SX_OK;
}

// The rows of a call; `total` is the number of rows of its arrays, which may be NULL where there are none.
sx_status rows_of(const char* who, const sx_plan* p, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                  bool by_token, void* stream, sx::F8Rows* r, int64_t* total) {
  if (max_rows < 0) return reportf(SX_EINVAL, "%s: max_rows must be >= 0", who);
  *r = sx::F8Rows{nullptr, nullptr, n_rows, max_rows, 1};
  *total = max_rows;
  if (!p) {
    if (rows) return reportf(SX_EINVAL, "%s: a row list needs a plan", who);
    if (SX_DEVICE_CHECKS && n_rows && max_rows > 0) {
      int v[4] = {0, 0, 0, 0};
      const hipError_t e = sx::device_check_index(n_rows, 1, 0, (int64_t)max_rows + 1, (hipStream_t)stream, v);
      return verdict(who, e, v);
    }
    return SX_OK;
  }
  if (p->desc.dtype != SX_BF16) return reportf(SX_EUNSUPPORTED, "%s: the layer body runs on bfloat16 plans", who);
  if (!n_rows || (by_token && !rows)) return reportf(SX_EINVAL, "%s: NULL row list", who);
  if (max_rows > p->max_T) return reportf(SX_ESHAPE, "%s: max_rows %d exceeds the longest request (%d)", who, max_rows, p->max_T);
  if (p->n_req > kMaxRequests) return reportf(SX_EUNSUPPORTED, "%s: more than %d requests", who, kMaxRequests);
  *r = sx::F8Rows{p->d_req, by_token ? rows : nullptr, n_rows, max_rows, p->n_req};
  *total = p->total;
  if (max_rows == 0) return SX_OK;
  return sx::check_row_list(p, rows, n_rows, max_rows, stream, who);
}

sx_status gemm_launch(const char* who, sx::F8GemmK& a, int rows, int64_t n, const char* what, void* stream) {
  const hipError_t e = sx::launch_gemm_f8(a, sx::cu_count(), (hipStream_t)stream);
  if (e == hipErrorInvalidConfiguration)
    return reportf(SX_EUNSUPPORTED, "%s: %d rows x %lld features exceed one launch", who, rows, (long long)n);
  return sx::launch_status(e, what);
}

Arg n_rows_arg(const sx_plan* p, const int32_t* n_rows) { return {n_rows, 4ll * (p ? p->n_req : 1), "n_rows"}; }
Arg rows_arg(const sx_plan* p, const int32_t* rows) { return {rows, p ? 4 * p->total : 0, "rows"}; }

}  // namespace

extern "C" {

sx_status sx_f8_scale_ld(int32_t k, int32_t* ld) {
  const sx_status st = width_ok("sx_f8_scale_ld", "k", k, INT32_MAX);
  if (st != SX_OK) return st;
  if (!ld) return reportf(SX_EINVAL, "sx_f8_scale_ld: ld is NULL");
  *ld = sx::f8_ld(k);
  return SX_OK;
}

sx_status sx_f8_pack_weight(const void* w, int64_t n, int32_t k, void* codes, void* scales, void* stream) {
  const char* who = "sx_f8_pack_weight";
  if (n == 0) return SX_OK;
  sx_status st = width_ok(who, "n", n, (int64_t)1 << 36);
  if (st != SX_OK) return st;
  if ((st = width_ok(who, "k", k, 1 << 24)) != SX_OK) return st;
  if (!w || !codes || !scales) return reportf(SX_EINVAL, "%s: NULL argument", who);
  const Arg in[] = {{w, 2 * n * k, "w"}}, out[] = {{codes, n * k, "codes"}, {scales, n / sx::kF8Group * sx::f8_ld(k), "scales"}};
  if ((st = aligned(who, in)) != SX_OK || (st = aligned(who, out)) != SX_OK) return st;
  if ((st = apart(who, out, in)) != SX_OK) return st;
  return sx::launch_status(sx::launch_f8_pack_weight((const uint16_t*)w, n, k, (uint8_t*)codes, (uint8_t*)scales, (hipStream_t)stream),
                           "sx_f8_pack_weight launch");
}

sx_status sx_add_rmsnorm_f8(const sx_plan* plan, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                            const void* x, int32_t x_by_token, const void* delta, const void* gamma, float eps,
                            int32_t h, void* x_out, void* y16, void* y8, void* y_scale, int32_t y_by_token,
                            void* stream) {
  const char* who = "sx_add_rmsnorm_f8";
  sx::F8NormK a{};
  int64_t total;
  sx_status st = rows_of(who, plan, rows, n_rows, max_rows, x_by_token || y_by_token, stream, &a.r, &total);
  if (st != SX_OK) return st;
  if ((st = width_ok(who, "h", h, 1 << 24)) != SX_OK) return st;
  if (!x && total > 0) return reportf(SX_EINVAL, "%s: x is NULL", who);
  if (!y8 != !y_scale) return reportf(SX_EINVAL, "%s: y8 and y_scale come together", who);
  if (!y8 && !y16 && !x_out && total > 0) return reportf(SX_EINVAL, "%s: no output", who);
  if (x_out && !delta) return reportf(SX_EINVAL, "%s: x_out needs delta", who);
  if (y16 && !gamma) return reportf(SX_EINVAL, "%s: y16 needs gamma", who);
  if (gamma && (!(eps > 0.0f) || !std::isfinite(eps))) return reportf(SX_EINVAL, "%s: eps must be finite and > 0", who);
  const int64_t row = 2ll * h;
  const Arg in[] = {{x, total * row, "x"}, {delta, total * row, "delta"}, {gamma, row, "gamma"}, rows_arg(plan, rows),
                    n_rows_arg(plan, n_rows)};
  const Arg out[] = {{x_out, total * row, "x_out"}, {y16, total * row, "y16"}, {y8, total * h, "y8"},
                     {y_scale, total * sx::f8_ld(h), "y_scale"}};
  const Arg wide[] = {in[0], in[1], in[2]};
  if ((st = aligned(who, wide)) != SX_OK || (st = aligned(who, out)) != SX_OK) return st;
  if ((st = apart(who, out, in, 0)) != SX_OK) return st;
  if (max_rows == 0) return SX_OK;
  a.x = (const uint16_t*)x;
  a.delta = (const uint16_t*)delta;
  a.gamma = (const uint16_t*)gamma;
  a.x_out = (uint16_t*)x_out;
  a.y16 = (uint16_t*)y16;
  a.y8 = (uint8_t*)y8;
  a.ys = (uint8_t*)y_scale;
  a.eps = eps;
  a.h = h;
  a.ld = sx::f8_ld(h);
  a.x_tok = x_by_token != 0;
  a.y_tok = y_by_token != 0;
  if ((int64_t)max_rows * 256 >= kMaxThreads) return reportf(SX_EUNSUPPORTED, "%s: %d rows exceed one launch", who, max_rows);
  return sx::launch_status(sx::launch_add_rmsnorm_f8(a, (hipStream_t)stream), "sx_add_rmsnorm_f8 launch");
}

sx_status sx_silu_mul_f8(const sx_plan* plan, const int32_t* n_rows, int32_t max_rows, const void* gate_up,
                         int32_t f, void* y8, void* y_scale, void* stream) {
  const char* who = "sx_silu_mul_f8";
  sx::F8SiluK a{};
  int64_t total;
  sx_status st = rows_of(who, plan, nullptr, n_rows, max_rows, false, stream, &a.r, &total);
  if (st != SX_OK) return st;
  if ((st = width_ok(who, "f", f, 1 << 24)) != SX_OK) return st;
  if ((!gate_up || !y8 || !y_scale) && total > 0) return reportf(SX_EINVAL, "%s: NULL argument", who);
  const Arg in[] = {{gate_up, total * 4 * f, "gate_up"}, n_rows_arg(plan, n_rows)};
  const Arg out[] = {{y8, total * f, "y8"}, {y_scale, total * sx::f8_ld(f), "y_scale"}};
  const Arg wide[] = {in[0]};
  if ((st = aligned(who, wide)) != SX_OK || (st = aligned(who, out)) != SX_OK) return st;
  if ((st = apart(who, out, in)) != SX_OK) return st;
  if (max_rows == 0) return SX_OK;
  a.gu = (const uint16_t*)gate_up;
  a.y8 = (uint8_t*)y8;
  a.ys = (uint8_t*)y_scale;
  a.f = f;
  a.ld = sx::f8_ld(f);
  if ((int64_t)max_rows * ((f + 511) / 512) * 64 >= kMaxThreads)
    return reportf(SX_EUNSUPPORTED, "%s: %d rows of %d exceed one launch", who, max_rows, f);
  return sx::launch_status(sx::launch_silu_mul_f8(a, (hipStream_t)stream), "sx_silu_mul_f8 launch");
}

sx_status sx_gemm_f8(const sx_plan* plan, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                     const void* x8, const void* x_scale, int32_t x_by_token, const void* w8, const void* w_scale,
                     int32_t k, int32_t n_parts, const int32_t* part_n, const void* residual, void* const* y_parts,
                     int32_t y_by_token, void* stream) {
  const char* who = "sx_gemm_f8";
  sx::F8GemmK a{};
  int64_t total;
  sx_status st = rows_of(who, plan, rows, n_rows, max_rows, x_by_token || y_by_token, stream, &a.r, &total);
  if (st != SX_OK) return st;
  if (((!x8 || !x_scale) && total > 0) || !w8 || !w_scale || !part_n || !y_parts) return reportf(SX_EINVAL, "%s: NULL argument", who);
  if (n_parts < 1 || n_parts > sx::kF8MaxParts) return reportf(SX_EINVAL, "%s: n_parts %d outside 1..%d", who, n_parts, sx::kF8MaxParts);
  if (residual && n_parts != 1) return reportf(SX_EINVAL, "%s: a residual needs one part", who);
  if ((st = width_ok(who, "k", k, sx::kF8MaxK)) != SX_OK) return st;
  int64_t n = 0;
  Arg out[sx::kF8MaxParts] = {{nullptr, 0, "y"}, {nullptr, 0, "y part 1"}, {nullptr, 0, "y part 2"}, {nullptr, 0, "y part 3"}};
  for (int i = 0; i < n_parts; ++i) {
    if (!y_parts[i] && total > 0) return reportf(SX_EINVAL, "%s: output part %d is NULL", who, i);
    if ((st = width_ok(who, "a part's width", part_n[i], 1 << 24)) != SX_OK) return st;
    a.y[i] = (uint16_t*)y_parts[i];
    a.pn[i] = (int)n;
    n += part_n[i];
    out[i].p = y_parts[i];
    out[i].bytes = total * 2 * part_n[i];
  }
  for (int i = n_parts; i <= sx::kF8MaxParts; ++i) a.pn[i] = (int)n;
  a.n_parts = n_parts;
  a.K = k;
  a.N = (int)n;
  a.ld = sx::f8_ld(k);
  const Arg in[] = {{x8, total * k, "x8"}, {w8, n * k, "w8"}, {residual, total * 2 * n, "residual"},
                    {x_scale, total * a.ld, "x_scale"}, {w_scale, n / sx::kF8Group * a.ld, "w_scale"}, rows_arg(plan, rows),
                    n_rows_arg(plan, n_rows)};
  const Arg wide[] = {in[0], in[1], in[2], in[3], in[4]};
  if ((st = aligned(who, wide)) != SX_OK || (st = aligned(who, out)) != SX_OK) return st;
  if ((st = apart(who, out, in, 2)) != SX_OK) return st;
  if (max_rows == 0) return SX_OK;
  a.x = (const uint8_t*)x8;
  a.xs = (const uint8_t*)x_scale;
  a.w = (const uint8_t*)w8;
  a.ws = (const uint8_t*)w_scale;
  a.res = (const uint16_t*)residual;
  a.x_tok = x_by_token != 0;
  a.y_tok = y_by_token != 0;
  return gemm_launch(who, a, max_rows, n, "sx_gemm_f8 launch", stream);
}

sx_status sx_moe_route_workspace(int32_t n_experts, int32_t top_k, int32_t n_requests, int32_t max_rows, int64_t* bytes) {
  const char* who = "sx_moe_route_workspace";
  if (n_experts < 1 || n_experts > sx::kMoeMaxExperts || top_k < 1 || top_k > n_experts || top_k > sx::kMoeMaxTop)
    return reportf(SX_EUNSUPPORTED, "%s: top_k %d of %d experts (at most %d of %d)", who, top_k, n_experts, sx::kMoeMaxTop, sx::kMoeMaxExperts);
  if (n_requests < 0 || max_rows < 0) return reportf(SX_EINVAL, "%s: negative size", who);
  if (!bytes) return reportf(SX_EINVAL, "%s: bytes is NULL", who);
  sx::MoeRouteK a{};
  sx::moe_blocks(n_requests < 1 ? 1 : n_requests, max_rows, &a);
  *bytes = ((int64_t)a.blocks * n_experts * 4 + 15) / 16 * 16;
  return SX_OK;
}

sx_status sx_moe_route(const sx_plan* plan, const int32_t* n_rows, int32_t max_rows, const void* logits,
                       int32_t logits_dtype, int32_t n_experts, int32_t top_k, int32_t renormalise, int32_t* ids,
                       float* weights, int32_t* offsets, int32_t* order, void* workspace, int64_t workspace_bytes,
                       void* stream) {
  const char* who = "sx_moe_route";
  sx::MoeRouteK a{};
  int64_t total, need;
  sx_status st = rows_of(who, plan, nullptr, n_rows, max_rows, false, stream, &a.r, &total);
  if (st != SX_OK) return st;
  if (logits_dtype != SX_F32 && logits_dtype != SX_BF16) return reportf(SX_EUNSUPPORTED, "%s: logits_dtype %d", who, logits_dtype);
  if ((st = sx_moe_route_workspace(n_experts, top_k, a.r.n_req, max_rows, &need)) != SX_OK) return st;
  if (((!logits || !ids || !weights || !order) && total > 0) || !offsets || !workspace) return reportf(SX_EINVAL, "%s: NULL argument", who);
  if (workspace_bytes < need)
    return reportf(SX_ESHAPE, "%s needs %lld bytes of workspace, got %lld", who, (long long)need, (long long)workspace_bytes);
  if (total * top_k > INT32_MAX) return reportf(SX_EUNSUPPORTED, "%s: %lld rows x %d experts exceed 2^31", who, (long long)total, top_k);
  const Arg in[] = {{logits, total * n_experts * (logits_dtype == SX_F32 ? 4 : 2), "logits"}, n_rows_arg(plan, n_rows)};
  const Arg out[] = {{ids, 4 * total * top_k, "ids"}, {weights, 4 * total * top_k, "weights"}, {order, 4 * total * top_k, "order"},
                     {offsets, 4ll * (n_experts + 1), "offsets"}, {workspace, need, "workspace"}};
  const Arg wide[] = {in[0], out[0], out[1], out[2], out[3], out[4]};
  if ((st = aligned(who, wide)) != SX_OK) return st;
  if ((st = apart(who, out, in)) != SX_OK) return st;
  a.logits = logits;
  a.ids = ids;
  a.weights = weights;
  a.offsets = offsets;
  a.order = order;
  a.counts = (int32_t*)workspace;
  a.n_experts = n_experts;
  a.top_k = top_k;
  a.renormalise = renormalise != 0;
  sx::moe_blocks(a.r.n_req < 1 ? 1 : a.r.n_req, max_rows, &a);
  return sx::launch_status(sx::launch_moe_route(a, logits_dtype == SX_F32, (hipStream_t)stream), "sx_moe_route launch");
}

sx_status sx_gemm_experts_f8(const int32_t* offsets, const int32_t* order, int32_t n_experts, int32_t n_places,
                             const void* x8, const void* x_scale, int32_t x_rows, int32_t gather, const void* w8,
                             const void* w_scale, int32_t k, int32_t n, void* y, int32_t scatter, void* stream) {
  const char* who = "sx_gemm_experts_f8";
  if (n_experts < 1 || n_experts > 65536) return reportf(SX_EUNSUPPORTED, "%s: %d experts (1 .. 65536)", who, n_experts);
  if (n_places < 0 || x_rows < 0 || gather < 0) return reportf(SX_EINVAL, "%s: negative size", who);
  sx_status st = width_ok(who, "k", k, sx::kF8MaxK);
  if (st != SX_OK) return st;
  if ((st = width_ok(who, "n", n, 1 << 24)) != SX_OK) return st;
  if (n_places == 0) return SX_OK;
  if (x_rows == 0) return reportf(SX_ESHAPE, "%s: no rows of x for %d places", who, n_places);
  if (!offsets || !x8 || !x_scale || !w8 || !w_scale || !y || ((gather || scatter) && !order))
    return reportf(SX_EINVAL, "%s: NULL argument", who);
  sx::F8GemmK a{};
  a.ld = sx::f8_ld(k);
  const int64_t rows = n_places, xr = x_rows;
  const Arg in[] = {{x8, xr * k, "x8"}, {w8, (int64_t)n_experts * n * k, "w8"}, {x_scale, xr * a.ld, "x_scale"},
                    {w_scale, (int64_t)n_experts * (n / sx::kF8Group) * a.ld, "w_scale"}, {offsets, 4ll * (n_experts + 1), "offsets"},
                    {order, 4 * rows, "order"}};
  const Arg out[] = {{y, rows * 2 * n, "y"}};
  if ((st = aligned(who, in)) != SX_OK || (st = aligned(who, out)) != SX_OK) return st;
  if ((st = apart(who, out, in)) != SX_OK) return st;
  if (SX_DEVICE_CHECKS) {
    int v[4] = {0, 0, 0, 0};
    // (without gather a place is a row of x too)
    hipError_t e = sx::device_check_offsets(offsets, n_experts, gather || x_rows > n_places ? n_places : x_rows, (hipStream_t)stream, v);
    if ((st = verdict(who, e, v)) != SX_OK) return st;
    if (order) {   // the places that are in use
      e = sx::device_check_order(offsets, n_experts, order, n_places, gather, gather ? x_rows : n_places, (hipStream_t)stream, v);
      if ((st = verdict(who, e, v)) != SX_OK) return st;
    }
  }
  a.r = sx::F8Rows{nullptr, nullptr, nullptr, n_places, 1};
  a.offsets = offsets;
  a.order = order;
  a.x = (const uint8_t*)x8;
  a.xs = (const uint8_t*)x_scale;
  a.w = (const uint8_t*)w8;
  a.ws = (const uint8_t*)w_scale;
  a.y[0] = (uint16_t*)y;
  for (int i = 1; i <= sx::kF8MaxParts; ++i) a.pn[i] = n;
  a.n_parts = 1;
  a.K = k;
  a.N = n;
  a.n_experts = n_experts;
  a.n_places = n_places;
  a.x_rows = x_rows;
  a.gather = gather;
  a.scatter = scatter != 0;
  return gemm_launch(who, a, n_places, n, "sx_gemm_experts_f8 launch", stream);
}

sx_status sx_moe_combine(const sx_plan* plan, const int32_t* rows, const int32_t* n_rows, int32_t max_rows,
                         const void* y, const float* weights, int32_t top_k, int32_t h, const void* residual, void* out,
                         int32_t out_by_token, void* stream) {
  const char* who = "sx_moe_combine";
  sx::MoeCombineK a{};
  int64_t total;
  sx_status st = rows_of(who, plan, rows, n_rows, max_rows, out_by_token != 0, stream, &a.r, &total);
  if (st != SX_OK) return st;
  if (top_k < 1 || top_k > sx::kMoeMaxTop) return reportf(SX_EUNSUPPORTED, "%s: top_k %d outside 1..%d", who, top_k, sx::kMoeMaxTop);
  if (h <= 0 || h % 8 != 0 || h > (1 << 24)) return reportf(SX_EUNSUPPORTED, "%s needs h a positive multiple of 8 up to 2^24 (%d)", who, h);
  if ((!y || !weights || !out) && total > 0) return reportf(SX_EINVAL, "%s: NULL argument", who);
  const Arg in[] = {{y, total * top_k * 2 * h, "y"}, {residual, total * 2 * h, "residual"}, {weights, 4 * total * top_k, "weights"},
                    rows_arg(plan, rows), n_rows_arg(plan, n_rows)};
  const Arg to[] = {{out, total * 2 * h, "out"}};
  const Arg wide[] = {in[0], in[1], in[2]};
  if ((st = aligned(who, wide)) != SX_OK || (st = aligned(who, to)) != SX_OK) return st;
  if ((st = apart(who, to, in, 1)) != SX_OK) return st;
  if (max_rows == 0) return SX_OK;
  a.y = (const uint16_t*)y;
  a.weights = weights;
  a.res = (const uint16_t*)residual;
  a.out = (uint16_t*)out;
  a.top_k = top_k;
  a.h = h;
  a.out_tok = out_by_token != 0;
  if ((int64_t)max_rows * (h / 8) >= kMaxThreads) return reportf(SX_EUNSUPPORTED, "%s: %d rows of %d exceed one launch", who, max_rows, h);
  return sx::launch_status(sx::launch_moe_combine(a, (hipStream_t)stream), "sx_moe_combine launch");
}

}  // extern "C"

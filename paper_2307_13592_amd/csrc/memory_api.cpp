// C ABI of the layer norm, the operators along time that a trajectory's memory is
// made of, and gradient clipping (include/mgn.h): argument checks and launches.
// Only a list of tensors holds state, in host memory.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "api_check.h"

using namespace mgn;

// The tensors' tables as the kernels take them.
struct mgn_grads {
  std::vector<GradTable> tables;
};

extern "C" {

mgn_status mgn_layer_norm(const void* x, const void* res, int32_t type, int64_t rows, int32_t cols, const float* weight,
                          const float* bias, float eps, void* total, void* y, int32_t y_type, float* y_scale,
                          mgn_stream stream) {
  const char* fn = "mgn_layer_norm";
  if (cols < 1 || cols > MGN_ROW_MAX_COLS || !size_ok(rows, cols)) return bad(fn, "bad sizes");
  if (!float_type(type) || !(float_type(y_type) || y_type == MGN_E4M3)) return bad(fn, "unknown storage type");
  if (!std::isnormal(eps) || eps < 0.f) return bad(fn, "eps must be positive (a normal number)");
  if ((y_type == MGN_E4M3) != (y_scale != nullptr) && rows > 0) return bad(fn, "y_scale goes with 8-bit rows");
  if (rows == 0) return MGN_OK;
  if (!x || !y) return bad(fn, "NULL argument");
  const int64_t ts = type_size(type), n = rows * cols;
  if (!aligned(x, ts) || !aligned(res, ts) || !aligned(total, ts) || !aligned(y, type_size(y_type)) ||
      !aligned(weight, 4) || !aligned(bias, 4) || !aligned(y_scale, 4))
    return bad(fn, "misaligned pointer");
  // results may stand on an input, element for element; that input is then a written array
  const void* own_total = apart(total, {x, res});
  const void* own_y = y_type == type ? apart(y, {x, res}) : y;
  const auto written = [&](const void* p) { return p && (p == total || (p == y && y_type == type)); };
  if ((total && total == y) ||
      clash({Span{x, n * ts, written(x)}, Span{apart(res, {x}), n * ts, written(res)}, rd(weight, 4 * (int64_t)cols),
             rd(bias, 4 * (int64_t)cols), to(own_total, n * ts), to(own_y, n * type_size(y_type)),
             to(y_scale, 4 * rows * blocks(cols))}))
    return bad(fn, "overlapping arrays");
  LayerArgs a{};
  a.x = x;
  a.res = res;
  a.w = weight;
  a.b = bias;
  a.total = total;
  a.y = y;
  a.y_scale = y_scale;
  a.rows = rows;
  a.cols = cols;
  a.eps = eps;
  return launched(launch_layer_norm(a, type, y_type, (hipStream_t)stream), fn);
}

mgn_status mgn_layer_norm_grad(const void* total, int32_t type, const float* weight, float eps, const void* dy,
                               const void* d_total, int64_t rows, int32_t cols, void* dx, float* dweight, float* dbias,
                               int32_t accumulate, float* work, mgn_stream stream) {
  const char* fn = "mgn_layer_norm_grad";
  if (cols < 1 || cols > MGN_ROW_MAX_COLS || !size_ok(rows, cols)) return bad(fn, "bad sizes");
  if (!float_type(type)) return bad(fn, "unknown storage type");
  if (!std::isnormal(eps) || eps < 0.f) return bad(fn, "eps must be positive (a normal number)");
  if (rows > 0 && (!total || !dy || !dx)) return bad(fn, "NULL argument");
  const bool sums = dweight || dbias;
  if (sums && !work) return bad(fn, "dweight and dbias need work");
  const int64_t ts = type_size(type), n = rows * cols, w = 4 * (int64_t)cols;
  if (!aligned(total, ts) || !aligned(dy, ts) || !aligned(d_total, ts) || !aligned(dx, ts) || !aligned(weight, 4) ||
      !aligned(dweight, 4) || !aligned(dbias, 4) || !aligned(work, 4))
    return bad(fn, "misaligned pointer");
  if (clash({Span{total, n * ts, total == dx}, Span{apart(dy, {total}), n * ts, dy == dx},
             Span{apart(d_total, {total, dy}), n * ts, d_total == dx}, rd(weight, w),
             to(apart(dx, {total, dy, d_total}), n * ts), to(dweight, w), to(dbias, w),
             to(work, sums ? MGN_LAYER_WORK_PER_COL * w : 0)}))
    return bad(fn, "overlapping arrays");
  if (rows == 0 && !sums) return MGN_OK;
  LayerArgs a{};
  a.x = total;
  a.res = d_total;
  a.dy = dy;
  a.w = weight;
  a.total = dx;
  a.part = sums ? work : nullptr;
  a.rows = rows;
  a.cols = cols;
  a.eps = eps;
  return launched(launch_layer_norm_grad(a, type, dweight, dbias, accumulate != 0, (hipStream_t)stream), fn);
}

}  // extern "C"

namespace {

// Sizes [steps][rows][cols], with `per` numbers for a column of a row.
bool steps_ok(int64_t steps, int64_t rows, int32_t cols, int64_t per) {
  return cols >= 1 && cols <= MGN_ROW_MAX_COLS && size_ok(rows, cols * per) && steps >= 0 &&
         (rows == 0 || size_ok(steps, rows * cols * per));
}

// Checks shared by the convolution and its backward, the argument record filled.
mgn_status conv_args(const char* fn, ConvArgs& a, const void* x, int32_t type, const float* weight, int32_t width,
                     const float* bias, const uint8_t* starts, const void* past, int64_t steps, int64_t rows,
                     int32_t cols, int32_t silu) {
  if (width < 1 || width > MGN_CONV_MAX_WIDTH) return bad(fn, "width must be 1 .. MGN_CONV_MAX_WIDTH");
  if (!steps_ok(steps, rows, cols, MGN_CONV_MAX_WIDTH)) return bad(fn, "bad sizes");
  if (!float_type(type)) return bad(fn, "unknown storage type");
  if (steps > 0 && rows > 0 && (!x || !weight)) return bad(fn, "NULL argument");
  const int64_t ts = type_size(type);
  if (!aligned(x, ts) || !aligned(past, ts) || !aligned(weight, 4) || !aligned(bias, 4))
    return bad(fn, "misaligned pointer");
  a.x = x;
  a.past = width > 1 ? past : nullptr;
  a.w = weight;
  a.b = bias;
  a.starts = starts;
  a.steps = steps;
  a.rows = rows;
  a.cols = cols;
  a.silu = silu != 0;
  return MGN_OK;
}

}  // namespace

extern "C" {

mgn_status mgn_causal_conv(const void* x, int32_t type, const float* weight, int32_t width, const float* bias,
                           const uint8_t* starts, const void* past, int64_t steps, int64_t rows, int32_t cols,
                           int32_t silu, void* y, void* past_out, mgn_stream stream) {
  const char* fn = "mgn_causal_conv";
  ConvArgs a{};
  const mgn_status s = conv_args(fn, a, x, type, weight, width, bias, starts, past, steps, rows, cols, silu);
  if (s) return s;
  if (width == 1) past_out = nullptr;
  if (rows == 0 || (steps == 0 && !past_out)) return MGN_OK;
  if (steps > 0 && !y) return bad(fn, "NULL argument");
  const int64_t ts = type_size(type), m = rows * cols, n = steps * m, before = (width - 1) * m;
  if (!aligned(y, ts) || !aligned(past_out, ts)) return bad(fn, "misaligned pointer");
  if (clash({rd(x, n * ts), rd(weight, 4 * (int64_t)cols * width), rd(bias, 4 * (int64_t)cols), rd(starts, steps),
             rd(apart(a.past, {past_out}), before * ts), to(y, n * ts), to(past_out, before * ts)}))
    return bad(fn, "overlapping arrays");
  a.y = y;
  a.past_out = past_out;
  return launched(launch_conv(a, type, width, (hipStream_t)stream), fn);
}

mgn_status mgn_causal_conv_grad(const void* x, int32_t type, const float* weight, int32_t width, const float* bias,
                                const uint8_t* starts, const void* past, const void* dy, const float* d_past_out,
                                int64_t steps, int64_t rows, int32_t cols, int32_t silu, void* dx, float* dweight,
                                float* dbias, int32_t accumulate, float* d_past, float* work, mgn_stream stream) {
  const char* fn = "mgn_causal_conv_grad";
  ConvArgs a{};
  const mgn_status s = conv_args(fn, a, x, type, weight, width, bias, starts, past, steps, rows, cols, silu);
  if (s) return s;
  if (width == 1) d_past = nullptr, d_past_out = nullptr;
  const bool sums = dweight || dbias;
  if (steps > 0 && rows > 0 && (!dy || !dx)) return bad(fn, "NULL argument");
  if (sums && !work) return bad(fn, "dweight and dbias need work");
  const int64_t ts = type_size(type), m = rows * cols, n = steps * m, before = 4 * (width - 1) * m;
  if (!aligned(dy, ts) || !aligned(dx, ts) || !aligned(d_past_out, 4) || !aligned(d_past, 4) || !aligned(dweight, 4) ||
      !aligned(dbias, 4) || !aligned(work, 4))
    return bad(fn, "misaligned pointer");
  const int64_t wb = 4 * (int64_t)cols * width, bb = 4 * (int64_t)cols;
  if (clash({rd(x, n * ts), rd(weight, wb), rd(bias, bb), rd(starts, steps), rd(a.past, (width - 1) * m * ts),
             rd(dy, n * ts), rd(d_past_out, before), to(dx, n * ts), to(dweight, wb), to(dbias, bb), to(d_past, before),
             to(work, sums ? 4 * conv_work_floats(cols, width) : 0)}))
    return bad(fn, "overlapping arrays");
  a.dy = dy;
  a.d_past_out = d_past_out;
  a.d_past = d_past;
  a.y = dx;
  a.part = sums ? work : nullptr;
  return launched(launch_conv_grad(a, type, width, dweight, dbias, accumulate != 0, (hipStream_t)stream), fn);
}

}  // extern "C"

namespace {

mgn_status ssm_sizes(const char* fn, int64_t steps, int64_t rows, int32_t cols, int32_t n) {
  if (n < 1 || n > MGN_STATES_MAX) return bad(fn, "n must be 1 .. MGN_STATES_MAX");
  if (!steps_ok(steps, rows, cols, n)) return bad(fn, "bad sizes");
  return MGN_OK;
}

int64_t marks_bytes(const mgn_ssm& s) {
  return 4 * ((s.steps + MGN_MARK_STEPS - 1) / MGN_MARK_STEPS) * s.rows * s.cols * s.n;
}

// Checks shared by the scan and its backward, the argument record filled.
mgn_status ssm_args(const char* fn, SsmArgs& a, const mgn_ssm* s, const void* work, size_t work_bytes, bool grad) {
  if (!s) return bad(fn, "NULL argument");
  if (const mgn_status st = ssm_sizes(fn, s->steps, s->rows, s->cols, s->n)) return st;
  if (!float_type(s->type)) return bad(fn, "unknown storage type");
  const bool any = s->steps > 0 && s->rows > 0;
  if (any && (!s->x || !s->dt || !s->B || !s->C || !s->A)) return bad(fn, "NULL argument");
  const int64_t ts = type_size(s->type);
  for (const void* p : {s->x, s->dt, s->B, s->C, s->z})
    if (!aligned(p, ts)) return bad(fn, "misaligned pointer");
  for (const void* p : {s->A, s->D, s->dt_bias})
    if (!aligned(p, 4)) return bad(fn, "misaligned pointer");
  if (!aligned(work, 16)) return bad(fn, "misaligned pointer");
  const size_t need = (grad ? ssm_grad_work_bytes : ssm_work_bytes)(s->steps, s->rows, s->cols, s->n);
  if (work_bytes < need || (need && !work))
    return set_error(nullptr, MGN_E_NOMEM,
                     std::string(fn) + ": work too small (need " + std::to_string(need) + " bytes)");
  a.x = s->x;
  a.dt = s->dt;
  a.B = s->B;
  a.C = s->C;
  a.z = s->z;
  a.A = s->A;
  a.D = s->D;
  a.bias = s->dt_bias;
  a.starts = s->starts;
  a.steps = s->steps;
  a.rows = s->rows;
  a.cols = s->cols;
  a.n = s->n;
  a.softplus = s->softplus != 0;
  return MGN_OK;
}

mgn_status work_size(const char* fn, int64_t steps, int64_t rows, int32_t cols, int32_t n, size_t* bytes, bool grad) {
  if (!bytes) return bad(fn, "bytes is NULL");
  if (const mgn_status st = ssm_sizes(fn, steps, rows, cols, n)) return st;
  *bytes = (grad ? ssm_grad_work_bytes : ssm_work_bytes)(steps, rows, cols, n);
  return MGN_OK;
}

}  // namespace

extern "C" {

mgn_status mgn_selective_scan_work(int64_t steps, int64_t rows, int32_t cols, int32_t n, size_t* bytes) {
  return work_size("mgn_selective_scan_work", steps, rows, cols, n, bytes, false);
}
mgn_status mgn_selective_scan_grad_work(int64_t steps, int64_t rows, int32_t cols, int32_t n, size_t* bytes) {
  return work_size("mgn_selective_scan_grad_work", steps, rows, cols, n, bytes, true);
}

mgn_status mgn_selective_scan(const mgn_ssm* s, const float* h0, void* y, float* h_last, float* marks, void* work,
                              size_t work_bytes, mgn_stream stream) {
  const char* fn = "mgn_selective_scan";
  SsmArgs a{};
  if (const mgn_status st = ssm_args(fn, a, s, work, work_bytes, false)) return st;
  if (s->rows == 0 || (s->steps == 0 && !h_last)) return MGN_OK;
  if (s->steps > 0 && !y) return bad(fn, "NULL argument");
  const int64_t ts = type_size(s->type), m = s->rows * s->cols, n = s->steps * m * ts, pair = s->steps * s->rows * s->n * ts;
  const int64_t an = 4 * (int64_t)s->cols * s->n, cn = 4 * (int64_t)s->cols, hn = 4 * m * s->n;
  if (!aligned(y, ts) || !aligned(h0, 4) || !aligned(h_last, 4) || !aligned(marks, 4))
    return bad(fn, "misaligned pointer");
  if (clash({rd(s->x, n), rd(s->dt, n), rd(s->z, n), rd(s->B, pair), rd(s->C, pair), rd(s->A, an), rd(s->D, cn),
             rd(s->dt_bias, cn), rd(s->starts, s->steps), rd(apart(h0, {h_last}), hn), to(y, n), to(h_last, hn),
             to(marks, marks_bytes(*s)), to(work, (int64_t)ssm_work_bytes(s->steps, s->rows, s->cols, s->n))}))
    return bad(fn, "overlapping arrays");
  a.h0 = h0;
  a.y = y;
  a.h_last = h_last;
  a.marks = marks;
  return launched(launch_ssm(a, s->type, work, (hipStream_t)stream), fn);
}

mgn_status mgn_selective_scan_grad(const mgn_ssm* s, const float* marks, const void* dy, const float* dh_last,
                                   const mgn_ssm_grads* grads, float* dh0, void* work, size_t work_bytes,
                                   mgn_stream stream) {
  const char* fn = "mgn_selective_scan_grad";
  SsmArgs a{};
  if (const mgn_status st = ssm_args(fn, a, s, work, work_bytes, true)) return st;
  if (!grads) return bad(fn, "NULL argument");
  const mgn_ssm_grads& g = *grads;
  const bool any = s->steps > 0 && s->rows > 0;
  if (any && (!marks || !dy || !g.dx || !g.ddt || !g.dB || !g.dC)) return bad(fn, "NULL argument");
  if (any && (s->z != nullptr) != (g.dz != nullptr)) return bad(fn, "dz goes with z");
  const int64_t ts = type_size(s->type), m = s->rows * s->cols, n = s->steps * m * ts, pair = s->steps * s->rows * s->n * ts;
  const int64_t an = 4 * (int64_t)s->cols * s->n, cn = 4 * (int64_t)s->cols, hn = 4 * m * s->n;
  for (const void* p : {dy, (const void*)g.dx, (const void*)g.ddt, (const void*)g.dB, (const void*)g.dC, (const void*)g.dz})
    if (!aligned(p, ts)) return bad(fn, "misaligned pointer");
  for (const void* p : {marks, dh_last, (const float*)dh0, (const float*)g.dA, (const float*)g.dD, (const float*)g.d_bias})
    if (!aligned(p, 4)) return bad(fn, "misaligned pointer");
  if (clash({rd(s->x, n), rd(s->dt, n), rd(s->z, n), rd(s->B, pair), rd(s->C, pair), rd(s->A, an), rd(s->D, cn),
             rd(s->dt_bias, cn), rd(s->starts, s->steps), rd(marks, marks_bytes(*s)), rd(dy, n),
             rd(apart(dh_last, {dh0}), hn), to(g.dx, n), to(g.ddt, n), to(g.dz, n), to(g.dB, pair), to(g.dC, pair),
             to(g.dA, an), to(g.dD, cn), to(g.d_bias, cn), to(dh0, hn),
             to(work, (int64_t)ssm_grad_work_bytes(s->steps, s->rows, s->cols, s->n))}))
    return bad(fn, "overlapping arrays");
  a.marks = const_cast<float*>(marks);
  a.dy = dy;
  a.dh_last = dh_last;
  a.dx = g.dx;
  a.ddt = g.ddt;
  a.dB = g.dB;
  a.dC = g.dC;
  a.dz = g.dz;
  a.dh0 = dh0;
  return launched(launch_ssm_grad(a, s->type, g.dA, g.dD, g.d_bias, g.accumulate != 0, work, (hipStream_t)stream), fn);
}

}  // extern "C"

namespace {

// Whether a written tensor overlaps another one: spans in order of their
// addresses, each against the furthest end before it.
bool overlaps(const mgn_grad* t, int64_t count) {
  std::vector<Span> all;
  all.reserve(2 * count);
  for (int64_t k = 0; k < count; ++k) {
    const int64_t b = t[k].n * type_size(t[k].type);
    if (b == 0) continue;
    const bool in_place = !t[k].out || t[k].out == t[k].grad;
    all.push_back(Span{t[k].grad, b, in_place});
    if (!in_place) all.push_back(to(t[k].out, b));
  }
  std::sort(all.begin(), all.end(), [](const Span& a, const Span& b) { return (uintptr_t)a.p < (uintptr_t)b.p; });
  uintptr_t any = 0, written = 0;  // ends
  for (const Span& s : all) {
    const uintptr_t p = (uintptr_t)s.p, e = p + (uintptr_t)s.bytes;
    if (p < written || (s.written && p < any)) return true;
    any = std::max(any, e);
    if (s.written) written = std::max(written, e);
  }
  return false;
}

mgn_status grads_checked(const char* fn, const mgn_grads* list, const float* norm, const void* work, size_t work_bytes) {
  if (!list || !norm) return bad(fn, "NULL argument");
  if (!aligned(norm, 4) || !aligned(work, 16)) return bad(fn, "misaligned pointer");
  const size_t need = 8 * (size_t)grad_work_doubles((int64_t)list->tables.size());
  if (work_bytes < need || !work)
    return set_error(nullptr, MGN_E_NOMEM,
                     std::string(fn) + ": work too small (need " + std::to_string(need) + " bytes)");
  if (clash({to(norm, 4), to(work, (int64_t)need)})) return bad(fn, "overlapping arrays");
  for (const GradTable& t : list->tables)
    for (int k = 0; k < t.count; ++k) {
      const int64_t b = t.n(k) * (t.is_bf16(k) ? 2 : 4);
      for (const Span& s : {to(norm, 4), to(work, (int64_t)need)})
        if (touch(s, rd(t.g(k), b)) || touch(s, rd(t.out(k), b))) return bad(fn, "overlapping arrays");
    }
  return MGN_OK;
}

}  // namespace

extern "C" {

mgn_status mgn_grads_create(const mgn_grad* tensors, int64_t count, mgn_grads** out) {
  const char* fn = "mgn_grads_create";
  if (!out || count < 0 || (count > 0 && !tensors)) return bad(fn, "NULL argument or bad count");
  *out = nullptr;
  for (int64_t k = 0; k < count; ++k) {
    const mgn_grad& t = tensors[k];
    if (!float_type(t.type)) return bad(fn, "unknown storage type");
    if (!size_ok(t.n, 1) || t.n / GRAD_TILE >= 1 << 24) return bad(fn, "bad sizes");
    if (t.n > 0 && !t.grad) return bad(fn, "NULL argument");
    if (((uint64_t)t.grad | (uint64_t)t.out) >> 48) return bad(fn, "not a device address");
    if (!aligned(t.grad, type_size(t.type)) || !aligned(t.out, type_size(t.type))) return bad(fn, "misaligned pointer");
  }
  mgn_grads* list = nullptr;
  try {
    if (overlaps(tensors, count)) return bad(fn, "overlapping arrays");
    list = new mgn_grads;
    for (int64_t k = 0; k < count; ++k) {
      const mgn_grad& t = tensors[k];
      if (t.n == 0) continue;
      if (list->tables.empty() || list->tables.back().count == GRAD_TABLE) list->tables.emplace_back(GradTable{});
      GradTable& to = list->tables.back();
      const int i = to.count++;
      const uint64_t g = (uint64_t)t.grad, out = t.out ? (uint64_t)t.out : g;
      to.g_lo[i] = (uint32_t)g, to.g_hi[i] = (uint16_t)(g >> 32);
      to.out_lo[i] = (uint32_t)out, to.out_hi[i] = (uint16_t)(out >> 32);
      to.rem[i] = (uint16_t)((t.n - 1) % GRAD_TILE);
      to.first[i + 1] = to.first[i] + (uint32_t)((t.n + GRAD_TILE - 1) / GRAD_TILE);
      if (t.type == MGN_BF16) to.bf16[i / 32] |= 1u << (i % 32);
    }
  } catch (const std::bad_alloc&) {
    delete list;
    return set_error(nullptr, MGN_E_NOMEM, std::string(fn) + ": out of host memory");
  }
  *out = list;
  return MGN_OK;
}

void mgn_grads_destroy(mgn_grads* list) { delete list; }

mgn_status mgn_grads_work(const mgn_grads* list, size_t* bytes) {
  if (!list || !bytes) return bad("mgn_grads_work", "NULL argument");
  *bytes = 8 * (size_t)grad_work_doubles((int64_t)list->tables.size());
  return MGN_OK;
}

mgn_status mgn_grad_norm(const mgn_grads* list, float* norm, void* work, size_t work_bytes, mgn_stream stream) {
  const char* fn = "mgn_grad_norm";
  if (const mgn_status s = grads_checked(fn, list, norm, work, work_bytes)) return s;
  return launched(launch_grads(list->tables.data(), (int64_t)list->tables.size(), -1.f, false, norm, (double*)work,
                               (hipStream_t)stream), fn);
}

mgn_status mgn_grad_clip(const mgn_grads* list, float max_norm, int32_t given, float* norm, void* work,
                         size_t work_bytes, mgn_stream stream) {
  const char* fn = "mgn_grad_clip";
  if (!(max_norm > 0.f) || !std::isfinite(max_norm)) return bad(fn, "max_norm must be positive and finite");
  if (const mgn_status s = grads_checked(fn, list, norm, work, work_bytes)) return s;
  return launched(launch_grads(list->tables.data(), (int64_t)list->tables.size(), max_norm, given != 0, norm,
                               (double*)work, (hipStream_t)stream), fn);
}

}  // extern "C"

// C ABI of the row and time operators (include/mgn.h): argument checks and
// launches.  Nothing here holds state.
#include <cmath>

#include "api_check.h"

using namespace mgn;

namespace {

mgn_status check_rows8(const char* fn, const void* p, int32_t type, int64_t n_rows, int32_t cols, const int32_t* rows,
                       const int32_t* slots, int64_t n, const uint8_t* q, const float* scale, int64_t n_slots) {
  if (cols < 1 || cols > MGN_ROW_MAX_COLS) return bad(fn, "cols must be 1 .. MGN_ROW_MAX_COLS");
  if (!float_type(type)) return bad(fn, "the rows' type must be MGN_FP32 or MGN_BF16");
  if (!size_ok(n, cols) || !size_ok(n_rows, cols) || !size_ok(n_slots, cols)) return bad(fn, "bad sizes");
  if ((!rows && n > n_rows) || (!slots && n > n_slots)) return bad(fn, "more rows than the arrays hold");
  if (n == 0) return MGN_OK;
  if (!p || !q || !scale) return bad(fn, "NULL argument");
  if (!aligned(p, type_size(type)) || !aligned(scale, 4) || !aligned(rows, 4) || !aligned(slots, 4))
    return bad(fn, "misaligned pointer");
  return MGN_OK;
}

}  // namespace

extern "C" {

mgn_status mgn_rows_store8(const void* src, int32_t src_type, int64_t n_src, int32_t cols, const int32_t* src_rows,
                           const int32_t* slots, int64_t n, uint8_t* q, float* scale, int64_t n_slots,
                           mgn_stream stream) {
  const char* fn = "mgn_rows_store8";
  mgn_status s = check_rows8(fn, src, src_type, n_src, cols, src_rows, slots, n, q, scale, n_slots);
  if (s || n == 0) return s;
  if (clash({rd(src, n_src * cols * type_size(src_type)), rd(src_rows, 4 * n), rd(slots, 4 * n), to(q, n_slots * cols),
             to(scale, 4 * n_slots * blocks(cols))}))
    return bad(fn, "overlapping arrays");
  Rows8Args a{};
  a.x = src;
  a.rows = src_rows;
  a.slots = slots;
  a.q = q;
  a.scale = scale;
  a.n = n;
  a.n_rows = n_src;
  a.n_slots = n_slots;
  a.cols = cols;
  return launched(launch_rows_store8(a, src_type, (hipStream_t)stream), fn);
}

mgn_status mgn_rows_load8(const uint8_t* q, const float* scale, int64_t n_slots, int32_t cols, const int32_t* slots,
                          const int32_t* dst_rows, int64_t n, void* dst, int32_t dst_type, int64_t n_dst, int32_t add,
                          mgn_stream stream) {
  const char* fn = "mgn_rows_load8";
  mgn_status s = check_rows8(fn, dst, dst_type, n_dst, cols, dst_rows, slots, n, q, scale, n_slots);
  if (s) return s;
  if (add && dst_type != MGN_FP32) return bad(fn, "sums are kept in MGN_FP32 only");
  if (n == 0) return MGN_OK;
  if (clash({rd(q, n_slots * cols), rd(scale, 4 * n_slots * blocks(cols)), rd(dst_rows, 4 * n), rd(slots, 4 * n),
             to(dst, n_dst * cols * type_size(dst_type))}))
    return bad(fn, "overlapping arrays");
  Rows8Args a{};
  a.out = dst;
  a.rows = dst_rows;
  a.slots = slots;
  a.q = const_cast<uint8_t*>(q);
  a.scale = const_cast<float*>(scale);
  a.n = n;
  a.n_rows = n_dst;
  a.n_slots = n_slots;
  a.cols = cols;
  a.add = add != 0;
  return launched(launch_rows_load8(a, dst_type, (hipStream_t)stream), fn);
}

mgn_status mgn_rms_norm(const void* x, const void* res, int32_t type, int64_t rows, int32_t cols, const float* weight,
                        float eps, void* total, void* y, int32_t y_type, float* y_scale, mgn_stream stream) {
  const char* fn = "mgn_rms_norm";
  if (cols < 1 || cols > MGN_ROW_MAX_COLS || !size_ok(rows, cols)) return bad(fn, "bad sizes");
  if (!float_type(type) || !(float_type(y_type) || y_type == MGN_E4M3)) return bad(fn, "unknown storage type");
  if (!std::isnormal(eps) || eps < 0.f) return bad(fn, "eps must be positive (a normal number)");
  if ((y_type == MGN_E4M3) != (y_scale != nullptr) && rows > 0) return bad(fn, "y_scale goes with 8-bit rows");
  if (rows == 0) return MGN_OK;
  if (!x || !y) return bad(fn, "NULL argument");
  const int64_t ts = type_size(type), n = rows * cols;
  if (!aligned(x, ts) || !aligned(res, ts) || !aligned(total, ts) || !aligned(y, type_size(y_type)) ||
      !aligned(weight, 4) || !aligned(y_scale, 4))
    return bad(fn, "misaligned pointer");
  // results may stand on an input, element for element; that input is then a written array
  const void* own_total = apart(total, {x, res});
  const void* own_y = y_type == type ? apart(y, {x, res}) : y;
  const auto written = [&](const void* p) { return p && (p == total || (p == y && y_type == type)); };
  if ((total && total == y) ||
      clash({Span{x, n * ts, written(x)}, Span{apart(res, {x}), n * ts, written(res)}, rd(weight, 4 * (int64_t)cols),
             to(own_total, n * ts), to(own_y, n * type_size(y_type)), to(y_scale, 4 * rows * blocks(cols))}))
    return bad(fn, "overlapping arrays");
  RmsArgs a{};
  a.x = x;
  a.res = res;
  a.w = weight;
  a.total = total;
  a.y = y;
  a.y_scale = y_scale;
  a.rows = rows;
  a.cols = cols;
  a.eps = eps;
  return launched(launch_rms_norm(a, type, y_type, (hipStream_t)stream), fn);
}

mgn_status mgn_rms_norm_grad(const void* total, int32_t type, const float* weight, float eps, const void* dy,
                             const void* d_total, int64_t rows, int32_t cols, void* dx, float* dweight,
                             int32_t accumulate, float* work, mgn_stream stream) {
  const char* fn = "mgn_rms_norm_grad";
  if (cols < 1 || cols > MGN_ROW_MAX_COLS || !size_ok(rows, cols)) return bad(fn, "bad sizes");
  if (!float_type(type)) return bad(fn, "unknown storage type");
  if (!std::isnormal(eps) || eps < 0.f) return bad(fn, "eps must be positive (a normal number)");
  if (rows > 0 && (!total || !dy || !dx)) return bad(fn, "NULL argument");
  if (dweight && !work) return bad(fn, "dweight needs work");
  const int64_t ts = type_size(type), n = rows * cols;
  if (!aligned(total, ts) || !aligned(dy, ts) || !aligned(d_total, ts) || !aligned(dx, ts) || !aligned(weight, 4) ||
      !aligned(dweight, 4) || !aligned(work, 4))
    return bad(fn, "misaligned pointer");
  const int64_t wb = dweight ? (int64_t)MGN_RMS_WORK_PER_COL * cols * 4 : 0;
  if (clash({Span{total, n * ts, total == dx}, Span{apart(dy, {total}), n * ts, dy == dx},
             Span{apart(d_total, {total, dy}), n * ts, d_total == dx}, rd(weight, 4 * (int64_t)cols),
             to(apart(dx, {total, dy, d_total}), n * ts), to(dweight, 4 * (int64_t)cols), to(work, wb)}))
    return bad(fn, "overlapping arrays");
  if (rows == 0 && !dweight) return MGN_OK;
  RmsArgs a{};
  a.x = total;
  a.res = d_total;
  a.dy = dy;
  a.w = weight;
  a.total = dx;
  a.part = dweight ? work : nullptr;
  a.rows = rows;
  a.cols = cols;
  a.eps = eps;
  return launched(launch_rms_norm_grad(a, type, dweight, accumulate != 0, (hipStream_t)stream), fn);
}

mgn_status mgn_gated_scan_work(int64_t steps, int64_t rows, int32_t cols, size_t* bytes) {
  const char* fn = "mgn_gated_scan_work";
  if (!bytes) return bad(fn, "bytes is NULL");
  if (cols < 1 || cols > MGN_ROW_MAX_COLS || !size_ok(rows, cols) || steps < 0 ||
      (rows > 0 && !size_ok(steps, rows * cols)))
    return bad(fn, "bad sizes");
  *bytes = scan_work_bytes(steps, rows, cols);
  return MGN_OK;
}

}  // extern "C"

namespace {

// Checks shared by the recurrence and its backward, the argument record filled.
mgn_status scan_args(const char* fn, ScanArgs& a, const void* g, int32_t g_type, const void* x, int32_t x_type,
                     const float* x_scale, const uint8_t* starts, const float* h0, int64_t steps, int64_t rows,
                     int32_t cols, void* work, size_t work_bytes) {
  if (cols < 1 || cols > MGN_ROW_MAX_COLS || !size_ok(rows, cols) || steps < 0 ||
      (rows > 0 && !size_ok(steps, rows * cols)))
    return bad(fn, "bad sizes");
  if (!float_type(g_type) || !(x_type == g_type || x_type == MGN_E4M3))
    return bad(fn, "g must be MGN_FP32 or MGN_BF16, x of g's type or MGN_E4M3");
  const bool any = steps > 0 && rows > 0;
  if (any && (!g || !x)) return bad(fn, "NULL argument");
  if (any && (x_type == MGN_E4M3) != (x_scale != nullptr)) return bad(fn, "x_scale goes with 8-bit x");
  if (!aligned(g, type_size(g_type)) || !aligned(x, type_size(x_type)) || !aligned(x_scale, 4) || !aligned(h0, 4) ||
      !aligned(work, 16))
    return bad(fn, "misaligned pointer");
  const size_t need = any ? scan_work_bytes(steps, rows, cols) : 0;
  if (work_bytes < need || (need && !work))
    return set_error(nullptr, MGN_E_NOMEM,
                     std::string(fn) + ": work too small (need " + std::to_string(need) + " bytes)");
  a.g = g;
  a.x = x;
  a.x_scale = x_scale;
  a.starts = starts;
  a.h0 = h0;
  a.steps = steps;
  a.rows = rows;
  a.cols = cols;
  a.work = work;
  return MGN_OK;
}

}  // namespace

extern "C" {

mgn_status mgn_gated_scan(const void* g, int32_t g_type, const void* x, int32_t x_type, const float* x_scale,
                          const uint8_t* starts, const float* h0, int64_t steps, int64_t rows, int32_t cols, float* h,
                          float* h_last, void* work, size_t work_bytes, mgn_stream stream) {
  const char* fn = "mgn_gated_scan";
  ScanArgs a{};
  mgn_status s = scan_args(fn, a, g, g_type, x, x_type, x_scale, starts, h0, steps, rows, cols, work, work_bytes);
  if (s) return s;
  if (rows == 0 || (steps == 0 && !h_last)) return MGN_OK;
  if (!h && !h_last) return bad(fn, "neither h nor h_last is wanted");
  if (!aligned(h, 4) || !aligned(h_last, 4)) return bad(fn, "misaligned pointer");
  const int64_t m = rows * cols, n = steps * m;
  if (clash({rd(g, n * type_size(g_type)), rd(x, n * type_size(x_type)), rd(x_scale, 4 * steps * rows * blocks(cols)),
             rd(starts, steps), rd(apart(h0, {h_last}), 4 * m), to(h, 4 * n), to(h_last, 4 * m),
             to(work, (int64_t)scan_work_bytes(steps, rows, cols))}))
    return bad(fn, "overlapping arrays");
  a.h = h;
  a.h_last = h_last;
  return launched(launch_scan(a, g_type, x_type, (hipStream_t)stream), fn);
}

mgn_status mgn_gated_scan_grad(const void* g, int32_t g_type, const void* x, int32_t x_type, const float* x_scale,
                               const uint8_t* starts, const float* h0, const float* h, const float* dh,
                               const float* dh_last, int64_t steps, int64_t rows, int32_t cols, void* dg, void* dx,
                               float* dh0, void* work, size_t work_bytes, mgn_stream stream) {
  const char* fn = "mgn_gated_scan_grad";
  ScanArgs a{};
  mgn_status s = scan_args(fn, a, g, g_type, x, x_type, x_scale, starts, h0, steps, rows, cols, work, work_bytes);
  if (s) return s;
  if (rows == 0 || (steps == 0 && !dh0)) return MGN_OK;
  if (steps > 0 && (!h || !dg || !dx)) return bad(fn, "NULL argument");
  const int32_t d_type = x_type == MGN_E4M3 ? g_type : x_type;
  if (!aligned(h, 4) || !aligned(dh, 4) || !aligned(dh_last, 4) || !aligned(dh0, 4) || !aligned(dg, type_size(g_type)) ||
      !aligned(dx, type_size(d_type)))
    return bad(fn, "misaligned pointer");
  const int64_t m = rows * cols, n = steps * m;
  if (clash({rd(g, n * type_size(g_type)), rd(x, n * type_size(x_type)), rd(x_scale, 4 * steps * rows * blocks(cols)),
             rd(starts, steps), rd(h0, 4 * m), rd(h, 4 * n), rd(dh, 4 * n), rd(apart(dh_last, {dh0}), 4 * m),
             to(dg, n * type_size(g_type)), to(dx, n * type_size(d_type)), to(dh0, 4 * m),
             to(work, (int64_t)scan_work_bytes(steps, rows, cols))}))
    return bad(fn, "overlapping arrays");
  a.h = const_cast<float*>(h);
  a.dh = dh;
  a.dh_last = dh_last;
  a.dg = dg;
  a.dx = dx;
  a.dh0 = dh0;
  return launched(launch_scan_grad(a, g_type, x_type, (hipStream_t)stream), fn);
}

}  // extern "C"

// C ABI of the 8-bit operators: argument validation on the host, then dispatch to the kernel launchers.
#include "api_check.h"
#include "common.h"

using namespace mb;

namespace {

mb_status check_dtype(mb_dtype dt) {
  MB_REQUIRE(dt == MB_F32 || dt == MB_BF16, MB_ERR_INVALID_ARG, "unknown dtype %d", (int)dt);
  return MB_OK;
}

// The kernels form a tile's offsets, 256 rows at most, in 32 bits and count tiles in 32 bits.
constexpr int kMaxRows = 1 << 30, kMaxWidth = 1 << 20, kMaxStride = 1 << 21;

mb_status check_rows(int T_cap) {
  MB_REQUIRE(T_cap >= 0, MB_ERR_INVALID_ARG, "T_cap must be >= 0 (got %d)", T_cap);
  MB_REQUIRE(T_cap <= kMaxRows, MB_ERR_UNSUPPORTED, "T_cap=%d exceeds 2^30", T_cap);
  return MB_OK;
}
mb_status check_width(int W, int multiple, const char* name) {
  MB_REQUIRE(W > 0, MB_ERR_INVALID_ARG, "%s must be positive (got %d)", name, W);
  MB_REQUIRE(W % multiple == 0, MB_ERR_UNSUPPORTED, "%s must be a multiple of %d (got %d)", name, multiple, W);
  MB_REQUIRE(W <= kMaxWidth, MB_ERR_UNSUPPORTED, "%s=%d exceeds 2^20", name, W);
  return MB_OK;
}
mb_status check_stride(int64_t stride, int W, mb_dtype dt, const char* name) {
  MB_REQUIRE(stride >= W, MB_ERR_INVALID_ARG, "%s=%lld is smaller than the row's %d elements", name, (long long)stride, W);
  MB_REQUIRE(stride < kMaxStride, MB_ERR_UNSUPPORTED, "%s=%lld elements exceeds 2^21", name, (long long)stride);
  MB_REQUIRE(stride * (int64_t)elem_size(dt) % 16 == 0, MB_ERR_INVALID_ARG, "%s=%lld elements is not a multiple of 16 bytes",
             name, (long long)stride);
  return MB_OK;
}
#define MB_CHECK(call)                \
  do {                                \
    const mb_status st_ = (call);     \
    if (st_ != MB_OK) return st_;     \
  } while (0)

// (the row kernels count a row's pieces of 16 in 32 bits, and a launch has less than 2^32 threads: 8 to a block)
mb_status check_matrix(int T_cap, int W) {
  MB_REQUIRE((int64_t)T_cap * W < ((int64_t)1 << 35), MB_ERR_UNSUPPORTED, "matrix of 2^35 elements or more (%d x %d)", T_cap, W);
  MB_REQUIRE((int64_t)T_cap * ((W + 127) / 128) < ((int64_t)1 << 29), MB_ERR_UNSUPPORTED, "2^29 blocks of 128 or more (%d x %d)", T_cap, W);
  return MB_OK;
}
mb_status check_product(int T_cap, int n_in, int n_out) {
  MB_CHECK(check_rows(T_cap));
  MB_CHECK(check_width(n_in, 16, "n_in"));
  MB_CHECK(check_width(n_out, 16, "n_out"));
  MB_REQUIRE((int64_t)T_cap * n_out < ((int64_t)1 << 38), MB_ERR_UNSUPPORTED, "T_cap * n_out of 2^38 or more (%d, %d)", T_cap, n_out);
  return MB_OK;
}
// (partial gradients are added up by two threads for an element at most, of less than 2^32 in a launch)
mb_status check_gradient(int T_cap, int n_in, int n_out) {
  MB_CHECK(check_product(T_cap, n_in, n_out));
  MB_REQUIRE((int64_t)n_in * n_out < ((int64_t)1 << 31), MB_ERR_UNSUPPORTED, "gradient of 2^31 elements or more (%d x %d)", n_out, n_in);
  return MB_OK;
}

}  // namespace

extern "C" {

mb_status mb_fp8_quant(const void* x, int64_t x_row_stride, int T_cap, const int32_t* meta_dev, int W, mb_dtype dt, uint8_t* q,
                       uint8_t* s, void* stream) {
  clear_error();
  MB_CHECK(check_dtype(dt));
  MB_CHECK(check_rows(T_cap));
  MB_CHECK(check_width(W, 16, "W"));
  MB_CHECK(check_matrix(T_cap, W));
  MB_CHECK(check_stride(x_row_stride, W, dt, "x_row_stride"));
  if (T_cap == 0) return MB_OK;
  MB_CHECK_PTR(x);
  MB_CHECK_PTR(q);
  MB_CHECK_PTR(s);
  return launch_fp8_quant(dt, x, x_row_stride, T_cap, meta_dev, W, q, s, (hipStream_t)stream);
}

mb_status mb_fp8_dequant(const uint8_t* q, const uint8_t* s, int T_cap, const int32_t* meta_dev, int W, mb_dtype dt, void* x,
                         int64_t x_row_stride, void* stream) {
  clear_error();
  MB_CHECK(check_dtype(dt));
  MB_CHECK(check_rows(T_cap));
  MB_CHECK(check_width(W, 16, "W"));
  MB_CHECK(check_matrix(T_cap, W));
  MB_CHECK(check_stride(x_row_stride, W, dt, "x_row_stride"));
  if (T_cap == 0) return MB_OK;
  MB_CHECK_PTR(q);
  MB_CHECK_PTR(s);
  MB_CHECK_PTR(x);
  return launch_fp8_dequant(dt, q, s, T_cap, meta_dev, W, x, x_row_stride, (hipStream_t)stream);
}

mb_status mb_fp8_quant_weight(const void* w, int n_out, int n_in, mb_dtype dt, uint8_t* q, uint8_t* s, uint8_t* qt, uint8_t* st,
                              void* stream) {
  clear_error();
  MB_CHECK(check_dtype(dt));
  MB_CHECK(check_width(n_out, 16, "n_out"));
  MB_CHECK(check_width(n_in, 16, "n_in"));
  MB_REQUIRE((qt == nullptr) == (st == nullptr), MB_ERR_INVALID_ARG, "qt and st are given together or not at all");
  MB_CHECK_PTR(w);
  MB_CHECK_PTR(q);
  MB_CHECK_PTR(s);
  if (qt != nullptr) {
    MB_CHECK_PTR(qt);
    MB_CHECK_PTR(st);
  }
  return launch_fp8_quant_weight(dt, w, n_out, n_in, q, s, qt, st, (hipStream_t)stream);
}

mb_status mb_linear_fp8_fwd(const uint8_t* xq, const uint8_t* xs, const uint8_t* wq, const uint8_t* ws, int T_cap,
                            const int32_t* meta_dev, int n_in, int n_out, mb_dtype dt, void* y, int64_t y_row_stride,
                            void* stream) {
  clear_error();
  MB_CHECK(check_dtype(dt));
  MB_CHECK(check_product(T_cap, n_in, n_out));
  MB_CHECK(check_stride(y_row_stride, n_out, dt, "y_row_stride"));
  if (T_cap == 0) return MB_OK;
  MB_CHECK_PTR(xq);
  MB_CHECK_PTR(xs);
  MB_CHECK_PTR(wq);
  MB_CHECK_PTR(ws);
  MB_CHECK_PTR(y);
  return launch_linear_fp8_fwd(xq, xs, wq, ws, T_cap, meta_dev, n_in, n_out, dt, y, y_row_stride, (hipStream_t)stream);
}

size_t mb_linear_fp8_wgrad_workspace_bytes(int T_cap, int n_in, int n_out) {
  if (check_gradient(T_cap, n_in, n_out) != MB_OK) return 0;
  return linear_fp8_wgrad_workspace_bytes(T_cap, n_in, n_out);
}

mb_status mb_linear_fp8_wgrad(const void* dy, const uint8_t* dys, int64_t dy_row_stride, const uint8_t* xq, const uint8_t* xs,
                              int T_cap, const int32_t* meta_dev, int n_in, int n_out, float* dw, void* workspace,
                              size_t workspace_bytes, void* stream) {
  clear_error();
  MB_CHECK(check_gradient(T_cap, n_in, n_out));
  if (dys == nullptr) MB_CHECK(check_stride(dy_row_stride, n_out, MB_BF16, "dy_row_stride"));
  else MB_REQUIRE(dy_row_stride == n_out, MB_ERR_INVALID_ARG, "8-bit rows of dy are contiguous: dy_row_stride=%lld, n_out=%d",
                  (long long)dy_row_stride, n_out);
  MB_CHECK_PTR(dw);
  if (T_cap > 0) {
    MB_CHECK_PTR(dy);
    if (dys != nullptr) MB_CHECK_PTR(dys);
    MB_CHECK_PTR(xq);
    MB_CHECK_PTR(xs);
  }
  const size_t need = linear_fp8_wgrad_workspace_bytes(T_cap, n_in, n_out);
  if (need > 0) {
    MB_REQUIRE(workspace != nullptr && workspace_bytes >= need, MB_ERR_WORKSPACE,
               "workspace of %zu bytes given, %zu needed", workspace ? workspace_bytes : (size_t)0, need);
    MB_REQUIRE(aligned16(workspace), MB_ERR_INVALID_ARG, "workspace is not 16-byte aligned");
  }
  return launch_linear_fp8_wgrad(dy, dys, dy_row_stride, xq, xs, T_cap, meta_dev, n_in, n_out, dw, workspace, (hipStream_t)stream);
}

mb_status mb_geglu_fp8_act(const uint8_t* xq, const uint8_t* xs, const uint8_t* w1vq, const uint8_t* w1vs, int T_cap,
                           const int32_t* meta_dev, int hidden, int inter, uint8_t* actq, uint8_t* acts, void* stream) {
  clear_error();
  MB_CHECK(check_rows(T_cap));
  MB_CHECK(check_width(hidden, 16, "hidden"));
  MB_CHECK(check_width(inter, 128, "inter"));
  MB_REQUIRE(2 * (int64_t)inter * hidden < ((int64_t)1 << 31), MB_ERR_UNSUPPORTED,
             "weight of 2^31 elements or more (hidden=%d inter=%d)", hidden, inter);
  MB_REQUIRE((int64_t)T_cap * inter < ((int64_t)1 << 38), MB_ERR_UNSUPPORTED, "T_cap * inter of 2^38 or more (%d, %d)", T_cap, inter);
  if (T_cap == 0) return MB_OK;
  MB_CHECK_PTR(xq);
  MB_CHECK_PTR(xs);
  MB_CHECK_PTR(w1vq);
  MB_CHECK_PTR(w1vs);
  MB_CHECK_PTR(actq);
  MB_CHECK_PTR(acts);
  return launch_geglu_fp8_act(xq, xs, w1vq, w1vs, T_cap, meta_dev, hidden, inter, actq, acts, (hipStream_t)stream);
}

mb_status mb_gelu_gate_fp8_bwd(const void* da, const void* hg, const uint8_t* hgs, int T_cap, const int32_t* meta_dev, int inter,
                               uint8_t* dhgq, uint8_t* dhgs, void* stream) {
  clear_error();
  MB_CHECK(check_rows(T_cap));
  MB_CHECK(check_width(inter, 128, "inter"));
  MB_CHECK(check_matrix(T_cap, inter));
  if (T_cap == 0) return MB_OK;
  MB_CHECK_PTR(da);
  MB_CHECK_PTR(hg);
  if (hgs != nullptr) MB_CHECK_PTR(hgs);
  MB_CHECK_PTR(dhgq);
  MB_CHECK_PTR(dhgs);
  return launch_gelu_gate_fp8_bwd(da, hg, hgs, T_cap, meta_dev, inter, dhgq, dhgs, (hipStream_t)stream);
}

}  // extern "C"

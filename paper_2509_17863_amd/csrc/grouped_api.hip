// C ABI of the separate products of an expert layer: host-side validation and
// kernel enqueueing, under the conventions of eaas_api.hip (nothing is
// allocated, nothing waits, a refused call enqueues nothing).
#include <limits.h>
#include <stdint.h>

#include <algorithm>

#include "common.h"
#include "internal.h"

namespace {

using namespace eaas;

constexpr long long kMaxLd = 1 << 22;

int hip_status(hipError_t e) { return e == hipSuccess ? EAAS_OK : EAAS_ERR_HIP; }

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// Rows of `width` bytes, `pitch` bytes apart.
struct Span {
  uintptr_t at;
  unsigned long long bytes, pitch, width;
};
Span rows_span(const void* p, long long rows, long long ld, long long width, int esz) {
  return {(uintptr_t)p, rows > 0 ? (unsigned long long)((rows - 1) * ld + width) * esz : 0,
          (unsigned long long)ld * esz, (unsigned long long)width * esz};
}
bool overlap(const Span& a, const Span& b) {
  if (a.at >= b.at + b.bytes || b.at >= a.at + a.bytes) return false;
  if (a.pitch != b.pitch) return true;
  // rows of one wider array: side by side, or one over the other
  const Span &lo = a.at <= b.at ? a : b, &hi = a.at <= b.at ? b : a;
  const unsigned long long d = (hi.at - lo.at) % lo.pitch;
  return d < lo.width || d + hi.width > lo.pitch;
}

int check_group(const eaas_group_shape* s) {
  if (!s || s->R < 0 || s->E <= 0 || s->N <= 0 || s->K <= 0) return EAAS_ERR_INVALID_ARG;
  if (s->E > kMaxExperts || (long long)s->N * s->K > INT_MAX) return EAAS_ERR_UNSUPPORTED;
  return EAAS_OK;
}

int check_ld(long long ld, int width) {
  if (ld < width) return EAAS_ERR_INVALID_ARG;
  return ld > kMaxLd ? EAAS_ERR_UNSUPPORTED : EAAS_OK;
}

// Rows of x, with or without a perm.
int check_gather(const eaas_group_shape* s, const int32_t* perm, int32_t k, long long ldx,
                 long long* rows) {
  *rows = s->R;
  if (!perm) return EAAS_OK;
  if (k < 1 || s->R % k) return EAAS_ERR_INVALID_ARG;
  *rows = s->R / k;
  return *rows * ldx > INT_MAX ? EAAS_ERR_UNSUPPORTED : EAAS_OK;
}

bool out_type(int t) { return t == EAAS_BF16 || t == EAAS_FP32; }

GroupedArgs args_of(const eaas_group_shape* s, int dir, bool i8) {
  GroupedArgs a{};
  a.dir = dir;
  a.i8 = i8;
  a.R = s->R;
  a.E = s->E;
  a.N = s->N;
  a.K = s->K;
  return a;
}

int enqueue(GroupedArgs& a, void* ws, size_t ws_bytes, void* stream) {
  const size_t need = grouped_workspace(a);
  if (need > 0 && (!ws || !aligned(ws, 16) || ws_bytes < need)) return EAAS_ERR_WORKSPACE;
  a.ws = ws;
  return hip_status(launch_grouped(a, reinterpret_cast<hipStream_t>(stream)));
}

// The forward product of either operand type (esz: bytes of x's and w's elements).
int forward(const eaas_group_shape* s, const void* x, long long ldx, const float* xs,
            const int32_t* perm, int32_t k, const int32_t* offsets, const void* w,
            const float* wscale, void* y, long long ldy, int y_dtype, bool i8, void* ws,
            size_t ws_bytes, void* stream) {
  const int esz = i8 ? 1 : 2, osz = y_dtype == EAAS_FP32 ? 4 : 2;
  int st = check_group(s);
  if (st != EAAS_OK) return st;
  if (i8 && s->K >= 1 << 17) return EAAS_ERR_UNSUPPORTED;
  if (!out_type(y_dtype)) return EAAS_ERR_INVALID_ARG;
  if ((st = check_ld(ldx, s->K)) != EAAS_OK || (st = check_ld(ldy, s->N)) != EAAS_OK) return st;
  long long rows;
  if ((st = check_gather(s, perm, k, ldx, &rows)) != EAAS_OK) return st;
  if (s->R == 0) return EAAS_OK;
  if (!x || !offsets || !w || !y || (i8 && (!xs || !wscale))) return EAAS_ERR_INVALID_ARG;
  if (!aligned(x, esz) || !aligned(w, 16) || !aligned(y, osz) || !aligned(offsets, 4) ||
      (perm && !aligned(perm, 4)) || (i8 && (!aligned(xs, 4) || !aligned(wscale, 4))))
    return EAAS_ERR_INVALID_ARG;
  const Span out = rows_span(y, s->R, ldy, s->N, osz);
  if (overlap(out, rows_span(x, rows, ldx, s->K, esz)) ||
      overlap(out, rows_span(w, (long long)s->E * s->N, s->K, s->K, esz)))
    return EAAS_ERR_INVALID_ARG;
  GroupedArgs a = args_of(s, kForward, i8);
  a.a = x;
  a.lda = ldx;
  a.b = w;
  a.perm = perm;
  a.k = perm ? k : 1;
  a.offsets = offsets;
  a.out = y;
  a.ldo = ldy;
  a.out_fp32 = y_dtype == EAAS_FP32;
  a.row_scale = xs;
  a.col_scale = wscale;
  return enqueue(a, ws, ws_bytes, stream);
}

int check_rows(int64_t rows, int32_t width, int32_t most) {
  if (rows < 0 || width <= 0) return EAAS_ERR_INVALID_ARG;
  return rows > INT_MAX || width > most ? EAAS_ERR_UNSUPPORTED : EAAS_OK;
}

}  // namespace

extern "C" {

size_t eaas_grouped_workspace_bytes(const eaas_group_shape* s) {
  if (check_group(s) != EAAS_OK) return 0;
  size_t n = 256;
  for (int dir = kForward; dir <= kGradWeights; ++dir)
    n = std::max(n, grouped_workspace_most(args_of(s, dir, false)));
  n = std::max(n, grouped_workspace_most(args_of(s, kForward, true)));
  return (n + 255) / 256 * 256;
}

int eaas_grouped_matmul(const eaas_group_shape* s, const void* x, int64_t ldx,
                        const int32_t* perm, int32_t k, const int32_t* offsets, const void* w,
                        void* y, int64_t ldy, int y_dtype, void* ws, size_t ws_bytes,
                        void* stream) {
  return forward(s, x, ldx, nullptr, perm, k, offsets, w, nullptr, y, ldy, y_dtype, false, ws,
                 ws_bytes, stream);
}

int eaas_grouped_matmul_int8(const eaas_group_shape* s, const void* xq, const float* xs,
                             const int32_t* perm, int32_t k, const int32_t* offsets,
                             const void* wq, const float* wscale, void* y, int64_t ldy,
                             int y_dtype, void* ws, size_t ws_bytes, void* stream) {
  return forward(s, xq, s ? s->K : 0, xs, perm, k, offsets, wq, wscale, y, ldy, y_dtype, true, ws,
                 ws_bytes, stream);
}

int eaas_grouped_matmul_dx(const eaas_group_shape* s, const void* dy, int64_t lddy,
                           const int32_t* offsets, const void* w, void* dx, int64_t lddx,
                           int dx_dtype, void* ws, size_t ws_bytes, void* stream) {
  const int osz = dx_dtype == EAAS_FP32 ? 4 : 2;
  int st = check_group(s);
  if (st != EAAS_OK) return st;
  if (!out_type(dx_dtype)) return EAAS_ERR_INVALID_ARG;
  if ((st = check_ld(lddy, s->N)) != EAAS_OK || (st = check_ld(lddx, s->K)) != EAAS_OK) return st;
  if (s->R == 0) return EAAS_OK;
  if (!dy || !offsets || !w || !dx) return EAAS_ERR_INVALID_ARG;
  if (!aligned(dy, 2) || !aligned(w, 16) || !aligned(dx, osz) || !aligned(offsets, 4))
    return EAAS_ERR_INVALID_ARG;
  const Span out = rows_span(dx, s->R, lddx, s->K, osz);
  if (overlap(out, rows_span(dy, s->R, lddy, s->N, 2)) ||
      overlap(out, rows_span(w, (long long)s->E * s->N, s->K, s->K, 2)))
    return EAAS_ERR_INVALID_ARG;
  GroupedArgs a = args_of(s, kGradRows, false);
  a.a = dy;
  a.lda = lddy;
  a.b = w;
  a.k = 1;
  a.offsets = offsets;
  a.out = dx;
  a.ldo = lddx;
  a.out_fp32 = dx_dtype == EAAS_FP32;
  return enqueue(a, ws, ws_bytes, stream);
}

int eaas_grouped_matmul_dw(const eaas_group_shape* s, const void* dy, int64_t lddy,
                           const void* x, int64_t ldx, const int32_t* perm, int32_t k,
                           const int32_t* offsets, void* dw, int dw_dtype, int accumulate,
                           void* ws, size_t ws_bytes, void* stream) {
  const int osz = dw_dtype == EAAS_FP32 ? 4 : 2;
  int st = check_group(s);
  if (st != EAAS_OK) return st;
  if (!out_type(dw_dtype) || (accumulate && dw_dtype != EAAS_FP32)) return EAAS_ERR_INVALID_ARG;
  if ((st = check_ld(lddy, s->N)) != EAAS_OK || (st = check_ld(ldx, s->K)) != EAAS_OK) return st;
  long long rows;
  if ((st = check_gather(s, perm, k, ldx, &rows)) != EAAS_OK) return st;
  if (s->R == 0 && accumulate) return EAAS_OK;
  if ((s->R > 0 && (!dy || !x)) || !offsets || !dw) return EAAS_ERR_INVALID_ARG;
  if (!aligned(dy, 2) || !aligned(x, 2) || !aligned(dw, 16) || !aligned(offsets, 4) ||
      (perm && !aligned(perm, 4)))
    return EAAS_ERR_INVALID_ARG;
  const Span out = rows_span(dw, (long long)s->E * s->N, s->K, s->K, osz);
  if (overlap(out, rows_span(dy, s->R, lddy, s->N, 2)) ||
      overlap(out, rows_span(x, rows, ldx, s->K, 2)))
    return EAAS_ERR_INVALID_ARG;
  GroupedArgs a = args_of(s, kGradWeights, false);
  a.a = dy;
  a.lda = lddy;
  a.b = x;
  a.ldb = ldx;
  a.perm = perm;
  a.k = perm ? k : 1;
  a.offsets = offsets;
  a.out = dw;
  a.ldo = s->K;
  a.out_fp32 = dw_dtype == EAAS_FP32;
  a.accumulate = accumulate != 0;
  return enqueue(a, ws, ws_bytes, stream);
}

int eaas_quantize_rows_int8(const void* x, int64_t ldx, int64_t rows, int32_t K, void* q,
                            float* s, void* stream) {
  int st = check_rows(rows, K, (int32_t)kMaxLd);
  if (st != EAAS_OK || (st = check_ld(ldx, K)) != EAAS_OK) return st;
  if (rows == 0) return EAAS_OK;
  if (!x || !q || !s || !aligned(x, 2) || !aligned(s, 4)) return EAAS_ERR_INVALID_ARG;
  const Span in = rows_span(x, rows, ldx, K, 2);
  if (overlap(in, rows_span(q, rows, K, K, 1)) || overlap(in, rows_span(s, rows, 1, 1, 4)))
    return EAAS_ERR_INVALID_ARG;
  return hip_status(launch_quantize_int8(static_cast<const uint16_t*>(x), ldx, rows, K,
                                         static_cast<int8_t*>(q), s,
                                         reinterpret_cast<hipStream_t>(stream)));
}

int eaas_swiglu(const void* gu, int64_t rows, int32_t I, const int32_t* n_rows, void* h,
                void* stream) {
  const int st = check_rows(rows, I, 1 << 21);
  if (st != EAAS_OK) return st;
  if (rows == 0) return EAAS_OK;
  if (!gu || !h || !aligned(gu, 2) || !aligned(h, 2) || !aligned(n_rows, 4))
    return EAAS_ERR_INVALID_ARG;
  if (overlap(rows_span(gu, rows, 2LL * I, 2LL * I, 2), rows_span(h, rows, I, I, 2)))
    return EAAS_ERR_INVALID_ARG;
  return hip_status(launch_swiglu(static_cast<const uint16_t*>(gu), rows, I, n_rows,
                                  static_cast<uint16_t*>(h),
                                  reinterpret_cast<hipStream_t>(stream)));
}

int eaas_swiglu_int8(const void* gu, int64_t rows, int32_t I, const int32_t* n_rows, void* q,
                     float* s, void* stream) {
  const int st = check_rows(rows, I, 1 << 21);
  if (st != EAAS_OK) return st;
  if (rows == 0) return EAAS_OK;
  if (!gu || !q || !s || !aligned(gu, 2) || !aligned(s, 4) || !aligned(n_rows, 4))
    return EAAS_ERR_INVALID_ARG;
  const Span in = rows_span(gu, rows, 2LL * I, 2LL * I, 2);
  if (overlap(in, rows_span(q, rows, I, I, 1)) || overlap(in, rows_span(s, rows, 1, 1, 4)))
    return EAAS_ERR_INVALID_ARG;
  return hip_status(launch_swiglu_int8(static_cast<const uint16_t*>(gu), rows, I, n_rows,
                                       static_cast<int8_t*>(q), s,
                                       reinterpret_cast<hipStream_t>(stream)));
}

int eaas_swiglu_backward(const void* gu, const void* dh, int64_t rows, int32_t I,
                         const int32_t* n_rows, void* dgu, void* stream) {
  const int st = check_rows(rows, I, 1 << 21);
  if (st != EAAS_OK) return st;
  if (rows == 0) return EAAS_OK;
  if (!gu || !dh || !dgu || !aligned(gu, 2) || !aligned(dh, 2) || !aligned(dgu, 2) ||
      !aligned(n_rows, 4))
    return EAAS_ERR_INVALID_ARG;
  const Span out = rows_span(dgu, rows, 2LL * I, 2LL * I, 2);
  if ((gu != dgu && overlap(out, rows_span(gu, rows, 2LL * I, 2LL * I, 2))) ||
      overlap(out, rows_span(dh, rows, I, I, 2)))
    return EAAS_ERR_INVALID_ARG;
  return hip_status(launch_swiglu_backward(static_cast<const uint16_t*>(gu),
                                           static_cast<const uint16_t*>(dh), rows, I, n_rows,
                                           static_cast<uint16_t*>(dgu),
                                           reinterpret_cast<hipStream_t>(stream)));
}

int eaas_unpermute_combine_backward(const eaas_shape* s, const void* dout, int dout_dtype,
                                    const float* y_perm, const eaas_routing* r,
                                    const float* topk_weights, void* dy_perm, float* dweights,
                                    void* stream) {
  // the shape rules of eaas_unpermute_combine
  if (eaas_workspace_bytes(s, EAAS_BF16) == 0)
    return !s || s->T < 0 || s->H <= 0 || s->I <= 0 || s->E <= 0 || s->k <= 0
               ? EAAS_ERR_INVALID_ARG : EAAS_ERR_UNSUPPORTED;
  if (!out_type(dout_dtype)) return EAAS_ERR_INVALID_ARG;
  if (s->T == 0) return EAAS_OK;
  if (!dout || !y_perm || !r || !r->inv || !topk_weights || !dy_perm || !dweights ||
      !aligned(dout, 16) || !aligned(y_perm, 16) || !aligned(r->inv, 16) || !aligned(dy_perm, 16))
    return EAAS_ERR_INVALID_ARG;
  const long long R = (long long)s->T * s->k;
  const Span dy = rows_span(dy_perm, R, s->H, s->H, 2), dw = rows_span(dweights, R, 1, 1, 4);
  const Span in[3] = {rows_span(dout, s->T, s->H, s->H, dout_dtype == EAAS_FP32 ? 4 : 2),
                      rows_span(y_perm, R, s->H, s->H, 4), rows_span(topk_weights, R, 1, 1, 4)};
  if (overlap(dy, dw)) return EAAS_ERR_INVALID_ARG;
  for (const Span& i : in)
    if (overlap(dy, i) || overlap(dw, i)) return EAAS_ERR_INVALID_ARG;
  return hip_status(launch_combine_backward(dout, dout_dtype == EAAS_FP32, y_perm, r->inv,
                                            topk_weights, s->T, s->H, s->k,
                                            static_cast<uint16_t*>(dy_perm), dweights,
                                            reinterpret_cast<hipStream_t>(stream)));
}

// Not part of the ABI: the kernel that a product takes, for tests and measurements
// (grouped_plan_code), or -1 for what the library rejects.  dir: 0 forward, 1 gradient
// in the rows, 2 in the weights; i8: in 8-bit integers; in16: sizes, strides and bases
// in multiples of 16 bytes.
int eaas_internal_grouped_plan(const eaas_group_shape* s, int dir, int i8, int in16) {
  if (check_group(s) != EAAS_OK || dir < kForward || dir > kGradWeights || (i8 && dir != kForward))
    return -1;
  return grouped_plan_code(args_of(s, dir, i8 != 0), in16 != 0);
}

}  // extern "C"

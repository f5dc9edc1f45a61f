// C ABI of microscaled 4-bit floating point (include/mxfp4.h): argument checks and the launch sequence.
#pragma GCC visibility push(default)
#include "../../include/mxfp4.h"
#pragma GCC visibility pop

#include "layer.h"
#include "mxfp4.h"

namespace sla {
void launch_mxfp4_quantize(const void* x, int R, int K, uint8_t* codes, uint8_t* exps, hipStream_t stream);
void launch_mxfp4_dequantize(const uint8_t* codes, const uint8_t* exps, int R, int K, void* x, hipStream_t stream);
void launch_mxfp4_pack(const uint8_t* from, const uint8_t* from_exps, int R, int K, uint8_t* codes, uint8_t* exps, hipStream_t stream);
void launch_mxfp4_unpack(const uint8_t* codes, const uint8_t* exps, int R, int K, uint8_t* to, uint8_t* to_exps, hipStream_t stream);
void launch_mxfp4_gemm(const uint8_t* x, const uint8_t* xe, const uint8_t* w, const uint8_t* we, const void* bias, void* y, int M,
                       int N, int K, hipStream_t stream);
bool launch_mxfp4_linear_few(const void* x, const uint8_t* w, const uint8_t* we, const void* bias, void* y, int M, int N, int K,
                             hipStream_t stream);
}  // namespace sla

using namespace sla;

namespace {

bool width_ok(int K) { return K >= 8 && K <= 65536 && !(K & 7); }
bool rows_ok(int R) { return R >= 1 && R <= (1 << 22); }
bool dims_ok(int R, int K) { return rows_ok(R) && width_ok(K); }
// the exponents of an object
const uint8_t* exps_of(const void* q, int R, int K) { return (const uint8_t*)q + mx_codes_bytes(R, K); }
uint8_t* exps_of(void* q, int R, int K) { return (uint8_t*)q + mx_codes_bytes(R, K); }
int check_object(const void* q, size_t bytes, int R, int K) { return check_ws(q, bytes, mx_object_bytes(R, K)); }
// what every form of the layer checks of weight, bias and result
int layer_out(const void* wq, size_t wq_bytes, const void* bias, const void* y, int N, int K) {
  if (int st = check_object(wq, wq_bytes, N, K)) return st;
  return aligned16(y) && aligned16(bias) ? SLA_OK : SLA_ERR_LAYOUT;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

size_t mxfp4_bytes(int R, int K) { return dims_ok(R, K) ? mx_object_bytes(R, K) : 0; }

int mxfp4_quantize(const void* x, int R, int K, void* q, size_t q_bytes, sla_stream_t stream) {
  if (!x || !q) return SLA_ERR_NULL;
  if (!dims_ok(R, K)) return SLA_ERR_SHAPE;
  if (int st = check_object(q, q_bytes, R, K)) return st;
  if (!aligned16(x)) return SLA_ERR_LAYOUT;
  launch_mxfp4_quantize(x, R, K, (uint8_t*)q, exps_of(q, R, K), (hipStream_t)stream);
  return launch_status();
}

int mxfp4_dequantize(const void* q, size_t q_bytes, int R, int K, void* x, sla_stream_t stream) {
  if (!x || !q) return SLA_ERR_NULL;
  if (!dims_ok(R, K)) return SLA_ERR_SHAPE;
  if (int st = check_object(q, q_bytes, R, K)) return st;
  if (!aligned16(x)) return SLA_ERR_LAYOUT;
  launch_mxfp4_dequantize((const uint8_t*)q, exps_of(q, R, K), R, K, x, (hipStream_t)stream);
  return launch_status();
}

int mxfp4_pack(const uint8_t* codes, const uint8_t* exponents, int R, int K, void* q, size_t q_bytes, sla_stream_t stream) {
  if (!codes || !exponents || !q) return SLA_ERR_NULL;
  if (!dims_ok(R, K)) return SLA_ERR_SHAPE;
  if (int st = check_object(q, q_bytes, R, K)) return st;
  launch_mxfp4_pack(codes, exponents, R, K, (uint8_t*)q, exps_of(q, R, K), (hipStream_t)stream);
  return launch_status();
}

int mxfp4_unpack(const void* q, size_t q_bytes, int R, int K, uint8_t* codes, uint8_t* exponents, sla_stream_t stream) {
  if (!q) return SLA_ERR_NULL;
  if (!dims_ok(R, K)) return SLA_ERR_SHAPE;
  if (int st = check_object(q, q_bytes, R, K)) return st;
  if (codes || exponents) launch_mxfp4_unpack((const uint8_t*)q, exps_of(q, R, K), R, K, codes, exponents, (hipStream_t)stream);
  return launch_status();
}

int mxfp4_gemm_fwd(const void* xq, size_t xq_bytes, const void* wq, size_t wq_bytes, const void* bias, void* y, int M, int N,
                   int K, sla_stream_t stream) {
  if (!xq || !wq || !y) return SLA_ERR_NULL;
  if (!dims_ok(M, K) || !width_ok(N)) return SLA_ERR_SHAPE;
  if (int st = check_object(xq, xq_bytes, M, K)) return st;
  if (int st = layer_out(wq, wq_bytes, bias, y, N, K)) return st;
  launch_mxfp4_gemm((const uint8_t*)xq, exps_of(xq, M, K), (const uint8_t*)wq, exps_of(wq, N, K), bias, y, M, N, K,
                    (hipStream_t)stream);
  return launch_status();
}

int mxfp4_linear_fwd(const void* x, const void* wq, size_t wq_bytes, const void* bias, void* y, int M, int N, int K,
                     void* workspace, size_t workspace_bytes, sla_stream_t stream) {
  if (!x || !wq || !y) return SLA_ERR_NULL;
  if (!dims_ok(M, K) || !width_ok(N)) return SLA_ERR_SHAPE;
  if (int st = check_object(workspace, workspace_bytes, M, K)) return st;
  if (int st = layer_out(wq, wq_bytes, bias, y, N, K)) return st;
  if (!aligned16(x)) return SLA_ERR_LAYOUT;
  if (launch_mxfp4_linear_few(x, (const uint8_t*)wq, exps_of(wq, N, K), bias, y, M, N, K, (hipStream_t)stream)) return launch_status();
  uint8_t *codes = (uint8_t*)workspace, *exps = exps_of(workspace, M, K);
  launch_mxfp4_quantize(x, M, K, codes, exps, (hipStream_t)stream);
  if (int st = launch_status()) return st;
  launch_mxfp4_gemm(codes, exps, (const uint8_t*)wq, exps_of(wq, N, K), bias, y, M, N, K, (hipStream_t)stream);
  return launch_status();
}

int mxfp4_norm_quantize(const void* x, const void* res, const void* w, const void* b, const norm_modulation* mod, void* h,
                        void* q, size_t q_bytes, int M, int K, double eps, sla_stream_t stream) {
  if (!q) return SLA_ERR_NULL;
  LayerArgs a;
  if (int st = layer_args(x, res, w, b, mod, h, M, K, eps, &a)) return st;
  if (int st = check_object(q, q_bytes, M, K)) return st;
  a.codes = (uint8_t*)q;
  a.exps = exps_of(q, M, K);
  launch_layer_fwd(a, (hipStream_t)stream);
  return launch_status();
}

int mxfp4_norm_linear_fwd(const void* x, const void* res, const void* norm_w, const void* norm_b, const norm_modulation* mod,
                          void* h, const void* wq, size_t wq_bytes, const void* bias, void* y, int M, int N, int K, double eps,
                          void* workspace, size_t workspace_bytes, sla_stream_t stream) {
  if (!wq || !y) return SLA_ERR_NULL;
  LayerArgs a;
  if (int st = layer_args(x, res, norm_w, norm_b, mod, h, M, K, eps, &a)) return st;
  if (!width_ok(N)) return SLA_ERR_SHAPE;
  if (int st = check_object(workspace, workspace_bytes, M, K)) return st;
  if (int st = layer_out(wq, wq_bytes, bias, y, N, K)) return st;
  a.codes = (uint8_t*)workspace;
  a.exps = exps_of(workspace, M, K);
  launch_layer_fwd(a, (hipStream_t)stream);
  if (int st = launch_status()) return st;
  launch_mxfp4_gemm(a.codes, a.exps, (const uint8_t*)wq, exps_of(wq, N, K), bias, y, M, N, K, (hipStream_t)stream);
  return launch_status();
}

}  // extern "C"
#pragma GCC visibility pop

// C-ABI entry points: descriptor validation and dispatch.  All device work is in the kernel files.
#include "vq_common.hpp"
#include "vq_kv.hpp"
#include "vq_lend.h"
#include <algorithm>
#include <cfloat>
#include <cstdlib>
#include <cstring>
#include <mutex>

namespace vq {

int cu_count() {
  static const int n = [] {
    int dev = 0, c = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&c, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || c < 1) c = 256;
    return c;
  }();
  return n;
}

namespace {
thread_local Switches g_switches;
}
const Switches &switches() { return g_switches; }

// VQ_SWITCHES = "name=value,name=value": unknown names are ignored.
void read_switches() {
  Switches sw;
  const char *e = getenv("VQ_SWITCHES");
  while (e && *e) {
    const char *eq = strchr(e, '='), *end = strchr(e, ',');
    if (!end) end = e + strlen(e);
    if (eq && eq < end) {
      const size_t n = (size_t)(eq - e);
      const char v = eq[1] == ',' ? '\0' : eq[1];
      if (n == 4 && !strncmp(e, "gemv", 4)) sw.gemv = v;
      else if (n == 4 && !strncmp(e, "gemm", 4)) sw.gemm = v;
      else if (n == 7 && !strncmp(e, "dequant", 7)) sw.dequant = v;
      else if (n == 6 && !strncmp(e, "groups", 6)) sw.groups_loop = v == 'l';
      else if (n == 5 && !strncmp(e, "multi", 5)) sw.multi_off = v == '0';
      else if (n == 4 && !strncmp(e, "rows", 4)) sw.rows = v == '0' ? 0 : v == '1' ? 1 : -1;
      else if (n == 8 && !strncmp(e, "products", 8)) sw.products = v == '0' ? 0 : v == '1' ? 1 : -1;
      else if (n == 9 && !strncmp(e, "attention", 9)) sw.attention = v;
      else if (n == 6 && !strncmp(e, "shared", 6)) sw.shared = v >= '0' && v <= '2' ? v : 0;
      else if (n == 6 && !strncmp(e, "prefix", 6)) sw.prefix = v;
      else if (n == 12 && !strncmp(e, "prefix_parts", 12)) sw.prefix_parts = v >= '0' && v <= '5' ? v - '0' : -1;
      else if (n == 5 && !strncmp(e, "parts", 5)) sw.parts = v >= '0' && v <= '6' ? v - '0' : -1;
      else if (n == 5 && !strncmp(e, "dense", 5)) sw.dense = v >= '0' && v <= '9' ? v - '0' : -1;
    }
    e = *end ? end + 1 : end;
  }
  g_switches = sw;
}

static bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

static int check_stream(const void *idx, long long stride, int per_row, int bits) {
  if (!idx) return VQ_ERR_NULL;
  if (stride < ((long long)per_row * bits + 7) / 8) return VQ_ERR_SHAPE;
  if (stride % 16 != 0 || !aligned(idx, 16)) return VQ_ERR_ALIGNMENT;
  return VQ_OK;
}

int make_params(const vq_layer_desc *d, Params *p) {
  if (!d) return VQ_ERR_NULL;
  if (d->struct_size != sizeof(vq_layer_desc) && d->struct_size != VQ_LAYER_DESC_SIZE_V1 && d->struct_size != VQ_LAYER_DESC_SIZE_V2)
    return VQ_ERR_SHAPE;
  const bool v2 = d->struct_size != VQ_LAYER_DESC_SIZE_V1;
  const int group_vectors = v2 ? d->group_vectors : 0;
  const int orientation = v2 ? d->orientation : 0;
  const int32_t *col_perm = d->struct_size == sizeof(vq_layer_desc) ? d->col_perm : nullptr;
  if (col_perm && !aligned(col_perm, 4)) return VQ_ERR_ALIGNMENT;
  if (group_vectors < 0 || (orientation != 0 && orientation != 1)) return VQ_ERR_SHAPE;
  const int lim = 1 << 24;
  if (d->out_features < 1 || d->out_features > lim || d->in_features < 1 || d->in_features > lim) return VQ_ERR_SHAPE;
  if (d->v < 1 || d->v > 16 || d->k < 2 || d->k > 65536) return VQ_ERR_SHAPE;
  if (d->k_res != 0 && (d->k_res < 2 || d->k_res > 65536)) return VQ_ERR_SHAPE;
  if (d->n_outlier_cols < 0) return VQ_ERR_SHAPE;
  if (d->n_outlier_cols > 0) {
    if (d->v_out < 1 || d->v_out > 16 || d->k_out < 2 || d->k_out > 65536) return VQ_ERR_SHAPE;
    if ((orientation == 0 && d->n_outlier_cols % d->v_out != 0) || d->n_outlier_cols >= d->in_features) return VQ_ERR_SHAPE;
  }
  Params q{};
  q.out_features = d->out_features; q.in_features = d->in_features;
  q.v = d->v; q.k = d->k; q.bits = index_bits(d->k);
  q.k_res = d->k_res; q.bits_res = d->k_res ? index_bits(d->k_res) : 0;
  q.n_out = d->n_outlier_cols;
  q.v_out = q.n_out ? d->v_out : 1; q.k_out = q.n_out ? d->k_out : 0; q.bits_out = q.n_out ? index_bits(d->k_out) : 0;
  q.orientation = orientation;
  if (orientation == 0) {
    q.P = (d->in_features - q.n_out + d->v - 1) / d->v;
    q.Q = q.n_out ? q.n_out / d->v_out : 0;
    q.S = d->out_features; q.S_out = q.n_out ? d->out_features : 0;
  } else {
    q.P = d->in_features - q.n_out;
    q.Q = q.n_out;
    q.S = (d->out_features + d->v - 1) / d->v; q.S_out = q.n_out ? (d->out_features + d->v_out - 1) / d->v_out : 0;
  }
  q.Pg = group_vectors > 0 && group_vectors < q.P ? group_vectors : q.P;
  q.n_groups = (q.P + q.Pg - 1) / q.Pg;
  if (!d->codebook) return VQ_ERR_NULL;
  if (!aligned(d->codebook, 16)) return VQ_ERR_ALIGNMENT;
  int rc = check_stream(d->idx, d->idx_row_stride, q.P, q.bits);
  if (rc != VQ_OK) return rc;
  if (q.k_res) {
    if (!d->codebook_res) return VQ_ERR_NULL;
    if (!aligned(d->codebook_res, 16)) return VQ_ERR_ALIGNMENT;
    rc = check_stream(d->idx_res, d->idx_res_row_stride, q.P, q.bits_res);
    if (rc != VQ_OK) return rc;
  }
  if (q.n_out) {
    if (!d->codebook_out) return VQ_ERR_NULL;
    if (!aligned(d->codebook_out, 16)) return VQ_ERR_ALIGNMENT;
    rc = check_stream(d->idx_out, d->idx_out_row_stride, q.Q, q.bits_out);
    if (rc != VQ_OK) return rc;
  }
  if ((d->scale && !aligned(d->scale, 2)) || (d->bias && !aligned(d->bias, 2))) return VQ_ERR_ALIGNMENT;
  q.cb = static_cast<const __half *>(d->codebook);
  q.cb_res = q.k_res ? static_cast<const __half *>(d->codebook_res) : nullptr;
  q.cb_out = q.n_out ? static_cast<const __half *>(d->codebook_out) : nullptr;
  q.idx = static_cast<const uint8_t *>(d->idx); q.stride = d->idx_row_stride;
  q.idx_res = q.k_res ? static_cast<const uint8_t *>(d->idx_res) : nullptr; q.stride_res = q.k_res ? d->idx_res_row_stride : 0;
  q.idx_out = q.n_out ? static_cast<const uint8_t *>(d->idx_out) : nullptr; q.stride_out = q.n_out ? d->idx_out_row_stride : 0;
  q.scale = static_cast<const __half *>(d->scale);
  q.bias = static_cast<const __half *>(d->bias);
  q.perm = col_perm;
  if (p) *p = q;
  return VQ_OK;
}

}  // namespace vq

using vq::aligned;

extern "C" int vq_validate(const vq_layer_desc *desc) { return vq::make_params(desc, nullptr); }

extern "C" int vq_dequant(const vq_layer_desc *desc, void *W, int64_t ldw, void *hip_stream) {
  vq::read_switches();
  vq::Params p;
  int rc = vq::make_params(desc, &p);
  if (rc != VQ_OK) return rc;
  if (!W) return VQ_ERR_NULL;
  if (ldw < p.in_features) return VQ_ERR_SHAPE;
  if (!aligned(W, 2)) return VQ_ERR_ALIGNMENT;
  return vq::launch_dequant(p, static_cast<__half *>(W), ldw, static_cast<hipStream_t>(hip_stream));
}

extern "C" int vq_gemv(const vq_layer_desc *desc, const void *x, int64_t ldx, int32_t batch,
                       void *y, int64_t ldy, void *hip_stream) {
  vq::read_switches();
  vq::Params p;
  int rc = vq::make_params(desc, &p);
  if (rc != VQ_OK) return rc;
  if (!x || !y) return VQ_ERR_NULL;
  if (batch < 1 || batch > 16 || ldx < p.in_features || ldy < p.out_features) return VQ_ERR_SHAPE;
  if (!aligned(x, 2) || !aligned(y, 2)) return VQ_ERR_ALIGNMENT;
  return vq::launch_gemv(p, static_cast<const __half *>(x), ldx, batch, static_cast<__half *>(y), ldy,
                         static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t vq_gemv_workspace_bytes(const vq_layer_desc *desc, int32_t batch) {
  vq::read_switches();
  vq::Params p;
  if (vq::make_params(desc, &p) != VQ_OK || batch < 1 || batch > 16) return 0;
  // the size does not depend on x; the fast kernels' conditions on x are checked again at the call
  return vq::gemv_workspace_bytes(p, nullptr, p.in_features + (p.in_features & 1), batch);
}

extern "C" size_t vq_lend_gemv_bytes(const vq_layer_desc *desc, int32_t batch) {
  vq::read_switches();
  vq::Params p;
  if (vq::make_params(desc, &p) != VQ_OK || batch < 1 || batch > 16) return 0;
  const bool plain = desc->group_vectors || (p.v == 6 && p.k > 2048 && !p.perm), odd = p.v == 6 && (p.in_features & 1);
  return plain && !odd ? 0 : vq::gemv_lent_bytes(p, batch);
}

extern "C" int vq_gemv_with_workspace(const vq_layer_desc *desc, const void *x, int64_t ldx, int32_t batch, void *y, int64_t ldy,
                                      void *workspace, size_t workspace_bytes, void *hip_stream) {
  vq::read_switches();
  vq::Params p;
  int rc = vq::make_params(desc, &p);
  if (rc != VQ_OK) return rc;
  if (!x || !y) return VQ_ERR_NULL;
  if (batch < 1 || batch > 16 || ldx < p.in_features || ldy < p.out_features) return VQ_ERR_SHAPE;
  if (!aligned(x, 2) || !aligned(y, 2)) return VQ_ERR_ALIGNMENT;
  if (workspace && workspace_bytes && !aligned(workspace, 256)) return VQ_ERR_ALIGNMENT;
  return vq::launch_gemv_ws(p, static_cast<const __half *>(x), ldx, batch, static_cast<__half *>(y), ldy, workspace, workspace_bytes,
                            static_cast<hipStream_t>(hip_stream));
}

// ---- vq_gemv_with_workspace for callers that cannot allocate: the workspace is a device array of this library.
// In host code the array's name is only a handle for hipGetSymbolAddress; what kernels and the launchers get is the
// device address that call returns, looked up once per device (every device holds its own copy of the array).
namespace vq {
static __device__ __align__(256) unsigned char scratch[VQ_GEMV_STATIC_WORKSPACE_BYTES];
namespace {
constexpr int MAX_DEVICES = 64;
void *g_scratch_ptr[MAX_DEVICES];
std::mutex g_scratch_mutex;

int static_workspace(void **ptr) {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return VQ_ERR_HIP;
  std::lock_guard<std::mutex> lock(g_scratch_mutex);
  if (!g_scratch_ptr[dev]) {
    void *q = nullptr;
    if (hipGetSymbolAddress(&q, HIP_SYMBOL(scratch)) != hipSuccess || !q) return VQ_ERR_HIP;
    g_scratch_ptr[dev] = q;
  }
  *ptr = g_scratch_ptr[dev];
  return VQ_OK;
}
}  // namespace
}  // namespace vq

extern "C" int vq_gemv_static_workspace(const vq_layer_desc *desc, const void *x, int64_t ldx, int32_t batch, void *y, int64_t ldy,
                                        void *hip_stream) {
  vq::read_switches();
  vq::Params p;
  int rc = vq::make_params(desc, &p);
  if (rc != VQ_OK) return rc;
  if (!x || !y) return VQ_ERR_NULL;
  if (batch < 1 || batch > 16 || ldx < p.in_features || ldy < p.out_features) return VQ_ERR_SHAPE;
  if (!aligned(x, 2) || !aligned(y, 2)) return VQ_ERR_ALIGNMENT;
  const size_t need = vq::gemv_workspace_bytes(p, static_cast<const __half *>(x), ldx, batch);
  if (need > (size_t)VQ_GEMV_STATIC_WORKSPACE_BYTES) return VQ_ERR_WORKSPACE;
  void *ws = nullptr;
  if (need) {
    rc = vq::static_workspace(&ws);
    if (rc != VQ_OK) return rc;
  }
  return vq::launch_gemv_ws(p, static_cast<const __half *>(x), ldx, batch, static_cast<__half *>(y), ldy, ws,
                            ws ? (size_t)VQ_GEMV_STATIC_WORKSPACE_BYTES : 0, static_cast<hipStream_t>(hip_stream));
}

extern "C" int vq_gemv_multi(const vq_layer_desc *const *descs, int32_t n_layers, const void *x, int64_t ldx, int32_t batch,
                             void *const *y, const int64_t *ldy, void *hip_stream) {
  vq::read_switches();
  constexpr int MAX_LAYERS = 8;
  if (!descs || !y || !ldy || !x) return VQ_ERR_NULL;
  if (n_layers < 1 || n_layers > MAX_LAYERS || batch < 1 || batch > 16) return VQ_ERR_SHAPE;
  vq::Params p[MAX_LAYERS];
  __half *ys[MAX_LAYERS];
  long long ldys[MAX_LAYERS];
  for (int i = 0; i < n_layers; ++i) {
    const int rc = vq::make_params(descs[i], &p[i]);
    if (rc != VQ_OK) return rc;
    if (!y[i]) return VQ_ERR_NULL;
    if (p[i].in_features != p[0].in_features || ldx < p[i].in_features || ldy[i] < p[i].out_features) return VQ_ERR_SHAPE;
    if (!aligned(x, 2) || !aligned(y[i], 2)) return VQ_ERR_ALIGNMENT;
    ys[i] = static_cast<__half *>(y[i]); ldys[i] = ldy[i];
  }
  return vq::launch_gemv_multi(p, n_layers, static_cast<const __half *>(x), ldx, batch, ys, ldys, static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t vq_gemm_workspace_bytes(const vq_layer_desc *desc, int32_t tokens) {
  vq::read_switches();
  vq::Params p;
  if (vq::make_params(desc, &p) != VQ_OK || tokens < 1) return 0;
  return vq::gemm_workspace_bytes(p, tokens);
}

extern "C" size_t vq_gemm_fast_workspace_bytes(const vq_layer_desc *desc, int32_t tokens) {
  vq::read_switches();
  vq::Params p;
  if (vq::make_params(desc, &p) != VQ_OK || tokens < 1) return 0;
  return vq::gemm_fast_workspace_bytes(p, tokens);
}

extern "C" size_t vq_gemm_default_workspace_bytes(const vq_layer_desc *desc, int32_t tokens) {
  vq::read_switches();
  vq::Params p;
  if (vq::make_params(desc, &p) != VQ_OK || tokens < 1) return 0;
  return vq::gemm_default_workspace_bytes(p, tokens, true);
}

extern "C" size_t vq_lend_gemm_least_bytes(const vq_layer_desc *desc, int32_t tokens) {
  vq::read_switches();
  vq::Params p;
  if (vq::make_params(desc, &p) != VQ_OK || tokens < 1) return 0;
  return vq::gemm_default_workspace_bytes(p, tokens, false);
}

namespace vq {
namespace {
// vq_gemm and vq_gemm_default: the same arguments, checks and errors
template <typename Launch>
int checked_gemm(const vq_layer_desc *desc, const void *X, int64_t ldx, int32_t tokens, void *Y, int64_t ldy, void *workspace, size_t workspace_bytes,
                 void *hip_stream, Launch launch) {
  read_switches();
  Params p;
  int rc = make_params(desc, &p);
  if (rc != VQ_OK) return rc;
  if (!X || !Y) return VQ_ERR_NULL;
  if (tokens < 1 || tokens > (1 << 24) || ldx < p.in_features || ldy < p.out_features) return VQ_ERR_SHAPE;
  if (!aligned(X, 16) || (ldx & 7) || !aligned(Y, 2)) return VQ_ERR_ALIGNMENT;
  const size_t need = gemm_workspace_bytes(p, tokens);
  if (need && (!workspace || workspace_bytes < need)) return VQ_ERR_WORKSPACE;
  if (workspace && workspace_bytes && !aligned(workspace, 16)) return VQ_ERR_ALIGNMENT;
  return launch(p, static_cast<const __half *>(X), ldx, tokens, static_cast<__half *>(Y), ldy, workspace, workspace_bytes, static_cast<hipStream_t>(hip_stream));
}
}  // namespace
}  // namespace vq

extern "C" int vq_gemm(const vq_layer_desc *desc, const void *X, int64_t ldx, int32_t tokens,
                       void *Y, int64_t ldy, void *workspace, size_t workspace_bytes, void *hip_stream) {
  return vq::checked_gemm(desc, X, ldx, tokens, Y, ldy, workspace, workspace_bytes, hip_stream, vq::launch_gemm);
}

extern "C" int vq_gemm_default(const vq_layer_desc *desc, const void *X, int64_t ldx, int32_t tokens,
                               void *Y, int64_t ldy, void *workspace, size_t workspace_bytes, void *hip_stream) {
  return vq::checked_gemm(desc, X, ldx, tokens, Y, ldy, workspace, workspace_bytes, hip_stream, vq::launch_gemm_default);
}

static int checked_assign(const void *W, const void *B, int64_t ld, int32_t rows, int32_t cols, const void *codebook, int32_t v, int32_t k, void *idx,
                          int64_t idx_row_stride, bool down, bool clear, void *hip_stream) {
  if (!W || !codebook || !idx) return VQ_ERR_NULL;
  const int lim = 1 << 24;
  if (rows < 1 || rows > lim || cols < 1 || cols > lim || ld < cols || v < 1 || v > 16 || k < 2 || k > 65536) return VQ_ERR_SHAPE;
  const long long P = down ? cols : ((long long)cols + v - 1) / v;
  const long long need = ((P * vq::index_bits(k) + 31) / 32) * 4;             // whole dwords
  if (idx_row_stride < need) return VQ_ERR_SHAPE;
  if (!aligned(W, 2) || (B && !aligned(B, 2)) || !aligned(codebook, 2)) return VQ_ERR_ALIGNMENT;
  if (!aligned(idx, 16) || idx_row_stride % 16 != 0) return VQ_ERR_ALIGNMENT;
  return (down ? vq::launch_assign_down : vq::launch_assign)(static_cast<const __half *>(W), static_cast<const __half *>(B), ld, rows, cols,
                                                             static_cast<const __half *>(codebook), v, k, static_cast<unsigned char *>(idx), idx_row_stride,
                                                             clear, static_cast<hipStream_t>(hip_stream));
}

extern "C" int vq_assign(const void *W, const void *B, int64_t ld, int32_t rows, int32_t cols, const void *codebook, int32_t v, int32_t k,
                         void *idx, int64_t idx_row_stride, void *hip_stream) {
  return checked_assign(W, B, ld, rows, cols, codebook, v, k, idx, idx_row_stride, false, false, hip_stream);
}

extern "C" int vq_assign_down(const void *W, const void *B, int64_t ld, int32_t rows, int32_t cols, const void *codebook, int32_t v,
                              int32_t k, void *idx, int64_t idx_row_stride, void *hip_stream) {
  return checked_assign(W, B, ld, rows, cols, codebook, v, k, idx, idx_row_stride, true, false, hip_stream);
}

extern "C" int vq_lend_assign(const void *W, const void *B, int64_t ld, int32_t rows, int32_t cols, const void *codebook, int32_t v, int32_t k,
                              void *idx, int64_t idx_row_stride, int32_t down, void *hip_stream) {
  const long long bits = (down ? (long long)cols : ((long long)cols + v - 1) / std::max(v, 1)) * vq::index_bits(std::max(k, 2));
  if (idx_row_stride > (bits + 127) / 128 * 16) return VQ_ERR_SHAPE;          // (three dwords of padding at most)
  return checked_assign(W, B, ld, rows, cols, codebook, v, k, idx, idx_row_stride, down != 0, true, hip_stream);
}

extern "C" size_t vq_quantize_columns_workspace_bytes(int32_t rows, int32_t v, int32_t k, int32_t k_res) {
  if (rows < 1 || rows > (1 << 24) || v < 1 || v > 16 || k < 2 || k > 65536 || (k_res != 0 && (k_res < 2 || k_res > 65536))) return 0;
  return vq::quantize_columns_workspace_bytes(rows, v, k, k_res);
}

extern "C" int vq_quantize_columns(void *W, int64_t ldw, int32_t rows, int32_t cols, const void *Hinv, int64_t ldh, const void *codebook,
                                   int32_t v, int32_t k, const void *codebook_res, int32_t k_res, int32_t block, void *idx,
                                   int64_t idx_row_stride, void *idx_res, int64_t idx_res_row_stride, void *T, int64_t ldt, void *workspace,
                                   size_t workspace_bytes, void *hip_stream) {
  if (!W || !Hinv || !codebook || !idx) return VQ_ERR_NULL;
  const int lim = 1 << 24;
  if (rows < 1 || rows > lim || cols < 1 || cols > lim || ldw < cols || ldh < cols || v < 1 || v > 16 || k < 2 || k > 65536) return VQ_ERR_SHAPE;
  if (k_res != 0 && (k_res < 2 || k_res > 65536)) return VQ_ERR_SHAPE;
  if (k_res && (!codebook_res || !idx_res)) return VQ_ERR_NULL;
  if (block < 1 || block > 128 || (T && ldt < cols)) return VQ_ERR_SHAPE;
  if (idx_row_stride < (((long long)cols * vq::index_bits(k) + 31) / 32) * 4) return VQ_ERR_SHAPE;
  if (k_res && idx_res_row_stride < (((long long)cols * vq::index_bits(k_res) + 31) / 32) * 4) return VQ_ERR_SHAPE;
  if (!aligned(W, 4) || !aligned(Hinv, 4) || (T && !aligned(T, 4)) || !aligned(codebook, 2) || (k_res && !aligned(codebook_res, 2))) return VQ_ERR_ALIGNMENT;
  if (!aligned(idx, 16) || idx_row_stride % 16 != 0 || (k_res && (!aligned(idx_res, 16) || idx_res_row_stride % 16 != 0))) return VQ_ERR_ALIGNMENT;
  const size_t need = vq::quantize_columns_workspace_bytes(rows, v, k, k_res);
  if (!workspace || workspace_bytes < need) return VQ_ERR_WORKSPACE;
  if (!aligned(workspace, 256)) return VQ_ERR_ALIGNMENT;
  return vq::launch_quantize_columns(static_cast<float *>(W), ldw, rows, cols, static_cast<const float *>(Hinv), ldh,
                                     static_cast<const __half *>(codebook), v, k, static_cast<const __half *>(codebook_res), k_res, block,
                                     static_cast<unsigned char *>(idx), idx_row_stride, static_cast<unsigned char *>(idx_res),
                                     idx_res_row_stride, static_cast<float *>(T), ldt, workspace, static_cast<hipStream_t>(hip_stream));
}

// ---- paged cache, attention, norms ----
namespace vq {

int make_kv_params(const vq_kv_desc *d, KvParams *p) {
  if (!d) return VQ_ERR_NULL;
  if (d->struct_size != sizeof(vq_kv_desc) || d->reserved != 0) return VQ_ERR_SHAPE;
  if (d->type != VQ_KV_FP16 && d->type != VQ_KV_E4M3) return VQ_ERR_SHAPE;
  const bool e4m3 = d->type == VQ_KV_E4M3;
  if (d->kv_heads < 1 || d->kv_heads > 65535 || d->head_dim < 16 || d->head_dim > 256 || d->head_dim % 16 != 0) return VQ_ERR_SHAPE;
  int shift = 4;
  while (shift < 8 && (1 << shift) != d->page_tokens) ++shift;
  if ((1 << shift) != d->page_tokens) return VQ_ERR_SHAPE;
  if (d->n_pages < 1 || d->n_seqs < 1 || d->n_tokens < 1 || d->n_tokens > 1 << 30 || d->max_new < 1 || d->max_new > d->n_tokens || d->max_length < 0 || d->max_length > 1 << 30) return VQ_ERR_SHAPE;
  if (d->table_pages < 0 || d->max_length > (long long)d->table_pages * d->page_tokens || d->table_stride < d->table_pages) return VQ_ERR_SHAPE;
  if (!d->starts && (d->n_tokens % d->n_seqs != 0 || d->max_new < d->n_tokens / d->n_seqs)) return VQ_ERR_SHAPE;
  if (!d->k_pages || !d->v_pages || !d->lengths || (!d->page_table && d->table_pages) || (e4m3 && (!d->k_scales || !d->v_scales))) return VQ_ERR_NULL;
  const long long page = (long long)d->kv_heads * d->page_tokens * d->head_dim, element = e4m3 ? 1 : 2, most = (1ll << 32) / element - 1;
  if (d->k_page_stride < page || d->v_page_stride < page || d->k_page_stride > most || d->v_page_stride > most) return VQ_ERR_SHAPE;
  if (!aligned(d->k_pages, 16) || !aligned(d->v_pages, 16) || d->k_page_stride * element % 16 || d->v_page_stride * element % 16) return VQ_ERR_ALIGNMENT;
  if (!aligned(d->lengths, 4) || !aligned(d->page_table, 4) || !aligned(d->starts, 4) || (e4m3 && (!aligned(d->k_scales, 4) || !aligned(d->v_scales, 4))))
    return VQ_ERR_ALIGNMENT;
  KvParams q{};
  q.e4m3 = e4m3;
  q.kv_heads = d->kv_heads; q.head_dim = d->head_dim; q.page_shift = shift; q.n_pages = d->n_pages;
  q.n_seqs = d->n_seqs; q.n_tokens = d->n_tokens; q.max_new = d->max_new; q.max_length = d->max_length; q.table_pages = d->table_pages;
  q.each = d->starts ? 0 : d->n_tokens / d->n_seqs;
  q.k_pages = static_cast<unsigned char *>(d->k_pages); q.v_pages = static_cast<unsigned char *>(d->v_pages);
  q.k_page_bytes = d->k_page_stride * element; q.v_page_bytes = d->v_page_stride * element; q.table_stride = d->table_stride;
  q.k_scales = e4m3 ? d->k_scales : nullptr; q.v_scales = e4m3 ? d->v_scales : nullptr;
  q.page_table = d->page_table; q.lengths = d->lengths; q.starts = d->starts;
  if (p) *p = q;
  return VQ_OK;
}

// Query heads, window and first tokens of a call of vq_attention.
static int make_attention_params(const KvParams &c, int32_t q_heads, int32_t window, int32_t sinks, AttentionParams *a) {
  if (q_heads < 1 || q_heads > 65535 || q_heads % c.kv_heads != 0 || window < 0 || sinks < 0) return VQ_ERR_SHAPE;
  *a = AttentionParams{};
  a->q_heads = q_heads; a->group = q_heads / c.kv_heads;
  a->by_group = a->group > 1 ? (unsigned)((1ull << 32) / a->group) + 1 : 0;
  if ((long long)c.max_new * a->group * a->group >= 1ll << 30) return VQ_ERR_SHAPE;          // (by_group is good for so many rows and more)
  constexpr int32_t most = 1 << 30;                                                          // (as long as any sequence, and places less it are numbers of 32 bits)
  a->window = window < most ? window : most; a->sinks = window ? (sinks < most ? sinks : most) : 0;
  return VQ_OK;
}

// The prefixes of a call; what they bound is cut to what the call can have.
static int make_prefixes(const vq_prefix_desc *d, const KvParams &c, Prefixes *x) {
  if (!d) return VQ_ERR_NULL;
  if (d->struct_size != sizeof(vq_prefix_desc) || d->n_prefixes < 1 || d->n_prefixes > 65535 || d->max_members < 1 || d->max_length < 0 || d->max_length > 1 << 30 || d->max_own < 0)
    return VQ_ERR_SHAPE;
  if (d->table_pages < 0 || d->max_length > ((long long)d->table_pages << c.page_shift) || d->table_stride < d->table_pages) return VQ_ERR_SHAPE;
  if (!d->members && d->n_prefixes != 1) return VQ_ERR_SHAPE;
  if (!d->lengths || (!d->page_table && d->table_pages)) return VQ_ERR_NULL;
  if (!aligned(d->lengths, 4) || !aligned(d->page_table, 4) || !aligned(d->members, 4)) return VQ_ERR_ALIGNMENT;
  *x = Prefixes{};
  x->n = d->n_prefixes; x->most = std::min(d->max_members, c.n_seqs); x->max_length = std::min(d->max_length, c.max_length); x->max_own = std::min(d->max_own, c.max_length);
  x->n_seqs = c.n_seqs; x->table_pages = d->table_pages; x->table_stride = d->table_stride;
  x->rows_most = (int)std::min<long long>((long long)x->most * c.max_new, c.n_tokens);
  x->partial_tokens = std::min((long long)x->n * x->rows_most, (long long)c.n_tokens);
  x->by_token = (long long)x->n * x->rows_most > c.n_tokens;
  x->page_table = d->page_table; x->lengths = d->lengths; x->members = d->members;
  return VQ_OK;
}

}  // namespace vq

extern "C" int vq_kv_append(const vq_kv_desc *cache, const void *k, int64_t ldk, const void *v, int64_t ldv, const void *q, int64_t ldq,
                            int32_t q_heads, void *q_out, int64_t ldq_out, const vq_rotary *rotary, void *hip_stream) {
  vq::KvParams c;
  const int rc = vq::make_kv_params(cache, &c);
  if (rc != VQ_OK) return rc;
  if (!k || !v || (q && !q_out)) return VQ_ERR_NULL;
  const long long kv_width = (long long)c.kv_heads * c.head_dim;
  if (ldk < kv_width || ldv < kv_width) return VQ_ERR_SHAPE;
  if (q && (q_heads < 1 || q_heads > 65535 || ldq < (long long)q_heads * c.head_dim || ldq_out < (long long)q_heads * c.head_dim)) return VQ_ERR_SHAPE;
  if (!aligned(k, 2) || !aligned(v, 2) || (q && (!aligned(q, 2) || !aligned(q_out, 2)))) return VQ_ERR_ALIGNMENT;
  vq::Rotary r{};
  if (rotary) {
    if (!rotary->cos || !rotary->sin) return VQ_ERR_NULL;
    if (rotary->positions < 1 || rotary->rotary_dim < 2 || rotary->rotary_dim % 2 != 0 || rotary->rotary_dim > c.head_dim || rotary->ld < rotary->rotary_dim / 2)
      return VQ_ERR_SHAPE;
    if (!aligned(rotary->cos, 4) || !aligned(rotary->sin, 4) || !aligned(rotary->position, 4)) return VQ_ERR_ALIGNMENT;
    r = vq::Rotary{rotary->cos, rotary->sin, rotary->ld, rotary->positions, rotary->rotary_dim, rotary->interleaved != 0, rotary->position};
  }
  return vq::launch_kv_append(c, static_cast<const __half *>(k), ldk, static_cast<const __half *>(v), ldv, static_cast<const __half *>(q), ldq,
                              q ? q_heads : 0, static_cast<__half *>(q_out), ldq_out, r, static_cast<hipStream_t>(hip_stream));
}

static int checked_attention(const vq::KvParams &c, const void *q, int64_t ldq, int32_t q_heads, float softmax_scale, int32_t window, int32_t sinks, void *out, int64_t ldo,
                             float *lse, void *workspace, vq::AttentionParams *a) {
  if (!q || !out) return VQ_ERR_NULL;
  const int rc = vq::make_attention_params(c, q_heads, window, sinks, a);
  if (rc != VQ_OK) return rc;
  const long long width = (long long)q_heads * c.head_dim;
  if (ldq < width || ldo < width || !(softmax_scale > 0.f && softmax_scale <= 1e30f)) return VQ_ERR_SHAPE;
  if (!aligned(q, 2) || !aligned(out, 2) || !aligned(lse, 4) || !aligned(workspace, 256)) return VQ_ERR_ALIGNMENT;
  a->q = static_cast<const __half *>(q); a->ldq = ldq;
  a->out = static_cast<__half *>(out); a->ldo = ldo;
  a->lse = lse;
  a->scale = softmax_scale * 1.4426950408889634f;
  return VQ_OK;
}

extern "C" size_t vq_attention_workspace_bytes(const vq_kv_desc *cache, int32_t q_heads, int32_t window, int32_t sinks) {
  vq::read_switches();
  vq::KvParams c;
  vq::AttentionParams a;
  if (vq::make_kv_params(cache, &c) != VQ_OK || vq::make_attention_params(c, q_heads, window, sinks, &a) != VQ_OK) return 0;
  return vq::attention_workspace_bytes(c, a);
}

extern "C" int vq_attention(const vq_kv_desc *cache, const void *q, int64_t ldq, int32_t q_heads, float softmax_scale, int32_t window, int32_t sinks,
                            void *out, int64_t ldo, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  vq::read_switches();
  vq::KvParams c;
  vq::AttentionParams a;
  int rc = vq::make_kv_params(cache, &c);
  if (rc != VQ_OK) return rc;
  if ((rc = checked_attention(c, q, ldq, q_heads, softmax_scale, window, sinks, out, ldo, lse, workspace, &a)) != VQ_OK) return rc;
  return vq::launch_attention(c, a, workspace, workspace ? workspace_bytes : 0, static_cast<hipStream_t>(hip_stream));
}

extern "C" size_t vq_attention_shared_workspace_bytes(const vq_kv_desc *cache, const vq_prefix_desc *prefix, int32_t q_heads) {
  vq::read_switches();
  vq::KvParams c;
  vq::Prefixes x;
  vq::AttentionParams a;
  if (vq::make_kv_params(cache, &c) != VQ_OK || vq::make_prefixes(prefix, c, &x) != VQ_OK || vq::make_attention_params(c, q_heads, 0, 0, &a) != VQ_OK) return 0;
  return vq::attention_shared_workspace_bytes(c, x, a);
}

extern "C" int vq_attention_shared(const vq_kv_desc *cache, const vq_prefix_desc *prefix, const void *q, int64_t ldq, int32_t q_heads, float softmax_scale, void *out,
                                   int64_t ldo, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  vq::read_switches();
  vq::KvParams c;
  vq::Prefixes x;
  vq::AttentionParams a;
  int rc = vq::make_kv_params(cache, &c);
  if (rc != VQ_OK || (rc = vq::make_prefixes(prefix, c, &x)) != VQ_OK) return rc;
  if ((rc = checked_attention(c, q, ldq, q_heads, softmax_scale, 0, 0, out, ldo, lse, workspace, &a)) != VQ_OK) return rc;
  return vq::launch_attention_shared(c, x, a, workspace, workspace ? workspace_bytes : 0, static_cast<hipStream_t>(hip_stream));
}

extern "C" int vq_embed(const int32_t *ids, int32_t rows, const void *table, int64_t ld, int32_t vocabulary, int32_t width, float scale, int32_t stream32, void *y,
                        int64_t ldy, void *hip_stream) {
  if (!ids || !table || !y) return VQ_ERR_NULL;
  const int lim = 1 << 24;
  if (rows < 1 || vocabulary < 1 || vocabulary > lim || width < 1 || width > lim || ld < width || ldy < width || !(scale >= -FLT_MAX && scale <= FLT_MAX)) return VQ_ERR_SHAPE;
  if (!aligned(ids, 4) || !aligned(table, 2) || !aligned(y, stream32 ? 4 : 2)) return VQ_ERR_ALIGNMENT;
  return vq::launch_embed(ids, rows, static_cast<const __half *>(table), ld, vocabulary, width, scale, stream32 != 0, y, ldy, static_cast<hipStream_t>(hip_stream));
}

extern "C" int vq_sample(const void *logits, int64_t ld, int32_t rows, int32_t vocabulary, const float *uniform, const vq_sampling *how, int32_t *tokens, float *probabilities,
                         void *hip_stream) {
  if (!logits || !uniform || !how || !tokens) return VQ_ERR_NULL;
  if (how->struct_size != sizeof(vq_sampling) || rows < 1 || vocabulary < 1 || vocabulary > 1 << 24 || ld < vocabulary) return VQ_ERR_SHAPE;
  if (!aligned(logits, 2) || !aligned(uniform, 4) || !aligned(tokens, 4) || !aligned(probabilities, 4) || !aligned(how->temperatures, 4) || !aligned(how->top_ks, 4) ||
      !aligned(how->top_ps, 4) || !aligned(how->min_ps, 4))
    return VQ_ERR_ALIGNMENT;
  const vq::SampleParams p{static_cast<const __half *>(logits), ld, vocabulary, how->top_k, how->temperature, how->top_p, how->min_p, uniform, how->temperatures, how->top_ps,
                           how->min_ps, how->top_ks, tokens, probabilities};
  return vq::launch_sample(p, rows, static_cast<hipStream_t>(hip_stream));
}

extern "C" int vq_residual_norm(const void *h, int64_t ldh, const void *x, int64_t ldx, const void *w_post, const void *gate, int64_t ldgate,
                                float scale, const void *w_pre, float eps, int32_t stream32, int32_t rows, int32_t width, void *y, int64_t ldy,
                                void *z, int64_t ldz, void *hip_stream) {
  if (!x || (!y && !z) || (z && !w_pre) || (!h && (w_post || gate))) return VQ_ERR_NULL;
  if (rows < 1 || width < 1 || width > 32768 || ldx < width || (h && ldh < width) || (y && ldy < width) || (z && ldz < width)) return VQ_ERR_SHAPE;
  if ((gate && ldgate != 0 && ldgate < width) || !(eps >= 0.f)) return VQ_ERR_SHAPE;
  const uintptr_t stream = stream32 ? 4 : 2;
  if (!aligned(x, stream) || !aligned(y, stream) || !aligned(h, 2) || !aligned(z, 2) || !aligned(w_post, 2) || !aligned(gate, 2) || !aligned(w_pre, 2))
    return VQ_ERR_ALIGNMENT;
  return vq::launch_residual_norm(static_cast<const __half *>(h), ldh, x, ldx, static_cast<const __half *>(w_post), static_cast<const __half *>(gate), ldgate,
                                  scale, static_cast<const __half *>(w_pre), eps, stream32 != 0, rows, width, y, ldy, static_cast<__half *>(z), ldz,
                                  static_cast<hipStream_t>(hip_stream));
}

extern "C" const char *vq_status_string(int status) {
  switch (status) {
    case VQ_OK: return "ok";
    case VQ_ERR_NULL: return "a required pointer is NULL";
    case VQ_ERR_SHAPE: return "size, stride or leading dimension out of range";
    case VQ_ERR_ALIGNMENT: return "pointer or stride misaligned";
    case VQ_ERR_UNSUPPORTED: return "no kernel handles this layer";
    case VQ_ERR_HIP: return "HIP launch error";
    case VQ_ERR_WORKSPACE: return "workspace missing or too small";
    default: return "unknown status";
  }
}

extern "C" int vq_version(void) { return 100; }

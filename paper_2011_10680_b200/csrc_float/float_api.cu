// C ABI of the operators on floating-point activations: argument checks and the choice of kernel.  Host code only.
#include <mutex>

#include <cuda.h>

#include "float_internal.cuh"

namespace {

constexpr long long kMaxExtent = 1ll << 30;     // 32-bit indexes of a tile or a group may reach past the last row or column

CUresult (*g_current_context)(CUcontext*) = nullptr;
CUresult (*g_set_context)(CUcontext) = nullptr;

// The context of the handle's device for the duration of a call, then again whatever the thread had: the context of another device, one
// that the program has made itself (a stream and memory of this handle are nothing to it, although the device may be the
// same), or none.
class ContextScope {
 public:
  explicit ContextScope(const hq_handle* h) {
    const CUcontext wanted = (CUcontext)h->context;
    ok_ = g_current_context && g_current_context(&before_) == CUDA_SUCCESS && (before_ == wanted || g_set_context(wanted) == CUDA_SUCCESS);
    changed_ = ok_ && before_ != wanted;
  }
  ~ContextScope() { if (changed_) g_set_context(before_); }
  ContextScope(const ContextScope&) = delete;
  ContextScope& operator=(const ContextScope&) = delete;
  bool ok() const { return ok_; }

 private:
  CUcontext before_ = nullptr;
  bool ok_ = false, changed_ = false;
};

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

hq_status check_matrix(const hq_matrix* m, bool f32) {
  if (!m) return HQ_ERR_INVALID_ARG;
  if (!(m->type == HQ_F16 || m->type == HQ_BF16 || (m->type == HQ_F32 && f32))) return HQ_ERR_INVALID_ARG;
  if (m->rows < 0 || m->cols < 1 || m->row_stride < m->cols) return HQ_ERR_INVALID_ARG;
  if (m->rows > kMaxExtent || m->cols > kMaxExtent || m->row_stride > (1ll << 40)) return HQ_ERR_UNSUPPORTED;
  if (m->rows > 0 && !m->data) return HQ_ERR_INVALID_ARG;
  return aligned(m->data, 16) ? HQ_OK : HQ_ERR_ALIGNMENT;
}
inline bool same_shape(const hq_matrix* a, const hq_matrix* b) { return a->rows == b->rows && a->cols == b->cols && a->type == b->type; }

hq_status check_w4(const hq_w4* w) {
  if (!w || !w->q || !w->scale) return HQ_ERR_INVALID_ARG;
  if (w->n < 1 || w->k < 2 || (w->k & 1) || w->group < 32 || w->group % 32) return HQ_ERR_INVALID_ARG;
  if (w->n > kMaxExtent || w->k > kMaxExtent) return HQ_ERR_UNSUPPORTED;
  return aligned(w->q, 16) && aligned(w->scale, 16) ? HQ_OK : HQ_ERR_ALIGNMENT;
}

hq_status check_saved(const hq_saved8* s, long long rows, long long cols) {
  if (!s || s->rows != rows || s->cols != cols) return HQ_ERR_INVALID_ARG;
  if (!(s->group == 32 || s->group == 64 || s->group == 128 || s->group == 256)) return HQ_ERR_INVALID_ARG;
  if (rows > 0 && (!s->q || !s->scale)) return HQ_ERR_INVALID_ARG;
  return aligned(s->q, 16) && aligned(s->scale, 16) ? HQ_OK : HQ_ERR_ALIGNMENT;
}

// A launch that failed leaves no error behind for the caller's next CUDA call.
inline hq_status launched(cudaError_t e) {
  if (e == cudaSuccess) return HQ_OK;
  cudaGetLastError();
  return HQ_ERR_CUDA;
}
inline hq_status launched(hq_status st) {
  if (st == HQ_ERR_CUDA) cudaGetLastError();
  return st;
}

inline int groups_of(long long cols, int group) { return (int)((cols + group - 1) / group); }

hq_status product(hq_handle* h, ProductKind kind, int type, const ProductArgs& a, void* stream) {
  const ContextScope context(h);
  if (!context.ok()) return HQ_ERR_CUDA;
  if (kind == PRODUCT_FORWARD && hq_product_few_supported(a, h->sm_count)) return launched(hq_launch_product_few(h, type, a, (cudaStream_t)stream));
  if (hq_product_tc_supported(kind, a)) {
    const hq_status st = launched(hq_launch_product_tc(h, kind, type, a, (cudaStream_t)stream));
    if (st != HQ_ERR_UNSUPPORTED) return st;
  }
  return launched(hq_launch_product_any(kind, type, a, (cudaStream_t)stream));
}

// What hq_act_save8 and hq_act_backward8 share.
hq_status act_args(const hq_handle* h, const hq_matrix* shape, const hq_saved8* saved_x, const hq_saved8* saved_gate, int32_t act, ActArgs& a) {
  if (act < HQ_ACT_NONE || act > HQ_ACT_SILU) return HQ_ERR_INVALID_ARG;
  hq_status st = check_saved(saved_x, shape->rows, shape->cols);
  if (st != HQ_OK) return st;
  if (saved_gate) {
    st = check_saved(saved_gate, shape->rows, shape->cols);
    if (st != HQ_OK) return st;
    if (saved_gate->group != saved_x->group) return HQ_ERR_INVALID_ARG;
    a.gq = saved_gate->q; a.gs = saved_gate->scale;
  }
  a.xq = saved_x->q; a.xs = saved_x->scale;
  a.rows = shape->rows; a.cols = (int32_t)shape->cols; a.group = saved_x->group; a.groups = groups_of(shape->cols, saved_x->group);
  a.act = act; a.sm_count = h->sm_count;
  return HQ_OK;
}

}  // namespace

// From hq_create, with the handle's device current.
bool hq_float_init(hq_handle* h) {
  static std::mutex lock;
  const std::lock_guard<std::mutex> held(lock);
  void *get = nullptr, *set = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPoint("cuCtxGetCurrent", &get, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess ||
      cudaGetDriverEntryPoint("cuCtxSetCurrent", &set, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return false;
  if (!g_current_context) {
    g_set_context = (CUresult (*)(CUcontext))set;
    g_current_context = (CUresult (*)(CUcontext*))get;
  }
  CUcontext context = nullptr;
  if (g_current_context(&context) != CUDA_SUCCESS || !context) return false;
  h->context = context;
  return true;
}

extern "C" {

hq_status hq_linear_w4(hq_handle* h, const hq_matrix* x, const hq_w4* w, const void* bias, hq_matrix* out, void* stream) {
  if (!h) return HQ_ERR_INVALID_ARG;
  hq_status st = check_w4(w);
  if (st == HQ_OK) st = check_matrix(x, false);
  if (st == HQ_OK) st = check_matrix(out, false);
  if (st != HQ_OK) return st;
  if (x->type != out->type || x->rows != out->rows || x->cols != w->k || out->cols != w->n) return HQ_ERR_INVALID_ARG;
  if (!aligned(bias, 2)) return HQ_ERR_ALIGNMENT;
  if (x->rows == 0) return HQ_OK;
  ProductArgs a{};
  a.q = w->q; a.scale = w->scale; a.q_cols = w->k; a.groups = groups_of(w->k, w->group); a.group = w->group;
  a.b = x->data; a.b_stride = x->row_stride; a.bias = bias; a.out = out->data; a.out_stride = out->row_stride;
  a.i = w->n; a.j = (int32_t)x->rows; a.r = w->k;
  return product(h, PRODUCT_FORWARD, x->type, a, stream);
}

hq_status hq_linear_w4_dgrad(hq_handle* h, const hq_matrix* dy, const hq_w4* w, hq_matrix* dx, void* stream) {
  if (!h) return HQ_ERR_INVALID_ARG;
  hq_status st = check_w4(w);
  if (st == HQ_OK) st = check_matrix(dy, false);
  if (st == HQ_OK) st = check_matrix(dx, false);
  if (st != HQ_OK) return st;
  if (dy->type != dx->type || dy->rows != dx->rows || dy->cols != w->n || dx->cols != w->k) return HQ_ERR_INVALID_ARG;
  if (dy->rows == 0) return HQ_OK;
  ProductArgs a{};
  a.q = w->q; a.scale = w->scale; a.q_cols = w->k; a.groups = groups_of(w->k, w->group); a.group = w->group;
  a.b = dy->data; a.b_stride = dy->row_stride; a.out = dx->data; a.out_stride = dx->row_stride;
  a.i = w->k; a.j = (int32_t)dy->rows; a.r = w->n;
  return product(h, PRODUCT_DGRAD, dy->type, a, stream);
}

hq_status hq_linear_wgrad8(hq_handle* h, const hq_matrix* dy, const hq_saved8* saved, hq_matrix* dw, void* stream) {
  if (!h) return HQ_ERR_INVALID_ARG;
  hq_status st = check_matrix(dy, false);
  if (st == HQ_OK) st = check_matrix(dw, false);
  if (st == HQ_OK) st = check_saved(saved, dy->rows, dw->cols);
  if (st != HQ_OK) return st;
  if (dw->type != dy->type || dw->rows != dy->cols) return HQ_ERR_INVALID_ARG;
  ProductArgs a{};
  a.q = saved->q; a.scale = saved->scale; a.q_cols = (int32_t)saved->cols; a.groups = groups_of(saved->cols, saved->group); a.group = saved->group;
  a.b = dy->data; a.b_stride = dy->row_stride; a.out = dw->data; a.out_stride = dw->row_stride;
  a.i = (int32_t)dw->cols; a.j = (int32_t)dw->rows; a.r = (int32_t)dy->rows;
  return product(h, PRODUCT_WGRAD, dy->type, a, stream);
}

hq_status hq_linear_plan(int32_t product, int32_t m, int32_t n, int32_t k, int32_t group, int32_t sm_count, hq_product_plan* plan) {
  if (product < HQ_PRODUCT_LINEAR || product > HQ_PRODUCT_WGRAD || m < 1 || n < 1 || k < 1 || sm_count < 1 || !plan) return HQ_ERR_INVALID_ARG;
  if (product != HQ_PRODUCT_WGRAD && (k & 1)) return HQ_ERR_INVALID_ARG;
  if (group < 32 || group % 32) return HQ_ERR_INVALID_ARG;
  if (m > kMaxExtent || n > kMaxExtent || k > kMaxExtent) return HQ_ERR_UNSUPPORTED;
  ProductArgs a{};
  a.q_cols = k; a.groups = groups_of(k, group); a.group = group;
  a.i = product == HQ_PRODUCT_LINEAR ? n : k; a.j = product == HQ_PRODUCT_WGRAD ? n : m;
  a.r = product == HQ_PRODUCT_LINEAR ? k : product == HQ_PRODUCT_DGRAD ? n : m;
  a.b_stride = product == HQ_PRODUCT_LINEAR ? k : n;
  *plan = hq_product_plan{};
  if (product == HQ_PRODUCT_LINEAR && hq_plan_product_few(a, sm_count, plan)) plan->kernel = HQ_KERNEL_FEW_ROWS;
  else if (hq_plan_product_tc((ProductKind)product, a, sm_count, plan)) plan->kernel = HQ_KERNEL_TENSOR_MEMORY;
  else plan->kernel = HQ_KERNEL_CUDA_CORES;
  return HQ_OK;
}

hq_status hq_act_save8(hq_handle* h, const hq_matrix* x, const hq_matrix* gate, int32_t act, hq_matrix* y,
                       hq_saved8* saved_x, hq_saved8* saved_gate, void* stream) {
  if (!h || !saved_x || (gate != nullptr) != (saved_gate != nullptr)) return HQ_ERR_INVALID_ARG;
  hq_status st = check_matrix(x, true);
  if (st == HQ_OK && gate) st = check_matrix(gate, true);
  if (st == HQ_OK && y) st = check_matrix(y, true);
  if (st != HQ_OK) return st;
  if ((gate && !same_shape(x, gate)) || (y && !same_shape(x, y))) return HQ_ERR_INVALID_ARG;
  ActArgs a{};
  st = act_args(h, x, saved_x, saved_gate, act, a);
  if (st != HQ_OK || x->rows == 0) return st;
  a.x = x->data; a.x_stride = x->row_stride;
  if (gate) { a.gate = gate->data; a.gate_stride = gate->row_stride; }
  if (y) { a.y = y->data; a.y_stride = y->row_stride; }
  const ContextScope context(h);
  if (!context.ok()) return HQ_ERR_CUDA;
  return launched(hq_launch_act_save8(x->type, a, (cudaStream_t)stream));
}

hq_status hq_act_backward8(hq_handle* h, const hq_matrix* dy, const hq_saved8* saved_x, const hq_saved8* saved_gate, int32_t act,
                           hq_matrix* dx, hq_matrix* dgate, void* stream) {
  if (!h || !saved_x || !dx || (dgate != nullptr) != (saved_gate != nullptr)) return HQ_ERR_INVALID_ARG;
  hq_status st = check_matrix(dy, true);
  if (st == HQ_OK) st = check_matrix(dx, true);
  if (st == HQ_OK && dgate) st = check_matrix(dgate, true);
  if (st != HQ_OK) return st;
  if (!same_shape(dy, dx) || (dgate && !same_shape(dy, dgate))) return HQ_ERR_INVALID_ARG;
  ActArgs a{};
  st = act_args(h, dy, saved_x, saved_gate, act, a);
  if (st != HQ_OK || dy->rows == 0) return st;
  a.x = dy->data; a.x_stride = dy->row_stride; a.y = dx->data; a.y_stride = dx->row_stride;
  if (dgate) { a.dgate = dgate->data; a.dgate_stride = dgate->row_stride; }
  const ContextScope context(h);
  if (!context.ok()) return HQ_ERR_CUDA;
  return launched(hq_launch_act_backward8(dy->type, a, (cudaStream_t)stream));
}

}  // extern "C"

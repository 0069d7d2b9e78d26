// C-ABI of the softmax operators: handle, argument checks, workspace.
#include <cmath>
#include <new>
#include <string>

#include "softmax.h"

using namespace esspt;

namespace {

struct Carve {
  size_t status, q, self, scores, part, stat, dh;
  size_t words, act, pos, units_h, units_w, scale_h, scale_w, row_max, row_sum, score, col, col_top, col_m, col_f, item_top, slot_stat, out, key[2], val[2], again, tile_first, run_sum[2], sort;
  size_t sort_bytes, total;
};

}  // namespace

struct esspt_softmax {
  esspt_softmax_config cfg{};
  cudaStream_t st = nullptr;
  char* base = nullptr;
  Carve k{};
  cudaStream_t side = nullptr;
  cudaEvent_t fork = nullptr, join = nullptr;
  int sms = 0;
  char err[256] = "";
};

namespace {

thread_local char g_create_err[256] = "";

esspt_status fail(esspt_softmax* sm, esspt_status code, const char* msg) {
  snprintf(sm ? sm->err : g_create_err, 256, "%s", msg);
  return code;
}
esspt_status cuda_fail(esspt_softmax* sm, cudaError_t e, const char* where) {
  snprintf(sm ? sm->err : g_create_err, 256, "%s: %s", where, cudaGetErrorString(e));
  return ESSPT_ECUDA;
}

void release(esspt_softmax* sm) {
  if (sm->fork) cudaEventDestroy(sm->fork);
  if (sm->join) cudaEventDestroy(sm->join);
  if (sm->side) cudaStreamDestroy(sm->side);
  delete sm;
}

#define SOFTMAX_CUDA(sm, call)                                   \
  do {                                                           \
    cudaError_t e_ = (call);                                     \
    if (e_ != cudaSuccess) return cuda_fail((sm), e_, #call);    \
  } while (0)

const char* config_fault(const esspt_softmax_config* c) {
  if (!c) return "null config";
  if (c->max_rows < 1 || c->max_rows > (1 << 20)) return "max_rows must be in [1, 2^20]";
  if (c->n_items < 1 || c->n_items > (1 << 30)) return "n_items must be in [1, 2^30]";
  if (c->width < 1 || c->width > 512) return "width must be in [1, 512]";
  if (c->dtype < ESSPT_F32 || c->dtype > ESSPT_F16) return "unknown dtype";
  if (c->max_top < 1 || c->max_rows * c->max_top >= (int64_t)INT32_MAX)
    return "max_top must be >= 1 and max_rows * max_top < 2^31";
  return nullptr;
}


constexpr int kMaxSms = 256;  // what the workspace is sized for
constexpr int kStatusBytes = 256, kDoneAt = 64;  // the status word, and FewScratch::done behind it
static_assert(kDoneAt + kSmallRows / kFewRows * sizeof(uint32_t) <= kStatusBytes, "counters outgrow their place");

Carve carve(const esspt_softmax_config& c) {
  Carve k{};
  size_t o = 0;
  auto take = [&o](size_t bytes) {
    const size_t at = o;
    o += (bytes + 255) & ~size_t(255);
    return at;
  };
  const size_t n = (size_t)c.max_rows, V = (size_t)c.n_items, D = (size_t)c.width;
  k.status = take(kStatusBytes);
  k.q = take(n * c.max_top * sizeof(float));
  k.self = take(n * sizeof(float));
  const size_t groups = (size_t)few_groups(c.max_rows, c.n_items, c.width, c.dtype, c.backward != 0);
  const size_t few = groups > (size_t)few_blocks(kMaxSms) ? groups : (size_t)few_blocks(kMaxSms);
  k.scores = take(groups * V * kFewRows * sizeof(float));
  k.part = take(few * kFewRows * sizeof(float2));
  k.stat = take(2 * groups * kFewRows * sizeof(float));
  k.dh = take(c.backward ? few * kFewRows * D * sizeof(float) : 0);
  if (c.max_rows > kFewRows) {
    const ManySizes z = many_sizes(c.max_rows, c.n_items, c.width, c.dtype, c.max_top, c.backward != 0, kMaxSms);
    const size_t back = c.backward ? 1 : 0, entries = back * n * c.max_top * sizeof(uint32_t);
    k.words = take(sizeof(ManyWords));
    k.act = take(n * sizeof(int32_t));
    k.pos = take(n * sizeof(int32_t));
    k.units_h = take(z.units_h);
    k.units_w = take(z.units_w);
    k.scale_h = take(c.dtype == ESSPT_F32 ? (n + 128) * sizeof(RowScale) : 0);
    k.scale_w = take(c.dtype == ESSPT_F32 ? (V + 128) * sizeof(RowScale) : 0);
    k.slot_stat = take(z.stat);
    k.row_max = take(back * n * sizeof(float));
    k.row_sum = take(back * n * sizeof(float));
    k.score = take(entries);
    k.col = take(back * (n + 128) * sizeof(float2));
    for (size_t* p : {&k.col_top, &k.col_m, &k.col_f}) *p = take(back * (n + 128) * sizeof(float));
    k.item_top = take(back * V * sizeof(uint32_t));
    k.out = take(z.out);
    for (int i = 0; i < 2; ++i) k.key[i] = take(entries), k.val[i] = take(entries);
    k.again = take(c.dtype != ESSPT_F32 && c.max_top > 1 ? back * n * c.max_top : 0);
    k.tile_first = take(back * ((V + 127) / 128 + 1) * sizeof(int32_t));
    for (int i = 0; i < 2; ++i) k.run_sum[i] = take(z.run_sum[i]);
    k.sort = take(z.sort);
    k.sort_bytes = z.sort;
  }
  k.total = o;
  return k;
}

esspt_status run(esspt_softmax* sm, const void* h, int64_t h_stride, const void* w, int64_t w_stride,
                 const int32_t* ids, const float* logits, int32_t top, int64_t n, const float* weight, float b,
                 float* loss, float* lse, void* grad_h, void* grad_w) {
  const esspt_softmax_config& c = sm->cfg;
  const size_t size = c.dtype == ESSPT_F32 ? 4 : 2;
  auto off = [](const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; };
  if (n < 0 || n > c.max_rows) return fail(sm, ESSPT_EINVAL, "n must be in [0, max_rows]");
  if (top < 1 || top > c.max_top) return fail(sm, ESSPT_EINVAL, "top must be in [1, max_top]");
  if (!(b > 0.f) || !std::isfinite(b)) return fail(sm, ESSPT_EINVAL, "inv_temperature must be positive and finite");
  if (!w || (n > 0 && (!h || !ids || !loss || !lse))) return fail(sm, ESSPT_EINVAL, "null pointer");
  if (h_stride < c.width || w_stride < c.width) return fail(sm, ESSPT_EINVAL, "a row stride is below the width");
  if (!grad_w != !grad_h && n > 0) return fail(sm, ESSPT_EINVAL, "both gradients or neither");
  if (grad_w && !c.backward) return fail(sm, ESSPT_EINVAL, "the handle was made without backward");
  if (off(h, size) || off(w, size) || off(grad_h, size) || off(grad_w, size) || off(ids, 4) || off(logits, 4) ||
      off(weight, 4) || off(loss, 4) || off(lse, 4))
    return fail(sm, ESSPT_EINVAL, "a pointer is not aligned to its type");
  if (n == 0) {
    if (grad_w) SOFTMAX_CUDA(sm, cudaMemsetAsync(grad_w, 0, (size_t)c.n_items * c.width * size, sm->st));
    return ESSPT_OK;
  }
  const Carve& k = sm->k;
  SoftmaxArgs a{};
  a.h = h, a.w = w, a.h_stride = h_stride, a.w_stride = w_stride, a.n = n;
  a.V = (int32_t)c.n_items, a.D = c.width, a.dtype = c.dtype;
  a.target = TargetArgs{ids, logits, top, n, a.V, b, reinterpret_cast<float*>(sm->base + k.q),
                        reinterpret_cast<float*>(sm->base + k.self), reinterpret_cast<uint32_t*>(sm->base + k.status), nullptr};
  if (c.dtype != ESSPT_F32 && grad_w && logits && top > 1 && top <= kAgainByWarp && n > kFewRows)  // (k.again holds lists)
    a.target.again = reinterpret_cast<uint8_t*>(sm->base + k.again);
  a.weight = weight, a.b = b, a.loss = loss, a.lse = lse, a.grad_h = grad_h, a.grad_w = grad_w;
  a.st = sm->st, a.sms = sm->sms;
  if (logits) SOFTMAX_CUDA(sm, launch_targets(a.target, a.st));
  auto at = [&](size_t offset) { return static_cast<void*>(sm->base + offset); };
  if (few_rows(n, c.n_items, c.width, c.dtype, grad_w != nullptr)) {
    const FewScratch s{static_cast<float*>(at(k.scores)), static_cast<float2*>(at(k.part)),
                       static_cast<float*>(at(k.stat)), static_cast<float*>(at(k.dh)),
                       static_cast<uint32_t*>(at(k.status + kDoneAt))};
    SOFTMAX_CUDA(sm, launch_few_rows(a, s));
    return ESSPT_OK;
  }
  ManyScratch s{};
  s.words = static_cast<ManyWords*>(at(k.words));
  s.act = static_cast<int32_t*>(at(k.act)), s.pos = static_cast<int32_t*>(at(k.pos));
  s.units_h = static_cast<char*>(at(k.units_h)), s.units_w = static_cast<char*>(at(k.units_w));
  s.scale_h = static_cast<RowScale*>(at(k.scale_h)), s.scale_w = static_cast<RowScale*>(at(k.scale_w));
  s.row_max = static_cast<float*>(at(k.row_max)), s.row_sum = static_cast<float*>(at(k.row_sum));
  s.score = static_cast<float*>(at(k.score));
  s.col = static_cast<float*>(at(k.col)), s.col_top = static_cast<float*>(at(k.col_top));
  s.col_m = static_cast<float*>(at(k.col_m)), s.col_f = static_cast<float*>(at(k.col_f));
  s.item_top = static_cast<uint32_t*>(at(k.item_top)), s.stat = static_cast<float2*>(at(k.slot_stat));
  s.out = static_cast<float*>(at(k.out));
  for (int i = 0; i < 2; ++i)
    s.key[i] = static_cast<uint32_t*>(at(k.key[i])), s.val[i] = static_cast<uint32_t*>(at(k.val[i]));
  s.again = static_cast<uint8_t*>(at(k.again));
  s.tile_first = static_cast<int32_t*>(at(k.tile_first));
  for (int i = 0; i < 2; ++i) s.run_sum[i] = static_cast<float*>(at(k.run_sum[i]));
  s.sort_tmp = at(k.sort), s.sort_bytes = k.sort_bytes;
  s.side = sm->side, s.fork = sm->fork, s.join = sm->join;
  SOFTMAX_CUDA(sm, launch_many_rows(a, s));
  return ESSPT_OK;
}

}  // namespace

extern "C" {

size_t esspt_softmax_workspace_bytes(const esspt_softmax_config* cfg) {
  return config_fault(cfg) ? 0 : carve(*cfg).total;
}

esspt_status esspt_softmax_create(const esspt_softmax_config* cfg, void* d_workspace, size_t bytes,
                                  esspt_softmax** out) {
  if (const char* why = config_fault(cfg)) return fail(nullptr, ESSPT_EINVAL, why);
  if (!out || !d_workspace || reinterpret_cast<uintptr_t>(d_workspace) % 256 != 0)
    return fail(nullptr, ESSPT_EINVAL, "null or misaligned pointer");
  if (bytes < carve(*cfg).total) return fail(nullptr, ESSPT_ENOSPC, "workspace too small");
  int dev = 0, sms = 0;
  SOFTMAX_CUDA(nullptr, cudaGetDevice(&dev));
  SOFTMAX_CUDA(nullptr, cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  SOFTMAX_CUDA(nullptr, cudaMemsetAsync(d_workspace, 0, kStatusBytes, static_cast<cudaStream_t>(cfg->stream)));
  esspt_softmax* sm = new (std::nothrow) esspt_softmax;
  if (!sm) return fail(nullptr, ESSPT_ENOSPC, "out of host memory");
  sm->cfg = *cfg;
  sm->st = static_cast<cudaStream_t>(cfg->stream);
  sm->base = static_cast<char*>(d_workspace);
  sm->k = carve(*cfg);
  sm->sms = sms < kMaxSms ? sms : kMaxSms;
  if (cfg->backward && cfg->max_rows > kFewRows) {
    cudaError_t e = cudaStreamCreateWithFlags(&sm->side, cudaStreamNonBlocking);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&sm->fork, cudaEventDisableTiming);
    if (e == cudaSuccess) e = cudaEventCreateWithFlags(&sm->join, cudaEventDisableTiming);
    if (e != cudaSuccess) {
      release(sm);
      return cuda_fail(nullptr, e, "esspt_softmax_create");
    }
  }
  *out = sm;
  return ESSPT_OK;
}

esspt_status esspt_softmax_destroy(esspt_softmax* sm) {
  if (!sm) return ESSPT_OK;
  cudaError_t e = cudaStreamSynchronize(sm->st);
  if (e == cudaSuccess && sm->side) e = cudaStreamSynchronize(sm->side);  // (after a call that failed half-way)
  release(sm);
  return e == cudaSuccess ? ESSPT_OK : cuda_fail(nullptr, e, "esspt_softmax_destroy");
}

esspt_status esspt_softmax_loss(esspt_softmax* sm, const void* d_h, int64_t h_stride, const void* d_w,
                                int64_t w_stride, const int32_t* d_targets, int64_t n, const float* d_weight,
                                float inv_temperature, float* d_loss, float* d_lse, void* d_grad_h, void* d_grad_w) {
  if (!sm) return ESSPT_EINVAL;
  sm->err[0] = 0;
  return run(sm, d_h, h_stride, d_w, w_stride, d_targets, nullptr, 1, n, d_weight, inv_temperature, d_loss, d_lse,
             d_grad_h, d_grad_w);
}

esspt_status esspt_softmax_distill(esspt_softmax* sm, const void* d_h, int64_t h_stride, const void* d_w,
                                   int64_t w_stride, const int32_t* d_ids, const float* d_logits, int32_t top,
                                   int64_t n, const float* d_weight, float inv_temperature, float* d_loss,
                                   float* d_lse, void* d_grad_h, void* d_grad_w) {
  if (!sm) return ESSPT_EINVAL;
  sm->err[0] = 0;
  if (!d_logits && n > 0) return fail(sm, ESSPT_EINVAL, "null pointer");
  return run(sm, d_h, h_stride, d_w, w_stride, d_ids, d_logits, top, n, d_weight, inv_temperature, d_loss, d_lse,
             d_grad_h, d_grad_w);
}

esspt_status esspt_softmax_poll(esspt_softmax* sm) {
  if (!sm) return ESSPT_EINVAL;
  sm->err[0] = 0;
  uint32_t bits = 0;
  SOFTMAX_CUDA(sm, cudaMemcpyAsync(&bits, sm->base, sizeof(bits), cudaMemcpyDeviceToHost, sm->st));
  SOFTMAX_CUDA(sm, cudaStreamSynchronize(sm->st));
  if (!bits) return ESSPT_OK;
  SOFTMAX_CUDA(sm, cudaMemsetAsync(sm->base, 0, sizeof(bits), sm->st));
  if (bits & kErrStuck) return fail(sm, ESSPT_ECUDA, "a wait inside a kernel ran out");
  return fail(sm, ESSPT_EINVAL, "a target or item id is outside the catalogue");
}

const char* esspt_softmax_last_error(const esspt_softmax* sm) { return sm ? sm->err : g_create_err; }

}  // extern "C"

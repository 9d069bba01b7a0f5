// C entries of the operators on device tensors (unifiednn.h): checks of the
// arguments, the device of the stream, and the launch. Nothing is enqueued
// before every check has passed.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "operators.h"

using namespace un;

namespace {

un_status bad(const char* call, const char* what, un_status s = UN_ERR_INVALID) {
  return fail_call(s, (std::string(call) + ": " + what).c_str());
}
un_status device_error(const char* call, hipError_t e) {
  (void)hipGetLastError();  // not the next call's
  return fail_call(UN_ERR_DEVICE, (std::string(call) + ": " + hipGetErrorString(e)).c_str());
}

// Makes the stream's device current for the life of this object.
class OnDevice {
 public:
  OnDevice(hipStream_t s) {
    if (!s) return;  // the current device's default stream
    int want = 0;
    err = hipStreamGetDevice(s, &want);
    if (err == hipSuccess) err = hipGetDevice(&was_);
    if (err == hipSuccess && want != was_) {
      err = hipSetDevice(want);
      back_ = err == hipSuccess;
    }
  }
  ~OnDevice() {
    if (back_) (void)hipSetDevice(was_);
  }
  hipError_t err = hipSuccess;

 private:
  int was_ = 0;
  bool back_ = false;
};

template <typename F> un_status enqueue(const char* call, void* stream, F&& f) {
  OnDevice on((hipStream_t)stream);
  if (on.err != hipSuccess) return device_error(call, on.err);
  const hipError_t e = f((hipStream_t)stream);
  return e == hipSuccess ? UN_OK : device_error(call, e);
}

// A launch's threads are counted in 32 bits.
bool too_many(int64_t workgroups, int threads) { return workgroups > (((int64_t)1 << 32) - 1) / threads; }

bool type_ok(int32_t t) { return t == UN_TYPE_F32 || t == UN_TYPE_BF16; }

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------
// RMS norm
// ---------------------------------------------------------------------------
un_status un_rms_norm(const un_rms_norm_args* a, void* stream) {
  const char* F = "un_rms_norm";
  if (!a) return bad(F, "args is NULL");
  if (!type_ok(a->type)) return bad(F, "unknown type");
  if (a->rows < 0 || a->width < 1) return bad(F, "rows >= 0 and width >= 1 expected");
  if (a->width > NORM_MAX_D) return bad(F, "width above 16384 is not supported", UN_ERR_UNSUPPORTED);
  if (!(a->eps >= 0.f) || !std::isfinite(a->eps)) return bad(F, "eps must be finite and >= 0");
  if (a->rows == 0) return UN_OK;
  if (!a->x || !a->weight || !a->y) return bad(F, "x, weight or y is NULL");
  const int64_t d = a->width;
  if (a->rows > 1 && (a->ldx < d || a->ldy < d || (a->residual && a->ldr < d) || (a->sum && a->lds < d)))
    return bad(F, "a row stride is smaller than the width");
  const NormPlan plan = norm_plan(a->type == UN_TYPE_BF16, a->width);
  if (too_many((a->rows + plan.group - 1) / plan.group, 256 > plan.tpr ? 256 : plan.tpr)) return bad(F, "too many rows", UN_ERR_UNSUPPORTED);
  NormProb p{};
  p.x = a->x;
  p.ldx = a->ldx;
  p.r = a->residual;
  p.ldr = a->ldr;
  p.w = a->weight;
  p.s = a->sum;
  p.lds = a->lds;
  p.y = a->y;
  p.ldy = a->ldy;
  p.rstd = a->rstd;
  p.scale = a->scale;
  p.rows = a->rows;
  p.d = a->width;
  p.eps = a->eps;
  return enqueue(F, stream, [&](hipStream_t s) { return launch_norm(a->type == UN_TYPE_BF16, a->scale != nullptr, plan, p, s); });
}

un_status un_rms_norm_workspace(int32_t type, int64_t rows, int32_t width, size_t* bytes) {
  const char* F = "un_rms_norm_workspace";
  if (!bytes) return bad(F, "bytes is NULL");
  if (!type_ok(type)) return bad(F, "unknown type");
  if (rows < 0 || width < 1) return bad(F, "rows >= 0 and width >= 1 expected");
  if (width > NORM_MAX_D) return bad(F, "width above 16384 is not supported", UN_ERR_UNSUPPORTED);
  *bytes = (size_t)norm_blocks(norm_plan(type == UN_TYPE_BF16, width), rows) * width * 4;
  return UN_OK;
}

un_status un_rms_norm_backward(const un_rms_norm_grad_args* a, void* stream) {
  const char* F = "un_rms_norm_backward";
  if (!a) return bad(F, "args is NULL");
  size_t need = 0;
  const un_status st = un_rms_norm_workspace(a->type, a->rows, a->width, &need);
  if (st != UN_OK) return st;
  if (!a->dweight || !a->weight) return bad(F, "weight or dweight is NULL");
  if (a->rows > 0 && (!a->dy || !a->s || !a->rstd)) return bad(F, "dy, s or rstd is NULL");
  const int64_t d = a->width;
  if (a->rows > 1 && (a->lddy < d || a->lds < d || (a->ds && a->ldds < d) || (a->dx && a->lddx < d)))
    return bad(F, "a row stride is smaller than the width");
  if (a->workspace_bytes < need || !a->workspace) return bad(F, "workspace too small (un_rms_norm_workspace)", UN_ERR_BUFSIZE);
  const NormPlan plan = norm_plan(a->type == UN_TYPE_BF16, a->width);
  NormProb p{};
  p.x = a->s;
  p.ldx = a->lds;
  p.r = a->ds;
  p.ldr = a->ldds;
  p.dy = a->dy;
  p.lddy = a->lddy;
  p.w = a->weight;
  p.y = a->dx;
  p.ldy = a->lddx;
  p.rstd = const_cast<float*>(a->rstd);
  p.part = (float*)a->workspace;
  p.rows = a->rows;
  p.d = a->width;
  p.blocks = norm_blocks(plan, a->rows);
  return enqueue(F, stream, [&](hipStream_t s) {
    const hipError_t e = launch_norm_bwd(a->type == UN_TYPE_BF16, plan, p, s);
    return e != hipSuccess ? e : launch_norm_dw(p.part, p.blocks, p.d, a->dweight, s);
  });
}

// ---------------------------------------------------------------------------
// Gated linear recurrence
// ---------------------------------------------------------------------------
namespace {
// sizes that a direction's launch plan and the kernels can count; that plan
un_status scan_sizes_ok(const char* F, int32_t B, int32_t T, int32_t d, bool bwd, ScanPlan* plan) {
  if (B < 0 || T < 0 || d < 0) return bad(F, "negative size");
  if (T > (1 << 30)) return bad(F, "more than 2^30 tokens are not supported", UN_ERR_UNSUPPORTED);
  if (d > SCAN_MAX_LD) return bad(F, "a width of 2^24 or more is not supported", UN_ERR_UNSUPPORTED);
  *plan = scan_plan(B, T, d, bwd);
  if (too_many((int64_t)plan->tiles * B * plan->nseg, plan->kind >= SCAN_CHUNKS ? 64 * SCAN_W : 64))
    return bad(F, "too many sequences and channels", UN_ERR_UNSUPPORTED);
  return UN_OK;
}
}  // namespace

un_status un_gated_scan_sizes(int32_t batch, int32_t tokens, int32_t width, size_t* states, size_t* workspace_bytes) {
  const char* F = "un_gated_scan_sizes";
  ScanPlan fwd;  // (the backward pass has no fewer workgroups)
  const un_status st = scan_sizes_ok(F, batch, tokens, width, false, &fwd);
  if (st != UN_OK) return st;
  if (states) *states = (size_t)batch * scan_chunks(tokens) * width;
  if (workspace_bytes)
    *workspace_bytes = 8 * (size_t)std::max(scan_ws_words(fwd, batch, width),
                                            scan_ws_words(scan_plan(batch, tokens, width, true), batch, width));
  return UN_OK;
}

namespace {
// what both directions check: sizes, strides and the workspace
un_status scan_common(const char* F, int32_t type, int32_t B, int32_t T, int32_t d, int64_t ld, int64_t ld2, int64_t ld3,
                      int64_t seq_out, const void* workspace, size_t bytes, bool bwd, ScanPlan* plan) {
  if (!type_ok(type)) return bad(F, "unknown type");
  un_status st = scan_sizes_ok(F, B, T, d, bwd, plan);
  if (st != UN_OK) return st;
  if (T > 1 && (ld > SCAN_MAX_LD || ld2 > SCAN_MAX_LD || ld3 > SCAN_MAX_LD))
    return bad(F, "a token stride of 2^24 or more is not supported", UN_ERR_UNSUPPORTED);
  if (T > 1 && (ld < d || ld2 < d || ld3 < d)) return bad(F, "a token stride is smaller than the width");
  if (B > 1 && T > 0 && seq_out < d) return bad(F, "the output's sequence stride is smaller than the width");
  size_t need = 0;
  st = un_gated_scan_sizes(B, T, d, nullptr, &need);
  if (st != UN_OK) return st;
  if (need && (!workspace || bytes < need)) return bad(F, "workspace too small (un_gated_scan_sizes)", UN_ERR_BUFSIZE);
  if (need && (uintptr_t)workspace % 8) return bad(F, "workspace is not 8-byte aligned");
  return UN_OK;
}
}  // namespace

un_status un_gated_scan(const un_gated_scan_args* a, void* stream) {
  const char* F = "un_gated_scan";
  if (!a) return bad(F, "args is NULL");
  ScanPlan plan;
  const un_status st = scan_common(F, a->type, a->batch, a->tokens, a->width, a->ld_in, a->ld_h, a->ld_h, a->seq_h,
                                   a->workspace, a->workspace_bytes, false, &plan);
  if (st != UN_OK) return st;
  if (a->batch == 0 || a->width == 0) return UN_OK;
  if (a->tokens > 0 && (!a->gate || !a->value || !a->h)) return bad(F, "gate, value or h is NULL");
  ScanProb p{};
  p.gate = a->gate;
  p.value = a->value;
  p.ldi = a->ld_in;
  p.bsi = a->seq_in;
  p.o1 = a->h;
  p.ldo = a->ld_h;
  p.bso = a->seq_h;
  p.lens = a->lens;
  p.start = a->start;
  p.end = a->last;
  p.states = a->states;
  p.joint = (uint64_t*)a->workspace;
  p.B = a->batch;
  p.T = a->tokens;
  p.d = a->width;
  return enqueue(F, stream, [&](hipStream_t s) { return launch_scan(a->type == UN_TYPE_BF16, false, plan, p, s); });
}

un_status un_gated_scan_backward(const un_gated_scan_grad_args* a, void* stream) {
  const char* F = "un_gated_scan_backward";
  if (!a) return bad(F, "args is NULL");
  ScanPlan plan;
  const un_status st = scan_common(F, a->type, a->batch, a->tokens, a->width, a->ld_in, a->ld_dh, a->ld_out, a->seq_out,
                                   a->workspace, a->workspace_bytes, true, &plan);
  if (st != UN_OK) return st;
  if (a->batch == 0 || a->width == 0) return UN_OK;
  if (a->tokens > 0 && (!a->gate || !a->value || !a->dh || !a->states || !a->dgate || !a->dvalue))
    return bad(F, "gate, value, states, dh, dgate or dvalue is NULL");
  ScanProb p{};
  p.gate = a->gate;
  p.value = a->value;
  p.ldi = a->ld_in;
  p.bsi = a->seq_in;
  p.dh = a->dh;
  p.lddh = a->ld_dh;
  p.bsdh = a->seq_dh;
  p.o1 = a->dgate;
  p.o2 = a->dvalue;
  p.ldo = a->ld_out;
  p.bso = a->seq_out;
  p.lens = a->lens;
  p.start = a->dlast;
  p.end = a->dstart;
  p.states = const_cast<float*>(a->states);
  p.joint = (uint64_t*)a->workspace;
  p.B = a->batch;
  p.T = a->tokens;
  p.d = a->width;
  return enqueue(F, stream, [&](hipStream_t s) { return launch_scan(a->type == UN_TYPE_BF16, true, plan, p, s); });
}

// ---------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------
struct un_adamw {
  int device = 0;
  bool g16 = false, eight = false;
  char* table = nullptr;   // the tensors, then the workgroups' (tensor, chunk)
  size_t map_at = 0;
  int nblocks = 0;
  int64_t bytes = 0;       // of the tensors, gradients and states
};

un_status un_adamw_create(const un_adamw_tensor* t, int32_t n, int32_t grad_type, int32_t bits, un_adamw** out) {
  const char* F = "un_adamw_create";
  if (!out) return bad(F, "out is NULL");
  *out = nullptr;
  if (!t || n < 1) return bad(F, "no tensors");
  if (!type_ok(grad_type)) return bad(F, "unknown gradient type");
  if (bits != 32 && bits != 8) return bad(F, "state_bits must be 32 or 8");
  int64_t blocks = 0;
  for (int i = 0; i < n; ++i) {
    if (t[i].elements < 0) return bad(F, "negative element count");
    if (t[i].elements == 0) continue;
    if (!t[i].weight || !t[i].grad || !t[i].m || !t[i].v) return bad(F, "a tensor's weight, grad, m or v is NULL");
    if (bits == 8 && (!t[i].m_scale || !t[i].v_scale)) return bad(F, "8-bit states need m_scale and v_scale");
    if (bits == 32 && (t[i].m_scale || t[i].v_scale)) return bad(F, "32-bit states have no scales");
    if (t[i].elements > ((int64_t)1 << 42)) return bad(F, "tensor too large", UN_ERR_UNSUPPORTED);
    blocks += (t[i].elements + AW_CHUNK - 1) / AW_CHUNK;
  }
  if (too_many(blocks, 256)) return bad(F, "too many elements", UN_ERR_UNSUPPORTED);
  un_adamw* a = nullptr;
  try {
    a = new un_adamw();
    a->g16 = grad_type == UN_TYPE_BF16;
    a->eight = bits == 8;
    a->nblocks = (int)blocks;
    std::vector<AdamwTensor> ts((size_t)n);
    std::vector<int32_t> map;
    map.reserve((size_t)blocks * 2);
    uint32_t base = 0;
    for (int i = 0; i < n; ++i) {
      const un_adamw_tensor& q = t[i];
      ts[i] = AdamwTensor{q.weight, q.grad, q.copy, q.m, q.v, q.m_scale, q.v_scale, q.elements, base, 0};
      const int64_t nb = (q.elements + AW_CHUNK - 1) / AW_CHUNK;
      for (int64_t b = 0; b < nb; ++b) {
        map.push_back(i);
        map.push_back((int32_t)b);
      }
      base += (uint32_t)((q.elements + AW_BLOCK - 1) / AW_BLOCK * AW_BLOCK);
      a->bytes += q.elements * (4 + (a->g16 ? 2 : 4) + (q.copy ? 2 : 0) + (a->eight ? 2 : 8));
    }
    a->map_at = (ts.size() * sizeof(AdamwTensor) + 255) / 256 * 256;
    std::vector<char> host(a->map_at + map.size() * 4);
    memcpy(host.data(), ts.data(), ts.size() * sizeof(AdamwTensor));
    memcpy(host.data() + a->map_at, map.data(), map.size() * 4);
    hipError_t e = hipGetDevice(&a->device);
    if (e == hipSuccess) e = hipMalloc((void**)&a->table, host.size() + 256);
    if (e != hipSuccess) {
      delete a;
      (void)hipGetLastError();
      return fail_call(e == hipErrorOutOfMemory ? UN_ERR_OOM : UN_ERR_DEVICE, (std::string(F) + ": " + hipGetErrorString(e)).c_str());
    }
    e = hipMemcpy(a->table, host.data(), host.size(), hipMemcpyHostToDevice);
    if (e != hipSuccess) {
      (void)hipFree(a->table);
      delete a;
      return device_error(F, e);
    }
  } catch (const std::bad_alloc&) {
    if (a && a->table) (void)hipFree(a->table);
    delete a;
    return bad(F, "out of host memory", UN_ERR_OOM);
  }
  *out = a;
  return UN_OK;
}

un_status un_adamw_step(un_adamw* a, const un_adamw_hyper* h, void* stream) {
  const char* F = "un_adamw_step";
  if (!a || !h) return bad(F, "plan or hyper-parameters NULL");
  auto unit = [](double x) { return x >= 0.0 && (float)x < 1.f; };
  if (!std::isfinite(h->lr) || h->lr < 0.0 || !std::isfinite(h->decay) || h->decay < 0.0) return bad(F, "lr and decay must be finite and >= 0");
  if (!(h->lr * h->decay < 1.0)) return bad(F, "lr * decay must be below 1");
  if (!unit(h->beta1) || !unit(h->beta2)) return bad(F, "beta1 and beta2 must be in [0, 1)");
  if (!std::isfinite(h->eps) || !((float)h->eps > 0.f)) return bad(F, "eps must be finite and > 0");
  if (h->t < 1) return bad(F, "t counts from 1");
  OnDevice on((hipStream_t)stream);
  if (on.err != hipSuccess) return device_error(F, on.err);
  int dev = 0;
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  hipError_t e = hipGetDevice(&dev);
  if (e == hipSuccess) e = hipStreamIsCapturing((hipStream_t)stream, &cap);
  if (e != hipSuccess) return device_error(F, e);
  if (cap != hipStreamCaptureStatusNone)
    return bad(F, "a captured step would repeat its rates and count", UN_ERR_UNSUPPORTED);
  if (dev != a->device) return bad(F, "the stream is on another device than the plan");
  const double t = (double)h->t;
  AdamwHp hp;
  hp.decay = (float)(h->lr * h->decay);
  hp.key = h->key;
  hp.lr = (float)(h->lr / (1.0 - std::pow(h->beta1, t)));
  hp.b1 = (float)h->beta1;
  hp.b2 = (float)h->beta2;
  hp.c1 = (float)(1.0 - h->beta1);
  hp.c2 = (float)(1.0 - h->beta2);
  hp.isb2 = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, t)));
  hp.eps = (float)h->eps;
  e = launch_adamw(a->g16, a->eight, (const AdamwTensor*)a->table, (const int32_t*)(a->table + a->map_at), a->nblocks, a->bytes, hp, nullptr,
                   (hipStream_t)stream);
  return e == hipSuccess ? UN_OK : device_error(F, e);
}

void un_adamw_destroy(un_adamw* a) {
  if (!a) return;
  int was = 0;
  const bool set = hipGetDevice(&was) == hipSuccess && was != a->device && hipSetDevice(a->device) == hipSuccess;
  (void)hipFree(a->table);  // waits for the device
  if (set) (void)hipSetDevice(was);
  delete a;
}

}  // extern "C"

// C ABI of libjetvit: argument validation, dispatch, device status.
// Every argument error is reported before anything is launched.
#include <atomic>
#include <initializer_list>
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "attn_diff.cuh"
#include "common.cuh"
#include "scan.cuh"

namespace jv {
namespace {

__device__ int g_status_word = 0;          // sticky error bits written by kernels
std::atomic<uint64_t> g_launches{0};
std::atomic<int32_t> g_force_generic{0};

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// [a, a + na) and [b, b + nb) share at least one byte
bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + nb && y < x + na;
}

size_t tensor_bytes(const jv_shape* s) {
  return (size_t)s->B * s->H * shape_tokens(*s) * s->D * (s->dtype == JV_F32 ? 4 : 2);
}

jv_status check_shape(const jv_shape* s) {
  if (!s) return JV_ERR_INVALID_ARG;
  if (s->B <= 0 || s->H <= 0 || s->Hg <= 0 || s->Wg <= 0 || s->D <= 0 || s->P < 0) return JV_ERR_INVALID_ARG;
  if (s->dtype != JV_F32 && s->dtype != JV_BF16) return JV_ERR_INVALID_ARG;
  if ((int64_t)s->Hg * s->Wg + s->P > (1 << 24)) return JV_ERR_UNSUPPORTED;
  if ((int64_t)s->B * s->H > 65535) return JV_ERR_UNSUPPORTED;
  if (s->D > 128) return JV_ERR_UNSUPPORTED;
  // rows must keep 16-byte alignment for the vector loads
  const int esz = s->dtype == JV_F32 ? 4 : 2;
  if ((s->D * esz) % 16 != 0) return JV_ERR_UNSUPPORTED;
  if (s->in_layout != JV_LAYOUT_BHND && s->in_layout != JV_LAYOUT_BNHD) return JV_ERR_INVALID_ARG;
  if (s->in_layout == JV_LAYOUT_BNHD) {
    const int64_t row = (int64_t)s->H * s->D;
    if (s->in_tok_stride != 0 && s->in_tok_stride < row) return JV_ERR_INVALID_ARG;   // token rows would overlap
    if ((s->in_tok_stride * esz) % 16 != 0) return JV_ERR_INVALID_ARG;
    if (s->in_tok_stride > ((int64_t)1 << 31)) return JV_ERR_UNSUPPORTED;
  } else if (s->in_tok_stride != 0) {
    return JV_ERR_INVALID_ARG;
  }
  return JV_OK;
}

// bytes from the first to one past the last element of an input tensor (q, k or v)
size_t input_bytes(const jv_shape* s) {
  if (!in_strided(*s)) return tensor_bytes(s);
  const InStrides in = in_strides(*s);
  const size_t esz = s->dtype == JV_F32 ? 4 : 2;
  return (size_t)((int64_t)(s->B - 1) * in.batch + (int64_t)(shape_tokens(*s) - 1) * in.tok + (int64_t)s->H * s->D) * esz;
}

jv_status check_tensors(const void* q, const void* k, const void* v, const void* o, const jv_shape* s) {
  if (!q || !k || !v || !o) return JV_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16)) return JV_ERR_INVALID_ARG;
  const size_t n = tensor_bytes(s), ni = input_bytes(s);      // o may not share a byte with an input
  if (overlaps(o, n, q, ni) || overlaps(o, n, k, ni) || overlaps(o, n, v, ni)) return JV_ERR_INVALID_ARG;
  return JV_OK;
}

jv_status check_dwc(const jv_dwc* d) {
  if (!d) return JV_OK;
  if (d->k != 3 && d->k != 5) return JV_ERR_INVALID_ARG;
  if (d->R < 0 || d->R > 1024) return JV_ERR_INVALID_ARG;
  if (d->token_wise != 0 && d->token_wise != 1) return JV_ERR_INVALID_ARG;
  if (d->token_wise && d->R == 0) return JV_ERR_INVALID_ARG;  // per-token kernels need the generator
  if (d->R == 0) return d->b2 ? JV_OK : JV_ERR_INVALID_ARG;   // static kernels live in b2
  if (!d->W1 || !d->W2) return JV_ERR_INVALID_ARG;
  return JV_OK;
}

jv_status check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return JV_OK;
  if (!ws || !aligned(ws, 256) || ws_bytes < need) return JV_ERR_WORKSPACE;
  return JV_OK;
}

jv_status check_window(const jv_shape* s, int wh, int ww) {
  if (wh <= 0 || ww <= 0) return JV_ERR_INVALID_ARG;
  const int64_t nwin = (int64_t)ceil_div(s->Hg, wh < s->Hg ? wh : s->Hg) * ceil_div(s->Wg, ww < s->Wg ? ww : s->Wg);
  if (nwin > 65535) return JV_ERR_UNSUPPORTED;
  return JV_OK;
}

jv_status check_device() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return JV_ERR_CUDA; }
  int major = 0;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess) {
    cudaGetLastError();
    return JV_ERR_CUDA;
  }
  return major == 10 ? JV_OK : JV_ERR_UNSUPPORTED;
}

// ptrs[0 .. nin) are inputs, ptrs[nin .. nptr) outputs; bytes[i] is the extent of ptrs[i]
jv_status check_proj(const jv_shape* s, const void* const* ptrs, const size_t* bytes, int nptr, int nin) {
  jv_status st = check_shape(s);
  if (st != JV_OK) return st;
  for (int i = 0; i < nptr; ++i)
    if (!ptrs[i] || !aligned(ptrs[i], 16)) return JV_ERR_INVALID_ARG;
  if (s->dtype != JV_BF16 || s->D != 64) return JV_ERR_UNSUPPORTED;   // (the extents below assume both)
  if (in_strided(*s)) return JV_ERR_UNSUPPORTED;                        // the projections have layouts of their own
  for (int i = nin; i < nptr; ++i)           // outputs overlap neither an input nor each other
    for (int j = 0; j < i; ++j)
      if (overlaps(ptrs[i], bytes[i], ptrs[j], bytes[j])) return JV_ERR_INVALID_ARG;
  return JV_OK;
}

jv_status from_cuda(cudaError_t e) {
  if (e == cudaSuccess) return JV_OK;
  if (getenv("JETVIT_DEBUG")) fprintf(stderr, "libjetvit: CUDA error %d (%s)\n", (int)e, cudaGetErrorString(e));
  return JV_ERR_CUDA;
}

// A stretch of memory that a call reads or writes
struct Span {
  const void* p;
  size_t bytes;
};
// every output against every input and the outputs before it; null pointers take no part
bool outputs_clash(const Span* in, int nin, const Span* out, int nout) {
  for (int i = 0; i < nout; ++i) {
    if (!out[i].p) continue;
    for (int j = 0; j < nin; ++j)
      if (in[j].p && overlaps(out[i].p, out[i].bytes, in[j].p, in[j].bytes)) return true;
    for (int j = 0; j < i; ++j)
      if (out[j].p && overlaps(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return true;
  }
  return false;
}

jv_status check_norm(const jv_norm_shape* s) {
  if (!s || s->rows <= 0 || s->C <= 0) return JV_ERR_INVALID_ARG;
  if (s->dtype != JV_F32 && s->dtype != JV_BF16) return JV_ERR_INVALID_ARG;
  if (s->C > 16384 || s->rows > 0x7fffffffll) return JV_ERR_UNSUPPORTED;
  if ((s->x_stride != 0 && s->x_stride < s->C) || (s->dy_stride != 0 && s->dy_stride < s->C)) return JV_ERR_INVALID_ARG;
  for (int64_t stride : {s->x_stride, s->dy_stride})          // (extents are counted in 64 bits of bytes)
    if (stride > ((int64_t)1 << 56) / s->rows) return JV_ERR_UNSUPPORTED;
  return JV_OK;
}
size_t norm_rows_bytes(const jv_norm_shape* s, int64_t stride) {
  return (size_t)((s->rows - 1) * (stride ? stride : s->C) + s->C) * (s->dtype == JV_F32 ? 4 : 2);
}

// {token rows, batch elements} of a [B, L, C] tensor; false if token rows would overlap or run backwards
bool token_rows(const int64_t* s, int L, int C, Rows* out) {
  out->tok = s[0] ? s[0] : C;
  out->batch = s[1] ? s[1] : L * out->tok;
  return out->tok >= C && out->batch > 0;
}
// extents are counted in 64 bits of bytes (L is at most 2^24)
bool far_rows(const Rows& r, int B) { return r.tok > (int64_t)1 << 31 || r.batch > ((int64_t)1 << 56) / B; }

// {tokens, heads, batch elements}; a zero entry only where all are zero (contiguous)
bool diff_strides(const int64_t* s, int heads, int n, int D, InStrides* out) {
  if (!s[0] && !s[1] && !s[2]) {
    *out = InStrides{(int64_t)D, (int64_t)n * D, (int64_t)heads * n * D};
    return true;
  }
  *out = InStrides{s[0], s[1], s[2]};
  return s[0] > 0 && s[1] > 0 && s[2] > 0;
}
size_t diff_bytes(const InStrides& s, int B, int heads, int n, int D, size_t e) {
  return (size_t)((B - 1) * s.batch + (heads - 1) * s.head + (n - 1) * s.tok + D) * e;
}
jv_status check_diff(const jv_diff_shape* s, InStrides* qs, InStrides* ks) {
  if (!s || s->B <= 0 || s->H <= 0 || s->Hkv <= 0 || s->Nq <= 0 || s->Nk <= 0 || s->D <= 0) return JV_ERR_INVALID_ARG;
  if (s->dtype != JV_F32 && s->dtype != JV_BF16) return JV_ERR_INVALID_ARG;
  if (s->causal != 0 && s->causal != 1) return JV_ERR_INVALID_ARG;
  if (s->H % 2 || s->Hkv % 2 || s->H % s->Hkv) return JV_ERR_INVALID_ARG;
  if (s->Nq > (1 << 24) || s->Nk > (1 << 24) || (int64_t)s->B * s->H > 65535 || s->D > 64) return JV_ERR_UNSUPPORTED;
  // tiles of 128 queries and keys: a block counts its share of them in 32 bits
  if ((int64_t)s->B * (s->H / 2) * ceil_div(s->Nq, 128) * ceil_div(s->Nk, 128) > (int64_t)1 << 36) return JV_ERR_UNSUPPORTED;
  const int64_t e = s->dtype == JV_F32 ? 4 : 2;
  if (s->D * e % 16) return JV_ERR_UNSUPPORTED;
  if (!diff_strides(s->q_stride, s->H, s->Nq, s->D, qs) || !diff_strides(s->kv_stride, s->Hkv, s->Nk, s->D, ks)) return JV_ERR_INVALID_ARG;
  for (const InStrides* x : {qs, ks})
    for (int64_t v : {x->tok, x->head, x->batch}) {
      if (v * e % 16) return JV_ERR_INVALID_ARG;
      if (v > (int64_t)1 << 37) return JV_ERR_UNSUPPORTED;
    }
  return JV_OK;
}

jv_status check_conv(const jv_conv_shape* s, Rows* xs) {
  if (!s || s->B <= 0 || s->L <= 0 || s->C <= 0 || s->K <= 0) return JV_ERR_INVALID_ARG;
  if (s->dtype != JV_F32 && s->dtype != JV_BF16) return JV_ERR_INVALID_ARG;
  if ((s->silu != 0 && s->silu != 1) || !token_rows(s->x_stride, s->L, s->C, xs)) return JV_ERR_INVALID_ARG;
  if (s->K < 2 || s->K > 4 || s->B > 65535 || s->C > (1 << 20) || s->L > (1 << 24) || far_rows(*xs, s->B)) return JV_ERR_UNSUPPORTED;
  return (int64_t)s->B * s->L * s->C > ((int64_t)1 << 40) ? JV_ERR_UNSUPPORTED : JV_OK;
}

struct ScanRows {
  Rows u, dt, b, c, z;
};
jv_status check_scan(const jv_scan_shape* s, ScanRows* r) {
  if (!s || s->B <= 0 || s->L <= 0 || s->C <= 0 || s->Ns <= 0) return JV_ERR_INVALID_ARG;
  if (s->dtype != JV_F32 && s->dtype != JV_BF16) return JV_ERR_INVALID_ARG;
  if (s->softplus != 0 && s->softplus != 1) return JV_ERR_INVALID_ARG;
  if (!token_rows(s->u_stride, s->L, s->C, &r->u) || !token_rows(s->dt_stride, s->L, s->C, &r->dt) || !token_rows(s->z_stride, s->L, s->C, &r->z) ||
      !token_rows(s->b_stride, s->L, s->Ns, &r->b) || !token_rows(s->c_stride, s->L, s->Ns, &r->c))
    return JV_ERR_INVALID_ARG;
  for (const Rows& v : {r->u, r->dt, r->b, r->c, r->z})
    if (far_rows(v, s->B)) return JV_ERR_UNSUPPORTED;
  if (s->Ns > 64 || s->B > 65535 || s->C > (1 << 20) || s->L > (1 << 24)) return JV_ERR_UNSUPPORTED;
  return JV_OK;
}
size_t token_rows_bytes(int B, int L, const Rows& r, int C, size_t e) { return (size_t)(r.at(B - 1, L - 1) + C) * e; }

float pick_scale(float scale, int D) { return scale > 0.f ? scale : 1.f / sqrtf((float)D); }

// ---- enqueue helpers (arguments already validated) ---------------------------
jv_status run_attn(const void* q, const void* k, const void* v, void* o, const jv_shape* s, int wh, int ww,
                   float scale, bool full, cudaStream_t st) {
  AttnArgs a{q, k, v, o, s->B * s->H, s->Hg, s->Wg, s->D, s->H, in_strides(*s), in_strided(*s),
             s->P, wh, ww, pick_scale(scale, s->D), s->dtype};
  const bool one_window = full || (wh >= s->Hg && ww >= s->Wg);
  if (one_window) {      // every token attends all P + N tokens: where a token sits does not matter
    a.Hg = 1;
    a.Wg = shape_tokens(*s);
    a.P = 0;
    a.wh = a.Hg;
    a.ww = a.Wg;
  }
  if (!g_force_generic.load() && one_window && a.Wg <= 256) {
    // A sequence of at most two tiles is a window one token wide: two heads at a time per CTA.  Measured against the two-tile
    // kernel: 384 heads of 256 tokens 15.8 / 17.1 us, of 144 15.8 / 18.1; 192 of 100: 7.6 / 9.3; 6 of 256: 7.8 / 7.7.
    AttnArgs w = a;
    w.Hg = a.Wg;
    w.Wg = 1;
    w.wh = 256;
    w.ww = 1;
    if (attn_w4_supported(w)) {
      int* status = device_status_ptr();
      if (!status) return JV_ERR_CUDA;
      return from_cuda(launch_attn_w4(w, status, st));
    }
  }
  if (!g_force_generic.load() && one_window && attn_split_supported(a)) {
    int* status = device_status_ptr();
    if (!status) return JV_ERR_CUDA;
    return from_cuda(launch_attn_split(a, status, st));
  }
  if (!g_force_generic.load() && one_window && attn_f4_supported(a)) {
    int* status = device_status_ptr();
    if (!status) return JV_ERR_CUDA;
    return from_cuda(launch_attn_f4(a, status, st));
  }
  if (!g_force_generic.load() && attn_d128_supported(a, full)) {
    int* status = device_status_ptr();
    if (!status) return JV_ERR_CUDA;
    return from_cuda(launch_attn_d128(a, full, status, st));
  }
  if (!g_force_generic.load() && !one_window && attn_w4_supported(a)) {
    int* status = device_status_ptr();
    if (!status) return JV_ERR_CUDA;
    if (a.P > 0) {                                        // the P prefix queries, which attend everything
      const jv_status r = from_cuda(launch_attn_prefix(a, device_sm_count() - attn_w4_ctas(a), status, st));
      if (r != JV_OK) return r;
    }
    return from_cuda(launch_attn_w4(a, status, st));
  }
  if (!g_force_generic.load() && attn_tc_supported(a, full)) {
    int* status = device_status_ptr();
    if (!status) return JV_ERR_CUDA;
    if (a.strided && a.P > 0) return JV_ERR_UNSUPPORTED;  // the prefix queries' kernel reads contiguous tensors
    if (a.P > 0) {
      const jv_status r = from_cuda(launch_attn_prefix(a, device_sm_count() - attn_tc_ctas(a, full), status, st));
      if (r != JV_OK) return r;
    }
    return from_cuda(launch_attn_tc(a, full, status, st));
  }
  if (a.strided) return JV_ERR_UNSUPPORTED;               // the fp32 and generic kernels read contiguous tensors
  if (!g_force_generic.load() && attn_f32_supported(a)) return from_cuda(launch_attn_f32(a, st));
  return from_cuda(launch_attn_generic(a, st));
}

jv_status run_linear(const void* q, const void* k, const void* v, void* o, const jv_shape* s, float eps,
                     const jv_dwc* dwc, void* ws, cudaStream_t st) {
  LinArgs a{q, k, v, o, *s, eps, dwc, ws};
  if (!dwc && s->P > 0) {   // without the convolution the block is global: where a token sits does not matter
    a.s.Hg = 1;
    a.s.Wg = shape_tokens(*s);
    a.s.P = 0;
  }
  const LinPlan p = lin_plan(*s, dwc);
  if (!g_force_generic.load() && linear_fast_supported(a)) return from_cuda(launch_linear_fast(a, p, st));
  if (!g_force_generic.load() && linear_d128_supported(a)) return from_cuda(launch_linear_d128(a, p, st));
  if (!g_force_generic.load() && linear_f32_supported(a)) return from_cuda(launch_linear_f32(a, p, st));
  if (in_strided(*s)) return JV_ERR_UNSUPPORTED;          // the generic kernels read contiguous tensors
  return from_cuda(launch_linear_generic(a, p, st));
}

}  // namespace

int* device_status_ptr() {
  // One address per device; looked up once per device and cached.
  static int* cache[64] = {nullptr};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
  if (!cache[dev]) {
    int* p = nullptr;
    if (cudaGetSymbolAddress((void**)&p, g_status_word) != cudaSuccess) { cudaGetLastError(); return nullptr; }
    cache[dev] = p;
  }
  return cache[dev];
}

void count_launch(int n) { g_launches.fetch_add((uint64_t)n, std::memory_order_relaxed); }

int current_device() {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return -1; }
  return dev;
}

int device_sm_count() {
  static std::atomic<int> cache[kMaxDevices] = {};
  const int dev = current_device();
  if (dev < 0 || dev >= kMaxDevices) return kDefaultSmCount;
  int n = cache[dev].load(std::memory_order_relaxed);
  if (n > 0) return n;
  if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) {
    cudaGetLastError();
    return kDefaultSmCount;
  }
  cache[dev].store(n, std::memory_order_relaxed);
  return n;
}

}  // namespace jv

using namespace jv;

extern "C" {

size_t jv_workspace_bytes(char mixer, const jv_shape* shape, const jv_dwc* dwc) {
  if (check_shape(shape) != JV_OK || check_dwc(dwc) != JV_OK) return 0;
  switch (mixer) {
    case 'L':
    case 'S':
      return lin_plan(*shape, dwc).total;   // W and F need no scratch
    case 'f':   // the linear block with the focused feature map: two tensors for phi(q), phi(k) behind the block's own scratch
      return align_up(lin_plan(*shape, dwc).total, 256) + 2 * align_up(tensor_bytes(shape), 256);
    case 'W':
    case 'F':
      return 0;
    default:
      return 0;
  }
}

jv_status jv_linear_attn(const void* q, const void* k, const void* v, void* o, const jv_shape* shape, float eps,
                         const jv_dwc* dwc, void* ws, size_t ws_bytes, void* cuda_stream) {
  jv_status st = check_shape(shape);
  if (st != JV_OK) return st;
  if ((st = check_tensors(q, k, v, o, shape)) != JV_OK) return st;
  if (!(eps >= 0.f)) return JV_ERR_INVALID_ARG;
  if ((st = check_dwc(dwc)) != JV_OK) return st;
  if ((st = check_ws(ws, ws_bytes, lin_plan(*shape, dwc).total)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  return run_linear(q, k, v, o, shape, eps, dwc, ws, (cudaStream_t)cuda_stream);
}

jv_status jv_linear_attn_focused(const void* q, const void* k, const void* v, void* o, const jv_shape* shape, float eps,
                                 float focus_p, const jv_dwc* dwc, void* ws, size_t ws_bytes, void* cuda_stream) {
  jv_status st = check_shape(shape);
  if (st != JV_OK) return st;
  if ((st = check_tensors(q, k, v, o, shape)) != JV_OK) return st;
  if (!(eps >= 0.f) || !(focus_p > 0.f) || !(focus_p <= 16.f)) return JV_ERR_INVALID_ARG;
  if ((st = check_dwc(dwc)) != JV_OK) return st;
  if (in_strided(*shape)) return JV_ERR_UNSUPPORTED;      // the feature-map pass reads contiguous q and k
  const size_t lin = align_up(lin_plan(*shape, dwc).total, 256), tb = align_up(tensor_bytes(shape), 256);
  if ((st = check_ws(ws, ws_bytes, lin + 2 * tb)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  void* qf = (char*)ws + lin;
  void* kf = (char*)ws + lin + tb;
  if ((st = from_cuda(launch_focus_map(q, k, qf, kf, *shape, focus_p, stream))) != JV_OK) return st;
  return run_linear(qf, kf, v, o, shape, eps, dwc, ws, stream);
}

jv_status jv_window_attn(const void* q, const void* k, const void* v, void* o, const jv_shape* shape,
                         int32_t win_h, int32_t win_w, float scale, void* ws, size_t ws_bytes,
                         void* cuda_stream) {
  (void)ws; (void)ws_bytes;
  jv_status st = check_shape(shape);
  if (st != JV_OK) return st;
  if ((st = check_tensors(q, k, v, o, shape)) != JV_OK) return st;
  if ((st = check_window(shape, win_h, win_w)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  return run_attn(q, k, v, o, shape, win_h, win_w, scale, false, (cudaStream_t)cuda_stream);
}

jv_status jv_full_attn(const void* q, const void* k, const void* v, void* o, const jv_shape* shape, float scale,
                       void* ws, size_t ws_bytes, void* cuda_stream) {
  (void)ws; (void)ws_bytes;
  jv_status st = check_shape(shape);
  if (st != JV_OK) return st;
  if ((st = check_tensors(q, k, v, o, shape)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  return run_attn(q, k, v, o, shape, shape->Hg, shape->Wg, scale, true, (cudaStream_t)cuda_stream);
}

jv_status jv_hybrid_mixers(int32_t n_layers, const char* schedule, const void* const* q, const void* const* k,
                           const void* const* v, void* const* o, const jv_shape* shape, int32_t win_h,
                           int32_t win_w, float scale, float eps, const jv_dwc* const* dwc, void* ws,
                           size_t ws_bytes, void* cuda_stream) {
  if (n_layers <= 0 || !schedule || !q || !k || !v || !o) return JV_ERR_INVALID_ARG;
  jv_status st = check_shape(shape);
  if (st != JV_OK) return st;
  if (!(eps >= 0.f)) return JV_ERR_INVALID_ARG;
  size_t need = 0;
  bool any_w = false;
  for (int l = 0; l < n_layers; ++l) {
    const char m = schedule[l];
    if (m != 'L' && m != 'W' && m != 'F') return JV_ERR_INVALID_ARG;   // also catches an early '\0'
    if ((st = check_tensors(q[l], k[l], v[l], o[l], shape)) != JV_OK) return st;
    if (m == 'W') any_w = true;
    if (m == 'L') {
      const jv_dwc* d = dwc ? dwc[l] : nullptr;
      if ((st = check_dwc(d)) != JV_OK) return st;
      const size_t n = lin_plan(*shape, d).total;
      if (n > need) need = n;
    }
  }
  if (any_w && (st = check_window(shape, win_h, win_w)) != JV_OK) return st;
  if ((st = check_ws(ws, ws_bytes, need)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  cudaStream_t stream = (cudaStream_t)cuda_stream;
  for (int l = 0; l < n_layers; ++l) {
    switch (schedule[l]) {
      case 'L': st = run_linear(q[l], k[l], v[l], o[l], shape, eps, dwc ? dwc[l] : nullptr, ws, stream); break;
      case 'W': st = run_attn(q[l], k[l], v[l], o[l], shape, win_h, win_w, scale, false, stream); break;
      default:  st = run_attn(q[l], k[l], v[l], o[l], shape, shape->Hg, shape->Wg, scale, true, stream); break;
    }
    if (st != JV_OK) return st;
  }
  return JV_OK;
}

jv_status jv_qkv_proj(const void* x, const void* w, const float* bias, void* q, void* k, void* v,
                      const jv_shape* shape, void* cuda_stream) {
  if (!shape) return JV_ERR_INVALID_ARG;
  const void* ptrs[5] = {x, w, q, k, v};
  const size_t C = (size_t)shape->H * shape->D, nt = (size_t)shape->B * shape_tokens(*shape) * C * 2;
  const size_t bytes[5] = {nt, 3 * C * C * 2, nt, nt, nt};
  jv_status st = check_proj(shape, ptrs, bytes, 5, 2);
  if (st != JV_OK) return st;
  if (bias && !aligned(bias, 16)) return JV_ERR_INVALID_ARG;
  if ((st = check_device()) != JV_OK) return st;
  if (!proj_tc_available()) return JV_ERR_CUDA;
  int* status = device_status_ptr();
  if (!status) return JV_ERR_CUDA;
  return from_cuda(launch_proj_tc(true, x, w, bias, q, k, v, *shape, status, (cudaStream_t)cuda_stream));
}

jv_status jv_out_proj(const void* o, const void* w, const float* bias, void* y, const jv_shape* shape,
                      void* cuda_stream) {
  if (!shape) return JV_ERR_INVALID_ARG;
  const void* ptrs[3] = {o, w, y};
  const size_t C = (size_t)shape->H * shape->D, nt = (size_t)shape->B * shape_tokens(*shape) * C * 2;
  const size_t bytes[3] = {nt, C * C * 2, nt};
  jv_status st = check_proj(shape, ptrs, bytes, 3, 2);
  if (st != JV_OK) return st;
  if (bias && !aligned(bias, 16)) return JV_ERR_INVALID_ARG;
  if ((st = check_device()) != JV_OK) return st;
  if (!proj_tc_available()) return JV_ERR_CUDA;
  int* status = device_status_ptr();
  if (!status) return JV_ERR_CUDA;
  return from_cuda(launch_proj_tc(false, o, w, bias, y, nullptr, nullptr, *shape, status, (cudaStream_t)cuda_stream));
}

jv_status jv_layer_norm(const void* x, const float* w, const float* b, void* y, float* mean, float* rstd,
                        const jv_norm_shape* shape, float eps, void* cuda_stream) {
  jv_status st = check_norm(shape);
  if (st != JV_OK) return st;
  const size_t e = shape->dtype == JV_F32 ? 4 : 2;
  if (!x || !y || (!mean != !rstd) || !(eps >= 0.f)) return JV_ERR_INVALID_ARG;
  if (!aligned(x, e) || !aligned(y, e) || !aligned(w, 4) || !aligned(b, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return JV_ERR_INVALID_ARG;
  const size_t vec = (size_t)shape->C * 4, per_row = (size_t)shape->rows * 4;
  const Span in[3] = {{x, norm_rows_bytes(shape, shape->x_stride)}, {w, vec}, {b, vec}};
  const Span out[3] = {{y, norm_rows_bytes(shape, 0)}, {mean, per_row}, {rstd, per_row}};
  if (outputs_clash(in, 3, out, 3)) return JV_ERR_INVALID_ARG;
  if ((st = check_device()) != JV_OK) return st;
  const NormArgs a{x, nullptr, w, b, y, mean, rstd, shape->rows, shape->x_stride ? shape->x_stride : shape->C, 0, shape->C, shape->dtype, eps};
  return from_cuda(launch_layer_norm(a, (cudaStream_t)cuda_stream));
}

size_t jv_layer_norm_grad_workspace_bytes(const jv_norm_shape* shape) {
  if (check_norm(shape) != JV_OK) return 0;
  return (size_t)layer_norm_grad_blocks(shape->rows, shape->C) * 2 * shape->C * 4;
}

jv_status jv_layer_norm_grad(const void* dy, const void* x, const float* w, const float* mean, const float* rstd, void* dx,
                             float* dw, float* db, const jv_norm_shape* shape, void* ws, size_t ws_bytes, void* cuda_stream) {
  jv_status st = check_norm(shape);
  if (st != JV_OK) return st;
  const size_t e = shape->dtype == JV_F32 ? 4 : 2;
  if (!dy || !x || !mean || !rstd || !dx) return JV_ERR_INVALID_ARG;
  if (!aligned(dy, e) || !aligned(x, e) || !aligned(dx, e) || !aligned(w, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(dw, 4) ||
      !aligned(db, 4))
    return JV_ERR_INVALID_ARG;
  const size_t vec = (size_t)shape->C * 4, per_row = (size_t)shape->rows * 4;
  const size_t need = dw || db ? jv_layer_norm_grad_workspace_bytes(shape) : 0;
  const Span in[5] = {{dy, norm_rows_bytes(shape, shape->dy_stride)}, {x, norm_rows_bytes(shape, shape->x_stride)}, {w, vec}, {mean, per_row}, {rstd, per_row}};
  const Span out[4] = {{dx, norm_rows_bytes(shape, 0)}, {dw, vec}, {db, vec}, {need ? ws : nullptr, need}};
  if (outputs_clash(in, 5, out, 4)) return JV_ERR_INVALID_ARG;
  if ((st = check_ws(ws, ws_bytes, need)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  const NormArgs a{x, dy, w, nullptr, dx, const_cast<float*>(mean), const_cast<float*>(rstd), shape->rows,
                   shape->x_stride ? shape->x_stride : shape->C, shape->dy_stride ? shape->dy_stride : shape->C, shape->C, shape->dtype, 0.f};
  return from_cuda(launch_layer_norm_grad(a, (float*)ws, dw, db, (cudaStream_t)cuda_stream));
}

size_t jv_diff_attn_workspace_bytes(const jv_diff_shape* shape) {
  InStrides qs, ks;
  if (check_diff(shape, &qs, &ks) != JV_OK) return 0;
  if (shape->dtype != JV_BF16 || shape->D != 64) return 0;                // (the fp32 kernel needs none)
  const int pairs = shape->H / 2, kv_pairs = shape->Hkv / 2;
  const size_t tiles = diff_tc_plan(shape->B, pairs, shape->Nq, shape->Nk).total;
  const size_t rows = diff_rows_plan(shape->B, kv_pairs, shape->Nk).total;
  return (int64_t)(pairs / kv_pairs) * shape->Nq <= 16 ? rows : tiles;
}

jv_status jv_diff_attn(const void* q, const void* k, const void* v, void* o, const jv_diff_shape* shape, const jv_diff* diff,
                       float scale, void* ws, size_t ws_bytes, void* cuda_stream) {
  InStrides qs, ks;
  jv_status st = check_diff(shape, &qs, &ks);
  if (st != JV_OK) return st;
  if (!q || !k || !v || !o || !diff || !diff->lambda) return JV_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16)) return JV_ERR_INVALID_ARG;
  if (!aligned(diff->lambda, 4) || !aligned(diff->norm_w, 16) || !aligned(diff->kv_len, 4) || !aligned(diff->q_pos, 4)) return JV_ERR_INVALID_ARG;
  if (!isfinite(diff->lambda_init) || (diff->norm_w && !(diff->norm_eps >= 0.f))) return JV_ERR_INVALID_ARG;
  const int B = shape->B, D = shape->D;
  const size_t e = shape->dtype == JV_F32 ? 4 : 2, need = jv_diff_attn_workspace_bytes(shape), nkv = diff_bytes(ks, B, shape->Hkv, shape->Nk, D, e);
  const Span in[7] = {{q, diff_bytes(qs, B, shape->H, shape->Nq, D, e)}, {k, nkv}, {v, nkv}, {diff->lambda, (size_t)16 * D},
                      {diff->norm_w, (size_t)8 * D}, {diff->kv_len, (size_t)4 * B}, {diff->q_pos, (size_t)4 * B}};
  const Span out[2] = {{o, (size_t)B * shape->H * shape->Nq * D * e}, {need ? ws : nullptr, need}};
  if (outputs_clash(in, 7, out, 2)) return JV_ERR_INVALID_ARG;
  if ((st = check_ws(ws, ws_bytes, need)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  const DiffArgs a{q, k, v, o, B, shape->H / 2, shape->Hkv / 2, shape->Nq, shape->Nk, D, shape->dtype, shape->causal != 0, qs, ks,
                   diff->lambda, diff->lambda_init, diff->norm_w, diff->norm_eps, diff->kv_len, diff->q_pos, pick_scale(scale, D)};
  if (!g_force_generic.load() && diff_tc_supported(a)) {
    int* status = device_status_ptr();
    if (!status) return JV_ERR_CUDA;
    return from_cuda(diff_rows_supported(a) ? launch_diff_rows(a, ws, status, (cudaStream_t)cuda_stream)
                                            : launch_diff_tc(a, ws, status, (cudaStream_t)cuda_stream));
  }
  return from_cuda(launch_diff_generic(a, (cudaStream_t)cuda_stream));
}

jv_status jv_causal_conv(const void* x, const float* w, const float* bias, const void* state_in, void* u, void* state_out,
                         const int32_t* lens, const jv_conv_shape* shape, void* cuda_stream) {
  Rows xs;
  jv_status st = check_conv(shape, &xs);
  if (st != JV_OK) return st;
  const size_t e = shape->dtype == JV_F32 ? 4 : 2;
  if (!x || !w || !u) return JV_ERR_INVALID_ARG;
  if (!aligned(x, e) || !aligned(u, e) || !aligned(state_in, e) || !aligned(state_out, e) || !aligned(w, 4) || !aligned(bias, 4) || !aligned(lens, 4))
    return JV_ERR_INVALID_ARG;
  const int B = shape->B, L = shape->L, C = shape->C, K = shape->K;
  const size_t state = (size_t)B * (K - 1) * C * e;
  const Span in[5] = {{x, token_rows_bytes(B, L, xs, C, e)}, {w, (size_t)C * K * 4}, {bias, (size_t)C * 4}, {lens, (size_t)B * 4},
                      {state_in == state_out ? nullptr : state_in, state}};
  const Span out[2] = {{u, (size_t)B * L * C * e}, {state_out, state}};
  if (outputs_clash(in, 5, out, 2) || (state_in && overlaps(u, out[0].bytes, state_in, state))) return JV_ERR_INVALID_ARG;
  if ((st = check_device()) != JV_OK) return st;
  const ConvArgs a{x, w, bias, state_in, u, state_out, lens, B, L, C, K, shape->dtype, shape->silu, xs};
  return from_cuda(launch_causal_conv(a, (cudaStream_t)cuda_stream));
}

size_t jv_selective_scan_workspace_bytes(const jv_scan_shape* shape) {
  ScanRows r;
  if (check_scan(shape, &r) != JV_OK) return 0;
  return scan_plan(shape->B, shape->L, shape->C, shape->Ns).total;
}

jv_status jv_selective_scan(const void* u, const void* dt, const float* A, const void* Bm, const void* Cm, const float* D,
                            const void* z, const float* dt_bias, const float* state_in, void* y, float* state_out,
                            const int32_t* lens, const jv_scan_shape* shape, void* ws, size_t ws_bytes, void* cuda_stream) {
  ScanRows r;
  jv_status st = check_scan(shape, &r);
  if (st != JV_OK) return st;
  const size_t e = shape->dtype == JV_F32 ? 4 : 2;
  if (!u || !dt || !A || !Bm || !Cm || !y) return JV_ERR_INVALID_ARG;
  for (const void* p : {u, dt, Bm, Cm, z, (const void*)y})
    if (!aligned(p, e)) return JV_ERR_INVALID_ARG;
  for (const void* p : {(const void*)A, (const void*)D, (const void*)dt_bias, (const void*)state_in, (const void*)state_out, (const void*)lens})
    if (!aligned(p, 4)) return JV_ERR_INVALID_ARG;
  const int B = shape->B, L = shape->L, C = shape->C, Ns = shape->Ns;
  const size_t state = (size_t)B * C * Ns * 4;
  const ScanPlan plan = scan_plan(B, L, C, Ns);
  const Span in[10] = {{u, token_rows_bytes(B, L, r.u, C, e)}, {dt, token_rows_bytes(B, L, r.dt, C, e)}, {Bm, token_rows_bytes(B, L, r.b, Ns, e)},
                       {Cm, token_rows_bytes(B, L, r.c, Ns, e)}, {z, token_rows_bytes(B, L, r.z, C, e)}, {A, (size_t)C * Ns * 4},
                       {D, (size_t)C * 4}, {dt_bias, (size_t)C * 4}, {lens, (size_t)B * 4}, {state_in == state_out ? nullptr : state_in, state}};
  const Span out[3] = {{y, (size_t)B * L * C * e}, {state_out, state}, {plan.total ? ws : nullptr, plan.total}};
  if (outputs_clash(in, 10, out, 3)) return JV_ERR_INVALID_ARG;
  if (state_in && (overlaps(y, out[0].bytes, state_in, state) || (out[2].p && overlaps(ws, plan.total, state_in, state)))) return JV_ERR_INVALID_ARG;
  if ((st = check_ws(ws, ws_bytes, plan.total)) != JV_OK) return st;
  if ((st = check_device()) != JV_OK) return st;
  const ScanArgs a{u, dt, Bm, Cm, z, A, D, dt_bias, state_in, state_out, y, lens, B, L, C, Ns, shape->dtype, shape->softplus, r.u, r.dt, r.b, r.c, r.z};
  return from_cuda(launch_selective_scan(a, plan, ws, (cudaStream_t)cuda_stream));
}

jv_status jv_device_status(void* cuda_stream) {
  if (cudaStreamSynchronize((cudaStream_t)cuda_stream) != cudaSuccess) { cudaGetLastError(); return JV_ERR_CUDA; }
  int word = 0;
  if (cudaMemcpyFromSymbol(&word, g_status_word, sizeof(int)) != cudaSuccess) { cudaGetLastError(); return JV_ERR_CUDA; }
  if (word != 0) {
    const int zero = 0;
    cudaMemcpyToSymbol(g_status_word, &zero, sizeof(int));
    return JV_ERR_TIMEOUT;
  }
  return JV_OK;
}

int32_t jv_set_force_generic(int32_t on) { return g_force_generic.exchange(on ? 1 : 0); }

uint64_t jv_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

const char* jv_status_string(jv_status s) {
  switch (s) {
    case JV_OK: return "ok";
    case JV_ERR_INVALID_ARG: return "invalid argument";
    case JV_ERR_UNSUPPORTED: return "unsupported shape, dtype or device";
    case JV_ERR_WORKSPACE: return "workspace missing, misaligned or too small";
    case JV_ERR_CUDA: return "CUDA call failed";
    case JV_ERR_TIMEOUT: return "a kernel gave up on a bounded wait";
    default: return "unknown status";
  }
}

const char* jv_version(void) { return "jetvit-b200 0.1.0 (sm_100a)"; }

}  // extern "C"

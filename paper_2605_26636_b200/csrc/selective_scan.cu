// The selective scan of a state-space mixer: every channel carries Ns states through its sequence.
//   d_t = softplus(dt_t + dt_bias),  h_t = exp(d_t A) h_(t-1) + d_t B_t u_t,  y_t = (C_t . h_t + D u_t) z_t / (1 + exp(-z_t))
//
// Four lanes share a channel, a quarter of its states each in registers; a warp has 8 channels, a block 64.  Tiles of 32 tokens of u, dt, z, B, C
// pass through shared memory (the next one's loads are in flight meanwhile), where d_t and d_t u_t are formed once per token
// and channel.  Four tokens at a time: the lanes' shares of four y are exchanged so that every lane ends up with the sum of one.
//
// What bounds it: the exponentials, Ns a token and channel on the MUFU unit (16 a clock and SM), three times what
// the bytes take at Ns = 16 in bf16.
//
// A sequence is cut into chunks where the channels alone leave SMs idle: one pass for the chunks' own states from zero, a
// second that carries the state from chunk to chunk (h_end = exp(A sum d) h_begin + own), a third like the single pass, from
// the states that the second left.
#include "scan.cuh"

namespace jv {
namespace {

constexpr int kCh = 64;               // channels of a block
constexpr int kLanes = 4;             // lanes of a channel
constexpr int kThreads = kCh * kLanes;
constexpr int kTT = 32;               // tokens of a tile
constexpr int kStepTokens = 4;        // calls of at most this many tokens walk without tiles
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float softplus(float x) { return x > 20.f ? x : log1pf(__expf(x)); }
__device__ __forceinline__ float silu(float x) { return x / (1.f + __expf(-x)); }

__device__ __forceinline__ int length_of(const ScanArgs& a, int b) { return a.lens ? min(max(__ldg(a.lens + b), 0), a.L) : a.L; }

// A channel's coefficients and states: state n of lane s is s * NPL + n; states past Ns are zeros all through
template <int NPL>
__device__ __forceinline__ void load_A(const ScanArgs& a, int c, int s, float (&A2)[NPL]) {
#pragma unroll
  for (int n = 0; n < NPL; ++n) A2[n] = s * NPL + n < a.Ns ? __ldg(a.A + (int64_t)c * a.Ns + s * NPL + n) * kLog2e : 0.f;
}
template <int NPL>
__device__ __forceinline__ void load_state(const float* h, int Ns, int s, float (&st)[NPL]) {
#pragma unroll
  for (int n = 0; n < NPL; ++n) st[n] = h && s * NPL + n < Ns ? h[s * NPL + n] : 0.f;
}
template <int NPL>
__device__ __forceinline__ void store_state(float* h, int Ns, int s, const float (&st)[NPL]) {
#pragma unroll
  for (int n = 0; n < NPL; ++n)
    if (s * NPL + n < Ns) h[s * NPL + n] = st[n];
}

// ---- a few tokens: straight from global memory ------------------------------------------------------------------------
template <typename T, int NPL>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(const ScanArgs a) {
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.y, c = blockIdx.x * kCh + (int)threadIdx.x / kLanes, s = threadIdx.x % kLanes;
  const int cc = min(c, a.C - 1);                      // (lanes past the last channel follow it: the sums need whole warps)
  const int64_t ch = (int64_t)b * a.C + cc;
  const int len = length_of(a, b);
  float A2[NPL], h[NPL];
  load_A<NPL>(a, cc, s, A2);
  load_state<NPL>(a.h_in ? a.h_in + ch * a.Ns : nullptr, a.Ns, s, h);
  const float bias = a.dt_bias ? __ldg(a.dt_bias + cc) : 0.f, D = a.D ? __ldg(a.D + cc) : 0.f;
  for (int t = 0; t < len; ++t) {
    const float u = to_f32(((const T*)a.u)[a.us.at(b, t) + cc]);
    float d = to_f32(((const T*)a.dt)[a.ds.at(b, t) + cc]) + bias;
    if (a.softplus) d = softplus(d);
    const float du = d * u;
    float y = 0.f;
#pragma unroll
    for (int n = 0; n < NPL; ++n) {
      const int i = s * NPL + n;
      const float bm = i < a.Ns ? to_f32(((const T*)a.Bm)[a.bs.at(b, t) + i]) : 0.f;
      const float cm = i < a.Ns ? to_f32(((const T*)a.Cm)[a.cs.at(b, t) + i]) : 0.f;
      h[n] = fmaf(ex2(d * A2[n]), h[n], du * bm);
      y = fmaf(h[n], cm, y);
    }
    y += __shfl_xor_sync(0xffffffffu, y, 1);
    y += __shfl_xor_sync(0xffffffffu, y, 2);
    if (s == 0 && c < a.C) {
      y = fmaf(D, u, y);
      if (a.z) y *= silu(to_f32(((const T*)a.z)[a.zs.at(b, t) + c]));
      from_f32((T*)a.y + ((int64_t)b * a.L + t) * a.C + c, y);
    }
  }
  if (a.h_out && c < a.C) store_state<NPL>(a.h_out + ch * a.Ns, a.Ns, s, h);
}

// ---- tiles of tokens ------------------------------------------------------------------------------------------------------
template <typename T, int NPL>
struct Smem {
  float d[kTT][kCh], du[kTT][kCh];
  float Bm[kTT][kLanes * NPL], Cm[kTT][kLanes * NPL];
  T u[kTT][kCh], z[kTT][kCh];         // u: y takes its place
};

// kY: the whole thing; else the chunk's own state from zero and the sum of its steps only
template <typename T, int NPL, bool WIDE, bool kY>
__global__ void __launch_bounds__(kThreads) scan_kernel(const ScanArgs a, int chunk, int nchunk, float* ws_state, float* ws_sum) {
  constexpr int kVec = WIDE ? 16 / sizeof(T) : 1;             // elements of a load
  constexpr int kLoads = kTT * kCh / kThreads / kVec;         // loads of a thread and tile from each of u, dt, z
  constexpr int kRow = kCh / kVec;                            // loads of a token
  constexpr int kNs = kLanes * NPL;
  constexpr int kBC = (kTT * kNs + kThreads - 1) / kThreads;  // elements of a thread and tile from each of B, C
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Smem<T, NPL>& sm = *reinterpret_cast<Smem<T, NPL>*>(smem_raw);
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.z, ck = blockIdx.y, c0 = blockIdx.x * kCh, tid = threadIdx.x;
  const int lc = tid / kLanes, s = tid % kLanes, c = c0 + lc, cc = min(c, a.C - 1);
  const int len = length_of(a, b);
  const int t_begin = ck * chunk, t_end = min(t_begin + chunk, len);
  const int64_t ch = ((int64_t)b * nchunk + ck) * a.C + cc;    // of the workspace's arrays
  float A2[NPL], h[NPL], sum = 0.f;
  load_A<NPL>(a, cc, s, A2);
  if (kY && nchunk > 1) load_state<NPL>(ws_state + ch * a.Ns, a.Ns, s, h);
  else load_state<NPL>(kY && a.h_in ? a.h_in + ((int64_t)b * a.C + cc) * a.Ns : nullptr, a.Ns, s, h);
  const float D = a.D ? __ldg(a.D + cc) : 0.f;

  using Raw = typename std::conditional<WIDE, uint4, T>::type;
  Raw ru[kLoads], rd[kLoads], rz[kLoads];
  T rb[kBC], rc[kBC];
  auto fetch = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int e = i * kThreads + tid, t = t0 + e / kRow, col = c0 + (e % kRow) * kVec;
      const bool in = t < t_end && col < a.C;                  // (16 bytes at a time: C is a multiple of them)
      Raw zero;
      memset(&zero, 0, sizeof(Raw));
      ru[i] = in ? *reinterpret_cast<const Raw*>((const T*)a.u + a.us.at(b, t) + col) : zero;
      rd[i] = in ? *reinterpret_cast<const Raw*>((const T*)a.dt + a.ds.at(b, t) + col) : zero;
      if (kY) rz[i] = in && a.z ? *reinterpret_cast<const Raw*>((const T*)a.z + a.zs.at(b, t) + col) : zero;
    }
#pragma unroll
    for (int i = 0; i < kBC; ++i) {
      const int e = i * kThreads + tid, t = t0 + e / kNs, n = e % kNs;
      const bool in = t < t_end && n < a.Ns && e < kTT * kNs;
      rb[i] = in ? ((const T*)a.Bm)[a.bs.at(b, t) + n] : T(0.f);
      if (kY) rc[i] = in ? ((const T*)a.Cm)[a.cs.at(b, t) + n] : T(0.f);
    }
  };
  auto put = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int e = i * kThreads + tid, t = e / kRow, col = (e % kRow) * kVec;
      T uu[kVec], dd[kVec];
      memcpy(uu, &ru[i], sizeof(Raw));
      memcpy(dd, &rd[i], sizeof(Raw));
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        float d = 0.f;                                          // a token past the end: exp(0) h + 0
        if (t0 + t < t_end) {
          d = to_f32(dd[v]) + (a.dt_bias ? __ldg(a.dt_bias + min(c0 + col + v, a.C - 1)) : 0.f);
          if (a.softplus) d = softplus(d);
        }
        sm.d[t][col + v] = d;
        sm.du[t][col + v] = d * to_f32(uu[v]);
      }
      if (kY) {
        *reinterpret_cast<Raw*>(&sm.u[t][col]) = ru[i];
        *reinterpret_cast<Raw*>(&sm.z[t][col]) = rz[i];
      }
    }
#pragma unroll
    for (int i = 0; i < kBC; ++i) {
      const int e = i * kThreads + tid;
      if (e < kTT * kNs) {
        sm.Bm[e / kNs][e % kNs] = to_f32(rb[i]);
        if (kY) sm.Cm[e / kNs][e % kNs] = to_f32(rc[i]);
      }
    }
  };
  auto flush = [&](int t0) {                                    // the tile of y to global memory
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int e = i * kThreads + tid, t = e / kRow, col = (e % kRow) * kVec;
      if (t0 + t < t_end && c0 + col < a.C)
        *reinterpret_cast<Raw*>((T*)a.y + ((int64_t)b * a.L + t0 + t) * a.C + c0 + col) = *reinterpret_cast<const Raw*>(&sm.u[t][col]);
    }
  };

  if (t_begin < t_end) fetch(t_begin);
  for (int t0 = t_begin; t0 < t_end; t0 += kTT) {
    put(t0);
    __syncthreads();
    if (t0 + kTT < t_end) fetch(t0 + kTT);
#pragma unroll 2
    for (int t = 0; t < kTT; t += kLanes) {
      float y[kLanes];
#pragma unroll
      for (int j = 0; j < kLanes; ++j) {
        const float d = sm.d[t + j][lc], du = sm.du[t + j][lc];
        y[j] = 0.f;
        if (!kY) sum += d;
#pragma unroll
        for (int n = 0; n < NPL; ++n) {
          h[n] = fmaf(ex2(d * A2[n]), h[n], du * sm.Bm[t + j][s * NPL + n]);
          if (kY) y[j] = fmaf(h[n], sm.Cm[t + j][s * NPL + n], y[j]);
        }
      }
      if (kY) {
        // lanes s and s ^ 1 exchange: an even one keeps tokens 0 and 2, an odd one 1 and 3; then s and s ^ 2
        const float a0 = (s & 1) ? y[1] : y[0], a1 = (s & 1) ? y[3] : y[2], o0 = (s & 1) ? y[0] : y[1], o1 = (s & 1) ? y[2] : y[3];
        const float p0 = a0 + __shfl_xor_sync(0xffffffffu, o0, 1), p1 = a1 + __shfl_xor_sync(0xffffffffu, o1, 1);
        float r = (s & 2) ? p1 : p0;
        r += __shfl_xor_sync(0xffffffffu, (s & 2) ? p0 : p1, 2);   // token t + s
        r = fmaf(D, to_f32(sm.u[t + s][lc]), r);
        if (a.z) r *= silu(to_f32(sm.z[t + s][lc]));
        from_f32(&sm.u[t + s][lc], r);
      }
    }
    __syncthreads();
    if (kY) flush(t0);                                          // (a thread reads and refills the same places of u)
  }
  if (c >= a.C) return;
  if (kY) {
    // the state behind the last token: by the chunk that has it, the first one of an empty sequence
    if (a.h_out && (t_begin < t_end ? t_end == len : len == 0 && ck == 0)) store_state<NPL>(a.h_out + ((int64_t)b * a.C + c) * a.Ns, a.Ns, s, h);
  } else {
    store_state<NPL>(ws_state + ch * a.Ns, a.Ns, s, h);
    if (s == 0) ws_sum[ch] = sum;
  }
}

// State from chunk to chunk, in place: a chunk's own state out, the state that it begins with in
__global__ void __launch_bounds__(256) scan_carry_kernel(const ScanArgs a, int nchunk, float* ws_state, const float* ws_sum) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)a.C * a.Ns;
  const int b = (int)(id / per);
  if (b >= a.B) return;
  const int64_t e = id - b * per;
  const int c = (int)(e / a.Ns);
  const float A2 = __ldg(a.A + e) * kLog2e;
  float h = a.h_in ? a.h_in[b * per + e] : 0.f;
  for (int k = 0; k < nchunk; ++k) {
    float* st = ws_state + ((int64_t)b * nchunk + k) * per + e;
    const float own = *st, sum = ws_sum[((int64_t)b * nchunk + k) * a.C + c];
    *st = h;
    h = fmaf(ex2(sum * A2), h, own);
  }
}

template <typename T, int NPL, bool WIDE>
cudaError_t launch_tiles(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  const dim3 grid((unsigned)ceil_div(a.C, kCh), (unsigned)p.nchunk, (unsigned)a.B);
  const size_t smem = sizeof(Smem<T, NPL>);
  static OncePerDevice opt_in;
  cudaError_t e = opt_in.run([] {
    const cudaError_t r = cudaFuncSetAttribute(scan_kernel<T, NPL, WIDE, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<T, NPL>));
    return r != cudaSuccess ? r : cudaFuncSetAttribute(scan_kernel<T, NPL, WIDE, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem<T, NPL>));
  });
  if (e != cudaSuccess) return e;
  float* state = p.nchunk > 1 ? (float*)((char*)ws + p.off_state) : nullptr;
  float* sum = p.nchunk > 1 ? (float*)((char*)ws + p.off_sum) : nullptr;
  if (p.nchunk > 1) {
    e = launch_programmatic(scan_kernel<T, NPL, WIDE, false>, grid, kThreads, smem, st, a, p.chunk, p.nchunk, state, sum);
    if (e != cudaSuccess) return e;
    const int64_t n = (int64_t)a.B * a.C * a.Ns;
    e = launch_programmatic(scan_carry_kernel, dim3((unsigned)((n + 255) / 256)), 256, 0, st, a, p.nchunk, state, (const float*)sum);
    if (e != cudaSuccess) return e;
  }
  return launch_programmatic(scan_kernel<T, NPL, WIDE, true>, grid, kThreads, smem, st, a, p.chunk, p.nchunk, state, sum);
}

template <typename T, int NPL>
cudaError_t launch_states(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  if (a.L <= kStepTokens) return launch_programmatic(scan_step_kernel<T, NPL>, dim3((unsigned)ceil_div(a.C, kCh), (unsigned)a.B), kThreads, 0, st, a);
  const size_t e = sizeof(T);
  const bool wide = ((uintptr_t)a.u | (uintptr_t)a.dt | (uintptr_t)a.z | (uintptr_t)a.y | a.C * e | a.us.tok * e | a.us.batch * e |
                     a.ds.tok * e | a.ds.batch * e | (a.z ? (a.zs.tok | a.zs.batch) * e : 0)) % 16 == 0;
  return wide ? launch_tiles<T, NPL, true>(a, p, ws, st) : launch_tiles<T, NPL, false>(a, p, ws, st);
}

template <typename T>
cudaError_t launch_type(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  const int npl = ceil_div(a.Ns, kLanes);
  if (npl <= 1) return launch_states<T, 1>(a, p, ws, st);
  if (npl <= 2) return launch_states<T, 2>(a, p, ws, st);
  if (npl <= 4) return launch_states<T, 4>(a, p, ws, st);
  if (npl <= 8) return launch_states<T, 8>(a, p, ws, st);
  return launch_states<T, 16>(a, p, ws, st);
}

}  // namespace

ScanPlan scan_plan(int B, int L, int C, int Ns) {
  ScanPlan p{1, L, 0, 0, 0};
  if (L <= kStepTokens) return p;
  // one pass where the channels give every SM a block; else chunks (which walk the exponentials twice) for two blocks an SM
  const int64_t blocks = (int64_t)B * ceil_div(C, kCh), sms = device_sm_count();
  if (blocks < sms / 2) {
    const int want = (int)(2 * sms / blocks), tiles = ceil_div(L, kTT);
    p.chunk = ceil_div(tiles, want < tiles ? want : tiles) * kTT;
    p.nchunk = ceil_div(L, p.chunk);
  }
  if (p.nchunk > 1) {
    p.off_sum = align_up((size_t)B * p.nchunk * C * Ns * 4, 256);
    p.total = p.off_sum + (size_t)B * p.nchunk * C * 4;
  }
  return p;
}

cudaError_t launch_selective_scan(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  return a.dtype == JV_F32 ? launch_type<float>(a, p, ws, st) : launch_type<__nv_bfloat16>(a, p, ws, st);
}

}  // namespace jv

// The short causal convolution of a state-space mixer: every channel on its own, over the token and the K - 1 before it.
//   u_t = act(b + sum_j w_j x_(t - K + 1 + j)),  act = x / (1 + exp(-x)) or nothing;   state: the last K - 1 inputs
//
// x is read once and u written once; what bounds it is not HBM yet but instructions and latency (half of the issue slots: every token
// moves the past ones on by a register each; four loads of a thread in flight).  2 x 4096 tokens of 2048 channels 24 us in bf16 (its
// bytes: 10.2), 26.6 in fp32 (20.5).  A thread owns 16 bytes of channels and a run of tokens, which it walks with
// the last K - 1 inputs in registers; neighbouring threads own neighbouring channels.  The K - 1 inputs ahead of a run
// come from the run before (L2 has them), those ahead of the first from the state.  The new state is written by the thread of the
// first run, the only one that reads the old one: both may be the same memory.
#include "scan.cuh"

namespace jv {
namespace {

// VEC consecutive values as they lie in memory
template <typename T, int VEC, typename Raw>
__device__ __forceinline__ void widen(const Raw& r, float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    f[0] = to_f32(r);
  } else {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        f[i] = __uint_as_float(u[i]);
      } else {
        f[2 * i] = __uint_as_float(u[i] << 16);
        f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      }
    }
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, float (&f)[VEC]) {
  if constexpr (VEC == 1) widen<T, VEC>(*p, f);
  else widen<T, VEC>(*reinterpret_cast<const uint4*>(p), f);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    from_f32(p, f[0]);
  } else {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        u[i] = __float_as_uint(f[i]);
      } else {
        const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&t);
      }
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  }
}

constexpr int kThreads = 128;
constexpr int kAhead = 4;            // tokens whose loads are in flight together; runs are multiples of it, and no shorter than K - 1

template <typename T, int VEC, int K>
__global__ void __launch_bounds__(kThreads, VEC == 8 ? 4 : 1) causal_conv_kernel(const ConvArgs a, int run, int runs) {
  griddep_wait();
  griddep_launch_dependents();
  const int ncv = a.C / VEC;
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t br = id / ncv;
  if (br >= (int64_t)a.B * runs) return;
  const int c = (int)(id - br * ncv) * VEC, b = (int)(br / runs), r = (int)(br - (int64_t)b * runs);
  const int len = a.lens ? min(max(__ldg(a.lens + b), 0), a.L) : a.L;
  const int t0 = r * run, t1 = min(t0 + run, len);
  if (r > 0 && t0 >= t1) return;
  const T* x = (const T*)a.x + a.xs.at(b, 0) + c;
  T* u = (T*)a.u + (int64_t)b * a.L * a.C + c;
  const T* s_in = a.s_in ? (const T*)a.s_in + (int64_t)b * (K - 1) * a.C + c : nullptr;
  float past[K - 1][VEC];                          // the inputs ahead of the token in turn
#pragma unroll
  for (int j = 0; j < K - 1; ++j) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) past[j][i] = 0.f;
    if (r > 0) load_vec<T, VEC>(x + (int64_t)(t0 - (K - 1) + j) * a.xs.tok, past[j]);
    else if (s_in) load_vec<T, VEC>(s_in + (int64_t)j * a.C, past[j]);
  }
  float w[VEC][K], bias[VEC];                      // (a thread's filters are VEC * K consecutive values: 16 bytes at a time)
  if constexpr (VEC > 1) {
    float f[VEC * K];
#pragma unroll
    for (int i = 0; i < VEC * K; i += 4) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(a.w + (int64_t)c * K + i));
      f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i)
#pragma unroll
      for (int j = 0; j < K; ++j) w[i][j] = f[i * K + j];
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const float4 v = a.b ? __ldg(reinterpret_cast<const float4*>(a.b + c + i)) : make_float4(0.f, 0.f, 0.f, 0.f);
      bias[i] = v.x; bias[i + 1] = v.y; bias[i + 2] = v.z; bias[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < K; ++j) w[0][j] = __ldg(a.w + (int64_t)c * K + j);
    bias[0] = a.b ? __ldg(a.b + c) : 0.f;
  }
  // kAhead tokens in turn, as they lie in memory, and the next kAhead on their way
  using Raw = typename std::conditional<VEC == 1, T, uint4>::type;
  Raw now[kAhead], next[kAhead];
  auto fetch = [&](Raw (&q)[kAhead], int t) {
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (t + n < t1) q[n] = *reinterpret_cast<const Raw*>(x + (int64_t)(t + n) * a.xs.tok);
  };
  if (t0 < t1) fetch(now, t0);
  for (int t = t0; t < t1; t += kAhead) {
    fetch(next, t + kAhead);
#pragma unroll
    for (int n = 0; n < kAhead; ++n)
      if (t + n < t1) {
        float in[VEC], o[VEC];
        widen<T, VEC>(now[n], in);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          float s = bias[i];
#pragma unroll
          for (int j = 0; j < K - 1; ++j) s = fmaf(w[i][j], past[j][i], s);
          s = fmaf(w[i][K - 1], in[i], s);
          o[i] = a.silu ? __fdividef(s, 1.f + __expf(-s)) : s;
#pragma unroll
          for (int j = 0; j + 1 < K - 1; ++j) past[j][i] = past[j + 1][i];
          past[K - 2][i] = in[i];
        }
        store_vec<T, VEC>(u + (int64_t)(t + n) * a.C, o);
      }
#pragma unroll
    for (int n = 0; n < kAhead; ++n) now[n] = next[n];
  }
  if (r == 0 && a.s_out) {
    T* s_out = (T*)a.s_out + (int64_t)b * (K - 1) * a.C + c;
    // Row j: token len - (K - 1) + j, or row len + j of the old state where that is before the first.  In ascending order, so that a
    // state in its own place is read ahead of the rows that are written.
    for (int j = 0; j < K - 1; ++j) {
      float f[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) f[i] = 0.f;
      if (len + j >= K - 1) load_vec<T, VEC>(x + (int64_t)(len + j - (K - 1)) * a.xs.tok, f);
      else if (s_in) load_vec<T, VEC>(s_in + (int64_t)(len + j) * a.C, f);
      store_vec<T, VEC>(s_out + (int64_t)j * a.C, f);
    }
  }
}

template <typename T, int VEC>
cudaError_t launch(const ConvArgs& a, cudaStream_t st) {
  const int ncv = a.C / VEC;
  // Runs of 32 tokens (the K - 1 tokens ahead of a run are read again), shorter ones until every SM has 256 threads.  Measured with 1024 / 512 /
  // 256: 2 x 4096 tokens of 2048 channels 29 / 25 / 24 us, 8 x 2048 47 / 41 / 42, 1 x 4096 20 / 16 / 14.
  int run = 32;
  while (run > kAhead && (int64_t)a.B * ceil_div(a.L, run) * ncv < 256ll * device_sm_count()) run /= 2;
  const int runs = ceil_div(a.L, run);
  const int64_t blocks = ((int64_t)a.B * runs * ncv + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)blocks);
  switch (a.K) {
    case 2: return launch_programmatic(causal_conv_kernel<T, VEC, 2>, grid, kThreads, 0, st, a, run, runs);
    case 3: return launch_programmatic(causal_conv_kernel<T, VEC, 3>, grid, kThreads, 0, st, a, run, runs);
    default: return launch_programmatic(causal_conv_kernel<T, VEC, 4>, grid, kThreads, 0, st, a, run, runs);
  }
}

}  // namespace

cudaError_t launch_causal_conv(const ConvArgs& a, cudaStream_t st) {
  const size_t e = a.dtype == JV_F32 ? 4 : 2;
  const bool wide = ((uintptr_t)a.x | (uintptr_t)a.u | (uintptr_t)a.s_in | (uintptr_t)a.s_out | (uintptr_t)a.w | (uintptr_t)a.b | a.C * e | a.xs.tok * e | a.xs.batch * e) % 16 == 0;
  if (a.dtype == JV_F32) return wide ? launch<float, 4>(a, st) : launch<float, 1>(a, st);
  return wide ? launch<__nv_bfloat16, 8>(a, st) : launch<__nv_bfloat16, 1>(a, st);
}

}  // namespace jv

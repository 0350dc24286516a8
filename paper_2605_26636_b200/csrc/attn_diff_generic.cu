// Differential attention for what has no kernel of its own: f32 tensors, and bf16 ones with D other than 64.  One warp per query row and
// pair, fp32 arithmetic: a lane takes a key of 32 for the scores of both maps, then 2 D / 32 channels for the products.
#include "attn_diff.cuh"

namespace jv {
namespace {

using namespace diff;

constexpr int kRowWarps = 4;
constexpr int kMaxD = 64;

template <typename T>
__device__ __forceinline__ void load16(const T* p, float (&f)[16 / sizeof(T)]) {
  const uint4 r = __ldg(reinterpret_cast<const uint4*>(p));
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

// the larger; no number if one of them is none
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}

template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) diff_generic_kernel(const DiffArgs a) {
  __shared__ float sq[kRowWarps][2][kMaxD];
  griddep_wait();
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = blockIdx.x * kRowWarps + warp, b = blockIdx.y / a.pairs, p = blockIdx.y % a.pairs;
  if (i >= a.Nq) return;
  const int g = p / (a.pairs / a.kv_pairs), D = a.D;
  const T* q = (const T*)a.q + b * a.qs.batch + i * a.qs.tok;
  const T* k = (const T*)a.k + b * a.ks.batch + 2 * g * a.ks.head;
  const T* v = (const T*)a.v + b * a.ks.batch + 2 * g * a.ks.head;
  for (int c = lane; c < 2 * D; c += 32) sq[warp][c / D][c % D] = to_f32(q[(2 * p + c / D) * a.qs.head + c % D]);
  __syncwarp();
  const float lam = lambda_of(Tail{a.lambda, a.lambda_init, a.norm_w, a.norm_eps, D});
  const int limit = reach_of(a.kv_len, a.q_pos, b, a.Nq, a.Nk, a.causal).limit(i);
  const float sl2 = a.scale * 1.4426950408889634f;
  constexpr int kPer = 2 * kMaxD / 32;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, acc[2][kPer] = {};
  for (int j0 = 0; j0 < limit; j0 += 32) {
    float pr[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float s = -INFINITY;
      if (j0 + lane < limit) {
        const T* kr = k + (int64_t)(j0 + lane) * a.ks.tok + h * a.ks.head;
        s = 0.f;
        for (int c = 0; c < D; c += 16 / sizeof(T)) {
          float f[16 / sizeof(T)];
          load16(kr + c, f);
#pragma unroll
          for (int x = 0; x < (int)(16 / sizeof(T)); ++x) s = fmaf(f[x], sq[warp][h][c + x], s);
        }
        s *= sl2;
      }
      float mx = s;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float mn = max_nan(m[h], mx), ref = mn == -INFINITY ? 0.f : mn;       // no key of weight so far: weight 0, not NaN
      const float alpha = exp2f(m[h] - ref);
      m[h] = mn;
      pr[h] = exp2f(s - ref);
      l[h] = l[h] * alpha + warp_sum(pr[h]);
#pragma unroll
      for (int x = 0; x < kPer; ++x) acc[h][x] *= alpha;
    }
    const int nk = min(32, limit - j0);
    for (int j = 0; j < nk; ++j) {
      const T* vr = v + (int64_t)(j0 + j) * a.ks.tok;
      const float p0 = __shfl_sync(0xffffffffu, pr[0], j), p1 = __shfl_sync(0xffffffffu, pr[1], j);
#pragma unroll
      for (int x = 0; x < kPer; ++x) {
        const int c = lane + 32 * x;
        if (c < 2 * D) {
          const float f = to_f32(vr[(c / D) * a.ks.head + c % D]);
          acc[0][x] = fmaf(p0, f, acc[0][x]);
          acc[1][x] = fmaf(p1, f, acc[1][x]);
        }
      }
    }
  }
  // a row that sees no key is 0; one whose keys all weigh nothing is no number (0 / 0)
  float x[kPer], ss = 0.f;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    x[j] = limit > 0 ? acc[0][j] / l[0] - lam * (acc[1][j] / l[1]) : 0.f;
    if (lane + 32 * j < 2 * D) ss = fmaf(x[j], x[j], ss);
  }
  const float r = a.norm_w ? (1.f - a.lambda_init) * rsqrtf(warp_sum(ss) / (2 * D) + a.norm_eps) : 1.f;
  T* o = (T*)a.o + (((int64_t)b * 2 * a.pairs + 2 * p) * a.Nq + i) * D;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int c = lane + 32 * j;
    if (c < 2 * D) from_f32(o + (c / D) * (int64_t)a.Nq * D + c % D, a.norm_w ? x[j] * r * __ldg(a.norm_w + c) : x[j]);
  }
}

}  // namespace

cudaError_t launch_diff_generic(const DiffArgs& a, cudaStream_t st) {
  const dim3 grid((unsigned)ceil_div(a.Nq, kRowWarps), (unsigned)(a.B * a.pairs));
  if (a.dtype == JV_F32) return launch_programmatic(diff_generic_kernel<float>, grid, kRowWarps * 32, 0, st, a);
  return launch_programmatic(diff_generic_kernel<__nv_bfloat16>, grid, kRowWarps * 32, 0, st, a);
}

}  // namespace jv

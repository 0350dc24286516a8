// Differential attention for what has no kernel of its own: f32 tensors, and bf16 ones with D other than 64.  One warp per query row and
// pair, fp32 arithmetic (diff_row in attn_diff.cuh).
//
// It is right, not fast: no row shares a key with another in registers or shared memory and no row's keys are split, so latency bounds
// it.  f32, D = 64, 8 pairs: 64 queries against 64 keys 85 us, two causal prompts of 4096 tokens 50 ms, single tokens of 32 sequences of up
// to 16384 keys, two pairs of keys, 39 ms.
#include "attn_diff.cuh"

namespace jv {
namespace {

using namespace diff;

constexpr int kRowWarps = 4;

template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) diff_generic_kernel(const DiffArgs a) {
  __shared__ float sq[kRowWarps][2 * 64];
  griddep_wait();
  griddep_launch_dependents();
  const int warp = threadIdx.x >> 5, i = blockIdx.x * kRowWarps + warp;
  if (i >= a.Nq) return;
  const float lam = lambda_of(Tail{a.lambda, a.lambda_init, a.norm_w, a.norm_eps, a.D});
  diff_row<T>(a, blockIdx.y / a.pairs, blockIdx.y % a.pairs, i, lam, sq[warp]);
}

}  // namespace

cudaError_t launch_diff_generic(const DiffArgs& a, cudaStream_t st) {
  const dim3 grid((unsigned)ceil_div(a.Nq, kRowWarps), (unsigned)(a.B * a.pairs));
  if (a.dtype == JV_F32) return launch_programmatic(diff_generic_kernel<float>, grid, kRowWarps * 32, 0, st, a);
  return launch_programmatic(diff_generic_kernel<__nv_bfloat16>, grid, kRowWarps * 32, 0, st, a);
}

}  // namespace jv

// The calls of a state-space mixer: host launchers of causal_conv.cu and selective_scan.cu.  Internal.
#pragma once

#include "common.cuh"

namespace jv {

// Token rows of a [B, L, ...] tensor: elements from token to token, and from batch element to batch element
struct Rows {
  int64_t tok, batch;
  __host__ __device__ int64_t at(int b, int t) const { return b * batch + t * tok; }
};

struct ConvArgs {
  const void* x;                    // [B, L, C]
  const float *w, *b;               // [C, K]; [C] or null
  const void* s_in;                 // [B, K - 1, C] or null
  void *u, *s_out;                  // [B, L, C]; [B, K - 1, C] or null
  const int* lens;                  // [B] or null
  int B, L, C, K, dtype, silu;
  Rows xs;
};
cudaError_t launch_causal_conv(const ConvArgs& a, cudaStream_t st);

struct ScanArgs {
  const void *u, *dt, *Bm, *Cm, *z;  // [B, L, C], [B, L, C], [B, L, Ns] twice, [B, L, C] or null
  const float *A, *D, *dt_bias;      // [C, Ns]; [C] or null
  const float* h_in;                 // [B, C, Ns] or null
  float* h_out;                      // or null
  void* y;                           // [B, L, C] contiguous
  const int* lens;
  int B, L, C, Ns, dtype, softplus;
  Rows us, ds, bs, cs, zs;
};
struct ScanPlan {
  int lanes;                         // of a channel
  int nchunk, chunk;                 // chunks of a sequence (1: no scratch) and their tokens
  size_t off_state, off_sum, total;  // bytes: [B, nchunk, C, Ns] states, [B, nchunk, C] sums of steps
};
ScanPlan scan_plan(int B, int L, int C, int Ns);
cudaError_t launch_selective_scan(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st);

}  // namespace jv

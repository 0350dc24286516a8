// Differential attention, the second launch of a call on the tensor cores: partial results merged in the order of their keys, and rows that
// the first has marked done again (see attn_diff.cuh and attn_diff.cu).
#include "attn_diff.cuh"
#include "tc_common.cuh"

namespace jv {
namespace {

using namespace tc;
using namespace diff;

// ---- the partials of an item merged, and rows done again ----------------------------------------------------------------
// Block (c, y), rows y, y + gridDim.y, ... of eight by its warps: the marked rows of the whole items of block c of the main launch; and
// the item that block c takes up in its middle, if c is the first that does.  A lane holds four channels of both maps.
constexpr int kMergeWarps = 8;
__global__ void __launch_bounds__(kMergeWarps * 32, 4) diff_merge_kernel(const DiffParams p, int rows, int blocks) {
  __shared__ int last, begun;
  __shared__ float sq[kMergeWarps][kV];
  griddep_wait();
  griddep_launch_dependents();
  const int c = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Start s = p.starts[c];
  if (s.tiles == 0 || s.left) return;
  const float lam = lambda_of(p.tail);
  if (s.redo) {
    Walk it;
    it.begin(s);
    while (it.next(p.items)) {
      if (!it.whole()) continue;
      for (int r = blockIdx.y * kMergeWarps + warp; r < rows; r += gridDim.y * kMergeWarps) {
        const int i = it.iqt * kTile + r;                 // (only items of tiles have marked rows)
        if (i < p.items.Nq && p.mark[((size_t)it.ib * p.pairs + it.ipair) * p.items.Nq + i])
          diff_row<__nv_bfloat16>(p.args, it.ib, it.ipair, i, lam, sq[warp]);
      }
    }
  }
  if (s.tile == 0) return;
  auto same = [&](const Start& a) { return a.b == s.b && a.qt == s.qt && a.pair == s.pair; };
  if (threadIdx.x == 0) {
    // blocks without tiles lie between; the one before with tiles holds the item's beginning, or takes it up in its middle, too
    int b = c - 1;
    while (b > 0 && p.starts[b].tiles == 0) --b;
    const Start before = p.starts[b];
    begun = same(before) && before.tile > 0 ? -1 : b;
    int e = c;
    bool left = before.left != 0;
    for (int k = c + 1; k < blocks; ++k) {
      const Start a = p.starts[k];
      if (a.tiles == 0) continue;
      if (!same(a) || a.tile == 0) break;
      e = k;
      left = left || a.left != 0;
    }
    last = left ? -1 : e;
  }
  __syncthreads();
  if (begun < 0 || last < 0) return;         // another block's item; or one whose blocks have left without a result
  const Reach reach = reach_of(p.items.kv_len, p.items.q_pos, s.b, p.items.Nq, p.items.Nk, p.items.causal != 0);
  for (int r = blockIdx.y * kMergeWarps + warp; r < rows; r += gridDim.y * kMergeWarps) {
    int pair, i;
    p.row(s.qt, s.pair, r, pair, i);
    if (i >= p.items.Nq) break;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    const float* src = p.partial + r * kPartial;
#pragma unroll 4
    for (int k = begun; k <= last; ++k) {
      // (a block without tiles has left nothing in its slots: what lies there is loaded and dropped)
      const float* at = src + (size_t)(2 * k + (k == begun ? 1 : 0)) * p.slot_rows * kPartial;
      const float4 st = __ldcg(reinterpret_cast<const float4*>(at));
      const float4 a4[2] = {__ldcg(reinterpret_cast<const float4*>(at + 4) + lane), __ldcg(reinterpret_cast<const float4*>(at + 4 + kV) + lane)};
      const bool none = k > begun && p.starts[k].tiles == 0;
      const float pm[2] = {st.x, st.z}, pl[2] = {st.y, st.w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (none || pm[h] == -INFINITY) continue;       // no keys of this row
        const float mn = max3(m[h], pm[h], pm[h]), f = ex2(m[h] - mn), g = ex2(pm[h] - mn);
        m[h] = mn;
        l[h] = l[h] * f + pl[h] * g;
        acc[h].x = acc[h].x * f + a4[h].x * g;
        acc[h].y = acc[h].y * f + a4[h].y * g;
        acc[h].z = acc[h].z * f + a4[h].z * g;
        acc[h].w = acc[h].w * f + a4[h].w * g;
      }
    }
    const bool any = reach.limit(i) > 0;
    const float f0 = any ? 1.f / l[0] : 0.f, f1 = any ? -lam / l[1] : 0.f;
    float x[4] = {acc[0].x * f0 + acc[1].x * f1, acc[0].y * f0 + acc[1].y * f1, acc[0].z * f0 + acc[1].z * f1, acc[0].w * f0 + acc[1].w * f1};
    float ss = 0.f;
#pragma unroll
    for (int y = 0; y < 4; ++y) ss = fmaf(x[y], x[y], ss);
    ss = warp_sum(ss);
    if (!(ss < INFINITY)) {                     // a part that says so, or values out of range
      diff_row<__nv_bfloat16>(p.args, s.b, pair, i, lam, sq[warp]);
      continue;
    }
    if (p.tail.norm_w) {
      const float rn = (1.f - p.tail.lambda_init) * rsqrtf(ss * (1.f / kV) + p.tail.norm_eps);
      const float4 w = __ldg(reinterpret_cast<const float4*>(p.tail.norm_w + 4 * lane));
      x[0] *= rn * w.x; x[1] *= rn * w.y; x[2] *= rn * w.z; x[3] *= rn * w.w;
    }
    __nv_bfloat16* dst = p.o + (((size_t)s.b * 2 * p.pairs + 2 * pair + (lane >> 4)) * p.items.Nq + i) * kD + 4 * (lane & 15);
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  }
}

}  // namespace

cudaError_t launch_diff_merge(const DiffParams& p, int blocks, int rows, cudaStream_t st) {
  return launch_programmatic(diff_merge_kernel, dim3((unsigned)blocks, (unsigned)ceil_div(rows, kMergeWarps)), kMergeWarps * 32, 0, st, p, rows, blocks);
}

}  // namespace jv

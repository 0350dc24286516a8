// Differential attention, the second launch of a call on the tensor cores: partial results merged in the order of their keys, and rows that
// the first has marked done again (see attn_diff.cuh and attn_diff.cu).
#include "attn_diff.cuh"
#include "tc_common.cuh"

namespace jv {
namespace {

using namespace tc;
using namespace diff;

// Block (c, y): the marked rows of the whole items of block c of the main launch; and sixteen rows, 16 y on, of the item that block c
// takes up in its middle, if c is the first that does.  A thread has eight channels of both maps of one row.
constexpr int kMergeWarps = 8;
constexpr int kMergeRows = 16;
static_assert(kMergeRows == kPartialRows && kMergeWarps * 32 == kMergeRows * kV / 8, "threads of the rows that lie side by side");
__global__ void __launch_bounds__(kMergeWarps * 32, 4) diff_merge_kernel(const DiffParams p, int rows, int blocks) {
  __shared__ float sq[kMergeWarps][kV], square[kMergeWarps][kMergeRows];
  griddep_wait();
  griddep_launch_dependents();
  const int c = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Start s = p.starts[c];
  if (s.tiles == 0 || s.left || (!s.redo && s.tile == 0)) return;
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
  // The block before (blocks without tiles may lie between) holds the item's beginning, or takes it up in its middle, too: then the
  // item is another block's.
  int begun = c - 1;
  Start before = p.starts[begun];
  while (before.tiles == 0 && begun > 0) before = p.starts[--begun];
  if (same(before) && before.tile > 0) return;
  int last = c;
  bool left = before.left != 0;
  for (int k0 = c + 1; k0 < blocks; k0 += 32) {           // 32 of the blocks behind at a time
    const int k = k0 + lane;
    const Start a = p.starts[min(k, blocks - 1)];
    const bool in = k < blocks && (a.tiles == 0 || (same(a) && a.tile > 0));
    const uint32_t out = __ballot_sync(0xffffffffu, !in);
    const int n = out ? __ffs(out) - 1 : 32;
    const uint32_t parts = __ballot_sync(0xffffffffu, lane < n && a.tiles > 0), gone = __ballot_sync(0xffffffffu, lane < n && a.tiles > 0 && a.left);
    if (parts) last = k0 + 31 - __clz(parts);
    left = left || gone;
    if (n < 32) break;
  }
  if (left) return;                          // blocks that have left without a result
  const Reach reach = reach_of(p.items.kv_len, p.items.q_pos, s.b, p.items.Nq, p.items.Nk, p.items.causal != 0);
  const int row = lane & 15, r = kMergeRows * blockIdx.y + row, ch = 8 * (2 * warp + (lane >> 4));
  int pair, i;
  p.row(s.qt, s.pair, min(r, rows - 1), pair, i);
  const bool mine = r < rows && i < p.items.Nq;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, acc[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int y = 0; y < 8; ++y) acc[h][y] = 0.f;
  const float* src = p.partial + partial_at(r);
#pragma unroll 2
  for (int k = begun; k <= (mine ? last : -1); ++k) {
    // (a block without tiles has left nothing in its slots: what lies there is loaded and dropped)
    const float* at = src + (size_t)(2 * k + (k == begun ? 1 : 0)) * p.slot_rows * kPartial;
    const float4 st = __ldcg(reinterpret_cast<const float4*>(at));
    float4 q[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int y = 0; y < 2; ++y) q[h][y] = __ldcg(reinterpret_cast<const float4*>(at + (1 + (kV * h + ch) / 4 + y) * kPiece));
    const bool none = k > begun && p.starts[k].tiles == 0;
    const float pm[2] = {st.x, st.z}, pl[2] = {st.y, st.w};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (none || pm[h] == -INFINITY) continue;       // no keys of this row
      const float mn = max3(m[h], pm[h], pm[h]), f = ex2(m[h] - mn), g = ex2(pm[h] - mn);
      m[h] = mn;
      l[h] = l[h] * f + pl[h] * g;
      const float v[8] = {q[h][0].x, q[h][0].y, q[h][0].z, q[h][0].w, q[h][1].x, q[h][1].y, q[h][1].z, q[h][1].w};
#pragma unroll
      for (int y = 0; y < 8; ++y) acc[h][y] = acc[h][y] * f + v[y] * g;
    }
  }
  const bool any = reach.limit(i) > 0;
  const float f0 = any ? 1.f / l[0] : 0.f, f1 = any ? -lam / l[1] : 0.f;
  float x[8], ss = 0.f;
#pragma unroll
  for (int y = 0; y < 8; ++y) {
    x[y] = acc[0][y] * f0 + acc[1][y] * f1;
    ss = fmaf(x[y], x[y], ss);
  }
  ss += __shfl_xor_sync(0xffffffffu, ss, 16);
  if (lane < kMergeRows) square[warp][row] = ss;
  __syncthreads();                           // (all of a block comes here, or none of it)
  ss = 0.f;
#pragma unroll
  for (int w = 0; w < kMergeWarps; ++w) ss += square[w][row];
  // a part that says so, values out of range, or (with a norm) a mean square that is not safely within fp32
  const bool again = mine && any && !(p.tail.norm_w ? square_fine(ss * (1.f / kV) + p.tail.norm_eps) : ss < INFINITY);
  if (p.tail.norm_w) {
    const float rn = (1.f - p.tail.lambda_init) * rsqrtf(ss * (1.f / kV) + p.tail.norm_eps);
#pragma unroll
    for (int y = 0; y < 8; y += 4) {
      const float4 w = __ldg(reinterpret_cast<const float4*>(p.tail.norm_w + ch + y));
      x[y] *= rn * w.x; x[y + 1] *= rn * w.y; x[y + 2] *= rn * w.z; x[y + 3] *= rn * w.w;
    }
  }
  if (!any)
#pragma unroll
    for (int y = 0; y < 8; ++y) x[y] = 0.f;  // (whatever the norm makes of zeros)
  if (mine && !again) {
    __nv_bfloat16* dst = p.o + (((size_t)s.b * 2 * p.pairs + 2 * pair + (ch >> 6)) * p.items.Nq + i) * kD + (ch & 63);
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
  const uint32_t redo = __ballot_sync(0xffffffffu, again);     // (rows in bits 0 to 15, alike in all warps)
  if (redo == 0) return;
#pragma unroll 1
  for (int h = warp; h < kMergeRows; h += kMergeWarps)
    if (redo >> h & 1u) {
      int pr, qi;
      p.row(s.qt, s.pair, kMergeRows * blockIdx.y + h, pr, qi);
      diff_row<__nv_bfloat16>(p.args, s.b, pr, qi, lam, sq[warp]);
    }
}

}  // namespace

cudaError_t launch_diff_merge(const DiffParams& p, int blocks, int rows, cudaStream_t st) {
  return launch_programmatic(diff_merge_kernel, dim3((unsigned)blocks, (unsigned)ceil_div(rows, kMergeRows)), kMergeWarps * 32, 0, st, p, rows, blocks);
}

}  // namespace jv

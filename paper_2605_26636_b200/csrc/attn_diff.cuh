// Differential attention: what its kernels share.  Internal.
//
// Pair p of heads (2 p, 2 p + 1) has two softmax maps over the same keys and one row of values, the two value heads side by side:
//   x = softmax(s q_0 k_0^T) v - lambda softmax(s q_1 k_1^T) v,   lambda = exp(lq1 . lk1) - exp(lq2 . lk2) + lambda_init,
// with a norm weight w:  o = (1 - lambda_init) w x / sqrt(mean x^2 + eps) over the pair's 2 D channels.
// Each map's normaliser is known only behind its last key, so both products with v are kept and subtracted at the end.
//
// Work in units of 128-key tiles.  An item is a set of query rows of one pair that walk the same keys (a tile of 128 queries, or all the rows
// of one key pair); its tiles form a stretch of the list of all items' tiles, and block c of G takes tiles
// [c T / G, (c + 1) T / G) of that list whatever the sequences' lengths are.  A block that has an item's whole stretch writes o;
// a part of one leaves a partial (reference, sum and product of both maps per row, fp32) in the workspace, and a second launch
// merges an item's partials in the order of its keys.  No atomics: results repeat bit for bit.
#pragma once

#include "common.cuh"

namespace jv {

struct DiffArgs {
  const void *q, *k, *v;
  void* o;                           // [B, H, Nq, D] contiguous
  int B, pairs, kv_pairs, Nq, Nk, D, dtype;
  bool causal;
  InStrides qs, ks;                  // of q; of k and v
  const float* lambda;               // [4, D]
  float lambda_init;
  const float* norm_w;               // [2 D] or null
  float norm_eps;
  const int *kv_len, *q_pos;         // [B] or null
  float scale;
};

namespace diff {

constexpr int kD = 64, kV = 128;     // channels of a map; of a value row
constexpr int kTile = 128;           // keys of a tile
constexpr int kPartial = 4 + 2 * kV; // floats of a row's partial: reference (log2) and sum of map 0, of map 1, product 0, product 1

// Keys that a batch element has, and the position of its first query among them.  A query i sees the keys [0, limit(i)).
struct Reach {
  int len, pos;
  bool causal;
  __device__ __forceinline__ int limit(int i) const { return causal ? min(len, pos + i + 1) : len; }
};
__device__ __forceinline__ Reach reach_of(const int* kv_len, const int* q_pos, int b, int Nq, int Nk, bool causal) {
  Reach r;
  r.len = kv_len ? min(max(__ldg(kv_len + b), 0), Nk) : Nk;
  r.pos = q_pos ? min(__ldg(q_pos + b), Nk) : Nk - Nq;       // (a position past the last key sees them all)
  r.causal = causal;
  return r;
}

// The list of items: groups (batch element, query tile), the pairs of a group side by side, each of `tiles(group)` key tiles.
struct Items {
  int B, qtiles, width;              // width: pairs of a group
  int Nq, Nk, qrows;                 // qrows: queries of a tile
  int causal;
  const int *kv_len, *q_pos;
  __device__ __forceinline__ int tiles(int b, int qt) const {
    const Reach r = reach_of(kv_len, q_pos, b, Nq, Nk, causal);
    // an item without keys takes one tile, all of it masked: its rows are written like any other's
    return max(1, (r.limit(min(Nq, (qt + 1) * qrows) - 1) + kTile - 1) / kTile);
  }
};

// Where a block begins, and how far it goes.  Also what it leaves in the workspace for the launch that merges.
struct Start {
  int b, qt, pair, tile;             // first item, and the first of its tiles
  int tiles;                         // tiles of the block
  int left;                          // the block has left without a result
};

// To be called by all threads of a block (a multiple of 32, at most 1024): start of block c of G.  tmp: 33 64-bit words of
// shared memory; *out in shared memory, valid behind the barrier that the call ends with.
__device__ __forceinline__ void find_start(const Items& it, int c, int G, long long* tmp, Start* out) {
  const int groups = it.B * it.qtiles, n = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long base = 0, total = 0;
  for (int pass = 0; pass < 2; ++pass) {                    // the sum, then the place (one round each up to n groups)
    const long long lo = pass ? (long long)c * total / G : 0, hi = pass ? (long long)(c + 1) * total / G : 0;
    base = 0;
    for (int g0 = 0; g0 < groups; g0 += n) {
      const int g = g0 + (int)threadIdx.x;
      int b = 0, qt = 0, per = 0;
      long long w = 0;
      if (g < groups) {
        b = g / it.qtiles;
        qt = g - b * it.qtiles;
        per = it.tiles(b, qt);
        w = (long long)per * it.width;
      }
      long long incl = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long up = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += up;
      }
      __syncthreads();
      if (lane == 31) tmp[warp] = incl;
      __syncthreads();
      long long before = base, all = 0;
      for (int i = 0; i < n / 32; ++i) {
        if (i < warp) before += tmp[i];
        all += tmp[i];
      }
      const long long excl = before + incl - w;
      if (pass && w && lo >= excl && lo < excl + w) {
        const long long d = lo - excl;
        *out = Start{b, qt, (int)(d / per), (int)(d % per), (int)(hi - lo), 0};
      }
      base += all;
    }
    total = base;
  }
  __syncthreads();
}

// A block's walk over its tiles, item by item
struct Walk {
  int b, qt, pair, tile, left;       // the next item, the first of its tiles, tiles left to the block
  int n, t0, t1;                     // the present item: its tiles, and those of them that are this block's
  int ib, iqt, ipair;
  __device__ __forceinline__ void begin(const Start& s) { b = s.b; qt = s.qt; pair = s.pair; tile = s.tile; left = s.tiles; }
  __device__ __forceinline__ bool next(const Items& it) {
    if (left <= 0) return false;
    ib = b; iqt = qt; ipair = pair;
    n = it.tiles(b, qt);
    t0 = tile;
    t1 = min(n, tile + left);
    left -= t1 - t0;
    tile = 0;
    if (++pair == it.width) {
      pair = 0;
      if (++qt == it.qtiles) { qt = 0; ++b; }
    }
    return true;
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == n; }
};
// Partials of block c: 0 of an item that began in an earlier block, 1 of one that begins in it and ends in a later one
__device__ __forceinline__ int partial_slot(int c, int t0) { return 2 * c + (t0 == 0 ? 1 : 0); }

// What turns both maps' results into o
struct Tail {
  const float* lambda;
  float lambda_init;
  const float* norm_w;
  float norm_eps;
  int D;
};
// lambda, by a whole warp
__device__ __forceinline__ float lambda_of(const Tail& t) {
  float a = 0.f, b = 0.f;
  for (int i = threadIdx.x & 31; i < t.D; i += 32) {
    a = fmaf(__ldg(t.lambda + i), __ldg(t.lambda + t.D + i), a);
    b = fmaf(__ldg(t.lambda + 2 * t.D + i), __ldg(t.lambda + 3 * t.D + i), b);
  }
  return expf(warp_sum(a)) - expf(warp_sum(b)) + t.lambda_init;
}

}  // namespace diff

size_t diff_workspace_bytes(int B, int pairs, int kv_pairs, int Nq, int Nk, int D, int dtype, bool causal);
// any f32 or bf16 tensors, D <= 64: one warp per query row, fp32 arithmetic
cudaError_t launch_diff_generic(const DiffArgs& a, cudaStream_t st);
// bf16, D == 64: tiles of 128 queries on the tensor cores
bool diff_tc_supported(const DiffArgs& a);
cudaError_t launch_diff_tc(const DiffArgs& a, void* ws, int* status, cudaStream_t st);

}  // namespace jv

// Differential attention: what its kernels share.  Internal.
//
// Pair p of heads (2 p, 2 p + 1) has two softmax maps over the same keys and one row of values, the two value heads side by side:
//   x = softmax(s q_0 k_0^T) v - lambda softmax(s q_1 k_1^T) v,   lambda = exp(lq1 . lk1) - exp(lq2 . lk2) + lambda_init,
// with a norm weight w:  o = (1 - lambda_init) w x / sqrt(mean x^2 + eps) over the pair's 2 D channels.
// Each map's normaliser is known only behind its last key, so both products with v are kept and subtracted at the end.
//
// Work in units of 128-key tiles.  An item is a set of query rows of one pair that walk the same keys (a tile of 128 queries, or all the rows
// of one key pair).  All items' tiles, `lead` units for what an item costs beside its tiles ahead of them, form a list of U units, and
// block c of G takes the units [c U / G, (c + 1) U / G) of it, whatever the sequences' lengths are.  A block that has all of an
// item's tiles writes o; a part of them leaves a partial (reference, sum and product of both maps per row, fp32) in the
// workspace, and a second launch merges an item's partials in the order of its keys.  No atomics: results repeat bit for bit.
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
// A row's partial: 65 pieces of 16 bytes, reference (log2) and sum of map 0 and of map 1, product 0, product 1.  The pieces of sixteen rows
// lie side by side, [16 rows / piece / row]: threads that own rows write, and threads that own channels of sixteen rows read, 256
// bytes in a row.  (Row by row the main launch's stores, 16 bytes of 32 rows at a time, took a quarter of 256 queries against
// 16384 keys.)
constexpr int kPartial = 4 + 2 * kV, kPartialRows = 16, kPiece = 4 * kPartialRows;   // floats of a row; rows side by side; floats from piece to piece
__host__ __device__ constexpr size_t partial_at(size_t row) { return row / kPartialRows * (kPartialRows * kPartial) + row % kPartialRows * 4; }

// Keys that a batch element has, and the position of its first query among them.  A query i sees the keys [0, limit(i)).
struct Reach {
  int len, pos;
  bool causal;
  __device__ __forceinline__ int limit(int i) const { return causal ? min(len, pos + i + 1) : len; }
};
__device__ __forceinline__ Reach reach_of(const int* kv_len, const int* q_pos, int b, int Nq, int Nk, bool causal) {
  Reach r;
  r.len = kv_len ? min(max(__ldg(kv_len + b), 0), Nk) : Nk;
  // a position past the last key sees them all, one that the last query does not bring up to key 0 sees none, however far off it is
  r.pos = q_pos ? max(min(__ldg(q_pos + b), Nk), -Nq) : Nk - Nq;
  r.causal = causal;
  return r;
}

// The list of items: groups (batch element, query tile), the pairs of a group side by side, each of `tiles(group)` key tiles.
struct Items {
  int B, qtiles, width;              // width: pairs of a group
  int Nq, Nk, qrows;                 // qrows: queries of a tile
  int causal;
  int lead, whole;                   // units ahead of an item's tiles; no part of an item has fewer tiles than `whole`
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
  int redo;                          // some of its whole items' rows are marked to be done again
};

// To be called by all threads of a block (a multiple of 32, at most 1024): start of block c of G.  tmp: 34 64-bit words of
// shared memory; *out in shared memory, valid behind the barrier that the call ends with.
__device__ __forceinline__ void find_start(const Items& it, int c, int G, long long* tmp, Start* out) {
  const int groups = it.B * it.qtiles, n = blockDim.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long total = 0;                                      // units of the list
  for (int pass = 0; pass < 2; ++pass) {                    // the sum, then the places (one round each up to n groups)
    const long long lo = pass ? (long long)c * total / G : -1, hi = pass ? (long long)(c + 1) * total / G : -1;
    long long base = 0;
    for (int g0 = 0; g0 < groups; g0 += n) {
      const int g = g0 + (int)threadIdx.x;
      int b = 0, qt = 0, per = 0;
      long long w = 0;
      if (g < groups) {
        b = g / it.qtiles;
        qt = g - b * it.qtiles;
        per = it.tiles(b, qt);
        w = (long long)(per + it.lead) * it.width;
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
      // the place of a unit: pair, tile (of the item, or 0 of the next where a part would be too short), tiles ahead of it
      auto place = [&](long long at, int& pair, int& tile) {
        const long long d = at - excl;
        pair = (int)(d / (per + it.lead));
        tile = max(0, (int)(d % (per + it.lead)) - it.lead);
        if (tile < it.whole) tile = 0;
        else if (per - tile < it.whole) tile = per;
        if (tile == per) { ++pair; tile = 0; }
        return excl - (long long)(g) * it.width * it.lead + (long long)pair * per + tile;
      };
      if (pass && w) {
        int pair, tile;
        if (lo >= excl && lo < excl + w) {
          const long long ahead = place(lo, pair, tile);
          if (pair == it.width) {                           // the first item of the next group (if there is none, no tiles are left)
            pair = 0;
            if (++qt == it.qtiles) { qt = 0; ++b; }
          }
          *out = Start{b, qt, pair, tile, 0, 0, 0};
          tmp[32] = ahead;
        }
        if (hi >= excl && hi < excl + w) tmp[33] = place(hi, pair, tile);
        else if (hi == total && g == groups - 1) tmp[33] = total - (long long)groups * it.width * it.lead;
      }
      base += all;
    }
    total = base;
  }
  __syncthreads();
  if (threadIdx.x == 0) out->tiles = (int)(tmp[33] - tmp[32]);
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

// The norm of a row: x times what this returns is x / sqrt(mean x^2 + eps).  A warp holds the row, N values a lane, inv_n = 1 / (their
// number).  Where the mean square is not safely within fp32, x is scaled by a power of two first (values from 2^-149 to 2^128 then have
// squares from 2^-98 to 2^96), and eps with it.
constexpr float kSquareMin = 1e-30f;        // smallest mean square that is taken as it is
__device__ __forceinline__ bool square_fine(float ms) { return ms >= kSquareMin && ms < INFINITY; }
template <int N>
__device__ __forceinline__ float inverse_rms(float (&x)[N], float inv_n, float eps) {
  auto mean_square = [&](float e) {
    float ss = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) ss = fmaf(x[j], x[j], ss);
    return fmaf(warp_sum(ss), inv_n, e);
  };
  const float ms = mean_square(eps);
  if (square_fine(ms)) return rsqrtf(ms);
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j) top = fmaxf(top, fabsf(x[j]));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (!(top > 0.f && top < INFINITY)) return rsqrtf(ms);      // zeros; an infinity (no numbers stay so either way)
  const float s = top > 1.f ? 0x1p-80f : 0x1p+100f;
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] *= s;
  return rsqrtf(mean_square(eps * s * s));
}

// One query row of one pair, by a whole warp, in fp32: a lane takes a key of 32 for the scores of both maps, then 2 D / 32 channels for
// the products.  sq: 2 D floats of shared memory of the warp.
template <typename T>
__device__ __forceinline__ void diff_row(const DiffArgs& a, int b, int p, int i, float lam, float* sq) {
  constexpr int kMaxD = 64, kPer = 2 * kMaxD / 32;
  const int lane = threadIdx.x & 31, g = p / (a.pairs / a.kv_pairs), D = a.D;
  const T* q = (const T*)a.q + b * a.qs.batch + i * a.qs.tok;
  const T* k = (const T*)a.k + b * a.ks.batch + 2 * g * a.ks.head;
  const T* v = (const T*)a.v + b * a.ks.batch + 2 * g * a.ks.head;
  __syncwarp();
  for (int c = lane; c < 2 * D; c += 32) sq[c] = to_f32(q[(2 * p + c / D) * a.qs.head + c % D]);
  __syncwarp();
  const int limit = reach_of(a.kv_len, a.q_pos, b, a.Nq, a.Nk, a.causal).limit(i);
  const float sl2 = a.scale * 1.4426950408889634f;
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
          for (int x = 0; x < (int)(16 / sizeof(T)); ++x) s = fmaf(f[x], sq[h * D + c + x], s);
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
  float x[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) x[j] = limit > 0 && lane + 32 * j < 2 * D ? acc[0][j] / l[0] - lam * (acc[1][j] / l[1]) : 0.f;
  const float r = a.norm_w ? (1.f - a.lambda_init) * inverse_rms(x, 1.f / (float)(2 * D), a.norm_eps) : 1.f;
  T* o = (T*)a.o + (((int64_t)b * 2 * a.pairs + 2 * p) * a.Nq + i) * D;
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int c = lane + 32 * j;
    if (c < 2 * D) {
      const float y = a.norm_w ? x[j] * r * __ldg(a.norm_w + c) : x[j];
      from_f32(o + (c / D) * (int64_t)a.Nq * D + c % D, limit > 0 ? y : 0.f);      // (no key: 0 whatever the norm makes of zeros)
    }
  }
}

// What the main launches and the one that merges share
struct DiffParams {
  Items items;
  Tail tail;
  DiffArgs args;
  __nv_bfloat16* o;        // [B, 2 pairs, Nq, 64]
  unsigned char* mark;     // [B, pairs, Nq]: rows of whole items to be done again (tiles of queries only)
  Start* starts;           // [blocks]
  float* partial;          // [2 blocks, slot_rows, kPartial]
  int* status;
  int pairs, share;        // share: pairs of queries to a pair of keys
  int slot_rows;
  float scale_log2;
  // Row r of an item: query and pair.  Items of tiles (slot_rows = kTile) have one pair and 128 queries; items of rows have all queries of
  // the pairs that share their keys.
  __device__ __forceinline__ void row(int qt, int item_pair, int r, int& pair, int& i) const {
    if (slot_rows == kTile) {
      pair = item_pair;
      i = qt * kTile + r;
    } else {
      pair = item_pair * share + r / items.Nq;
      i = r % items.Nq;
    }
  }
};

}  // namespace diff

// Blocks of a call's main launch, and where its arrays are in the workspace
struct DiffPlan {
  int blocks;
  size_t off_partial, off_mark, total;
};
inline DiffPlan diff_plan(int blocks, int slot_rows, int64_t marks) {
  DiffPlan p;
  p.blocks = blocks;
  p.off_partial = align_up((size_t)blocks * sizeof(diff::Start), 256);
  p.off_mark = p.off_partial + (size_t)2 * blocks * slot_rows * diff::kPartial * 4;
  p.total = p.off_mark + (size_t)marks;
  return p;
}
inline diff::DiffParams diff_params(const DiffArgs& a, const DiffPlan& plan, const diff::Items& items, int slot_rows, void* ws, int* status) {
  diff::DiffParams p;
  p.items = items;
  p.tail = diff::Tail{a.lambda, a.lambda_init, a.norm_w, a.norm_eps, diff::kD};
  p.args = a;
  p.o = (__nv_bfloat16*)a.o;
  p.starts = (diff::Start*)ws;
  p.partial = (float*)((char*)ws + plan.off_partial);
  p.mark = (unsigned char*)ws + plan.off_mark;
  p.status = status;
  p.pairs = a.pairs;
  p.share = a.pairs / a.kv_pairs;
  p.slot_rows = slot_rows;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  return p;
}
cudaError_t launch_diff_merge(const diff::DiffParams& p, int blocks, int rows, cudaStream_t st);

// any f32 or bf16 tensors, D <= 64: one warp per query row, fp32 arithmetic
cudaError_t launch_diff_generic(const DiffArgs& a, cudaStream_t st);
// bf16, D == 64, on the tensor cores: all queries of the pairs that share their keys at a time, at most 16 rows ...
bool diff_rows_supported(const DiffArgs& a);
DiffPlan diff_rows_plan(int B, int kv_pairs, int Nk);
cudaError_t launch_diff_rows(const DiffArgs& a, void* ws, int* status, cudaStream_t st);
// ... or tiles of 128 queries of a pair
bool diff_tc_supported(const DiffArgs& a);
DiffPlan diff_tc_plan(int B, int pairs, int Nq, int Nk);
cudaError_t launch_diff_tc(const DiffArgs& a, void* ws, int* status, cudaStream_t st);

}  // namespace jv

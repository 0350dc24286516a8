// Differential attention on the 5th-generation tensor cores: bf16, 64 channels a map, tiles of 128 queries of a pair of heads.
//
// The kernel of head_dim 128 (attn_d128.cu) with its two query tiles turned into the two maps of one: a tile of 128 tokens lies in
// shared memory as two 128-byte-swizzled halves of 64 channels, the two heads of the pair.  Map m is S_m = Q_m K_m^T over half m alone (4
// MMAs of K = 16), and both maps multiply the same values, O_m += P_m V over both halves of V (2 x 4 MMAs).  Tensor memory: per
// map two 64-column score buffers (the bf16 probabilities written over the scores they came from) and one 128-column accumulator,
// 512 columns.  Warp roles (11 warps): a TMA producer (two buffers of Q, K through a ring of three tiles, V through one of two), an MMA
// issuer per map, four softmax warps per map, one thread per query row.  Steps of 64 keys, exact two-pass softmax per step
// against a lazily raised reference.
//
// Behind an item's last key a thread of map m takes channels 64 m .. 64 m + 63 of its row from both accumulators: the sums of
// the maps and the shares of the row's mean square are exchanged through shared memory, and the difference is normalised and written as one
// contiguous row of 128 bytes.  Parts of an item (see attn_diff.cuh) go to the workspace as they are.
//
// Keys that a row does not see are set to -inf behind the load of the scores; rows of V that lie behind a length may hold anything, and
// are overwritten with zeros in shared memory before the first product of their tile.
//
// Every wait is bounded: one that runs out sets the device status word and every role falls through to the teardown.
#include "attn_diff.cuh"
#include "tc_common.cuh"

namespace jv {
namespace {

using namespace tc;
using namespace diff;

constexpr uint32_t kSuspendNs = 4000;       // suspend-time hint of the barrier waits (tc_common.cuh)
constexpr int kHalfBytes = kTile * kD * 2;  // one head's half of a tile: 16 KB
constexpr int kTileBytes = 2 * kHalfBytes;
constexpr int kQB = 2, kKS = 3, kVS = 2;    // query buffers, ring depths
constexpr int kWarps = 11;
constexpr int kThreads = kWarps * 32;
constexpr int kFirstSoftmaxWarp = 3;
constexpr uint32_t kTmemCols = 512;
constexpr int kSub = 64;                    // keys per step
constexpr int kPolyOf8 = 3, kPolyDeg = 4;   // of every 8 score pairs, this many take the polynomial exponential, of this degree
// Tensor-memory columns: score buffer h of map m at 128 m + 64 h, O_m at 256 + 128 m
constexpr uint32_t kColS = 0, kColO = 256;

struct DiffParams {
  Items items;
  Tail tail;
  __nv_bfloat16* o;        // [B, 2 pairs, Nq, 64]
  Start* starts;           // [blocks], for the launch that merges
  float* partial;          // [2 blocks, 128, kPartial]
  int* status;
  int pairs, share;        // share: pairs of queries to a pair of keys
  float scale_log2;
};

struct __align__(8) Barriers {
  uint64_t q_full[kQB], q_empty[kQB];
  uint64_t k_full[kKS], k_empty[kKS], v_full[kVS], v_empty[kVS];
  uint64_t s_full[2][2], p_full[2][2];   // per map and score buffer
  uint64_t pv_done[2];                   // two phases per item: its last but one, its last P V has retired
  uint64_t sums_in, read_out;            // per item written whole: the maps' sums are there; the accumulators have been read
  uint64_t drain;
  union {
    long long scan[33];                  // for find_start
    float swap[2][kTile];                // what the two threads of a row tell each other
  };
  Start start;
  uint32_t tmem_base;
  volatile uint32_t abort_flag;
};
constexpr size_t kSmemTiles = (kQB + kKS + kVS) * (size_t)kTileBytes;          // 224 KB
constexpr size_t kSmemBytes = kSmemTiles + sizeof(Barriers) + 1024;            // + alignment slack
static_assert(kSmemBytes <= 227 * 1024, "shared memory of one block");

constexpr uint32_t kIdescQK = idesc(kTile, kSub, 0);       // S = Q K^T: M128 N64, both operands K-major
constexpr uint32_t kIdescPV = idesc(kTile, kD, 1);         // O half = P V half: M128 N64, V MN-major

__global__ void __launch_bounds__(kThreads, 1)
attn_diff_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK,
                 const __grid_constant__ CUtensorMap mapV, const DiffParams p) {
  extern __shared__ unsigned char smem_raw[];
  if (threadIdx.x == 32) {
    prefetch_map(&mapQ);
    prefetch_map(&mapK);
    prefetch_map(&mapV);
  }
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  Barriers* bar = reinterpret_cast<Barriers*>(smem + kSmemTiles);
  const uint32_t sQ = smem_u32(smem), sK = sQ + kQB * kTileBytes, sV = sK + kKS * kTileBytes;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kQB; ++i) {
      mbar_init(&bar->q_full[i], 1);
      mbar_init(&bar->q_empty[i], 2);         // one commit from each issuer
    }
    for (int m = 0; m < 2; ++m) {
      for (int h = 0; h < 2; ++h) {
        mbar_init(&bar->s_full[m][h], 1);
        mbar_init(&bar->p_full[m][h], 128);
      }
      mbar_init(&bar->pv_done[m], 1);
    }
    for (int s = 0; s < kKS; ++s) {
      mbar_init(&bar->k_full[s], 1);
      mbar_init(&bar->k_empty[s], 2);
    }
    for (int s = 0; s < kVS; ++s) {
      mbar_init(&bar->v_full[s], 1);
      mbar_init(&bar->v_empty[s], 2);
    }
    mbar_init(&bar->sums_in, 256);
    mbar_init(&bar->read_out, 256);
    mbar_init(&bar->drain, 2);
    bar->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 0) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar->tmem_base)),
                 "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, bar->tmem_base, 0);

  griddep_wait();                 // what is read and written from here on may belong to the launch ahead
  griddep_launch_dependents();
  // a timeout flagged earlier (by any CTA or launch) makes the rest leave at once
  if (threadIdx.x == 0 && *reinterpret_cast<volatile int*>(p.status) != 0) bar->abort_flag = 1;
  find_start(p.items, blockIdx.x, gridDim.x, bar->scan, &bar->start);    // (ends with a barrier)
  if (threadIdx.x == 0) {
    Start s = bar->start;
    s.left = bar->abort_flag;
    p.starts[blockIdx.x] = s;
  }
  if (bar->abort_flag) {
    if (warp == 0)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    return;
  }
  Walk it;
  it.begin(bar->start);

  if (warp == 0) {
    // ================= TMA producer =================
    // a tile = two boxes of 64 channels x 128 tokens, one per head of the pair
    auto load_tile = [&](uint32_t dst, const CUtensorMap* map, uint64_t* full, int row, int h, int b) {
      mbar_expect_tx(full, kTileBytes);
      tma_load_4d(dst, map, full, 0, row, h, b);
      tma_load_4d(dst + kHalfBytes, map, full, 0, row, h + 1, b);
    };
    bool ok = true;
    int n = 0;                 // items seen
    int ks = 0, vs = 0;        // ring stages of the next K and V tile
    uint32_t kpar = 1, vpar = 1;   // parity of the "empty" phase this pass over each ring waits for
    int issued_v = 0;          // for the abort path: V copies issued so far
    while (ok && it.next(p.items)) {
      const int hk = 2 * (it.ipair / p.share), qb = n & 1;
      ok = warp_wait<kSuspendNs>(&bar->q_empty[qb], ((n >> 1) & 1) ^ 1, &bar->abort_flag, p.status);
      if (!ok) break;
      if (elect_one()) load_tile(sQ + qb * kTileBytes, &mapQ, &bar->q_full[qb], it.iqt * kTile, 2 * it.ipair, it.ib);
      __syncwarp();
      for (int j = it.t0; j < it.t1 && ok; ++j) {
        ok = warp_wait<kSuspendNs>(&bar->k_empty[ks], kpar, &bar->abort_flag, p.status);
        if (!ok) break;
        if (elect_one()) load_tile(sK + ks * kTileBytes, &mapK, &bar->k_full[ks], j * kTile, hk, it.ib);
        __syncwarp();
        if (++ks == kKS) { ks = 0; kpar ^= 1; }
        ok = warp_wait<kSuspendNs>(&bar->v_empty[vs], vpar, &bar->abort_flag, p.status);
        if (!ok) break;
        if (elect_one()) load_tile(sV + vs * kTileBytes, &mapV, &bar->v_full[vs], j * kTile, hk, it.ib);
        __syncwarp();
        ++issued_v;
        if (++vs == kVS) { vs = 0; vpar ^= 1; }
      }
      ++n;
    }
    if (!ok && lane == 0) {
      // let the copies still in flight land before the CTA leaves (bounded by the same limit): those of V by their
      // barriers, those of K and Q around them by a millisecond from here
      const unsigned long long t0 = globaltimer();
      for (int g = max(0, issued_v - kVS); g < issued_v; ++g)
        while (!mbar_try(&bar->v_full[g % kVS], (g / kVS) & 1) && globaltimer() - t0 < kWaitLimitNs) {}
      while (globaltimer() - t0 < 1000000ull) {}
    }
  } else if (warp < kFirstSoftmaxWarp) {
    // ================= MMA issuer of map x =================
    // Per item the work is a chain over 64-key steps u (key tile u / 2, half u % 2):
    //   S(u) = Q_x K_x(u)^T      4 MMAs, M128 N64 K16, operands in shared memory
    //   O   += P(u) V(u)         2 x 4 MMAs, M128 N64 K16, A = P in tensor memory, one per channel half of V
    // S(u + 2) goes into the buffer that P(u) V(u) has just read: the tensor pipe executes one thread's MMAs in issue order, so
    // the commit that publishes S(u + 1) also says that P(u - 1) V(u - 1) has retired; behind the last scores pv_done says so.
    const int x = warp - 1;
    bool ok = true;
    int n = 0;
    int sk = 0, sv = 0;                     // ring stages of the score key tile and of the P V key tile
    uint32_t phk = 0, phv = 0;              // and their "full" parities
    uint32_t pcnt[2] = {0, 0};              // publications seen so far per buffer: parity of p_full
    while (ok && it.next(p.items)) {
      const int nsteps = 2 * (it.t1 - it.t0), qb = n & 1;
      const uint64_t dq = smem_desc(sQ + qb * kTileBytes + x * kHalfBytes);
      auto scores = [&](int u) {
        const uint64_t dk = smem_desc(sK + sk * kTileBytes + x * kHalfBytes + (u & 1) * (kSub * kD * 2));
        if (elect_one()) {
#pragma unroll
          for (int c = 0; c < kD / 16; ++c)
            mma_ss_1(tmem + kColS + x * 128 + (u & 1) * kSub, desc_advance(dq, c * 32), desc_advance(dk, c * 32), kIdescQK, c > 0 ? 1u : 0u);
        }
        __syncwarp();
        tc_commit(&bar->s_full[x][u & 1]);
        if ((u & 1) == 1) {
          tc_commit(&bar->k_empty[sk]);
          if (++sk == kKS) { sk = 0; phk ^= 1; }
        }
        if (u == nsteps - 1) tc_commit(&bar->q_empty[qb]);    // the item's last scores: its query tile may be replaced
      };
      auto key_landed = [&](int u) -> bool {
        return (u & 1) == 1 || warp_wait<kSuspendNs>(&bar->k_full[sk], phk, &bar->abort_flag, p.status);
      };
      ok = warp_wait<kSuspendNs>(&bar->q_full[qb], (n >> 1) & 1, &bar->abort_flag, p.status);
      ++n;
      for (int u = 0; u < 2 && ok; ++u) {   // (a key tile is two steps: nsteps >= 2)
        ok = key_landed(u);
        if (!ok) break;
        tc_fence_after();
        scores(u);
      }
      for (int u = 0; u < nsteps && ok; ++u) {
        const int hb = u & 1;
        const bool more = u + 2 < nsteps;   // the buffer of step u is free behind its P V: the scores of step u + 2 go there
        if (hb == 0) ok = warp_wait<kSuspendNs>(&bar->v_full[sv], phv, &bar->abort_flag, p.status);   // P V of a first half: its V must have landed
        if (ok && more) ok = key_landed(u + 2);
        if (ok) ok = warp_wait<kSuspendNs>(&bar->p_full[x][hb], pcnt[hb] & 1, &bar->abort_flag, p.status);
        if (!ok) break;
        ++pcnt[hb];
        const uint32_t vb = sV + sv * kTileBytes + hb * (kSub * kD * 2);
        tc_fence_after();
        if (elect_one()) {                 // one lane issues the step's MMAs back to back
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const uint64_t dv = smem_desc(vb + half * kHalfBytes);
#pragma unroll
            for (int c = 0; c < kSub / 16; ++c)
              mma_ts_1(tmem + kColO + x * kV + half * kD, tmem + kColS + x * 128 + hb * kSub + c * 8, desc_advance(dv, c * 2048),
                       kIdescPV, (u > 0 || c > 0) ? 1u : 0u);
          }
        }
        __syncwarp();
        if (u >= nsteps - 2) tc_commit(&bar->pv_done[x]);
        if (hb == 1) {                      // both halves of the V tile are in flight or done
          tc_commit(&bar->v_empty[sv]);
          if (++sv == kVS) { sv = 0; phv ^= 1; }
        }
        if (more) scores(u + 2);
      }
    }
    // Teardown: every MMA issued so far must have retired before tensor memory is released.
    tc_commit(&bar->drain);
    if (lane == 0) {
      const unsigned long long t0 = globaltimer();
      while (!mbar_try(&bar->drain, 0) && globaltimer() - t0 < kWaitLimitNs) {}
    }
    __syncwarp();
  } else {
    // ================= softmax + epilogue: one thread per query row and map =================
    const int x = (warp - kFirstSoftmaxWarp) >> 2;  // map of this warp
    const int q4 = warp & 3;                        // tensor-memory quadrant a warp may touch: warp % 4
    const int r = 32 * q4 + lane;                   // row of the tile
    const uint32_t lane_base = (uint32_t)(q4 << 5) << 16;
    const uint32_t tS0 = tmem + lane_base + kColS + x * 128;   // score buffer 0 (buffer 1: + 64); probabilities over a buffer's first 32 columns
    const uint32_t tO = tmem + lane_base + kColO + x * kV;
    const float sl2 = p.scale_log2;
    const float kLazy = 8.f / sl2;                 // the reference maximum moves only when it grew by > 2^8
    const uint64_t sl2x2 = pack2(sl2, sl2);
    const float lam = x == 0 ? 1.f : -lambda_of(p.tail);
    bool ok = true;
    uint32_t sc = 0;                  // parity of s_full[x][h] in bit h
    int vt = 0;                       // V tiles walked so far
    uint32_t whole = 0;               // items written whole so far: parity of sums_in and read_out

    while (ok && it.next(p.items)) {
      const int nsteps = 2 * (it.t1 - it.t0);
      const Reach reach = reach_of(p.items.kv_len, p.items.q_pos, it.ib, p.items.Nq, p.items.Nk, p.items.causal != 0);
      const int i = it.iqt * kTile + r;                                                  // this thread's query
      const int limit = reach.limit(i), limit0 = reach.limit(it.iqt * kTile + 32 * q4);    // its keys; the fewest of the warp
      // first step of the tile with the last key: rows of V behind it may hold anything, and 0 times that need not be 0
      const int zero_step = reach.len < min(it.n * kTile, p.items.Nk) && it.t1 == it.n ? nsteps - 2 : -1;
      float m = -INFINITY, l = 0.f;
      for (int u = 0; u < nsteps; ++u) {
        const uint32_t tS = tS0 + (u & 1) * kSub;
        const int key0 = (it.t0 + (u >> 1)) * kTile + (u & 1) * kSub;
        ok = warp_wait<kSuspendNs>(&bar->s_full[x][u & 1], (sc >> (u & 1)) & 1, &bar->abort_flag, p.status);
        if (!ok) break;
        sc ^= 1u << (u & 1);
        tc_fence_after();
        uint32_t va[32], vb2[32];
        // ---- pass 1: the step's maximum; both halves of the scores stay in registers for pass 2
        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        tmem_ld32(tS, va);
        tmem_ld32(tS + 32, vb2);
        tmem_wait_ld(va);
        tmem_wait_ld(vb2);
        if (key0 + kSub > limit0) {                 // keys that some row of the warp does not see
          const int nv = limit - key0;
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            if (c >= nv) va[c] = kNegInf;           // exp2(-inf) = 0 and -inf never wins the maximum
            if (c + 32 >= nv) vb2[c] = kNegInf;
          }
        }
        if (u == zero_step) {
          const int s = (vt + (u >> 1)) % kVS;
          ok = warp_wait<kSuspendNs>(&bar->v_full[s], ((vt + (u >> 1)) / kVS) & 1, &bar->abort_flag, p.status);
          if (!ok) break;
          if (key0 + r >= reach.len) {              // (both maps' threads write the same zeros: each map's products wait for its own)
            unsigned char* row = smem + (kQB + kKS + s) * kTileBytes + r * (kD * 2);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              *reinterpret_cast<uint4*>(row + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
              *reinterpret_cast<uint4*>(row + kHalfBytes + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        max32(va, mx4);
        max32(vb2, mx4);
        const float mx = max_of(mx4);
        if (u == nsteps - 1) {         // (a key tile is two steps: u > 0)
          ok = warp_wait<kSuspendNs>(&bar->pv_done[x], 0, &bar->abort_flag, p.status);
          if (!ok) break;
        }
        float o_scale = 1.f;
        if (ref_moves(mx, m, kLazy)) { // always true on the first step, unless all of its scores are -inf
          o_scale = ref_scale(m, mx, sl2);            // first step: 0
          l *= o_scale;
          m = mx;
        }
        if (u > 0 && __any_sync(0xffffffffu, o_scale != 1.f)) {
          // Rare: the reference moved.  O may be touched once the previous step's P V has retired, which the next step's scores
          // say (a look at their barrier; the next step waits for the same phase); the next P V waits for this step's P.
          if (u < nsteps - 1) {
            ok = warp_wait<kSuspendNs>(&bar->s_full[x][(u + 1) & 1], (sc >> ((u + 1) & 1)) & 1, &bar->abort_flag, p.status);
            if (!ok) break;
          }
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < kV / 32; ++c) {
            uint32_t v[32];
            tmem_ld32(tO + 32 * c, v);
            tmem_wait_ld(v);
#pragma unroll
            for (int y = 0; y < 32; ++y) v[y] = __float_as_uint(__uint_as_float(v[y]) * o_scale);
            tmem_st32(tO + 32 * c, v);
          }
          tmem_wait_st();
        }
        // ---- pass 2: exponentials against the reference, P over the scores just consumed
        const float mneg = ref_negative(m, sl2);
        const uint64_t mnegx2 = pack2(mneg, mneg);
        uint64_t lsum[4] = {0ull, 0ull, 0ull, 0ull};
        uint32_t pk[16];
        exp32<false, kPolyOf8, kPolyDeg>(va, sl2x2, mnegx2, lsum, pk, mx4);
        tmem_st16(tS, pk);
        exp32<false, kPolyOf8, kPolyDeg>(vb2, sl2x2, mnegx2, lsum, pk, mx4);
        tmem_st16(tS + 16, pk);
        float a0, a1, b0, b1;
        unpack2(add2(lsum[0], lsum[1]), a0, a1);
        unpack2(add2(lsum[2], lsum[3]), b0, b1);
        l += (a0 + a1) + (b0 + b1);
        // publish P
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&bar->p_full[x][u & 1]);
      }
      if (!ok) break;
      vt += nsteps >> 1;
      ok = warp_wait<kSuspendNs>(&bar->pv_done[x], 1, &bar->abort_flag, p.status);   // the item's last P V
      if (!ok) break;
      tc_fence_after();
      if (!it.whole()) {
        // ---- a part: reference, sum and product of this map as they are
        float* dst = p.partial + ((size_t)partial_slot(blockIdx.x, it.t0) * kTile + r) * kPartial;
        *reinterpret_cast<float2*>(dst + 2 * x) = make_float2(m * sl2, l);
        dst += 4 + kV * x;
#pragma unroll 1
        for (int c = 0; c < kV / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(tO + 32 * c, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int y = 0; y < 8; ++y)
            *reinterpret_cast<uint4*>(dst + 32 * c + 4 * y) = make_uint4(v[4 * y], v[4 * y + 1], v[4 * y + 2], v[4 * y + 3]);
        }
        tc_fence_before();
        continue;
      }
      // ---- the whole: x = O_0 / l_0 - lambda O_1 / l_1 on this thread's 64 channels
      const float mine = lam * ref_inverse(m, l);
      bar->swap[x][r] = mine;
      tc_fence_before();
      mbar_arrive(&bar->sums_in);
      ok = warp_wait<kSuspendNs>(&bar->sums_in, whole & 1, &bar->abort_flag, p.status);
      if (!ok) break;
      tc_fence_after();
      const float other = bar->swap[x ^ 1][r], f0 = x == 0 ? mine : other, f1 = x == 0 ? other : mine;
      const uint32_t tX = tmem + lane_base + kColO + x * kD;
      float out[kD], ss = 0.f;
#pragma unroll
      for (int c = 0; c < kD / 32; ++c) {
        uint32_t v0[32], v1[32];
        tmem_ld32(tX + 32 * c, v0);
        tmem_ld32(tX + kV + 32 * c, v1);
        tmem_wait_ld(v0);
        tmem_wait_ld(v1);
#pragma unroll
        for (int y = 0; y < 32; ++y) {
          const float d = fmaf(__uint_as_float(v0[y]), f0, __uint_as_float(v1[y]) * f1);
          out[32 * c + y] = limit > 0 ? d : 0.f;    // a row that sees no key
          ss = fmaf(out[32 * c + y], out[32 * c + y], ss);
        }
      }
      bar->swap[x ^ 1][r] = ss;                     // (the place that this thread has just read, and nobody else does)
      tc_fence_before();
      mbar_arrive(&bar->read_out);
      ok = warp_wait<kSuspendNs>(&bar->read_out, whole & 1, &bar->abort_flag, p.status);
      if (!ok) break;
      tc_fence_after();
      ++whole;
      float rn = 1.f;
      if (p.tail.norm_w)
        rn = (1.f - p.tail.lambda_init) * rsqrtf((x == 0 ? ss + bar->swap[x][r] : bar->swap[x][r] + ss) * (1.f / kV) + p.tail.norm_eps);
      if (i < p.items.Nq) {
        __nv_bfloat16* dst = p.o + (((size_t)it.ib * 2 * p.pairs + 2 * it.ipair + x) * p.items.Nq + i) * kD;
#pragma unroll
        for (int c = 0; c < kD / 8; ++c) {
          float w[8];
#pragma unroll
          for (int y = 0; y < 8; y += 4) {
            const float4 g = p.tail.norm_w ? __ldg(reinterpret_cast<const float4*>(p.tail.norm_w + kD * x + 8 * c + y)) : make_float4(1.f, 1.f, 1.f, 1.f);
            w[y] = g.x; w[y + 1] = g.y; w[y + 2] = g.z; w[y + 3] = g.w;
          }
          uint32_t pk[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) pk[y] = pack_bf16(out[8 * c + 2 * y] * rn * w[2 * y], out[8 * c + 2 * y + 1] * rn * w[2 * y + 1]);
          *reinterpret_cast<uint4*>(dst + 8 * c) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
        }
      }
    }
  }

  // ================= common teardown =================
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// ---- the partials of an item merged ------------------------------------------------------------------------------------
// Block (c, y): the item that block c of the main launch takes up in its middle, if c is the first that does; rows y, y + gridDim.y, ... by
// the warps.  A lane holds four channels of both maps.
constexpr int kMergeWarps = 8;
__global__ void __launch_bounds__(kMergeWarps * 32) diff_merge_kernel(const DiffParams p, int rows, int blocks) {
  __shared__ int last, begun;
  griddep_wait();
  griddep_launch_dependents();
  const int c = blockIdx.x + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Start s = p.starts[c];
  if (s.tiles == 0 || s.tile == 0) return;
  auto same = [&](const Start& a) { return a.b == s.b && a.qt == s.qt && a.pair == s.pair; };
  if (threadIdx.x == 0) {
    // blocks without tiles lie between; the one before with tiles holds the item's beginning, or takes it up in its middle, too
    int b = c - 1;
    while (b > 0 && p.starts[b].tiles == 0) --b;
    const Start before = p.starts[b];
    begun = same(before) && before.tile > 0 ? -1 : b;
    int e = c;
    bool left = before.left != 0 || s.left != 0;
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
  const float lam = lambda_of(p.tail);
  const Reach reach = reach_of(p.items.kv_len, p.items.q_pos, s.b, p.items.Nq, p.items.Nk, p.items.causal != 0);
  for (int r = blockIdx.y * kMergeWarps + warp; r < rows; r += gridDim.y * kMergeWarps) {
    const int i = s.qt * kTile + r;
    if (i >= p.items.Nq) break;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int k = begun; k <= last; ++k) {
      if (k > begun && p.starts[k].tiles == 0) continue;
      const float* src = p.partial + ((size_t)(2 * k + (k == begun ? 1 : 0)) * kTile + r) * kPartial;
      const float4 st = *reinterpret_cast<const float4*>(src);
      const float pm[2] = {st.x, st.z}, pl[2] = {st.y, st.w};
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float4 a = *reinterpret_cast<const float4*>(src + 4 + kV * h + 4 * lane);
        const float mn = max3(m[h], pm[h], pm[h]), ref = mn == -INFINITY ? 0.f : mn;    // no key of weight so far: weight 0, not NaN
        const float f = ex2(m[h] - ref), g = ex2(pm[h] - ref);
        m[h] = mn;
        l[h] = l[h] * f + pl[h] * g;
        acc[h].x = acc[h].x * f + a.x * g;
        acc[h].y = acc[h].y * f + a.y * g;
        acc[h].z = acc[h].z * f + a.z * g;
        acc[h].w = acc[h].w * f + a.w * g;
      }
    }
    const float f0 = ref_inverse(m[0], l[0]), f1 = -lam * ref_inverse(m[1], l[1]);
    float x[4] = {acc[0].x * f0 + acc[1].x * f1, acc[0].y * f0 + acc[1].y * f1, acc[0].z * f0 + acc[1].z * f1, acc[0].w * f0 + acc[1].w * f1};
    float ss = 0.f;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      if (reach.limit(i) <= 0) x[y] = 0.f;
      ss = fmaf(x[y], x[y], ss);
    }
    if (p.tail.norm_w) {
      const float rn = (1.f - p.tail.lambda_init) * rsqrtf(warp_sum(ss) * (1.f / kV) + p.tail.norm_eps);
      const float4 w = __ldg(reinterpret_cast<const float4*>(p.tail.norm_w + 4 * lane));
      x[0] *= rn * w.x; x[1] *= rn * w.y; x[2] *= rn * w.z; x[3] *= rn * w.w;
    }
    __nv_bfloat16* dst = p.o + (((size_t)s.b * 2 * p.pairs + 2 * s.pair + (lane >> 4)) * p.items.Nq + i) * kD + 4 * (lane & 15);
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  }
}

// Blocks of a call, one per SM at most: one for every item, or for every kTilesMin tiles of the longest that the items can be
constexpr int kTilesMin = 4;
int diff_blocks(int B, int pairs, int Nq, int Nk, bool causal) {
  (void)causal;
  const int64_t items = (int64_t)B * pairs * ceil_div(Nq, kTile), tiles = items * ceil_div(Nk, kTile);
  const int64_t want = items > tiles / kTilesMin ? items : tiles / kTilesMin;
  const int sms = device_sm_count();
  return (int)(want < sms ? want : sms);
}

}  // namespace

size_t diff_workspace_bytes(int B, int pairs, int kv_pairs, int Nq, int Nk, int D, int dtype, bool causal) {
  (void)kv_pairs;
  if (dtype != JV_BF16 || D != kD) return 0;
  const int blocks = diff_blocks(B, pairs, Nq, Nk, causal);
  return align_up((size_t)blocks * sizeof(Start), 256) + (size_t)2 * blocks * kTile * kPartial * 4;
}

bool diff_tc_supported(const DiffArgs& a) { return a.dtype == JV_BF16 && a.D == kD && encode_fn() != nullptr; }

cudaError_t launch_diff_tc(const DiffArgs& a, void* ws, int* status, cudaStream_t st) {
  EncodeFn enc = encode_fn();
  if (!enc) return cudaErrorNotSupported;
  CUtensorMap maps[3];
  const void* ptrs[3] = {a.q, a.k, a.v};
  for (int i = 0; i < 3; ++i) {
    const InStrides& s = i == 0 ? a.qs : a.ks;
    // (channels, tokens, heads, batch elements) with the caller's strides; a box is 128 tokens of one head
    const cuuint64_t dims[4] = {(cuuint64_t)kD, (cuuint64_t)(i == 0 ? a.Nq : a.Nk), (cuuint64_t)(2 * (i == 0 ? a.pairs : a.kv_pairs)), (cuuint64_t)a.B};
    const cuuint64_t strides[3] = {(cuuint64_t)s.tok * 2, (cuuint64_t)s.head * 2, (cuuint64_t)s.batch * 2};
    const cuuint32_t box[4] = {(cuuint32_t)kD, (cuuint32_t)kTile, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    const CUresult r = enc(&maps[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptrs[i]), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cudaErrorInvalidValue;
  }
  static OncePerDevice smem_opt_in;   // > 48 KB of dynamic shared memory: a per-device function attribute
  cudaError_t e = smem_opt_in.run([] {
    return cudaFuncSetAttribute(attn_diff_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const int blocks = diff_blocks(a.B, a.pairs, a.Nq, a.Nk, a.causal);
  DiffParams p;
  p.items = Items{a.B, ceil_div(a.Nq, kTile), a.pairs, a.Nq, a.Nk, kTile, a.causal ? 1 : 0, a.kv_len, a.q_pos};
  p.tail = Tail{a.lambda, a.lambda_init, a.norm_w, a.norm_eps, kD};
  p.o = (__nv_bfloat16*)a.o;
  p.starts = (Start*)ws;
  p.partial = (float*)((char*)ws + align_up((size_t)blocks * sizeof(Start), 256));
  p.status = status;
  p.pairs = a.pairs;
  p.share = a.pairs / a.kv_pairs;
  p.scale_log2 = a.scale * 1.4426950408889634f;
  e = launch_programmatic(attn_diff_kernel, dim3((unsigned)blocks), kThreads, kSmemBytes, st, maps[0], maps[1], maps[2], p);
  if (e != cudaSuccess || blocks == 1) return e;
  const int rows = a.Nq < kTile ? a.Nq : kTile;
  return launch_programmatic(diff_merge_kernel, dim3((unsigned)(blocks - 1), (unsigned)ceil_div(rows, kMergeWarps)), kMergeWarps * 32, 0, st, p, rows, blocks);
}

}  // namespace jv

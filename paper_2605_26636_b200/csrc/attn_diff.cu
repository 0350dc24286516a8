// Differential attention on the 5th-generation tensor cores: bf16, 64 channels a map, tiles of 128 queries of a pair of heads.
//
// A tile of 128 tokens lies in shared memory as two 128-byte-swizzled halves of 64 channels, the two heads of the pair.  Map m is
// S_m = Q_m K_m^T over half m alone (4 MMAs of K = 16), and both maps multiply the same values, O_m += P_m V over both halves of V
// (4 MMAs).  Warp roles (20 warps): a TMA producer, an MMA issuer per map, and four sets of four softmax warps, one thread per query
// row: set (m, h) takes the steps of 64 keys u = h, h + 2, ... of map m.  Tensor memory, 512 columns: 64 of scores per map, 32
// of probabilities (bf16) per set, 128 of accumulator per map.
//
// A set takes its 64 scores a row into registers at once, so the buffer is free for the next step's as soon as they are read: the other
// set of the map finds them there when it is done with its step before, and neither ever waits for the tensor pipe in the steady
// state.  (With probabilities over the scores they came from, as the other kernels here have them, the chain  scores -> softmax -> product ->
// next scores  was in the open a third of the time, with two softmax warps per sub-core or with four: four grids of 73 x 73 tokens, 8
// pairs, 882 and 856 us.)
//
// The two sets of a map add to one accumulator, so they share its reference: a row's reference lies in shared memory, every step looks at
// it and raises it lazily.  The issuer sees to the order: it issues the scores of step u + 1 when the reference of step u stands, which
// is also when that step's scores have been read.  Each set keeps its own sum.
//
// Behind an item's last key each of a row's four threads takes 32 channels from both accumulators: the sums and the shares of
// the row's mean square are exchanged through shared memory, the difference is normalised and written.  Parts of an item (see
// attn_diff.cuh) go to the workspace as they are.
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
constexpr int kQB = 2, kKS = 2, kVS = 2;    // query buffers, ring depths
constexpr int kWarps = 20;
constexpr int kThreads = kWarps * 32;
constexpr int kFirstSoftmaxWarp = 4;
// Registers: a block is launched with 96 a thread; the first four warps hand back 64 each, the sixteen softmax warps take 16 each, so
// that a step's 64 scores stay in registers between the maximum and the exponentials
constexpr int kRegsRoles = 32, kRegsSoftmax = 112;
static_assert(128 * kRegsRoles + 512 * kRegsSoftmax <= kThreads * 96, "registers of a block");
constexpr uint32_t kTmemCols = 512;
constexpr int kSub = 64;                    // keys per step
constexpr int kPolyOf8 = 2, kPolyDeg = 3;   // of every 8 score pairs, this many take the polynomial exponential, of this degree
// Tensor-memory columns: scores of map m at 64 m, probabilities of set s at 128 + 32 s, O_m at 256 + 128 m
constexpr uint32_t kColS = 0, kColP = 128, kColO = 256;

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
  // per map and set, once a step: its scores are there; they have been read and its reference stands; its probabilities are
  // there; its product has retired
  uint64_t s_full[2][2], decided[2][2], p_full[2][2], pv_done[2][2];
  uint64_t sums_in, read_out;            // per item: the sets' sums are there; they and the accumulators have been read
  uint64_t drain;
  long long scan[33];                    // for find_start
  Start start;
  float ref[2][kTile], base[2][kTile], sum[2][2][kTile], square[4][kTile];   // base: the reference of set (m, 0)'s sum
  uint32_t tmem_base;
  volatile uint32_t abort_flag;
};
constexpr size_t kSmemTiles = (kQB + kKS + kVS) * (size_t)kTileBytes;          // 224 KB
constexpr size_t kSmemBytes = kSmemTiles + sizeof(Barriers) + 1024;            // + alignment slack
static_assert(kSmemBytes <= 227 * 1024, "shared memory of one block");

constexpr uint32_t kIdescQK = idesc(kTile, kSub, 0);       // S = Q K^T: M128 N64, both operands K-major
constexpr uint32_t kIdescPV = idesc(kTile, kV, 1);         // O = P V: M128 N128, V MN-major

// tcgen05.commit of everything this thread has issued, to be called by one lane
__device__ __forceinline__ void commit_1(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

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
        mbar_init(&bar->p_full[m][h], 4);       // one arrival from each warp of the set
        mbar_init(&bar->decided[m][h], 4);
        mbar_init(&bar->pv_done[m][h], 1);
      }
    }
    for (int s = 0; s < kKS; ++s) {
      mbar_init(&bar->k_full[s], 1);
      mbar_init(&bar->k_empty[s], 2);
    }
    for (int s = 0; s < kVS; ++s) {
      mbar_init(&bar->v_full[s], 1);
      mbar_init(&bar->v_empty[s], 2);
    }
    mbar_init(&bar->sums_in, 512);
    mbar_init(&bar->read_out, 512);
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

  if (warp < kFirstSoftmaxWarp) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRoles));
  else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));

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
  } else if (warp < 3) {
    // ================= MMA issuer of map x =================
    // Over the block's steps g of 64 keys, one item behind the other (key tile g / 2, half g % 2):
    //   S(g) = Q_x K_x(g)^T      4 MMAs, M128 N64 K16, operands in shared memory
    //   O   += P(g) V(g)         4 MMAs, M128 N128 K16, A = P in tensor memory, V from both heads' halves
    // S(g + 1) is issued when step g has read its scores, the product of step g - 1 behind it; at the first step of an item the other way
    // round, since its set first has to see the item before to its end.  One election a phase, addresses from running descriptors.
    const int x = warp - 1;
    const uint32_t dS = tmem + kColS + x * kSub, dP = tmem + kColP + x * kSub, dO = tmem + kColO + x * kV;
    const uint64_t dQ0 = smem_desc(sQ + x * kHalfBytes), dK0 = smem_desc(sK + x * kHalfBytes);
    const uint64_t dV0 = (smem_desc(sV) & ~(0x3FFFull << 16)) | ((uint64_t)(kHalfBytes >> 4) << 16);   // the next 64 channels lie kHalfBytes on
    bool ok = true;
    Walk itv = it;                          // the products' walk (it: the scores')
    int qn = 0, sk = 0, sv = 0;             // items of the scores' walk, ring stages of the next key and value tile
    uint32_t phk = 0, phv = 0;              // and their "full" parities
    int s_left = 0, v_left = 0;             // steps left of the walks' items
    bool v_first = false;                   // the next product is an item's first
    // Scores of the next step, of half h of its tile; false if there is none (or the wait has run out: ok)
    auto next_scores = [&](uint32_t h) -> bool {
      if (s_left == 0) {
        if (!it.next(p.items)) return false;
        s_left = 2 * (it.t1 - it.t0);
        ok = warp_wait<kSuspendNs>(&bar->q_full[qn & 1], (qn >> 1) & 1, &bar->abort_flag, p.status);
        if (!ok) return false;
        ++qn;
      }
      if (h == 0) {
        ok = warp_wait<kSuspendNs>(&bar->k_full[sk], phk, &bar->abort_flag, p.status);
        if (!ok) return false;
      }
      tc_fence_after();
      const int qb = (qn - 1) & 1;
      --s_left;
      if (elect_one()) {
        const uint64_t dq = dQ0 + (uint64_t)(qb * (kTileBytes >> 4)), dk = dK0 + (uint64_t)(sk * (kTileBytes >> 4));
#pragma unroll
        for (int c = 0; c < kD / 16; ++c)
          mma_ss_1(dS, desc_advance(dq, c * 32), desc_advance(dk, h * (kSub * kD * 2) + c * 32), kIdescQK, c > 0 ? 1u : 0u);
        commit_1(&bar->s_full[x][h]);
        if (h == 1) commit_1(&bar->k_empty[sk]);
        if (s_left == 0) commit_1(&bar->q_empty[qb]);        // the item's last scores: its query tile may be replaced
      }
      __syncwarp();
      if (h == 1 && ++sk == kKS) { sk = 0; phk ^= 1; }
      return true;
    };
    // Product of the next step, of half h of its tile; par: parity of its probabilities' barrier
    auto next_product = [&](uint32_t h, uint32_t par) {
      if (v_left == 0) {
        itv.next(p.items);
        v_left = 2 * (itv.t1 - itv.t0);
        v_first = true;
      }
      if (h == 0) ok = warp_wait<kSuspendNs>(&bar->v_full[sv], phv, &bar->abort_flag, p.status);
      if (ok) ok = warp_wait<kSuspendNs>(&bar->p_full[x][h], par, &bar->abort_flag, p.status);
      if (!ok) return;
      tc_fence_after();
      if (elect_one()) {
        const uint64_t dv = dV0 + (uint64_t)(sv * (kTileBytes >> 4));
#pragma unroll
        for (int c = 0; c < kSub / 16; ++c)
          mma_ts_1(dO, dP + h * 32 + c * 8, desc_advance(dv, h * (kSub * kD * 2) + c * 2048), kIdescPV, c > 0 || !v_first ? 1u : 0u);
        commit_1(&bar->pv_done[x][h]);
        if (h == 1) commit_1(&bar->v_empty[sv]);
      }
      __syncwarp();
      v_first = false;
      --v_left;
      if (h == 1 && ++sv == kVS) { sv = 0; phv ^= 1; }
    };
    bool more = next_scores(0);
    for (uint32_t g = 0; more && ok; ++g) {           // step g has its scores
      const uint32_t h = g & 1, par = (g >> 1) & 1;
      const bool first = g > 0 && v_left == 1;        // step g begins an item: the product before it is an item's last
      if (first) next_product(h ^ 1, ((g - 1) >> 1) & 1);
      if (ok) ok = warp_wait<kSuspendNs>(&bar->decided[x][h], par, &bar->abort_flag, p.status);
      if (!ok) break;
      more = next_scores(h ^ 1);
      if (ok && g > 0 && !first) next_product(h ^ 1, ((g - 1) >> 1) & 1);
      if (ok && !more) next_product(h, par);          // the block's last step
    }
    // Teardown: every MMA issued so far must have retired before tensor memory is released.
    tc_commit(&bar->drain);
    if (lane == 0) {
      const unsigned long long t0 = globaltimer();
      while (!mbar_try(&bar->drain, 0) && globaltimer() - t0 < kWaitLimitNs) {}
    }
    __syncwarp();
  } else if (warp >= kFirstSoftmaxWarp) {
    // ================= softmax + epilogue: one thread per query row, map and parity of the step =================
    const int set = (warp - kFirstSoftmaxWarp) >> 2, x = set >> 1, hb = set & 1;   // map, and parity of the steps, of this warp
    const int q4 = warp & 3;                        // tensor-memory quadrant a warp may touch: warp % 4
    const int r = 32 * q4 + lane;                   // row of the tile
    const uint32_t lane_base = (uint32_t)(q4 << 5) << 16;
    const uint32_t tS = tmem + lane_base + kColS + x * kSub, tP = tmem + lane_base + kColP + 32 * set;
    const uint32_t tO = tmem + lane_base + kColO + x * kV;
    const float sl2 = p.scale_log2;
    const float kLazy = 8.f / sl2;                 // the reference moves only when the maximum grew by > 2^8
    const uint64_t sl2x2 = pack2(sl2, sl2);
    const float lam = lambda_of(p.tail);
    bool ok = true;
    uint32_t n = 0;                   // steps of this set so far: parity of its barriers; the map's other set has done as many before an item
    int vt = 0;                       // V tiles walked so far
    uint32_t items = 0;               // items so far: parity of sums_in and read_out

    while (ok && it.next(p.items)) {
      const int nsteps = 2 * (it.t1 - it.t0);
      const Reach reach = reach_of(p.items.kv_len, p.items.q_pos, it.ib, p.items.Nq, p.items.Nk, p.items.causal != 0);
      const int i = it.iqt * kTile + r;                                                  // this thread's query
      const int limit = reach.limit(i), limit0 = reach.limit(it.iqt * kTile + 32 * q4);    // its keys; the fewest of the warp
      // steps of the tile with the last key: rows of V behind it may hold anything, and 0 times that need not be 0
      const int zero_step = reach.len < min(it.n * kTile, p.items.Nk) && it.t1 == it.n ? nsteps - 2 + hb : -1;
      float m = -INFINITY, l = 0.f;
      for (int u = hb; u < nsteps; u += 2, ++n) {
        const int key0 = (it.t0 + (u >> 1)) * kTile + hb * kSub;
        ok = warp_wait<kSuspendNs>(&bar->s_full[x][hb], n & 1, &bar->abort_flag, p.status);
        if (!ok) break;
        tc_fence_after();
        const bool masked = key0 + kSub > limit0;       // keys that some row of the warp does not see
        uint32_t va[32], vb[32];
        if (u == zero_step) {
          const int s = (vt + (u >> 1)) % kVS;
          ok = warp_wait<kSuspendNs>(&bar->v_full[s], ((vt + (u >> 1)) / kVS) & 1, &bar->abort_flag, p.status);
          if (!ok) break;
          // this step's half of the tile, both maps' threads the same zeros: each map's products wait for its own
          const int row = hb * kSub + (r >> 1);
          if (key0 + (r >> 1) >= reach.len) {
            unsigned char* dst = smem + (kQB + kKS + s) * kTileBytes + (r & 1) * kHalfBytes + row * (kD * 2);
#pragma unroll
            for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(dst + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        // ---- pass 1: the step's maximum
        float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        tmem_ld32(tS, va);
        tmem_ld32(tS + 32, vb);
        const float now = bar->ref[x][r];              // the reference as the step before has left it
        tmem_wait_ld(va);
        tmem_wait_ld(vb);
        if (masked) {
          const int nv = limit - key0;
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            if (c >= nv) va[c] = kNegInf;              // exp2(-inf) = 0 and -inf never wins the maximum
            if (c + 32 >= nv) vb[c] = kNegInf;
          }
        }
        max32(va, mx4);
        max32(vb, mx4);
        const float mx = max_of(mx4);
        if (u > 0 && now != m) {       // the step before has moved the reference (no number: always)
          l *= ref_scale(m, now, sl2);
          m = now;
        }
        float o_scale = 1.f;
        if (ref_moves(mx, m, kLazy)) { // always on the first step, unless all of its scores are -inf
          o_scale = ref_scale(m, mx, sl2);              // first step: 0
          l *= o_scale;
          m = mx;
          bar->ref[x][r] = m;
        } else if (u == 0) {
          bar->ref[x][r] = m;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->decided[x][hb]);
        if (u > 0 && __any_sync(0xffffffffu, o_scale != 1.f)) {
          // Rare: the reference moved.  O may be touched once the previous step's P V has retired; the next one waits for this step's P.
          ok = warp_wait<kSuspendNs>(&bar->pv_done[x][hb ^ 1], (n + hb + 1) & 1, &bar->abort_flag, p.status);
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < kV; c += 8) {    // (few registers: the scores stay where they are)
            uint32_t v[8];
            asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];\n\ttcgen05.wait::ld.sync.aligned;"
                         : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "r"(tO + c) : "memory");
#pragma unroll
            for (int y = 0; y < 8; ++y) v[y] = __float_as_uint(__uint_as_float(v[y]) * o_scale);
            asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                         ::"r"(tO + c), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
          }
          tmem_wait_st();
        }
        // ---- pass 2: exponentials against the reference
        const float mneg = ref_negative(m, sl2);
        const uint64_t mnegx2 = pack2(mneg, mneg);
        uint64_t lsum[4] = {0ull, 0ull, 0ull, 0ull};
        uint32_t pk[16];
        exp32<false, kPolyOf8, kPolyDeg>(va, sl2x2, mnegx2, lsum, pk, mx4);
        if (n > 0) {                   // P(u - 2) has been read
          ok = warp_wait<kSuspendNs>(&bar->pv_done[x][hb], (n + 1) & 1, &bar->abort_flag, p.status);
          if (!ok) break;
          tc_fence_after();
        }
        tmem_st16(tP, pk);
        exp32<false, kPolyOf8, kPolyDeg>(vb, sl2x2, mnegx2, lsum, pk, mx4);
        tmem_st16(tP + 16, pk);
        float a0, a1, b0, b1;
        unpack2(add2(lsum[0], lsum[1]), a0, a1);
        unpack2(add2(lsum[2], lsum[3]), b0, b1);
        l += (a0 + a1) + (b0 + b1);
        // publish P
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->p_full[x][hb]);
      }
      if (!ok) break;
      vt += nsteps >> 1;
      bar->sum[x][hb][r] = l;
      if (hb == 0) {
        bar->base[x][r] = m;           // (the last step, the other set's, may still move the reference)
      } else {                         // the item's last product: the sets of parity 1 wait for it, the others for them
        ok = warp_wait<kSuspendNs>(&bar->pv_done[x][1], (n + 1) & 1, &bar->abort_flag, p.status);
        if (!ok) break;
      }
      tc_fence_after();
      tc_fence_before();
      mbar_arrive(&bar->sums_in);
      ok = warp_wait<kSuspendNs>(&bar->sums_in, items & 1, &bar->abort_flag, p.status);
      if (!ok) break;
      tc_fence_after();
      auto total = [&](int map) {
        const float now = bar->ref[map][r], was = bar->base[map][r], s = bar->sum[map][0][r];
        return (now != was ? s * ref_scale(was, now, sl2) : s) + bar->sum[map][1][r];
      };
      if (!it.whole()) {
        // ---- a part: reference, sum and product of this map as they are, half the channels to each set
        float* dst = p.partial + ((size_t)partial_slot(blockIdx.x, it.t0) * kTile + r) * kPartial;
        if (hb == 0) *reinterpret_cast<float2*>(dst + 2 * x) = make_float2(bar->ref[x][r] * sl2, total(x));
        dst += 4 + kV * x + kD * hb;
#pragma unroll 1
        for (int c = 0; c < kD / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(tO + kD * hb + 32 * c, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int y = 0; y < 8; ++y)
            *reinterpret_cast<uint4*>(dst + 32 * c + 4 * y) = make_uint4(v[4 * y], v[4 * y + 1], v[4 * y + 2], v[4 * y + 3]);
        }
        tc_fence_before();
        mbar_arrive(&bar->read_out);
        ok = warp_wait<kSuspendNs>(&bar->read_out, items & 1, &bar->abort_flag, p.status);
        ++items;
        continue;
      }
      // ---- the whole: x = O_0 / l_0 - lambda O_1 / l_1 on this thread's 32 channels
      const float f0 = ref_inverse(bar->ref[0][r], total(0));
      const float f1 = -lam * ref_inverse(bar->ref[1][r], total(1));
      const uint32_t tX = tmem + lane_base + kColO + 32 * set;
      float out[32], ss = 0.f;
      {
        uint32_t v[32];
        tmem_ld32(tX, v);
        tmem_wait_ld(v);
#pragma unroll
        for (int y = 0; y < 32; ++y) out[y] = __uint_as_float(v[y]) * f0;
        tmem_ld32(tX + kV, v);
        tmem_wait_ld(v);
#pragma unroll
        for (int y = 0; y < 32; ++y) {
          const float d = fmaf(__uint_as_float(v[y]), f1, out[y]);
          out[y] = limit > 0 ? d : 0.f;             // a row that sees no key
          ss = fmaf(out[y], out[y], ss);
        }
      }
      bar->square[set][r] = ss;
      tc_fence_before();
      mbar_arrive(&bar->read_out);
      ok = warp_wait<kSuspendNs>(&bar->read_out, items & 1, &bar->abort_flag, p.status);
      if (!ok) break;
      tc_fence_after();
      ++items;
      float rn = 1.f;
      if (p.tail.norm_w)
        rn = (1.f - p.tail.lambda_init) *
             rsqrtf(((bar->square[0][r] + bar->square[1][r]) + (bar->square[2][r] + bar->square[3][r])) * (1.f / kV) + p.tail.norm_eps);
      if (i < p.items.Nq) {
        __nv_bfloat16* dst = p.o + (((size_t)it.ib * 2 * p.pairs + 2 * it.ipair + x) * p.items.Nq + i) * kD + 32 * hb;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float w[8];
#pragma unroll
          for (int y = 0; y < 8; y += 4) {
            const float4 g = p.tail.norm_w ? __ldg(reinterpret_cast<const float4*>(p.tail.norm_w + 32 * set + 8 * c + y)) : make_float4(1.f, 1.f, 1.f, 1.f);
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
    cudaFuncAttributes attr;       // the split of the registers counts on those that a block is launched with
    const cudaError_t r = cudaFuncGetAttributes(&attr, attn_diff_kernel);
    if (r != cudaSuccess) return r;
    if (attr.numRegs * kThreads < 128 * kRegsRoles + 512 * kRegsSoftmax) return cudaErrorInvalidConfiguration;
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

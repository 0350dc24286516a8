// Differential attention on the 5th-generation tensor cores: bf16, 64 channels a map, tiles of 128 queries of a pair of heads.
//
// A tile of 128 tokens lies in shared memory as two 128-byte-swizzled halves of 64 channels, the two heads of the pair.  Map m is
// S_m = Q_m K_m^T over half m alone (4 MMAs of K = 16), and both maps multiply the same values, O_m += P_m V over both halves of V
// (4 MMAs).  Warp roles (20 warps): a TMA producer, an issuer of both maps' scores, an issuer of each map's products, and four sets of
// four softmax warps, one thread per query row: set (m, h) takes the steps of 64 keys u = h, h + 2, ... of map m.  Tensor memory, 512
// columns: 64 of scores per map, 32 of probabilities (bf16) per set, 128 of accumulator per map.
//
// A set takes its 64 scores a row into registers at once, so the buffer is free for the next step's as soon as they are read: the other
// set of the map finds them there when it is done with its step before, and no set waits for the tensor pipe in the steady
// state.
//
// The softmax has no running maximum.  The two sets of a map add to one accumulator, so all their exponentials are against one reference
// a row: the maximum of the first 64 keys of the item, or of the block's part of it.  A later score may lie far above it: probabilities,
// sums and accumulators are floating point with 8 bits of exponent, and as precise at 2^60 as at 1.  A row whose sum leaves
// [2^-60, 2^60] in some part, whose result is not finite, or whose mean square is not safely within fp32, is marked, and done again by
// the second launch, exactly and slowly, from the inputs (so are infinities and NaN among them).  That takes a score 41 above every one of
// those 64 keys (or, where none of them weighs anything, 41 off zero).  A call all of whose rows are so takes 60 ms where it takes 0.13 (two
// causal prompts of 4096 tokens, 8 pairs).  It saves the maximum of every other
// step, and its order between the sets: half of a step's instructions.  The exponentials are all the MUFU unit's: it gives 0 for a key
// that scores -inf, and two of eight by a polynomial are no faster (B = 4, 8 pairs, 73 x 73 tokens, without second terms: 651 us, 661).
//
// What bounds a step is the latency between its roles (MUFU unit 59 %, issue slots 54 %, tensor pipe 51 % of two causal prompts of 4096
// tokens), first the chain of the warps that issue for it: beside four busy softmax warps in its sub-core an instruction takes such a
// warp some 8 clocks, a look at a barrier 110 and more.  Scores and products from one warp per map, each phase elected and
// voted on by the whole warp, cost it 1300 clocks a step, whatever was left out of the arithmetic.  So one lane per role, three
// issuers, and the softmax warps' looks at their barriers ahead of the arithmetic that hides them.
//
// The difference of the maps is smaller than either: bf16 probabilities left o at 2.6e-3 of the exact result (its own rounding: 1.7e-3).
// So map 0, which weighs most, has its probabilities of kLoKeys of every 64 keys as two bf16 terms: what the rounding took off them
// goes through shared memory (tensor memory is full) into products of their own: 2.4e-3, and 652 us become 735 at 73 x 73 tokens.
//
// Behind an item's last key each of a row's four threads takes 32 channels from both accumulators: the sums and the shares of
// the row's mean square are exchanged through shared memory, the difference is normalised and written.  Parts of an item (see
// attn_diff.cuh) go to the workspace as they are.
//
// Measured, with the launch that merges: B = 4, 8 pairs, 73 x 73 tokens 735 us (850 at the power cap; 698 GF: 950 TF), two causal prompts
// of 4096 tokens, 8 pairs, 127 to 143 us by the board, 256 queries against 16384 keys, 8 pairs, 48 us.
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
constexpr uint32_t kTmemCols = 512;
constexpr int kSub = 64;                    // keys per step
constexpr int kLoKeys = 32;                 // of them, the first, with a second term in map 0
constexpr int kLoBytes = kTile * kLoKeys * 2;   // of a set: rows of 64 bytes, 64-byte swizzle
constexpr float kFine = 1152921504606846976.f;   // 2^60: sums between this and its inverse are used as they are
// Tensor-memory columns: scores of map m at 64 m, probabilities of set s at 128 + 32 s, O_m at 256 + 128 m
constexpr uint32_t kColS = 0, kColP = 128, kColO = 256;

struct __align__(8) Barriers {
  uint64_t q_full[kQB], q_empty[kQB];
  uint64_t k_full[kKS], k_empty[kKS], v_full[kVS], v_empty[kVS];
  // per map and set, once a step: its scores are there; they have been read; its probabilities are there; its product has retired
  uint64_t s_full[2][2], s_read[2][2], p_full[2][2], pv_done[2][2];
  uint64_t ref_set[2];                   // per map, once an item: its references stand
  uint64_t sums_in, read_out;            // per item: the sets' sums are there; they and the accumulators have been read
  uint64_t drain;
  long long scan[34];                    // for find_start
  Start start;
  float ref[2][kTile], sum[2][2][kTile], square[4][kTile];   // ref: minus the reference, times the scale
  uint32_t tmem_base;
  volatile uint32_t abort_flag;
  int redo;
};
constexpr size_t kSmemTiles = (kQB + kKS + kVS) * (size_t)kTileBytes;          // 192 KB
constexpr size_t kSmemLo = 2 * (size_t)kLoBytes;                               // the two sets of map 0
constexpr size_t kSmemBytes = kSmemTiles + kSmemLo + sizeof(Barriers) + 1024;  // + alignment slack
static_assert(kSmemBytes <= 227 * 1024, "shared memory of one block");

constexpr uint32_t kIdescQK = idesc(kTile, kSub, 0);       // S = Q K^T: M128 N64, both operands K-major
constexpr uint32_t kIdescPV = idesc(kTile, kV, 1);         // O = P V: M128 N128, V MN-major

// tcgen05.commit of everything this thread has issued, to be called by one lane
__device__ __forceinline__ void commit_1(uint64_t* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// Descriptor of a K-major operand in rows of 64 bytes, 64-byte swizzle (16-byte chunk c of row r at c ^ (r / 2 % 4)), 8-row groups 512
// bytes apart; 32 bytes on per K step of 16
__device__ __forceinline__ uint64_t smem_desc_64(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (1ull << 16) /* LBO (unused) */ | (32ull << 32) /* SBO = 512 B */ |
         (1ull << 46) /* descriptor version */ | (4ull << 61) /* SWIZZLE_64B */;
}
// p = exp2(s * sl2 + neg) for 32 scores; adds them into four packed partial sums and packs them to bf16 pairs (even key low).  lo: where
// what the rounding takes off goes, this thread's row in four chunks of 16 bytes (chunk c at lo + 16 (c ^ turn)); null: nowhere.
__device__ __forceinline__ void weights32(const uint32_t (&v)[32], uint64_t sl2x2, uint64_t neg2, uint64_t (&lsum)[4], uint32_t (&pk)[16],
                                          unsigned char* lo, int turn) {
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint64_t pp[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = 4 * c + j;
      float x0, x1;
      unpack2(fma2(pack2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), sl2x2, neg2), x0, x1);
      const float p0 = ex2(x0), p1 = ex2(x1);
      pp[j] = pack2(p0, p1);
      lsum[j] = add2(lsum[j], pp[j]);
      pk[i] = pack_bf16(p0, p1);
    }
    if (lo) {
      uint32_t r[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t h = pk[4 * c + j];
        float r0, r1;
        unpack2(fma2(pack2(__uint_as_float(h << 16), __uint_as_float(h & 0xffff0000u)), pack2(-1.f, -1.f), pp[j]), r0, r1);
        r[j] = pack_bf16(r0, r1);
      }
      *reinterpret_cast<uint4*>(lo + 16 * (c ^ turn)) = make_uint4(r[0], r[1], r[2], r[3]);
    }
  }
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
  Barriers* bar = reinterpret_cast<Barriers*>(smem + kSmemTiles + kSmemLo);
  const uint32_t sQ = smem_u32(smem), sK = sQ + kQB * kTileBytes, sV = sK + kKS * kTileBytes, sLo = sV + kVS * kTileBytes;

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kQB; ++i) {
      mbar_init(&bar->q_full[i], 1);
      mbar_init(&bar->q_empty[i], 1);
    }
    for (int m = 0; m < 2; ++m) {
      for (int h = 0; h < 2; ++h) {
        mbar_init(&bar->s_full[m][h], 1);
        mbar_init(&bar->p_full[m][h], 4);       // one arrival from each warp of the set
        mbar_init(&bar->s_read[m][h], 4);
        mbar_init(&bar->pv_done[m][h], 1);
      }
      mbar_init(&bar->ref_set[m], 4);
    }
    for (int s = 0; s < kKS; ++s) {
      mbar_init(&bar->k_full[s], 1);
      mbar_init(&bar->k_empty[s], 1);
    }
    for (int s = 0; s < kVS; ++s) {
      mbar_init(&bar->v_full[s], 1);
      mbar_init(&bar->v_empty[s], 2);         // one commit from each issuer of products
    }
    mbar_init(&bar->sums_in, 512);
    mbar_init(&bar->read_out, 512);
    mbar_init(&bar->drain, 3);
    bar->abort_flag = 0;
    bar->redo = 0;
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
    s.left = bar->abort_flag;          // (redo follows at the end)
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
    // ================= TMA producer (one lane) =================
    if (elect_one()) {
      // a tile = two boxes of 64 channels x 128 tokens, one per head of the pair
      auto load_tile = [&](uint32_t dst, const CUtensorMap* map, uint64_t* full, int row, int h, int b) {
        mbar_expect_tx(full, kTileBytes);
        tma_load_4d(dst, map, full, 0, row, h, b);
        tma_load_4d(dst + kHalfBytes, map, full, 0, row, h + 1, b);
      };
      auto wait = [&](uint64_t* b, uint32_t parity) { return mbar_wait<kSuspendNs>(b, parity, &bar->abort_flag, p.status); };
      bool ok = true;
      int n = 0;                 // items seen
      int ks = 0, vs = 0;        // ring stages of the next K and V tile
      uint32_t kpar = 1, vpar = 1;   // parity of the "empty" phase this pass over each ring waits for
      int issued_q = 0, issued_k = 0, issued_v = 0;   // for the abort path: tiles whose copies have been issued so far
      while (ok && it.next(p.items)) {
        const int hk = 2 * (it.ipair / p.share), qb = n & 1;
        ok = wait(&bar->q_empty[qb], ((n >> 1) & 1) ^ 1);
        if (!ok) break;
        load_tile(sQ + qb * kTileBytes, &mapQ, &bar->q_full[qb], it.iqt * kTile, 2 * it.ipair, it.ib);
        ++issued_q;
        for (int j = it.t0; j < it.t1; ++j) {
          ok = wait(&bar->k_empty[ks], kpar);
          if (!ok) break;
          load_tile(sK + ks * kTileBytes, &mapK, &bar->k_full[ks], j * kTile, hk, it.ib);
          ++issued_k;
          if (++ks == kKS) { ks = 0; kpar ^= 1; }
          ok = wait(&bar->v_empty[vs], vpar);
          if (!ok) break;
          load_tile(sV + vs * kTileBytes, &mapV, &bar->v_full[vs], j * kTile, hk, it.ib);
          ++issued_v;
          if (++vs == kVS) { vs = 0; vpar ^= 1; }
        }
        ++n;
      }
      if (!ok) {
        // let the copies still in flight land before the CTA leaves (bounded by the same limit)
        const unsigned long long t0 = globaltimer();
        auto landed = [&](uint64_t* full, int ring, int issued) {
          for (int g = max(0, issued - ring); g < issued; ++g)
            while (!mbar_try(&full[g % ring], (g / ring) & 1) && globaltimer() - t0 < kWaitLimitNs) {}
        };
        landed(bar->q_full, kQB, issued_q);
        landed(bar->k_full, kKS, issued_k);
        landed(bar->v_full, kVS, issued_v);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ================= issuer of scores (one lane) =================
    // S_x(g) = Q_x K_x(g)^T for both maps x over the block's steps g of 64 keys, one item behind the other (key tile g / 2, half g % 2):
    // 4 MMAs, M128 N64 K16, operands in shared memory, once step g - 1 of the map has read its scores.
    if (elect_one()) {
      const uint64_t dQ0 = smem_desc(sQ), dK0 = smem_desc(sK);
      auto wait = [&](uint64_t* b, uint32_t parity) { return mbar_wait(b, parity, &bar->abort_flag, p.status); };
      bool ok = true, begun = false;
      int n = 0, sk = 0;
      uint32_t phk = 0, par = 0;              // parity of the ring, and of a tile's barriers
      while (ok && it.next(p.items)) {
        const int qb = n & 1;
        const uint64_t dq = dQ0 + (uint64_t)(qb * (kTileBytes >> 4));
        ok = wait(&bar->q_full[qb], (n >> 1) & 1);
        for (int j = it.t0; j < it.t1 && ok; ++j) {
          const uint64_t dk = dK0 + (uint64_t)(sk * (kTileBytes >> 4));
          ok = wait(&bar->k_full[sk], phk);
          tc_fence_after();
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              // the step before: half 1 of the tile before, or half 0 of this one
              if (ok && (h == 1 || begun)) ok = wait(&bar->s_read[x][h ^ 1], h == 1 ? par : par ^ 1);
              if (!ok) break;
              tc_fence_after();
#pragma unroll
              for (int c = 0; c < kD / 16; ++c)
                mma_ss_1(tmem + kColS + x * kSub, desc_advance(dq, x * kHalfBytes + c * 32),
                         desc_advance(dk, x * kHalfBytes + h * (kSub * kD * 2) + c * 32), kIdescQK, c > 0 ? 1u : 0u);
              commit_1(&bar->s_full[x][h]);
            }
          if (!ok) break;
          commit_1(&bar->k_empty[sk]);
          if (j + 1 == it.t1) commit_1(&bar->q_empty[qb]);     // the item's last scores: its query tile may be replaced
          begun = true;
          par ^= 1;
          if (++sk == kKS) { sk = 0; phk ^= 1; }
        }
        ++n;
      }
      // Teardown: every MMA issued so far must have retired before tensor memory is released.
      commit_1(&bar->drain);
      const unsigned long long t0 = globaltimer();
      while (!mbar_try(&bar->drain, 0) && globaltimer() - t0 < kWaitLimitNs) {}
    }
    __syncwarp();
  } else if (warp < kFirstSoftmaxWarp) {
    // ================= issuer of map x's products (one lane) =================
    // O_x += P_x(g) V(g): 4 MMAs, M128 N128 K16, A = P in tensor memory, V from both heads' halves.
    if (elect_one()) {
      const int x = warp - 2;
      const uint32_t dP = tmem + kColP + x * 64, dO = tmem + kColO + x * kV;
      const uint64_t dV0 = (smem_desc(sV) & ~(0x3FFFull << 16)) | ((uint64_t)(kHalfBytes >> 4) << 16);   // the next 64 channels lie kHalfBytes on
      auto wait = [&](uint64_t* b, uint32_t parity) { return mbar_wait(b, parity, &bar->abort_flag, p.status); };
      bool ok = true;
      int sv = 0;
      uint32_t phv = 0, par = 0;
      while (ok && it.next(p.items)) {
        for (int j = it.t0; j < it.t1 && ok; ++j) {
          const uint64_t dv = dV0 + (uint64_t)(sv * (kTileBytes >> 4));
          ok = wait(&bar->v_full[sv], phv);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (ok) ok = wait(&bar->p_full[x][h], par);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < kSub / 16; ++c)
              mma_ts_1(dO, dP + h * 32 + c * 8, desc_advance(dv, h * (kSub * kD * 2) + c * 2048), kIdescPV, c > 0 || h > 0 || j > it.t0 ? 1u : 0u);
            if (x == 0) {
              const uint64_t dl = smem_desc_64(sLo + h * kLoBytes);
#pragma unroll
              for (int c = 0; c < kLoKeys / 16; ++c)
                mma_ss_1(dO, desc_advance(dl, c * 32), desc_advance(dv, h * (kSub * kD * 2) + c * 2048), kIdescPV, 1u);
            }
            commit_1(&bar->pv_done[x][h]);
          }
          if (!ok) break;
          commit_1(&bar->v_empty[sv]);
          par ^= 1;
          if (++sv == kVS) { sv = 0; phv ^= 1; }
        }
      }
      commit_1(&bar->drain);
      const unsigned long long t0 = globaltimer();
      while (!mbar_try(&bar->drain, 0) && globaltimer() - t0 < kWaitLimitNs) {}
    }
    __syncwarp();
  } else {
    // ================= softmax + epilogue: one thread per query row, map and parity of the step =================
    const int set = (warp - kFirstSoftmaxWarp) >> 2, x = set >> 1, hb = set & 1;   // map, and parity of the steps, of this warp
    const int q4 = warp & 3;                        // tensor-memory quadrant a warp may touch: warp % 4
    const int r = 32 * q4 + lane;                   // row of the tile
    const uint32_t lane_base = (uint32_t)(q4 << 5) << 16;
    const uint32_t tS = tmem + lane_base + kColS + x * kSub, tP = tmem + lane_base + kColP + 32 * set;
    const uint32_t tO = tmem + lane_base + kColO;
    const float sl2 = p.scale_log2;
    const uint64_t sl2x2 = pack2(sl2, sl2);
    const float lam = lambda_of(p.tail);
    unsigned char* lo = x == 0 ? smem + kSmemTiles + hb * kLoBytes + r * (kLoKeys * 2) : nullptr;
    bool ok = true;
    uint32_t n = 0;                   // steps of this set so far: parity of its barriers
    uint32_t items = 0;               // items so far
    int vt = 0;                       // V tiles walked so far

    while (ok && it.next(p.items)) {
      const int nsteps = 2 * (it.t1 - it.t0);
      const Reach reach = reach_of(p.items.kv_len, p.items.q_pos, it.ib, p.items.Nq, p.items.Nk, p.items.causal != 0);
      const int i = it.iqt * kTile + r;                                                  // this thread's query
      const int limit = reach.limit(i), limit0 = reach.limit(it.iqt * kTile + 32 * q4);    // its keys; the fewest of the warp
      // steps of the tile with the last key: rows of V behind it may hold anything, and 0 times that need not be 0
      const int zero_step = reach.len < min(it.n * kTile, p.items.Nk) && it.t1 == it.n ? nsteps - 2 + hb : -1;
      float neg = 0.f, l = 0.f;       // minus the reference (log2); the sum
      for (int u = hb; u < nsteps; u += 2, ++n) {
        const int key0 = (it.t0 + (u >> 1)) * kTile + hb * kSub;
        ok = warp_wait<kSuspendNs>(&bar->s_full[x][hb], n & 1, &bar->abort_flag, p.status);
        if (!ok) break;
        tc_fence_after();
        if (u == zero_step) {
          const int s = (vt + (u >> 1)) % kVS;
          ok = warp_wait<kSuspendNs>(&bar->v_full[s], ((vt + (u >> 1)) / kVS) & 1, &bar->abort_flag, p.status);
          if (!ok) break;
          // this step's half of the tile, both maps' threads the same zeros: each map's products wait for its own
          if (key0 + (r >> 1) >= reach.len) {
            unsigned char* dst = smem + (kQB + kKS + s) * kTileBytes + (r & 1) * kHalfBytes + (hb * kSub + (r >> 1)) * (kD * 2);
#pragma unroll
            for (int c = 0; c < 8; ++c) *reinterpret_cast<uint4*>(dst + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        uint32_t va[32], vb[32];
        tmem_ld32(tS, va);
        tmem_ld32(tS + 32, vb);
        tmem_wait_ld(va);
        tmem_wait_ld(vb);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->s_read[x][hb]);
        if (key0 + kSub > limit0) {                   // keys that some row of the warp does not see
          const int nv = limit - key0;
#pragma unroll
          for (int c = 0; c < 32; ++c) {
            if (c >= nv) va[c] = kNegInf;
            if (c + 32 >= nv) vb[c] = kNegInf;
          }
        }
        if (u == 0) {
          float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
          max32(va, mx4);
          max32(vb, mx4);
          neg = ref_negative(max_of(mx4), sl2);       // (0 where none of the keys weighs anything)
          bar->ref[x][r] = neg;
          __syncwarp();
          if (lane == 0) mbar_arrive(&bar->ref_set[x]);
        } else if (u == 1) {
          ok = warp_wait<kSuspendNs>(&bar->ref_set[x], items & 1, &bar->abort_flag, p.status);
          if (!ok) break;
          neg = bar->ref[x][r];
        }
        // exponentials against the reference, 64 scores to 32 columns of bf16 pairs
        const uint64_t neg2 = pack2(neg, neg);
        uint64_t lsum[4] = {0ull, 0ull, 0ull, 0ull};
        uint32_t pa[16], pb[16];
        weights32(vb, sl2x2, neg2, lsum, pb, nullptr, 0);
        if (n > 0) {                                  // P(u - 2) has been read
          if (!__all_sync(0xffffffffu, mbar_test(&bar->pv_done[x][hb], (n + 1) & 1))) {
            ok = warp_wait<kSuspendNs>(&bar->pv_done[x][hb], (n + 1) & 1, &bar->abort_flag, p.status);
            if (!ok) break;
          }
          tc_fence_after();
        }
        tmem_st16(tP + 16, pb);
        weights32(va, sl2x2, neg2, lsum, pa, lo, (r >> 1) & 3);
        tmem_st16(tP, pa);
        float a0, a1, b0, b1;
        unpack2(add2(lsum[0], lsum[1]), a0, a1);
        unpack2(add2(lsum[2], lsum[3]), b0, b1);
        l += (a0 + a1) + (b0 + b1);
        // publish P
        tmem_wait_st();
        if (x == 0) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->p_full[x][hb]);
      }
      if (!ok) break;
      vt += nsteps >> 1;
      bar->sum[x][hb][r] = l;
      if (hb == 1) {                   // the item's last product: the sets of parity 1 wait for it, the others for them
        ok = warp_wait<kSuspendNs>(&bar->pv_done[x][1], (n + 1) & 1, &bar->abort_flag, p.status);
        if (!ok) break;
      }
      tc_fence_after();
      tc_fence_before();
      mbar_arrive(&bar->sums_in);
      ok = warp_wait<kSuspendNs>(&bar->sums_in, items & 1, &bar->abort_flag, p.status);
      if (!ok) break;
      tc_fence_after();
      auto fine = [](float s) { return s >= 1.f / kFine && s <= kFine; };
      if (!it.whole()) {
        // ---- a part: reference, sum and product of this map as they are, half the channels to each set.  Reference -inf: no
        // keys of this row; none at all: the row has to be done again.
        float* dst = p.partial + partial_at((size_t)partial_slot(blockIdx.x, it.t0) * kTile + r);
        if (hb == 0) {
          const float s = bar->sum[x][0][r] + bar->sum[x][1][r];
          const float ref = limit <= it.t0 * kTile ? -INFINITY : fine(s) ? -bar->ref[x][r] : __uint_as_float(0x7fc00000u);
          *reinterpret_cast<float2*>(dst + 2 * x) = make_float2(ref, s);
        }
        dst += (1 + (kV * x + kD * hb) / 4) * kPiece;
#pragma unroll
        for (int c = 0; c < kD / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(tO + kV * x + kD * hb + 32 * c, v);
          tmem_wait_ld(v);
#pragma unroll
          for (int y = 0; y < 8; ++y)
            *reinterpret_cast<uint4*>(dst + (8 * c + y) * kPiece) = make_uint4(v[4 * y], v[4 * y + 1], v[4 * y + 2], v[4 * y + 3]);
        }
        tc_fence_before();
        mbar_arrive(&bar->read_out);
        ok = warp_wait<kSuspendNs>(&bar->read_out, items & 1, &bar->abort_flag, p.status);
        ++items;
        continue;
      }
      // ---- the whole: x = O_0 / l_0 - lambda O_1 / l_1 on this thread's 32 channels
      const float s0 = bar->sum[0][0][r] + bar->sum[0][1][r], s1 = bar->sum[1][0][r] + bar->sum[1][1][r];
      const float f0 = 1.f / s0, f1 = -lam / s1;
      float out[32], ss = 0.f;
      {
        uint32_t v[32];
        tmem_ld32(tO + 32 * set, v);
        tmem_wait_ld(v);
#pragma unroll
        for (int y = 0; y < 32; ++y) out[y] = __uint_as_float(v[y]) * f0;
        tmem_ld32(tO + kV + 32 * set, v);
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
      if (i < p.items.Nq) {
        const float square = (bar->square[0][r] + bar->square[1][r]) + (bar->square[2][r] + bar->square[3][r]);
        if (set == 0) {
          // (with a norm also where the mean square is not safely within fp32)
          const bool good = p.tail.norm_w ? square_fine(square * (1.f / kV) + p.tail.norm_eps) : square < INFINITY;
          const bool again = limit > 0 && !(fine(s0) && fine(s1) && good);
          p.mark[((size_t)it.ib * p.pairs + it.ipair) * p.items.Nq + i] = again ? 1 : 0;
          if (again) bar->redo = 1;
        }
        const float rn = p.tail.norm_w ? (1.f - p.tail.lambda_init) * rsqrtf(square * (1.f / kV) + p.tail.norm_eps) : 1.f;
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
          for (int y = 0; y < 4; ++y)           // (no key: 0 whatever the norm makes of zeros)
            pk[y] = limit > 0 ? pack_bf16(out[8 * c + 2 * y] * rn * w[2 * y], out[8 * c + 2 * y + 1] * rn * w[2 * y + 1]) : 0u;
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
  if (threadIdx.x == 0) {
    p.starts[blockIdx.x].redo = bar->redo;
    if (bar->abort_flag) p.starts[blockIdx.x].left = 1;   // a wait has run out: its partials are not to be merged
  }
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// Blocks of a call, one per SM at most: one for every item, or for every kTilesMin tiles of the longest that the items can be
constexpr int kTilesMin = 4;
// An item costs as much as four tiles beside its own (first scores, epilogue).  Measured, in units of 1 / 2 / 3 / 4 / 6 tiles: two
// causal prompts of 4096 tokens, 8 pairs, on one board 173 / 137 / 127 / 127 / 132 us; 73 x 73 tokens 744 to 784 either way.
constexpr int kLead = 4, kWhole = 2;
int diff_blocks(int B, int pairs, int Nq, int Nk) {
  const int64_t items = (int64_t)B * pairs * ceil_div(Nq, kTile), tiles = items * ceil_div(Nk, kTile);
  const int64_t want = items > tiles / kTilesMin ? items : tiles / kTilesMin;
  const int sms = device_sm_count();
  return (int)(want < sms ? want : sms);
}

}  // namespace

DiffPlan diff_tc_plan(int B, int pairs, int Nq, int Nk) {
  return diff_plan(diff_blocks(B, pairs, Nq, Nk), kTile, (int64_t)B * pairs * Nq);
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
  const DiffPlan plan = diff_tc_plan(a.B, a.pairs, a.Nq, a.Nk);
  const DiffParams p = diff_params(a, plan, Items{a.B, ceil_div(a.Nq, kTile), a.pairs, a.Nq, a.Nk, kTile, a.causal ? 1 : 0, kLead, kWhole, a.kv_len, a.q_pos},
                                   kTile, ws, status);
  e = launch_programmatic(attn_diff_kernel, dim3((unsigned)plan.blocks), kThreads, kSmemBytes, st, maps[0], maps[1], maps[2], p);
  if (e != cudaSuccess) return e;
  return launch_diff_merge(p, plan.blocks, a.Nq < kTile ? a.Nq : kTile, st);
}

}  // namespace jv

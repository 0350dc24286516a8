// Differential attention for few queries: single tokens (or a few) against a long cache, bf16, 64 channels a map.
//
// All queries of the pairs that share a pair of keys, at most 16 rows, are the M dimension of mma.sync m16n8k16: the work is reading K and
// V once (512 bytes a key and pair), far below what needs tcgen05.  Keys come in boxes of 64 through a TMA ring of four (128 KB in
// flight per SM) to sixteen warps: eight per map, four of them to the even boxes, four to the odd ones, 16 keys each, with fragments by
// ldmatrix from the swizzled rows.  Every warp keeps its own running reference, sum and product (16 x 128) in registers; the reference
// moves when a score outgrows it by 2^8, which one vote per box decides.  At the end of an item the warps' results are summed
// through shared memory, and written, or left as a partial where the item goes on in another block (see attn_diff.cuh: blocks take
// equal shares of all items' keys, so sequences of any lengths keep all SMs busy to the end).
//
// What bounds it: HBM, and what a call costs beside it.  32 sequences of up to 16384 keys, two pairs of keys, four pairs of queries to
// each: 77 to 86 us by the board, with the launch that merges, for 336 MB (51 us at the rate of a copy); 67.5 us where the warps only
// take boxes in.  With eight warps for both maps, 168 registers a thread, 75.3 us where these sixteen took 74.3 (second terms in
// map 0 alone).  Second terms of both maps' probabilities in place of map 0's alone, on one board: 81.4 -> 82.9 us, o at 1.67e-3 of the
// exact result instead of 2.14e-3.
#include "attn_diff.cuh"
#include "tc_common.cuh"

namespace jv {
namespace {

using namespace tc;
using namespace diff;

constexpr int kRows = 16;
static_assert(kRows % kPartialRows == 0, "slots of whole groups of rows");
constexpr int kBox = 64;                      // keys of a box
constexpr int kStages = 4;
constexpr int kBoxBytes = kBox * kD * 2;      // one head's: 8 KB
constexpr int kStageBytes = 4 * kBoxBytes;    // K of both heads, V of both
constexpr int kWorkers = 16;                  // warps that compute
constexpr int kPerMap = kWorkers / 2;
constexpr int kThreads = (kWorkers + 1) * 32;
constexpr int kQStride = kV * 2 + 16;         // bytes between rows of queries: ldmatrix's eight rows in different banks
constexpr int kSumStride = kV + 4;            // floats between rows of the warps' results: rows g and g + 1 in different banks

struct __align__(16) Shared {
  uint64_t full[kStages], empty[kStages];
  long long scan[34];
  Start start;
  float m[2][kPerMap][kRows], l[2][kPerMap][kRows];
  volatile uint32_t abort_flag;
  uint32_t leave;                             // what the workers go by: one of them reads the flag for all
  __align__(16) unsigned char q[kRows][kQStride];
};
constexpr size_t kSumBytes = (size_t)kPerMap * kRows * kSumStride * 4;
constexpr size_t kSmemBytes = kStages * (size_t)kStageBytes + kSumBytes + sizeof(Shared) + 1024;
static_assert(kSmemBytes <= 227 * 1024, "shared memory of one block");

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// what a rounding to bf16 pairs has taken off
__device__ __forceinline__ uint32_t rest_bf16(float a, float b, uint32_t h) {
  return pack_bf16(a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xffff0000u));
}
__device__ __forceinline__ void workers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kWorkers * 32) : "memory"); }

__global__ void __launch_bounds__(kThreads, 1)
diff_rows_kernel(const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV, const DiffParams p) {
  extern __shared__ unsigned char smem_raw[];
  if (threadIdx.x == kWorkers * 32) {
    prefetch_map(&mapK);
    prefetch_map(&mapV);
  }
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  float* sums = reinterpret_cast<float*>(smem + kStages * kStageBytes);           // [warp of a map][row][channel], one map at a time
  Shared* sh = reinterpret_cast<Shared*>(smem + kStages * kStageBytes + kSumBytes);
  const uint32_t ring = smem_u32(smem);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh->full[s], 1);
      mbar_init(&sh->empty[s], 8);            // the eight warps that read it
    }
    sh->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  griddep_wait();                 // what is read and written from here on may belong to the launch ahead
  griddep_launch_dependents();
  if (threadIdx.x == 0 && *reinterpret_cast<volatile int*>(p.status) != 0) sh->abort_flag = 1;
  find_start(p.items, blockIdx.x, gridDim.x, sh->scan, &sh->start);    // (ends with a barrier)
  if (threadIdx.x == 0) {
    Start s = sh->start;
    s.left = sh->abort_flag;
    p.starts[blockIdx.x] = s;
  }
  if (sh->abort_flag) return;
  Walk it;
  it.begin(sh->start);
  const int rows = p.share * p.items.Nq;

  // boxes of the present item: [first, last) of 64 keys; none where no query sees a key
  auto boxes = [&](const Reach& reach, int& first, int& last) {
    first = 2 * it.t0;
    last = min(2 * it.t1, (max(reach.limit(p.items.Nq - 1), 0) + kBox - 1) / kBox);
  };
  auto reach_b = [&]() { return reach_of(p.items.kv_len, p.items.q_pos, it.ib, p.items.Nq, p.items.Nk, p.items.causal != 0); };

  if (warp == kWorkers) {
    // ================= TMA producer (one lane) =================
    if (elect_one()) {
      bool ok = true;
      uint32_t n = 0;              // boxes so far
      while (ok && it.next(p.items)) {
        int first, last;
        boxes(reach_b(), first, last);
        const int h = 2 * it.ipair;
        for (int x = first; x < last; ++x, ++n) {
          const uint32_t s = n % kStages, dst = ring + s * kStageBytes;
          ok = mbar_wait(&sh->empty[s], ((n / kStages) & 1) ^ 1, &sh->abort_flag, p.status);
          if (!ok) break;
          mbar_expect_tx(&sh->full[s], kStageBytes);
          tma_load_4d(dst, &mapK, &sh->full[s], 0, x * kBox, h, it.ib);
          tma_load_4d(dst + kBoxBytes, &mapK, &sh->full[s], 0, x * kBox, h + 1, it.ib);
          tma_load_4d(dst + 2 * kBoxBytes, &mapV, &sh->full[s], 0, x * kBox, h, it.ib);
          tma_load_4d(dst + 3 * kBoxBytes, &mapV, &sh->full[s], 0, x * kBox, h + 1, it.ib);
        }
      }
      // Nobody may leave with copies in flight: the last ones are waited for (bounded), whether their readers are done or gave up
      const unsigned long long t0 = globaltimer();
      for (uint32_t g = n > kStages ? n - kStages : 0; g < n; ++g)
        while (!mbar_try(&sh->full[g % kStages], (g / kStages) & 1) && globaltimer() - t0 < kWaitLimitNs) {}
    }
    __syncwarp();
    return;
  }

  // ================= sixteen warps =================
  const int g = lane >> 2, t = lane & 3;
  const int part = warp & 3, m = (warp >> 2) & 1, half = warp >> 3;   // keys 16 part .. of the boxes n with n % 2 == half; map
  const int mine = 4 * half + part;         // of the warps of the map
  const float lam = lambda_of(p.tail);
  const float sl2 = p.scale_log2;
  // ldmatrix addresses within a box: row (key) and 16-byte chunk of a lane, chunks swizzled by the row
  const int krow = 16 * part + (lane & 7) + ((lane & 16) >> 1), kchunk = (lane >> 3) & 1;    // x4: keys 0-7 | chunks 0, 1; keys 8-15 | chunks 0, 1
  const int vrow = 16 * part + (lane & 15), vchunk = lane >> 4;                              // x4: keys 0-7, 8-15 of chunk 0; of chunk 1
  const uint32_t qaddr = smem_u32(&sh->q[lane & 15][16 * (lane >> 4)]) + m * (kD * 2);   // x4: rows 0-7, 8-15 of chunk 0; of chunk 1
  uint32_t n = 0;
  bool ok = true;
  while (it.next(p.items)) {
    __syncwarp();
    const Reach reach = reach_b();
    int first, last;
    boxes(reach, first, last);
    int lim[2];                               // keys of rows g and g + 8
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int pair, i;
      p.row(0, it.ipair, g + 8 * h, pair, i);
      lim[h] = g + 8 * h < rows ? reach.limit(i) : 0;
    }
    if (threadIdx.x < kRows * 16) {           // queries of both maps, zeros past the rows: 16 bytes a thread
      const int r = threadIdx.x >> 4, c = threadIdx.x & 15;
      int pair, i;
      p.row(0, it.ipair, r, pair, i);
      const __nv_bfloat16* q = (const __nv_bfloat16*)p.args.q + it.ib * p.args.qs.batch + (int64_t)i * p.args.qs.tok + (2 * pair + (c >> 3)) * p.args.qs.head + 8 * (c & 7);
      *reinterpret_cast<uint4*>(&sh->q[r][16 * c]) = r < rows ? *reinterpret_cast<const uint4*>(q) : make_uint4(0u, 0u, 0u, 0u);
    }
    workers_sync();
    const int least = p.items.causal ? reach.limit(0) : reach.len;      // keys that every row sees
    float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};           // rows g, g + 8
    float acc[16][4];
#pragma unroll
    for (int j = 0; j < 16; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[j][c] = 0.f;

    for (int x = first; x < last; ++x, ++n) {
      if ((int)(n & 1) != half) continue;
      const uint32_t s = n % kStages, base = ring + s * kStageBytes;
      ok = warp_wait(&sh->full[s], (n / kStages) & 1, &sh->abort_flag, p.status);
      if (!ok) break;
      float sc[2][4];
#pragma unroll
      for (int c = 0; c < 4; ++c) sc[0][c] = sc[1][c] = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t qa[4], b[4];                 // b: keys 0-7: channels 16 k .., + 8; keys 8-15: the same
        ldsm4(qa, qaddr + 32 * k);
        ldsm4(b, base + m * kBoxBytes + krow * 128 + (((2 * k + kchunk) ^ (krow & 7)) << 4));
        mma16816(sc[0], qa, b[0], b[1]);
        mma16816(sc[1], qa, b[2], b[3]);
      }
      const int key0 = x * kBox + 16 * part;
      const bool edge = key0 + 16 > least;    // some row does not see some key
      bool moves = false;
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float v = sc[j][c] * sl2;
          if (edge && key0 + 8 * j + 2 * t + (c & 1) >= lim[c >> 1]) v = -INFINITY;
          sc[j][c] = v;
          moves |= !(v <= ref[c >> 1] + 8.f);
        }
      if (__any_sync(0xffffffffu, moves)) {   // a score outgrows its row's reference, or is no number: the first box always
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float mx = max3(max3(sc[0][2 * h], sc[0][2 * h + 1], sc[1][2 * h]), sc[1][2 * h + 1], ref[h]);
          mx = max3(mx, __shfl_xor_sync(0xffffffffu, mx, 1), mx);
          mx = max3(mx, __shfl_xor_sync(0xffffffffu, mx, 2), mx);
          const float f = mx == -INFINITY ? 1.f : ex2(ref[h] - mx) + (mx - mx);    // +inf, no number: no number
          ref[h] = mx;
          l[h] *= f;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            acc[j][2 * h] *= f;
            acc[j][2 * h + 1] *= f;
          }
        }
      }
      // A fragments of the probabilities, as two bf16 terms: the difference of the maps is smaller than either, and their roundings
      // left o at 2.6e-3 of the exact result.
      uint32_t pa[4], pb[4];
      const float r0 = ref[0] == -INFINITY ? 0.f : ref[0], r1 = ref[1] == -INFINITY ? 0.f : ref[1];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float p0 = ex2(sc[j][0] - r0), p1 = ex2(sc[j][1] - r0), p2 = ex2(sc[j][2] - r1), p3 = ex2(sc[j][3] - r1);
        l[0] += p0 + p1;
        l[1] += p2 + p3;
        pa[2 * j] = pack_bf16(p0, p1);
        pa[2 * j + 1] = pack_bf16(p2, p3);
        pb[2 * j] = rest_bf16(p0, p1, pa[2 * j]);
        pb[2 * j + 1] = rest_bf16(p2, p3, pa[2 * j + 1]);
      }
      const bool behind = key0 + 16 > reach.len;   // rows of V that may hold anything: they count as zeros
      const int k0 = key0 + 2 * t;
      const uint32_t keep0 = (k0 < reach.len ? 0xffffu : 0u) | (k0 + 1 < reach.len ? 0xffff0000u : 0u);
      const uint32_t keep1 = (k0 + 8 < reach.len ? 0xffffu : 0u) | (k0 + 9 < reach.len ? 0xffff0000u : 0u);
#pragma unroll
      for (int j = 0; j < 16; j += 2) {       // channels 8 j .. 8 j + 15
        uint32_t b[4];                        // channels 8 j: keys 0-7, 8-15; channels 8 j + 8: the same
        ldsm4_t(b, base + (2 + (j >> 3)) * kBoxBytes + vrow * 128 + ((((j & 7) + vchunk) ^ (vrow & 7)) << 4));
        if (behind) {
          b[0] &= keep0; b[1] &= keep1; b[2] &= keep0; b[3] &= keep1;
        }
        mma16816(acc[j], pa, b[0], b[1]);
        mma16816(acc[j + 1], pa, b[2], b[3]);
        mma16816(acc[j], pb, b[0], b[1]);
        mma16816(acc[j + 1], pb, b[2], b[3]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->empty[s]);
    }
    // ---- the warps' results.  (A wait that ran out leaves all of them, by the flag, before anybody waits for the others.)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      if (t == 0) {
        sh->m[m][mine][g + 8 * h] = ref[h];
        sh->l[m][mine][g + 8 * h] = l[h];
      }
    }
    workers_sync();
    float f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kPerMap; ++w) top = max3(top, sh->m[m][w][g + 8 * h], top);
      f[h] = ref[h] == -INFINITY ? 0.f : ex2(ref[h] - top);
    }
    // from here on a warp has row `warp`, four channels a lane
    const int tr = warp, ch = 4 * lane;
    float M[2], total[2], res[2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      M[x] = -INFINITY;
      total[x] = 0.f;
#pragma unroll
      for (int w = 0; w < kPerMap; ++w) M[x] = max3(M[x], sh->m[x][w][tr], M[x]);
#pragma unroll
      for (int w = 0; w < kPerMap; ++w) total[x] += sh->m[x][w][tr] == -INFINITY ? 0.f : sh->l[x][w][tr] * ex2(sh->m[x][w][tr] - M[x]);
      if (m == x)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            *reinterpret_cast<float2*>(sums + (mine * kRows + g + 8 * h) * kSumStride + 8 * j + 2 * t) = make_float2(acc[j][2 * h] * f[h], acc[j][2 * h + 1] * f[h]);
      workers_sync();
#pragma unroll
      for (int y = 0; y < 4; ++y) res[x][y] = 0.f;
#pragma unroll
      for (int w = 0; w < kPerMap; ++w) {
        const float4 v = *reinterpret_cast<const float4*>(sums + (w * kRows + tr) * kSumStride + ch);
        res[x][0] += v.x; res[x][1] += v.y; res[x][2] += v.z; res[x][3] += v.w;
      }
      if (threadIdx.x == 0) sh->leave = sh->abort_flag;
      workers_sync();                         // (the other map's turn, or the next item's)
    }
    if (sh->leave) {                          // a wait has run out: no result of this item is complete, and none to be merged
      if (threadIdx.x == 0) p.starts[blockIdx.x].left = 1;
      break;
    }
    if (tr >= rows) continue;
    if (!it.whole()) {
      float* dst = p.partial + partial_at((size_t)partial_slot(blockIdx.x, it.t0) * kRows + tr);
      if (lane == 0) *reinterpret_cast<float4*>(dst) = make_float4(M[0], total[0], M[1], total[1]);
#pragma unroll
      for (int x = 0; x < 2; ++x) *reinterpret_cast<float4*>(dst + (1 + (kV * x + ch) / 4) * kPiece) = make_float4(res[x][0], res[x][1], res[x][2], res[x][3]);
      continue;
    }
    int pair, i;
    p.row(0, it.ipair, tr, pair, i);
    const bool any = reach.limit(i) > 0;      // (a row that sees keys, none of weight: 0 / 0)
    const float f0 = 1.f / total[0], f1 = -lam / total[1];
    float xv[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) xv[y] = any ? res[0][y] * f0 + res[1][y] * f1 : 0.f;
    if (p.tail.norm_w) {
      const float rn = (1.f - p.tail.lambda_init) * inverse_rms(xv, 1.f / kV, p.tail.norm_eps);
      const float4 w = __ldg(reinterpret_cast<const float4*>(p.tail.norm_w + ch));
      xv[0] *= rn * w.x; xv[1] *= rn * w.y; xv[2] *= rn * w.z; xv[3] *= rn * w.w;
    }
    if (!any) xv[0] = xv[1] = xv[2] = xv[3] = 0.f;   // (whatever the norm makes of zeros)
    __nv_bfloat16* dst = p.o + (((size_t)it.ib * 2 * p.pairs + 2 * pair + (ch >> 6)) * p.items.Nq + i) * kD + (ch & 63);
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16(xv[0], xv[1]), pack_bf16(xv[2], xv[3]));
  }
}

// Blocks of a call: one per SM, or per tile of the longest that the items can be
int rows_blocks(int B, int kv_pairs, int Nk) {
  const int64_t tiles = (int64_t)B * kv_pairs * ceil_div(Nk, kTile);
  const int sms = device_sm_count();
  return (int)(tiles < sms ? tiles : sms);
}

}  // namespace

bool diff_rows_supported(const DiffArgs& a) {
  return a.dtype == JV_BF16 && a.D == kD && (int64_t)(a.pairs / a.kv_pairs) * a.Nq <= kRows && encode_fn() != nullptr;
}

DiffPlan diff_rows_plan(int B, int kv_pairs, int Nk) { return diff_plan(rows_blocks(B, kv_pairs, Nk), kRows, 0); }

cudaError_t launch_diff_rows(const DiffArgs& a, void* ws, int* status, cudaStream_t st) {
  EncodeFn enc = encode_fn();
  if (!enc) return cudaErrorNotSupported;
  CUtensorMap maps[2];
  const void* ptrs[2] = {a.k, a.v};
  for (int i = 0; i < 2; ++i) {
    // (channels, tokens, heads, batch elements) with the caller's strides; a box is 64 tokens of one head
    const cuuint64_t dims[4] = {(cuuint64_t)kD, (cuuint64_t)a.Nk, (cuuint64_t)(2 * a.kv_pairs), (cuuint64_t)a.B};
    const cuuint64_t strides[3] = {(cuuint64_t)a.ks.tok * 2, (cuuint64_t)a.ks.head * 2, (cuuint64_t)a.ks.batch * 2};
    const cuuint32_t box[4] = {(cuuint32_t)kD, (cuuint32_t)kBox, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    const CUresult r = enc(&maps[i], CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptrs[i]), dims, strides, box, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return cudaErrorInvalidValue;
  }
  static OncePerDevice smem_opt_in;
  cudaError_t e = smem_opt_in.run([] {
    return cudaFuncSetAttribute(diff_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemBytes);
  });
  if (e != cudaSuccess) return e;
  const DiffPlan plan = diff_rows_plan(a.B, a.kv_pairs, a.Nk);
  const DiffParams p = diff_params(a, plan, Items{a.B, 1, a.kv_pairs, a.Nq, a.Nk, a.Nq, a.causal ? 1 : 0, 1, 1, a.kv_len, a.q_pos}, kRows, ws, status);
  e = launch_programmatic(diff_rows_kernel, dim3((unsigned)plan.blocks), kThreads, kSmemBytes, st, maps[0], maps[1], p);
  if (e != cudaSuccess) return e;
  return launch_diff_merge(p, plan.blocks, (a.pairs / a.kv_pairs) * a.Nq, st);
}

}  // namespace jv

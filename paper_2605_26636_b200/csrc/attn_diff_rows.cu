// Differential attention for few queries: single tokens (or a few) against a long cache, bf16, 64 channels a map.
//
// All queries of the pairs that share a pair of keys, at most 16 rows, are the M dimension of mma.sync m16n8k16: the work is reading K and
// V once (512 bytes a key and pair), far below what needs tcgen05.  Keys come in boxes of 64 through a TMA ring of four (128 KB in
// flight per SM) to eight warps: four take the even boxes, four the odd ones, 16 keys each, with fragments by ldmatrix from the
// swizzled rows.  Every warp keeps its own running reference, sum and products (both maps, 16 x 128) in registers; the reference
// moves when a score outgrows it by 2^8, which one vote per box decides.  At the end of an item the eight warps' results are summed
// through shared memory, and written, or left as a partial where the item goes on in another block (see attn_diff.cuh: blocks take
// equal shares of all items' keys, so sequences of any lengths keep all SMs busy to the end).
//
// What bounds it: HBM.
#include "attn_diff.cuh"
#include "tc_common.cuh"

namespace jv {
namespace {

using namespace tc;
using namespace diff;

constexpr int kRows = 16;
constexpr int kBox = 64;                      // keys of a box
constexpr int kStages = 4;
constexpr int kBoxBytes = kBox * kD * 2;      // one head's: 8 KB
constexpr int kStageBytes = 4 * kBoxBytes;    // K of both heads, V of both
constexpr int kWorkers = 8;                   // warps that compute
constexpr int kThreads = (kWorkers + 1) * 32;
constexpr int kQStride = kV * 2 + 16;         // bytes between rows of queries: ldmatrix's eight rows in different banks
constexpr int kSumStride = kV + 4;            // floats between rows of the warps' results: rows g and g + 1 in different banks

struct __align__(16) Shared {
  uint64_t full[kStages], empty[kStages];
  long long scan[34];
  Start start;
  float m[kWorkers][2][kRows], l[kWorkers][2][kRows];
  volatile uint32_t abort_flag;
  uint32_t leave;                             // what the workers go by: one of them reads the flag for all
  __align__(16) unsigned char q[kRows][kQStride];
};
constexpr size_t kSumBytes = (size_t)kWorkers * kRows * kSumStride * 4;
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
  float* sums = reinterpret_cast<float*>(smem + kStages * kStageBytes);           // [warp][row][channel], one map at a time
  Shared* sh = reinterpret_cast<Shared*>(smem + kStages * kStageBytes + kSumBytes);
  const uint32_t ring = smem_u32(smem);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sh->full[s], 1);
      mbar_init(&sh->empty[s], 4);            // the four warps that read it
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

  // ================= eight warps =================
  const int tr = threadIdx.x >> 4, tc = threadIdx.x & 15;     // where a thread has a row's eight channels: row tr, channels 8 tc ..
  const int g = lane >> 2, t = lane & 3, half = warp >> 2, part = warp & 3;   // boxes n with n % 2 == half; keys 16 part .. of them
  const float lam = lambda_of(p.tail);
  const float sl2 = p.scale_log2;
  // ldmatrix addresses within a box: row (key) and 16-byte chunk of a lane, chunks swizzled by the row
  const int krow = 16 * part + (lane & 7) + ((lane & 16) >> 1), kchunk = (lane >> 3) & 1;    // x4: keys 0-7 | chunks 0, 1; keys 8-15 | chunks 0, 1
  const int vrow = 16 * part + (lane & 15), vchunk = lane >> 4;                              // x4: keys 0-7, 8-15 of chunk 0; of chunk 1
  const uint32_t qaddr = smem_u32(&sh->q[lane & 15][16 * (lane >> 4)]);   // x4: rows 0-7, 8-15 of chunk 0; of chunk 1
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
    {                                         // queries of both maps, zeros past the rows: 16 bytes a thread
      int pair, i;
      p.row(0, it.ipair, tr, pair, i);
      const __nv_bfloat16* q = (const __nv_bfloat16*)p.args.q + it.ib * p.args.qs.batch + (int64_t)i * p.args.qs.tok + (2 * pair + (tc >> 3)) * p.args.qs.head + 8 * (tc & 7);
      *reinterpret_cast<uint4*>(&sh->q[tr][16 * tc]) = tr < rows ? *reinterpret_cast<const uint4*>(q) : make_uint4(0u, 0u, 0u, 0u);
      workers_sync();
    }
    const int least = p.items.causal ? reach.limit(0) : reach.len;      // keys that every row sees
    float ref[2][2] = {{-INFINITY, -INFINITY}, {-INFINITY, -INFINITY}}, l[2][2] = {{0.f, 0.f}, {0.f, 0.f}};   // [map][row g, g + 8]
    float acc[2][16][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int j = 0; j < 16; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[m][j][c] = 0.f;

    for (int x = first; x < last; ++x, ++n) {
      if ((int)(n & 1) != half) continue;
      const uint32_t s = n % kStages, base = ring + s * kStageBytes;
      ok = warp_wait(&sh->full[s], (n / kStages) & 1, &sh->abort_flag, p.status);
      if (!ok) break;
      float sc[2][2][4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
#pragma unroll
        for (int c = 0; c < 4; ++c) sc[m][0][c] = sc[m][1][c] = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t qa[4], b[4];               // b: keys 0-7: channels 16 k .., + 8; keys 8-15: the same
          ldsm4(qa, qaddr + m * (kD * 2) + 32 * k);
          ldsm4(b, base + m * kBoxBytes + krow * 128 + (((2 * k + kchunk) ^ (krow & 7)) << 4));
          mma16816(sc[m][0], qa, b[0], b[1]);
          mma16816(sc[m][1], qa, b[2], b[3]);
        }
      }
      const int key0 = x * kBox + 16 * part;
      const bool edge = key0 + 16 > least;    // some row does not see some key
      bool moves = false;
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            float v = sc[m][j][c] * sl2;
            if (edge && key0 + 8 * j + 2 * t + (c & 1) >= lim[c >> 1]) v = -INFINITY;
            sc[m][j][c] = v;
            moves |= !(v <= ref[m][c >> 1] + 8.f);
          }
      if (__any_sync(0xffffffffu, moves)) {   // a score outgrows its row's reference, or is no number: the first box always
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float mx = max3(max3(sc[m][0][2 * h], sc[m][0][2 * h + 1], sc[m][1][2 * h]), sc[m][1][2 * h + 1], ref[m][h]);
            mx = max3(mx, __shfl_xor_sync(0xffffffffu, mx, 1), mx);
            mx = max3(mx, __shfl_xor_sync(0xffffffffu, mx, 2), mx);
            const float f = mx == -INFINITY ? 1.f : ex2(ref[m][h] - mx) + (mx - mx);    // +inf, no number: no number
            ref[m][h] = mx;
            l[m][h] *= f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              acc[m][j][2 * h] *= f;
              acc[m][j][2 * h + 1] *= f;
            }
          }
      }
      // A fragments of the probabilities, those of map 0 (which weighs most) as two bf16 terms: the difference of the maps is smaller
      // than either, and their roundings left o at 2.6e-3 of the exact result (its own rounding: 1.7e-3).  Both maps so: 1.64e-3, 92 us.
      uint32_t pa[2][4], pb[4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        const float r0 = ref[m][0] == -INFINITY ? 0.f : ref[m][0], r1 = ref[m][1] == -INFINITY ? 0.f : ref[m][1];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float p0 = ex2(sc[m][j][0] - r0), p1 = ex2(sc[m][j][1] - r0), p2 = ex2(sc[m][j][2] - r1), p3 = ex2(sc[m][j][3] - r1);
          l[m][0] += p0 + p1;
          l[m][1] += p2 + p3;
          pa[m][2 * j] = pack_bf16(p0, p1);
          pa[m][2 * j + 1] = pack_bf16(p2, p3);
          if (m == 0) {
            pb[2 * j] = rest_bf16(p0, p1, pa[m][2 * j]);
            pb[2 * j + 1] = rest_bf16(p2, p3, pa[m][2 * j + 1]);
          }
        }
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
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          mma16816(acc[m][j], pa[m], b[0], b[1]);
          mma16816(acc[m][j + 1], pa[m], b[2], b[3]);
          if (m == 0) {
            mma16816(acc[m][j], pb, b[0], b[1]);
            mma16816(acc[m][j + 1], pb, b[2], b[3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh->empty[s]);
    }
    // ---- the eight warps' results.  (A wait that ran out leaves all of them, by the flag, before anybody waits for the others.)
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        l[m][h] += __shfl_xor_sync(0xffffffffu, l[m][h], 1);
        l[m][h] += __shfl_xor_sync(0xffffffffu, l[m][h], 2);
        if (t == 0) {
          sh->m[warp][m][g + 8 * h] = ref[m][h];
          sh->l[warp][m][g + 8 * h] = l[m][h];
        }
      }
    workers_sync();
    float M[2], total[2], res[2][8];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      M[m] = -INFINITY;
      total[m] = 0.f;
#pragma unroll
      for (int w = 0; w < kWorkers; ++w) M[m] = max3(M[m], sh->m[w][m][tr], M[m]);
#pragma unroll
      for (int w = 0; w < kWorkers; ++w) total[m] += sh->m[w][m][tr] == -INFINITY ? 0.f : sh->l[w][m][tr] * ex2(sh->m[w][m][tr] - M[m]);
      float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int w = 0; w < kWorkers; ++w)
#pragma unroll
        for (int h = 0; h < 2; ++h) top[h] = max3(top[h], sh->m[w][m][g + 8 * h], top[h]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float f = ref[m][h] == -INFINITY ? 0.f : ex2(ref[m][h] - top[h]);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          *reinterpret_cast<float2*>(sums + (warp * kRows + g + 8 * h) * kSumStride + 8 * j + 2 * t) = make_float2(acc[m][j][2 * h] * f, acc[m][j][2 * h + 1] * f);
      }
      workers_sync();
#pragma unroll
      for (int y = 0; y < 8; ++y) res[m][y] = 0.f;
#pragma unroll
      for (int w = 0; w < kWorkers; ++w)
#pragma unroll
        for (int y = 0; y < 8; y += 4) {
          const float4 v = *reinterpret_cast<const float4*>(sums + (w * kRows + tr) * kSumStride + 8 * tc + y);
          res[m][y] += v.x; res[m][y + 1] += v.y; res[m][y + 2] += v.z; res[m][y + 3] += v.w;
        }
      if (threadIdx.x == 0) sh->leave = sh->abort_flag;
      workers_sync();                         // (the other map's turn, or the next item's)
    }
    if (sh->leave) {                          // a wait has run out: no result of this item is complete, and none to be merged
      if (threadIdx.x == 0) p.starts[blockIdx.x].left = 1;
      break;
    }
    if (!it.whole()) {
      if (tr >= rows) continue;
      float* dst = p.partial + ((size_t)partial_slot(blockIdx.x, it.t0) * kRows + tr) * kPartial;
      if (tc == 0) *reinterpret_cast<float4*>(dst) = make_float4(M[0], total[0], M[1], total[1]);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int y = 0; y < 8; y += 4)
          *reinterpret_cast<float4*>(dst + 4 + kV * m + 8 * tc + y) = make_float4(res[m][y], res[m][y + 1], res[m][y + 2], res[m][y + 3]);
      continue;
    }
    int pair, i;
    p.row(0, it.ipair, tr, pair, i);
    const bool any = reach.limit(i) > 0;      // (a row that sees keys, none of weight: 0 / 0)
    const float f0 = 1.f / total[0], f1 = -lam / total[1];
    float xv[8], ss = 0.f;
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      xv[y] = any ? res[0][y] * f0 + res[1][y] * f1 : 0.f;
      ss = fmaf(xv[y], xv[y], ss);
    }
    if (p.tail.norm_w) {
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);          // the 16 lanes of a row
      const float rn = (1.f - p.tail.lambda_init) * rsqrtf(ss * (1.f / kV) + p.tail.norm_eps);
#pragma unroll
      for (int y = 0; y < 8; ++y) xv[y] *= rn * __ldg(p.tail.norm_w + 8 * tc + y);
    }
    __nv_bfloat16* dst = p.o + (((size_t)it.ib * 2 * p.pairs + 2 * pair + (tc >> 3)) * p.items.Nq + i) * kD + 8 * (tc & 7);
    if (tr < rows) *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16(xv[0], xv[1]), pack_bf16(xv[2], xv[3]), pack_bf16(xv[4], xv[5]), pack_bf16(xv[6], xv[7]));
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

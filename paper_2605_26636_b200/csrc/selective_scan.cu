// The selective scan of a state-space mixer: every channel carries Ns states through its sequence.
//   d_t = softplus(dt_t + dt_bias),  h_t = exp(d_t A) h_(t-1) + d_t B_t u_t,  y_t = (C_t . h_t + D u_t) z_t / (1 + exp(-z_t))
//
// Four or eight lanes share a channel, each with a share of its states in registers; a block has 64 or 32 channels in eight warps.
// Eight more warps bring tiles of 2048 values (32 or 64 tokens) of u, dt, z with their B and C into one of two buffers in shared
// memory, form d_t and d_t u_t once per token and channel on the way, and take y out of them through D and the gate.  (Bringing
// tiles in between steps of the computing warps themselves left both kinds of work waiting: two prompts of 4096 tokens, 2048
// channels, 16 states 231 us against 183.)  As many tokens at a time as a channel has lanes: the lanes' shares of their y are
// exchanged so that every lane ends up with the sum of one.  States in pairs (the packed fp32 arithmetic of sm_100).
//
// What bounds it: the exponentials, Ns a token and channel on the MUFU unit (16 a clock and SM), more than twice what
// the bytes take at Ns = 16 in bf16.
//
// A sequence is cut into chunks where the channels alone leave SMs idle: one pass for the chunks' own states from zero, a
// second that carries the state from chunk to chunk (h_end = exp(A sum d) h_begin + own), a third like the single pass, from
// the states that the second left.
#include "scan.cuh"
#include "tc_common.cuh"   // packed fp32 arithmetic

namespace jv {
namespace {

using tc::add2;
using tc::ex2;
using tc::fma2;
using tc::mul2;
using tc::pack2;
using tc::unpack2;

constexpr int kThreads = 256;         // that compute
// ... and that bring tiles in and out.  Measured with 256 / 128 of them, B x L tokens of 2048 channels: 2 x 4096 183 / 220 us, 4 x 2048 163 / 234,
// 8 x 2048 286 / 315.
constexpr int kStagers = 256;
constexpr int kTile = 2048;           // tokens times channels of a tile
constexpr int kStepTokens = 4;        // calls of at most this many tokens walk without tiles
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLog2eLo = (float)(1.4426950408889634 - (double)1.4426950408889634f);

// log(1 + e^x) = max(x, 0) + log1p(t), t = e^-|x|;  log1p(t) = 2 artanh(t / (2 + t)), the series of artanh up to the 15th power:
// its argument is 1/3 at most, so what is left out is below 2^-26 of it
__device__ __forceinline__ float softplus(float x) {
  // the exponent's product with log2 e is off by half a unit of its last place, a few 2^-22 of t: what is off is put back; the quotient with
  // one step of refinement
  const float e = -fabsf(x), hi = e * kLog2e, lo = fmaf(e, kLog2e, -hi) + e * kLog2eLo;
  float t = ex2(hi);
  if (hi > -120.f) t = fmaf(t, lo * 0.69314718f, t);       // (below, and at -inf, there is nothing to put back)
  const float r = __fdividef(1.f, 2.f + t), s0 = t * r, s = fmaf(fmaf(-s0, 2.f + t, t), r, s0), q = s * s;
  float a = fmaf(q, 1.f / 15.f, 1.f / 13.f);
  a = fmaf(q, a, 1.f / 11.f);
  a = fmaf(q, a, 1.f / 9.f);
  a = fmaf(q, a, 1.f / 7.f);
  a = fmaf(q, a, 1.f / 5.f);
  a = fmaf(q, a, 1.f / 3.f);
  a = fmaf(q, a, 1.f);
  const float top = x > 0.f ? x : x == x ? 0.f : x;        // (no number stays none)
  return fmaf(2.f * s, a, top);
}
__device__ __forceinline__ float silu(float x) { return __fdividef(x, 1.f + ex2(-x * kLog2e)); }

__device__ __forceinline__ int length_of(const ScanArgs& a, int b) { return a.lens ? min(max(__ldg(a.lens + b), 0), a.L) : a.L; }

// A coefficient, for powers of 2.  Infinities (minus: a state that is forgotten at once) as the numbers farthest from 0: a step of 0, as
// tokens and chunks past the end have it, then leaves the state alone, as it does elsewhere.
__device__ __forceinline__ float coefficient(float A) {
  const float a = A * kLog2e, most = 3.4028235e38f;
  return a < -most ? -most : a > most ? most : a;          // (no number stays none)
}
// A channel's coefficients and states: state n of lane s is s * NPL + n; states past Ns are zeros all through
template <int NPL>
__device__ __forceinline__ void load_A(const ScanArgs& a, int c, int s, float (&A2)[NPL]) {
  if (NPL % 4 == 0 && a.Ns % 4 == 0 && ((uintptr_t)a.A & 15) == 0) {        // 16 bytes at a time
#pragma unroll
    for (int n = 0; n + 3 < NPL; n += 4) {
      const float4 v = s * NPL + n < a.Ns ? __ldg(reinterpret_cast<const float4*>(a.A + (int64_t)c * a.Ns + s * NPL + n)) : make_float4(0.f, 0.f, 0.f, 0.f);
      A2[n] = coefficient(v.x); A2[n + 1] = coefficient(v.y); A2[n + 2] = coefficient(v.z); A2[n + 3] = coefficient(v.w);
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < NPL; ++n) A2[n] = s * NPL + n < a.Ns ? coefficient(__ldg(a.A + (int64_t)c * a.Ns + s * NPL + n)) : 0.f;
}
template <int NPL>
__device__ __forceinline__ void load_state(const float* h, int Ns, int s, float (&st)[NPL]) {
  if (NPL % 4 == 0 && h && Ns % 4 == 0 && ((uintptr_t)h & 15) == 0) {      // 16 bytes at a time
#pragma unroll
    for (int n = 0; n + 3 < NPL; n += 4) {
      const float4 v = s * NPL + n < Ns ? *reinterpret_cast<const float4*>(h + s * NPL + n) : make_float4(0.f, 0.f, 0.f, 0.f);
      st[n] = v.x; st[n + 1] = v.y; st[n + 2] = v.z; st[n + 3] = v.w;
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < NPL; ++n) st[n] = h && s * NPL + n < Ns ? h[s * NPL + n] : 0.f;
}
template <int NPL>
__device__ __forceinline__ void store_state(float* h, int Ns, int s, const float (&st)[NPL]) {
  if (NPL % 4 == 0 && Ns % 4 == 0 && ((uintptr_t)h & 15) == 0) {
#pragma unroll
    for (int n = 0; n + 3 < NPL; n += 4)
      if (s * NPL + n < Ns) *reinterpret_cast<float4*>(h + s * NPL + n) = make_float4(st[n], st[n + 1], st[n + 2], st[n + 3]);
    return;
  }
#pragma unroll
  for (int n = 0; n < NPL; ++n)
    if (s * NPL + n < Ns) h[s * NPL + n] = st[n];
}

// A lane's values of B or C of a token
template <typename T, int NPL>
__device__ __forceinline__ void load_row(const T* row, int Ns, int s, float (&v)[NPL]) {
  if (NPL % 4 == 0 && Ns % 4 == 0 && ((uintptr_t)row % (4 * sizeof(T))) == 0) {       // four at a time
#pragma unroll
    for (int n = 0; n + 3 < NPL; n += 4) {
      if (s * NPL + n >= Ns) {
        v[n] = v[n + 1] = v[n + 2] = v[n + 3] = 0.f;
      } else if constexpr (sizeof(T) == 4) {
        const float4 q = *reinterpret_cast<const float4*>(row + s * NPL + n);
        v[n] = q.x; v[n + 1] = q.y; v[n + 2] = q.z; v[n + 3] = q.w;
      } else {
        const uint2 q = *reinterpret_cast<const uint2*>(row + s * NPL + n);
        v[n] = __uint_as_float(q.x << 16);
        v[n + 1] = __uint_as_float(q.x & 0xffff0000u);
        v[n + 2] = __uint_as_float(q.y << 16);
        v[n + 3] = __uint_as_float(q.y & 0xffff0000u);
      }
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < NPL; ++n) v[n] = s * NPL + n < Ns ? to_f32(row[s * NPL + n]) : 0.f;
}

// ---- a few tokens: straight from global memory ------------------------------------------------------------------------
template <typename T, int NPL>
__global__ void __launch_bounds__(kThreads) scan_step_kernel(const ScanArgs a) {
  constexpr int kLanes = 4, kCh = kThreads / kLanes;
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.y, c = blockIdx.x * kCh + (int)threadIdx.x / kLanes, s = threadIdx.x % kLanes;
  const int cc = min(c, a.C - 1);                      // (lanes past the last channel follow it: the sums need whole warps)
  const int64_t ch = (int64_t)b * a.C + cc;
  const int len = length_of(a, b);
  float A2[NPL], h[NPL];
  load_A<NPL>(a, cc, s, A2);
  load_state<NPL>(a.h_in ? a.h_in + ch * a.Ns : nullptr, a.Ns, s, h);
  const float bias = a.dt_bias ? __ldg(a.dt_bias + cc) : 0.f, D = a.D ? __ldg(a.D + cc) : 0.f;
  for (int t = 0; t < len; ++t) {
    const float u = to_f32(((const T*)a.u)[a.us.at(b, t) + cc]);
    float d = to_f32(((const T*)a.dt)[a.ds.at(b, t) + cc]) + bias;
    const float z = a.z ? to_f32(((const T*)a.z)[a.zs.at(b, t) + cc]) : 0.f;
    float bm[NPL], cm[NPL];
    load_row<T, NPL>((const T*)a.Bm + a.bs.at(b, t), a.Ns, s, bm);
    load_row<T, NPL>((const T*)a.Cm + a.cs.at(b, t), a.Ns, s, cm);
    if (a.softplus) d = softplus(d);
    const float du = d * u;
    float y = 0.f;
#pragma unroll
    for (int n = 0; n < NPL; ++n) {
      h[n] = s * NPL + n < a.Ns ? fmaf(ex2(d * A2[n]), h[n], du * bm[n]) : 0.f;     // (0 times an infinite d or d u is no number)
      y = fmaf(h[n], cm[n], y);
    }
    y += __shfl_xor_sync(0xffffffffu, y, 1);
    y += __shfl_xor_sync(0xffffffffu, y, 2);
    if (s == 0 && c < a.C) {
      y = fmaf(D, u, y);
      if (a.z) y *= silu(z);
      from_f32((T*)a.y + ((int64_t)b * a.L + t) * a.C + c, y);
    }
  }
  if (a.h_out && c < a.C) store_state<NPL>(a.h_out + ch * a.Ns, a.Ns, s, h);
}

// ---- tiles of tokens ------------------------------------------------------------------------------------------------------
template <typename T, int S, int NPL>
struct Smem {
  static constexpr int kCh = kThreads / S, kTT = kTile / kCh;
  // bf16 pairs of B and C stay as they are: what a lane's registers take from shared memory, 32 lanes x 4 bytes a clock, is the
  // tightest resource beside the exponentials
  static constexpr bool kPacked = sizeof(T) == 2 && NPL > 1;
  using Pack = typename std::conditional<kPacked, T, float>::type;
  float2 d[kTT][kCh + 2];             // d, d u       (rows padded to lie in different banks)
  float y[kTT][kCh + 4];              // sum over the states
  Pack bc[kTT][S][2 * NPL];           // B, then C, of a lane's states
  T u[kTT][kCh], z[kTT][kCh];
};

// Barriers of a block: a buffer is full (it waits for the warps that bring tiles in); a buffer is done with (they wait for the others)
constexpr int kFull = 1, kDone = 3;
__device__ __forceinline__ void barrier_sync(int id) { asm volatile("bar.sync %0, %1;" ::"r"(id), "n"(kThreads + kStagers) : "memory"); }
__device__ __forceinline__ void barrier_arrive(int id) { asm volatile("bar.arrive %0, %1;" ::"r"(id), "n"(kThreads + kStagers) : "memory"); }

// The warps that bring tiles in, two ahead of the others, and y out
template <typename T, int S, int NPL, bool WIDE, bool kY>
__device__ __forceinline__ void stage_tiles(const ScanArgs& a, Smem<T, S, NPL>* buf, int b, int c0, int t_begin, int t_end, int tiles) {
  using Sm = Smem<T, S, NPL>;
  constexpr int kCh = Sm::kCh, kTT = Sm::kTT;
  constexpr int kVec = WIDE ? 16 / sizeof(T) : 1;             // elements of a load
  constexpr int kLoads = kTile / kStagers / kVec;             // loads of a thread and tile from each of u, dt, z
  constexpr int kRow = kCh / kVec;                            // loads of a token
  constexpr int kNs = S * NPL;
  constexpr int kBC = (kTT * kNs + kStagers - 1) / kStagers;  // elements of a thread and tile from each of B, C
  const int tid = threadIdx.x - kThreads;
  float bias[kVec], D[kVec];                                    // of the columns that this thread loads
#pragma unroll
  for (int v = 0; v < kVec; ++v) bias[v] = D[v] = 0.f;
  constexpr bool kOneColumn = kStagers % kRow == 0;             // every load of a thread is of the same columns
  static_assert(kOneColumn, "a thread's loads are of one set of columns");
  const int lcol = (tid % kRow) * kVec;
  if (a.dt_bias)
#pragma unroll
    for (int v = 0; v < kVec; ++v) bias[v] = __ldg(a.dt_bias + min(c0 + lcol + v, a.C - 1));
  if (a.D)
#pragma unroll
    for (int v = 0; v < kVec; ++v) D[v] = __ldg(a.D + min(c0 + lcol + v, a.C - 1));

  using Raw = typename std::conditional<WIDE, uint4, T>::type;
  Raw ru[kLoads], rd[kLoads], rz[kLoads];
  T rb[kBC], rc[kBC];
  auto fetch = [&](int t0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int t = t0 + (i * kStagers + tid) / kRow, col = c0 + lcol;
      const bool in = t < t_end && col < a.C;                  // (16 bytes at a time: C is a multiple of them)
      Raw zero;
      memset(&zero, 0, sizeof(Raw));
      ru[i] = in ? *reinterpret_cast<const Raw*>((const T*)a.u + a.us.at(b, t) + col) : zero;
      rd[i] = in ? *reinterpret_cast<const Raw*>((const T*)a.dt + a.ds.at(b, t) + col) : zero;
      if (kY) rz[i] = in && a.z ? *reinterpret_cast<const Raw*>((const T*)a.z + a.zs.at(b, t) + col) : zero;
    }
#pragma unroll
    for (int i = 0; i < kBC; ++i) {
      const int e = i * kStagers + tid, t = t0 + e / kNs, n = e % kNs;
      const bool in = t < t_end && n < a.Ns && e < kTT * kNs;
      rb[i] = in ? ((const T*)a.Bm)[a.bs.at(b, t) + n] : T(0.f);
      if (kY) rc[i] = in ? ((const T*)a.Cm)[a.cs.at(b, t) + n] : T(0.f);
    }
  };
  auto put = [&](Sm& sm, int t0) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int t = (i * kStagers + tid) / kRow;
      T uu[kVec], dd[kVec];
      memcpy(uu, &ru[i], sizeof(Raw));
      memcpy(dd, &rd[i], sizeof(Raw));
      float d_even = 0.f, du_even = 0.f;
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        float d = to_f32(dd[v]) + bias[v];
        if (a.softplus) d = softplus(d);
        if (t0 + t >= t_end) d = 0.f;                           // a token past the end: exp(0) h + 0
        const float du = d * to_f32(uu[v]);
        if constexpr (kVec == 1) {
          sm.d[t][lcol] = make_float2(d, du);
        } else {
          if (v & 1) *reinterpret_cast<float4*>(&sm.d[t][lcol + v - 1]) = make_float4(d_even, du_even, d, du);
          d_even = d;
          du_even = du;
        }
      }
      if (kY) {
        *reinterpret_cast<Raw*>(&sm.u[t][lcol]) = ru[i];
        *reinterpret_cast<Raw*>(&sm.z[t][lcol]) = rz[i];
      }
    }
#pragma unroll
    for (int i = 0; i < kBC; ++i) {
      const int e = i * kStagers + tid;
      if (e < kTT * kNs) {
        const int n = e % kNs;
        if constexpr (Sm::kPacked) {
          sm.bc[e / kNs][n / NPL][n % NPL] = rb[i];
          if (kY) sm.bc[e / kNs][n / NPL][NPL + n % NPL] = rc[i];
        } else {
          sm.bc[e / kNs][n / NPL][n % NPL] = to_f32(rb[i]);
          if (kY) sm.bc[e / kNs][n / NPL][NPL + n % NPL] = to_f32(rc[i]);
        }
      }
    }
  };
  auto flush = [&](const Sm& sm, int t0) {                      // y = (sum + D u) gate to global memory
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int t = (i * kStagers + tid) / kRow;
      if (t0 + t < t_end && c0 + lcol < a.C) {
        T uu[kVec], zz[kVec], yy[kVec];
        float sum[kVec];
        if constexpr (kVec == 1) {
          sum[0] = sm.y[t][lcol];
        } else {
#pragma unroll
          for (int v = 0; v < kVec; v += 4) {
            const float4 q = *reinterpret_cast<const float4*>(&sm.y[t][lcol + v]);
            sum[v] = q.x; sum[v + 1] = q.y; sum[v + 2] = q.z; sum[v + 3] = q.w;
          }
        }
        const Raw pu = *reinterpret_cast<const Raw*>(&sm.u[t][lcol]), pz = *reinterpret_cast<const Raw*>(&sm.z[t][lcol]);
        memcpy(uu, &pu, sizeof(Raw));
        memcpy(zz, &pz, sizeof(Raw));
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
          float r = fmaf(D[v], to_f32(uu[v]), sum[v]);
          if (a.z) r *= silu(to_f32(zz[v]));
          from_f32(&yy[v], r);
        }
        Raw py;
        memcpy(&py, yy, sizeof(Raw));
        *reinterpret_cast<Raw*>((T*)a.y + ((int64_t)b * a.L + t0 + t) * a.C + c0 + lcol) = py;
      }
    }
  };

  for (int i = 0; i < min(2, tiles); ++i) {
    fetch(t_begin + i * kTT);
    put(buf[i], t_begin + i * kTT);
    barrier_arrive(kFull + i);
  }
  for (int i = 0; i < tiles; ++i) {
    const int t0 = t_begin + i * kTT;
    if (i + 2 < tiles) fetch(t0 + 2 * kTT);
    barrier_sync(kDone + (i & 1));
    if (kY) flush(buf[i & 1], t0);                              // (a thread reads and refills the same places of u)
    if (i + 2 < tiles) {
      put(buf[i & 1], t0 + 2 * kTT);
      barrier_arrive(kFull + (i & 1));
    }
  }
}

// S lanes a channel, NPL states a lane.  kY: the whole thing; else the chunk's own state from zero and the sum of its steps only.
// kPad: there are states past Ns, to be kept at zero where d or d u are infinite (0 times that is no number); without kY they reach nothing.
template <typename T, int S, int NPL, bool WIDE, bool kY, bool kPad>
__global__ void __launch_bounds__(kThreads + kStagers, S == 4 && NPL <= 4 ? 2 : 1) scan_kernel(const ScanArgs a, int chunk, int nchunk, float* ws_state, float* ws_sum) {
  using Sm = Smem<T, S, NPL>;
  constexpr int kCh = Sm::kCh, kTT = Sm::kTT;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Sm* buf = reinterpret_cast<Sm*>(smem_raw);
  griddep_wait();
  griddep_launch_dependents();
  const int b = blockIdx.z, ck = blockIdx.y, c0 = blockIdx.x * kCh, tid = threadIdx.x;
  const int len = length_of(a, b);
  const int t_begin = ck * chunk, t_end = min(t_begin + chunk, len), tiles = max(0, (t_end - t_begin + kTT - 1) / kTT);

  if (tid >= kThreads) {
    stage_tiles<T, S, NPL, WIDE, kY>(a, buf, b, c0, t_begin, t_end, tiles);
    return;
  }
  const int lc = tid / S, s = tid % S, c = c0 + lc, cc = min(c, a.C - 1);
  const int64_t ch = ((int64_t)b * nchunk + ck) * a.C + cc;    // of the workspace's arrays
  float A2[NPL], h[NPL], sum = 0.f;
  load_A<NPL>(a, cc, s, A2);
  if (kY && nchunk > 1) load_state<NPL>(ws_state + ch * a.Ns, a.Ns, s, h);
  else load_state<NPL>(kY && a.h_in ? a.h_in + ((int64_t)b * a.C + cc) * a.Ns : nullptr, a.Ns, s, h);
  constexpr int kPairs = NPL / 2;
  uint64_t A2p[NPL > 1 ? kPairs : 1], hp[NPL > 1 ? kPairs : 1];
#pragma unroll
  for (int n = 0; n < kPairs; ++n) {
    A2p[n] = pack2(A2[2 * n], A2[2 * n + 1]);
    hp[n] = pack2(h[2 * n], h[2 * n + 1]);
  }
  auto keep = [&](int n) { return s * NPL + n < a.Ns ? 0xffffffffu : 0u; };
  for (int i = 0; i < tiles; ++i) {
    Sm& sm = buf[i & 1];
    const int t0 = t_begin + i * kTT;
    barrier_sync(kFull + (i & 1));
    const int tokens = min(kTT, t_end - t0);
#pragma unroll 1
    for (int t = 0; t < tokens; t += S) {                       // (kTT is a multiple of S; tokens past the end change nothing)
      float y[S];
#pragma unroll
      for (int j = 0; j < S; ++j) {
        const float2 q = sm.d[t + j][lc];
        const typename Sm::Pack* bc = sm.bc[t + j][s];
        if (!kY) sum += q.x;
        if constexpr (NPL == 1) {
          h[0] = fmaf(ex2(q.x * A2[0]), h[0], q.y * bc[0]);
          if (kPad) h[0] = __uint_as_float(__float_as_uint(h[0]) & keep(0));
          if (kY) y[j] = h[0] * bc[1];
        } else {
          constexpr int kUse = kY ? 2 * NPL : NPL;              // B, and C
          float v[kUse];
          constexpr int kWords = Sm::kPacked ? kUse / 2 : kUse;   // of 32 bits
          uint32_t words[kWords];
#pragma unroll
          for (int n = 0; n < kWords; n += kWords % 4 == 0 ? 4 : kWords % 2 == 0 ? 2 : 1) {
            const uint32_t* at = reinterpret_cast<const uint32_t*>(bc) + n;
            if constexpr (kWords % 4 == 0) {
              const uint4 x = *reinterpret_cast<const uint4*>(at);
              words[n] = x.x; words[n + 1] = x.y; words[n + 2] = x.z; words[n + 3] = x.w;
            } else if constexpr (kWords % 2 == 0) {
              const uint2 x = *reinterpret_cast<const uint2*>(at);
              words[n] = x.x; words[n + 1] = x.y;
            } else {
              words[n] = *at;
            }
          }
#pragma unroll
          for (int n = 0; n < kUse; ++n) {
            if constexpr (Sm::kPacked) v[n] = __uint_as_float(n & 1 ? words[n / 2] & 0xffff0000u : words[n / 2] << 16);
            else v[n] = __uint_as_float(words[n]);
          }
          const uint64_t dd = pack2(q.x, q.x), du = pack2(q.y, q.y);
          uint64_t yp = 0ull;
#pragma unroll
          for (int n = 0; n < kPairs; ++n) {
            float e0, e1;
            unpack2(mul2(dd, A2p[n]), e0, e1);
            hp[n] = fma2(pack2(ex2(e0), ex2(e1)), hp[n], mul2(du, pack2(v[2 * n], v[2 * n + 1])));
            if constexpr (kPad) hp[n] &= (uint64_t)keep(2 * n) | (uint64_t)keep(2 * n + 1) << 32;
            if constexpr (kY) {
              const uint64_t cn = pack2(v[NPL + 2 * n], v[NPL + 2 * n + 1]);
              yp = n == 0 ? mul2(hp[n], cn) : fma2(hp[n], cn, yp);
            }
          }
          if (kY) {
            float y0, y1;
            unpack2(yp, y0, y1);
            y[j] = y0 + y1;
          }
        }
      }
      if (kY) {
        // lanes that differ in bit k of their number exchange: each keeps the tokens whose bit k is its own, and token t + s is left
#pragma unroll
        for (int k = 1, left = S; left > 1; k <<= 1, left >>= 1)
#pragma unroll
          for (int i = 0; i < left / 2; ++i) {
            const float give = (s & k) ? y[2 * i] : y[2 * i + 1], keep = (s & k) ? y[2 * i + 1] : y[2 * i];
            y[i] = keep + __shfl_xor_sync(0xffffffffu, give, k);
          }
        sm.y[t + s][lc] = y[0];
      }
    }
    barrier_arrive(kDone + (i & 1));
  }
  if (c >= a.C) return;
#pragma unroll
  for (int n = 0; n < kPairs; ++n) unpack2(hp[n], h[2 * n], h[2 * n + 1]);
  if (kY) {
    // the state behind the last token: by the chunk that has it, the first one of an empty sequence
    if (a.h_out && (t_begin < t_end ? t_end == len : len == 0 && ck == 0)) store_state<NPL>(a.h_out + ((int64_t)b * a.C + c) * a.Ns, a.Ns, s, h);
  } else {
    store_state<NPL>(ws_state + ch * a.Ns, a.Ns, s, h);
    if (s == 0) ws_sum[ch] = sum;
  }
}

// h after steps of sum: exp(A sum) h, x = sum * A2.  Far powers in three parts: one that leaves fp32 may take h, or what is left of it, back
// into it, as the steps one by one do.  No state stays none, whatever it is multiplied with.
__device__ __forceinline__ float carried(float h, float x) {
  if (fabsf(x) <= 120.f) return ex2(x) * h;
  const float f = ex2(x * (1.f / 3.f));
  return h == 0.f ? 0.f : h * f * f * f;
}

// State from chunk to chunk, in place: a chunk's own state out, the state that it begins with in
__global__ void __launch_bounds__(256) scan_carry_kernel(const ScanArgs a, int nchunk, float* ws_state, const float* ws_sum) {
  griddep_wait();
  griddep_launch_dependents();
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)a.C * a.Ns;
  const int b = (int)(id / per);
  if (b >= a.B) return;
  const int64_t e = id - b * per;
  const int c = (int)(e / a.Ns);
  const float A2 = coefficient(__ldg(a.A + e));
  float h = a.h_in ? a.h_in[b * per + e] : 0.f;
  for (int k = 0; k < nchunk; ++k) {
    float* st = ws_state + ((int64_t)b * nchunk + k) * per + e;
    const float own = *st, sum = ws_sum[((int64_t)b * nchunk + k) * a.C + c];
    *st = h;
    h = carried(h, sum * A2) + own;
  }
}

template <typename T, int S, int NPL, bool WIDE, bool kPad>
cudaError_t launch_tiles(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  using Sm = Smem<T, S, NPL>;
  const dim3 grid((unsigned)ceil_div(a.C, Sm::kCh), (unsigned)p.nchunk, (unsigned)a.B);
  static OncePerDevice opt_in;
  cudaError_t e = opt_in.run([] {
    const cudaError_t r = cudaFuncSetAttribute(scan_kernel<T, S, NPL, WIDE, true, kPad>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * (int)sizeof(Sm));
    return r != cudaSuccess ? r : cudaFuncSetAttribute(scan_kernel<T, S, NPL, WIDE, false, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * (int)sizeof(Sm));
  });
  if (e != cudaSuccess) return e;
  float* state = p.nchunk > 1 ? (float*)((char*)ws + p.off_state) : nullptr;
  float* sum = p.nchunk > 1 ? (float*)((char*)ws + p.off_sum) : nullptr;
  if (p.nchunk > 1) {
    e = launch_programmatic(scan_kernel<T, S, NPL, WIDE, false, false>, grid, kThreads + kStagers, 2 * sizeof(Sm), st, a, p.chunk, p.nchunk, state, sum);
    if (e != cudaSuccess) return e;
    const int64_t n = (int64_t)a.B * a.C * a.Ns;
    e = launch_programmatic(scan_carry_kernel, dim3((unsigned)((n + 255) / 256)), 256, 0, st, a, p.nchunk, state, (const float*)sum);
    if (e != cudaSuccess) return e;
  }
  return launch_programmatic(scan_kernel<T, S, NPL, WIDE, true, kPad>, grid, kThreads + kStagers, 2 * sizeof(Sm), st, a, p.chunk, p.nchunk, state, sum);
}

template <typename T, int S, int NPL>
cudaError_t launch_states(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  const size_t e = sizeof(T);
  const bool wide = ((uintptr_t)a.u | (uintptr_t)a.dt | (uintptr_t)a.z | (uintptr_t)a.y | a.C * e | a.us.tok * e | a.us.batch * e |
                     a.ds.tok * e | a.ds.batch * e | (a.z ? (a.zs.tok | a.zs.batch) * e : 0)) % 16 == 0;
  if (a.Ns < S * NPL) return wide ? launch_tiles<T, S, NPL, true, true>(a, p, ws, st) : launch_tiles<T, S, NPL, false, true>(a, p, ws, st);
  return wide ? launch_tiles<T, S, NPL, true, false>(a, p, ws, st) : launch_tiles<T, S, NPL, false, false>(a, p, ws, st);
}

template <typename T>
cudaError_t launch_type(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  if (a.L <= kStepTokens) {
    const dim3 grid((unsigned)ceil_div(a.C, kThreads / 4), (unsigned)a.B);
    const int npl = ceil_div(a.Ns, 4);
    if (npl <= 1) return launch_programmatic(scan_step_kernel<T, 1>, grid, kThreads, 0, st, a);
    if (npl <= 2) return launch_programmatic(scan_step_kernel<T, 2>, grid, kThreads, 0, st, a);
    if (npl <= 4) return launch_programmatic(scan_step_kernel<T, 4>, grid, kThreads, 0, st, a);
    if (npl <= 8) return launch_programmatic(scan_step_kernel<T, 8>, grid, kThreads, 0, st, a);
    return launch_programmatic(scan_step_kernel<T, 16>, grid, kThreads, 0, st, a);
  }
  const int npl = ceil_div(a.Ns, p.lanes);
  if (p.lanes == 4) {
    if (npl <= 1) return launch_states<T, 4, 1>(a, p, ws, st);
    if (npl <= 2) return launch_states<T, 4, 2>(a, p, ws, st);
    if (npl <= 4) return launch_states<T, 4, 4>(a, p, ws, st);
    return launch_states<T, 4, 8>(a, p, ws, st);
  }
  if (npl <= 1) return launch_states<T, 8, 1>(a, p, ws, st);
  if (npl <= 2) return launch_states<T, 8, 2>(a, p, ws, st);
  if (npl <= 4) return launch_states<T, 8, 4>(a, p, ws, st);
  return launch_states<T, 8, 8>(a, p, ws, st);
}

}  // namespace

ScanPlan scan_plan(int B, int L, int C, int Ns) {
  ScanPlan p{4, 1, L, 0, 0, 0};
  if (L <= kStepTokens) return p;
  // Four lanes a channel where the channels give two of three SMs a block all the same, eight where they do with half as many
  // channels a block (and above 32 states, which eight lanes hold); chunks, which walk the exponentials twice, for two blocks an SM elsewhere
  const int64_t sms = device_sm_count(), four = (int64_t)B * ceil_div(C, kThreads / 4), eight = (int64_t)B * ceil_div(C, kThreads / 8);
  // (Measured: 2 x 4096 tokens of 2048 channels, four lanes 308 us, eight 184, chunks 255; 4 x 2048, four / eight 163 / 181; 1 x 4096, chunks
  // of four / eight lanes 124 / 155.  Eight lanes against chunks: 2 x 4096 tokens of 1600 channels, just above two thirds of the SMs,
  // 185 / 209; 5 x 1369 of 768, fp32, 67 / 94.  Blocks cannot know the lengths, so a ragged call takes as long as its longest sequence.)
  const bool pass = 3 * four >= 2 * sms || 3 * eight >= 2 * sms;
  p.lanes = Ns > 32 || (pass && 3 * four < 2 * sms) ? 8 : 4;
  if (!pass) {
    const int64_t blocks = p.lanes == 8 ? eight : four;
    const int tt = kTile / (kThreads / p.lanes), want = (int)(2 * sms / blocks), tiles = ceil_div(L, tt);
    p.chunk = ceil_div(tiles, want < tiles ? want : tiles) * tt;
    p.nchunk = ceil_div(L, p.chunk);
  }
  if (p.nchunk > 1) {
    p.off_sum = align_up((size_t)B * p.nchunk * C * Ns * 4, 256);
    p.total = p.off_sum + (size_t)B * p.nchunk * C * 4;
  }
  return p;
}

cudaError_t launch_selective_scan(const ScanArgs& a, const ScanPlan& p, void* ws, cudaStream_t st) {
  return a.dtype == JV_F32 ? launch_type<float>(a, p, ws, st) : launch_type<__nv_bfloat16>(a, p, ws, st);
}

}  // namespace jv

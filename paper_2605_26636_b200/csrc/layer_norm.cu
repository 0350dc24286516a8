// Layer norm of token rows and its gradient, in front of the projections of a block.
//
//   y = (x - m) r w + b,  m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps)             per row of C values
//   g = dy w,  xh = (x - m) r:   dx = r (g - mean g - xh mean(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// Both are bound by HBM: a row is read once, held in registers, and written once.  A row of up to 1024 values belongs to a warp
// (up to 32 values a lane, in 16-byte pieces 32 lanes side by side), a longer one to a block; sums are fp32, the variance is
// that of the centred values (no cancellation where a row's mean is large against its spread).
//
// Measured: 32768 rows of 1024 bf16 values 22.7 us (gradient 39.6), 21845 of 1536 31.0 (150), 16384 of 2048 29.5 (131); floors 20.5 (30.7).
// The gradient of rows longer than 1024 waits for each row where it needs it, at two blocks of few warps per SM; so it does for rows read
// value by value (32768 of 1023: 198 us, forward 52.7).
//
// The gradient's blocks are persistent: every lane keeps the sums of its columns for dw and db in registers over the rows that its
// warp walks, the warps of a block add theirs through shared memory, the blocks' partials go to the workspace and a second
// launch adds them up, all in a fixed order: no atomics, results repeat bit for bit.
#include "common.cuh"
#include "tc_common.cuh"   // packed fp32 arithmetic

namespace jv {
namespace {

template <typename T, int VEC>
struct Piece;                       // VEC consecutive values as they lie in memory
template <>
struct Piece<__nv_bfloat16, 8> {
  uint4 r;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    r = make_uint4(u[0], u[1], u[2], u[3]);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = r; }
};
template <>
struct Piece<float, 4> {
  float4 r;
  __device__ __forceinline__ void load(const float* p) { r = __ldcs(reinterpret_cast<const float4*>(p)); }
  __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
  __device__ __forceinline__ void set(const float (&f)[4]) { r = make_float4(f[0], f[1], f[2], f[3]); }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = r; }
};
template <typename T>
struct Piece<T, 1> {
  T r;
  __device__ __forceinline__ void load(const T* p) { r = __ldcs(p); }
  __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = to_f32(r); }
  __device__ __forceinline__ void set(const float (&f)[1]) { from_f32(&r, f[0]); }
  __device__ __forceinline__ void store(T* p) const { *p = r; }
};

// VEC fp32 values: weights and biases, partial sums
template <int VEC>
__device__ __forceinline__ void load_f32(const float* p, float (&f)[VEC]) {
  if constexpr (VEC == 1) {
    f[0] = __ldg(p);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const float4 v = __ldg(reinterpret_cast<const float4*>(p + i));
      f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
    }
  }
}

// Sums over the threads that share a row: a warp, or the block (red: 2 x 32 floats of shared memory, used in turn)
template <bool BLOCK, int N>
__device__ __forceinline__ void row_sums(float (&s)[N], float* red, int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = warp_sum(s[i]);
  if (!BLOCK) return;
  const int warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  float* dst = red + turn * 32 * N;                 // the other half: the one before may still be read
  turn ^= 1;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) dst[N * warp + i] = s[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    s[i] = 0.f;
    for (int w = 0; w < nwarps; ++w) s[i] += dst[N * w + i];
  }
}

struct NormParams {
  const void *x, *dy;
  const float *w, *b;
  void* y;                          // y, or dx
  float *mean, *rstd;               // written by the forward pass unless null, read by the gradient
  float* partial;                   // gradient: [blocks, 2, C]
  int64_t rows, x_stride, dy_stride;
  int C;
  float eps;
};

// A row whose variance is not safely within fp32 (values some 1e17 apart and more, or, without an eps, 1e-15 and less), by the threads that
// share it, once more from the start: the row, and eps with it, times the power of two k.  A call of its own at the end of the kernel, so that
// the rest of it keeps its registers (in its middle it took 17 % of the rows read value by value).
template <typename T, bool BLOCK>
__device__ __noinline__ void far_row(const T* x, const float* w, const float* b, T* y, float* mean, float* rstd, int C, float eps, float k,
                                     float* red, int turn) {
  const int tl = BLOCK ? threadIdx.x : threadIdx.x & 31, nl = BLOCK ? blockDim.x : 32;
  const float inv_c = 1.f / (float)C;
  float s[1] = {0.f};
  for (int c = tl; c < C; c += nl) s[0] += to_f32(x[c]) * k;
  row_sums<BLOCK, 1>(s, red, turn);
  const float m = s[0] * inv_c;
  s[0] = 0.f;
  for (int c = tl; c < C; c += nl) {
    const float d = fmaf(to_f32(x[c]), k, -m);
    s[0] = fmaf(d, d, s[0]);
  }
  row_sums<BLOCK, 1>(s, red, turn);
  const float r = rsqrtf(fmaf(s[0], inv_c, eps * k * k));
  if (!BLOCK) __syncwarp();                         // (what is written here other threads have written before)
  for (int c = tl; c < C; c += nl) from_f32(y + c, fmaf(fmaf(to_f32(x[c]), k, -m) * r, w ? __ldg(w + c) : 1.f, b ? __ldg(b + c) : 0.f));
  if (mean && tl == 0) {
    *mean = m * (k > 1.f ? 0x1p-100f : 0x1p+80f);
    *rstd = r * k;
  }
}

// Columns of lane `tl` (of `nl` that share a row): pieces tl, tl + nl, ...  R rows of a warp at a time: w and b pass through L1 once for
// them (for one row of bf16 values they are four times the row's bytes).
template <typename T, int VEC, int NCH, bool BLOCK, int R>
__global__ void __launch_bounds__(BLOCK ? 512 : 128, 1) layer_norm_kernel(const NormParams p) {
  __shared__ float red[64];
  griddep_wait();
  griddep_launch_dependents();
  const int tl = BLOCK ? threadIdx.x : threadIdx.x & 31, nl = BLOCK ? blockDim.x : 32;
  const int64_t row0 = BLOCK ? blockIdx.x : ((int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5)) * R;
  if (row0 >= p.rows) return;        // (whole warps or blocks)
  Piece<T, VEC> in[R][NCH];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const T* x = (const T*)p.x + min(row0 + r, p.rows - 1) * p.x_stride;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = (j * nl + tl) * VEC;
      if (c < p.C) in[r][j].load(x + c);
    }
  }
  const float inv_c = 1.f / (float)p.C;
  int turn = 0;
  float mean[R], rstd[R], s[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    s[r] = 0.f;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if ((j * nl + tl) * VEC < p.C) {
        float f[VEC];
        in[r][j].get(f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[r] += f[i];
      }
  }
  row_sums<BLOCK, R>(s, red, turn);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    mean[r] = s[r] * inv_c;
    s[r] = 0.f;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if ((j * nl + tl) * VEC < p.C) {
        float f[VEC];
        in[r][j].get(f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) s[r] = fmaf(f[i] - mean[r], f[i] - mean[r], s[r]);
      }
  }
  row_sums<BLOCK, R>(s, red, turn);
#pragma unroll
  for (int r = 0; r < R; ++r) rstd[r] = rsqrtf(fmaf(s[r], inv_c, p.eps));
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    const int c = (j * nl + tl) * VEC;
    if (c < p.C) {
      float w[VEC], b[VEC];
#pragma unroll
      for (int i = 0; i < VEC; ++i) { w[i] = 1.f; b[i] = 0.f; }
      if (p.w) load_f32<VEC>(p.w + c, w);
      if (p.b) load_f32<VEC>(p.b + c, b);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float f[VEC];
        in[r][j].get(f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = fmaf((f[i] - mean[r]) * rstd[r], w[i], b[i]);
        in[r][j].set(f);
        if (R == 1 || row0 + r < p.rows) in[r][j].store((T*)p.y + (row0 + r) * p.C + c);
      }
    }
  }
  if (p.mean && tl == 0)
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (row0 + r < p.rows) {
        p.mean[row0 + r] = mean[r];
        p.rstd[row0 + r] = rstd[r];
      }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    // variances from 1e-30 to fp32's end; beside a mean of 1 and more a smaller one is 0, no two values are that close
    const bool tiny = rstd[r] > 1e15f;
    if ((rstd[r] > 0.f && !tiny) || (tiny && fabsf(mean[r]) >= 1.f) || row0 + r >= p.rows) continue;
    const int64_t row = row0 + r;
    far_row<T, BLOCK>((const T*)p.x + row * p.x_stride, p.w, p.b, (T*)p.y + row * p.C, p.mean ? p.mean + row : nullptr,
                      p.mean ? p.rstd + row : nullptr, p.C, p.eps, tiny ? 0x1p+100f : 0x1p-80f, red, turn);
  }
}

// stages of a warp's ring: 1 KB for a piece of x and dy each
template <int NCH>
constexpr int kGradStages = 16 / NCH < 2 ? 2 : 16 / NCH > 4 ? 4 : 16 / NCH;

// ---- gradient, rows of a warp in 16-byte pieces --------------------------------------------------------------------------
// The rows ahead are on their way into shared memory (cp.async: every lane copies the pieces that it will read, so no barrier
// is in it) while this one is worked on, twice, from there: registers hold the sums of dw and db and the weights only.
// One block of twelve warps per SM: few partials, and a ring of 16 KB at most to each warp.
constexpr int kGradWarps = 12;
template <typename T, int VEC, int NCH>
__global__ void __launch_bounds__(kGradWarps * 32, 1) layer_norm_grad_rows_kernel(const NormParams p) {
  constexpr int kStages = kGradStages<NCH>, kRing = kStages * 2 * NCH * 512;
  extern __shared__ __align__(16) unsigned char ring[];   // [warp][stage][x, dy][piece][lane] of 16 bytes; at the end [warp][dw, db][columns]
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const int64_t first = (int64_t)blockIdx.x * nwarps + warp, step = (int64_t)gridDim.x * nwarps;
  unsigned char* mine = ring + (size_t)warp * kRing + lane * 16;
  auto fetch = [&](int64_t row, int stage) {
    if (row < p.rows) {
      const T *x = (const T*)p.x + row * p.x_stride, *dy = (const T*)p.dy + row * p.dy_stride;
#pragma unroll
      for (int j = 0; j < NCH; ++j) {
        const int c = (j * 32 + lane) * VEC;
        if (c < p.C) {
          const uint32_t dst = (uint32_t)__cvta_generic_to_shared(mine + (stage * 2 * NCH + j) * 512);
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(x + c) : "memory");
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + NCH * 512), "l"(dy + c) : "memory");
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // Pairs of values in the packed arithmetic of sm_100: with single values the instructions of a row of bf16, not its bytes, bounded
  // this (32768 rows of 1024: 50 us).
  using namespace tc;
  constexpr int kPairs = VEC / 2;
  uint64_t dw[NCH][kPairs], db[NCH][kPairs], w[NCH][kPairs];
#pragma unroll
  for (int j = 0; j < NCH; ++j) {
    float f[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) f[i] = 1.f;
    if (p.w && (j * 32 + lane) * VEC < p.C) load_f32<VEC>(p.w + (j * 32 + lane) * VEC, f);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      dw[j][i] = db[j][i] = 0ull;
      w[j][i] = pack2(f[2 * i], f[2 * i + 1]);
    }
  }
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) fetch(first + s * step, s);
  const float inv_c = 1.f / (float)p.C;
  int stage = 0;
  // a row's statistics are loaded a row ahead, too (where they were needed at once every warp waited for them, row after row: 32768 rows
  // of 1024 bf16 values 46.9 us, now 40.0; 21316 of 768 fp32 34 to 36 us either way)
  float mean_next = 0.f, rstd_next = 0.f;
  auto statistics = [&](int64_t row) {
    if (row < p.rows) {
      mean_next = __ldg(p.mean + row);
      rstd_next = __ldg(p.rstd + row);
    }
  };
  statistics(first);
  for (int64_t row = first; row < p.rows; row += step) {
    fetch(row + (kStages - 1) * step, stage == 0 ? kStages - 1 : stage - 1);
    const float mean = mean_next, rstd = rstd_next;
    statistics(row + step);
    const uint64_t nmean2 = pack2(-mean, -mean), rstd2 = pack2(rstd, rstd);
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    const unsigned char* at = mine + stage * 2 * NCH * 512;
    auto pairs = [&](const unsigned char* src, uint64_t (&v)[kPairs]) {
      Piece<T, VEC> q;
      q.r = *reinterpret_cast<const decltype(q.r)*>(src);
      float f[VEC];
      q.get(f);
#pragma unroll
      for (int i = 0; i < kPairs; ++i) v[i] = pack2(f[2 * i], f[2 * i + 1]);
    };
    uint64_t s0 = 0ull, s1 = 0ull;
#pragma unroll
    for (int j = 0; j < NCH; ++j)
      if ((j * 32 + lane) * VEC < p.C) {
        uint64_t x[kPairs], d[kPairs];
        pairs(at + j * 512, x);
        pairs(at + (NCH + j) * 512, d);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          const uint64_t xh = mul2(add2(x[i], nmean2), rstd2), g = mul2(d[i], w[j][i]);
          dw[j][i] = fma2(d[i], xh, dw[j][i]);
          db[j][i] = add2(db[j][i], d[i]);
          s0 = add2(s0, g);
          s1 = fma2(g, xh, s1);
        }
      }
    float a, b;
    unpack2(s0, a, b);
    const float mg = warp_sum(a + b) * inv_c;
    unpack2(s1, a, b);
    const float mgx = warp_sum(a + b) * inv_c;
    const uint64_t nmg2 = pack2(-mg, -mg), nmgx2 = pack2(-mgx, -mgx);
    T* dx = (T*)p.y + row * p.C;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = (j * 32 + lane) * VEC;
      if (c < p.C) {
        uint64_t x[kPairs], d[kPairs];
        pairs(at + j * 512, x);
        pairs(at + (NCH + j) * 512, d);
        float f[VEC];
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          const uint64_t xh = mul2(add2(x[i], nmean2), rstd2);
          unpack2(mul2(rstd2, fma2(xh, nmgx2, fma2(d[i], w[j][i], nmg2))), f[2 * i], f[2 * i + 1]);
        }
        Piece<T, VEC> q;
        q.set(f);
        q.store(dx + c);
      }
    }
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
  if (!p.partial) return;
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncwarp();                                           // (a warp's sums take its own ring's place)
  constexpr int kCols = NCH * 32 * VEC;
  float* own = reinterpret_cast<float*>(ring + (size_t)warp * kRing);
#pragma unroll
  for (int j = 0; j < NCH; ++j)
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const int c = (j * 32 + lane) * VEC + 2 * i;
      *reinterpret_cast<uint64_t*>(own + c) = dw[j][i];
      *reinterpret_cast<uint64_t*>(own + kCols + c) = db[j][i];
    }
  __syncthreads();
  float* part = p.partial + (size_t)blockIdx.x * 2 * p.C;
  for (int c = threadIdx.x; c < 2 * p.C; c += blockDim.x) {
    const int at = c < p.C ? c : c - p.C + kCols;
    float s = 0.f;
    for (int k = 0; k < nwarps; ++k) s += reinterpret_cast<const float*>(ring + (size_t)k * kRing)[at];
    part[c] = s;
  }
}

// ---- gradient of other rows: read value by value, or (BLOCK) longer than 1024 ----------------------------------------------
// Shared memory: BLOCK: 128 floats; else the block's sums, 2 C floats, added to by its warps one after the other
template <typename T, int VEC, int NCH, bool BLOCK>
__global__ void __launch_bounds__(BLOCK ? 512 : 128, 1) layer_norm_grad_kernel(const NormParams p) {
  extern __shared__ float sm[];
  griddep_wait();
  griddep_launch_dependents();
  const int tl = BLOCK ? threadIdx.x : threadIdx.x & 31, nl = BLOCK ? blockDim.x : 32;
  const int warp = threadIdx.x >> 5, nwarps = blockDim.x >> 5;
  const int64_t first = BLOCK ? blockIdx.x : (int64_t)blockIdx.x * nwarps + warp;
  const int64_t step = BLOCK ? gridDim.x : (int64_t)gridDim.x * nwarps;
  float dw[NCH][VEC], db[NCH][VEC];
#pragma unroll
  for (int j = 0; j < NCH; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) dw[j][i] = db[j][i] = 0.f;
  const float inv_c = 1.f / (float)p.C;
  int turn = 0;
  for (int64_t row = first; row < p.rows; row += step) {
    const T *x = (const T*)p.x + row * p.x_stride, *dy = (const T*)p.dy + row * p.dy_stride;
    Piece<T, VEC> px[NCH], pd[NCH];
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = (j * nl + tl) * VEC;
      if (c < p.C) {
        px[j].load(x + c);
        pd[j].load(dy + c);
      }
    }
    const float mean = __ldg(p.mean + row), rstd = __ldg(p.rstd + row);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = (j * nl + tl) * VEC;
      if (c < p.C) {
        float f[VEC], d[VEC], w[VEC];
        px[j].get(f);
        pd[j].get(d);
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[i] = 1.f;
        if (p.w) load_f32<VEC>(p.w + c, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float xh = (f[i] - mean) * rstd, g = d[i] * w[i];
          dw[j][i] = fmaf(d[i], xh, dw[j][i]);
          db[j][i] += d[i];
          s[0] += g;
          s[1] = fmaf(g, xh, s[1]);
        }
      }
    }
    row_sums<BLOCK, 2>(s, sm, turn);
    const float mg = s[0] * inv_c, mgx = s[1] * inv_c;
    T* dx = (T*)p.y + row * p.C;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
      const int c = (j * nl + tl) * VEC;
      if (c < p.C) {
        float f[VEC], d[VEC], w[VEC];
        px[j].get(f);
        pd[j].get(d);
#pragma unroll
        for (int i = 0; i < VEC; ++i) w[i] = 1.f;
        if (p.w) load_f32<VEC>(p.w + c, w);
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = rstd * (d[i] * w[i] - mg - (f[i] - mean) * rstd * mgx);
        px[j].set(f);
        px[j].store(dx + c);
      }
    }
  }
  if (!p.partial) return;
  float* part = p.partial + (size_t)blockIdx.x * 2 * p.C;
  if (BLOCK) {
#pragma unroll
    for (int j = 0; j < NCH; ++j)
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        const int c = (j * nl + tl) * VEC + i;
        if (c < p.C) {
          part[c] = dw[j][i];
          part[p.C + c] = db[j][i];
        }
      }
  } else {
    for (int w = 0; w < nwarps; ++w) {
      if (w == warp)
#pragma unroll
        for (int j = 0; j < NCH; ++j)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const int c = (j * nl + tl) * VEC + i;
            if (c < p.C) {
              sm[c] = (w ? sm[c] : 0.f) + dw[j][i];
              sm[p.C + c] = (w ? sm[p.C + c] : 0.f) + db[j][i];
            }
          }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < 2 * p.C; c += blockDim.x) part[c] = sm[c];
  }
}

// Column sums of the blocks' partials [n, 2, C]: 32 columns a block, kSumParts threads a column (a call of 32768 rows of 1024 with 8 / 16:
// 41.3 / 40.0 us)
constexpr int kSumParts = 16;
__global__ void __launch_bounds__(kSumParts * 32) layer_norm_sum_kernel(const float* __restrict__ partial, int n, int C, float* dw, float* db) {
  __shared__ float red[kSumParts][33];
  griddep_wait();
  griddep_launch_dependents();
  const int lane = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < 2 * C) {
#pragma unroll 8
    for (int i = part; i < n; i += kSumParts) s += __ldcg(partial + (size_t)i * 2 * C + c);
  }
  red[part][lane] = s;
  __syncthreads();
  if (part == 0 && c < 2 * C) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < kSumParts; ++i) s += red[i][lane];
    if (c < C) {
      if (dw) dw[c] = s;
    } else if (db) {
      db[c - C] = s;
    }
  }
}

constexpr int kWarpCols = 1024;         // longest row that one warp takes
constexpr int kNormWarps = 4;           // warps of a block that take a row each

int norm_block_warps(int C) { return (C + kWarpCols - 1) / kWarpCols; }

// 16-byte pieces where every row starts on such a boundary, single values elsewhere
bool norm_wide(const NormArgs& a) {
  const size_t e = a.dtype == JV_F32 ? 4 : 2;
  const uintptr_t low = (uintptr_t)a.x | (uintptr_t)a.dy | (uintptr_t)a.y | (uintptr_t)a.w | (uintptr_t)a.b | a.C * e | a.x_stride * e | a.dy_stride * e;
  return low % 16 == 0;
}

template <typename T, int VEC, int NCH>
cudaError_t launch_norm_rows(const NormParams& p, int64_t blocks, cudaStream_t st) {
  // Two rows of bf16 values a warp where there are enough to fill the chip all the same.  Measured, one / two / four rows a warp: 32768
  // rows of 1024 values 27.3 / 24.1 / 24.4 us (5.6 TB/s, what a plain copy of this size reaches), of 384 13.8 / 12.9 / 12.9; fp32, whose rows
  // are twice the bytes against the same weights, 21316 of 768: 22.5 / 22.7 / 23.1.
  if (VEC == 8 && p.rows >= 2ll * 16 * device_sm_count())
    return launch_programmatic(layer_norm_kernel<T, VEC, NCH, false, (VEC == 8 ? 2 : 1)>, dim3((unsigned)((blocks + 1) / 2)), kNormWarps * 32, 0, st, p);
  return launch_programmatic(layer_norm_kernel<T, VEC, NCH, false, 1>, dim3((unsigned)blocks), kNormWarps * 32, 0, st, p);
}
template <typename T, int VEC, int NCH>
cudaError_t launch_grad_rows(const NormParams& p, int64_t blocks, cudaStream_t st) {
  if constexpr (VEC > 1) {
    constexpr size_t smem = (size_t)kGradWarps * kGradStages<NCH> * 2 * NCH * 512;
    static_assert(kGradStages<NCH> * 2 * NCH * 512 >= 2 * NCH * 32 * VEC * (int)sizeof(float), "a warp's sums take its ring's place");
    static OncePerDevice opt_in;
    const cudaError_t e = opt_in.run([] { return cudaFuncSetAttribute(layer_norm_grad_rows_kernel<T, VEC, NCH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
    if (e != cudaSuccess) return e;
    return launch_programmatic(layer_norm_grad_rows_kernel<T, VEC, NCH>, dim3((unsigned)blocks), kGradWarps * 32, smem, st, p);
  } else {
    return launch_programmatic(layer_norm_grad_kernel<T, VEC, NCH, false>, dim3((unsigned)blocks), kNormWarps * 32, 2 * (size_t)p.C * sizeof(float), st, p);
  }
}

template <typename T, int VEC, bool GRAD>
cudaError_t launch_norm(const NormArgs& a, const NormParams& p, int blocks, cudaStream_t st) {
  constexpr int kAll = 32 / VEC;        // pieces of a lane that holds 32 values
  if (a.C > kWarpCols) {
    const int threads = norm_block_warps(a.C) * 32;
    if (GRAD) return launch_programmatic(layer_norm_grad_kernel<T, VEC, kAll, true>, dim3((unsigned)blocks), threads, 128 * sizeof(float), st, p);
    return launch_programmatic(layer_norm_kernel<T, VEC, kAll, true, 1>, dim3((unsigned)blocks), threads, 0, st, p);
  }
  const int quarter = (a.C + 255) / 256;                 // 8, 16, 24 or 32 values a lane
  switch (quarter) {
    case 1: return GRAD ? launch_grad_rows<T, VEC, kAll / 4>(p, blocks, st) : launch_norm_rows<T, VEC, kAll / 4>(p, blocks, st);
    case 2: return GRAD ? launch_grad_rows<T, VEC, kAll / 2>(p, blocks, st) : launch_norm_rows<T, VEC, kAll / 2>(p, blocks, st);
    case 3: return GRAD ? launch_grad_rows<T, VEC, kAll / 4 * 3>(p, blocks, st) : launch_norm_rows<T, VEC, kAll / 4 * 3>(p, blocks, st);
    default: return GRAD ? launch_grad_rows<T, VEC, kAll>(p, blocks, st) : launch_norm_rows<T, VEC, kAll>(p, blocks, st);
  }
}

template <bool GRAD>
cudaError_t dispatch_norm(const NormArgs& a, const NormParams& p, int blocks, cudaStream_t st) {
  const bool wide = norm_wide(a);
  if (a.dtype == JV_F32) return wide ? launch_norm<float, 4, GRAD>(a, p, blocks, st) : launch_norm<float, 1, GRAD>(a, p, blocks, st);
  return wide ? launch_norm<__nv_bfloat16, 8, GRAD>(a, p, blocks, st) : launch_norm<__nv_bfloat16, 1, GRAD>(a, p, blocks, st);
}

}  // namespace

namespace {
// Blocks of the gradient's launch: of twelve rows at a time, of four where rows are read value by value, of one where they are long
int grad_blocks(int64_t rows, int C, bool wide) {
  const int64_t per_block = C > kWarpCols ? 1 : wide ? kGradWarps : kNormWarps;
  const int64_t most = (C > kWarpCols ? 2ll : wide ? 1ll : 3ll) * device_sm_count(), need = (rows + per_block - 1) / per_block;
  return (int)(need < most ? need : most);
}
}  // namespace

int layer_norm_grad_blocks(int64_t rows, int C) {
  const int a = grad_blocks(rows, C, false), b = grad_blocks(rows, C, true);
  return a > b ? a : b;
}

cudaError_t launch_layer_norm(const NormArgs& a, cudaStream_t st) {
  const NormParams p{a.x, nullptr, a.w, a.b, a.y, a.mean, a.rstd, nullptr, a.rows, a.x_stride, 0, a.C, a.eps};
  const int64_t blocks = a.C > kWarpCols ? a.rows : (a.rows + kNormWarps - 1) / kNormWarps;
  return dispatch_norm<false>(a, p, (int)blocks, st);
}

cudaError_t launch_layer_norm_grad(const NormArgs& a, float* partial, float* dw, float* db, cudaStream_t st) {
  const bool sums = dw || db;
  const int blocks = grad_blocks(a.rows, a.C, norm_wide(a));
  const NormParams p{a.x, a.dy, a.w, nullptr, a.y, a.mean, a.rstd, sums ? partial : nullptr, a.rows, a.x_stride, a.dy_stride, a.C, 0.f};
  const cudaError_t e = dispatch_norm<true>(a, p, blocks, st);
  if (e != cudaSuccess || !sums) return e;
  return launch_programmatic(layer_norm_sum_kernel, dim3((unsigned)ceil_div(2 * a.C, 32)), kSumParts * 32, 0, st, (const float*)partial, blocks, a.C, dw, db);
}

}  // namespace jv

// Layer norm over the rows of a matrix [M][N], and its gradients.
//   forward   mu = mean_j x,  v = mean_j (x - mu)^2,  r = 1/sqrt(v + eps),  xhat = (x - mu) r,  y = gamma xhat + beta
//   backward  g = gamma dy;  dx = r (g - mean_j g - xhat mean_j(g xhat)) [+ addend];  dgamma = sum_i dy xhat,  dbeta = sum_i dy
// A row is read once and stays in registers: the variance is taken about the mean itself, not as a difference of two sums.  All of it is
// fp32, the rows' sums too (a sum of N terms in a tree of 8 or more branches); the sums of the columns are joined in float64.
// Every reduction has a fixed order.
#include <algorithm>

#include "dense.h"

namespace resist {
namespace {

constexpr int kThreads = 256;
constexpr int kHeldCols = 8192;   // widest row that the threads of a workgroup hold in registers

struct LnArgs {
  const void *x, *dy, *addend;
  void *out;                       // y, or dx
  const float *gamma, *beta;
  float *mean, *rstd;              // written by the forward pass, read by the backward pass
  float *part;                     // [parts][2][N]: sums over a workgroup's rows of dy xhat, and of dy
  long long M, ldx, lddy, lda, ldo;
  int N;
  float eps;
};

// the sum over the TPR threads of a row; `red`: [waves of the workgroup] when a row is a workgroup's
template <int TPR> __device__ inline float row_sum(float v, float *red) {
#pragma unroll
  for (int d = 1; d < (TPR < 64 ? TPR : 64); d <<= 1) v += __shfl_xor(v, d, 64);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) v += red[w];
  }
  return v;
}

// TPR threads a row, NV vectors of eight each
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(kThreads) void ln_fwd_kernel(LnArgs a) {
  __shared__ float red[kThreads / 64];
  constexpr int RPW = kThreads / TPR;
  const int t = threadIdx.x % TPR;
  const long long row = (long long)blockIdx.x * RPW + threadIdx.x / TPR;
  const bool live = row < a.M;
  const T *x = static_cast<const T *>(a.x) + (live ? row : 0) * a.ldx;
  float v[NV][8];
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8;
    row_load(x + c, a.N - c, v[i]);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) s += ((v[i][0] + v[i][1]) + (v[i][2] + v[i][3])) + ((v[i][4] + v[i][5]) + (v[i][6] + v[i][7]));
  const float mu = row_sum<TPR>(s, red) / (float)a.N;
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = c + e < a.N ? v[i][e] - mu : 0.f;
      v[i][e] = d;
      q += d * d;
    }
  }
  const float r = 1.f / sqrtf(row_sum<TPR>(q, red) / (float)a.N + a.eps);
  if (!live) return;
  T *y = static_cast<T *>(a.out) + row * a.ldo;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8, left = a.N - c;
    if (left <= 0) break;
    float g[8], b[8];
    if (a.gamma) row_load(a.gamma + c, left, g);
    if (a.beta) row_load(a.beta + c, left, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float o = v[i][e] * r;
      if (a.gamma) o *= g[e];
      if (a.beta) o += b[e];
      v[i][e] = o;
    }
    row_store(y + c, left, v[i]);
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
}

// rows that do not fit: a workgroup reads each three times (the second and third from L2)
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_fwd_long_kernel(LnArgs a) {
  __shared__ float red[kThreads / 64];
  const long long row = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + row * a.ldx;
  T *y = static_cast<T *>(a.out) + row * a.ldo;
  float s = 0.f, v[8];
  for (int c = threadIdx.x * 8; c < a.N; c += kThreads * 8) {
    row_load(x + c, a.N - c, v);
    s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  }
  const float mu = row_sum<kThreads>(s, red) / (float)a.N;
  float q = 0.f;
  for (int c = threadIdx.x * 8; c < a.N; c += kThreads * 8) {
    row_load(x + c, a.N - c, v);
    float p = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float d = c + e < a.N ? v[e] - mu : 0.f;
      p += d * d;
    }
    q += p;
  }
  const float r = 1.f / sqrtf(row_sum<kThreads>(q, red) / (float)a.N + a.eps);
  for (int c = threadIdx.x * 8; c < a.N; c += kThreads * 8) {
    float g[8], b[8];
    row_load(x + c, a.N - c, v);
    if (a.gamma) row_load(a.gamma + c, a.N - c, g);
    if (a.beta) row_load(a.beta + c, a.N - c, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float o = (v[e] - mu) * r;
      if (a.gamma) o *= g[e];
      if (a.beta) o += b[e];
      v[e] = o;
    }
    row_store(y + c, a.N - c, v);
  }
  if (threadIdx.x == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
}

// A workgroup takes rows blockIdx.x, + gridDim.x, ... (a row per TPR threads): its threads keep their columns, so dy xhat and dy are summed
// over its rows in registers.  The threads of other rows add theirs through LDS at the end.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(kThreads) void ln_bwd_kernel(LnArgs a) {
  constexpr int RPW = kThreads / TPR;
  __shared__ float red[kThreads / 64];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float sg[NV][8], sb[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sg[i][e] = sb[i][e] = 0.f;
  const long long step = (long long)gridDim.x * RPW;
  for (long long row0 = (long long)blockIdx.x * RPW; row0 < a.M; row0 += step) {
    const long long row = row0 + sub;
    const bool live = row < a.M;
    const long long rr = live ? row : 0;
    const T *x = static_cast<const T *>(a.x) + rr * a.ldx, *dy = static_cast<const T *>(a.dy) + rr * a.lddy;
    const float mu = a.mean[rr], r = a.rstd[rr];
    float g[NV][8], h[NV][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8, left = live ? a.N - c : 0;
      row_load(x + c, left, h[i]);
      row_load(dy + c, left, g[i]);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8, left = live ? a.N - c : 0;
      float w[8];
      if (a.gamma) row_load(a.gamma + c, left, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[i][e] = e < left ? (h[i][e] - mu) * r : 0.f;
        sg[i][e] += g[i][e] * h[i][e];
        sb[i][e] += g[i][e];
        if (a.gamma) g[i][e] *= w[e];
        s1 += g[i][e];
        s2 += g[i][e] * h[i][e];
      }
    }
    s1 = row_sum<TPR>(s1, red) / (float)a.N;
    s2 = row_sum<TPR>(s2, red) / (float)a.N;
    if (!live) continue;
    T *dx = static_cast<T *>(a.out) + row * a.ldo;
    const T *ad = static_cast<const T *>(a.addend) + row * a.lda;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (t + i * TPR) * 8, left = a.N - c;
      if (left <= 0) break;
      float o[8];
      if (a.addend) row_load(ad + c, left, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = r * (g[i][e] - s1 - h[i][e] * s2);
        o[e] = a.addend ? o[e] + d : d;
      }
      row_store(dx + c, left, o);
    }
  }
  if (!a.part) return;
  if constexpr (RPW > 1) {
    __shared__ float cols[RPW][TPR * 8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float (&m)[8] = half ? sb[i] : sg[i];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) cols[sub][t * 8 + e] = m[e];
        __syncthreads();
        if (sub == 0) {
#pragma unroll
          for (int k = 1; k < RPW; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) m[e] += cols[k][t * 8 + e];
        }
      }
    }
    if (sub != 0) return;
  }
  float *p = a.part + (size_t)blockIdx.x * 2 * a.N;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (t + i * TPR) * 8, left = a.N - c;
    if (left <= 0) break;
    row_store(p + c, left, sg[i]);
    row_store(p + a.N + c, left, sb[i]);
  }
}

// rows that do not fit: the sums of the rows first ...
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_bwd_rows_kernel(LnArgs a, float *sums) {
  __shared__ float red[kThreads / 64];
  const long long row = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + row * a.ldx, *dy = static_cast<const T *>(a.dy) + row * a.lddy;
  const float mu = a.mean[row], r = a.rstd[row];
  float s1 = 0.f, s2 = 0.f;
  for (int c = threadIdx.x * 8; c < a.N; c += kThreads * 8) {
    float h[8], g[8], w[8], p1 = 0.f, p2 = 0.f;
    row_load(x + c, a.N - c, h);
    row_load(dy + c, a.N - c, g);
    if (a.gamma) row_load(a.gamma + c, a.N - c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (a.gamma) g[e] *= w[e];
      p1 += g[e];
      p2 += c + e < a.N ? g[e] * ((h[e] - mu) * r) : 0.f;
    }
    s1 += p1; s2 += p2;
  }
  s1 = row_sum<kThreads>(s1, red) / (float)a.N;
  s2 = row_sum<kThreads>(s2, red) / (float)a.N;
  if (threadIdx.x == 0) { sums[2 * row] = s1; sums[2 * row + 1] = s2; }
}
// ... then, 2048 columns of a range of rows to a workgroup, the gradients
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_bwd_cols_kernel(LnArgs a, const float *sums) {
  const int c = (blockIdx.y * kThreads + threadIdx.x) * 8, left = a.N - c;
  if (left <= 0) return;
  float sg[8] = {}, sb[8] = {}, w[8];
  if (a.gamma) row_load(a.gamma + c, left, w);
  for (long long row = blockIdx.x; row < a.M; row += gridDim.x) {
    const float mu = a.mean[row], r = a.rstd[row], s1 = sums[2 * row], s2 = sums[2 * row + 1];
    float h[8], g[8], o[8];
    row_load(static_cast<const T *>(a.x) + row * a.ldx + c, left, h);
    row_load(static_cast<const T *>(a.dy) + row * a.lddy + c, left, g);
    if (a.addend) row_load(static_cast<const T *>(a.addend) + row * a.lda + c, left, o);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float xh = e < left ? (h[e] - mu) * r : 0.f;
      sg[e] += g[e] * xh;
      sb[e] += g[e];
      const float d = r * ((a.gamma ? g[e] * w[e] : g[e]) - s1 - xh * s2);
      o[e] = a.addend ? o[e] + d : d;
    }
    row_store(static_cast<T *>(a.out) + row * a.ldo + c, left, o);
  }
  if (!a.part) return;
  float *p = a.part + (size_t)blockIdx.x * 2 * a.N;
  row_store(p + c, left, sg);
  row_store(p + a.N + c, left, sb);
}

// columns [2][N] of `parts` parts, in float64: 64 columns to a workgroup, 16 ranges of parts, joined in order
__global__ __launch_bounds__(1024) void ln_params_kernel(const float *part, int parts, int N, float *dgamma, float *dbeta) {
  __shared__ double red[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
  double s = 0.;
  if (c < 2 * N)
    for (int p = k; p < parts; p += 16) s += (double)part[(size_t)p * 2 * N + c];
  red[k][threadIdx.x & 63] = s;
  __syncthreads();
  if (k != 0 || c >= 2 * N) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += red[i][threadIdx.x];
  float *out = c < N ? dgamma : dbeta;
  if (out) out[c < N ? c : c - N] = (float)s;
}

// threads a row and vectors a thread
struct Held { int tpr, nv; };
Held held_shape(int N) {
  Held h;
  h.tpr = N > 1024 ? 256 : 64;
  h.nv = 1;
  while (h.tpr * h.nv * 8 < N) h.nv *= 2;
  return h;
}
int bwd_parts(int64_t M, int N) {
  const int64_t rpw = N > kHeldCols ? 1 : kThreads / held_shape(N).tpr;
  return (int)std::max<int64_t>(1, std::min<int64_t>(512, (M + rpw - 1) / rpw));
}

template <typename T> int fwd(const LnArgs &a, hipStream_t st) {
  if (a.N > kHeldCols) {
    ln_fwd_long_kernel<T><<<dim3((unsigned)a.M), kThreads, 0, st>>>(a);
  } else {
    const Held h = held_shape(a.N);
    const dim3 grid((unsigned)((a.M + kThreads / h.tpr - 1) / (kThreads / h.tpr)));
    if (h.tpr == 64 && h.nv == 1) ln_fwd_kernel<T, 64, 1><<<grid, kThreads, 0, st>>>(a);
    else if (h.tpr == 64) ln_fwd_kernel<T, 64, 2><<<grid, kThreads, 0, st>>>(a);
    else if (h.nv == 1) ln_fwd_kernel<T, 256, 1><<<grid, kThreads, 0, st>>>(a);
    else if (h.nv == 2) ln_fwd_kernel<T, 256, 2><<<grid, kThreads, 0, st>>>(a);
    else ln_fwd_kernel<T, 256, 4><<<grid, kThreads, 0, st>>>(a);
  }
  RESIST_CHECK_LAUNCH("layernorm_fwd");
  return RESIST_OK;
}
template <typename T> int bwd(const LnArgs &a, int parts, float *sums, hipStream_t st) {
  if (a.N > kHeldCols) {
    ln_bwd_rows_kernel<T><<<dim3((unsigned)a.M), kThreads, 0, st>>>(a, sums);
    ln_bwd_cols_kernel<T><<<dim3(parts, (a.N + kThreads * 8 - 1) / (kThreads * 8)), kThreads, 0, st>>>(a, sums);
  } else {
    const Held h = held_shape(a.N);
    if (h.tpr == 64 && h.nv == 1) ln_bwd_kernel<T, 64, 1><<<parts, kThreads, 0, st>>>(a);
    else if (h.tpr == 64) ln_bwd_kernel<T, 64, 2><<<parts, kThreads, 0, st>>>(a);
    else if (h.nv == 1) ln_bwd_kernel<T, 256, 1><<<parts, kThreads, 0, st>>>(a);
    else if (h.nv == 2) ln_bwd_kernel<T, 256, 2><<<parts, kThreads, 0, st>>>(a);
    else ln_bwd_kernel<T, 256, 4><<<parts, kThreads, 0, st>>>(a);
  }
  RESIST_CHECK_LAUNCH("layernorm_bwd");
  return RESIST_OK;
}

}  // namespace

int64_t layernorm_workspace_floats(int64_t M, int N) {
  return (int64_t)bwd_parts(M, N) * 2 * N + (N > kHeldCols ? 2 * M : 0);
}

int layernorm_fwd(int dt, const LayerNorm &l, void *y, int64_t ldy, hipStream_t st) {
  if (l.M == 0) return RESIST_OK;
  LnArgs a{};
  a.x = l.x; a.out = y; a.gamma = l.gamma; a.beta = l.beta; a.mean = l.mean; a.rstd = l.rstd;
  a.M = l.M; a.N = l.N; a.ldx = l.ldx; a.ldo = ldy; a.eps = l.eps;
  prof::Scope sc("layernorm_fwd", 8. * l.M * l.N, 2. * l.M * l.N * esize(dt), st);
  return dt == DT_F32 ? fwd<float>(a, st) : fwd<__bf16>(a, st);
}

int layernorm_bwd(int dt, const LayerNorm &l, const void *dy, int64_t lddy, const void *addend, int64_t lda, void *dx, int64_t lddx,
                  float *dgamma, float *dbeta, float *work, hipStream_t st) {
  const bool params = dgamma || dbeta;
  if (l.M == 0) {
    if (dgamma) RESIST_TRY(fill_zero_f32(dgamma, l.N, st));
    if (dbeta) RESIST_TRY(fill_zero_f32(dbeta, l.N, st));
    return RESIST_OK;
  }
  const int parts = bwd_parts(l.M, l.N);
  LnArgs a{};
  a.x = l.x; a.dy = dy; a.addend = addend; a.out = dx; a.gamma = l.gamma; a.mean = l.mean; a.rstd = l.rstd;
  a.M = l.M; a.N = l.N; a.ldx = l.ldx; a.lddy = lddy; a.lda = lda; a.ldo = lddx;
  a.part = params ? work : nullptr;
  {
    prof::Scope sc("layernorm_bwd", 14. * l.M * l.N, (addend ? 4. : 3.) * l.M * l.N * esize(dt), st);
    float *sums = work + (size_t)parts * 2 * l.N;
    RESIST_TRY(dt == DT_F32 ? bwd<float>(a, parts, sums, st) : bwd<__bf16>(a, parts, sums, st));
  }
  if (params) {
    prof::Scope sc("layernorm_params", 0., (double)parts * 2 * l.N * 4, st);
    ln_params_kernel<<<(2 * l.N + 63) / 64, 1024, 0, st>>>(work, parts, l.N, dgamma, dbeta);
    RESIST_CHECK_LAUNCH("layernorm_params");
  }
  return RESIST_OK;
}

}  // namespace resist

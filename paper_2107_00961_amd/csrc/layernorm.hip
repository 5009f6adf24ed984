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
constexpr int threads_of(int tpr) { return tpr > kThreads ? tpr : kThreads; }   // of a workgroup whose rows take tpr threads each
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

// The sum over LANES neighbouring lanes (16, 32 or 64), in every one of them, on the vector unit alone (a shuffle goes through LDS): of lanes one and
// two apart, of the mirrored halves of eight and sixteen, of rows of sixteen, of halves of the wave.
template <int LANES> __device__ inline float lanes_sum(float v) {
  auto moved = [&](auto ctrl) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true)); };
  v += moved(std::integral_constant<int, 0xb1>{});    // quad_perm 1 0 3 2
  v += moved(std::integral_constant<int, 0x4e>{});    // quad_perm 2 3 0 1
  v += moved(std::integral_constant<int, 0x141>{});   // row_half_mirror
  v += moved(std::integral_constant<int, 0x140>{});   // row_mirror
  // v in both operands swaps every second row (half) of one with the row before it of the other: one gets each pair's first row twice, the other
  // its second.
  if constexpr (LANES > 16) {
    const unsigned x = __builtin_bit_cast(unsigned, v);
    const auto p = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const unsigned first = p[0], second = p[1];   // (a bit cast of a vector's element itself takes the first one)
    v = __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
  }
  if constexpr (LANES > 32) {
    const unsigned x = __builtin_bit_cast(unsigned, v);
    const auto p = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const unsigned first = p[0], second = p[1];   // (a bit cast of a vector's element itself takes the first one)
    v = __builtin_bit_cast(float, first) + __builtin_bit_cast(float, second);
  }
  return v;
}
// The sums over the TPR threads of a row.  red: [2][waves of the workgroup], where a row is more than a wave's; `turn` alternates from call to call, so
// that one barrier is enough: who writes a turn's words has met everyone since they were read.
template <int TPR> __device__ inline void row_sums(float &a, float &b, float2 (*red)[8], int turn) {
  a = lanes_sum<(TPR < 64 ? TPR : 64)>(a);
  b = lanes_sum<(TPR < 64 ? TPR : 64)>(b);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) red[turn][threadIdx.x >> 6] = float2{a, b};
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) {
      const float2 t = red[turn][threadIdx.x / TPR * (TPR / 64) + w];
      a += t.x;
      b += t.y;
    }
  }
}
template <int TPR> __device__ inline float row_sum(float v, float2 (*red)[8], int turn) {
  float none = 0.f;
  row_sums<TPR>(v, none, red, turn);
  return v;
}

// Where a thread's eight elements from column c on are taken from: the last vector of a row ends with the row, so that all of them are whole (of rows of
// eight or more), and its first `skip` elements are another thread's too, who counts them (both store the same).  All eight are skipped past the row's
// end.  16384 x 1100 bf16, with the last vector's elements one by one: forward 26 us, backward 54; so 23 and 39.
struct Place {
  int c, skip, count;
  __device__ inline Place(int at, int N) : c(min(at, max(N - 8, 0))), skip(at - c), count(min(N, 8)) {}
  __device__ inline bool counts(int e) const { return (unsigned)(e - skip) < (unsigned)count; }
};

// TPR threads a row, NV vectors of eight each.  Bound by memory: 16384 x 4096 bf16 46 us (5.8 TB/s; a copy of 1 GiB reaches 5.1), fp32 109 us (4.9),
// 5003 x 1001 fp32, whose rows start anywhere, 9.8 us (4.1); one row of 4096 3.3 us, a launch.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(threads_of(TPR)) void ln_fwd_kernel(LnArgs a) {
  __shared__ float2 red[2][8];
  constexpr int RPW = threads_of(TPR) / TPR;
  const int t = threadIdx.x % TPR;
  const long long row = (long long)blockIdx.x * RPW + threadIdx.x / TPR;
  const bool live = row < a.M;
  const T *x = static_cast<const T *>(a.x) + (live ? row : 0) * a.ldx;
  float v[NV][8];
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place p((t + i * TPR) * 8, a.N);
    row_load(x + p.c, a.N - p.c, v[i]);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place p((t + i * TPR) * 8, a.N);
    float m[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = p.counts(e) ? v[i][e] : 0.f;
    s += ((m[0] + m[1]) + (m[2] + m[3])) + ((m[4] + m[5]) + (m[6] + m[7]));
  }
  const float mu = row_sum<TPR>(s, red, 0) / (float)a.N;
  float q = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place p((t + i * TPR) * 8, a.N);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[i][e] -= mu;
      q += p.counts(e) ? v[i][e] * v[i][e] : 0.f;
    }
  }
  const float r = 1.f / sqrtf(row_sum<TPR>(q, red, 1) / (float)a.N + a.eps);
  if (!live) return;
  T *y = static_cast<T *>(a.out) + row * a.ldo;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place p((t + i * TPR) * 8, a.N);
    const int left = a.N - p.c;
    if (p.skip >= 8) break;
    float g[8], b[8];
    if (a.gamma) row_load(a.gamma + p.c, left, g);
    if (a.beta) row_load(a.beta + p.c, left, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float o = v[i][e] * r;
      if (a.gamma) o *= g[e];
      if (a.beta) o += b[e];
      v[i][e] = o;
    }
    row_store(y + p.c, left, v[i]);
  }
  if (t == 0) {
    if (a.mean) a.mean[row] = mu;
    if (a.rstd) a.rstd[row] = r;
  }
}

// rows that do not fit: a workgroup reads each three times (the second and third from a cache).  4096 x 16384 bf16 77 us (3.5 TB/s of what is read once)
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_fwd_long_kernel(LnArgs a) {
  __shared__ float2 red[2][8];
  const long long row = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + row * a.ldx;
  T *y = static_cast<T *>(a.out) + row * a.ldo;
  float s = 0.f, v[8];
  for (int c = threadIdx.x * 8; c < a.N; c += kThreads * 8) {
    row_load(x + c, a.N - c, v);
    s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
  }
  const float mu = row_sum<kThreads>(s, red, 0) / (float)a.N;
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
  const float r = 1.f / sqrtf(row_sum<kThreads>(q, red, 1) / (float)a.N + a.eps);
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
// over its rows in registers.  The threads of other rows add theirs through LDS at the end.  Bound by memory, of few rows by the trips to it, a
// row's for each turn.  With ln_params_kernel, 16384 x 4096 bf16 88 ... 98 us whether or not with an
// addend (5.5 TB/s with), 16384 x 2048 43 us, 16384 x 1024 27, 777 x 513 fp32 9.9.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(threads_of(TPR)) void ln_bwd_kernel(LnArgs a) {
  constexpr int RPW = threads_of(TPR) / TPR;
  __shared__ float2 red[2][8];
  const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  float sg[NV][8], sb[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) sg[i][e] = sb[i][e] = 0.f;
  const long long step = (long long)gridDim.x * RPW;
  // a row's operands are asked for while the one before it is worked on
  Raw8<T> rx[NV], rdy[NV], rad[NV];
  float mu, r;
  auto ask = [&](long long row) {
    const bool live = row < a.M;
    const long long rr = live ? row : 0;
    const T *x = static_cast<const T *>(a.x) + rr * a.ldx, *dy = static_cast<const T *>(a.dy) + rr * a.lddy, *ad = static_cast<const T *>(a.addend) + rr * a.lda;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = Place((t + i * TPR) * 8, a.N).c, left = live ? a.N - c : 0;
      raw_load(x + c, left, rx[i]);
      raw_load(dy + c, left, rdy[i]);
      if (a.addend) raw_load(ad + c, left, rad[i]);
    }
    mu = live ? a.mean[rr] : 0.f;
    r = live ? a.rstd[rr] : 0.f;
  };
  float w[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = Place((t + i * TPR) * 8, a.N).c;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[i][e] = 1.f;
    if (a.gamma) row_load(a.gamma + c, a.N - c, w[i]);
  }
  const bool full = a.N == TPR * NV * 8;   // no thread without elements, or with another's: 16384 x 4096 in bf16 99 -> 88 us
  int turn = 0;
  ask((long long)blockIdx.x * RPW + sub);
  for (long long row0 = (long long)blockIdx.x * RPW; row0 < a.M; row0 += step) {
    const long long row = row0 + sub;
    const bool live = row < a.M;
    const float rs = r;
    float g[NV][8], h[NV][8], s1 = 0.f, s2 = 0.f;
    Raw8<T> add[NV];
    auto terms = [&](auto masked) {
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const Place p((t + i * TPR) * 8, a.N);
        widen(rx[i], h[i]);
        widen(rdy[i], g[i]);
        add[i] = rad[i];
        // where dx takes the addend's place, another thread may store into a vector that overlaps this one once the row's sums are joined
        if (decltype(masked)::value && a.addend) arrived(add[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          h[i][e] = (h[i][e] - mu) * rs;
          sg[i][e] += g[i][e] * h[i][e];
          sb[i][e] += g[i][e];
          g[i][e] *= w[i][e];
          const bool counts = !decltype(masked)::value || p.counts(e);
          s1 += counts ? g[i][e] : 0.f;
          s2 += counts ? g[i][e] * h[i][e] : 0.f;
        }
      }
    };
    if (full) terms(std::false_type{});
    else terms(std::true_type{});
    ask(row + step);
    row_sums<TPR>(s1, s2, red, turn);
    turn ^= 1;
    s1 /= (float)a.N;
    s2 /= (float)a.N;
    if (!live) continue;
    T *dx = static_cast<T *>(a.out) + row * a.ldo;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Place p((t + i * TPR) * 8, a.N);
      if (p.skip >= 8) break;
      float o[8];
      if (a.addend) widen(add[i], o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = rs * (g[i][e] - s1 - h[i][e] * s2);
        o[e] = a.addend ? o[e] + d : d;
      }
      row_store(dx + p.c, a.N - p.c, o);
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
  float *part = a.part + (size_t)blockIdx.x * 2 * a.N;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const Place p((t + i * TPR) * 8, a.N);
    if (p.skip == 0 && p.count == 8) {
      row_store(part + p.c, 8, sg[i]);
      row_store(part + a.N + p.c, 8, sb[i]);
      continue;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (p.counts(e)) {
        part[p.c + e] = sg[i][e];
        part[a.N + p.c + e] = sb[i][e];
      }
  }
}

// rows that do not fit: the sums of the rows first (4096 x 16384 bf16, all three kernels, 158 us) ...
template <typename T>
__global__ __launch_bounds__(kThreads) void ln_bwd_rows_kernel(LnArgs a, float *sums) {
  __shared__ float2 red[2][8];
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
  row_sums<kThreads>(s1, s2, red, 0);
  s1 /= (float)a.N;
  s2 /= (float)a.N;
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

// Columns [2][N] of `parts` parts, in float64: 64 columns to a workgroup, 16 ranges of parts, joined in order.  A part was written on any XCD, so that each
// trip to it takes microseconds: all of a thread's are asked for at once (512 parts of 512 columns: 11 us
// with eight at a time, 5 with 32; of 64 parts eight are 2.4 us, 32 with most of them past the end 5).
__global__ __launch_bounds__(1024) void ln_params_kernel(const float *part, int parts, int N, float *dgamma, float *dbeta) {
  __shared__ double red[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
  double s = 0.;
  if (c < 2 * N) s = parts > 128 ? parts_sum<32>(part + c, (size_t)2 * N, k, 16, parts) : parts_sum<8>(part + c, (size_t)2 * N, k, 16, parts);
  red[k][threadIdx.x & 63] = s;
  __syncthreads();
  if (k != 0 || c >= 2 * N) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) s += red[i][threadIdx.x];
  float *out = c < N ? dgamma : dbeta;
  if (out) out[c < N ? c : c - N] = (float)s;
}

// Threads a row and vectors a thread: as few threads as hold a row in one or two vectors each, so that a wave or a workgroup takes several short rows at
// once (16384 x 2048 bf16 in 128 threads or 256: forward 26 | 30 us, backward 43 | 50; in 64, four vectors each: 26 and 61).
struct Held { int tpr, nv; };
Held held_shape(int N) {
  if (N <= 128) return Held{16, 1};
  if (N <= 256) return Held{32, 1};
  if (N <= 512) return Held{64, 1};
  if (N <= 1024) return Held{64, 2};
  if (N <= 2048) return Held{128, 2};
  return N <= 4096 ? Held{256, 2} : Held{512, 2};
}
// Workgroups of the backward pass, each of which leaves a part of the columns' sums: two a CU (one where it is 512 threads) where there are rows enough for
// two or more apiece (four where a part is long); with up to 64 rows (or groups of them) a row each, which is quicker than a second turn.
// us, M x N, number of workgroups in brackets, the chosen one first:
//   777x513 fp32 (98) 10.2, (192) 13.6, (64) 12.6     2000x300 bf16 (250) 11.0, (500) 10.3, (128) 11.6
//   1000x4096 fp32 (250) 21.3, (500) 21.6, (1000) 28.2     4096x1024 bf16 (512) 14.4, (1024) 20.2, (256) 14.9     16384x4096 bf16 (512) 88, (1024) 100, (256) 134
//   4096x8192 bf16 (256) 50, (512) 55, (192) 58     16384x2048 bf16 (512) 43, (256) 57, (1024) 48     4000x1100 bf16 (512) 21.5, (256) 27, (768) 23
int bwd_parts(int64_t M, int N) {
  const Held h = held_shape(N);
  const int64_t rpw = N > kHeldCols ? 1 : threads_of(h.tpr) / h.tpr, turns = (M + rpw - 1) / rpw, each = N > 2048 ? 4 : 2;
  const int64_t most = h.tpr == 512 && N <= kHeldCols ? 256 : 512;
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, std::max<int64_t>(std::min<int64_t>(64, turns), (turns + each - 1) / each)));
}
// call(kernel<T, TPR, NV>, threads) for the shape of N
#define LN_HELD(kernel, T, N, call)                                               \
  do {                                                                            \
    const Held h = held_shape(N);                                                 \
    if (h.tpr == 16) call((kernel<T, 16, 1>), 16);                                \
    else if (h.tpr == 32) call((kernel<T, 32, 1>), 32);                           \
    else if (h.tpr == 64 && h.nv == 1) call((kernel<T, 64, 1>), 64);              \
    else if (h.tpr == 64) call((kernel<T, 64, 2>), 64);                           \
    else if (h.tpr == 128) call((kernel<T, 128, 2>), 128);                        \
    else if (h.tpr == 256) call((kernel<T, 256, 2>), 256);                        \
    else call((kernel<T, 512, 2>), 512);                                          \
  } while (0)

// Rows that one launch takes where a workgroup of `threads` takes `rows`: with 2^32 threads or more it would count them modulo 2^32, and
// leave rows out without an error.
long long rows_a_launch(int threads, int rows) { return (long long)(kMaxThreads / threads) * rows; }

template <typename T> int fwd(const LnArgs &all, hipStream_t st) {
  const int tpr = all.N > kHeldCols ? kThreads : held_shape(all.N).tpr, rpw = threads_of(tpr) / tpr;
  const long long most = rows_a_launch(threads_of(tpr), rpw);
  for (long long at = 0; at < all.M; at += most) {
    LnArgs a = all;
    a.M = std::min(most, all.M - at);
    a.x = static_cast<const T *>(all.x) + at * all.ldx;
    a.out = static_cast<T *>(all.out) + at * all.ldo;
    if (all.mean) a.mean = all.mean + at;
    if (all.rstd) a.rstd = all.rstd + at;
    const unsigned wgs = (unsigned)((a.M + rpw - 1) / rpw);
    if (a.N > kHeldCols) {
      ln_fwd_long_kernel<T><<<wgs, kThreads, 0, st>>>(a);
    } else {
#define FWD(k, tpr) k<<<wgs, threads_of(tpr), 0, st>>>(a)
      LN_HELD(ln_fwd_kernel, T, a.N, FWD);
#undef FWD
    }
    RESIST_CHECK_LAUNCH("layernorm_fwd");
  }
  return RESIST_OK;
}
template <typename T> int bwd(const LnArgs &a, int parts, float *sums, hipStream_t st) {
  if (a.N > kHeldCols) {
    const long long most = rows_a_launch(kThreads, 1);
    for (long long at = 0; at < a.M; at += most) {
      LnArgs b = a;
      b.x = static_cast<const T *>(a.x) + at * a.ldx;
      b.dy = static_cast<const T *>(a.dy) + at * a.lddy;
      b.mean = a.mean + at;
      b.rstd = a.rstd + at;
      ln_bwd_rows_kernel<T><<<(unsigned)std::min(most, a.M - at), kThreads, 0, st>>>(b, sums + 2 * at);
    }
    ln_bwd_cols_kernel<T><<<dim3(parts, (a.N + kThreads * 8 - 1) / (kThreads * 8)), kThreads, 0, st>>>(a, sums);
  } else {
#define BWD(k, tpr) k<<<parts, threads_of(tpr), 0, st>>>(a)
    LN_HELD(ln_bwd_kernel, T, a.N, BWD);
#undef BWD
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

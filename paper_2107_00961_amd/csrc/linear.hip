// Dense layers on rows of activations: x [M][K], w [N][K].
//   forward          z = x w' + bias,  y = residual + drop(a(z))
//   data gradient    dx = a'(z) drop(dz w)        (z, a, drop: of the layer that produced x)
//   weight gradient  dw = dz' x,  db = column sums of dz
// Products on the matrix cores, sums in fp32, one rounding where a result is stored.
#include <algorithm>

#include "conv_tile.h"
#include "dense.h"

namespace resist {
namespace {

constexpr int kThreads = 256;

// what becomes of a product on its way to memory
struct Epilogue {
  void *out;
  const float *bias;        // forward
  void *z_out;              // forward, optional
  const void *res;          // forward, optional
  const void *z_in;         // data gradient, optional
  long long ldo, ldz, ldr;
  Dropout d;
  int act, words;
};

// out(i, j) = sum over r of a(i, r) b(j, r); element (i, r) is a[i * ai + r * ar]
struct GemmArgs {
  const void *a, *b;
  long long ai, ar, bj, br;
  long long I;
  int J, tiles_j;
  long long R;
  Epilogue e;
};

// element (i, j)
template <typename T>
__device__ inline void finish(const Epilogue &e, long long i, int j, float v, u64 base) {
  float t[1] = {v};
  if (e.bias) t[0] += e.bias[j];
  if (e.z_out) static_cast<T *>(e.z_out)[i * e.ldz + j] = (T)t[0];
  if (!e.z_in) activate<1>(t, e.act);
  if (e.d.rng) {
    const u64 w = splitmix(base + ((u64)i * (unsigned)e.words + (unsigned)(j >> 1)) * kGolden);
    t[0] = (unsigned)(j & 1 ? w >> 32 : w) < e.d.thr ? 0.f : t[0] * e.d.scale;
  }
  if (e.z_in) {
    const float z[1] = {(float)static_cast<const T *>(e.z_in)[i * e.ldz + j]};
    times_slope<1>(t, z, e.act);
  }
  if (e.res) t[0] += (float)static_cast<const T *>(e.res)[i * e.ldr + j];
  static_cast<T *>(e.out)[i * e.ldo + j] = (T)t[0];
}

// Any strides: 64x64 outputs to a workgroup, 32 steps of the reduction staged at a time, an element per load.  AR, BR: whether the
// reduction index is the contiguous one.  T: operands, O: results.
template <typename T, typename O, bool AR, bool BR>
__global__ __launch_bounds__(kThreads) void gemm_any_kernel(GemmArgs g) {
  using E = Elem<T>;
  constexpr int BK = 32, PITCH = BK + E::VEC;
  __shared__ __attribute__((aligned(16))) T As[64][PITCH], Bs[64][PITCH];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const int bid = blockIdx.x;
  const long long i0 = (long long)(bid / g.tiles_j) * 64;
  const int j0 = bid % g.tiles_j * 64;
  const T *a = static_cast<const T *>(g.a), *b = static_cast<const T *>(g.b);
  f32x16 acc = {};
  for (long long r0 = 0; r0 < g.R; r0 += BK) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = AR ? tid >> 2 : tid & 63, r = AR ? (tid & 3) * 8 + e : (tid >> 6) * 8 + e;
      As[i][r] = i0 + i < g.I && r0 + r < g.R ? a[(i0 + i) * g.ai + (r0 + r) * g.ar] : (T)0.f;
      const int j = BR ? tid >> 2 : tid & 63, q = BR ? (tid & 3) * 8 + e : (tid >> 6) * 8 + e;
      Bs[j][q] = j0 + j < g.J && r0 + q < g.R ? b[(j0 + j) * g.bj + (r0 + q) * g.br] : (T)0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < BK; k += 2 * E::VEC) {
      const f32x4 fa = *reinterpret_cast<const f32x4 *>(&As[wm * 32 + (lane & 31)][k + (lane >> 5) * E::VEC]);
      const f32x4 fb = *reinterpret_cast<const f32x4 *>(&Bs[wn * 32 + (lane & 31)][k + (lane >> 5) * E::VEC]);
      E::mma(acc, fa, fb);
    }
    __syncthreads();
  }
  const u64 base = g.e.d.rng ? dropout_base(g.e.d.rng) : 0;
  const int j = j0 + wn * 32 + (lane & 31);
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const long long i = i0 + wm * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3);
    if (i < g.I && j < g.J) finish<O>(g.e, i, j, acc[e], base);
  }
}

// db: 64 columns of dz to a workgroup, four ranges of rows
template <typename T>
__global__ __launch_bounds__(kThreads) void col_sum_kernel(const T *dz, long long M, int N, long long ld, float *db) {
  __shared__ double red[4][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
  double s = 0.;
  if (c < N)
    for (long long m = k; m < M; m += 4) s += (double)(float)dz[m * ld + c];
  red[k][threadIdx.x & 63] = s;
  __syncthreads();
  if (k == 0 && c < N) db[c] = (float)(((red[0][threadIdx.x] + red[1][threadIdx.x]) + red[2][threadIdx.x]) + red[3][threadIdx.x]);
}

template <typename T, typename O, bool AR, bool BR> int gemm_any(GemmArgs &g, hipStream_t st) {
  g.tiles_j = (g.J + 63) / 64;
  const long long tiles = (g.I + 63) / 64 * g.tiles_j;
  if (tiles > 0x7fffffffLL) return set_error(RESIST_ESHAPE, "linear: too many outputs");
  gemm_any_kernel<T, O, AR, BR><<<(unsigned)tiles, kThreads, 0, st>>>(g);
  RESIST_CHECK_LAUNCH("linear");
  return RESIST_OK;
}

}  // namespace

int64_t linear_workspace(const LinearShape &s, int dt, int op) { (void)s; (void)dt; (void)op; return 0; }

int linear_fwd(const LinearShape &s, int dt, const void *x, const void *w, const LinearEpilogue &le, void *y, void *, hipStream_t st) {
  if (s.M == 0) return RESIST_OK;
  GemmArgs g{};
  g.a = x; g.ai = s.ldx; g.ar = 1; g.I = s.M;
  g.b = w; g.bj = s.K; g.br = 1; g.J = s.N; g.R = s.K;
  g.e.out = y; g.e.ldo = s.ldy; g.e.bias = le.bias; g.e.z_out = le.z; g.e.ldz = le.ldz; g.e.res = le.residual; g.e.ldr = le.ldr;
  g.e.act = le.act; g.e.d = make_dropout(le.drop); g.e.words = (s.N + 1) / 2;
  prof::Scope sc("linear_fwd", 2. * s.M * s.N * s.K, ((double)s.M * s.K + (double)s.N * s.K + (double)s.M * s.N) * esize(dt), st);
  return dt == DT_F32 ? gemm_any<float, float, true, true>(g, st) : gemm_any<__bf16, __bf16, true, true>(g, st);
}

int linear_dgrad(const LinearShape &s, int dt, const void *dz, const void *w, const LinearThrough &lt, void *dx, void *, hipStream_t st) {
  if (s.M == 0) return RESIST_OK;
  GemmArgs g{};
  g.a = dz; g.ai = s.ldy; g.ar = 1; g.I = s.M;
  g.b = w; g.bj = 1; g.br = s.K; g.J = s.K; g.R = s.N;
  g.e.out = dx; g.e.ldo = s.ldx; g.e.z_in = lt.act == RESIST_ACT_NONE ? nullptr : lt.z; g.e.ldz = lt.ldz; g.e.act = lt.act;
  g.e.d = make_dropout(lt.drop); g.e.words = (s.K + 1) / 2;
  prof::Scope sc("linear_dgrad", 2. * s.M * s.N * s.K, ((double)s.M * s.K + (double)s.N * s.K + (double)s.M * s.N) * esize(dt), st);
  return dt == DT_F32 ? gemm_any<float, float, true, false>(g, st) : gemm_any<__bf16, __bf16, true, false>(g, st);
}

int linear_wgrad(const LinearShape &s, int dt, const void *dz, const void *x, float *dw, float *db, void *, hipStream_t st) {
  GemmArgs g{};
  g.a = dz; g.ai = 1; g.ar = s.ldy; g.I = s.N;
  g.b = x; g.bj = 1; g.br = s.ldx; g.J = s.K; g.R = s.M;
  g.e.out = dw; g.e.ldo = s.K;
  if (dw) {
    prof::Scope sc("linear_wgrad", 2. * s.M * s.N * s.K, ((double)s.M * s.K + (double)s.M * s.N) * esize(dt) + 4. * s.N * s.K, st);
    RESIST_TRY((dt == DT_F32 ? gemm_any<float, float, false, false>(g, st) : gemm_any<__bf16, float, false, false>(g, st)));
  }
  if (!db) return RESIST_OK;
  prof::Scope sc("linear_bias", 0., (double)s.M * s.N * esize(dt), st);
  if (dt == DT_F32) col_sum_kernel<float><<<(s.N + 63) / 64, kThreads, 0, st>>>(static_cast<const float *>(dz), s.M, s.N, s.ldy, db);
  else col_sum_kernel<__bf16><<<(s.N + 63) / 64, kThreads, 0, st>>>(static_cast<const __bf16 *>(dz), s.M, s.N, s.ldy, db);
  RESIST_CHECK_LAUNCH("linear_bias");
  return RESIST_OK;
}

}  // namespace resist

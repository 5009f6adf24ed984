// Dropout whose mask is a function of {seed, offset} and position (dense.h), so that nothing but the tensor itself is read or stored:
//   forward   y  = [residual +] kept ? x / (1 - p) : 0
//   backward  dx = a'(z) * (kept ? dy / (1 - p) : 0)      a: the activation in front of the dropout, z: what it was applied to
// A thread takes eight consecutive elements of a row: four words of the sequence, which are two 64-bit products each.  Bound by memory: 16384 x 4096
// bf16 51 us, with a residual 74 ... 77 (5.2 TB/s), fp32 137 (5.9); in bf16 through GELU's gradient, where the arithmetic shows, 91 us (4.4 TB/s).
#include <algorithm>

#include "conv_tile.h"
#include "dense.h"

namespace resist {
namespace {

constexpr int kThreads = 256;

struct DropArgs {
  const void *x, *res, *z;
  void *out;
  long long M, ldx, ldr, ldz, ldo, units;   // units: vectors of eight, M * nvec
  int N, nvec, words, act;                   // words a row
  FastDiv div;                                // by nvec
  Dropout d;
};

template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(DropArgs a) {
  const u64 base = a.d.rng ? dropout_base(a.d.rng) : 0;
  for (long long first = (long long)blockIdx.x * kThreads; first < a.units; first += (long long)gridDim.x * kThreads) {
    const long long row0 = first / a.nvec;                           // the same for all threads
    const int rest = (int)(first - row0 * a.nvec) + (int)threadIdx.x;
    const int r = fdiv(rest, a.div), vec = rest - r * a.nvec;
    const long long row = row0 + r;
    if (row >= a.M) break;
    const int c = vec * 8, left = a.N - c;
    float v[8], o[8];
    row_load(static_cast<const T *>(a.x) + row * a.ldx + c, left, v);
    if (a.res) row_load(static_cast<const T *>(a.res) + row * a.ldr + c, left, o);
    if (a.z) row_load(static_cast<const T *>(a.z) + row * a.ldz + c, left, o);
    if (a.d.rng) dropout8(base + ((u64)row * (unsigned)a.words + (unsigned)(c >> 1)) * kGolden, a.d.thr, a.d.scale, v);
    if (a.z) times_slope(v, o, a.act);
    if (a.res) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += o[e];
    }
    row_store(static_cast<T *>(a.out) + row * a.ldo + c, left, v);
  }
}

}  // namespace

int dropout(int dt, int64_t M, int N, const void *x, int64_t ldx, const void *res, int64_t ldr, int act, const void *z, int64_t ldz,
            const DropSpec &d, void *out, int64_t ldo, hipStream_t st) {
  if (M == 0) return RESIST_OK;
  DropArgs a{};
  a.x = x; a.res = res; a.z = act == RESIST_ACT_NONE ? nullptr : z; a.out = out;
  a.M = M; a.N = N; a.ldx = ldx; a.ldr = ldr; a.ldz = ldz; a.ldo = ldo;
  a.nvec = (N + 7) / 8; a.words = (N + 1) / 2; a.units = M * a.nvec; a.act = act;
  a.div = make_fastdiv((unsigned)a.nvec);
  a.d = make_dropout(d);
  const long long wgs = std::min<long long>((a.units + kThreads - 1) / kThreads, 1 << 20);
  prof::Scope sc("dropout", 2. * M * N, (2. + (res != nullptr) + (a.z != nullptr)) * M * N * esize(dt), st);
  if (dt == DT_F32) dropout_kernel<float><<<(unsigned)wgs, kThreads, 0, st>>>(a);
  else dropout_kernel<__bf16><<<(unsigned)wgs, kThreads, 0, st>>>(a);
  RESIST_CHECK_LAUNCH("dropout");
  return RESIST_OK;
}

}  // namespace resist

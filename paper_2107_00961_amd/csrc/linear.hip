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

// ---- bf16 operands, tiled -------------------------------------------------------------------------------------------
// Operand tiles go from memory straight into LDS (16 bytes a lane, 1 KB a wave and instruction, in lane order), STAGES deep, and from there
// in fragments to the matrix cores.  Four waves, a quarter of the BM x BN tile each: the larger a wave's share, the fewer times a
// staged element is read from LDS (256x256: 1024 clocks of reading and 512 of arriving for 2048 of products).
// Layout in LDS.  Lane order leaves no room for padding, so what keeps rows off each other's banks is which 16-byte piece a lane asks for:
//   reduction contiguous (R): a row is an index i, BK values of r: piece c of row i lies at c ^ f(i), f = i & 7 (BK 64, 128 bytes a row),
//     (i >> 1) & 3 (BK 32, two rows to 128 bytes): eight consecutive rows' pieces c fill 128 bytes;
//   other index contiguous: a row is an r, BM values of i: piece c of row r lies at c ^ 4 (r & 3): the four rows of a transpose
//     read, 64 bytes each, fill 256 bytes.
// Bounds: an operand's descriptor starts at the tile and ends with the operand (rows past it, and steps past it, come as zeros); its
// contiguous axis is a multiple of eight where it is the reduction (a tail's pieces are not asked for) and may end in a piece where it is
// not (what a tile has past its last column goes into outputs that are not stored).
template <bool R, int B, int BK> struct Stage {
  static constexpr int kBytes = B * BK * 2, kLoads = kBytes / 4096;   // a wave's instructions
  static constexpr int kRow = R ? BK * 2 : B * 2, kPieces = kRow / 16, kRows = 1024 / kRow;   // rows an instruction
  // row and piece of the tile that lane `l` of wave `w` asks for with instruction p
  __device__ static inline int row(int p, int w, int l) { return (p * 4 + w) * kRows + l / kPieces; }
  __device__ static inline int piece(int r, int l) {
    const int f = R ? (BK == 64 ? r & 7 : (r >> 1) & 3) : (r & 3) << 2;
    return (l % kPieces) ^ f;
  }
};

struct TileArgs {
  const __bf16 *a, *b;
  long long lda, ldb;       // elements between rows (of i, or of r)
  long long I, R;
  int J, tiles_i, tiles_j, group;
  int splits;
  long long per_split;      // steps of the reduction, a multiple of the tile's
  float *part;              // [splits][I][J] where the reduction is split
  Epilogue e;
};

// eight outputs of a row.  bias: of their columns; side: what the epilogue reads beside them, z (data gradient) or the residual (forward)
template <typename O>
__device__ inline void finish8(const Epilogue &e, long long i, int j, int left, float (&v)[8], const float (&bias)[8], const Raw8<O> &side, u64 base) {
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] += bias[k];
  if (e.z_out) row_store(static_cast<O *>(e.z_out) + i * e.ldz + j, left, v);
  if (!e.z_in) activate(v, e.act);
  if (e.d.rng) dropout8(base, (u64)i * (unsigned)e.words + (unsigned)(j >> 1), e.d.thr, e.d.scale, v);
  if (e.z_in || e.res) {
    float s[8];
    widen(side, s);
    if (e.z_in) {
      times_slope(v, s, e.act);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += s[k];
    }
  }
  row_store(static_cast<O *>(e.out) + i * e.ldo + j, left, v);
}
template <typename O> __device__ inline const O *side_of(const Epilogue &e, long long &ld) {
  ld = e.z_in ? e.ldz : e.ldr;
  return static_cast<const O *>(e.z_in ? e.z_in : e.res);
}
__device__ inline void bias_of(const Epilogue &e, int j, int left, float (&b)[8]) {
#pragma unroll
  for (int k = 0; k < 8; ++k) b[k] = 0.f;
  if (e.bias) row_load(e.bias + j, left, b);
}

// 16 bytes a lane from a buffer to LDS at `to` and on, in lane order.  Written out because the compiler, which sees that LDS is written, waits for
// all transfers before the next read of any of it; what is waited for, and where, is wait_and_meet's.
__device__ inline void transfer(__amdgpu_buffer_rsrc_t r, unsigned off, unsigned to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(r), "s"(to) : "memory");
}
template <int N> __device__ inline void wait_and_meet() {   // at most N of this wave's transfers to LDS under way, all of its reads done
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// the tile's place: `group` rows of tiles are walked column by column, an XCD's workgroups one after the other
__device__ inline void tile_of(int bid, int tiles_i, int tiles_j, int group, int &ti, int &tj) {
  const int per = group * tiles_j, g = bid / per, rest = bid - g * per;
  const int rows = min(group, tiles_i - g * group);
  tj = rest / rows;
  ti = g * group + rest - tj * rows;
}

template <typename O, bool AR, bool BR, int BM, int BN, int BK, int STAGES, int WGS>
__global__ __launch_bounds__(kThreads, WGS) void gemm_tile_kernel(TileArgs g) {
  using SA = Stage<AR, BM, BK>;
  using SB = Stage<BR, BN, BK>;
  constexpr int WTM = BM / 2, WTN = BN / 2, TM = WTM / 32, TN = WTN / 32, NK = BK / 16;
  constexpr int kStage = SA::kBytes + SB::kBytes, kLoads = SA::kLoads + SB::kLoads;
  constexpr int kPitch = WTN * 4 + 16, kOut = 4 * 2 * 32 * kPitch;
  static_assert(STAGES >= 2, "stages");
  static_assert(TM <= 4, "tile");
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * kStage > kOut ? STAGES * kStage : kOut];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  int ti, tj, bid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int split = bid / (g.tiles_i * g.tiles_j);
  tile_of(bid - split * g.tiles_i * g.tiles_j, g.tiles_i, g.tiles_j, g.group, ti, tj);
  const long long i0 = (long long)ti * BM, rbeg = split * g.per_split, rend = min(g.R, rbeg + g.per_split);
  const int j0 = tj * BN;
  const int steps = (int)((rend - rbeg + BK - 1) / BK);

  // ---- operands to LDS.  left: bytes from the tile's current corner to the operand's end
  const char *pa = reinterpret_cast<const char *>(g.a + (AR ? i0 * g.lda + rbeg : rbeg * g.lda + i0));
  const char *pb = reinterpret_cast<const char *>(g.b + (BR ? (long long)j0 * g.ldb + rbeg : rbeg * g.ldb + j0));
  long long left_a = AR ? ((g.I - i0 - 1) * g.lda + (rend - rbeg)) * 2 : ((rend - rbeg - 1) * g.lda + (g.I - i0 + 7) / 8 * 8) * 2;
  long long left_b = BR ? ((g.J - j0 - 1) * g.ldb + (rend - rbeg)) * 2 : ((rend - rbeg - 1) * g.ldb + (g.J - j0 + 7) / 8 * 8) * 2;
  unsigned va[SA::kLoads], vb[SB::kLoads];
#pragma unroll
  for (int p = 0; p < SA::kLoads; ++p) {
    const int r = SA::row(p, wave, lane);
    va[p] = (unsigned)(r * g.lda * 2) + SA::piece(r, lane) * 16;
  }
#pragma unroll
  for (int p = 0; p < SB::kLoads; ++p) {
    const int r = SB::row(p, wave, lane);
    vb[p] = (unsigned)(r * g.ldb * 2) + SB::piece(r, lane) * 16;
  }
  // of a row of BK reduction steps: the first step of this lane's piece (the same in every instruction)
  const int ka = SA::piece(SA::row(0, wave, lane), lane) * 8, kb = SB::piece(SB::row(0, wave, lane), lane) * 8;
  int left_r = (int)min(rend - rbeg, (long long)0x40000000);
  const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds) + wave * 1024;
  auto request = [&](int p, int stage) {   // instruction p of the step
    const bool is_a = p < SA::kLoads;
    const __amdgpu_buffer_rsrc_t r = is_a ? make_rsrc(pa, left_a > 0 ? (unsigned)min(left_a, 0x7ffffff0LL) : 0u)
                                          : make_rsrc(pb, left_b > 0 ? (unsigned)min(left_b, 0x7ffffff0LL) : 0u);
    unsigned v = is_a ? va[p] : vb[p - SA::kLoads];
    if (is_a ? AR : BR) v = (is_a ? ka : kb) < left_r ? v : kOOB;
    transfer(r, v, lds_at + stage * kStage + (is_a ? p * 4096 : SA::kBytes + (p - SA::kLoads) * 4096));
  };
  auto advance = [&]() {
    const long long da = (AR ? BK : BK * g.lda) * 2, db = (BR ? BK : BK * g.ldb) * 2;
    pa += da; left_a -= da;
    pb += db; left_b -= db;
    left_r -= BK;
  };

  // ---- fragments from LDS: eight consecutive steps of the reduction of one index per lane, as they lie or by two transpose reads
  const int lr = lane & 31, lg = lane >> 5;
  int oa[AR ? NK : TM], ob[BR ? NK : TN];
  if constexpr (AR) {
#pragma unroll
    for (int k = 0; k < NK; ++k) oa[k] = (wm * WTM + lr) * SA::kRow + (((k * 2 + lg) ^ (BK == 64 ? lr & 7 : (lr >> 1) & 3)) << 4);
  } else {
    const int fr = lg * 8 + ((lane & 15) >> 2), fc = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int c = wm * WTM + i * 32 + fc;
      oa[i] = fr * SA::kRow + (((c >> 3) ^ ((fr & 3) << 2)) << 4) + (c & 7) * 2;
    }
  }
  if constexpr (BR) {
#pragma unroll
    for (int k = 0; k < NK; ++k) ob[k] = (wn * WTN + lr) * SB::kRow + (((k * 2 + lg) ^ (BK == 64 ? lr & 7 : (lr >> 1) & 3)) << 4);
  } else {
    const int fr = lg * 8 + ((lane & 15) >> 2), fc = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
      const int c = wn * WTN + j * 32 + fc;
      ob[j] = fr * SB::kRow + (((c >> 3) ^ ((fr & 3) << 2)) << 4) + (c & 7) * 2;
    }
  }
  bf16x8 fa[2][TM], fb[2][TN];
  auto fetch = [&](int n, int set, int stage, int k) {   // fragment n, in the order the products want them: A's first, B's, the rest of A's
    const char *A = lds + stage * kStage, *B = A + SA::kBytes;
    if (n == 0 || n > TN) {
      const int i = n == 0 ? 0 : n - TN;
      if constexpr (AR) fa[set][i] = *reinterpret_cast<const bf16x8 *>(A + oa[k] + i * 32 * SA::kRow);
      else fa[set][i] = lds_read_tr_pair(A + oa[i] + k * 16 * SA::kRow, A + oa[i] + (k * 16 + 4) * SA::kRow);
    } else {
      const int j = n - 1;
      if constexpr (BR) fb[set][j] = *reinterpret_cast<const bf16x8 *>(B + ob[k] + j * 32 * SB::kRow);
      else fb[set][j] = lds_read_tr_pair(B + ob[j] + k * 16 * SB::kRow, B + ob[j] + (k * 16 + 4) * SB::kRow);
    }
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // A step of the reduction asks for the tile STAGES steps ahead, whose place in LDS is free once all waves have met at the end of
  // the step before it: an NK-th of its transfers then, an NK-th with each of the first NK-1 of its NK products of depth 16.
  constexpr int kEach = kLoads / NK;
  static_assert(kLoads % NK == 0 && (STAGES - 2) * kLoads + kEach < 64, "transfers");
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
#pragma unroll
    for (int p = 0; p < kLoads; ++p) request(p, s);
    advance();
  }
#pragma unroll
  for (int p = 0; p < kEach; ++p) request(p, STAGES - 1);
  wait_and_meet<(STAGES - 2) * kLoads + kEach>();
#pragma unroll
  for (int n = 0; n < TM + TN; ++n) fetch(n, 0, 0, 0);
  __builtin_amdgcn_sched_barrier(0);
  int stage = 0, refill = STAGES - 1;
  auto step = [&](auto kc, int next) {
    constexpr int k = decltype(kc)::value, MF = TM * TN, DS = TM + TN, MD = MF * 3 / 4;
    constexpr bool last = k + 1 == NK;
    if constexpr (last) {
      advance();
      wait_and_meet<(STAGES - 2) * kLoads>();
    }
    int ds = 0, vm = 0;
#pragma unroll
    for (int m = 0; m < MF; ++m) {   // a product, then what goes on beside it, in this order
      const int i = m / TN, j = m % TN;
      acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[k & 1][j], fa[k & 1][i], acc[i][j], 0, 0, 0);
#pragma unroll
      for (; ds < (m < MD ? (m + 1) * DS / MD : DS); ++ds) fetch(ds, (k + 1) & 1, last ? next : stage, last ? 0 : k + 1);
#pragma unroll
      for (; vm < (m < MF / 2 ? (m + 1) * kEach / (MF / 2) : kEach); ++vm) request(last ? vm : (k + 1) * kEach + vm, last ? stage : refill);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  for (int t = 0; t < steps; ++t) {
    const int next = stage + 1 == STAGES ? 0 : stage + 1;
    step(std::integral_constant<int, 0>{}, next);
    step(std::integral_constant<int, 1>{}, next);
    if constexpr (NK > 2) {
      step(std::integral_constant<int, 2>{}, next);
      step(std::integral_constant<int, 3>{}, next);
    }
    refill = stage;
    stage = next;
  }

  // ---- out: 32 rows of a wave's share at a time through LDS, so that memory sees whole rows of it.  One wave a SIMD has nothing to hide a
  // wait behind but its own next rows: they are on their way from LDS, what the epilogue reads beside them for the next kAhead passes from
  // memory, while a pass is worked on.  One copy of the code (it is long, and the instruction cache is shared).
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the steps past the end have arrived too
  char *const mine = lds + wave * 2 * 32 * kPitch;
  const bool whole = g.splits == 1;
  const u64 base = g.e.d.rng && whole ? dropout_base(g.e.d.rng) : 0;
  constexpr int LPR = WTN / 8, RPP = 64 / LPR, PASSES = 32 / RPP, kAhead = sizeof(O) == 2 ? 8 : 4;   // lanes a row, rows a pass, passes of 32 rows
  const int c = (lane % LPR) * 8, j = j0 + wn * WTN + c, left = g.J - j;
  const long long row0 = i0 + wm * WTM + lane / LPR;
  auto put = [&](auto kc) {
    constexpr int k = decltype(kc)::value;
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4 *>(mine + (k & 1) * 32 * kPitch + lr * kPitch + (n * 32 + q * 8 + lg * 4) * 4) =
            f32x4{acc[k][n][q * 4], acc[k][n][q * 4 + 1], acc[k][n][q * 4 + 2], acc[k][n][q * 4 + 3]};
    asm volatile("" ::"n"(k));   // left alone, the compiler makes one of the calls, with an index, and keeps the sums in memory for it
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  f32x4 v0, v1;
  auto get = [&](int pass) {   // rows of pass `pass` of all
    const char *p = mine + (pass / PASSES & 1) * 32 * kPitch + (pass % PASSES * RPP + lane / LPR) * kPitch + c * 4;
    v0 = *reinterpret_cast<const f32x4 *>(p);
    v1 = *reinterpret_cast<const f32x4 *>(p + 16);
  };
  long long ld_side;
  const O *side = side_of<O>(g.e, ld_side);
  const bool has_side = side != nullptr && whole;
  Raw8<O> ahead[kAhead] = {};
  auto ask = [&](int pass, Raw8<O> &r) {
    const long long row = row0 + pass * RPP;
    if (pass < TM * PASSES && row < g.I && left > 0) raw_load(side + row * ld_side + j, left, r);
  };
  float bias[8] = {};
  if (whole) bias_of(g.e, j, left, bias);
  if (has_side) {
#pragma unroll
    for (int p = 0; p < kAhead; ++p) ask(p, ahead[p]);
  }
  put(std::integral_constant<int, 0>{});
  get(0);
#pragma unroll 1
  for (int pass = 0; pass < TM * PASSES; ++pass) {
    if (TM > 1 && pass == 0) put(std::integral_constant<int, TM - 1 < 1 ? TM - 1 : 1>{});
    if (TM > 2 && pass == PASSES) put(std::integral_constant<int, TM - 1 < 2 ? TM - 1 : 2>{});
    if (TM > 3 && pass == 2 * PASSES) put(std::integral_constant<int, TM - 1 < 3 ? TM - 1 : 3>{});
    float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
    get(pass + 1 < TM * PASSES ? pass + 1 : pass);
    const Raw8<O> now = ahead[0];
    if (has_side) {
#pragma unroll
      for (int p = 0; p + 1 < kAhead; ++p) ahead[p] = ahead[p + 1];
      ask(pass + kAhead, ahead[kAhead - 1]);
    }
    const long long row = row0 + pass * RPP;
    if (row >= g.I || left <= 0) continue;
    if (whole) finish8<O>(g.e, row, j, left, v, bias, now, base);
    else row_store(g.part + ((long long)split * g.I + row) * g.J + j, left, v);
  }
}

// the parts of a split reduction, in order
template <typename O>
__global__ __launch_bounds__(kThreads) void gemm_join_kernel(const float *part, int splits, long long I, int J, Epilogue e) {
  const int nvec = (J + 7) / 8;
  const long long u = (long long)blockIdx.x * kThreads + threadIdx.x;
  const long long row = u / nvec;
  const int j = (int)(u - row * nvec) * 8, left = J - j;
  if (row >= I) return;
  float v[8];
  row_load(part + row * J + j, left, v);
  for (int s = 1; s < splits; ++s) {
    float w[8];
    row_load(part + ((long long)s * I + row) * J + j, left, w);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += w[k];
  }
  float bias[8];
  bias_of(e, j, left, bias);
  long long ld;
  const O *side = side_of<O>(e, ld);
  Raw8<O> now = {};
  if (side) raw_load(side + row * ld + j, left, now);
  finish8<O>(e, row, j, left, v, bias, now, e.d.rng ? dropout_base(e.d.rng) : 0);
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

template <typename O, bool AR, bool BR, int BM, int BN, int BK, int STAGES, int WGS> int gemm_tiles_of(TileArgs &t, hipStream_t st) {
  t.tiles_i = (int)((t.I + BM - 1) / BM);
  t.tiles_j = (int)((t.J + BN - 1) / BN);
  t.group = 8; t.splits = 1; t.per_split = (t.R + BK - 1) / BK * BK;
  gemm_tile_kernel<O, AR, BR, BM, BN, BK, STAGES, WGS><<<t.tiles_i * t.tiles_j, kThreads, 0, st>>>(t);
  RESIST_CHECK_LAUNCH("linear");
  return RESIST_OK;
}
#ifndef RESIST_CFG
#define RESIST_CFG 256, 256, 64, 2, 1
#endif
template <typename O, bool AR, bool BR> int gemm_tiles(TileArgs &t, hipStream_t st) {
  return gemm_tiles_of<O, AR, BR, RESIST_CFG>(t, st);
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
  if (dt == DT_BF16 && s.K % 8 == 0 && s.ldx % 8 == 0) {
    TileArgs t{};
    t.a = (const __bf16 *)x; t.b = (const __bf16 *)w; t.lda = s.ldx; t.ldb = s.K; t.I = s.M; t.J = s.N; t.R = s.K; t.e = g.e;
    return gemm_tiles<__bf16, true, true>(t, st);
  }
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
  if (dt == DT_BF16 && s.N % 8 == 0 && s.K % 8 == 0 && s.ldy % 8 == 0) {
    TileArgs t{};
    t.a = (const __bf16 *)dz; t.b = (const __bf16 *)w; t.lda = s.ldy; t.ldb = s.K; t.I = s.M; t.J = s.K; t.R = s.N; t.e = g.e;
    return gemm_tiles<__bf16, true, false>(t, st);
  }
  prof::Scope sc("linear_dgrad", 2. * s.M * s.N * s.K, ((double)s.M * s.K + (double)s.N * s.K + (double)s.M * s.N) * esize(dt), st);
  return dt == DT_F32 ? gemm_any<float, float, true, false>(g, st) : gemm_any<__bf16, __bf16, true, false>(g, st);
}

int linear_wgrad(const LinearShape &s, int dt, const void *dz, const void *x, float *dw, float *db, void *, hipStream_t st) {
  GemmArgs g{};
  g.a = dz; g.ai = 1; g.ar = s.ldy; g.I = s.N;
  g.b = x; g.bj = 1; g.br = s.ldx; g.J = s.K; g.R = s.M;
  g.e.out = dw; g.e.ldo = s.K;
  if (dw && dt == DT_BF16 && s.ldx % 8 == 0 && s.ldy % 8 == 0) {
    TileArgs t{};
    t.a = (const __bf16 *)dz; t.b = (const __bf16 *)x; t.lda = s.ldy; t.ldb = s.ldx; t.I = s.N; t.J = s.K; t.R = s.M; t.e = g.e;
    RESIST_TRY((gemm_tiles<float, false, false>(t, st)));
  } else if (dw) {
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

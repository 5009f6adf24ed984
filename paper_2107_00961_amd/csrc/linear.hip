// Dense layers on rows of activations: x [M][K], w [N][K].
//   forward          z = x w' + bias,  y = residual + drop(a(z))
//   data gradient    dx = a'(z) drop(dz w)        (z, a, drop: of the layer that produced x)
//   weight gradient  dw = dz' x,  db = column sums of dz
// All three are one product, out(i, j) = sum over r of a(i, r) b(j, r), with either index contiguous in either operand.  Products on the matrix
// cores, sums in fp32, one rounding where a result is stored.  Three ways:
//   tiles      (gemm_tile_kernel) bf16 operands, or the three bf16 parts of fp32 ones (conv3.hip says why that loses nothing)
//   few rows   (few_rows_*_kernel) w straight from memory into fragments, or dw straight from registers: bound by its bytes
//   plain      (plain_tile) what of an fp32 product three parts do not hold, on the fp32 matrix instruction
// Operands whose rows are not 16-byte aligned, and those in parts, are laid out in the workspace first (lay_out_kernel).
#include <algorithm>

#include "conv_tile.h"
#include "dense.h"

namespace resist {
namespace {

constexpr int kThreads = 256;
constexpr long long kMaxWgs = kMaxThreads / kThreads;   // of a launch (HIP counts threads modulo 2^32)

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

// element (i, j)
template <typename T>
__device__ inline void finish(const Epilogue &e, long long i, int j, float v, u64 base) {
  float t[1] = {v};
  if (e.bias) t[0] += e.bias[j];
  if (e.z_out) static_cast<T *>(e.z_out)[i * e.ldz + j] = (T)t[0];
  if (!e.z_in) activate(t, e.act);
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

// ---- operands in the workspace --------------------------------------------------------------------------------------
// A matrix [rows][n] with `ld` elements between rows becomes [rows][to_ld] of bf16, to_ld a multiple of eight, with zeros behind a row's end:
// a copy (bf16), or three planes of parts (fp32).  Parts whose rows are the reduction's axis lie [to_ld/32][rows][32], to_ld a multiple of 32: the
// tiles read them 32 at a time, of which a row's 64 bytes would be half a line each.  Of parts, each 64x64 block also leaves a word: whether it has a value that three parts
// do not hold (conv3.hip: not finite or rounding to infinity, or below 2^-110).  2000 x 1024 and 1024 x 1024 in fp32, 31 MB in and out: 8 us.
struct LayOut {
  const void *from;
  __bf16 *to;
  unsigned *flags;          // [ceil(rows/64)][ceil(to_ld/64)]
  float *sums;              // optional [ceil(rows/64)][n]: of the columns, 64 rows each
  long long rows, ld, plane;   // plane: elements between planes
  int n, to_ld, blocks_n, blocks, panels;   // panels: [to_ld/32][rows][32]
};
struct LayOutArgs { LayOut m[2]; int first; };   // first: the launch's first block
// split_check, and for NaN: what two parts leave of a value that is not finite or rounds to infinity
__device__ inline void parts_check(const f32x4 &v, unsigned long long &missed) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    unsigned long long lanes;
    asm("v_cmp_class_f32 %0, %1, %2" : "=s"(lanes) : "v"(v[e]), "s"(0x93));   // subnormal of either sign, NaN
    missed |= lanes;
  }
}
template <int NP>
__global__ __launch_bounds__(kThreads) void lay_out_kernel(LayOutArgs a) {
  using T = std::conditional_t<NP == 3, float, __bf16>;
  const int at = a.first + (int)blockIdx.x, second = at >= a.m[0].blocks;
  const LayOut &m = a.m[second];
  const int b = at - (second ? a.m[0].blocks : 0);
  const int bi = b / m.blocks_n, bj = b - bi * m.blocks_n;
  const int c = bj * 64 + (threadIdx.x & 7) * 8;
  unsigned long long missed = 0;
  float sum[8] = {};
#pragma unroll
  for (int p = 0; p < 2; ++p) {
    const long long row = (long long)bi * 64 + p * 32 + (threadIdx.x >> 3);
    if (row >= m.rows || c >= m.to_ld) continue;
    float v[8];
    row_load(static_cast<const T *>(m.from) + row * m.ld + c, m.n - c, v);
    __bf16 *to = m.to + (m.panels ? ((long long)(c >> 5) * m.rows + row) * 32 + (c & 31) : row * m.to_ld + c);
    if constexpr (NP == 3) {
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] += v[e];
      f32x4 lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        if (q == 2) {
          parts_check(lo, missed);
          parts_check(hi, missed);
        }
        const u32x2 x = split_part(lo), y = split_part(hi);
        *reinterpret_cast<u32x4 *>(to + q * m.plane) = u32x4{x[0], x[1], y[0], y[1]};
      }
    } else {
      row_store(to, 8, v);
    }
  }
  if constexpr (NP == 3) {
    const int any = __syncthreads_or(missed != 0);
    if (threadIdx.x == 0) m.flags[b] = any;
    if (m.sums) {
      __shared__ float cols[32][65];
#pragma unroll
      for (int e = 0; e < 8; ++e) cols[threadIdx.x >> 3][(threadIdx.x & 7) * 8 + e] = sum[e];
      __syncthreads();
      const int k = threadIdx.x;
      if (k < 64 && bj * 64 + k < m.n) {
        float t = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) t += cols[r][k];
        m.sums[(size_t)bi * m.n + bj * 64 + k] = t;
      }
    }
  }
}

// ---- tiles --------------------------------------------------------------------------------------------
// Operand tiles go from memory straight into LDS (16 bytes a lane, 1 KB a wave and instruction, in lane order), STAGES deep, and from there
// in fragments to the matrix cores.  Four waves, a quarter of the BM x BN tile each: the larger a wave's share, the fewer times a
// staged element is read from LDS (256x256: 1024 clocks of reading and 512 of arriving for 2048 of products).  Bound by the matrix cores and what
// the chip's power leaves of its clock: 8192 x 8192 -> 2048 in bf16 192 us (1.43 PFLOP/s, the cores at work in 72 % of 362 thousand clocks at 1.86 GHz),
// 2000 x 1024 -> 1024 in fp32 30 us beside 8 of laying out.  The epilogue's arithmetic is not hidden, one workgroup having a compute unit to itself: with GELU,
// dropout and z 8192 x 2048 -> 8192 takes 290 ... 328 us for 213 ... 240 (making the mask between the products, though it fits, saved 1 %).
// Layout in LDS.  Lane order leaves no room for padding, so what keeps rows off each other's banks is which 16-byte piece a lane asks for:
//   reduction contiguous (R): a row is an index i, BK values of r: piece c of row i lies at c ^ f(i), f = (i >> 1) & 7 (BK 64, two rows to 256
//     bytes), (i >> 2) & 3 (BK 32, four rows): sixteen consecutive rows' pieces c fill the 256 bytes of the 64 banks;
//   other index contiguous: a row is an r, BM values of i: piece c of row r lies at c ^ 4 (r & 3) (64 values, two rows to 256 bytes:
//     c ^ 2 (r & 2)): the four rows of a transpose read, 64 bytes each, fill 256 bytes.  In fragments of 16 it has eight rows r, r + 1, .. r + 3, r + 8, ..
//     of 32 bytes each: c ^ 2 (r & 3) ^ (r & 8).
// Bounds: an operand's descriptor starts at the tile and ends with the operand (rows past it, and steps past it, come as zeros); its
// contiguous axis is a multiple of eight where it is the reduction (a tail's pieces are not asked for) and may end in a piece where it is
// not (what a tile has past its last column goes into outputs that are not stored).
// Operands in three parts are three such tiles each, and a product is six (small ones first).
template <bool R, int B, int BK, int FR> struct Stage {
  static constexpr int kBytes = B * BK * 2, kLoads = kBytes / 4096;   // of a plane; a wave's instructions
  static constexpr int kRow = R ? BK * 2 : B * 2, kPieces = kRow / 16, kRows = 1024 / kRow;   // rows an instruction
  __device__ static inline int swizzle(int row) {
    if (R) return BK == 64 ? (row >> 1) & 7 : (row >> 2) & 3;
    if (FR == 16) return (row & 3) << 1 | (row & 8);
    return kPieces == 8 ? (row & 2) << 1 : (row & 3) << 2;
  }
  // row and piece of the tile that lane `l` of wave `w` asks for with instruction p
  __device__ static inline int row(int p, int w, int l) { return (p * 4 + w) * kRows + l / kPieces; }
  __device__ static inline int piece(int r, int l) { return (l % kPieces) ^ swizzle(r); }
};

struct TileArgs {
  const __bf16 *a, *b;
  long long lda, ldb;       // elements between rows (of i, or of r)
  long long I, R;
  int J, tiles_i, tiles_j, group;
  int splits;
  long long per_split;      // steps of the reduction, a multiple of the tile's
  float *part;              // [splits][I][J] where the reduction is split
  float *sums;              // optional (neither reduction contiguous): [splits * tiles_j * 2][I], parts of the sums of a over r
  // operands in parts: elements between planes, the words of their blocks, and the operands themselves
  long long plane_a, plane_b;
  const unsigned *flags_a, *flags_b;
  const float *a32, *b32;
  long long lda32, ldb32;
  Epilogue e;
};

// Eight outputs of each of H rows (those that are `ok`), at `out`; z goes to `z_out` (optional), `word` is where the dropout's sequence is for them.  bias: of
// their columns; side: what the epilogue reads beside them, z (data gradient) or the residual (forward).  Several rows at once, as every
// branch costs a wave that has its SIMD to itself as much as a dozen instructions.
template <typename O, int H>
__device__ inline void finish_rows(const Epilogue &e, O *const (&out)[H], O *const (&z_out)[H], const u64 (&word)[H], int left, const bool (&ok)[H], float (&v)[H][8],
                                   const float (&bias)[8], const Raw8<O> (&side)[H]) {
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int k = 0; k < 8; ++k) v[h][k] += bias[k];
  auto store = [&](O *const (&to)[H]) {
    if (left >= 8) {
#pragma unroll
      for (int h = 0; h < H; ++h)
        if (ok[h]) Row<O>::store(to[h], v[h]);
    } else {
#pragma unroll
      for (int h = 0; h < H; ++h)
        if (ok[h]) row_store(to[h], left, v[h]);
    }
  };
  float(&all)[H * 8] = reinterpret_cast<float(&)[H * 8]>(v);
  if (e.z_out) store(z_out);
  if (!e.z_in) activate(all, e.act);
  if (e.d.rng) {
#pragma unroll
    for (int h = 0; h < H; ++h) dropout8(word[h], e.d.thr, e.d.scale, v[h]);
  }
  if (e.z_in || e.res) {
    float s[H][8];
#pragma unroll
    for (int h = 0; h < H; ++h) widen(side[h], s[h]);
    float(&flat)[H * 8] = reinterpret_cast<float(&)[H * 8]>(s);
    if (e.z_in) {
      times_slope(all, flat, e.act);
    } else {
#pragma unroll
      for (int k = 0; k < H * 8; ++k) all[k] += flat[k];
    }
  }
  store(out);
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
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(r), "s"(to) : "memory", "m0");
}
template <int N> __device__ inline void wait_and_meet() {   // at most N of this wave's transfers to LDS under way, all of its reads done
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

__device__ inline void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }   // all reads done

// f(0), f(1), ... as constants
template <int... M, typename F> __device__ inline void each(std::integer_sequence<int, M...>, F f) { (f(std::integral_constant<int, M>{}), ...); }

// the tile's place: `group` rows of tiles are walked column by column, an XCD's workgroups one after the other
__device__ inline void tile_of(int bid, int tiles_i, int tiles_j, int group, int &ti, int &tj) {
  const int per = group * tiles_j, g = bid / per, rest = bid - g * per;
  const int rows = min(group, tiles_i - g * group);
  tj = rest / rows;
  ti = g * group + rest - tj * rows;
}

// BM x BN outputs from the operands as they are, in fp32 on its own matrix instruction, 64x64 at a time: for operands and results that three parts do
// not hold.  Bound by its loads, an element each with two barriers every 32 steps: 2000 x 1024 -> 1024 with one such value in x takes 186 us for 40, 8192 x 2048 -> 2048
// 1835 for 354 (one tile's time, most of it), with one in every block 3171.  `lds`: 18 KB.  to(i, j, v) takes an output.
template <bool AR, bool BR, int BM, int BN, typename To>
__device__ inline void plain_tile(const TileArgs &g, long long i0, int j0, long long rbeg, long long rend, char *lds, To to) {
  constexpr int BK = 32;
  float (*As)[BK + 4] = reinterpret_cast<float (*)[BK + 4]>(lds), (*Bs)[BK + 4] = As + 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
  const long long ai = AR ? g.lda32 : 1, ar = AR ? 1 : g.lda32, bj = BR ? g.ldb32 : 1, br = BR ? 1 : g.ldb32;
#pragma unroll 1
  for (int s = 0; s < (BM / 64) * (BN / 64); ++s) {
    const long long i1 = i0 + s / (BN / 64) * 64;
    const int j1 = j0 + s % (BN / 64) * 64;
    f32x16 acc = {};
#pragma unroll 1
    for (long long r0 = rbeg; r0 < rend; r0 += BK) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = AR ? tid >> 2 : tid & 63, r = AR ? (tid & 3) * 8 + e : (tid >> 6) * 8 + e;
        As[i][r] = i1 + i < g.I && r0 + r < rend ? g.a32[(i1 + i) * ai + (r0 + r) * ar] : 0.f;
        const int j = BR ? tid >> 2 : tid & 63, q = BR ? (tid & 3) * 8 + e : (tid >> 6) * 8 + e;
        Bs[j][q] = j1 + j < g.J && r0 + q < rend ? g.b32[(j1 + j) * bj + (r0 + q) * br] : 0.f;
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < BK; k += 8)
        Elem<float>::mma(acc, *reinterpret_cast<const f32x4 *>(&As[wm * 32 + (lane & 31)][k + (lane >> 5) * 4]),
                         *reinterpret_cast<const f32x4 *>(&Bs[wn * 32 + (lane & 31)][k + (lane >> 5) * 4]));
    }
    const int j = j1 + wn * 32 + (lane & 31);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const long long i = i1 + wm * 32 + (e >> 2) * 8 + (lane >> 5) * 4 + (e & 3);
      if (i < g.I && j < g.J) to(i, j, acc[e]);
    }
  }
}

template <typename O, bool AR, bool BR, int NP, int BM, int BN, int BK, int STAGES, int WGS>
__global__ __launch_bounds__(kThreads, WGS) void gemm_tile_kernel(TileArgs g) {
  constexpr bool EARLY = STAGES == 2 && BK == 64 && NP == 1;
  // Fragments of FR rows by FK of the reduction.  v_mfma_f32_16x16x32_bf16 moves less through the registers than 32x32x16 (a result is added to half as
  // often), and the clock that the power limit leaves is what counts: 2.0 PFLOP/s with it alone, 1.8 with the other.
  constexpr int FR = EARLY ? 16 : 32, FK = 512 / FR;
  using SA = Stage<AR, BM, BK, FR>;
  using SB = Stage<BR, BN, BK, FR>;
  constexpr int WTM = BM / 2, WTN = BN / 2, TM = WTM / 32, FM = WTM / FR, FN = WTN / FR, NK = BK / FK;
  constexpr int kLoadsA = NP * SA::kLoads, kLoads = kLoadsA + NP * SB::kLoads, kA = NP * SA::kBytes, kStage = kA + NP * SB::kBytes;
  constexpr int kPitch = WTN * 4 + 16, kSide = AR ? 32 * WTN * (int)sizeof(O) : 0, kOut = 4 * (32 * kPitch + kSide);
  static_assert(STAGES >= 2, "stages");
  // Two stages only (EARLY): a step's fragments are read in its first half, and what is staged next goes where they came from in the second half:
  // transfers have half a step and more to arrive in, and a stage less does.  (Fragments are read a product ahead else, and a stage is free a step later.
  // Waiting for transfers took 11 % of the 256x256 tile's time then.  Spread over all of a step, the 128x128 tile of 4096 x 2048 x 2048 took 38 and, as
  // weight gradient, 55 us for 37 and 49.)
  static_assert(TM <= 4, "tile");
  __shared__ __attribute__((aligned(1024))) char lds[STAGES * kStage > kOut ? STAGES * kStage : kOut];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 1, wn = wave & 1;
  int ti, tj, bid = xcd_contiguous(blockIdx.x, gridDim.x);
  const int split = bid / (g.tiles_i * g.tiles_j);
  tile_of(bid - split * g.tiles_i * g.tiles_j, g.tiles_i, g.tiles_j, g.group, ti, tj);
  const long long i0 = (long long)ti * BM, rbeg = split * g.per_split, rend = min(g.R, rbeg + g.per_split);
  const int j0 = tj * BN;
  const int steps = (int)((rend - rbeg + BK - 1) / BK);

  // ---- operands to LDS
  constexpr bool PA = AR && NP == 3, PB = BR && NP == 3;   // in panels of 32 steps: [R/32][I][32]
  static_assert(NP == 1 || BK == 32, "panels");
  const char *pa = reinterpret_cast<const char *>(g.a + (PA ? (rbeg >> 5) * g.I * 32 + i0 * 32 : AR ? i0 * g.lda + rbeg : rbeg * g.lda + i0));
  const char *pb = reinterpret_cast<const char *>(g.b + (PB ? (rbeg >> 5) * g.J * 32 + (long long)j0 * 32 : BR ? (long long)j0 * g.ldb + rbeg : rbeg * g.ldb + j0));
  unsigned va[SA::kLoads], vb[SB::kLoads];
#pragma unroll
  for (int p = 0; p < SA::kLoads; ++p) {
    const int r = SA::row(p, wave, lane);
    va[p] = (PA ? r * 64u : (unsigned)(r * g.lda * 2)) + SA::piece(r, lane) * 16;
  }
#pragma unroll
  for (int p = 0; p < SB::kLoads; ++p) {
    const int r = SB::row(p, wave, lane);
    vb[p] = (PB ? r * 64u : (unsigned)(r * g.ldb * 2)) + SB::piece(r, lane) * 16;
  }
  // of a row of BK reduction steps: the first step of this lane's piece (the same in every instruction)
  const int ka = SA::piece(SA::row(0, wave, lane), lane) * 8, kb = SB::piece(SB::row(0, wave, lane), lane) * 8;
  int left_r = (int)(rend - rbeg);   // steps are rows of a matrix, or fewer
  // Bytes of an operand from the tile's current corner on.  Where the reduction is contiguous, to the end of the last row: rows past it begin there or
  // later at any step, and steps past the end are not asked for.  Else the rows that this step has, at most BK of them.
  auto capped = [](long long n) { return (unsigned)min(n, 0x7ffffff0LL); };
  unsigned size_a = PA ? capped((g.I - i0) * 64) : AR ? capped(((g.I - i0 - 1) * g.lda + (rend - rbeg + 7) / 8 * 8) * 2) : 0u;
  unsigned size_b = PB ? capped((long long)(g.J - j0) * 64) : BR ? capped(((g.J - j0 - 1) * g.ldb + (rend - rbeg + 7) / 8 * 8) * 2) : 0u;
  const unsigned row_a = (unsigned)g.lda * 2, row_b = (unsigned)g.ldb * 2, last_a = AR ? 0u : (unsigned)((g.I - i0 + 7) / 8 * 8) * 2, last_b = BR ? 0u : (unsigned)((g.J - j0 + 7) / 8 * 8) * 2;
  auto measure = [&]() {
    const int rows = min(left_r, BK);
    if constexpr (!AR) size_a = rows > 0 ? (rows - 1) * row_a + last_a : 0u;
    if constexpr (!BR) size_b = rows > 0 ? (rows - 1) * row_b + last_b : 0u;
  };
  measure();
  const unsigned lds_at = __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds) + wave * 1024;
  auto aim = [&](int p, int stage, unsigned &v, unsigned &to) {   // of instruction p of the step: where from, where to
    const bool is_a = p < kLoadsA;
    const int q = is_a ? p : p - kLoadsA, per = is_a ? SA::kLoads : SB::kLoads;
    v = is_a ? va[q % per] : vb[q % per];
    if (is_a ? AR : BR) v = (is_a ? ka : kb) < left_r ? v : kOOB;
    to = lds_at + stage * kStage + (is_a ? 0 : kA) + q * 4096;
    asm volatile("" : "+v"(v), "+s"(to));   // here, that is
  };
  auto go = [&](int p, unsigned v, unsigned to) {
    const bool is_a = p < kLoadsA;
    const int plane = is_a ? p / SA::kLoads : (p - kLoadsA) / SB::kLoads;
    transfer(is_a ? make_rsrc(pa + plane * g.plane_a * 2, size_a) : make_rsrc(pb + plane * g.plane_b * 2, size_b), v, to);
  };
  auto request = [&](int p, int stage) {
    unsigned v, to;
    aim(p, stage, v, to);
    go(p, v, to);
  };
  const long long da = PA ? g.I * 64 : (AR ? BK : BK * g.lda) * 2, db = PB ? g.J * 64LL : (BR ? BK : BK * g.ldb) * 2;
  // To the next step, in three pieces that fit beside a product each.  (Left alone, the compiler makes all of them at the loop's end, where nothing
  // goes on beside them.)
  auto advance = [&](int piece) {
    if (piece == 0) {
      pa += da;
      asm volatile("" : "+s"(pa));
    } else if (piece == 1) {
      pb += db;
      asm volatile("" : "+s"(pb));
    } else {
      left_r -= BK;
      asm volatile("" : "+s"(left_r));
      measure();
    }
  };

  // ---- fragments from LDS: eight consecutive steps of the reduction of one index per lane, as they lie or by two transpose reads
  const int lr = lane % FR, lg = lane / FR;
  int oa[AR ? NK : FM], ob[BR ? NK : FN];
  auto frag_r = [&](int at, int k, int row_bytes, int swizzle) { return (at + lr) * row_bytes + (((k * (FK / 8) + lg) ^ swizzle) << 4); };
  const int fr = lg * 8 + ((lane & 15) >> 2), fc = (FR == 32 ? ((lane >> 4) & 1) * 16 : 0) + (lane & 3) * 4;
  auto frag_t = [&](int at, int row_bytes, int swizzle) { return fr * row_bytes + ((((at + fc) >> 3) ^ swizzle) << 4) + ((at + fc) & 7) * 2; };
  if constexpr (AR) {
#pragma unroll
    for (int k = 0; k < NK; ++k) oa[k] = frag_r(wm * WTM, k, SA::kRow, SA::swizzle(lr));
  } else {
#pragma unroll
    for (int i = 0; i < FM; ++i) oa[i] = frag_t(wm * WTM + i * FR, SA::kRow, SA::swizzle(fr));
  }
  if constexpr (BR) {
#pragma unroll
    for (int k = 0; k < NK; ++k) ob[k] = frag_r(wn * WTN, k, SB::kRow, SB::swizzle(lr));
  } else {
#pragma unroll
    for (int j = 0; j < FN; ++j) ob[j] = frag_t(wn * WTN + j * FR, SB::kRow, SB::swizzle(fr));
  }
  bf16x8 fa[2][NP][FM], fb[2][NP][FN];
  constexpr int kFrags = NP * (FM + FN);
  auto fetch_a = [&](int i, int p, int set, int stage, int k) {
    const char *A = lds + stage * kStage + p * SA::kBytes;
    if constexpr (AR) fa[set][p][i] = *reinterpret_cast<const bf16x8 *>(A + oa[k] + i * FR * SA::kRow);
    else fa[set][p][i] = lds_read_tr_pair(A + oa[i] + k * FK * SA::kRow, A + oa[i] + (k * FK + 4) * SA::kRow);
  };
  auto fetch_b = [&](int j, int p, int set, int stage, int k) {
    const char *B = lds + stage * kStage + kA + p * SB::kBytes;
    if constexpr (BR) fb[set][p][j] = *reinterpret_cast<const bf16x8 *>(B + ob[k] + j * FR * SB::kRow);
    else fb[set][p][j] = lds_read_tr_pair(B + ob[j] + k * FK * SB::kRow, B + ob[j] + (k * FK + 4) * SB::kRow);
  };
  // Fragment n: plane by plane from the smallest part on, of a plane A's first, B's, the rest of A's.  Early, half of A's and of B's in that order, then the
  // rest of B's, the rest of A's.
  auto fetch = [&](int n, int set, int stage, int k) {
    if constexpr (EARLY) {
      if (n == 0) fetch_a(0, 0, set, stage, k);
      else if (n <= FN / 2) fetch_b(n - 1, 0, set, stage, k);
      else if (n < FN / 2 + FM / 2) fetch_a(n - FN / 2, 0, set, stage, k);
      else if (n < FN + FM / 2) fetch_b(n - FM / 2, 0, set, stage, k);
      else fetch_a(n - FN, 0, set, stage, k);
    } else {
      const int p = NP - 1 - n / (FM + FN), m = n % (FM + FN);
      if (m == 0 || m > FN) fetch_a(m == 0 ? 0 : m - FN, p, set, stage, k);
      else fetch_b(m - 1, p, set, stage, k);
    }
  };

  std::conditional_t<FR == 16, f32x4, f32x16> acc[FM][FN];   // a lane's: 4 or 16 columns, in runs of four, of row lr
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < FR * FR / 64; ++e) acc[i][j][e] = 0.f;

  // A step of the reduction asks for the tile STAGES steps ahead, whose place in LDS is free once all waves have met: an NK-th of its transfers with
  // each of NK products of depth FK, from the last of the step before on.  Early: all of them in the second of two.
  static_assert((STAGES - 1) * kLoads < 64, "transfers");
  auto cut = [](int k) constexpr { return k * kLoads / NK; };   // a tile's transfers cut(k) .. cut(k + 1) go together
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s) {
#pragma unroll
    for (int p = 0; p < kLoads; ++p) request(p, s);
#pragma unroll
    for (int p = 0; p < 3; ++p) advance(p);
  }
  constexpr int kFirst = EARLY ? kLoads : cut(1);
#pragma unroll
  for (int p = 0; p < kFirst; ++p) request(p, STAGES - 1);
  wait_and_meet<(STAGES - 2) * kLoads + kFirst>();
  // Early: fragments that a step finds read; the rest go beside its first products (where those are few, there is no time for any)
  constexpr int kReady = !EARLY || FM * FN < 64 ? kFrags : kFrags / 2;
#pragma unroll
  for (int n = 0; n < kReady; ++n) fetch(n, 0, 0, 0);
  __builtin_amdgcn_sched_barrier(0);
  int stage = 0, refill = STAGES - 1;
  // sums of a over r (the gradient of a bias): of the steps t with t % tiles_j == tj, the first waves in the even, the second in the odd products of depth FK
  constexpr bool kSums = !AR && NP == 1;
  float sums[FM] = {};
  int sums_at = kSums && g.sums ? tj : 0x7fffffff;
  auto sum_up = [&](int set) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sums[i] += (float)fa[set][0][i][e];
  };
  auto multiply = [](auto &c, const bf16x8 &b, const bf16x8 &a) {
    if constexpr (sizeof(c) == 16) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0);
    else c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0);
  };
  auto step = [&](auto kc, int next, bool take) {
    constexpr int k = decltype(kc)::value, PAIRS = NP == 3 ? 6 : 1, MF = PAIRS * FM * FN, MD = MF > 1 ? MF * 3 / 4 : 1, MH = MF == 1 ? MF : MF / 2;
    constexpr bool last = k + 1 == NK;
    constexpr int set = k & 1, part = (k + 1) % NK, v0 = cut(part), VM = cut(part + 1) - v0, DS = kFrags;
    if constexpr (last) {
#pragma unroll
      for (int p = 0; p < 3; ++p) advance(p);
      wait_and_meet<(STAGES - 2) * kLoads>();   // the next stage is there
    }
    int ds = 0, vm = 0;   // the next product's fragments are read beside this one's
#pragma unroll
    for (int m = 0; m < MF; ++m) {   // a product, then what goes on beside it, in this order
      const int pair = m / (FM * FN), i = m / FN % FM, j = m % FN;
      const int pa_ = NP == 1 ? 0 : pair == 0 ? 2 : pair == 1 ? 0 : pair == 2 ? 1 : pair == 3 ? 1 : 0;   // parts l h', h l', m m', m h', h m', h h'
      const int pb_ = NP == 1 ? 0 : pair == 0 ? 0 : pair == 1 ? 2 : pair == 2 ? 1 : pair == 3 ? 0 : pair == 4 ? 1 : 0;
      multiply(acc[i][j], fb[set][pb_][j], fa[set][pa_][i]);
#pragma unroll
      for (; ds < (m + 1 < MD ? (m + 1) * DS / MD : DS); ++ds) fetch(ds, (k + 1) & 1, last ? next : stage, last ? 0 : k + 1);
#pragma unroll
      for (; vm < (m + 1 < MH ? (m + 1) * VM / MH : VM); ++vm) request(v0 + vm, last ? stage : refill);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (kSums)
      if (take && (k & 1) == wn) sum_up(set);
  };
  // Early: products in four blocks, A's and B's first halves, then B's second, then A's: their fragments may come one after the other.  What goes on
  // beside a product has 12 clocks, three instructions, so a transfer takes two products' (its address, then itself).
  auto early_step = [&](auto kc, int next, bool take) {
    constexpr int k = decltype(kc)::value, P = FM * FN, HM = FM / 2, HN = FN / 2, MD = P * 3 / 4, LATE = kFrags - kReady, VH = kLoads / 2, EACH = EARLY ? P / 2 / VH : 2;
    static_assert(!EARLY || (EACH >= 2 && NK == 2), "transfers");
    unsigned v = 0, to = 0;
    auto due = [](int m) constexpr {   // fragments read before product m
      if (k == 0) return m < MD ? m * (LATE + kFrags) / MD : LATE + kFrags;
      return m < P / 2 ? 0 : m < P / 2 + MD / 2 ? (m - P / 2) * kReady / (MD / 2) : kReady;
    };
    each(std::make_integer_sequence<int, P>{}, [&](auto mc) {
      constexpr int m = decltype(mc)::value, b = m / (P / 4), q = m % (P / 4), d0 = due(m), d1 = due(m + 1);
      constexpr int i = b == 0 ? q / HN : b == 1 ? q % HM : b == 2 ? HM + q / HN : HM + q % HM, j = b == 0 ? q % HN : b == 1 ? HN + q / HM : b == 2 ? HN + q % HN : q / HM;
      if constexpr (k == 1 && m == 0) meet();                  // everyone has read this stage
      if constexpr (k == 1 && m == P / 2) wait_and_meet<VH>(); // the next stage is there
      multiply(acc[i][j], fb[k][0][j], fa[k][0][i]);
      each(std::make_integer_sequence<int, d1 - d0>{}, [&](auto dc) {
        constexpr int d = d0 + decltype(dc)::value;
        if constexpr (k == 1) fetch(d, 0, next, 0);            // the next step's first
        else if constexpr (d < LATE) fetch(kReady + d, 0, stage, 0);   // what is missing of this product's
        else fetch(d - LATE, 1, stage, 1);                     // the next one's
      });
      if constexpr (k == 0 && m + 3 >= P) advance(m + 3 - P);
      if constexpr (k == 1 && m % EACH == EACH - 2) aim(m / EACH, stage, v, to);
      if constexpr (k == 1 && m % EACH == EACH - 1) go(m / EACH, v, to);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (kSums)
      if (take && k == wn) sum_up(k);
  };
  for (int t = 0; t < steps; ++t) {
    const int next = stage + 1 == STAGES ? 0 : stage + 1;
    const bool take = kSums && t == sums_at;
    if (take) sums_at += g.tiles_j;
    if constexpr (EARLY) {
      early_step(std::integral_constant<int, 0>{}, next, take);
      early_step(std::integral_constant<int, 1>{}, next, take);
    } else {
      step(std::integral_constant<int, 0>{}, next, take);
      step(std::integral_constant<int, 1>{}, next, take);
      if constexpr (NK > 2) {
        step(std::integral_constant<int, 2>{}, next, take);
        step(std::integral_constant<int, 3>{}, next, take);
      }
    }
    refill = stage;
    stage = next;
  }

  // ---- out: 32 rows of a wave's share at a time through LDS, so that memory sees whole rows of it.  What the epilogue reads beside them is asked for
  // up front, all of it (the fragments' registers are free), and passes through LDS, too, where a loop can index it: one wave a SIMD has nothing
  // else to hide a wait behind, and a copy of the code for each pass would not fit the instruction cache.
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the steps past the end have arrived too
  if constexpr (kSums) {
    if (g.sums) {
      float *to = g.sums + ((size_t)(split * g.tiles_j + tj) * 2 + wn) * g.I;
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        float s = sums[i] + __shfl_xor(sums[i], 32, 64);
        if (FR == 16) s += __shfl_xor(s, 16, 64);
        const long long at = i0 + wm * WTM + i * FR + lr;
        if (lg == 0 && at < g.I) to[at] = s;
      }
    }
  }
  if constexpr (NP == 3) {
    int bad = 0;
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) bad |= !(fabsf(acc[i][j][e]) <= 3.4028234e38f);
    // the blocks of 64x64 whose values went into this tile
    const int r0 = (int)(rbeg >> 6), r1 = (int)((rend + 63) >> 6), nr = r1 - r0, wide_a = AR ? (int)((g.R + 63) >> 6) : (int)((g.I + 63) >> 6),
              wide_b = BR ? (int)((g.R + 63) >> 6) : (g.J + 63) >> 6;
    const int ia = (int)(i0 >> 6), na = (int)min((long long)BM / 64, ((g.I + 63) >> 6) - ia), jb = j0 >> 6, nb = min(BN / 64, ((g.J + 63) >> 6) - jb);
    for (int u = tid; u < nr * na; u += kThreads) {
      const int r = r0 + u / na, i = ia + u % na;
      bad |= g.flags_a[AR ? (size_t)i * wide_a + r : (size_t)r * wide_a + i];
    }
    for (int u = tid; u < nr * nb; u += kThreads) {
      const int r = r0 + u / nb, j = jb + u % nb;
      bad |= g.flags_b[BR ? (size_t)j * wide_b + r : (size_t)r * wide_b + j];
    }
    if (__syncthreads_or(bad)) {
      const u64 base = g.e.d.rng && g.splits == 1 ? dropout_base(g.e.d.rng) : 0;
      plain_tile<AR, BR, BM, BN>(g, i0, j0, rbeg, rend, lds, [&](long long i, int j, float v) {
        if (g.splits > 1) g.part[((long long)split * g.I + i) * g.J + j] = v;
        else finish<O>(g.e, i, j, v, base);
      });
      return;
    }
  }
  const bool whole = g.splits == 1;
  const u64 base = g.e.d.rng && whole ? dropout_base(g.e.d.rng) : 0;
  constexpr int LPR = WTN / 8, RPP = 64 / LPR, PASSES = 32 / RPP;   // lanes a row, rows a pass, passes of 32 rows
  static_assert(PASSES % 2 == 0 && (!AR || sizeof(Raw8<O>) * PASSES * 64 <= (size_t)kSide), "passes");
  char *const mine = lds + wave * (32 * kPitch + kSide);
  Raw8<O> *const mine_side = reinterpret_cast<Raw8<O> *>(mine + 32 * kPitch) + lane;   // a lane's own
  const int c = (lane % LPR) * 8, j = j0 + wn * WTN + c, left = g.J - j;
  const long long row0 = i0 + wm * WTM + lane / LPR;
  const int rows = left <= 0 ? 0 : (int)min(g.I - row0, (long long)BM);   // of the operand from this lane's first on
  auto put = [&](auto kc) {
    constexpr int k = decltype(kc)::value;
#pragma unroll
    for (int i = 0; i < 32 / FR; ++i)
#pragma unroll
      for (int n = 0; n < FN; ++n)
#pragma unroll
        for (int q = 0; q < FR * FR / 256; ++q) {
          const auto &c = acc[k * (32 / FR) + i][n];
          *reinterpret_cast<f32x4 *>(mine + (i * FR + lr) * kPitch + (n * FR + q * 8 + lg * 4) * 4) = f32x4{c[q * 4], c[q * 4 + 1], c[q * 4 + 2], c[q * 4 + 3]};
        }
    asm volatile("" ::"n"(k));   // left alone, the compiler makes one of the calls, with an index, and keeps the sums in memory for it
  };
  auto meet_lanes = [&]() {   // LDS takes a wave's accesses in order: it is the compiler that has to
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  f32x4 v0, v1;
  auto get = [&](int p) {   // pass p of the 32 rows
    const char *at = mine + (p * RPP + lane / LPR) * kPitch + c * 4;
    v0 = *reinterpret_cast<const f32x4 *>(at);
    v1 = *reinterpret_cast<const f32x4 *>(at + 16);
  };
  if (j0 + BN > g.J || (whole && (g.e.act != RESIST_ACT_NONE || g.e.d.rng || g.e.z_out || g.e.res || g.e.z_in))) {
    // Addresses are a base for the wave, which goes on from pass to pass, and a lane's part, which does not
    long long ld_side;
    const O *side0 = side_of<O>(g.e, ld_side);
    const long long wrow = i0 + wm * WTM, wcol = j0 + wn * WTN;
    const int lrow = lane / LPR;
    const char *side = reinterpret_cast<const char *>(side0 + wrow * ld_side + wcol);
    const unsigned vside = (unsigned)((lrow * ld_side + c) * sizeof(O)), vout = (unsigned)((lrow * g.e.ldo + c) * sizeof(O)), vz = (unsigned)((lrow * g.e.ldz + c) * sizeof(O)),
                   vpart = (unsigned)(((long long)lrow * g.J + c) * 4);
    char *out = reinterpret_cast<char *>(static_cast<O *>(g.e.out) + wrow * g.e.ldo + wcol), *z_out = reinterpret_cast<char *>(static_cast<O *>(g.e.z_out) + wrow * g.e.ldz + wcol),
         *part = reinterpret_cast<char *>(g.part + ((long long)split * g.I + wrow) * g.J + wcol);
    u64 word = base + ((u64)row0 * (unsigned)g.e.words + (unsigned)(j >> 1)) * kGolden;
    const u64 word_step = (u64)(RPP * (unsigned)g.e.words) * kGolden;
    constexpr bool kSided = AR;   // a weight gradient has nothing beside it
    const bool has_side = kSided && whole && (g.e.z_in || g.e.res), early = has_side && j0 + BN <= g.J;
    float bias[8] = {};
    if (whole) bias_of(g.e, j, left, bias);
    Raw8<O> ahead[kSided ? TM : 1][PASSES];
    if (kSided && early) {
#pragma unroll
      for (int k = 0; k < TM; ++k)
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
          const int r = (k * PASSES + p) * RPP;
          raw_load(side0 + (rows > 0 ? row0 + (r < rows ? r : 0) : 0) * ld_side + j, 8, ahead[kSided ? k : 0][p]);   // of a row that is there, whichever
        }
    }
    auto bring = [&](auto kc) {
      put(kc);
      if (kSided && early) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) mine_side[p * 64] = ahead[kSided ? decltype(kc)::value : 0][p];
      }
    };
    int at = 0;   // rows behind
#pragma unroll 1
    for (int k = 0; k < TM; ++k) {
      if (k == 0) bring(std::integral_constant<int, 0>{});
      if (TM > 1 && k == 1) bring(std::integral_constant<int, TM - 1 < 1 ? TM - 1 : 1>{});
      if (TM > 2 && k == 2) bring(std::integral_constant<int, TM - 1 < 2 ? TM - 1 : 2>{});
      if (TM > 3 && k == 3) bring(std::integral_constant<int, TM - 1 < 3 ? TM - 1 : 3>{});
      meet_lanes();
#pragma unroll 1
      for (int p = 0; p < PASSES; p += 2, at += 2 * RPP) {
        float v[2][8];
        Raw8<O> vs[2] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          get(p + h);
#pragma unroll
          for (int e = 0; e < 4; ++e) { v[h][e] = v0[e]; v[h][e + 4] = v1[e]; }
          if (early) vs[h] = mine_side[(p + h) * 64];
        }
        const bool ok[2] = {at < rows, at + RPP < rows};
        if (whole) {
          if (has_side && !early) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (ok[h]) raw_load(reinterpret_cast<const O *>(side + h * RPP * ld_side * (int)sizeof(O) + vside), left, vs[h]);
          }
          O *const outs[2] = {reinterpret_cast<O *>(out + vout), reinterpret_cast<O *>(out + RPP * g.e.ldo * (int)sizeof(O) + vout)};
          O *const zs[2] = {reinterpret_cast<O *>(z_out + vz), reinterpret_cast<O *>(z_out + RPP * g.e.ldz * (int)sizeof(O) + vz)};
          const u64 words[2] = {word, word + word_step};
          finish_rows<O, 2>(g.e, outs, zs, words, left, ok, v, bias, vs);
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (ok[h]) row_store(reinterpret_cast<float *>(part + h * (long long)RPP * g.J * 4 + vpart), left, v[h]);
        }
        side += 2 * RPP * ld_side * (int)sizeof(O);
        part += 2 * (long long)RPP * g.J * 4;
        out += 2 * RPP * g.e.ldo * (int)sizeof(O);
        z_out += 2 * RPP * g.e.ldz * (int)sizeof(O);
        word += 2 * word_step;
      }
      meet_lanes();
    }
  } else {
    // Sums on their own, or with a bias, in whole vectors: a pass is little more than its store, unrolled
    float bias[8] = {};
    if (whole) bias_of(g.e, j, 8, bias);
    auto all = [&](auto *out, long long ld) {
      auto chunk = [&](auto kc) {
        constexpr int k = decltype(kc)::value;
        if constexpr (k < TM) {
          put(kc);
          meet_lanes();
#pragma unroll
          for (int p = 0; p < PASSES; ++p) {
            get(p);
            float v[8] = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += bias[e];
            if ((k * PASSES + p) * RPP < rows) Row<std::remove_pointer_t<decltype(out)>>::store(out, v);
            out += RPP * ld;
          }
          meet_lanes();
        }
      };
      chunk(std::integral_constant<int, 0>{});
      chunk(std::integral_constant<int, 1>{});
      chunk(std::integral_constant<int, 2>{});
      chunk(std::integral_constant<int, 3>{});
    };
    if (whole) all(static_cast<O *>(g.e.out) + row0 * g.e.ldo + j, g.e.ldo);
    else all(g.part + ((long long)split * g.I + row0) * g.J + j, (long long)g.J);
  }
}

// What follows a split reduction and the sums of columns: workgroups 0 .. sum_wgs-1 join `sum_parts` rows of sums of 64 columns each, in float64,
// the others the parts of eight outputs a thread; in order.
struct JoinArgs {
  const float *part, *sums;
  float *db;
  long long I;
  int splits, J, sum_parts, sum_n, sum_wgs;
  Epilogue e;
};
template <typename O>
__global__ __launch_bounds__(kThreads) void gemm_join_kernel(JoinArgs a) {
  if ((int)blockIdx.x < a.sum_wgs) {
    __shared__ double red[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), k = threadIdx.x >> 6;
    const double s = c < a.sum_n ? parts_sum<16>(a.sums + c, (size_t)a.sum_n, k, 4, a.sum_parts) : 0.;
    red[k][threadIdx.x & 63] = s;
    __syncthreads();
    if (k == 0 && c < a.sum_n) a.db[c] = (float)(((red[0][threadIdx.x] + red[1][threadIdx.x]) + red[2][threadIdx.x]) + red[3][threadIdx.x]);
    return;
  }
  const int nvec = (a.J + 7) / 8;
  const long long u = (long long)(blockIdx.x - a.sum_wgs) * kThreads + threadIdx.x;
  const long long row = u / nvec;
  const int j = (int)(u - row * nvec) * 8, left = a.J - j;
  if (row >= a.I) return;
  float bias[8];
  bias_of(a.e, j, left, bias);
  long long ld;
  const O *side = side_of<O>(a.e, ld);
  Raw8<O> now[1] = {};
  if (side) raw_load(side + row * ld + j, left, now[0]);
  float v[1][8];
  row_load(a.part + row * a.J + j, left, v[0]);
  for (int s = 1; s < a.splits; s += 3) {   // three on their way at once (past the last one that again)
    float w[3][8];
#pragma unroll
    for (int u = 0; u < 3; ++u) row_load(a.part + ((long long)min(s + u, a.splits - 1) * a.I + row) * a.J + j, left, w[u]);
#pragma unroll
    for (int u = 0; u < 3; ++u)
#pragma unroll
      for (int k = 0; k < 8; ++k) v[0][k] += s + u < a.splits ? w[u][k] : 0.f;
  }
  O *const out[1] = {static_cast<O *>(a.e.out) + row * a.e.ldo + j}, *const z_out[1] = {static_cast<O *>(a.e.z_out) + row * a.e.ldz + j};
  const u64 word[1] = {a.e.d.rng ? dropout_base(a.e.d.rng) + ((u64)row * (unsigned)a.e.words + (unsigned)(j >> 1)) * kGolden : 0};
  const bool ok[1] = {true};
  finish_rows<O, 1>(a.e, out, z_out, word, left, ok, v, bias, now);
}

// ---- few rows -------------------------------------------------------------------------------------------------------
// The time is that of reading w once (forward, data gradient) or of writing dw once, so w comes straight from memory into fragments, from rows that
// start anywhere, several loads in flight, and nothing is laid out.  16 of w by 16 rows, MG times, on v_mfma_f32_16x16x32_bf16 or
// v_mfma_f32_16x16x4_f32.  A workgroup's eight waves take every eighth piece of its range of the reduction, and their sums are joined in LDS,
// in order; where there are few workgroups the reduction is split among several (gemm_join_kernel).  Rows and columns past the last are
// read as the last one and not stored.
struct FewArgs {
  const void *a, *w;        // x or dz, [M][K] or [M][N]
  long long lda;
  int M, K, N;
  int splits, per;          // ranges of the reduction, one per blockIdx.y; their length
  float *part;              // [splits][M][outputs of a row]
  Epilogue e;
};
template <typename T> struct Four;   // four elements
template <> struct Four<float> { typedef f32x4 Raw; typedef f32x4_any Any; };
typedef u32x2 u32x2_any __attribute__((aligned(2)));
template <> struct Four<__bf16> { typedef u32x2 Raw; typedef u32x2_any Any; };
__device__ inline f32x4 widen4(const f32x4 &r) { return r; }
__device__ inline f32x4 widen4(const u32x2 &r) { return f32x4{bf16_lo(r[0]), bf16_hi(r[0]), bf16_lo(r[1]), bf16_hi(r[1])}; }
// 16 or 8 bytes of a row from element k on, with zeros from element n on
template <typename T, typename Raw> __device__ inline Raw piece(const T *p, int k, int n) {
  constexpr int V = (int)(sizeof(Raw) / sizeof(T));
  Raw out = {};
#pragma unroll
  for (int e = 0; e < V; ++e)
    if (k + e < n) {
      if constexpr (sizeof(T) == 4) out[e] = p[k + e];
      else out[e >> 1] |= (unsigned)__builtin_bit_cast(unsigned short, p[k + e]) << (e & 1 ? 16 : 0);
    }
  return out;
}

// y = x w': 16 rows of w to a workgroup
template <typename T, int MG>
__global__ __launch_bounds__(512) void few_rows_fwd_kernel(FewArgs a) {
  constexpr int V = 16 / (int)sizeof(T), STEP = 4 * V, AHEAD = MG == 1 ? 8 : 4;   // elements a lane, of the reduction a wave and load; loads in flight
  typedef std::conditional_t<sizeof(T) == 4, f32x4, u32x4> Piece;
  typedef std::conditional_t<sizeof(T) == 4, f32x4_any, u32x4_any> Any;
  __shared__ float red[8][16][17];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, kk = (lane >> 4) * V;
  const int beg = blockIdx.y * a.per, end = min(a.K, beg + a.per);
  const T *w = static_cast<const T *>(a.w) + (long long)min((int)blockIdx.x * 16 + row, a.N - 1) * a.K, *x[MG];
#pragma unroll
  for (int g = 0; g < MG; ++g) x[g] = static_cast<const T *>(a.a) + min(g * 16 + row, a.M - 1) * a.lda;
  f32x4 acc[MG] = {};
  auto multiply = [&](const Piece &fw, const Piece (&fx)[MG]) {
#pragma unroll
    for (int g = 0; g < MG; ++g) {
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[e], fx[g][e], acc[g], 0, 0, 0);
      } else {
        acc[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw), __builtin_bit_cast(bf16x8, fx[g]), acc[g], 0, 0, 0);
      }
    }
  };
  int k0 = beg + wave * STEP;
  for (; k0 + (AHEAD * 8 - 7) * STEP <= end; k0 += 8 * STEP * AHEAD) {   // all of these pieces are whole
    Piece fw[AHEAD], fx[AHEAD][MG];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      fw[u] = *reinterpret_cast<const Any *>(w + k0 + u * 8 * STEP + kk);
#pragma unroll
      for (int g = 0; g < MG; ++g) fx[u][g] = *reinterpret_cast<const Any *>(x[g] + k0 + u * 8 * STEP + kk);
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) multiply(fw[u], fx[u]);
  }
#pragma unroll 1
  for (; k0 < end; k0 += 8 * STEP) {
    Piece fw, fx[MG];
    if (k0 + STEP <= end) {
      fw = *reinterpret_cast<const Any *>(w + k0 + kk);
#pragma unroll
      for (int g = 0; g < MG; ++g) fx[g] = *reinterpret_cast<const Any *>(x[g] + k0 + kk);
    } else {
      fw = piece<T, Piece>(w, k0 + kk, end);
#pragma unroll
      for (int g = 0; g < MG; ++g) fx[g] = piece<T, Piece>(x[g], k0 + kk, end);
    }
    multiply(fw, fx);
  }
  const u64 base = a.e.d.rng && a.splits == 1 ? dropout_base(a.e.d.rng) : 0;
#pragma unroll
  for (int g = 0; g < MG; ++g) {
    if (g > 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) red[wave][row][(lane >> 4) * 4 + e] = acc[g][e];   // lane: row `row` of x, four columns
    __syncthreads();
    const int m = g * 16 + (threadIdx.x >> 4), c = threadIdx.x & 15, j = blockIdx.x * 16 + c;
    if (threadIdx.x < 256 && m < a.M && j < a.N) {
      float v = red[0][m & 15][c];
#pragma unroll
      for (int s = 1; s < 8; ++s) v += red[s][m & 15][c];
      if (a.splits > 1) a.part[((long long)blockIdx.y * a.M + m) * a.N + j] = v;
      else finish<T>(a.e, m, j, v, base);
    }
  }
}

// dx = dz w in fp32: 64 columns of w to a workgroup.  A lane loads four columns of four rows and four elements of dz: 16 of the reduction a wave
// and piece.  Column 4 i + c of the 64 is row i of the c-th product, so that a lane ends up with 16 columns next to each other.  (In bf16 the
// tiles read half the bytes and are as quick.)
template <int MG>
__global__ __launch_bounds__(512) void few_rows_dgrad_kernel(FewArgs a) {
  constexpr int AHEAD = MG == 4 ? 2 : 4;
  __shared__ float red[8][16][65];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 15, nn = (lane >> 4) * 4;
  const int c0 = blockIdx.x * 64 + row * 4, beg = blockIdx.y * a.per, end = min(a.N, beg + a.per);
  const bool inside = blockIdx.x * 64 + 64 <= (unsigned)a.K;
  const float *w = static_cast<const float *>(a.w), *z[MG];
#pragma unroll
  for (int g = 0; g < MG; ++g) z[g] = static_cast<const float *>(a.a) + min(g * 16 + row, a.M - 1) * a.lda;
  f32x4 acc[MG][4] = {};
  auto multiply = [&](const f32x4 (&fw)[4], const f32x4 (&fz)[MG]) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int g = 0; g < MG; ++g)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[g][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(fw[e][c], fz[g][e], acc[g][c], 0, 0, 0);
  };
  int n0 = beg + wave * 16;
  if (inside)
    for (; n0 + (AHEAD * 8 - 7) * 16 <= end; n0 += 8 * 16 * AHEAD) {   // all of these pieces are whole
      f32x4 fw[AHEAD][4], fz[AHEAD][MG];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const int n = n0 + u * 8 * 16 + nn;
#pragma unroll
        for (int e = 0; e < 4; ++e) fw[u][e] = *reinterpret_cast<const f32x4_any *>(w + (long long)(n + e) * a.K + c0);
#pragma unroll
        for (int g = 0; g < MG; ++g) fz[u][g] = *reinterpret_cast<const f32x4_any *>(z[g] + n);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) multiply(fw[u], fz[u]);
    }
#pragma unroll 1
  for (; n0 < end; n0 += 8 * 16) {
    const int n = n0 + nn;
    f32x4 fw[4], fz[MG];
#pragma unroll
    for (int e = 0; e < 4; ++e) fw[e] = n + e < end ? piece<float, f32x4>(w + (long long)(n + e) * a.K, c0, a.K) : f32x4{};
#pragma unroll
    for (int g = 0; g < MG; ++g) fz[g] = piece<float, f32x4>(z[g], n, end);
    multiply(fw, fz);
  }
  const u64 base = a.e.d.rng && a.splits == 1 ? dropout_base(a.e.d.rng) : 0;
#pragma unroll
  for (int g = 0; g < MG; ++g) {
    if (g > 0) __syncthreads();
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) red[wave][row][(lane >> 4) * 16 + r * 4 + c] = acc[g][c][r];
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = (threadIdx.x >> 6) + h * 8, m = g * 16 + r, c = threadIdx.x & 63, j = blockIdx.x * 64 + c;
      if (m >= a.M || j >= a.K) continue;
      float v = red[0][r][c];
#pragma unroll
      for (int s = 1; s < 8; ++s) v += red[s][r][c];
      if (a.splits > 1) a.part[((long long)blockIdx.y * a.M + m) * a.K + j] = v;
      else finish<float>(a.e, m, j, v, base);
    }
  }
}

// dw = dz' x, db: 64 rows by 256 columns of dw to a workgroup, 16 rows to a wave, four columns of all rows of x in each lane's registers.
template <typename T, int MR>
__global__ __launch_bounds__(kThreads) void few_rows_wgrad_kernel(const T *dz, long long ldz, const T *x, long long ldx, int M, int N, int K, float *dw, float *db) {
  __shared__ __attribute__((aligned(16))) float z[64][MR + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n0 = blockIdx.y * 64, c = blockIdx.x * 256 + lane * 4;
  for (int u = threadIdx.x; u < 64 * MR; u += kThreads) {
    const int m = u >> 6, n = u & 63;
    z[n][m] = m < M && n0 + n < N ? (float)dz[m * ldz + n0 + n] : 0.f;
  }
  f32x4 v[MR];
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    typename Four<T>::Raw r = {};
    if (m < M && c + 4 <= K) r = *reinterpret_cast<const typename Four<T>::Any *>(x + m * ldx + c);
    else if (m < M) r = piece<T, typename Four<T>::Raw>(x + m * ldx, c, K);
    v[m] = widen4(r);
  }
  __syncthreads();
  if (db && blockIdx.x == 0 && threadIdx.x < 64 && n0 + (int)threadIdx.x < N) {
    float s = 0.f;
#pragma unroll
    for (int m = 0; m < MR; ++m) s += z[threadIdx.x][m];
    db[n0 + threadIdx.x] = s;
  }
  const int left = K - c;
  for (int r = 0; r < 16; ++r) {
    const int n = wave * 16 + r;
    if (n0 + n >= N || left <= 0) break;
    f32x4 s = {};
#pragma unroll
    for (int m = 0; m < MR; m += 4) {
      const f32x4 q = *reinterpret_cast<const f32x4 *>(&z[n][m]);
#pragma unroll
      for (int e = 0; e < 4; ++e) s += q[e] * v[m + e];
    }
    float *to = dw + (long long)(n0 + n) * K + c;
    if (left >= 4) {
      *reinterpret_cast<f32x4_any *>(to) = s;
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (e < left) to[e] = s[e];
    }
  }
}

// ---- plans ----------------------------------------------------------------------------------------------------------
// Up to this many rows go without tiles; a bf16 forward pass of more than 16 rows does while its weights are few (fewer of odd length, whose rows start anywhere).
// us, 4096 -> 4096, tiles (with what they lay out and join) -> few rows:
//   fp32 1 row: forward 50 -> 15, data gradient 53 -> 16, weight gradient 33 -> 13      17 rows: 50 -> 20, 55 -> 20, 34 (tiles)
//   fp32 64 rows: 51 -> 39, 55 -> 41     bf16 1 row: forward 11.6 -> 7.4 (4.5 TB/s), data gradient 11 (tiles; 40 with 64 columns to a workgroup), weight gradient 23 -> 13.4 (5 TB/s)
//   bf16 16 rows: forward 12.5 -> 10.1, weight gradient 24 -> 16.5
// bf16 forward, 17 | 32 rows, tiles -> few rows:  512 -> 512 5.8 -> 3.7 | 5.8 -> 4.0     1024 -> 4096 8.6 -> 5.6 | 8.7 -> 6.4     2048 -> 2048 9.6 -> 8.0 | 9.8 -> 9.4
//   2048 -> 8192 12.3 -> 12.9 | 12.6 -> 15.9     4096 -> 4096 12.3 -> 13.7 | 12.6 -> 16.2     8192 -> 2048 13.6 -> 23.0 | 13.7 -> 27.6
//   511 -> 512 9.6 -> 7.3 | 9.6 -> 8.8     1023 -> 1024 11.7 -> 10.9 | 11.7 -> 13.7     2047 -> 1024 13.5 -> 17.2 | 13.6 -> 22.7
int few(const LinearShape &s, int dt, int op) {
  if (op == 2) return 16;
  if (dt == DT_F32) return 64;
  if (op == 1) return 0;
  return (int64_t)s.K * s.N <= (s.K % 2 ? 1 << 19 : 1 << 22) ? 32 : 16;
}
// Ranges of the reduction: a few hundred workgroups where there are less than one for every other CU, as long as each wave has whole turns of loads.
struct FewPlan { int wgs, splits, per; };
FewPlan plan_few(int dt, int op, long long M, int J, int R) {
  FewPlan p;
  const int cols = op == 0 ? 16 : 64, groups = M <= 16 ? 1 : M <= 32 ? 2 : 4;
  const int turn = op == 0 ? 8 * (dt == DT_F32 ? 16 : 32) * (groups == 1 ? 8 : 4) : 8 * 16 * (groups == 4 ? 2 : 4);
  p.wgs = (J + cols - 1) / cols;
  p.splits = 1;
  if (p.wgs < 128) p.splits = std::max(1, std::min(R / turn, 384 / p.wgs));
  if (p.splits < 3) p.splits = 1;   // a launch more than they save
  p.per = ((R + p.splits - 1) / p.splits + turn - 1) / turn * turn;
  p.splits = (R + p.per - 1) / p.per;
  return p;
}

// Which tiles, and how many ranges of the reduction (`splits`): the least time by a model of the kernels, us, with what was measured alone on the chip:
// a launch, then rounds of as many workgroups as fit (one or two a CU), each its start and epilogue and `step` per 64 of the reduction
// (`low` with a quarter of that many, `half`, `full` with all: the clock gives way under the products, and two share a CU); a split reduction writes
// its parts and reads them back, from a cache, in a launch of its own.  Either side of the choice, us measured, bf16 forward unless said
// (M x K x N: 256x256 | 128x128 | 64x64):
//   8192x8192x2048  190 | 230 | 389     4096x2048x2048  46 | 35 | 55     512x4096x4096  76 | 35 | 28      64x512x512  16 | 7.9 | 5.4
//   128x4096x512, 64x64: 1 split 17.7, 2 13.4, 4 10.1, 8 10.0, 16 11.5   128x512x4096, 64x64: 1 split 5.7, 2 9.5, 4 11.7
//   fp32 (256x128 | 128x128 | 64x64)  8192x2048x2048  329 | 345 | 397     2048x1024x4096  94 | 99 | 109     2000x1024x1024  62 | 46 (2 splits 40) | 36
struct TileCost { int bm, bn, fit; double start, low, half, full; };
constexpr int kSizes = 3;
constexpr TileCost kTiles[2][kSizes] = {{{256, 256, 256, 10.0, 1.1, 1.25, 1.41}, {128, 128, 512, 4.0, 0.5, 0.53, 0.91}, {64, 64, 512, 1.4, 0.26, 0.27, 0.41}},
                                   {{256, 128, 256, 5.0, 2.9, 3.75, 4.6}, {128, 128, 256, 9.0, 1.5, 1.6, 2.15}, {64, 64, 512, 1.5, 0.65, 0.9, 1.55}}};
constexpr double kLaunch = 2.0, kJoin = 2.5, kJoinPart = 0.4, kBytesPerUs = 8e6;
struct Plan {
  int size;                  // of the tiles: an index into kTiles
  int bm, bn, splits;
  long long per_split;
};
// Ranges are of 2^18 of the reduction at most: a sum in fp32 that has grown past 2^20 of its terms loses their bits (plain_tile's, a term or two at a time:
// weight gradients of 2^28 rows in 32 ranges were off by 4e-3 of their magnitude, in 1025 by 2e-5).
constexpr long long kMostSteps = (1 << 18) / 64;
Plan plan_tiles(int np, long long I, long long J, long long R) {
  const long long steps = (R + 63) / 64, least_splits = (steps + kMostSteps - 1) / kMostSteps;
  Plan best{};
  double least = 0.;
  for (int size = 0; size < kSizes; ++size) {
    const TileCost &c = kTiles[np == 3][size];
    const long long tiles = ((I + c.bm - 1) / c.bm) * ((J + c.bn - 1) / c.bn);
    if (tiles > kMaxWgs && size > 0) continue;   // (of the largest: layout_of refuses the call)
    for (const int some : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32}) {
      const long long want = std::max<long long>(some, least_splits);
      if (want > least_splits && (want > steps / 4 || tiles * want > 2 * c.fit)) break;
      const long long per = (steps + want - 1) / want, splits = (steps + per - 1) / per, wgs = tiles * splits;
      const long long rounds = wgs / c.fit, rest = wgs - rounds * c.fit;
      double t = kLaunch + rounds * (c.start + per * c.full);
      if (rest > 0) t += c.start + per * (rest * 4 <= c.fit ? c.low : rest * 2 <= c.fit ? c.half : c.full);
      if (splits > 1) t += kJoin + kJoinPart * splits + 8. * splits * I * J / kBytesPerUs;
      if (best.splits == 0 || t < least) {
        least = t;
        best = Plan{size, c.bm, c.bn, (int)splits, per * 64};
      }
    }
  }
  return best;
}

// An operand of a call: `rows` rows of n elements; whether it has to be laid out, and where.
struct Operand {
  long long rows, ld;
  int n;
  bool moved, panels;
  long long to_ld, plane;    // as the kernel reads it
  int64_t at, flags_at;      // bytes into the workspace
};
struct Layout {
  Operand a, b;
  int np;
  Plan plan;
  int64_t part_at, sums_at, bytes;   // bytes: -1 of a call with more workgroups than a launch takes (2^40 outputs and more)
  int sum_parts;
};
int64_t align256(int64_t n) { return (n + 255) & ~(int64_t)255; }
int64_t blocks64(long long rows, long long n) { return ((rows + 63) / 64) * ((n + 63) / 64); }
// `whole`: the reduction is the contiguous axis, so that a row's end has to be one of eight elements
Operand operand(int dt, long long rows, int n, long long ld, bool whole, int64_t *at) {
  Operand o{rows, ld, n, false, false, ld, 0, 0, 0};
  o.moved = dt == DT_F32 || ld % 8 != 0 || (whole && n % 8 != 0);
  if (!o.moved) return o;
  o.panels = dt == DT_F32 && whole;
  o.to_ld = o.panels ? (n + 31) / 32 * 32 : (n + 7) / 8 * 8;
  o.plane = rows * o.to_ld;
  o.at = *at;
  *at += align256(o.plane * 2 * (dt == DT_F32 ? 3 : 1));
  if (dt == DT_F32) {
    o.flags_at = *at;
    *at += align256(blocks64(rows, n) * 4);
  }
  return o;
}
// op 0 forward, 1 data gradient, 2 weight gradient
Layout layout_of(const LinearShape &s, int dt, int op) {
  Layout l{};
  l.np = dt == DT_F32 ? 3 : 1;
  const long long I = op == 2 ? s.N : s.M, J = op == 0 ? s.N : s.K, R = op == 0 ? s.K : op == 1 ? s.N : s.M;
  l.plan = plan_tiles(l.np, I, J, R);
  int64_t at = 0;
  if (op == 0) {
    l.a = operand(dt, s.M, s.K, s.ldx, true, &at);
    l.b = operand(dt, s.N, s.K, s.K, true, &at);
  } else if (op == 1) {
    l.a = operand(dt, s.M, s.N, s.ldy, true, &at);
    l.b = operand(dt, s.N, s.K, s.K, false, &at);
  } else {
    l.a = operand(dt, s.M, s.N, s.ldy, false, &at);
    l.b = operand(dt, s.M, s.K, s.ldx, false, &at);
  }
  l.part_at = at;
  if (l.plan.splits > 1) at += align256(l.plan.splits * I * J * 4);
  if (op == 2) {
    l.sums_at = at;
    l.sum_parts = dt == DT_F32 ? (int)((s.M + 63) / 64) : (int)((J + l.plan.bn - 1) / l.plan.bn) * l.plan.splits * 2;
    at += align256((int64_t)l.sum_parts * s.N * 4);
  }
  const long long tiles = ((I + l.plan.bm - 1) / l.plan.bm) * ((J + l.plan.bn - 1) / l.plan.bn);
  l.bytes = tiles * l.plan.splits > kMaxWgs || blocks64(l.a.rows, l.a.n) + blocks64(l.b.rows, l.b.n) > 0x7fffffff ? -1 : at;
  return l;
}

template <typename O, bool AR, bool BR, int NP, int BM, int BN, int BK, int STAGES, int WGS> int launch_tiles(TileArgs &t, hipStream_t st) {
  t.tiles_i = (int)((t.I + BM - 1) / BM);
  t.tiles_j = (t.J + BN - 1) / BN;
  t.group = 8;
  const long long wgs = (long long)t.tiles_i * t.tiles_j * t.splits;
  gemm_tile_kernel<O, AR, BR, NP, BM, BN, BK, STAGES, WGS><<<(unsigned)wgs, kThreads, 0, st>>>(t);
  RESIST_CHECK_LAUNCH("linear");
  return RESIST_OK;
}

template <typename O> int join(const JoinArgs &j, hipStream_t st) {
  const long long wgs = j.sum_wgs + (j.splits > 1 ? (j.I * ((j.J + 7) / 8) + kThreads - 1) / kThreads : 0);
  if (wgs > kMaxWgs) return set_error(RESIST_ESHAPE, "linear: too many outputs");
  prof::Scope sc("linear_join", 0., j.splits > 1 ? (double)j.splits * j.I * j.J * 4 : 0., st);
  gemm_join_kernel<O><<<(unsigned)wgs, kThreads, 0, st>>>(j);
  RESIST_CHECK_LAUNCH("linear_join");
  return RESIST_OK;
}

// the product of a call, its operands laid out first where they have to be, what was split joined after
template <typename O, int NP, bool AR, bool BR>
int product(const Layout &l, const void *a, const void *b, long long I, int J, long long R, const Epilogue &e, float *db, void *work, const char *name,
            double flops, double bytes, hipStream_t st) {
  char *ws = static_cast<char *>(work);
  float *sums = db ? reinterpret_cast<float *>(ws + l.sums_at) : nullptr;
  if (l.a.moved || l.b.moved) {
    LayOutArgs args{};
    int n = 0;
    double moved = 0.;
    auto add = [&](const Operand &o, const void *from, float *to_sums) {
      if (!o.moved) return;
      LayOut &m = args.m[n++];
      m = LayOut{from, reinterpret_cast<__bf16 *>(ws + o.at), reinterpret_cast<unsigned *>(ws + o.flags_at), to_sums, o.rows, o.ld, o.plane, o.n, (int)o.to_ld, 0, 0, o.panels};
      m.blocks_n = (o.n + 63) / 64;
      m.blocks = (int)((o.rows + 63) / 64 * m.blocks_n);
      moved += (NP == 3 ? 10. : 4.) * o.rows * o.n;
    };
    add(l.a, a, NP == 3 ? sums : nullptr);
    add(l.b, b, nullptr);
    const long long blocks = (long long)args.m[0].blocks + args.m[1].blocks;
    prof::Scope sc("linear_lay_out", 0., moved, st);
    for (long long first = 0; first < blocks; first += kMaxWgs) {
      args.first = (int)first;
      lay_out_kernel<NP><<<(unsigned)std::min(kMaxWgs, blocks - first), kThreads, 0, st>>>(args);
      RESIST_CHECK_LAUNCH("linear_lay_out");
    }
  }
  TileArgs t{};
  t.a = reinterpret_cast<const __bf16 *>(l.a.moved ? ws + l.a.at : static_cast<const char *>(a));
  t.b = reinterpret_cast<const __bf16 *>(l.b.moved ? ws + l.b.at : static_cast<const char *>(b));
  t.lda = l.a.to_ld; t.ldb = l.b.to_ld; t.I = I; t.J = J; t.R = R;
  t.splits = l.plan.splits; t.per_split = l.plan.per_split; t.part = reinterpret_cast<float *>(ws + l.part_at);
  t.sums = NP == 1 ? sums : nullptr;
  if (NP == 3) {
    t.plane_a = l.a.plane; t.plane_b = l.b.plane;
    t.flags_a = reinterpret_cast<const unsigned *>(ws + l.a.flags_at); t.flags_b = reinterpret_cast<const unsigned *>(ws + l.b.flags_at);
    t.a32 = static_cast<const float *>(a); t.b32 = static_cast<const float *>(b); t.lda32 = l.a.ld; t.ldb32 = l.b.ld;
  }
  t.e = e;
  {
    prof::Scope sc(name, flops, bytes, st);
    if constexpr (NP == 1) {
      if (l.plan.size == 0) RESIST_TRY((launch_tiles<O, AR, BR, 1, 256, 256, 64, 2, 1>(t, st)));
      else if (l.plan.size == 1) RESIST_TRY((launch_tiles<O, AR, BR, 1, 128, 128, 64, 2, 2>(t, st)));
      else RESIST_TRY((launch_tiles<O, AR, BR, 1, 64, 64, 64, 4, 2>(t, st)));
    } else {
      if (l.plan.size == 0) RESIST_TRY((launch_tiles<O, AR, BR, 3, 256, 128, 32, 2, 1>(t, st)));
      else if (l.plan.size == 1) RESIST_TRY((launch_tiles<O, AR, BR, 3, 128, 128, 32, 3, 1>(t, st)));
      else RESIST_TRY((launch_tiles<O, AR, BR, 3, 64, 64, 32, 3, 2>(t, st)));
    }
  }
  if (t.splits == 1 && !db) return RESIST_OK;
  JoinArgs j{};
  j.part = t.part; j.splits = t.splits; j.I = I; j.J = J; j.e = e;
  j.sums = sums; j.db = db; j.sum_parts = l.sum_parts; j.sum_n = (int)I; j.sum_wgs = db ? (int)((I + 63) / 64) : 0;
  return join<O>(j, st);
}

double flops_of(const LinearShape &s) { return 2. * s.M * s.N * s.K; }
// forward (op 0) or data gradient (op 1, fp32) of few rows
int few_rows(const LinearShape &s, int dt, int op, const void *a, int64_t lda, const void *w, const Epilogue &e, void *work, const char *name, double bytes, hipStream_t st) {
  const int J = op == 0 ? s.N : s.K;
  const FewPlan p = plan_few(dt, op, s.M, J, op == 0 ? s.K : s.N);
  const FewArgs f{a, w, lda, (int)s.M, s.K, s.N, p.splits, p.per, static_cast<float *>(work), e};
  const dim3 wgs(p.wgs, p.splits);
  {
    prof::Scope sc(name, flops_of(s), bytes, st);
    if (op == 1) {
      if (s.M <= 16) few_rows_dgrad_kernel<1><<<wgs, 512, 0, st>>>(f);
      else if (s.M <= 32) few_rows_dgrad_kernel<2><<<wgs, 512, 0, st>>>(f);
      else few_rows_dgrad_kernel<4><<<wgs, 512, 0, st>>>(f);
    } else if (dt == DT_F32) {
      if (s.M <= 16) few_rows_fwd_kernel<float, 1><<<wgs, 512, 0, st>>>(f);
      else if (s.M <= 32) few_rows_fwd_kernel<float, 2><<<wgs, 512, 0, st>>>(f);
      else few_rows_fwd_kernel<float, 4><<<wgs, 512, 0, st>>>(f);
    } else {
      if (s.M <= 16) few_rows_fwd_kernel<__bf16, 1><<<wgs, 512, 0, st>>>(f);
      else few_rows_fwd_kernel<__bf16, 2><<<wgs, 512, 0, st>>>(f);
    }
    RESIST_CHECK_LAUNCH(name);
  }
  if (p.splits == 1) return RESIST_OK;
  JoinArgs j{};
  j.part = f.part; j.splits = p.splits; j.I = s.M; j.J = J; j.e = e;
  return dt == DT_F32 ? join<float>(j, st) : join<__bf16>(j, st);
}
double bytes_of(const LinearShape &s, int dt, double outs) { return ((double)s.M * s.K + (double)s.N * s.K + (double)s.M * s.N) * esize(dt) + outs; }

}  // namespace

int64_t linear_workspace(const LinearShape &s, int dt, int op) {
  if (s.M == 0) return 0;
  if (s.M <= few(s, dt, op)) {
    if (op == 2) return 0;
    const int J = op == 0 ? s.N : s.K;
    const FewPlan p = plan_few(dt, op, s.M, J, op == 0 ? s.K : s.N);
    return p.splits > 1 ? align256((int64_t)p.splits * s.M * J * 4) : 0;
  }
  return layout_of(s, dt, op).bytes;
}

int linear_fwd(const LinearShape &s, int dt, const void *x, const void *w, const LinearEpilogue &le, void *y, void *work, hipStream_t st) {
  if (s.M == 0) return RESIST_OK;
  Epilogue e{};
  e.out = y; e.ldo = s.ldy; e.bias = le.bias; e.z_out = le.z; e.ldz = le.ldz; e.res = le.residual; e.ldr = le.ldr; e.act = le.act;
  e.d = make_dropout(le.drop); e.words = (s.N + 1) / 2;
  const double bytes = bytes_of(s, dt, (double)s.M * s.N * esize(dt) * ((le.z != nullptr) + (le.residual != nullptr)));
  if (s.M <= few(s, dt, 0)) return few_rows(s, dt, 0, x, s.ldx, w, e, work, "linear_few_rows_fwd", bytes, st);
  const Layout l = layout_of(s, dt, 0);
  return dt == DT_F32 ? product<float, 3, true, true>(l, x, w, s.M, s.N, s.K, e, nullptr, work, "linear_fwd", flops_of(s), bytes, st)
                      : product<__bf16, 1, true, true>(l, x, w, s.M, s.N, s.K, e, nullptr, work, "linear_fwd", flops_of(s), bytes, st);
}

int linear_dgrad(const LinearShape &s, int dt, const void *dz, const void *w, const LinearThrough &lt, void *dx, void *work, hipStream_t st) {
  if (s.M == 0) return RESIST_OK;
  Epilogue e{};
  e.out = dx; e.ldo = s.ldx; e.z_in = lt.act == RESIST_ACT_NONE ? nullptr : lt.z; e.ldz = lt.ldz; e.act = lt.act;
  e.d = make_dropout(lt.drop); e.words = (s.K + 1) / 2;
  const double bytes = bytes_of(s, dt, e.z_in ? (double)s.M * s.K * esize(dt) : 0.);
  if (s.M <= few(s, dt, 1)) return few_rows(s, dt, 1, dz, s.ldy, w, e, work, "linear_few_rows_dgrad", bytes, st);
  const Layout l = layout_of(s, dt, 1);
  return dt == DT_F32 ? product<float, 3, true, false>(l, dz, w, s.M, s.K, s.N, e, nullptr, work, "linear_dgrad", flops_of(s), bytes, st)
                      : product<__bf16, 1, true, false>(l, dz, w, s.M, s.K, s.N, e, nullptr, work, "linear_dgrad", flops_of(s), bytes, st);
}

int linear_wgrad(const LinearShape &s, int dt, const void *dz, const void *x, float *dw, float *db, void *work, hipStream_t st) {
  const double bytes = ((double)s.M * s.K + (double)s.M * s.N) * esize(dt) + 4. * s.N * s.K;
  if (s.M <= few(s, dt, 2)) {
    const dim3 wgs((s.K + 255) / 256, (s.N + 63) / 64);
    const int M = (int)s.M;
    prof::Scope sc("linear_few_rows_wgrad", flops_of(s), bytes, st);
    auto launch = [&](auto kernel, auto type) {
      typedef decltype(type) T;
      kernel<<<wgs, kThreads, 0, st>>>(static_cast<const T *>(dz), s.ldy, static_cast<const T *>(x), s.ldx, M, s.N, s.K, dw, db);
    };
    if (dt == DT_F32) {
      if (M <= 4) launch(few_rows_wgrad_kernel<float, 4>, float{});
      else launch(few_rows_wgrad_kernel<float, 16>, float{});
    } else {
      if (M <= 4) launch(few_rows_wgrad_kernel<__bf16, 4>, __bf16{});
      else launch(few_rows_wgrad_kernel<__bf16, 16>, __bf16{});
    }
    RESIST_CHECK_LAUNCH("linear_few_rows_wgrad");
    return RESIST_OK;
  }
  Epilogue e{};
  e.out = dw; e.ldo = s.K;
  const Layout l = layout_of(s, dt, 2);
  return dt == DT_F32 ? product<float, 3, false, false>(l, dz, x, s.N, s.K, s.M, e, db, work, "linear_wgrad", flops_of(s), bytes, st)
                      : product<float, 1, false, false>(l, dz, x, s.N, s.K, s.M, e, db, work, "linear_wgrad", flops_of(s), bytes, st);
}

}  // namespace resist

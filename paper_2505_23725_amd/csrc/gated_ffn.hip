// The gated feed-forward block and its gradient, on the matrix cores.
//
//   g = x Wg^T ; u = x Wu^T ; h = act(g) u ; y = h Wd^T                              x [t][d], Wg, Wu [f][d], Wd [d][f]
//   dh = dy Wd ; dg = dh u act'(g) ; du = dh act(g)
//   dx = dg Wg + du Wu ; dWg = dg^T x ; dWu = du^T x ; dWd = dy^T h
//
// in five kernels of one tile scheme, which differ in how their operands lie in memory and in what is done with the
// accumulators:
//   UP    both projections at once: the tile's columns are half columns of g and half of u, dealt to the lanes so that a lane
//         holds g and u of the same elements; h leaves from there, and for training the factors of the gradients, act(g)
//         and u act'(g)
//   NT    y = h Wd^T
//   DH    dy Wd, whose accumulators times the two factors are du and dg
//   NN    dx: one sum over the 2 f columns of dg and du
//   TN    the weights' gradients, three products in one launch
// bf16 operands, fp32 sums.  h, the factors, dg and du are rounded to bf16 where they are stored (h, dg and du are the next
// product's operands); all are formed from unrounded g and u.  A caller who keeps the factors in fp32 (twice their memory) saves
// one of the three roundings on the way to dx and the projections' gradients: relative to fp64 2.4e-3 instead of 2.9e-3, where one
// rounding alone gives 1.7e-3 (16384 x 2048 x 5632: forward 840 -> 857 us, backward 1647 -> 1707).  The factors are kept instead of g and u because DH's epilogue has
// the matrix cores wait for it: with the activation's slope in it (20 instructions an element, two of them quarter rate)
// a tile of 256 x 256 took 24 us beside its 46 us of products.
//
// 16384 x 2048 x 5632 (tiles of 256): UP 575 us, 1.32 PFLOP/s; NT 280, 1.35; DH 402, 0.94; NN 522, 1.45; TN 789, 1.44: the matrix cores at
// the power limit, but for the epilogues of UP and DH.
//
// Tiles: 256 threads, 2 x 2 wavefronts, operands straight from memory to LDS in a ring of 64-deep K tiles, the fragments of one
// 32-deep slice read while the matrix cores work on the one before it: the scheme of the Newton-Schulz products
// (ns_gemm.hip), with nothing padded: what lies outside a matrix is beyond the end of its buffer resource, whose loads give
// 0 and whose stores are dropped.
#include <atomic>
#include <utility>

#include "common.h"
#include "ffn_plan.h"
#include "mfma_tile.h"

namespace mlc {
namespace {

constexpr int NTHREADS = 256;
constexpr int NUM_XCD = 8;
constexpr int GROUP_M = 8;                          // tile rows per group of the tile order
constexpr unsigned int BUFFER_END = 0xfffffff0u;    // no buffer reaches it: a load there gives 0, a store is dropped
constexpr int MAX_PROBLEMS = 3;
enum Form { UP, NT, DH, NN, TN, UP32, DH32 };       // the last two: with fp32 factors

struct Problem {
  const bf16_t* A[2]; const bf16_t* B[2];           // NN: of the two halves of the sum; UP: B of g and of u
  long lda, ldb;
  bf16_t* D; long ldd;                              // UP: h; DH: dg
  int M, N, K;                                      // K: of one half
  int tiles_m, tiles_n, first;                      // first: index of its first tile
};
// The work is a list of items: `whole` tiles, then the others, `splits` items each, which leave fp32 sums over a part of K in
// `partial`, [item][BM][BN], for ffn_join_kernel.
struct GemmArgs {
  Problem p[MAX_PROBLEMS];
  int problems, tiles, whole, splits;
  float* partial;
  void* gate; void* up;                             // act(g) and u act'(g), bf16 or fp32; UP: out (may be null); DH: in
  bf16_t* du;                                       // DH: out
};
struct Place { int problem, m0, n0; };
template <int BM, int COLS>
__device__ __forceinline__ Place locate(const GemmArgs& g, int t) {
  Place r;
  r.problem = 0;
  while (r.problem + 1 < g.problems && t >= g.p[r.problem + 1].first) ++r.problem;
  const Problem& P = g.p[r.problem];
  t -= P.first;
  // groups of GROUP_M tile rows, column by column inside a group
  const int per_group = GROUP_M * P.tiles_n, grp = t / per_group, rest = t - grp * per_group;
  const int rows = min(P.tiles_m - grp * GROUP_M, GROUP_M);
  const int tn = rest / rows, tm = grp * GROUP_M + (rest - tn * rows);
  r.m0 = tm * BM;
  r.n0 = tn * COLS;
  return r;
}
// Workgroups go round the XCDs; an XCD has a contiguous range of the whole tiles and one of the rest, and its workgroups take them
// in order, one after the other.
struct Share { int whole0, whole, rest0, rest; };
__device__ __forceinline__ Share share_of(const GemmArgs& g, int xcd) {
  const int rest = (g.tiles - g.whole) * g.splits, w8 = (g.whole + NUM_XCD - 1) / NUM_XCD, r8 = (rest + NUM_XCD - 1) / NUM_XCD;
  Share s;
  s.whole0 = xcd * w8;
  s.whole = min(max(g.whole - s.whole0, 0), w8);
  s.rest0 = g.whole + xcd * r8;
  s.rest = min(max(g.whole + rest - s.rest0, 0), r8);
  return s;
}

// f(I<0>), f(I<1>), ... f(I<N - 1>): loops that are too long for the compiler's own unrolling.
template <int... N, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, N...>, F&& f) { (f(I<N>{}), ...); }
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) { each_of(std::make_integer_sequence<int, N>{}, f); }

// (the hardware's reciprocal, an ulp of fp32 off: all of this is rounded to bf16 next)
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.f + __expf(-x)); }
constexpr float GELU_C = 0.7978845608028654f, GELU_A = 0.044715f;
// act(g) and act'(g)
template <int ACT>
__device__ __forceinline__ void activation(float g, float& a, float& da) {
  if (ACT == MLC_ACT_SILU) {
    const float s = sigmoid(g);
    a = g * s;
    da = s + (a - a * s);
  } else {
    // 1/2 (1 + tanh(x)) = sigmoid(2 x), whose relative error stays an ulp or two where 1 + tanh(x) cancels
    // (from |g| = 10 on it is 0 or 1 in fp32, whatever the cubic; at 16 its square cannot overflow against that 0)
    const float h = __builtin_amdgcn_fmed3f(g, -16.f, 16.f), s = sigmoid(2.f * GELU_C * (h + GELU_A * h * h * h));
    a = g * s;
    da = s + a * (1.f - s) * (2.f * GELU_C) * (1.f + 3.f * GELU_A * h * h);
  }
}

// An operand's place in memory: a buffer that begins at its tile and ends where the matrix does, or before.  All offsets of a tile
// are below LOAD_END; an offset of LOAD_END or more gives 0.
constexpr unsigned int LOAD_END = 0x80000000u;
struct Cursor {
  unsigned long base; long left;                    // bytes to the end of the matrix
  __device__ __forceinline__ i32x4 rsrc() const {
    const int hi = (int)(left >> 32);
    const unsigned int lo = (unsigned int)left;
    i32x4 r;
    r.x = (int)(unsigned int)base;
    r.y = (int)((unsigned int)(base >> 32) & 0xffffu);
    r.z = (int)(hi < 0 ? 0u : hi > 0 || lo > LOAD_END ? LOAD_END : lo);
    r.w = 0x00020000;
    return r;
  }
  __device__ __forceinline__ void forward(long bytes) { base += (unsigned long)bytes; left -= bytes; }
};

// Of a 128 x 128 or smaller tile the compiler's own MFMAs; the 256 x 256 one's are written out (see mfma_tile.h).
// ACT: of UP.
template <int KIND, int ACT, int BM, int BN, int NB>
__global__ __launch_bounds__(NTHREADS, NB == 5 && BM != 256 ? 2 : 1) void ffn_gemm_kernel(GemmArgs g) {
  constexpr bool WIDE = KIND == UP32 || KIND == DH32;
  constexpr int FORM = KIND == UP32 ? UP : KIND == DH32 ? DH : KIND;
  constexpr bool AKS = FORM == TN, BKS = FORM == DH || FORM == NN || FORM == TN, DUAL = FORM == UP;
  constexpr int TI = BM / 32, TJ = BN / 32, NM = TI * TJ;
  constexpr int NCHA = BM / 32, NCHB = BN / 32;     // transfers per thread and buffer
  constexpr unsigned int BUF = (BM > BN ? BM : BN) * BK * 2, RING = NB * BUF;
  constexpr int D = (NB - 1) / 2;                   // K tiles requested ahead
  constexpr bool HAND = BM == 256;
  static_assert(D >= 2 && NB % 2 == 1 && TJ % 4 == 0, "");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  typedef __attribute__((address_space(3))) unsigned char lds_byte;
  const unsigned int lds0 = (unsigned int)(unsigned long)(lds_byte*)smem;

  constexpr int COLS = DUAL ? BN / 2 : BN;          // columns of the result in a tile
  const int kt_half = (g.p[0].K + BK - 1) / BK, kt_all = FORM == NN ? 2 * kt_half : kt_half;
  // this workgroup's turns: `turn`, turn + turn_step, ... below `turns`
  const Share share = share_of(g, (int)blockIdx.x % NUM_XCD);
  const int turn_step = (int)gridDim.x / NUM_XCD, turns = share.whole + share.rest;
  int turn = (int)blockIdx.x / NUM_XCD;
  if (turn >= turns) return;
  struct Tile { int problem, m0, n0, k_first, k_last, part, live; };
  auto tile_of = [&](int at) {
    Tile r;
    int t = share.whole0 + at, part = -1, k_first = 0, k_last = kt_all;
    if (at >= share.whole) {
      part = share.rest0 + at - share.whole - g.whole;
      const int n = part / g.splits, split = part - n * g.splits;
      t = g.whole + n;
      k_first = kt_all * split / g.splits;
      k_last = kt_all * (split + 1) / g.splits;
    }
    const Place place = locate<BM, COLS>(g, t);
    r.problem = __builtin_amdgcn_readfirstlane(place.problem);
    r.m0 = __builtin_amdgcn_readfirstlane(place.m0);
    r.n0 = __builtin_amdgcn_readfirstlane(place.n0);
    r.k_first = __builtin_amdgcn_readfirstlane(k_first);
    r.k_last = __builtin_amdgcn_readfirstlane(k_last);
    r.part = __builtin_amdgcn_readfirstlane(part);
    r.live = 1;
    return r;
  };

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int idx = lane & 15, lg = lane >> 4;
  const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);

  // ---- transfers.  LDS chunk c = it * 256 + tid (16 bytes) of a buffer.  K-contiguous operands lie there as [slot][64 k] with
  // slot = 32 (pair of accumulator tiles) + 16 (odd) + idx and chunks swizzled by the slot; K-strided ones as [k][rows], chunks
  // swizzled by k: see ns_gemm.hip.  Accumulator tile i of a wavefront holds rows 32 (i / 2) + 8 (idx / 4) + 4 (i % 2) + idx % 4, so
  // that a lane's two tiles of a pair are 8 adjacent columns; so does transfer `it` fetch rows from 32 it on.
  const int slot = tid >> 3, sidx = slot & 15;
  const unsigned int srow = 8 * (sidx >> 2) + 4 * (slot >> 4) + (sidx & 3);
  const unsigned int kchunk = (unsigned int)((tid & 7) ^ ((tid >> 4) & 7));
  auto ks_swizzle = [](int b, int k) { return b == 64 ? 4 * ((k >> 1) & 1) : 4 * (k & 3); };
  auto ks_voff = [&](int b, unsigned int ld2) {
    const int cpr = b / 8;
    return (unsigned int)(tid / cpr) * ld2 + (unsigned int)(((tid % cpr) ^ ks_swizzle(b, tid / cpr)) * 16);
  };
  // the last, partial K tile: of a K-contiguous operand the chunks behind the row's end are not its own
  const int tail = g.p[0].K % BK;
  const bool cut = tail && (int)kchunk * 8 >= tail;
  const unsigned int lds_wave = lds0 + (unsigned int)wave * 1024;

  // ---- where the transfers stand: K tile `ask` of the tile of turn `ask_turn`, one of this workgroup's next ones.  They run on from
  // tile to tile, so that the ring is full when a tile begins.
  int ask_turn = turn;
  Tile asked = tile_of(turn);
  int ask = asked.k_first;
  Cursor ca{0, 0}, cb{0, 0};
  unsigned int voffA = 0, voffB = 0, stepA = 0, stepB = 0;
  long advA = 0, advB = 0;                          // of a K-strided operand, from K tile to K tile
  i32x4 rsA = {0, 0, 0, 0}, rsB = rsA, rsB2 = rsA;
  auto aim = [&] {                                  // everything at K tile `ask` of `asked`
    const Problem& P = g.p[asked.problem];
    const unsigned int lda2 = (unsigned int)(P.lda * 2), ldb2 = (unsigned int)(P.ldb * 2);
    voffA = AKS ? ks_voff(BM, lda2) : srow * lda2 + kchunk * 16;
    voffB = BKS ? ks_voff(BN, ldb2) : srow * ldb2 + kchunk * 16;
    stepA = AKS ? (unsigned int)(NTHREADS / (BM / 8)) * lda2 : 32u * lda2;
    stepB = BKS ? (unsigned int)(NTHREADS / (BN / 8)) * ldb2 : 32u * ldb2;
    advA = AKS ? (long)BK * lda2 : 0;
    advB = BKS ? (long)BK * ldb2 : 0;
    const int half = FORM == NN && ask >= kt_half ? 1 : 0, kt = ask - half * kt_half;
    // K-contiguous: the buffer begins at the tile's first row, and the K tile is in the lanes' offsets; K-strided: at the K tile
    auto at = [&](const bf16_t* p, bool ks, long ld2, int row0, int rows_all) {
      const long start = ks ? (long)row0 * 2 + kt * ld2 * BK : (long)row0 * ld2;
      const long bytes = ks ? ((long)P.K - 1) * ld2 + (long)rows_all * 2 : ((long)rows_all - 1) * ld2 + (long)P.K * 2;
      return Cursor{(unsigned long)p + (unsigned long)start, asked.live ? bytes - start : 0};
    };
    ca = at(P.A[half], AKS, lda2, asked.m0, P.M);
    cb = at(P.B[FORM == NN ? half : 0], BKS, ldb2, asked.n0, P.N);
    if (!AKS) voffA += (unsigned int)kt * (BK * 2);
    if (!BKS) voffB += (unsigned int)kt * (BK * 2);
    rsA = ca.rsrc();
    rsB = cb.rsrc();
    if constexpr (DUAL) rsB2 = at(P.B[1], BKS, ldb2, asked.n0, P.N).rsrc();
  };
  unsigned int runA = 0, runB = 0;                  // lane offsets of the next transfer
  // What the transfers of K tile `ask` start from, and what follows them.  PLAIN: neither is it a row's last, partial one nor the
  // last one of its half or tile.
  auto request = [&](auto plain_tag) {
    const bool last = !decltype(plain_tag)::value && tail && (ask + 1 == kt_half || ask + 1 == 2 * kt_half);
    runA = !AKS && last && cut ? LOAD_END : voffA;
    runB = !BKS && last && cut ? LOAD_END : voffB;
  };
  auto forward = [&] {
    if constexpr (AKS) {
      ca.forward(advA);
      rsA = ca.rsrc();
    } else {
      voffA += BK * 2;
    }
    if constexpr (BKS) {
      cb.forward(advB);
      rsB = cb.rsrc();
    } else {
      voffB += BK * 2;
    }
  };
  auto advance = [&](auto plain_tag) {
    ++ask;
    if (decltype(plain_tag)::value) {
      forward();
    } else if (ask >= asked.k_last) {
      ask_turn += turn_step;
      const bool more = ask_turn < turns;
      asked = tile_of(more ? ask_turn : turn);
      ask = asked.k_first;
      if (!more) {                                  // beyond the last tile they fetch nothing
        asked.live = 0;
        asked.k_last = 0x7fffffff;
      }
      aim();
    } else if (FORM == NN && ask == kt_half) {
      aim();
    } else {
      forward();
    }
  };
  // K tiles from `ask` on that are plain
  auto plain_ones = [&] { return (FORM == NN && ask < kt_half ? min(kt_half, asked.k_last) : asked.k_last) - 1 - ask; };
  auto next_a = [&] { runA += stepA; };
  auto next_b = [&](int it) { if (!DUAL || (it & 1)) runB += stepB; };
  auto dma_a = [&](auto it_tag, unsigned int dst) {
    constexpr int it = decltype(it_tag)::value;
    dma16<it * 4096>(rsA, runA, 0, dst);
    next_a();
  };
  auto dma_b = [&](auto it_tag, unsigned int dst) {
    constexpr int it = decltype(it_tag)::value;
    dma16<it * 4096>(DUAL && (it & 1) ? rsB2 : rsB, runB, 0, dst);
    next_b(it);
  };
  auto with = [&](int n, auto&& f) {                // f(I<n>): n is a constant after unrolling
    switch (n) {
      case 0: f(I<0>{}); break;
      case 1: f(I<1>{}); break;
      case 2: f(I<2>{}); break;
      case 3: f(I<3>{}); break;
      case 4: f(I<4>{}); break;
      case 5: f(I<5>{}); break;
      case 6: f(I<6>{}); break;
      default: f(I<7>{}); break;
    }
  };

  // ---- fragments: offsets inside a buffer, and the reads
  const unsigned int swz = (unsigned int)((idx >> 1) & 7);
  const int k4 = idx >> 2, q = idx & 3;
  unsigned int fragA[AKS ? TI / 2 : 1], fragB[BKS ? TJ / 2 : 1];
  if constexpr (AKS) {
#pragma unroll
    for (int n = 0; n < TI / 2; ++n)
      fragA[n] = (unsigned int)(8 * lg + k4) * (BM * 2) + (unsigned int)(((wm / 8 + 4 * n + q) ^ ks_swizzle(BM, k4)) * 16);
  } else {
    fragA[0] = (unsigned int)(wm + idx) * 128 + (((unsigned int)lg ^ swz) * 16);
  }
  if constexpr (BKS) {
#pragma unroll
    for (int n = 0; n < TJ / 2; ++n)
      fragB[n] = (unsigned int)(8 * lg + k4) * (BN * 2) + (unsigned int)(((wn / 8 + 4 * n + q) ^ ks_swizzle(BN, k4)) * 16);
  } else {
    fragB[0] = (unsigned int)(wn + idx) * 128 + (((unsigned int)lg ^ swz) * 16);
  }
  u32x4 fa[2][TI], fb[2][TJ];
  f32x4 acc[TI][TJ];
  constexpr int NRA = AKS ? 2 * TI : TI, NRB = BKS ? 2 * TJ : TJ, NR = NRA + NRB;        // LDS reads per slice
  constexpr int RSTEP = NM / 2 / NR > 0 ? NM / 2 / NR : 1, RPER = (NR + NM - 1) / NM;
  unsigned int bufA = 0, bufB = 0;                  // what the reads are from
  int kk = 0;
  auto tr_read = [&](unsigned int at) {
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)((lds_byte*)smem + at)));
  };
  auto read_a = [&](int set, int r) {
    if constexpr (AKS) {
      const int i = r >> 1, h = r & 1;
      const u32x2 w = tr_read(fragA[i >> 1] + bufA + (kk ? 32u * BM * 2 : 0u) + (i & 1) * 8 + h * 4 * (BM * 2));
      fa[set][i][2 * h] = w.x;
      fa[set][i][2 * h + 1] = w.y;
    } else {
      fa[set][r] = *reinterpret_cast<const u32x4*>(smem + ((fragA[0] ^ (kk ? 64u : 0u)) + bufA) + r * 2048);
    }
  };
  auto read_b = [&](int set, int r) {
    if constexpr (BKS) {
      const int j = r >> 1, h = r & 1;
      const u32x2 w = tr_read(fragB[j >> 1] + bufB + (kk ? 32u * BN * 2 : 0u) + (j & 1) * 8 + h * 4 * (BN * 2));
      fb[set][j][2 * h] = w.x;
      fb[set][j][2 * h + 1] = w.y;
    } else {
      fb[set][r] = *reinterpret_cast<const u32x4*>(smem + ((fragB[0] ^ (kk ? 64u : 0u)) + bufB) + r * 2048);
    }
  };
  // read r of a slice: the first of A, all of B, the rest of A
  constexpr int FIRST_A = AKS ? 2 : 1;
  auto read_one = [&](int set, int r) {
    if (r < FIRST_A) read_a(set, r);
    else if (r < FIRST_A + NRB) read_b(set, r - FIRST_A);
    else read_a(set, r - NRB);
  };

  // One slice: NM MFMAs on fragment set S, with the reads of the next slice and the transfers of one operand between them.
  // ZERO: the sums begin here.
  auto slice = [&](auto set_tag, auto zero_tag, auto b_tag, unsigned int dst) {
    constexpr int S = decltype(set_tag)::value;
    constexpr bool ZERO = decltype(zero_tag)::value;
    constexpr bool OPB = decltype(b_tag)::value;
    constexpr int NCH = OPB ? NCHB : NCHA, DSTEP = NM / NCH;
#pragma unroll
    for (int n = 0; n < NM; ++n) {
      const int i = n / TJ, j = (i & 1) ? TJ - 1 - n % TJ : n % TJ;
      if constexpr (!HAND) {
        f32x4 c = acc[i][j];
        if constexpr (ZERO) c = f32x4{0.f, 0.f, 0.f, 0.f};
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[S][j]),
                                                            __builtin_bit_cast(bf16x8, fa[S][i]), c, 0, 0, 0);
        if (n % DSTEP == 1) with(n / DSTEP, [&](auto it) { if constexpr (OPB) dma_b(it, dst); else dma_a(it, dst); });
      } else if (n % DSTEP == 1) {
        with(n / DSTEP, [&](auto it) {
          constexpr int x = decltype(it)::value;
          mfma_dma<ZERO, x * 4096>(acc[i][j], fb[S][j], fa[S][i], OPB ? (DUAL && (x & 1) ? rsB2 : rsB) : rsA, OPB ? runB : runA, 0, dst);
        });
      } else {
        mfma<ZERO>(acc[i][j], fb[S][j], fa[S][i]);
        if (n % DSTEP == 2) { if constexpr (OPB) next_b(n / DSTEP); else next_a(); }
      }
#pragma unroll
      for (int r = 0; r < RPER; ++r)
        if (n % RSTEP == 0 && n / RSTEP * RPER + r < NR) read_one(1 - S, n / RSTEP * RPER + r);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto wrap = [](unsigned int p) { return p >= RING ? p - RING : p; };

  aim();
#pragma unroll
  for (int n = 0; n < D; ++n) {
    request(std::false_type{});
#pragma unroll
    for (int it = 0; it < NCHA; ++it) with(it, [&](auto x) { if constexpr (decltype(x)::value < NCHA) dma_a(x, lds_wave + (2 * n) * BUF); });
#pragma unroll
    for (int it = 0; it < NCHB; ++it) with(it, [&](auto x) { if constexpr (decltype(x)::value < NCHB) dma_b(x, lds_wave + (2 * n + 1) * BUF); });
    advance(std::false_type{});
  }
  wait_vmcnt<(D - 1) * (NCHA + NCHB)>();
  block_sync();
  unsigned int p = 0;                               // buffer of operand A of the current K tile

  // Transfers that may be in flight at a K tile's barrier, which publishes the next K tile: all requested after it, and on a tile's
  // first K tile the stores of the epilogue before it.
  constexpr int STEADY = (D - 2) * (NCHA + NCHB) + NCHA;
  constexpr int JC = DUAL ? TJ / 4 : TJ / 2;        // runs of 8 columns of a lane's row
  constexpr int STORES = TI * JC;                   // of one result, at least
  constexpr auto most = [](int n) { return n < 63 ? n : 63; };      // (what the counter holds)
  bool stored = false;
  auto step = [&](auto first_tag, auto plain_tag) {
    request(plain_tag);
    const unsigned int pa1 = wrap(p + 2 * BUF), pb1 = wrap(p + 3 * BUF);
    const unsigned int free0 = lds_wave + (p == 0 ? RING - BUF : p - BUF), free1 = lds_wave + p;
    bufA = p; bufB = wrap(p + BUF); kk = 1;
    slice(I<0>{}, first_tag, std::false_type{}, free0);
    if (decltype(first_tag)::value && stored) {
      if (FORM == DH || (FORM == UP && g.gate)) wait_vmcnt<most(STEADY + 2 * STORES)>();
      else wait_vmcnt<most(STEADY + STORES)>();
    } else {
      wait_vmcnt<STEADY>();
    }
    block_sync();
    bufA = pa1; bufB = pb1; kk = 0;
    slice(I<1>{}, std::false_type{}, std::true_type{}, free1);
    advance(plain_tag);
    p = pa1;
  };
  while (true) {
  const Tile tile = tile_of(turn);
  const Problem& P = g.p[tile.problem];
  const int m0 = tile.m0, n0 = tile.n0;
  bufA = p; bufB = wrap(p + BUF); kk = 0;
#pragma unroll
  for (int r = 0; r < NR; ++r) read_one(0, r);
  step(std::true_type{}, std::false_type{});        // (of no K tiles at all: one of zeros)
  for (int n = tile.k_first + 1; n < tile.k_last;) {
    // the loop that counts knows of no tile's end (with the turn to the next tile in it a K tile took 7 % longer)
    const int plain = min(tile.k_last - n, plain_ones());
#pragma unroll 1
    for (int x = 0; x < plain; ++x) step(std::false_type{}, std::true_type{});
    n += max(plain, 0);
    if (n < tile.k_last) {
      step(std::false_type{}, std::false_type{});
      ++n;
    }
  }
  if constexpr (HAND) acc_settle(acc);

  // ---- epilogue: lane (idx, lg) holds, for each i and J, 8 adjacent columns of row 32 (i / 2) + 8 (idx / 4) + 4 (i % 2) + idx % 4.
  // A store meets 64 bytes of each of 16 rows; lanes of neighbouring rows therefore swap what is 32 columns apart (pair_rows),
  // and a store covers 8 whole lines.  Places outside the result lie beyond the buffers' ends.
  const int col0 = (DUAL ? wn / 2 : wn) + 8 * lg, odd = lane & 1;
  const unsigned int ldd2 = (unsigned int)(P.ldd * 2);
  const long origin = (long)m0 * P.ldd + n0;
  auto row_at = [&](int i) { return wm + 32 * (i >> 1) + 8 * (idx >> 2) + 4 * (i & 1) + (idx & 3); };
  const int rows_left = P.M - m0, cols_left = P.N - n0;
  auto place = [&](int row, int col) {              // byte offset from the tile's origin
    const bool in = (row < rows_left) & (col < cols_left);
    return in ? (unsigned int)row * ldd2 + (unsigned int)col * 2 : BUFFER_END;
  };
  auto take = [&](int i, int J, float (&v)[8]) {
    const f32x4 a = HAND ? acc_read(acc[i][2 * J]) : acc[i][2 * J], b = HAND ? acc_read(acc[i][2 * J + 1]) : acc[i][2 * J + 1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  };
  auto rsrc_of = [&](const bf16_t* q) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(q) + origin, 0, BUFFER_END, 0x00020000); };
  // the factors' buffers, and the places of 8 (4 fp32) of their elements there
  constexpr int FACTOR = WIDE ? 2 : 1;              // times two bytes an element
  auto rsrc_factor = [&](void* q) { return __builtin_amdgcn_make_buffer_rsrc((bf16_t*)q + origin * FACTOR, 0, BUFFER_END, 0x00020000); };
  auto place_factor = [&](int row, int col) {
    const unsigned int at = place(row, col);
    return at == BUFFER_END ? BUFFER_END : at * FACTOR;
  };
  auto store_row = [&](__amdgpu_buffer_rsrc_t r, int i, const u32x4 (&w)[JC]) {
    const int row = row_at(i);
    if constexpr (JC == 1) {
      __builtin_amdgcn_raw_buffer_store_b128(w[0], r, place(row, col0), 0, 0);
    } else {
#pragma unroll
      for (int J = 0; J < JC; J += 2) {
        u32x4 x, y;
        pair_rows(w[J], w[J + 1], odd, x, y);
        const int col = col0 + 32 * (J + odd);
        __builtin_amdgcn_raw_buffer_store_b128(x, r, place(row & ~1, col), 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(y, r, place(row | 1, col), 0, 0);
      }
    }
  };
  if constexpr (FORM == UP) {
    const __amdgpu_buffer_rsrc_t rh = rsrc_of(P.D), rg = rsrc_factor(g.gate), ru = rsrc_factor(g.up);
    auto all = [&](auto keep_tag) {                 // keep: the backward call's factors too
      constexpr bool KEEP = decltype(keep_tag)::value;
      each<TI>([&](auto row_tag) {
        constexpr int i = decltype(row_tag)::value;
        u32x4 wg[JC], wu[JC], wh[JC];
#pragma unroll
        for (int J = 0; J < JC; ++J) {
          float v[8], u[8], h[8];
          take(i, 2 * J, v);
          take(i, 2 * J + 1, u);
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            float a, da;
            activation<ACT>(v[x], a, da);
            h[x] = a * u[x];
            v[x] = a;
            u[x] *= da;
          }
          wh[J] = Vec8<bf16_t>::pack(h);
          if (KEEP && !WIDE) { wg[J] = Vec8<bf16_t>::pack(v); wu[J] = Vec8<bf16_t>::pack(u); }
          if constexpr (KEEP && WIDE) {
            const unsigned int at = place_factor(row_at(i), col0 + 32 * J), next = at == BUFFER_END ? at : at + 16;
            auto four = [](const float* q) { return u32x4{__float_as_uint(q[0]), __float_as_uint(q[1]), __float_as_uint(q[2]), __float_as_uint(q[3])}; };
            __builtin_amdgcn_raw_buffer_store_b128(four(v), rg, at, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b128(four(v + 4), rg, next, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b128(four(u), ru, at, 0, 0);
            __builtin_amdgcn_raw_buffer_store_b128(four(u + 4), ru, next, 0, 0);
          }
        }
        store_row(rh, i, wh);
        if (KEEP && !WIDE) {
          store_row(rg, i, wg);
          store_row(ru, i, wu);
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    if constexpr (WIDE) all(std::true_type{});
    else if (g.gate) all(std::true_type{});
    else all(std::false_type{});
  } else if constexpr (FORM == DH) {
    const __amdgpu_buffer_rsrc_t rd = rsrc_of(P.D), rdu = rsrc_of(g.du), rg = rsrc_factor(g.gate), ru = rsrc_factor(g.up);
    u32x4 gt[2][JC * FACTOR], up[2][JC * FACTOR];   // this row's and the next one's
    auto fetch = [&](int i) {
#pragma unroll
      for (int J = 0; J < JC; ++J) {
        const unsigned int at = place_factor(row_at(i), col0 + 32 * J);
#pragma unroll
        for (int half = 0; half < FACTOR; ++half) {
          const unsigned int there = half && at != BUFFER_END ? at + 16 : at;
          gt[i & 1][J * FACTOR + half] = __builtin_amdgcn_raw_buffer_load_b128(rg, there, 0, 0);
          up[i & 1][J * FACTOR + half] = __builtin_amdgcn_raw_buffer_load_b128(ru, there, 0, 0);
        }
      }
    };
    auto factors = [&](const u32x4* w, float (&f)[8]) {
      if constexpr (WIDE) {
#pragma unroll
        for (int x = 0; x < 8; ++x) f[x] = __uint_as_float(w[x / 4][x % 4]);
      } else {
        Vec8<bf16_t>::unpack(w[0], f);
      }
    };
    fetch(0);
    each<TI>([&](auto row_tag) {
      constexpr int i = decltype(row_tag)::value;
      if (i + 1 < TI) fetch(i + 1);
      __builtin_amdgcn_sched_barrier(0);
      u32x4 wg[JC], wu[JC];
#pragma unroll
      for (int J = 0; J < JC; ++J) {
        float v[8], gv[8], uv[8];
        take(i, J, v);
        factors(&gt[i & 1][J * FACTOR], gv);
        factors(&up[i & 1][J * FACTOR], uv);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          gv[x] *= v[x];
          uv[x] *= v[x];
        }
        wg[J] = Vec8<bf16_t>::pack(uv); wu[J] = Vec8<bf16_t>::pack(gv);
      }
      store_row(rd, i, wg);
      store_row(rdu, i, wu);
      __builtin_amdgcn_sched_barrier(0);
    });
  } else if (tile.part >= 0) {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(g.partial + (long)tile.part * (BM * BN), 0, BM * BN * 4, 0x00020000);
    each<TI>([&](auto row_tag) {
      constexpr int i = decltype(row_tag)::value;
#pragma unroll
      for (int J = 0; J < JC; ++J) {
        const f32x4 a = HAND ? acc_read(acc[i][2 * J]) : acc[i][2 * J], b = HAND ? acc_read(acc[i][2 * J + 1]) : acc[i][2 * J + 1];
        const unsigned int at = (unsigned int)(row_at(i) * BN + col0 + 32 * J) * 4;
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, a), r, at, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, b), r, at + 16, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  } else {
    const __amdgpu_buffer_rsrc_t r = rsrc_of(P.D);
    each<TI>([&](auto row_tag) {
      constexpr int i = decltype(row_tag)::value;
      u32x4 w[JC];
#pragma unroll
      for (int J = 0; J < JC; ++J) {
        float v[8];
        take(i, J, v);
        w[J] = Vec8<bf16_t>::pack(v);
      }
      store_row(r, i, w);
      __builtin_amdgcn_sched_barrier(0);
    });
  }
  stored = true;
  turn += turn_step;
  if (turn >= turns) break;
  }
  // nothing may land in the ring after this workgroup has left it
  __builtin_amdgcn_s_waitcnt(0x0f70);
  block_sync();
}

// ---- few tokens: up to 16 TM rows of x against all of a matrix, which is read once, straight into the MFMAs' operands.
//
// A workgroup takes 16 rows of the weights (of both matrices for UP), its wavefronts share the K range in pieces of 128, and the
// partial sums meet in LDS, in the order of the wavefronts.  Bound by the stream of the weights: a wavefront keeps a piece's
// loads under way (16 bytes a lane each), and there are enough wavefronts a workgroup that a few hundred rows of
// weights keep the chip's memory busy.
constexpr int STEPS = 4;                            // MFMA steps of 32 k in a piece
template <bool DUAL, int ACT, int TM, bool WIDE>
__global__ __launch_bounds__(1024) void ffn_few_kernel(const bf16_t* x, const bf16_t* w0, const bf16_t* w1, int M, int N, int K,
                                                       bf16_t* out, void* gate, void* up) {
  constexpr int NW = DUAL ? 2 : 1;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  f32x4* const held = (f32x4*)smem;                 // [wavefront][TM][NW][lane]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int idx = lane & 15, lg = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const unsigned int ld2 = (unsigned int)K * 2;
  auto rsrc = [&](const bf16_t* p, long row0, long rows) {
    const long bytes = (rows - row0) * (long)ld2;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t*>(p) + row0 * K, 0,
                                             (unsigned int)(bytes < (long)BUFFER_END ? bytes : (long)BUFFER_END), 0x00020000);
  };
  const __amdgpu_buffer_rsrc_t rx = rsrc(x, 0, M), r0 = rsrc(w0, n0, N), r1 = rsrc(DUAL ? w1 : w0, n0, N);
  f32x4 acc[TM][NW];
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int w = 0; w < NW; ++w) acc[m][w] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int k0 = wave * 32 * STEPS; k0 < K; k0 += waves * 32 * STEPS) {
    u32x4 fw[STEPS][NW], fx[STEPS][TM];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int k = k0 + 32 * s + 8 * lg;
      const unsigned int at = k < K ? (unsigned int)k * 2 : BUFFER_END;       // (a row's end is not the buffer's)
      const unsigned int row = at == BUFFER_END ? 0 : (unsigned int)idx * ld2;
      fw[s][0] = __builtin_amdgcn_raw_buffer_load_b128(r0, at + row, 0, 0);
      if constexpr (DUAL) fw[s][1] = __builtin_amdgcn_raw_buffer_load_b128(r1, at + row, 0, 0);
#pragma unroll
      for (int m = 0; m < TM; ++m)
        fx[s][m] = __builtin_amdgcn_raw_buffer_load_b128(rx, at + (at == BUFFER_END ? 0 : row + 16u * m * ld2), 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);              // all loads first
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
      for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int w = 0; w < NW; ++w)
          acc[m][w] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw[s][w]),
                                                              __builtin_bit_cast(bf16x8, fx[s][m]), acc[m][w], 0, 0, 0);
  }
#pragma unroll
  for (int m = 0; m < TM; ++m)
#pragma unroll
    for (int w = 0; w < NW; ++w) held[((wave * TM + m) * NW + w) * 64 + lane] = acc[m][w];
  __syncthreads();
  // lane (idx, lg) of tile m: columns n0 + 4 lg .. + 3 of token 16 m + idx
  for (int e = threadIdx.x; e < TM * 64; e += blockDim.x) {
    const int m = e >> 6, token = 16 * m + (e & 15), col = n0 + 4 * ((e >> 4) & 3);
    if (token >= M || col >= N) continue;
    f32x4 v[NW];
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      v[w] = held[(m * NW + w) * 64 + (e & 63)];
      for (int q = 1; q < waves; ++q) v[w] += held[((q * TM + m) * NW + w) * 64 + (e & 63)];
    }
    const long at = (long)token * N + col;
    auto put = [&](bf16_t* p, const f32x4& f) {
      u32x2 b;
      b.x = pack_bf16x2(f.x, f.y);
      b.y = pack_bf16x2(f.z, f.w);
      *reinterpret_cast<u32x2*>(p + at) = b;
    };
    if constexpr (DUAL) {
      f32x4 h;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        float a, da;
        activation<ACT>(v[0][c], a, da);
        h[c] = a * v[1][c];
        v[0][c] = a;
        v[1][c] *= da;
      }
      put(out, h);
      if constexpr (WIDE) {
        *reinterpret_cast<f32x4*>((float*)gate + at) = v[0];
        *reinterpret_cast<f32x4*>((float*)up + at) = v[1];
      } else if (gate) {
        put((bf16_t*)gate, v[0]);
        put((bf16_t*)up, v[1]);
      }
    } else {
      put(out, v[0]);
    }
  }
}

// The split tiles: sums of their items' sums, in the order of K.  A workgroup takes 2048 elements of a tile.
template <int BM, int BN>
__global__ __launch_bounds__(NTHREADS) void ffn_join_kernel(GemmArgs g) {
  constexpr int PER = BM * BN / (NTHREADS * 8);
  const int n = (int)blockIdx.x / PER, e = ((int)blockIdx.x % PER * NTHREADS + (int)threadIdx.x) * 8;
  const Place at = locate<BM, BN>(g, g.whole + n);
  const Problem& P = g.p[at.problem];
  const int row = at.m0 + e / BN, col = at.n0 + e % BN;
  if (row >= P.M || col >= P.N) return;
  const float* const from = g.partial + (long)n * g.splits * (BM * BN) + e;
  float sum[8], v[8];
  Vec8<float>::load(from, sum);
  for (int s = 1; s < g.splits; ++s) {
    Vec8<float>::load(from + (long)s * (BM * BN), v);
#pragma unroll
    for (int x = 0; x < 8; ++x) sum[x] += v[x];
  }
  Vec8<bf16_t>::store(P.D + (long)row * P.ldd + col, sum);
}

int check_launch() { return hipGetLastError() == hipSuccess ? MLC_OK : MLC_ERR_LAUNCH; }

template <bool DUAL, int ACT, bool WIDE = false>
int launch_few(const bf16_t* x, const bf16_t* w0, const bf16_t* w1, int64_t M, int64_t N, int64_t K, bf16_t* out, void* gate, void* up,
               hipStream_t stream) {
  const int tm = (int)((M + 15) / 16);
  // wavefronts: two pieces of the K range each where that is long enough for 16 of them
  int waves = 4;
  while (waves < (DUAL ? 8 : 16) && (int64_t)waves * 2 * 32 * STEPS * 2 <= K) waves *= 2;
  const dim3 grid((unsigned)((N + 15) / 16)), block(64 * waves);
  const unsigned int lds = (unsigned)(waves * tm * (DUAL ? 2 : 1) * 64 * sizeof(f32x4));
  LaunchScope scope(MLC_KERNEL_FFN, stream, (DUAL ? 4.0 : 2.0) * M * N * K, 2.0 * ((DUAL ? 2.0 : 1.0) * N * K + (double)M * (N + K)));
#define MLC_FEW(TM) \
  hipLaunchKernelGGL((ffn_few_kernel<DUAL, ACT, TM, WIDE>), grid, block, lds, stream, x, w0, w1, (int)M, (int)N, (int)K, out, gate, up)
  if (tm == 1) MLC_FEW(1); else MLC_FEW(2);
#undef MLC_FEW
  return check_launch();
}

template <int FORM, int ACT, int BM, int BN, int NB>
int launch_tile(GemmArgs& g, const Plan& plan, double flops, double bytes, hipStream_t stream) {
  constexpr int COLS = FORM == UP || FORM == UP32 ? BN / 2 : BN;
  long tiles = 0;
  for (int i = 0; i < g.problems; ++i) {
    Problem& p = g.p[i];
    p.tiles_m = (p.M + BM - 1) / BM;
    p.tiles_n = (p.N + COLS - 1) / COLS;
    p.first = (int)tiles;
    tiles += (long)p.tiles_m * p.tiles_n;
    if (tiles > (1L << 28)) return MLC_ERR_SHAPE;
  }
  g.tiles = (int)tiles;
  g.splits = plan.splits;
  g.whole = plan.splits > 1 ? plan.whole : g.tiles;
  constexpr unsigned int lds = (BM > BN ? BM : BN) * BK * 2 * NB;
  auto kern = ffn_gemm_kernel<FORM, ACT, BM, BN, NB>;
  static std::atomic<bool> ready[MAX_DEVICES];
  const int dev = device_slot();
  if (dev < 0 || !ready[dev].load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds) != hipSuccess) return MLC_ERR_LAUNCH;
    if (dev >= 0) ready[dev].store(true, std::memory_order_release);
  }
  // as many workgroups on every XCD
  const int most = UNITS / NUM_XCD * plan.per_unit;
  const int rest = g.tiles - g.whole, per_xcd = (g.whole + NUM_XCD - 1) / NUM_XCD + (rest * g.splits + NUM_XCD - 1) / NUM_XCD;
  {
    LaunchScope scope(MLC_KERNEL_FFN, stream, flops, bytes);
    hipLaunchKernelGGL(kern, dim3((unsigned)(per_xcd < most ? per_xcd : most) * NUM_XCD), dim3(NTHREADS), lds, stream, g);
    const int rc = check_launch();
    if (rc != MLC_OK || g.whole == g.tiles) return rc;
  }
  LaunchScope scope(MLC_KERNEL_FFN, stream, 0.0, (4.0 * g.splits + 2.0) * rest * BM * BN);
  hipLaunchKernelGGL((ffn_join_kernel<BM, BN>), dim3((unsigned)rest * (BM * BN / (NTHREADS * 8))), dim3(NTHREADS), 0, stream, g);
  return check_launch();
}

template <int FORM, int ACT = 0>
int launch_form(GemmArgs& g, const Plan& plan, hipStream_t stream) {
  double flops = 0.0, bytes = 0.0;
  for (int i = 0; i < g.problems; ++i) {
    const Problem& p = g.p[i];
    constexpr bool both = FORM == UP || FORM == UP32;
    const double twice = both || FORM == NN ? 2.0 : 1.0;
    flops += 2.0 * twice * p.M * p.N * (double)p.K;
    bytes += 2.0 * (twice * ((double)p.M * p.K / (both ? 2 : 1) + (double)p.N * p.K) + (double)p.M * p.N);
  }
  if (plan.bm == 256) return launch_tile<FORM, ACT, 256, 256, 5>(g, plan, flops, bytes, stream);
  if (plan.bm == 128 && plan.per_unit == 1) return launch_tile<FORM, ACT, 128, 128, 9>(g, plan, flops, bytes, stream);
  if (plan.bm == 128) return launch_tile<FORM, ACT, 128, 128, 5>(g, plan, flops, bytes, stream);
  if (plan.per_unit == 1) return launch_tile<FORM, ACT, 64, 128, 9>(g, plan, flops, bytes, stream);
  return launch_tile<FORM, ACT, 64, 128, 5>(g, plan, flops, bytes, stream);
}

Problem problem(const bf16_t* A, long lda, const bf16_t* B, long ldb, bf16_t* D, long ldd, int64_t M, int64_t N, int64_t K) {
  Problem p{};
  p.A[0] = A; p.B[0] = B; p.lda = lda; p.ldb = ldb; p.D = D; p.ldd = ldd;
  p.M = (int)M; p.N = (int)N; p.K = (int)K;
  return p;
}

}  // namespace

size_t ffn_forward_workspace(const FfnShape& s) { return few(s.t, s.d, s.f) ? 0 : partial_bytes(plan_down(s.t, s.d, s.f)); }
size_t ffn_backward_workspace(const FfnShape& s) {
  const size_t dx = partial_bytes(plan_dx(s.t, s.d, s.f)), dw = partial_bytes(plan_dw(s.t, s.d, s.f));
  return 2 * (size_t)round_up(s.t * s.f * 2, 256) + (dx > dw ? dx : dw);
}

int launch_ffn_forward(const FfnShape& s, const bf16_t* x, const bf16_t* wg, const bf16_t* wu, const bf16_t* wd, void* gate, void* up,
                       bf16_t* hidden, bf16_t* y, void* workspace, hipStream_t stream) {
  int rc;
  const bool silu = s.act == MLC_ACT_SILU;
  if (few(s.t, s.f, s.d)) {
    auto launch = [&](auto act, auto wide) {
      return launch_few<true, decltype(act)::value, decltype(wide)::value>(x, wg, wu, s.t, s.f, s.d, hidden, gate, up, stream);
    };
    if (s.wide && gate) rc = silu ? launch(I<MLC_ACT_SILU>{}, std::true_type{}) : launch(I<MLC_ACT_GELU_TANH>{}, std::true_type{});
    else rc = silu ? launch(I<MLC_ACT_SILU>{}, std::false_type{}) : launch(I<MLC_ACT_GELU_TANH>{}, std::false_type{});
  } else {
    GemmArgs g{};
    g.problems = 1;
    g.p[0] = problem(x, s.d, wg, s.d, hidden, s.f, s.t, s.f, s.d);
    g.p[0].B[1] = wu;
    g.gate = gate; g.up = up;
    const Plan both = plan_up(s.t, s.d, s.f);
    if (s.wide && gate) rc = silu ? launch_form<UP32, MLC_ACT_SILU>(g, both, stream) : launch_form<UP32, MLC_ACT_GELU_TANH>(g, both, stream);
    else rc = silu ? launch_form<UP, MLC_ACT_SILU>(g, both, stream) : launch_form<UP, MLC_ACT_GELU_TANH>(g, both, stream);
  }
  if (rc != MLC_OK) return rc;
  if (few(s.t, s.d, s.f)) return launch_few<false, 0>(hidden, wd, wd, s.t, s.d, s.f, y, nullptr, nullptr, stream);
  GemmArgs n{};
  n.problems = 1;
  n.p[0] = problem(hidden, s.f, wd, s.f, y, s.d, s.t, s.d, s.f);
  n.partial = (float*)workspace;
  return launch_form<NT>(n, plan_down(s.t, s.d, s.f), stream);
}

int launch_ffn_backward(const FfnShape& s, const bf16_t* dy, const bf16_t* x, const bf16_t* wg, const bf16_t* wu, const bf16_t* wd,
                        const void* gate, const void* up, const bf16_t* hidden, bf16_t* dx, bf16_t* dwg, bf16_t* dwu, bf16_t* dwd,
                        void* workspace, hipStream_t stream) {
  bf16_t* const dg = (bf16_t*)workspace;
  bf16_t* const du = (bf16_t*)((unsigned char*)workspace + round_up(s.t * s.f * 2, 256));
  float* const partial = (float*)((unsigned char*)workspace + 2 * round_up(s.t * s.f * 2, 256));
  int rc = MLC_OK;
  if (s.t) {
    GemmArgs g{};
    g.problems = 1;
    g.p[0] = problem(dy, s.d, wd, s.f, dg, s.f, s.t, s.f, s.d);
    g.gate = const_cast<void*>(gate); g.up = const_cast<void*>(up); g.du = du;
    const Plan inner = plan_inner(s.t, s.d, s.f);
    rc = s.wide ? launch_form<DH32>(g, inner, stream) : launch_form<DH>(g, inner, stream);
    if (rc != MLC_OK) return rc;
    GemmArgs n{};
    n.problems = 1;
    n.p[0] = problem(dg, s.f, wg, s.d, dx, s.d, s.t, s.d, s.f);
    n.p[0].A[1] = du; n.p[0].B[1] = wu;
    n.partial = partial;
    rc = launch_form<NN>(n, plan_dx(s.t, s.d, s.f), stream);
    if (rc != MLC_OK) return rc;
  }
  GemmArgs w{};
  w.problems = 3;
  w.p[0] = problem(dg, s.f, x, s.d, dwg, s.d, s.f, s.d, s.t);
  w.p[1] = problem(du, s.f, x, s.d, dwu, s.d, s.f, s.d, s.t);
  w.p[2] = problem(dy, s.d, hidden, s.f, dwd, s.f, s.d, s.f, s.t);
  w.partial = partial;
  return launch_form<TN>(w, plan_dw(s.t, s.d, s.f), stream);
}

}  // namespace mlc

// Norm of every query and key head with the position rotation in the same pass, and its gradient.
//
// A head x of `dim` values at position p, gain w (plus an offset, 0 or 1), over its first `rot` values turned pairwise:
//   r = 1 / sqrt(mean(x^2) + eps) ; n = x r (w + offset)
//   y_a = n_a cos - n_b sin ; y_b = n_b cos + n_a sin         (cos, sin: row p of the tables; the rest of n passes)
// and backwards, with dn the rotation of dy by the negative angle:
//   dw += dn x r ; d = dn (w + offset) ; dx = r (d - x r^2 mean(d x))
// Everything is computed in fp32 from the stored values and rounded once, where it is stored.  The backward pass reads x again
// instead of a stored r: the row has to come in anyway.
//
// Bound by the memory stream: a row is read once and written once (backwards two rows in, one out).  L lanes share a row, a lane
// holds four pairs, and a group of L lanes takes HEADS heads of one token after the other, so that a row of the tables is read
// once for them, their loads are all under way together and the gains stay in registers.  16384 tokens x 32 heads of 128 in bf16: forward
// 62 us, 337 MB with the tables for every four heads, 5.4 TB/s; backward 83, 471 MB, 5.7 TB/s, and 5 for the gains' sums.  Where head or
// rotated width is no multiple of 8, elements go one by one: half that rate (100 / 100: forward 99 us, 210 MB).
//
// The gains' gradients are sums over all tokens and heads: a lane keeps its own elements' sums in registers over all rows it
// meets, a workgroup adds its lanes' and writes one partial row, and a second kernel adds the partial rows, each
// in a fixed order: the same bits whatever the timing.
#include "common.h"

namespace mlc {
namespace {

constexpr int THREADS = 256;
constexpr int MAX_HEADS = 4;
static_assert(2 * QK_MAX_HEADS <= QK_MAX_PARTIALS, "a partial row for every head");

// Four adjacent elements at an address aligned to the element, as they sit in memory (raw_t) and as floats.
template <typename T> struct Vec4;
template <> struct Vec4<float> {
  typedef f32x4 __attribute__((aligned(4))) vec_t;
  typedef f32x4 raw_t;
  static __device__ __forceinline__ raw_t raw(const float* p) { return *reinterpret_cast<const vec_t*>(p); }
  static __device__ __forceinline__ void unpack(const raw_t& a, float* v) { v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; }
  static __device__ __forceinline__ void load(const float* p, float* v) { unpack(raw(p), v); }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    f32x4 a;
    a.x = v[0]; a.y = v[1]; a.z = v[2]; a.w = v[3];
    *reinterpret_cast<vec_t*>(p) = a;
  }
};
template <> struct Vec4<bf16_t> {
  typedef u32x2 __attribute__((aligned(2))) vec_t;
  typedef u32x2 raw_t;
  static __device__ __forceinline__ raw_t raw(const bf16_t* p) { return *reinterpret_cast<const vec_t*>(p); }
  static __device__ __forceinline__ void unpack(const raw_t& a, float* v) {
    v[0] = bf16lo(a.x); v[1] = bf16hi(a.x); v[2] = bf16lo(a.y); v[3] = bf16hi(a.y);
  }
  static __device__ __forceinline__ void load(const bf16_t* p, float* v) { unpack(raw(p), v); }
  static __device__ __forceinline__ void store(bf16_t* p, const float* v) {
    u32x2 a;
    a.x = pack_bf16x2(v[0], v[1]);
    a.y = pack_bf16x2(v[2], v[3]);
    *reinterpret_cast<vec_t*>(p) = a;
  }
};

// Sum over the L lanes of an aligned group, in every one of them.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float((unsigned int)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int L>
__device__ __forceinline__ float group_sum(float x) {
  static_assert(L >= 8 && L <= 64, "8 to 64 lanes a row");
  x = add_dpp<0xb1>(x);
  x = add_dpp<0x4e>(x);
  x = add_dpp<0x141>(x);
  if constexpr (L >= 16) x = add_dpp<0x140>(x);
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

// Which elements of a head a lane holds: four pairs (a[i], b[i]).
// VEC: dim and rot are multiples of 8; pairs 4 lane .. 4 lane + 3, two runs of four adjacent elements, which are all turned or
// all passed on.  Otherwise pairs lane + L i, element by element.
template <bool VEC, bool INTER, int L>
struct Place {
  int lane, dim, rot;
  __device__ __forceinline__ int pair(int i) const { return VEC ? 4 * lane + i : lane + L * i; }
  __device__ __forceinline__ bool has(int i) const { return 2 * pair(i) < dim; }
  __device__ __forceinline__ bool turned(int i) const { return 2 * pair(i) < rot; }
  // elements of pair i (one that is passed on: any two adjacent ones)
  __device__ __forceinline__ int first(int i) const { const int p = pair(i); return !INTER && 2 * p < rot ? p : 2 * p; }
  __device__ __forceinline__ int second(int i) const { const int p = pair(i); return !INTER && 2 * p < rot ? p + rot / 2 : 2 * p + 1; }
  // of VEC: the two runs
  __device__ __forceinline__ int run0() const { return !INTER && 8 * lane < rot ? 4 * lane : 8 * lane; }
  __device__ __forceinline__ int run1() const { return !INTER && 8 * lane < rot ? 4 * lane + rot / 2 : 8 * lane + 4; }

  // a row's elements as they sit in memory, held until their head's turn: half the registers for bf16
  template <typename T> struct Raw { typename Vec4<T>::raw_t a, b; float e[VEC ? 1 : 8]; };
  template <typename T>
  __device__ __forceinline__ void fetch(const T* row, Raw<T>& r) const {
    if constexpr (VEC) {
      if (has(0)) { r.a = Vec4<T>::raw(row + run0()); r.b = Vec4<T>::raw(row + run1()); }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r.e[i] = has(i) ? Vec8<T>::load1(row + first(i)) : 0.f;
        r.e[4 + i] = has(i) ? Vec8<T>::load1(row + second(i)) : 0.f;
      }
    }
  }
  template <typename T>
  __device__ __forceinline__ void unpack(const Raw<T>& r, float (&a)[4], float (&b)[4]) const {
    if constexpr (VEC) {
      float v[8];
      Vec4<T>::unpack(r.a, v);
      Vec4<T>::unpack(r.b, v + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = has(0) ? v[INTER ? 2 * i : i] : 0.f;
        b[i] = has(0) ? v[INTER ? 2 * i + 1 : 4 + i] : 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) { a[i] = r.e[i]; b[i] = r.e[4 + i]; }
    }
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* row, float (&a)[4], float (&b)[4]) const {
    Raw<T> r;
    fetch(row, r);
    unpack(r, a, b);
  }
  template <typename T>
  __device__ __forceinline__ void store(T* row, const float (&a)[4], const float (&b)[4]) const {
    if constexpr (VEC) {
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[INTER ? 2 * i : i] = a[i]; v[INTER ? 2 * i + 1 : 4 + i] = b[i]; }
      if (has(0)) { Vec4<T>::store(row + run0(), v); Vec4<T>::store(row + run1(), v + 4); }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (has(i)) { Vec8<T>::store1(row + first(i), a[i]); Vec8<T>::store1(row + second(i), b[i]); }
    }
  }
  __device__ __forceinline__ void gain(const void* w, int dtype, float offset, float (&a)[4], float (&b)[4]) const {
    if (dtype == MLC_F32) load((const float*)w, a, b);
    else load((const bf16_t*)w, a, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] += offset; b[i] += offset; }
  }
  // cos and sin of the lane's pairs (1 and 0 where they pass); a position outside the tables reads nothing of them (they may have
  // no rows at all) and gives NaN
  __device__ __forceinline__ void angles(const QkArgs& g, long token, float (&c)[4], float (&s)[4]) const {
    if (rot == 0) {                                 // the norm alone: no positions
#pragma unroll
      for (int i = 0; i < 4; ++i) { c[i] = 1.f; s[i] = 0.f; }
      return;
    }
    const long p = g.pos64 ? ((const long*)g.positions)[token] : (long)((const int*)g.positions)[token];
    const bool in = p >= 0 && p < g.table_rows;
    const long at = in ? p * (rot / 2) : 0;
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < 4; ++i) { c[i] = 1.f; s[i] = 0.f; }
      if (in && turned(0)) { Vec4<float>::load(g.cos + at + pair(0), c); Vec4<float>::load(g.sin + at + pair(0), s); }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = in && turned(i) ? g.cos[at + pair(i)] : 1.f;
        s[i] = in && turned(i) ? g.sin[at + pair(i)] : 0.f;
      }
    }
    if (!in)
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = s[i] = __uint_as_float(0x7fc00000u);
  }
  // pair i turned by that angle; two elements that are passed on have nothing to do with each other (0 times one that is not finite
  // would be NaN in the other)
  __device__ __forceinline__ void turn(int i, float a, float b, float c, float s, float& ya, float& yb) const {
    ya = a * c - (turned(i) ? b * s : 0.f);
    yb = b * c + (turned(i) ? a * s : 0.f);
  }
};

// A workgroup's share: HEADS neighbouring heads, of the queries or of the keys, of every step-th token.  Workgroups with the
// heads of one token come one after the other.
struct Share { int key, head, heads; long token, step; };
template <int HEADS, int GROUPS>
__device__ __forceinline__ Share share_of(const QkArgs& g) {
  const int cq = (g.q_heads + HEADS - 1) / HEADS, per = cq + (g.k_heads + HEADS - 1) / HEADS;
  const int c = (int)blockIdx.x % per, n = (int)blockIdx.x / per;
  Share r;
  r.key = c >= cq;
  r.head = (r.key ? c - cq : c) * HEADS;
  r.heads = min(HEADS, (r.key ? g.k_heads : g.q_heads) - r.head);
  r.token = (long)n * GROUPS;
  r.step = (long)((int)gridDim.x / per) * GROUPS;
  return r;
}
// First row of the share's heads for a lane group's token.
template <typename T>
__device__ __forceinline__ T* rows_of(const QkRows& q, const QkRows& k, const Share& x, long token) {
  const QkRows& r = x.key ? k : q;
  return (T*)r.p + token * r.token_stride + (long)x.head * r.head_stride;
}

template <typename T, bool VEC, bool INTER, int L, int HEADS>
__global__ __launch_bounds__(THREADS) void qk_norm_rope_kernel(QkArgs g) {
  constexpr int GROUPS = THREADS / L;
  const Place<VEC, INTER, L> at{(int)threadIdx.x % L, g.dim, g.rot};
  const Share x = share_of<HEADS, GROUPS>(g);
  const long in_step = x.key ? g.k.head_stride : g.q.head_stride, out_step = x.key ? g.k_out.head_stride : g.q_out.head_stride;
  float wa[4], wb[4];
  at.gain(x.key ? g.k_gain : g.q_gain, g.gain_dtype, g.offset, wa, wb);
  for (long token = x.token + (int)threadIdx.x / L; token < g.tokens; token += x.step) {
    const T* const in = rows_of<const T>(g.q, g.k, x, token);
    T* const out = rows_of<T>(g.q_out, g.k_out, x, token);
    typename Place<VEC, INTER, L>::template Raw<T> raw[HEADS];
    float c[4], s[4];
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
      if (h < x.heads) at.fetch(in + h * in_step, raw[h]);
    at.angles(g, token, c, s);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (h >= x.heads) break;
      float a[4], b[4], ss = 0.f;
      at.unpack(raw[h], a, b);
#pragma unroll
      for (int i = 0; i < 4; ++i) ss += a[i] * a[i] + b[i] * b[i];
      const float r = rsqrtf(group_sum<L>(ss) * g.inv_dim + g.eps);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float na = a[i] * r * wa[i], nb = b[i] * r * wb[i];
        at.turn(i, na, nb, c[i], s[i], a[i], b[i]);
      }
      at.store(out + h * out_step, a, b);
    }
  }
}

template <typename T, bool VEC, bool INTER, int L, int HEADS>
__global__ __launch_bounds__(THREADS, !VEC ? 2 : sizeof(T) == 2 ? 4 : 3) void qk_norm_rope_backward_kernel(QkArgs g) {
  constexpr int GROUPS = THREADS / L;
  const Place<VEC, INTER, L> at{(int)threadIdx.x % L, g.dim, g.rot};
  const Share x = share_of<HEADS, GROUPS>(g);
  const long in_step = x.key ? g.k.head_stride : g.q.head_stride, dy_step = x.key ? g.dk_out.head_stride : g.dq_out.head_stride,
             dx_step = x.key ? g.dk.head_stride : g.dq.head_stride;
  float wa[4], wb[4], sum[8];                       // sum: the lane's part of the gain's gradient
  at.gain(x.key ? g.k_gain : g.q_gain, g.gain_dtype, g.offset, wa, wb);
#pragma unroll
  for (int i = 0; i < 8; ++i) sum[i] = 0.f;
  for (long token = x.token + (int)threadIdx.x / L; token < g.tokens; token += x.step) {
    const T* const in = rows_of<const T>(g.q, g.k, x, token);
    const T* const dy = rows_of<const T>(g.dq_out, g.dk_out, x, token);
    T* const dx = rows_of<T>(g.dq, g.dk, x, token);
    typename Place<VEC, INTER, L>::template Raw<T> raw[HEADS], rawy[HEADS];
    float c[4], s[4];
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
      if (h < x.heads) {
        at.fetch(in + h * in_step, raw[h]);
        at.fetch(dy + h * dy_step, rawy[h]);
      }
    at.angles(g, token, c, s);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (h >= x.heads) break;
      float a[4], b[4], na[4], nb[4], ss = 0.f, dot = 0.f;
      at.unpack(raw[h], a, b);
      at.unpack(rawy[h], na, nb);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ya = na[i], yb = nb[i];
        at.turn(i, ya, yb, c[i], -s[i], na[i], nb[i]);
        ss += a[i] * a[i] + b[i] * b[i];
        dot += na[i] * wa[i] * a[i] + nb[i] * wb[i] * b[i];
      }
      const float r = rsqrtf(group_sum<L>(ss) * g.inv_dim + g.eps);
      const float pull = group_sum<L>(dot) * g.inv_dim * r * r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum[i] += na[i] * (a[i] * r);
        sum[4 + i] += nb[i] * (b[i] * r);
        a[i] = r * (na[i] * wa[i] - a[i] * pull);
        b[i] = r * (nb[i] * wb[i] - b[i] * pull);
      }
      at.store(dx + h * dx_step, a, b);
    }
  }
  // the workgroup's row of the partial sums: its groups one after the other
  __shared__ float held[GROUPS][8 * L];
#pragma unroll
  for (int i = 0; i < 8; ++i) held[threadIdx.x / L][i * L + threadIdx.x % L] = sum[i];
  __syncthreads();
  float* const out = g.partials + (long)blockIdx.x * g.dim;
  for (int e = threadIdx.x; e < 8 * L; e += THREADS) {
    float v = 0.f;
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) v += held[q][e];
    const Place<VEC, INTER, L> from{e % L, g.dim, g.rot};
    const int i = e / L;
    if (from.has(i % 4)) {
      // (VEC lanes' pairs that are passed on lie in two runs unless they are interleaved)
      int el = i < 4 ? from.first(i % 4) : from.second(i % 4);
      if (VEC && !INTER && !from.turned(i % 4)) el = 8 * from.lane + i;
      out[el] = v;
    }
  }
}

// Sums of the partial rows' columns, of the queries' rows and (blockIdx.y = 1) of the keys': row n is of the queries where
// n % per < cq.  8 columns a workgroup, 128 lanes each.
constexpr int SUM_COLS = 8, SUM_LANES = 128, SUM_THREADS = SUM_COLS * SUM_LANES;
__global__ __launch_bounds__(SUM_THREADS) void qk_gain_sum_kernel(const float* partials, int rows, int cq, int per, int dim,
                                                                  float* dq_gain, float* dk_gain) {
  const int col = blockIdx.x * SUM_COLS + threadIdx.x % SUM_COLS, lane = threadIdx.x / SUM_COLS;
  const int c0 = blockIdx.y ? cq : 0, cs = blockIdx.y ? per - cq : cq, n = rows / per * cs;      // rows of this kind
  float v = 0.f;
  if (col < dim)
#pragma unroll 4
    for (int r = lane; r < n; r += SUM_LANES) v += partials[(long)(r / cs * per + c0 + r % cs) * dim + col];
  __shared__ float held[SUM_LANES][SUM_COLS + 1];
  held[lane][threadIdx.x % SUM_COLS] = v;
  __syncthreads();
  for (int w = SUM_LANES / 2; w > 0; w /= 2) {
    if (lane < w) held[lane][threadIdx.x % SUM_COLS] += held[lane + w][threadIdx.x % SUM_COLS];
    __syncthreads();
  }
  float* const out = blockIdx.y ? dk_gain : dq_gain;
  if (lane == 0 && col < dim && out) out[col] = held[0][threadIdx.x];
}

int check_launch() { return hipGetLastError() == hipSuccess ? MLC_OK : MLC_ERR_LAUNCH; }

template <typename T, bool VEC, bool INTER, int L>
int launch_one(QkArgs& g, bool backward, hipStream_t stream) {
  constexpr int GROUPS = THREADS / L;
  auto chunks = [](int n, int heads) { return (n + heads - 1) / heads; };
  const long blocks = (g.tokens + GROUPS - 1) / GROUPS;
  // Several heads a group once that leaves every compute unit eight workgroups; before that the rows are spread out.  (Heads that
  // are loaded element by element go one by one: four of them need more registers than there are.)
  constexpr int MANY = VEC ? MAX_HEADS : 1;
  const bool many = blocks * (chunks(g.q_heads, MANY) + chunks(g.k_heads, MANY)) >= 2048;
  const int heads = many ? MANY : 1, cq = chunks(g.q_heads, heads), per = cq + chunks(g.k_heads, heads);
  const long most = (backward ? QK_MAX_PARTIALS : 1L << 20) / per;
  const unsigned int grid = (unsigned int)(blocks > most ? most : blocks > 0 ? blocks : 1) * per;      // (no tokens: gradients of 0)
  const double row_bytes = (double)g.tokens * (g.q_heads + g.k_heads) * g.dim * sizeof(T);
  LaunchScope scope(MLC_KERNEL_QK_NORM, stream, 0.0, row_bytes * (backward ? 3 : 2));
#define MLC_QK(KERN, H) hipLaunchKernelGGL((KERN<T, VEC, INTER, L, H>), dim3(grid), dim3(THREADS), 0, stream, g)
  if (backward) {
    if (many) MLC_QK(qk_norm_rope_backward_kernel, MANY); else MLC_QK(qk_norm_rope_backward_kernel, 1);
    const int rc = check_launch();
    if (rc != MLC_OK) return rc;
    hipLaunchKernelGGL(qk_gain_sum_kernel, dim3((unsigned)((g.dim + SUM_COLS - 1) / SUM_COLS), g.dk_gain ? 2 : 1), dim3(SUM_THREADS),
                       0, stream, g.partials, (int)grid, cq, per, g.dim, g.dq_gain, g.dk_gain);
  } else {
    if (many) MLC_QK(qk_norm_rope_kernel, MANY); else MLC_QK(qk_norm_rope_kernel, 1);
  }
#undef MLC_QK
  return check_launch();
}

template <typename T, bool VEC, bool INTER>
int launch_lanes(QkArgs& g, bool backward, hipStream_t stream) {
  const int pairs = g.dim / 2;                      // four a lane
  if (pairs <= 4 * 8) return launch_one<T, VEC, INTER, 8>(g, backward, stream);
  if (pairs <= 4 * 16) return launch_one<T, VEC, INTER, 16>(g, backward, stream);
  if (pairs <= 4 * 32) return launch_one<T, VEC, INTER, 32>(g, backward, stream);
  return launch_one<T, VEC, INTER, 64>(g, backward, stream);
}
template <typename T>
int launch_form(QkArgs& g, int interleaved, bool backward, hipStream_t stream) {
  const bool vec = g.dim % 8 == 0 && g.rot % 8 == 0;
  if (interleaved) return vec ? launch_lanes<T, true, true>(g, backward, stream) : launch_lanes<T, false, true>(g, backward, stream);
  return vec ? launch_lanes<T, true, false>(g, backward, stream) : launch_lanes<T, false, false>(g, backward, stream);
}

}  // namespace

int launch_qk_norm_rope(QkArgs g, int dtype, int interleaved, bool backward, hipStream_t stream) {
  return dtype == MLC_F32 ? launch_form<float>(g, interleaved, backward, stream) : launch_form<bf16_t>(g, interleaved, backward, stream);
}

}  // namespace mlc

// AdamW with both states held in 8 bits, over many tensors (paper Sec. 4 "AdamW inner updates" for the step itself):
//   m <- b1 m + (1 - b1) g ; v <- b2 v + (1 - b2) g^2
//   theta <- theta - lr * (m * c1) / (sqrt(v) * c2 + eps) - lr * lambda * theta
// as in adamw_kernel (inner_elementwise.hip), with m and v read from and written to codes.
//
// A tensor's elements, in their order in memory, form blocks of 256 that share two fp32 scales, the block's largest |m| and
// largest v.  A code is a small floating-point number relative to the scale: for m a sign, four exponent and three
// mantissa bits (1.125 2^-15 .. 1, and 0), for v, which is never negative but spans the square of the range, five exponent
// and three mantissa bits (1.125 2^-31 .. 1, and 0).  Evenly spaced levels would send the smaller half of a block's second
// moments to 0 and their steps to m / eps; here a v > 0 keeps at least the smallest code, so sqrt(v) >= 2^-15.4 of the
// block's largest and m, which is 0 below 2^-14.9 of its largest, cannot outgrow it.  The largest element's code stands for
// exactly the scale, so a block's magnitude follows its moving average without rounding.
//
// Rounding, from the first level on: to the nearest code, or (with a seed) up with the probability that makes the mean exact.  To the
// nearest, an average that moves by less than half a step of its code (1 / 16 of its value) stands still next to its
// block's largest; with rounding by chance it moves at the right rate on average.  Below the first level neither holds: an m up to
// 2^-15 of its block's largest becomes 0 whatever the seed (so an element with gradients that small beside an outlier's is moved by
// its newest gradient's part of the average alone), and a v > 0 becomes the first level.  The 20 bits per element come from a
// hash of (seed, block), moved on by an odd constant from element to element: one hash per block, and over the steps every
// element's sequence is as the hash's.  (A tensor's blocks count from 0: tensors of one call share their blocks' hashes.)
//
// All sums and products of the states are single fp32 operations in a fixed order (no contraction), so that codes are
// reproducible bit for bit.
#include "common.h"

namespace mlc {
namespace {

constexpr int THREADS = 256;
constexpr int BLOCK = MLC_ADAMW8_BLOCK;
constexpr int LANES = BLOCK / 8;                  // lanes per block, 8 elements each
constexpr int CHUNK = THREADS * 8 * 4;            // elements of a workgroup: whole blocks
static_assert(CHUNK % BLOCK == 0 && LANES == 32, "a block is half a wavefront's elements");
constexpr unsigned int M_OFF = 896, M_TOP = 120;  // exponent of the first code and the code of 1.0, eight codes an exponent
constexpr unsigned int V_OFF = 768, V_TOP = 248;

struct Seg { void* theta; const void* grad; uint8_t* m8; uint8_t* v8; float* scales; long n; };
template <int SEG> struct Table { Seg s[SEG]; unsigned int blk0[SEG]; };
struct ValueSeg { const uint8_t* m8; const uint8_t* v8; const float* scales; float* m; float* v; long n; };
template <int SEG> struct ValueTable { ValueSeg s[SEG]; unsigned int blk0[SEG]; };
struct Scalars { float b1, a1, b2, a2, lr, eps, decay, c1, c2; unsigned int seed; };

// Up to 8 codes from an address of any alignment; those beyond cnt are 0.
typedef u32x2 __attribute__((aligned(1))) u32x2_any;
__device__ __forceinline__ u32x2 load_codes(const uint8_t* p, int cnt) {
  if (cnt >= 8) return *reinterpret_cast<const u32x2_any*>(p);
  u32x2 w = {0u, 0u};
#pragma unroll
  for (int j = 0; j < 8; ++j) if (j < cnt) w[j / 4] |= (unsigned int)p[j] << (8 * (j & 3));
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, u32x2 w, int cnt) {
  if (cnt >= 8) {
    *reinterpret_cast<u32x2_any*>(p) = w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) if (j < cnt) p[j] = (uint8_t)(w[j / 4] >> (8 * (j & 3)));
  }
}

// Value of a code relative to the scale, without its sign.
__device__ __forceinline__ float level(unsigned int code, unsigned int off) {
  return code ? __uint_as_float((code + off) << 20) : 0.f;
}
__device__ __forceinline__ float m_value(unsigned int code, float scale) {
  const float x = __uint_as_float(__float_as_uint(level(code & 127u, M_OFF)) | ((code & 128u) << 24));
  return x * scale;
}

// The largest of 32 lanes' values (of an aligned half of the wavefront), in every one of them.
template <int CTRL>
__device__ __forceinline__ unsigned int max_dpp(unsigned int x) {
  return max(x, (unsigned int)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ unsigned int half_max(unsigned int x) {
  x = max_dpp<0xb1>(x);        // the neighbour
  x = max_dpp<0x4e>(x);        // two further
  x = max_dpp<0x141>(x);       // mirrored within 8
  x = max_dpp<0x140>(x);       // mirrored within 16
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);       // the other 16
  return max(r[0], r[1]);
}

__device__ __forceinline__ unsigned int block_hash(unsigned int block, unsigned int seed) {
  unsigned int h = block * 0x9E3779B1u + seed;
  h = (h ^ (h >> 16)) * 0x6C8E9CF5u;
  h = (h ^ (h >> 15)) * 0x7D1A93B7u;
  return h ^ (h >> 16);
}

// SEG: entries of the table (one lane each).
template <int SEG, typename Tab>
__device__ __forceinline__ int find_seg(const Tab& tab) {
  static_assert(SEG == 1 || SEG == 64, "one lane per tensor");
  if (SEG == 1) return 0;
  const bool below = blockIdx.x >= tab.blk0[threadIdx.x & 63];      // 0xffffffff beyond the last tensor
  return __builtin_amdgcn_readfirstlane(__popcll(__ballot(below)) - 1);
}

// One lane's 8 elements and its half of a wavefront's block.  FULL: all 8 are there, of every lane.
template <typename WT, typename GT, bool DITHER, bool FULL>
__device__ __forceinline__ void eight(const Seg& sg, long off, const Scalars& h) {
#pragma clang fp contract(off)
  WT* const theta = (WT*)sg.theta + off;
  const GT* const grad = (const GT*)sg.grad + off;
  const int cnt = FULL ? 8 : (int)max(0L, min(8L, sg.n - off));
  const long blk = off / BLOCK;
  float th[8], g[8], m[8], v[8];
  u32x2 cm = {0u, 0u}, cv = {0u, 0u};
  float sm = 0.f, sv = 0.f;
  if (!FULL)
#pragma unroll
    for (int j = 0; j < 8; ++j) th[j] = g[j] = 0.f;
  if (cnt > 0) {
    Vec8<WT>::unpack(Vec8U<WT>::load_raw(theta, cnt), th);
    Vec8<GT>::unpack(Vec8U<GT>::load_raw(grad, cnt), g);
    cm = load_codes(sg.m8 + off, cnt);
    cv = load_codes(sg.v8 + off, cnt);
    sm = sg.scales[2 * blk];
    sv = sg.scales[2 * blk + 1];
  }
  unsigned int tm = 0, tv = 0;                      // largest |m| and v, as bits: what is not finite is larger than all that is
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float m0 = m_value((cm[j / 4] >> (8 * (j & 3))) & 255u, sm);
    const float v0 = level((cv[j / 4] >> (8 * (j & 3))) & 255u, V_OFF) * sv;
    m[j] = h.b1 * m0 + h.a1 * g[j];
    v[j] = h.b2 * v0 + (h.a2 * g[j]) * g[j];
    if (!FULL && j >= cnt) m[j] = v[j] = 0.f;       // (the scale of a block that is not finite times nothing)
    tm = max(tm, __float_as_uint(m[j]) & 0x7fffffffu);
    tv = max(tv, __float_as_uint(v[j]));
  }
  tm = half_max(tm);
  tv = half_max(tv) & 0x7fffffffu;                  // (v is not negative; NaN may carry a sign)
  // The step itself.  Not needed bit for bit: the hardware's root and reciprocal, an ulp off, as long as eps outweighs what they
  // make of numbers below the normal ones (1e-19 after the root).
  if (h.eps >= 1e-12f) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float step = (m[j] * h.c1) * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[j]), h.c2, h.eps));
      th[j] = fmaf(-h.lr, step, fmaf(-h.decay, th[j], th[j]));
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float step = (m[j] * h.c1) / (sqrtf(v[j]) * h.c2 + h.eps);
      th[j] = th[j] - h.lr * step - h.decay * th[j];
    }
  }
  // (below the normal numbers a scale has no reciprocal: such a block counts as 0)
  if (tm < 0x00800000u) tm = 0;
  if (tv < 0x00800000u) tv = 0;
  const float im = tm ? 1.0f / __uint_as_float(tm) : 0.f, iv = tv ? 1.0f / __uint_as_float(tv) : 0.f;
  const unsigned int least = tv ? 1u : 0u;
  // what is added to a value's bits: half a step, or a part of one by chance, less the place of code 0
  int rm = (1 << 19) - (int)(M_OFF << 20), rv = (1 << 19) - (int)(V_OFF << 20);
  unsigned int hm = 0, hv = 0;
  if (DITHER) {
    const unsigned int hash = block_hash((unsigned int)blk, h.seed), e = 8u * (threadIdx.x % LANES);
    hm = hash + e * 0x9E3779B1u;
    hv = (hash ^ 0x5A5A5A5Au) + e * 0x85EBCA77u;
  }
  cm = cv = u32x2{0u, 0u};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    if (DITHER) {
      rm = (int)((hm + j * 0x9E3779B1u) >> 12) - (int)(M_OFF << 20);
      rv = (int)((hv + j * 0x85EBCA77u) >> 12) - (int)(V_OFF << 20);
    }
    const int bm = __float_as_int(fabsf(m[j]) * im) & 0x7fffffff, bv = __float_as_int(v[j] * iv) & 0x7fffffff;
    const int em = min(max((bm + rm) >> 20, 0), (int)M_TOP);
    const int ev = min(max((bv + rv) >> 20, (int)min(__float_as_uint(v[j]), least)), (int)V_TOP);
    const unsigned int sign = m[j] < 0.f ? 128u : 0u;
    cm[j / 4] |= ((unsigned int)em | sign) << (8 * (j & 3));
    cv[j / 4] |= (unsigned int)ev << (8 * (j & 3));
  }
  if (cnt > 0) {
    Vec8U<WT>::store(theta, th, cnt);
    store_codes(sg.m8 + off, cm, cnt);
    store_codes(sg.v8 + off, cv, cnt);
    if (threadIdx.x % LANES == 0) {
      sg.scales[2 * blk] = __uint_as_float(tm);
      sg.scales[2 * blk + 1] = __uint_as_float(tv);
    }
  }
}

// 10 bytes an element for bf16 parameters and gradients, bound by their stream: 65.5 million in 140 us (4.7 TB/s), 164 million in 290
// (5.7).
template <typename WT, typename GT, int SEG, bool DITHER>
__global__ __launch_bounds__(THREADS) void adamw8_kernel(Table<SEG> tab, Scalars h) {
  const int si = find_seg<SEG>(tab);
  const Seg sg = tab.s[si];
  const long first = (long)(blockIdx.x - tab.blk0[si]) * CHUNK;
#pragma unroll 1
  for (int u = 0; u < CHUNK / (THREADS * 8); ++u) {
    const long base = first + (long)u * THREADS * 8, off = base + (int)threadIdx.x * 8;
    if (base >= sg.n) break;                        // the whole workgroup
    if (base + THREADS * 8 <= sg.n) eight<WT, GT, DITHER, true>(sg, off, h);
    else eight<WT, GT, DITHER, false>(sg, off, h);
  }
}

// The values that states stand for: 2 bytes read and 8 written an element, four elements a lane, so that a wavefront's stores
// are whole kilobytes, past the caches: 109 us for 65.5 million elements, 0.66 GB (eight a lane, half lines at a time, 170), and 290
// to 330 for 164 million, 1.64 GB.
template <int SEG>
__global__ __launch_bounds__(THREADS) void adamw8_values_kernel(ValueTable<SEG> tab) {
  typedef unsigned int __attribute__((aligned(1))) u32_any;
  typedef f32x4 __attribute__((aligned(4))) f32x4_any;
  const int si = find_seg<SEG>(tab);
  const ValueSeg sg = tab.s[si];
  const long first = (long)(blockIdx.x - tab.blk0[si]) * CHUNK;
#pragma unroll
  for (int u = 0; u < CHUNK / (THREADS * 4); ++u) {
    const long off = first + (u * THREADS + (int)threadIdx.x) * 4;
    if (off >= sg.n) break;
    const int cnt = (int)min(4L, sg.n - off);
    const float sm = sg.scales[2 * (off / BLOCK)], sv = sg.scales[2 * (off / BLOCK) + 1];
    if (cnt == 4) {
      const unsigned int cm = *reinterpret_cast<const u32_any*>(sg.m8 + off), cv = *reinterpret_cast<const u32_any*>(sg.v8 + off);
      f32x4 m, v;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        m[j] = m_value((cm >> (8 * j)) & 255u, sm);
        v[j] = level((cv >> (8 * j)) & 255u, V_OFF) * sv;
      }
      __builtin_nontemporal_store(m, reinterpret_cast<f32x4_any*>(sg.m + off));
      __builtin_nontemporal_store(v, reinterpret_cast<f32x4_any*>(sg.v + off));
    } else {
      for (int j = 0; j < cnt; ++j) {
        sg.m[off + j] = m_value(sg.m8[off + j], sm);
        sg.v[off + j] = level(sg.v8[off + j], V_OFF) * sv;
      }
    }
  }
}

int check_launch() { return hipGetLastError() == hipSuccess ? MLC_OK : MLC_ERR_LAUNCH; }

// First workgroups of n tensors; false where they are too many for one launch.
template <typename Group>
bool deal_chunks(const Group* gs, int n, int seg, unsigned int* blk0, unsigned long* blocks) {
  unsigned long blk = 0;
  for (int i = 0; i < seg; ++i) {
    blk0[i] = i < n ? (unsigned int)blk : 0xffffffffu;
    if (i < n) blk += (unsigned long)((gs[i].count + CHUNK - 1) / CHUNK);
    if (blk > 0x7fffffffUL) return false;
  }
  *blocks = blk;
  return true;
}

template <int SEG>
int launch_step(const mlc_adamw8_group* gs, int n, const Scalars& h, bool dither, hipStream_t stream) {
  Table<SEG> tab;
  unsigned long blk;
  if (!deal_chunks(gs, n, SEG, tab.blk0, &blk)) return MLC_ERR_SHAPE;
  const int wd = gs[0].param_dtype, gd = gs[0].grad_dtype;
  double bytes = 0.0;
  for (int i = 0; i < SEG; ++i) {
    const mlc_adamw8_group& g = gs[i < n ? i : 0];
    tab.s[i] = Seg{g.param, g.grad, g.exp_avg, g.exp_avg_sq, g.scales, (long)g.count};
    if (i < n) bytes += (double)g.count * (2 * (wd == MLC_F32 ? 4 : 2) + (gd == MLC_F32 ? 4 : 2) + 4 + 16.0 / BLOCK);
  }
  LaunchScope scope(MLC_KERNEL_ADAMW8, stream, 0.0, bytes);
#define MLC_AW(WT, GT)                                                                                                       \
  do {                                                                                                                       \
    if (dither) hipLaunchKernelGGL((adamw8_kernel<WT, GT, SEG, true>), dim3((unsigned)blk), dim3(THREADS), 0, stream, tab, h); \
    else hipLaunchKernelGGL((adamw8_kernel<WT, GT, SEG, false>), dim3((unsigned)blk), dim3(THREADS), 0, stream, tab, h);     \
  } while (0)
  if (wd == MLC_F32 && gd == MLC_F32) MLC_AW(float, float);
  else if (wd == MLC_F32) MLC_AW(float, bf16_t);
  else if (gd == MLC_F32) MLC_AW(bf16_t, float);
  else MLC_AW(bf16_t, bf16_t);
#undef MLC_AW
  return check_launch();
}

template <int SEG>
int launch_values(const mlc_adamw8_group* gs, float* const* m, float* const* v, int n, hipStream_t stream) {
  ValueTable<SEG> tab;
  unsigned long blk;
  if (!deal_chunks(gs, n, SEG, tab.blk0, &blk)) return MLC_ERR_SHAPE;
  double bytes = 0.0;
  for (int i = 0; i < SEG; ++i) {
    const int x = i < n ? i : 0;
    tab.s[i] = ValueSeg{gs[x].exp_avg, gs[x].exp_avg_sq, gs[x].scales, m[x], v[x], (long)gs[x].count};
    if (i < n) bytes += (double)gs[x].count * (10 + 8.0 / BLOCK);
  }
  LaunchScope scope(MLC_KERNEL_ADAMW8, stream, 0.0, bytes);
  hipLaunchKernelGGL((adamw8_values_kernel<SEG>), dim3((unsigned)blk), dim3(THREADS), 0, stream, tab);
  return check_launch();
}

}  // namespace

int launch_adamw8(const mlc_adamw8_group* gs, int n, float lr, float b1, float b2, float eps, float decay, float c1, float c2,
                  bool dither, unsigned int seed, hipStream_t stream) {
  const Scalars h{b1, 1.0f - b1, b2, 1.0f - b2, lr, eps, decay, c1, c2, seed};
  return n == 1 ? launch_step<1>(gs, n, h, dither, stream) : launch_step<ADAMW_MAX_SEG>(gs, n, h, dither, stream);
}

int launch_adamw8_values(const mlc_adamw8_group* gs, float* const* m, float* const* v, int n, hipStream_t stream) {
  return n == 1 ? launch_values<1>(gs, m, v, n, stream) : launch_values<ADAMW_MAX_SEG>(gs, m, v, n, stream);
}

}  // namespace mlc

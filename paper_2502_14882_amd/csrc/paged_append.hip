// Rotary positions with several axes, and growth of the paged e4m3 cache.
//
// Rotation.  Pair (a, b) of channels of a head, angle t = position on the pair's axis * frequency:
//     a' = a cos t - b sin t,   b' = b cos t + a sin t;
// its gradient is the rotation by -t.  The angle is formed in fp64 (the product of an int32 and an fp32 is exact there),
// brought to a fraction of a turn with 1 / (2 pi) in two parts, and cos and sin are Taylor sums on [-pi/4, pi/4] to 2e-16,
// rounded to fp32: positions of millions of tokens keep all of fp32's bits, and no table has to be read.  About 35
// fp64 instructions for a pair, shared by the heads that a thread turns.
// Bound: HBM, every element is read and written once.
//
// Append.  For page and head: e = exponent of the largest new magnitude, scale 2^e, codes = e4m3(x / scale).
// A workgroup takes one page of one head of the keys or of the values, so it alone decides the scale; its new elements stay in
// registers between the maximum and the codes.  The values lie channel by channel in a page (attention then
// reads a channel's tokens as one operand), so they turn in LDS on the way.
#include "paged_device.h"

namespace cq {
namespace {

struct CosSin {
  float c[8], s[8];
};

// cos and sin of a (radians), to fp64 accuracy before the one rounding
__device__ inline void cos_sin(double a, float* c, float* s) {
  constexpr double kTurnHi = 0x1.45f306dc9c883p-3, kTurnLo = -0x1.6b01ec5417056p-57;   // 1 / (2 pi)
  constexpr double kTwoPi = 0x1.921fb54442d18p+2;
  const double n = __builtin_rint(a * kTurnHi);
  const double r = __builtin_fma(a, kTurnHi, -n) + a * kTurnLo;     // turns, in [-1/2, 1/2]
  const double quarter = __builtin_rint(4.0 * r);
  const double x = __builtin_fma(quarter, -0.25, r) * kTwoPi, y = x * x;
  double p = 1.0 / 6227020800.0;                                    // x^13 / 13!
  p = __builtin_fma(p, y, -1.0 / 39916800.0);
  p = __builtin_fma(p, y, 1.0 / 362880.0);
  p = __builtin_fma(p, y, -1.0 / 5040.0);
  p = __builtin_fma(p, y, 1.0 / 120.0);
  p = __builtin_fma(p, y, -1.0 / 6.0);
  const double sn = __builtin_fma(p * y, x, x);
  double q = -1.0 / 87178291200.0;                                  // x^14 / 14!
  q = __builtin_fma(q, y, 1.0 / 479001600.0);
  q = __builtin_fma(q, y, -1.0 / 3628800.0);
  q = __builtin_fma(q, y, 1.0 / 40320.0);
  q = __builtin_fma(q, y, -1.0 / 720.0);
  q = __builtin_fma(q, y, 1.0 / 24.0);
  q = __builtin_fma(q, y, -0.5);
  const double cs = __builtin_fma(q, y, 1.0);
  const int k = (int)quarter & 3;                                   // NaN and infinities: x is NaN, whatever k is
  const float fs = (float)((k & 1) ? cs : sn), fc = (float)((k & 1) ? sn : cs);
  *s = (k & 2) ? -fs : fs;
  *c = ((k + 1) & 2) ? -fc : fc;
}

// A unit: 16 channels of a head in two pieces of eight.  Units below half / 8 hold eight whole pairs: channels 8 u.. and
// half + 8 u.. of halves, 16 u.. of adjacent pairs.  The units behind them are not turned.
__device__ inline void unit_channels(const RopeArgs& rope, int u, int* c0, int* c1) {
  if (8 * u < rope.half && !rope.adjacent) {
    *c0 = 8 * u;
    *c1 = rope.half + 8 * u;
  } else {
    *c0 = 16 * u;
    *c1 = 16 * u + 8;
  }
}
__device__ inline bool unit_turns(const RopeArgs& rope, int u) { return 8 * u < rope.half; }

__device__ inline void unit_angles(const RopeArgs& rope, int n_tokens, int token, int u, CosSin* cs) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int pair = 8 * u + i;
    const int pos = rope.positions[(size_t)rope.axis_of[pair] * n_tokens + token];
    cos_sin((double)pos * (double)rope.inv_freq[pair], &cs->c[i], &cs->s[i]);
    cs->s[i] *= rope.sign;
  }
}

__device__ inline void turn_unit(const RopeArgs& rope, const CosSin& cs, float* x) {
#pragma clang fp contract(off)
  if (rope.adjacent) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[2 * i], b = x[2 * i + 1];
      x[2 * i] = a * cs.c[i] - b * cs.s[i];
      x[2 * i + 1] = b * cs.c[i] + a * cs.s[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float a = x[i], b = x[8 + i];
      x[i] = a * cs.c[i] - b * cs.s[i];
      x[8 + i] = b * cs.c[i] + a * cs.s[i];
    }
  }
}

template <bool BF16>
__device__ inline void load_unit(const HeadRows& t, long long token, int head, int c0, int c1, float* x) {
  const uint16_t* p = static_cast<const uint16_t*>(t.data) + token * t.token_stride + head * t.head_stride;
  const v4u a = *reinterpret_cast<const v4u*>(p + c0), b = *reinterpret_cast<const v4u*>(p + c1);
  widen8<BF16>(a, x);
  widen8<BF16>(b, x + 8);
}

// Thread -> (token, group of heads, unit), units fastest.  The heads of two tensors are counted through.
struct RotateWork {
  HeadRows in[2], out[2];
  int n_tokens, units, heads_per_thread, groups;
};

template <bool BF16>
__device__ inline void rotate_thread(const RopeArgs& rope, const RotateWork& w, long long i) {
  const int u = (int)(i % w.units);
  const long long rest = i / w.units;
  const int group = (int)(rest % w.groups);
  const long long token = rest / w.groups;
  if (token >= w.n_tokens) return;
  const int heads = w.in[0].heads + w.in[1].heads;
  const int h0 = group * w.heads_per_thread;
  const int h1 = h0 + w.heads_per_thread < heads ? h0 + w.heads_per_thread : heads;
  int c0, c1;
  unit_channels(rope, u, &c0, &c1);
  const bool turns = unit_turns(rope, u);
  CosSin cs;
  if (turns) unit_angles(rope, w.n_tokens, (int)token, u, &cs);
  for (int h = h0; h < h1; ++h) {
    const int t = h >= w.in[0].heads, head = t ? h - w.in[0].heads : h;
    float x[16];
    load_unit<BF16>(w.in[t], token, head, c0, c1, x);
    if (turns) turn_unit(rope, cs, x);
    uint16_t* p = static_cast<uint16_t*>(w.out[t].data) + token * w.out[t].token_stride + head * w.out[t].head_stride;
    *reinterpret_cast<v4u*>(p + c0) = narrow8<BF16>(x);
    *reinterpret_cast<v4u*>(p + c1) = narrow8<BF16>(x + 8);
  }
}

template <bool BF16>
__global__ void __launch_bounds__(256) rotate_kernel(RopeArgs rope, RotateWork w) {
  rotate_thread<BF16>(rope, w, (long long)blockIdx.x * 256 + threadIdx.x);
}

// As many heads to a thread as leave the chip 2^18 threads (four waves to a SIMD), eight at most: the angles are then formed
// once for them.
RotateWork plan_rotate(int n_tokens, int d, const HeadRows* in, const HeadRows* out, int n_tensors) {
  RotateWork w = {};
  for (int i = 0; i < n_tensors; ++i) {
    w.in[i] = in[i];
    w.out[i] = out[i];
  }
  w.n_tokens = n_tokens;
  w.units = d / 16;
  const int heads = w.in[0].heads + w.in[1].heads;
  const long long items = (long long)n_tokens * w.units * heads;
  const long long per = items >> 18;
  w.heads_per_thread = per < 1 ? 1 : per > 8 ? 8 : (int)per;
  if (w.heads_per_thread > heads) w.heads_per_thread = heads;
  w.groups = ceil_div(heads, w.heads_per_thread);
  return w;
}
long long rotate_threads(const RotateWork& w) { return (long long)w.n_tokens * w.units * w.groups; }

// ---- append
constexpr int kItems = 4;          // units that a thread holds
constexpr float kMinScale = 0x1p-100f;

// The smallest power of two s >= 2^-100 with m <= 448 s: 448 = 1.75 * 2^8, so the exponent rises where the
// significand of m is above 1.75.
__device__ inline float scale_for(float m) {
  const unsigned bits = __builtin_bit_cast(unsigned, m) + 0x1fffffu;
  const int e = (int)(bits >> 23) - 127 - 8;
  return e < -100 ? kMinScale : __builtin_bit_cast(float, (unsigned)(e + 127) << 23);
}

struct AppendArgs {
  PagedCacheArgs cache;
  PagedBatch batch;
  HeadRows k, v;
  RopeArgs rope;
  RotateWork q;
  int tasks;               // pages that a sequence's new tokens can reach
  unsigned page_blocks;    // workgroups for pages; those behind turn queries
};

// x / scale for codes: NaN for what is not finite
__device__ inline float coded(float x, float inv) { return __builtin_isfinite(x) ? x * inv : __builtin_nanf(""); }

template <bool BF16>
__global__ void __launch_bounds__(1024) append_kernel(AppendArgs a) {
  extern __shared__ __align__(16) uint8_t s_turn[];          // values: [d][page + 4]
  __shared__ float s_most[16];
  const int tid = threadIdx.x, threads = blockDim.x;
  unsigned id = blockIdx.x;
  if (id >= a.page_blocks) {
    rotate_thread<BF16>(a.rope, a.q, (long long)(id - a.page_blocks) * threads + tid);
    return;
  }
  const PagedCacheArgs& C = a.cache;
  const bool value = id & 1;
  id >>= 1;
  const int h = (int)(id % (unsigned)C.heads);
  id /= (unsigned)C.heads;
  const int task = (int)(id % (unsigned)a.tasks), b = (int)(id / (unsigned)a.tasks);
  const Sequence s = load_sequence(a.batch, b);
  if (s.n == 0) return;
  // the sequence's places [from, to) that have a new row
  const int from = s.pos0 > 0 ? s.pos0 : 0, to = s.pos0 + s.n;
  const int index = (from >> C.page_log2) + task, place = index << C.page_log2;
  if (place >= to || to <= from) return;
  const int pid = a.batch.page_table[(size_t)b * a.batch.max_pages + index];      // place < to <= len: within the row
  if ((unsigned)pid >= (unsigned)C.n_pages) return;
  const int s0 = from > place ? from - place : 0, s1 = to - place < C.page ? to - place : C.page;
  const int live = s1 - s0, units = C.d / 16;
  const int row0 = s.first + place + s0 - s.pos0;

  // the new elements, and their largest magnitude
  float x[kItems][16];
  int c0[kItems], c1[kItems];
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int item = tid + i * threads;
    if (item < live * units) {
      const int row = row0 + item / units, u = item % units;
      if (value) {
        c0[i] = 16 * u;
        c1[i] = 16 * u + 8;
        load_unit<BF16>(a.v, row, h, c0[i], c1[i], x[i]);
      } else {
        unit_channels(a.rope, u, &c0[i], &c1[i]);
        load_unit<BF16>(a.k, row, h, c0[i], c1[i], x[i]);
        if (unit_turns(a.rope, u)) {
          CosSin cs;
          unit_angles(a.rope, a.batch.n_tokens, row, u, &cs);
          turn_unit(a.rope, cs, x[i]);
        }
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) most = fmaxf(most, __builtin_isfinite(x[i][j]) ? fabsf(x[i][j]) : 0.f);
    }
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
  if ((tid & 63) == 0) s_most[tid >> 6] = most;
  __syncthreads();
  most = s_most[0];
  for (int w = 1; w < (threads >> 6); ++w) most = fmaxf(most, s_most[w]);

  const size_t head = (size_t)pid * C.heads + h;
  float* scale_at = (value ? C.v_scale : C.k_scale) + head;
  uint8_t* codes = (value ? C.v_codes : C.k_codes) + (head << C.page_log2) * C.d;
  float scale = scale_for(most);
  if (s0 > 0) {
    const float old = *scale_at;
    if (old >= scale) {
      scale = old;
    } else {
      const float ratio = old / scale;
      for (int i = tid; i < C.page * C.d / 16; i += threads) {
        v4u w = reinterpret_cast<v4u*>(codes)[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[j], true);
          w[j] = code4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
        }
        reinterpret_cast<v4u*>(codes)[i] = w;
      }
    }
    __syncthreads();       // everybody has read the scale; the old codes are in place before the new ones
  }
  if (tid == 0) *scale_at = scale;

  const float inv = 1.0f / scale;       // exact: a power of two
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    const int item = tid + i * threads;
    if (item >= live * units) continue;
    const int slot = s0 + item / units;
    unsigned w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = code4(coded(x[i][4 * j], inv), coded(x[i][4 * j + 1], inv), coded(x[i][4 * j + 2], inv),
                   coded(x[i][4 * j + 3], inv));
    if (!value) {
      uint8_t* p = codes + (size_t)slot * C.d;
      *reinterpret_cast<v2u*>(p + c0[i]) = (v2u){w[0], w[1]};
      *reinterpret_cast<v2u*>(p + c1[i]) = (v2u){w[2], w[3]};
    } else if (live < 4) {
#pragma unroll
      for (int j = 0; j < 16; ++j) codes[((size_t)(c0[i] + j) << C.page_log2) + slot] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
    } else {
#pragma unroll
      for (int j = 0; j < 16; ++j) s_turn[(c0[i] + j) * (C.page + 4) + slot] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
    }
  }
  if (value && live >= 4) {
    __syncthreads();
    const int quads = C.page / 4;
    for (int i = tid; i < C.d * quads; i += threads) {
      const int c = i / quads, t = 4 * (i % quads);
      const uint8_t* from_lds = s_turn + c * (C.page + 4) + t;
      uint8_t* p = codes + ((size_t)c << C.page_log2) + t;
      if (t >= s0 && t + 4 <= s1) {
        *reinterpret_cast<unsigned*>(p) = *reinterpret_cast<const unsigned*>(from_lds);
      } else {
        for (int j = 0; j < 4; ++j)
          if (t + j >= s0 && t + j < s1) p[j] = from_lds[j];
      }
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RopeArgs& rope, int n_tokens, int d, bool bf16, const HeadRows* in, const HeadRows* out,
                         int n_tensors, hipStream_t stream) {
  const RotateWork w = plan_rotate(n_tokens, d, in, out, n_tensors);
  const long long blocks = (rotate_threads(w) + 255) / 256;
  if (blocks >= 1ll << 24) return hipErrorInvalidValue;      // 2^32 threads
  if (bf16) rotate_kernel<true><<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(rope, w);
  else rotate_kernel<false><<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(rope, w);
  return hipGetLastError();
}

hipError_t launch_append(const PagedCacheArgs& cache, const PagedBatch& batch, bool bf16, const HeadRows& k,
                         const HeadRows& v, const RopeArgs& rope, const HeadRows& q_in, const HeadRows& q_out,
                         hipStream_t stream) {
  AppendArgs a = {};
  a.cache = cache;
  a.batch = batch;
  a.k = k;
  a.v = v;
  a.rope = rope;
  const int bound = batch.max_new < batch.len_bound ? batch.max_new : batch.len_bound;
  a.tasks = (bound + cache.page - 2) / cache.page + 1;       // the new tokens can begin in a page's last slot
  const int threads = cache.page * cache.d / 16 / kItems < 64 ? 64 : cache.page * cache.d / 16 / kItems;
  const long long pages = 2ll * batch.batch * cache.heads * a.tasks;
  long long q_blocks = 0;
  if (q_in.heads > 0) {
    a.q = plan_rotate(batch.n_tokens, cache.d, &q_in, &q_out, 1);
    q_blocks = (rotate_threads(a.q) + threads - 1) / threads;
  }
  if ((pages + q_blocks) * threads >= 1ll << 32) return hipErrorInvalidValue;
  a.page_blocks = (unsigned)pages;
  const dim3 grid((unsigned)(pages + q_blocks)), block((unsigned)threads);
  const size_t lds = (size_t)cache.d * (cache.page + 4);
  const auto kernel = bf16 ? append_kernel<true> : append_kernel<false>;
  static std::atomic<size_t> raised[2][kPagedDevices];
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(kernel), lds, raised[bf16]);
  if (e != hipSuccess) return e;
  kernel<<<grid, block, lds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace cq

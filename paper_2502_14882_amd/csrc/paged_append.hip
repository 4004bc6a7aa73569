// Rotary positions with several axes, and growth of the paged e4m3 cache.
//
// Rotation.  Pair (a, b) of channels of a head, angle t = position on the pair's axis * frequency:
//     a' = a cos t - b sin t,   b' = b cos t + a sin t;
// its gradient is the rotation by -t.  The angle is formed in fp64 (the product of an int32 and an fp32 is exact there),
// brought to a fraction of a turn with 1 / (2 pi) in two parts, and cos and sin are Taylor sums on [-pi/4, pi/4] to 2e-16,
// rounded to fp32: positions of millions of tokens keep all of fp32's bits, and no table has to be read.  About 35
// fp64 instructions for a pair, shared by the heads that a thread turns.
// Bound: HBM, every element is read and written once.  32 + 8 heads of 128 channels, 16384 tokens on three axes: 331 MB in 66 us, 5.0
// TB/s (a plain copy 5.5); 56 heads with 64 of 128 channels turned, 3003 tokens: 86 MB in 17 us.
//
// Append.  For page and head: e = exponent of the largest new magnitude, scale 2^e, codes = e4m3(x / scale).
// A workgroup takes one page of one or some heads of the keys or of the values, so it alone decides their scales; its new elements stay
// in registers between the maximum and the codes.  The values lie channel by channel in a page (attention then
// reads a channel's tokens as one operand), so they turn in LDS on the way.
// Bound: HBM for many tokens - with the queries 364 MB for 16384 tokens (32 + 8 heads of 128 channels) in 91 us, 4.0 TB/s; of it the
// keys and values 42 us for 96 MB, since a block loads, waits for the largest, and stores, and the angles' fp64 work lies in between (27 us
// without rotation).  Non-temporal loads or stores change nothing or cost 6 %; a head per block, without shared angles, takes 105 us.
// A token for each of 64 sequences: 6 us of the kernel, the trips to the sequence and its page; the call, 9 us, is the host's.
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

typedef float v4f_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ inline void unit_angles(const RopeArgs& rope, int n_tokens, int token, int u, CosSin* cs) {
  const unsigned long long axes = *reinterpret_cast<const unsigned long long*>(rope.axis_of + 8 * u);
  const v4f_any* freq = reinterpret_cast<const v4f_any*>(rope.inv_freq + 8 * u);
  const v4f f0 = freq[0], f1 = freq[1];
  // the token's place on every axis
  const int32_t* at = rope.positions + token;
  const int p0 = at[0], p1 = rope.n_axes > 1 ? at[n_tokens] : 0;
  const int p2 = rope.n_axes > 2 ? at[2 * (size_t)n_tokens] : 0, p3 = rope.n_axes > 3 ? at[3 * (size_t)n_tokens] : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int axis = (int)(axes >> (8 * i)) & 3;
    const int pos = axis & 2 ? (axis & 1 ? p3 : p2) : (axis & 1 ? p1 : p0);
    cos_sin((double)pos * (double)(i < 4 ? f0[i & 3] : f1[i & 3]), &cs->c[i], &cs->s[i]);
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

__device__ inline const uint16_t* row_of(const HeadRows& t, long long token, int head) {
  return static_cast<const uint16_t*>(t.data) + token * t.token_stride + head * t.head_stride;
}
__device__ inline v4u load8(const uint16_t* p) { return *reinterpret_cast<const v4u*>(p); }

// Thread -> (token, group of heads, unit), units fastest.  The heads of two tensors are counted through.
struct RotateWork {
  HeadRows in[2], out[2];
  const int32_t *from, *to;     // NULL, or where the device keeps the first token and the end of those that are turned
  int n_tokens, units, heads_per_thread, groups;
};

template <bool BF16>
__device__ inline void rotate_thread(const RopeArgs& rope, const RotateWork& w, long long i) {
  const int u = (int)(i % w.units);
  const long long rest = i / w.units;
  const int group = (int)(rest % w.groups);
  const long long token = rest / w.groups;
  if (token >= w.n_tokens || (w.from && (token < *w.from || token >= *w.to))) return;
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
    const uint16_t* from = row_of(w.in[t], token, head);
    const v4u lo = load8(from + c0), hi = load8(from + c1);
    widen8<BF16>(lo, x);
    widen8<BF16>(hi, x + 8);
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
constexpr int kMostThreads = 1024;
constexpr float kMinScale = 0x1p-100f;

// The smallest power of two s >= 2^-100 with m <= 448 s: 448 = 1.75 * 2^8, so the exponent rises where the
// significand of m is above 1.75.
__device__ inline float scale_for(float m) {
  const unsigned bits = __builtin_bit_cast(unsigned, m) + 0x1fffffu;
  const int e = (int)(bits >> 23) - 127 - 8;
  return e < -100 ? kMinScale : __builtin_bit_cast(float, (unsigned)(e + 127) << 23);
}

struct AppendArgs {
  RopeArgs rope;
  PagedCacheArgs cache;
  PagedBatch batch;
  HeadRows k, v;
  RotateWork q;
  int one_each;            // every sequence's new token lies in one page
  int heads_per_block, groups;
  unsigned page_blocks;    // workgroups for pages; those behind turn queries
};

__device__ inline float magnitude(float x) { return __builtin_isfinite(x) ? fabsf(x) : 0.f; }
// x / scale for codes: NaN for what is not finite
__device__ inline float coded(float x, float inv) { return __builtin_isfinite(x) ? x * inv : __builtin_nanf(""); }

// The largest of a wave's magnitudes into `most` (bits of floats >= 0 compare as they do); `spread`: lanes hold values of different heads.
__device__ inline void fold_most(unsigned* most, float x, bool spread) {
  if (spread) {
    atomicMax(most, __builtin_bit_cast(unsigned, x));
    return;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  if ((threadIdx.x & 63) == 0) atomicMax(most, __builtin_bit_cast(unsigned, x));
}

// One page of a sequence, heads_per_block heads of the keys or of the values.
//   keys:   thread -> (token, 16 channels that hold whole pairs), a slot per head: the angles serve all of them
// kSlots: pieces of 16 elements of the keys that a thread holds, half as many of 32 of the values.  Two leave six waves to a SIMD, with
// which queries are turned in the same launch in the time of a kernel of their own; four, for pages of over 32768 elements, four
// (and took 2 % longer where both can be had).
//   values: thread -> (head, 4 tokens, 8 channels): a channel's four codes are one word, which turn in LDS
template <int kSlots, bool BF16>
__global__ void __launch_bounds__(kMostThreads) append_kernel(AppendArgs a) {
  extern __shared__ __align__(16) uint8_t s_turn[];          // values: [heads][d][page + 4]
  __shared__ unsigned s_most[kSlots];
  const int tid = threadIdx.x, threads = blockDim.x;
  unsigned id = blockIdx.x;
  if (id >= a.page_blocks) {
    rotate_thread<BF16>(a.rope, a.q, (long long)(id - a.page_blocks) * threads + tid);
    return;
  }
  const PagedCacheArgs& C = a.cache;
  const bool value = id & 1;
  id >>= 1;
  const int h0 = (int)(id % (unsigned)a.groups) * a.heads_per_block;
  const int heads = C.heads - h0 < a.heads_per_block ? C.heads - h0 : a.heads_per_block;
  id /= (unsigned)a.groups;
  // the sequence's places [from, to) that have a new row, and the pages that they lie in
  auto pages_of = [&](const Sequence& s) {
    const int from = s.pos0 > 0 ? s.pos0 : 0, to = s.pos0 + s.n;
    return to <= from ? 0 : ((to - 1) >> C.page_log2) - (from >> C.page_log2) + 1;
  };
  const Item item = a.one_each ? item_of(a.batch, (int)id, 0) : a.batch.batch == 1 ? item_of(a.batch, 0, (int)id) : locate(a.batch, (int)id, pages_of);
  if (item.b < 0) return;
  const int b = item.b;
  const Sequence s = item.s;
  if (item.local >= pages_of(s)) return;
  const int from = s.pos0 > 0 ? s.pos0 : 0, to = s.pos0 + s.n;
  const int index = (from >> C.page_log2) + item.local, place = index << C.page_log2;
  const int pid = a.batch.page_table[(size_t)b * a.batch.max_pages + index];      // place < to <= len: within the row
  const bool there = (unsigned)pid < (unsigned)C.n_pages;      // looked at when the new rows are on their way
  const int s0 = from > place ? from - place : 0, s1 = to - place < C.page ? to - place : C.page;
  const int live = s1 - s0;
  const int row0 = s.first + place - s.pos0;                 // row of the page's slot 0
  const size_t head0 = (size_t)(unsigned)pid * C.heads + h0;
  float* const scales = (value ? C.v_scale : C.k_scale) + head0;
  uint8_t* const codes = (value ? C.v_codes : C.k_codes) + (head0 << C.page_log2) * C.d;
  const int head_bytes = C.d << C.page_log2;
  if (tid < kSlots) s_most[tid] = 0;
  __syncthreads();

  // Scale of a head: every thread forms it from s_most; the old codes are brought to it before anybody writes new ones.
  auto grown = [&](int i, float old) {
    const float now = scale_for(__builtin_bit_cast(float, s_most[i]));
    return s0 > 0 && old >= now ? old : now;
  };
  auto settle = [&]() {
    if (s0 > 0) {
      for (int i = 0; i < heads; ++i) {
        const float old = scales[i], now = grown(i, old);
        if (old >= now) continue;
        const float ratio = old / now;
        v4u* const held = reinterpret_cast<v4u*>(codes + (size_t)i * head_bytes);
        for (int j = tid; j < head_bytes / 16; j += threads) {
          v4u w = held[j];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[e], true);
            w[e] = code4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
          }
          held[j] = w;
        }
      }
    }
  };

  if (!value) {
    const int units = C.d / 16, items = live * units;
    const int rounds = kSlots / a.heads_per_block;           // (token, unit) items of a thread
    float x[kSlots][16];
    v4u raw[kSlots][2];
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int round = i % rounds, hh = i / rounds, item = tid + round * threads;
      if (hh < heads && item < items) {
        int c0, c1;
        unit_channels(a.rope, item % units, &c0, &c1);
        const uint16_t* p = row_of(a.k, row0 + s0 + item / units, h0 + hh);
        raw[i][0] = load8(p + c0);
        raw[i][1] = load8(p + c1);
      }
    }
    if (!there) return;
    CosSin cs;
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      // (slots of a round follow each other in the order of the heads: rounds are 1, 2 or 4 and so are the heads)
      const int round = i % rounds, hh = i / rounds, item = tid + round * threads;
      float most = 0.f;
      if (hh < heads && item < items) {
        const int u = item % units;
        widen8<BF16>(raw[i][0], x[i]);
        widen8<BF16>(raw[i][1], x[i] + 8);
        if (unit_turns(a.rope, u)) {
          if (rounds > 1 || i == 0) unit_angles(a.rope, a.batch.n_tokens, row0 + s0 + item / units, u, &cs);
          turn_unit(a.rope, cs, x[i]);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) most = fmaxf(most, magnitude(x[i][j]));
      }
      if (hh < heads) fold_most(&s_most[hh], most, false);
    }
    __syncthreads();
    float scale[kSlots];
#pragma unroll
    for (int i = 0; i < kSlots; ++i) scale[i] = i / rounds < heads ? grown(i / rounds, s0 > 0 ? scales[i / rounds] : 0.f) : 1.f;
    settle();
    __syncthreads();                                         // everybody has read the scales, and the old codes are in place
#pragma unroll
    for (int i = 0; i < kSlots; ++i) {
      const int round = i % rounds, hh = i / rounds, item = tid + round * threads;
      if (hh >= heads) continue;
      if (tid == 0 && round == 0) scales[hh] = scale[i];
      if (item >= items) continue;
      const float inv = inverse_of_power(scale[i]);
      int c0, c1;
      unit_channels(a.rope, item % units, &c0, &c1);
      uint8_t* p = codes + (size_t)hh * head_bytes + (size_t)(s0 + item / units) * C.d;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float* y = x[i] + 8 * j;
        *reinterpret_cast<v2u*>(p + (j ? c1 : c0)) =
            (v2u){code4(coded(y[0], inv), coded(y[1], inv), coded(y[2], inv), coded(y[3], inv)),
                  code4(coded(y[4], inv), coded(y[5], inv), coded(y[6], inv), coded(y[7], inv))};
      }
    }
    return;
  }

  const int octets = C.d / 8, quad0 = s0 >> 2, quads = ((s1 + 3) >> 2) - quad0, per_head = quads * octets, items = heads * per_head;
  const bool spread = (per_head & 63) != 0;
  v4u raw[kSlots / 2][4];
#pragma unroll
  for (int i = 0; i < kSlots / 2; ++i) {
    const int item = tid + i * threads, hh = item / per_head, rest = item - hh * per_head;
    const int slot = 4 * (quad0 + rest / octets), c = 8 * (rest % octets);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool live_row = item < items && slot + t >= s0 && slot + t < s1;
      raw[i][t] = live_row ? load8(row_of(a.v, row0 + slot + t, h0 + hh) + c) : (v4u){0, 0, 0, 0};
    }
  }
  if (!there) return;
  float x[kSlots / 2][4][8];
#pragma unroll
  for (int i = 0; i < kSlots / 2; ++i) {
    const int item = tid + i * threads, hh = item / per_head;
    if (item < items) {
      float most = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        widen8<BF16>(raw[i][t], x[i][t]);
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, magnitude(x[i][t][j]));
      }
      fold_most(&s_most[hh], most, spread);
    }
  }
  __syncthreads();
  float scale[kSlots / 2];
#pragma unroll
  for (int i = 0; i < kSlots / 2; ++i) {
    const int item = tid + i * threads, hh = item < items ? item / per_head : 0;
    scale[i] = grown(hh, s0 > 0 ? scales[hh] : 0.f);
  }
  const float first_scale = tid < heads ? grown(tid, s0 > 0 ? scales[tid] : 0.f) : 0.f;
  settle();
  __syncthreads();
  if (tid < heads) scales[tid] = first_scale;
  const int stride = C.page + 4;
#pragma unroll
  for (int i = 0; i < kSlots / 2; ++i) {
    const int item = tid + i * threads, hh = item / per_head, rest = item - hh * per_head;
    if (item >= items) continue;
    const int slot = 4 * (quad0 + rest / octets), c = 8 * (rest % octets);
    const float inv = inverse_of_power(scale[i]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const unsigned w = code4(coded(x[i][0][j], inv), coded(x[i][1][j], inv), coded(x[i][2][j], inv), coded(x[i][3][j], inv));
      if (live < 4) {
        uint8_t* p = codes + (size_t)hh * head_bytes + ((size_t)(c + j) << C.page_log2) + slot;
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (slot + t >= s0 && slot + t < s1) p[t] = (uint8_t)(w >> (8 * t));
      } else {
        *reinterpret_cast<unsigned*>(s_turn + (size_t)(hh * C.d + c + j) * stride + slot) = w;
      }
    }
  }
  if (live < 4) return;
  __syncthreads();
  if (live == C.page) {
    const int words = C.page / 16;
    for (int i = tid; i < heads * C.d * words; i += threads) {
      const int c = i / words, t = 16 * (i % words);         // channel of the heads one after the other
      const unsigned* from_lds = reinterpret_cast<const unsigned*>(s_turn + (size_t)c * stride + t);
      *reinterpret_cast<v4u*>(codes + ((size_t)c << C.page_log2) + t) = (v4u){from_lds[0], from_lds[1], from_lds[2], from_lds[3]};
    }
    return;
  }
  for (int i = tid; i < heads * C.d * quads; i += threads) {
    const int c = i / quads, t = 4 * (quad0 + i % quads);
    const uint8_t* from_lds = s_turn + (size_t)c * stride + t;
    uint8_t* p = codes + ((size_t)c << C.page_log2) + t;
    if (t >= s0 && t + 4 <= s1) {
      *reinterpret_cast<unsigned*>(p) = *reinterpret_cast<const unsigned*>(from_lds);
    } else {
      for (int j = 0; j < 4; ++j)
        if (t + j >= s0 && t + j < s1) p[j] = from_lds[j];
    }
  }
}

}  // namespace

hipError_t launch_rotate(const RopeArgs& rope, int n_tokens, int d, bool bf16, const HeadRows* in, const HeadRows* out,
                         int n_tensors, hipStream_t stream) {
  const RotateWork w = plan_rotate(n_tokens, d, in, out, n_tensors);
  const long long blocks = (rotate_threads(w) + 255) / 256;
  if (blocks >= 1ll << 24) return hipErrorInvalidConfiguration;      // 2^32 threads
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
  a.one_each = bound == 1;
  // pages that a sequence's new tokens can reach (they can begin in a page's last slot), and those that all tokens can
  const long long each = (bound + cache.page - 2) / cache.page + 1, most = each * batch.batch;
  const long long by_tokens = (long long)batch.n_tokens / cache.page + 2ll * batch.batch;
  const long long pages = 2 * (by_tokens < most ? by_tokens : most);     // keys and values
  const int tokens = bound < cache.page ? bound : cache.page, units = tokens * (cache.d / 16);
  // Heads to a block: their keys share the angles, but blocks are fewer.  As many as the slots allow, while four blocks are
  // left to a CU.
  const int slots = units <= 2 * kMostThreads ? 2 : 4;
  int heads = units <= kMostThreads ? slots : 1;
  while (heads > 1 && (heads > cache.heads || pages * ceil_div(cache.heads, heads) < 4 * device_cu_count())) heads /= 2;
  a.heads_per_block = heads;
  a.groups = ceil_div(cache.heads, heads);
  const int rounds = slots / heads;                          // a thread's (token, unit) items of the keys
  int threads = ceil_div(units, rounds);
  // the values' (head, 4 tokens, 8 channels): a quad more than the tokens fill can be touched
  const int quads = (tokens + 3) / 4 + (tokens < cache.page ? 1 : 0);
  const int value_threads = ceil_div(heads * (quads < cache.page / 4 ? quads : cache.page / 4) * (cache.d / 8), slots / 2);
  if (threads < value_threads) threads = value_threads;
  threads = ceil_div(threads, 64) * 64;
  const long long page_blocks = pages * a.groups;
  long long q_blocks = 0;
  if (q_in.heads > 0) {
    a.q = plan_rotate(batch.n_tokens, cache.d, &q_in, &q_out, 1);
    a.q.from = batch.q_start;
    a.q.to = batch.q_start + batch.batch;
    q_blocks = (rotate_threads(a.q) + threads - 1) / threads;
  }
  if ((page_blocks + q_blocks) * threads >= 1ll << 32) return hipErrorInvalidConfiguration;
  a.page_blocks = (unsigned)page_blocks;
  const dim3 grid((unsigned)(page_blocks + q_blocks)), block((unsigned)threads);
  const size_t lds = bound < 4 ? 0 : (size_t)heads * cache.d * (cache.page + 4);
  const auto kernel = slots == 2 ? (bf16 ? append_kernel<2, true> : append_kernel<2, false>)
                                 : (bf16 ? append_kernel<4, true> : append_kernel<4, false>);
  static std::atomic<size_t> raised[4][kPagedDevices];
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(kernel), lds, raised[(slots == 2 ? 2 : 0) + bf16]);
  if (e != hipSuccess) return e;
  kernel<<<grid, block, lds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace cq

// Device helpers shared by the kernels of the paged 8-bit cache (paged_append.hip, paged_few.hip, paged_prompt.hip): the
// sequences of a step, 16-bit rows, e4m3 codes.  Internal to libcq.
#ifndef CQ_PAGED_DEVICE_H_
#define CQ_PAGED_DEVICE_H_

#include "decode_device.h"
#include "paged_internal.h"

namespace cq {
namespace {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef unsigned int v4u __attribute__((ext_vector_type(4)));

// One sequence of the step as the device sees it, brought into range.
struct Sequence {
  int first;   // its first row
  int n;       // rows that are served
  int pos0;    // place of its first row in the sequence (below 0: rows of no token)
  int len;     // tokens in the cache
};
__device__ inline int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ inline Sequence sequence_of(const PagedBatch& s, int from, int to, int len) {
  Sequence q;
  q.first = clamp_int(from, 0, s.n_tokens);
  const int rows = clamp_int(to, q.first, s.n_tokens) - q.first;
  q.n = rows < s.max_new ? rows : s.max_new;
  q.len = clamp_int(len, 0, s.len_bound);
  q.pos0 = q.len - rows;
  return q;
}
// b is the same for all lanes, and the result is known to be to the compiler: branches on it are scalar
__device__ inline Sequence load_sequence(const PagedBatch& s, int b) {
  return sequence_of(s, __builtin_amdgcn_readfirstlane(s.q_start[b]), __builtin_amdgcn_readfirstlane(s.q_start[b + 1]),
                     __builtin_amdgcn_readfirstlane(s.seq_lens[b]));
}

// Work items counted through the sequences, count(sequence) of each: whose the item `index` is, which of its items, and that sequence;
// sequence -1: there are not as many.  A launch then needs workgroups for the items that the tokens can make, not for the most of every sequence.
struct Item {
  int b, local;
  Sequence s;
};
__device__ inline Item item_of(const PagedBatch& s, int b, int local) { return {b, local, load_sequence(s, b)}; }
template <class F>
__device__ inline Item locate(const PagedBatch& s, int index, F count) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < s.batch; base += 64) {
    const int b = base + lane;
    Sequence seq = {0, 0, 0, 0};
    if (b < s.batch) seq = sequence_of(s, s.q_start[b], s.q_start[b + 1], s.seq_lens[b]);
    const int own = b < s.batch ? count(seq) : 0;
    int sum = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o);
      if (lane >= o) sum += x;
    }
    const int all = __builtin_amdgcn_readlane(sum, 63);
    if (index < all) {
      const int at = __builtin_ctzll(__ballot(sum > index));
      return {base + at, index - __builtin_amdgcn_readlane(sum - own, at),
              {__builtin_amdgcn_readlane(seq.first, at), __builtin_amdgcn_readlane(seq.n, at), __builtin_amdgcn_readlane(seq.pos0, at),
               __builtin_amdgcn_readlane(seq.len, at)}};
    }
    index -= all;
  }
  return {-1, 0, {0, 0, 0, 0}};
}

// ---- 16-bit elements, eight of them as they lie in memory
template <bool BF16>
__device__ inline float widen(unsigned lo16) {
  if constexpr (BF16) return __builtin_bit_cast(float, lo16 << 16);
  else return (float)__builtin_bit_cast(_Float16, (unsigned short)lo16);
}
template <bool BF16>
__device__ inline void widen8(v4u w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
    } else {
      const unsigned u = w[i];       // (the builtin would read element 0 of the vector for any other)
      const v2h h = __builtin_bit_cast(v2h, u);
      x[2 * i] = (float)h[0];
      x[2 * i + 1] = (float)h[1];
    }
  }
}
// round to nearest even (the compiler's conversion; NaN stays NaN)
template <bool BF16>
__device__ inline unsigned narrow(float x) {
  if constexpr (BF16) return __builtin_bit_cast(unsigned short, (__bf16)x);
  else return __builtin_bit_cast(unsigned short, (_Float16)x);
}
template <bool BF16>
__device__ inline v4u narrow8(const float* x) {
  v4u w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = narrow<BF16>(x[2 * i]) | narrow<BF16>(x[2 * i + 1]) << 16;
  return w;
}

// ---- e4m3 codes
// Four codes, nearest even; |x| <= 448 or NaN.
__device__ inline unsigned code4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
// Eight codes (two words) as fp16 times the power of two `scale`: exact for codes times 2^-15 to 2^7.
__device__ inline v8h codes_to_half(unsigned lo, unsigned hi, float scale) {
  const v2h a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, false);
  const v2h b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, scale, true);
  const v2h c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, false);
  const v2h d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, scale, true);
  return __builtin_shufflevector(__builtin_shufflevector(a, b, 0, 1, 2, 3), __builtin_shufflevector(c, d, 0, 1, 2, 3),
                                 0, 1, 2, 3, 4, 5, 6, 7);
}
// The top bit of every byte that holds a NaN code (0x7f or 0xff); no carry leaves a byte.
__device__ inline unsigned nan_codes(unsigned w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// The power of two that brings the largest magnitude of a row of queries into [2^14, 2^15): fp16 then holds all that is not 2^-28
// of it.  1 for rows of zeros.
__device__ inline float row_unit(float most) {
  const int e = most > 0x1p-100f ? (int)(__builtin_bit_cast(unsigned, most) >> 23) - 127 - 14 : 0;
  return __builtin_bit_cast(float, (unsigned)(127 - e) << 23);
}

// 1 / x of a power of two between 2^-126 and 2^126
__device__ inline float inverse_of_power(float x) { return __builtin_bit_cast(float, 0x7f000000u - __builtin_bit_cast(unsigned, x)); }

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kNoMax = -3.0e38f;   // running maximum before the first token: finite, below every logit
constexpr float kLn2 = 0.6931471805599453f;

}  // namespace
}  // namespace cq

#endif  // CQ_PAGED_DEVICE_H_

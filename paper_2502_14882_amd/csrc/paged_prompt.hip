// Attention over the paged e4m3 cache for many query rows per KV head: prompts, and pieces of them.
//
// Rows: the (new token, query head) pairs of one KV head, 32 to a wave as columns of its products.  For 64 tokens at a time:
//     S^T = K Q^T      A = keys (token rows), B = queries                    v_mfma_f32_32x32x16_f16
//     p = exp2(s - m)  with the row's running reference m and sum l
//     O^T += V^T P^T   A = values (channel rows), B = weights
// Bound: the matrix cores, 4 d flops for each pair of a row and a token - or rather the chip's power: with zeros for inputs the
// same instructions take a fifth less time (a plain matrix product of 8192 x 8192 x 8192 a quarter less).  What keeps the cores fed:
//   - the codes are turned into fp16 once per workgroup, on their way into LDS (exactly: a code has four significant bits), and
//     lie there operand by operand (1 KB, lane by lane), so that an operand is one linear 16-byte read per lane;
//   - which token is which row of S^T is chosen such that the weights a lane has computed are its operand of the second product:
//     token 16 u + 8 f + 4 j + b of 32 is row 16 u + 8 j + 4 f + b, f being the half of the wave;
//   - products, softmax and the codes' way into LDS are interleaved within a wave (half_step): a wave whose next product waits
//     for the cores also keeps the other wave's vector instructions waiting (one wave with 16 products and one with 64 adds
//     take the sum of their times), while vector instructions between two products of a wave cost next to nothing - except
//     v_dot2, which runs on the cores, so the weights are summed by additions;
//   - m follows a row's largest logit only when that is more than 2^8 above it (weights up to 256 fit fp16 as well as those
//     up to 1), so that O is rescaled a few times per row and not at every step.
// 8192 rows of 32 heads over 8192 tokens, each up to its own, 128 channels: 580 to 600 us, 0.94 PFLOP/s, where a matrix product
// reaches 1.26 on such data; 512 new tokens of each of three sequences of 16384 tokens 440 us, 0.85 PFLOP/s, 19 of them the splits' joining.
// Two row tiles per wave and one wave to a SIMD read half as much from LDS, but took 850 us where this takes 589 (8192 rows of 32 heads
// over 8192 tokens, 128 channels): the accumulators then travel between the two register files.
#include <type_traits>
#include <utility>

#include "paged_device.h"

namespace cq {
namespace {

// f(std::integral_constant<int, 0>{}) .. of N: loops whose index the body needs at compile time
template <class F, int... I>
__device__ inline void static_for_each(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ inline void static_for(F&& f) {
  static_for_each(f, std::make_integer_sequence<int, N>{});
}

template <int D>
struct Prompt {
  // two to a SIMD while 256 registers hold what one needs (192 channels 350 us, 365 with four waves; 256 channels 805 us, 452 with four; for few
  // blocks four would be a little faster, 3 x 1060 rows 24 us and 27, 2 x 1043 x 4 rows 41 and 44, but 8192 tokens take 617 and 573)
  static constexpr int kWaves = D <= 192 ? 8 : 4;
  static constexpr int kThreads = 64 * kWaves, kRows = 32 * kWaves;
  static constexpr int kOps = D / 16;                                 // operands of 32 keys, and of 32 tokens' values
  static constexpr int kValueTiles = D / 32;
  static constexpr int kPieces = (4 * D + kThreads - 1) / kThreads;   // of 16 codes, per thread, for keys as for values
  static constexpr bool kEven = 4 * D % kThreads == 0;
  // bytes of an operand in LDS: padded such that the writes of eight neighbouring lanes fall into eight different banks' groups
  static constexpr int kKeyStride = 1024 + 16, kValueStride = 1024 + 32;
  static constexpr int kKeyBytes = 2 * kOps * kKeyStride, kValueBytes = 2 * kOps * kValueStride;
  static constexpr int kOutStride = D + 8;                            // fp16 elements between the rows of the result in LDS
  static constexpr int kOutBytes = kRows * kOutStride * 2;
  static constexpr int kTileBytes = 2 * (kKeyBytes + kValueBytes);
  static constexpr int kLds = kTileBytes > kOutBytes ? kTileBytes : kOutBytes;
};

// Of the four groups of 16 tokens of a step, lane l holds group l % 4.
struct Groups {
  int pid;            // page, -1: not there
  float ks, vs;       // scales; keys: 1, values: 0 where the group is not there
};

template <int D, bool BF16>
__global__ void __launch_bounds__(Prompt<D>::kThreads) prompt_kernel(PagedAttention a) {
  using T = Prompt<D>;
  extern __shared__ __align__(16) uint8_t s_tiles[];                  // [2][keys], [2][values]
  __shared__ unsigned s_nan[3][2];
  uint8_t* const s_keys = s_tiles;
  uint8_t* const s_values = s_tiles + 2 * T::kKeyBytes;
  const PagedCacheArgs& C = a.cache;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 31, half = lane >> 5;

  // KV heads fastest: with eight of them a head's workgroups share an XCD and its L2; of the rows the last first, whose tokens are
  // the most where rows see up to their own; splits slowest: workgroups go to an XCD's shader engines in turn, and neighbours have like
  // work then (2048 tokens in two splits beside each other 103 us)
  unsigned id = blockIdx.x;
  const int h = (int)(id % (unsigned)C.heads);
  id /= (unsigned)C.heads;
  const int split = (int)(id / (unsigned)a.plan.prompt_blocks);
  id %= (unsigned)a.plan.prompt_blocks;
  auto blocks_of = [&](const Sequence& s) {
    const int rows = s.n * a.g;
    return a.plan.few && rows <= kFewRows ? 0 : ceil_div(rows, T::kRows);
  };
  const Item item = a.batch.batch == 1 ? item_of(a.batch, 0, (int)id) : locate(a.batch, (int)id, blocks_of);
  if (item.b < 0) return;
  const int b = item.b;
  const Sequence s = item.s;
  const int rows = s.n * a.g, rb = blocks_of(s) - 1 - item.local, block0 = rb * T::kRows;
  if (rb < 0) return;
  const int parts = ceil_div(ceil_div(s.len, kStep), a.plan.prompt_split_steps);
  if (split >= (parts > 1 ? parts : 1)) return;

  auto sees = [&](int r) { return a.causal ? clamp_int(s.pos0 + r / a.g + 1, 0, s.len) : s.len; };
  const int block_last = (block0 + T::kRows < rows ? block0 + T::kRows : rows) - 1;
  const int block_lo = sees(block0), block_hi = sees(block_last);
  const int r0 = block0 + 32 * wave;                                   // this wave's rows
  const int step0 = split * a.plan.prompt_split_steps;
  int step1 = step0 + a.plan.prompt_split_steps;
  if (step1 > ceil_div(block_hi, kStep)) step1 = ceil_div(block_hi, kStep);
  const int steps = step1 - step0;
  if (steps <= 0 && split > 0) return;                                // no row sees a token of this split: nobody reads its results

  const int row = r0 + n, row_new = row / a.g;                        // this lane's row, as column of the products
  const bool row_there = row < rows;
  const long long row_token = s.first + row_new;
  const int row_head = h * a.g + row - row_new * a.g, limit = row_there ? sees(row) : 0;
  v8h q[T::kOps];
  float row_scale;
  {
    const uint16_t* p = static_cast<const uint16_t*>(a.q.data);
    if (row_there) p += row_token * a.q.token_stride + row_head * a.q.head_stride;
    v4u raw[T::kOps];
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < T::kOps; ++j) {
      raw[j] = row_there ? *reinterpret_cast<const v4u*>(p + 16 * j + 8 * half) : (v4u){0, 0, 0, 0};
      float x[8];
      widen8<BF16>(raw[j], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, __builtin_isfinite(x[e]) ? fabsf(x[e]) : 0.f);
    }
    most = fmaxf(most, __shfl_xor(most, 32));
    const float up = row_unit(most);
    row_scale = a.scale_log2 / up;
#pragma unroll
    for (int j = 0; j < T::kOps; ++j) {
      float x[8];
      widen8<BF16>(raw[j], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) q[j][e] = (_Float16)(x[e] * up);
    }
  }

  // ---- where the codes lie
  const int32_t* table = a.batch.page_table + (size_t)b * a.batch.max_pages;
  auto page_of = [&](int step) {
    const int tok = step * kStep + 16 * (lane & 3);
    const int pid = tok < s.len ? table[tok >> C.page_log2] : -1;
    return (unsigned)pid < (unsigned)C.n_pages ? pid : -1;
  };
  auto load_scales = [&](Groups* w) {
    const size_t i = (size_t)(w->pid < 0 ? 0 : w->pid) * C.heads + h;
    const float ks = C.k_scale[i], vs = C.v_scale[i];
    w->ks = w->pid < 0 ? 1.f : ks;
    w->vs = w->pid < 0 ? 0.f : vs;
  };
  // a page's codes of this head: first + pid * stride, one multiplication (the host has checked that the stride fits 32 bits)
  const unsigned page_bytes = (unsigned)(C.heads * C.page * D);
  const uint8_t* const first_keys = C.k_codes + (((size_t)h << C.page_log2)) * D;
  const uint8_t* const first_values = C.v_codes + (((size_t)h * D) << C.page_log2);
  v4u key[T::kPieces], val[T::kPieces];
  auto load_keys = [&](int step, int pid_of_lane) {
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + T::kThreads * j, tok = p / T::kOps, c = 16 * (p % T::kOps);
      const int pid = __shfl(pid_of_lane, (tok >> 4) & 3);
      if (T::kEven || p < 4 * D) {
        const unsigned offset = (unsigned)((step * kStep + tok) & (C.page - 1)) * D + c;
        key[j] = *reinterpret_cast<const v4u*>(first_keys + ((unsigned long long)(unsigned)(pid < 0 ? 0 : pid) * page_bytes + offset));
      }
    }
  };
  auto load_values = [&](int step, int pid) {
    const unsigned offset = (unsigned)(step * kStep + 16 * (lane & 3)) & (unsigned)(C.page - 1);
    const uint8_t* from = first_values + ((unsigned long long)(unsigned)(pid < 0 ? 0 : pid) * page_bytes + offset);
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + T::kThreads * j, c = p >> 2;
      if (T::kEven || p < 4 * D) val[j] = *reinterpret_cast<const v4u*>(from + ((unsigned)c << C.page_log2));
    }
  };
  auto store_keys = [&](int buffer) {
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + T::kThreads * j, tok = p / T::kOps, op = p % T::kOps;
      if (T::kEven || p < 4 * D) {
        const int t = tok & 31, m = (t & 0x13) | (t & 4) << 1 | (t & 8) >> 1;
        uint8_t* to = s_keys + buffer * T::kKeyBytes + ((tok >> 5) * T::kOps + op) * T::kKeyStride + m * 16;
        *reinterpret_cast<v8h*>(to) = codes_to_half(key[j][0], key[j][1], 1.f);
        *reinterpret_cast<v8h*>(to + 512) = codes_to_half(key[j][2], key[j][3], 1.f);
      }
    }
  };
  // values in units of `unit`; where some row does not see some of the 64 tokens, those that nobody sees or that are not
  // there are cleared, and NaN codes of the others too: their tokens are noted, whose logits become NaN
  auto store_values = [&](int buffer, int step, const Groups& w, float unit) {
    const float rel = w.vs == 0.f ? 1.f : w.vs * inverse_of_power(unit);
    const int tok = step * kStep + 16 * (lane & 3);
    const bool cut = step * kStep + kStep > block_lo || __any(w.pid < 0);
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + T::kThreads * j, c = p >> 2;
      if (T::kEven || p < 4 * D) {
        v4u x = val[j];
        if (cut) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int live = w.pid < 0 ? 0 : clamp_int(block_hi - tok - 4 * i, 0, 4);
            unsigned y = x[i] & (live == 4 ? 0xffffffffu : (1u << (8 * live)) - 1u);
            const unsigned bad = nan_codes(y) >> 7;
            x[i] = y & ~(bad * 0xffu);
            if (bad) {
              const unsigned four = (bad & 1) | (bad >> 7 & 2) | (bad >> 14 & 4) | (bad >> 21 & 8);
              atomicOr(&s_nan[step % 3][(lane & 3) >> 1], four << (16 * (lane & 1) + 4 * i));
            }
          }
        }
        uint8_t* to = s_values + buffer * T::kValueBytes + ((c >> 5) * 4 + (lane & 3)) * T::kValueStride + (c & 31) * 16;
        *reinterpret_cast<v8h*>(to) = codes_to_half(x[0], x[1], rel);
        *reinterpret_cast<v8h*>(to + 512) = codes_to_half(x[2], x[3], rel);
      }
    }
  };
  // The unit of a step's values in LDS: the one so far while all of the step's scales lie within 2^-15 to 1 of it (codes times those are
  // exact in fp16), otherwise the largest of them.
  auto unit_of = [&](float unit, const Groups& w) {
    unsigned top = 0, low = 0xffffffffu;                              // positive floats compare as their bits
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned x = (unsigned)__builtin_amdgcn_readlane(__builtin_bit_cast(int, w.vs), i);
      top = x > top ? x : top;
      low = x - 1 < low ? x - 1 : low;                                // groups that are not there, 0, come last
    }
    if (top == 0) return unit;
    const float most = __builtin_bit_cast(float, top), least = __builtin_bit_cast(float, low + 1);
    return most > unit || least < unit * 0x1p-15f ? most : unit;
  };

  v16f acc[T::kValueTiles];
  float m = kNoMax, l = 0.f, acc_unit = 1.f;
#pragma unroll
  for (int c = 0; c < T::kValueTiles; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[c][e] = 0.f;

  // The largest of each group's eight logits (raw) of a lane.
  auto largest = [&](const v16f& sc, float (&best)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      best[i] = fmaxf(sc[8 * i], sc[8 * i + 1]);
#pragma unroll
      for (int e = 2; e < 8; e += 2) best[i] = fmaxf(fmaxf(best[i], sc[8 * i + e]), sc[8 * i + e + 1]);
    }
  };
  // Half h of the sequence of halves of steps (32 tokens each).  Things that do not depend on each other are dealt out in groups of
  // two products each, so that the vector unit works under the matrix cores: a wave whose next product waits for the cores keeps the
  // other wave's vector instructions waiting too, so the overlap has to be within a wave.
  //   logits of half h + 1 (`next`) | most of the weights of half h (from `now`, to `p`), and what `beside` does
  //   products of half h - 1's weights (`before`) with its values | the other weights, the largest of `next`
  auto half_step = [&](const uint8_t* keys, const uint8_t* values, int step, int t, const Groups& w, v16f& now, float (&best)[2], v16f& next,
                       v8h (&p)[2], v8h (&before)[2], auto&& beside) {
    // operands in the order [keys: 16 channels] [values: 16 tokens][32 channels]; in LDS the four value operands of 32 channels lie together
    auto op = [&](auto J) {
      constexpr int j = decltype(J)::value, v = j - T::kOps;
      if constexpr (v < 0) return *reinterpret_cast<const v8h*>(keys + j * T::kKeyStride);
      else return *reinterpret_cast<const v8h*>(values + (v % T::kValueTiles * 4 + v / T::kValueTiles) * T::kValueStride);
    };
    constexpr int kAhead = 4;                                         // operands on their way from LDS
    v8h ring[kAhead];
    static_for<kAhead>([&](auto J) { ring[decltype(J)::value] = op(J); });
    __builtin_amdgcn_sched_barrier(0);
    if (step * kStep + kStep > block_lo || __any(w.pid < 0)) {        // where store_values looks for NaN codes
      const unsigned long long there = __ballot(w.pid >= 0) >> (2 * t);      // bit i: group i
      const unsigned nan = s_nan[step % 3][t];
#pragma unroll
      for (int i = 0; i < 2; ++i) {                                   // group of 16 tokens, eight of them this lane's
        const int first = 16 * i + 8 * half;
        const unsigned bad = nan >> first;
        const int live = there >> i & 1 ? limit - step * kStep - 32 * t - first : 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = now[8 * i + e];
          now[8 * i + e] = e < live ? (bad >> e & 1 ? __builtin_nanf("") : x) : -__builtin_inff();
        }
        __builtin_amdgcn_sched_barrier(0);                            // (all comparisons at once would not fit the scalar registers)
      }
      largest(now, best);
    }
    float f[2], top = kNoMax;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // (above 0, as tiny queries over pages of zeros would not have it: a masked logit, -infinity, stays what it is)
      f[i] = fmaxf(row_scale * __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w.ks), 2 * t + i)), 0x1p-126f);
      top = fmaxf(top, best[i] * f[i]);
    }
    if (__any(top > m + 8.f)) {
      // the weights before are relative to the old reference: their products are added first
      static_for<T::kOps>([&](auto J) {
        constexpr int j = decltype(J)::value, c = j % T::kValueTiles;
        const v8h o = op(std::integral_constant<int, T::kOps + j>{});
        acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o, before[j / T::kValueTiles], acc[c], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      });
#pragma unroll
      for (int i = 0; i < 2; ++i) before[i] = (v8h){0, 0, 0, 0, 0, 0, 0, 0};
      top = fmaxf(top, __shfl_xor(top, 32));
      const float to = fmaxf(m, top), g = exp2_fast(m - to);
      m = to;
      l *= g;
#pragma unroll
      for (int c = 0; c < T::kValueTiles; ++c) acc[c] *= g;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) next[e] = 0.f;
    __builtin_amdgcn_s_setprio(1);
    constexpr int kUnder = T::kOps > 2 ? 6 : 8;                       // pairs of weights under the logits, of 8
    static_for<2 * T::kOps>([&](auto J) {
      constexpr int j = decltype(J)::value;
      const v8h o = ring[j % kAhead];
      if constexpr (j + kAhead < 2 * T::kOps) ring[j % kAhead] = op(std::integral_constant<int, j + kAhead>{});
      if constexpr (j < T::kOps) {
        next = __builtin_amdgcn_mfma_f32_32x32x16_f16(o, q[j], next, 0, 0, 0);
      } else {
        constexpr int v = j - T::kOps, c = v % T::kValueTiles;
        acc[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(o, before[v / T::kValueTiles], acc[c], 0, 0, 0);
      }
      if constexpr (j % 2 == 1) {                                     // behind every second product
        constexpr int groups = T::kOps / 2, group = j / 2;
        constexpr int at = group % groups, base = group < groups ? 0 : kUnder, many = group < groups ? kUnder : 8 - kUnder;
        constexpr int first = base + many * at / groups, last = base + many * (at + 1) / groups;
        static_for<last - first>([&](auto P) {
          constexpr int pair = first + decltype(P)::value, i = pair / 4, e = 2 * pair;
          const float x = exp2_fast(__builtin_fmaf(now[e], f[i], -m)), y = exp2_fast(__builtin_fmaf(now[e + 1], f[i], -m));
          v2h two = {(_Float16)x, (_Float16)y};
          asm volatile("" : "+v"(two));      // here, and not where the next half uses it
          l += x + y;
          p[i][e & 7] = two[0];
          p[i][(e & 7) + 1] = two[1];
        });
        beside(group);
        if constexpr (j == 2 * T::kOps - 1) {
          largest(next, best);
          asm volatile("" : "+v"(best[0]), "+v"(best[1]));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    __builtin_amdgcn_s_setprio(0);
  };

  if (steps > 0) {
    // Step i: its halves 2 i and 2 i + 1; logits of 2 i + 1 and 2 i + 2, values of 2 i - 1 and 2 i.  Behind the barrier between the two nobody reads
    // the keys of i and the values of i - 1 any more: keys of i + 2 and values of i + 1 take their places; asked for: keys of
    // i + 3, values of i + 2.  Beyond the last step the last one's codes are loaded again, and not used.
    auto at = [&](int i) { return step0 + (i < steps ? i : steps - 1); };
    auto keys_of = [&](int i, int t) { return s_keys + (i & 1) * T::kKeyBytes + t * T::kOps * T::kKeyStride + lane * 16; };
    auto values_of = [&](int i, int t) { return s_values + (i & 1) * T::kValueBytes + 2 * t * T::kValueStride + lane * 16; };
    Groups g0, g1, g2;
    if (tid < 6) s_nan[tid >> 1][tid & 1] = 0;
    // the values "before" the first half are multiplied by 0
    for (int i = tid; i < T::kValueBytes / 16; i += T::kThreads)
      *reinterpret_cast<v4u*>(s_values + T::kValueBytes + 16 * i) = (v4u){0, 0, 0, 0};
    g0.pid = page_of(at(0));
    g1.pid = page_of(at(1));
    g2.pid = page_of(at(2));
    load_scales(&g0);
    load_scales(&g1);
    load_keys(at(0), g0.pid);
    load_values(at(0), g0.pid);
    store_keys(0);
    load_keys(at(1), g1.pid);
    __syncthreads();                                                  // s_nan
    float unit = unit_of(1.f, g0);
    store_values(0, at(0), g0, unit);
    load_values(at(1), g1.pid);
    store_keys(1);
    load_keys(at(2), g2.pid);
    int pid = page_of(at(3));
    __syncthreads();
    v16f sc0, sc1;
    float best[2];
    v8h p0[2], p1[2];
#pragma unroll
    for (int e = 0; e < 16; ++e) sc0[e] = 0.f;
#pragma unroll
    for (int j = 0; j < T::kOps; ++j)
      sc0 = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const v8h*>(keys_of(0, 0) + j * T::kKeyStride), q[j], sc0, 0, 0, 0);
    largest(sc0, best);
#pragma unroll
    for (int i = 0; i < 2; ++i) p1[i] = (v8h){0, 0, 0, 0, 0, 0, 0, 0};
    acc_unit = unit;
    for (int i = 0; i < steps; ++i) {
      if (at(i) * kStep + kStep > block_lo || __any(g0.pid < 0)) __syncthreads();        // s_nan of this step
      half_step(keys_of(i, 1), values_of(i + 1, 1), at(i), 0, g0, sc0, best, sc1, p0, p1, [](int) {});   // values_of(i - 1, 1): the same buffer
      __syncthreads();
      if (tid < 2) s_nan[(step0 + i + 2) % 3][tid] = 0;               // last read a step ago
      if (unit != acc_unit) {
        const float f = acc_unit * inverse_of_power(unit);
#pragma unroll
        for (int c = 0; c < T::kValueTiles; ++c) acc[c] *= f;
        acc_unit = unit;
      }
      if (i + 1 < steps) unit = unit_of(unit, g1);
      half_step(keys_of(i + 1, 0), values_of(i, 0), at(i), 1, g0, sc1, best, sc0, p1, p0, [&](int group) {
        // (beyond the last step the last one's codes again, which nobody reads)
        if (group == 0) {
          store_values((i + 1) & 1, at(i + 1), g1, unit);
          load_values(at(i + 2), g2.pid);
        }
        if (group == (T::kOps > 2 ? 1 : 0)) {
          store_keys(i & 1);
          load_keys(at(i + 3), pid);
          load_scales(&g2);
        }
      });
      g0 = g1;
      g1 = g2;
      g2.pid = pid;
      pid = page_of(at(i + 4));
    }
    const uint8_t* values = values_of(steps - 1, 1);
#pragma unroll
    for (int j = 0; j < T::kOps; ++j)
      acc[j % T::kValueTiles] = __builtin_amdgcn_mfma_f32_32x32x16_f16(
          *reinterpret_cast<const v8h*>(values + (j % T::kValueTiles * 4 + j / T::kValueTiles) * T::kValueStride), p1[j / T::kValueTiles],
          acc[j % T::kValueTiles], 0, 0, 0);
  }

  // ---- results
  l += __shfl_xor(l, 32);
  if (parts <= 1) {
    __syncthreads();                                                  // the tiles are no longer read
    uint16_t* const s_out = reinterpret_cast<uint16_t*>(s_tiles) + wave * 32 * T::kOutStride;
    const float inv = l == 0.f ? 0.f : acc_unit / l;
#pragma unroll
    for (int c = 0; c < T::kValueTiles; ++c)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<v2u*>(s_out + n * T::kOutStride + 32 * c + 2 * e + 4 * half) =
            (v2u){narrow<BF16>(acc[c][e] * inv) | narrow<BF16>(acc[c][e + 1] * inv) << 16,
                  narrow<BF16>(acc[c][e + 2] * inv) | narrow<BF16>(acc[c][e + 3] * inv) << 16};
    __builtin_amdgcn_wave_barrier();                                  // a wave reads what it wrote itself: in order
    for (int i = lane; i < 32 * (D / 8); i += 64) {
      const int at_row = r0 + i / (D / 8), c = 8 * (i % (D / 8));
      if (at_row < rows) {
        const int tok = at_row / a.g;
        uint16_t* to = static_cast<uint16_t*>(a.out.data) + (long long)(s.first + tok) * a.out.token_stride +
                       (long long)(h * a.g + at_row - tok * a.g) * a.out.head_stride + c;
        *reinterpret_cast<v4u*>(to) = *reinterpret_cast<const v4u*>(s_out + (i / (D / 8)) * T::kOutStride + c);
      }
    }
    if (a.lse && half == 0 && row_there)
      a.lse[row_token * a.q.heads + row_head] = l == 0.f ? -__builtin_inff() : (m + log2f(l)) * kLn2;
  } else if (row_there) {
    const size_t part = (row_token * a.q.heads + row_head) * a.plan.splits + split;
#pragma unroll
    for (int c = 0; c < T::kValueTiles; ++c)
#pragma unroll
      for (int e = 0; e < 16; e += 4)
        *reinterpret_cast<v4f*>(a.acc + part * D + 32 * c + 2 * e + 4 * half) =
            (v4f){acc[c][e], acc[c][e + 1], acc[c][e + 2], acc[c][e + 3]} * acc_unit;
    if (half == 0) *reinterpret_cast<v2f*>(a.ml + part * 2) = (v2f){m, l};
  }
}

template <int D>
hipError_t launch_prompt_d(const PagedAttention& a, bool bf16, hipStream_t stream) {
  const long long blocks = (long long)a.cache.heads * a.plan.prompt_blocks * a.plan.prompt_splits;
  const auto kernel = bf16 ? prompt_kernel<D, true> : prompt_kernel<D, false>;
  static std::atomic<size_t> raised[2][kPagedDevices];
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(kernel), Prompt<D>::kLds, raised[bf16]);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)blocks), dim3(Prompt<D>::kThreads), Prompt<D>::kLds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int prompt_rows(int d) { return d <= 192 ? Prompt<192>::kRows : Prompt<256>::kRows; }

hipError_t launch_paged_prompt(const PagedAttention& a, bool bf16, hipStream_t stream) { CQ_FOR_HEAD_DIM(launch_prompt_d); }

}  // namespace cq

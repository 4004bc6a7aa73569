// Attention over the paged e4m3 cache for many query rows per KV head: prompts, and pieces of them.
//
// Rows: the (new token, query head) pairs of one KV head, 32 to a tile of the matrix cores, kRowTiles tiles to a wave, four waves
// to a workgroup.  For 64 tokens at a time:
//     S^T = K Q^T      A = keys (token rows), B = queries                    v_mfma_f32_32x32x16_f16
//     p = exp2(s - m)  with the row's running reference m and sum l
//     O^T += V^T P^T   A = values (channel rows), B = weights
// Bound: the matrix cores, 4 d flops for each pair of a row and a token.  What keeps them fed:
//   - the codes are turned into fp16 once per workgroup, on their way into LDS (exactly: a code has four significant bits), and
//     lie there operand by operand (1 KB, lane by lane), so that an operand is one linear 16-byte read per lane; each is used for two
//     products (two row tiles) - with one the LDS would bound;
//   - which token is which row of S^T is chosen such that the weights a lane has computed are its operand of the second product:
//     token 16 u + 8 f + 4 j + b of 32 is row 16 u + 8 j + 4 f + b, f being the half of the wave;
//   - two tiles of keys, two of values and the next codes in registers are under way at once: while a wave turns the
//     logits of one step into weights, its products with the next step's keys are in the matrix cores; one barrier a step;
//   - m follows a row's largest logit only when that is more than 2^8 above it (weights up to 256 fit fp16 as well as those
//     up to 1), so that O is rescaled a few times per row and not at every step.
// The sum l is taken of the rounded weights, which takes their common error out of the result.
#include "paged_device.h"

namespace cq {
namespace {

constexpr int kPromptWaves = 4;
constexpr int kPromptThreads = 64 * kPromptWaves;

template <int D>
struct Prompt {
  static constexpr int kRowTiles = D <= 128 ? 2 : 1;                 // O takes 16 D / 32 registers for each
  static constexpr int kRows = 32 * kRowTiles * kPromptWaves;
  static constexpr int kKeyOps = D / 16;                              // operands of a tile of 32 keys
  static constexpr int kValueTiles = D / 32;
  static constexpr int kPieces = (4 * D + kPromptThreads - 1) / kPromptThreads;   // of 16 codes, per thread, for keys as for values
  static constexpr bool kEven = 4 * D % kPromptThreads == 0;
  // bytes of an operand in LDS: padded such that the writes of eight neighbouring lanes fall into eight different banks' groups
  static constexpr int kKeyStride = 1024 + 16, kValueStride = 1024 + 32;
  static constexpr int kKeyBytes = 2 * kKeyOps * kKeyStride, kValueBytes = 4 * kValueTiles * kValueStride;
  static constexpr int kOutStride = D + 8;                            // fp16 elements between the rows of the result in LDS
  static constexpr int kOutBytes = kPromptWaves * 32 * kOutStride * 2;
  static constexpr int kKeyBuffers = D == 256 ? 2 : 3;                // three of 256 channels do not fit, and take a second barrier
  static constexpr int kTileBytes = kKeyBuffers * kKeyBytes + 2 * kValueBytes;
  static constexpr int kLds = kTileBytes > kOutBytes ? kTileBytes : kOutBytes;
};

// Of the four groups of 16 tokens of a step, lane l holds group l % 4.
struct Groups {
  int pid;            // page, -1: not there
  float ks, vs;       // scales; keys: 1, values: 0 where the group is not there
};

template <int D, bool BF16>
__global__ void __launch_bounds__(kPromptThreads, 1) prompt_kernel(PagedAttention a) {
  using T = Prompt<D>;
  constexpr int R = T::kRowTiles;
  extern __shared__ __align__(16) uint8_t s_tiles[];                  // [kKeyBuffers][keys], [2][values]
  __shared__ unsigned s_nan[3][2];
  uint8_t* const s_keys = s_tiles;
  uint8_t* const s_values = s_tiles + T::kKeyBuffers * T::kKeyBytes;
  const PagedCacheArgs& C = a.cache;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, n = lane & 31, half = lane >> 5;

  // KV heads fastest: with eight of them a head's workgroups share an XCD and its L2; of the rows the last first, whose tokens are
  // the most where rows see up to their own
  unsigned id = blockIdx.x;
  const int h = (int)(id % (unsigned)C.heads);
  id /= (unsigned)C.heads;
  const int b = (int)(id % (unsigned)a.batch.batch);
  id /= (unsigned)a.batch.batch;
  const int split = (int)(id % (unsigned)a.plan.prompt_splits);
  const int rb = a.plan.prompt_blocks - 1 - (int)(id / (unsigned)a.plan.prompt_splits);
  const Sequence s = load_sequence(a.batch, b);
  const int rows = s.n * a.g, block0 = rb * T::kRows;
  if (block0 >= rows || (a.plan.few && rows <= kFewRows)) return;
  const int parts = ceil_div(ceil_div(s.len, kStep), a.plan.prompt_split_steps);
  if (split >= (parts > 1 ? parts : 1)) return;

  auto sees = [&](int r) { return a.causal ? clamp_int(s.pos0 + r / a.g + 1, 0, s.len) : s.len; };
  const int block_last = (block0 + T::kRows < rows ? block0 + T::kRows : rows) - 1;
  const int block_lo = sees(block0), block_hi = sees(block_last);
  const int r0 = block0 + 32 * R * wave;                              // this wave's rows
  const int wave_last = (r0 + 32 * R < rows ? r0 + 32 * R : rows) - 1;
  const int wave_hi = r0 < rows ? sees(wave_last) : 0;
  const int step0 = split * a.plan.prompt_split_steps;
  int step1 = step0 + a.plan.prompt_split_steps;
  if (step1 > ceil_div(block_hi, kStep)) step1 = ceil_div(block_hi, kStep);
  const int steps = step1 - step0;                                    // may be <= 0

  int limit[R];
  v8h q[R][T::kKeyOps];
  float row_scale[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = r0 + 32 * r + n, i = row / a.g;
    const bool there = row < rows;
    limit[r] = there ? sees(row) : 0;
    const uint16_t* p = static_cast<const uint16_t*>(a.q.data);
    if (there) p += (long long)(s.first + i) * a.q.token_stride + (long long)(h * a.g + row - i * a.g) * a.q.head_stride;
    v4u raw[T::kKeyOps];
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < T::kKeyOps; ++j) {
      raw[j] = there ? *reinterpret_cast<const v4u*>(p + 16 * j + 8 * half) : (v4u){0, 0, 0, 0};
      float x[8];
      widen8<BF16>(raw[j], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) most = fmaxf(most, __builtin_isfinite(x[e]) ? fabsf(x[e]) : 0.f);
    }
    most = fmaxf(most, __shfl_xor(most, 32));
    const float up = row_unit(most);                                  // a power of two: the largest element into [2^14, 2^15)
    row_scale[r] = a.scale_log2 / up;
#pragma unroll
    for (int j = 0; j < T::kKeyOps; ++j) {
      float x[8];
      widen8<BF16>(raw[j], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) q[r][j][e] = (_Float16)(x[e] * up);
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
  v4u key[T::kPieces], val[T::kPieces];
  auto load_keys = [&](int step, int pid_of_lane) {
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + kPromptThreads * j, tok = p / T::kKeyOps, c = 16 * (p % T::kKeyOps);
      const int pid = __shfl(pid_of_lane, (tok >> 4) & 3);
      if (T::kEven || p < 4 * D) {
        const int offset = (step * kStep + tok) & (C.page - 1);
        key[j] = *reinterpret_cast<const v4u*>(C.k_codes + ((((size_t)(pid < 0 ? 0 : pid) * C.heads + h) << C.page_log2) + offset) * D + c);
      }
    }
  };
  auto load_values = [&](int step, int pid) {
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + kPromptThreads * j, c = p >> 2;
      if (T::kEven || p < 4 * D) {
        const int offset = (step * kStep + 16 * (lane & 3)) & (C.page - 1);
        val[j] = *reinterpret_cast<const v4u*>(C.v_codes + ((((size_t)(pid < 0 ? 0 : pid) * C.heads + h) * D + c) << C.page_log2) + offset);
      }
    }
  };
  auto store_keys = [&](int buffer) {
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + kPromptThreads * j, tok = p / T::kKeyOps, op = p % T::kKeyOps;
      if (T::kEven || p < 4 * D) {
        const int t = tok & 31, m = (t & 0x13) | (t & 4) << 1 | (t & 8) >> 1;
        uint8_t* to = s_keys + buffer * T::kKeyBytes + ((tok >> 5) * T::kKeyOps + op) * T::kKeyStride + m * 16;
        *reinterpret_cast<v8h*>(to) = codes_to_half(key[j][0], key[j][1], 1.f);
        *reinterpret_cast<v8h*>(to + 512) = codes_to_half(key[j][2], key[j][3], 1.f);
      }
    }
  };
  // values in units of `unit`; where some row does not see some of the 64 tokens, those that nobody sees or that are not
  // there are cleared, and NaN codes of the others too: their tokens are noted, whose logits become NaN
  auto store_values = [&](int buffer, int step, const Groups& w, float unit) {
    const float rel = w.vs == 0.f ? 1.f : w.vs / unit;
    const int tok = step * kStep + 16 * (lane & 3);
    const bool cut = step * kStep + kStep > block_lo || __any(w.pid < 0);
#pragma unroll
    for (int j = 0; j < T::kPieces; ++j) {
      const int p = tid + kPromptThreads * j, c = p >> 2;
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
    float top = fmaxf(w.vs, __shfl_xor(w.vs, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    float low = w.vs == 0.f ? top : w.vs;
    low = fminf(low, __shfl_xor(low, 1));
    low = fminf(low, __shfl_xor(low, 2));
    const float next = top > unit || low < unit * 0x1p-15f ? top : unit;
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, top == 0.f ? unit : next)));
  };

  v16f acc[R][T::kValueTiles];
  float m[R], l[R], acc_unit = 1.f;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = kNoMax;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < T::kValueTiles; ++c)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[r][c][e] = 0.f;
  }

  // The 32 tokens 32 t .. of a step: logits, weights, products with the values.
  auto logits = [&](int buffer, int t, v16f (&sc)[R]) {
    const uint8_t* from = s_keys + buffer * T::kKeyBytes + t * T::kKeyOps * T::kKeyStride + lane * 16;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[r][e] = 0.f;
#pragma unroll
    for (int j = 0; j < T::kKeyOps; ++j) {
      const v8h k = *reinterpret_cast<const v8h*>(from + j * T::kKeyStride);
#pragma unroll
      for (int r = 0; r < R; ++r) sc[r] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, q[r][j], sc[r], 0, 0, 0);
    }
  };
  auto weights = [&](int step, int t, const Groups& w, v16f (&sc)[R], v8h (&p)[R][2]) {
    float ks[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      ks[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w.ks), 2 * t + i));
    if (step * kStep + kStep > block_lo || __any(w.pid < 0)) {        // where store_values looks for NaN codes
      const unsigned long long there = __ballot(w.pid >= 0) >> (2 * t);      // bit i: group i
      const unsigned nan = s_nan[step % 3][t];
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i) {                                 // group of 16 tokens, eight of them this lane's
          const int first = 16 * i + 8 * half;
          const unsigned bad = nan >> first;
          const int live = there >> i & 1 ? limit[r] - step * kStep - 32 * t - first : 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = sc[r][8 * i + e];
            sc[r][8 * i + e] = e < live ? (bad >> e & 1 ? __builtin_nanf("") : x) : -__builtin_inff();
          }
          __builtin_amdgcn_sched_barrier(0);                          // (all comparisons at once would not fit the scalar registers)
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float f[2], top = kNoMax;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f[i] = ks[i] * row_scale[r];
        float best = sc[r][8 * i];
#pragma unroll
        for (int e = 1; e < 8; ++e) best = fmaxf(best, sc[r][8 * i + e]);
        top = fmaxf(top, best * f[i]);
      }
      if (__any(top > m[r] + 8.f)) {
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m[r], top), g = exp2_fast(m[r] - now);
        m[r] = now;
        l[r] *= g;
#pragma unroll
        for (int c = 0; c < T::kValueTiles; ++c) {
          acc[r][c] *= g;
          __builtin_amdgcn_sched_barrier(0);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float x = exp2_fast(__builtin_fmaf(sc[r][8 * i + e], f[i], -m[r]));
          const float y = exp2_fast(__builtin_fmaf(sc[r][8 * i + e + 1], f[i], -m[r]));
          const v2h two = {(_Float16)x, (_Float16)y};
          l[r] = __builtin_amdgcn_fdot2(two, (v2h){(_Float16)1.f, (_Float16)1.f}, l[r], false);
          p[r][i][e] = two[0];
          p[r][i][e + 1] = two[1];
        }
    }
  };
  auto values = [&](int buffer, int t, const v8h (&p)[R][2]) {
    const uint8_t* from = s_values + buffer * T::kValueBytes + 2 * t * T::kValueStride + lane * 16;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int c = 0; c < T::kValueTiles; ++c) {
        const v8h v = *reinterpret_cast<const v8h*>(from + (c * 4 + i) * T::kValueStride);
#pragma unroll
        for (int r = 0; r < R; ++r) acc[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[r][i], acc[r][c], 0, 0, 0);
      }
  };

  if (steps > 0) {
    // Step i: logits of its second 32 tokens and of the next step's first, weights and values of both its 32; written to LDS: keys of
    // i + 2, values of i + 1; asked for: keys of i + 3, values of i + 2.  Beyond the last step the last one's codes are loaded again,
    // and not used.
    auto at = [&](int i) { return step0 + (i < steps ? i : steps - 1); };
    Groups g0, g1, g2, g3;
    float next_unit = 1.f;
    if (tid < 6) s_nan[tid >> 1][tid & 1] = 0;
    g0.pid = page_of(at(0));
    g1.pid = page_of(at(1));
    g2.pid = page_of(at(2));
    load_scales(&g0);
    load_scales(&g1);
    load_keys(at(0), g0.pid);
    load_values(at(0), g0.pid);
    store_keys(0);
    __syncthreads();                                                  // s_nan
    next_unit = unit_of(next_unit, g0);
    store_values(0, at(0), g0, next_unit);
    load_keys(at(1), g1.pid);
    store_keys(1);
    load_keys(at(2), g2.pid);
    load_values(at(1), g1.pid);
    __syncthreads();
    v16f sc0[R], sc1[R];
    if (at(0) * kStep < wave_hi) logits(0, 0, sc0);
    int key_buffer = 0;                                               // of step i
    for (int i = 0; i < steps; ++i) {
      const int key_next = key_buffer + 1 == T::kKeyBuffers ? 0 : key_buffer + 1;
      const int key_store = key_next + 1 == T::kKeyBuffers ? 0 : key_next + 1;
      if (i > 0) __syncthreads();
      const float unit = next_unit;
      if (tid < 2) s_nan[(step0 + i + 2) % 3][tid] = 0;               // last read a step ago
      if (i + 1 < steps) {
        next_unit = unit_of(unit, g1);
        store_values((i + 1) & 1, at(i + 1), g1, next_unit);
      }
      load_values(at(i + 2), g2.pid);
      if constexpr (T::kKeyBuffers == 3) {
        if (i + 2 < steps) store_keys(key_store);
        g3.pid = page_of(at(i + 3));
        load_keys(at(i + 3), g3.pid);
      }
      load_scales(&g2);
      const bool live = at(i) * kStep < wave_hi;
      v8h p[R][2];
      if (live) {
        if (unit != acc_unit) {
          const float f = acc_unit / unit;
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < T::kValueTiles; ++c) {
              acc[r][c] *= f;
              __builtin_amdgcn_sched_barrier(0);
            }
          acc_unit = unit;
        }
        logits(key_buffer, 1, sc1);
        weights(at(i), 0, g0, sc0, p);
        values(i & 1, 0, p);
      }
      if constexpr (T::kKeyBuffers == 2) {
        __syncthreads();
        if (i + 2 < steps) store_keys(key_store);
        g3.pid = page_of(at(i + 3));
        load_keys(at(i + 3), g3.pid);
      }
      if (i + 1 < steps && at(i + 1) * kStep < wave_hi) logits(key_next, 0, sc0);
      if (live) {
        weights(at(i), 1, g0, sc1, p);
        values(i & 1, 1, p);
      }
      g0 = g1;
      g1 = g2;
      g2.pid = g3.pid;
      key_buffer = key_next;
    }
  }

  // ---- results
#pragma unroll
  for (int r = 0; r < R; ++r) l[r] += __shfl_xor(l[r], 32);
  if (parts <= 1) {
    __syncthreads();                                                  // the tiles are no longer read
    uint16_t* const s_out = reinterpret_cast<uint16_t*>(s_tiles) + wave * 32 * T::kOutStride;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float inv = l[r] == 0.f ? 0.f : acc_unit / l[r];
#pragma unroll
      for (int c = 0; c < T::kValueTiles; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          float x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = acc[r][c][e + i] * inv;
          *reinterpret_cast<v2u*>(s_out + n * T::kOutStride + 32 * c + 2 * e + 4 * half) =
              (v2u){narrow<BF16>(x[0]) | narrow<BF16>(x[1]) << 16, narrow<BF16>(x[2]) | narrow<BF16>(x[3]) << 16};
        }
      __builtin_amdgcn_wave_barrier();                                // a wave reads what it wrote itself: in order
      const int row0 = r0 + 32 * r;
      for (int i = lane; i < 32 * (D / 8); i += 64) {
        const int row = row0 + i / (D / 8), c = 8 * (i % (D / 8));
        if (row < rows) {
          const int tok = row / a.g;
          uint16_t* to = static_cast<uint16_t*>(a.out.data) + (long long)(s.first + tok) * a.out.token_stride +
                         (long long)(h * a.g + row - tok * a.g) * a.out.head_stride + c;
          *reinterpret_cast<v4u*>(to) = *reinterpret_cast<const v4u*>(s_out + (i / (D / 8)) * T::kOutStride + c);
        }
      }
      __builtin_amdgcn_wave_barrier();
      const int row = row0 + n, tok = row / a.g;
      if (a.lse && half == 0 && row < rows)
        a.lse[(size_t)(s.first + tok) * a.q.heads + h * a.g + row - tok * a.g] =
            l[r] == 0.f ? -__builtin_inff() : (m[r] + log2f(l[r])) * kLn2;
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int row = r0 + 32 * r + n, tok = row / a.g;
      if (row >= rows) continue;
      const size_t part = ((size_t)(s.first + tok) * a.q.heads + h * a.g + row - tok * a.g) * a.plan.splits + split;
#pragma unroll
      for (int c = 0; c < T::kValueTiles; ++c)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<v4f*>(a.acc + part * D + 32 * c + 2 * e + 4 * half) =
              (v4f){acc[r][c][e], acc[r][c][e + 1], acc[r][c][e + 2], acc[r][c][e + 3]} * acc_unit;
      if (half == 0) *reinterpret_cast<v2f*>(a.ml + part * 2) = (v2f){m[r], l[r]};
    }
  }
}

template <int D>
hipError_t launch_prompt_d(const PagedAttention& a, bool bf16, hipStream_t stream) {
  const long long blocks = (long long)a.batch.batch * a.cache.heads * a.plan.prompt_blocks * a.plan.prompt_splits;
  if (blocks >= 1ll << 24) return hipErrorInvalidValue;      // 2^32 threads
  const auto kernel = bf16 ? prompt_kernel<D, true> : prompt_kernel<D, false>;
  static std::atomic<size_t> raised[2][kPagedDevices];
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(kernel), Prompt<D>::kLds, raised[bf16]);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)blocks), dim3(kPromptThreads), Prompt<D>::kLds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int prompt_rows(int d) { return d <= 128 ? 64 * kPromptWaves : 32 * kPromptWaves; }

hipError_t launch_paged_prompt(const PagedAttention& a, bool bf16, hipStream_t stream) { CQ_FOR_HEAD_DIM(launch_prompt_d); }

}  // namespace cq

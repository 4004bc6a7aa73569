// Attention over the paged e4m3 cache for few query rows per KV head: single tokens, drafted ones.
//
// Rows: the (new token, query head) pairs of one KV head, 16 to a tile of the matrix cores.  A wave takes 64 tokens at a time:
//     S^T = K Q^T      A = key codes as fp16 (token rows), B = queries          v_mfma_f32_16x16x32_f16
//     p = exp2(s - m)  with the row's running maximum m and sum l
//     O^T += V^T P^T   A = value codes as fp16 (channel rows), B = weights
// Lane l holds, of every product's result, column (query row) l % 16.  Which token is which row of S^T is free, and is chosen such that
// the weights a lane has computed ARE its operand of the second product: row 4 a + i of tile t is token 16 a + 4 t + i of the 64,
// so lane group l / 16 holds the weights of the 16 tokens 16 (l / 16) .. + 15, and its piece of the values is 16
// consecutive bytes of a channel - which is why a page has its values channel by channel.  Nothing crosses
// lanes but the maximum, nothing passes through LDS before the end, and since a page holds at least 16 tokens all of a
// lane's weights have one key scale and one value scale.
//
// Bound: HBM, 2 d bytes per token and KV head.  Each wave keeps the keys or the values of its next step in flight while it
// works on the other (8 KB each at 128 channels).  The four waves of a workgroup take the steps in turn and join
// their (m, l, O) in LDS; a long sequence is split over workgroups, whose partials the one that ends last joins while they are
// few, and another launch otherwise (make_paged_plan).
// 64 sequences of up to 8192 tokens, 8 KV heads of 128 channels: 961 MB in 156 us, 6.2 TB/s (a plain read 7.1); 8 of up to 65536: 1071
// MB in 170 us, 6.3 TB/s.  One sequence of 1000 tokens takes 10 us, and 8 drafted tokens of 16 sequences (3328 tokens, 64 channels, 32 rows
// per KV head) 15: the trips to memory that follow each other - the sequence, its pages, their codes, the parts' meeting - and a launch.
#include "paged_device.h"
#include "decode_meet.h"

namespace cq {
namespace {

constexpr int kWaves = 4;

template <int D, int NT, bool BF16>
struct Few {
  static constexpr int kPieces = D / 64;            // 16-byte pieces of a key row that a lane loads,
  static constexpr bool kHalfPiece = D % 64 != 0;   // and one of 8 bytes
  static constexpr int kKeyOps = D / 32;            // products of 32 channels
  static constexpr int kValueTiles = D / 16;
  static constexpr bool kPair = !BF16;              // weights as pairs of fp16: below the rounding of an fp16 result
};

// Whether, and where, 16 tokens lie: lane group by lane group.
struct Place {
  int pid;        // page, -1: not there or behind the end
  int offset;     // of the 16 tokens in their page
};

// Four channels of a row's result, o / sum.
template <bool BF16>
__device__ inline void store_result(const PagedAttention& a, size_t row, int hq, int c, v4f o, float sum, float top) {
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  uint16_t* p = static_cast<uint16_t*>(a.out.data) + row * a.out.token_stride + hq * a.out.head_stride + c;
  *reinterpret_cast<v2u*>(p) = (v2u){narrow<BF16>(o[0] * inv) | narrow<BF16>(o[1] * inv) << 16,
                                     narrow<BF16>(o[2] * inv) | narrow<BF16>(o[3] * inv) << 16};
  if (a.lse && c == 0) a.lse[row * a.q.heads + hq] = sum == 0.f ? -__builtin_inff() : (top + log2f(sum)) * kLn2;
}

template <int D, int NT, bool BF16>
__global__ void __launch_bounds__(256, D * NT <= 128 ? 2 : 1) few_kernel(PagedAttention a) {
  using T = Few<D, NT, BF16>;
  constexpr int kRows = 16 * NT;
  extern __shared__ __align__(16) float s_acc[];        // [kWaves][kRows][D + 4]
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ bool s_last;
  const PagedCacheArgs& C = a.cache;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, n = lane & 15, grp = lane >> 4;
  // blocks of rows of the same tokens eight apart: an XCD takes every eighth workgroup, and they meet in its L2
  const unsigned blocks = (unsigned)a.plan.row_blocks;
  const int rb = (int)(blockIdx.x / 8 % blocks);
  unsigned id = blocks == 1 ? blockIdx.x : blockIdx.x / (8 * blocks) * 8 + blockIdx.x % 8;
  const int split = (int)(id % (unsigned)a.plan.few_splits);
  id /= (unsigned)a.plan.few_splits;
  const int h = (int)(id % (unsigned)C.heads), b = (int)(id / (unsigned)C.heads);
  if (b >= a.batch.batch) return;                       // the grid is rounded up
  const Sequence s = load_sequence(a.batch, b);
  const int rows = s.n * a.g, r0 = (blocks == 1 ? 0 : rb) * kRows;
  if (r0 >= rows || (a.plan.prompts && rows > kFewRows)) return;
  const int parts = ceil_div(ceil_div(s.len, kStep), a.plan.split_steps);      // splits of this sequence
  if (split >= (parts > 1 ? parts : 1)) return;
  const bool joins = parts > 1 && a.plan.few_joins;
  u64* const count = a.counts + ((size_t)b * C.heads + h) * blocks + (blocks == 1 ? 0 : rb);
  u64 seen = 0;
  if (joins && tid == 255) seen = count_open(count, a.tag);

  // this lane's rows
  int limit[NT], at_row[NT], at_head[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = r0 + 16 * t + n, i = r / a.g;
    at_row[t] = s.first + i;
    at_head[t] = h * a.g + (r - i * a.g);
    limit[t] = r >= rows ? 0 : a.causal ? clamp_int(s.pos0 + i + 1, 0, s.len) : s.len;
  }
  // the fewest and the most tokens that a row of the workgroup sees
  const int last_row = (r0 + kRows < rows ? r0 + kRows : rows) - 1;
  const int lim_lo = a.causal ? clamp_int(s.pos0 + r0 / a.g + 1, 0, s.len) : s.len;
  const int lim_hi = a.causal ? clamp_int(s.pos0 + last_row / a.g + 1, 0, s.len) : s.len;
  const int step0 = split * a.plan.split_steps;
  int step1 = step0 + a.plan.split_steps;
  if (step1 > ceil_div(lim_hi, kStep)) step1 = ceil_div(lim_hi, kStep);

  const bool once = C.page <= 64 && a.plan.row_blocks == 1;
  const int32_t* table = a.batch.page_table + (size_t)b * a.batch.max_pages;
  auto place_of = [&](int step) {
    const int tok = step * kStep + 16 * grp;
    Place w;
    w.pid = tok < s.len ? table[tok >> C.page_log2] : -1;
    if ((unsigned)w.pid >= (unsigned)C.n_pages) w.pid = -1;
    w.offset = tok & (C.page - 1);
    return w;
  };
  int step = step0 + wave;
  Place here = {-1, 0}, next = {-1, 0};
  if (step < step1) here = place_of(step);
  // everything that the first step needs is asked for before the queries are made operands
  v4u raw[NT][T::kKeyOps];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint16_t* p = static_cast<const uint16_t*>(a.q.data);
    const bool there = r0 + 16 * t + n < rows;
    if (there) p += at_row[t] * a.q.token_stride + at_head[t] * a.q.head_stride;
#pragma unroll
    for (int j = 0; j < T::kKeyOps; ++j) {
      const int c = j < 2 * T::kPieces ? (j / 2) * 64 + grp * 16 + (j % 2) * 8 : T::kPieces * 64 + grp * 8;
      raw[t][j] = there ? *reinterpret_cast<const v4u*>(p + c) : (v4u){0, 0, 0, 0};
    }
  }
  v4u key[4][T::kPieces > 0 ? T::kPieces : 1];
  v2u key_half[4];
  v4u val[T::kValueTiles];
  float key_scale, val_scale, next_key_scale = 1.f, next_val_scale = 1.f;
  auto load_keys = [&](const Place& w) {
    // row n of tile t is token 4 t + n % 4 of lane group n / 4
    const int pid = __shfl(w.pid, 16 * (n >> 2)), offset = __shfl(w.offset, 16 * (n >> 2));
    const uint8_t* p = C.k_codes + ((((size_t)(pid < 0 ? 0 : pid) * C.heads + h) << C.page_log2) + offset + (n & 3)) * D;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int j = 0; j < T::kPieces; ++j) key[t][j] = *reinterpret_cast<const v4u*>(p + 4 * t * D + 64 * j + 16 * grp);
      if constexpr (T::kHalfPiece) key_half[t] = *reinterpret_cast<const v2u*>(p + 4 * t * D + 64 * T::kPieces + 8 * grp);
    }
  };
  auto load_values = [&](const Place& w) {
    const uint8_t* p = C.v_codes + ((((size_t)(w.pid < 0 ? 0 : w.pid) * C.heads + h) * D + n) << C.page_log2) + w.offset;
    // non-temporal where one instruction covers whole lines and nobody else reads them: a page's channel rows of 128 bytes and more
    // are read half by half
    if (once) {
      asm volatile("; once");           // (without these the compiler makes one ordinary load of the two)
#pragma unroll
      for (int t = 0; t < T::kValueTiles; ++t) val[t] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p + ((size_t)(16 * t) << C.page_log2)));
      asm volatile("; once");
    } else {
#pragma unroll
      for (int t = 0; t < T::kValueTiles; ++t) val[t] = *reinterpret_cast<const v4u*>(p + ((size_t)(16 * t) << C.page_log2));
    }
  };
  auto load_scales = [&](const Place& w) {
    const size_t i = (size_t)(w.pid < 0 ? 0 : w.pid) * C.heads + h;
    next_key_scale = C.k_scale[i];
    next_val_scale = w.pid < 0 ? 0.f : C.v_scale[i];     // 0 marks tokens that are not there
  };

  if (step < step1) {
    load_scales(here);
    load_keys(here);
    load_values(here);
    next = place_of(step + kWaves < step1 ? step + kWaves : step);
  }
  // queries: every row scaled by a power of two
  v8h q[NT][T::kKeyOps];
  float row_scale[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float most = 0.f;
#pragma unroll
    for (int j = 0; j < T::kKeyOps; ++j) {
      float x[8];
      widen8<BF16>(raw[t][j], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) most = fmaxf(most, __builtin_isfinite(x[i]) ? fabsf(x[i]) : 0.f);
    }
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    const float up = row_unit(most);
    row_scale[t] = a.scale_log2 / up;
#pragma unroll
    for (int j = 0; j < T::kKeyOps; ++j) {
      float x[8];
      widen8<BF16>(raw[t][j], x);
#pragma unroll
      for (int i = 0; i < 8; ++i) q[t][j][i] = (_Float16)(x[i] * up);
    }
  }

  v4f acc[NT][T::kValueTiles];
  float m[NT], l[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    m[t] = kNoMax;
    l[t] = 0.f;
#pragma unroll
    for (int c = 0; c < T::kValueTiles; ++c) acc[t][c] = (v4f){0.f, 0.f, 0.f, 0.f};
  }

  for (; step < step1; step += kWaves) {
    key_scale = next_key_scale;
    val_scale = next_val_scale;
    // ---- logits
    v4f sc[NT][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int r = 0; r < NT; ++r) sc[r][t] = (v4f){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < T::kKeyOps; ++j) {
        v8h k8;
        if (j < 2 * T::kPieces) k8 = codes_to_half(key[t][j / 2][2 * (j % 2)], key[t][j / 2][2 * (j % 2) + 1], 1.f);
        else k8 = codes_to_half(key_half[t][0], key_half[t][1], 1.f);
#pragma unroll
        for (int r = 0; r < NT; ++r) sc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k8, q[r][j], sc[r][t], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_sched_barrier(0);
    const bool more = step + kWaves < step1;
    if (more) {
      load_scales(next);
      load_keys(next);
    }
    const bool there = here.pid >= 0;
    const int tok = step * kStep + 16 * grp;
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      const float f = key_scale * row_scale[r];
#pragma unroll
      for (int t = 0; t < 4; ++t) sc[r][t] *= f;
    }
    // ---- tokens that some row does not see
    if (step * kStep + kStep > lim_lo || !__all(there)) {
      // NaN codes of the values must not reach rows whose weight is 0: they are cleared, and the token's logit becomes the NaN
      unsigned nan[4] = {0, 0, 0, 0};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        // bytes of tokens that no row sees, or that are not there
        const int live = there ? clamp_int(lim_hi - tok - 4 * w, 0, 4) : 0;
        const unsigned keep = live == 4 ? 0xffffffffu : (1u << (8 * live)) - 1u;
#pragma unroll
        for (int c = 0; c < T::kValueTiles; ++c) {
          unsigned x = val[c][w] & keep;
          const unsigned bad = nan_codes(x);
          nan[w] |= bad;
          val[c][w] = x & ~((bad >> 7) * 0xffu);
        }
        nan[w] |= __shfl_xor(nan[w], 1);
        nan[w] |= __shfl_xor(nan[w], 2);
        nan[w] |= __shfl_xor(nan[w], 4);
        nan[w] |= __shfl_xor(nan[w], 8);
      }
#pragma unroll
      for (int r = 0; r < NT; ++r)
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (nan[t] >> (8 * i + 7) & 1) sc[r][t][i] = __builtin_nanf("");
            if (!there || tok + 4 * t + i >= limit[r]) sc[r][t][i] = -__builtin_inff();
          }
    }
    // ---- softmax
    v8h p_hi[NT][2], p_lo[NT][2];
#pragma unroll
    for (int r = 0; r < NT; ++r) {
      float top = sc[r][0][0];
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, sc[r][t][i]);
      if (__any(top > m[r])) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = fmaxf(m[r], top), f = exp2_fast(m[r] - now);
        m[r] = now;
        l[r] *= f;
#pragma unroll
        for (int c = 0; c < T::kValueTiles; ++c) acc[r][c] *= f;
      }
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_fast(sc[r][t][i] - m[r]);
          l[r] += p;
          const _Float16 hi = (_Float16)p;
          p_hi[r][t / 2][4 * (t % 2) + i] = hi;
          if constexpr (T::kPair) p_lo[r][t / 2][4 * (t % 2) + i] = (_Float16)(p - (float)hi);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    // ---- values, in units of the largest scale of the 64 tokens
    float unit = fmaxf(val_scale, __shfl_xor(val_scale, 16));
    unit = fmaxf(unit, __shfl_xor(unit, 32));
    const bool near = val_scale == 0.f || val_scale >= unit * 0x1p-15f;
    // pages whose scales lie too far apart for one fp16 range: lane group by lane group, the others' weights 0
    const bool together = __all(near);
#pragma unroll 1
    for (int part = 0; part < (together ? 1 : 4); ++part) {
      const float f = together ? unit : __shfl(val_scale, 16 * part);
      float rel = together && val_scale != 0.f ? val_scale / unit : 1.f;
      asm volatile("" : "+v"(rel));          // the values become fp16 here, and are not kept as such for the next round
      const unsigned mine = together || grp == part ? 0xffffffffu : 0u;
      v8h w_hi[NT][2], w_lo[NT][2];
#pragma unroll
      for (int r = 0; r < NT; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w_hi[r][i] = __builtin_bit_cast(v8h, __builtin_bit_cast(v4u, p_hi[r][i]) & mine);
          if constexpr (T::kPair) w_lo[r][i] = __builtin_bit_cast(v8h, __builtin_bit_cast(v4u, p_lo[r][i]) & mine);
        }
#pragma unroll
      for (int c = 0; c < T::kValueTiles; ++c) {
        const v8h v0 = codes_to_half(val[c][0], val[c][1], rel), v1 = codes_to_half(val[c][2], val[c][3], rel);
#pragma unroll
        for (int r = 0; r < NT; ++r) {
          v4f o = {0.f, 0.f, 0.f, 0.f};
          o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w_hi[r][0], o, 0, 0, 0);
          o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w_hi[r][1], o, 0, 0, 0);
          if constexpr (T::kPair) {
            o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, w_lo[r][0], o, 0, 0, 0);
            o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, w_lo[r][1], o, 0, 0, 0);
          }
          acc[r][c] += o * f;
        }
        if (c % 2) __builtin_amdgcn_sched_barrier(0);
      }
    }
    here = next;
    if (more) {
      load_values(next);
      if (step + 2 * kWaves < step1) next = place_of(step + 2 * kWaves);
    }
  }

  // ---- the four waves' parts
#pragma unroll
  for (int r = 0; r < NT; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    if (grp == 0) {
      s_m[wave][16 * r + n] = m[r];
      s_l[wave][16 * r + n] = l[r];
    }
#pragma unroll
    for (int c = 0; c < T::kValueTiles; ++c)
      *reinterpret_cast<v4f*>(s_acc + (size_t)(wave * kRows + 16 * r + n) * (D + 4) + 16 * c + 4 * grp) = acc[r][c];
  }
  __syncthreads();
  for (int i = tid; i < kRows * (D / 4); i += 256) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    if (r0 + r >= rows) break;
    float top = s_m[0][r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
    float sum = 0.f;
    v4f o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = exp2_fast(s_m[w][r] - top);
      sum += s_l[w][r] * f;
      o += *reinterpret_cast<const v4f*>(s_acc + (size_t)(w * kRows + r) * (D + 4) + c) * f;
    }
    const int i_new = (r0 + r) / a.g, hq = h * a.g + (r0 + r) - i_new * a.g;
    const size_t row = (size_t)(s.first + i_new);
    if (parts <= 1) {
      store_result<BF16>(a, row, hq, c, o, sum, top);
    } else {
      const size_t part = (row * a.q.heads + hq) * a.plan.splits + split;
      store_device(a.acc + part * D + c, o[0], o[1]);
      store_device(a.acc + part * D + c + 2, o[2], o[3]);
      if (c == 0) store_device(a.ml + part * 2, top, sum);
    }
  }
  if (!joins) return;

  // ---- the workgroup that is counted last joins the splits, in their order
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");          // this wave's part has reached memory
  __syncthreads();
  if (tid == 255) s_last = count_in(count, a.tag, seen) == parts - 1;
  __syncthreads();
  if (!s_last) return;
  const int live = rows - r0 < kRows ? rows - r0 : kRows;
  auto first_part = [&](int r) {
    const int i_new = (r0 + r) / a.g;
    return ((size_t)(s.first + i_new) * a.q.heads + h * a.g + (r0 + r) - i_new * a.g) * a.plan.splits;
  };
  for (int i = tid; i < live * (D / 4); i += 256) {
    const int r = i / (D / 4), c = 4 * (i % (D / 4));
    const size_t first = first_part(r);
    float top = kNoMax, sum = 0.f;
    v4f o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; p0 < parts; p0 += 8) {        // eight parts' loads at once: each is a trip to memory
      v2f w[8], x[8], y[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const size_t p = first + (p0 + u < parts ? p0 + u : parts - 1);
        w[u] = load_device(a.ml + 2 * p);
        x[u] = load_device(a.acc + p * D + c);
        y[u] = load_device(a.acc + p * D + c + 2);
      }
      float to = top;
#pragma unroll
      for (int u = 0; u < 8; ++u) to = fmaxf(to, w[u][0]);
      const float keep = exp2_fast(top - to);
      top = to;
      sum *= keep;
      o *= keep;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float f = p0 + u < parts ? exp2_fast(w[u][0] - top) : 0.f;
        sum += w[u][1] * f;
        o += (v4f){x[u][0], x[u][1], y[u][0], y[u][1]} * f;
      }
    }
    const int i_new = (r0 + r) / a.g;
    store_result<BF16>(a, (size_t)(s.first + i_new), h * a.g + (r0 + r) - i_new * a.g, c, o, sum, top);
  }
  if (tid == 0) *count = 0;
}

// Joins the splits of rows: a workgroup of four waves, a wave to some heads of a token, a lane to pairs of channels.  Bound: the trips to memory
// that follow each other, so four parts' maxima, sums and results are asked for together; 94 MB of parts of 1425 tokens of 32 heads, four
// heads to a wave, in 18.5 us, 5.6 TB/s (25 with a head to a wave, 30 with a part after the other).
template <int D, bool BF16>
__global__ void __launch_bounds__(256) combine_splits_kernel(PagedAttention a, int heads_per_wave, unsigned groups) {
  constexpr int kPairs = (D + 127) / 128, kAtOnce = 4;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const unsigned id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(wave);       // (the host holds rows below 2^26)
  const int hq0 = (int)(id % groups) * heads_per_wave, at = (int)(id / groups);               // row of the tokens
  const int first_row = clamp_int(__builtin_amdgcn_readfirstlane(a.batch.q_start[0]), 0, a.batch.n_tokens);
  if (at < first_row) return;
  const Item item = locate(a.batch, at - first_row, [&](const Sequence& s) { return s.len - s.pos0; });      // all rows of a sequence
  if (item.b < 0) return;
  const int i = item.local;
  const Sequence s = item.s;
  const bool few = a.plan.few && (!a.plan.prompts || s.n * a.g <= kFewRows);
  if (few && a.plan.few_joins) return;
  const int split_steps = few ? a.plan.split_steps : a.plan.prompt_split_steps;
  if (i >= s.n || ceil_div(ceil_div(s.len, kStep), split_steps) <= 1) return;
  // the parts that hold a token which the row sees
  const int limit = a.causal ? clamp_int(s.pos0 + i + 1, 0, s.len) : s.len;
  const int parts = ceil_div(ceil_div(limit, kStep), split_steps);
  const int hq1 = hq0 + heads_per_wave < a.q.heads ? hq0 + heads_per_wave : a.q.heads;
  for (int hq = hq0; hq < hq1; ++hq) {
    const size_t row = (size_t)(s.first + i), first = (row * a.q.heads + hq) * a.plan.splits;
    const v2f* const ml = reinterpret_cast<const v2f*>(a.ml) + first;
    const float* const acc = a.acc + first * D;
    float top = kNoMax, sum = 0.f;
    v2f o[kPairs];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) o[j] = (v2f){0.f, 0.f};
    for (int p0 = 0; p0 < parts; p0 += kAtOnce) {
      v2f w[kAtOnce], x[kAtOnce][kPairs];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int p = p0 + u < parts ? p0 + u : parts - 1;
        w[u] = ml[p];
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
          const int c = 2 * lane + 128 * j;
          x[u][j] = *reinterpret_cast<const v2f*>(acc + (size_t)p * D + (c < D ? c : 0));
        }
      }
      float to = top;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) to = fmaxf(to, w[u][0]);
      const float keep = exp2_fast(top - to);
      top = to;
      sum *= keep;
#pragma unroll
      for (int j = 0; j < kPairs; ++j) o[j] *= keep;
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const float f = p0 + u < parts ? exp2_fast(w[u][0] - top) : 0.f;
        sum += w[u][1] * f;
#pragma unroll
        for (int j = 0; j < kPairs; ++j) o[j] += x[u][j] * f;
      }
    }
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    uint16_t* p = static_cast<uint16_t*>(a.out.data) + row * a.out.token_stride + hq * a.out.head_stride;
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
      const int c = 2 * lane + 128 * j;
      if (c < D) *reinterpret_cast<unsigned*>(p + c) = narrow<BF16>(o[j][0] * inv) | narrow<BF16>(o[j][1] * inv) << 16;
    }
    if (a.lse && lane == 0) a.lse[row * a.q.heads + hq] = sum == 0.f ? -__builtin_inff() : (top + log2f(sum)) * kLn2;
  }
}

template <int D, int NT>
hipError_t launch_few(const PagedAttention& a, bool bf16, hipStream_t stream) {
  long long blocks = (long long)a.batch.batch * a.cache.heads * a.plan.few_splits;
  if (a.plan.row_blocks > 1) blocks = (blocks + 7) / 8 * 8 * a.plan.row_blocks;
  const size_t lds = (size_t)kWaves * 16 * NT * (D + 4) * sizeof(float);
  const auto kernel = bf16 ? few_kernel<D, NT, true> : few_kernel<D, NT, false>;
  static std::atomic<size_t> raised[2][kPagedDevices];
  const hipError_t e = raise_lds(reinterpret_cast<const void*>(kernel), lds, raised[bf16]);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)blocks), dim3(256), lds, stream>>>(a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_few_d(const PagedAttention& a, bool bf16, hipStream_t stream) {
  return a.plan.row_tiles == 1 ? launch_few<D, 1>(a, bf16, stream) : launch_few<D, 2>(a, bf16, stream);
}

template <int D>
hipError_t launch_combine_d(const PagedAttention& a, bool bf16, hipStream_t stream) {
  // four heads to a wave while they leave the chip a full round of waves (32 to a CU)
  const long long rows = (long long)a.batch.n_tokens * a.q.heads;
  const int heads = rows >= 4 * 32ll * device_cu_count() ? 4 : 1;
  const unsigned groups = (unsigned)ceil_div(a.q.heads, heads);
  const unsigned blocks = (unsigned)(((long long)a.batch.n_tokens * groups + 3) / 4);
  if (bf16) combine_splits_kernel<D, true><<<dim3(blocks), dim3(256), 0, stream>>>(a, heads, groups);
  else combine_splits_kernel<D, false><<<dim3(blocks), dim3(256), 0, stream>>>(a, heads, groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_few(const PagedAttention& a, bool bf16, hipStream_t stream) { CQ_FOR_HEAD_DIM(launch_few_d); }
hipError_t launch_paged_combine(const PagedAttention& a, bool bf16, hipStream_t stream) { CQ_FOR_HEAD_DIM(launch_combine_d); }

// Few rows: a workgroup per (sequence, KV head, tile of rows) and split.  Splits are of a fixed number of tokens, so that sequences of
// different lengths have as many as they need: as many workgroups as are resident at once (two to a CU while their registers
// allow it) if sequences are of the same length, a step for every wave at least (two: 1 x 1000
// tokens, recorded, 10.7 us and 9.2, 4 x 2000 11.2 and 9.9).  Twice as many took 1 to 5 % longer at 64 x 8192, 8 x 65536
// and 32 x 8192 tokens, 20 % at 8 x 4096 and 1 x 65536; 1.5 times as many up to 18 %.
// Over 16 rows a workgroup takes two tiles of them, which share the codes' way to fp16 - but for little work (16 steps of 64 tokens to a
// CU) workgroups of one tile, twice as many: 32 rows, 64 x 3328 tokens, 64 channels 15.3 and 18.4 us; 32 x 4096 tokens, 128 channels 17.3
// and 20.5 with 32 rows, 23 and 27 with 64; but 16 x 43681 tokens 52 and 46, 256 x 8192, 64 channels 100 and 79, and from 192 channels
// on, where a CU holds one workgroup of either, 88 x 1844 tokens 63 and 51.
// While the partial results of a row of workgroups are few (256 KB), the one that ends last joins them;
// otherwise a launch of its own does, whose waves are many.
// Many rows (over kFewRows per KV head): a workgroup takes a block of rows over a split; a CU holds one.  The splits taken are those whose
// time is the least: rounds of workgroups of so many steps each, the partial results' way to memory and back and the launch that joins them
// (the constants are measured).  580 rows over 2373 tokens 30 us, 86 whole and 39 in four splits; 512 x 4 rows over 1024 tokens 32 in
// four, 41 whole; 2048 x 4 rows over as many tokens 72 whole, 83 in two; 3437 x 7 rows, two sequences, 2 heads, 129 whole, 163 in two.
// In a batch some sequences can have few rows all the same, whose workgroups are those of the other kernel - but for caches of up to
// kShortCache tokens, which the first takes in less than a launch (3 x 64 new tokens of 141 17.6 us, 19.4 with both).
PagedPlan make_paged_plan(const PagedCacheArgs& cache, const PagedBatch& batch, int n_q_heads) {
  PagedPlan p;
  const long long cus = device_cu_count();
  const int g = n_q_heads / cache.heads;
  const long long rows = (long long)batch.max_new * g;
  const int steps = ceil_div(batch.len_bound, kStep);
  p.prompts = rows > kFewRows;
  p.few = !p.prompts || (batch.batch > 1 && g <= kFewRows && batch.len_bound > kShortCache);
  if (p.few) {
    const long long few = rows < kFewRows ? rows : kFewRows;
    p.row_tiles = few > 16 && (cache.d > 128 || (long long)batch.batch * cache.heads * steps > 16 * cus) ? 2 : 1;
    p.row_blocks = (int)((few + 16 * p.row_tiles - 1) / (16 * p.row_tiles));
    const long long beside = (long long)batch.batch * cache.heads * p.row_blocks;
    long long want = cus * (cache.d * p.row_tiles <= 128 ? 2 : 1) / beside;
    long long most = ceil_div(steps, 4);
    if (most > kMostSplits) most = kMostSplits;
    if (want > most) want = most;
    if (want < 1) want = 1;
    p.split_steps = ceil_div(steps, (int)want);
    p.few_splits = p.splits = ceil_div(steps, p.split_steps);
    const long long parts = few * p.few_splits;
    p.few_joins = p.few_splits > 1 && parts * cache.d <= 65536;
  }
  if (p.prompts) {
    const int block = prompt_rows(cache.d);
    // all tokens' rows in whole blocks, and one begun for each sequence; of one sequence, or of even ones, what the longest takes
    const long long most_blocks = (rows + block - 1) / block * batch.batch, token_blocks = (long long)batch.n_tokens * g / block + batch.batch;
    p.prompt_blocks = (int)(token_blocks < most_blocks ? token_blocks : most_blocks);
    const long long beside = (long long)cache.heads * p.prompt_blocks;
    const long long most = steps / 2 < 32 ? steps / 2 : 32;
    const double step_us = cache.d <= 64 ? 1.1 : 1.1 * cache.d / 64, begin_us = 3.0, join_us = 4.0, join_bytes_per_us = 3.3e6;
    const double bytes_per_split = (double)batch.n_tokens * n_q_heads * (cache.d + 2) * sizeof(float) * 2;       // written and read
    // how much fewer steps the blocks have than the longest, on the average, where rows see up to their own token
    const double fewer = 0.5 * (batch.max_new < batch.len_bound ? batch.max_new : batch.len_bound) / batch.len_bound;
    int best = 1;
    double least = 0;
    for (int n = 1; n <= (most > 1 ? most : 1); ++n) {
      // Equal blocks take whole rounds; unequal ones, the longest first, end together, but not before the longest.
      const double one = ceil_div(steps, n) * step_us + begin_us, rounds = (double)((beside * n + cus - 1) / cus) * one;
      const double mean = (1.0 - fewer) * (steps * step_us + n * begin_us) * beside / cus + (1.0 - 2.0 * fewer) * one;
      const double work = rounds < mean ? rounds : mean > one ? mean : one;
      const double us = work + (n > 1 ? join_us + (n - fewer * (n - 1)) * bytes_per_split / join_bytes_per_us : 0.0);
      if (n == 1 || us < 0.98 * least) {
        best = n;
        least = us;
      }
    }
    p.prompt_split_steps = ceil_div(steps, best);
    p.prompt_splits = ceil_div(steps, p.prompt_split_steps);
    if (p.prompt_splits > p.splits) p.splits = p.prompt_splits;
  }
  if (p.splits > 1) {
    const size_t parts = (size_t)batch.n_tokens * n_q_heads * p.splits;
    if (p.few_joins) p.ws_ml_floats = ((size_t)batch.batch * cache.heads * p.row_blocks * 2 + 63) / 64 * 64;
    p.ws_acc_floats = p.ws_ml_floats + (parts * 2 + 63) / 64 * 64;
    p.ws_bytes = ((p.ws_acc_floats + parts * cache.d) * sizeof(float) + 255) / 256 * 256;
    if (p.ws_bytes == 0) p.ws_bytes = 256;
  }
  // what a launch takes: 2^32 threads
  p.fits = rows < 1ll << 30 && (!p.few || ((long long)batch.batch * cache.heads * p.few_splits + 8) * p.row_blocks < 1ll << 24) &&
           (!p.prompts || (long long)cache.heads * p.prompt_blocks * p.prompt_splits < 1ll << 23) &&
           (long long)batch.n_tokens * n_q_heads < 1ll << 26;
  return p;
}

}  // namespace cq

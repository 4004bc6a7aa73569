// Declarations shared by the host side and the kernels of the paged 8-bit cache.  Not part of the ABI
// (see include/cq_paged.h for that).
#ifndef CQ_PAGED_INTERNAL_H_
#define CQ_PAGED_INTERNAL_H_

#include <atomic>

#include "cq_internal.h"
#include "cq_paged.h"

namespace cq {

constexpr int kStep = 64;   // tokens that the attention kernels take at a time: 16 to 64 of them lie in one page

struct PagedCacheArgs {
  uint8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
  int n_pages, heads, d;
  int page, page_log2;
};

struct PagedBatch {
  const int32_t *page_table, *seq_lens, *q_start;
  int batch, max_pages, max_new, n_tokens;
  int len_bound;   // min(max_len, max_pages * page)
};

struct HeadRows {
  void* data;
  long long token_stride, head_stride;
  int heads;
};

struct RopeArgs {
  uint8_t axis_of[128];  // read eight at a time
  const float* inv_freq;
  const int32_t* positions;
  int half;              // pairs; 0: nothing is turned
  int n_axes;
  int adjacent;          // how they lie
  float sign;            // of the angles
};

// Raises a kernel's limit of dynamic LDS once per device; `raised` holds what it is on each, and only grows.
// Concurrent callers may both raise it, which is harmless.
constexpr int kPagedDevices = 64;
inline hipError_t raise_lds(const void* kernel, size_t bytes, std::atomic<size_t>* raised) {
  if (bytes <= 48 * 1024) return hipSuccess;
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kPagedDevices) return hipErrorInvalidDevice;
  if (bytes <= raised[dev].load(std::memory_order_acquire)) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e != hipSuccess) return e;
  size_t seen = raised[dev].load(std::memory_order_relaxed);
  while (seen < bytes && !raised[dev].compare_exchange_weak(seen, bytes, std::memory_order_release)) {
  }
  return hipSuccess;
}

hipError_t launch_rotate(const RopeArgs& rope, int n_tokens, int d, bool bf16, const HeadRows* in, const HeadRows* out,
                         int n_tensors, hipStream_t stream);
// q_in->heads == 0: no queries
hipError_t launch_append(const PagedCacheArgs& cache, const PagedBatch& batch, bool bf16, const HeadRows& k,
                         const HeadRows& v, const RopeArgs& rope, const HeadRows& q_in, const HeadRows& q_out,
                         hipStream_t stream);

// How the attention of a step is spread: sequences of at most kFewRows (new token, query head) rows per KV head go to one kernel
// (paged_few.hip), those of more to another (paged_prompt.hip).
// At 65 to 96 rows, three blocks of the first, it depends: 72 rows, 8 x 3000 tokens 41 us there and 67 here, 96 rows, 16 x 4096 tokens 97
// and 85; 64 rows, 16 x 4096 tokens 56 and 82, 160 rows 143 and 93 (64 query heads, 128 channels).
constexpr int kFewRows = 64;
constexpr int kShortCache = 512;   // tokens, up to which a batch with sequences of more rows is the second kernel's alone
constexpr int kMostSplits = 128;   // below the 256 that a count holds
struct PagedPlan {
  bool prompts = false;    // sequences of more rows are possible
  bool few = true;         // the first kernel runs
  int row_tiles = 1;       // its tiles of 16 rows per workgroup, 1 or 2
  int row_blocks = 1;      // its workgroups beside each other for the rows of a (sequence, KV head)
  int split_steps = 1;     // its steps of kStep tokens per split of a sequence
  int few_splits = 1;      // of the longest sequence
  bool few_joins = false;  // it joins them itself
  int prompt_blocks = 1;   // blocks of rows of the second kernel, of all sequences
  int prompt_split_steps = 1, prompt_splits = 1;
  int splits = 1;          // the larger number of splits
  size_t ws_ml_floats = 0, ws_acc_floats = 0;   // workspace: [counts | m, l | acc], the latter two [rows][splits]
  size_t ws_bytes = 256;
  bool fits = true;        // every launch has a size that launches take
};
int prompt_rows(int d);    // rows of a workgroup of the second kernel
PagedPlan make_paged_plan(const PagedCacheArgs& cache, const PagedBatch& batch, int n_q_heads);

struct PagedAttention {
  PagedCacheArgs cache;
  PagedBatch batch;
  HeadRows q, out;
  float* lse;
  int g;                   // query heads per KV head
  int causal;
  float scale_log2;        // softmax scale times log2(e)
  PagedPlan plan;
  unsigned long long* counts;   // [batch][KV heads][row blocks] workgroups that have ended (decode_meet.h)
  unsigned long long tag;       // of the call
  float* ml;               // [rows][splits][2] partial maxima and sums
  float* acc;              // [rows][splits][d]
};
hipError_t launch_paged_few(const PagedAttention& a, bool bf16, hipStream_t stream);
hipError_t launch_paged_prompt(const PagedAttention& a, bool bf16, hipStream_t stream);
hipError_t launch_paged_combine(const PagedAttention& a, bool bf16, hipStream_t stream);

#define CQ_FOR_HEAD_DIM(call)              \
  switch (a.cache.d) {                     \
    case 32: return call<32>(a, bf16, stream);   \
    case 64: return call<64>(a, bf16, stream);   \
    case 96: return call<96>(a, bf16, stream);   \
    case 128: return call<128>(a, bf16, stream); \
    case 160: return call<160>(a, bf16, stream); \
    case 192: return call<192>(a, bf16, stream); \
    case 224: return call<224>(a, bf16, stream); \
    case 256: return call<256>(a, bf16, stream); \
  }                                        \
  return hipErrorInvalidValue

}  // namespace cq

#endif  // CQ_PAGED_INTERNAL_H_

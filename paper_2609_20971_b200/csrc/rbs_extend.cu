// rbs_paged_extend: pages, block-table entries, positions and slots of new tokens, from lengths that stand on the device.
// Whole numbers only.  With c the prefix sums of the new lengths (cut at the rows there are) and
//   first_s = ceil(past_s / P),  last_s = ceil((past_s + c_{s+1} - c_s) / P),  a_s = prefix sums of last_s - first_s
// page p of sequence s, first_s <= p < last_s, is entry free_used + a_s + p - first_s of the free list.
// Bound by its launch: a decode step of 64 sequences moves 2 KB, half a million prompt tokens 4.8 MB.
#include "rbs_common.cuh"

namespace rbs {

constexpr int kExtendThreads = 1024;
constexpr int kExtendMaxSeqs = 8192;

struct ExtendParams {
  const int* seq_lens;
  const int* new_lens;
  const int* free_pages;
  const int* free_used;   // nullable
  int* table;
  int* out_lens;
  int* cu_new;
  int* positions;
  int* slots;
  int* free_used_out;
  int S, P, n_pages, max_pages, stride, n_free, T;
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Exclusive prefix sum of one value per thread over the block; `total` = the sum.  `part`: 32 values of shared memory.
__device__ __forceinline__ long long block_scan(long long v, long long* part, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();   // `part` may still be read for the scan before
  if (lane == 31) part[warp] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kExtendThreads / 32; ++w) {
    const long long p = part[w];
    before += w < warp ? p : 0;
    all += p;
  }
  *total = all;
  return before + x - v;
}

// The last index s in [0, n) with a[s] <= v, where a[0] <= v.
__device__ __forceinline__ int last_not_above(const int* a, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] <= v) lo = mid; else hi = mid;
  }
  return lo;
}

// Every CTA scans all lengths for itself (two block scans over at most 8 values per thread, from L2), so that nothing
// is handed from CTA to CTA; then the CTAs share out the sequences, the new table entries and the token rows.
__global__ void __launch_bounds__(kExtendThreads)
extend_kernel(const ExtendParams p) {
  extern __shared__ int shared[];
  int* cu = shared;                  // [S + 1]
  int* at = shared + p.S + 1;        // [S + 1]
  __shared__ long long part[kExtendThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int cap = p.max_pages * p.P;
  const int per = ceil_div(p.S, kExtendThreads);
  const int s0 = min(static_cast<int>(threadIdx.x) * per, p.S), s1 = min(s0 + per, p.S);

  long long sum = 0, total;
  for (int s = s0; s < s1; ++s) sum += max(p.new_lens[s], 0);
  long long run = block_scan(sum, part, &total);
  for (int s = s0; s < s1; ++s) {
    cu[s] = static_cast<int>(min(run, static_cast<long long>(p.T)));
    run += max(p.new_lens[s], 0);
  }
  if (threadIdx.x == 0) cu[p.S] = static_cast<int>(min(total, static_cast<long long>(p.T)));
  __syncthreads();

  sum = 0;
  for (int s = s0; s < s1; ++s) {
    const int past = min(max(p.seq_lens[s], 0), cap);
    sum += ceil_div(min(past + cu[s + 1] - cu[s], cap), p.P) - ceil_div(past, p.P);
  }
  run = block_scan(sum, part, &total);
  for (int s = s0; s < s1; ++s) {
    const int past = min(max(p.seq_lens[s], 0), cap);
    at[s] = static_cast<int>(run);
    run += ceil_div(min(past + cu[s + 1] - cu[s], cap), p.P) - ceil_div(past, p.P);
  }
  if (threadIdx.x == 0) at[p.S] = static_cast<int>(total);
  __syncthreads();

  const int me = blockIdx.x * kExtendThreads + threadIdx.x, step = gridDim.x * kExtendThreads;
  const int used = p.free_used != nullptr ? max(p.free_used[0], 0) : 0;
  const int fresh = at[p.S], n_new = cu[p.S];
  if (me == 0) p.free_used_out[0] = static_cast<int>(min(static_cast<long long>(used) + fresh, 0x7fffffffll));
  for (int s = me; s <= p.S; s += step) {
    p.cu_new[s] = cu[s];
    if (s < p.S) p.out_lens[s] = min(min(max(p.seq_lens[s], 0), cap) + cu[s + 1] - cu[s], cap);
  }
  for (int k = me; k < fresh; k += step) {
    const int s = last_not_above(at, p.S, k);
    const int past = min(max(p.seq_lens[s], 0), cap);
    const long long f = static_cast<long long>(used) + k;
    p.table[static_cast<int64_t>(s) * p.stride + ceil_div(past, p.P) + k - at[s]] = f < p.n_free ? p.free_pages[f] : -1;
  }
  for (long long row = me; row < p.T; row += step) {
    const int i = static_cast<int>(row);
    int pos = 0, slot = -1;
    if (i < n_new) {
      const int s = last_not_above(cu, p.S, i);
      const int past = min(max(p.seq_lens[s], 0), cap);
      pos = past + i - cu[s];
      if (pos < cap) {
        const int page_index = pos / p.P, first = ceil_div(past, p.P);
        int page = -1;
        if (page_index < first) {
          page = p.table[static_cast<int64_t>(s) * p.stride + page_index];   // the page that the sequence had begun
        } else {
          const long long f = static_cast<long long>(used) + at[s] + page_index - first;
          if (f < p.n_free) page = p.free_pages[f];
        }
        if (page >= 0 && page < p.n_pages) slot = page * p.P + pos % p.P;
      }
    }
    p.positions[i] = pos;
    p.slots[i] = slot;
  }
}

}  // namespace rbs

extern "C" rbs_status rbs_paged_extend(const rbs_paged_shape* shape, const int* seq_lens, const int* new_lens,
                                       const int* free_pages, int n_free, const int* free_used, int n_tokens,
                                       int* block_table, int* out_lens, int* cu_new, int* positions, int* slots,
                                       int* free_used_out, void* stream) {
  using namespace rbs;
  NvtxRange range("rbs_paged_extend");
  rbs_status st = check_paged_table(shape);
  if (st != RBS_OK) return st;
  if (n_free < 0 || n_tokens < 0) return RBS_ERR_INVALID_ARG;
  if (seq_lens == nullptr || new_lens == nullptr || block_table == nullptr || out_lens == nullptr || cu_new == nullptr ||
      free_used_out == nullptr)
    return RBS_ERR_INVALID_ARG;
  if ((n_free > 0 && free_pages == nullptr) || (n_tokens > 0 && (positions == nullptr || slots == nullptr)))
    return RBS_ERR_INVALID_ARG;
  if (out_lens == seq_lens || out_lens == new_lens || free_used_out == free_used) return RBS_ERR_INVALID_ARG;
  if (shape->n_seqs > kExtendMaxSeqs) return RBS_ERR_UNSUPPORTED;
  if (static_cast<long long>(shape->max_pages) * shape->page_size + n_tokens >= 0x7fffffffll) return RBS_ERR_UNSUPPORTED;
  ExtendParams p;
  p.seq_lens = seq_lens; p.new_lens = new_lens; p.free_pages = free_pages; p.free_used = free_used;
  p.table = block_table; p.out_lens = out_lens; p.cu_new = cu_new; p.positions = positions; p.slots = slots;
  p.free_used_out = free_used_out;
  p.S = shape->n_seqs; p.P = shape->page_size; p.n_pages = shape->n_pages; p.max_pages = shape->max_pages;
  p.stride = shape->table_stride; p.n_free = n_free; p.T = n_tokens;
  const size_t smem = 2 * (static_cast<size_t>(p.S) + 1) * sizeof(int);
  if ((st = ensure_dynamic_smem(reinterpret_cast<const void*>(extend_kernel), smem)) != RBS_OK) return st;
  const int work = p.T > p.S ? p.T : p.S, sms = sm_count();
  const int ctas = work / kExtendThreads + 1;
  RBS_CUDA_OK(launch_pdl(extend_kernel, ctas < sms ? ctas : sms, 1, kExtendThreads, smem, static_cast<cudaStream_t>(stream), p));
  return RBS_OK;
}

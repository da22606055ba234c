// rbs_paged_extend: pages, block-table entries, positions and slots of new tokens, from lengths that stand on the device.
// Whole numbers only.  With c the prefix sums of the new lengths (cut at the rows there are) and
//   first_s = ceil(past_s / P),  last_s = ceil((past_s + c_{s+1} - c_s) / P),  a_s = prefix sums of last_s - first_s
// page p of sequence s, first_s <= p < last_s, is entry free_used + a_s + p - first_s of the free list.
// A decode step of 64 sequences moves 2 KB and is bound by its launch (2.8 us); 1.2 million prompt tokens move 9.6 MB and are bound by
// the scan in front of their stores (8.1 us).
#include "rbs_common.cuh"
#include "rbs_sm100.cuh"

namespace rbs {

constexpr int kExtendThreads = 1024;
constexpr int kExtendFew = 256;         // threads where there is little to do: barriers of fewer warps are shorter
constexpr int kExtendMaxSeqs = 8192;
constexpr int kExtendRows = 4;          // token rows of a thread, one after the other (a 16-byte store), in large calls
constexpr int kExtendGroups = 2;        // and how many times, a warp's width apart

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
  bool aligned;           // positions and slots take 16-byte stores
  unsigned int* status;   // of the debug build's checks
};

// of a >= 0, without passing 31 bits for lengths and page sizes that come near them
__device__ __forceinline__ int ceil_div(int a, int b) { return a / b + (a % b != 0); }

struct TokensPages {
  long long tokens;
  int pages;
};

// Exclusive prefix sums of one pair per thread over the block; `total` = the sums.
template <int THREADS>
__device__ __forceinline__ TokensPages block_scan(const TokensPages& v, TokensPages* total) {
  constexpr int kWarps = THREADS / 32;
  __shared__ TokensPages part[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto scan = [&](TokensPages& x) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, x.tokens, o);
      const int g = __shfl_up_sync(0xffffffffu, x.pages, o);
      if (lane >= o) {
        x.tokens += t;
        x.pages += g;
      }
    }
  };
  TokensPages x = v;
  scan(x);
  __syncthreads();   // `part` may still be read for the scan before
  if (lane == 31) part[warp] = x;
  __syncthreads();
  TokensPages y = lane < kWarps ? part[lane] : TokensPages{0, 0};
  scan(y);
  total->tokens = __shfl_sync(0xffffffffu, y.tokens, 31);
  total->pages = __shfl_sync(0xffffffffu, y.pages, 31);
  const long long t = __shfl_sync(0xffffffffu, y.tokens, (warp + 31) & 31);
  const int g = __shfl_sync(0xffffffffu, y.pages, (warp + 31) & 31);
  return {x.tokens - v.tokens + (warp > 0 ? t : 0), x.pages - v.pages + (warp > 0 ? g : 0)};
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

// Every CTA scans all lengths for itself (from L2, into shared memory), so that nothing is handed from CTA to CTA; then the
// CTAs share out the sequences, the new table entries and the token rows.  One CTA per SM and 16-byte stores where there are many
// rows (1.2 million rows of 301 prompts: 8.1 us, of which the scan 2.5; two CTAs per SM 10.3; eight rows one after the other, whose
// stores leave gaps, 8.7); one row per thread otherwise (a decode step of 64 sequences: 2.8 us, 4.9 with eight).
template <int THREADS, int ROWS, int GROUPS>
__global__ void __launch_bounds__(THREADS)
extend_kernel(const ExtendParams p) {
  extern __shared__ int shared[];
  int* cu = shared;                  // [S + 1] tokens in front of sequence s
  int* at = cu + p.S + 1;            // [S + 1] new pages in front of it
  int* past = at + p.S + 1;          // [S] its tokens so far
  int* begun = past + p.S;           // [S] the page that they have begun and not filled, on its way during the scan
  pdl_trigger();
  pdl_wait();
  const int cap = p.max_pages * p.P;
  const int per = ceil_div(p.S, THREADS);
  const int s0 = min(static_cast<int>(threadIdx.x) * per, p.S), s1 = min(s0 + per, p.S);
  const int used = p.free_used != nullptr ? max(p.free_used[0], 0) : 0;
  auto pages = [&](int have, int more) { return ceil_div(have + min(more, cap - have), p.P) - ceil_div(have, p.P); };

  TokensPages sum = {0, 0}, total;
  int page0 = -1;
  for (int s = s0; s < s1; ++s) {
    const int have = min(max(p.seq_lens[s], 0), cap), more = max(p.new_lens[s], 0);
    past[s] = have;
    cu[s] = more;      // until the prefix sums are known
    const int page = have / p.P;
    const int entry = have < cap && page * p.P < have ? p.table[static_cast<int64_t>(s) * p.stride + page] : -1;
    if (s == s0) page0 = entry; else begun[s] = entry;
    sum.tokens += more;
    sum.pages += pages(have, more);
  }
  TokensPages run = block_scan<THREADS>(sum, &total);
  if (total.tokens > p.T) {      // not all tokens fit: count the pages of those that do
    long long before = run.tokens;
    sum.pages = 0;
    for (int s = s0; s < s1; ++s) {
      const long long end = before + cu[s];
      cu[s] = static_cast<int>(min(end, static_cast<long long>(p.T)) - min(before, static_cast<long long>(p.T)));
      sum.pages += pages(past[s], cu[s]);
      before = end;
    }
    sum.tokens = 0;
    run.tokens = min(run.tokens, static_cast<long long>(p.T));
    TokensPages again;
    run.pages = block_scan<THREADS>(sum, &again).pages;
    total.tokens = p.T;
    total.pages = again.pages;
  }
  if (s0 < s1) begun[s0] = page0;
  for (int s = s0; s < s1; ++s) {
    const int more = cu[s];
    cu[s] = static_cast<int>(run.tokens);
    at[s] = run.pages;
    run.tokens += more;
    run.pages += pages(past[s], more);
  }
  if (threadIdx.x == 0) {
    cu[p.S] = static_cast<int>(total.tokens);
    at[p.S] = total.pages;
  }
  __syncthreads();

  const int me = blockIdx.x * THREADS + threadIdx.x, step = gridDim.x * THREADS;
  const int fresh = total.pages, n_new = static_cast<int>(total.tokens);
  auto free_page = [&](int k) {      // page k of those that are taken
    const long long f = static_cast<long long>(used) + k;
    return f >= 0 && f < p.n_free ? p.free_pages[f] : -1;
  };
  if (me == 0) p.free_used_out[0] = static_cast<int>(min(static_cast<long long>(used) + fresh, 0x7fffffffll));
  for (int s = me; s <= p.S; s += step) {
    p.cu_new[s] = cu[s];
    if (s < p.S) p.out_lens[s] = past[s] + min(cu[s + 1] - cu[s], cap - past[s]);
  }
  for (int k = me; k < fresh; k += step) {
    const int s = last_not_above(at, p.S, k);
    const int entry = ceil_div(past[s], p.P) + k - at[s];
    if (RBS_DBG_OK(entry >= 0 && entry < p.max_pages, p.status, kDbgExtendEntry)) p.table[static_cast<int64_t>(s) * p.stride + entry] = free_page(k);
  }
  const int lane = threadIdx.x & 31;
  for (long long warp_row = static_cast<long long>(me >> 5) * (32 * ROWS * GROUPS); warp_row < p.T; warp_row += static_cast<long long>(step) * ROWS * GROUPS) {
    int s = -1, behind = 0;      // the sequence of the last row, and the first row behind it
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
      const long long row64 = warp_row + (g * 32 + lane) * ROWS;
      if (row64 >= p.T) break;
      const int row0 = static_cast<int>(row64);
      int pos[ROWS], slot[ROWS];
      int page = -1, off = 0, index = 0, first = 0;
      bool good = false, begin = true;      // begin: position and page are worked out, not counted on
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const int row = row0 + i;
        pos[i] = 0;
        slot[i] = -1;
        if (row >= n_new) continue;
        if (row >= behind) {
          if (begin) s = last_not_above(cu, p.S, row);
          else do ++s; while (cu[s + 1] <= row);
          behind = cu[s + 1];
          begin = true;
        }
        bool look = begin;
        if (begin) {
          pos[i] = past[s] + row - cu[s];
          index = pos[i] / p.P;
          off = pos[i] - index * p.P;
          first = ceil_div(past[s], p.P);
          begin = false;
        } else {
          pos[i] = pos[i > 0 ? i - 1 : 0] + 1;
          if (++off == p.P) {
            off = 0;
            ++index;
            look = true;
          }
        }
        if (look) {
          page = -1;
          if (pos[i] < cap)      // the page that the sequence had begun, or a new one
            page = index < first ? begun[s] : free_page(at[s] + index - first);
          good = page >= 0 && page < p.n_pages;
        }
        if (good && pos[i] < cap) slot[i] = page * p.P + off;
      }
      if (ROWS == 4 && p.aligned && row0 <= p.T - ROWS) {      // row0 + ROWS may pass 31 bits
        *reinterpret_cast<int4*>(p.positions + row0) = make_int4(pos[0], pos[1 % ROWS], pos[2 % ROWS], pos[3 % ROWS]);
        *reinterpret_cast<int4*>(p.slots + row0) = make_int4(slot[0], slot[1 % ROWS], slot[2 % ROWS], slot[3 % ROWS]);
      } else {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
          if (row0 + i < p.T) {
            p.positions[row0 + i] = pos[i];
            p.slots[row0 + i] = slot[i];
          }
        }
      }
    }
  }
}

template <int THREADS, int ROWS, int GROUPS>
static rbs_status launch_extend(const ExtendParams& p, cudaStream_t stream) {
  const size_t smem = (4 * static_cast<size_t>(p.S) + 2) * sizeof(int);
  const rbs_status st = ensure_dynamic_smem(reinterpret_cast<const void*>(extend_kernel<THREADS, ROWS, GROUPS>), smem);
  if (st != RBS_OK) return st;
  const int groups = p.T > 0 ? (p.T - 1) / (ROWS * GROUPS) + 1 : 0, work = groups > p.S + 1 ? groups : p.S + 1;
  const int ctas = (work - 1) / THREADS + 1, most = sm_count();
  RBS_CUDA_OK(launch_pdl(extend_kernel<THREADS, ROWS, GROUPS>, static_cast<unsigned>(ctas < most ? ctas : most), 1, THREADS, smem, stream, p));
  return RBS_OK;
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
  p.status = debug_status();
  p.aligned = (reinterpret_cast<uintptr_t>(positions) | reinterpret_cast<uintptr_t>(slots)) % 16 == 0;
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  if (p.S < kExtendFew && p.T <= kExtendFew) return launch_extend<kExtendFew, 1, 1>(p, cs);
  return p.T <= sm_count() * kExtendThreads ? launch_extend<kExtendThreads, 1, 1>(p, cs) : launch_extend<kExtendThreads, kExtendRows, kExtendGroups>(p, cs);
}

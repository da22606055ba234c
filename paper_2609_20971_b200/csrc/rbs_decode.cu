// rbs_paged_decode: attention of one new token per sequence over a paged key/value cache.
// One pass over the keys and values with the running maximum and sum of the softmax.  The cache is read once: 512 bytes per
// token and KV head against 4 * 128 * G operations, far below what either kind of unit can do, so HBM is the bound and all
// else is arranged to keep loads in flight.
#include "rbs_common.cuh"

namespace rbs {

constexpr int kDecWarps = 4;            // warps of a CTA, each with keys of its own
constexpr int kDecKeys = 16;            // keys of a warp's tile
constexpr int kDecTile = kDecWarps * kDecKeys;
constexpr int kDecStages = 2;
constexpr int kDecWorkers = 148 * 3;    // CTAs, three per SM
constexpr int kDecTileBytes = kDecKeys * kHeadDim * 2;                 // K or V of a warp's tile
constexpr int kDecRow = kHeadDim + 4;                                  // floats of a row of O on its way between warps
constexpr int kDecOffO = kDecWarps * kDecStages * 2 * kDecTileBytes;   // two buffers [8 heads][kDecRow]
constexpr int kDecOffMl = kDecOffO + 2 * 8 * kDecRow * 4;              // [warp][head][m, l]

struct DecodeParams {
  const __nv_bfloat16* Q; int64_t qst, qsh;
  const __nv_bfloat16* K; int64_t kp, kt, kh;     // page, token, head strides
  const __nv_bfloat16* V; int64_t vp, vt, vh;
  __nv_bfloat16* O; int64_t ost, osh;
  float* lse;                                     // nullable
  const int* table;
  const int* lens;
  int S, Hq, Hkv, G, P, n_pages, max_pages, stride;
  int cuts, gh;    // a KV head's G query heads are `cuts` items of up to gh (<= 16) heads
  int items;       // Hkv * cuts
  float scale_log2;
  float* part_o;   // [slot][HT * 8][128] sums of parts of items
  float2* part_ml; // [slot][HT * 8] their maxima (log2 units) and normalisers
  int4* cut;       // [worker] the item that begins in its share and goes on: sequence (-1: none), first head | heads << 24,
                   // slot of its first part, worker of its last part
};

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

// The running softmax of up to 8 * HT heads over the keys that a warp has seen.  Keys are the M side of both products:
//   S^T [16 keys x 8 heads] = K Q^T,   O^T [128 x 8 heads] += V^T P^T
// so that 8 heads fill the N side.  Lane (g, t) = (lane / 4, lane % 4) has heads 2t, 2t + 1 of each group of 8: of S^T keys g and
// g + 8, of O^T elements 16 j + g and 16 j + g + 8.
template <int HT>
struct Softmax {
  uint32_t q[HT][16];     // Q^T, the B operand of the eight steps over the head dimension
  float o[HT][8][4];
  float m[HT][2], l[HT][2];   // m in units of log2; l over this lane's keys only

  __device__ __forceinline__ void start(const __nv_bfloat16* Q, int64_t qsh, int heads) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
    for (int n = 0; n < HT; ++n) {
      const int h = 8 * n + g;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        q[n][i] = h < heads ? *reinterpret_cast<const uint32_t*>(Q + h * qsh + 8 * i + 2 * t) : 0u;
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][j][i] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
    }
  }

  // Scores of 16 keys; `valid`: a bit per key.  p: their probabilities against the new maximum, as the B operand of P V
  // (rounded to bf16, at most 2^-8 relative each; l sums them unrounded, so that lse does not see the rounding).
  __device__ __forceinline__ void scores(uint32_t ktile, uint32_t valid, float scale_log2, uint32_t (&p)[HT][2]) {
    const int lane = threadIdx.x & 31, g = lane >> 2;
    float c[HT][4];
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) c[n][i] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t a[4];
      ldmatrix_x4(a[0], a[1], a[2], a[3], ktile + tile_off(lane & 15, 2 * k + (lane >> 4)));
#pragma unroll
      for (int n = 0; n < HT; ++n) mma_bf16_16816(c[n], a, q[n][2 * k], q[n][2 * k + 1]);
    }
    const bool lo = (valid >> g) & 1, hi = (valid >> (g + 8)) & 1;
#pragma unroll
    for (int n = 0; n < HT; ++n) {
      float top[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) c[n][i] = (i < 2 ? lo : hi) ? c[n][i] * scale_log2 : -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[i] = fmaxf(c[n][i], c[n][i + 2]);
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], s));
        top[i] = fmaxf(top[i], m[n][i]);
        const float base = top[i] == -INFINITY ? 0.f : top[i];   // nothing seen yet: no inf - inf
        const float fade = fast_exp2(m[n][i] - base);
        m[n][i] = top[i];
        c[n][i] = fast_exp2(c[n][i] - base);
        c[n][i + 2] = fast_exp2(c[n][i + 2] - base);
        l[n][i] = l[n][i] * fade + c[n][i] + c[n][i + 2];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          o[n][j][i] *= fade;
          o[n][j][i + 2] *= fade;
        }
      }
      p[n][0] = transpose_8x8(pack_bf16(c[n][0], c[n][1]));
      p[n][1] = transpose_8x8(pack_bf16(c[n][2], c[n][3]));
    }
  }

  __device__ __forceinline__ void values(uint32_t vtile, const uint32_t (&p)[HT][2]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t a[4];
      ldmatrix_x4_trans(a[0], a[1], a[2], a[3], vtile + tile_off((lane & 7) + (lane >> 4) * 8, 2 * j + ((lane >> 3) & 1)));
#pragma unroll
      for (int n = 0; n < HT; ++n) mma_bf16_16816(o[n][j], a, p[n][0], p[n][1]);
    }
  }
};

// The sums of a CTA's warps become one: all to the largest maximum, then (0 + 2) + (1 + 3).  `whole`: the item is complete, its
// output is written; otherwise the sum goes to the workspace.
template <int HT>
__device__ __forceinline__ void finish_item(const DecodeParams& p, Softmax<HT>& sm, float* part_o, float* part_ml, int s, int h0, int heads,
                                            bool whole, int slot) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int k = 0; k < HT; ++k) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) sm.l[k][i] += __shfl_xor_sync(0xffffffffu, sm.l[k][i], x);
      if (g == 0) {
        part_ml[(warp * 8 + 2 * t + i) * 2] = sm.m[k][i];
        part_ml[(warp * 8 + 2 * t + i) * 2 + 1] = sm.l[k][i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) top = fmaxf(top, part_ml[(w * 8 + 2 * t + i) * 2]);
      const float f = fast_exp2(sm.m[k][i] - (top == -INFINITY ? 0.f : top));
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        sm.o[k][j][i] *= f;
        sm.o[k][j][i + 2] *= f;
      }
    }
    float* mine = part_o + (warp & 1) * 8 * kDecRow;
#pragma unroll
    for (int round = 1; round >= 0; --round) {
      if (warp >> 1 == round) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float* x = mine + (2 * t + (i & 1)) * kDecRow + 16 * j + g + (i >> 1) * 8;
            *x = round == 1 ? sm.o[k][j][i] : *x + sm.o[k][j][i];
          }
      }
      __syncthreads();
    }
    // a thread per eight elements of a head
    const int h = threadIdx.x >> 4, c = (threadIdx.x & 15) * 8;
    if (8 * k + h < heads) {
      float top = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) top = fmaxf(top, part_ml[(w * 8 + h) * 2]);
      const float base = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < kDecWarps; ++w) sum += part_ml[(w * 8 + h) * 2 + 1] * fast_exp2(part_ml[(w * 8 + h) * 2] - base);
      const float4* x = reinterpret_cast<const float4*>(part_o + h * kDecRow + c);
      const float4* y = reinterpret_cast<const float4*>(part_o + (8 + h) * kDecRow + c);
      float4 a = x[0], b = x[1];
      a.x += y[0].x; a.y += y[0].y; a.z += y[0].z; a.w += y[0].w;
      b.x += y[1].x; b.y += y[1].y; b.z += y[1].z; b.w += y[1].w;
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        const int hq = h0 + 8 * k + h;
        *reinterpret_cast<uint4*>(p.O + s * p.ost + hq * p.osh + c) =
            make_uint4(pack_bf16(a.x * inv, a.y * inv), pack_bf16(a.z * inv, a.w * inv), pack_bf16(b.x * inv, b.y * inv), pack_bf16(b.z * inv, b.w * inv));
        if (c == 0 && p.lse != nullptr)
          p.lse[static_cast<int64_t>(s) * p.Hq + hq] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.6931471805599453f;
      } else {
        const int64_t row = static_cast<int64_t>(slot) * (HT * 8) + 8 * k + h;
        float4* o = reinterpret_cast<float4*>(p.part_o + row * kHeadDim + c);
        o[0] = a;
        o[1] = b;
        if (c == 0) p.part_ml[row] = make_float2(top, sum);
      }
    }
    __syncthreads();
  }
}

// A place in the order of all work: sequence by sequence, in it item by item (KV head, cut of its query heads), in it tile by
// tile of kDecTile tokens.  A sequence has at least one tile, so that its outputs are written even if it has no token.
struct Place {
  int s, item, tile, n, len, next_len;   // n: tiles of an item of sequence s; next_len: length of sequence s + 1
};

__device__ __forceinline__ int clamped_len(const DecodeParams& p, int s) {
  return s < p.S ? min(max(p.lens[s], 0), p.max_pages * p.P) : 0;
}
__device__ __forceinline__ int tiles_of(int len) { return len <= kDecTile ? 1 : (len - 1) / kDecTile + 1; }

// One tile on.  True if it was the last of its item.
__device__ __forceinline__ bool step(const DecodeParams& p, Place& at) {
  if (++at.tile < at.n) return false;
  at.tile = 0;
  if (++at.item == p.items) {
    at.item = 0;
    ++at.s;
    at.len = at.next_len;
    at.n = tiles_of(at.len);
    at.next_len = clamped_len(p, at.s + 1);
  }
  return true;
}

// The page-table entry of this lane's row of a warp's 16 keys (lanes 0 - 15) or values (lanes 16 - 31, the same rows).
struct Lookup {
  int page, off, hk;
};
__device__ __forceinline__ Lookup look_up(const DecodeParams& p, const Place& at, int warp) {
  const int pos = at.tile * kDecTile + warp * kDecKeys + (threadIdx.x & 15);
  Lookup r = {-1, 0, at.item / p.cuts};
  if (pos < at.len) {
    const int index = pos / p.P;
    r.off = pos - index * p.P;
    r.page = p.table[static_cast<int64_t>(at.s) * p.stride + index];
  }
  return r;
}

// Which of the 16 keys there are, a bit each, and where this lane's row starts.
__device__ __forceinline__ uint32_t row_offset(const DecodeParams& p, const Lookup& r, int64_t& at) {
  const bool there = r.page >= 0 && r.page < p.n_pages;
  at = 0;
  if (there)
    at = (threadIdx.x & 16) ? r.page * p.vp + r.off * p.vt + r.hk * p.vh : r.page * p.kp + r.off * p.kt + r.hk * p.kh;
  return __ballot_sync(0xffffffffu, there) & 0xffffu;
}

// Starts the copy of 16 rows, whose offsets lanes first .. first + 15 hold; rows that are not there become zeros, so that no
// stale page contents reach a product.
__device__ __forceinline__ void copy_rows(const __nv_bfloat16* base, int64_t at, int first, uint32_t valid, uint32_t tile) {
  const int lane = threadIdx.x & 31, chunk = lane & 15, half = lane >> 4;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = 2 * i + half;
    const int64_t from = __shfl_sync(0xffffffffu, at, row + first);
    cp_async16_zfill(tile + tile_off(row, chunk), base + from + chunk * 8, (valid >> row) & 1);
  }
  cp_async_commit();
}

// Where tile t of all `total` tiles falls when `workers` share them in order, and where worker w's share begins.
__device__ __forceinline__ int worker_of(long long t, long long total, int workers) {
  return static_cast<int>(((t + 1) * workers - 1) / total);
}
__device__ __forceinline__ long long share_begin(int w, long long total, int workers) { return total * w / workers; }

// Sum over the CTA of one value per thread and this thread's exclusive prefix sum.
__device__ __forceinline__ long long scan_cta(long long v, long long* part, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    before += w < warp ? part[w] : 0;
    all += part[w];
  }
  *total = all;
  return before + x - v;
}

// Finds the total number of tiles and the place where this CTA's share of them begins.  A chunk of four lengths per thread
// at a time; up to 512 sequences are one chunk and are read once.
__device__ __forceinline__ void find_share(const DecodeParams& p, Place& at, long long& begin, long long& end, int& workers,
                                           long long& all_tiles) {
  __shared__ long long part[kDecWarps];
  __shared__ int found[2];
  constexpr int kChunk = kDecWarps * 32 * 4;
  int n[4];
  auto load = [&](int base) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = base + threadIdx.x * 4 + i;
      n[i] = s < p.S ? tiles_of(clamped_len(p, s)) : 0;
      sum += n[i];
    }
    return static_cast<long long>(sum);
  };
  long long total = 0, sum = 0, before = 0;
  if (p.S <= kChunk) {
    before = scan_cta(load(0), part, &total);
  } else {
    for (int base = 0; base < p.S; base += kChunk) sum += load(base);
    scan_cta(sum, part, &total);
  }
  all_tiles = total * p.items;
  workers = static_cast<int>(min(static_cast<long long>(kDecWorkers), all_tiles));
  const int w = blockIdx.x;
  begin = w < workers ? share_begin(w, all_tiles, workers) : all_tiles;
  end = w < workers ? share_begin(w + 1, all_tiles, workers) : all_tiles;
  if (begin == end) return;
  const long long in_seqs = begin / p.items;      // tiles of one item's worth of sequences in front of the share
  long long base_tiles = 0;
  for (int base = 0; base < p.S; base += kChunk) {
    if (p.S > kChunk) before = scan_cta(load(base), part, &total);
    long long first = base_tiles + before;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (first <= in_seqs && in_seqs < first + n[i]) {
        found[0] = base + threadIdx.x * 4 + i;
        found[1] = static_cast<int>(begin - first * p.items);      // the share's first tile within the sequence's
      }
      first += n[i];
    }
    base_tiles += total;
    if (in_seqs < base_tiles) break;
  }
  __syncthreads();
  at.s = found[0];
  at.len = clamped_len(p, at.s);
  at.next_len = clamped_len(p, at.s + 1);
  at.n = tiles_of(at.len);
  at.item = found[1] / at.n;
  at.tile = found[1] % at.n;
}

// One CTA per worker: an equal share of the tiles of all sequences, in order.  Items inside the share are finished here;
// the first and the last one may reach into other shares: their sums go to the workspace (slot 2 w for the first item
// of the share, 2 w + 1 for the last one), and the worker in whose share a cut item begins says in whole[w] which workers follow.
template <int HT>
__global__ void __launch_bounds__(kDecWarps * 32, 3)
decode_kernel(const DecodeParams p) {
  extern __shared__ __align__(128) unsigned char smem[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
  const uint32_t tiles = smem_u32(smem) + warp * kDecStages * 2 * kDecTileBytes;
  float* part_o = reinterpret_cast<float*>(smem + kDecOffO);
  float* part_ml = reinterpret_cast<float*>(smem + kDecOffMl);
  pdl_trigger();
  pdl_wait();
  Place at;
  long long begin, end, total;
  int workers;
  const int w = blockIdx.x;
  find_share(p, at, begin, end, workers, total);
  if (begin == end) {
    if (threadIdx.x == 0) p.cut[w] = make_int4(-1, 0, 0, 0);
    return;
  }
  const int count = static_cast<int>(end - begin);

  // consumer's side: the item that is being summed
  int s = at.s, item = at.item, done = 0, item_begin = at.tile == 0 ? 0 : -1;   // item_begin: in tiles of the share, -1 before it
  bool first_item = true;

  // the pipeline: tiles i + 2 on their way while tile i is worked on, the table entries of tile i + 3 as well
  Lookup look = look_up(p, at, warp);
  int ahead = 0;
  auto info = [&](uint32_t valid, bool last) { return valid | (last ? 0x10000u : 0u); };
  uint32_t queue[kDecStages];
  int64_t from;
  auto begin_keys = [&](uint32_t kt) {      // returns the tile's word
    uint32_t word = 0;
    if (ahead < count) {
      const uint32_t valid = row_offset(p, look, from);
      copy_rows(p.K, from, 0, valid, kt);
      ++ahead;
      const bool last = step(p, at);
      if (ahead < count) look = look_up(p, at, warp);
      word = info(valid, last);
    } else {
      cp_async_commit();
    }
    return word;
  };
  auto begin_values = [&](uint32_t vt, uint32_t word, bool there) {
    if (there) copy_rows(p.V, from, 16, word & 0xffffu, vt);
    else cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kDecStages; ++i) {
    const bool there = ahead < count;
    queue[i] = begin_keys(tiles + 2 * i * kDecTileBytes);
    begin_values(tiles + (2 * i + 1) * kDecTileBytes, queue[i], there);
  }

  Softmax<HT> sm;
  int h0 = 0, heads = 0;
  auto open_item = [&]() {
    const int hk = item / p.cuts, c = item - hk * p.cuts;
    h0 = hk * p.G + c * p.gh;
    heads = min(p.gh, p.G - c * p.gh);
    sm.start(p.Q + s * p.qst + h0 * p.qsh, p.qsh, heads);
  };
  open_item();
  for (; done < count; ++done) {
    const uint32_t kt = tiles + 2 * (done % kDecStages) * kDecTileBytes, vt = kt + kDecTileBytes;
    const uint32_t word = queue[0];
    queue[0] = queue[1];
    uint32_t pr[HT][2];
    cp_async_wait<2 * kDecStages - 1>();
    __syncwarp();
    sm.scores(kt, word & 0xffffu, p.scale_log2, pr);
    __syncwarp();
    const bool more = ahead < count;
    queue[1] = begin_keys(kt);
    cp_async_wait<2 * kDecStages - 1>();
    __syncwarp();
    sm.values(vt, pr);
    __syncwarp();
    begin_values(vt, queue[1], more);

    const bool last = word & 0x10000u;
    if (!last && done + 1 < count) continue;
    // the end of the item, or of the share
    const bool whole = last && item_begin >= 0;
    finish_item<HT>(p, sm, part_o, part_ml, s, h0, heads, whole, 2 * w + (first_item ? 0 : 1));
    if (done + 1 == count) {
      if (threadIdx.x == 0) {
        int4 c = make_int4(-1, 0, 0, 0);
        if (!last && item_begin >= 0)      // the item begins here and goes on; `at` stands inside it
          c = make_int4(s, h0 | heads << 24, 2 * w + (first_item ? 0 : 1), worker_of(begin + item_begin + at.n - 1, total, workers));
        p.cut[w] = c;
      }
      break;
    }
    first_item = false;
    item_begin = done + 1;
    if (++item == p.items) { item = 0; ++s; }
    open_item();
  }
}

// Joins the parts of the item that begins in worker w's share and goes on behind it: one CTA per worker and head, a quarter of
// the parts per warp, four elements per lane.  The order depends on the lengths alone.
template <int HT>
__global__ void __launch_bounds__(128)
join_kernel(const DecodeParams p) {
  __shared__ float4 sums[3][32];
  __shared__ float norm[3];
  pdl_trigger();
  pdl_wait();
  const int w = blockIdx.x, head = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int4 c = p.cut[w];
  if (c.x < 0 || head >= c.y >> 24) return;
  const int n = c.w - w + 1;      // part 0 in slot c.z, part i in slot 2 (w + i)
  auto ml_of = [&](int i) { return p.part_ml[(i == 0 ? c.z : 2 * (w + i)) * (HT * 8) + head]; };
  float top = -INFINITY;
  for (int i = lane; i < n; i += 32) top = fmaxf(top, ml_of(i).x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float base = top == -INFINITY ? 0.f : top;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  float sum = 0.f;
#pragma unroll 4
  for (int i = warp; i < n; i += 4) {
    const float2 ml = ml_of(i);
    const float f = fast_exp2(ml.x - base);
    const float4 o = *reinterpret_cast<const float4*>(
        p.part_o + (static_cast<int64_t>(i == 0 ? c.z : 2 * (w + i)) * (HT * 8) + head) * kHeadDim + 4 * lane);
    sum = fmaf(ml.y, f, sum);
    acc.x = fmaf(o.x, f, acc.x); acc.y = fmaf(o.y, f, acc.y); acc.z = fmaf(o.z, f, acc.z); acc.w = fmaf(o.w, f, acc.w);
  }
  if (warp > 0) {
    sums[warp - 1][lane] = acc;
    if (lane == 0) norm[warp - 1] = sum;
  }
  __syncthreads();
  if (warp > 0) return;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const float4 o = sums[i][lane];
    acc.x += o.x; acc.y += o.y; acc.z += o.z; acc.w += o.w;
    sum += norm[i];
  }
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
  const int h = (c.y & 0xffffff) + head;
  *reinterpret_cast<uint2*>(p.O + c.x * p.ost + h * p.osh + 4 * lane) =
      make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
  if (lane == 0 && p.lse != nullptr)
    p.lse[static_cast<int64_t>(c.x) * p.Hq + h] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.6931471805599453f;
}

struct DecodeWorkspace {
  size_t off_o, off_ml, off_cut, bytes;
};
static DecodeWorkspace decode_workspace(int G) {
  const size_t rows = static_cast<size_t>(2 * kDecWorkers) * (G <= 8 ? 8 : 16);
  DecodeWorkspace w;
  size_t off = 0;
  w.off_o = off; off = align_up(off + rows * kHeadDim * sizeof(float), 256);
  w.off_ml = off; off = align_up(off + rows * sizeof(float2), 256);
  w.off_cut = off; off = align_up(off + kDecWorkers * sizeof(int4), 256);
  w.bytes = off;
  return w;
}

}  // namespace rbs

extern "C" size_t rbs_paged_decode_workspace_bytes(const rbs_paged_shape* shape) {
  using namespace rbs;
  if (check_paged_table(shape) != RBS_OK || check_paged_cache(shape) != RBS_OK) return 0;
  return decode_workspace(shape->n_q_heads / shape->n_kv_heads).bytes;
}

extern "C" rbs_status rbs_paged_decode(const rbs_paged_shape* shape, rbs_tensor Q, rbs_tensor k_cache, rbs_tensor v_cache,
                                       const int* block_table, const int* seq_lens, rbs_tensor O, float* lse,
                                       float softmax_scale, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace rbs;
  NvtxRange range("rbs_paged_decode");
  rbs_status st = check_paged_table(shape);
  if (st != RBS_OK || (st = check_paged_cache(shape)) != RBS_OK) return st;
  if (block_table == nullptr || seq_lens == nullptr || !(fabsf(softmax_scale) <= 3.4028235e38f)) return RBS_ERR_INVALID_ARG;
  Q.stride_batch = O.stride_batch = 0;
  if ((st = check_tensor(Q)) != RBS_OK || (st = check_tensor(O)) != RBS_OK || (st = check_tensor(k_cache)) != RBS_OK ||
      (st = check_tensor(v_cache)) != RBS_OK)
    return st;
  DecodeParams p = {};
  p.Q = static_cast<const __nv_bfloat16*>(Q.ptr); p.qst = Q.stride_token; p.qsh = Q.stride_head;
  p.K = static_cast<const __nv_bfloat16*>(k_cache.ptr); p.kp = k_cache.stride_batch; p.kt = k_cache.stride_token; p.kh = k_cache.stride_head;
  p.V = static_cast<const __nv_bfloat16*>(v_cache.ptr); p.vp = v_cache.stride_batch; p.vt = v_cache.stride_token; p.vh = v_cache.stride_head;
  p.O = static_cast<__nv_bfloat16*>(O.ptr); p.ost = O.stride_token; p.osh = O.stride_head;
  p.lse = lse; p.table = block_table; p.lens = seq_lens;
  p.S = shape->n_seqs; p.Hq = shape->n_q_heads; p.Hkv = shape->n_kv_heads; p.G = p.Hq / p.Hkv;
  p.P = shape->page_size; p.n_pages = shape->n_pages; p.max_pages = shape->max_pages; p.stride = shape->table_stride;
  p.cuts = (p.G + 15) / 16;
  p.gh = (p.G + p.cuts - 1) / p.cuts;
  p.items = p.Hkv * p.cuts;
  if (p.Hq >= 1 << 24) return RBS_ERR_UNSUPPORTED;
  const DecodeWorkspace ws = decode_workspace(p.G);
  if (workspace == nullptr || workspace_bytes < ws.bytes || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return RBS_ERR_WORKSPACE;
  unsigned char* base = static_cast<unsigned char*>(workspace);
  p.part_o = reinterpret_cast<float*>(base + ws.off_o);
  p.part_ml = reinterpret_cast<float2*>(base + ws.off_ml);
  p.cut = reinterpret_cast<int4*>(base + ws.off_cut);
  const float scale = softmax_scale == 0.f ? 1.0f / sqrtf(static_cast<float>(kHeadDim)) : softmax_scale;
  p.scale_log2 = scale * kLog2e;
  auto* kernel = p.gh <= 8 ? decode_kernel<1> : decode_kernel<2>;
  const size_t smem = kDecOffMl + kDecWarps * 8 * 2 * sizeof(float);
  if ((st = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem)) != RBS_OK) return st;
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  RBS_CUDA_OK(launch_pdl(kernel, kDecWorkers, 1, kDecWarps * 32, smem, cs, p));
  RBS_CUDA_OK(launch_pdl(p.gh <= 8 ? join_kernel<1> : join_kernel<2>, kDecWorkers, p.gh, 128, 0, cs, p));
  return RBS_OK;
}

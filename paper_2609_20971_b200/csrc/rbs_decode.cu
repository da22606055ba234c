// rbs_paged_decode: attention of one new token per sequence over a paged key/value cache.
// One pass over the keys and values with the running maximum and sum of the softmax.  The cache is read once: 512 bytes per
// token and KV head against 4 * 128 * G operations, far below what either kind of unit can do, so HBM is the bound for groups of up
// to 8 heads (64 sequences of 64 heads: 211 us, 6.5 TB/s) and all else is arranged to keep loads in flight.  With 16 heads to
// a KV head the products of a warp take longer than its loads (257 us for the same bytes); larger groups are cut, and
// each cut reads the cache anew (32 heads: 65 us where 16 take 40).
//
// The work of all sequences stands in one order -- sequence by sequence, item by item (KV head, cut of its query heads), tile by
// tile of 16 tokens -- and is cut into equal shares, one per warp, whatever the lengths are.  A warp works alone: its own
// ring of K and V tiles in shared memory, items that lie inside its share finished from its registers.  Only the first and
// the last item of a share can be in pieces; pieces of one item are joined by the thread block at its end, and by a second
// kernel where an item goes on in other thread blocks.  All joins are in the order of the tokens.
#include "rbs_common.cuh"
#include "rbs_sm100.cuh"

namespace rbs {

constexpr int kDecWarps = 4;
constexpr int kDecWave = 148 * 3;       // CTAs that are resident at a time, three per SM
constexpr int kDecRest = 148 * 3 / 2;   // CTAs behind them, for a tenth of the work of large calls
constexpr int kDecCtas = kDecWave + kDecRest;
constexpr int kDecRestTiles = 32;       // where a warp's share is at least that much
constexpr int kDecKeys = 16;            // tokens of a tile
constexpr int kDecStages = 2;
constexpr int kDecTileBytes = kDecKeys * kHeadDim * 2;                 // K or V of a tile
constexpr int kDecRing = kDecStages * 2 * kDecTileBytes;               // of a warp
constexpr int kDecRow = kHeadDim + 4;                                  // floats of a row of O in shared memory
constexpr int kDecSlots = kDecCtas * (2 + kDecWarps - 1);
constexpr int kDecItemCost = 2;         // what the end of an item costs a warp, in tiles: shares are equal with it counted
constexpr float kDecSlack = 8.f;        // log2 units by which a score may pass the maximum in use

struct DecodeParams {
  const __nv_bfloat16* Q; int64_t qst, qsh;
  const __nv_bfloat16* K; int64_t kp, kt, kh;     // page, token, head strides
  const __nv_bfloat16* V; int64_t vp, vt, vh;
  __nv_bfloat16* O; int64_t ost, osh;
  float* lse;                                     // nullable
  const int* table;
  const int* lens;
  int S, Hq, Hkv, G, P, n_pages, max_pages, stride;
  int page_tiles;  // tiles per page; 0: a tile may lie in several pages
  int cuts, gh;    // a KV head's G query heads are `cuts` items of up to gh (<= 16) heads
  int items;       // Hkv * cuts
  float scale_log2;
  // Pieces of items, [slot][HT * 8 heads]: slot 2 c: of the item that CTA c found begun, 2 c + 1: of the one that it left unfinished,
  // 2 CTAs + 3 c + w - 1: of the item that warp w > 0 of CTA c found begun and finished
  float* part_o;   // [..][128] sums
  float2* part_ml; // maxima in use (log2 units) and normalisers
  unsigned int* status;   // of the debug build's checks
  int4* found;     // [CTA] the item that its share finds begun: sequence (-1: none), first head | heads << 24, CTAs of its begin and end
};

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// A bf16 number below x > 0, by 2^-9 to 2^-6 of x, as fp32 bits; 0 for 0, NaN for NaN.  What is left of x in two steps has at most 10
// bits and is positive.  (Below some 2^-110 the last part is lost: an infinite value with a weight that small gives NaN, as it does
// where the weight itself underflows.)
__device__ __forceinline__ uint32_t bf16_below(float x) {
  return static_cast<uint32_t>(max(__float_as_int(x) - 0x8000, 0)) & 0xffff0000u;
}
// x += y of two neighbouring numbers, in one instruction
__device__ __forceinline__ void add_pair(float* x, const float* y) {
  f2_unpack(f2_add(f2_pack(x[0], x[1]), f2_pack(y[0], y[1])), x[0], x[1]);
}
// The value that exponentials are taken against: nothing seen yet must not give inf - inf.
__device__ __forceinline__ float exp_base(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (exp_base(m) + log2f(l)) * 0.6931471805599453f; }

// Q^T of up to 8 * HT heads, the B operand of the eight steps over the head dimension.
template <int HT>
struct Queries {
  uint32_t q[HT][16];
  __device__ __forceinline__ void load(const __nv_bfloat16* Q, int64_t qsh, int heads) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
    for (int n = 0; n < HT; ++n) {
      const __nv_bfloat16* row = Q + (8 * n + g) * qsh + 2 * t;
#pragma unroll
      for (int i = 0; i < 16; ++i) q[n][i] = 8 * n + g < heads ? *reinterpret_cast<const uint32_t*>(row + 8 * i) : 0u;
    }
  }
};

// The running softmax of up to 8 * HT heads over the keys that a warp has seen.  Keys are the M side of both products:
//   S^T [16 keys x 8 heads] = K Q^T,   O^T [128 x 8 heads] += V^T P^T
// so that 8 heads fill the N side.  Lane (g, t) = (lane / 4, lane % 4) has heads 2t, 2t + 1 of each group of 8: of S^T keys g and
// g + 8, of O^T elements 16 j + g and 16 j + g + 8.
template <int HT>
struct Softmax {
  float o[HT][8][4];
  float m[HT][2], l[HT][2];   // maximum in use, log2 units; sum over this lane's keys

  __device__ __forceinline__ void start() {
#pragma unroll
    for (int n = 0; n < HT; ++n) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][j][i] = 0.f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
    }
  }

  // Scores of 16 keys and, in c, their probabilities against the maximum in use; `valid`: a bit per key.
  // The maximum moves only when a score passes it by kDecSlack: probabilities of up to 2^8 round no worse, and a tile that
  // leaves it alone has no exchange between lanes and no rescaling.
  __device__ __forceinline__ void scores(const Queries<HT>& q, uint32_t ktile, uint32_t valid, float scale_log2, float (&c)[HT][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2;
    float c2[HT][4];
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) c[n][i] = c2[n][i] = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {      // two sums of four steps: half as many roundings in a row
      uint32_t a[4];
      ldmatrix_x4(a[0], a[1], a[2], a[3], ktile + tile_off(lane & 15, 2 * k + (lane >> 4)));
#pragma unroll
      for (int n = 0; n < HT; ++n) mma_bf16_16816(k & 1 ? c2[n] : c[n], a, q.q[n][2 * k], q.q[n][2 * k + 1]);
    }
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 4; i += 2) add_pair(c[n] + i, c2[n] + i);
    const bool lo = (valid >> g) & 1, hi = (valid >> (g + 8)) & 1;
    bool move = false;
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        c[n][i] = lo ? c[n][i] * scale_log2 : -INFINITY;
        c[n][i + 2] = hi ? c[n][i + 2] * scale_log2 : -INFINITY;
        move |= fmaxf(c[n][i], c[n][i + 2]) > m[n][i] + kDecSlack;
      }
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int n = 0; n < HT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float top = fmaxf(c[n][i], c[n][i + 2]);
#pragma unroll
          for (int s = 4; s < 32; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
          top = fmaxf(top, m[n][i]);
          const float fade = fast_exp2(m[n][i] - exp_base(top));
          m[n][i] = top;
          l[n][i] *= fade;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            o[n][j][i] *= fade;
            o[n][j][i + 2] *= fade;
          }
        }
    }
#pragma unroll
    for (int n = 0; n < HT; ++n) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float base = exp_base(m[n][i]);
        c[n][i] = fast_exp2(c[n][i] - base);
        c[n][i + 2] = fast_exp2(c[n][i + 2] - base);
        l[n][i] += c[n][i] + c[n][i + 2];
      }
    }
  }

  // Adds P V of 16 keys.  A probability goes into the product as three bf16 numbers, which together are the fp32 number, off by 2^-24
  // of it, and none of which is zero or below: an infinite value stays what it is in each of the three products.
  // The sums of the product drop bits where a plain addition rounds, and over the hundred tiles of a share those would add up in
  // one direction: a tile is summed from zero, the smallest parts first, and added by itself.  Against 64 bits rounded to bf16,
  // 2-norm, 64 sequences of 64 heads: two bf16 numbers and one running sum 1.2e-4 (207.9 us), three numbers the same (210.2),
  // with tiles summed by themselves 3.9e-5 (212.7), with the scores' product in two sums as well 2.9e-5 (212.9); plain fp32
  // operations 5.8e-5.
  // Products of four times 16 elements go side by side, because the three of a sum wait for each other: 17 sequences with pages of 24
  // 16.75 -> 16.25 us, 64 sequences of 128 heads in groups of 16 272 -> 257 (232 with two numbers and one running sum: there the
  // products and their instructions count, not HBM).
  __device__ __forceinline__ void values(uint32_t vtile, const float (&c)[HT][4]) {
    const int lane = threadIdx.x & 31;
    uint32_t p[HT][6];
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = c[n][2 * i], y = c[n][2 * i + 1];
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          const uint32_t px = bf16_below(x), py = bf16_below(y);
          p[n][2 * part + i] = transpose_8x8(__byte_perm(px, py, 0x7632));
          x -= __uint_as_float(px);
          y -= __uint_as_float(py);
        }
        p[n][4 + i] = transpose_8x8(pack_bf16(x, y));
      }
    constexpr int kSide = 4;
#pragma unroll
    for (int j = 0; j < 8; j += kSide) {
      uint32_t a[kSide][4];
      float sum[kSide][HT][4] = {};
#pragma unroll
      for (int b = 0; b < kSide; ++b)
        ldmatrix_x4_trans(a[b][0], a[b][1], a[b][2], a[b][3], vtile + tile_off((lane & 7) + (lane >> 4) * 8, 2 * (j + b) + ((lane >> 3) & 1)));
#pragma unroll
      for (int part = 4; part >= 0; part -= 2)
#pragma unroll
        for (int b = 0; b < kSide; ++b)
#pragma unroll
          for (int n = 0; n < HT; ++n) mma_bf16_16816(sum[b][n], a[b], p[n][part], p[n][part + 1]);
#pragma unroll
      for (int b = 0; b < kSide; ++b)
#pragma unroll
        for (int n = 0; n < HT; ++n)
#pragma unroll
          for (int i = 0; i < 4; i += 2) add_pair(o[n][j + b] + i, sum[b][n] + i);
    }
  }

  // l becomes the sum over all keys of the warp
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int s = 4; s < 32; s <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], s);
  }
  // O and lse of a whole item
  __device__ __forceinline__ void write(const DecodeParams& p, int s, int h0, int heads) const {
    if (!RBS_DBG_OK(s >= 0 && s < p.S && h0 >= 0 && heads > 0 && h0 + heads <= p.Hq, p.status, kDbgDecodeRow)) return;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < HT; ++n) {
      float inv[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        inv[i] = l[n][i] == 0.f ? 0.f : 1.0f / l[n][i];
        const int h = 8 * n + 2 * t + i;
        if (p.lse != nullptr && g == 0 && h < heads) p.lse[static_cast<int64_t>(s) * p.Hq + h0 + h] = lse_of(m[n][i], l[n][i]);
      }
      __nv_bfloat16* row = p.O + s * p.ost + (h0 + 8 * n + g) * p.osh + 2 * t;      // behind the transposition
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t x = transpose_8x8(pack_bf16(o[n][j][2 * i] * inv[0], o[n][j][2 * i + 1] * inv[1]));
          if (8 * n + g < heads) *reinterpret_cast<uint32_t*>(row + 16 * j + 8 * i) = x;
        }
    }
  }
  // a piece of an item: rows of `stride` floats, maxima and normalisers
  __device__ __forceinline__ void put(float* rows, int stride, float2* ml) const {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int h = 8 * n + 2 * t + i;
        if (g == 0) ml[h] = make_float2(m[n][i], l[n][i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          rows[h * stride + 16 * j + g] = o[n][j][i];
          rows[h * stride + 16 * j + g + 8] = o[n][j][i + 2];
        }
      }
  }
};

// A place in the order of all work.  A sequence has at least one tile per item, so that its outputs are written even if it has
// no token.
struct Place {
  int s, item, tile, n, len, next_len;   // n: tiles of an item of sequence s; next_len: length of sequence s + 1, as it was read
  int hk, cut;                           // of the item
  int page, in_page;                     // of the tile: entry of the table row, tile within the page (where pages hold whole tiles)
  unsigned unit;                         // of all work (see Cuts)
};

__device__ __forceinline__ int read_len(const DecodeParams& p, int s) { return s < p.S ? p.lens[s] : 0; }
__device__ __forceinline__ int clamped(const DecodeParams& p, int len) { return min(max(len, 0), p.max_pages * p.P); }
__device__ __forceinline__ int tiles_of(int len) { return len <= kDecKeys ? 1 : (len - 1) / kDecKeys + 1; }

// One tile on.  True if it was the last of its item.
__device__ __forceinline__ bool step(const DecodeParams& p, Place& at) {
  if (++at.in_page == p.page_tiles) {
    at.in_page = 0;
    ++at.page;
  }
  ++at.unit;
  if (++at.tile < at.n) return false;
  at.unit += kDecItemCost;
  at.tile = at.page = at.in_page = 0;
  if (++at.cut == p.cuts) {
    at.cut = 0;
    ++at.hk;
  }
  if (++at.item == p.items) {
    at.item = at.hk = at.cut = 0;
    ++at.s;
    at.len = clamped(p, at.next_len);
    at.n = tiles_of(at.len);
    at.next_len = read_len(p, at.s + 1);
  }
  return true;
}

// The table entry of a tile, fetched a tile ahead.  WHOLE (pages hold whole tiles): one entry for the warp, and the tile's place in
// the page; otherwise lane r or r + 16 has row r's entry and its offset in the page.
struct Lookup {
  int page, off, count, hk;
};
template <bool WHOLE>
__device__ __forceinline__ Lookup look_up(const DecodeParams& p, const Place& at) {
  const int* row = p.table + static_cast<int64_t>(at.s) * p.stride;
  Lookup r;
  r.hk = at.hk;
  r.page = -1;
  r.count = min(at.len - at.tile * kDecKeys, kDecKeys);
  if (WHOLE) {
    r.off = at.in_page * kDecKeys;
    if (r.count > 0) r.page = row[at.page];
  } else {
    const int in_tile = threadIdx.x & 15, pos = at.tile * kDecKeys + in_tile;
    r.off = 0;
    if (in_tile < r.count) {
      const int index = pos / p.P;
      r.off = pos - index * p.P;
      r.page = row[index];
    }
  }
  return r;
}

// The copies of a tile's rows; rows that are not there become zeros, so that no stale page contents reach a product.
template <bool WHOLE>
struct TileSource {
  int64_t k, v;     // WHOLE: this lane's first row of keys and of values; otherwise k: lanes 0 - 15 key rows, 16 - 31 value rows
  uint32_t valid;

  __device__ __forceinline__ void set(const DecodeParams& p, const Lookup& r) {
    const bool there = r.page >= 0 && r.page < p.n_pages;
    const int lane = threadIdx.x & 31;
    if (WHOLE) {
      valid = there ? 0xffffu >> (kDecKeys - r.count) : 0u;
      const int off = r.off + (lane >> 4), page = there ? r.page : 0;
      k = page * p.kp + off * p.kt + r.hk * p.kh + (lane & 15) * 8;
      v = page * p.vp + off * p.vt + r.hk * p.vh + (lane & 15) * 8;
    } else {
      k = 0;
      if (there) k = lane >= 16 ? r.page * p.vp + r.off * p.vt + r.hk * p.vh : r.page * p.kp + r.off * p.kt + r.hk * p.kh;
      valid = __ballot_sync(0xffffffffu, there) & 0xffffu;
    }
  }
  template <bool VALUES>
  __device__ __forceinline__ void copy(const DecodeParams& p, uint32_t tile) const {
    const int lane = threadIdx.x & 31, chunk = lane & 15, half = lane >> 4;
    const __nv_bfloat16* base = VALUES ? p.V : p.K;
    if (WHOLE) base += VALUES ? v : k;
    const int64_t two_rows = 2 * (VALUES ? p.vt : p.kt);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 2 * i + half;
      const bool ok = (valid >> row) & 1;
      if (WHOLE) {
        cp_async16_zfill(tile + tile_off(row, chunk), base, ok);
        base += two_rows;
      } else {
        const int64_t from = __shfl_sync(0xffffffffu, k, row + (VALUES ? 16 : 0));
        cp_async16_zfill(tile + tile_off(row, chunk), base + from + chunk * 8, ok);
      }
    }
  }
};

// Shares are cut in units of work: the tiles of an item, and behind them kDecItemCost for its end (in all fewer than 2^31).  The
// first wave of CTAs gets equal shares.  CTAs do not end together, though: SMs differ in what they get of the memory.  So large
// calls leave a tenth to a second wave of smaller shares, which the first CTAs to end make room for: 64 sequences of 64 heads
// 229 -> 213 us.  In smaller ones their start costs more than that.
struct Cuts {
  unsigned total, first;              // units; those of the first wave
  unsigned ctas, wave;                // CTAs with a share; those of the first wave
  unsigned each, over, each2, over2;  // units of a share of each wave, and how many shares have one more

  __device__ __forceinline__ void set(unsigned units) {
    total = units;
    wave = min(static_cast<unsigned>(kDecWave), (units + kDecWarps - 1) / kDecWarps);
    const bool rest = units >= static_cast<unsigned>(kDecWave) * kDecWarps * kDecRestTiles;
    first = rest ? units - units / 10 : units;
    ctas = rest ? kDecCtas : wave;
    each = first / wave;
    over = first - each * wave;
    each2 = (total - first) / kDecRest;
    over2 = total - first - each2 * kDecRest;
  }
  __device__ __forceinline__ unsigned begin(unsigned c) const {
    return c <= wave ? c * each + min(c, over) : first + (c - wave) * each2 + min(c - wave, over2);
  }
  __device__ __forceinline__ unsigned cta_of(unsigned u) const {
    const bool in_first = u < first;
    const unsigned x = in_first ? u : u - first, e = in_first ? each : each2, o = in_first ? over : over2;
    const unsigned c = x < o * (e + 1) ? x / (e + 1) : o + (x - o * (e + 1)) / e;
    return in_first ? c : wave + c;
  }
};

// Sum over the CTA of one value per thread and this thread's exclusive prefix sum.
__device__ __forceinline__ unsigned scan_cta(unsigned v, unsigned* part, unsigned* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) part[warp] = x;
  __syncthreads();
  unsigned before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kDecWarps; ++w) {
    before += w < warp ? part[w] : 0;
    all += part[w];
  }
  *total = all;
  return before + x - v;
}

struct Share {
  Cuts cuts;
  unsigned end;      // the unit where this warp's share ends
};

// Finds this warp's share and the place where it begins, four lengths per thread at a time.  Up to 128 sequences every warp
// reads and searches them alone; more are searched by the CTA, up to 512 of them at a time, which are read once if that is all.
// (One sequence of 4,001 tokens: 0.25 us less than with the CTA's search.)
__device__ __forceinline__ Share find_share(const DecodeParams& p, Place& at) {
  __shared__ unsigned part[kDecWarps];
  __shared__ uint4 shared_found[kDecWarps];
  constexpr int kChunk = kDecWarps * 32 * 4;
  const int warp = threadIdx.x >> 5;
  int len[5];
  unsigned n[4];
  auto load = [&](int s) {      // lengths s .. s + 4, units of sequences s .. s + 3; their sum
    unsigned sum = 0;
#pragma unroll
    for (int i = 0; i < 5; ++i) len[i] = read_len(p, s + i);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      n[i] = s + i < p.S ? (tiles_of(clamped(p, len[i])) + kDecItemCost) * p.items : 0;
      sum += n[i];
    }
    return sum;
  };
  Share sh;
  sh.end = at.unit = 0;
  unsigned begin, units;
  uint4 f;      // where this warp's share begins: sequence, its length, unit within it, length of the one behind it
  auto my_share = [&](unsigned total) {      // of the CTA; false if it has none
    sh.cuts.set(total);
    if (blockIdx.x >= sh.cuts.ctas) return false;
    begin = sh.cuts.begin(blockIdx.x);
    units = sh.cuts.begin(blockIdx.x + 1) - begin;
    return true;
  };
  if (p.S <= 128) {
    const int lane = threadIdx.x & 31;
    const unsigned sum = load(lane * 4);
    unsigned x = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (!my_share(__shfl_sync(0xffffffffu, x, 31))) return sh;
    const unsigned want = begin + units * warp / kDecWarps;
    unsigned first = x - sum;
    bool here = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (want - first < n[i]) {      // wraps where the sequence lies behind
        f = make_uint4(lane * 4 + i, len[i], want - first, len[i + 1]);
        here = true;
      }
      first += n[i];
    }
    const int from = __ffs(__ballot_sync(0xffffffffu, here)) - 1;
    f = make_uint4(__shfl_sync(0xffffffffu, f.x, from), __shfl_sync(0xffffffffu, f.y, from), __shfl_sync(0xffffffffu, f.z, from),
                   __shfl_sync(0xffffffffu, f.w, from));
  } else {
    unsigned total = 0, sum = 0, before = 0;
    if (p.S <= kChunk) {
      before = scan_cta(load(threadIdx.x * 4), part, &total);
    } else {
      for (int base = 0; base < p.S; base += kChunk) sum += load(base + threadIdx.x * 4);
      scan_cta(sum, part, &total);
    }
    if (!my_share(total)) return sh;
    unsigned seen = 0;
    for (int base = 0; base < p.S; base += kChunk) {
      if (p.S > kChunk) before = scan_cta(load(base + threadIdx.x * 4), part, &total);
      unsigned first = seen + before;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int w = 0; w < kDecWarps; ++w) {
          const unsigned in = begin + units * w / kDecWarps - first;
          if (in < n[i]) shared_found[w] = make_uint4(base + threadIdx.x * 4 + i, len[i], in, len[i + 1]);
        }
        first += n[i];
      }
      seen += total;
      if (begin + units < seen) break;
    }
    __syncthreads();
    f = shared_found[warp];
  }
  sh.end = begin + units * (warp + 1) / kDecWarps;
  at.unit = begin + units * warp / kDecWarps;
  at.s = f.x;
  at.len = clamped(p, f.y);
  at.next_len = f.w;
  at.n = tiles_of(at.len);
  const unsigned cost = at.n + kDecItemCost;
  at.item = f.z / cost;
  at.tile = f.z - at.item * cost;
  at.hk = p.cuts == 1 ? at.item : at.item / p.cuts;
  at.cut = at.item - at.hk * p.cuts;
  at.page = at.in_page = 0;
  if (at.tile >= at.n) {      // the end of an item: on to the next one
    at.unit += at.n - 1 - at.tile;      // its last tile, from where a step leads there
    at.tile = at.n - 1;
    at.in_page = -1;
    step(p, at);
  } else if (p.page_tiles > 0) {
    at.page = at.tile / p.page_tiles;
    at.in_page = at.tile - at.page * p.page_tiles;
  }
  return sh;
}

// What a CTA's warps leave to its end: pieces of items, in order; piece 2 w: of the item that warp w found begun and finished (in the
// workspace), 2 w + 1: of the one that it has left unfinished (in shared memory, where its ring was).
struct Piece {
  int flags, s, h0_heads;
};
enum { kPieceThere = 1, kPieceBegins = 2, kPieceEnds = 4 };

template <int HT>
__device__ __forceinline__ void join_pieces(const DecodeParams& p, const unsigned char* smem, const Piece* pieces) {
  constexpr int kHeads = HT * 8;
  const int c = blockIdx.x;
  unsigned there = 0, begun = 0, ended = 0;      // a bit per piece
#pragma unroll
  for (int i = 0; i < 2 * kDecWarps; ++i) {
    const int f = pieces[i].flags;
    there |= f & kPieceThere ? 1u << i : 0u;
    begun |= f & kPieceBegins ? 1u << i : 0u;
    ended |= f & kPieceEnds ? 1u << i : 0u;
  }
  while (there != 0) {
    // the pieces of one item: those of shared memory up to one in the workspace that ends it, or to the end of the share
    const int first = __ffs(there) - 1, end = ended != 0 ? __ffs(ended) - 1 : 2 * kDecWarps;
    const unsigned mine = there & ((2u << end) - 1);
    const bool begins = begun >> first & 1, ends = end < 2 * kDecWarps;
    there &= ~mine;
    ended &= ~mine;
    const int s = pieces[first].s, h0 = pieces[first].h0_heads & 0xffffff, heads = pieces[first].h0_heads >> 24;
    if (!RBS_DBG_OK(s >= 0 && s < p.S && h0 >= 0 && heads > 0 && h0 + heads <= p.Hq, p.status, kDbgDecodeRow)) continue;
#pragma unroll
    for (int n = 0; n < HT; ++n) {
      const int h = 8 * n + (threadIdx.x >> 4), e = (threadIdx.x & 15) * 8;
      if (h >= heads) continue;
      float2 ml[kDecWarps + 1];
      float4 a[kDecWarps + 1], b[kDecWarps + 1];
#pragma unroll
      for (int w = 0; w <= kDecWarps; ++w) {
        ml[w] = make_float2(-INFINITY, 0.f);
        a[w] = b[w] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (w < kDecWarps && (mine >> (2 * w + 1) & 1)) {
          const unsigned char* from = smem + w * kDecRing;
          ml[w] = reinterpret_cast<const float2*>(from + kHeads * kDecRow * 4)[h];
          const float4* o = reinterpret_cast<const float4*>(from + (h * kDecRow + e) * 4);
          a[w] = o[0];
          b[w] = o[1];
        }
        if (w == kDecWarps && ends) {
          const int64_t row = static_cast<int64_t>(2 * kDecCtas + (kDecWarps - 1) * c + (end >> 1) - 1) * kHeads + h;
          ml[w] = __ldcg(p.part_ml + row);
          const float4* o = reinterpret_cast<const float4*>(p.part_o + row * kHeadDim + e);
          a[w] = __ldcg(o);
          b[w] = __ldcg(o + 1);
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w <= kDecWarps; ++w) top = fmaxf(top, ml[w].x);
      const float base = exp_base(top);
      float acc[8] = {}, sum = 0.f;
#pragma unroll
      for (int w = 0; w <= kDecWarps; ++w) {
        const float f = fast_exp2(ml[w].x - base);
        sum = fmaf(ml[w].y, f, sum);
        acc[0] = fmaf(a[w].x, f, acc[0]); acc[1] = fmaf(a[w].y, f, acc[1]); acc[2] = fmaf(a[w].z, f, acc[2]); acc[3] = fmaf(a[w].w, f, acc[3]);
        acc[4] = fmaf(b[w].x, f, acc[4]); acc[5] = fmaf(b[w].y, f, acc[5]); acc[6] = fmaf(b[w].z, f, acc[6]); acc[7] = fmaf(b[w].w, f, acc[7]);
      }
      if (begins && ends) {
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        *reinterpret_cast<uint4*>(p.O + s * p.ost + (h0 + h) * p.osh + e) =
            make_uint4(pack_bf16(acc[0] * inv, acc[1] * inv), pack_bf16(acc[2] * inv, acc[3] * inv), pack_bf16(acc[4] * inv, acc[5] * inv),
                       pack_bf16(acc[6] * inv, acc[7] * inv));
        if (e == 0 && p.lse != nullptr) p.lse[static_cast<int64_t>(s) * p.Hq + h0 + h] = lse_of(top, sum);
      } else {
        const int64_t row = static_cast<int64_t>(2 * c + (begins ? 1 : 0)) * kHeads + h;
        float4* o = reinterpret_cast<float4*>(p.part_o + row * kHeadDim + e);
        o[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        o[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
        if (e == 0) p.part_ml[row] = make_float2(top, sum);
      }
    }
  }
}

template <int HT, bool WHOLE>
__global__ void __launch_bounds__(kDecWarps * 32, 3)
decode_kernel(const DecodeParams p) {
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ Piece pieces[2 * kDecWarps];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  unsigned char* ring_bytes = smem + warp * kDecRing;
  const uint32_t ring = smem_u32(ring_bytes);
  if (lane < 2) pieces[2 * warp + lane].flags = 0;
  pdl_wait();
  Place at;
  const Share share = find_share(p, at);
  if (blockIdx.x >= share.cuts.ctas) {
    if (threadIdx.x == 0) p.found[blockIdx.x] = make_int4(-1, 0, 0, 0);
    return;
  }
  // the item that the CTA finds begun, for the kernel below: warp 0's share begins where the CTA's does
  const int4 begun = make_int4(at.tile == 0 ? -1 : at.s, (at.hk * p.G + at.cut * p.gh) | min(p.gh, p.G - at.cut * p.gh) << 24, at.unit - at.tile,
                               at.unit - at.tile + at.n - 1);
  auto write_found = [&]() {
    if (threadIdx.x == 0)
      p.found[blockIdx.x] = begun.x < 0 ? begun
                                        : make_int4(begun.x, begun.y, share.cuts.cta_of(begun.z), share.cuts.cta_of(begun.w));
  };
  if (at.unit < share.end) {
    // the item that is summed, and how many items this warp has begun, on the copying side and on this one
    int s = at.s, hk = at.hk, cut = at.cut, item = at.item;
    bool begun_here = at.tile == 0, finished = false;
    int copied_items = 0, item_no = 0;

    // tiles i + 1 and i + 2 are on their way while tile i is worked on, the table entry of tile i + 3 as well
    Lookup look = look_up<WHOLE>(p, at);
    TileSource<WHOLE> source;
    uint32_t queue[kDecStages];      // a word per tile, 0 behind the last one: bits 0 - 15: the keys that there are
    constexpr uint32_t kTile = 0x20000u, kLast = 0x10000u;      // there is a tile; it is the last one of its item
    auto begin_keys = [&](uint32_t tile) {
      uint32_t word = 0;
      if (at.unit < share.end) {
        source.set(p, look);
        source.template copy<false>(p, tile);
        const bool last = step(p, at);
        if (at.unit < share.end) {
          look = look_up<WHOLE>(p, at);
          copied_items += last;
        }
        word = kTile | source.valid | (last ? kLast : 0u);
      }
      cp_async_commit();
      return word;
    };
    auto begin_values = [&](uint32_t tile, bool there) {
      if (there) source.template copy<true>(p, tile);
      cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < kDecStages; ++i) {
      queue[i] = begin_keys(ring + 2 * i * kDecTileBytes);
      begin_values(ring + (2 * i + 1) * kDecTileBytes, queue[i] != 0);
    }

    write_found();
    Queries<HT> q, q_next;
    int h0, heads, next_no = 0;      // q_next: queries of item next_no of this warp, if that is ahead of item_no
    auto heads_of = [&](int k, int c) {
      h0 = k * p.G + c * p.gh;
      heads = min(p.gh, p.G - c * p.gh);
    };
    auto fetch_next = [&]() {
      if (HT == 1 && next_no == item_no && copied_items > item_no) {
        int ns = s, nk = hk, nc = cut + 1;
        if (nc == p.cuts) { nc = 0; ++nk; }
        if (item + 1 == p.items) { nk = 0; ++ns; }
        q_next.load(p.Q + ns * p.qst + (nk * p.G + nc * p.gh) * p.qsh, p.qsh, min(p.gh, p.G - nc * p.gh));
        next_no = item_no + 1;
      }
    };
    heads_of(hk, cut);
    q.load(p.Q + s * p.qst + h0 * p.qsh, p.qsh, heads);
    fetch_next();
    Softmax<HT> sm;
    sm.start();
    for (int i = 0; queue[0] != 0; ++i) {
      const uint32_t kt = ring + 2 * (i % kDecStages) * kDecTileBytes, vt = kt + kDecTileBytes;
      const uint32_t word = queue[0];
      queue[0] = queue[1];
      float pr[HT][4];
      cp_async_wait<2 * kDecStages - 1>();
      __syncwarp();
      sm.scores(q, kt, word & 0xffffu, p.scale_log2, pr);
      __syncwarp();
      queue[1] = begin_keys(kt);
      fetch_next();
      cp_async_wait<2 * kDecStages - 1>();
      __syncwarp();
      sm.values(vt, pr);
      __syncwarp();
      begin_values(vt, queue[1] != 0);
      finished = word & kLast;
      if (!finished) continue;

      // the end of the item
      sm.finish();
      if (begun_here) {
        sm.write(p, s, h0, heads);
      } else {
        const int64_t slot = warp == 0 ? 2 * blockIdx.x : 2 * kDecCtas + (kDecWarps - 1) * blockIdx.x + warp - 1;
        if (RBS_DBG_OK(slot >= 0 && slot < kDecSlots, p.status, kDbgDecodeSlot))
          sm.put(p.part_o + slot * (HT * 8) * kHeadDim, kHeadDim, p.part_ml + slot * (HT * 8));
        if (warp > 0 && lane == 0) pieces[2 * warp] = {kPieceThere | kPieceEnds, s, h0 | heads << 24};
      }
      begun_here = true;
      ++item_no;
      if (++cut == p.cuts) { cut = 0; ++hk; }
      if (++item == p.items) { item = hk = 0; ++s; }
      if (queue[0] != 0) {
        heads_of(hk, cut);
        if (next_no == item_no) q = q_next;
        else q.load(p.Q + s * p.qst + h0 * p.qsh, p.qsh, heads), next_no = item_no;
        fetch_next();
        sm.start();
      }
    }
    if (!finished) {      // an item is left unfinished
      sm.finish();
      sm.put(reinterpret_cast<float*>(ring_bytes), kDecRow, reinterpret_cast<float2*>(ring_bytes + HT * 8 * kDecRow * 4));
      if (lane == 0) pieces[2 * warp + 1] = {kPieceThere | (begun_here ? kPieceBegins : 0), s, h0 | heads << 24};
    }
  } else {
    write_found();
  }
  pdl_trigger();      // see join_kernel
  __syncthreads();
  join_pieces<HT>(p, smem, pieces);
}

constexpr int kJoinThreads = 256;

// Joins the pieces of the items that lie in several CTAs' shares.  The CTAs that found an item begun share out its 1024 * HT
// sums: the more pieces, the narrower the strip of each, so that every CTA reads about as much as one piece holds.  Thread
// (group, column) takes four sums of every groups-th piece, with the maximum as it goes, so that all its loads can be on
// their way together; the groups are joined in order, maxima first.  The order depends on the lengths alone.
// It becomes resident at the end of the kernel above, and lets no later kernel do so before its own end: the kernel above fills
// every SM exactly, and where waiting CTAs had taken places of its own its last CTAs started late (64 sequences of 64 heads:
// 224 us instead of 213 with triggers at both kernels' begins).
template <int HT>
__global__ void __launch_bounds__(kJoinThreads)
join_kernel(const DecodeParams p) {
  constexpr int kColumns = HT * 8 * kHeadDim / 4;
  __shared__ float4 sums[kJoinThreads];
  __shared__ float2 mls[kJoinThreads];
  pdl_wait();
  const int4 found = p.found[blockIdx.x];
  if (found.x < 0) return;
  const int c0 = found.z, sharers = found.w - c0, rank = blockIdx.x - c0 - 1;
  // columns of a strip: a power of two, at least a quarter of a warp's 16-byte loads
  const int fair = (kColumns + sharers - 1) / sharers;
  const int width = fair <= 4 ? 4 : 1 << (32 - __clz(fair - 1));
  if (rank * width >= kColumns) return;
  const int heads = found.y >> 24, h0 = found.y & 0xffffff;
  if (!RBS_DBG_OK(found.x < p.S && heads > 0 && h0 + heads <= p.Hq && c0 >= 0 && found.w < kDecCtas, p.status, kDbgDecodeRow)) return;
  const int lanes = min(width, kJoinThreads), shift = __ffs(lanes) - 1, groups = kJoinThreads >> shift;      // powers of two
  const int group = threadIdx.x >> shift, lane = threadIdx.x & (lanes - 1), apart = max(lanes, 32);
  for (int column = rank * width + lane; column < (rank + 1) * width; column += lanes) {      // once but for strips wider than the CTA
    const int head = column / (kHeadDim / 4);
    float top = -INFINITY, sum = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    auto fade = [&](float high) {      // everything against the maximum `high` from here on
      const float f = fast_exp2(top - exp_base(high));
      top = high;
      sum *= f;
      acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
    };
    if (head < heads) {
#pragma unroll 4
      for (int i = group; i <= sharers; i += groups) {      // piece 0 in slot 2 c0 + 1, piece i in slot 2 (c0 + i)
        const int64_t slot = i == 0 ? 2 * c0 + 1 : 2 * (c0 + i);
        const float2 ml = p.part_ml[slot * (HT * 8) + head];
        const float4 o = *reinterpret_cast<const float4*>(p.part_o + slot * (HT * 8 * kHeadDim) + 4 * column);
        fade(fmaxf(top, ml.x));
        const float w = fast_exp2(ml.x - exp_base(top));
        sum = fmaf(ml.y, w, sum);
        acc.x = fmaf(o.x, w, acc.x); acc.y = fmaf(o.y, w, acc.y); acc.z = fmaf(o.z, w, acc.z); acc.w = fmaf(o.w, w, acc.w);
      }
    }
    // the groups of a warp, then those of the warps: first the maximum, then plain sums
    if (lanes < 32) {
      float high = top;
      for (int o = lanes; o < 32; o *= 2) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
      fade(high);
      for (int o = lanes; o < 32; o *= 2) {
        sum += __shfl_down_sync(0xffffffffu, sum, o);
        acc.x += __shfl_down_sync(0xffffffffu, acc.x, o);
        acc.y += __shfl_down_sync(0xffffffffu, acc.y, o);
        acc.z += __shfl_down_sync(0xffffffffu, acc.z, o);
        acc.w += __shfl_down_sync(0xffffffffu, acc.w, o);
      }
    }
    if (groups > 1) {
      __syncthreads();
      sums[threadIdx.x] = acc;
      mls[threadIdx.x] = make_float2(top, sum);
      __syncthreads();
      if (group == 0) {
        float high = top;
#pragma unroll
        for (int k = 1; k < kJoinThreads / 32; ++k)
          if (threadIdx.x + k * apart < kJoinThreads) high = fmaxf(high, mls[threadIdx.x + k * apart].x);
        fade(high);
#pragma unroll
        for (int k = 1; k < kJoinThreads / 32; ++k) {
          const int i = threadIdx.x + k * apart;
          if (i >= kJoinThreads) break;
          const float2 ml = mls[i];
          const float4 o = sums[i];
          const float w = fast_exp2(ml.x - exp_base(high));
          sum = fmaf(ml.y, w, sum);
          acc.x = fmaf(o.x, w, acc.x); acc.y = fmaf(o.y, w, acc.y); acc.z = fmaf(o.z, w, acc.z); acc.w = fmaf(o.w, w, acc.w);
        }
      }
    }
    if (group == 0 && head < heads) {
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      const int e = 4 * column % kHeadDim;
      *reinterpret_cast<uint2*>(p.O + found.x * p.ost + (h0 + head) * p.osh + e) =
          make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
      if (e == 0 && p.lse != nullptr) p.lse[static_cast<int64_t>(found.x) * p.Hq + h0 + head] = lse_of(top, sum);
    }
  }
}

struct DecodeWorkspace {
  size_t off_o, off_ml, off_found, bytes;
};
static DecodeWorkspace decode_workspace(int G) {
  const size_t rows = static_cast<size_t>(kDecSlots) * (G <= 8 ? 8 : 16);
  DecodeWorkspace w;
  size_t off = 0;
  w.off_o = off; off = align_up(off + rows * kHeadDim * sizeof(float), 256);
  w.off_ml = off; off = align_up(off + rows * sizeof(float2), 256);
  w.off_found = off; off = align_up(off + kDecCtas * sizeof(int4), 256);
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
  if (block_table == nullptr || seq_lens == nullptr || !(fabsf(softmax_scale * kLog2e) <= 3.4028235e38f)) return RBS_ERR_INVALID_ARG;
  Q.stride_batch = O.stride_batch = 0;
  if ((st = check_tensor(Q)) != RBS_OK || (st = check_tensor(O)) != RBS_OK || (st = check_tensor(k_cache)) != RBS_OK ||
      (st = check_tensor(v_cache)) != RBS_OK)
    return st;
  DecodeParams p = {};
  p.Q = static_cast<const __nv_bfloat16*>(Q.ptr); p.qst = Q.stride_token; p.qsh = Q.stride_head;
  p.K = static_cast<const __nv_bfloat16*>(k_cache.ptr); p.kp = k_cache.stride_batch; p.kt = k_cache.stride_token; p.kh = k_cache.stride_head;
  p.V = static_cast<const __nv_bfloat16*>(v_cache.ptr); p.vp = v_cache.stride_batch; p.vt = v_cache.stride_token; p.vh = v_cache.stride_head;
  p.O = static_cast<__nv_bfloat16*>(O.ptr); p.ost = O.stride_token; p.osh = O.stride_head;
  p.status = debug_status();
  p.lse = lse; p.table = block_table; p.lens = seq_lens;
  p.S = shape->n_seqs; p.Hq = shape->n_q_heads; p.Hkv = shape->n_kv_heads; p.G = p.Hq / p.Hkv;
  p.P = shape->page_size; p.n_pages = shape->n_pages; p.max_pages = shape->max_pages; p.stride = shape->table_stride;
  p.cuts = (p.G + 15) / 16;
  p.gh = (p.G + p.cuts - 1) / p.cuts;
  p.items = p.Hkv * p.cuts;
  // heads share a word with a count, units of work are counted in 31 bits
  const double most_units = static_cast<double>(p.S) * p.items * (static_cast<double>(p.max_pages) * p.P / kDecKeys + 1 + kDecItemCost);
  if (p.Hq >= 1 << 24 || most_units >= 2147483647.0) return RBS_ERR_UNSUPPORTED;
  const DecodeWorkspace ws = decode_workspace(p.G);
  if (workspace == nullptr || workspace_bytes < ws.bytes || reinterpret_cast<uintptr_t>(workspace) % 256 != 0) return RBS_ERR_WORKSPACE;
  unsigned char* base = static_cast<unsigned char*>(workspace);
  p.part_o = reinterpret_cast<float*>(base + ws.off_o);
  p.part_ml = reinterpret_cast<float2*>(base + ws.off_ml);
  p.found = reinterpret_cast<int4*>(base + ws.off_found);
  const float scale = softmax_scale == 0.f ? 1.0f / sqrtf(static_cast<float>(kHeadDim)) : softmax_scale;
  p.scale_log2 = scale * kLog2e;
  p.page_tiles = p.P % kDecKeys == 0 ? p.P / kDecKeys : 0;
  auto* kernel = p.page_tiles > 0 ? (p.gh <= 8 ? decode_kernel<1, true> : decode_kernel<2, true>)
                                  : (p.gh <= 8 ? decode_kernel<1, false> : decode_kernel<2, false>);
  const size_t smem = static_cast<size_t>(kDecWarps) * kDecRing;
  if ((st = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem)) != RBS_OK) return st;
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  // no more CTAs than the table could have work for (four units each)
  const unsigned ctas = static_cast<unsigned>(most_units / kDecWarps + 1 < kDecCtas ? most_units / kDecWarps + 1 : kDecCtas);
  RBS_CUDA_OK(launch_pdl(kernel, ctas, 1, kDecWarps * 32, smem, cs, p));
  RBS_CUDA_OK(launch_pdl(p.gh <= 8 ? join_kernel<1> : join_kernel<2>, ctas, 1, kJoinThreads, 0, cs, p));
  return RBS_OK;
}

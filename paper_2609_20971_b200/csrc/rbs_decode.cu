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
  float scale_log2;
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

// Starts the copy of a warp's 16 keys and values from token `tok` on; returns which of them there are (a bit per key; the
// others are filled with zeros, so that no stale page contents reach a product).  Lanes 0 - 15 look up the key rows, lanes
// 16 - 31 the value rows.
__device__ __forceinline__ uint32_t fetch_tile(const DecodeParams& p, const int* table_row, int tok, int len, int hk, uint32_t ktile,
                                               uint32_t vtile) {
  const int lane = threadIdx.x & 31, r = lane & 15, pos = tok + r;
  int page = -1, off = 0;
  if (pos < len) {
    page = table_row[pos / p.P];
    off = pos % p.P;
  }
  const bool there = page >= 0 && page < p.n_pages;
  const bool is_v = lane >= 16;
  int64_t at = 0;
  if (there) at = is_v ? page * p.vp + off * p.vt + hk * p.vh : page * p.kp + off * p.kt + hk * p.kh;
  const uint32_t valid = __ballot_sync(0xffffffffu, there) & 0xffffu;
  const int chunk = lane & 15, half = lane >> 4;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int row = 2 * i + half;
    const int64_t k_at = __shfl_sync(0xffffffffu, at, row), v_at = __shfl_sync(0xffffffffu, at, row + 16);
    const bool ok = (valid >> row) & 1;
    cp_async16_zfill(ktile + tile_off(row, chunk), p.K + k_at + chunk * 8, ok);
    cp_async16_zfill(vtile + tile_off(row, chunk), p.V + v_at + chunk * 8, ok);
  }
  return valid;
}

// One CTA per (sequence, KV head, cut of its query heads).
template <int HT>
__global__ void __launch_bounds__(kDecWarps * 32)
decode_kernel(const DecodeParams p) {
  extern __shared__ __align__(128) unsigned char smem[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t tiles = smem_u32(smem) + warp * kDecStages * 2 * kDecTileBytes;
  float* part_o = reinterpret_cast<float*>(smem + kDecOffO);
  float* part_ml = reinterpret_cast<float*>(smem + kDecOffMl);
  pdl_trigger();
  pdl_wait();
  const int item = blockIdx.x;
  const int cut = item % p.cuts, hk = item / p.cuts % p.Hkv, s = item / p.cuts / p.Hkv;
  const int h0 = hk * p.G + cut * p.gh, heads = min(p.gh, p.G - cut * p.gh);
  const int len = min(max(p.lens[s], 0), p.max_pages * p.P);
  const int* row = p.table + static_cast<int64_t>(s) * p.stride;

  Softmax<HT> sm;
  sm.start(p.Q + s * p.qst + h0 * p.qsh, p.qsh, heads);
  const int n = (len + kDecTile - 1) / kDecTile;
  uint32_t valid[kDecStages];
#pragma unroll
  for (int i = 0; i < kDecStages; ++i) {
    valid[i] = 0;
    if (i < n) valid[i] = fetch_tile(p, row, i * kDecTile + warp * kDecKeys, len, hk, tiles + 2 * i * kDecTileBytes, tiles + (2 * i + 1) * kDecTileBytes);
    cp_async_commit();
  }
  for (int i = 0; i < n; ++i) {
    const uint32_t kt = tiles + 2 * (i % kDecStages) * kDecTileBytes, vt = kt + kDecTileBytes;
    cp_async_wait<kDecStages - 1>();
    __syncwarp();
    uint32_t pr[HT][2];
    sm.scores(kt, valid[0], p.scale_log2, pr);
    sm.values(vt, pr);
    __syncwarp();
    valid[0] = valid[1];
    if (i + kDecStages < n) valid[1] = fetch_tile(p, row, (i + kDecStages) * kDecTile + warp * kDecKeys, len, hk, kt, vt);
    cp_async_commit();
  }

  // the warps' sums become one: all to the largest maximum, then (0 + 2) + (1 + 3)
  const int g = lane >> 2, t = lane & 3;
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
      const float* x = part_o + h * kDecRow + c;
      const float inv = sum == 0.f ? 0.f : 1.0f / sum;
      uint32_t out[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        out[i] = pack_bf16((x[2 * i] + x[8 * kDecRow + 2 * i]) * inv, (x[2 * i + 1] + x[8 * kDecRow + 2 * i + 1]) * inv);
      const int hq = h0 + 8 * k + h;
      *reinterpret_cast<uint4*>(p.O + s * p.ost + hq * p.osh + c) = make_uint4(out[0], out[1], out[2], out[3]);
      if (c == 0 && p.lse != nullptr)
        p.lse[static_cast<int64_t>(s) * p.Hq + hq] = sum == 0.f ? -INFINITY : (base + log2f(sum)) * 0.6931471805599453f;
    }
    __syncthreads();
  }
}

}  // namespace rbs

extern "C" size_t rbs_paged_decode_workspace_bytes(const rbs_paged_shape* shape) {
  using namespace rbs;
  if (check_paged_table(shape) != RBS_OK || check_paged_cache(shape) != RBS_OK) return 0;
  return 0;
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
  const float scale = softmax_scale == 0.f ? 1.0f / sqrtf(static_cast<float>(kHeadDim)) : softmax_scale;
  p.scale_log2 = scale * kLog2e;
  auto* kernel = p.gh <= 8 ? decode_kernel<1> : decode_kernel<2>;
  const size_t smem = kDecOffMl + kDecWarps * 8 * 2 * sizeof(float);
  if ((st = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem)) != RBS_OK) return st;
  const long long items = static_cast<long long>(p.S) * p.Hkv * p.cuts;
  if (items > 0x7fffffffll) return RBS_ERR_UNSUPPORTED;
  (void)workspace; (void)workspace_bytes;
  RBS_CUDA_OK(launch_pdl(kernel, static_cast<unsigned>(items), 1, kDecWarps * 32, smem, static_cast<cudaStream_t>(stream), p));
  return RBS_OK;
}

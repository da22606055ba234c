// rbs_qk_norm_rope and rbs_qk_norm_rope_paged: norm of each head and rotation by position in one pass over the rows of Q
// and K (256 bytes each), in the paged form with the keys and the values going to their slots of the cache.
// A stream: 512 bytes read and written per row against some 60 instructions of half a warp.
#include "rbs_common.cuh"

namespace rbs {

struct RopeParams {
  const __nv_bfloat16* Q; int64_t qsb, qst, qsh;
  const __nv_bfloat16* K; int64_t ksb, kst, ksh;
  const __nv_bfloat16* V; int64_t vst, vsh;
  __nv_bfloat16* Qo; int64_t qosb, qost, qosh;
  __nv_bfloat16* Ko; int64_t kosb, kost, kosh;       // nullable in the paged form
  __nv_bfloat16* Kc; int64_t kcp, kct, kch;          // cache: page, token, head strides
  __nv_bfloat16* Vc; int64_t vcp, vct, vch;
  const int* positions;
  const int* slots;
  const float* inv_freq;
  const float* q_norm;   // nullable
  const float* k_norm;   // nullable
  float eps, magnitude;
  int rot, Hq, Hkv, N, page;
  int slot_rows, cache_rows;   // entries of slots; rows of the cache
  long long tokens;      // batch * N
  int halves;            // halves of warps per token: 2, 4, 8 or 16
};

constexpr int kRopeThreads = 256;
constexpr int kRopeHalves = kRopeThreads / 16;   // halves of warps of a CTA
constexpr int kRopeBatch = 4;                    // rows that half a warp has in flight
constexpr int kRopeTokens = 8;                   // most tokens of a CTA

// Half a warp per row.  Lane u (of 16) of a row holds two groups A, B of four elements:
//   half layout, u < rot / 8: A = 4u.., B = rot/2 + 4u.., so that pair 4u + k is (A[k], B[k]);
//   otherwise 8 neighbours: A = 8u.., B = 8u + 4..; interleaved, pairs 4u .. 4u + 3 are (A0,A1) (A2,A3) (B0,B1) (B2,B3).
// In both layouts lane u turns pairs 4u .. 4u + 3 iff u < rot / 8: no exchange between lanes but the sum of squares, and
// an output may be its own input.  Pair (x, y) becomes (x c0 - y s1, y c1 + x s0) * r with r = 1 / sqrt(mean + eps) and the norm's
// weights in c and s, which stay in registers while a half walks over the heads of its token.
template <bool INTERLEAVED>
struct RopeLane {
  float c0[4], s1[4], c1[4], s0[4];
  int a, b;
  unsigned mask;     // the lanes of this half
  float eps;
  bool turns, norm;

  __device__ __forceinline__ void weigh(const float2* angles, const float* weights) {
    const int u = threadIdx.x & 15;
    norm = weights != nullptr;
    float w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = norm ? weights[(k < 4 ? a : b - 4) + k] : 1.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 cs = turns ? angles[4 * u + k] : make_float2(1.0f, 0.0f);
      const float w0 = INTERLEAVED ? w[2 * k] : w[k], w1 = INTERLEAVED ? w[2 * k + 1] : w[4 + k];
      c0[k] = w0 * cs.x; s1[k] = w1 * cs.y; c1[k] = w1 * cs.x; s0[k] = w0 * cs.y;
    }
  }
  __device__ __forceinline__ void turn(uint2& xa, uint2& xb) const {
    const float x[8] = {bf16lo(xa.x), bf16hi(xa.x), bf16lo(xa.y), bf16hi(xa.y), bf16lo(xb.x), bf16hi(xb.x), bf16lo(xb.y), bf16hi(xb.y)};
    float r = 1.0f;
    if (norm) {
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) ss = fmaf(x[k], x[k], ss);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(mask, ss, o);
      r = rsqrtf(ss * (1.0f / kHeadDim) + eps);
    }
    float y[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = INTERLEAVED ? 2 * k : k, j = INTERLEAVED ? 2 * k + 1 : 4 + k;
      y[i] = x[i] * c0[k];
      y[j] = x[j] * c1[k];
      if (turns) {      // elsewhere a zero would still carry an infinite neighbour over
        y[i] = fmaf(-x[j], s1[k], y[i]);
        y[j] = fmaf(x[i], s0[k], y[j]);
      }
      if (norm) {
        y[i] *= r;
        y[j] *= r;
      }
    }
    xa = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
    xb = make_uint2(pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
  }
};

// Up to kRopeBatch rows from head h on, every step-th.
template <bool INTERLEAVED>
__device__ __forceinline__ void load_rows(const RopeLane<INTERLEAVED>& lane, const __nv_bfloat16* src, int64_t stride, int h, int heads, int step,
                                          uint2 (&xa)[kRopeBatch], uint2 (&xb)[kRopeBatch]) {
#pragma unroll
  for (int i = 0; i < kRopeBatch; ++i) {
    if (h + i * step < heads) {
      const __nv_bfloat16* row = src + (h + i * step) * stride;
      xa[i] = *reinterpret_cast<const uint2*>(row + lane.a);
      xb[i] = *reinterpret_cast<const uint2*>(row + lane.b);
    }
  }
}

// The heads h, h + step, .. of one token; the first batch has been loaded.  Each row goes to one or two places.
template <bool TURN, bool INTERLEAVED>
__device__ __forceinline__ void walk_heads(const RopeLane<INTERLEAVED>& lane, const __nv_bfloat16* src, int64_t stride, int h, int heads, int step,
                                           uint2 (&xa)[kRopeBatch], uint2 (&xb)[kRopeBatch], __nv_bfloat16* dst, int64_t dst_stride,
                                           __nv_bfloat16* dst2, int64_t dst2_stride) {
  while (h < heads) {
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      const int at = h + i * step;
      if (at < heads) {
        if (TURN) lane.turn(xa[i], xb[i]);
        if (dst != nullptr) {
          *reinterpret_cast<uint2*>(dst + at * dst_stride + lane.a) = xa[i];
          *reinterpret_cast<uint2*>(dst + at * dst_stride + lane.b) = xb[i];
        }
        if (dst2 != nullptr) {
          *reinterpret_cast<uint2*>(dst2 + at * dst2_stride + lane.a) = xa[i];
          *reinterpret_cast<uint2*>(dst2 + at * dst2_stride + lane.b) = xb[i];
        }
      }
    }
    h += kRopeBatch * step;
    if (h < heads) load_rows(lane, src, stride, h, heads, step, xa, xb);
  }
}

// A CTA has 16 / halves tokens, `halves` halves of warps for each.  Its threads compute the tokens' angles once, behind the
// first rows' loads.
template <bool INTERLEAVED, bool PAGED>
__global__ void __launch_bounds__(kRopeThreads, 4)
rope_kernel(const RopeParams p) {
  __shared__ float2 angles[kRopeTokens][kHeadDim / 2];
  const int u = threadIdx.x & 15, half = threadIdx.x >> 4;
  const int per_cta = kRopeHalves / p.halves, mine = half / p.halves, h0 = half - mine * p.halves;
  const long long token0 = static_cast<long long>(blockIdx.x) * per_cta, token = token0 + mine;
  RopeLane<INTERLEAVED> lane;
  lane.turns = u < p.rot / 8;
  lane.a = lane.turns && !INTERLEAVED ? 4 * u : 8 * u;
  lane.b = lane.turns && !INTERLEAVED ? p.rot / 2 + 4 * u : 8 * u + 4;
  lane.mask = 0xffffu << (threadIdx.x & 16);
  lane.eps = p.eps;
  pdl_trigger();
  pdl_wait();
  const bool live = token < p.tokens;
  const int64_t l = token < p.N ? 0 : token / p.N, t = token - l * p.N;
  const __nv_bfloat16* Q = p.Q + l * p.qsb + t * p.qst;
  const __nv_bfloat16* K = p.K + l * p.ksb + t * p.kst;
  const int n_q = live ? p.Hq : 0;
  uint2 xa[kRopeBatch], xb[kRopeBatch];
  load_rows(lane, Q, p.qsh, h0, n_q, p.halves, xa, xb);

  // Angles in revolutions, as fractions of 2^64: positions are whole numbers, so whole revolutions of the frequency drop out of
  // the product by themselves, and an angle is off by 2^-33 of a revolution at most however far the position is.
  const int pairs = p.rot / 2;
  for (int i = threadIdx.x; i < per_cta * (kHeadDim / 2); i += kRopeThreads) {
    const int which = i / (kHeadDim / 2), k = i % (kHeadDim / 2);
    if (k < pairs && token0 + which < p.tokens) {
      double f = static_cast<double>(p.inv_freq[k]) * 0.15915494309189535;
      f = (f - floor(f)) * 18446744073709551616.0;
      const long long pos = p.positions[(token0 + which) % p.N];
      const unsigned long long turn = static_cast<unsigned long long>(pos) * __double2ull_rn(f);
      float sn, cs;
      sincospif(static_cast<float>(static_cast<int>(turn >> 32)) * 4.656612873077393e-10f, &sn, &cs);   // 2^-31: half revolutions
      angles[which][k] = make_float2(cs * p.magnitude, sn * p.magnitude);
    }
  }
  __syncthreads();
  if (!live) return;

  lane.weigh(angles[mine], p.q_norm);
  walk_heads<true>(lane, Q, p.qsh, h0, n_q, p.halves, xa, xb, p.Qo + l * p.qosb + t * p.qost, p.qosh, nullptr, 0);

  __nv_bfloat16 *kc = nullptr, *vc = nullptr;
  if (PAGED) {
    const int slot = t < p.slot_rows ? p.slots[t] : -1;
    if (slot >= 0 && slot < p.cache_rows) {
      const int64_t page = slot / p.page, off = slot - page * p.page;
      kc = p.Kc + page * p.kcp + off * p.kct;
      vc = p.Vc + page * p.vcp + off * p.vct;
    }
    if (vc != nullptr) {
      const __nv_bfloat16* V = p.V + t * p.vst;
      load_rows(lane, V, p.vsh, h0, p.Hkv, p.halves, xa, xb);
      walk_heads<false>(lane, V, p.vsh, h0, p.Hkv, p.halves, xa, xb, vc, p.vch, nullptr, 0);
    }
  }
  if (!PAGED || kc != nullptr || p.Ko != nullptr) {
    load_rows(lane, K, p.ksh, h0, p.Hkv, p.halves, xa, xb);
    lane.weigh(angles[mine], p.k_norm);
    walk_heads<true>(lane, K, p.ksh, h0, p.Hkv, p.halves, xa, xb, PAGED && p.Ko == nullptr ? nullptr : p.Ko + l * p.kosb + t * p.kost, p.kosh, kc,
                     p.kch);
  }
}

static rbs_status check_rope(const rbs_rope* r, int n_tokens) {
  if (r == nullptr || n_tokens <= 0 || r->positions == nullptr) return RBS_ERR_INVALID_ARG;
  if (!(r->eps >= 0.f) || r->eps > 3.0e38f || !(fabsf(r->magnitude) <= 3.4028235e38f)) return RBS_ERR_INVALID_ARG;
  if (r->rot_dim < 0 || (r->interleaved != 0 && r->interleaved != 1)) return RBS_ERR_INVALID_ARG;
  if (r->rot_dim > kHeadDim || r->rot_dim % 8 != 0) return RBS_ERR_UNSUPPORTED;
  if (r->rot_dim > 0 && r->inv_freq == nullptr) return RBS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(r->q_norm) % 16 != 0 || reinterpret_cast<uintptr_t>(r->k_norm) % 16 != 0) return RBS_ERR_INVALID_ARG;
  return RBS_OK;
}

static void set_rope(RopeParams& p, const rbs_rope* r) {
  p.positions = r->positions; p.inv_freq = r->inv_freq; p.q_norm = r->q_norm; p.k_norm = r->k_norm;
  p.eps = r->eps; p.magnitude = r->magnitude; p.rot = r->rot_dim;
}

// A token is spread over as many halves of warps as leave all CTAs resident at a time, four per SM, and over two where that
// does not fit.
static rbs_status launch_rope(RopeParams p, long long tokens, bool interleaved, bool paged, cudaStream_t s) {
  const long long room = 4ll * sm_count();
  p.halves = kRopeHalves;
  while (p.halves > kRopeHalves / kRopeTokens && (tokens * p.halves + kRopeHalves - 1) / kRopeHalves > room) p.halves /= 2;
  const long long per_cta = kRopeHalves / p.halves, ctas = (tokens + per_cta - 1) / per_cta;
  if (ctas > 0x7fffffffll) return RBS_ERR_UNSUPPORTED;
  p.tokens = tokens;
  auto* kernel = paged ? (interleaved ? rope_kernel<true, true> : rope_kernel<false, true>)
                       : (interleaved ? rope_kernel<true, false> : rope_kernel<false, false>);
  RBS_CUDA_OK(launch_pdl(kernel, static_cast<unsigned>(ctas), 1, kRopeThreads, 0, s, p));
  return RBS_OK;
}

}  // namespace rbs

extern "C" rbs_status rbs_qk_norm_rope(int batch, int n_tokens, int n_q_heads, int n_kv_heads, int head_dim, rbs_tensor Q,
                                       rbs_tensor K, const rbs_rope* rope, rbs_tensor Q_out, rbs_tensor K_out, void* stream) {
  using namespace rbs;
  NvtxRange range("rbs_qk_norm_rope");
  if (batch <= 0 || n_q_heads <= 0 || n_kv_heads <= 0) return RBS_ERR_INVALID_ARG;
  if (head_dim != kHeadDim) return RBS_ERR_UNSUPPORTED;
  rbs_status st = check_rope(rope, n_tokens);
  if (st != RBS_OK) return st;
  if ((st = check_tensor(Q)) != RBS_OK || (st = check_tensor(K)) != RBS_OK || (st = check_tensor(Q_out)) != RBS_OK ||
      (st = check_tensor(K_out)) != RBS_OK)
    return st;
  RopeParams p = {};
  p.Q = static_cast<const __nv_bfloat16*>(Q.ptr); p.qsb = Q.stride_batch; p.qst = Q.stride_token; p.qsh = Q.stride_head;
  p.K = static_cast<const __nv_bfloat16*>(K.ptr); p.ksb = K.stride_batch; p.kst = K.stride_token; p.ksh = K.stride_head;
  p.Qo = static_cast<__nv_bfloat16*>(Q_out.ptr); p.qosb = Q_out.stride_batch; p.qost = Q_out.stride_token; p.qosh = Q_out.stride_head;
  p.Ko = static_cast<__nv_bfloat16*>(K_out.ptr); p.kosb = K_out.stride_batch; p.kost = K_out.stride_token; p.kosh = K_out.stride_head;
  set_rope(p, rope);
  p.Hq = n_q_heads; p.Hkv = n_kv_heads; p.N = n_tokens; p.page = 1;
  return launch_rope(p, static_cast<long long>(batch) * n_tokens, rope->interleaved != 0, false, static_cast<cudaStream_t>(stream));
}

extern "C" rbs_status rbs_qk_norm_rope_paged(const rbs_paged_shape* shape, int n_tokens, rbs_tensor Q, rbs_tensor K,
                                             rbs_tensor V, const rbs_rope* rope, const int* slots, int n_slots,
                                             rbs_tensor Q_out, rbs_tensor K_out, rbs_tensor k_cache, rbs_tensor v_cache, void* stream) {
  using namespace rbs;
  NvtxRange range("rbs_qk_norm_rope_paged");
  rbs_status st = check_paged_cache(shape);
  if (st != RBS_OK || (st = check_rope(rope, n_tokens)) != RBS_OK) return st;
  if (n_slots < 0 || n_slots > n_tokens || (n_slots > 0 && slots == nullptr)) return RBS_ERR_INVALID_ARG;
  // rows have no batch stride here, and a tensor's stays out of the checks
  Q.stride_batch = K.stride_batch = V.stride_batch = Q_out.stride_batch = K_out.stride_batch = 0;
  if ((st = check_tensor(Q)) != RBS_OK || (st = check_tensor(K)) != RBS_OK || (st = check_tensor(V)) != RBS_OK ||
      (st = check_tensor(Q_out)) != RBS_OK || (st = check_tensor(k_cache)) != RBS_OK || (st = check_tensor(v_cache)) != RBS_OK)
    return st;
  if (K_out.ptr != nullptr && (st = check_tensor(K_out)) != RBS_OK) return st;
  RopeParams p = {};
  p.Q = static_cast<const __nv_bfloat16*>(Q.ptr); p.qst = Q.stride_token; p.qsh = Q.stride_head;
  p.K = static_cast<const __nv_bfloat16*>(K.ptr); p.kst = K.stride_token; p.ksh = K.stride_head;
  p.V = static_cast<const __nv_bfloat16*>(V.ptr); p.vst = V.stride_token; p.vsh = V.stride_head;
  p.Qo = static_cast<__nv_bfloat16*>(Q_out.ptr); p.qost = Q_out.stride_token; p.qosh = Q_out.stride_head;
  p.Ko = static_cast<__nv_bfloat16*>(K_out.ptr); p.kost = K_out.stride_token; p.kosh = K_out.stride_head;
  p.Kc = static_cast<__nv_bfloat16*>(k_cache.ptr); p.kcp = k_cache.stride_batch; p.kct = k_cache.stride_token; p.kch = k_cache.stride_head;
  p.Vc = static_cast<__nv_bfloat16*>(v_cache.ptr); p.vcp = v_cache.stride_batch; p.vct = v_cache.stride_token; p.vch = v_cache.stride_head;
  p.slots = slots;
  set_rope(p, rope);
  p.Hq = shape->n_q_heads; p.Hkv = shape->n_kv_heads; p.N = n_tokens; p.page = shape->page_size;
  p.slot_rows = n_slots; p.cache_rows = shape->n_pages * shape->page_size;
  return launch_rope(p, n_tokens, rope->interleaved != 0, true, static_cast<cudaStream_t>(stream));
}

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
};

// One warp per token, half a warp per row.  Lane u (of 16) of a row holds two groups A, B of four elements:
//   half layout, u < rot / 8: A = 4u.., B = rot/2 + 4u.., so that pair 4u + k is (A[k], B[k]);
//   otherwise 8 neighbours: A = 8u.., B = 8u + 4..; interleaved, pairs 4u .. 4u + 3 are (A0,A1) (A2,A3) (B0,B1) (B2,B3).
// In both layouts lane u turns pairs 4u .. 4u + 3 iff u < rot / 8: no exchange between lanes but the sum of squares.
template <bool INTERLEAVED, bool PAGED>
__global__ void __launch_bounds__(256)
rope_kernel(const RopeParams p) {
  const int lane = threadIdx.x & 31, u = lane & 15, side = lane >> 4;
  const bool turns = u < p.rot / 8;
  const int a = turns && !INTERLEAVED ? 4 * u : 8 * u;
  const int b = turns && !INTERLEAVED ? p.rot / 2 + 4 * u : 8 * u + 4;
  pdl_trigger();
  pdl_wait();
  // revolutions per position, in fp64: position * frequency is reduced to a part of a turn before it becomes fp32
  double turn[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) turn[k] = turns ? static_cast<double>(p.inv_freq[4 * u + k]) * 0.15915494309189535 : 0.0;

  const long long warps = static_cast<long long>(gridDim.x) * (blockDim.x >> 5);
  for (long long row = static_cast<long long>(blockIdx.x) * (blockDim.x >> 5) + (threadIdx.x >> 5); row < p.tokens; row += warps) {
    const int l = static_cast<int>(row / p.N), t = static_cast<int>(row - static_cast<long long>(l) * p.N);
    float cs[4], sn[4];
    const double pos = static_cast<double>(p.positions[t]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      double r = pos * turn[k];
      r -= rint(r);
      sincospif(2.0f * static_cast<float>(r), &sn[k], &cs[k]);
      const float m = turns ? p.magnitude : 1.0f;
      sn[k] *= m;
      cs[k] *= m;
    }
    int64_t page = 0, off = 0;
    bool kept = false;
    if (PAGED) {
      const int slot = t < p.slot_rows ? p.slots[t] : -1;
      kept = slot >= 0 && slot < p.cache_rows;
      if (kept) { page = slot / p.page; off = slot % p.page; }
    }
    const int rows = p.Hq + p.Hkv * (!PAGED ? 1 : kept ? 2 : p.Ko != nullptr ? 1 : 0);
    for (int h0 = 0; h0 < rows; h0 += 2) {
      const int h = h0 + side;
      const bool live = h < rows;
      const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
      const int hk = is_v ? h - p.Hq - p.Hkv : h - p.Hq;
      uint2 xa = make_uint2(0, 0), xb = make_uint2(0, 0);
      if (live) {
        const __nv_bfloat16* src = is_q ? p.Q + l * p.qsb + t * p.qst + h * p.qsh
                                 : is_v ? p.V + t * p.vst + hk * p.vsh : p.K + l * p.ksb + t * p.kst + hk * p.ksh;
        xa = *reinterpret_cast<const uint2*>(src + a);
        xb = *reinterpret_cast<const uint2*>(src + b);
      }
      float x[8] = {bf16lo(xa.x), bf16hi(xa.x), bf16lo(xa.y), bf16hi(xa.y), bf16lo(xb.x), bf16hi(xb.x), bf16lo(xb.y), bf16hi(xb.y)};
      const float* w = is_q ? p.q_norm : p.k_norm;
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) ss = fmaf(x[k], x[k], ss);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (live && !is_v) {
        if (w != nullptr) {
          const float r = rsqrtf(ss * (1.0f / kHeadDim) + p.eps);
          const float4 wa = *reinterpret_cast<const float4*>(w + a), wb = *reinterpret_cast<const float4*>(w + b);
          x[0] *= r * wa.x; x[1] *= r * wa.y; x[2] *= r * wa.z; x[3] *= r * wa.w;
          x[4] *= r * wb.x; x[5] *= r * wb.y; x[6] *= r * wb.z; x[7] *= r * wb.w;
        }
        if (turns) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float& y0 = INTERLEAVED ? x[2 * k] : x[k];
            float& y1 = INTERLEAVED ? x[2 * k + 1] : x[4 + k];
            const float n0 = y0 * cs[k] - y1 * sn[k], n1 = y1 * cs[k] + y0 * sn[k];
            y0 = n0;
            y1 = n1;
          }
        }
        xa = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
        xb = make_uint2(pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
      }
      if (!live) continue;
      auto put = [&](__nv_bfloat16* dst) {
        *reinterpret_cast<uint2*>(dst + a) = xa;
        *reinterpret_cast<uint2*>(dst + b) = xb;
      };
      if (is_q) put(p.Qo + l * p.qosb + t * p.qost + h * p.qosh);
      else if (is_v) put(p.Vc + page * p.vcp + off * p.vct + hk * p.vch);
      else {
        if (!PAGED || p.Ko != nullptr) put(p.Ko + l * p.kosb + t * p.kost + hk * p.kosh);
        if (PAGED && kept) put(p.Kc + page * p.kcp + off * p.kct + hk * p.kch);
      }
    }
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

static rbs_status launch_rope(const RopeParams& p, bool interleaved, bool paged, cudaStream_t s) {
  const long long want = (p.tokens + 7) / 8, most = static_cast<long long>(sm_count()) * 8;
  const unsigned ctas = static_cast<unsigned>(want < most ? want : most);
  auto* kernel = paged ? (interleaved ? rope_kernel<true, true> : rope_kernel<false, true>)
                       : (interleaved ? rope_kernel<true, false> : rope_kernel<false, false>);
  RBS_CUDA_OK(launch_pdl(kernel, ctas, 1, 256, 0, s, p));
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
  p.tokens = static_cast<long long>(batch) * n_tokens;
  return launch_rope(p, rope->interleaved != 0, false, static_cast<cudaStream_t>(stream));
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
  p.tokens = n_tokens;
  return launch_rope(p, rope->interleaved != 0, true, static_cast<cudaStream_t>(stream));
}

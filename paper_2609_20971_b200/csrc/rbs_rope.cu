// rbs_qk_norm_rope and rbs_qk_norm_rope_paged: norm of each head and rotation by position in one pass over the rows of Q
// and K (256 bytes each), in the paged form with the keys and the values going to their slots of the cache.
// A stream: 512 bytes read and written per row against some 50 instructions of half a warp.  128K tokens of 32 + 4 heads: 364 us
// = 6.64 TB/s, a little above what a plain copy reaches.  Instructions count all the same: with a quarter more of them (offsets by
// head, weights one by one, rsqrtf's care for denormals) 400 us.
#include <type_traits>

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
  int spread;            // log2 of the warps per token: 0 .. 3
};

constexpr int kRopeThreads = 256;
constexpr int kRopeWarps = kRopeThreads / 32;
constexpr int kRopeResident = 4;                 // CTAs of an SM
constexpr int kRopeAhead = 2;                    // groups of rows that a warp has in flight, in shared memory
constexpr int kRopeGroup = 2;                    // pairs of rows of a group: the shuffles of one pair fill the waits of the other

__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(d)) : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)));
  return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<uint64_t&>(d))
      : "l"(reinterpret_cast<uint64_t&>(a)), "l"(reinterpret_cast<uint64_t&>(b)), "l"(reinterpret_cast<uint64_t&>(c)));
  return d;
}

constexpr double kInvTwoPiLow = -9.839338337591243e-18;      // 1 / 2 pi - 0.15915494309189535
// of a normal number
__device__ __forceinline__ float fast_rsqrt(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Half a warp per row.  Lane u (of 16) of a row holds two groups A, B of four elements:
//   half layout, u < rot / 8: A = 4u.., B = rot/2 + 4u.., so that pair 4u + k is (A[k], B[k]);
//   otherwise 8 neighbours: A = 8u.., B = 8u + 4..; interleaved, pairs 4u .. 4u + 3 are (A0,A1) (A2,A3) (B0,B1) (B2,B3).
// In both layouts lane u turns pairs 4u .. 4u + 3 iff u < rot / 8: no exchange between lanes but the sum of squares, and
// an output may be its own input.  The norm's weights are in c and s, which stay in registers while a
// half walks over the heads of its token; 1 / sqrt(mean + eps) comes last.
// WHOLE: all of the head is turned.
template <bool INTERLEAVED, bool WHOLE>
struct RopeLane {
  float2 c[4], s[4];   // element j of this lane becomes x_j c_j + x_(partner of j) s_j
  int a, gap;          // A's first element, elements from there to B's: a constant where that helps
  float eps;
  bool turns;

  __device__ __forceinline__ void place(int rot) {
    const int u = threadIdx.x & 15;
    turns = WHOLE || u < rot / 8;
    a = turns && !INTERLEAVED ? 4 * u : 8 * u;
    gap = turns && !INTERLEAVED ? rot / 2 : 4;
  }
  __device__ __forceinline__ int to_b() const { return INTERLEAVED ? 4 : WHOLE ? kHeadDim / 2 : gap; }
  __device__ __forceinline__ void weigh(const float2* angles, const float* weights) {
    const int u = threadIdx.x & 15;
    const bool norm = weights != nullptr;
    float w[8], cj[8], sj[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = 1.0f;
    if (norm) {
      const float4 wa = *reinterpret_cast<const float4*>(weights + a), wb = *reinterpret_cast<const float4*>(weights + a + to_b());
      w[0] = wa.x; w[1] = wa.y; w[2] = wa.z; w[3] = wa.w;
      w[4] = wb.x; w[5] = wb.y; w[6] = wb.z; w[7] = wb.w;
    }
    float4 two[2] = {make_float4(1.f, 0.f, 1.f, 0.f), make_float4(1.f, 0.f, 1.f, 0.f)};
    if (WHOLE || turns) {
      two[0] = *reinterpret_cast<const float4*>(angles + 4 * u);
      two[1] = *reinterpret_cast<const float4*>(angles + 4 * u + 2);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 cs = k & 1 ? make_float2(two[k >> 1].z, two[k >> 1].w) : make_float2(two[k >> 1].x, two[k >> 1].y);
      const int f = INTERLEAVED ? 2 * k : k, g = INTERLEAVED ? 2 * k + 1 : 4 + k;
      cj[f] = w[f] * cs.x; sj[f] = -w[g] * cs.y;
      cj[g] = w[g] * cs.x; sj[g] = w[f] * cs.y;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c[k] = make_float2(cj[2 * k], cj[2 * k + 1]);
      s[k] = make_float2(sj[2 * k], sj[2 * k + 1]);
    }
  }
  // Two neighbouring elements at a time (packed fp32 instructions), N rows side by side.
  template <bool NORM, int N>
  __device__ __forceinline__ void turn(uint2 (&xa)[N], uint2 (&xb)[N]) const {
    float2 y[N][4];
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float2 x[4] = {make_float2(bf16lo(xa[i].x), bf16hi(xa[i].x)), make_float2(bf16lo(xa[i].y), bf16hi(xa[i].y)),
                           make_float2(bf16lo(xb[i].x), bf16hi(xb[i].x)), make_float2(bf16lo(xb[i].y), bf16hi(xb[i].y))};
#pragma unroll
      for (int k = 0; k < 4; ++k) y[i][k] = mul2(x[k], c[k]);
      if (WHOLE || turns) {      // elsewhere a zero would still carry an infinite neighbour over
#pragma unroll
        for (int k = 0; k < 4; ++k) y[i][k] = fma2(INTERLEAVED ? make_float2(x[k].y, x[k].x) : x[k ^ 2], s[k], y[i][k]);
      }
      float2 ss = mul2(x[0], x[0]);
#pragma unroll
      for (int k = 1; k < 4; ++k) ss = fma2(x[k], x[k], ss);
      sum[i] = ss.x + ss.y;
    }
    if (NORM) {
#pragma unroll
      for (int o = 8; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float r = fast_rsqrt(sum[i] * (1.0f / kHeadDim) + eps);
#pragma unroll
        for (int k = 0; k < 4; ++k) y[i][k] = mul2(y[i][k], make_float2(r, r));
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      xa[i] = make_uint2(pack_bf16(y[i][0].x, y[i][0].y), pack_bf16(y[i][1].x, y[i][1].y));
      xb[i] = make_uint2(pack_bf16(y[i][2].x, y[i][2].y), pack_bf16(y[i][3].x, y[i][3].y));
    }
  }
};

// The rows of one warp, two heads at a time, in order: its heads of Q, of K, of V.  kRopeAhead groups of kRopeGroup such pairs are on
// their way to a ring of its own in shared memory (in registers they would cost as many as the arithmetic; a chunk of 8,191 tokens
// of 64 heads takes 59.8 us pair by pair, 57.7 with two pairs).  All but the second head of a last pair is the same for both
// halves, so that the warp stays together: halves that went through loops of their own took twice the instructions (447 us instead
// of 367 for 128K tokens of 36 heads).
struct RopeRows {
  const __nv_bfloat16* at;       // this half's row that is fetched next, at this lane's 16 bytes
  int64_t skip;                  // elements from it to the one behind it
  int kind, left, mine;          // its kind; pairs of that kind that are left, and rows of this half
  uint32_t fill, read;           // shared memory: the group filled next at this lane's 16 bytes, and the one read next at its A;
  int hop;                       // from it to the ring's other one

  template <typename Open>
  __device__ __forceinline__ void fetch(Open& open) {
    if (left <= 0 && kind < 2) open(*this, kind + 1);
#pragma unroll
    for (int j = 0; j < kRopeGroup; ++j) {
      if (j < mine) cp_async16_zfill(fill + j * 512, at, true);
      at += skip;
    }
    left -= kRopeGroup;
    mine -= kRopeGroup;
    cp_async_commit();
    fill += hop;
    read += hop;
    hop = -hop;
  }
  // the next group has arrived: the address of A of this half's row of its first pair
  __device__ __forceinline__ uint32_t wait() {
    cp_async_wait<kRopeAhead - 1>();
    __syncwarp();
    return read;
  }
  template <typename Open>
  __device__ __forceinline__ void done(Open& open) {
    __syncwarp();
    fetch(open);
  }
};
// Both are filled before the first is read, and each is filled again as soon as it is read: the group to fill is the one to read.
static_assert(kRopeAhead == 2, "two groups take turns");
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}

// A CTA has eight warps, 2^spread for each of its tokens.  Its threads compute the tokens' angles once, behind the first rows'
// loads.
template <bool INTERLEAVED, bool WHOLE, bool PAGED>
__global__ void __launch_bounds__(kRopeThreads, kRopeResident)
rope_kernel(const RopeParams p) {
  __shared__ __align__(16) float2 angles[kRopeWarps][kHeadDim / 2];
  __shared__ __align__(16) unsigned char rings[kRopeWarps * kRopeAhead * kRopeGroup * 512];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), u = threadIdx.x & 15, side = (threadIdx.x >> 4) & 1;
  const int per_cta = kRopeWarps >> p.spread, mine = warp >> p.spread, pair0 = warp - (mine << p.spread), h0 = 2 * pair0 + side;
  const long long token0 = static_cast<long long>(blockIdx.x) * per_cta, token = token0 + mine;
  RopeLane<INTERLEAVED, WHOLE> lane;
  lane.place(p.rot);
  lane.eps = p.eps;
  pdl_trigger();
  pdl_wait();
  // What is needed behind the first rows' arrival is asked for before them: the frequency and the position of this thread's first
  // angle, and the norms' weights (to L2).
  const int k = threadIdx.x & (kHeadDim / 2 - 1), first = threadIdx.x / (kHeadDim / 2);
  const unsigned t0 = static_cast<unsigned>(token0 < p.N ? token0 : token0 % p.N);
  auto position = [&](int i) { return p.positions[t0 + i < static_cast<unsigned>(p.N) ? t0 + i : (t0 + i) % p.N]; };
  const bool angle = k < p.rot / 2 && first < per_cta && token0 + first < p.tokens;
  const float freq = angle ? p.inv_freq[k] : 0.f;
  int pos = angle ? position(first) : 0;
  if (p.spread > 0 && threadIdx.x < 2 * kHeadDim * 4 / 128) {
    const float* w = threadIdx.x & 1 ? p.k_norm : p.q_norm;
    if (w != nullptr) asm volatile("prefetch.global.L2 [%0];" ::"l"(w + (threadIdx.x >> 1) * 32));
  }
  const bool live = token < p.tokens;
  const int64_t l = token < p.N ? 0 : token / p.N, t = token - l * p.N;
  __nv_bfloat16 *kc = nullptr, *vc = nullptr;
  if (PAGED && live) {
    const int slot = t < p.slot_rows ? p.slots[t] : -1;
    if (slot >= 0 && slot < p.cache_rows) {
      const int64_t page = slot / p.page, off = slot - page * p.page;
      kc = p.Kc + page * p.kcp + off * p.kct;
      vc = p.Vc + page * p.vcp + off * p.vct;
    }
  }
  // pairs of heads of this warp
  auto pairs = [&](int heads) { return (((heads + 1) >> 1) - pair0 + (1 << p.spread) - 1) >> p.spread; };
  const int n_q = live ? pairs(p.Hq) : 0;
  const int n_k = live && (!PAGED || kc != nullptr || p.Ko != nullptr) ? pairs(p.Hkv) : 0;
  const int n_v = PAGED && vc != nullptr ? n_k : 0;
  const int step = 2 << p.spread;
  auto rows_of = [&](int heads) { return (heads - h0 + step - 1) >> (p.spread + 1); };      // of this half
  auto open = [&](RopeRows& r, int kind) {      // the first row of that kind, or of the next one that there is
    if (kind == 0 && n_q == 0) kind = 1;
    const bool q = kind == 0, k = kind == 1;
    if (!PAGED && !q && !k) return;
    const int64_t stride = q ? p.qsh : k ? p.ksh : p.vsh;
    r.at = (q ? p.Q + l * p.qsb + t * p.qst : k ? p.K + l * p.ksb + t * p.kst : p.V + t * p.vst) + h0 * stride + 8 * u;
    r.skip = step * stride;
    r.left = q ? n_q : k ? n_k : kind == 2 ? n_v : 0;
    r.kind = kind;
    r.mine = min(r.left, rows_of(q ? p.Hq : p.Hkv));
  };
  RopeRows rows;
  rows.left = rows.mine = 0;
  rows.fill = smem_u32(rings) + warp * kRopeAhead * kRopeGroup * 512 + side * 256 + u * 16;
  rows.read = rows.fill - u * 16 + lane.a * 2;
  rows.hop = kRopeGroup * 512;
  open(rows, 0);
#pragma unroll
  for (int i = 0; i < kRopeAhead; ++i) rows.fetch(open);

  // Angles in revolutions, as fractions of 2^64: positions are whole numbers, so whole revolutions of the frequency drop out of
  // the product by themselves.  The frequency is taken in two fp64 numbers (1 / 2 pi in 106 bits), off by 2^-64 of a revolution for
  // frequencies up to 2^40, which a position makes 2^-33 at most.  What counts is the fp32 number of half revolutions in front
  // of the sine: an angle is off by 2^-26 of a revolution, however far the position is.
  if (angle) {
    const double f = static_cast<double>(freq), high = f * 0.15915494309189535, low = fma(f, 0.15915494309189535, -high) + f * kInvTwoPiLow;
    auto of_turn = [](double x) { return static_cast<unsigned long long>(__double2ll_rn((x - rint(x)) * 18446744073709551616.0)); };
    const unsigned long long each = of_turn(high) + of_turn(low);
    const float magnitude = fabsf(freq) <= 3.4028235e38f ? p.magnitude : __int_as_float(0x7fffffff);      // no angle, no result
    for (int i = first;;) {
      float sn, cs;
      sincospif(static_cast<float>(static_cast<int>(static_cast<unsigned long long>(static_cast<long long>(pos)) * each >> 32)) *
                    4.656612873077393e-10f, &sn, &cs);      // 2^-31: in half revolutions
      angles[i][k] = make_float2(cs * magnitude, sn * magnitude);
      i += kRopeThreads / (kHeadDim / 2);
      if (i >= per_cta || token0 + i >= p.tokens) break;
      pos = position(i);
    }
  }
  __syncthreads();
  if (!live) return;

  // rows of `dst` (and of `dst2`) at this lane's A
  auto turn_rows = [&](auto norm, int n, int mine, __nv_bfloat16* dst, int64_t skip, __nv_bfloat16* dst2, int64_t skip2) {
    auto put = [&](__nv_bfloat16* at, const uint2& xa, const uint2& xb) {
      *reinterpret_cast<uint2*>(at) = xa;
      *reinterpret_cast<uint2*>(at + lane.to_b()) = xb;
    };
    for (; n > 0; n -= kRopeGroup, mine -= kRopeGroup) {
      const uint32_t from = rows.wait();
      uint2 xa[kRopeGroup], xb[kRopeGroup];
#pragma unroll
      for (int j = 0; j < kRopeGroup; ++j) {      // a row that is not there is turned and not written
        xa[j] = lds64(from + j * 512);
        xb[j] = lds64(from + j * 512 + lane.to_b() * 2);
      }
      rows.done(open);
      lane.template turn<decltype(norm)::value>(xa, xb);
#pragma unroll
      for (int j = 0; j < kRopeGroup; ++j) {
        if (j < mine) {
          if (!PAGED || dst != nullptr) put(dst, xa[j], xb[j]);
          if (PAGED && dst2 != nullptr) put(dst2, xa[j], xb[j]);
        }
        if (!PAGED || dst != nullptr) dst += skip;
        if (PAGED && dst2 != nullptr) dst2 += skip2;
      }
    }
  };
  if (n_q > 0) {
    lane.weigh(angles[mine], p.q_norm);
    __nv_bfloat16* out = p.Qo + l * p.qosb + t * p.qost + h0 * p.qosh + lane.a;
    if (p.q_norm != nullptr) turn_rows(std::true_type(), n_q, rows_of(p.Hq), out, step * p.qosh, nullptr, 0);
    else turn_rows(std::false_type(), n_q, rows_of(p.Hq), out, step * p.qosh, nullptr, 0);
  }
  if (n_k > 0) {
    lane.weigh(angles[mine], p.k_norm);
    __nv_bfloat16* out = PAGED && p.Ko == nullptr ? nullptr : p.Ko + l * p.kosb + t * p.kost + h0 * p.kosh + lane.a;
    __nv_bfloat16* out2 = PAGED && kc != nullptr ? kc + h0 * p.kch + lane.a : nullptr;
    if (p.k_norm != nullptr) turn_rows(std::true_type(), n_k, rows_of(p.Hkv), out, step * p.kosh, out2, step * p.kch);
    else turn_rows(std::false_type(), n_k, rows_of(p.Hkv), out, step * p.kosh, out2, step * p.kch);
  }
  if (PAGED) {
    __nv_bfloat16* dst = vc + h0 * p.vch + 8 * u;
    int mine = rows_of(p.Hkv);
    for (int n = n_v; n > 0; n -= kRopeGroup, mine -= kRopeGroup) {
      const uint32_t from = rows.wait() - lane.a * 2 + u * 16;
      uint4 x[kRopeGroup];
#pragma unroll
      for (int j = 0; j < kRopeGroup; ++j) x[j] = lds128(from + j * 512);
      rows.done(open);
#pragma unroll
      for (int j = 0; j < kRopeGroup; ++j, dst += step * p.vch)
        if (j < mine) *reinterpret_cast<uint4*>(dst) = x[j];
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
  p.eps = fmaxf(r->eps, 1.17549435e-38f); p.magnitude = r->magnitude; p.rot = r->rot_dim;
}

// A token is spread over as many of 8, 4, 2 warps as leave all CTAs resident at a time, and stays with one warp where that does not
// fit: a spread shortens the row of pairs that a warp goes through, and costs the weights of each warp.  us with 1 / 2 / 4 / 8 warps,
// 36 heads: 400 tokens 6.2 / 4.9 / 4.5 / 4.3; 1,003 7.9 / 7.3 / 6.3 / 7.7; 2,000 10.6 / 9.2 / 10.2 / 12.3; 3,000 12.2 / 13.1 / 13.6 / 16.8.
// Where a token has many rows two warps go on paying for four times as many (80 rows: 4,000 tokens 32.3 / 29.7, 8,000 56.3 / 55.4).
static rbs_status launch_rope(RopeParams p, long long tokens, bool interleaved, bool paged, cudaStream_t s) {
  const long long room = static_cast<long long>(kRopeResident) * sm_count() * kRopeWarps;
  const bool many = p.Hq + p.Hkv * (paged ? 2 : 1) >= 64;
  p.spread = tokens * 8 <= room ? 3 : tokens * 4 <= room ? 2 : tokens * 2 <= (many ? 4 : 1) * room ? 1 : 0;
  const long long per_cta = kRopeWarps >> p.spread, ctas = (tokens + per_cta - 1) / per_cta;
  if (ctas > 0x7fffffffll) return RBS_ERR_UNSUPPORTED;
  p.tokens = tokens;
  using Kernel = void (*)(const RopeParams);
  static const Kernel kernels[8] = {rope_kernel<false, false, false>, rope_kernel<false, false, true>, rope_kernel<false, true, false>,
                                    rope_kernel<false, true, true>,   rope_kernel<true, false, false>, rope_kernel<true, false, true>,
                                    rope_kernel<true, true, false>,   rope_kernel<true, true, true>};
  const Kernel kernel = kernels[(interleaved ? 4 : 0) + (p.rot == kHeadDim ? 2 : 0) + (paged ? 1 : 0)];
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
  if (batch > 1 && (Q_out.stride_batch == 0 || K_out.stride_batch == 0)) return RBS_ERR_INVALID_ARG;
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

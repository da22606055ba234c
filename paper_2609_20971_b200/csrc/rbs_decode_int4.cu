// rbs_paged_decode_int4: attention of one new token per sequence over a paged key/value cache held in 4 bits.
// The order of all work, its equal shares, the pieces and their joins are those of rbs_paged_decode (rbs_decode.cuh); tiles have 32
// tokens, because a row is a quarter as long.  Per token and KV head 144 bytes are read, against 256 numbers that have to be made
// from them, so the instructions of a warp are what has to be saved:
//   - four bits become fp16 numbers by one and-or for two of them (1024 + c or 64 + c, by where the bits stand) and one fused
//     multiply-add, s (1024 + c) - 1032 s, which is exact: (c - 8) s has at most 7 bits, 1032 s = 129 * 8 s has 11.
//   - rows are stored in their natural order; the elements of a row that meet in a step of the product over the head, and the
//     tokens that meet in a step of the product over the tokens, are chosen so that a lane finds all of its bits in 16 (keys)
//     or 8 (values) bytes in a row.
//   - a probability is two fp16 numbers of 11 bits each.
#include "rbs_decode.cuh"
#include "rbs_int4.cuh"

#include <cuda_fp16.h>
#include <string.h>

namespace rbs {

constexpr int kKeys4 = 32;                                              // tokens of a tile
constexpr int kCodes4 = kKeys4 * kHeadDim / 2, kScales4 = kKeys4 * 8;   // bytes of K's or V's
constexpr int kTile4 = 2 * (kCodes4 + kScales4);                        // codes of K, of V, scales of K, of V
constexpr int kStages4 = 2;

template <int HT>
struct Int4Tiles {
  static constexpr int kPerSm = HT == 1 ? 3 : 2;      // CTAs per SM
  // no second wave: the SMs' instructions bound large calls, not what each gets of the memory (64 sequences of 64 heads 84.4 -> 82.8 us)
  static constexpr int kWarps = 4, kWave = 148 * kPerSm, kRest = 0, kCtas = kWave, kRestTiles = 0;
  static constexpr int kKeys = kKeys4, kRing = kStages4 * kTile4, kSlots = kCtas * (2 + kWarps - 1), kItemCost = 2;
  static_assert(kRing >= HT * 8 * (kDecRow * 4 + 8), "an unfinished item is left in the ring");
};

// Probabilities are kept against 2^11 below the maximum (2^15 is the most that fp16 holds, 2^-24 the least): the maximum in use moves
// when a score passes it by 4 in units of log 2.
constexpr float kLift4 = 11.f, kSlack4 = 15.f;
constexpr float kValueScale = 8.f;      // scales are taken as fp16 numbers of an eighth of their value

struct Decode4Params : DecodeCommon {
  const unsigned char* K; int64_t kp, kt, kh;     // codes: page, token, head strides
  const unsigned char* V; int64_t vp, vt, vh;
  const unsigned char* KS; int64_t ksp, kst, ksh; // scales
  const unsigned char* VS; int64_t vsp, vst, vsh;
  Divide by_page;
};

// ------------------------------------------------------------------------------------------------ small things

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src));
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src));
}
__device__ __forceinline__ void cp_async8_zfill(uint32_t dst, const void* src, bool valid) {
  const uint32_t n = valid ? 8u : 0u;
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(n));
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}
__device__ __forceinline__ uint32_t lds1(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(at));
  return v;
}
__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
// D(16x8, fp32) += A(16x16, fp16, row) * B(16x8, fp16, col)
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// D = A * B
__device__ __forceinline__ void mma_f16_16816_zero(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// A pair of scales as fp16 numbers of an eighth of their value, and what takes the offset of the codes away: a scale byte is the upper
// byte but one bit of such a number (a byte of 255 is no number there as well).  The bytes are brought to their places by products,
// which leave the units of the masks and shifts alone (64 sequences of 64 heads 82.0 -> 81.2 us).
struct Scale2 {
  uint32_t s, low, high;
  __device__ __forceinline__ void set(uint32_t pair) {
    s = pair;
    low = h2_mul(s, 0xe408e408u);       // -1032
    high = h2_mul(s, 0xd480d480u);      // -72
  }
  __device__ __forceinline__ void set_both(uint32_t byte) { set(byte * 0x00800080u); }
  __device__ __forceinline__ void set_each(uint32_t lower, uint32_t upper) { set(lower * 0x80u + upper * 0x800000u); }
};
// An instruction has room for one constant: where the compiler knows both of (w & mask) | bits it makes two of it.  So the masks are
// in memory that it does not look into (1,027 -> 898 instructions of a warp per tile, 128K tokens 32.4 -> 29.6 us).
__constant__ uint32_t kMasks[2] = {0x000f000fu, 0x00f000f0u};

// (c - 8) s of the four pairs of codes in bits 4 j .. 4 j + 3 of the halves of w
__device__ __forceinline__ void expand(uint32_t w, const Scale2& s, uint32_t (&out)[4]) {
  const uint32_t v = w >> 8;
  out[0] = h2_fma((w & kMasks[0]) | 0x64006400u, s.s, s.low);
  out[1] = h2_fma((w & kMasks[1]) | 0x54005400u, s.s, s.high);
  out[2] = h2_fma((v & kMasks[0]) | 0x64006400u, s.s, s.low);
  out[3] = h2_fma((v & kMasks[1]) | 0x54005400u, s.s, s.high);
}

// Row k (0 .. 15) of a product's step over 16 tokens is token token_of(k): 2 t -> t, 2 t + 1 -> 4 + (t ^ 1), the same for the upper
// eight.  So the two tokens that a lane (g, t) multiplies its values of, and the two key rows that lanes next to each other
// read, stand in shared memory where no two of them meet in a bank (16-byte chunk c of row r stands at chunk c ^ (r & 2)).
__device__ __forceinline__ int token_of(int k) { return (k & 8) | (k & 1 ? 4 + ((k >> 1 & 3) ^ 1) : k >> 1 & 3); }

// ------------------------------------------------------------------------------------------------ queries

// Q^T of up to 8 * HT heads, the B operand of the eight steps over the head dimension: lane (g, t) has elements 32 t .. 32 t + 31 of heads
// 8 n + g, in fp16 and times the power of two that brings the head's largest element to [2^14, 2^15) (at most 2^127, which leaves
// subnormal ones between 2^-6 and 2).  So bf16 numbers of down to 2^-31 of the largest keep all of their bits and smaller ones are off by up to
// 2^-39 of it; sums of 128 products with keys of up to 8 * 480 / kValueScale stay below 2^31.
template <int HT>
struct Queries4 {
  uint4 raw[HT][4];      // bf16, as they are loaded
  uint32_t q[HT][16];
  float scale[HT][2];    // of heads 8 n + 2 t, + 1: what takes their sums to scores in units of log 2

  __device__ __forceinline__ void load(const __nv_bfloat16* Q, int64_t qsh, int heads) {
    const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
#pragma unroll
    for (int n = 0; n < HT; ++n) {
      const uint4* row = reinterpret_cast<const uint4*>(Q + (8 * n + g) * qsh + 32 * t);
#pragma unroll
      for (int i = 0; i < 4; ++i) raw[n][i] = 8 * n + g < heads ? row[i] : make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void convert(float scale_log2) {
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int n = 0; n < HT; ++n) {
      uint32_t top = 0;      // of the numbers' bits without sign, two at a time
#pragma unroll
      for (int i = 0; i < 4; ++i)
        top = __vmaxu2(__vmaxu2(__vmaxu2(top, raw[n][i].x & 0x7fff7fffu), __vmaxu2(raw[n][i].y & 0x7fff7fffu, raw[n][i].z & 0x7fff7fffu)),
                       raw[n][i].w & 0x7fff7fffu);
      uint32_t most = max(top & 0xffffu, top >> 16);
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
      const int power = min(141 - static_cast<int>(most >> 7), 127);      // 14 less the exponent of the largest
      // a negative scale goes into the queries
      const float down = __uint_as_float(static_cast<uint32_t>(127 + power) << 23 | (__float_as_uint(scale_log2) & 0x80000000u));
      // kValueScale |scale| / 2^power: what its parts make beyond 32 bits must not make it infinite, nor anything make it zero, which the
      // scores of zero and the scores of keys that are left out would not stand
      const int half = power / 2;
      const float halves[2] = {__uint_as_float(static_cast<uint32_t>(127 - half) << 23), __uint_as_float(static_cast<uint32_t>(127 + half - power) << 23)};
      const float up = fminf(fmaxf(fabsf(scale_log2) * halves[0] * kValueScale * halves[1], 0x1p-126f), 3.4028235e38f);
      scale[n][0] = __shfl_sync(0xffffffffu, up, 8 * t);
      scale[n][1] = __shfl_sync(0xffffffffu, up, 8 * t + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {      // eight elements: pairs j, j + 4
        const uint4 w = raw[n][i];
        q[n][4 * i + 0] = pack_half(bf16lo(w.x) * down, bf16lo(w.z) * down);
        q[n][4 * i + 1] = pack_half(bf16hi(w.x) * down, bf16hi(w.z) * down);
        q[n][4 * i + 2] = pack_half(bf16lo(w.y) * down, bf16lo(w.w) * down);
        q[n][4 * i + 3] = pack_half(bf16hi(w.y) * down, bf16hi(w.w) * down);
      }
    }
  }
};

// ------------------------------------------------------------------------------------------------ softmax over a warp's keys

// As in rbs_decode.cu, S^T = K Q^T and O^T += V^T P^T with 16 tokens and 8 heads to a product.  Lane (g, t) = (lane / 4, lane % 4) has heads
// 2 t, 2 t + 1 of each group of 8: of S^T tokens token_of(g) and token_of(g + 8), of O^T elements 16 g + 2 j (o[.][j][0], o[.][j][1]) and
// 16 g + 2 j + 1 (o[.][j][2], o[.][j][3]).
template <int HT>
struct Softmax4 {
  float o[HT][8][4];
  float m[HT][2], l[HT][2];   // maximum in use less kLift4, log2 units; sum over this lane's keys

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

  // Probabilities c of the 32 keys of a tile against the maximum in use; `valid`: a bit per key.
  __device__ __forceinline__ void scores(const Queries4<HT>& q, uint32_t tile, uint32_t valid, float (&c)[2][HT][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3, row = token_of(g);
    const uint32_t codes = tile + row * 64 + ((t ^ (row & 2)) << 4), scales = tile + 2 * kCodes4 + row * 8 + 2 * t;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4 lo = lds16(codes + h * 1024), hi = lds16(codes + h * 1024 + 512);
      const uint32_t slo[2] = {lds1(scales + h * 128), lds1(scales + h * 128 + 1)}, shi[2] = {lds1(scales + h * 128 + 64), lds1(scales + h * 128 + 65)};
      const uint32_t wlo[4] = {lo.x, lo.y, lo.z, lo.w}, whi[4] = {hi.x, hi.y, hi.z, hi.w};
      float c2[HT][4];
      Scale2 sa, sb;
#pragma unroll
      for (int w = 0; w < 4; ++w) {      // eight elements of each row; two sums of four steps: half as many roundings in a row
        if (w % 2 == 0) {
          sa.set_both(slo[w / 2]);
          sb.set_both(shi[w / 2]);
        }
        uint32_t x[4], y[4];
        expand(wlo[w], sa, x);
        expand(whi[w], sb, y);
        const uint32_t a[4] = {x[0], y[0], x[1], y[1]}, b[4] = {x[2], y[2], x[3], y[3]};
#pragma unroll
        for (int n = 0; n < HT; ++n) {
          if (w == 0) {
            mma_f16_16816_zero(c[h][n], a, q.q[n][0], q.q[n][1]);
            mma_f16_16816_zero(c2[n], b, q.q[n][2], q.q[n][3]);
          } else {
            mma_f16_16816(c[h][n], a, q.q[n][4 * w], q.q[n][4 * w + 1]);
            mma_f16_16816(c2[n], b, q.q[n][4 * w + 2], q.q[n][4 * w + 3]);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < HT; ++n)
#pragma unroll
        for (int i = 0; i < 4; i += 2) add_pair(c[h][n] + i, c2[n] + i);
    }
    // c: sums, not yet times q.scale, which is above zero
    if (valid != 0xffffffffu) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool first = valid >> (16 * h + row) & 1, second = valid >> (16 * h + 8 + row) & 1;
#pragma unroll
        for (int n = 0; n < HT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            c[h][n][i] = first ? c[h][n][i] : -INFINITY;
            c[h][n][i + 2] = second ? c[h][n][i + 2] : -INFINITY;
          }
      }
    }
    float top[HT][2];
    bool move = false;
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        top[n][i] = fmaxf(fmaxf(c[0][n][i], c[0][n][i + 2]), fmaxf(c[1][n][i], c[1][n][i + 2])) * q.scale[n][i];
        move |= top[n][i] > m[n][i] + kSlack4;
      }
    if (__any_sync(0xffffffffu, move)) {
#pragma unroll
      for (int n = 0; n < HT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float high = top[n][i];
#pragma unroll
          for (int s = 4; s < 32; s <<= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, s));
          high = fmaxf(high - kLift4, m[n][i]);
          const float fade = fast_exp2(m[n][i] - exp_base(high));
          m[n][i] = high;
          l[n][i] *= fade;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            o[n][j][i] *= fade;
            o[n][j][i + 2] *= fade;
          }
        }
    }
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float base = -exp_base(m[n][i]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          c[h][n][i] = fast_exp2(fmaf(c[h][n][i], q.scale[n][i], base));
          c[h][n][i + 2] = fast_exp2(fmaf(c[h][n][i + 2], q.scale[n][i], base));
        }
        l[n][i] += (c[0][n][i] + c[0][n][i + 2]) + (c[1][n][i] + c[1][n][i + 2]);
      }
  }

  // Adds P V of a tile.  A probability of up to 2^15 goes into the product as two fp16 numbers, its first 11 bits and what is left, to 2^-22
  // of it (2^-24 at the least, which is 2^-35 of the largest probability).  One number takes 81 us instead of 92 (64 sequences of 64 heads),
  // but leaves values that cancel 11 bits, and outputs differ from those of 32-bit operations by 6e-4 of their norm instead of 6e-5.
  // The sums of the product drop bits in one direction, so a tile is summed from zero, the small parts first, and added by itself.
  __device__ __forceinline__ void values(uint32_t tile, const float (&c)[2][HT][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint32_t p[2][2][HT][2];      // half of the tile; what is left, first bits
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < HT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float x = c[h][n][2 * i], y = c[h][n][2 * i + 1];
          const float fx = __uint_as_float(__float_as_uint(x) & 0xffffe000u), fy = __uint_as_float(__float_as_uint(y) & 0xffffe000u);
          p[h][1][n][i] = transpose_8x8(pack_half(fx, fy));
          p[h][0][n][i] = transpose_8x8(pack_half(x - fx, y - fy));
        }
    // tokens t, 4 + (t ^ 1) and those eight further on; elements 16 g .. 16 g + 15
    const int other = 4 + (t ^ 1);
    const uint32_t chunk = (((g >> 1) ^ (t & 2)) << 4) + ((g & 1) << 3);
    const uint32_t ta = tile + kCodes4 + t * 64 + chunk, tb = tile + kCodes4 + other * 64 + chunk;
    const uint32_t sa = tile + 2 * kCodes4 + kScales4 + t * 8 + g, sb = tile + 2 * kCodes4 + kScales4 + other * 8 + g;
    uint2 a[2][2], b[2][2];
    Scale2 s[2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        a[h][e] = lds8(ta + h * 1024 + e * 512);
        b[h][e] = lds8(tb + h * 1024 + e * 512);
        s[h][e].set_each(lds1(sa + h * 128 + e * 64), lds1(sb + h * 128 + e * 64));
      }
#pragma unroll
    for (int k = 0; k < 4; ++k) {      // elements 16 g + 4 k .. + 3
      float sum[2][HT][4];
      uint32_t v[2][2][4];             // half, step j of two, operand
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t x[4], y[4];
        expand(__byte_perm(k < 2 ? a[h][0].x : a[h][0].y, k < 2 ? b[h][0].x : b[h][0].y, k % 2 ? 0x7632 : 0x5410), s[h][0], x);
        expand(__byte_perm(k < 2 ? a[h][1].x : a[h][1].y, k < 2 ? b[h][1].x : b[h][1].y, k % 2 ? 0x7632 : 0x5410), s[h][1], y);
        v[h][0][0] = x[0]; v[h][0][1] = x[1]; v[h][0][2] = y[0]; v[h][0][3] = y[1];
        v[h][1][0] = x[2]; v[h][1][1] = x[3]; v[h][1][2] = y[2]; v[h][1][3] = y[3];
      }
#pragma unroll
      for (int part = 0; part < 2; ++part)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int n = 0; n < HT; ++n) {
              if (part == 0 && h == 0) mma_f16_16816_zero(sum[j][n], v[h][j], p[h][part][n][0], p[h][part][n][1]);
              else mma_f16_16816(sum[j][n], v[h][j], p[h][part][n][0], p[h][part][n][1]);
            }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < HT; ++n)
#pragma unroll
          for (int i = 0; i < 4; i += 2) add_pair(o[n][2 * k + j] + i, sum[j][n] + i);
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
  __device__ __forceinline__ void write(const DecodeCommon& p, int s, int h0, int heads) const {
    if (!RBS_DBG_OK(s >= 0 && s < p.S && h0 >= 0 && heads > 0 && h0 + heads <= p.Hq, p.status, kDbgDecodeRow)) return;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int n = 0; n < HT; ++n)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int h = 8 * n + 2 * t + i;
        if (h >= heads) continue;
        const float inv = l[n][i] == 0.f ? 0.f : kValueScale / l[n][i];
        if (p.lse != nullptr && g == 0) p.lse[static_cast<int64_t>(s) * p.Hq + h0 + h] = lse_of(m[n][i], l[n][i]);
        uint32_t x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = pack_bf16(o[n][j][i] * inv, o[n][j][i + 2] * inv);
        uint4* row = reinterpret_cast<uint4*>(p.O + s * p.ost + (h0 + h) * p.osh + 16 * g);
        row[0] = make_uint4(x[0], x[1], x[2], x[3]);
        row[1] = make_uint4(x[4], x[5], x[6], x[7]);
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
        float4* row = reinterpret_cast<float4*>(rows + h * stride + 16 * g);
#pragma unroll
        for (int j = 0; j < 8; j += 2)
          row[j / 2] = make_float4(o[n][j][i] * kValueScale, o[n][j][i + 2] * kValueScale, o[n][j + 1][i] * kValueScale, o[n][j + 1][i + 2] * kValueScale);
      }
  }
};

// ------------------------------------------------------------------------------------------------ tiles on their way

// What a warp copies: the tiles of its share, item by item; all that changes from item to item is done at an item's end.  Rows that are not
// there become zeros (codes of 0 with a scale of 0: zeros), so that no stale page contents reach a product.
// RUNS: pages hold halves of a tile (16 tokens) as one run of bytes per tensor -- rows of a head one behind the other, page_size a multiple
// of 16.  A lane copies from its half's page, four times 16 bytes of codes that lie 256 apart, so a whole tile is four addresses and ten
// copies at constant distances from them.  (Bulk copies need their operands in uniform registers: eight lanes' copies, which differ, were
// run one after the other, and a tile took 138 instructions to copy.)
// Otherwise lane r has the table entry of row r, and a row's codes are copied by four lanes.
template <class C, bool RUNS>
struct Source {
  Place at;                       // the item's first tile of the share
  unsigned end;                   // the unit where the share ends
  int left;                       // tiles of the item that are not begun yet; 0: none of the share
  bool ends;                      // the share reaches the item's end
  const int* row;                 // of the block table
  const unsigned char *k, *v, *ks, *vs;      // RUNS: this lane's bytes of page 0 at the item's head
  int next;                       // of the next tile: token of this lane (RUNS: the first one of its half), ..
  int page, offset, count;        // .. its page, row in the page, and how many tokens from there on

  __device__ __forceinline__ void look_up(const Decode4Params& p) {
    const int index = p.by_page(next);
    offset = next - index * p.P;
    count = at.len - next;
    page = count > 0 ? row[index] : -1;
    next += kKeys4;
  }
  __device__ __forceinline__ void item(const Decode4Params& p) {
    const int whole = at.n - at.tile, lane = threadIdx.x & 31;
    left = min(whole, static_cast<int>(end - at.unit));
    ends = left == whole;
    row = p.table + static_cast<int64_t>(at.s) * p.stride;
    next = at.tile * kKeys4 + (RUNS ? lane & 16 : lane);
    if (RUNS) {
      k = p.K + at.hk * p.kh + (lane & 15) * 16;
      v = p.V + at.hk * p.vh + (lane & 15) * 16;
      ks = p.KS + at.hk * p.ksh + (lane & 15) * 8;
      vs = p.VS + at.hk * p.vsh + (lane & 15) * 8;
    }
    look_up(p);
  }
  // Begins a tile, if there is one.  `keys`: a bit per token; true if it is the last one of its item.
  __device__ __forceinline__ bool begin(const Decode4Params& p, uint32_t tile, uint32_t& keys) {
    keys = RUNS ? copy_runs(p, tile) : copy_rows(p, tile);
    if (--left > 0) {
      look_up(p);
      return false;
    }
    if (!ends) return false;
    at.unit += at.n - at.tile + C::kItemCost;
    if (at.unit < end) {
      at.tile = 0;
      if (++at.cut == p.cuts) {
        at.cut = 0;
        ++at.hk;
      }
      if (++at.item == p.items) {
        at.item = at.hk = at.cut = 0;
        ++at.s;
        at.len = clamped(p, at.next_len);
        at.n = tiles_of<C>(at.len);
        at.next_len = read_len(p, at.s + 1);
      }
      item(p);
    }
    return true;
  }
  __device__ __forceinline__ uint32_t copy_runs(const Decode4Params& p, uint32_t tile) const {
    const int lane = threadIdx.x & 31, r = lane >> 2 & 3;      // row of the half, less a multiple of 4
    const bool there = page >= 0 && page < p.n_pages;
    const uint32_t in = there ? page : 0;
    const uint64_t row64 = static_cast<uint32_t>(offset), at64 = row64 * 64, at8 = row64 * 8;      // beyond 32 bits in pages of 2^26 tokens and more
    // a 32-bit number times a 64-bit one
    auto from = [&](const unsigned char* base, int64_t stride) { return base + in * static_cast<uint64_t>(stride); };
    const unsigned char *from_k = from(k, p.kp) + at64, *from_v = from(v, p.vp) + at64, *from_ks = from(ks, p.ksp) + at8, *from_vs = from(vs, p.vsp) + at8;
    const uint32_t to = tile + (lane >> 4) * 1024 + r * 64 + (((lane & 3) ^ (r & 2)) << 4), to_s = tile + 2 * kCodes4 + lane * 8;
    if (__all_sync(0xffffffffu, there && count >= 16)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        cp_async16(to + i * 256, from_k + i * 256);
        cp_async16(to + kCodes4 + i * 256, from_v + i * 256);
      }
      cp_async8(to_s, from_ks);
      cp_async8(to_s + kScales4, from_vs);
      return 0xffffffffu;
    }
    const uint32_t mine = there ? 0xffffu >> (16 - min(count, 16)) : 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool ok = mine >> (4 * i + r) & 1;
      cp_async16_zfill(to + i * 256, from_k + i * 256, ok);
      cp_async16_zfill(to + kCodes4 + i * 256, from_v + i * 256, ok);
    }
    const bool ok = mine >> (lane & 15) & 1;
    cp_async8_zfill(to_s, from_ks, ok);
    cp_async8_zfill(to_s + kScales4, from_vs, ok);
    return __shfl_sync(0xffffffffu, mine, 0) | __shfl_sync(0xffffffffu, mine, 16) << 16;
  }
  __device__ __forceinline__ uint32_t copy_rows(const Decode4Params& p, uint32_t tile) const {
    const bool there = page >= 0 && page < p.n_pages;
    const int lane = threadIdx.x & 31, chunk = lane & 3;
    const uint32_t valid = __ballot_sync(0xffffffffu, there);
    const int64_t in = there ? page : 0, head = at.hk;
    const int off = there ? offset : 0;
    const int64_t k = in * p.kp + off * p.kt + head * p.kh, v = in * p.vp + off * p.vt + head * p.vh;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 8 * i + (lane >> 2);
      const bool ok = valid >> r & 1;
      const uint32_t to = tile + r * 64 + ((chunk ^ (r & 2)) << 4);
      cp_async16_zfill(to, p.K + __shfl_sync(0xffffffffu, k, r) + chunk * 16, ok);
      cp_async16_zfill(to + kCodes4, p.V + __shfl_sync(0xffffffffu, v, r) + chunk * 16, ok);
    }
    cp_async8_zfill(tile + 2 * kCodes4 + lane * 8, p.KS + in * p.ksp + off * p.kst + head * p.ksh, there);
    cp_async8_zfill(tile + 2 * kCodes4 + kScales4 + lane * 8, p.VS + in * p.vsp + off * p.vst + head * p.vsh, there);
    return valid;
  }
};

template <int HT, bool RUNS>
__global__ void __launch_bounds__(Int4Tiles<HT>::kWarps * 32, Int4Tiles<HT>::kPerSm)
decode_int4_kernel(const Decode4Params p) {
  using C = Int4Tiles<HT>;
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ Piece pieces[2 * C::kWarps];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  unsigned char* ring_bytes = smem + warp * C::kRing;
  const uint32_t ring = smem_u32(ring_bytes);
  if (lane < 2) pieces[2 * warp + lane].flags = 0;
  pdl_wait();
  Source<C, RUNS> source;
  Place& at = source.at;
  const Share<C> share = find_share<C>(p, at);
  if (blockIdx.x >= share.cuts.ctas) {
    if (threadIdx.x == 0) p.found[blockIdx.x] = make_int4(-1, 0, 0, 0);
    return;
  }
  // the item that the CTA finds begun, for the kernel that joins: warp 0's share begins where the CTA's does
  const int4 begun = make_int4(at.tile == 0 ? -1 : at.s, (at.hk * p.G + at.cut * p.gh) | min(p.gh, p.G - at.cut * p.gh) << 24, at.unit - at.tile,
                               at.unit - at.tile + at.n - 1);
  auto write_found = [&]() {
    if (threadIdx.x == 0)
      p.found[blockIdx.x] = begun.x < 0 ? begun
                                        : make_int4(begun.x, begun.y, share.cuts.cta_of(begun.z), share.cuts.cta_of(begun.w));
  };
  if (at.unit < share.end) {
    int s = at.s, hk = at.hk, cut = at.cut, item = at.item;      // the item that is summed
    bool begun_here = at.tile == 0, finished = false;

    // tile i + 1 is on its way while tile i is worked on, the table entries of tile i + 2 as well
    source.end = share.end;
    source.item(p);
    uint32_t valid[kStages4];
    unsigned state[kStages4];
    constexpr unsigned kTile = 1, kLast = 2;      // there is a tile; it is the last one of its item
    auto begin_tile = [&](uint32_t tile, uint32_t& keys) {
      unsigned word = 0;
      if (source.left > 0) word = source.begin(p, tile, keys) ? kTile | kLast : kTile;
      cp_async_commit();
      return word;
    };
#pragma unroll
    for (int i = 0; i < kStages4; ++i) state[i] = begin_tile(ring + i * kTile4, valid[i]);

    write_found();
    Queries4<HT> q;
    int h0, heads;
    auto begin_item = [&]() {
      h0 = hk * p.G + cut * p.gh;
      heads = min(p.gh, p.G - cut * p.gh);
      q.load(p.Q + s * p.qst + h0 * p.qsh, p.qsh, heads);
      q.convert(p.scale_log2);
    };
    begin_item();
    Softmax4<HT> sm;
    sm.start();
    for (uint32_t tile = ring; state[0] != 0; tile = tile == ring + (kStages4 - 1) * kTile4 ? ring : tile + kTile4) {
      const unsigned word = state[0];
      float pr[2][HT][4];
      cp_async_wait<kStages4 - 1>();
      __syncwarp();
      sm.scores(q, tile, valid[0], pr);
      sm.values(tile, pr);
      __syncwarp();
#pragma unroll
      for (int i = 0; i + 1 < kStages4; ++i) state[i] = state[i + 1], valid[i] = valid[i + 1];
      state[kStages4 - 1] = begin_tile(tile, valid[kStages4 - 1]);
      finished = word & kLast;
      if (!finished) continue;

      // the end of the item
      sm.finish();
      if (begun_here) {
        sm.write(p, s, h0, heads);
      } else {
        const int64_t slot = warp == 0 ? 2 * blockIdx.x : 2 * C::kCtas + (C::kWarps - 1) * blockIdx.x + warp - 1;
        if (RBS_DBG_OK(slot >= 0 && slot < C::kSlots, p.status, kDbgDecodeSlot))
          sm.put(p.part_o + slot * (HT * 8) * kHeadDim, kHeadDim, p.part_ml + slot * (HT * 8));
        if (warp > 0 && lane == 0) pieces[2 * warp] = {kPieceThere | kPieceEnds, s, h0 | heads << 24};
      }
      begun_here = true;
      if (++cut == p.cuts) { cut = 0; ++hk; }
      if (++item == p.items) { item = hk = 0; ++s; }
      if (state[0] != 0) {
        begin_item();
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
  join_pieces<C, HT>(p, smem, pieces);
}

template <int HT>
static rbs_status decode_int4(Decode4Params& p, bool runs, void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  using C = Int4Tiles<HT>;
  unsigned ctas = 0;
  rbs_status st = decode_grid<C>(p, workspace, workspace_bytes, &ctas);
  if (st != RBS_OK) return st;
  auto* kernel = runs ? decode_int4_kernel<HT, true> : decode_int4_kernel<HT, false>;
  const size_t smem = static_cast<size_t>(C::kWarps) * C::kRing;
  if ((st = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem)) != RBS_OK) return st;
  RBS_CUDA_OK(launch_pdl(kernel, ctas, 1, C::kWarps * 32, smem, stream, p));
  RBS_CUDA_OK(launch_pdl(join_kernel<C, HT>, ctas, 1, kJoinThreads, 0, stream, static_cast<const DecodeCommon&>(p)));
  return RBS_OK;
}

}  // namespace rbs

extern "C" size_t rbs_paged_decode_int4_workspace_bytes(const rbs_paged_shape* shape) {
  using namespace rbs;
  if (check_paged_table(shape) != RBS_OK || check_paged_cache(shape) != RBS_OK) return 0;
  const int G = shape->n_q_heads / shape->n_kv_heads;
  return G <= 8 ? decode_workspace<Int4Tiles<1>>(G).bytes : decode_workspace<Int4Tiles<2>>(G).bytes;
}

extern "C" rbs_status rbs_paged_decode_int4(const rbs_paged_shape* shape, rbs_tensor Q, rbs_cache_int4 k_cache, rbs_cache_int4 v_cache,
                                            const int* block_table, const int* seq_lens, rbs_tensor O, float* lse,
                                            float softmax_scale, void* workspace, size_t workspace_bytes, void* stream) {
  using namespace rbs;
  NvtxRange range("rbs_paged_decode_int4");
  Decode4Params p = {};
  rbs_status st = decode_arguments(p, shape, Q, block_table, seq_lens, O, lse, softmax_scale);
  if (st != RBS_OK || (st = check_cache_int4(k_cache)) != RBS_OK || (st = check_cache_int4(v_cache)) != RBS_OK) return st;
  auto take = [](const unsigned char*& ptr, int64_t& page, int64_t& token, int64_t& head, const rbs_tensor& t) {
    ptr = static_cast<const unsigned char*>(t.ptr);
    page = t.stride_batch; token = t.stride_token; head = t.stride_head;
  };
  take(p.K, p.kp, p.kt, p.kh, k_cache.codes);
  take(p.V, p.vp, p.vt, p.vh, v_cache.codes);
  take(p.KS, p.ksp, p.kst, p.ksh, k_cache.scales);
  take(p.VS, p.vsp, p.vst, p.vsh, v_cache.scales);
  auto run = [](const rbs_tensor& codes, const rbs_tensor& scales) { return codes.stride_token == 64 && scales.stride_token == 8; };
  const bool runs = p.P % 16 == 0 && run(k_cache.codes, k_cache.scales) && run(v_cache.codes, v_cache.scales);
  p.by_page.set(p.P);
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  return p.gh <= 8 ? decode_int4<1>(p, runs, workspace, workspace_bytes, cs) : decode_int4<2>(p, runs, workspace, workspace_bytes, cs);
}

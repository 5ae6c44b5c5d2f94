// The KV pool in 4 bits (RECG_FLAG_KV_4BIT).
//
// A row x (one token, one kv head, K or V; d values) is held as d codes c of 4 bits, a minimum m and a step s:
//   m = min x,  s = bf16((max x - m) / 15),  c = nearest whole number to (x - m) / s, ties to even (0 where s is 0)
// and stands for m + s c.  m is one of the bf16 inputs, hence exact in 16 bits; s rounded to bf16 moves the largest value by at
// most 15 s 2^-8 = 0.06 s, an eighth of what rounding to codes does.  One pair (s, m) per row, not per 32 or 64 values: the
// products q.(m + s c) = s (q.c) + m sum(q) and sum_j p_j (m_j + s_j c_j) then need the pairs outside of the matrix products
// only, whose operands, the codes, are exact.  A row with a value that is not finite (or whose range overflows) gets s = NaN.
//
// Pool = [layer][page][kv_head] blocks of 16 d + 128 bytes, one bulk copy each:
//   [K codes: 16 tokens x d/2 bytes][V codes][K pairs: 16 x {s, m} bf16][V pairs]
// The codes of eight consecutive values 8 j .. 8 j + 7 make one 32-bit word: nibble i of the low half is value 8 j + 2 i, nibble
// i of the high half value 8 j + 2 i + 1, so that (word >> 4 i) & 0x000f000f is a pair of neighbours, as a matrix operand
// along the values takes them.  K: word j of token t at t d/2 + 4 j.  V is contracted over tokens: the halves of the words of tokens
// 2 p and 2 p + 1 are exchanged, the even values' halves at p d + 8 j and the odd values' at p d + 8 j + 4, token 2 p low and
// 2 p + 1 high.  A lane of an mma.sync B operand thus finds all it needs of a token (K) or token pair (V) in one 16-byte read.
#pragma once
#include "common.cuh"

namespace recg {

__host__ __device__ constexpr int kv4_block_bytes(int d) { return 16 * d + 128; }
__host__ __device__ constexpr int kv4_v_codes(int d) { return 8 * d; }      // offsets inside a block
__host__ __device__ constexpr int kv4_k_pairs(int d) { return 16 * d; }
__host__ __device__ constexpr int kv4_v_pairs(int d) { return 16 * d + 64; }
__host__ __device__ __forceinline__ size_t kv4_block_base(int64_t n_pages, int n_kv, int d, int layer, int64_t page, int kv_head) {
  return (((size_t)layer * n_pages + page) * n_kv + kv_head) * (size_t)kv4_block_bytes(d);
}
__host__ __device__ __forceinline__ int kv4_k_word(int tok, int j, int d) { return tok * (d >> 1) + 4 * j; }
__host__ __device__ __forceinline__ int kv4_v_word(int tok, int j, int odd, int d) { return kv4_v_codes(d) + (tok >> 1) * d + 8 * j + 4 * odd; }

__device__ __forceinline__ float pow2(int e) { return __int_as_float((127 + e) << 23); }       // 2^e, a normal number
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// {s, m} of a row
__device__ __forceinline__ float kv4_step(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float kv4_min(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {       // of bf16 pairs; NaN stays
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Which of its neighbours a value on the border between two codes (or next to it) goes to: r the bits of the code tried, e = a - r s,
// |e| at least half a step.  On the border to the even one, or, where a = x - lo was rounded onto it, to where the difference lies.
__device__ __forceinline__ uint32_t kv4_settle(uint32_t r, float e, float half, float x, float lo, float a) {
  const int toward = e > 0.f ? 1 : -1;
  if (fabsf(e) > half) return r + toward;
  if (fabsf(e) < half) return r;
  const float back = __fsub_rn(a, x), err = __fsub_rn(__fsub_rn(x, __fsub_rn(a, back)), __fadd_rn(lo, back));      // (x - lo) - a
  return (err == 0.f ? (r & 1u) != 0 : (err > 0.f) == (toward > 0)) ? r + toward : r;
}
// Eight values of a row, whose other values the LANES threads around this one (consecutive lanes of a warp, aligned) hold:
// their word of codes; *pair receives the row's {s, m}.
template <int LANES>
__device__ __forceinline__ uint32_t kv4_quantise(const uint4& raw, uint32_t* pair) {
  const uint32_t in[4] = {raw.x, raw.y, raw.z, raw.w};
  // {max x, max -x} of the row as a bf16 pair
  const uint32_t up = max2_nan(max2_nan(in[0], in[1]), max2_nan(in[2], in[3]));
  const uint32_t down = max2_nan(max2_nan(in[0] ^ 0x80008000u, in[1] ^ 0x80008000u), max2_nan(in[2] ^ 0x80008000u, in[3] ^ 0x80008000u));
  uint32_t top = max2_nan(__byte_perm(up, down, 0x5410), __byte_perm(up, down, 0x7632));
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) top = max2_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
  const float hi = __uint_as_float(top << 16), lo = __uint_as_float((top & 0xffff0000u) ^ 0x80000000u);
  // the quotient by 15, correctly rounded: the reciprocal is, and one step of the remainder follows
  const float span = __fsub_rn(hi, lo), first = __fmul_rn(span, 1.f / 15.f);
  const __nv_bfloat16 step = __float2bfloat16_rn(__fmaf_rn(__fmaf_rn(-first, 15.f, span), 1.f / 15.f, first));
  uint32_t sb = __bfloat16_as_ushort(step);
  if ((sb & 0x7f80u) == 0x7f80u) sb = 0x7fc0u;          // a value, or the range, is not finite
  else if ((sb & 0x7f80u) < 0x0400u) sb = 0;            // (a step below 2^-119, whose half may be no normal number: the row is its minimum)
  *pair = sb | (__float_as_uint(lo) & 0xffff0000u);
  const float s = __uint_as_float(sb << 16);
  if (!(s > 0.f)) return 0;
  // 2^23 + 2^22 added to a number below 2^22 rounds it to a whole one, which then stands in the low bits (conversion instructions run at an
  // eighth of the rate).  r is the quotient rounded, or next to it; the remainder e = a - r s is exact and says whether: it is as long as the
  // reciprocal is good to 2^-19.  Every code is a nibble of the word: a sum of bits << shift, less that of the bits of 0.
  constexpr float kWhole = 12582912.f;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  const float half = .5f * s;
  const float2 lo2 = make_float2(-lo, -lo), inv2 = make_float2(inv, inv), whole2 = make_float2(kWhole, kWhole), minus2 = make_float2(-kWhole, -kWhole),
               s2 = make_float2(-s, -s);
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x = make_float2(__uint_as_float(in[i] << 16), __uint_as_float(in[i] & 0xffff0000u)), a = add2(x, lo2), q = fma2(a, inv2, whole2),
                 e = fma2(add2(q, minus2), s2, a);
    uint32_t r0 = __float_as_uint(q.x), r1 = __float_as_uint(q.y);
    if (fmaxf(fabsf(e.x), fabsf(e.y)) >= half) {
      r0 = kv4_settle(r0, e.x, half, x.x, lo, a.x);
      r1 = kv4_settle(r1, e.y, half, x.y, lo, a.y);
    }
    word += (r0 << (4 * i)) + (r1 << (4 * i + 16));
  }
  constexpr uint32_t kZero = 0x4b400000u;               // the bits of kWhole
  return word - (kZero + (kZero << 4) + (kZero << 8) + (kZero << 12) + (kZero << 16) + (kZero << 20) + (kZero << 24) + (kZero << 28));
}
// The eight bf16 values that a word stands for, rounded once, in pairs: 128 + c is the bf16 number 0x4300 | c.  (In fp32, with a
// conversion at the end, reading was bound by instructions: 14400 rows of 8 heads 17.4 us, now 14.6.)
__device__ __forceinline__ uint4 kv4_values(uint32_t word, uint32_t pair) {
  const uint32_t s = __byte_perm(pair, pair, 0x1010), m = __byte_perm(pair, pair, 0x3232);
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t c;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(((word >> (4 * i)) & 0x000f000fu) | 0x43004300u), "r"(0x43004300u));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(out[i]) : "r"(s), "r"(c), "r"(m));
  }
  return make_uint4(out[0], out[1], out[2], out[3]);
}

}  // namespace recg

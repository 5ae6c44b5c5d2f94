// The KV pool in 4 bits (RECG_FLAG_KV_4BIT).
//
// A row x (one token, one kv head, K or V; d values) is held as d codes c of 4 bits, a minimum m and a step s:
//   m = min x,  s = bf16((max x - m) / 15),  c = nearest whole number to (x - m) / s, ties to even (0 where s is 0)
// and stands for m + s c.  m is one of the bf16 inputs, hence exact in 16 bits; s rounded to bf16 moves the largest value by at
// most 15 s 2^-9 = 0.03 s, a sixteenth of what rounding to codes does.  One pair (s, m) per row, not per 32 or 64 values: the
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

// Pair i of a word of codes as two bf16 values c - 8 (exact: 128 + c is 0x4300 | c, and 136 is subtracted).  Centred, because sums
// of products with values of one sign grow and lose low bits in the accumulators of the matrix units.
__device__ __forceinline__ uint32_t kv4_pair(uint32_t word, int i) {
  const uint32_t x = ((word >> (4 * i)) & 0x000f000fu) | 0x43004300u;
  const __nv_bfloat162 off = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));   // 136
  const __nv_bfloat162 r = __hsub2(reinterpret_cast<const __nv_bfloat162&>(x), off);
  return reinterpret_cast<const uint32_t&>(r);
}
// {s, m} of a row
__device__ __forceinline__ float kv4_step(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float kv4_min(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// Eight values of a row, whose other values the LANES threads around this one (consecutive lanes of a warp, aligned) hold:
// their word of codes; *pair receives the row's {s, m}.
template <int LANES>
__device__ __forceinline__ uint32_t kv4_quantise(const uint4& raw, uint32_t* pair) {
  const uint32_t in[4] = {raw.x, raw.y, raw.z, raw.w};
  float x[8];
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(in[i] << 16);
    x[2 * i + 1] = __uint_as_float(in[i] & 0xffff0000u);
    bad |= (in[i] & 0x7f80u) == 0x7f80u || (in[i] & 0x7f800000u) == 0x7f800000u;
  }
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
  }
#pragma unroll
  for (int o = LANES / 2; o; o >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    bad |= __shfl_xor_sync(0xffffffffu, (int)bad, o) != 0;
  }
  const __nv_bfloat16 step = __float2bfloat16_rn(__fdiv_rn(__fsub_rn(hi, lo), 15.f));
  uint32_t sb = __bfloat16_as_ushort(step);
  if (bad || (sb & 0x7f80u) == 0x7f80u) sb = 0x7fc0u;
  else if ((sb & 0x7f80u) < 0x0400u) sb = 0;            // (a step below 2^-119, whose half may be no normal number: the row is its minimum)
  *pair = sb | (__float_as_uint(lo) & 0xffff0000u);
  const float s = __uint_as_float(sb << 16);
  if (!(s > 0.f)) return 0;
  const float inv = __frcp_rn(s), half = .5f * s;
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // r is the quotient rounded, or next to it; the remainder a - r s is exact and says which
    const float a = __fsub_rn(x[i], lo);
    float r = rintf(a * inv);
    const float e = __fmaf_rn(-r, s, a);
    if (e > half) r += 1.f;
    else if (e < -half) r -= 1.f;
    else if (fabsf(e) == half) {                        // on the border, or a was rounded onto it
      const float low = e > 0.f ? r : r - 1.f;
      const double at = (double)x[i] - (double)lo, border = ((double)low + .5) * (double)s;
      r = at > border ? low + 1.f : (at < border ? low : 2.f * rintf(.5f * (low + .5f)));
    }
    const uint32_t c = (uint32_t)fminf(fmaxf(r, 0.f), 15.f);
    word |= c << (4 * (i >> 1) + 16 * (i & 1));
  }
  return word;
}
// the eight bf16 values that a word stands for
__device__ __forceinline__ uint4 kv4_values(uint32_t word, uint32_t pair) {
  const float s = kv4_step(pair), m = kv4_min(pair);
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    out[i] = pack_bf16(__fmaf_rn(s, (float)((word >> (4 * i)) & 15u), m), __fmaf_rn(s, (float)((word >> (4 * i + 16)) & 15u), m));
  return make_uint4(out[0], out[1], out[2], out[3]);
}

}  // namespace recg

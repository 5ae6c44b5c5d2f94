// Hybrid-mask paged attention over a pool in 4 bits on the 5th-generation tensor cores (head_dim 128, many query rows per kv head).
//
// Work items, masks and the combine kernel are those of attention_tc.cu.  The operands are fp16: with x = m + s c (kv4.cuh) a product
// s (c - 8) of an 8-bit step and a code has 11 significant bits, which is what fp16 holds, and so have q and m.  Hence
//   score = q . (s_K (c_K - 8))  +  (m_K + 8 s_K) sum(q)
// is exact up to fp32 sums: the second term is one more step of 16 of the contraction, in which both factors stand as sums of
// two fp16 numbers.  (K as m + s c rounded to 16 bits would leave the log-sum-exp of a few tokens good to 1e-4 only; steps applied
// in fp32 behind the product have to be broadcast to every row's thread, and that alone took more of the shared memory's
// bandwidth than all operands: 325 us instead of the 192 us that this took then, for 1001 rows over 6000 tokens of 40 / 8 heads.)
// V stands as m + s c rounded once, and P as fp16 too: 2^-11 of each term by either, a quarter of the rounding of the result together.
//
// Range.  fp16 has five bits of exponent, so everything is scaled by powers of two, in steps of 2^8: a query row by its own largest
// value, K and V of 32 tokens by theirs, or, where tokens lie 2^16 apart, each by its own (a row may see one and not the other).  The
// scale of a row of Q and of 32 tokens of K is one factor of the score, that of a single token is applied to it.  The scale of V joins
// the exponent of the probabilities, relative to the largest one that the row has seen (its O is rescaled when that grows); that of
// a single token is applied to P.  So K and V lose at most what is 2^-20 of the largest of their 32 tokens where none lies below 2^-16 of
// it, and P what is 2^-31 of the reference, 2^(e - e_j) times as much for a token whose V is on a scale 2^(e - e_j) below the row's.
//
// Per CTA (20 warps = 5 warpgroups, one CTA per SM, persistent over the work list), stages of 128 tokens:
//   warp 0     streams the blocks of the pool (codes and pairs of a page and head: one bulk copy) into a ring of two raw stages, and
//              the item's Q rows by TMA
//   warps 4-7  turn a raw stage into the operand K (K-major) and warps 8-11 into V (MN-major), 32 tokens a warp: 16 tokens x 128 values
//              in 128-byte-swizzled atoms as the tensor core reads them.  Every lane turns words of eight codes into 16-byte stores;
//              the words of a lane are taken in an order in which no two lanes of a store meet a bank.  Warps 4-7 also turn the
//              rows of Q, one a thread.  (One warpgroup for both had a chain of latencies longer than a stage: 272 us, where two took 201 at the time.)
//   warp 1     one elected lane issues S = Q K^T (two stages ahead) and per softmax group O_g += P_g V_g (P from TMEM)
//   warps 12-15 and 16-19  two softmax groups: group g takes tokens [64 g, 64 g + 64) of every stage, one thread one query row, its
//              own O accumulator and running (reference maximum, sum); merged at the end of an item.
// The registers are moved to the softmax warps: 4 x (56 + 64 + 64 + 144 + 144) x 32 of the 20 x 96 x 32 of the launch.
// Every wait is bounded; a wait that runs out raises a CTA-wide flag after which no wait blocks, so the kernel always ends.
#include <cuda_fp16.h>
#include <cstdio>

#include "attention_tc.cuh"
#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

constexpr int D = 128;
constexpr int kBT = 128;                         // tokens per stage
constexpr int kPages = kBT / kPageSize;
constexpr int kBlock = kv4_block_bytes(D);       // 2176
constexpr int kRawBytes = kPages * kBlock;
constexpr int kOperand = kBT * D * 2;            // 32 KB: K or V of a stage, or Q
constexpr int kRaw = 2, kRing = 2;               // raw stages; stages of K and of V operands
constexpr int kInfo = 4;                         // stages of what the softmax needs to know of 32 tokens (see the writer)
constexpr int kExt = 128 * 32;                   // the 16 further values of the contraction: 128 rows x 32 bytes, not swizzled
constexpr int kThreads = 640;
constexpr uint32_t kSpin = 1u << 22;             // polls of a wait
constexpr int kTmemCols = 512;                   // two S buffers of 128 columns; O of group g at 256 + 128 g
constexpr int kTmemO = 2 * kBT;
constexpr float kNoRef = -1e30f;       // reference maximum of a row that has seen no token yet
constexpr int kNoScale = -1000;        // scale of its O
constexpr float kHeadroom = 8.f;       // a row's reference maximum moves when it is outgrown by more than 2^8
constexpr float kLift = 7.f;           // probabilities stand as 2^7 p: at most 2^15, and 2^-31 of the reference is not lost yet

constexpr int kOffQ = 0;
constexpr int kOffK = kOffQ + kOperand;
constexpr int kOffV = kOffK + kRing * kOperand;
constexpr int kOffQExt = kOffV + kRing * kOperand;
constexpr int kOffKExt = kOffQExt + kExt;
constexpr int kOffRaw = kOffKExt + kRing * kExt;
constexpr int kOffScratch = kOffRaw + kRaw * kRawBytes;            // 2 KB per softmax warp: partial rows on their way out
constexpr int kOffML = kOffScratch + 8 * 2048;                     // per row, both groups: reference; sum; scale of O
constexpr int kOffQF = kOffML + 3 * 2 * 128 * 4;                   // per row: the factor of its scores
constexpr int kOffInfo = kOffQF + 128 * 4;                         // [kInfo][4] of 32 tokens: K stands scaled by 1 / x, V by 2^-y; z: those whose V
                                                                   // is not finite (it stands as zero, a row that sees one is NaN); w: 1, 2 where
                                                                   // K, V of every token stand on a scale of their own (x is 1, y the largest)
constexpr int kOffExp = kOffInfo + kInfo * 4 * 16;                 // [kInfo][128] those scales: two signed bytes
constexpr int kOffBar = kOffExp + kInfo * 128 * 2;
constexpr int kNumBars = 2 * kRaw + 4 * kRing + 3 + 2 + 4 + 3;
constexpr int kSmemBytes = kOffBar + kNumBars * 8 + 16;
static_assert(kSmemBytes <= 227 * 1024, "shared memory budget");

struct Params {
  const AttnItem* items;
  const int* cta_off;
  const int* page_table;
  int pt_stride;
  const int* tok_climit;
  const int* tok_lo;
  const int* tok_hi;
  __nv_bfloat16* o;
  float* lse;
  const uint8_t* pool;
  int64_t n_pages;
  int layer, n_q, n_kv, group;
  float scale_log2;
  float* part_o;
  float* part_ml;
  int* status;
};

__device__ __forceinline__ void softmax_bar() { asm volatile("bar.sync 1, 256;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void regs_inc() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_dec() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

constexpr uint32_t kIdescF16QK = kIdescQK & ~((1u << 7) | (1u << 10));      // fp16 operands
constexpr uint32_t kIdescF16PV = kIdescPV & ~((1u << 7) | (1u << 10));
// K-major operand of 16 values per row without swizzle: 8 rows x 16 bytes make a core matrix, the second one 128 bytes behind the
// first, the next 8 rows 256 bytes
__device__ __forceinline__ uint64_t desc_ext(uint32_t addr) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(128 >> 4) << 16) | ((uint64_t)(256 >> 4) << 32) | ((uint64_t)1 << 46);
}
__device__ __forceinline__ int ext_row(int row) { return (row >> 3) * 256 + (row & 7) * 16; }

// A bounded wait that sleeps NS nanoseconds between polls: 20 warps that poll take issue slots from those that work.
template <int NS>
__device__ __forceinline__ bool wait_asleep(uint64_t* bar, uint32_t parity) {
#pragma unroll 1
  for (uint32_t i = 0; i < kSpin; ++i) {
    __nanosleep(NS);
    if (mbar_test_wait(bar, parity)) return true;
  }
  return false;
}

// Multiples of eight E with 2^-E v in [1, 2^8) for the v whose exponent field is `field` (clamped where a factor 2^E or 2^-E would
// not be a normal number, or products of two not)
__device__ __forceinline__ int scale_exp(int field) { return max(-56, min(120, ((field - 127) >> 3) << 3)); }
// The scales of 32 tokens, a token a lane, of which `top` is the largest value (0: nothing that has to be held).
struct Scale {
  int all, own;
  bool loses;      // this token is two steps of 2^8 or more below the scale of all
};
__device__ __forceinline__ Scale token_scale(float top) {
  Scale s;
  const int field = __float_as_int(top) >> 23;
  s.own = scale_exp(field);
  s.all = scale_exp(__reduce_max_sync(0xffffffffu, field));
  s.loses = top > 0.f && s.own + 8 < s.all;
  return s;
}
// the largest value of V of a token with this {step, minimum}
__device__ __forceinline__ float v_top(uint32_t pair, bool* bad) {
  *bad = (pair & 0x7f80u) == 0x7f80u;
  return *bad ? 0.f : fmaxf(fabsf(kv4_min(pair)), fabsf(fmaf(15.f, kv4_step(pair), kv4_min(pair))));
}
__device__ __forceinline__ uint32_t h2_bits(const __half2& h) { return reinterpret_cast<const uint32_t&>(h); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { return h2_bits(__floats2half2_rn(lo, hi)); }
__device__ __forceinline__ uint32_t add_h2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
// The constants of a conversion.  They are made where the compiler does not see their values: it would split every (word & mask) |
// exponent into two instructions with an immediate each.
struct CodeConst {
  uint32_t exponent, whole, part, sixteenth;      // 1024 in both halves; off - 1024, off - 64; 1 / 16
};
__device__ __forceinline__ uint32_t opaque(uint32_t v) {
  uint32_t d;
  asm volatile("mov.b32 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}
__device__ __forceinline__ CodeConst code_const(float off) {
  return CodeConst{opaque(0x64006400u), opaque(pack_f16(off - 1024.f, off - 1024.f)), opaque(pack_f16(off - 64.f, off - 64.f)), opaque(0x2c002c00u)};
}
template <uint32_t MASK>
__device__ __forceinline__ uint32_t code_bits(uint32_t w, uint32_t exponent) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(w), "n"(MASK), "r"(exponent));     // (w & MASK) | exponent
  return d;
}
// the pairs of a word of codes as fp16 c + off: 1024 + c is 0x6400 | c, 1024 + 16 c is 0x6400 | (c << 4)
__device__ __forceinline__ void word_codes(uint32_t w, const CodeConst& k, uint32_t (&x)[4]) {
  const uint32_t v = w >> 8;
  x[0] = add_h2(code_bits<0x000f000fu>(w, k.exponent), k.whole);
  x[1] = fma_h2(code_bits<0x00f000f0u>(w, k.exponent), k.sixteenth, k.part);
  x[2] = add_h2(code_bits<0x000f000fu>(v, k.exponent), k.whole);
  x[3] = fma_h2(code_bits<0x00f000f0u>(v, k.exponent), k.sixteenth, k.part);
}
// s (c - 8), exact; m + s c, rounded once
__device__ __forceinline__ uint4 k_values(uint32_t w, const CodeConst& k, uint32_t s) {
  uint32_t x[4];
  word_codes(w, k, x);
  return make_uint4(mul_h2(x[0], s), mul_h2(x[1], s), mul_h2(x[2], s), mul_h2(x[3], s));
}
__device__ __forceinline__ uint4 v_values(uint32_t w, const CodeConst& k, uint32_t s, uint32_t m) {
  uint32_t x[4];
  word_codes(w, k, x);
  return make_uint4(fma_h2(x[0], s, m), fma_h2(x[1], s, m), fma_h2(x[2], s, m), fma_h2(x[3], s, m));
}

__global__ void __launch_bounds__(kThreads, 1) attention_kv4_tc_kernel(const __grid_constant__ CUtensorMap qmap, Params P) {
  extern __shared__ __align__(1024) uint8_t smem[];
  if (smem_u32(smem) & 1023u) {          // the swizzled operand layouts need a 1 KB aligned base
    if (threadIdx.x == 0) set_status(P.status, DEV_BAD_INDEX);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBar);
  uint64_t* raw_full = bars;                     // [kRaw]
  uint64_t* raw_empty = raw_full + kRaw;         // [kRaw]   the eight converting warps
  uint64_t* k_full = raw_empty + kRaw;           // [kRing]
  uint64_t* k_empty = k_full + kRing;
  uint64_t* v_full = k_empty + kRing;
  uint64_t* v_empty = v_full + kRing;
  uint64_t* q_full = v_empty + kRing;            // [1]
  uint64_t* q_empty = q_full + 1;                // [1]   the item's last S product, and the eight softmax warps (factor of the row)
  uint64_t* q_ready = q_empty + 1;               // [1]   the four converting warps
  uint64_t* s_full = q_ready + 1;                // [2]   per S buffer
  uint64_t* p_full = s_full + 2;                 // [4]   2 g + (stage & 1)
  uint64_t* pv_done = p_full + 4;
  uint64_t* o_full = pv_done + 1;
  uint64_t* o_empty = o_full + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* ml_smem = reinterpret_cast<float*>(smem + kOffML);
  float* qf_smem = reinterpret_cast<float*>(smem + kOffQF);
  // (the MMA issuer and the softmax warps, whom the stage waits for, poll more often)
  auto bwait = [&](uint64_t* bar, uint32_t parity, int code) {
    if (mbar_test_wait(bar, parity) || *abort_flag) return;
    if (!wait_asleep<20>(bar, parity)) {
      set_status(P.status, code);
      *abort_flag = 1;
    }
  };
  auto lazy_wait = [&](uint64_t* bar, uint32_t parity, int code) {
    if (mbar_test_wait(bar, parity) || *abort_flag) return;
    if (!wait_asleep<100>(bar, parity)) {
      set_status(P.status, code);
      *abort_flag = 1;
    }
  };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kRaw; ++s) {
      mbar_init(&raw_full[s], 1);
      mbar_init(&raw_empty[s], 8);
    }
    for (int s = 0; s < kRing; ++s) {
      mbar_init(&k_full[s], 4);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_full[s], 4);
      mbar_init(&v_empty[s], 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 9);
    mbar_init(q_ready, 4);
    for (int s = 0; s < 2; ++s) mbar_init(&s_full[s], 1);
    for (int s = 0; s < 4; ++s) mbar_init(&p_full[s], 4);
    mbar_init(pv_done, 1);
    mbar_init(o_full, 1);
    mbar_init(o_empty, 8);
    fence_barrier_init();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&qmap) : "memory");
  }
  for (int i = threadIdx.x; i < (1 + kRing) * kExt / 16; i += kThreads)     // (12 of the 16 further values stay zero)
    reinterpret_cast<uint4*>(smem + kOffQExt)[i] = make_uint4(0, 0, 0, 0);
  fence_proxy_async();
  if (warp == 1) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const uint32_t smem_base = smem_u32(smem);
  griddep_wait();

  // the CTA walks two ranges of the item list one after the other (see the layout kernel)
  const int4 r4 = *reinterpret_cast<const int4*>(P.cta_off + 4 * blockIdx.x);
  const int range_n0 = r4.y - r4.x, item_end = range_n0 + (r4.w - r4.z);
  auto item_at = [&](int i) { return i < range_n0 ? r4.x + i : r4.z + (i - range_n0); };
  auto stages_of = [&](const AttnItem& w) { return (min(w.blk_end * 64, w.kv_len) - w.blk_begin * 64 + kBT - 1) / kBT; };

  if (warp < 4) {
    regs_dec<56>();
    if (warp == 0) {
      // ------------------------------------ producer: raw stages and Q ------------------------------------
      uint32_t blk = 0;
      for (int item = 0; item < item_end; ++item) {
        const AttnItem w = P.items[item_at(item)];
        const int tok_begin = w.blk_begin * 64, tok_end = min(w.blk_end * 64, w.kv_len), nblk = stages_of(w);
        const int* pt = P.page_table + (size_t)w.req * P.pt_stride;
        auto fetch_page = [&](int n) -> int {        // lanes 0..7, one stage ahead of their use
          const int pos = tok_begin + n * kBT + lane * kPageSize;
          return lane < kPages && n < nblk && pos < tok_end ? __ldg(pt + pos / kPageSize) : -1;
        };
        int pg_next = fetch_page(0);
        for (int n = 0; n < nblk; ++n, ++blk) {
          int my_pg = pg_next;
          pg_next = fetch_page(n + 1);
          if (my_pg >= P.n_pages) {
            set_status(P.status, DEV_BAD_INDEX);
            my_pg = -1;
          }
          const int s = blk % kRaw;
          lazy_wait(&raw_empty[s], ((blk / kRaw) & 1) ^ 1, DEV_TIMEOUT_EMPTY);
          const unsigned mask = __ballot_sync(0xffffffffu, my_pg >= 0);
          if (lane == 0) {
            if (mask == 0) mbar_arrive(&raw_full[s]);
            else mbar_arrive_expect_tx(&raw_full[s], __popc(mask) * kBlock);
          }
          __syncwarp();
          if (my_pg >= 0)
            bulk_g2s(smem + kOffRaw + s * kRawBytes + lane * kBlock, P.pool + kv4_block_base(P.n_pages, P.n_kv, D, P.layer, my_pg, w.kv_head),
                     kBlock, &raw_full[s]);
          __syncwarp();
          if (n == 0) {
            // Q rows of the item (see attention_tc.cu); the first raw stage went ahead, since the item before may still read its Q
            lazy_wait(q_empty, (item & 1) ^ 1, DEV_TIMEOUT_EMPTY);
            if (lane == 0) {
              mbar_arrive_expect_tx(q_full, 2u * 128u * (uint32_t)(P.group * (128 / P.group)));
              tma_load_3d(smem_base + kOffQ, &qmap, 0, w.kv_head * P.group, w.tok0, q_full);
              tma_load_3d(smem_base + kOffQ + kOperand / 2, &qmap, 64, w.kv_head * P.group, w.tok0, q_full);
            }
            __syncwarp();
          }
        }
      }
      if (*abort_flag && lane == 0) {     // gave up somewhere: let the copies in flight land before exiting
        for (int s = 0; s < kRaw + 1; ++s)
          for (uint32_t i = 0; i < (1u << 14); ++i) {
            uint64_t* b = s < kRaw ? &raw_full[s] : q_full;
            if (mbar_try_wait(b, 0) || mbar_try_wait(b, 1)) break;
            __nanosleep(64);
          }
      }
    } else if (warp == 1) {
      // ------------------------------------ MMA issuer ------------------------------------
      if (elect_one()) {
        uint32_t blk = 0;
        const uint64_t dq0 = desc_kmajor(smem_base + kOffQ), dq1 = desc_ext(smem_base + kOffQExt);
        for (int item = 0; item < item_end; ++item) {
          const AttnItem w = P.items[item_at(item)];
          const int nblk = stages_of(w);
          auto issue_qk = [&](uint32_t b, bool last) {
            const int s = b % kRing;
            bwait(&k_full[s], (b / kRing) & 1, DEV_TIMEOUT_FULL);
            tc_fence_after();
            const uint64_t dk0 = desc_kmajor(smem_base + kOffK + s * kOperand, 2048);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)
              umma_bf16(tmem_base + (b & 1) * kBT, dq0 + (uint64_t)((((kk >> 2) * (128 * 128)) + (kk & 3) * 32) >> 4),
                        dk0 + (uint64_t)((((kk >> 2) * 1024) + (kk & 3) * 32) >> 4), kIdescF16QK, kk ? 1u : 0u);
            umma_bf16(tmem_base + (b & 1) * kBT, dq1, desc_ext(smem_base + kOffKExt + s * kExt), kIdescF16QK, 1u);
            umma_commit(&s_full[b & 1]);
            umma_commit(&k_empty[s]);
            if (last) umma_commit(q_empty);
          };
          bwait(q_ready, item & 1, DEV_TIMEOUT_FULL);
          tc_fence_after();
          issue_qk(blk, nblk == 1);
          if (nblk > 1) issue_qk(blk + 1, nblk == 2);
          for (int n = 0; n < nblk; ++n, ++blk) {
            const int s = blk % kRing;
            const uint64_t dv0 = desc_mnmajor(smem_base + kOffV + s * kOperand, 1024, 2048);
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              bwait(&p_full[2 * g + (blk & 1)], (blk >> 1) & 1, DEV_TIMEOUT_MMA);
              if (g == 0) {
                if (n == 0) bwait(o_empty, (item & 1) ^ 1, DEV_TIMEOUT_MMA);
                bwait(&v_full[s], (blk / kRing) & 1, DEV_TIMEOUT_FULL);
              }
              tc_fence_after();
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)
                umma_bf16_ts(tmem_base + kTmemO + g * D, tmem_base + (blk & 1) * kBT + g * 64 + kk * 8,
                             dv0 + (uint64_t)(((4 * g + kk) * 4096) >> 4), kIdescF16PV, (n | kk) ? 1u : 0u);
            }
            umma_commit(pv_done);
            umma_commit(&v_empty[s]);
            if (n == nblk - 1) umma_commit(o_full);
            if (n + 2 < nblk) issue_qk(blk + 2, n + 3 == nblk);
          }
        }
      }
    }
  } else if (warp < 8) {
    // ------------------------------------ codes to K; the rows of Q ------------------------------------
    regs_dec<64>();
    const CodeConst kc = code_const(-8.f);
    const int wq = warp - 4;                     // takes tokens [32 wq, 32 wq + 32) of every stage, and rows 32 wq .. of Q
    uint32_t blk = 0;
    for (int item = 0; item < item_end; ++item) {
      const AttnItem w = P.items[item_at(item)];
      const int nblk = stages_of(w), tok_begin = w.blk_begin * 64, tok_end = min(w.blk_end * 64, w.kv_len);
      for (int n = 0; n < nblk; ++n, ++blk) {
        const int rs = blk % kRaw, s = blk % kRing;
        const uint8_t* raw = smem + kOffRaw + rs * kRawBytes + 2 * wq * kBlock;
        lazy_wait(&raw_full[rs], (blk / kRaw) & 1, DEV_TIMEOUT_FULL);
        // ---- steps and minima, a token a lane: what is not there, or not finite, counts nothing ----
        const uint8_t* pg = raw + (lane >> 4) * kBlock;
        const bool there = tok_begin + n * kBT + 32 * wq + lane < tok_end;
        const uint32_t kp = there ? *reinterpret_cast<const uint32_t*>(pg + kv4_k_pairs(D) + 4 * (lane & 15)) : 0u;
        const uint32_t vp = there ? *reinterpret_cast<const uint32_t*>(pg + kv4_v_pairs(D) + 4 * (lane & 15)) : 0u;
        const float k_mid = fmaf(8.f, kv4_step(kp), kv4_min(kp));                       // m + 8 s
        const float k_top = (kp & 0x7f80u) == 0x7f80u ? 0.f : fmaxf(fabsf(k_mid), 8.f * kv4_step(kp));
        bool v_bad;
        const Scale k_scale = token_scale(k_top), v_scale = token_scale(v_top(vp, &v_bad));
        const unsigned bad = __ballot_sync(0xffffffffu, v_bad);
        int apart = 0;
        if (__any_sync(0xffffffffu, k_scale.loses || v_scale.loses))
          apart = (__any_sync(0xffffffffu, k_scale.loses) ? 1 : 0) | (__any_sync(0xffffffffu, v_scale.loses) ? 2 : 0);
        const float ks = pow2(-((apart & 1) ? k_scale.own : k_scale.all));
        const float mid = k_mid * ks, hi = __half2float(__float2half_rn(mid));
        const uint32_t terms = pack_f16(hi, mid - hi);                                  // met by {a, a, b, b} of the row's sum a + b
        const uint32_t k_step = pack_f16(kv4_step(kp) * ks, kv4_step(kp) * ks);
        lazy_wait(&k_empty[s], ((blk / kRing) & 1) ^ 1, DEV_TIMEOUT_EMPTY);
        // (A ring of four stages is enough: the S product of stage blk - 2, whose K stood here, was issued behind the P V products of
        // stage blk - 4, which had waited for every softmax warp.)
        if (lane == 0)
          reinterpret_cast<int4*>(smem + kOffInfo)[(blk % kInfo) * 4 + wq] =
              make_int4(__float_as_int((apart & 1) ? 1.f : pow2(k_scale.all)), v_scale.all, (int)bad, apart);
        if (apart) reinterpret_cast<char2*>(smem + kOffExp)[(blk % kInfo) * 128 + 32 * wq + lane] = make_char2((char)k_scale.own, (char)v_scale.own);
        *reinterpret_cast<uint4*>(smem + kOffKExt + s * kExt + ext_row(32 * wq + lane)) = make_uint4(terms, terms, 0, 0);
        // unit: 16 bytes = values [32 q, 32 q + 32) of a token; atom (token group, q >> 1), chunks (q & 1) * 4 + word
        const int q = lane & 3, r = lane >> 2;
        const uint8_t* src = raw + r * (D / 2) + q * 16;
        uint8_t* dst = smem + kOffK + s * kOperand + wq * 8192 + (q >> 1) * 1024 + r * 128;
        uint4 next = *reinterpret_cast<const uint4*>(src);
        // (two units at a time in K and V: 187.0 us instead of 189.5 for one; all four, whose code is twice as long, as slow as one)
#pragma unroll 2
        for (int u = 0; u < 4; ++u) {
          const uint4 v = (q & 2) ? make_uint4(next.z, next.w, next.x, next.y) : next;
          if (u < 3) next = *reinterpret_cast<const uint4*>(src + ((u + 1) >> 1) * kBlock + ((u + 1) & 1) * (4 * D));
          const uint32_t step = __shfl_sync(0xffffffffu, k_step, u * 8 + r);
          const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int x = 0; x < 4; ++x)
            *reinterpret_cast<uint4*>(dst + u * 2048 + ((((q & 1) * 4 + (x ^ (q & 2))) ^ r) << 4)) = k_values(word[x], kc, step);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&raw_empty[rs]);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&k_full[s]);
        if (n == 0) {
          // ---- Q: one row a thread, scaled by its largest value, in place; its sum; the factor of its scores ----
          const int row = 32 * wq + lane;
          uint8_t* qrow = smem + kOffQ + row * 128;
          lazy_wait(q_full, item & 1, DEV_TIMEOUT_FULL);
          uint32_t top = 0;
          float sum = 0.f;
#pragma unroll 4
          for (int c = 0; c < 16; ++c) {
            const uint4 v = *reinterpret_cast<const uint4*>(qrow + (c >> 3) * (kOperand / 2) + (((c & 7) ^ (row & 7)) << 4));
            const uint32_t e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              top = max(top, max(e[i] & 0x7fffu, (e[i] >> 16) & 0x7fffu));
              sum += __uint_as_float(e[i] << 16) + __uint_as_float(e[i] & 0xffff0000u);
            }
          }
          const int qe = scale_exp((int)(top >> 7));
          const float qs = pow2(-qe);
#pragma unroll 4
          for (int c = 0; c < 16; ++c) {
            uint4* at = reinterpret_cast<uint4*>(qrow + (c >> 3) * (kOperand / 2) + (((c & 7) ^ (row & 7)) << 4));
            uint4 v = *at;
            v.x = pack_f16(__uint_as_float(v.x << 16) * qs, __uint_as_float(v.x & 0xffff0000u) * qs);
            v.y = pack_f16(__uint_as_float(v.y << 16) * qs, __uint_as_float(v.y & 0xffff0000u) * qs);
            v.z = pack_f16(__uint_as_float(v.z << 16) * qs, __uint_as_float(v.z & 0xffff0000u) * qs);
            v.w = pack_f16(__uint_as_float(v.w << 16) * qs, __uint_as_float(v.w & 0xffff0000u) * qs);
            *at = v;
          }
          sum *= qs;
          const float hi = __half2float(__float2half_rn(sum)), lo = sum - hi;
          *reinterpret_cast<uint4*>(smem + kOffQExt + ext_row(row)) = make_uint4(pack_f16(hi, hi), pack_f16(lo, lo), 0, 0);
          qf_smem[row] = P.scale_log2 * pow2(qe);
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(q_ready);
        }
      }
    }
  } else if (warp < 12) {
    // ------------------------------------ codes to V ------------------------------------
    regs_dec<64>();
    const CodeConst vc = code_const(0.f);
    const int wq = warp - 8;
    uint32_t blk = 0;
    for (int item = 0; item < item_end; ++item) {
      const AttnItem w = P.items[item_at(item)];
      const int nblk = stages_of(w), tok_begin = w.blk_begin * 64, tok_end = min(w.blk_end * 64, w.kv_len);
      for (int n = 0; n < nblk; ++n, ++blk) {
        const int rs = blk % kRaw, s = blk % kRing;
        const uint8_t* raw = smem + kOffRaw + rs * kRawBytes + 2 * wq * kBlock;
        lazy_wait(&raw_full[rs], (blk / kRaw) & 1, DEV_TIMEOUT_FULL);
        const bool there = tok_begin + n * kBT + 32 * wq + lane < tok_end;
        uint32_t vp = there ? *reinterpret_cast<const uint32_t*>(raw + (lane >> 4) * kBlock + kv4_v_pairs(D) + 4 * (lane & 15)) : 0u;
        bool v_bad;
        const Scale v_scale = token_scale(v_top(vp, &v_bad));
        const float vs = pow2(-(__any_sync(0xffffffffu, v_scale.loses) ? v_scale.own : v_scale.all));
        if (v_bad) vp = 0;
        const uint32_t v_pair = pack_f16(kv4_step(vp) * vs, kv4_min(vp) * vs);
        lazy_wait(&v_empty[s], ((blk / kRing) & 1) ^ 1, DEV_TIMEOUT_EMPTY);
        // unit: 16 bytes = values [16 g, 16 g + 16) of a token pair, chunks 2 g and 2 g + 1 of both tokens
        const int g = lane & 7, r = lane >> 3;
        const uint8_t* src = raw + kv4_v_codes(D) + r * D + g * 16;
        uint8_t* dst = smem + kOffV + s * kOperand + wq * 8192 + (g >> 2) * 1024 + 2 * r * 128;
        uint4 next = *reinterpret_cast<const uint4*>(src);
#pragma unroll 2
        for (int u = 0; u < 4; ++u) {
          const uint4 v = (g & 4) ? make_uint4(next.z, next.w, next.x, next.y) : next;
          if (u < 3) next = *reinterpret_cast<const uint4*>(src + ((u + 1) >> 1) * kBlock + ((u + 1) & 1) * (4 * D));
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t sm = __shfl_sync(0xffffffffu, v_pair, u * 8 + 2 * r + e);
            const uint32_t step = __byte_perm(sm, sm, 0x1010), low = __byte_perm(sm, sm, 0x3232);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t a = x ? v.z : v.x, b = x ? v.w : v.y;
              *reinterpret_cast<uint4*>(dst + u * 2048 + e * 128 + (((2 * (g & 3) + (x ^ (g >> 2))) ^ (2 * r + e)) << 4)) =
                  v_values(e ? __byte_perm(a, b, 0x7632) : __byte_perm(a, b, 0x5410), vc, step, low);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&raw_empty[rs]);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&v_full[s]);
      }
    }
  } else {
    // ------------------------------------ softmax ------------------------------------
    regs_inc<144>();
    const int g = (warp - 12) >> 2;             // softmax group: takes tokens [64 g, 64 g + 64) of every stage
    const int quad = warp & 3;
    const int row = quad * 32 + lane;          // query row of the tile = TMEM lane
    const uint32_t lane_addr = tmem_base + ((uint32_t)(quad * 32) << 16);
    const uint32_t s_addr = lane_addr + g * 64, o_addr = lane_addr + kTmemO + g * D;
    uint32_t cs = 0;                           // stages so far
    for (int item = 0; item < item_end; ++item) {
      const AttnItem w = P.items[item_at(item)];
      const int R = w.ntok * P.group;
      const int tok_begin = w.blk_begin * 64, tok_end = min(w.blk_end * 64, w.kv_len), nblk = stages_of(w);
      const bool rvalid = row < R, warp_valid = quad * 32 < R;
      int climit = -1, vlo = 0, vhi = 0;
      if (rvalid) {
        const int t = w.tok0 + row / P.group;
        climit = P.tok_climit[t];
        vlo = P.tok_lo[t];
        vhi = P.tok_hi[t];
      }
      bwait(q_ready, item & 1, DEV_TIMEOUT_FULL);
      const float qf = qf_smem[row];               // (a row that does not exist: whatever)
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty);
      // Reference maximum (powers of two, a whole number: adding exponents to it is exact), sum and scale of O of the row.
      float m_ref = rvalid ? kNoRef : 0.f, l_run = 0.f;
      int o_exp = kNoScale;

      for (int n = 0; n < nblk; ++n, ++cs) {
        const uint32_t s_buf = s_addr + (cs & 1) * kBT;
        bwait(&s_full[cs & 1], (cs >> 1) & 1, DEV_TIMEOUT_MMA);
        tc_fence_after();
        const int pos0 = tok_begin + n * kBT + g * 64;
        if (warp_valid) {
          const int4* info = reinterpret_cast<const int4*>(smem + kOffInfo) + (cs % kInfo) * 4 + 2 * g;
          const int4 i0 = info[0], i1 = info[1];
          const float f[2] = {qf * __int_as_float(i0.x), qf * __int_as_float(i1.x)};
          uint32_t sr[2][32];   // the S row of this thread: 64 scores, in units of 1 / f
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_ld32_nowait(s_buf + c * 32, sr[c]);
          tmem_ld_wait();
          const int lim = min(climit, tok_end - 1);
          const int apart[2] = {i0.w, i1.w};
          // words of two tokens: scales of K and V of the first, of K and V of the second
          const uint32_t* scales = reinterpret_cast<const uint32_t*>(smem + kOffExp) + (cs % kInfo) * 64 + g * 32;
          const bool need_mask = __any_sync(0xffffffffu, (rvalid && pos0 + 63 > lim) || (apart[0] | apart[1]));
          unsigned bad[2] = {(unsigned)i0.z, (unsigned)i1.z};
          int ev[2] = {i0.y, i1.y};            // the largest scale of V among those of the 32 tokens that the row sees
          if (need_mask) {
            // visible tokens of this row within the 64: [0, a] and [b, c), as a 64-bit mask over tokens
            const int a = lim - pos0, b = vlo - pos0, cc = min(vhi, tok_end) - pos0;
            auto ones = [](int k) -> unsigned long long { return k <= 0 ? 0ull : (k >= 64 ? ~0ull : ((1ull << k) - 1ull)); };
            const unsigned long long see = ones(a + 1) | (ones(cc) & ~ones(b));
            bad[0] &= (unsigned)see;
            bad[1] &= (unsigned)(see >> 32);
            if ((unsigned)see == 0u) ev[0] = kNoScale;
            if ((unsigned)(see >> 32) == 0u) ev[1] = kNoScale;
            if (apart[0] | apart[1]) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                int most = kNoScale;
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                  const int both = (int)(scales[c * 16 + (i >> 1)] << ((i & 1) ? 0 : 16)), k = (both << 8) >> 24, v = both >> 24;
                  if (apart[c] & 1) sr[c][i] = __float_as_uint(__uint_as_float(sr[c][i]) * pow2(k));
                  if ((see >> (c * 32 + i)) & 1ull) most = max(most, v);
                }
                if (apart[c] & 2) ev[c] = most;
              }
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (((see >> (c * 32 + i)) & 1ull) == 0ull) sr[c][i] = 0xff800000u;   // -inf
          }
          if (__any_sync(0xffffffffu, m_ref == kNoRef)) {      // a row that has seen no token yet: what it has summed up is nothing
            float mx[2][2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              mx[c][0] = mx[c][1] = -INFINITY;
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                mx[c][0] = fmaxf(mx[c][0], fmaxf(__uint_as_float(sr[c][i]), __uint_as_float(sr[c][i + 1])));
                mx[c][1] = fmaxf(mx[c][1], fmaxf(__uint_as_float(sr[c][i + 2]), __uint_as_float(sr[c][i + 3])));
              }
            }
            const float z = fmaxf(__fmul_rn(fmaxf(mx[0][0], mx[0][1]), f[0]), __fmul_rn(fmaxf(mx[1][0], mx[1][1]), f[1]));
            if (m_ref == kNoRef && z > m_ref) m_ref = rintf(z);
          }
          const int e_new = max(o_exp, max(ev[0], ev[1]));
          const bool rescale = n > 0 && e_new != o_exp && o_exp != kNoScale;      // (without a scale it is zero)
          // (see attention_tc.cu: probabilities relative to the standing reference; a stage in which a row outgrows it is done again)
#pragma unroll 1
          for (int pass = 0; pass < 2; ++pass) {
            float2 lsa[2][2] = {};
            float mxa[2][2];
            const int lower[2] = {max(-64, ev[0] - e_new), max(-64, ev[1] - e_new)};     // (at -64 nothing of P is left)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const float2 f2 = make_float2(f[c], f[c]);
              const float shift = kLift + (float)lower[c] - m_ref;
              const float2 shift2 = make_float2(shift, shift);
              mxa[c][0] = mxa[c][1] = -INFINITY;
              uint32_t pk[16];     // 32 tokens -> 16 packed columns over the start of this S buffer
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const int k = (i >> 1) & 1;
                const float2 t = make_float2(__uint_as_float(sr[c][i]), __uint_as_float(sr[c][i + 1])), y = fma2(t, f2, shift2);
                mxa[c][k] = fmaxf(mxa[c][k], fmaxf(t.x, t.y));
                const float2 p = make_float2(exp2f(y.x), exp2f(y.y));   // exp2(-inf) = 0 for masked
                lsa[c][k] = add2(lsa[c][k], p);
                pk[i >> 1] = pack_f16(p.x, p.y);
              }
              tmem_st16(s_buf + c * 16, pk);
            }
            const float z = fmaxf(__fmul_rn(fmaxf(mxa[0][0], mxa[0][1]), f[0]), __fmul_rn(fmaxf(mxa[1][0], mxa[1][1]), f[1]));
            const bool grow = rvalid && n > 0 && z > m_ref + kHeadroom;
            if (pass == 1 || !__any_sync(0xffffffffu, grow || rescale)) {
              const float2 l0 = add2(lsa[0][0], lsa[0][1]), l1 = add2(lsa[1][0], lsa[1][1]);
              l_run += (l0.x + l0.y) * pow2(-lower[0]) + (l1.x + l1.y) * pow2(-lower[1]);
              break;
            }
            // O is rescaled in TMEM, once the group's P V of the previous stage has completed
            bwait(pv_done, (cs - 1) & 1, DEV_TIMEOUT_MMA);
            tc_fence_after();
            const float m_new = grow ? rintf(z) : m_ref;
            const float fl = exp2f(m_ref - m_new), fo = rescale ? fl * pow2(max(-120, o_exp - e_new)) : fl;
            m_ref = m_new;
            l_run *= fl;
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t r[16];
              tmem_ld16(o_addr + c * 16, r);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * fo);
              tmem_st16(o_addr + c * 16, r);
            }
            tmem_st_wait();
          }
          // the tokens' own scales of V, on P as it stands.  (This code and that for K in front of the masks is rarely run, and takes 6 us of
          // 184 for 1001 rows over 6000 tokens of 40 / 8 heads by being there; inside of the loop it took 18.)
          if ((apart[0] | apart[1]) & 2) {
            tmem_st_wait();
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
              if (!((c ? apart[1] : apart[0]) & 2)) continue;
              const int most = c ? ev[1] : ev[0];
              auto by = [&](int v) { return __int_as_float(max(127 + min(v - most, 0), 0) << 23); };      // (one that the row does not see: P is 0)
              uint32_t pk[16];
              tmem_ld16(s_buf + c * 16, pk);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int both = (int)scales[c * 16 + i];
                const float2 p = __half22float2(reinterpret_cast<const __half2&>(pk[i]));
                pk[i] = pack_f16(p.x * by((both << 16) >> 24), p.y * by(both >> 24));
              }
              tmem_st16(s_buf + c * 16, pk);
            }
          }
          o_exp = e_new;
          if (bad[0] | bad[1]) l_run = __int_as_float(0x7fc00000);      // the row sees V that is not finite
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[2 * g + (cs & 1)]);
      }

      // ---- merge the two groups' partial attentions and write out: this group finishes dims [64 g, 64 g + 64) ----
      bwait(o_full, item & 1, DEV_TIMEOUT_MMA);
      tc_fence_after();
      // (the sum is of lifted probabilities, relative to a reference lower by as much)
      ml_smem[g * 128 + row] = m_ref - kLift;
      ml_smem[256 + g * 128 + row] = l_run;
      ml_smem[512 + g * 128 + row] = pow2(max(-56, o_exp));
      softmax_bar();
      if (warp_valid) {
        const float r0 = ml_smem[row], r1 = ml_smem[128 + row], m_all = fmaxf(r0, r1);
        const float w0 = exp2f(r0 - m_all), w1 = exp2f(r1 - m_all);
        const float l_all = ml_smem[256 + row] * w0 + ml_smem[384 + row] * w1;
        const float inv = (w.part < 0) ? (l_all > 0.f ? 1.f / l_all : 0.f * l_all) : (l_all == l_all ? 1.f : l_all);
        const float f0 = w0 * ml_smem[512 + row] * inv, f1 = w1 * ml_smem[640 + row] * inv;
        const size_t orow = (size_t)(w.tok0 + row / P.group) * P.n_q + w.kv_head * P.group + row % P.group;
        float4* s4 = reinterpret_cast<float4*>(smem + kOffScratch + (warp - 12) * 2048);
        const int nrow = min(32, R - quad * 32);
#pragma unroll 1
        for (int cc = 0; cc < 4; ++cc) {
          const int c = 4 * g + cc;               // 16-dim chunk of the output row
          uint32_t ra[16], rb[16];
          tmem_ld16(lane_addr + kTmemO + c * 16, ra);
          tmem_ld16(lane_addr + kTmemO + D + c * 16, rb);
          tmem_ld_wait();
          float v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = fmaf(__uint_as_float(rb[i]), f1, __uint_as_float(ra[i]) * f0);
          if (w.part < 0) {
            if (rvalid) {
              uint4* dst = reinterpret_cast<uint4*>(P.o + orow * D + c * 16);
              dst[0] = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
              dst[1] = make_uint4(pack_bf16(v[8], v[9]), pack_bf16(v[10], v[11]), pack_bf16(v[12], v[13]), pack_bf16(v[14], v[15]));
            }
          } else {
            // fp32 partial rows: through shared memory (chunk q of row r at q ^ ((r >> 1) & 3)), so that a store writes 64-byte pieces
#pragma unroll
            for (int q = 0; q < 4; ++q) s4[lane * 4 + (q ^ ((lane >> 1) & 3))] = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            __syncwarp();
            const int rq = lane >> 2, q = lane & 3;
            float4* dst = reinterpret_cast<float4*>(P.part_o + ((size_t)w.part * 128 + quad * 32) * D + c * 16) + q;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int rr = 8 * j + rq;
              const float4 t = s4[rr * 4 + (q ^ ((rr >> 1) & 3))];
              if (rr < nrow) __stcg(dst + (size_t)rr * (D / 4), t);
            }
            __syncwarp();
          }
        }
        if (g == 0 && rvalid) {
          if (w.part >= 0) {
            P.part_ml[((size_t)w.part * 128 + row) * 2 + 0] = m_all;
            P.part_ml[((size_t)w.part * 128 + row) * 2 + 1] = l_all;
          } else if (P.lse) {
            P.lse[orow] = log_sum_exp(m_all, l_all);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(o_empty);
      softmax_bar();          // the exchange area may be rewritten
    }
  }

  griddep_launch();
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols);
  }
}

}  // namespace

bool launch_attention_kv4_tc(const BatchLayout& bl, const Dims& dm, int layer, const void* q, void* o, float* lse, const void* kv_pool,
                             int64_t n_pages, float* part_o, float* part_ml, int n_sm, int* status, cudaStream_t st) {
  static bool configured[kMaxDevices] = {false};
  if (first_use_on_device(configured))
    cudaFuncSetAttribute(attention_kv4_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  Params P;
  P.items = bl.items;
  P.cta_off = bl.cta_off;
  P.page_table = bl.page_table;
  P.pt_stride = bl.pt_stride;
  P.tok_climit = bl.tok_climit;
  P.tok_lo = bl.tok_lo;
  P.tok_hi = bl.tok_hi;
  P.o = static_cast<__nv_bfloat16*>(o);
  P.lse = lse;
  P.pool = static_cast<const uint8_t*>(kv_pool);
  P.n_pages = n_pages;
  P.layer = layer;
  P.n_q = dm.n_q;
  P.n_kv = dm.n_kv;
  P.group = dm.n_q / dm.n_kv;
  P.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  P.part_o = part_o;
  P.part_ml = part_ml;
  P.status = status;
  CUtensorMap qmap;
  if (!q_tensor_map(q, bl.n_tok, dm.n_q, P.group, &qmap)) return false;
  launch_pdl(attention_kv4_tc_kernel, dim3(n_sm), dim3(kThreads), kSmemBytes, st, qmap, P);
  return true;
}

}  // namespace recg

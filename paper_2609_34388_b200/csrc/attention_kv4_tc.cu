// Hybrid-mask paged attention over a pool in 4 bits on the 5th-generation tensor cores (head_dim 128, many query rows per kv head).
//
// Work items, masks and the combine kernel are those of attention_tc.cu, the mathematics are those of attention_kv4.cu: the tensor
// cores multiply codes (c - 8 as bf16, exact), steps and minima enter in fp32 beside the softmax,
//   score = s_K (q . (c_K - 8)) + (m_K + 8 s_K) sum(q),    o = sum_j (p_j s_Vj) (c_Vj - 8) + sum_j p_j (m_Vj + 8 s_Vj).
// Values with their steps applied would have to be rounded to bf16 before the products, K and V both: an error of 3.2e-3 against
// 2.3e-3 for scores of unit variance, and a log-sum-exp that is good to 1e-4 only.
//
// Per CTA (16 warps = 4 warpgroups, one CTA per SM, persistent over the work list), stages of 128 tokens:
//   warp 0     streams the blocks of the pool (codes and pairs of a page and head: one bulk copy) into a ring of two raw stages, and
//              the item's Q rows by TMA
//   warps 4-7  turn a raw stage into the operands: K (K-major) and V (MN-major), 16 tokens x 128 values in 128-byte-swizzled atoms as
//              the tensor core reads them, and the steps and minima as fp32 pairs.  Every lane turns words of eight codes into
//              16-byte stores; words of a lane are taken in an order in which no two lanes of a store meet a bank.
//   warp 1     one elected lane issues S = Q C_K^T (two stages ahead) and per softmax group O_g += P_g C_V (P from TMEM)
//   warps 8-11 and 12-15  two softmax groups: group g takes tokens [64 g, 64 g + 64) of every stage, one thread one query row, its
//              own O accumulator and running (reference maximum, sum, sum of p m); merged at the end of an item.
// The registers are moved to the softmax warps: 4 x (88 + 88 + 168 + 168) x 32 = 16 x 128 x 32 of the launch.
// Every wait is bounded; a wait that runs out raises a CTA-wide flag after which no wait blocks, so the kernel always ends.
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
constexpr int kParams = 4;                       // stages of steps and minima (see the writer)
constexpr int kParamBytes = (kBT / 2) * 32;      // per token pair {s_K, s_K', m_K, m_K'} and {s_V, s_V', m_V, m_V'}
constexpr int kThreads = 512;
constexpr uint32_t kSpin = 1u << 22;
constexpr int kTmemCols = 512;                   // two S buffers of 128 columns; O of group g at 256 + 128 g
constexpr int kTmemO = 2 * kBT;
constexpr float kNoRef = -1e30f;
constexpr float kHeadroom = 8.f;

constexpr int kOffQ = 0;
constexpr int kOffK = kOffQ + kOperand;
constexpr int kOffV = kOffK + kRing * kOperand;
constexpr int kOffRaw = kOffV + kRing * kOperand;
constexpr int kOffParam = kOffRaw + kRaw * kRawBytes;
constexpr int kOffScratch = kOffParam + kParams * kParamBytes;     // 2 KB per softmax warp: partial rows on their way out
constexpr int kOffML = kOffScratch + 8 * 2048;                     // float4 [2 groups][128 rows]: reference, sum, sum of p m
constexpr int kOffBar = kOffML + 2 * 128 * 16;
constexpr int kNumBars = 2 * kRaw + 4 * kRing + 2 + 2 + 4 + 3;
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
__device__ __forceinline__ float2 mul2(const float2& a, const float2& b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)));
  return reinterpret_cast<float2&>(d);
}
// eight values c - 8 as four bf16 pairs
__device__ __forceinline__ uint4 word_values(uint32_t w) { return make_uint4(kv4_pair(w, 0), kv4_pair(w, 1), kv4_pair(w, 2), kv4_pair(w, 3)); }

__global__ void __launch_bounds__(kThreads, 1) attention_kv4_tc_kernel(const __grid_constant__ CUtensorMap qmap, Params P) {
  extern __shared__ __align__(1024) uint8_t smem[];
  if (smem_u32(smem) & 1023u) {          // the swizzled operand layouts need a 1 KB aligned base
    if (threadIdx.x == 0) set_status(P.status, DEV_BAD_INDEX);
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kOffBar);
  uint64_t* raw_full = bars;                     // [kRaw]
  uint64_t* raw_empty = raw_full + kRaw;         // [kRaw]   the four converting warps
  uint64_t* k_full = raw_empty + kRaw;           // [kRing]
  uint64_t* k_empty = k_full + kRing;
  uint64_t* v_full = k_empty + kRing;
  uint64_t* v_empty = v_full + kRing;
  uint64_t* q_full = v_empty + kRing;            // [1]
  uint64_t* q_empty = q_full + 1;                // [1]   the item's last S product, and the eight softmax warps (sum of the row)
  uint64_t* s_full = q_empty + 1;                // [2]   per S buffer
  uint64_t* p_full = s_full + 2;                 // [4]   2 g + (stage & 1)
  uint64_t* pv_done = p_full + 4;
  uint64_t* o_full = pv_done + 1;
  uint64_t* o_empty = o_full + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float4* ml_smem = reinterpret_cast<float4*>(smem + kOffML);
  auto bwait = [&](uint64_t* bar, uint32_t parity, int code) {
    if (mbar_test_wait(bar, parity) || *abort_flag) return;
    if (!mbar_wait(bar, parity, kSpin)) {
      set_status(P.status, code);
      *abort_flag = 1;
    }
  };
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int s = 0; s < kRaw; ++s) {
      mbar_init(&raw_full[s], 1);
      mbar_init(&raw_empty[s], 4);
    }
    for (int s = 0; s < kRing; ++s) {
      mbar_init(&k_full[s], 4);
      mbar_init(&k_empty[s], 1);
      mbar_init(&v_full[s], 4);
      mbar_init(&v_empty[s], 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 9);
    for (int s = 0; s < 2; ++s) mbar_init(&s_full[s], 1);
    for (int s = 0; s < 4; ++s) mbar_init(&p_full[s], 4);
    mbar_init(pv_done, 1);
    mbar_init(o_full, 1);
    mbar_init(o_empty, 8);
    fence_barrier_init();
    asm volatile("prefetch.tensormap [%0];" ::"l"(&qmap) : "memory");
  }
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
    regs_dec<88>();
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
          bwait(&raw_empty[s], ((blk / kRaw) & 1) ^ 1, DEV_TIMEOUT_EMPTY);
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
            bwait(q_empty, (item & 1) ^ 1, DEV_TIMEOUT_EMPTY);
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
        const uint64_t dq0 = desc_kmajor(smem_base + kOffQ);
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
                        dk0 + (uint64_t)((((kk >> 2) * 1024) + (kk & 3) * 32) >> 4), kIdescQK, kk ? 1u : 0u);
            umma_commit(&s_full[b & 1]);
            umma_commit(&k_empty[s]);
            if (last) umma_commit(q_empty);
          };
          bwait(q_full, item & 1, DEV_TIMEOUT_FULL);
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
                             dv0 + (uint64_t)(((4 * g + kk) * 4096) >> 4), kIdescPV, (n | kk) ? 1u : 0u);
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
    // ------------------------------------ codes to operands ------------------------------------
    regs_dec<88>();
    const int tid = threadIdx.x - 128;
    uint32_t blk = 0;
    for (int item = 0; item < item_end; ++item) {
      const AttnItem w = P.items[item_at(item)];
      const int nblk = stages_of(w), tok_begin = w.blk_begin * 64, tok_end = min(w.blk_end * 64, w.kv_len);
      for (int n = 0; n < nblk; ++n, ++blk) {
        const int rs = blk % kRaw, s = blk % kRing;
        const uint8_t* raw = smem + kOffRaw + rs * kRawBytes;
        bwait(&raw_full[rs], (blk / kRaw) & 1, DEV_TIMEOUT_FULL);
        bwait(&k_empty[s], ((blk / kRing) & 1) ^ 1, DEV_TIMEOUT_EMPTY);
        // Steps and minima: thread = token.  The ring of them is four deep: the V operands of the stage before this one went where the P V
        // product of stage blk - 3 had read, which waited for every softmax warp to be done with stage blk - 3.
        {
          const uint8_t* pg = raw + (tid >> 4) * kBlock;
          const bool there = tok_begin + n * kBT + tid < tok_end;          // what is not there counts nothing, whatever the slot holds
          const uint32_t kp = there ? *reinterpret_cast<const uint32_t*>(pg + kv4_k_pairs(D) + 4 * (tid & 15)) : 0u;
          const uint32_t vp = there ? *reinterpret_cast<const uint32_t*>(pg + kv4_v_pairs(D) + 4 * (tid & 15)) : 0u;
          float* out = reinterpret_cast<float*>(smem + kOffParam + (blk % kParams) * kParamBytes) + (tid >> 1) * 8 + (tid & 1);
          out[0] = kv4_step(kp) * P.scale_log2;
          out[2] = fmaf(8.f, kv4_step(kp), kv4_min(kp)) * P.scale_log2;
          out[4] = kv4_step(vp);
          out[6] = fmaf(8.f, kv4_step(vp), kv4_min(vp));
        }
        uint8_t* kdst = smem + kOffK + s * kOperand;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          // unit: 16 bytes = values [32 q, 32 q + 32) of a token; atom (token group, q >> 1), chunks (q & 1) * 4 + word
          const int i = u * 128 + tid, tok = i >> 2, q = i & 3;
          uint4 v = *reinterpret_cast<const uint4*>(raw + (tok >> 4) * kBlock + (tok & 15) * (D / 2) + q * 16);
          if (q & 2) v = make_uint4(v.z, v.w, v.x, v.y);
          const uint32_t word[4] = {v.x, v.y, v.z, v.w};
          uint8_t* row = kdst + (tok >> 3) * 2048 + (q >> 1) * 1024 + (tok & 7) * 128;
#pragma unroll
          for (int x = 0; x < 4; ++x)
            *reinterpret_cast<uint4*>(row + ((((q & 1) * 4 + (x ^ (q & 2))) ^ (tok & 7)) << 4)) = word_values(word[x]);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&k_full[s]);
        bwait(&v_empty[s], ((blk / kRing) & 1) ^ 1, DEV_TIMEOUT_EMPTY);
        uint8_t* vdst = smem + kOffV + s * kOperand;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          // unit: 16 bytes = values [16 g, 16 g + 16) of a token pair, chunks 2 g and 2 g + 1 of both tokens
          const int i = u * 128 + tid, pair = i >> 3, g = i & 7;
          uint4 v = *reinterpret_cast<const uint4*>(raw + (pair >> 3) * kBlock + kv4_v_codes(D) + (pair & 7) * D + g * 16);
          if (g & 4) v = make_uint4(v.z, v.w, v.x, v.y);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int tok = 2 * pair + e;
            uint8_t* row = vdst + (tok >> 3) * 2048 + (g >> 2) * 1024 + (tok & 7) * 128;
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const uint32_t a = x ? v.z : v.x, b = x ? v.w : v.y;
              *reinterpret_cast<uint4*>(row + (((2 * (g & 3) + (x ^ (g >> 2))) ^ (tok & 7)) << 4)) =
                  word_values(e ? __byte_perm(a, b, 0x7632) : __byte_perm(a, b, 0x5410));
            }
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&v_full[s]);
          mbar_arrive(&raw_empty[rs]);
        }
      }
    }
  } else {
    // ------------------------------------ softmax ------------------------------------
    regs_inc<168>();
    const int g = (warp - 8) >> 2;             // softmax group: takes tokens [64 g, 64 g + 64) of every stage
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
      // the sum of the row's query values
      float qsum = 0.f;
      bwait(q_full, item & 1, DEV_TIMEOUT_FULL);
      if (rvalid) {
#pragma unroll 4
        for (int c = 0; c < 16; ++c) {
          const uint4 v = *reinterpret_cast<const uint4*>(smem + kOffQ + (c >> 3) * (kOperand / 2) + row * 128 + (((c & 7) ^ (row & 7)) << 4));
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) qsum += __uint_as_float(u[i] << 16) + __uint_as_float(u[i] & 0xffff0000u);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty);
      float m_ref = rvalid ? kNoRef : 0.f, l_run = 0.f, om_run = 0.f;

      for (int n = 0; n < nblk; ++n, ++cs) {
        const uint32_t s_buf = s_addr + (cs & 1) * kBT;
        bwait(&s_full[cs & 1], (cs >> 1) & 1, DEV_TIMEOUT_MMA);
        tc_fence_after();
        const int pos0 = tok_begin + n * kBT + g * 64;
        const float4* param = reinterpret_cast<const float4*>(smem + kOffParam + (cs % kParams) * kParamBytes) + g * 64;
        if (warp_valid) {
          uint32_t sr[2][32];   // 64 products of this thread's row
#pragma unroll
          for (int c = 0; c < 2; ++c) tmem_ld32_nowait(s_buf + c * 32, sr[c]);
          tmem_ld_wait();
          const int lim = min(climit, tok_end - 1);
          const bool need_mask = __any_sync(0xffffffffu, rvalid && (pos0 + 63 > lim));
          unsigned long long see = ~0ull;          // visible tokens of this row within the 64: [0, a] and [b, c)
          if (need_mask) {
            const int a = lim - pos0, b = vlo - pos0, cc = min(vhi, tok_end) - pos0;
            auto ones = [](int k) -> unsigned long long { return k <= 0 ? 0ull : (k >= 64 ? ~0ull : ((1ull << k) - 1ull)); };
            see = ones(a + 1) | (ones(cc) & ~ones(b));
          }
          const float2 qsum2 = make_float2(qsum, qsum);
          // scores (in powers of two) of tokens i, i + 1 of half c, less `ref`
          auto score2 = [&](int c, int i, const float2& neg_ref2) {
            const float4 kp = param[2 * ((c * 32 + i) >> 1)];
            return fma2(make_float2(__uint_as_float(sr[c][i]), __uint_as_float(sr[c][i + 1])), make_float2(kp.x, kp.y),
                        fma2(make_float2(kp.z, kp.w), qsum2, neg_ref2));
          };
          auto row_max = [&]() {
            float mx = -INFINITY;
            const float2 none = make_float2(0.f, 0.f);
#pragma unroll 1
            for (int c = 0; c < 2; ++c)
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const float4 kp = param[2 * ((c * 32 + i) >> 1)];
                const float2 t = c ? make_float2(__uint_as_float(sr[1][i]), __uint_as_float(sr[1][i + 1]))
                                   : make_float2(__uint_as_float(sr[0][i]), __uint_as_float(sr[0][i + 1]));
                const float2 y = fma2(t, make_float2(kp.x, kp.y), fma2(make_float2(kp.z, kp.w), qsum2, none));
                const unsigned bits = (unsigned)(see >> (c * 32 + i)) & 3u;
                if (bits & 1u) mx = fmaxf(mx, y.x);
                if (bits & 2u) mx = fmaxf(mx, y.y);
              }
            return mx;
          };
          if (__any_sync(0xffffffffu, m_ref == kNoRef)) {      // a row that has seen no token yet: what it has summed up is nothing
            const float mx = row_max();
            if (m_ref == kNoRef && mx > m_ref) m_ref = mx;
          }
          // (see attention_tc.cu: probabilities relative to the standing reference; a stage in which a row outgrows it is done again)
#pragma unroll 1
          for (int pass = 0; pass < 2; ++pass) {
            const float2 neg_ref2 = make_float2(-m_ref, -m_ref);
            float2 lsa[2] = {}, oma[2] = {};
            float mxa[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t pk[16];
              if (!need_mask) {
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                  const int k = (i >> 1) & 1;
                  const float2 y = score2(c, i, neg_ref2);
                  const float4 vp = param[2 * ((c * 32 + i) >> 1) + 1];
                  mxa[k] = fmaxf(mxa[k], fmaxf(y.x, y.y));
                  const float2 p = make_float2(exp2f(y.x), exp2f(y.y));
                  lsa[k] = add2(lsa[k], p);
                  oma[k] = fma2(p, make_float2(vp.z, vp.w), oma[k]);
                  const float2 ps = mul2(p, make_float2(vp.x, vp.y));
                  pk[i >> 1] = pack_bf16(ps.x, ps.y);
                }
              } else {
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                  const int k = (i >> 1) & 1;
                  float2 y = score2(c, i, neg_ref2);
                  const bool s0 = (see >> (c * 32 + i)) & 1ull, s1 = (see >> (c * 32 + i + 1)) & 1ull;
                  if (!s0) y.x = -INFINITY;
                  if (!s1) y.y = -INFINITY;
                  const float4 vp = param[2 * ((c * 32 + i) >> 1) + 1];
                  mxa[k] = fmaxf(mxa[k], fmaxf(y.x, y.y));
                  const float2 p = make_float2(exp2f(y.x), exp2f(y.y));
                  lsa[k] = add2(lsa[k], p);
                  // (a token that this row does not see may hold anything, infinities too)
                  oma[k] = add2(oma[k], make_float2(s0 ? p.x * vp.z : 0.f, s1 ? p.y * vp.w : 0.f));
                  pk[i >> 1] = pack_bf16(s0 ? p.x * vp.x : 0.f, s1 ? p.y * vp.y : 0.f);
                }
              }
              tmem_st16(s_buf + c * 16, pk);
            }
            const bool grow = rvalid && n > 0 && fmaxf(mxa[0], mxa[1]) > kHeadroom;
            if (pass == 1 || !__any_sync(0xffffffffu, grow)) {
              const float2 ls = add2(lsa[0], lsa[1]), os = add2(oma[0], oma[1]);
              l_run += ls.x + ls.y;
              om_run += os.x + os.y;
              break;
            }
            // O is rescaled in TMEM, once the group's P V of the previous stage has completed
            bwait(pv_done, (cs - 1) & 1, DEV_TIMEOUT_MMA);
            tc_fence_after();
            const float mx = row_max();
            const float m_new = grow ? fmaxf(m_ref, mx) : m_ref;
            const float f = exp2f(m_ref - m_new);
            m_ref = m_new;
            l_run *= f;
            om_run *= f;
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint32_t r[16];
              tmem_ld16(o_addr + c * 16, r);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
              tmem_st16(o_addr + c * 16, r);
            }
            tmem_st_wait();
          }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[2 * g + (cs & 1)]);
      }

      // ---- merge the two groups' partial attentions and write out: this group finishes dims [64 g, 64 g + 64) ----
      bwait(o_full, item & 1, DEV_TIMEOUT_MMA);
      tc_fence_after();
      ml_smem[g * 128 + row] = make_float4(m_ref, l_run, om_run, 0.f);
      softmax_bar();
      if (warp_valid) {
        const float4 a0 = ml_smem[row], a1 = ml_smem[128 + row];
        const float m_all = fmaxf(a0.x, a1.x);
        float f0 = exp2f(a0.x - m_all), f1 = exp2f(a1.x - m_all);
        const float l_all = a0.y * f0 + a1.y * f1;
        const float inv = (w.part < 0) ? (l_all > 0.f ? 1.f / l_all : 0.f) : 1.f;
        f0 *= inv;
        f1 *= inv;
        const float om = a0.z * f0 + a1.z * f1;
        const size_t orow = (size_t)(w.tok0 + row / P.group) * P.n_q + w.kv_head * P.group + row % P.group;
        float4* s4 = reinterpret_cast<float4*>(smem + kOffScratch + (warp - 8) * 2048);
        const int nrow = min(32, R - quad * 32);
#pragma unroll 1
        for (int cc = 0; cc < 4; ++cc) {
          const int c = 4 * g + cc;               // 16-dim chunk of the output row
          uint32_t r[16], r1[16];
          tmem_ld16(lane_addr + kTmemO + c * 16, r);
          tmem_ld16(lane_addr + kTmemO + D + c * 16, r1);
          tmem_ld_wait();
          float v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = fmaf(__uint_as_float(r1[i]), f1, fmaf(__uint_as_float(r[i]), f0, om));
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

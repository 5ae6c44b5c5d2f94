// The attention weight that cached tokens gather (recg_kv_weights): per kv head and position j
//   out[j] = (j < L ? decay in[j] : 0) + sum over the rows t and the query heads of the group of w_t exp(score_tj - lse_t).
// With the log-sum-exp of every row from the attention kernel each probability follows from its score alone, so one pass over K
// gives them: S^T = K Q^T (mma.sync) with the tokens as rows of the product.  A warp owns the 16 tokens of a page, has their K as A
// operands in registers and walks over the query rows; the sum over rows is a sum over the columns of its accumulators, which stays in
// the warp.  Nothing is added by atomics: a position belongs to one warp, which takes the rows in order, so results repeat bit for bit.
//
// Bound by the bytes of K as long as rows are few.  The pages of all requests and heads are one line, of which every CTA takes an
// equal piece.  The rows that count (weight not zero) of as many (request, head) pairs of the piece as fit are staged in shared memory
// together, and the warps stream the pairs' pages past them in one go, each into a ring of its own, 16 bytes a lane.  (Pair by pair, each
// with its staging and its barriers: sixteen decoding requests 25.5 us, a serving batch on a bf16 pool 57.8; now 18.9 and 47.1.  One CTA per 128
// tokens, with its own staging and K by plain loads: 41.5 and 140.)
//
// Operands.  A bf16 pool: its tiles are what ldmatrix takes.  A pool in 4 bits: a lane holds the values [D / 4 t, D / 4 (t + 1)) of two
// tokens (t its number in the quad), the contraction index is permuted accordingly; codes as subnormal fp16 numbers, a row of Q scaled by a
// power of two of its own, steps and minima in fp32 (attention_kv4.cu has the reasons).  Q is staged in the order in which a lane takes
// two k-steps at once.
#include <cuda_fp16.h>
#include <type_traits>

#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

constexpr int kChunkRows = 128;             // query rows staged at a time

struct Params {
  const int* ctx_len;
  const int* cu_tok;
  const int* page_table;
  int pt_stride, n_req;
  const int* verify_len;
  const int* tok_climit;
  const int* tok_lo;
  const int* tok_hi;
  const __nv_bfloat16* q;
  const float* lse;
  const float* row_weight;    // null: one each
  const float* in;            // null: nothing gathered so far
  float* out;
  float decay;
  const uint8_t* pool;
  int64_t n_pages;
  int layer, n_q, n_kv, group;
  float scale_log2;
  int* status;
};

template <int D, bool FOUR>
struct Shape {
  static constexpr int kWarps = 16, kThreads = kWarps * 32;
  static constexpr int kBlock = FOUR ? kv4_block_bytes(D) : 4 * kPageSize * D;      // of a page and head in the pool
  static constexpr int kCodes = FOUR ? kPageSize * D / 2 : kPageSize * D * 2;       // its K: codes or values ...
  static constexpr int kWeights = kCodes + (FOUR ? 64 : 0);                         // ... and pairs; the weights so far;
  static constexpr int kId = kWeights + 64;                                         // the page's id
  static constexpr int kPage = kId + 16;
  static constexpr int kSlots = FOUR ? 4 : 2;                                       // pages that a warp has on their way
  static constexpr int kRowBytes = 2 * D + 64;      // from staged row to staged row: lanes of eight rows meet no bank twice
  static constexpr int kRing = kWarps * kSlots * kPage;
  static constexpr int kRowsOff = kRing;
  static constexpr int kInfoOff = kRowsOff + kChunkRows * kRowBytes;
  static constexpr int kVisOff = kInfoOff + kChunkRows * 16;
  static constexpr int kListOff = kVisOff + kChunkRows * 16;
  static constexpr int kTotal = kListOff + kChunkRows * 8;
  static_assert(kPage % 16 == 0 && kTotal % 16 == 0, "16-byte pieces");
};

// d (+)= a b; FIRST: the accumulator starts from zero
template <bool HALF, bool FIRST>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  const float c0 = FIRST ? 0.f : d[0], c1 = FIRST ? 0.f : d[1], c2 = FIRST ? 0.f : d[2], c3 = FIRST ? 0.f : d[3];
  if (HALF)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c0), "f"(c1), "f"(c2), "f"(c3));
}
__device__ __forceinline__ uint32_t scaled_f16(uint32_t pair, float by) {
  const __half2 h = __floats2half2_rn(__uint_as_float(pair << 16) * by, __uint_as_float(pair & 0xffff0000u) * by);
  return reinterpret_cast<const uint32_t&>(h);
}

template <int D, bool FOUR>
__global__ void __launch_bounds__(Shape<D, FOUR>::kThreads, 1) kv_weights_kernel(const __grid_constant__ Params P) {
  using SH = Shape<D, FOUR>;
  constexpr int kWarps = SH::kWarps, kThreads = SH::kThreads;
  constexpr int NW = D / 32, kChunks = D / 8;           // 16-byte chunks a lane holds of a row; of a row
  extern __shared__ __align__(128) uint8_t smem[];
  // a staged row: sum of its values times the scale, -lse (powers of two), weight, what makes a product of codes a score
  float4* s_info = reinterpret_cast<float4*>(smem + SH::kInfoOff);
  int4* s_vis = reinterpret_cast<int4*>(smem + SH::kVisOff);
  int2* s_src = reinterpret_cast<int2*>(smem + SH::kListOff);          // a staged row: its place in lse (-1: fills up an eight); row of the batch | segment << 20
  int* s_cost = reinterpret_cast<int*>(smem + SH::kTotal);             // [n_req] cost of a page and head of request r
  long long* s_first = reinterpret_cast<long long*>(smem);             // [n_req + 1] cost in front of request r (where rings and rows are later)
  __shared__ long long s_scan[kWarps];
  // segments, (request, head) pairs whose rows are staged together
  __shared__ int s_req[kWarps], s_head[kWarps], s_page0[kWarps], s_pages[kWarps], s_tok0[kWarps], s_new[kWarps], s_ctx[kWarps];
  __shared__ int s_cum[kWarps], s_row0[kWarps], s_rows8[kWarps], s_count[kWarps], s_next[kWarps], s_lim[kWarps];
  __shared__ long long s_ahead[kWarps];                                // cost in front of what follows the segment
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  griddep_wait();
  griddep_launch();
  // The line of pages [request][kv head][page], each as long as it takes: kPageCost for K and one for eight rows.  (With pages of one
  // length the CTAs of requests with few rows waited for the others: a serving batch on a bf16 pool 86 us, 61 with this.)  Where rows are
  // weighted the verify rows are taken to be the ones that count.
  constexpr int kPageCost = 3;
  const int per = (P.n_req + kThreads - 1) / kThreads, my_r0 = min(P.n_req, tid * per), my_r1 = min(P.n_req, my_r0 + per);
  {
    long long mine = 0;
    for (int r = my_r0; r < my_r1; ++r) {
      const int n_new = P.cu_tok[r + 1] - P.cu_tok[r], verify = P.verify_len[r];
      const int cost = kPageCost + ((P.row_weight && verify > 0 ? verify : n_new) * P.group + 7) / 8;
      s_cost[r] = cost;
      s_first[r] = mine;
      // (a device-resident round that was refused has no rows, and lengths that may be anything)
      if (n_new > 0) mine += (long long)((P.ctx_len[r] + n_new + kPageSize - 1) / kPageSize * P.n_kv) * cost;
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    long long at = incl - mine;
    for (int k = 0; k < warp; ++k) at += s_scan[k];
    for (int r = my_r0; r < my_r1; ++r) s_first[r] += at;
    if (tid == kThreads - 1) s_first[P.n_req] = at + mine;
    __syncthreads();
  }
  // this CTA's piece of it: the pages that begin there
  const long long total = s_first[P.n_req], piece = (total + gridDim.x - 1) / gridDim.x;
  const long long begin = piece * blockIdx.x, end = min(total, begin + piece);
  const uint32_t ring_at = smem_u32(smem + warp * SH::kSlots * SH::kPage) + lane * 16;
  const unsigned pool_pages = (unsigned)min(P.n_pages, (int64_t)0x7fffffff);

  const size_t out_layer = (size_t)P.layer * P.n_pages * P.n_kv * kPageSize;
  const uint8_t* base = P.pool + (size_t)P.layer * P.n_pages * P.n_kv * SH::kBlock + lane * 16;
  float* out_at = P.out + out_layer + g + 8 * (t & 1);

  int pair = 0;                                        // (request, head) the piece begins in, and the cost in front of it
  long long ahead = 0;
  if (begin < end) {
    int r = 0, hi_r = P.n_req;                         // largest r with s_first[r] <= begin: it has pages
    while (hi_r - r > 1) {
      const int mid = (r + hi_r) >> 1;
      if (s_first[mid] <= begin) r = mid; else hi_r = mid;
    }
    const long long one = (s_first[r + 1] - s_first[r]) / P.n_kv;
    const int h = (int)((begin - s_first[r]) / one);
    pair = r * P.n_kv + h;
    ahead = s_first[r] + h * one;
  }
  __syncthreads();
  const int n_pairs = P.n_req * P.n_kv;
  while (begin < end && pair < n_pairs && ahead < end) {
    // ---- the next segments: a lane one of them ----
    if (warp == 0) {
      const int q = pair + lane, r = q < n_pairs ? q / P.n_kv : 0;
      int first_tok = 0, n_new = 0, L = 0, n_pages = 0;
      if (lane < kWarps && q < n_pairs) {
        first_tok = P.cu_tok[r];
        n_new = P.cu_tok[r + 1] - first_tok;
        L = P.ctx_len[r];
        if (n_new > 0) n_pages = (L + n_new + kPageSize - 1) / kPageSize;
      }
      const int cost = s_cost[r];
      const long long mine = (long long)n_pages * cost;
      long long upto = mine;
#pragma unroll
      for (int o = 1; o < kWarps; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += y;
      }
      upto += ahead;
      const long long from = upto - mine;
      const int lo = begin > from ? (int)min((long long)n_pages, (begin - from + cost - 1) / cost) : 0;
      const int hi = from < end ? (int)min((long long)n_pages, (end - from + cost - 1) / cost) : 0;
      if (lane < kWarps) {
        s_req[lane] = r;
        s_head[lane] = q - r * P.n_kv;
        s_page0[lane] = lo;
        s_pages[lane] = max(0, hi - lo);
        s_tok0[lane] = first_tok;
        s_new[lane] = n_new;
        s_ctx[lane] = L;
        s_ahead[lane] = upto;
        s_count[lane] = hi > lo ? n_new : 0;
        s_lim[lane] = 0x7fffffff;
      }
    }
    __syncthreads();
    // ---- how many rows of each count; those whose rows fit are taken together (or one, in pieces) ----
    if (P.row_weight) {
      const int first_tok = s_tok0[warp], n_new = s_count[warp];
      int n = 0;
      for (int at = lane; at < n_new; at += 32) n += P.row_weight[first_tok + at] != 0.f;
      n = __reduce_add_sync(0xffffffffu, n);
      __syncwarp();
      if (lane == 0) s_count[warp] = n;
      __syncthreads();
    }
    int cum, nseg, total, row0;                          // (row0: of the warp's segment)
    {
      const int rows_of = lane < kWarps ? (s_count[lane] * P.group + 7) & ~7 : 0, pages = lane < kWarps ? s_pages[lane] : 0;
      int rows_to = rows_of, pages_to = pages;
#pragma unroll
      for (int o = 1; o < kWarps; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, rows_to, o), z = __shfl_up_sync(0xffffffffu, pages_to, o);
        if (lane >= o) {
          rows_to += y;
          pages_to += z;
        }
      }
      const unsigned fit = __ballot_sync(0xffffffffu, lane < kWarps && rows_to <= kChunkRows);
      nseg = max(1, __ffs(~fit) - 1);
      total = __shfl_sync(0xffffffffu, pages_to, nseg - 1);
      cum = lane < nseg ? pages_to - pages : 0x7fffffff;
      row0 = __shfl_sync(0xffffffffu, rows_to - rows_of, warp);
      if (warp == 0 && lane < nseg) {
        s_cum[lane] = cum;
        s_row0[lane] = rows_to - rows_of;
      }
    }
    const bool whole = nseg > 1 || (s_count[0] * P.group + 7) / 8 * 8 <= kChunkRows;

    for (int first_tok = 0, chunk = 0;; ++chunk) {
      // what the weights are added to: those so far, or what the chunk of rows before this one left
      const uint8_t* old = reinterpret_cast<const uint8_t*>(chunk ? P.out : (P.decay != 0.f ? P.in : nullptr));
      if (old) old += out_layer * 4 + (lane & 3) * 16;
      const float keep = chunk ? 1.f : P.decay;
      // ---- the warp's pages on their way; ids 32 at a time, a lane one of them (and its head) ----
      int next = warp, ids = 0, heads = 0, used = 0;
      auto load_ids = [&]() {
        used = 0;
        const int at = next + lane * kWarps;
        int k = 0;
        for (int x = 1; x < nseg; ++x) k += at >= __shfl_sync(0xffffffffu, cum, x);
        const int from = __shfl_sync(0xffffffffu, cum, k);
        heads = s_head[k];
        ids = at < total ? __ldg(P.page_table + (size_t)s_req[k] * P.pt_stride + s_page0[k] + at - from) : 0;
      };
      auto request = [&](uint32_t slot_at) {            // one group of copies per call, be it empty
        if (next < total) {
          const unsigned id = __shfl_sync(0xffffffffu, ids, used), head = __shfl_sync(0xffffffffu, heads, used);
          const uint32_t dst = ring_at + slot_at;
          if (id < pool_pages) {
            const uint64_t block = (uint64_t)id * (unsigned)P.n_kv + head;
            const uint8_t* src = base + block * SH::kBlock;
#pragma unroll
            for (int x = 0; x < SH::kCodes / 512; ++x) copy_async16(dst + x * 512, src + x * 512);
            if (lane < 4) {
              if (FOUR) copy_async16(dst + SH::kCodes, src + kv4_k_pairs(D));
              if (old) copy_async16(dst + SH::kWeights, old + block * (kPageSize * 4));
            }
          } else {
            set_status(P.status, DEV_BAD_INDEX);
          }
          if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + SH::kId), "r"(id) : "memory");
          next += kWarps;
          if (++used == 32) load_ids();
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
      load_ids();
      for (int x = 0; x < SH::kSlots; ++x) request(x * SH::kPage);

      // ---- the rows that count, as many as fit: a warp those of a segment ----
      if (warp < nseg) {
        const int fit = kChunkRows / P.group, tok0 = s_tok0[warp], n_new = s_pages[warp] ? s_new[warp] : 0, h = s_head[warp];
        int2* src = s_src + row0;
        int n = 0, at = first_tok;
        while (at < n_new && n < fit) {
          const bool counts = at + lane < n_new && (!P.row_weight || P.row_weight[tok0 + at + lane] != 0.f);
          unsigned m = __ballot_sync(0xffffffffu, counts);
          const int mine = n + __popc(m & ((1u << lane) - 1)), tok = tok0 + at + lane;
          if (counts && mine < fit)
            for (int x = 0; x < P.group; ++x) src[mine * P.group + x] = make_int2(tok * P.n_q + h * P.group + x, tok | warp << 20);
          if (n + __popc(m) > fit) {                     // up to the last one that fits
            for (int k = fit - n; k > 1; --k) m &= m - 1;
            at += __ffs(m);
            n = fit;
          } else {
            n += __popc(m);
            at += 32;
          }
        }
        const int rows = n * P.group, rows8 = (rows + 7) & ~7;
        if (lane < rows8 - rows) src[rows + lane] = make_int2(-1, warp << 20);
        if (lane == 0) {
          s_rows8[warp] = rows8;
          s_next[warp] = min(at, n_new);
        }
      }
      __syncthreads();
      first_tok = s_next[0];
      const int staged = s_row0[nseg - 1] + s_rows8[nseg - 1];
      // (chunk c of a row: its values 8 c .. 8 c + 7)
      constexpr int kPer = kChunkRows * kChunks / kThreads;
      static_assert(kPer * kThreads == kChunkRows * kChunks, "a turn stages whole rows");
      uint4 raw[kPer];
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int i = tid + k * kThreads, row = i / kChunks, c = i % kChunks;
        raw[k] = make_uint4(0, 0, 0, 0);
        if (row < staged) {
          const int at = s_src[row].x;
          if (at >= 0) raw[k] = __ldg(reinterpret_cast<const uint4*>(P.q + (size_t)at * D) + c);
        }
      }
      for (int row = tid; row < staged; row += kThreads) {
        const int2 from = s_src[row];
        float minus_lse = -1e30f, weight = 0.f;                   // (a row that fills up the last eight: probability 0)
        int4 vis = make_int4(-1, 0, 0, 0);
        if (from.x >= 0) {
          const int tok = from.y & 0xfffff;
          minus_lse = -1.4426950408889634f * P.lse[from.x];
          weight = P.row_weight ? P.row_weight[tok] : 1.f;
          vis = make_int4(P.tok_climit[tok], P.tok_lo[tok], P.tok_hi[tok], 0);
          atomicMin(&s_lim[from.y >> 20], vis.x);
        }
        s_info[row].y = minus_lse;
        s_info[row].z = weight;
        s_vis[row] = vis;
      }
#pragma unroll
      for (int k = 0; k < kPer; ++k) {
        const int i = tid + k * kThreads, row = i / kChunks, c = i % kChunks;
        if (row >= staged) continue;
        const uint4 v = raw[k];
        uint8_t* at = smem + SH::kRowsOff + row * SH::kRowBytes;
        // (staged * kChunks is a multiple of 64 and kThreads of kChunks: whole quarter and half warps come here together)
        const unsigned together = (kChunks == 16 ? 0xffffu : 0xffu) << (lane & ~(kChunks - 1));
        if (FOUR) {
          // the row's largest value goes to [2^8, 2^9) (as far as the exponent allows)
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
          float sum = 0.f;
          unsigned top = 0;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            sum += __uint_as_float(u[x] << 16) + __uint_as_float(u[x] & 0xffff0000u);
            const unsigned lo = u[x] & 0x7fffu, hi = (u[x] >> 16) & 0x7fffu;
            top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
          }
#pragma unroll
          for (int o = kChunks / 2; o; o >>= 1) {
            sum += __shfl_xor_sync(together, sum, o);
            top = max(top, __shfl_xor_sync(together, top, o));
          }
          const int e = max(-100, min(100, (int)(top >> 7) - 127 - 8));
          if (c == 0) {
            s_info[row].x = sum * P.scale_log2;
            s_info[row].w = pow2(e) * 16777216.f * P.scale_log2;
          }
          const float down = pow2(-e), down16 = pow2(-e - 4);
          // where lane c / NW of a quad looks for its word c % NW
          *reinterpret_cast<uint4*>(at + ((c % NW) * 4 + c / NW) * 16) =
              make_uint4(scaled_f16(v.x, down), scaled_f16(v.y, down16), scaled_f16(v.z, down), scaled_f16(v.w, down16));
        } else {
          // pair i of the chunk belongs to lane i of a quad, which takes the pairs of four chunks at once: two k-steps
          uint32_t* to = reinterpret_cast<uint32_t*>(at + (c >> 2) * 64) + (c & 3);
          to[0] = v.x;
          to[4] = v.y;
          to[8] = v.z;
          to[12] = v.w;
        }
      }
      __syncthreads();

      // ---- pages past the rows ----
      uint32_t slot_at = 0;
      int seg_end = 0, to_page = 0, L = 0, kv_len = 0, h = 0, lim = 0, rows8 = 0;
      const uint8_t* rows_at = smem + SH::kRowsOff;      // of the segment
      const float4* info_at = s_info;
      const int4* vis_at = s_vis;
      for (int i = warp; i < total; i += kWarps) {
        if (i >= seg_end) {
          const int k = 31 - __clz(__ballot_sync(0xffffffffu, cum <= i)), seg_row0 = s_row0[k];
          to_page = s_page0[k] - s_cum[k];
          seg_end = s_cum[k] + s_pages[k];
          L = s_ctx[k];
          kv_len = L + s_new[k];
          h = s_head[k];
          lim = s_lim[k];
          rows8 = s_rows8[k];
          rows_at = smem + SH::kRowsOff + seg_row0 * SH::kRowBytes;
          info_at = s_info + seg_row0;
          vis_at = s_vis + seg_row0;
        }
        const int p = i + to_page;
        asm volatile("cp.async.wait_group %0;" ::"n"(SH::kSlots - 1) : "memory");
        __syncwarp();
        const uint8_t* pg = smem + warp * SH::kSlots * SH::kPage + slot_at;
        const int pos0 = p * kPageSize;
        const unsigned id = *reinterpret_cast<const unsigned*>(pg + SH::kId);
        const int tok = g + 8 * t;                       // lane 0 of a quad stores row g, lane 1 row g + 8
        const bool stores = t < 2 && id < pool_pages && pos0 + tok < kv_len;
        float before = 0.f;
        if (old && stores && (chunk || pos0 + tok < L)) before = keep * reinterpret_cast<const float*>(pg + SH::kWeights)[tok];
        uint32_t a[D / 16][4];
        float sk[2] = {P.scale_log2, P.scale_log2}, mk[2] = {0.f, 0.f};
#pragma unroll
        for (int e2 = 0; e2 < 2; ++e2) {
          const int tk = g + 8 * e2;
          if (FOUR) {
            uint32_t word[4];
            if (NW == 4) {
              const uint4 v = *reinterpret_cast<const uint4*>(pg + tk * (D / 2) + t * 16);
              word[0] = v.x; word[1] = v.y; word[2] = v.z; word[3] = v.w;
            } else {
              const uint2 v = *reinterpret_cast<const uint2*>(pg + tk * (D / 2) + t * 8);
              word[0] = v.x; word[1] = v.y;
            }
            const uint32_t pair = *reinterpret_cast<const uint32_t*>(pg + SH::kCodes + 4 * tk);
            sk[e2] = kv4_step(pair);
            mk[e2] = kv4_min(pair);
#pragma unroll
            for (int j = 0; j < NW; ++j)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const uint32_t w = u ? word[j] >> 8 : word[j];
                a[2 * j + u][e2] = w & 0x000f000fu;
                a[2 * j + u][e2 + 2] = w & 0x00f000f0u;
              }
          }
        }
        if (!FOUR) {           // matrices: tokens 0..7 and 8..15 of values 16 k .., then of 16 k + 8 ..
          const uint32_t tk = lane & 15, half = lane >> 4, pg_at = smem_u32(pg);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)
            ldmatrix_x4(a[k][0], a[k][1], a[k][2], a[k][3], pg_at + 2 * kv_tile_offset(tk, 16 * k + 8 * half, D));
        }
        __syncwarp();
        request(slot_at);
        slot_at = slot_at == (SH::kSlots - 1) * SH::kPage ? 0 : slot_at + SH::kPage;
        float acc[2] = {0.f, 0.f};
        auto walk = [&](auto masked) {
          constexpr bool MASK = decltype(masked)::value;
#pragma unroll 1
          for (int nt = 0; nt < rows8; nt += 8) {
            float sc[2][4];
#pragma unroll
            for (int j = 0; j < NW; ++j) {
              const uint4 b = *reinterpret_cast<const uint4*>(rows_at + (nt + g) * SH::kRowBytes + (j * 4 + t) * 16);
              if (j == 0) {
                mma<FOUR, true>(sc[0], a[0], b.x, b.y);
                mma<FOUR, true>(sc[1], a[1], b.z, b.w);
              } else {
                mma<FOUR, false>(sc[0], a[2 * j], b.x, b.y);
                mma<FOUR, false>(sc[1], a[2 * j + 1], b.z, b.w);
              }
            }
            const float4 i0 = info_at[nt + 2 * t], i1 = info_at[nt + 2 * t + 1];
            int4 v0, v1;
            if (MASK) {
              v0 = vis_at[nt + 2 * t];
              v1 = vis_at[nt + 2 * t + 1];
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float4& ri = (x & 1) ? i1 : i0;
              const float shift = FOUR ? fmaf(mk[x >> 1], ri.x, ri.y) : ri.y;
              const float p_ = exp2f(fmaf(sc[0][x] + sc[1][x], FOUR ? sk[x >> 1] * ri.w : sk[x >> 1], shift));
              if (MASK) {
                const int4& vi = (x & 1) ? v1 : v0;
                const int pos = pos0 + g + 8 * (x >> 1);
                if (pos <= vi.x || (pos >= vi.y && pos < vi.z)) acc[x >> 1] = fmaf(p_, ri.z, acc[x >> 1]);
              } else {
                acc[x >> 1] = fmaf(p_, ri.z, acc[x >> 1]);
              }
            }
          }
        };
        if (pos0 + kPageSize - 1 > lim) walk(std::true_type{});
        else walk(std::false_type{});
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          acc[x] += __shfl_xor_sync(0xffffffffu, acc[x], 1);
          acc[x] += __shfl_xor_sync(0xffffffffu, acc[x], 2);
        }
        if (stores) out_at[((uint64_t)id * (unsigned)P.n_kv + h) * kPageSize] = before + (t ? acc[1] : acc[0]);
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
      const bool more = first_tok < s_new[0] && !whole;
      __syncthreads();                                   // the staged rows may be replaced
      if (!more) break;
      if (tid == 0) s_lim[0] = 0x7fffffff;
    }
    pair += nseg;
    ahead = s_ahead[nseg - 1];
    __syncthreads();
  }
}

template <int D, bool FOUR>
void launch_shape(const Params& P, int n_sm, cudaStream_t st) {
  constexpr int kMost = Shape<D, FOUR>::kTotal + kMaxLayoutRequests * (int)sizeof(int);
  static_assert(Shape<D, FOUR>::kTotal >= (kMaxLayoutRequests + 1) * (int)sizeof(long long), "the sums fit where rings and rows are");
  static_assert(kMost <= 227 * 1024, "shared memory budget");
  static bool configured[kMaxDevices] = {false};
  if (first_use_on_device(configured)) cudaFuncSetAttribute(kv_weights_kernel<D, FOUR>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
  launch_pdl(kv_weights_kernel<D, FOUR>, dim3(n_sm), dim3(Shape<D, FOUR>::kThreads), Shape<D, FOUR>::kTotal + P.n_req * sizeof(int), st, P);
}

}  // namespace

void launch_kv_weights(const BatchLayout& bl, const Dims& dm, int layer, const void* q, const float* lse, const float* row_weight,
                       float decay, const float* in, float* out, const void* pool, int64_t n_pages, bool four, int n_sm, int* status,
                       cudaStream_t st) {
  Params P;
  P.ctx_len = bl.ctx_len;
  P.cu_tok = bl.cu_tok;
  P.page_table = bl.page_table;
  P.pt_stride = bl.pt_stride;
  P.n_req = bl.n_req;
  P.verify_len = bl.verify_len;
  P.tok_climit = bl.tok_climit;
  P.tok_lo = bl.tok_lo;
  P.tok_hi = bl.tok_hi;
  P.q = static_cast<const __nv_bfloat16*>(q);
  P.lse = lse;
  P.row_weight = row_weight;
  P.in = in;
  P.out = out;
  P.decay = decay;
  P.pool = static_cast<const uint8_t*>(pool);
  P.n_pages = n_pages;
  P.layer = layer;
  P.n_q = dm.n_q;
  P.n_kv = dm.n_kv;
  P.group = dm.n_q / dm.n_kv;
  P.scale_log2 = 1.4426950408889634f / sqrtf((float)dm.head_dim);
  P.status = status;
  if (dm.head_dim == 128) (four ? launch_shape<128, true> : launch_shape<128, false>)(P, n_sm, st);
  else (four ? launch_shape<64, true> : launch_shape<64, false>)(P, n_sm, st);
}

}  // namespace recg

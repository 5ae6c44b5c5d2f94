// The attention weight that cached tokens gather (recg_kv_weights): per kv head and position j
//   out[j] = (j < L ? decay in[j] : 0) + sum over the rows t and the query heads of the group of w_t exp(score_tj - lse_t).
// With the log-sum-exp of every row from the attention kernel each probability follows from its score alone, so one pass over K
// gives them: S^T = K Q^T with the tokens as rows of the product.  A warp owns the 16 tokens of a page, keeps their K as A operands in
// registers and walks over the query rows; the sum over rows is a sum over the columns of its accumulators, which stay in the
// warp.  Nothing is added by atomics: a position belongs to one warp, which takes the rows in order, so results repeat bit for bit.
//
// K of either kind of pool is read straight into operands: a lane holds the values [D / 4 t, D / 4 (t + 1)) of two tokens (t its
// number in the quad), which are contiguous; the contraction index is permuted accordingly and Q is staged in shared memory in
// that order.  Codes are exact in bf16, steps and minima enter in fp32 (kv4.cuh), so the scores are those of the attention kernel.
#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kTileTokens = kWarps * kPageSize;
constexpr int kChunkRows = 64;              // query rows staged at a time

struct Params {
  const int* ctx_len;
  const int* cu_tok;
  const int* page_table;
  int pt_stride, n_req;
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

struct RowInfo {              // a staged query row
  float qsum, lse2, weight;   // sum of its values, its log-sum-exp in powers of two, what its probabilities count
  int climit, lo, hi;
};

template <int D, bool FOUR>
__global__ void __launch_bounds__(kThreads, 2) kv_weights_kernel(Params P) {
  constexpr int NW = D / 32, kChunks = D / 8;
  constexpr int kRowChunks = kChunks + 4;     // 16-byte chunks from row to row: lanes of eight rows meet no bank twice
  __shared__ uint4 s_q[kChunkRows * kRowChunks];
  __shared__ RowInfo s_row[kChunkRows];
  __shared__ int s_scan[kWarps];
  extern __shared__ int s_tiles[];            // [n_req + 1] token tiles (one kv head) in front of request r
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  griddep_wait();
  griddep_launch();
  auto kv_len_of = [&](int r) { return P.ctx_len[r] + P.cu_tok[r + 1] - P.cu_tok[r]; };
  {
    const int per = (P.n_req + kThreads - 1) / kThreads, r0 = min(P.n_req, tid * per), r1 = min(P.n_req, r0 + per);
    int mine = 0;
    for (int r = r0; r < r1; ++r) mine += (kv_len_of(r) + kTileTokens - 1) / kTileTokens;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) s_scan[warp] = incl;
    __syncthreads();
    int at = incl - mine;
    for (int k = 0; k < warp; ++k) at += s_scan[k];
    for (int r = r0; r < r1; ++r) {
      s_tiles[r] = at;
      at += (kv_len_of(r) + kTileTokens - 1) / kTileTokens;
    }
    if (tid == kThreads - 1) s_tiles[P.n_req] = at;
    __syncthreads();
  }
  const int n_items = s_tiles[P.n_req] * P.n_kv;     // (item = token tile * n_kv + head)

  for (int item = blockIdx.x; item < n_items; item += gridDim.x) {
    const int tile = item / P.n_kv, h = item - tile * P.n_kv;
    int lo_r = 0, hi_r = P.n_req;                     // largest r with s_tiles[r] <= tile (every request has a tile)
    while (hi_r - lo_r > 1) {
      const int mid = (lo_r + hi_r) >> 1;
      if (s_tiles[mid] <= tile) lo_r = mid; else hi_r = mid;
    }
    const int r = lo_r, tok_first = P.cu_tok[r], n_new = P.cu_tok[r + 1] - tok_first, L = P.ctx_len[r], kv_len = L + n_new;
    const int pos0 = (tile - s_tiles[r]) * kTileTokens + warp * kPageSize;
    int page = -1;
    if (pos0 < kv_len) {
      page = P.page_table[(size_t)r * P.pt_stride + pos0 / kPageSize];
      if (page < 0 || page >= P.n_pages) {
        set_status(P.status, DEV_BAD_INDEX);
        page = -1;
      }
    }
    // ---- K of the warp's page as A operands: rows g and g + 8 are its tokens ----
    uint32_t a[D / 16][4];
    float sk[2] = {P.scale_log2, P.scale_log2}, mk[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < D / 16; ++k) a[k][0] = a[k][1] = a[k][2] = a[k][3] = 0;
    if (page >= 0) {
      if (FOUR) {
        const uint8_t* block = P.pool + kv4_block_base(P.n_pages, P.n_kv, D, P.layer, page, h);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          uint32_t word[4];
          const uint8_t* src = block + (g + 8 * e) * (D / 2) + t * (NW * 4);
          if (NW == 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(src));
            word[0] = v.x; word[1] = v.y; word[2] = v.z; word[3] = v.w;
          } else {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(src));
            word[0] = v.x; word[1] = v.y;
          }
          const uint32_t pair = __ldg(reinterpret_cast<const uint32_t*>(block + kv4_k_pairs(D)) + g + 8 * e);
          sk[e] = kv4_step(pair) * P.scale_log2;
          mk[e] = fmaf(8.f, kv4_step(pair), kv4_min(pair)) * P.scale_log2;
#pragma unroll
          for (int j = 0; j < NW; ++j)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              a[2 * j + u][e] = kv4_pair(word[j], 2 * u);
              a[2 * j + u][e + 2] = kv4_pair(word[j], 2 * u + 1);
            }
        }
      } else {
        const uint8_t* block = P.pool + 2 * kv_tile_base(P.n_pages, P.n_kv, D, P.layer, page, h);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int j = 0; j < NW; ++j) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(block + 2 * kv_tile_offset(g + 8 * e, t * (D / 4) + 8 * j, D)));
            a[2 * j][e] = v.x;
            a[2 * j][e + 2] = v.y;
            a[2 * j + 1][e] = v.z;
            a[2 * j + 1][e + 2] = v.w;
          }
      }
    }
    float acc[2] = {0.f, 0.f};
    const int R = n_new * P.group;
    for (int row0 = 0; row0 < R; row0 += kChunkRows) {
      // ---- stage the next rows: chunk c of a row at (c % NW) * 4 + c / NW, where lane c / NW of a quad looks for it ----
      __syncthreads();
      const int rows = min(kChunkRows, R - row0), rows8 = (rows + 7) & ~7;
      for (int i = tid; i < rows8 * kChunks; i += kThreads) {
        const int row = i / kChunks, c = i - row * kChunks, rho = row0 + row;
        const int tok = tok_first + rho / P.group, head = h * P.group + rho % P.group;
        const uint4 v = row < rows ? __ldg(reinterpret_cast<const uint4*>(P.q + ((size_t)tok * P.n_q + head) * D) + c) : make_uint4(0, 0, 0, 0);
        s_q[row * kRowChunks + (c % NW) * 4 + c / NW] = v;
        float sum = 0.f;
        if (FOUR) {
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) sum += __uint_as_float(u[k] << 16) + __uint_as_float(u[k] & 0xffff0000u);
          // (rows8 * kChunks is a multiple of 64 and kThreads of kChunks: whole quarter and half warps come here together)
          const unsigned group_mask = (kChunks == 16 ? 0xffffu : 0xffu) << (lane & ~(kChunks - 1));
#pragma unroll
          for (int o = kChunks / 2; o; o >>= 1) sum += __shfl_xor_sync(group_mask, sum, o);
        }
        if (c == 0) {
          RowInfo ri = {sum, 0.f, 0.f, 0x7fffffff, 0, 0};
          if (row < rows) {
            ri.weight = P.row_weight ? P.row_weight[tok] : 1.f;
            ri.lse2 = P.lse[(size_t)tok * P.n_q + head] * 1.4426950408889634f;
            ri.climit = P.tok_climit[tok];
            ri.lo = P.tok_lo[tok];
            ri.hi = P.tok_hi[tok];
          }
          s_row[row] = ri;
        }
      }
      __syncthreads();
      if (page < 0) continue;
      for (int nt = 0; nt < rows8; nt += 8) {
        const RowInfo r0 = s_row[nt + 2 * t], r1 = s_row[nt + 2 * t + 1];
        if (!__any_sync(0xffffffffu, r0.weight != 0.f || r1.weight != 0.f)) continue;
        float sc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NW; ++j) {
          const uint4 b = s_q[(nt + g) * kRowChunks + j * 4 + t];
          mma_bf16_16816(sc, a[2 * j], b.x, b.y);
          mma_bf16_16816(sc, a[2 * j + 1], b.z, b.w);
        }
        const bool need_mask = __any_sync(0xffffffffu, pos0 + kPageSize - 1 > min(r0.climit, r1.climit));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const RowInfo& ri = (e & 1) ? r1 : r0;
          float p = exp2f(fmaf(sc[e], sk[e >> 1], fmaf(mk[e >> 1], ri.qsum, -ri.lse2)));
          const int pos = pos0 + g + 8 * (e >> 1);
          bool counts = ri.weight != 0.f;
          if (need_mask) counts = counts && (pos <= ri.climit || (pos >= ri.lo && pos < ri.hi));
          if (counts) acc[e >> 1] = fmaf(p, ri.weight, acc[e >> 1]);
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 1);
      acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 2);
    }
    const int tok = g + 8 * t, pos = pos0 + tok;       // lane 0 of a quad stores row g, lane 1 row g + 8
    if (t < 2 && page >= 0 && pos < kv_len) {
      const size_t at = (((size_t)P.layer * P.n_pages + page) * P.n_kv + h) * kPageSize + tok;
      const float before = P.in && pos < L && P.decay != 0.f ? P.decay * P.in[at] : 0.f;
      P.out[at] = before + (t ? acc[1] : acc[0]);
    }
  }
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
  auto* kernel = dm.head_dim == 128 ? (four ? kv_weights_kernel<128, true> : kv_weights_kernel<128, false>)
                                    : (four ? kv_weights_kernel<64, true> : kv_weights_kernel<64, false>);
  launch_pdl(kernel, dim3(2 * n_sm), dim3(kThreads), (bl.n_req + 1) * sizeof(int), st, P);
}

}  // namespace recg

// Eviction from the cache by gathered attention weight: which positions every kv head of every layer keeps (recg_kv_select), and
// the move of their K, V and weights to the front of the request's pages or to other pages (recg_kv_compact).
#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

// ---- selection ------------------------------------------------------------------------------------------------------------
// Per (layer, request, kv head) the n-th largest weight is found by counting the keys' digits from the top (11, 11 and 10 bits),
// and one more pass lists what lies above it, with the first of its equals, in ascending order.  A thread takes a page, 64
// contiguous bytes; the weights are read from memory once and from L2 after that.  All counts are integers: the list does not depend
// on the order of threads.
constexpr int kSelThreads = 512;
constexpr int kBins = 2048;

// larger weight, larger key; -0 and 0 are equal, NaN is below everything
__device__ __forceinline__ uint32_t weight_key(float w) {
  uint32_t u = __float_as_uint(w);      // (compared as bits: the arithmetic of this build takes subnormal numbers for zero)
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if ((u << 1) == 0) u = 0;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelThreads) kv_select_kernel(EvictDesc E, const float* __restrict__ weights, int64_t n_pages, int n_kv,
                                                                int* __restrict__ keep, int keep_stride) {
  __shared__ int hist[kBins];
  __shared__ int s_scan[2][kSelThreads / 32];
  __shared__ int s_pick[2];
  const int h = blockIdx.x, r = blockIdx.y, layer = E.layer_begin + blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  griddep_wait();
  griddep_launch();
  const int L = E.ctx_len[r], n_keep = E.kept[r];
  int* out = keep + (((size_t)blockIdx.z * E.n_req + r) * n_kv + h) * keep_stride;
  for (int i = n_keep + tid; i < keep_stride; i += kSelThreads) out[i] = -1;
  if (n_keep >= L) {
    for (int i = tid; i < n_keep; i += kSelThreads) out[i] = i;
    return;
  }
  const int* pt = E.page_table + (size_t)r * E.pt_stride;
  const int lo = E.n_sink, hi = L - E.n_recent;        // candidates; n_sink + n_recent <= n_keep < L
  const int pages = (L + kPageSize - 1) / kPageSize;
  auto page_keys = [&](int p, uint32_t (&key)[kPageSize]) {
    const float4* src = reinterpret_cast<const float4*>(weights + (((size_t)layer * n_pages + pt[p]) * n_kv + h) * kPageSize);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4 v = src[c];
      key[4 * c] = weight_key(v.x);
      key[4 * c + 1] = weight_key(v.y);
      key[4 * c + 2] = weight_key(v.z);
      key[4 * c + 3] = weight_key(v.w);
    }
  };
  // ---- the key of the last one that stays, and how many of its equals do ----
  uint32_t prefix = 0, known = 0;                      // digits found so far, and the mask of their bits
  int want = n_keep - E.n_sink - E.n_recent;           // among the keys with that prefix
  const bool none = want == 0;
  for (int pass = 0; pass < 3 && !none; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : kBins;
    for (int i = tid; i < bins; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int p = lo / kPageSize + tid; p < pages; p += kSelThreads) {
      uint32_t key[kPageSize];
      page_keys(p, key);
#pragma unroll
      for (int i = 0; i < kPageSize; ++i) {
        const int j = p * kPageSize + i;
        if (j >= lo && j < hi && (key[i] & known) == prefix) atomicAdd(&hist[(key[i] >> shift) & (bins - 1)], 1);
      }
    }
    __syncthreads();
    // the bin in which the want-th largest lies: a scan from the top, four (two) bins a thread
    const int per = bins / kSelThreads, top = bins - 1 - tid * per;
    int mine = 0;
    for (int k = 0; k < per; ++k) mine += hist[top - k];
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 31) s_scan[0][warp] = incl;
    __syncthreads();
    for (int k = 0; k < warp; ++k) incl += s_scan[0][k];
    int above = incl - mine;
    if (above < want && want <= incl)
      for (int k = 0; k < per; ++k) {
        const int c = hist[top - k];
        if (above < want && want <= above + c) {
          s_pick[0] = top - k;
          s_pick[1] = want - above;
        }
        above += c;
      }
    __syncthreads();
    prefix |= (uint32_t)s_pick[0] << shift;
    known |= (uint32_t)(bins - 1) << shift;
    want = s_pick[1];
    __syncthreads();
  }
  // ---- the list: pages in order, kSelThreads at a time ----
  int n_out = 0, n_eq = 0;
  for (int p0 = 0; p0 < pages; p0 += kSelThreads) {
    const int p = p0 + tid;
    unsigned sure = 0, equal = 0;                      // bits of the page's tokens
    if (p < pages) {
      uint32_t key[kPageSize];
      page_keys(p, key);
#pragma unroll
      for (int i = 0; i < kPageSize; ++i) {
        const int j = p * kPageSize + i;
        if (j < L && (j < lo || j >= hi || (!none && key[i] > prefix))) sure |= 1u << i;
        else if (j < L && !none && key[i] == prefix) equal |= 1u << i;
      }
    }
    int a = __popc(sure), b = __popc(equal);
    int ia = a, ib = b;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int ya = __shfl_up_sync(0xffffffffu, ia, o), yb = __shfl_up_sync(0xffffffffu, ib, o);
      if (lane >= o) { ia += ya; ib += yb; }
    }
    if (lane == 31) { s_scan[0][warp] = ia; s_scan[1][warp] = ib; }
    __syncthreads();
    int ta = 0, tb = 0;
    for (int k = 0; k < kSelThreads / 32; ++k) {
      if (k < warp) { ia += s_scan[0][k]; ib += s_scan[1][k]; }
      ta += s_scan[0][k];
      tb += s_scan[1][k];
    }
    const int eq_before = n_eq + ib - b;               // equals in front of this page: the first `want` of all stay
    int at = n_out + (ia - a) + min(eq_before, want) - min(n_eq, want);
    int eq = eq_before;
    for (unsigned m = sure | equal; m; m &= m - 1) {
      const int i = __ffs(m) - 1;
      const bool stays = ((sure >> i) & 1u) || eq++ < want;
      if (stays) out[at++] = p * kPageSize + i;
    }
    n_out += ta + min(n_eq + tb, want) - min(n_eq, want);
    n_eq += tb;
    __syncthreads();
  }
}

// ---- compaction -----------------------------------------------------------------------------------------------------------
// Slot i takes what lies in slot keep[i], a warp a page of 16 at a time: K, V and weight of its tokens are read, and when every
// read that an earlier write could spoil is done, written.  In place keep[i] >= i, so the pages of a round read nothing in front of
// the first of them: one barrier between the reads and the writes of a round is all the order that there has to be.
constexpr int kMoveWarps = 8, kMoveThreads = kMoveWarps * 32;

template <int D, bool FOUR>
__global__ void __launch_bounds__(kMoveThreads) kv_compact_kernel(EvictDesc E, uint8_t* pool, float* weights, int64_t n_pages, int n_kv,
                                                                  const int* __restrict__ keep, int keep_stride, int* status) {
  const int h = blockIdx.x, r = blockIdx.y / E.splits, split = blockIdx.y % E.splits, layer = E.layer_begin + blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  griddep_wait();
  griddep_launch();
  const int L = E.ctx_len[r], n_keep = E.kept[r];
  const bool in_place = E.dst_table == nullptr;
  if (in_place && n_keep >= L) return;
  const int* list = keep + (((size_t)blockIdx.z * E.n_req + r) * n_kv + h) * keep_stride;
  const int* src_pt = E.page_table + (size_t)r * E.pt_stride;
  const int* dst_pt = in_place ? src_pt : E.dst_table + (size_t)r * E.dst_stride;
  const int pages = (n_keep + kPageSize - 1) / kPageSize;
  constexpr int kBlock = FOUR ? kv4_block_bytes(D) : 4 * kPageSize * D;       // bytes of a page and head
  auto block_of = [&](int page) { return pool + (((size_t)layer * n_pages + page) * n_kv + h) * (size_t)kBlock; };
  // (out of place: `splits` CTAs share the pages; in place one CTA takes them in order)
  const int step = kMoveWarps * E.splits;
  for (int p0 = split * kMoveWarps; p0 < pages; p0 += step) {
    const int p = p0 + warp;
    // lane i < 16: where token i of the page comes from
    int src = -1;
    if (p < pages && lane < kPageSize && p * kPageSize + lane < n_keep) {
      src = list[p * kPageSize + lane];
      if (src < 0 || src >= L || (in_place && src < p * kPageSize + lane)) {
        set_status(status, DEV_BAD_INDEX);
        src = -1;
      }
    }
    const int src_page = src >= 0 ? src_pt[src / kPageSize] : 0;
    const unsigned valid = __ballot_sync(0xffffffffu, src >= 0);
    const bool moves = __any_sync(0xffffffffu, src >= 0 && (!in_place || src != p * kPageSize + lane));
    uint8_t* dst = p < pages ? block_of(dst_pt[p]) : nullptr;
    float wt = 0.f;
    const size_t w_head = (size_t)n_kv * kPageSize;
    if (moves && weights && src >= 0) wt = weights[((size_t)layer * n_pages + src_page) * w_head + h * kPageSize + (src & 15)];
    if constexpr (FOUR) {
      constexpr int kC = D / 32;           // 16-byte chunks of a K row
      constexpr int kK = kC / 2 > 0 ? 16 * kC / 32 : 1, kV = 8 * (D / 4) / 32;
      uint4 kr[kK];
      uint32_t vr[kV], pair = 0;
      if (moves) {
#pragma unroll
        for (int u = 0; u < kK; ++u) {
          const int i = u * 32 + lane, tok = i / kC, c = i % kC;
          const int s = __shfl_sync(0xffffffffu, src, tok), sp = __shfl_sync(0xffffffffu, src_page, tok);
          if (s >= 0) kr[u] = *reinterpret_cast<const uint4*>(block_of(sp) + kv4_k_word(s & 15, 4 * c, D));
        }
#pragma unroll
        for (int u = 0; u < kV; ++u) {     // word x of token pair q: halves of the same word of two source tokens
          const int i = u * 32 + lane, q = i / (D / 4), x = i % (D / 4);
          uint32_t half[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int s = __shfl_sync(0xffffffffu, src, 2 * q + e), sp = __shfl_sync(0xffffffffu, src_page, 2 * q + e);
            half[e] = s >= 0 ? *reinterpret_cast<const uint16_t*>(block_of(sp) + kv4_v_codes(D) + ((s & 15) >> 1) * D + 4 * x + 2 * (s & 1)) : 0;
          }
          vr[u] = half[0] | half[1] << 16;
        }
        // lanes 0..15 the K pairs, 16..31 the V pairs
        const int s = __shfl_sync(0xffffffffu, src, lane & 15), sp = __shfl_sync(0xffffffffu, src_page, lane & 15);
        if (s >= 0) pair = *reinterpret_cast<const uint32_t*>(block_of(sp) + (lane < 16 ? kv4_k_pairs(D) : kv4_v_pairs(D)) + 4 * (s & 15));
      }
      if (in_place) __syncthreads();
      if (moves) {
#pragma unroll
        for (int u = 0; u < kK; ++u) {
          const int i = u * 32 + lane, tok = i / kC, c = i % kC;
          if ((valid >> tok) & 1u) *reinterpret_cast<uint4*>(dst + kv4_k_word(tok, 4 * c, D)) = kr[u];
        }
#pragma unroll
        for (int u = 0; u < kV; ++u) {
          const int i = u * 32 + lane, q = i / (D / 4), x = i % (D / 4);
          uint8_t* at = dst + kv4_v_codes(D) + q * D + 4 * x;
          const unsigned have = (valid >> (2 * q)) & 3u;
          if (have == 3u) *reinterpret_cast<uint32_t*>(at) = vr[u];
          else if (have == 1u) *reinterpret_cast<uint16_t*>(at) = (uint16_t)vr[u];
          else if (have == 2u) *reinterpret_cast<uint16_t*>(at + 2) = (uint16_t)(vr[u] >> 16);
        }
        if ((valid >> (lane & 15)) & 1u)
          *reinterpret_cast<uint32_t*>(dst + (lane < 16 ? kv4_k_pairs(D) : kv4_v_pairs(D)) + 4 * (lane & 15)) = pair;
      }
    } else {
      constexpr int kC = D / 8, kN = kPageSize * kC / 32;      // 16-byte chunks of a row; per lane of a tile
      uint4 kr[kN], vr[kN];
      if (moves) {
#pragma unroll
        for (int u = 0; u < kN; ++u) {
          const int i = u * 32 + lane, tok = i / kC, c = i % kC;
          const int s = __shfl_sync(0xffffffffu, src, tok), sp = __shfl_sync(0xffffffffu, src_page, tok);
          if (s < 0) continue;
          const uint8_t* at = block_of(sp) + 2 * kv_tile_offset(s & 15, 8 * c, D);
          kr[u] = *reinterpret_cast<const uint4*>(at);
          vr[u] = *reinterpret_cast<const uint4*>(at + 2 * kPageSize * D);
        }
      }
      if (in_place) __syncthreads();
      if (moves) {
#pragma unroll
        for (int u = 0; u < kN; ++u) {
          const int i = u * 32 + lane, tok = i / kC, c = i % kC;
          if (!((valid >> tok) & 1u)) continue;
          uint8_t* at = dst + 2 * kv_tile_offset(tok, 8 * c, D);
          *reinterpret_cast<uint4*>(at) = kr[u];
          *reinterpret_cast<uint4*>(at + 2 * kPageSize * D) = vr[u];
        }
      }
    }
    if (moves && weights && src >= 0) weights[((size_t)layer * n_pages + dst_pt[p]) * w_head + h * kPageSize + lane] = wt;
  }
}

}  // namespace

void launch_kv_select(const EvictDesc& E, const float* weights, int64_t n_pages, int n_kv, int n_layers, int* keep, int keep_stride,
                      cudaStream_t st) {
  launch_pdl(kv_select_kernel, dim3(n_kv, E.n_req, n_layers), dim3(kSelThreads), 0, st, E, weights, n_pages, n_kv, keep, keep_stride);
}

void launch_kv_compact(EvictDesc E, const Dims& dm, void* pool, float* weights, int64_t n_pages, bool four, int n_layers, int max_keep,
                       const int* keep, int keep_stride, int* status, cudaStream_t st) {
  const int rounds = (max_keep + kMoveWarps * kPageSize - 1) / (kMoveWarps * kPageSize);
  E.splits = E.dst_table ? (rounds < 8 ? (rounds > 0 ? rounds : 1) : 8) : 1;
  auto* kernel = dm.head_dim == 128 ? (four ? kv_compact_kernel<128, true> : kv_compact_kernel<128, false>)
                                    : (four ? kv_compact_kernel<64, true> : kv_compact_kernel<64, false>);
  launch_pdl(kernel, dim3(dm.n_kv, E.n_req * E.splits, n_layers), dim3(kMoveThreads), 0, st, E, static_cast<uint8_t*>(pool), weights, n_pages,
             dm.n_kv, keep, keep_stride, status);
}

}  // namespace recg

// Eviction from the cache by gathered attention weight: which positions every kv head of every layer keeps (recg_kv_select), and
// the move of their K, V and weights to the front of the request's pages or to other pages (recg_kv_compact).
#include <type_traits>

#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

// ---- selection ------------------------------------------------------------------------------------------------------------
// Per (layer, request, kv head) the key of the last weight that stays is found bit by bit from the top, by counting the keys that are
// not below the bits so far and the next one.  A thread keeps the keys of its pages in registers, so a bit costs it a comparison a key
// and one sum over the threads (over the CTAs of a cluster for long contexts); bits that all keys share are not counted, and when the
// keys in question are few every warp goes on by itself.  Then every
// thread lists what stays of its pages, behind those in front of it.  All counts are integers: the list does not depend on the order of
// threads.  (Counting digits in shared memory instead: weights lie close together and many are zero, so that the counters were hit by
// many lanes at once: 38 us for four requests of 8192 to 16384 tokens, 8 heads, 8 layers; now 28.)
constexpr int kSelThreads = 1024, kSelWarps = kSelThreads / 32;      // at most: a CTA has as many as there are pages for
constexpr int kMaxCluster = 8;
constexpr int kClose = 256;                           // keys in question that every warp resolves by itself

// larger weight, larger key; -0 and 0 are equal, NaN is below everything
__device__ __forceinline__ uint32_t weight_key(float w) {
  uint32_t u = __float_as_uint(w);      // (compared as bits: the arithmetic of this build takes subnormal numbers for zero)
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0;
  if ((u << 1) == 0) u = 0;
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// KEPT: pages whose keys a thread keeps (0: any number, read again for every bit)
template <int KEPT>
__global__ void __launch_bounds__(kSelThreads) kv_select_kernel(EvictDesc E, const float* __restrict__ weights, int64_t n_pages, int n_kv,
                                                                int* __restrict__ keep, int keep_stride) {
  __shared__ int s_warp[2][kSelWarps];
  __shared__ uint32_t s_close[kClose];
  __shared__ int s_n_close;
  __shared__ int s_cta[2][2][kMaxCluster];             // [use][sure, equal] of every CTA of the cluster
  const int h = blockIdx.x / E.splits, rank = blockIdx.x % E.splits, r = blockIdx.y, layer = E.layer_begin + blockIdx.z;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, ctas = E.splits, threads = blockDim.x, n_warps = threads >> 5;
  griddep_wait();
  griddep_launch();
  const int L = E.ctx_len[r], n_keep = E.kept[r];
  int* out = keep + (((size_t)blockIdx.z * E.n_req + r) * n_kv + h) * keep_stride;
  for (int i = n_keep + rank * threads + tid; i < keep_stride; i += ctas * threads) out[i] = -1;
  if (n_keep >= L) {                                   // (the whole cluster)
    for (int i = rank * threads + tid; i < n_keep; i += ctas * threads) out[i] = i;
    return;
  }
  const int* pt = E.page_table + (size_t)r * E.pt_stride;
  const int lo = E.n_sink, hi = L - E.n_recent;        // candidates; n_sink + n_recent <= n_keep < L
  const int pages = (L + kPageSize - 1) / kPageSize, per = (pages + ctas * threads - 1) / (ctas * threads);
  const int page0 = min(pages, (rank * threads + tid) * per), page1 = min(pages, page0 + per);      // this thread's
  // keys of a page; 0, which no weight but NaN has, for what is no candidate (found: it is one)
  auto page_keys = [&](int p, uint32_t (&key)[kPageSize], unsigned& candidates) {
    candidates = 0;
    if (p >= page1) {
#pragma unroll
      for (int i = 0; i < kPageSize; ++i) key[i] = 0;
      return;
    }
    const float4* src = reinterpret_cast<const float4*>(weights + (((size_t)layer * n_pages + pt[p]) * n_kv + h) * kPageSize);
    const int from = max(lo - p * kPageSize, 0), to = min(hi - p * kPageSize, kPageSize);
    candidates = to > from ? (0xffffu >> (kPageSize - to)) & (0xffffu << from) : 0u;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float4 v = src[c];
      key[4 * c] = weight_key(v.x);
      key[4 * c + 1] = weight_key(v.y);
      key[4 * c + 2] = weight_key(v.z);
      key[4 * c + 3] = weight_key(v.w);
    }
    if (candidates != 0xffffu) {
#pragma unroll
      for (int i = 0; i < kPageSize; ++i) key[i] = (candidates >> i) & 1u ? key[i] : 0u;
    }
  };
  constexpr int kHeld = KEPT ? KEPT : 1;
  uint32_t key[kHeld][kPageSize];
  unsigned candidates[kHeld];
  if (KEPT) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) page_keys(page0 + k, key[k], candidates[k]);
  }
  if (ctas > 1) asm volatile("barrier.cluster.arrive.aligned;\n barrier.cluster.wait.aligned;" ::: "memory");      // all have started
  int use = 0;
  // the sum (or largest) over all threads of the cluster
  auto over_all = [&](uint32_t mine, auto largest) {
    constexpr bool MAX = decltype(largest)::value;
    auto over_warp = [](uint32_t v) { return MAX ? __reduce_max_sync(0xffffffffu, v) : __reduce_add_sync(0xffffffffu, v); };
    const uint32_t w = over_warp(mine);
    use ^= 1;
    if (lane == 0) s_warp[use][warp] = (int)w;
    __syncthreads();
    uint32_t total = over_warp(lane < n_warps ? (uint32_t)s_warp[use][lane] : 0u);
    if (ctas > 1) {
      if (tid < ctas) {
        uint32_t at;
        asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&s_cta[use][0][rank])), "r"(tid));
        asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(total) : "memory");
      }
      asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
      total = 0;
      for (int c = 0; c < ctas; ++c) {
        const uint32_t v = (uint32_t)s_cta[use][0][c];
        total = MAX ? max(total, v) : total + v;
      }
    }
    return total;
  };
  auto sum_all = [&](int n) { return (int)over_all((uint32_t)n, std::false_type{}); };
  auto each_key = [&](auto f) {                        // f(key, is it a candidate's)
    if (KEPT) {
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
#pragma unroll
        for (int i = 0; i < kPageSize; ++i) f(key[k][i], (candidates[k] >> i) & 1u);
    } else {
      for (int p = page0; p < page1; ++p) {
        page_keys(p, key[0], candidates[0]);
#pragma unroll
        for (int i = 0; i < kPageSize; ++i) f(key[0][i], (candidates[0] >> i) & 1u);
      }
    }
  };
  // ---- the largest bound that at least `want` keys reach; if more do, its equals are taken in order ----
  const int want = n_keep - E.n_sink - E.n_recent;
  uint32_t bound = 0, above = 0xffffffffu;             // as many keys as wanted reach the bound, fewer reach `above`
  int reach = hi - lo, reach_above = 0;
  int bit = -1;
  if (want > 0) {
    // (the bits that all keys share need no counting)
    uint32_t top = 0, low = 0;
    each_key([&](uint32_t k, unsigned is) {
      top = max(top, k);
      low = max(low, is ? ~k : 0u);
    });
    top = over_all(top, std::true_type{});
    low = ~over_all(low, std::true_type{});
    bit = top == low ? -1 : 31 - __clz(top ^ low);
    bound = bit < 0 ? top : (bit == 31 ? 0u : top & ~((2u << bit) - 1u));
  }
  for (; bit >= 0 && reach != want && (ctas > 1 || reach - reach_above > kClose); --bit) {
    const uint32_t test = bound | (1u << bit);
    int n = 0;
    each_key([&](uint32_t k, unsigned) { n += k >= test; });
    const int total = sum_all(n);
    if (total >= want) {
      bound = test;
      reach = total;
    } else {
      above = test;
      reach_above = total;
    }
  }
  if (bit >= 0 && reach != want) {
    // few enough are left between the two: every warp goes on with them by itself, without a barrier per bit
    if (tid == 0) s_n_close = 0;
    __syncthreads();
    each_key([&](uint32_t k, unsigned is) {
      if (is && k >= bound && k < above) s_close[atomicAdd(&s_n_close, 1)] = k;
    });
    __syncthreads();
    uint32_t mine[kClose / 32];
#pragma unroll
    for (int i = 0; i < kClose / 32; ++i) mine[i] = i * 32 + lane < s_n_close ? s_close[i * 32 + lane] : 0u;
    for (; bit >= 0 && reach != want; --bit) {
      const uint32_t test = bound | (1u << bit);
      int n = 0;
#pragma unroll
      for (int i = 0; i < kClose / 32; ++i) n += mine[i] >= test;
      const int total = reach_above + __reduce_add_sync(0xffffffffu, n);
      if (total >= want) {
        bound = test;
        reach = total;
      }
    }
  }
  // ---- the list: what is above the bound, and the first equals of it ----
  auto split = [&](int k, int p, unsigned& sure, unsigned& equal) {
    sure = equal = 0;
    if (p >= page1) return;
    if (!KEPT) page_keys(p, key[0], candidates[0]);
    const int there = min(L - p * kPageSize, kPageSize);
    unsigned over = 0, same = 0;
#pragma unroll
    for (int i = 0; i < kPageSize; ++i) {
      over |= (unsigned)(key[k][i] > bound) << i;
      same |= (unsigned)(key[k][i] == bound) << i;
    }
    sure = ~candidates[k] & (0xffffu >> (kPageSize - there));
    if (want > 0) {
      sure |= over;
      equal = same & candidates[k];
    }
  };
  unsigned stays[kHeld], maybe[kHeld];
  int n_sure = 0, n_equal = 0;
  if (KEPT) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      split(k, page0 + k, stays[k], maybe[k]);
      n_sure += __popc(stays[k]);
      n_equal += __popc(maybe[k]);
    }
  } else {
    for (int p = page0; p < page1; ++p) {
      unsigned a, b;
      split(0, p, a, b);
      n_sure += __popc(a);
      n_equal += __popc(b);
    }
  }
  // in front of this thread: inclusive sums over the warp, then warps, then CTAs
  int ia = n_sure, ib = n_equal;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int ya = __shfl_up_sync(0xffffffffu, ia, o), yb = __shfl_up_sync(0xffffffffu, ib, o);
    if (lane >= o) { ia += ya; ib += yb; }
  }
  __syncthreads();
  if (lane == 31) { s_warp[0][warp] = ia; s_warp[1][warp] = ib; }
  __syncthreads();
  int sure_before = ia - n_sure, equal_before = ib - n_equal;
  sure_before += __reduce_add_sync(0xffffffffu, lane < warp ? s_warp[0][lane] : 0);
  equal_before += __reduce_add_sync(0xffffffffu, lane < warp ? s_warp[1][lane] : 0);
  int sure_all = __reduce_add_sync(0xffffffffu, lane < n_warps ? s_warp[0][lane] : 0);
  if (ctas > 1) {
    const int equal_all = __reduce_add_sync(0xffffffffu, lane < n_warps ? s_warp[1][lane] : 0);
    use ^= 1;
    if (tid < 2 * ctas) {
      uint32_t at;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(&s_cta[use][tid & 1][rank])), "r"(tid >> 1));
      asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"((tid & 1) ? equal_all : sure_all) : "memory");
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
    sure_all = 0;
    for (int c = 0; c < ctas; ++c) {
      if (c < rank) {
        sure_before += s_cta[use][0][c];
        equal_before += s_cta[use][1][c];
      }
      sure_all += s_cta[use][0][c];
    }
  }
  const int equals = n_keep - sure_all;                // how many equals stay: the first ones
  int at = sure_before + min(equal_before, equals), eq = equal_before;
  auto list = [&](int p, unsigned sure, unsigned equal) {
    const int n = __popc(equal), room = max(0, equals - eq);
    eq += n;
    for (int drop = n - room; drop > 0; --drop) equal &= ~(0x80000000u >> __clz(equal));      // behind the last one that stays
    for (unsigned m = sure | equal; m; m &= m - 1) out[at++] = p * kPageSize + __ffs(m) - 1;
  };
  if (KEPT) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) list(page0 + k, stays[k], maybe[k]);
  } else {
    for (int p = page0; p < page1; ++p) {
      unsigned a, b;
      split(0, p, a, b);
      list(p, a, b);
    }
  }
  // (no CTA leaves while another one of the cluster may still write to it: every such write lies in front of a barrier that all passed)
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
      constexpr int kK = 16 * kC / 32, kP = D / 16, kV = 8 * kP / 32;       // K chunks a lane; 16-byte pieces of a token pair's V, and of them a lane
      uint4 kr[kK];
      uint4 vr[kV];
      uint32_t pair = 0;
      if (moves) {
#pragma unroll
        for (int u = 0; u < kK; ++u) {
          const int i = u * 32 + lane, tok = i / kC, c = i % kC;
          const int s = __shfl_sync(0xffffffffu, src, tok), sp = __shfl_sync(0xffffffffu, src_page, tok);
          if (s >= 0) kr[u] = *reinterpret_cast<const uint4*>(block_of(sp) + kv4_k_word(s & 15, 4 * c, D));
        }
#pragma unroll
        for (int u = 0; u < kV; ++u) {     // piece x of token pair q: halves of the words of the same piece of two source tokens
          const int i = u * 32 + lane, q = i / kP, x = i % kP;
          uint4 from[2];
          int odd[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int s = __shfl_sync(0xffffffffu, src, 2 * q + e), sp = __shfl_sync(0xffffffffu, src_page, 2 * q + e);
            odd[e] = s & 1;
            from[e] = s >= 0 ? *reinterpret_cast<const uint4*>(block_of(sp) + kv4_v_codes(D) + ((s & 15) >> 1) * D + 16 * x) : make_uint4(0, 0, 0, 0);
          }
          // low half from token 2 q, high half from token 2 q + 1
          const uint32_t pick = (odd[0] ? 0x32u : 0x10u) | (odd[1] ? 0x7600u : 0x5400u);
          vr[u] = make_uint4(__byte_perm(from[0].x, from[1].x, pick), __byte_perm(from[0].y, from[1].y, pick),
                             __byte_perm(from[0].z, from[1].z, pick), __byte_perm(from[0].w, from[1].w, pick));
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
          const int i = u * 32 + lane, q = i / kP, x = i % kP;
          uint8_t* at = dst + kv4_v_codes(D) + q * D + 16 * x;
          const unsigned have = (valid >> (2 * q)) & 3u;
          if (have == 3u) {
            *reinterpret_cast<uint4*>(at) = vr[u];
          } else if (have) {               // (the other token of the pair is not to be touched)
            const uint32_t w[4] = {vr[u].x, vr[u].y, vr[u].z, vr[u].w};
#pragma unroll
            for (int y = 0; y < 4; ++y) *reinterpret_cast<uint16_t*>(at + 4 * y + (have == 2u ? 2 : 0)) = (uint16_t)(have == 2u ? w[y] >> 16 : w[y]);
          }
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

void launch_kv_select(EvictDesc E, const float* weights, int64_t n_pages, int n_kv, int n_layers, int max_pages, int* keep, int keep_stride,
                      cudaStream_t st) {
  // as many CTAs as keep two pages a thread at most
  int ctas = 1;
  while (ctas < kMaxCluster && max_pages > ctas * 2 * kSelThreads) ctas *= 2;
  E.splits = ctas;
  const int per = (max_pages + ctas * kSelThreads - 1) / (ctas * kSelThreads);
  // Two pages a thread and half as many threads, so that two CTAs fit on an SM (one page a thread: 16 requests of 8192 tokens, 8 heads, 8 layers
  // 56.8 us instead of 46.0, 4 of 16384 38.3 instead of 31.1; one request of 16384, one layer 21.0 instead of 20.0), unless the pages are few.
  const int held = max_pages > 256 * ctas ? 2 : 1;
  auto* kernel = per <= 2 ? (held == 2 ? kv_select_kernel<2> : kv_select_kernel<1>) : kv_select_kernel<0>;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(n_kv * ctas, E.n_req, n_layers);
  const int need = (max_pages + ctas * held - 1) / (ctas * held);
  cfg.blockDim = dim3(need >= kSelThreads ? kSelThreads : (need < 128 ? 128 : (need + 31) / 32 * 32));
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  cudaLaunchKernelEx(&cfg, kernel, E, weights, n_pages, n_kv, keep, keep_stride);
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

// Hybrid-mask paged attention over a pool in 4 bits, few query rows per kv head (mma.sync).
//
// Work items, masks and the combine kernel are those of attention.cu.  With x_j = m_j + s_j c_j for a row of K or V (kv4.cuh):
//   score = s_K (q . (c_K - 8)) + (m_K + 8 s_K) sum(q)
//   o     = sum_j (p_j s_Vj) (c_Vj - 8) + sum_j p_j (m_Vj + 8 s_Vj)
// so the matrix instructions multiply codes, which bf16 holds exactly, and steps and minima enter in fp32: the scores are exact
// up to fp32 sums, and the only rounding ahead of the result is that of p s_V to bf16 (2^-9 of each term, like p in the bf16
// kernels).
//
// One producer warp streams the item's blocks of 64 tokens, one bulk copy per page and head, into a ring; eight consumer warps
// take 16 query rows each and share the blocks among themselves where there are fewer row tiles than warps.  The codes are
// laid out such that a lane reads its part of a B operand with one 16-byte access and nothing goes through registers of other
// lanes; the values of a row then stand at positions of the contraction that are permuted, and Q is loaded in the same order.
#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

constexpr int kBlockTokens = 64;
constexpr int kPagesPerBlock = kBlockTokens / kPageSize;
constexpr int kConsumers = 8;
constexpr int kThreads = (kConsumers + 1) * 32;
constexpr uint32_t kSpin = 1u << 22;
constexpr float kNoRef = -1e30f;       // reference maximum of a row that has seen no token yet
constexpr float kHeadroom = 8.f;       // a row's reference maximum moves when it is outgrown by more than 2^8

template <int D>
struct Smem {
  static constexpr int kBlock = kv4_block_bytes(D);
  static constexpr int kStage = kPagesPerBlock * kBlock;
  static constexpr int kMergeFloats = (D / 2 + 4) * 32;                     // per warp: o, reference maxima, sums
  static constexpr int kMerge = kConsumers * kMergeFloats * 4;
  static constexpr int kStages = 16;
  static constexpr int kBars = kStages * kStage + kMerge;
  static constexpr int kTotal = kBars + 2 * kStages * 8;
};

struct Params {
  const AttnItem* items;
  const int* cta_off;
  const int* page_table;
  int pt_stride;
  const int* tok_climit;
  const int* tok_lo;
  const int* tok_hi;
  const __nv_bfloat16* q;
  __nv_bfloat16* o;
  float* lse;         // may be null
  const uint8_t* pool;
  int64_t n_pages;
  int layer, n_q, n_kv, group;
  float scale_log2;   // log2(e) / sqrt(d)
  float* part_o;      // [part][128][D]
  float* part_ml;     // [part][128][2]
  int* status;
};

__device__ __forceinline__ void consumer_bar() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&w)[N], const uint8_t* p) {
  if constexpr (N == 4) {
    const uint4 t = *reinterpret_cast<const uint4*>(p);
    w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
  } else {
    const uint2 t = *reinterpret_cast<const uint2*>(p);
    w[0] = t.x; w[1] = t.y;
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) attention_kv4_kernel(Params P) {
  using SM = Smem<D>;
  constexpr int kStages = SM::kStages;
  constexpr int NW = D / 32;             // words of codes a lane holds of a token (K) or token pair (V)
  extern __shared__ __align__(128) uint8_t smem[];
  uint64_t* full_bar = reinterpret_cast<uint64_t*>(smem + SM::kBars);
  uint64_t* empty_bar = full_bar + kStages;
  float* merge = reinterpret_cast<float*>(smem + kStages * SM::kStage);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], kConsumers);
    }
    fence_barrier_init();
  }
  __syncthreads();
  griddep_wait();
  griddep_launch();

  // the CTA walks two ranges of the item list one after the other (see the layout kernel)
  const int4 r4 = *reinterpret_cast<const int4*>(P.cta_off + 4 * blockIdx.x);
  const int range_n0 = r4.y - r4.x;
  const int item_end = range_n0 + (r4.w - r4.z);
  auto item_at = [&](int i) { return i < range_n0 ? r4.x + i : r4.z + (i - range_n0); };
  uint32_t it = 0;  // running block counter, identical in producer and consumers
  bool aborted = false;

  if (warp == kConsumers) {
    // ------------------------------ producer ------------------------------
    for (int item = 0; item < item_end && !aborted; ++item) {
      const AttnItem w = P.items[item_at(item)];
      const int n_req_pages = (w.kv_len + kPageSize - 1) / kPageSize;
      const int* pt = P.page_table + (size_t)w.req * P.pt_stride;
      // lanes 0..3 each own one page of the block; ids are fetched one block ahead of their use
      auto fetch_page = [&](int n) -> int {
        const int lp = n * kPagesPerBlock + lane;
        return lane < kPagesPerBlock && n < w.blk_end && lp < n_req_pages ? __ldg(pt + lp) : -1;
      };
      int pg_next = fetch_page(w.blk_begin);
      for (int n = w.blk_begin; n < w.blk_end; ++n, ++it) {
        const int s = it % kStages;
        int my_pg = pg_next;
        pg_next = fetch_page(n + 1);
        if (my_pg >= P.n_pages) {
          set_status(P.status, DEV_BAD_INDEX);
          my_pg = -1;
        }
        if (!mbar_wait(&empty_bar[s], ((it / kStages) & 1) ^ 1, kSpin)) {
          set_status(P.status, DEV_TIMEOUT_EMPTY);
          aborted = true;
          break;
        }
        const unsigned valid = __ballot_sync(0xffffffffu, my_pg >= 0);
        if (lane == 0) {
          if (valid == 0) mbar_arrive(&full_bar[s]);
          else mbar_arrive_expect_tx(&full_bar[s], __popc(valid) * SM::kBlock);
        }
        __syncwarp();
        if (my_pg >= 0)
          bulk_g2s(smem + s * SM::kStage + lane * SM::kBlock, P.pool + kv4_block_base(P.n_pages, P.n_kv, D, P.layer, my_pg, w.kv_head),
                   SM::kBlock, &full_bar[s]);
        __syncwarp();
      }
    }
    if (aborted && lane == 0)         // let copies already in flight land before the CTA may exit
      for (int s = 0; s < kStages; ++s)
        for (uint32_t i = 0; i < (1u << 14); ++i) {
          if (mbar_try_wait(&full_bar[s], 0) || mbar_try_wait(&full_bar[s], 1)) break;
          __nanosleep(64);
        }
    return;
  }

  // ------------------------------ consumers ------------------------------
  const int g = lane >> 2, t = lane & 3;

  for (int item = 0; item < item_end; ++item) {
    const AttnItem w = P.items[item_at(item)];
    const int R = w.ntok * P.group;
    const int RW = (R + 15) >> 4, KW = kConsumers / RW;
    const int rw = warp % RW, kw = warp / RW;
    const bool active = kw < KW;

    // Q fragments and visibility of this lane's two rows (g and g + 8 of the warp's 16).  Lane t holds the values
    // [32 t, 32 t + 32) (d = 128) of a row, its word j of codes the values 8 j .. of these: k-step 2 j + u of the products
    // takes the pairs 2 u and 2 u + 1 of word j.
    uint32_t qf[D / 16][4];
    float qsum[2];
    int climit[2], vlo[2], vhi[2], row_tok[2], row_head[2];
    bool rvalid[2];
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int rho = rw * 16 + g + hh * 8;
      rvalid[hh] = active && rho < R;
      const int j = rho / P.group, hg = rho - j * P.group;
      const int tok = w.tok0 + (rvalid[hh] ? j : 0);
      row_tok[hh] = tok;
      row_head[hh] = w.kv_head * P.group + hg;
      climit[hh] = rvalid[hh] ? P.tok_climit[tok] : -1;
      vlo[hh] = rvalid[hh] ? P.tok_lo[tok] : 0;
      vhi[hh] = rvalid[hh] ? P.tok_hi[tok] : 0;
      const uint4* src = reinterpret_cast<const uint4*>(P.q + ((size_t)tok * P.n_q + row_head[hh]) * D) + t * NW;
      float sum = 0.f;
#pragma unroll
      for (int j2 = 0; j2 < NW; ++j2) {
        const uint4 v = rvalid[hh] ? __ldg(src + j2) : make_uint4(0, 0, 0, 0);
        qf[2 * j2][hh] = v.x;
        qf[2 * j2][hh + 2] = v.y;
        qf[2 * j2 + 1][hh] = v.z;
        qf[2 * j2 + 1][hh + 2] = v.w;
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += __uint_as_float(u[i] << 16) + __uint_as_float(u[i] & 0xffff0000u);
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      qsum[hh] = sum + __shfl_xor_sync(0xffffffffu, sum, 2);
    }

    float o[D / 8][4];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float ref[2] = {kNoRef, kNoRef};     // reference maximum (powers of two), the same in the four lanes of a row
    float l[2] = {0.f, 0.f};             // this lane's part of the row's sum of probabilities
    float om[2] = {0.f, 0.f};            // ... and of the part of o that all its values share: sum p (m + 8 s)

    for (int n = w.blk_begin; n < w.blk_end; ++n, ++it) {
      const int s = it % kStages;
      if (!aborted && !mbar_wait(&full_bar[s], (it / kStages) & 1, kSpin)) {
        set_status(P.status, DEV_TIMEOUT_FULL);
        aborted = true;
      }
      if (!aborted && active && ((n - w.blk_begin) % KW) == kw) {
        const int n_pg = min(kPagesPerBlock, (w.kv_len - n * kBlockTokens + kPageSize - 1) / kPageSize);
#pragma unroll 1
        for (int p = 0; p < n_pg; ++p) {
          const uint8_t* pg = smem + s * SM::kStage + p * SM::kBlock;
          const int pos0 = n * kBlockTokens + p * kPageSize;
          // ---- S = Q C_K^T over the page's 16 tokens: n-tile h holds tokens 8 h .. 8 h + 7 ----
          float sc[2][4];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t word[NW];
            load_words(word, pg + (g + 8 * h) * (D / 2) + t * (NW * 4));
            sc[h][0] = sc[h][1] = sc[h][2] = sc[h][3] = 0.f;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              mma_bf16_16816(sc[h], qf[k], kv4_pair(word[k >> 1], 2 * (k & 1)), kv4_pair(word[k >> 1], 2 * (k & 1) + 1));
          }
          // ---- scores in powers of two; columns 8 h + 2 t + c, rows e >> 1 ----
          float sk[2][2], mk[2][2], sv[2][2], mv[2][2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint2 kp = *reinterpret_cast<const uint2*>(pg + kv4_k_pairs(D) + 4 * (8 * h + 2 * t));
            const uint2 vp = *reinterpret_cast<const uint2*>(pg + kv4_v_pairs(D) + 4 * (8 * h + 2 * t));
            const uint32_t kk[2] = {kp.x, kp.y}, vv[2] = {vp.x, vp.y};
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              sk[h][c] = kv4_step(kk[c]) * P.scale_log2;
              mk[h][c] = fmaf(8.f, kv4_step(kk[c]), kv4_min(kk[c])) * P.scale_log2;
              sv[h][c] = kv4_step(vv[c]);
              mv[h][c] = fmaf(8.f, sv[h][c], kv4_min(vv[c]));
            }
          }
          // (rows that do not exist carry a limit of -1 and are masked everywhere)
          const bool need_mask = __any_sync(0xffffffffu, pos0 + kPageSize - 1 > min(climit[0], climit[1]));
          unsigned see = 0xff;
          if (need_mask) {
            see = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int pos = pos0 + 8 * h + 2 * t + (e & 1), hh = e >> 1;
                if (pos <= climit[hh] || (pos >= vlo[hh] && pos < vhi[hh])) see |= 1u << (4 * h + e);
              }
          }
          float pr[2][4];
          auto scores = [&]() {
            float top = -INFINITY;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float y = fmaf(sc[h][e], sk[h][e & 1], fmaf(mk[h][e & 1], qsum[e >> 1], -ref[e >> 1]));
                if (need_mask && !((see >> (4 * h + e)) & 1u)) y = -INFINITY;
                pr[h][e] = y;
                top = fmaxf(top, y);
              }
            return top;
          };
          if (__any_sync(0xffffffffu, scores() > kHeadroom)) {
            // some row's reference maximum moves, and what has been summed up is scaled to it
#pragma unroll
            for (int hh = 0; hh < 2; ++hh) {
              float z = -INFINITY;
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                  if ((see >> (4 * h + 2 * hh + c)) & 1u) z = fmaxf(z, fmaf(sc[h][2 * hh + c], sk[h][c], mk[h][c] * qsum[hh]));
              z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, 1));
              z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, 2));
              const float next = fmaxf(ref[hh], z), f = exp2f(ref[hh] - next);
              ref[hh] = next;
              l[hh] *= f;
              om[hh] *= f;
#pragma unroll
              for (int i = 0; i < D / 8; ++i) {
                o[i][2 * hh] *= f;
                o[i][2 * hh + 1] *= f;
              }
            }
            scores();
          }
          // ---- probabilities; O += (P s_V) C_V ----
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p_ = exp2f(pr[h][e]);
              l[e >> 1] += p_;
              float ps = p_ * sv[h][e & 1], pm = p_ * mv[h][e & 1];
              if (need_mask && !((see >> (4 * h + e)) & 1u)) ps = pm = 0.f;      // (the step of a token that nobody wrote may be NaN)
              om[e >> 1] += pm;
              pr[h][e] = ps;
            }
          const uint32_t a[4] = {pack_bf16(pr[0][0], pr[0][1]), pack_bf16(pr[0][2], pr[0][3]), pack_bf16(pr[1][0], pr[1][1]),
                                 pack_bf16(pr[1][2], pr[1][3])};
          uint32_t v0[NW], v1[NW];
          load_words(v0, pg + kv4_v_codes(D) + t * D + g * (D / 8));
          load_words(v1, pg + kv4_v_codes(D) + (t + 4) * D + g * (D / 8));
#pragma unroll
          for (int nt = 0; nt < D / 8; ++nt) mma_bf16_16816(o[nt], a, kv4_pair(v0[nt >> 2], nt & 3), kv4_pair(v1[nt >> 2], nt & 3));
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty_bar[s]);
    }

#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      l[hh] += __shfl_xor_sync(0xffffffffu, l[hh], 1);
      l[hh] += __shfl_xor_sync(0xffffffffu, l[hh], 2);
      om[hh] += __shfl_xor_sync(0xffffffffu, om[hh], 1);
      om[hh] += __shfl_xor_sync(0xffffffffu, om[hh], 2);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        o[i][2 * hh] += om[hh];
        o[i][2 * hh + 1] += om[hh];
      }
    }

    // ---- merge the warps that share a row tile ----
    if (KW > 1) {
      float* mine = merge + warp * SM::kMergeFloats;
      if (active && kw > 0) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) mine[(i * 4 + e) * 32 + lane] = o[i][e];
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          mine[(D / 2 + hh) * 32 + lane] = ref[hh];
          mine[(D / 2 + 2 + hh) * 32 + lane] = l[hh];
        }
      }
      consumer_bar();
      if (active && kw == 0)
        for (int k2 = 1; k2 < KW; ++k2) {
          const float* oth = merge + (k2 * RW + rw) * SM::kMergeFloats;
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            const float ro = oth[(D / 2 + hh) * 32 + lane], lo = oth[(D / 2 + 2 + hh) * 32 + lane];
            const float next = fmaxf(ref[hh], ro), fa = exp2f(ref[hh] - next), fb = exp2f(ro - next);
            ref[hh] = next;
            l[hh] = l[hh] * fa + lo * fb;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
              o[i][2 * hh] = o[i][2 * hh] * fa + oth[(i * 4 + 2 * hh) * 32 + lane] * fb;
              o[i][2 * hh + 1] = o[i][2 * hh + 1] * fa + oth[(i * 4 + 2 * hh + 1) * 32 + lane] * fb;
            }
          }
        }
      consumer_bar();  // scratch may be rewritten by the next item only after everyone has read it
    }

    // ---- write out: n-tile 4 w + i holds the values 8 (w / 2) + 2 i + (w & 1) of the D / 8 that column 2 t (+ 1) stands for ----
    if (active && kw == 0 && !aborted) {
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        if (!rvalid[hh]) continue;
        const int rho = rw * 16 + g + hh * 8;
        if (w.part < 0) {
          const float inv = l[hh] > 0.f ? 1.f / l[hh] : 0.f;
          __nv_bfloat16* dst = P.o + ((size_t)row_tok[hh] * P.n_q + row_head[hh]) * D + t * (D / 4);
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int x = 0; x < NW / 2; ++x) {
              uint32_t out[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) out[i] = pack_bf16(o[8 * x + i][2 * hh + c] * inv, o[8 * x + 4 + i][2 * hh + c] * inv);
              *reinterpret_cast<uint4*>(dst + c * (D / 8) + 8 * x) = make_uint4(out[0], out[1], out[2], out[3]);
            }
          if (P.lse && t == 0) P.lse[(size_t)row_tok[hh] * P.n_q + row_head[hh]] = log_sum_exp(ref[hh], l[hh]);
        } else {
          float* dst = P.part_o + ((size_t)w.part * 128 + rho) * D + t * (D / 4);
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int x = 0; x < NW / 2; ++x)
#pragma unroll
              for (int i = 0; i < 4; i += 2)
                *reinterpret_cast<float4*>(dst + c * (D / 8) + 8 * x + 2 * i) =
                    make_float4(o[8 * x + i][2 * hh + c], o[8 * x + 4 + i][2 * hh + c], o[8 * x + i + 1][2 * hh + c], o[8 * x + 5 + i][2 * hh + c]);
          if (t == 0) *reinterpret_cast<float2*>(P.part_ml + ((size_t)w.part * 128 + rho) * 2) = make_float2(ref[hh], l[hh]);
        }
      }
    }
  }
}

}  // namespace

void launch_attention_kv4(const BatchLayout& bl, const Dims& dm, int layer, const void* q, void* o, float* lse, const void* kv_pool,
                          int64_t n_pages, float* part_o, float* part_ml, int n_sm, int* status, cudaStream_t st) {
  static bool configured[kMaxDevices] = {false};
  if (first_use_on_device(configured)) {
    cudaFuncSetAttribute(attention_kv4_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<64>::kTotal);
    cudaFuncSetAttribute(attention_kv4_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, Smem<128>::kTotal);
  }
  Params P;
  P.items = bl.items;
  P.cta_off = bl.cta_off;
  P.page_table = bl.page_table;
  P.pt_stride = bl.pt_stride;
  P.tok_climit = bl.tok_climit;
  P.tok_lo = bl.tok_lo;
  P.tok_hi = bl.tok_hi;
  P.q = static_cast<const __nv_bfloat16*>(q);
  P.o = static_cast<__nv_bfloat16*>(o);
  P.lse = lse;
  P.pool = static_cast<const uint8_t*>(kv_pool);
  P.n_pages = n_pages;
  P.layer = layer;
  P.n_q = dm.n_q;
  P.n_kv = dm.n_kv;
  P.group = dm.n_q / dm.n_kv;
  P.scale_log2 = 1.4426950408889634f / sqrtf((float)dm.head_dim);
  P.part_o = part_o;
  P.part_ml = part_ml;
  P.status = status;
  if (dm.head_dim == 64) launch_pdl(attention_kv4_kernel<64>, dim3(n_sm), dim3(kThreads), Smem<64>::kTotal, st, P);
  else launch_pdl(attention_kv4_kernel<128>, dim3(n_sm), dim3(kThreads), Smem<128>::kTotal, st, P);
}

}  // namespace recg

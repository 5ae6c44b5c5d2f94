// Hybrid-mask paged attention over a pool in 4 bits, few query rows per kv head (mma.sync).
//
// Work items, masks and the combine kernel are those of attention.cu.  With x_j = m_j + s_j c_j for a row of K or V (kv4.cuh)
//   score = s_K (q . c_K) + m_K sum(q),      o = sum_j (p_j s_Vj) c_Vj + sum_j p_j m_Vj
// the matrix instructions multiply codes, which are exact, and steps and minima enter in fp32.  Both products are taken transposed,
// S^T = K Q^T and O^T = V^T P^T, since there are fewer rows (the 8 columns of a product) than tokens or values (its 16 rows): one
// token of four or five query heads fills half a product, not a quarter, and every lane needs the step and minimum of two tokens
// only, not of four.  P^T turns from accumulators to operand by one movmatrix per eight tokens.
//
// Single rows are bound by the bytes of the cache, if only the instructions that unpack the codes are few.  The operands are fp16,
// and a code masked out of its word in the lowest 8 bits of a half IS an fp16 number, a subnormal one: c 2^-24 or 16 c 2^-24.  So
// eight codes cost one shift and four ANDs, where bf16 takes three shifts, four masks with an exponent and four subtractions
// (694 instructions for a page of 16 tokens: 99.5 us for one token over 131072 of context, 32 / 8 heads; now 35.0).  What belongs to
// the 16 is divided out of Q and of the result.  Rows of Q are scaled by a power of two, one for all rows of a warp unless they lie
// far apart, and the steps of V, as factors of a row of P, by another that follows the largest step that the row sees.  So a value of
// q is off by 2^-21 of the row's largest at most, and p s_V by 2^-11 of itself or, where that is more, by 2^-31 of the largest step.
// (Rows with scales of their own, masks and large scores are a second form of the loop's body.  With one scale for whatever the
// warp has at hand, a row was wrong by half where another one's V was 2^30 as large; it took 34.3 instead of 35.0 us.)
//
// A warp is alone with its pages: it requests them itself, 16 bytes a lane into a ring of its own, and runs ahead of itself into the
// next item.  (One bulk copy per page and head and a barrier per slot: the one lane that issues them took 850 clocks for every 2100
// of work.)  The warps are divided among the item's row groups, those of a group share its pages among
// themselves, and their results are merged at the end of the item.
#include <cuda_fp16.h>
#include <type_traits>

#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

constexpr float kNoRef = -1e30f;       // reference maximum of a row that has seen no token yet
constexpr float kHeadroom = 8.f;       // a row's reference maximum moves when it is outgrown by more than 2^8
constexpr float kLift = 7.f;           // probabilities stand as 2^7 p: with steps below 1 at most 2^15
constexpr float kLarge = 512.f;        // scores (in powers of two) from which on the reference is subtracted exactly (see below)
constexpr int kNear = 8;               // rows of Q whose largest values are within 2^8 of each other stand on one scale

// NT: groups of eight query rows a warp has.  Two pages at a time are two independent chains of instructions (one token of one request,
// 131072 of context: 41.9 us with one page, 40.3 with two, before the merge of parts got shorter), for which sixteen rows leave no registers.
template <int D, int NT>
struct Shape {
  static constexpr int kWarps = 12;
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kPages = NT == 1 ? 2 : 1;                   // pages of a chunk, which a warp works on at once
  static constexpr int kSlots = NT == 1 ? 3 : 4;                   // chunks that a warp has on their way
  static constexpr int kBlock = kv4_block_bytes(D);
  static constexpr int kRing = kWarps * kSlots * kPages * kBlock;
  static constexpr int kRowPad = D + 4;                            // floats from row to row of a merged part
  static constexpr int kRows = 8 * NT;
  static constexpr int kMerge = kWarps * kRows * kRowPad * 4;      // [warp][row][value]; values D to D + 2: reference maximum, sum, scale of Q
  static constexpr int kItemsOff = kRing + kMerge;
  static constexpr int kItems = 32;                                // items of the CTA whose descriptors are kept on chip
  static constexpr int kTotal = kItemsOff + kItems * (int)sizeof(AttnItem);
  static_assert(kBlock % 16 == 0 && kTotal <= 227 * 1024, "shared memory budget");
  static_assert(kWarps * kRows >= 128 || NT == 1, "every row of a tile has a warp");
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
  int layer, n_q, n_kv, group, inv_group;      // inv_group: (rho * inv_group) >> 16 is rho / group for the rows of a tile
  float scale_log2;   // log2(e) / sqrt(d)
  float* part_o;      // [part][128][D]
  float* part_ml;     // [part][128][2]
  int* status;
  int early_desc;     // the work list is settled: it may be read before the wait for the kernel in front of this one
};

// D(16x8, f32) += A(16x16, f16, row) * B(16x8, f16, col)
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return reinterpret_cast<const uint32_t&>(h);
}
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
__device__ __forceinline__ float inverse(float power) { return __int_as_float(0x7f000000 - __float_as_int(power)); }       // of 2^e

template <int D, int NT>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1) attention_kv4_kernel(Params P) {
  using SH = Shape<D, NT>;
  constexpr int NW = D / 32;             // words of codes a lane holds of a token (K) or token pair (V)
  constexpr int W = SH::kWarps, PG = SH::kPages, kSlots = SH::kSlots, kSlot = PG * SH::kBlock;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * kSlots * kSlot;
  float* merge = reinterpret_cast<float*>(smem + SH::kRing);
  // scale of a row of Q of this warp, relative to the scale of all (in shared memory: as a register more in the loop 35.5 us
  // instead of 35.0 for one token over 131072 of context)
  auto below = [&](int nt, int column) -> float& { return merge[(warp * SH::kRows + nt * 8 + column) * SH::kRowPad + D + 2]; };
  // (where the work list is settled all reads of it, and of page ids, overlap the end of the kernel in front)
  if (!P.early_desc) griddep_wait();

  // the CTA walks two ranges of the item list one after the other (see the layout kernel)
  const int4 r4 = *reinterpret_cast<const int4*>(P.cta_off + 4 * blockIdx.x);
  const int range_n0 = r4.y - r4.x, item_end = range_n0 + (r4.w - r4.z);
  auto item_at = [&](int i) { return i < range_n0 ? r4.x + i : r4.z + (i - range_n0); };
  static_assert(sizeof(AttnItem) == 32, "two 16-byte pieces");
  uint4* kept = reinterpret_cast<uint4*>(smem + SH::kItemsOff);
  for (int i = threadIdx.x; i < 2 * min(item_end, SH::kItems); i += SH::kThreads)
    kept[i] = reinterpret_cast<const uint4*>(P.items + item_at(i >> 1))[i & 1];
  __syncthreads();
  auto item_of = [&](int i) { return i < SH::kItems ? reinterpret_cast<const AttnItem*>(kept)[i] : P.items[item_at(i)]; };
  // of an item: warps per row group; this warp's group; its first chunk of pages and the end of all
  struct Share { int warps, group, page, end; };
  auto share_of = [&](const AttnItem& w) {
    Share s;
    if (NT == 1) {                       // (one group)
      s.warps = W;
      s.group = 0;
    } else {
      s.warps = W / ((w.ntok * P.group + SH::kRows - 1) / SH::kRows);
      s.group = warp / s.warps;
    }
    s.end = s.group * SH::kRows < w.ntok * P.group ? min(w.blk_end * 4, (w.kv_len + kPageSize - 1) / kPageSize) : 0;
    s.page = w.blk_begin * 4 + (warp - s.group * s.warps) * PG;
    return s;
  };

  // ---- what the warp requests next: a chunk of an item.  Page ids are fetched 32 at a time, a lane one of them; a page's address is one
  // multiplication away from its id (with the general formula for a block's place a request took 100 instructions a page, as many as the
  // work on it leaves to the other warps of the scheduler) ----
  int f_item = -1, f_page = 0, f_step = 0, f_end = 0, f_used = 0, f_ids = 0;
  const int* f_table = nullptr;
  const uint8_t* f_base = nullptr;       // this lane's 16 bytes of the head's block in page 0 of the layer
  const unsigned page_bytes = (unsigned)P.n_kv * SH::kBlock, n_pages = (unsigned)min(P.n_pages, (int64_t)0x7fffffff);
  const uint32_t ring_at = smem_u32(ring) + lane * 16;
  auto load_ids = [&]() {
    f_used = 0;
    const int page = f_page + (lane / PG) * f_step + lane % PG;
    f_ids = page < f_end ? __ldg(f_table + page) : 0;
  };
  auto next_item = [&]() {
    do {
      if (++f_item >= item_end) {
        f_end = -1;
        return;
      }
      const AttnItem w = item_of(f_item);
      const Share s = share_of(w);
      f_page = s.page;
      f_step = s.warps * PG;
      f_end = s.end;
      f_table = P.page_table + (size_t)w.req * P.pt_stride;
      f_base = P.pool + kv4_block_base(P.n_pages, P.n_kv, D, P.layer, 0, w.kv_head) + lane * 16;
    } while (f_page >= f_end);
    load_ids();
  };
  auto request = [&](uint32_t slot_at) {        // one group of copies per call, be it empty
    if (f_end >= 0) {
#pragma unroll
      for (int i = 0; i < PG; ++i) {
        const unsigned id = __shfl_sync(0xffffffffu, f_ids, f_used + i);
        if (PG > 1 && i > 0 && f_page + i >= f_end) continue;
        if (id >= n_pages) {
          set_status(P.status, DEV_BAD_INDEX);
          continue;
        }
        const uint8_t* src = f_base + (uint64_t)id * page_bytes;
        const uint32_t dst = ring_at + slot_at + i * SH::kBlock;
#pragma unroll
        for (int x = 0; x < SH::kBlock / 512; ++x) copy_async16(dst + x * 512, src + x * 512);
        if (lane < SH::kBlock % 512 / 16) copy_async16(dst + SH::kBlock / 512 * 512, src + SH::kBlock / 512 * 512);
      }
      f_page += f_step;
      f_used += PG;
      if (f_page >= f_end) next_item();
      else if (f_used >= 32) load_ids();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  next_item();
  if (P.early_desc) griddep_wait();
  griddep_launch();

  // The rows of a warp's group in an item, read ahead of their use: column g of row group nt, of which lane t holds the values
  // [D / 4 t, D / 4 (t + 1)); and what the rows 2 t and 2 t + 1 see
  uint4 raw[NT][NW];
  int climit[NT][2], vlo[NT][2], vhi[NT][2];
  auto load_rows = [&](const AttnItem& w) {
    const int R = w.ntok * P.group, row0 = share_of(w).group * SH::kRows;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int rho = row0 + nt * 8 + g, j = (rho * P.inv_group) >> 16;
      const bool there = rho < R;
      const uint4* src = reinterpret_cast<const uint4*>(P.q + ((size_t)(w.tok0 + (there ? j : 0)) * P.n_q + w.kv_head * P.group + (there ? rho - j * P.group : 0)) * D) + t * NW;
#pragma unroll
      for (int k = 0; k < NW; ++k) raw[nt][k] = there ? __ldg(src + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rv = row0 + nt * 8 + 2 * t + e, tok = w.tok0 + ((rv * P.inv_group) >> 16);
        const bool is = rv < R;      // (a row that does not exist needs no mask: nobody reads it)
        climit[nt][e] = is ? P.tok_climit[tok] : 0x7fffffff;
        vlo[nt][e] = is ? P.tok_lo[tok] : 0;
        vhi[nt][e] = is ? P.tok_hi[tok] : 0;
      }
    }
  };
  if (item_end > 0) load_rows(item_of(0));
  for (int s = 0; s < kSlots; ++s) request(s * kSlot);

  uint32_t slot_at = 0;   // the slot of the next chunk
  for (int item = 0; item < item_end; ++item) {
    const AttnItem w = item_of(item);
    const int R = w.ntok * P.group;
    const Share sh = share_of(w);
    // ---- Q as B operands: k-step 2 j + u takes the pairs 2 u and 2 u + 1 of word j of codes, the second of which the K operand holds
    // times 16 ----
    uint32_t qf[NT][D / 16][2];
    float qs[NT][2];                     // sums of the rows 2 t and 2 t + 1, times the scale of the scores
    float factor;                        // what makes a product of scaled Q and codes 2^-24 c a score
    int lim = 0x7fffffff;                // the position up to which every row of the warp sees everything
    {
      uint32_t top[NT];                  // largest value of this quarter of row g
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        top[nt] = 0;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < NW; ++k) {
          const uint32_t u[4] = {raw[nt][k].x, raw[nt][k].y, raw[nt][k].z, raw[nt][k].w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            sum += __uint_as_float(u[i] << 16) + __uint_as_float(u[i] & 0xffff0000u);
            const uint32_t lo = u[i] & 0x7fffu, hi = (u[i] >> 16) & 0x7fffu;
            top[nt] = max(top[nt], max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));      // (a row that is not finite does not concern the others)
          }
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          qs[nt][c] = __shfl_sync(0xffffffffu, sum, (2 * t + c) * 4) * P.scale_log2;
          lim = min(lim, climit[nt][c]);
        }
      }
      lim = __reduce_min_sync(0xffffffffu, lim);
      // The largest value of all rows goes to [2^8, 2^9) (as far as the exponent allows: a factor and its inverse are normal numbers), or, where
      // the quarters of rows that the lanes hold lie far apart, each row's own.
      auto exponent = [](uint32_t largest) { return max(-100, min(100, (int)(largest >> 7) - 127 - 8)); };
      int e_most = -100, e_least = 100;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        e_most = max(e_most, exponent(top[nt]));
        if (top[nt]) e_least = min(e_least, exponent(top[nt]));
      }
      e_most = __reduce_max_sync(0xffffffffu, e_most);
      const bool far = __reduce_min_sync(0xffffffffu, e_least) + kNear < e_most;
      factor = pow2(e_most) * 16777216.f * P.scale_log2;
      if (far) lim = -1;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        int e = e_most;
        if (far) {
          uint32_t row = max(top[nt], __shfl_xor_sync(0xffffffffu, top[nt], 1));
          row = max(row, __shfl_xor_sync(0xffffffffu, row, 2));
          e = max(exponent(row), e_most - 126);
        }
        if (t == 0) below(nt, g) = pow2(e - e_most);
        const float down = pow2(-e), down16 = pow2(-e - 4);
#pragma unroll
        for (int k = 0; k < NW; ++k) {
          const uint4 v = raw[nt][k];
          qf[nt][2 * k][0] = pack_f16(__uint_as_float(v.x << 16) * down, __uint_as_float(v.x & 0xffff0000u) * down);
          qf[nt][2 * k][1] = pack_f16(__uint_as_float(v.y << 16) * down16, __uint_as_float(v.y & 0xffff0000u) * down16);
          qf[nt][2 * k + 1][0] = pack_f16(__uint_as_float(v.z << 16) * down, __uint_as_float(v.z & 0xffff0000u) * down);
          qf[nt][2 * k + 1][1] = pack_f16(__uint_as_float(v.w << 16) * down16, __uint_as_float(v.w & 0xffff0000u) * down16);
        }
      }
    }
    {
      float o[NT][D / 16][4];              // O^T: rows (values) i, columns 2 t and 2 t + 1; see the writer for which values
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
      // per row (columns 2 t, 2 t + 1; the same in all lanes of a column): reference maximum in powers of two, less kLift; this lane's
      // part of the sum of probabilities and of sum p m
      float ref[NT][2], l[NT][2], om[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        ref[nt][0] = ref[nt][1] = kNoRef;
        l[nt][0] = l[nt][1] = om[nt][0] = om[nt][1] = 0.f;
      }
      // Per row: the steps of V that it has seen are below s_top (a power of two), and P holds p s_V 2^7 / s_top.  They are the same for all
      // rows as long as all rows see everything; what a row does not see may be larger than what it does by more than fp16 holds.
      // s_least: the least of this lane's
      float s_top[NT][2], s_least = 0.f;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s_top[nt][0] = s_top[nt][1] = 0.f;

      for (int p = sh.page; p < sh.end; p += sh.warps * PG) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 1) : "memory");
        __syncwarp();
        const uint8_t* pg = ring + slot_at;
        const int pos0 = p * kPageSize;
        // Without MASK: every row sees everything, rows of Q stand on one scale and scores are not large (returns whether they turn out to be)
        auto work = [&](auto masked) {
          constexpr bool MASK = decltype(masked)::value;
          // ---- S^T = C_K Q^T: rows g and g + 8 of product i are tokens of page i ----
          float sc[PG][NT][4];
#pragma unroll
          for (int i = 0; i < PG; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sc[i][nt][0] = sc[i][nt][1] = sc[i][nt][2] = sc[i][nt][3] = 0.f;
          {
            uint32_t k0[PG][NW], k1[PG][NW];
#pragma unroll
            for (int i = 0; i < PG; ++i) {
              load_words(k0[i], pg + i * SH::kBlock + g * (D / 2) + t * (NW * 4));
              load_words(k1[i], pg + i * SH::kBlock + (g + 8) * (D / 2) + t * (NW * 4));
            }
#pragma unroll
            for (int j = 0; j < NW; ++j)
#pragma unroll
              for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < PG; ++i) {
                  const uint32_t w0 = u ? k0[i][j] >> 8 : k0[i][j], w1 = u ? k1[i][j] >> 8 : k1[i][j];
#pragma unroll
                  for (int nt = 0; nt < NT; ++nt)
                    mma_f16(sc[i][nt], w0 & 0x000f000fu, w1 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x00f000f0u, qf[nt][2 * j + u][0], qf[nt][2 * j + u][1]);
                }
          }
          if (MASK && lim < 0) {               // (rows on scales of their own, or large scores)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const float by = below(nt, 2 * t + c);
#pragma unroll
                for (int i = 0; i < PG; ++i) {
                  sc[i][nt][c] *= by;
                  sc[i][nt][2 + c] *= by;
                }
              }
          }
          // (token x = 2 i + h of this lane is token g + 8 h of page i)
          float sk[2 * PG], mk[2 * PG], sv[2 * PG], mv[2 * PG];
          float sv_top = 0.f;
#pragma unroll
          for (int x = 0; x < 2 * PG; ++x) {
            const uint8_t* pair = pg + (x >> 1) * SH::kBlock + 4 * (8 * (x & 1) + g);
            const uint32_t kp = *reinterpret_cast<const uint32_t*>(pair + kv4_k_pairs(D)), vp = *reinterpret_cast<const uint32_t*>(pair + kv4_v_pairs(D));
            sk[x] = kv4_step(kp) * factor;
            mk[x] = kv4_min(kp);
            sv[x] = kv4_step(vp);
            mv[x] = kv4_min(vp);
            // (a token behind the request's end is seen by no row: its step may be anything)
            if (MASK && pos0 + 16 * (x >> 1) + 8 * (x & 1) + g >= w.kv_len) sv[x] = mv[x] = 0.f;
            sv_top = fmaxf(sv_top, sv[x]);
          }
          auto sees = [&](int x, int nt, int c) {
            const int pos = pos0 + 16 * (x >> 1) + 8 * (x & 1) + g;
            return !MASK || pos <= climit[nt][c] || (pos >= vlo[nt][c] && pos < vhi[nt][c]);
          };
          // Score, and its distance from the reference.  Scores below kLarge: the reference joins the sum, whose terms are rounded as
          // coarsely as it is; beyond, it is subtracted from the rounded score whose maximum it was.
          auto score = [&](int x, int nt, int c) {
            return fmaf(sc[x >> 1][nt][2 * (x & 1) + c], sk[x], __fmul_rn(mk[x], qs[nt][c]));
          };
          float pr[PG][NT][4];
          auto scores = [&]() {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < PG; ++i)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int x = 2 * i + (e >> 1);
                  float y;
                  if (MASK) y = sees(x, nt, e & 1) ? __fsub_rn(score(x, nt, e & 1), ref[nt][e & 1]) : -INFINITY;
                  else y = fmaf(sc[i][nt][e], sk[x], fmaf(mk[x], qs[nt][e & 1], -ref[nt][e & 1]));
                  pr[i][nt][e] = y;
                  top = fmaxf(top, y);
                }
            return top;
          };
          if (__any_sync(0xffffffffu, scores() > kHeadroom + kLift || sv_top >= s_least)) {
            // some row's reference maximum moves, or its scale of the steps does: what has been summed up is scaled to the new ones
            float z[NT][2], step[NT][2], large = 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                z[nt][c] = -INFINITY;
                step[nt][c] = 0.f;
#pragma unroll
                for (int x = 0; x < 2 * PG; ++x)
                  if (sees(x, nt, c)) {
                    z[nt][c] = fmaxf(z[nt][c], score(x, nt, c));
                    if (MASK) step[nt][c] = fmaxf(step[nt][c], sv[x]);      // (NaN does not take part)
                  }
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) {
                  z[nt][c] = fmaxf(z[nt][c], __shfl_xor_sync(0xffffffffu, z[nt][c], x));
                  if (MASK) step[nt][c] = fmaxf(step[nt][c], __shfl_xor_sync(0xffffffffu, step[nt][c], x));
                }
                if (!MASK) large = fmaxf(large, fabsf(z[nt][c]));
              }
            const float step_all = MASK ? 0.f : __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(sv_top)));
            s_least = INFINITY;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                const float next_top = fmaxf(s_top[nt][c], pow2(max(-100, (int)(__float_as_uint(MASK ? step[nt][c] : step_all) >> 23) - 127 + 1)));
                const float fs = s_top[nt][c] * inverse(next_top);
                s_top[nt][c] = next_top;
                s_least = fminf(s_least, next_top);
                const float to = z[nt][c] - kLift;
                const float next = to > ref[nt][c] + kHeadroom || ref[nt][c] == kNoRef ? fmaxf(ref[nt][c], to) : ref[nt][c];
                const float f = exp2f(ref[nt][c] - next);
                ref[nt][c] = next;
                l[nt][c] *= f;
                om[nt][c] *= f;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                  o[nt][i][c] *= f * fs;
                  o[nt][i][2 + c] *= f * fs;
                }
              }
            scores();
            if (!MASK && __any_sync(0xffffffffu, large >= kLarge)) return true;
          }
          // ---- probabilities; O^T += C_V^T (P s_V)^T ----
          uint32_t b[PG][NT][2];
#pragma unroll
          for (int i = 0; i < PG; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float ps[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int x = 2 * i + (e >> 1);
                const float p_ = exp2f(pr[i][nt][e]);
                l[nt][e & 1] += p_;
                ps[e] = p_ * (sv[x] * inverse(MASK ? s_top[nt][e & 1] : s_top[0][0]));
                float pm = p_ * mv[x];
                if (MASK && !sees(x, nt, e & 1)) ps[e] = pm = 0.f;
                om[nt][e & 1] += pm;
              }
              b[i][nt][0] = transpose8x8(pack_f16(ps[0], ps[1]));
              b[i][nt][1] = transpose8x8(pack_f16(ps[2], ps[3]));
            }
#pragma unroll
          for (int i = 0; i < PG; ++i) {
            uint32_t v0[NW], v1[NW];
            load_words(v0, pg + i * SH::kBlock + kv4_v_codes(D) + t * D + g * (D / 8));
            load_words(v1, pg + i * SH::kBlock + kv4_v_codes(D) + (t + 4) * D + g * (D / 8));
#pragma unroll
            for (int j = 0; j < NW; ++j)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const uint32_t w0 = u ? v0[j] >> 8 : v0[j], w1 = u ? v1[j] >> 8 : v1[j];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                  mma_f16(o[nt][2 * j + u], w0 & 0x000f000fu, w0 & 0x00f000f0u, w1 & 0x000f000fu, w1 & 0x00f000f0u, b[i][nt][0], b[i][nt][1]);
              }
          }
          return false;
        };
        if (pos0 + PG * kPageSize - 1 <= lim && work(std::false_type{})) lim = -1;      // (to the end of the item)
        if (pos0 + PG * kPageSize - 1 > lim) work(std::true_type{});
        __syncwarp();
        request(slot_at);
        slot_at = slot_at == (kSlots - 1) * kSlot ? 0 : slot_at + kSlot;
      }

      if (item + 1 < item_end) load_rows(item_of(item + 1));
      __syncthreads();      // (the parts of the item before have been read)
      // ---- the warps' parts meet: row (column 2 t + c of group nt), the D / 8 values of g that this lane holds ----
      constexpr float k1 = 16777216.f, k16 = 1048576.f;      // 2^24 and 2^20
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float ls = l[nt][c], ms = om[nt][c];
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) {
            ls += __shfl_xor_sync(0xffffffffu, ls, x);
            ms += __shfl_xor_sync(0xffffffffu, ms, x);
          }
          float* row = merge + (warp * SH::kRows + nt * 8 + 2 * t + c) * SH::kRowPad;
          // tile 2 w + u: its row g is value 8 (w / 2) + 4 u + (w & 1) of the D / 8 of g, its row g + 8 the value two further, times 16
#pragma unroll
          for (int x = 0; x < NW / 2; ++x)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const float (&e)[4] = o[nt][4 * x + u];          // word 2 x: even values
              const float (&f)[4] = o[nt][4 * x + 2 + u];      // word 2 x + 1: odd values
              *reinterpret_cast<float4*>(row + g * (D / 8) + 8 * x + 4 * u) =
                  make_float4(fmaf(e[c] * k1, s_top[nt][c], ms), fmaf(f[c] * k1, s_top[nt][c], ms), fmaf(e[2 + c] * k16, s_top[nt][c], ms),
                              fmaf(f[2 + c] * k16, s_top[nt][c], ms));
            }
          if (g == 0) {
            row[D] = ref[nt][c];
            row[D + 1] = ls;
          }
        }
      __syncthreads();
      // a warp takes every kWarps-th row, a lane D / 32 consecutive values of it
      for (int rr = warp; rr < R; rr += W) {
        const float* part = merge + ((size_t)(rr / SH::kRows) * sh.warps * SH::kRows + rr % SH::kRows) * SH::kRowPad;   // of the group's first warp
        constexpr int kPart = SH::kRows * SH::kRowPad;
        const float m_mine = lane < sh.warps ? part[lane * kPart + D] : kNoRef, l_mine = lane < sh.warps ? part[lane * kPart + D + 1] : 0.f;
        float m_all = m_mine;
#pragma unroll
        for (int x = 16; x; x >>= 1) m_all = fmaxf(m_all, __shfl_xor_sync(0xffffffffu, m_all, x));
        const float f_mine = exp2f(m_mine - m_all);
        float l_all = f_mine * l_mine;
#pragma unroll
        for (int x = 16; x; x >>= 1) l_all += __shfl_xor_sync(0xffffffffu, l_all, x);
        constexpr int E = D / 32;
        float acc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll 4
        for (int k = 0; k < sh.warps; ++k) {
          const float f = __shfl_sync(0xffffffffu, f_mine, k);
          const float* src = part + k * kPart + lane * E;
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(f, src[e], acc[e]);
        }
        const int rho = rr, j = rho / P.group;
        if (w.part < 0) {
          const size_t row = (size_t)(w.tok0 + j) * P.n_q + w.kv_head * P.group + rho - j * P.group;
          const float inv = l_all > 0.f ? 1.f / l_all : 0.f * l_all;
          uint32_t* dst = reinterpret_cast<uint32_t*>(P.o + row * D + lane * E);
#pragma unroll
          for (int e = 0; e < E / 2; ++e) dst[e] = pack_bf16(acc[2 * e] * inv, acc[2 * e + 1] * inv);
          if (P.lse && lane == 0) P.lse[row] = log_sum_exp(m_all, l_all);
        } else {
          float* dst = P.part_o + ((size_t)w.part * 128 + rho) * D + lane * E;
          if constexpr (E == 4) *reinterpret_cast<float4*>(dst) = make_float4(acc[0], acc[1], acc[2], acc[3]);
          else *reinterpret_cast<float2*>(dst) = make_float2(acc[0], acc[1]);
          if (lane == 0) *reinterpret_cast<float2*>(P.part_ml + ((size_t)w.part * 128 + rho) * 2) = make_float2(m_all, l_all);
        }
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <int D, int NT>
void launch_rows(const Params& P, int n_sm, cudaStream_t st) {
  static bool configured[kMaxDevices] = {false};
  if (first_use_on_device(configured))
    cudaFuncSetAttribute(attention_kv4_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D, NT>::kTotal);
  launch_pdl(attention_kv4_kernel<D, NT>, dim3(n_sm), dim3(Shape<D, NT>::kThreads), Shape<D, NT>::kTotal, st, P);
}

}  // namespace

void launch_attention_kv4(const BatchLayout& bl, const Dims& dm, int layer, const void* q, void* o, float* lse, const void* kv_pool,
                          int64_t n_pages, float* part_o, float* part_ml, int n_sm, int max_rows, int* status, cudaStream_t st, bool list_settled) {
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
  P.inv_group = 65536 / P.group + 1;
  P.scale_log2 = 1.4426950408889634f / sqrtf((float)dm.head_dim);
  P.part_o = part_o;
  P.part_ml = part_ml;
  P.status = status;
  P.early_desc = list_settled ? 1 : 0;
  if (dm.head_dim == 64) (max_rows <= 8 ? launch_rows<64, 1> : launch_rows<64, 2>)(P, n_sm, st);
  else (max_rows <= 8 ? launch_rows<128, 1> : launch_rows<128, 2>)(P, n_sm, st);
}

}  // namespace recg

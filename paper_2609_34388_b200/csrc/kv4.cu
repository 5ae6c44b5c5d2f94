// Rows into and out of the KV pool: a request's positions for a pool in 4 bits (recg_kv_write, recg_kv_read), and the rows of a
// batch for either kind of pool (recg_kv_append, recg_kv_rows).
//
// Nothing is computed that counts, so the bytes bound it: 4 d in, d + 8 out per position and head (K and V) to write, the reverse
// to read.  The d / 8 lanes that share a row take eight values of it each, one 16-byte access, and reduce minimum and maximum by
// shuffles; each makes one word of codes.
#include <algorithm>
#include <cstring>

#include "kernels.h"
#include "kv4.cuh"

namespace recg {

namespace {

constexpr int kThreads = 256;
// Page ids travel with a launch: 3.5 KB of kernel parameters, or 16 of the 32 KB that there are for longer ranges.  (16001 positions in two
// launches of 3.5 KB, written and read: 41.8 us; in one: 37.6.)
constexpr int kFewPages = 896, kManyPages = 4000;
template <int N>
struct IoPages {
  int first;                         // logical page of ids[0]
  int ids[N];
};

// Positions [pos0, pos0 + n_pos) of a request; k, v [n_pos][n_kv][D].  Two positions of a token pair (2 p, 2 p + 1) and one head
// are 2 D / 8 consecutive lanes, so that a word of V, which holds both, is put together by one shuffle.
template <int D, bool WRITE, int N>
__global__ void __launch_bounds__(kThreads) kv4_io_kernel(uint8_t* pool, int64_t n_pages, int layer, int n_kv,
                                                          const __grid_constant__ IoPages<N> pages, int pos0, int n_pos,
                                                          uint4* __restrict__ k, uint4* __restrict__ v) {
  constexpr int kLanes = D / 8;
  griddep_launch();
  const unsigned unit = blockIdx.x * (kThreads / (2 * kLanes)) + threadIdx.x / (2 * kLanes);
  const int half = (threadIdx.x / kLanes) & 1, j = threadIdx.x % kLanes;
  const int first_pair = pos0 >> 1, n_pairs = ((pos0 + n_pos - 1) >> 1) - first_pair + 1;
  const int pair = (int)(unit / (unsigned)n_kv), h = (int)(unit - (unsigned)pair * (unsigned)n_kv);
  const int pos = 2 * (first_pair + pair) + half, i = pos - pos0;
  const bool mine = pair < n_pairs && i >= 0 && i < n_pos;
  const int tok = pos & (kPageSize - 1);
  uint8_t* block = nullptr;
  if (mine) block = pool + kv4_block_base(n_pages, n_kv, D, layer, pages.ids[pos / kPageSize - pages.first], h);
  const size_t at = mine ? ((size_t)i * n_kv + h) * kLanes + j : 0;
  griddep_wait();
  if (WRITE) {
    const uint4 kr = mine ? k[at] : make_uint4(0, 0, 0, 0), vr = mine ? v[at] : make_uint4(0, 0, 0, 0);
    uint32_t kp, vp;
    const uint32_t kw = kv4_quantise<kLanes>(kr, &kp), vw = kv4_quantise<kLanes>(vr, &vp);
    const uint32_t other = __shfl_xor_sync(0xffffffffu, vw, kLanes);
    const bool both = __shfl_xor_sync(0xffffffffu, (int)mine, kLanes) && mine;
    if (!mine) return;
    *reinterpret_cast<uint32_t*>(block + kv4_k_word(tok, j, D)) = kw;
    if (both) {       // the even position stores the word of the even values, the odd one that of the odd values
      *reinterpret_cast<uint32_t*>(block + kv4_v_word(tok, j, half, D)) = half ? __byte_perm(other, vw, 0x7632) : __byte_perm(vw, other, 0x5410);
    } else {
      *reinterpret_cast<uint16_t*>(block + kv4_v_word(tok, j, 0, D) + 2 * half) = (uint16_t)vw;
      *reinterpret_cast<uint16_t*>(block + kv4_v_word(tok, j, 1, D) + 2 * half) = (uint16_t)(vw >> 16);
    }
    if (j == 0) {
      *reinterpret_cast<uint32_t*>(block + kv4_k_pairs(D) + 4 * tok) = kp;
      *reinterpret_cast<uint32_t*>(block + kv4_v_pairs(D) + 4 * tok) = vp;
    }
  } else if (mine) {
    const uint32_t kw = *reinterpret_cast<const uint32_t*>(block + kv4_k_word(tok, j, D));
    const uint2 w = *reinterpret_cast<const uint2*>(block + kv4_v_word(tok, j, 0, D));
    const uint32_t kp = *reinterpret_cast<const uint32_t*>(block + kv4_k_pairs(D) + 4 * tok);
    const uint32_t vp = *reinterpret_cast<const uint32_t*>(block + kv4_v_pairs(D) + 4 * tok);
    k[at] = kv4_values(kw, kp);
    v[at] = kv4_values(half ? __byte_perm(w.x, w.y, 0x7632) : __byte_perm(w.x, w.y, 0x5410), vp);
  }
}

// The rows of a batch, row t to or from slot tok_slot[t]; rows row_stride elements apart.  FOUR: a pool in 4 bits.
// STAGED: row t of k and v lies in slot t of a bf16 pool of row_stride pages (v is not used).
template <int D, bool FOUR, bool WRITE, bool STAGED>
__global__ void __launch_bounds__(kThreads) kv_rows_kernel(uint8_t* pool, int64_t n_pages, int layer, int n_kv, const int* __restrict__ tok_slot,
                                                           int n_tok, const int* dyn, uint8_t* k, uint8_t* v, int64_t row_stride) {
  constexpr int kLanes = D / 8;
  griddep_launch();
  const unsigned unit = blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;      // (a row and head: below 2^20 n_kv)
  const int j = threadIdx.x % kLanes;
  const int t = (int)(unit / (unsigned)n_kv), h = (int)(unit - (unsigned)t * (unsigned)n_kv);
  const size_t at = STAGED ? 2 * (kv_tile_base(row_stride, n_kv, D, 0, t / kPageSize, h) + kv_tile_offset(t % kPageSize, 8 * j, D))
                           : ((size_t)t * row_stride + (size_t)h * D + 8 * j) * 2;
  if (STAGED) v = k + 2 * kv_tile_elems(D);
  griddep_wait();
  if (dyn) n_tok = dyn[0];
  const int slot = t < n_tok ? tok_slot[t] : -1;
  const bool mine = slot >= 0;                     // (a slot of a bad page is -1: the layout kernel has said so)
  const int tok = slot & (kPageSize - 1);
  const int64_t page = slot / kPageSize;
  if (FOUR) {
    uint8_t* block = mine ? pool + kv4_block_base(n_pages, n_kv, D, layer, page, h) : nullptr;
    if (WRITE) {
      const uint4 none = make_uint4(0, 0, 0, 0);
      const uint4 kr = mine ? *reinterpret_cast<const uint4*>(k + at) : none, vr = mine ? *reinterpret_cast<const uint4*>(v + at) : none;
      uint32_t kp, vp;
      const uint32_t kw = kv4_quantise<kLanes>(kr, &kp), vw = kv4_quantise<kLanes>(vr, &vp);
      if (!mine) return;
      *reinterpret_cast<uint32_t*>(block + kv4_k_word(tok, j, D)) = kw;
      *reinterpret_cast<uint16_t*>(block + kv4_v_word(tok, j, 0, D) + 2 * (tok & 1)) = (uint16_t)vw;
      *reinterpret_cast<uint16_t*>(block + kv4_v_word(tok, j, 1, D) + 2 * (tok & 1)) = (uint16_t)(vw >> 16);
      if (j == 0) {
        *reinterpret_cast<uint32_t*>(block + kv4_k_pairs(D) + 4 * tok) = kp;
        *reinterpret_cast<uint32_t*>(block + kv4_v_pairs(D) + 4 * tok) = vp;
      }
    } else if (mine) {
      const uint32_t kw = *reinterpret_cast<const uint32_t*>(block + kv4_k_word(tok, j, D));
      const uint2 w = *reinterpret_cast<const uint2*>(block + kv4_v_word(tok, j, 0, D));
      const uint32_t kp = *reinterpret_cast<const uint32_t*>(block + kv4_k_pairs(D) + 4 * tok);
      const uint32_t vp = *reinterpret_cast<const uint32_t*>(block + kv4_v_pairs(D) + 4 * tok);
      *reinterpret_cast<uint4*>(k + at) = kv4_values(kw, kp);
      *reinterpret_cast<uint4*>(v + at) = kv4_values((tok & 1) ? __byte_perm(w.x, w.y, 0x7632) : __byte_perm(w.x, w.y, 0x5410), vp);
    }
  } else if (mine) {
    uint8_t* tile = pool + 2 * (kv_tile_base(n_pages, n_kv, D, layer, page, h) + kv_tile_offset(tok, 8 * j, D));
    uint8_t* vtile = tile + 2 * kv_tile_elems(D);
    if (WRITE) {
      *reinterpret_cast<uint4*>(tile) = *reinterpret_cast<const uint4*>(k + at);
      *reinterpret_cast<uint4*>(vtile) = *reinterpret_cast<const uint4*>(v + at);
    } else {
      *reinterpret_cast<uint4*>(k + at) = *reinterpret_cast<const uint4*>(tile);
      *reinterpret_cast<uint4*>(v + at) = *reinterpret_cast<const uint4*>(vtile);
    }
  }
}

template <int N>
using IoKernel = void (*)(uint8_t*, int64_t, int, int, const IoPages<N>, int, int, uint4*, uint4*);
using RowsKernel = void (*)(uint8_t*, int64_t, int, int, const int*, int, const int*, uint8_t*, uint8_t*, int64_t);
template <int D>
RowsKernel rows_kernel(bool four, bool write) {
  if (four) return write ? kv_rows_kernel<D, true, true, false> : kv_rows_kernel<D, true, false, false>;
  return write ? kv_rows_kernel<D, false, true, false> : kv_rows_kernel<D, false, false, false>;
}

// As many of the positions as N page ids cover (whole pairs: a page is even); returns how many.
template <int N>
int launch_io(bool write, void* pool, int64_t n_pages, int layer, const Dims& dm, const int* page_row, int pos0, int n_pos, uint4* k, uint4* v,
              cudaStream_t st) {
  IoPages<N> pg;
  pg.first = pos0 / kPageSize;
  const int n = (int)std::min<int64_t>(n_pos, (int64_t)(pg.first + N) * kPageSize - pos0), last = (pos0 + n - 1) / kPageSize;
  memcpy(pg.ids, page_row + pg.first, (last - pg.first + 1) * sizeof(int));
  const size_t pairs = ((pos0 + n - 1) >> 1) - (pos0 >> 1) + 1, threads = pairs * dm.n_kv * (dm.head_dim / 4);
  IoKernel<N> kernel = dm.head_dim == 128 ? (write ? kv4_io_kernel<128, true, N> : kv4_io_kernel<128, false, N>)
                                          : (write ? kv4_io_kernel<64, true, N> : kv4_io_kernel<64, false, N>);
  launch_pdl(kernel, dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, static_cast<uint8_t*>(pool), n_pages, layer,
             dm.n_kv, pg, pos0, n, k, v);
  return n;
}

}  // namespace

void launch_kv4_io(bool write, void* pool, int64_t n_pages, int layer, const Dims& dm, const int* page_row, int pos0, int n_pos,
                   void* k, void* v, cudaStream_t st) {
  uint4 *kp = static_cast<uint4*>(k), *vp = static_cast<uint4*>(v);
  const size_t row = (size_t)dm.n_kv * (dm.head_dim / 8);
  while (n_pos > 0) {
    const bool few = (pos0 + n_pos - 1) / kPageSize - pos0 / kPageSize < kFewPages;
    const int n = few ? launch_io<kFewPages>(write, pool, n_pages, layer, dm, page_row, pos0, n_pos, kp, vp, st)
                      : launch_io<kManyPages>(write, pool, n_pages, layer, dm, page_row, pos0, n_pos, kp, vp, st);
    pos0 += n;
    n_pos -= n;
    kp += n * row;
    vp += n * row;
  }
}

void launch_kv_rows(bool write, bool four, const BatchLayout& bl, void* pool, int64_t n_pages, int layer, const Dims& dm, void* k,
                    void* v, int64_t row_stride, cudaStream_t st) {
  const int64_t threads = (int64_t)bl.n_tok * dm.n_kv * (dm.head_dim / 8);
  const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads));
  RowsKernel kernel = dm.head_dim == 128 ? rows_kernel<128>(four, write) : rows_kernel<64>(four, write);
  launch_pdl(kernel, grid, dim3(kThreads), 0, st, static_cast<uint8_t*>(pool), n_pages, layer, dm.n_kv, (const int*)bl.tok_slot,
             bl.n_tok, bl.dyn, static_cast<uint8_t*>(k), static_cast<uint8_t*>(v), row_stride);
}

void launch_kv_stage(const BatchLayout& bl, const void* stage, int stage_pages, void* pool, int64_t n_pages, int layer, const Dims& dm,
                     cudaStream_t st) {
  const int64_t threads = (int64_t)bl.n_tok * dm.n_kv * (dm.head_dim / 8);
  RowsKernel kernel = dm.head_dim == 128 ? kv_rows_kernel<128, true, true, true> : kv_rows_kernel<64, true, true, true>;
  uint8_t* from = const_cast<uint8_t*>(static_cast<const uint8_t*>(stage));
  launch_pdl(kernel, dim3((unsigned)((threads + kThreads - 1) / kThreads)), dim3(kThreads), 0, st, static_cast<uint8_t*>(pool), n_pages, layer,
             dm.n_kv, (const int*)bl.tok_slot, bl.n_tok, bl.dyn, from, from, (int64_t)stage_pages);
}

}  // namespace recg

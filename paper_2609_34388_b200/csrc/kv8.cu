// Rows into and out of a KV pool in 8 bits (kv8.cuh): a request's positions (recg_kv_write, recg_kv_read) and the rows of a batch
// (recg_kv_append, recg_kv_rows, rounds); and rows of a batch into any pool with their rotation on the way (recg_kv_append_rotary).
//
// A warp has a block of 16 tokens of one kv head, K or V, in its registers: what the new rows find there is read, the exponent follows
// all of them, and the block is written whole.  The bytes bound it: 4 d in and 2 d out per position and head (K and V) to write, the
// reverse to read.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "kernels.h"
#include "kv4.cuh"
#include "kv8.cuh"

namespace recg {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kFewPages = 896, kManyPages = 4000;      // page ids that travel with a launch (see kv4.cu)
template <int N>
struct IoPages {
  int first;                         // logical page of ids[0]
  int ids[N];
};

// A lane's values of a row, from a row of bf16
template <int D>
__device__ __forceinline__ void load_row(uint32_t (&x)[Kv8Block<D>::N], const uint8_t* row, int lane) {
  if constexpr (D == 128) {
    const uint2 t = *reinterpret_cast<const uint2*>(row + lane * 8);
    x[0] = t.x;
    x[1] = t.y;
  } else {
    x[0] = *reinterpret_cast<const uint32_t*>(row + lane * 4);
  }
}
template <int D>
__device__ __forceinline__ void store_row(const uint32_t (&x)[Kv8Block<D>::N], uint8_t* row, int lane) {
  if constexpr (D == 128) *reinterpret_cast<uint2*>(row + lane * 8) = make_uint2(x[0], x[1]);
  else *reinterpret_cast<uint32_t*>(row + lane * 4) = x[0];
}

// K (V: V) of one page and kv head: rows [first, end) of it, which `row(r)` finds in memory, written or read by a warp.
// `turn(x, r)`: what happens to a row of K on its way.
template <int D, bool V, bool WRITE, typename Row, typename Turn>
__device__ __forceinline__ void move_block(uint8_t* layer, int64_t n_pages, int n_kv, int64_t page, int h, int first, int end, int lane,
                                           Row row, Turn turn) {
  uint8_t* codes = layer + (page * n_kv + h) * kv8_block_bytes(D) + (V ? 16 * D : 0);
  uint32_t* header = reinterpret_cast<uint32_t*>(layer + kv8_headers(n_pages, n_kv, D)) + (page * n_kv + h) * 2 + (V ? 1 : 0);
  Kv8Block<D> b;
  if (WRITE) {
    if (first > 0) kv8_load<D, V>(b, codes, *header, first, lane);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      if (r >= first && r < end) load_row<D>(b.x[r], row(r), lane);
      else if (r >= end || first == 0)
#pragma unroll
        for (int i = 0; i < Kv8Block<D>::N; ++i) b.x[r][i] = 0;
    }
    if (!V)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (r >= first && r < end) turn(b.x[r], r);
    const uint32_t to = kv8_store<D, V>(b, codes, end, lane);
    if (lane == 0) *header = to;
  } else {
    kv8_load<D, V>(b, codes, *header, end, lane);
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (r >= first && r < end) store_row<D>(b.x[r], row(r), lane);
  }
}
struct AsItIs {
  template <int N>
  __device__ __forceinline__ void operator()(uint32_t (&)[N], int) const {}
};

// Positions [pos0, pos0 + n_pos) of a request; k, v [n_pos][n_kv][D].
template <int D, bool WRITE, int N>
__global__ void __launch_bounds__(kThreads) kv8_io_kernel(uint8_t* layer, int64_t n_pages, int n_kv, const __grid_constant__ IoPages<N> pages,
                                                          int pos0, int n_pos, uint8_t* k, uint8_t* v) {
  griddep_launch();
  const unsigned task = blockIdx.x * kWarps + (threadIdx.x >> 5), unit = task >> 1;
  const int lane = threadIdx.x & 31, p = (int)(unit / (unsigned)n_kv), h = (int)(unit - (unsigned)p * (unsigned)n_kv);
  const int start = (pages.first + p) * kPageSize, first = max(pos0 - start, 0), end = min(pos0 + n_pos - start, kPageSize);
  if (end <= first) return griddep_wait();
  const int64_t page = pages.ids[p];
  uint8_t* at = ((task & 1) ? v : k) + (size_t)h * (2 * D);
  const size_t stride = (size_t)n_kv * (2 * D);
  const auto row = [&](int r) { return at + (size_t)(start + r - pos0) * stride; };
  griddep_wait();
  if (task & 1) move_block<D, true, WRITE>(layer, n_pages, n_kv, page, h, first, end, lane, row, AsItIs());
  else move_block<D, false, WRITE>(layer, n_pages, n_kv, page, h, first, end, lane, row, AsItIs());
}

// What a CTA has of a batch: one page of one request, of which the rows [first, end) are the batch's rows t0 ..  A request with n rows touches
// at most n / 16 + 2 pages, so that the pages of request r can be numbered from cu_tok[r] / 16 + 2 r on without knowing the others'.
struct PageRows {
  int t0, first, end;
  int64_t page;                      // -1: no such page
};
__host__ __device__ __forceinline__ unsigned page_units(int n_tok, int n_req) { return (unsigned)(n_tok / kPageSize + 2 * n_req); }
__device__ __forceinline__ PageRows page_rows(const BatchLayout& bl, unsigned unit) {
  const int u = (int)unit;
  int r = 0;
  for (int r0 = 1; r0 < bl.n_req; r0 += kThreads) {
    const int i = r0 + threadIdx.x;
    r += __syncthreads_count(i < bl.n_req && bl.cu_tok[i] / kPageSize + 2 * i <= u);
  }
  const int cu = bl.cu_tok[r], L = bl.ctx_len[r], n = bl.cu_tok[r + 1] - cu;
  const int start = (L / kPageSize + u - (cu / kPageSize + 2 * r)) * kPageSize;
  PageRows p;
  p.first = max(L - start, 0);
  p.end = min(L + n - start, kPageSize);
  p.t0 = cu + start + p.first - L;
  p.page = -1;
  if (p.first < p.end) {
    const int slot = bl.tok_slot[p.t0];
    if (slot >= 0) p.page = slot / kPageSize;        // (a slot of a bad page is -1: the layout kernel has said so)
  }
  return p;
}

// Rows of a batch.  STAGED: row t of k and v lies in slot t of a bf16 pool of row_stride pages (v is not used).
template <int D, bool WRITE, bool STAGED>
__global__ void __launch_bounds__(kThreads) kv8_rows_kernel(const __grid_constant__ BatchLayout bl, uint8_t* layer, int64_t n_pages, int n_kv,
                                                            uint8_t* k, uint8_t* v, int64_t row_stride) {
  griddep_launch();
  griddep_wait();
  const PageRows p = page_rows(bl, blockIdx.x);
  if (p.page < 0) return;
  const int lane = threadIdx.x & 31;
  for (int task = blockIdx.y * kWarps + (threadIdx.x >> 5); task < 2 * n_kv; task += kWarps * gridDim.y) {
    const int h = task >> 1;
    const auto row = [&](int r) {
      const int t = p.t0 + r - p.first;
      if (STAGED)      // (a lane finds its values in the swizzled row by itself: they are less than a chunk)
        return k + 2 * (kv_tile_base(row_stride, n_kv, D, 0, t / kPageSize, h) + ((task & 1) ? kv_tile_elems(D) : 0) +
                        kv_tile_offset(t % kPageSize, lane * (D / 32), D) - lane * (D / 32));
      return ((task & 1) ? v : k) + ((size_t)t * row_stride + (size_t)h * D) * 2;
    };
    if (task & 1) move_block<D, true, WRITE>(layer, n_pages, n_kv, p.page, h, p.first, p.end, lane, row, AsItIs());
    else move_block<D, false, WRITE>(layer, n_pages, n_kv, p.page, h, p.first, p.end, lane, row, AsItIs());
  }
}

// ---- rotation and append -------------------------------------------------------------------------------------------------------
// The angles of the page's rows once per CTA, in 64 bits, for all heads.  K is rotated in 64 bits too (the result goes on to be rounded to
// codes, where the last bit of a sum next to a border decides between two of them), q in 32.
struct RotaryArgs {
  const uint8_t *q, *k, *v;
  uint8_t* q_out;                    // [n_tok][n_q][D]; q may be null
  int64_t q_stride, kv_stride;       // elements from row to row
  uint8_t* pool;                     // of 8 bits: the layer
  int64_t n_pages;
  int layer, n_q, n_kv;
  double turn[64];                   // base^(-2 i / D)
};
// y = x cos - (partner) sin in the first half of a row, x cos + (partner) sin in the second
__device__ __forceinline__ float turned(float x, float other, double2 cs, bool second) {
  return (float)((double)x * cs.x + (second ? cs.y : -cs.y) * (double)other);
}
__device__ __forceinline__ float turned(float x, float other, float2 cs, bool second) {
  return x * cs.x + (second ? cs.y : -cs.y) * other;
}
template <typename T>
__device__ __forceinline__ uint32_t turned_pair(uint32_t x, uint32_t other, const T* cs, bool second) {
  return pack_bf16(turned(__uint_as_float(x << 16), __uint_as_float(other << 16), cs[0], second),
                   turned(__uint_as_float(x & 0xffff0000u), __uint_as_float(other & 0xffff0000u), cs[1], second));
}
// Eight values of a row, chunk j of LANES that consecutive lanes hold
template <int LANES, typename T>
__device__ __forceinline__ uint4 turned_chunk(const uint4& x, const T* row, int j) {
  const uint32_t in[4] = {x.x, x.y, x.z, x.w};
  const bool second = j >= LANES / 2;
  const T* cs = row + 8 * (j % (LANES / 2));
  uint32_t out[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = turned_pair(in[i], __shfl_xor_sync(0xffffffffu, in[i], LANES / 2), cs + 2 * i, second);
  return make_uint4(out[0], out[1], out[2], out[3]);
}

// BITS: of the pool.
template <int D, int BITS>
__global__ void __launch_bounds__(kThreads) append_rotary_kernel(const __grid_constant__ BatchLayout bl, const __grid_constant__ RotaryArgs A) {
  constexpr int kLanes = D / 8;
  __shared__ double2 exact[kPageSize][D / 2];
  __shared__ float2 plain[kPageSize][D / 2];
  griddep_launch();
  griddep_wait();
  const PageRows p = page_rows(bl, blockIdx.x);
  const int rows = p.end - p.first;
  if (rows <= 0) return;
  for (int i = threadIdx.x; i < rows * (D / 2); i += kThreads) {
    const double angle = (double)bl.tok_pos[p.t0 + i / (D / 2)] * A.turn[i % (D / 2)];
    double2 cs;
    sincos(angle, &cs.y, &cs.x);
    exact[i / (D / 2)][i % (D / 2)] = cs;
    plain[i / (D / 2)][i % (D / 2)] = make_float2((float)cs.x, (float)cs.y);
  }
  __syncthreads();
  const int warp = blockIdx.y * kWarps + (threadIdx.x >> 5), n_warps = kWarps * gridDim.y, lane = threadIdx.x & 31, j = lane % kLanes;
  constexpr int kRows = 32 / kLanes;       // row heads that a warp moves at once
  int done = 0;                            // tasks that have been handed out, a warp each
  // ---- K and V ----
  if (BITS == 8) {
    const int tasks = p.page < 0 ? 0 : 2 * A.n_kv;
    for (int task = warp; task < tasks; task += n_warps) {
      const int h = task >> 1;
      const auto row = [&](int r) { return const_cast<uint8_t*>((task & 1) ? A.v : A.k) + ((size_t)(p.t0 + r - p.first) * A.kv_stride + (size_t)h * D) * 2; };
      const auto turn = [&](uint32_t (&x)[Kv8Block<D>::N], int r) {
        const double2* cs = exact[r - p.first] + (D / 32) * (lane & 15);
#pragma unroll
        for (int i = 0; i < Kv8Block<D>::N; ++i) x[i] = turned_pair(x[i], __shfl_xor_sync(0xffffffffu, x[i], 16), cs + 2 * i, lane >= 16);
      };
      if (task & 1) move_block<D, true, true>(A.pool, A.n_pages, A.n_kv, p.page, h, p.first, p.end, lane, row, AsItIs());
      else move_block<D, false, true>(A.pool, A.n_pages, A.n_kv, p.page, h, p.first, p.end, lane, row, turn);
    }
    done = tasks;
  } else {
    const int units = p.page < 0 ? 0 : rows * A.n_kv, tasks = (units + kRows - 1) / kRows;
    for (int task = warp; task < tasks; task += n_warps) {
      const int unit = task * kRows + lane / kLanes, r = unit / A.n_kv, h = unit - r * A.n_kv, tok = p.first + r;
      const bool mine = unit < units;
      const size_t at = ((size_t)(p.t0 + r) * A.kv_stride + (size_t)h * D + 8 * j) * 2;
      const uint4 none = make_uint4(0, 0, 0, 0);
      uint4 k = mine ? *reinterpret_cast<const uint4*>(A.k + at) : none, v = mine ? *reinterpret_cast<const uint4*>(A.v + at) : none;
      k = turned_chunk<kLanes>(k, exact[mine ? r : 0], j);
      if (BITS == 16) {
        if (!mine) continue;
        uint8_t* tile = A.pool + 2 * (kv_tile_base(A.n_pages, A.n_kv, D, A.layer, p.page, h) + kv_tile_offset(tok, 8 * j, D));
        *reinterpret_cast<uint4*>(tile) = k;
        *reinterpret_cast<uint4*>(tile + 2 * kv_tile_elems(D)) = v;
      } else {
        uint32_t kp, vp;
        const uint32_t kw = kv4_quantise<kLanes>(k, &kp), vw = kv4_quantise<kLanes>(v, &vp);
        if (!mine) continue;
        uint8_t* block = A.pool + kv4_block_base(A.n_pages, A.n_kv, D, A.layer, p.page, h);
        *reinterpret_cast<uint32_t*>(block + kv4_k_word(tok, j, D)) = kw;
        *reinterpret_cast<uint16_t*>(block + kv4_v_word(tok, j, 0, D) + 2 * (tok & 1)) = (uint16_t)vw;
        *reinterpret_cast<uint16_t*>(block + kv4_v_word(tok, j, 1, D) + 2 * (tok & 1)) = (uint16_t)(vw >> 16);
        if (j == 0) {
          *reinterpret_cast<uint32_t*>(block + kv4_k_pairs(D) + 4 * tok) = kp;
          *reinterpret_cast<uint32_t*>(block + kv4_v_pairs(D) + 4 * tok) = vp;
        }
      }
    }
    done = tasks;
  }
  // ---- q (its tasks go on where those of K and V have ended) ----
  if (!A.q) return;
  const int units = rows * A.n_q, tasks = (units + kRows - 1) / kRows;
  for (int task = (warp + n_warps - done % n_warps) % n_warps; task < tasks; task += n_warps) {
    const int unit = task * kRows + lane / kLanes, r = unit / A.n_q, h = unit - r * A.n_q;
    const bool mine = unit < units;
    const size_t t = p.t0 + (mine ? r : 0);
    uint4 x = make_uint4(0, 0, 0, 0);
    if (mine) x = *reinterpret_cast<const uint4*>(A.q + (t * A.q_stride + (size_t)h * D + 8 * j) * 2);
    x = turned_chunk<kLanes>(x, plain[mine ? r : 0], j);
    if (mine) *reinterpret_cast<uint4*>(A.q_out + ((t * A.n_q + h) * D + 8 * j) * 2) = x;
  }
}

template <int N>
using IoKernel = void (*)(uint8_t*, int64_t, int, const IoPages<N>, int, int, uint8_t*, uint8_t*);
using RowsKernel = void (*)(const BatchLayout, uint8_t*, int64_t, int, uint8_t*, uint8_t*, int64_t);

template <int N>
int launch_io(bool write, uint8_t* layer, int64_t n_pages, const Dims& dm, const int* page_row, int pos0, int n_pos, uint8_t* k, uint8_t* v,
              cudaStream_t st) {
  IoPages<N> pg;
  pg.first = pos0 / kPageSize;
  const int n = (int)std::min<int64_t>(n_pos, (int64_t)(pg.first + N) * kPageSize - pos0), last = (pos0 + n - 1) / kPageSize;
  memcpy(pg.ids, page_row + pg.first, (last - pg.first + 1) * sizeof(int));
  const unsigned tasks = (unsigned)(last - pg.first + 1) * dm.n_kv * 2;
  IoKernel<N> kernel = dm.head_dim == 128 ? (write ? kv8_io_kernel<128, true, N> : kv8_io_kernel<128, false, N>)
                                          : (write ? kv8_io_kernel<64, true, N> : kv8_io_kernel<64, false, N>);
  launch_pdl(kernel, dim3((tasks + kWarps - 1) / kWarps), dim3(kThreads), 0, st, layer, n_pages, dm.n_kv, pg, pos0, n, k, v);
  return n;
}

uint8_t* layer_of(void* pool, int64_t n_pages, int layer, const Dims& dm) {
  return static_cast<uint8_t*>(pool) + layer * kv8_layer_bytes(n_pages, dm.n_kv, dm.head_dim);
}
// CTAs that share a page: as many as it takes to fill the SMs, but no more than there are tasks for
int splits(unsigned units, int tasks) { return std::max(1, std::min((tasks + kWarps - 1) / kWarps, (int)(296 / std::max(units, 1u)))); }

}  // namespace

void launch_kv8_io(bool write, void* pool, int64_t n_pages, int layer, const Dims& dm, const int* page_row, int pos0, int n_pos,
                   void* k, void* v, cudaStream_t st) {
  uint8_t *at = layer_of(pool, n_pages, layer, dm), *kp = static_cast<uint8_t*>(k), *vp = static_cast<uint8_t*>(v);
  const size_t row = (size_t)dm.n_kv * dm.head_dim * 2;
  while (n_pos > 0) {
    const bool few = (pos0 + n_pos - 1) / kPageSize - pos0 / kPageSize < kFewPages;
    const int n = few ? launch_io<kFewPages>(write, at, n_pages, dm, page_row, pos0, n_pos, kp, vp, st)
                      : launch_io<kManyPages>(write, at, n_pages, dm, page_row, pos0, n_pos, kp, vp, st);
    pos0 += n;
    n_pos -= n;
    kp += n * row;
    vp += n * row;
  }
}

void launch_kv8_rows(bool write, bool staged, const BatchLayout& bl, void* pool, int64_t n_pages, int layer, const Dims& dm, void* k, void* v,
                     int64_t row_stride, cudaStream_t st) {
  const unsigned units = page_units(bl.n_tok, bl.n_req);
  RowsKernel kernel;
  if (dm.head_dim == 128) kernel = staged ? kv8_rows_kernel<128, true, true> : write ? kv8_rows_kernel<128, true, false> : kv8_rows_kernel<128, false, false>;
  else kernel = staged ? kv8_rows_kernel<64, true, true> : write ? kv8_rows_kernel<64, true, false> : kv8_rows_kernel<64, false, false>;
  launch_pdl(kernel, dim3(units, splits(units, 2 * dm.n_kv)), dim3(kThreads), 0, st, bl, layer_of(pool, n_pages, layer, dm), n_pages, dm.n_kv,
             static_cast<uint8_t*>(k), static_cast<uint8_t*>(v), row_stride);
}

void launch_append_rotary(int bits, const BatchLayout& bl, void* pool, int64_t n_pages, int layer, const Dims& dm, const void* q, int64_t q_stride,
                          void* q_out, const void* k, const void* v, int64_t kv_stride, cudaStream_t st) {
  RotaryArgs A;
  A.q = static_cast<const uint8_t*>(q);
  A.k = static_cast<const uint8_t*>(k);
  A.v = static_cast<const uint8_t*>(v);
  A.q_out = static_cast<uint8_t*>(q_out);
  A.q_stride = q_stride;
  A.kv_stride = kv_stride;
  A.pool = bits == 8 ? layer_of(pool, n_pages, layer, dm) : static_cast<uint8_t*>(pool);
  A.n_pages = n_pages;
  A.layer = layer;
  A.n_q = dm.n_q;
  A.n_kv = dm.n_kv;
  const int half = dm.head_dim / 2;
  for (int i = 0; i < half; ++i) A.turn[i] = exp(-log((double)dm.rope_base) * i / half);
  using Kernel = void (*)(const BatchLayout, const RotaryArgs);
  Kernel kernel;
  if (dm.head_dim == 128) kernel = bits == 16 ? append_rotary_kernel<128, 16> : bits == 8 ? append_rotary_kernel<128, 8> : append_rotary_kernel<128, 4>;
  else kernel = bits == 16 ? append_rotary_kernel<64, 16> : bits == 8 ? append_rotary_kernel<64, 8> : append_rotary_kernel<64, 4>;
  const unsigned units = page_units(bl.n_tok, bl.n_req);
  launch_pdl(kernel, dim3(units, splits(units, 2 * dm.n_kv + dm.n_q)), dim3(kThreads), 0, st, bl, A);
}

}  // namespace recg

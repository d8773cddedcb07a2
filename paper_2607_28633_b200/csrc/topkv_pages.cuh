// Page operators of a paged cache: fork, free, extend, compact, copy.
//
// The tables (block table, lengths, reference counts) are integers and every rule that picks a
// page takes the lowest free id first, so a call has one possible result whatever the order in
// which its CTAs run. Each call is one to three launches: the tables are copied when the caller
// wants them in other buffers (beside the planning, or before), one CTA works out who gets which page
// (fork, extend: prefix sums over the requests, then one walk over the reference counts up to the
// last page that is needed), and a wide grid rewrites rows and moves page contents.
//
// The contents are moved like every other page here: streaming 16- or 32-byte accesses, several
// in flight per thread, about 64 KiB per CTA and turn, so that part is bound by memory bandwidth (255
// pages of 72 KiB in 8 layers: 45.5 us for 301 MB, 1.0 of the measured copy); the planning CTA is
// bound by the latency of dependent rounds of loads and barriers: 5 us for a pool of up to 4,096 pages, one
// round. It grows with the pages in use, since the lowest free page lies behind them: extend and fork 10 us
// at 25,000 pages, 23 us at 80,000 nearly all in use (out of place, tables copied). In compact every
// planning CTA reads all counts, 25 us at 80,000 pages with nothing to move.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "topkv_common.cuh"

namespace topkv {

constexpr int kPlanThreads = 1024;
constexpr int kPlanPages = 4;  // reference counts per thread and round of the walk
constexpr int kMoveThreads = 256;

// What the page operators change: all three arrays are read and written in place.
struct PageTables {
  int32_t* bt;   // [R][maxp]
  int32_t* sl;   // [R]
  int32_t* ref;  // [num_pages]
  int R, maxp, P;
  int num_pages;
};

// Where the bytes of a page lie, and how a page is cut for moving.
struct PageGeom {
  uint8_t* pool;          // base of layer `first_layer`
  int64_t S_layer, S_page, S_kv, S_tok, S_unit;
  int64_t unit_bytes;     // contiguous bytes of one (token, plane[, head])
  int F, U, P;
  int layers;
  int linear;             // 1: consecutive tokens of one (plane[, head]) are adjacent
  int tps, cpp;           // tokens per part, parts per page
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (int)(((int64_t)a + b - 1) / b); }

// Exclusive sum of `x` over the CTA (up to 1,024 threads); *total = sum over all threads.
// s_scan: 33 words. The barrier at its start makes it safe to call in a loop.
template <typename T>
__device__ __forceinline__ T block_exclusive_sum(T x, T* s_scan, T* total) {
  const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5, nw = blockDim.x >> 5;
  T incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  __syncthreads();
  if (lane == 31) s_scan[wid] = incl;
  __syncthreads();
  if (wid == 0) {
    const T w = lane < nw ? s_scan[lane] : 0;
    T wi = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T up = __shfl_up_sync(0xffffffffu, wi, o);
      if (lane >= o) wi += up;
    }
    if (lane < nw) s_scan[lane] = wi - w;
    if (lane == 31) s_scan[32] = wi;
  }
  __syncthreads();
  *total = s_scan[32];
  return incl - x + s_scan[wid];
}

// The first `limit` free pages in ascending order, written to `list`; returns how many there are
// (at most limit). One CTA; stops at the page that completes the list.
__device__ __forceinline__ int list_free_pages(const int32_t* ref, int num_pages, int limit, int32_t* list,
                                               int* s_scan) {
  int found = 0;
  for (int64_t base = 0; base < num_pages && found < limit; base += kPlanThreads * kPlanPages) {
    const int64_t p0 = base + (int64_t)threadIdx.x * kPlanPages;
    bool f[kPlanPages];
    int n = 0;
#pragma unroll
    for (int k = 0; k < kPlanPages; ++k) {
      f[k] = p0 + k < num_pages && ref[p0 + k] <= 0;
      n += f[k];
    }
    int total;
    int rank = found + block_exclusive_sum(n, s_scan, &total);
#pragma unroll
    for (int k = 0; k < kPlanPages; ++k)
      if (f[k]) {
        if (rank < limit) list[rank] = (int32_t)(p0 + k);
        ++rank;
      }
    found += total;
  }
  __syncthreads();
  return min(found, limit);
}

// ---- tables into other buffers ------------------------------------------------------------------
struct TablesCopyParams {
  const int32_t* src[3];
  int32_t* dst[3];
  int64_t n[3];  // 0: stays where it is
};
__device__ __forceinline__ void copy_tables(const TablesCopyParams& p, int cta, int ctas) {
  const int64_t t = (int64_t)cta * blockDim.x + threadIdx.x, step = (int64_t)ctas * blockDim.x;
#pragma unroll
  for (int a = 0; a < 3; ++a)
    for (int64_t i = t; i < p.n[a]; i += step) p.dst[a][i] = p.src[a][i];
}
__global__ void __launch_bounds__(256) topkv_tables_copy_kernel(const TablesCopyParams p) {
  pdl_prologue(0);
  copy_tables(p, blockIdx.x, gridDim.x);
}

// ---- free ---------------------------------------------------------------------------------------
struct FreeParams {
  PageTables t;
  TablesCopyParams copy;  // done by the kernel itself (one CTA, small tables)
  const int32_t* rows;
  int n;
};
// A warp per listed row. Whoever takes the row's length (an exchange with 0) frees its pages, so a
// row that is listed twice is freed once; reference counts go down by integer atomics, whose order
// does not show in the result.
__global__ void __launch_bounds__(kPlanThreads) topkv_free_kernel(const FreeParams p) {
  pdl_prologue(0);
  if (gridDim.x == 1) {
    copy_tables(p.copy, 0, 1);
    __syncthreads();
  }
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)gridDim.x * (blockDim.x >> 5);
  for (int64_t i = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); i < p.n; i += warps) {
    const int r = p.rows[i];
    if (r < 0 || r >= p.t.R) {
      if (lane == 0) raise_error(kErrTable);
      continue;
    }
    int len = 0;
    if (lane == 0) len = atomicExch(p.t.sl + r, 0);
    len = __shfl_sync(0xffffffffu, len, 0);
    if (len <= 0) {
      if (lane == 0 && len < 0) raise_error(kErrTable);
      continue;
    }
    int pages = ceil_div(len, p.t.P);
    if (pages > p.t.maxp) {
      pages = p.t.maxp;
      if (lane == 0) raise_error(kErrTable);
    }
    int32_t* row = p.t.bt + (int64_t)r * p.t.maxp;
    for (int j = lane; j < p.t.maxp; j += 32) {
      if (j < pages) {
        const int pg = row[j];
        if (pg < 0 || pg >= p.t.num_pages) {
          raise_error(kErrTable);
        } else if (atomicSub(p.t.ref + pg, 1) <= 0) {  // it was free already: the count stays at 0
          atomicAdd(p.t.ref + pg, 1);
          raise_error(kErrTable);
        }
      }
      row[j] = -1;
    }
  }
}

// ---- extend -------------------------------------------------------------------------------------
struct ExtendParams {
  PageTables t;
  TablesCopyParams copy;  // done by the kernel itself
  const int32_t* add;  // [R]
  int32_t* prefix;     // workspace [R + 1]: pages wanted by the requests before r (cut off at num_pages + 1)
  int32_t* list;       // workspace [num_pages]
};
// Pages that request r wants, -1 when the request is unusable.
__device__ __forceinline__ int extend_need(const ExtendParams& p, int r, int* len, int* add) {
  *len = p.t.sl[r];
  *add = p.add[r];
  const int64_t row = (int64_t)p.t.maxp * p.t.P;
  if (*len < 0 || *add < 0 || (int64_t)*len + *add > row) return -1;
  return ceil_div(*len + *add, p.t.P) - ceil_div(*len, p.t.P);
}
// Requests are served in order: r gets its pages if the free ones suffice for it and all before it.
__global__ void __launch_bounds__(kPlanThreads) topkv_extend_kernel(const ExtendParams p) {
  __shared__ int64_t s_sum[33];
  __shared__ int s_scan[33];
  pdl_prologue(0);
  const int tid = threadIdx.x;
  copy_tables(p.copy, 0, 1);
  __syncthreads();
  const int64_t cap = (int64_t)p.t.num_pages + 1;  // more than this is never there
  int64_t carry = 0;
  for (int64_t base = 0; base < p.t.R; base += kPlanThreads) {
    const int64_t r = base + tid;
    int len, add, need = 0;
    if (r < p.t.R) {
      need = extend_need(p, (int)r, &len, &add);
      if (need < 0) {
        raise_error(kErrTable);
        need = 0;
      }
    }
    int64_t total;
    const int64_t before = carry + block_exclusive_sum((int64_t)need, s_sum, &total);
    if (r < p.t.R) p.prefix[r + 1] = (int32_t)min(before + need, cap);
    carry += total;
  }
  if (tid == 0) p.prefix[0] = 0;
  const int wanted = (int)min(carry, (int64_t)p.t.num_pages);
  const int found = wanted > 0 ? list_free_pages(p.t.ref, p.t.num_pages, wanted, p.list, s_scan) : 0;
  __syncthreads();
  for (int k = tid; k < found; k += kPlanThreads) {  // the k-th free page goes to the request r with
    int lo = 0, hi = p.t.R;                          // prefix[r] <= k < prefix[r + 1]
    while (hi - lo > 1) {
      const int mid = lo + ((hi - lo) >> 1);
      if (p.prefix[mid] <= k)
        lo = mid;
      else
        hi = mid;
    }
    if (p.prefix[lo + 1] > found) continue;  // not all of its pages are there
    const int pg = p.list[k];
    p.t.bt[(int64_t)lo * p.t.maxp + ceil_div(p.t.sl[lo], p.t.P) + (k - p.prefix[lo])] = pg;
    p.t.ref[pg] = 1;
  }
  __syncthreads();
  for (int r = tid; r < p.t.R; r += kPlanThreads) {
    int len, add;
    const int need = extend_need(p, r, &len, &add);
    if (need < 0) continue;
    if (need > 0 && p.prefix[r + 1] > found)
      raise_error(kErrPages);
    else
      p.t.sl[r] = len + add;
  }
}

// ---- moving page contents -----------------------------------------------------------------------
// Tokens [t0, t0 + v) of page `src` to page `dst` of one layer, all planes and heads, by one CTA.
template <int VEC>
__device__ __forceinline__ void move_page(const PageGeom& g, uint8_t* base, int src, int dst, int t0, int v) {
  constexpr int kUnroll = VEC == 32 ? 4 : 8;
  const int64_t run = g.linear ? (int64_t)v * g.unit_bytes : g.unit_bytes;  // bytes of one contiguous run
  const uint32_t cps = (uint32_t)(run / VEC);
  const uint32_t fu = (uint32_t)(g.F * g.U);
  const uint32_t total = cps * fu * (g.linear ? 1u : (uint32_t)v);
  const uint8_t* s = base + (int64_t)src * g.S_page + (int64_t)t0 * g.S_tok;
  uint8_t* d = base + (int64_t)dst * g.S_page + (int64_t)t0 * g.S_tok;
  for (uint32_t i0 = threadIdx.x; i0 < total; i0 += blockDim.x * kUnroll) {
    Vec<VEC> buf[kUnroll];
    int64_t off[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const uint32_t i = i0 + u * blockDim.x;
      if (i < total) {
        const uint32_t seg = i / cps, w = i - seg * cps;
        const uint32_t t = seg / fu, ch = seg - t * fu;  // linear runs: seg < fu, so t = 0
        const uint32_t c = ch / (uint32_t)g.U, h = ch - c * (uint32_t)g.U;
        off[u] = (int64_t)c * g.S_kv + (int64_t)h * g.S_unit + (int64_t)t * g.S_tok + (int64_t)w * VEC;
        buf[u].load(s + off[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i0 + u * blockDim.x < total) buf[u].store(d + off[u]);
  }
}

// Whole pages src[k] -> dst[k], k < n, in every layer. An item is one part of one page of one layer;
// the CTAs take them in turn, since the number of pages may be known on the device only.
template <int VEC>
__device__ __forceinline__ void move_pages(const PageGeom& g, const int32_t* src, const int32_t* dst, int64_t n,
                                           int num_pages) {
  const int64_t per_page = (int64_t)g.layers * g.cpp, items = n * per_page;
  for (int64_t it = blockIdx.x; it < items; it += gridDim.x) {
    const int64_t k = it / per_page;
    const int rest = (int)(it - k * per_page);
    const int layer = rest / g.cpp, part = rest - layer * g.cpp;
    const int s = src[k], d = dst[k];
    if (s < 0 || s >= num_pages || d < 0 || d >= num_pages) {
      if (threadIdx.x == 0) raise_error(kErrTable);
      continue;
    }
    if (s == d) continue;
    const int t0 = part * g.tps;
    move_page<VEC>(g, g.pool + (int64_t)layer * g.S_layer, s, d, t0, min(g.tps, g.P - t0));
  }
}
struct MoveParams {
  PageGeom g;
  const int32_t* src;  // [n] page ids
  const int32_t* dst;  // [n]
  int64_t n;
  int num_pages;
};
template <int VEC>
__global__ void __launch_bounds__(kMoveThreads, 3) topkv_page_move_kernel(const MoveParams p) {
  pdl_prologue(0);
  move_pages<VEC>(p.g, p.src, p.dst, p.n, p.num_pages);
}

// ---- fork ---------------------------------------------------------------------------------------
struct ForkRecord {
  int32_t parent, child, len, fresh;  // parent -1: refused; fresh -1: no page of its own needed
};
struct ForkParams {
  PageTables t;
  TablesCopyParams copy;
  PageGeom g;
  const int32_t* parents;
  const int32_t* children;
  int n;
  ForkRecord* rec;   // workspace [n]
  int32_t* claim;    // workspace [R]: the first fork that names the row as its child
  int32_t* list;     // workspace [n]: free pages
};
// Which fork is done, and with which page: everything the second kernel needs is in the records,
// so it never reads a row or a length that another of its CTAs writes.
__global__ void __launch_bounds__(kPlanThreads) topkv_fork_plan_kernel(const ForkParams p) {
  __shared__ int s_scan[33];
  pdl_prologue(0);
  if (blockIdx.x > 0) {  // the other CTAs copy the tables; this one reads them where they were
    copy_tables(p.copy, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  const int tid = threadIdx.x;
  const int32_t *bt = p.copy.src[0], *sl = p.copy.src[1], *ref = p.copy.src[2];
  for (int i = tid; i < p.n; i += kPlanThreads) {  // only the rows that are named have to be cleared
    const int c = p.children[i];
    if (c >= 0 && c < p.t.R) p.claim[c] = 0x7fffffff;
  }
  // as many free pages as the forks could want, whichever of them are done (its barriers serve the claims)
  const int found = list_free_pages(ref, p.t.num_pages, min(p.n, p.t.num_pages), p.list, s_scan);
  for (int i = tid; i < p.n; i += kPlanThreads) {
    const int c = p.children[i];
    if (c >= 0 && c < p.t.R) atomicMin(p.claim + c, i);
  }
  __syncthreads();
  int carry = 0;
  const int64_t row = (int64_t)p.t.maxp * p.t.P;
  for (int base = 0; base < p.n; base += kPlanThreads) {
    const int i = base + tid;
    int need = 0;
    ForkRecord rec = {-1, -1, 0, -1};
    if (i < p.n) {
      const int a = p.parents[i], c = p.children[i];
      bool ok = a >= 0 && a < p.t.R && c >= 0 && c < p.t.R && a != c;
      if (ok) ok = *(volatile int32_t*)(p.claim + c) == i && sl[c] == 0;
      const int len = ok ? sl[a] : 0;
      if (ok) ok = len >= 0 && len <= row;
      if (ok && len % p.t.P != 0) {  // the page that is shared in part must be a page of the pool
        const int pg = bt[(int64_t)a * p.t.maxp + len / p.t.P];
        ok = pg >= 0 && pg < p.t.num_pages;
        need = ok;
      }
      if (ok) {
        rec.parent = a;
        rec.child = c;
        rec.len = len;
      } else {
        raise_error(kErrTable);
      }
    }
    int total;
    const int rank = carry + block_exclusive_sum(need, s_scan, &total);
    if (need) rec.fresh = rank;
    if (i < p.n) p.rec[i] = rec;
    carry += total;
  }
  for (int i = tid; i < p.n; i += kPlanThreads) {  // this thread wrote these records itself
    const int rank = p.rec[i].fresh;
    if (rank < 0) continue;
    if (rank < found) {
      p.rec[i].fresh = p.list[rank];
    } else {
      p.rec[i].parent = -1;
      raise_error(kErrPages);
    }
  }
}
// blockIdx.y 0 writes the child's row, length and reference counts; blockIdx.y 1 + layer * cpp +
// part copies the tokens of the parent's last, partly filled page.
template <int VEC>
__global__ void __launch_bounds__(kMoveThreads, 3) topkv_fork_apply_kernel(const ForkParams p) {
  pdl_prologue(0);
  const ForkRecord rec = p.rec[blockIdx.x];
  if (rec.parent < 0) return;
  const int full = rec.len / p.t.P, tail = rec.len - full * p.t.P;
  const int32_t* from = p.t.bt + (int64_t)rec.parent * p.t.maxp;
  if (blockIdx.y == 0) {
    int32_t* row = p.t.bt + (int64_t)rec.child * p.t.maxp;
    for (int j = threadIdx.x; j < p.t.maxp; j += blockDim.x) {
      int pg = -1;
      if (j < full) {
        pg = from[j];
        if (pg < 0 || pg >= p.t.num_pages)
          raise_error(kErrTable);  // handed on as it is: readers skip it and say so again
        else
          atomicAdd(p.t.ref + pg, 1);
      } else if (j == full && tail > 0) {
        pg = rec.fresh;
        p.t.ref[pg] = 1;
      }
      row[j] = pg;
    }
    if (threadIdx.x == 0) p.t.sl[rec.child] = rec.len;
    return;
  }
  const int layer = (blockIdx.y - 1) / p.g.cpp, part = (blockIdx.y - 1) - layer * p.g.cpp;
  const int t0 = part * p.g.tps, v = min(p.g.tps, tail - t0);
  if (v > 0) move_page<VEC>(p.g, p.g.pool + (int64_t)layer * p.g.S_layer, from[full], rec.fresh, t0, v);
}

// ---- compact ------------------------------------------------------------------------------------
struct CompactParams {
  PageTables t;
  TablesCopyParams copy;
  int blocks;       // CTAs that plan; the others copy the tables
  int32_t* code;    // workspace [num_pages]: -1 free, p stays, -2 - k moves to holes[k]
  int32_t* holes;   // workspace [num_pages / 2 + 1]: free pages below the number in use, ascending
  int32_t* movers;  // workspace [num_pages / 2 + 1]: pages in use at or above it, ascending
  int32_t* moves;   // workspace [1]
  int32_t* num_used;
  int32_t* map;
};
// Every CTA counts the pages in use itself (the reference counts of even a large pool sit in L2:
// 4 bytes a page), then places the pages of its own block of 4,096.
__global__ void __launch_bounds__(kPlanThreads) topkv_compact_plan_kernel(const CompactParams p) {
  __shared__ int s_scan[33];
  pdl_prologue(0);
  if (blockIdx.x >= p.blocks) {
    copy_tables(p.copy, blockIdx.x - p.blocks, gridDim.x - p.blocks);
    return;
  }
  const int32_t* ref = p.copy.src[2];
  const int tid = threadIdx.x, N = p.t.num_pages;
  constexpr int kBlock = kPlanThreads * kPlanPages;
  const int mine = blockIdx.x * kBlock;
  int n = 0;
  bool u[kPlanPages];
  const int64_t p0 = (int64_t)mine + (int64_t)tid * kPlanPages;
#pragma unroll
  for (int k = 0; k < kPlanPages; ++k) {
    u[k] = p0 + k < N && ref[p0 + k] > 0;
    n += u[k];
  }
  int used, used_before = 0, used_low;  // pages in use: all, before this block, and those that stay
  int rank = block_exclusive_sum(n, s_scan, &used);
  int low = 0;
  if (p.blocks == 1) {  // the block is the pool
#pragma unroll
    for (int k = 0; k < kPlanPages; ++k) low += u[k] && p0 + k < used;
  } else {
    int all = 0, before = 0;
    for (int64_t i = tid; i < N; i += kPlanThreads) {
      const int v = ref[i] > 0;
      all += v;
      before += i < mine ? v : 0;
    }
    block_exclusive_sum(all, s_scan, &used);
    block_exclusive_sum(before, s_scan, &used_before);
    for (int i = tid; i < used; i += kPlanThreads) low += ref[i] > 0;
  }
  block_exclusive_sum(low, s_scan, &used_low);
  rank += used_before;  // pages in use below p0
#pragma unroll
  for (int k = 0; k < kPlanPages; ++k) {
    const int64_t pg = p0 + k;
    if (pg >= N) break;
    int code = -1;
    if (u[k]) {
      code = (int)pg;
      if (pg >= used) {
        code = -2 - (rank - used_low);
        p.movers[rank - used_low] = (int)pg;
      }
    } else if (pg < used) {
      p.holes[pg - rank] = (int)pg;
    }
    p.code[pg] = code;
    rank += u[k];
  }
  if (blockIdx.x == 0 && tid == 0) {
    *p.num_used = used;
    *p.moves = used - used_low;
  }
}
// The move itself, and the tables after it: new page ids in the rows, the reference counts beside
// their pages, the map. Sources lie at or above the number of pages in use and destinations below
// it, so no page is both; every table entry is read and written by one thread only.
template <int VEC>
__global__ void __launch_bounds__(kMoveThreads, 3) topkv_compact_apply_kernel(const CompactParams p, const PageGeom g) {
  pdl_prologue(0);
  const int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  const int moves = *p.moves;
  move_pages<VEC>(g, p.movers, p.holes, moves, p.t.num_pages);
  for (int64_t i = t; i < (int64_t)p.t.R * p.t.maxp; i += step) {
    const int r = (int)(i / p.t.maxp), j = (int)(i - (int64_t)r * p.t.maxp);
    const int len = p.t.sl[r];
    if (len < 0 || len > (int64_t)p.t.maxp * p.t.P) {
      if (j == 0) raise_error(kErrTable);
    }
    if (len <= 0 || j >= ceil_div(len, p.t.P)) continue;
    const int pg = p.t.bt[i];
    const int code = pg >= 0 && pg < p.t.num_pages ? p.code[pg] : -1;
    if (code == -1)
      raise_error(kErrTable);  // outside the pool, or a page that nobody is said to use
    else if (code <= -2)
      p.t.bt[i] = p.holes[-2 - code];
  }
  for (int64_t k = t; k < moves; k += step) {
    const int from = p.movers[k], to = p.holes[k];
    p.t.ref[to] = p.t.ref[from];
    p.t.ref[from] = 0;
  }
  for (int64_t i = t; i < p.t.num_pages; i += step) {
    const int code = p.code[i];
    p.map[i] = code <= -2 ? p.holes[-2 - code] : code;
  }
}

}  // namespace topkv

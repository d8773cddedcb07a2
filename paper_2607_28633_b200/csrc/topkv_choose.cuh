// Which pages a query looks at: bounds of each page's keys in 8 bits, and the choice of the pages that can
// score highest.
//
//   step = max |K| c, c = 1/127    lo[d] = floor(min K[d] / step)    hi[d] = ceil(max K[d] / step)
//   t = max |q| c                  q8[d] = rint(q[d] / t)
//   score = max over the heads of (sum_d q8[d] < 0 ? q8[d] lo[d] : q8[d] hi[d]) * (t * step)
//
// The sum is of whole numbers, and what is left are two roundings, so the choice does not depend on any order
// of summation. With q8 split into its negative and its positive part the sum is one product over 2 D
// elements, [negative | positive] . [lo | hi], formed four 8-bit products and sums at an instruction; four threads
// share a page, 16 consecutive bytes each at a time. (The warp-wide matrix instruction for 8-bit integers is
// no help: 100 cycles each, 26,000 for 1,024 pages a CTA.)
//
// What bounds it: the bounds, 2 D + 4 bytes a page and head (1/32 of a cache of 16-token pages), read once; in
// small calls the chain table -> bounds -> keys -> three passes over the keys -> list.
// A cluster of 1 to 8 CTAs has one request and KV head, each CTA an equal share of its pages. The keys go to the
// first CTA's shared memory, which then selects alone (a pass of the whole cluster takes 1.5 us for its barrier and
// the remote histograms); where they are more than it holds, each keeps its own, and histograms and counts are
// added up through the cluster's shared memory.
// Measured: 4 requests of 65,537 to 131,071 tokens, 128 of up to 8,192 pages a head, 8 x 4 heads of 128: 28 us here, of
// which the bounds are read at 5.4 TB/s in 10 and the selection takes 8, attention over the chosen 34 MB 16, its join 4: 49
// with both calls; two of 2,000 to 3,001 tokens 17 us, the calls (24 in a table of 65,536 columns, where the keys stay with
// their CTAs).
#pragma once
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <cfloat>
#include <cstdint>

#include "topkv_append.cuh"
#include "topkv_attend.cuh"
#include "topkv_common.cuh"

namespace topkv {

constexpr float k127th = 1.f / 127.f;

// ---- bounds ---------------------------------------------------------------------------------------
constexpr int kBoundThreads = 256;
struct BoundParams {
  const uint8_t* pool;  // this layer's slab
  const int32_t* bt;
  const int32_t* sl;
  int8_t* bounds;       // [pages][H][2][D]
  float* steps;         // [pages][H]
  int64_t S_page, S_tok, S_head;
  int64_t num_pages;
  uint32_t items;       // R * columns * H
  int maxp, P;
  uint32_t H;
  int D;
  int window;
  uint32_t columns;          // that the window can touch
};
// Pairs of 16-bit values; 8-bit ones are held as fp16, exactly. NaN wins.
template <bool BF16>
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
  uint32_t d;
  if constexpr (BF16) asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("min.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <bool BF16>
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t d;
  if constexpr (BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <bool BF16>
__device__ __forceinline__ float2 both(uint32_t v) {
  if constexpr (BF16) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  else return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
// A warp per page and head: lanes over the 16-byte chunks of a key, groups of them over the tokens. Minima and
// maxima stay in 16 bits, two to an instruction, which leaves registers for four CTAs of eight warps an SM with eight
// accesses under way each. What bounds it besides memory: the conversions and divisions, 59 % of the issue slots.
// Measured: 77 MB of keys of 16 requests of 512 to 4,096 tokens, 8 heads of 128, bf16: 22 us, 3.5 TB/s (25 with each
// lane's divisions its own, 32 with 32-bit extremes, 69 with a warp that walks over four pages).
template <int TYPE>
__global__ void __launch_bounds__(kBoundThreads, TYPE == kE4m3 ? 3 : 4) topkv_bound_pages_kernel(const BoundParams p) {
  constexpr bool kBf = TYPE == kBf16;
  constexpr int N = TYPE == kE4m3 ? 16 : 8, kPairs = N / 2;  // elements of 16 bytes
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  const int lane = threadIdx.x & 31;
  const uint32_t item = blockIdx.x * (kBoundThreads / 32) + (threadIdx.x >> 5);
  if (item >= p.items) return;
  const uint32_t at = item / p.H;
  const int h = (int)(item - at * p.H), r = (int)(at / p.columns), column = (int)(at - (uint32_t)r * p.columns);
  const int32_t* bt_row = p.bt + (int64_t)r * p.maxp;
  int page = p.window > 0 ? 0 : bt_row[column];  // under way beside the length
  int s = p.sl[r];
  const int64_t row = (int64_t)p.maxp * p.P;
  if (s < 0 || s > row) {
    if (lane == 0) raise_error(kErrTable);
    s = s < 0 ? 0 : (int)row;
  }
  const int j = (p.window > 0 ? max(s - p.window, 0) / p.P : 0) + column;
  if ((int64_t)j * p.P >= s) return;
  if (p.window > 0) page = bt_row[j];
  const int held = min(p.P, s - j * p.P);
  if (page < 0 || page >= p.num_pages) {
    if (lane == 0) raise_error(kErrTable);
    return;
  }
  const int chunks = p.D / N, groups = 32 / chunks, group = lane / chunks, c = lane - group * chunks;
  const uint8_t* src = p.pool + (int64_t)page * p.S_page + (int64_t)h * p.S_head + c * 16;
  uint32_t lo[kPairs], hi[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    lo[i] = kBf ? 0x7f807f80u : 0x7c007c00u;  // infinity
    hi[i] = kBf ? 0xff80ff80u : 0xfc00fc00u;
  }
  auto take = [&](int i, uint32_t v) {
    lo[i] = min2<kBf>(lo[i], v);
    hi[i] = max2<kBf>(hi[i], v);
  };
  if (group < groups) {
    constexpr int kAhead = 8;
    for (int t = group; t < held; t += groups * kAhead) {
      uint4 v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (t + u * groups < held) v[u] = *reinterpret_cast<const uint4*>(src + (int64_t)(t + u * groups) * p.S_tok);
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (t + u * groups >= held) continue;
        const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (TYPE == kE4m3) {
            uint32_t x, y;
            e4m3x4_to_f16(w[i], &x, &y);
            take(2 * i, x);
            take(2 * i + 1, y);
          } else {
            take(i, w[i]);
          }
        }
      }
    }
  }
  for (int k = 0; k < groups; ++k) {  // all groups' into each
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      const uint32_t a = __shfl_sync(0xffffffffu, lo[i], (c + k * chunks) & 31), b = __shfl_sync(0xffffffffu, hi[i], (c + k * chunks) & 31);
      lo[i] = min2<kBf>(lo[i], a);
      hi[i] = max2<kBf>(hi[i], b);
    }
  }
  float most = 0.f;
  bool nan = false;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const float2 a = both<kBf>(lo[i]), b = both<kBf>(hi[i]);
    if (group == 0) {
      most = fmaxf(most, fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(b.x), fabsf(b.y))));
      nan |= a.x != a.x || a.y != a.y;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
  if (__any_sync(0xffffffffu, nan)) most = NAN;
  const float step = __fmul_rn(most, k127th);
  const bool usable = step > 0.f && step < INFINITY;
  const int64_t to = (int64_t)page * p.H + h;
  if (lane == 0) p.steps[to] = step;
  // The first group divides the minima, the second the maxima (their negatives, rounded down as well): divisions are
  // most of what this kernel computes.
#pragma unroll 1
  for (int e = group; group < groups && e < 2; e += groups) {
    const float sign = e == 0 ? 1.f : -1.f;
    uint32_t w[N / 4] = {};
    if (usable) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 a = both<kBf>(e == 0 ? lo[i] : hi[i]);
        auto whole = [&](float x) { return (uint32_t)((int)(sign * fminf(fmaxf(floorf(__fdiv_rn(sign * x, step)), -127.f), 127.f)) & 255); };
        w[i / 2] |= (whole(a.x) | whole(a.y) << 8) << (i % 2 * 16);
      }
    }
    int8_t* out = p.bounds + (to * 2 + e) * p.D + c * N;
    if constexpr (N == 16)
      *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
    else
      *reinterpret_cast<uint2*>(out) = make_uint2(w[0], w[1]);
  }
}

// ---- choice ---------------------------------------------------------------------------------------
constexpr int kChooseThreads = 256;
constexpr int kChooseWarps = kChooseThreads / 32;
constexpr int kChooseCluster = 8;
struct ChooseParams {
  const int32_t* bt;
  const int32_t* sl;
  const uint8_t* q;
  const int8_t* bounds;
  const float* steps;
  int32_t* chosen;
  uint32_t* keys;       // workspace [R][H][maxp], or nullptr: they fit in shared memory
  int64_t q_req, q_head;
  int64_t num_pages;
  int maxp, P, H, G, D;
  int budget, firsts, lasts;
  int pitch;            // bytes of a head's queries in shared memory
};
// Rising floats as rising unsigned numbers.
__device__ __forceinline__ uint32_t score_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr int kChooseBits = 8, kChooseBins = 1 << kChooseBits;
constexpr int kGatherKeys = 24 * 1024;  // pages of a request up to which one CTA of the cluster selects
struct ChooseShared {
  uint32_t histogram[2][kChooseBins];
  uint32_t range[2];                 // the smallest and the largest key
  uint32_t count[2];                 // pages above the threshold, pages at it, of this CTA
  uint32_t sum[2][kChooseWarps];
  uint32_t found[2];                 // the pass's digit, and how many of its pages are still wanted
};

// Dynamic shared memory: q8 [heads][pitch], t [heads], keys.
template <int DP, bool BF16, bool GATHER>
__global__ void __launch_bounds__(kChooseThreads, 2) topkv_choose_pages_kernel(const ChooseParams p) {
  namespace cg = cooperative_groups;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ ChooseShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  int ctas = (int)cluster.num_blocks();
  const int rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int unit = blockIdx.x / ctas, r = unit / p.H, h = unit - r * p.H;
  const int heads = p.G;
  float* const s_t = reinterpret_cast<float*>(smem + heads * p.pitch);
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  int s = p.sl[r];
  const int64_t row = (int64_t)p.maxp * p.P;
  if (s < 0 || s > row) {
    if (tid == 0 && h == 0) raise_error(kErrTable);
    s = s < 0 ? 0 : (int)row;
  }
  const int pages = s / p.P + (s % p.P != 0);
  int32_t* const out = p.chosen + (int64_t)unit * p.budget;
  const int listed = min(pages, p.budget);
  for (int i = listed + rank * kChooseThreads + tid; i < p.budget; i += ctas * kChooseThreads) out[i] = -1;
  if (pages <= p.budget) {  // all of them; every CTA of the cluster comes here
    for (int i = rank * kChooseThreads + tid; i < pages; i += ctas * kChooseThreads) out[i] = i;
    return;
  }
  const int lasts = min(p.lasts, p.budget), firsts = min(p.firsts, p.budget - lasts);
  const int wanted = p.budget - lasts - firsts, end = pages - lasts;  // of the pages firsts .. end - 1
  if (rank == 0) {
    for (int i = tid; i < firsts; i += kChooseThreads) out[i] = i;
    for (int i = tid; i < lasts; i += kChooseThreads) out[p.budget - lasts + i] = end + i;
  }
  if (wanted == 0) return;
  // this CTA's pages
  const int each = ((end - firsts + ctas - 1) / ctas + 7) / 8 * 8;
  int j0 = min(firsts + rank * each, end), n = min(each, end - j0);
  const int32_t* bt_row = p.bt + (int64_t)r * p.maxp + j0;
  uint32_t* keys = p.keys != nullptr ? p.keys + (int64_t)unit * p.maxp + j0 : reinterpret_cast<uint32_t*>(smem + heads * (p.pitch + 4));
  for (int i = tid; i < kChooseBins; i += kChooseThreads) sh.histogram[0][i] = sh.histogram[1][i] = 0;
  if (tid == 0) {
    sh.range[0] = 0xffffffffu;
    sh.range[1] = 0;
  }
  uint32_t* range = sh.range;
  if (GATHER && ctas > 1) {  // keys go to the first CTA, which has to have begun
    cluster.sync();
    keys = cluster.map_shared_rank(keys, 0) + (j0 - firsts);
    range = cluster.map_shared_rank(range, 0);
  }
  // A warp has kAhead groups of eight pages under way at a time, the first ones while the queries are made.
  constexpr int kSets = DP / 32;  // four 16-byte chunks each, of 2 D bytes
  constexpr int kAhead = 16 / kSets < 4 ? 16 / kSets : 4;
  constexpr int kHop = kChooseWarps * 8 * kAhead;
  const int gr = lane >> 2, gc = lane & 3;
  const int chunks = p.D / 8;  // of 16 bytes, of 2 D bytes
  int page[kAhead];
  uint4 v[kAhead][kSets];
  float step[kAhead];
  auto pages_of = [&](int i) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) page[u] = i + u * 8 + gr < n ? bt_row[i + u * 8 + gr] : -1;
  };
  auto bring = [&](int i) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const bool ok = page[u] >= 0 && page[u] < p.num_pages;
      if (!ok && i + u * 8 + gr < n && gc == 0) raise_error(kErrTable);
      const int64_t at = (int64_t)(ok ? page[u] : 0) * p.H + h;
      step[u] = ok ? p.steps[at] : 0.f;
      const int8_t* from = p.bounds + at * 2 * p.D + gc * 16;
#pragma unroll
      for (int k = 0; k < kSets; ++k) {
        v[u][k] = make_uint4(0, 0, 0, 0);
        if (ok && k * 4 + gc < chunks) v[u][k] = *reinterpret_cast<const uint4*>(from + k * 64);
      }
    }
  };
  const int i_first = warp * 8 * kAhead;
  pages_of(i_first);
  bring(i_first);
  pages_of(i_first + kHop);

  // ---- the queries in 8 bits, negative part before positive part ------------------------------------
  for (int g = warp; g < heads; g += kChooseWarps) {
    uint8_t* to = smem + g * p.pitch;
    const uint8_t* src = p.q + r * p.q_req + ((int64_t)h * p.G + g) * p.q_head;
    float x[8], most = 0.f;
    bool nan = false;
    const bool mine = g < p.G && lane < p.D / 8;  // D is at most 256
    if (mine) {
      unpack8<BF16>(*reinterpret_cast<const uint4*>(src + lane * 16), x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        most = fmaxf(most, fabsf(x[i]));
        nan |= x[i] != x[i];
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
    float t = __fmul_rn(most, k127th);
    if (__any_sync(0xffffffffu, nan) || !(t > 0.f && t < INFINITY)) t = 0.f;
    if (lane == 0) s_t[g] = t;
    uint32_t neg[2] = {0, 0}, pos[2] = {0, 0};
    if (mine && t > 0.f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int v = (int)fminf(fmaxf(rintf(__fdiv_rn(x[i], t)), -127.f), 127.f);
        neg[i / 4] |= (uint32_t)(min(v, 0) & 255) << (i % 4 * 8);
        pos[i / 4] |= (uint32_t)(max(v, 0) & 255) << (i % 4 * 8);
      }
    }
    if (lane < p.D / 8) {
      *reinterpret_cast<uint2*>(to + lane * 8) = make_uint2(neg[0], neg[1]);
      *reinterpret_cast<uint2*>(to + p.D + lane * 8) = make_uint2(pos[0], pos[1]);
    }
    for (int i = 2 * p.D + lane * 8; i < kSets * 64; i += 32 * 8) *reinterpret_cast<uint2*>(to + i) = make_uint2(0, 0);
  }
  __syncthreads();

  // ---- scores: a warp takes eight pages at a time ----------------------------------------------------
  uint32_t least = 0xffffffffu, most = 0;
#pragma unroll 1
  for (int i0 = i_first; i0 < n; i0 += kHop) {
    float best[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) best[u] = -INFINITY;
#pragma unroll 1
    for (int g = 0; g < heads; ++g) {
      int dot[kAhead] = {};
      const uint8_t* from = smem + g * p.pitch + gc * 16;
#pragma unroll
      for (int k = 0; k < kSets; ++k) {
        const uint4 q = *reinterpret_cast<const uint4*>(from + k * 64);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          dot[u] = __dp4a((int)v[u][k].x, (int)q.x, dot[u]);
          dot[u] = __dp4a((int)v[u][k].y, (int)q.y, dot[u]);
          dot[u] = __dp4a((int)v[u][k].z, (int)q.z, dot[u]);
          dot[u] = __dp4a((int)v[u][k].w, (int)q.w, dot[u]);
        }
      }
      const float t = s_t[g];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        dot[u] += __shfl_xor_sync(0xffffffffu, dot[u], 1);
        dot[u] += __shfl_xor_sync(0xffffffffu, dot[u], 2);
        // kept finite, so that a sum of 0 stays 0
        best[u] = fmaxf(best[u], __fmul_rn((float)dot[u], fminf(__fmul_rn(t, step[u]), FLT_MAX)));
      }
    }
    if (gc == 0) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int j = i0 + u * 8 + gr;
        if (j < n) {
          // infinity without a finite step, as a score that has left the range is: such pages are equal
          const uint32_t key = score_key(step[u] < INFINITY ? __fadd_rn(best[u], 0.f) : INFINITY);
          keys[j] = key;
          least = min(least, key);
          most = max(most, key);
        }
      }
    }
    if (i0 + kHop < n) {
      bring(i0 + kHop);
      pages_of(i0 + 2 * kHop);
    }
  }
  least = __reduce_min_sync(0xffffffffu, least);
  most = __reduce_max_sync(0xffffffffu, most);
  if (lane == 0) {
    atomicMin(range, least);
    atomicMax(range + 1, most);
  }
  if (ctas > 1) cluster.sync(); else __syncthreads();
  if (GATHER && ctas > 1) {
    if (rank > 0) return;
    ctas = 1;
    j0 = firsts;
    n = end - firsts;
    keys = reinterpret_cast<uint32_t*>(smem + heads * (p.pitch + 4));
  }

  // ---- the key of the last page that is taken, kChooseBits bits a pass --------------------------------
  // The first pass begins at the highest bit in which keys differ, so that they spread over its bins.
  least = sh.range[0];
  most = sh.range[1];
  for (int k = 0; k < ctas && ctas > 1; ++k) {
    const uint32_t* there = cluster.map_shared_rank(sh.range, k);
    least = min(least, there[0]);
    most = max(most, there[1]);
  }
  int top = 32 - __clz((int)(least ^ most));  // bits below `top` are not known yet
  uint32_t prefix = top < 32 ? most >> top << top : 0, need = (uint32_t)wanted;
#pragma unroll 1
  for (int b = 0; top > 0; b ^= 1) {
    const int shift = max(top - kChooseBits, 0);
    const uint32_t digits = (1u << (top - shift)) - 1;
#pragma unroll 8
    for (int i = tid; i < n; i += kChooseThreads) {
      const uint32_t key = keys[i];
      if (top == 32 || (key ^ prefix) >> top == 0) atomicAdd(&sh.histogram[b][key >> shift & digits], 1u);
    }
    if (ctas > 1) cluster.sync(); else __syncthreads();
    // the whole cluster's histogram, a few bins a thread from the highest down, and how many pages lie above them
    constexpr int kBins = kChooseBins / kChooseThreads;
    const int bin0 = kChooseBins - 1 - tid * kBins;
    uint32_t bin[kBins] = {}, mine = 0;
    for (int k = 0; k < ctas; ++k) {
      const uint32_t* there = ctas > 1 ? cluster.map_shared_rank(sh.histogram[b], k) : sh.histogram[b];
#pragma unroll
      for (int i = 0; i < kBins; ++i) bin[i] += there[bin0 - i];
    }
#pragma unroll
    for (int i = 0; i < kBins; ++i) mine += bin[i];
    uint32_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) sh.sum[0][warp] = incl;
    // the other buffer: read by all before the barrier above, filled behind the one below
#pragma unroll
    for (int i = 0; i < kBins; ++i) sh.histogram[b ^ 1][tid + i * kChooseThreads] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kChooseWarps; ++w)
      if (w < warp) incl += sh.sum[0][w];
    uint32_t above = incl - mine;
    if (incl >= need && above < need) {  // exactly one thread
#pragma unroll
      for (int i = 0; i < kBins; ++i) {
        if (above < need && above + bin[i] >= need) {
          sh.found[0] = bin0 - i;
          sh.found[1] = need - above;
          above = need;  // none of the bins below
        } else {
          above += bin[i];
        }
      }
    }
    __syncthreads();
    prefix |= sh.found[0] << shift;
    need = sh.found[1];
    top = shift;
  }

  // ---- the list: pages above that key, and the first `need` at it, in order of their columns ------------
  const int per = (n + kChooseThreads - 1) / kChooseThreads | 1;  // odd: the threads' runs begin in different banks
  const int i0 = min(tid * per, n), i1 = min(i0 + per, n);
  // which of up to 32 keys from i on are above, which at the threshold
  auto look = [&](int i, uint32_t* above, uint32_t* at) {
    *above = *at = 0;
#pragma unroll 8
    for (int k = 0; k < 32; ++k) {
      if (i + k >= i1) break;
      const uint32_t key = keys[i + k];
      *above |= (uint32_t)(key > prefix) << k;
      *at |= (uint32_t)(key == prefix) << k;
    }
  };
  uint32_t mine[2] = {0, 0}, seen[2] = {0, 0};
  for (int i = i0; i < i1; i += 32) {
    look(i, &seen[0], &seen[1]);
    mine[0] += __popc(seen[0]);
    mine[1] += __popc(seen[1]);
  }
  uint32_t incl[2] = {mine[0], mine[1]};
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t up = __shfl_up_sync(0xffffffffu, incl[k], o);
      if (lane >= o) incl[k] += up;
    }
  if (lane == 31) {
    sh.sum[0][warp] = incl[0];
    sh.sum[1][warp] = incl[1];
  }
  __syncthreads();
  uint32_t before[2] = {incl[0] - mine[0], incl[1] - mine[1]}, total[2] = {0, 0};
#pragma unroll
  for (int w = 0; w < kChooseWarps; ++w)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (w < warp) before[k] += sh.sum[k][w];
      total[k] += sh.sum[k][w];
    }
  if (ctas > 1) {
    if (tid < 2) sh.count[tid] = total[tid];
    cluster.sync();
    for (int k = 0; k < rank; ++k) {
      const uint32_t* there = cluster.map_shared_rank(sh.count, k);
      before[0] += there[0];
      before[1] += there[1];
    }
    cluster.sync();  // nobody leaves while its counts are read
  }
  for (int i = i0; i < i1; i += 32) {
    if (i1 - i0 > 32) look(i, &seen[0], &seen[1]);
    for (uint32_t any = seen[0] | seen[1]; any != 0; any &= any - 1) {
      const int k = __ffs(any) - 1;
      const bool above = seen[0] >> k & 1;
      if (above || before[1] < need) out[firsts + before[0] + min(before[1], need)] = j0 + i + k;
      before[0] += above;
      before[1] += !above;
    }
  }
}

}  // namespace topkv

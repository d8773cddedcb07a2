// Attention of one new token per request over one layer of a paged cache with K and V planes.
//
//   x_i = scale * k_scale * q . K[i]      m = max x_i      l = sum exp(x_i - m)
//   out = v_scale * sum exp(x_i - m) V[i] / l              lse = m + ln l
// over the visible tokens i of the request. A window with first tokens that stay visible leaves two
// ranges, [0, ns) and [lo, s): the kernel numbers the visible tokens 0 .. n-1 straight through, so
// nothing that is masked is ever loaded, and a NaN left behind there cannot reach the result.
//
// What bounds it: every K and V byte is read once and used for G query heads, 2 G flops a byte at 16
// bits, so for the usual G <= 16 it is memory, far below the tensor rate; the matrix instructions
// are warp-wide m16n8k16 ones with the G query heads as rows (padded to 16), which need no shared
// staging of accumulators and keep the tensor pipe 14 % busy. Measured: 16 x 16,384 tokens, 8 KV heads of
// 128 in bf16, 176 us = 6.1 TB/s (0.93 of the measured copy); 16 x 512 to 4,096, 34 us, of which the
// 148 MB take 22.6, the start 2, the spread between the CTAs 4 and the join 4. Layout of the work:
//  * a CTA has 4 warps and one KV head; each warp takes its own 16 tokens of every 64 and runs its
//    own ring of cp.async stages, running maximum and sum, so the loop has no CTA barrier at all;
//  * the visible tokens of all requests, cut into tiles of 64, are shared out evenly between
//    `teams` of CTAs (one CTA per KV head and group of 16 query heads in a team, so that a team
//    reads whole token rows at about the same time), whatever the lengths: a long request is
//    split between teams, and several short ones may fall to one;
//  * a request that lies inside one team is finished by it. Of one that is cut, each team leaves
//    its (m, l, sum) in the workspace and topkv_attend_join_kernel joins the parts in their
//    order, so the result does not depend on which CTA ran when.
//  * many more short requests than CTAs fit at a time take a warp each: no cut, and nothing to join.
// Scores, maxima, sums and the accumulated values are 32-bit; the weights exp(x - m) are rounded to
// the 16-bit type of the values for the second product (to fp16 for an 8-bit cache): half a step of
// 2^-8 (bf16) or 2^-11 of each weight, which averages out over the tokens and stays at or below the
// rounding of the output; for bf16 up to 128 columns the rest of each weight is multiplied too.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "topkv_bulk.cuh"
#include "topkv_common.cuh"

namespace topkv {

constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = kAttendWarps * 32;
constexpr int kWarpTokens = 16;
constexpr int kTileTokens = kAttendWarps * kWarpTokens;
constexpr int kAttendRows = 16;      // query heads per CTA (rows of the matrix instruction)
constexpr int kUncutTiles = 4;       // requests of at most this many tiles are not cut
constexpr float kLazy = 8.f;         // a running maximum moves when it is exceeded by more than this (powers of two)
// Sum of a part none of whose tokens counted (their pages are outside the pool). A sum of zero will not do:
// tokens that count and score minus infinity have that one, and their result is not zero but 0 / 0.
constexpr float kNoneSeen = -1.f;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

enum AttendType { kBf16 = 1, kFp16 = 2, kE4m3 = 3 };

struct AttendParams {
  const uint8_t* pool;  // this layer's slab
  const int32_t* bt;
  const int32_t* sl;
  const uint8_t* q;
  uint8_t* out;
  float* lse;           // [R][Hq] or nullptr
  int64_t S_page, S_kv, S_tok, S_head;
  int64_t q_req, q_head, o_req, o_head;  // bytes
  int64_t num_pages;
  int R, maxp, P;
  int page_shift;       // log2 of P, or -1 if P is no power of two
  int H, G, gtiles;     // KV heads, query heads per KV head, groups of row_tile query heads per KV head
  int D, Dv;            // elements
  int window, sinks;
  float qk_scale;       // scale * k_scale * log2(e): scores are kept in powers of two
  float v_scale;
  int io_bf16;
  int teams;            // CTAs along x
  int uncut;            // 1: team t is request t
  int narrow;           // 1 (uncut only): a warp has a request to itself, team t the requests 4 t .. 4 t + 3
  int by_request;       // how the join records are indexed
  int start_cost;       // of a request, in tiles
  int late_wait;        // tables are settled
  int box;              // latent rows: tokens of a tensor copy (divides the page and 64), 0 = none are used
  int q_box;            // latent rows: 1 = Q comes by tensor copies too
  int rows;             // rows of a partial result, min(G, row_tile)
  int row_tile;         // query heads per CTA
  // workspace
  int4* joins;          // which requests were cut, see JoinRecord: [R] if by_request, else [teams]
  float2* ml;           // [teams][2][H * gtiles][rows]
  float* part;          // [teams][2][H * gtiles][rows][Dv]
};

// Visible tokens of a request: 0 .. n-1 stand for tokens 0 .. ns-1 and lo, lo+1, ..
struct Visible {
  int n, ns, lo;
};
__device__ __forceinline__ Visible visible_tokens(const AttendParams& p, int r, bool complain) {
  int s = p.sl[r];
  const int64_t row = (int64_t)p.maxp * p.P;
  if (s < 0 || s > row) {
    if (complain) raise_error(kErrTable);
    s = s < 0 ? 0 : (int)row;
  }
  Visible v;
  v.lo = p.window > 0 ? max(s - p.window, 0) : 0;
  v.ns = min(p.sinks, v.lo);
  v.n = v.ns + s - v.lo;
  return v;
}
__device__ __forceinline__ int attend_tiles(int n) { return n / kTileTokens + (n % kTileTokens != 0); }

// Which tiles are a team's. The requests are laid end to end, each `p.start_cost` + its tiles long (what
// it costs to begin with a request and to write its result, in tiles; an empty one 0), and cut into
// ranges of equal length; a range has the tiles that lie in it. In an uncut launch team t takes request
// t. Every CTA works it out from the lengths.
struct TeamRange {
  int r;          // first request
  int64_t off;    // where in it the range begins
  int64_t left;   // length of the range (uncut: the request)
};
struct TeamStart {  // in shared memory
  int64_t scan[16];
  int64_t pos;    // the range's start
  int64_t off;
  int64_t each;   // length of a range ...
  int more;       // ... and how many ranges are one longer
  int r;
};
// The tiles [t0, t1) of a request of n tiles that a range has which begins `off` into it and is `left` long;
// the return value is how much of the range the request takes.
__device__ __forceinline__ int64_t tiles_in_range(const AttendParams& p, int n, int64_t off, int64_t left, int* t0, int* t1) {
  const int c = p.uncut ? 0 : p.start_cost;
  const int64_t end = min(off + left, (int64_t)c + n);
  *t0 = (int)max(off - c, (int64_t)0);
  *t1 = (int)max(end - c, (int64_t)0);
  return end - off;
}
// The team whose range holds position x.
__device__ __forceinline__ int team_of(const TeamStart& t, int64_t x) {
  const int64_t wide = t.more * (t.each + 1);
  return x < wide ? (int)(x / (t.each + 1)) : t.more + (int)((x - wide) / t.each);
}
template <int THREADS>
__device__ __forceinline__ TeamRange team_range(const AttendParams& p, int team, TeamStart* s) {
  TeamRange out = {team, 0, 0x7fffffff};
  if (p.uncut) return out;
  constexpr int kWarps = THREADS / 32;
  static_assert(kWarps <= 16, "scan holds 16 warps");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (p.R + THREADS - 1) / THREADS;
  const int r0 = (int)min((int64_t)tid * per, (int64_t)p.R), r1 = min(r0 + per, p.R);
  int64_t mine = 0;
  auto length = [&](int i) {
    const int n = attend_tiles(visible_tokens(p, i, false).n);
    return n > 0 ? n + p.start_cost : 0;
  };
  for (int i = r0; i < r1; ++i) mine += length(i);
  int64_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) s->scan[warp] = incl;
  if (tid == 0) s->r = -1;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) incl += s->scan[w];
    total += s->scan[w];
  }
  const int teams = (int)min((int64_t)p.teams, total);  // no range is empty
  int64_t a = 0, b = 0;
  if (team < teams) {
    const bool narrow = total <= 0xffffffffll;  // a 32-bit division where that will do
    const int64_t each = narrow ? (uint32_t)total / (uint32_t)teams : total / teams;
    const int more = (int)(total - each * teams);
    a = each * team + min(team, more);
    b = a + each + (team < more ? 1 : 0);
    if (tid == 0) {
      s->pos = a;
      s->each = each;
      s->more = more;
    }
  }
  if (a < b && a >= incl - mine && a < incl) {  // exactly one thread
    int64_t at = incl - mine;
    for (int i = r0; i < r1; ++i) {
      const int n = length(i);
      if (a < at + n) {
        s->r = i;
        s->off = a - at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  out.r = s->r;
  out.off = s->off;
  out.left = out.r < 0 ? 0 : b - a;
  return out;
}
// What the joining kernel needs to know of a request that does not end in the team that begins it: its
// number, that team, which of the team's segments it is (0 the first, else 1), and how many teams hold
// a part (0: nothing to join). Written by the team that begins the request, behind the wait for earlier
// kernels: the join of the call before reads the records until then. Indexed by team, a record says
// what holds for the last request that the team begins: no other can be cut.
__device__ __forceinline__ void write_join(const AttendParams& p, int r, int team, int slot, int parts) {
  p.joins[p.by_request ? r : team] = make_int4(r, team, slot, parts);
}
// `begin`: where the request begins, from the start of the team's range (before it, if negative).
__device__ __forceinline__ void request_begins(const AttendParams& p, const TeamStart& s, int team, int r, bool first, int64_t begin,
                                               int tiles, bool whole) {
  write_join(p, r, team, first ? 0 : 1, whole ? 0 : team_of(s, s.pos + begin + p.start_cost + tiles - 1) - team + 1);
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool valid) {
  const int n = valid ? 16 : 0;  // 0: nothing is read, the 16 bytes become zero
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
template <bool BF16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if constexpr (BF16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  } else {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
}
__device__ __forceinline__ void store_io(uint8_t* p, float v, bool bf16) {
  if (bf16)
    *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v);
  else
    *reinterpret_cast<__half*>(p) = __float2half_rn(v);
}
__device__ __forceinline__ void store_io4(uint8_t* p, const float4& v, float f, bool bf16) {
  const uint2 w = bf16 ? make_uint2(pack2<true>(v.x * f, v.y * f), pack2<true>(v.z * f, v.w * f))
                       : make_uint2(pack2<false>(v.x * f, v.y * f), pack2<false>(v.z * f, v.w * f));
  *reinterpret_cast<uint2*>(p) = w;
}
// Requests with nothing to see get zeros and a log-sum-exp of minus infinity, `rows` heads from head0. Every
// lane looks at one request of the team's share, a warp writes what it finds.
template <int THREADS>
__device__ __forceinline__ void empty_requests(const AttendParams& p, int team, int64_t head0, int rows, bool complain) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int64_t first = team + (int64_t)p.teams * 32 * warp; first < p.R; first += (int64_t)p.teams * THREADS) {
    const int64_t e = first + (int64_t)p.teams * lane;
    const bool empty = e < p.R && visible_tokens(p, (int)e, complain).n == 0;
    if (empty && complain && !p.uncut && p.by_request) write_join(p, (int)e, 0, 0, 0);
    for (uint32_t left = __ballot_sync(0xffffffffu, empty); left != 0; left &= left - 1) {
      const int64_t r = first + (int64_t)p.teams * (__ffs(left) - 1);
      for (int i = lane; i < rows * p.Dv; i += 32) {
        const int g = i / p.Dv, d = i - g * p.Dv;
        store_io(p.out + r * p.o_req + (head0 + g) * p.o_head + d * 2, 0.f, p.io_bf16);
      }
      if (p.lse != nullptr)
        for (int g = lane; g < rows; g += 32) p.lse[r * p.H * p.G + head0 + g] = -INFINITY;
    }
  }
}
// 2^x by the hardware's approximation (2 ulp; results below 2^-126 become 0).
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Four 8-bit values to two pairs of fp16 values; exact.
__device__ __forceinline__ void e4m3x4_to_f16(uint32_t v, uint32_t* lo, uint32_t* hi) {
  asm("{ .reg .b16 a, b; mov.b32 {a, b}, %2; cvt.rn.f16x2.e4m3x2 %0, a; cvt.rn.f16x2.e4m3x2 %1, b; }"
      : "=r"(*lo), "=r"(*hi)
      : "r"(v));
}
// Shared memory: per warp a ring of stages, each 16 rows of K and 16 rows of V of DP elements.
// Rows are swizzled in 16-byte chunks so that the eight rows of a matrix load hit all banks. Stages
// and registers are set for several CTAs per SM: a warp works through a tile in a chain of dependent
// steps, so it takes 12 to 16 warps an SM to keep enough loads in flight.
template <int DP, int TYPE>
struct AttendShape {
  static constexpr int kElem = TYPE == kE4m3 ? 1 : 2;
  static constexpr int kRow = DP * kElem;                    // bytes of a row
  static constexpr int kChunks = kRow / 16;
  static constexpr int kStage = 2 * kWarpTokens * kRow;      // K rows, then V rows
  static constexpr int kCtas = DP == 64 ? 4 : DP == 128 ? 3 : TYPE == kE4m3 ? 2 : 1;  // per SM
  static constexpr int kStages = (kCtas == 4 ? 12288 : kCtas == 3 ? 16384 : kCtas == 2 ? 24576 : 49152) / kStage;
  static constexpr int kSmem = kAttendWarps * kStages * kStage;
  static_assert(kSmem >= kAttendWarps * kAttendRows * (DP + 8 + 2) * 4, "the epilogue reuses the ring");
  static __device__ __forceinline__ uint32_t swizzle(int token, int chunk) {
    const int s = kChunks >= 8 ? (token & 7) : ((token >> 1) & 3);
    return (uint32_t)((chunk ^ s) << 4);
  }
};
__host__ __device__ inline int attend_ctas_per_sm(int D, int type) {
  return D <= 64 ? 4 : D <= 128 ? 3 : type == kE4m3 ? 2 : 1;
}

template <int DP, int TYPE>
__global__ void __launch_bounds__(kAttendThreads, AttendShape<DP, TYPE>::kCtas) topkv_attend_kernel(const AttendParams p) {
  using S = AttendShape<DP, TYPE>;
  constexpr bool kMmaBf16 = TYPE == kBf16;
  constexpr float kShift = kMmaBf16 ? 0.f : 7.f;
  // bf16 keeps 8 bits of a weight. What that cuts off is multiplied as well: the error against 64 bits falls
  // from 1.4 to 1.0 times that of the output's own rounding, for 1 to 2 % of the time while memory sets
  // the pace. At 256 columns, with a single CTA per SM, it would be 5 %: left out there.
  constexpr bool kSecond = kMmaBf16 && DP <= 128;
  constexpr int kSteps = DP / 16;  // k-steps of the first product, pairs of n-tiles of the second
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ TeamStart s_team;
  __shared__ uint32_t s_mask[kAttendWarps][AttendShape<DP, TYPE>::kStages];
  __shared__ int s_seen[kAttendWarps];  // kUsable: a token of the warp's share counted; narrow: kVisible as well
  constexpr int kUsable = 1, kVisible = 2;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int team = blockIdx.x, unit = blockIdx.y;  // unit: KV head and group of 16 query heads
  const int h = unit / p.gtiles, g0 = (unit - h * p.gtiles) * kAttendRows;
  const int rows = min(p.G - g0, kAttendRows);
  if (!p.late_wait) pdl_wait_prior_grid();
  pdl_release_next_grid();

  const TeamRange mine = team_range<kAttendThreads>(p, team, &s_team);
  if (p.late_wait) pdl_wait_prior_grid();
  const int64_t q_head0 = (int64_t)h * p.G + g0;
  empty_requests<kAttendThreads>(p, team, q_head0, rows, unit == 0);
  const bool records = !p.uncut && unit == 0 && tid == 0;
  if (records && !p.by_request) write_join(p, 0, team, 0, 0);
  if (mine.left == 0) return;

  uint8_t* ring = smem + warp * S::kStages * S::kStage;
  const uint32_t ring_a = smem_addr(ring);
  if (p.D < DP) {  // columns past the head dimension stay zero
    for (int i = lane; i < S::kStages * S::kStage / 16; i += 32)
      reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
    __syncwarp();
  }
  const int chunks = p.D * S::kElem / 16;
  const uint8_t* k_base = p.pool + (int64_t)h * p.S_head;
  int64_t left = mine.left, off = mine.off;
  int r = mine.r;
  const int gr = lane >> 2, gc = lane & 3;  // row and column group of this thread in a matrix fragment

  if (p.narrow) r = team * kAttendWarps + warp;  // may lie behind the last request: the warp only keeps step then
  // from a warp's tile to its next: the CTA's four warps share a request, or each has its own
  const int hop = p.narrow ? kWarpTokens : kTileTokens;

  for (bool first = true; left > 0 && (r < p.R || p.narrow); ++r) {
    Visible vis = {0, 0, 0};
    if (r < p.R) vis = visible_tokens(p, r, false);
    const int tiles = attend_tiles(vis.n);
    if (tiles == 0 && !p.narrow) {
      if (p.uncut) return;
      continue;
    }
    int t0, t1;
    const int64_t taken = tiles_in_range(p, tiles, off, left, &t0, &t1);
    if (records && t0 == 0 && t1 > 0) request_begins(p, s_team, team, r, first, mine.left - left - off, tiles, t1 == tiles);
    left -= taken;
    off = 0;
    if (t0 == t1 && !p.narrow) continue;

    // ---- the query rows as fragments ----------------------------------------------------------
    uint32_t qf[kSteps][4];
    float row_scale[2] = {p.qk_scale, p.qk_scale};
    {
      const uint8_t* qp = p.q + r * p.q_req + q_head0 * p.q_head;
      float top[2] = {0.f, 0.f};
      // For an 8-bit cache a thread's four consecutive elements take the places (2c, 2c+1, 2c+8, 2c+9)
      // of a k-step, in Q and in K alike: that is how four 8-bit values of K arrive in one register.
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int row = gr + (j & 1) * 8;
          const int col = k * 16 + (TYPE == kE4m3 ? gc * 4 + (j >> 1) * 2 : gc * 2 + (j >> 1) * 8);
          uint32_t v = 0;
          if (row < rows && col < p.D && vis.n > 0) v = *reinterpret_cast<const uint32_t*>(qp + row * p.q_head + col * 2);
          qf[k][j] = v;
          if (TYPE == kE4m3 && p.io_bf16)
            top[j & 1] = fmaxf(top[j & 1], fmaxf(fabsf(__uint_as_float(v << 16)), fabsf(__uint_as_float(v & 0xffff0000u))));
        }
      if (TYPE == kE4m3 && p.io_bf16) {
        // bf16 queries become fp16 ones: exact after a power of two per row, except for elements
        // below 2^-14 of the row's largest, which keep an absolute error of 2^-25 of it
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
          top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
          int e = 0;
          if (top[i] > 0.f && top[i] < INFINITY) e = ilogbf(top[i]);
          // in two steps: a single factor of 2^-e may itself leave the range of a float
          const float half_up = exp2f((float)(-(e / 2))), rest_up = exp2f((float)(-(e - e / 2)));
          row_scale[i] = p.qk_scale * exp2f((float)(e / 2)) * exp2f((float)(e - e / 2));
#pragma unroll
          for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if ((j & 1) == i) {
                const uint32_t v = qf[k][j];
                qf[k][j] = pack2<false>(__uint_as_float(v << 16) * half_up * rest_up,
                                        __uint_as_float(v & 0xffff0000u) * half_up * rest_up);
              }
        }
      }
    }

    float o[2 * kSteps][4];
#pragma unroll
    for (int i = 0; i < 2 * kSteps; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[i][j] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, base[2] = {0.f, 0.f};

    // ---- this warp's 16 tokens of every tile: visible tokens v .. v + 15, `hop` further each time ----
    const int end = t1 == tiles ? vis.n : t1 * kTileTokens;
    const int32_t* bt_row = p.bt + (int64_t)r * p.maxp;
    auto token = [&](int v) { return v < vis.ns ? v : v + (vis.lo - vis.ns); };
    auto page_column = [&](int i) { return p.page_shift >= 0 ? i >> p.page_shift : i / p.P; };
    // The page of the tile's first token, one tile ahead of its use.
    auto page_of = [&](int v) { return v < end ? bt_row[page_column(token(v))] : 0; };
    constexpr int kRows = 32 / S::kChunks;   // rows that one warp-wide copy brings
    static_assert(kRows >= 1, "a row is at most 512 bytes");
    constexpr int kCopies = kWarpTokens * S::kChunks / 32;
    const int my_row = lane / S::kChunks, my_chunk = lane % S::kChunks;
    uint32_t slow = 0;  // bit s: stage s holds a tile whose s_mask says which tokens count
    auto issue = [&](int stage, int v, int pg) {
      const uint32_t dst = ring_a + stage * S::kStage;
      if (v >= end) return;  // nothing left: the stage is not read
      const int i0 = token(v), x0 = i0 - page_column(i0) * p.P;
      if (v + kWarpTokens <= end && (v >= vis.ns || v + kWarpTokens <= vis.ns) && x0 + kWarpTokens <= p.P && pg >= 0 &&
          pg < p.num_pages) {
        // all 16 tokens follow each other in one page: rows at a constant stride
        const uint8_t* src = k_base + (int64_t)pg * p.S_page + (int64_t)(x0 + my_row) * p.S_tok + my_chunk * 16;
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          const int row = i * kRows + my_row;
          const uint32_t to = dst + row * S::kRow + S::swizzle(row, my_chunk);
          if (my_chunk < chunks) {
            cp_async16(to, src, true);
            cp_async16(to + kWarpTokens * S::kRow, src + p.S_kv, true);
          }
          src += kRows * p.S_tok;
        }
        slow &= ~(1u << stage);
        return;
      }
      // the end of a request, pages of fewer than 16 tokens, a tile across pages or across the gap of
      // a window, a page outside the pool: every row for itself
      int64_t off = -1;
      if (v + (lane & 15) < end) {
        const int i = token(v + (lane & 15)), j = page_column(i), page = bt_row[j];
        if (page < 0 || page >= p.num_pages)
          raise_error(kErrTable);
        else
          off = (int64_t)page * p.S_page + (int64_t)(i - j * p.P) * p.S_tok;
      }
#pragma unroll 1
      for (int k = 0; k < kCopies; ++k) {
        const int row = k * kRows + my_row;
        const int64_t o = __shfl_sync(0xffffffffu, off, row);
        if (my_chunk < chunks) {
          const uint8_t* src = k_base + (o < 0 ? 0 : o) + my_chunk * 16;
          const uint32_t to = dst + row * S::kRow + S::swizzle(row, my_chunk);
          cp_async16(to, src, o >= 0);
          cp_async16(to + kWarpTokens * S::kRow, src + (o < 0 ? 0 : p.S_kv), o >= 0);
        }
      }
      const uint32_t mask = __ballot_sync(0xffffffffu, off >= 0) & 0xffffu;
      if (lane == 0) s_mask[warp][stage] = mask;
      slow |= 1u << stage;
    };
    int v = p.narrow ? 0 : t0 * kTileTokens + warp * kWarpTokens;
    int next = page_of(v);
#pragma unroll
    for (int s = 0; s < S::kStages - 1; ++s) {
      const int pg = next;
      next = page_of(v + (s + 1) * hop);
      issue(s, v + s * hop, pg);
      cp_async_commit();
    }
    // matrix loads: row and first chunk of this lane, K as it lies and V transposed
    const int k_row = TYPE == kE4m3 ? (lane & 7) + ((lane >> 3) & 1) * 8 : (lane & 7) + (lane >> 4) * 8;
    const int k_chunk = TYPE == kE4m3 ? lane >> 4 : (lane >> 3) & 1;
    const int v_row = (lane & 7) + ((lane >> 3) & 1) * 8, v_chunk = lane >> 4;
    constexpr int kOffsets = S::kChunks >= 8 ? 4 : 2;  // the swizzle repeats after 128 bytes (a row, if shorter)
    uint32_t k_off[kOffsets], v_off[kOffsets];
#pragma unroll
    for (int i = 0; i < kOffsets; ++i) {
      k_off[i] = ring_a + k_row * S::kRow + S::swizzle(k_row, 2 * i + k_chunk);
      v_off[i] = ring_a + (kWarpTokens + v_row) * S::kRow + S::swizzle(v_row, 2 * i + v_chunk);
    }
    int stage = 0;
    bool seen = false;  // a token of this warp's counted (uniform)
    for (; v < end; v += hop) {
      {
        const int pg = next;
        next = page_of(v + S::kStages * hop);
        issue(stage == 0 ? S::kStages - 1 : stage - 1, v + (S::kStages - 1) * hop, pg);
        cp_async_commit();
      }
      cp_async_wait<S::kStages - 1>();
      __syncwarp();
      const uint32_t at = stage * S::kStage;
      const uint32_t mask = slow >> stage & 1 ? s_mask[warp][stage] : 0xffffu;
      if (mask != 0) {
        seen = true;
        float s[2][4] = {};
        if constexpr (TYPE == kE4m3) {
#pragma unroll
          for (int k = 0; k < kSteps; k += 2) {
            uint32_t b4[4];
            ldmatrix4(b4, k_off[(k / 2) % kOffsets] + at + (k / 2 / kOffsets) * (kOffsets * 32));
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                uint32_t lo, hi;
                e4m3x4_to_f16(b4[u * 2 + j], &lo, &hi);
                mma16816<false>(s[j], qf[k + u], lo, hi);
              }
          }
        } else {
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            uint32_t b4[4];
            ldmatrix4(b4, k_off[k % kOffsets] + at + (k / kOffsets) * (kOffsets * 32));
            mma16816<kMmaBf16>(s[0], qf[k], b4[0], b4[1]);
            mma16816<kMmaBf16>(s[1], qf[k], b4[2], b4[3]);
          }
        }
        // scores of rows gr and gr + 8 at tokens gc*2, +1, +8, +9
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[j][e] *= row_scale[e >> 1];
        if (mask != 0xffffu) {
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!((mask >> (j * 8 + gc * 2 + (e & 1))) & 1)) s[j][e] = -INFINITY;
        }
        float top[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) top[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
        // The reference of a row moves only when a score exceeds it by more than 2^kLazy: most tiles
        // need one vote here, no exchange and no rescaling. Weights are at most 2^(kLazy + kShift).
        if (__any_sync(0xffffffffu, top[0] > m[0] + kLazy || top[1] > m[1] + kLazy)) {
          float alpha[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], 2));
            top[i] = fmaxf(top[i], m[i]);
            alpha[i] = top[i] == m[i] ? 1.f : exp2_approx(m[i] - top[i]);
            l[i] *= alpha[i];
            m[i] = top[i];
            base[i] = m[i] == -INFINITY ? 0.f : m[i] - kShift;
          }
#pragma unroll
          for (int i = 0; i < 2 * kSteps; ++i) {
            o[i][0] *= alpha[0];
            o[i][1] *= alpha[0];
            o[i][2] *= alpha[1];
            o[i][3] *= alpha[1];
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[j][e] = exp2_approx(s[j][e] - base[e >> 1]);
            l[e >> 1] += s[j][e];
          }
        uint32_t pf[4];
        pf[0] = pack2<kMmaBf16>(s[0][0], s[0][1]);
        pf[1] = pack2<kMmaBf16>(s[0][2], s[0][3]);
        pf[2] = pack2<kMmaBf16>(s[1][0], s[1][1]);
        pf[3] = pack2<kMmaBf16>(s[1][2], s[1][3]);
        uint32_t pl[4];
        if constexpr (kSecond) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            pl[i] = pack2<true>(s[i >> 1][(i & 1) * 2] - __uint_as_float(pf[i] << 16),
                                s[i >> 1][(i & 1) * 2 + 1] - __uint_as_float(pf[i] & 0xffff0000u));
        }
        if constexpr (TYPE == kE4m3) {
          // a transposed load of 16-bit units brings two neighbouring columns of two tokens: the
          // even columns of a 16-byte chunk form one n-tile, the odd ones the other
#pragma unroll
          for (int k = 0; k < kSteps; k += 2) {
            uint32_t b4[4];
            ldmatrix4_trans(b4, v_off[(k / 2) % kOffsets] + at + (k / 2 / kOffsets) * (kOffsets * 32));
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              // bytes: token 0 (even, odd column), token 1 (even, odd) -> both tokens' even, both odd
              uint32_t even0, odd0, even1, odd1;
              e4m3x4_to_f16(__byte_perm(b4[u * 2], 0, 0x3120), &even0, &odd0);
              e4m3x4_to_f16(__byte_perm(b4[u * 2 + 1], 0, 0x3120), &even1, &odd1);
              mma16816<false>(o[(k + u) * 2], pf, even0, even1);
              mma16816<false>(o[(k + u) * 2 + 1], pf, odd0, odd1);
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < kSteps; ++k) {
            uint32_t b4[4];
            ldmatrix4_trans(b4, v_off[k % kOffsets] + at + (k / kOffsets) * (kOffsets * 32));
            mma16816<kMmaBf16>(o[k * 2], pf, b4[0], b4[1]);
            mma16816<kMmaBf16>(o[k * 2 + 1], pf, b4[2], b4[3]);
            if constexpr (kSecond) {
              mma16816<true>(o[k * 2], pl, b4[0], b4[1]);
              mma16816<true>(o[k * 2 + 1], pl, b4[2], b4[3]);
            }
          }
        }
      }
      __syncwarp();
      if (++stage == S::kStages) stage = 0;
    }
    cp_async_wait<0>();
    __syncthreads();

    // ---- the four warps' results joined, through the ring's memory ------------------------------
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    }
    constexpr int kPitch = DP + 8;  // floats: the eight rows of a warp's store start in different banks
    float* s_o = reinterpret_cast<float*>(smem);                              // [warp][row][kPitch]
    float* s_m = s_o + kAttendWarps * kAttendRows * kPitch;                   // [warp][row]
    float* s_l = s_m + kAttendWarps * kAttendRows;
    if (lane == 0) s_seen[warp] = (seen ? kUsable : 0) | (vis.n > 0 ? kVisible : 0);
    if (gc == 0) {
      s_m[warp * kAttendRows + gr] = m[0] - kShift;
      s_m[warp * kAttendRows + gr + 8] = m[1] - kShift;
      s_l[warp * kAttendRows + gr] = l[0];
      s_l[warp * kAttendRows + gr + 8] = l[1];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (gr + i * 8 >= rows) continue;
      float* to = s_o + (warp * kAttendRows + gr + i * 8) * kPitch;
#pragma unroll
      for (int k = 0; k < 2 * kSteps; k += TYPE == kE4m3 ? 2 : 1) {
        if constexpr (TYPE == kE4m3)  // the tiles of even and of odd columns
          *reinterpret_cast<float4*>(to + k * 8 + gc * 4) =
              make_float4(o[k][2 * i], o[k + 1][2 * i], o[k][2 * i + 1], o[k + 1][2 * i + 1]);
        else
          *reinterpret_cast<float2*>(to + k * 8 + gc * 2) = make_float2(o[k][2 * i], o[k][2 * i + 1]);
      }
    }
    __syncthreads();
    const bool whole = t0 == 0 && t1 == tiles;
    const int64_t slot = ((int64_t)team * 2 + (first ? 0 : 1)) * gridDim.y + unit;
    const int quads = p.Dv / 4;
    if (p.narrow) {  // nothing to join: each warp's rows are a result
      for (int i = tid; i < kAttendWarps * rows * quads; i += kAttendThreads) {
        const int wg = i / quads, d = (i - wg * quads) * 4;
        const int w = wg / rows, g = wg - w * rows;
        if (s_seen[w] == 0) continue;  // empty_requests has written it
        const int64_t e = (int64_t)team * kAttendWarps + w;
        const float sum = s_l[w * kAttendRows + g];
        store_io4(p.out + e * p.o_req + (q_head0 + g) * p.o_head + d * 2,
                  *reinterpret_cast<const float4*>(&s_o[(w * kAttendRows + g) * kPitch + d]),
                  s_seen[w] & kUsable ? __fdividef(p.v_scale, sum) : 0.f, p.io_bf16);
        if (d == 0 && p.lse != nullptr)
          p.lse[e * p.H * p.G + q_head0 + g] = (s_m[w * kAttendRows + g] + log2f(sum)) * kLn2;
      }
      return;
    }
    const bool any = (s_seen[0] | s_seen[1] | s_seen[2] | s_seen[3]) & kUsable;
    static_assert(kAttendWarps == 4, "one flag per warp");
    for (int i = tid; i < rows * quads; i += kAttendThreads) {
      const int g = i / quads, d = (i - g * quads) * 4;
      float f[kAttendWarps], top = -INFINITY, sum = 0.f;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kAttendWarps; ++w) {
        f[w] = s_m[w * kAttendRows + g];
        top = fmaxf(top, f[w]);
      }
      const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < kAttendWarps; ++w) {
        const float c = exp2_approx(f[w] - from);
        const float4 v = *reinterpret_cast<const float4*>(&s_o[(w * kAttendRows + g) * kPitch + d]);
        sum += c * s_l[w * kAttendRows + g];
        acc.x += c * v.x;
        acc.y += c * v.y;
        acc.z += c * v.z;
        acc.w += c * v.w;
      }
      if (whole) {
        const float inv = any ? __fdividef(p.v_scale, sum) : 0.f;
        store_io4(p.out + r * p.o_req + (q_head0 + g) * p.o_head + d * 2, acc, inv, p.io_bf16);
        if (d == 0 && p.lse != nullptr) p.lse[(int64_t)r * p.H * p.G + q_head0 + g] = (top + log2f(sum)) * kLn2;
      } else {
        *reinterpret_cast<float4*>(&p.part[(slot * p.rows + g) * p.Dv + d]) = acc;
        if (d == 0) p.ml[slot * p.rows + g] = make_float2(top, any ? sum : kNoneSeen);
      }
    }
    __syncthreads();
    if (p.D < DP && left > 0) {  // the epilogue has written over the zero columns
      for (int i = lane; i < S::kStages * S::kStage / 16; i += 32)
        reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
      __syncwarp();
    }
    if (p.uncut) return;
    first = false;
  }
}

// Joins the parts of the requests that were cut, a CTA up to eight rows of one of them. First a warp per row turns the parts' maxima and sums into weights,
// then every thread adds up four neighbouring columns of a row over the parts; where rows and
// columns do not fill the CTA, groups of threads take every other part and are added up at the end,
// always in the same order.
constexpr int kJoinThreads = 256;
constexpr int kJoinRows = 8;
constexpr int kJoinParts = 640;  // more teams than a launch has
__global__ void __launch_bounds__(kJoinThreads, 4) topkv_attend_join_kernel(const AttendParams p) {
  __shared__ float s_w[kJoinRows][kJoinParts];
  __shared__ float4 s_acc[kJoinThreads];
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  const int unit = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int4 rec = p.joins[blockIdx.x];  // JoinRecord
  const int r = rec.x, team = rec.y, parts = rec.w, units = gridDim.y;
  if (parts == 0) return;
  const int h = unit / p.gtiles, g0 = (unit - h * p.gtiles) * p.row_tile;
  const int all_rows = min(p.G - g0, p.row_tile);
  const int per = (p.rows + gridDim.z - 1) / gridDim.z;  // at most kJoinRows
  const int row0 = blockIdx.z * per, rows = min(per, all_rows - row0);
  if (rows <= 0) return;
  const int64_t q_head0 = (int64_t)h * p.G + g0 + row0;
  // row `row0` of part k; the parts but the first lie at a constant stride (the host has checked that
  // the workspace's elements can be counted in 32 bits)
  const int slot0 = ((team * 2 + rec.z) * units + unit) * p.rows + row0;
  const int step = 2 * units * p.rows, slot1 = ((team + 1) * 2 * units + unit) * p.rows + row0 - step;
  auto slot = [&](int k) -> int { return k == 0 ? slot0 : slot1 + k * step; };

  const int quads = p.Dv / 4, items = rows * quads;  // quads: at most 128
  const int groups = max(kJoinThreads / items, 1), group = groups > 1 ? tid / items : 0;
  // Item i: columns 4 quad .. of row g; a thread's first item is loaded while the weights are formed.
  auto part_of = [&](int i) { return i / quads * p.Dv + (i % quads) * 4; };
  constexpr int kAhead = 4;
  float4 ahead[kAhead];
  const int item0 = tid - group * items;
  const bool mine = group < groups && item0 < items;
#pragma unroll
  for (int j = 0; j < kAhead; ++j) {
    const int k = group + j * groups;
    if (mine && k < parts) ahead[j] = *reinterpret_cast<const float4*>(&p.part[part_of(item0) + slot(k) * p.Dv]);
  }
  for (int g = warp; g < rows; g += kJoinThreads / 32) {
    // up to 64 parts are held by the warp's lanes, so that they are loaded once and all together
    constexpr int kHeld = 2;
    float2 held[kHeld];
    float top = -INFINITY, sum = 0.f;
    bool seen = false;  // a part has a token that counted; one that has none weighs 2^-inf = 0 below
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      const int k = lane + 32 * j;
      held[j] = k < parts ? p.ml[slot(k) + g] : make_float2(-INFINITY, kNoneSeen);
    }
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      top = fmaxf(top, held[j].x);
      seen |= held[j].y != kNoneSeen;
    }
    for (int k = lane + 32 * kHeld; k < parts; k += 32) {
      const float2 ml = p.ml[slot(k) + g];
      top = fmaxf(top, ml.x);
      seen |= ml.y != kNoneSeen;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) {
      held[j].x = exp2_approx(held[j].x - from);
      sum += held[j].x * held[j].y;
    }
    for (int k = lane + 32 * kHeld; k < parts; k += 32) {
      const float2 ml = p.ml[slot(k) + g];
      sum += exp2_approx(ml.x - from) * ml.y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const float inv = __any_sync(0xffffffffu, seen) ? p.v_scale / sum : 0.f;
#pragma unroll
    for (int j = 0; j < kHeld; ++j)
      if (lane + 32 * j < parts) s_w[g][lane + 32 * j] = held[j].x * inv;
    for (int k = lane + 32 * kHeld; k < parts; k += 32) s_w[g][k] = exp2_approx(p.ml[slot(k) + g].x - from) * inv;
    if (lane == 0 && p.lse != nullptr)
      p.lse[(int64_t)r * p.H * p.G + q_head0 + g] = (top + log2f(sum)) * kLn2;
  }
  __syncthreads();

  auto add = [](float4& acc, const float4& v, float f) {
    acc.x += f * v.x;
    acc.y += f * v.y;
    acc.z += f * v.z;
    acc.w += f * v.w;
  };
  for (int i = item0; mine && i < items; i += kJoinThreads) {
    const int g = i / quads;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    int k = group;
    if (i == item0) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j, k += groups)
        if (k < parts) add(acc, ahead[j], s_w[g][k]);
    }
#pragma unroll 4
    for (; k < parts; k += groups) add(acc, *reinterpret_cast<const float4*>(&p.part[part_of(i) + slot(k) * p.Dv]), s_w[g][k]);
    if (groups > 1)
      s_acc[tid] = acc;
    else
      store_io4(p.out + r * p.o_req + (q_head0 + g) * p.o_head + (i % quads) * 8, acc, 1.f, p.io_bf16);
  }
  if (groups == 1) return;
  __syncthreads();
  if (tid < items) {
    float4 acc = s_acc[tid];
    for (int k = 1; k < groups; ++k) add(acc, s_acc[k * items + tid], 1.f);
    store_io4(p.out + r * p.o_req + (q_head0 + tid / quads) * p.o_head + (tid % quads) * 8, acc, 1.f, p.io_bf16);
  }
}

}  // namespace topkv

// Attention of one new token per request where groups of requests share their first tokens: the plan of who
// shares what, the shared tokens' part, and the join with what each request has for itself.
//
//   part over the tokens i of a range:  m = max x_i, l = sum exp(x_i - m), o = sum exp(x_i - m) V[i]
//   parts join by  out = sum_k exp(m_k - m) o_k / sum_k exp(m_k - m) l_k,  m = max m_k
//
// The queries of a group's members and of a KV head's G query heads are the rows of one product with the
// prefix: members * G rows, and as many flops a byte at 16 bits (4 rows flops for 2 + 2 bytes of K and V), twice as
// many at 8. The tensor rate is 254 flop a byte of this memory, so 254 rows of 16 bits balance both and 128 leave the
// memory as the bound: the product runs on the tensor memory path (tcgen05), 128 rows to a tile and up to two tiles over
// the same tokens, rows in TMEM lanes, one thread a row, so that maxima and sums need no exchange:
//
//   S [128 x tokens] = Q [128 x D] K^T         both K-major in shared memory
//   O [128 x D]     += P [128 x tokens] V      P in TMEM, over the scores it was made of; V N-major. Of a bf16 cache P is
//                                              the sum of two bf16 matrices (up to 128 columns)
//
// A CTA, alone on its SM, has two accumulators that work by turns, the softmax of one under the products of the
// other: with more than 128 rows they are two tiles of rows over the same tokens, else the same rows over every
// other tile of tokens. (256 columns: one accumulator, two buffers of scores, 64 tokens a tile.) Roles:
//   warps 0-7    softmax: four per accumulator, one thread a row; also Q and the result
//   two warps    load K and V through the block table into a ring: tensor copies of page pieces, or 16-byte
//                copies (any page size and stride). Of an 8-bit cache one warp loads and four make fp16 of it (8 groups
//                of eight behind 4,096 tokens 81 us, 85 with two warps)
//   one warp     one thread issues the products
// The (group, KV head, 256 rows) units laid end to end, as long as their tiles, are cut into equal ranges, one
// per CTA; each leaves its part in 32 bits in the workspace, and the joining kernel adds them to those of the
// tokens behind the prefix, in order, so that results do not depend on timing.
// Waits are bounded and TMEM is held as in the latent-row kernel.
// What bounds it: with many rows the steps from one tile's scores to the next (with one bf16 value a weight a tile of 128
// tokens and 256 rows takes 4,400 cycles, of which the tensor core is busy 2,200 and a softmax job 2,600; the second value
// adds 1,100 to the tensor core's); with few rows a tile takes as long, and memory is at about half its rate. Measured, with
// the plan made before: 64 requests behind 16,384 tokens with 100 to 1,000 of their own, 8 x 8 heads of 128, bf16: 103 us,
// 61 in this kernel, 30 behind it, 11 in the join; 78 requests in 6 groups behind 500 to 4,000 tokens, e4m3: 68 us, 31 + 26 +
// 10. 32 requests behind 8,192 tokens, plan included: 4 x 8 heads of 256 72 us (floor 15), e4m3 84 (8); 8 x 8 heads of 64 50 (8).
#pragma once
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <cfloat>
#include <cstdint>

#include "topkv_attend.cuh"
#include "topkv_common.cuh"
#include "topkv_latent.cuh"

namespace topkv {

// ---- the plan -------------------------------------------------------------------------------------
constexpr int kPrefixPlanThreads = 1024;
struct PrefixPlanParams {
  const int32_t* bt;
  const int32_t* sl;
  int32_t* plan;
  int64_t num_pages;
  int R, maxp, P, min_tokens;
};
// Full pages of a row, as far as its table goes.
__device__ __forceinline__ int full_pages(const PrefixPlanParams& p, int r) {
  return min(max(p.sl[r], 0) / p.P, p.maxp);
}
// A warp looks at a row: the lowest row that begins with the same page, and how many pages both have in common.
__device__ __forceinline__ void plan_leader(const PrefixPlanParams& p, int r, int lane) {
  const int32_t* mine = p.bt + (int64_t)r * p.maxp;
  int full = full_pages(p, r), lead = r;
  const int page = full > 0 ? mine[0] : -1;
  if (lane == 0 && (p.sl[r] < 0 || p.sl[r] > (int64_t)p.maxp * p.P)) raise_error(kErrTable);
  constexpr int kAhead = 8;
  if (page >= 0 && page < p.num_pages) {
#pragma unroll 1
    for (int q0 = 0; q0 < r && lead == r; q0 += 32 * kAhead) {
      bool same[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int q = q0 + u * 32 + lane;
        same[u] = q < r && full_pages(p, q) > 0 && p.bt[(int64_t)q * p.maxp] == page;
      }
#pragma unroll
      for (int u = kAhead - 1; u >= 0; --u) {
        const uint32_t found = __ballot_sync(0xffffffffu, same[u]);
        if (found != 0) lead = q0 + u * 32 + __ffs(found) - 1;
      }
    }
  }
  const int32_t* first = p.bt + (int64_t)lead * p.maxp;
  full = min(full, full_pages(p, lead));
  int common = full;
#pragma unroll 1
  for (int j0 = 0; lead != r && j0 < common; j0 += 32 * kAhead) {
    bool differ[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u * 32 + lane;
      differ[u] = j < full && first[j] != mine[j];
    }
#pragma unroll
    for (int u = kAhead - 1; u >= 0; --u) {
      const uint32_t found = __ballot_sync(0xffffffffu, differ[u]);
      if (found != 0) common = j0 + u * 32 + __ffs(found) - 1;
    }
  }
  if (lane == 0) {
    p.plan[TOPKV_PLAN_LEADER * p.R + r] = lead;
    p.plan[TOPKV_PLAN_COMMON * p.R + r] = common * p.P;
  }
}
// ... and, over all rows, what its group shares, its size, and the row's place in the order.
__device__ __forceinline__ void plan_group(const PrefixPlanParams& p, int r, int lane) {
  // written by other CTAs of the cluster, or by the launch before: read from L2
  const int32_t* leader = p.plan + TOPKV_PLAN_LEADER * p.R;
  const int32_t* common = p.plan + TOPKV_PLAN_COMMON * p.R;
  const int lead = __ldcg(leader + r);
  int shared = 0x7fffffff, members = 0, place = 0;
#pragma unroll 4
  for (int q = lane; q < p.R; q += 32) {
    const int l = __ldcg(leader + q), c = __ldcg(common + q);
    if (l == lead) {
      shared = min(shared, c);
      ++members;
    }
    place += l < lead || (l == lead && q < r);
  }
  shared = __reduce_min_sync(0xffffffffu, shared);
  members = __reduce_add_sync(0xffffffffu, members);
  place = __reduce_add_sync(0xffffffffu, place);
  if (lane == 0) {
    p.plan[TOPKV_PLAN_SHARED * p.R + r] = members > 1 && shared >= p.min_tokens ? shared : 0;
    p.plan[TOPKV_PLAN_MEMBERS * p.R + r] = members;
    p.plan[TOPKV_PLAN_PLACE * p.R + r] = place;
    p.plan[TOPKV_PLAN_ORDER * p.R + place] = r;
  }
}
// A warp per row. Up to kPrefixPlanRows rows fit one cluster, whose barrier separates the two steps; more take a
// launch each. (7 rows: 7.8 us with the cluster, 10.0 with two launches; 253 rows of up to 410 pages 9.6; by two launches
// 1,000 rows 23.5, 3,000 63: every row looks at all others, twice.)
constexpr int kPrefixPlanCluster = 8, kPrefixPlanRows = kPrefixPlanCluster * kPrefixPlanThreads / 32;
__global__ void __launch_bounds__(kPrefixPlanThreads) topkv_plan_cluster_kernel(const PrefixPlanParams p) {
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  const int lane = threadIdx.x & 31, r = blockIdx.x * (kPrefixPlanThreads / 32) + (threadIdx.x >> 5);
  if (r < p.R) plan_leader(p, r, lane);
  __threadfence();
  cooperative_groups::this_cluster().sync();
  if (r < p.R) plan_group(p, r, lane);
}
__global__ void __launch_bounds__(kPrefixPlanThreads) topkv_plan_leaders_kernel(const PrefixPlanParams p) {
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  const int lane = threadIdx.x & 31, r = blockIdx.x * (kPrefixPlanThreads / 32) + (threadIdx.x >> 5);
  if (r < p.R) plan_leader(p, r, lane);
}
__global__ void __launch_bounds__(kPrefixPlanThreads) topkv_plan_groups_kernel(const PrefixPlanParams p) {
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  const int lane = threadIdx.x & 31, r = blockIdx.x * (kPrefixPlanThreads / 32) + (threadIdx.x >> 5);
  if (r < p.R) plan_group(p, r, lane);
}

// ---- the shared tokens' part ------------------------------------------------------------------------
constexpr int kPrefixRows = 128;    // rows of a tile
constexpr int kPrefixMaxStages = 8;
constexpr int kPrefixMaxRaw = 4;    // buffers of 8-bit tiles that wait to be converted
constexpr int kPrefixCtas = 148;    // at most

struct PrefixControl {
  uint64_t bar[2 * kPrefixMaxStages + 7 + 2 * kPrefixMaxRaw];
  int64_t scan[2][16];
  int off;
  int group[9];    // what is known of the first group; leader -1: nothing to do
  uint32_t tmem;
  volatile int dead;
  volatile int odd;   // a page outside the pool has been met
  float row_scale[2 * kPrefixRows];
};
template <int DP, int TYPE>
struct PrefixShape {
  static constexpr int kTiles = DP <= 128 ? 2 : 1;        // accumulators
  static constexpr int kTokens = DP <= 128 ? 128 : 64;    // per tile
  static constexpr int kQ = kPrefixRows * DP * 2;         // bytes of a tile of Q
  static constexpr int kStage = kTokens * DP * 2;         // ... of K or V
  static constexpr bool kConvert = TYPE == kE4m3;
  static constexpr int kRaws = !kConvert ? 0 : DP == 64 ? 4 : 2;
  static constexpr int kRaw = kTokens * DP;               // bytes of a tile of 8-bit values
  static constexpr int kRoom = (227 * 1024 - kTiles * kQ - kRaws * kRaw - (int)sizeof(PrefixControl)) / kStage;
  static constexpr int kStages = kRoom < kPrefixMaxStages ? kRoom : kPrefixMaxStages;
  static constexpr int kRawAt = kTiles * kQ + kStages * kStage;
  static constexpr int kControl = kRawAt + kRaws * kRaw;
  static constexpr int kSmem = kControl + (int)sizeof(PrefixControl);
  static constexpr int kSoftmaxWarps = 4 * kTiles;
  static constexpr int kLoadWarps = kConvert ? 4 : 2;     // that fill the ring
  static constexpr int kThreads = (kSoftmaxWarps + kLoadWarps + (kConvert ? 1 : 0) + 1) * 32;
  static constexpr uint32_t kScores = 0, kSums = 2 * kTokens;  // TMEM columns: two buffers of scores, the accumulators
  static_assert(2 * kTokens + kTiles * DP <= 512, "TMEM");
  static_assert(kStages >= 4, "the ring holds K of two tiles and V of the first");
};
// A group: its leader, and the geometry of its units.
struct PrefixGroup {
  int lead, place;   // its first row's place in the plan's order
  int tokens, n;     // shared tokens, tiles of them
  int rows;          // members * G
  int units;         // per KV head
  int full;          // length of a unit of all rows
  int length;        // of a KV head's units
  int begin;         // where the group's units begin on the line (the host has seen to it that this fits)
  int first;         // rows of the groups before it on the line, where its parts lie
  int pad[2];
};
// How the line is cut.
struct PrefixHeader {
  int each;      // length of a range ...
  int more;      // ... and how many are one longer
  int teams, pad;
};
struct PrefixParams {
  AttendParams a;          // teams is that of the tokens behind the prefix
  PrefixHeader* header;    // for the joining kernel, as are
  PrefixGroup* groups;     // [R], of leaders
  float2* ml;              // [rows of parts]
  float* part;             // [rows of parts][Dv]
  int tiles;               // accumulators, tokens per tile: those of the kernel's shape
  int tokens;
};
__device__ __forceinline__ PrefixGroup prefix_group(const PrefixParams& p, int lead) {
  const AttendParams& a = p.a;
  PrefixGroup g;
  g.lead = lead;
  // as shared_tokens() has it for the leader; all loads at once
  const int leader = a.plan[TOPKV_PLAN_LEADER * a.R + lead], shared = a.plan[TOPKV_PLAN_SHARED * a.R + lead];
  const int members = a.plan[TOPKV_PLAN_MEMBERS * a.R + lead], place = a.plan[TOPKV_PLAN_PLACE * a.R + lead], s = a.sl[lead];
  g.tokens = leader == lead && members >= 2 && shared > 0 && shared <= s && (int64_t)(members - a.spent) * shared >= a.least_saved ? (int)min((int64_t)shared, (int64_t)a.maxp * a.P) : 0;
  if (g.tokens == 0) return g;
  g.n = (g.tokens - 1) / p.tokens + 1;
  g.place = min(max(place, 0), a.R - 1);
  g.rows = min(members, a.R - g.place) * a.G;
  const int tall = kPrefixRows * p.tiles, rest = (g.rows - 1) % tall + 1;
  g.units = (g.rows - 1) / tall + 1;
  g.full = g.n * p.tiles;
  g.length = (g.units - 1) * g.full + (rest > kPrefixRows ? g.full : g.n);
  return g;
}
// One unit: rows first_row .. first_row + rows - 1 of a group with one KV head.
struct PrefixUnit {
  int h, first_row, rows;
  bool both;       // the accumulators hold different rows; a tile of tokens is as long as both
  int length;
  int64_t slot;    // row of parts where the unit's parts of team 0 would lie
};
__device__ __forceinline__ PrefixUnit prefix_unit(const PrefixParams& p, const PrefixGroup& g, int h, int i) {
  PrefixUnit u;
  const int tall = kPrefixRows * p.tiles;
  u.h = h;
  u.first_row = i * tall;
  u.rows = min(tall, g.rows - u.first_row);
  u.both = u.rows > kPrefixRows;
  u.length = u.both ? g.full : g.n;
  u.slot = p.tiles * ((int64_t)p.a.H * g.first + (int64_t)h * g.rows + u.first_row);
  return u;
}
__device__ __forceinline__ int prefix_team_of(const PrefixHeader& t, int x) {
  const int wide = t.more * (t.each + 1), past = x >= wide;
  return (x - past * wide) / (t.each + 1 - past) + past * t.more;
}
// The next leader of a group that shares, from row r on (a whole warp asks); R if there is none.
__device__ __forceinline__ int next_group(const PrefixParams& p, int r, int lane) {
  for (; r < p.a.R; r += 32) {
    const int mine = r + lane;
    const uint32_t found = __ballot_sync(0xffffffffu, mine < p.a.R && prefix_group(p, mine).tokens > 0);
    if (found != 0) return r + __ffs(found) - 1;
  }
  return p.a.R;
}

// Two products and sums at a time.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{ .reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%6, %7}; fma.rn.f32x2 x, x, y, z; mov.b64 {%0, %1}, x; }"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{ .reg .b64 x, y; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; add.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x; }"
      : "=f"(d.x), "=f"(d.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}
// What has been loaded is used only behind this, by name.
__device__ __forceinline__ void tmem_loaded(uint32_t (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]),
                 "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]),
                 "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}
// Arrives at the barrier once this thread's copies so far are there.
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tma_load5(uint32_t dst, const CUtensorMap* map, int x, int token, int head, int plane, int page, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
      "l"(map), "r"(x), "r"(token), "r"(head), "r"(plane), "r"(page), "r"(bar)
      : "memory");
}

__device__ __forceinline__ void tcgen05_mma_ta(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{ .reg .pred p; .reg .b64 db; mov.b64 db, {%2, %3}; setp.ne.u32 p, %5, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(hi), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}

template <int DP, int TYPE>
__global__ void __launch_bounds__(PrefixShape<DP, TYPE>::kThreads, 1) topkv_prefix_kernel(const PrefixParams p, const __grid_constant__ CUtensorMap map) {
  using S = PrefixShape<DP, TYPE>;
  constexpr bool kBf = TYPE == kBf16;
  constexpr float kShift = kBf ? 0.f : 7.f;
  // bf16 keeps 8 bits of a weight. What that cuts off is multiplied as well, as in the kernel of the other tokens, so
  // that shared tokens count as exactly as a request's own: behind 16,384 tokens the error against 64 bits falls from 0.0023
  // to 0.0017, the output's rounding, for half as many products again (64 requests 104 -> 112 us, the plan included).
  constexpr bool kSecond = kBf && DP <= 128;
  constexpr int kTokens = S::kTokens, kTiles = S::kTiles, kStages = S::kStages;
  // 8-bit values: a warp brings them, four convert
  constexpr int kRawWarp = S::kConvert ? S::kSoftmaxWarps : -1, kLoadWarp = S::kSoftmaxWarps + (S::kConvert ? 1 : 0);
  constexpr int kIssueWarp = kLoadWarp + S::kLoadWarps;
  constexpr int kSoftmaxThreads = S::kSoftmaxWarps * 32;
  constexpr int kBlock = kTokens * 128, kQBlock = kPrefixRows * 128;  // bytes of 64 columns
  extern __shared__ __align__(128) uint8_t smem[];
  const AttendParams& a = p.a;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, team = blockIdx.x;
  const uint32_t base = smem_addr(smem);
  if (base & 1023) {
    if (tid == 0) raise_error(kErrWait);
    return;
  }
  PrefixControl& ctl = *reinterpret_cast<PrefixControl*>(smem + S::kControl);
  volatile int& s_dead = ctl.dead;
  const uint32_t b_full = smem_addr(ctl.bar), b_free = b_full + 8 * kStages, b_score = b_free + 8 * kStages;
  const uint32_t b_weight = b_score + 16, b_sum = b_score + 32, b_query = b_score + 48;
  const uint32_t b_raw = b_query + 8, b_raw_free = b_raw + 8 * S::kRaws;
  if (tid == 0) {
    s_dead = 0;
    ctl.odd = 0;
    for (int i = 0; i < kStages; ++i) {
      mbar_init(b_full + 8 * i, S::kLoadWarps * 32);
      mbar_init(b_free + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(b_score + 8 * i, 1);
      mbar_init(b_weight + 8 * i, 128);
      mbar_init(b_sum + 8 * i, 1);
    }
    mbar_init(b_query, kSoftmaxThreads);
    for (int i = 0; i < S::kRaws; ++i) {
      mbar_init(b_raw + 8 * i, 32);
      mbar_init(b_raw_free + 8 * i, S::kLoadWarps * 32);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // The kernel behind this one does not wait for it: it may run once this one has waited. (It holds no TMEM, and
  // what comes after it starts when all its CTAs have, which is after this kernel's.)
  if (!a.late_wait) {
    pdl_wait_prior_grid();
    pdl_release_next_grid();
  }
  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)), "n"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    tcgen05_before_sync();
  }

  // ---- this CTA's range of the line --------------------------------------------------------------------
  int pos, left = 0;
  {
    const int per = (a.R + S::kThreads - 1) / S::kThreads;
    const int r0 = (int)min((int64_t)tid * per, (int64_t)a.R), r1 = min(r0 + per, a.R);
    PrefixGroup g = {};
    auto length = [&](int r) {
      if (per > 1 || g.n == 0) g = prefix_group(p, r);
      return g.tokens > 0 ? a.H * g.length : 0;
    };
    int64_t mine = 0, mine_rows = 0;
    for (int r = r0; r < r1; ++r) {
      const int n = length(r);
      mine += n;
      mine_rows += n > 0 ? g.rows : 0;
    }
    int64_t incl = mine, incl_rows = mine_rows;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t up = __shfl_up_sync(0xffffffffu, incl, o), up_rows = __shfl_up_sync(0xffffffffu, incl_rows, o);
      if (lane >= o) {
        incl += up;
        incl_rows += up_rows;
      }
    }
    if (lane == 31) {
      ctl.scan[0][warp] = incl;
      ctl.scan[1][warp] = incl_rows;
    }
    if (tid == 0) ctl.group[0] = -1;
    __syncthreads();
    int64_t sum = 0, sum_rows = 0;
    for (int w = 0; w < S::kThreads / 32; ++w) {
      if (w < warp) {
        incl += ctl.scan[0][w];
        incl_rows += ctl.scan[1][w];
      }
      sum += ctl.scan[0][w];
      sum_rows += ctl.scan[1][w];
    }
    // A plan whose groups overlap can come to more than the line counts, or than there is room for: it has no work then
    // (the host has seen to it that no other can).
    const bool fits = sum <= 0x7fffffff && sum_rows <= (int64_t)a.R * a.G;
    const int total = fits ? (int)sum : 0;
    if (!fits && tid == 0) raise_error(kErrTable);
    // a range is two tiles long at least: what a CTA costs to begin is about that
    const int teams = min((int)gridDim.x, (total + 1) / 2);
    PrefixHeader t;
    t.each = total / max(teams, 1);
    t.more = total - t.each * teams;
    t.teams = teams;
    pos = t.each * team + min(team, t.more);
    if (team < teams) left = t.each + (team < t.more ? 1 : 0);
    if (a.late_wait) {  // the join of the call before reads the workspace until then
      pdl_wait_prior_grid();
      pdl_release_next_grid();
    }
    int at = (int)(incl - mine), rows_at = (int)(incl_rows - mine_rows);
    const bool begins = left > 0 && pos >= at && pos < incl;  // exactly one thread
    if (begins || (team == 0 && total > 0)) {
      for (int r = r0; r < r1; ++r) {
        const int n = length(r);
        if (team == 0 && n > 0) {
          g.begin = at;
          g.first = rows_at;
          p.groups[r] = g;
        }
        if (begins && pos >= at && pos < at + n) {
          ctl.off = pos - at;
          const int known[9] = {r, g.place, g.tokens, g.n, g.rows, g.units, g.full, g.length, rows_at};
#pragma unroll
          for (int i = 0; i < 9; ++i) ctl.group[i] = known[i];
        }
        at += n;
        rows_at += n > 0 ? g.rows : 0;
      }
    }
    if (team == 0 && tid == 0) *p.header = t;
  }
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = ctl.tmem;

  auto wait = [&](uint32_t bar, uint32_t phase) {
    if (mbar_try_wait(bar, phase & 1)) return;
    const long long began = clock64();
    while (!mbar_try_wait(bar, phase & 1)) {
      if (s_dead) break;
      if (clock64() - began > kWaitClocks) {
        s_dead = 1;
        raise_error(kErrWait);
        break;
      }
    }
  };

  constexpr uint32_t kType = 1u << 4 | (kBf ? 1u : 0u) << 7 | (kBf ? 1u : 0u) << 10 | 8u << 24;  // M = 128
  constexpr uint32_t kScore = kType | (uint32_t)(kTokens >> 3) << 17;
  const uint32_t kValue = kType | 1u << 16 | (uint32_t)((a.D + 15) / 16 * 2) << 17;  // V is N-major
  const int ksteps = (a.D + 15) / 16;
  uint32_t seq = 0;                 // tiles of tokens before the current segment, in this CTA
  uint32_t done[2] = {0, 0};        // jobs before, by the buffer of scores they use
  uint32_t seg = 0;
  uint32_t issued = 0;              // load: entries whose copies are enqueued
  auto page_column = [&](int x) { return a.page_shift >= 0 ? x >> a.page_shift : x / a.P; };
  // Hands out what is this CTA's: tiles [t0, t1) of a unit at a time. Every role walks by itself, so that each has
  // registers of its own.
  auto walk = [&](auto body) {
    PrefixGroup g{ctl.group[0], ctl.group[1], ctl.group[2], ctl.group[3], ctl.group[4], ctl.group[5], ctl.group[6], ctl.group[7]};
    g.first = ctl.group[8];
    int off = ctl.off, rest = left;
    int lead = g.lead;
    while (rest > 0 && lead >= 0 && lead < a.R) {
      const int h = off / g.length, in_head = off - h * g.length, i = min(in_head / g.full, g.units - 1);
      const PrefixUnit u = prefix_unit(p, g, h, i);
      const int from = in_head - i * g.full, take = min(rest, u.length - from);
      const int scale = u.both ? kTiles : 1;
      const int t0 = (from + scale - 1) / scale, t1 = (from + take + scale - 1) / scale, count = t1 - t0, jobs = count * scale;
      body(g, u, t0, t1, jobs);
      seq += count;
      done[0] += (jobs + 1) / 2;
      done[1] += jobs / 2;
      if (jobs > 0) ++seg;
      rest -= take;
      off += take;
      if (off == a.H * g.length && rest > 0) {
        off = 0;
        lead = next_group(p, lead + 1, lane);
        const int first = g.first + g.rows;
        if (lead < a.R) g = prefix_group(p, lead);
        g.first = first;
      }
    }
  };

  if (warp >= S::kSoftmaxWarps) {
    if (warp == kRawWarp || (!S::kConvert && warp >= kLoadWarp && warp < kIssueWarp)) {
     walk([&](const PrefixGroup& g, const PrefixUnit& u, int t0, int t1, int jobs) {
      const int h = u.h;
      const int32_t* bt_row = a.bt + (int64_t)g.lead * a.maxp;
      // ---- load: 16-bit tiles into the ring, 8-bit tiles into buffers of their own ------------------------
      constexpr int kWarps = S::kConvert ? 1 : S::kLoadWarps, kElem = S::kConvert ? 1 : 2;
      constexpr int kDepth = S::kConvert ? S::kRaws : kStages, kBytes = S::kConvert ? S::kRaw : S::kStage;
      const int w = S::kConvert ? 0 : warp - kLoadWarp;
      const uint32_t b_there = S::kConvert ? b_raw : b_full, b_room = S::kConvert ? b_raw_free : b_free;
      const uint32_t to0 = base + (S::kConvert ? S::kRawAt : kTiles * S::kQ);
      const uint8_t* head = a.pool + (int64_t)h * a.S_head;
      constexpr int kRows = kTokens / kWarps, kGroups = kRows / 32;  // rows of this warp
      static_assert(kRows % 32 == 0, "a lane per row");
      const int chunks = a.D * kElem / 16, padded = S::kConvert ? chunks : ksteps * 2;  // of 16 bytes
      const int blocks = S::kConvert ? 1 : (a.D + 63) / 64;
      // Whole page pieces come by tensor copies, those outside the pool and behind the prefix as zeros from
      // outside the tensor. A prefix that ends inside a piece has its last tile copied row by row.
      const int box = a.box, boxes = box > 0 ? kTokens / box : 0;
      const uint32_t box_bytes = (uint32_t)(box * (S::kConvert ? a.D : 128));
      auto piece = [&](int t) {  // page of piece `lane` of a tile
        const int x = t * kTokens + lane * box;
        return t < t1 && lane < boxes && x < g.tokens ? bt_row[page_column(x)] : -1;
      };
      int pg = boxes > 0 ? piece(t0) : -1;
      for (int t = t0; t < t1; ++t) {
        if (__any_sync(0xffffffffu, s_dead)) break;
        if (boxes > 0 && (g.tokens >= (t + 1) * kTokens || g.tokens % box == 0)) {
          const int x = t * kTokens + lane * box;
          bool ok = lane < boxes && x < g.tokens;
          if (ok && (pg < 0 || pg >= a.num_pages)) {
            raise_error(kErrTable);
            ctl.odd = 1;
            ok = false;
          }
          const int z = ok ? pg : (int)a.num_pages, y = ok ? x - page_column(x) * a.P : 0;
          pg = piece(t + 1);
#pragma unroll 1
          for (int plane = 0; plane < 2; ++plane, ++issued) {
            const uint32_t stage = issued % kDepth, bar = b_there + 8 * stage;
            if (issued >= kDepth) wait(b_room + 8 * stage, issued / kDepth - 1);
            const uint32_t dst = to0 + stage * kBytes;
            if (lane == 0)
              mbar_expect_tx(bar, (uint32_t)((boxes + kWarps - 1 - w) / kWarps) * blocks * box_bytes);
            else
              bar_arrive(bar);
            __syncwarp();
            // the pieces' places are gathered by the whole warp, so that one thread's instructions follow each other
#pragma unroll 1
            for (int e0 = w; e0 < boxes; e0 += 4 * kWarps) {
              int ze[4], ye[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                ze[k] = __shfl_sync(0xffffffffu, z, (e0 + kWarps * k) & 31);
                ye[k] = __shfl_sync(0xffffffffu, y, (e0 + kWarps * k) & 31);
              }
              if (elect_one()) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const int e = e0 + kWarps * k;
                  if (e >= boxes) break;
#pragma unroll
                  for (int b = 0; b < (S::kConvert ? 1 : DP / 64); ++b)
                    if (b < blocks) tma_load5(dst + b * kBlock + e * box_bytes, &map, b * 64, ye[k], h, plane, ze[k], bar);
                }
              }
              __syncwarp();
            }
          }
          continue;
        }
        if (boxes > 0) pg = piece(t + 1);
        int64_t o[kGroups];
#pragma unroll
        for (int k = 0; k < kGroups; ++k) {
          const int x = t * kTokens + w * kRows + k * 32 + lane;
          o[k] = -1;
          if (x < g.tokens) {
            const int j = page_column(x), page = bt_row[j];
            if (page < 0 || page >= a.num_pages) {
              raise_error(kErrTable);
              ctl.odd = 1;
            } else {
              o[k] = (int64_t)page * a.S_page + (int64_t)(x - j * a.P) * a.S_tok;
            }
          }
        }
#pragma unroll 1
        for (int plane = 0; plane < 2; ++plane, ++issued) {
          const uint32_t stage = issued % kDepth;
          if (issued >= kDepth) wait(b_room + 8 * stage, issued / kDepth - 1);
          const uint32_t dst = to0 + stage * kBytes;
          const uint8_t* src0 = head + plane * a.S_kv;
          const int c = lane & 7, sub = lane >> 3;
#pragma unroll
          for (int k = 0; k < kGroups; ++k) {
#pragma unroll 2
            for (int rg = 0; rg < 8; ++rg) {
              const int row = rg * 4 + sub, in_tile = w * kRows + k * 32 + row;
              const int64_t ro = __shfl_sync(0xffffffffu, o[k], row);
#pragma unroll
              for (int b = 0; b < DP * kElem / 128; ++b) {
                const int ch = b * 8 + c;
                const uint32_t to = S::kConvert ? dst + in_tile * a.D + ch * 16 : dst + b * kBlock + in_tile * 128 + ((c ^ (row & 7)) << 4);
                const bool ok = ro >= 0 && ch < chunks;
                if (ch < padded) cp_async16(to, ok ? src0 + ro + ch * 16 : a.pool, ok);
              }
              if (DP * kElem < 128 && c < padded) {  // 64 columns of 8 bits
                const bool ok = ro >= 0;
                cp_async16(dst + in_tile * a.D + c * 16, ok ? src0 + ro + c * 16 : a.pool, ok);
              }
            }
          }
          cp_async_arrive(b_there + 8 * stage);
        }
      }
     });
    } else if (S::kConvert && warp >= kLoadWarp && warp < kIssueWarp) {
     walk([&](const PrefixGroup& g, const PrefixUnit& u, int t0, int t1, int jobs) {
      const int count = t1 - t0;
      // ---- convert: 16 bytes of a row at a time, a share of the rows each ----------------------------------
      constexpr int kRaws = S::kRaws > 0 ? S::kRaws : 1;
      constexpr int kChunks = DP / 16, kPer = 32 / kChunks, kRows = kTokens / S::kLoadWarps;
      const int c = lane % kChunks, sub = lane / kChunks, row0 = (warp - kLoadWarp) * kRows;
      for (int e = 0; e < 2 * count; ++e, ++issued) {
        const uint32_t stage = issued % kStages, raw = issued % kRaws;
        wait(b_raw + 8 * raw, issued / kRaws);
        if (issued >= kStages) wait(b_free + 8 * stage, issued / kStages - 1);
        if (__any_sync(0xffffffffu, s_dead)) break;
        const uint8_t* from = smem + S::kRawAt + raw * S::kRaw + c * 16;
        uint8_t* const to = smem + kTiles * S::kQ + stage * S::kStage + (c >> 2) * kBlock;
        const int ch = (c & 3) * 2;
        if (c * 16 < a.D) {
#pragma unroll 4
          for (int k = 0; k < kRows; k += kPer) {
            const int row = row0 + k + sub;
            const uint4 v = *reinterpret_cast<const uint4*>(from + row * a.D);
            uint32_t x8[8];
            e4m3x4_to_f16(v.x, &x8[0], &x8[1]);
            e4m3x4_to_f16(v.y, &x8[2], &x8[3]);
            e4m3x4_to_f16(v.z, &x8[4], &x8[5]);
            e4m3x4_to_f16(v.w, &x8[6], &x8[7]);
            *reinterpret_cast<uint4*>(to + row * 128 + ((ch ^ (row & 7)) << 4)) = make_uint4(x8[0], x8[1], x8[2], x8[3]);
            *reinterpret_cast<uint4*>(to + row * 128 + (((ch + 1) ^ (row & 7)) << 4)) = make_uint4(x8[4], x8[5], x8[6], x8[7]);
          }
        }
        bar_arrive(b_raw_free + 8 * raw);
        proxy_fence_smem();
        bar_arrive(b_full + 8 * stage);
      }
     });
    } else if (warp == kIssueWarp) {
     walk([&](const PrefixGroup& g, const PrefixUnit& u, int t0, int t1, int jobs) {
      // ---- products -----------------------------------------------------------------------------------
      // 16-byte copies are a thread's own writes, which the products see only behind a fence; a loader's own would
      // wait for all copies that it has under way. The first tile that comes so:
      const int rows_from = S::kConvert ? t1 : a.box == 0 ? t0 : g.tokens % a.box == 0 ? t1 : g.tokens / kTokens;
      if (jobs > 0) wait(b_query, seg);
      const uint32_t q0 = operand_lo(base, 16);
      const uint32_t kv0 = operand_lo(base + kTiles * S::kQ, 16), v00 = operand_lo(base + kTiles * S::kQ, kBlock);
      for (int j = 0; j < jobs + 2; ++j) {
        if (s_dead) break;
        if (j >= 2) {
          const int jj = j - 2, b = jj & 1, t = u.both ? jj >> 1 : jj;
          const uint32_t entry = 2 * (seq + t) + 1, stage = entry % kStages;
          wait(b_weight + 8 * b, done[b] + (jj >> 1));
          wait(b_full + 8 * stage, entry / kStages);
          if (t0 + t >= rows_from) proxy_fence_smem();  // what threads wrote and the barrier has shown, before the products read it
          tcgen05_after_sync();
          const uint32_t d = tmem + S::kSums + (kTiles == 2 ? b * DP : 0), w = tmem + b * kTokens, v0 = v00 + stage * (S::kStage >> 4);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < kTokens / 16; ++k) {
              const uint32_t p16 = kSecond ? w + 32 * (k >> 1) + 8 * (k & 1) : w + 8 * k;
              tcgen05_mma_ta(d, p16, v0 + 128 * k, kOperandHi, kValue, jj >= kTiles || k > 0);
              if (kSecond) tcgen05_mma_ta(d, p16 + 16, v0 + 128 * k, kOperandHi, kValue, true);
            }
            tcgen05_commit(b_sum + 8 * b);
            if (!u.both || b == 1) tcgen05_commit(b_free + 8 * stage);
          }
          __syncwarp();
        }
        if (j < jobs) {
          const int b = j & 1, t = u.both ? j >> 1 : j;
          const uint32_t entry = 2 * (seq + t), stage = entry % kStages;
          wait(b_full + 8 * stage, entry / kStages);
          if (t0 + t >= rows_from) proxy_fence_smem();
          tcgen05_after_sync();
          const uint32_t d = tmem + b * kTokens, k0 = kv0 + stage * (S::kStage >> 4), qa = q0 + (u.both ? b * (S::kQ >> 4) : 0);
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
              if (k < ksteps) tcgen05_mma(d, qa + (k >> 2) * (kQBlock >> 4) + 2 * (k & 3), k0 + (k >> 2) * (kBlock >> 4) + 2 * (k & 3), kOperandHi, kScore, k > 0);
            tcgen05_commit(b_score + 8 * b);
            if (!u.both || b == 1) tcgen05_commit(b_free + 8 * stage);
          }
          __syncwarp();
        }
      }
     });
    }
  } else {
    walk([&](const PrefixGroup& g, const PrefixUnit& u, int t0, int t1, int jobs) {
      const int h = u.h;
      const int32_t* bt_row = a.bt + (int64_t)g.lead * a.maxp;
      const int64_t slot = u.slot + (int64_t)team * (kPrefixRows * kTiles);
      // ---- softmax ------------------------------------------------------------------------------------
      const int acc = warp >> 2, row = (warp & 3) * 32 + lane;        // accumulator, TMEM lane
      const uint32_t lanes = (uint32_t)(warp & 3) << 21;
      const int my_row = u.both ? acc * kPrefixRows + row : row;      // of the unit
      const bool live = my_row < u.rows;
      if (jobs > 0) {
        // Q of the segment before is done with: both accumulators' last products have been waited for
        asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory");
        if (u.both || acc == 0) {
          const uint8_t* mine = nullptr;
          if (live) {
            const int gr = u.first_row + my_row, member = gr / a.G;
            int r = a.plan[TOPKV_PLAN_ORDER * a.R + g.place + member];
            r = min(max(r, 0), a.R - 1);
            mine = a.q + r * a.q_req + ((int64_t)h * a.G + gr - member * a.G) * a.q_head;
          }
          // kLanes lanes bring a row, so that a warp's accesses cover whole rows
          constexpr int kLanes = DP / 8, kPer = 32 / kLanes;
          const int chunks = a.D / 8, padded = ksteps * 2, c = lane % kLanes, sub = lane / kLanes;
          const uint32_t tile = base + (u.both ? acc * S::kQ : 0) + (warp & 3) * 32 * 128;
#pragma unroll 4
          for (int k = 0; k < 32; k += kPer) {
            const int rw = k + sub;
            const uint8_t* src = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), rw));
            const bool ok = src != nullptr && c < chunks;
            if (c < padded) cp_async16(tile + (c >> 3) * kQBlock + rw * 128 + (((c & 7) ^ (rw & 7)) << 4), ok ? src + c * 16 : a.q, ok);
          }
          cp_async_commit();
          cp_async_wait<0>();
          __syncwarp();
          // Scores times a factor that is not negative (a sign goes into Q); bf16 queries over 8-bit keys
          // become fp16 ones after a power of two for the row, see the kernel of the other tokens. A row a thread.
          float row_scale = fabsf(a.qk_scale);
          const uint32_t flip = a.qk_scale < 0.f ? 0x80008000u : 0u;
          const bool halves = TYPE == kE4m3 && a.io_bf16;
          if (halves || flip) {
            uint8_t* const at = smem + (tile - base) + lane * 128;
            float up = 1.f, rest = 1.f;
            if (halves) {
              float top = 0.f;
#pragma unroll 1
              for (int k = 0; k < chunks; ++k) {
                const uint4 v = *reinterpret_cast<const uint4*>(at + (k >> 3) * kQBlock + (((k & 7) ^ (lane & 7)) << 4));
                const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  top = fmaxf(top, fmaxf(fabsf(__uint_as_float(x[e] << 16)), fabsf(__uint_as_float(x[e] & 0xffff0000u))));
              }
              int e = 0;
              if (top > 0.f && top < INFINITY) e = ilogbf(top);
              // in two steps: a single factor of 2^-e may itself leave the range of a float
              up = exp2f((float)(-(e / 2)));
              rest = exp2f((float)(-(e - e / 2)));
              row_scale = row_scale * exp2f((float)(e / 2)) * exp2f((float)(e - e / 2));
            }
#pragma unroll 1
            for (int k = 0; k < chunks; ++k) {
              uint4* const v = reinterpret_cast<uint4*>(at + (k >> 3) * kQBlock + (((k & 7) ^ (lane & 7)) << 4));
              uint32_t x[4] = {v->x, v->y, v->z, v->w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if (halves)
                  x[e] = pack2<false>(__uint_as_float(x[e] << 16) * up * rest, __uint_as_float(x[e] & 0xffff0000u) * up * rest);
                x[e] ^= flip;
              }
              *v = make_uint4(x[0], x[1], x[2], x[3]);
            }
          }
          // Nor zero, as a product of small factors may be: masked scores are minus infinity before it is applied.
          ctl.row_scale[my_row] = fmaxf(row_scale, FLT_MIN);
          proxy_fence_smem();
        }
        tcgen05_before_sync();
        asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory");
        bar_arrive(b_query);
      }
      const float row_scale = ctl.row_scale[my_row];
      const bool some = __any_sync(0xffffffffu, live);  // a row of this warp counts
      float m = -INFINITY, l = 0.f, sub = 0.f;          // sub: what is subtracted from a score
      bool seen = false;
      int last = -1;  // this accumulator's last job
      for (int j = kTiles == 2 ? acc : 0; j < jobs; j += kTiles) {
        const int b = j & 1, t = t0 + (u.both ? j >> 1 : j);
        const uint32_t s_col = tmem + lanes + b * kTokens;
        wait(b_score + 8 * b, done[b] + (j >> 1));
        // no phase of a barrier is left out, since a wait tells them apart by parity alone
        if (j >= 2) wait(b_sum + 8 * b, done[b] + (j >> 1) - 1);
        if (__any_sync(0xffffffffu, s_dead)) break;
        tcgen05_after_sync();
        last = j;
        if (some) {
          // which of 32 tokens count; pages outside the pool are not visible, from the first one on every tile asks
          const int visible = g.tokens - t * kTokens;
          const bool odd = ctl.odd, partial = odd || visible < kTokens;
          auto valid = [&](int c) {
            const int n = visible - c * 32;
            uint32_t bits = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1;
            if (odd) {
              const int x = t * kTokens + c * 32 + lane;
              const int page = x < g.tokens ? bt_row[page_column(x)] : -1;
              bits &= __ballot_sync(0xffffffffu, page >= 0 && page < a.num_pages);
            }
            return bits;
          };
          // Two passes over the scores, whose code is kept short: it is fetched anew at every launch, at 9 cycles an
          // instruction (unrolled over the whole row, in variants, the first tiles took 9,000 cycles each).
          auto mask = [&](uint32_t (&x)[32], uint32_t bits) {
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (!(bits >> k & 1)) x[k] = 0xff800000u;  // minus infinity
          };
          float top = -INFINITY;
          uint32_t counted = 0;
          {
            uint32_t x[2][32];
            tmem_load<32>(x[0], s_col);
#pragma unroll 1
            for (int c = 0; c < kTokens / 32; c += 2) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                tmem_loaded(x[i]);
                if (i == 0 || c + 2 < kTokens / 32) tmem_load<32>(x[i ^ 1], s_col + (c + i + 1) * 32);
                if (partial) {
                  const uint32_t bits = valid(c + i);
                  counted |= bits;
                  if (bits != 0xffffffffu) mask(x[i], bits);
                }
                float part[2] = {top, -INFINITY};
#pragma unroll
                for (int k = 0; k < 32; k += 2) part[k / 2 & 1] = max3(part[k / 2 & 1], __uint_as_float(x[i][k]), __uint_as_float(x[i][k + 1]));
                top = fmaxf(part[0], part[1]);
              }
            }
          }
          seen |= !partial || counted != 0;
          top = top == -INFINITY ? top : top * row_scale;
          // The reference moves only when it is exceeded by more than 2^kLazy.
          if (__any_sync(0xffffffffu, top > m + kLazy)) {
            float alpha = 1.f;
            if (top > m) {
              alpha = exp2_approx(m - top);
              m = top;
              sub = m - kShift;
            }
            l *= alpha;
            if (j >= kTiles) {
              // With two accumulators the scores' arrival says that this one's products have ended, with one
              // those of the job before may still be running.
              if (kTiles == 1) {
                wait(b_sum + 8 * (b ^ 1), done[b ^ 1] + ((j - 1) >> 1));
                tcgen05_after_sync();
              }
#pragma unroll 1
              for (int c = 0; c * 32 < a.D; ++c) {
                uint32_t o[32];
                tmem_load<32>(o, tmem + lanes + S::kSums + acc * DP + c * 32);
                tmem_loaded(o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                tmem_store<32>(tmem + lanes + S::kSums + acc * DP + c * 32, o);
              }
            }
          }
          const float2 by = make_float2(row_scale, row_scale), less = make_float2(-sub, -sub);
          float2 sum[2] = {make_float2(l, 0.f), make_float2(0.f, 0.f)};
          {
            uint32_t x[2][32];
            tmem_load<32>(x[0], s_col);
#pragma unroll 1
            for (int c = 0; c < kTokens / 32; c += 2) {
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                tmem_loaded(x[i]);
                if (i == 0 || c + 2 < kTokens / 32) tmem_load<32>(x[i ^ 1], s_col + (c + i + 1) * 32);
                if (partial) {
                  const uint32_t bits = valid(c + i);
                  if (bits != 0xffffffffu) mask(x[i], bits);
                }
                uint32_t w[kSecond ? 32 : 16];
#pragma unroll
                for (int k = 0; k < 32; k += 2) {
                  float2 e = fma2(make_float2(__uint_as_float(x[i][k]), __uint_as_float(x[i][k + 1])), by, less);
                  e.x = exp2_approx(e.x);
                  e.y = exp2_approx(e.y);
                  sum[k / 2 & 1] = add2(sum[k / 2 & 1], e);
                  w[k / 2] = pack2<kBf>(e.x, e.y);
                  if constexpr (kSecond)
                    w[16 + k / 2] = pack2<true>(e.x - __uint_as_float(w[k / 2] << 16), e.y - __uint_as_float(w[k / 2] & 0xffff0000u));
                }
                // over scores that have been read; with what the weights' rounding cut off beside them
                tmem_store<kSecond ? 32 : 16>(s_col + (c + i) * (kSecond ? 32 : 16), w);
              }
            }
          }
          sum[0] = add2(sum[0], sum[1]);
          l = sum[0].x + sum[0].y;
          tmem_wait_store();
        }
        tcgen05_before_sync();
        bar_arrive(b_weight + 8 * b);
      }
      // ---- the segment's part --------------------------------------------------------------------------
      // Every accumulator of the unit leaves one: of its rows, or of the same rows and other tokens.
      if (last >= 0) {
        if (kTiles == 1 && last > 0) wait(b_sum + 8 * ((last - 1) & 1), done[(last - 1) & 1] + ((last - 1) >> 1));
        wait(b_sum + 8 * (last & 1), done[last & 1] + (last >> 1));
        tcgen05_after_sync();
      }
      const int64_t to = slot + (u.both || acc == 0 ? my_row : u.rows + my_row);
      if (live) p.ml[to] = make_float2(m - kShift, seen ? l : kNoneSeen);
      // Rows leave by way of shared memory, where Q is not needed any more once both accumulators have come here:
      // a warp's 32 rows of kWide columns, 16-byte chunks permuted by row, then whole rows at a time. (A row per
      // thread straight to memory: 8,000 cycles a segment.)
      if (jobs > 0) asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxThreads) : "memory");
      if (last >= 0 && some) {
        constexpr int kWide = DP / 2, kChunks = kWide / 4, kPer = 32 / kChunks;  // columns, their chunks, rows per access
        uint8_t* const mine = smem + (acc * 4 + (warp & 3)) * (32 * kWide * 4);
        const int rows_here = min(32, u.rows - (u.both ? acc * kPrefixRows : 0) - (warp & 3) * 32);
        const int c = lane % kChunks, sub = lane / kChunks;
#pragma unroll 1
        for (int half = 0; half < 2 && half * kWide < a.D; ++half) {
#pragma unroll 1
          for (int k = 0; k < kWide / 32; ++k) {
            uint32_t o[32];
            tmem_load<32>(o, tmem + lanes + S::kSums + acc * DP + half * kWide + k * 32);
            tmem_loaded(o);
#pragma unroll
            for (int e = 0; e < 8; ++e)
              *reinterpret_cast<uint4*>(mine + lane * (kWide * 4) + (((k * 8 + e) ^ (lane & (kChunks - 1))) << 4)) =
                  make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
          __syncwarp();
          float* const out = p.part + (to - lane) * a.Dv + half * kWide;
#pragma unroll 4
          for (int r0 = 0; r0 < 32; r0 += kPer) {
            const int rw = r0 + sub, at = c ^ (rw & (kChunks - 1));
            const uint4 v = *reinterpret_cast<const uint4*>(mine + rw * (kWide * 4) + (c << 4));
            if (rw < rows_here && half * kWide + at * 4 < a.D)
              *reinterpret_cast<uint4*>(out + (int64_t)rw * a.Dv + at * 4) = v;
          }
          __syncwarp();
        }
      }
      tcgen05_before_sync();
    });
  }
  cp_async_wait<0>();
  if (s_dead) {  // give the copies and products that are in flight a millisecond to end
    const long long began = clock64();
    while (clock64() - began < 2000000) __nanosleep(1000);
  }
  tcgen05_before_sync();
  __syncthreads();
  if (warp == kIssueWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
}

// ---- join -------------------------------------------------------------------------------------------
// A CTA takes up to kJoinRows heads of a request and KV head: parts of the tokens behind the prefix, then those
// of the prefix, in order. First a warp per row turns the parts' maxima and sums into weights, then threads add up
// four columns of a row each, several of them a row's parts in turns where they would have nothing to do. (The whole
// call, 8 requests behind 8,192 tokens: 40 us, 59 with a thread per four columns and parts in a row.)
constexpr int kPrefixJoinThreads = 256;
constexpr int kPrefixJoinParts = kJoinParts + 2 * kPrefixCtas;
__global__ void __launch_bounds__(kPrefixJoinThreads, 4) topkv_prefix_join_kernel(const PrefixParams p) {
  __shared__ float s_w[kJoinRows][kPrefixJoinParts];
  __shared__ int64_t s_first[kJoinRows];
  __shared__ int s_half[kJoinRows], s_teams[kJoinRows];
  __shared__ float4 s_sum[kPrefixJoinThreads];
  const AttendParams& a = p.a;
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = blockIdx.x, unit = blockIdx.y;
  const int4 rec = a.joins[r];
  const PrefixHeader t = *p.header;
  const int lead = rec.x, behind = rec.z, units = gridDim.y;
  if (behind < 0) return;  // written
  const int h = unit / a.gtiles, g0 = (unit - h * a.gtiles) * a.row_tile;
  const int per = (a.rows + gridDim.z - 1) / gridDim.z, row0 = blockIdx.z * per;
  const int rows = min(per, min(a.G - g0, a.row_tile) - row0);
  if (rows <= 0) return;
  PrefixGroup g = {};
  if (lead >= 0) g = p.groups[lead];
  const int64_t q_head0 = (int64_t)h * a.G + g0 + row0;
  // Where the parts of row `row` lie: those behind the prefix at a constant stride; of the prefix one to a team, or
  // two, `half` rows apart, where the accumulators hold the same rows.
  const int64_t b_first = ((int64_t)rec.y * units + unit) * a.rows + row0;
  const int b_step = units * a.rows, p_step = kPrefixRows * p.tiles;
  const int quads = a.Dv / 4, items = rows * quads;
  if (tid < rows) {
    int64_t first = 0;
    int half = 0, teams = 0;
    const int mine_at = rec.w * a.G + g0 + row0 + tid;
    if (lead >= 0 && t.teams > 0 && mine_at >= 0 && mine_at < g.rows) {
      const int i = mine_at / p_step;
      const PrefixUnit u = prefix_unit(p, g, h, i);
      const int pos = g.begin + h * g.length + i * g.full, t0 = prefix_team_of(t, pos);
      teams = prefix_team_of(t, pos + u.length - 1) - t0 + 1;
      first = u.slot + (int64_t)t0 * p_step + mine_at - u.first_row;
      half = u.both || p.tiles == 1 ? 0 : u.rows;
    }
    s_first[tid] = first;
    s_half[tid] = half;
    s_teams[tid] = teams;
  }
  __syncthreads();
  // part k of a row's columns d ..
  auto part_of = [&](int row, int d, int k) {
    if (k < behind) return reinterpret_cast<const float4*>(a.part + (b_first + row + (int64_t)k * b_step) * a.Dv + d);
    const int teams = s_teams[row], second = k - behind >= teams;
    return reinterpret_cast<const float4*>(p.part + (s_first[row] + second * s_half[row] + (int64_t)(k - behind - second * teams) * p_step) * a.Dv + d);
  };
  auto parts_of = [&](int row) { return behind + (s_half[row] > 0 ? 2 : 1) * s_teams[row]; };
  // Where there are more threads than items, several share an item's parts: part k goes to thread k % split. The first
  // parts of a thread's first item are under way while the weights are formed.
  constexpr int kAhead = 6;
  const int split = max(1, kPrefixJoinThreads / items), turn = split > 1 ? tid / items : 0;
  float4 ahead[kAhead];
  auto fetch = [&](int row, int d, int from, int parts) {  // parts from, from + split, ..; behind the last one the last one again
#pragma unroll
    for (int e = 0; e < kAhead; ++e) ahead[e] = *part_of(row, d, min(from + e * split, parts - 1));
  };
  const int item = tid - turn * items;
  if (item < items && turn < split) {
    const int row = item / quads, parts = parts_of(row);
    if (turn < parts) fetch(row, (item - row * quads) * 4, turn, parts);
  }
  for (int row = warp; row < rows; row += kPrefixJoinThreads / 32) {
    const int64_t first = s_first[row];
    const int half = s_half[row], teams = s_teams[row], parts = parts_of(row);
    // parts in the order: behind the prefix, the teams' first, the teams' second
    auto ml_of = [&](int k) {
      if (k < behind) return a.ml[b_first + row + (int64_t)k * b_step];
      k -= behind;
      return k < teams ? p.ml[first + (int64_t)k * p_step] : p.ml[first + half + (int64_t)(k - teams) * p_step];
    };
    // the first 32 parts are held by the lanes, the others read twice
    float2 held = make_float2(-INFINITY, kNoneSeen);
    if (lane < parts) held = ml_of(lane);
    float top = held.y != kNoneSeen ? held.x : -INFINITY, sum = 0.f;
    bool seen = held.y != kNoneSeen;
    for (int k = lane + 32; k < parts; k += 32) {
      const float2 ml = ml_of(k);
      if (ml.y != kNoneSeen) {
        seen = true;
        top = fmaxf(top, ml.x);
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float from = top == -INFINITY ? 0.f : top;
    const float mine = held.y != kNoneSeen ? exp2_approx(held.x - from) : 0.f;
    if (held.y != kNoneSeen) sum = mine * held.y;
    for (int k = lane + 32; k < parts; k += 32) {
      const float2 ml = ml_of(k);
      const float w = ml.y != kNoneSeen ? exp2_approx(ml.x - from) : 0.f;
      if (ml.y != kNoneSeen) sum += w * ml.y;
      s_w[row][k] = w;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    seen = __any_sync(0xffffffffu, seen);
    const float inv = seen ? a.v_scale / sum : 0.f;
    if (lane < parts) s_w[row][lane] = mine * inv;
    for (int k = lane + 32; k < parts; k += 32) s_w[row][k] *= inv;
    if (lane == 0 && a.lse != nullptr) a.lse[(int64_t)r * a.H * a.G + q_head0 + row] = seen ? (top + log2f(sum)) * kLn2 : -INFINITY;
  }
  __syncthreads();
  for (int i = item; i < items && turn < split; i += kPrefixJoinThreads) {
    const int row = i / quads, d = (i - row * quads) * 4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* w = s_w[row];
    const int parts = parts_of(row);
    for (int k = turn; k < parts; k += kAhead * split) {
      if (k != turn || i != item) fetch(row, d, k, parts);
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        // a part without weight may not have been written; no branch, so that the loads stay together
        const float f = k + e * split < parts ? w[k + e * split] : 0.f;
        acc.x = f != 0.f ? acc.x + f * ahead[e].x : acc.x;
        acc.y = f != 0.f ? acc.y + f * ahead[e].y : acc.y;
        acc.z = f != 0.f ? acc.z + f * ahead[e].z : acc.z;
        acc.w = f != 0.f ? acc.w + f * ahead[e].w : acc.w;
      }
    }
    if (split > 1) {
      s_sum[tid] = acc;
    } else {
      store_io4(a.out + r * a.o_req + (q_head0 + row) * a.o_head + d * 2, acc, 1.f, a.io_bf16);
    }
  }
  if (split == 1) return;
  __syncthreads();
  if (tid >= items) return;
  float4 acc = s_sum[tid];
  for (int k = 1; k < split; ++k) {
    const float4 v = s_sum[tid + k * items];
    acc.x += v.x;
    acc.y += v.y;
    acc.z += v.z;
    acc.w += v.w;
  }
  const int row = tid / quads;
  store_io4(a.out + r * a.o_req + (q_head0 + row) * a.o_head + (tid - row * quads) * 8, acc, 1.f, a.io_bf16);
}

}  // namespace topkv

// Attention of one new token over a cache of latent rows (multi-head latent attention in its absorbed
// form): every row is the key of all query heads and, in its first Dv elements, their value too.
//
//   x_i[a] = scale * q[a] . row[i]      out[a] = sum_i exp(x_i[a] - m) row[i][0:Dv] / l
//
// With 128 query heads a row of 1,152 bytes is used for 278 kflop, 242 flop a byte: bandwidth and
// tensor rate bind together, so this runs on the tensor memory path (tcgen05). Both products are
// formed transposed, with the cache as the A operand and the heads as the N columns:
//
//   S^T [64 tokens x N heads]  = rows [64 x D] * Q^T              (K-major A, K-major B)
//   O^T [Dv x N heads]        += rows^T [Dv x 64] * P^T           (M-major A, N-major B)
//
// so that one copy of the rows in shared memory (128-byte swizzle, 64 columns a block) serves both,
// the accumulator of 512 x N values fills TMEM lane by lane, N can follow the number of heads
// (16, 32, 64: a rank of a head-parallel model has 16), and a step of the second product has all 128
// rows of the tensor core busy, which N = 64 heads as rows would not have.
//
// A CTA has 64 or fewer heads of a request and takes the token tiles of its team, like the
// grouped-head kernel (same sharing-out, same join). More heads are more CTAs of the team, which read
// the same rows at about the same time, from L2. Roles:
//   warps 0-7   softmax: two warps per 32-lane quarter of TMEM, each with half of the heads; also
//               load Q, rescale and write out the accumulator
//   warps 8-11  load: two stages of 64 rows, one pair of warps each, through the block table: tensor
//               copies for full tiles, 16-byte copies for the rest (any page size and stride;
//               what is masked becomes zero)
//   warps 12, 13 one thread each issues the matrix instructions of the first and of the second product
// Running maxima move only when a tile exceeds them by more than 2^8, so the accumulator is rescaled
// a few times per request and not once per tile; the weights are at most 2^8 (fp16: scaled by
// 2^7, to stay below 2^15), which costs no precision in a floating type.
// Every wait on a barrier is bounded; one that runs out raises error bit 1 and lets the CTA finish. The
// allocation of TMEM waits for CTAs that hold it, which all end by themselves: the next launch is let in
// only once every CTA of this one has its share.
// Measured, 576 / 512 columns in bf16: 32 requests of 1,024 to 8,192 tokens, 128 heads: 75 us in bursts
// of 200 calls at 1.9 GHz, 80 in a run of seconds, where the power cap holds the clock at 1.78, 0.5 Pflop/s
// (0.64 at 16,384 tokens each), a tile of 64 tokens and 64 heads in 2,930 cycles, of which the tensor core
// needs 2,070; 16 heads, 32 x 16,384 tokens: 107 us = 5.6 TB/s. What remains is the time from giving up a
// stage to having it loaded again (2,000 cycles) in a ring of two: a third does not fit beside Q.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "topkv_attend.cuh"
#include "topkv_common.cuh"

namespace topkv {

constexpr int kLatentTile = 64;                  // tokens per tile
static_assert(kLatentTile == kTileTokens, "both kernels share out tiles of the same size");
constexpr int kSoftmaxWarps = 8, kLoadWarps = 4;
constexpr int kScoreWarp = kSoftmaxWarps + kLoadWarps, kValueWarp = kScoreWarp + 1;
constexpr int kLatentThreads = (kValueWarp + 1) * 32;
constexpr int kLatentBlock = kLatentTile * 128;  // bytes of 64 columns of a tile
constexpr int kLatentMaxD = 576, kLatentMaxDv = 512;
constexpr long long kWaitClocks = 1000000000ll;  // about half a second

template <int N>
__device__ __forceinline__ void tmem_load(uint32_t (&v)[N], uint32_t a);
template <int N>
__device__ __forceinline__ void tmem_store(uint32_t a, const uint32_t (&v)[N]);
template <>
__device__ __forceinline__ void tmem_load<8>(uint32_t (&v)[8], uint32_t a) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(a));
}
template <>
__device__ __forceinline__ void tmem_store<8>(uint32_t a, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

template <>
__device__ __forceinline__ void tmem_load<16>(uint32_t (&v)[16], uint32_t a) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
                 "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
                 "=r"(v[14]), "=r"(v[15])
               : "r"(a));
}
template <>
__device__ __forceinline__ void tmem_store<16>(uint32_t a, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}

template <>
__device__ __forceinline__ void tmem_load<32>(uint32_t (&v)[32], uint32_t a) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
                 "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
                 "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
                 "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
                 "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
               : "r"(a));
}
template <>
__device__ __forceinline__ void tmem_store<32>(uint32_t a, const uint32_t (&v)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}

// The 16 lanes of a quarter that hold scores, over all 32 threads: thread t gets, of columns
// 8 i + 2 (t % 4) and the next, row t / 4 in v[4 i], v[4 i + 1] and row t / 4 + 8 in v[4 i + 2], v[4 i + 3].
template <int N>
__device__ __forceinline__ void tmem_load_half(uint32_t (&v)[N], uint32_t a);
template <>
__device__ __forceinline__ void tmem_load_half<4>(uint32_t (&v)[4], uint32_t a) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
               : "r"(a));
}
template <>
__device__ __forceinline__ void tmem_load_half<8>(uint32_t (&v)[8], uint32_t a) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
               : "r"(a));
}
template <>
__device__ __forceinline__ void tmem_load_half<16>(uint32_t (&v)[16], uint32_t a) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
                 "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
                 "=r"(v[14]), "=r"(v[15])
               : "r"(a));
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// Operand descriptors are two words; only the low one (address, leading stride) differs between the
// steps of a product, so the steps cost one addition each.
__device__ __forceinline__ void tcgen05_mma(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{ .reg .pred p; .reg .b64 da, db; mov.b64 da, {%1, %3}; mov.b64 db, {%2, %3}; setp.ne.u32 p, %5, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p; }" ::"r"(d),
      "r"(a), "r"(b), "r"(hi), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void proxy_fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Barrier `id` of `threads` threads; whether the predicate holds for any of them.
__device__ __forceinline__ bool bar_any(int id, int threads, bool pred) {
  uint32_t r;
  asm volatile("{ .reg .pred p, q; setp.ne.u32 p, %3, 0; bar.red.or.pred q, %1, %2, p; selp.u32 %0, 1, 0, q; }"
               : "=r"(r)
               : "r"(id), "r"(threads), "r"((uint32_t)pred)
               : "memory");
  return r != 0;
}
// Box of the tensor map at (x, y, z) into shared memory (bytes counted by the barrier), or into L2 only.
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_prefetch(const CUtensorMap* map, int x, int y, int z) {
  asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global.tile [%0, {%1, %2, %3}];" ::"l"(map), "r"(x), "r"(y), "r"(z)
               : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(p));
  return p != 0;
}
// Joins C values of each thread over the eight threads t, t ^ 4, t ^ 8, ... of a warp: as long as a
// thread holds several columns, each step hands half of them over and joins the others. What is left
// is one column per thread, number `column_of` of the thread's own.
template <int C, typename Op>
__device__ __forceinline__ float join_rows(float (&v)[C], int lane, Op op) {
  int bit = 4;
#pragma unroll
  for (int n = C / 2; n >= 1; n /= 2, bit *= 2) {
    const bool up = lane & bit;
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float give = up ? v[j] : v[j + n];
      const float keep = up ? v[j + n] : v[j];
      v[j] = op(keep, __shfl_xor_sync(0xffffffffu, give, bit));
    }
  }
#pragma unroll
  for (; bit < 32; bit *= 2) v[0] = op(v[0], __shfl_xor_sync(0xffffffffu, v[0], bit));
  return v[0];
}
template <int C>
__device__ __forceinline__ int column_of(int lane) {  // 2 i + e, of column 8 i + 2 (lane % 4) + e
  int j = 0, bit = 4;
#pragma unroll
  for (int n = C / 2; n >= 1; n /= 2, bit *= 2) j |= (lane & bit) ? n : 0;
  return (j >> 1) * 8 + (lane & 3) * 2 + (j & 1);
}
// Shared-memory operand, 128-byte swizzle, 1,024 bytes from eight rows to the next eight; `lead` in bytes.
__device__ __forceinline__ uint32_t operand_lo(uint32_t addr, uint32_t lead) { return (addr & 0x3ffff) >> 4 | lead >> 4 << 16; }
constexpr uint32_t kOperandHi = 1024 >> 4 | 1u << 14 | 2u << 29;

// Layout of the dynamic shared memory. All operand blocks are multiples of 1,024 bytes.
struct LatentControl {
  float red[2 * 4 * 64];  // maxima and sums per quarter of TMEM and head, by turns
  uint64_t bar[15];
  TeamStart team;
  uint32_t valid[2][2];   // which of a stage's tokens count
  uint32_t tmem;
  volatile int dead;      // a wait ran out
};
struct LatentSmem {
  uint32_t q, kv, control, total;
  uint32_t p, p_step;  // weights of the first stage's tile, and from there to the second's
  uint32_t stage;      // bytes of a stage
};
__host__ __device__ constexpr LatentSmem latent_smem(int N, int D, int Dv) {
  const int blocks = (D + 63) / 64, vblocks = (Dv + 127) / 128 * 2;
  LatentSmem s = {};
  s.stage = (uint32_t)((blocks > vblocks ? blocks : vblocks) * kLatentBlock);
  s.q = 0;
  s.kv = (uint32_t)(blocks * N * 128);
  // The weights of a tile (64 tokens x 128 bytes) take the place of its first block behind the values,
  // which only the scores need; rows without such a block get two buffers.
  const bool inside = blocks > vblocks;
  s.p = s.kv + (inside ? (uint32_t)(vblocks * kLatentBlock) : 2 * s.stage);
  s.p_step = inside ? s.stage : (uint32_t)kLatentBlock;
  s.control = s.kv + 2 * s.stage + (inside ? 0 : 2 * kLatentBlock);
  s.total = s.control + (uint32_t)sizeof(LatentControl);
  return s;
}

// What a load warp waits for before it fills a stage again: the group of its i-th wait, -1 behind the last.
// A barrier tells its phases apart by parity only, so a wait that lies two phases back passes at once: no
// warp may wait for a group whose release of the tile before it has not seen. Products end in order, so
// the release of group 0 implies that of all groups one tile earlier; both lists therefore begin with it.
__host__ __device__ constexpr int rows_await(int i, int vblocks) {  // ..., then the last: the whole stage is free
  return i == 0 ? 0 : i == 1 && vblocks > 1 ? vblocks - 1 : -1;
}
__host__ __device__ constexpr int pieces_await(int i, int half, int vblocks) {  // ..., then the groups that the warp brings
  return i == 0 ? 0 : half + 2 * (i - 1) < vblocks ? half + 2 * (i - 1) : -1;
}

template <int N, bool BF16>
__global__ void __launch_bounds__(kLatentThreads, 1) topkv_latent_kernel(const AttendParams p, const __grid_constant__ CUtensorMap map, const __grid_constant__ CUtensorMap q_map) {
  constexpr int NC = N / 2;                       // heads per softmax warp
  constexpr int C = NC / 4;                       // ... per thread of it
  constexpr float kShift = BF16 ? 0.f : 7.f;
  constexpr uint32_t kCols = N == 64 ? 512 : N * 8;  // TMEM columns: 2 N for S^T, 4 N for O^T, a power of two
  extern __shared__ __align__(128) uint8_t smem[];

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int team = blockIdx.x, unit = blockIdx.y;
  const int g0 = unit * N, rows = min(p.G - g0, N);
  const uint32_t base = smem_addr(smem);
  if (base & 1023) {  // the swizzle wants 1,024; without static shared memory the base is there
    if (threadIdx.x == 0) raise_error(kErrWait);
    return;
  }
  const LatentSmem lay = latent_smem(N, p.D, p.Dv);
  LatentControl& ctl = *reinterpret_cast<LatentControl*>(smem + lay.control);
  volatile int& s_dead = ctl.dead;
  float* const s_red = ctl.red;  // [2][quarter][head]

  const int ksteps = (p.D + 15) / 16, vblocks = (p.Dv + 127) / 128;
  const int blocks = (p.D + 63) / 64;
  // Barriers. The blocks of a stage are given up in groups, one per 128 value columns (the blocks
  // behind the values, which hold the weights by then, belong to the last): a group is loaded again
  // while the products of the next one still run.
  //   rows loaded [2], rows used [2][4], scores ready [2], weights written [2], Q written
  const uint32_t bar0 = smem_addr(ctl.bar);
  const uint32_t b_full = bar0, b_free = bar0 + 16, b_score = bar0 + 80, b_weight = bar0 + 96, b_query = bar0 + 112;
  const int last = vblocks - 1;  // the group whose products come last
  if (tid == 0) {
    s_dead = 0;
    for (int i = 0; i < 2; ++i) {
      mbar_init(b_full + 8 * i, 64);
      mbar_init(b_score + 8 * i, 1);
      mbar_init(b_weight + 8 * i, kSoftmaxWarps * 32);
    }
    for (int i = 0; i < 8; ++i) mbar_init(b_free + 8 * i, 1);
    mbar_init(b_query, p.q_box ? 1 : kSoftmaxWarps * 32);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kScoreWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)), "n"(kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    tcgen05_before_sync();
  }
  if (!p.late_wait) pdl_wait_prior_grid();
  const TeamRange mine = team_range<kLatentThreads>(p, team, &ctl.team);
  if (p.late_wait) pdl_wait_prior_grid();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = ctl.tmem;
  // Not before this CTA has its TMEM: a CTA of the next launch that found room on this SM would hold some
  // while it waits for this grid, and a CTA of this grid could ask in vain.
  pdl_release_next_grid();
  const bool records = !p.uncut && unit == 0 && tid == 0;
  if (records && !p.by_request) write_join(p, 0, team, 0, 0);
  empty_requests<kLatentThreads>(p, team, (int64_t)g0, rows, unit == 0);

  // Waits until the barrier has completed its phase number `phase` (0, 1, 2, ...).
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

  constexpr uint32_t kType = 1u << 4 | (BF16 ? 1u : 0u) << 7 | (BF16 ? 1u : 0u) << 10 | (uint32_t)(N >> 3) << 17;
  uint32_t n = 0;    // tiles before the current segment, in this CTA: they number the phases
  uint32_t seg = 0;  // segments before
  int64_t left = mine.left, off = mine.off;  // left 0: no tiles
  bool first = true;
  for (int r = mine.r; left > 0 && r < p.R; ++r) {
    const Visible vis = visible_tokens(p, r, false);
    const int tiles = attend_tiles(vis.n);
    if (tiles == 0) {
      if (p.uncut) break;
      continue;
    }
    int t0, t1;
    const int64_t taken = tiles_in_range(p, tiles, off, left, &t0, &t1);
    if (records && t0 == 0 && t1 > 0) request_begins(p, ctl.team, team, r, first, mine.left - left - off, tiles, t1 == tiles);
    left -= taken;
    off = 0;
    const int count = t1 - t0;
    if (count == 0) continue;

    if (warp >= kSoftmaxWarps && warp < kSoftmaxWarps + kLoadWarps) {
      // ---- load: pair `g` of warps takes the stages g of its own parity ---------------------------
      const int g = (warp - kSoftmaxWarps) >> 1, half = (warp - kSoftmaxWarps) & 1;
      const int chunks = p.D / 8, padded = ksteps * 2;  // 16-byte chunks of a row, and up to the last k-step
      const int full = chunks / 8;                      // blocks that a row fills
      // A full tile of whole page pieces comes by tensor copies, one instruction per piece and block
      // of 64 columns, and its successor is brought to L2 meanwhile; any other tile comes by copies of
      // 16 bytes per thread. (Those alone, 43 cycles each to issue and 3,100 a tile: 100 us for 32
      // requests of 1,024 to 8,192 tokens and 128 heads, against 76 with tensor copies.)
      const int boxes = p.box > 0 ? kLatentTile / p.box : 0;  // pieces of a tile
      auto page_column = [&](int i) { return p.page_shift >= 0 ? i >> p.page_shift : i / p.P; };
      // Page and token of piece `lane` of tile i (tensor copies: no window, so token and place agree).
      auto piece = [&](int i, int* at) {
        *at = 0;
        const int v = (t0 + i) * kLatentTile + lane * p.box;
        if (i >= count || lane >= boxes || (int64_t)(t0 + i + 1) * kLatentTile > vis.n) return -1;
        const int j = page_column(v);
        *at = v - j * p.P;
        return p.bt[(int64_t)r * p.maxp + j];
      };
      int i = (g - (int)(n & 1)) & 1;
      int at, pg = piece(i, &at);
      for (; i < count; i += 2) {
        if (s_dead) break;
        const uint32_t k = n + i;
        const bool pieces = boxes > 0 && __all_sync(0xffffffffu, lane >= boxes || (pg >= 0 && pg < p.num_pages));
        if (pieces) {
          // ctl.valid of the tile before has been read when its products begin
          if (k >= 2) wait(b_free + 32 * g + 8 * pieces_await(0, half, vblocks), (k >> 1) - 1);
          // both warps come to the same answer; each takes every other group
          int own = half == (last & 1) ? max(blocks - 2 * vblocks, 0) : 0;  // blocks that this warp brings
          for (int v = half; v < vblocks; v += 2) own += min(2, blocks - 2 * v);
          if (lane == 0) {
            ctl.valid[g][half] = 0xffffffffu;
            mbar_expect_tx(b_full + 8 * g, (uint32_t)(own * kLatentBlock));
          } else {
            bar_arrive(b_full + 8 * g);
          }
          __syncwarp();
          const uint32_t dst = base + lay.kv + g * lay.stage;
          for (int w = 1, v; (v = pieces_await(w, half, vblocks)) >= 0; ++w) {
            if (k >= 2) wait(b_free + 32 * g + 8 * v, (k >> 1) - 1);
            for (int e = 0; e < boxes; ++e) {
              const int z = __shfl_sync(0xffffffffu, pg, e), y = __shfl_sync(0xffffffffu, at, e);
              if (elect_one()) {
                auto bring = [&](int b) {
                  tma_load(dst + b * kLatentBlock + e * p.box * 128, &map, b * 64, y, z, b_full + 8 * g);
                };
                bring(2 * v);
                if (2 * v + 1 < blocks) bring(2 * v + 1);
                if (v == last)
                  for (int b = 2 * vblocks; b < blocks; ++b) bring(b);
              }
              __syncwarp();
            }
          }
          pg = piece(i + 2, &at);
          if (__all_sync(0xffffffffu, lane >= boxes || (pg >= 0 && pg < p.num_pages))) {
            for (int e = 0; e < boxes; ++e) {
              const int z = __shfl_sync(0xffffffffu, pg, e), y = __shfl_sync(0xffffffffu, at, e);
              if (elect_one())
                for (int b = 2 * unit + half; b < blocks; b += 2 * gridDim.y) tma_prefetch(&map, b * 64, y, z);  // the team shares it
              __syncwarp();
            }
          }
          continue;
        }
        pg = piece(i + 2, &at);
        int64_t off = -1;
        const int place = (t0 + i) * kLatentTile + half * 32 + lane;
        if (place < vis.n) {
          const int tok = place < vis.ns ? place : place - vis.ns + vis.lo;
          const int j = page_column(tok), page = p.bt[(int64_t)r * p.maxp + j];
          if (page < 0 || page >= p.num_pages)
            raise_error(kErrTable);
          else
            off = (int64_t)page * p.S_page + (int64_t)(tok - j * p.P) * p.S_tok;
        }
        const uint32_t valid = __ballot_sync(0xffffffffu, off >= 0);
        if (k >= 2)
          for (int w = 0, v; (v = rows_await(w, vblocks)) >= 0; ++w) wait(b_free + 32 * g + 8 * v, (k >> 1) - 1);
        if (lane == 0) ctl.valid[g][half] = valid;
        // a warp-wide copy brings 128 bytes of four rows, so source and destination advance by a
        // constant from one block of 64 columns to the next
        const int c = lane & 7, sub = lane >> 3;
        const uint32_t dst = base + lay.kv + g * lay.stage + half * 32 * 128;
#pragma unroll 2
        for (int rg = 0; rg < 8; ++rg) {
          const int row = rg * 4 + sub;
          const int64_t o = __shfl_sync(0xffffffffu, off, row);
          const uint8_t* src = p.pool + (o < 0 ? 0 : o) + c * 16;
          uint32_t to = dst + row * 128 + ((c ^ (row & 7)) << 4);
#pragma unroll 3
          for (int b = 0; b < full; ++b, src += 128, to += kLatentBlock) cp_async16(to, src, o >= 0);
          if (full * 8 + c < padded) cp_async16(to, full * 8 + c < chunks ? src : p.pool, o >= 0 && full * 8 + c < chunks);
        }
        cp_async_commit();
        cp_async_wait<0>();
        proxy_fence_smem();
        bar_arrive(b_full + 8 * g);
      }
    } else if (warp == kScoreWarp) {
      // ---- scores -------------------------------------------------------------------------------------
      // The descriptors are formed by the whole warp and one elected thread issues: from inside a branch
      // of one thread each instruction took 70 cycles to issue, where the tensor core needs 35
      // (64 x 64) to 51 (128 x 64) for it. Two warps, one per product: one warp that takes whichever is
      // ready next lost 350 cycles from one product to the other.
      constexpr uint32_t kScore = kType | 4u << 24;  // M = 64, both K-major
      if (p.q_box) {
        if (n > 0) wait(b_score + 8 * ((n - 1) & 1), (n - 1) >> 1);  // Q of the segment before is done with
        if (elect_one()) {
          mbar_expect_tx(b_query, (uint32_t)(blocks * N * 128));
          for (int b = 0; b < blocks; ++b) tma_load(base + lay.q + b * (N * 128), &q_map, b * 64, g0, p.q_req > 0 ? r : 0, b_query);
        }
        __syncwarp();
      }
      wait(b_query, seg);
      const uint32_t q0 = operand_lo(base + lay.q, 16);
      for (int i = 0; i < count; ++i) {
        const uint32_t k = n + i, st = k & 1;
        if (k >= 2) wait(b_weight + 8 * st, (k >> 1) - 1);  // the scores two tiles before have been read
        wait(b_full + 8 * st, k >> 1);
        if (s_dead) break;
        tcgen05_after_sync();
        const uint32_t a0 = operand_lo(base + lay.kv + st * lay.stage, 16);
        const uint32_t d = tmem + st * N;
        if (elect_one()) {
#pragma unroll 3
          for (int b = 0; b < ksteps / 4; ++b)
#pragma unroll
            for (int u = 0; u < 4; ++u)
              tcgen05_mma(d, a0 + b * (kLatentBlock >> 4) + 2 * u, q0 + b * (N * 128 >> 4) + 2 * u, kOperandHi, kScore, b + u > 0);
          for (int s = ksteps & ~3; s < ksteps; ++s)
            tcgen05_mma(d, a0 + (s >> 2) * (kLatentBlock >> 4) + 2 * (s & 3), q0 + (s >> 2) * (N * 128 >> 4) + 2 * (s & 3), kOperandHi,
                        kScore, s > 0);
          tcgen05_commit(b_score + 8 * st);
        }
        __syncwarp();
      }
    } else if (warp == kValueWarp) {
      // ---- values -------------------------------------------------------------------------------------
      constexpr uint32_t kValue = kType | 1u << 15 | 1u << 16 | 8u << 24;  // M = 128, M- and N-major
      const uint32_t p00 = operand_lo(base + lay.p, kLatentBlock);
      for (int i = 0; i < count; ++i) {
        const uint32_t k = n + i, st = k & 1;
        wait(b_weight + 8 * st, k >> 1);
        if (s_dead) break;
        tcgen05_after_sync();
        const uint32_t a0 = operand_lo(base + lay.kv + st * lay.stage, kLatentBlock), p0 = p00 + st * (lay.p_step >> 4);
        if (elect_one()) {
#pragma unroll 4
          for (int v = 0; v < vblocks; ++v) {
#pragma unroll
            for (int u = 0; u < kLatentTile / 16; ++u)
              tcgen05_mma(tmem + 2 * N + v * N, a0 + v * (2 * kLatentBlock >> 4) + 128 * u, p0 + 128 * u, kOperandHi, kValue,
                          i > 0 || u > 0);
            tcgen05_commit(b_free + 32 * st + 8 * v);
          }
        }
        __syncwarp();
      }
    } else {
      // ---- softmax ------------------------------------------------------------------------------------
      const int quarter = warp & 3, half = warp >> 2;
      const uint32_t lanes = (uint32_t)quarter << 21;  // first TMEM lane of this warp's quarter, in an address
      const int c0 = half * NC;
      // Q: N rows of D elements, zero past the last head and column (where no tensor copy can bring it)
      if (!p.q_box) {
        const uint8_t* src = p.q + r * p.q_req + g0 * p.q_head;
        const int padded = ksteps * 2;
        for (int e = tid; e < N * padded; e += kSoftmaxWarps * 32) {
          const int row = e / padded, chunk = e - row * padded;
          const bool ok = row < rows && chunk < p.D / 8;
          cp_async16(base + lay.q + (chunk >> 3) * (N * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4),
                     ok ? src + row * p.q_head + chunk * 16 : src, ok);
        }
        cp_async_commit();
        cp_async_wait<0>();
        proxy_fence_smem();
        tcgen05_before_sync();  // the accumulator of the segment before has been read
        bar_arrive(b_query);
      }
      // A thread's scores: columns c0 + 8 i + 2 (lane % 4) + e of tokens row and row + 8.
      const int row = quarter * 16 + (lane >> 2);
      const int mine_col = column_of<C>(lane);
      float sum[C], from[C], limit[C];  // per column: what is subtracted, and up to where that will do
#pragma unroll
      for (int j = 0; j < C; ++j) {
        sum[j] = from[j] = 0.f;
        limit[j] = -INFINITY;
      }
      float top = -INFINITY;  // of head c0 + lane (lane < NC)
      uint32_t usable = 0;    // which of the tokens of this warp's half of the tiles counted, over all tiles
      for (int i = 0; i < count; ++i) {
        const uint32_t k = n + i, st = k & 1;
        wait(b_full + 8 * st, k >> 1);  // for ctl.valid
        wait(b_score + 8 * st, k >> 1);
        tcgen05_after_sync();
        uint32_t raw[2 * C];
        tmem_load_half<2 * C>(raw, tmem + lanes + st * N + c0);
        const uint32_t counted = ctl.valid[st][quarter >> 1], valid = counted >> ((quarter & 1) * 16 + (lane >> 2));
        usable |= counted;
        const bool seen0 = valid & 1, seen1 = valid >> 8 & 1;
        tmem_wait_load();
        float x[2 * C], e[2 * C];
        bool over = false;
#pragma unroll
        for (int j = 0; j < C; ++j) {  // j = 2 i + e; x[2 j] and x[2 j + 1] are the two tokens
          x[2 * j] = seen0 ? __uint_as_float(raw[(j >> 1) * 4 + (j & 1)]) * p.qk_scale : -INFINITY;
          x[2 * j + 1] = seen1 ? __uint_as_float(raw[(j >> 1) * 4 + (j & 1) + 2]) * p.qk_scale : -INFINITY;
          over |= fmaxf(x[2 * j], x[2 * j + 1]) > limit[j];
          e[2 * j] = exp2_approx(x[2 * j] - from[j]);
          e[2 * j + 1] = exp2_approx(x[2 * j + 1] - from[j]);
        }
        // Most tiles stay below the limits: one vote of the four warps that share these heads, and
        // nothing is exchanged. Otherwise they find the new maxima together.
        bool rescale = false;
        float alpha = 1.f;
        if (bar_any(1 + half, kSoftmaxWarps * 16, over)) {
          float most[C];
#pragma unroll
          for (int j = 0; j < C; ++j) most[j] = fmaxf(x[2 * j], x[2 * j + 1]);
          const float tile_top = join_rows<C>(most, lane, [](float a, float b) { return fmaxf(a, b); });
          float* const red = s_red + (k & 1) * 4 * N;
          red[quarter * N + c0 + mine_col] = tile_top;
          asm volatile("bar.sync %0, %1;" ::"r"(1 + half), "n"(kSoftmaxWarps * 16) : "memory");
          bool moved = false;
          if (lane < NC) {
            const int c = c0 + lane;
            const float m = fmaxf(fmaxf(red[c], red[N + c]), fmaxf(red[2 * N + c], red[3 * N + c]));
            if (m > top + kLazy) {
              moved = true;
              alpha = exp2_approx(top - m);
              top = m;
            }
          }
          rescale = __any_sync(0xffffffffu, moved);
          const float lane_from = top == -INFINITY ? 0.f : top - kShift;
#pragma unroll
          for (int j = 0; j < C; ++j) {
            const int col = (j >> 1) * 8 + (lane & 3) * 2 + (j & 1);
            sum[j] *= __shfl_sync(0xffffffffu, alpha, col);
            from[j] = __shfl_sync(0xffffffffu, lane_from, col);
            limit[j] = __shfl_sync(0xffffffffu, top, col) + kLazy;
            e[2 * j] = exp2_approx(x[2 * j] - from[j]);
            e[2 * j + 1] = exp2_approx(x[2 * j + 1] - from[j]);
          }
        }
        uint32_t w[C];  // w[2 i], w[2 i + 1]: the pair of columns, of the two tokens
#pragma unroll
        for (int j = 0; j < C; ++j) sum[j] += e[2 * j] + e[2 * j + 1];
#pragma unroll
        for (int j = 0; j < C; j += 2) {
          w[j] = pack2<BF16>(e[2 * j], e[2 * j + 2]);
          w[j + 1] = pack2<BF16>(e[2 * j + 1], e[2 * j + 3]);
        }
#pragma unroll
        for (int j = 0; j < C; j += 2) {
          uint8_t* to = smem + lay.p + st * lay.p_step + row * 128 + (((half * (NC / 8) + j / 2) ^ (row & 7)) << 4) + (lane & 3) * 4;
          *reinterpret_cast<uint32_t*>(to) = w[j];
          *reinterpret_cast<uint32_t*>(to + 8 * 128) = w[j + 1];  // row + 8: the same place of its swizzle
        }
        if (rescale && i > 0) {
          wait(b_free + 32 * (st ^ 1) + 8 * last, (k - 1) >> 1);  // the products of the tile before are in
          tcgen05_after_sync();
          for (int b = 0; b < vblocks; ++b) {
            uint32_t o[NC];
            tmem_load<NC>(o, tmem + lanes + 2 * N + b * N + c0);
            tmem_wait_load();
#pragma unroll
            for (int c = 0; c < NC; ++c)
              o[c] = __float_as_uint(__uint_as_float(o[c]) * __shfl_sync(0xffffffffu, alpha, c));
            tmem_store<NC>(tmem + lanes + 2 * N + b * N + c0, o);
          }
          tmem_wait_store();
        }
        proxy_fence_smem();
        tcgen05_before_sync();
        bar_arrive(b_weight + 8 * st);
      }
      // ---- the segment's result -----------------------------------------------------------------------
      wait(b_free + 32 * ((n + count - 1) & 1) + 8 * last, (n + count - 1) >> 1);
      tcgen05_after_sync();
      float total = join_rows<C>(sum, lane, [](float a, float b) { return a + b; });
      // the turn after the last tile's: its readers have passed the last tile's barrier; the next
      // tile's writers wait below until this turn has been read
      float* const red = s_red + ((n + count) & 1) * 4 * N;
      red[quarter * N + c0 + mine_col] = total;
      const bool seen = bar_any(1 + half, kSoftmaxWarps * 16, usable != 0);  // a token of the segment counted
      if (lane < NC) {  // from here on: of head c0 + lane
        const int c = c0 + lane;
        total = (red[c] + red[N + c]) + (red[2 * N + c] + red[3 * N + c]);
      }
      asm volatile("bar.sync %0, %1;" ::"r"(1 + half), "n"(kSoftmaxWarps * 16) : "memory");
      const bool whole = t0 == 0 && t1 == tiles;
      const int64_t slot = ((int64_t)team * 2 + (first ? 0 : 1)) * gridDim.y + unit;
      const int head = c0 + lane;
      const float inv = seen ? 1.f / total : 0.f;
      if (quarter == 0 && lane < NC && head < rows) {
        if (!whole)
          p.ml[slot * p.rows + head] = make_float2(top - kShift, seen ? total : kNoneSeen);
        else if (p.lse != nullptr)
          p.lse[(int64_t)r * p.G + g0 + head] = (top - kShift + log2f(total)) * kLn2;
      }
      for (int b = 0; b < vblocks; ++b) {
        uint32_t o[NC];
        tmem_load<NC>(o, tmem + lanes + 2 * N + b * N + c0);
        tmem_wait_load();
        const int d = b * 128 + quarter * 32 + lane;
        if (whole) {
          uint8_t* to = p.out + r * p.o_req + (int64_t)(g0 + c0) * p.o_head + d * 2;
#pragma unroll
          for (int c = 0; c < NC; ++c, to += p.o_head) {
            const float f = __shfl_sync(0xffffffffu, inv, c);
            if (c0 + c < rows && d < p.Dv) store_io(to, __uint_as_float(o[c]) * f, BF16);
          }
        } else {
          float* to = p.part + (slot * p.rows + c0) * p.Dv + d;
#pragma unroll
          for (int c = 0; c < NC; ++c, to += p.Dv)
            if (c0 + c < rows && d < p.Dv) *to = __uint_as_float(o[c]);
        }
      }
    }
    n += count;
    ++seg;
    first = false;
    if (p.uncut) break;
  }
  if (s_dead) {  // give the copies and products that are in flight a millisecond to end
    const long long began = clock64();
    while (clock64() - began < 2000000) __nanosleep(1000);
  }
  tcgen05_before_sync();
  __syncthreads();
  if (warp == kScoreWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kCols) : "memory");
}

}  // namespace topkv

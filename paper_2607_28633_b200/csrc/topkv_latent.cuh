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
//   warps 8-11  load: two stages of 64 rows, one pair of warps each, 16-byte asynchronous copies
//               through the block table (any page size and stride; what is masked becomes zero)
//   warp 12     one thread issues the matrix instructions
// Running maxima move only when a tile exceeds them by more than 2^8, so the accumulator is rescaled
// a few times per request and not once per tile; the weights are at most 2^8 (fp16: scaled by
// 2^7, to stay below 2^15), which costs no precision in a floating type.
// Every wait is bounded; one that runs out raises error bit 1 and lets the CTA finish.
#pragma once
#include <cuda_runtime.h>

#include <cstdint>

#include "topkv_attend.cuh"
#include "topkv_common.cuh"

namespace topkv {

constexpr int kLatentTile = 64;                  // tokens per tile
static_assert(kLatentTile == kTileTokens, "both kernels share out tiles of the same size");
constexpr int kSoftmaxWarps = 8, kLoadWarps = 4;
constexpr int kLatentThreads = (kSoftmaxWarps + kLoadWarps + 1) * 32;
constexpr int kLatentBlock = kLatentTile * 128;  // bytes of 64 columns of a tile
constexpr int kLatentMaxD = 576, kLatentMaxDv = 512;
constexpr float kLazy = 8.f;                     // a maximum moves when it is exceeded by more than this (powers of two)

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

__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tcgen05_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
      : "memory");
}
__device__ __forceinline__ void proxy_fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ float redux_max(float v) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// Shared-memory operand, 128-byte swizzle: `lead` and `stride` in bytes.
__device__ __forceinline__ uint64_t smem_operand(uint32_t addr, uint32_t lead, uint32_t stride) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46 |
         2ull << 61;
}

// Layout of the dynamic shared memory. All operand blocks are multiples of 1,024 bytes.
struct LatentControl {
  float red[2 * 4 * 64];  // maxima and sums per quarter of TMEM and head, by turns
  uint64_t bar[8];
  TeamStart team;
  uint32_t valid[2][2];   // which of a stage's tokens count
  uint32_t tmem;
  volatile int dead;      // a wait ran out
};
struct LatentSmem {
  uint32_t q, kv, p, control, total;
  uint32_t stage;  // bytes of a stage
};
__host__ __device__ inline LatentSmem latent_smem(int N, int D, int Dv) {
  const int blocks = (D + 63) / 64, vblocks = (Dv + 127) / 128 * 2;
  LatentSmem s;
  s.stage = (uint32_t)((blocks > vblocks ? blocks : vblocks) * kLatentBlock);
  s.q = 0;
  s.kv = (uint32_t)(blocks * N * 128);
  s.p = s.kv + 2 * s.stage;
  s.control = s.p + kLatentTile * 128;
  s.total = s.control + (uint32_t)sizeof(LatentControl);
  return s;
}

template <int N, bool BF16>
__global__ void __launch_bounds__(kLatentThreads, 1) topkv_latent_kernel(const AttendParams p) {
  constexpr int NC = N / 2;                       // heads per softmax warp
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

  // barriers: rows loaded [2], rows used [2], scores ready [2], weights written, Q written
  const uint32_t bar0 = smem_addr(ctl.bar);
  const uint32_t b_full = bar0, b_free = bar0 + 16, b_score = bar0 + 32, b_weight = bar0 + 48, b_query = bar0 + 56;
  if (tid == 0) {
    s_dead = 0;
    for (int i = 0; i < 2; ++i) {
      mbar_init(b_full + 8 * i, 64);
      mbar_init(b_free + 8 * i, 1);
      mbar_init(b_score + 8 * i, 1);
    }
    mbar_init(b_weight, kSoftmaxWarps * 32);
    mbar_init(b_query, kSoftmaxWarps * 32);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kSoftmaxWarps + kLoadWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)), "n"(kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    tcgen05_before_sync();
  }
  if (!p.late_wait) pdl_wait_prior_grid();
  pdl_release_next_grid();
  const TeamRange mine = team_range<kLatentThreads>(p, team, &ctl.team);
  if (p.late_wait) pdl_wait_prior_grid();
  __syncthreads();
  tcgen05_after_sync();
  const uint32_t tmem = ctl.tmem;
  if (unit == 0 && tid == 0) note_cut(p, team, mine);
  empty_requests<kLatentThreads>(p, team, (int64_t)g0, rows, unit == 0);

  // Waits until the barrier has completed its phase number `phase` (0, 1, 2, ...).
  auto wait = [&](uint32_t bar, uint32_t phase) {
    const long long began = clock64();
    while (!mbar_try_wait(bar, phase & 1)) {
      if (s_dead) break;
      if (clock64() - began > 1000000000ll) {  // about half a second
        s_dead = 1;
        raise_error(kErrWait);
        break;
      }
    }
  };

  const int ksteps = (p.D + 15) / 16, vblocks = (p.Dv + 127) / 128;
  uint32_t n = 0;    // tiles before the current segment, in this CTA: they number the phases
  uint32_t seg = 0;  // segments before
  int64_t left = mine.left;  // 0: no tiles
  int t0 = mine.t0;
  bool first = true;
  for (int r = mine.r; left > 0 && r < p.R; ++r) {
    const Visible vis = visible_tokens(p, r, false);
    const int tiles = attend_tiles(vis.n);
    if (tiles == 0) {
      if (p.uncut) break;
      t0 = 0;
      first = false;
      continue;
    }
    const int t1 = p.uncut ? tiles : (int)min((int64_t)tiles, t0 + left);
    const int count = t1 - t0;
    left -= p.uncut ? 1 : count;

    if (warp >= kSoftmaxWarps && warp < kSoftmaxWarps + kLoadWarps) {
      // ---- load: pair `g` of warps takes the stages g of its own parity ---------------------------
      const int g = (warp - kSoftmaxWarps) >> 1, half = (warp - kSoftmaxWarps) & 1;
      const int chunks = p.D / 8, padded = ksteps * 2;  // 16-byte chunks of a row, and up to the last k-step
      for (int i = (g - (int)(n & 1)) & 1; i < count; i += 2) {
        const uint32_t k = n + i;
        const int v = (t0 + i) * kLatentTile + half * 32 + lane;
        int64_t off = -1;
        if (v < vis.n) {
          const int tok = v < vis.ns ? v : v - vis.ns + vis.lo;
          const int j = tok / p.P;
          const int pg = p.bt[(int64_t)r * p.maxp + j];
          if (pg < 0 || pg >= p.num_pages)
            raise_error(kErrTable);
          else
            off = (int64_t)pg * p.S_page + (int64_t)(tok - j * p.P) * p.S_tok;
        }
        const uint32_t valid = __ballot_sync(0xffffffffu, off >= 0);
        if (k >= 2) wait(b_free + 8 * g, (k >> 1) - 1);
        if (lane == 0) ctl.valid[g][half] = valid;
        const uint32_t dst = base + lay.kv + g * lay.stage + half * 32 * 128;
        int row = 0, chunk = lane;
        while (chunk >= padded) {
          chunk -= padded;
          ++row;
        }
        for (int e = lane; e < 32 * padded; e += 32) {
          const int64_t o = __shfl_sync(0xffffffffu, off, row);
          const bool ok = o >= 0 && chunk < chunks;
          cp_async16(dst + (chunk >> 3) * kLatentBlock + row * 128 + (((chunk & 7) ^ (row & 7)) << 4),
                     p.pool + (ok ? o + chunk * 16 : 0), ok);
          chunk += 32;
          while (chunk >= padded) {
            chunk -= padded;
            ++row;
          }
        }
        cp_async_commit();
        cp_async_wait<0>();
        proxy_fence_smem();
        bar_arrive(b_full + 8 * g);
      }
    } else if (warp == kSoftmaxWarps + kLoadWarps) {
      // ---- matrix instructions ----------------------------------------------------------------------
      if (lane == 0) {
        constexpr uint32_t kType = 1u << 4 | (BF16 ? 1u : 0u) << 7 | (BF16 ? 1u : 0u) << 10 | (uint32_t)(N >> 3) << 17;
        constexpr uint32_t kScore = kType | 4u << 24;                        // M = 64, both K-major
        constexpr uint32_t kValue = kType | 1u << 15 | 1u << 16 | 8u << 24;  // M = 128, M- and N-major
        wait(b_query, seg);
        for (int i = 0; i <= count; ++i) {
          if (i < count) {
            const uint32_t k = n + i, st = k & 1;
            wait(b_full + 8 * st, k >> 1);
            tcgen05_after_sync();
            const uint32_t kv = base + lay.kv + st * lay.stage;
            if (!s_dead) {
              for (int s = 0; s < ksteps; ++s)
                tcgen05_mma(tmem + st * N, smem_operand(kv + (s >> 2) * kLatentBlock + (s & 3) * 32, 16, 1024),
                            smem_operand(base + lay.q + (s >> 2) * (N * 128) + (s & 3) * 32, 16, 1024), kScore, s > 0);
              tcgen05_commit(b_score + 8 * st);
            }
          }
          if (i > 0) {
            const uint32_t k = n + i - 1, st = k & 1;
            wait(b_weight, k);
            tcgen05_after_sync();
            const uint32_t kv = base + lay.kv + st * lay.stage;
            if (!s_dead) {
              for (int b = 0; b < vblocks; ++b)
#pragma unroll
                for (int s = 0; s < kLatentTile / 16; ++s)
                  tcgen05_mma(tmem + 2 * N + b * N, smem_operand(kv + 2 * b * kLatentBlock + s * 2048, kLatentBlock, 1024),
                              smem_operand(base + lay.p + s * 2048, kLatentBlock, 1024), kValue, i > 1 || s > 0);
              tcgen05_commit(b_free + 8 * st);
            }
          }
        }
      }
      __syncwarp();
    } else {
      // ---- softmax ------------------------------------------------------------------------------------
      const int quarter = warp & 3, half = warp >> 2;
      const uint32_t lanes = (uint32_t)quarter << 21;  // first TMEM lane of this warp's quarter, in an address
      const int token = quarter * 16 + lane;           // of a tile; lanes 16-31 of a quarter hold no scores
      const int c0 = half * NC;
      // Q: N rows of D elements, zero past the last head and column
      {
        const uint8_t* src = p.q + r * p.q_req + g0 * p.q_head;
        const int padded = ksteps * 2;
        for (int e = tid; e < N * padded; e += kSoftmaxWarps * 32) {
          const int row = e / padded, chunk = e - row * padded;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (row < rows && chunk < p.D / 8) v = *reinterpret_cast<const uint4*>(src + row * p.q_head + chunk * 16);
          *reinterpret_cast<uint4*>(smem + lay.q + (chunk >> 3) * (N * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)) = v;
        }
        proxy_fence_smem();
        tcgen05_before_sync();  // the accumulator of the segment before has been read
        bar_arrive(b_query);
      }
      float sum[NC];
#pragma unroll
      for (int c = 0; c < NC; ++c) sum[c] = 0.f;
      float top = -INFINITY;  // of head c0 + lane (lane < NC)
      for (int i = 0; i < count; ++i) {
        const uint32_t k = n + i, st = k & 1;
        wait(b_full + 8 * st, k >> 1);   // for ctl.valid
        wait(b_score + 8 * st, k >> 1);
        tcgen05_after_sync();
        uint32_t raw[NC];
        tmem_load<NC>(raw, tmem + lanes + st * N + c0);
        const bool seen = lane < 16 && (ctl.valid[st][quarter >> 1] >> ((quarter & 1) * 16 + (lane & 15)) & 1);
        tmem_wait_load();
        float x[NC], most = -INFINITY;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          x[c] = seen ? __uint_as_float(raw[c]) * p.qk_scale : -INFINITY;
          const float m = redux_max(x[c]);
          if (lane == c) most = m;
        }
        float* const red = s_red + (k & 1) * 4 * N;
        if (lane < NC) red[quarter * N + c0 + lane] = most;
        asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
        bool moved = false;
        float alpha = 1.f;
        if (lane < NC) {
          const int c = c0 + lane;
          const float m = fmaxf(fmaxf(red[c], red[N + c]), fmaxf(red[2 * N + c], red[3 * N + c]));
          if (m > top + kLazy) {
            moved = true;
            alpha = exp2f(top - m);
            top = m;
          }
        }
        const bool rescale = __any_sync(0xffffffffu, moved);
        const float from = top == -INFINITY ? 0.f : top - kShift;
        uint32_t w[NC / 2];
        if (rescale) {
#pragma unroll
          for (int c = 0; c < NC; ++c) sum[c] *= __shfl_sync(0xffffffffu, alpha, c);
        }
#pragma unroll
        for (int c = 0; c < NC; c += 2) {
          x[c] = exp2f(x[c] - __shfl_sync(0xffffffffu, from, c));
          x[c + 1] = exp2f(x[c + 1] - __shfl_sync(0xffffffffu, from, c + 1));
          w[c / 2] = pack2<BF16>(x[c], x[c + 1]);
          sum[c] += x[c];
          sum[c + 1] += x[c + 1];
        }
        // the second product of the tile before has to be done with the weights and the accumulator
        if (k > 0) wait(b_free + 8 * (st ^ 1), (k - 1) >> 1);
        if (lane < 16) {
          uint8_t* row = smem + lay.p + token * 128;
#pragma unroll
          for (int c = 0; c < NC / 8; ++c)
            *reinterpret_cast<uint4*>(row + (((half * (NC / 8) + c) ^ (token & 7)) << 4)) =
                make_uint4(w[c * 4], w[c * 4 + 1], w[c * 4 + 2], w[c * 4 + 3]);
        }
        if (rescale && i > 0) {
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
        bar_arrive(b_weight);
      }
      // ---- the segment's result -----------------------------------------------------------------------
      wait(b_free + 8 * ((n + count - 1) & 1), (n + count - 1) >> 1);
      tcgen05_after_sync();
      float total = 0.f;  // of head c0 + lane
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        float v = sum[c];
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        v = __shfl_sync(0xffffffffu, v, 0);  // lanes 0-15 hold the tokens
        if (lane == c) total = v;
      }
      // the turn after the last tile's: its readers have passed the last tile's barrier, and the next
      // tile's writers wait for scores that need every warp's arrival behind this read
      float* const red = s_red + ((n + count) & 1) * 4 * N;
      if (lane < NC) red[quarter * N + c0 + lane] = total;
      asm volatile("bar.sync 1, %0;" ::"n"(kSoftmaxWarps * 32) : "memory");
      if (lane < NC) {
        const int c = c0 + lane;
        total = (red[c] + red[N + c]) + (red[2 * N + c] + red[3 * N + c]);
      }
      const bool whole = t0 == 0 && t1 == tiles;
      const int64_t slot = ((int64_t)team * 2 + (first ? 0 : 1)) * gridDim.y + unit;
      const int head = c0 + lane;
      if (quarter == 0 && lane < NC && head < rows) {
        if (!whole)
          p.ml[slot * p.rows + head] = make_float2(top - kShift, total);
        else if (p.lse != nullptr)
          p.lse[(int64_t)r * p.G + g0 + head] = (top - kShift + log2f(total)) * kLn2;
      }
      for (int b = 0; b < vblocks; ++b) {
        uint32_t o[NC];
        tmem_load<NC>(o, tmem + lanes + 2 * N + b * N + c0);
        tmem_wait_load();
        const int d = b * 128 + quarter * 32 + lane;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const float l = __shfl_sync(0xffffffffu, total, c);
          if (c0 + c < rows && d < p.Dv) {
            if (whole)
              store_io(p.out + r * p.o_req + (g0 + c0 + c) * p.o_head + d * 2, __uint_as_float(o[c]) / l, BF16);
            else
              p.part[(slot * p.rows + c0 + c) * p.Dv + d] = __uint_as_float(o[c]);
          }
        }
      }
    }
    n += count;
    ++seg;
    first = false;
    t0 = 0;
    if (p.uncut) break;
  }
  tcgen05_before_sync();
  __syncthreads();
  if (warp == kSoftmaxWarps + kLoadWarps)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kCols) : "memory");
}

}  // namespace topkv

// New tokens of a layer: K and Q rotated by the tokens' positions, K and V converted and written into the
// paged cache through the block table.
//
//   a = 2 pi frac(position * turns_j / 2^64)      (x, y) -> scale * (x cos a - y sin a, x sin a + y cos a)
//
// A pair's advance per position is kept as a 64-bit fraction of a turn, so the product with a position drops
// its full turns exactly and the angle is good to 2^-26 turns wherever the token stands; in a float the
// angle of position 10^6 would be off by 0.06.
//
// What bounds it: memory, every element is read and written once (3 flops an element). The cosines of a token
// serve all its heads: a CTA takes few tokens, works out their count / 2 pairs each into shared memory, and
// its threads then keep to one 16-byte chunk of a head (and the one that holds the chunk's partners) and walk
// over the heads. Few tokens are spread over several CTAs by heads.
// Measured: 13,312 tokens of 8 x 4 heads of 128, bf16 into an e4m3 cache, 300 MB: 64 us, 4.7 TB/s (9 more with a loop over
// the tokens outside of that over the heads); 256 tokens of 128 heads of 576, 64 of whose elements turn: 18.8 us, 4.0 TB/s; four tokens 9
// us, the call and the launch.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "topkv_attend.cuh"
#include "topkv_common.cuh"

namespace topkv {

constexpr int kAppendThreads = 256;
constexpr int kAppendPairs = 2048;  // cosines in shared memory: tokens of a CTA times pairs

struct AppendParams {
  uint8_t* pool;  // this layer's slab
  const int32_t* bt;
  const int32_t* sl;
  const int64_t* cu;          // or nullptr: one row per request
  const int32_t* positions;   // or nullptr
  const uint64_t* turns;
  const uint8_t* in[3];       // q, k, v
  uint8_t* q_out;
  int64_t in_row[3], in_head[3];
  int64_t out_row, out_head;
  int64_t S_page, S_kv, S_tok, S_head;
  int64_t num_pages, num_rows;
  int R, maxp, P;
  int Hq, H, rows;            // rows of a token: Hq + H, and H more with values
  int D, first, half;         // elements; pairs
  int pairs;                  // neighbours, not halves
  int tokens;                 // per CTA
  float scale;
  float stored[2], inv[2];    // of K, V: what stored elements are divided by, see AppendTo
};

// Eight 16-bit elements as floats, and back.
template <bool BF16>
__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    } else {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}
template <bool BF16>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3]), pack2<BF16>(x[4], x[5]), pack2<BF16>(x[6], x[7]));
}
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {  // saturating, NaN stays NaN
  return __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
}
// Where row `row` of a token goes: q_out, or a plane of its page. E: bytes of an element there.
// Elements of an 8-bit plane are quotients: value / scale, rounded to 32 bits, then to 8. The product with the reciprocal is
// the same number only where the reciprocal has no rounding, i.e. for powers of two (scale 0 here); with other scales it leaves
// ties (1.5625 = 0.01068115234375 / (7 / 1024)) and comes out a step apart.
struct AppendTo {
  uint8_t* p;
  bool narrow;
  float scale, inv;
};
template <bool E8>
__device__ __forceinline__ AppendTo append_to(const AppendParams& p, int64_t token, int row, int64_t place) {
  if (row < p.Hq) return {p.q_out + token * p.out_row + row * p.out_head, false, 0.f, 1.f};
  const int h = row - p.Hq, plane = h >= p.H;
  return {p.pool + place + plane * p.S_kv + (h - plane * p.H) * p.S_head, E8, E8 ? p.stored[plane] : 0.f, E8 ? p.inv[plane] : 1.f};
}
__device__ __forceinline__ const uint8_t* append_from(const AppendParams& p, int64_t token, int row) {
  const int kind = row < p.Hq ? 0 : row < p.Hq + p.H ? 1 : 2;
  const int h = row - (kind == 0 ? 0 : kind == 1 ? p.Hq : p.Hq + p.H);
  return p.in[kind] + token * p.in_row[kind] + h * p.in_head[kind];
}
template <bool BF16, bool E8>
__device__ __forceinline__ void append_store8(const AppendTo& to, int d, float (&x)[8]) {
  if (E8 && to.narrow) {
    // The product is at most two units from the 32-bit quotient: one and a half of its two roundings, half a one of the
    // quotient's. Where neighbouring 8-bit values meet, the last 19 bits are zero, so only products within two units
    // of 16 such bits (four, for neighbours of powers of two) need the division. (13,312 tokens of 8 x 4 heads, V by 0.75, where
    // every warp has such products: 63.7 us, 64.5 if all are divided, 60.6 with products alone.)
    uint32_t near = 0xffffu;
    if (to.scale != 0.f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) near = min(near, (__float_as_uint(x[i] * to.inv) + 4) & 0xffffu);
    }
    if (near > 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= to.inv;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __fdiv_rn(x[i], to.scale);
    }
    *reinterpret_cast<uint2*>(to.p + d) = make_uint2(to_e4m3x2(x[0], x[1]) | to_e4m3x2(x[2], x[3]) << 16,
                                                     to_e4m3x2(x[4], x[5]) | to_e4m3x2(x[6], x[7]) << 16);
  } else {
    *reinterpret_cast<uint4*>(to.p + 2 * d) = pack8<BF16>(x);
  }
}
template <bool BF16>
__device__ __forceinline__ float load_io(const uint8_t* p) {
  if constexpr (BF16) return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p));
  else return __half2float(*reinterpret_cast<const __half*>(p));
}
template <bool BF16, bool E8>
__device__ __forceinline__ void append_store1(const AppendTo& to, int d, float x) {
  if (E8 && to.narrow)
    to.p[d] = (uint8_t)__nv_cvt_float_to_fp8(to.scale != 0.f ? __fdiv_rn(x, to.scale) : x * to.inv, __NV_SATFINITE, __NV_E4M3);
  else
    store_io(to.p + 2 * d, x, BF16);
}

// By chunks of eight elements if the rotated part begins, ends and is halved at multiples of eight (a rotation of
// neighbours: begins and ends), otherwise one pair at a time.
enum AppendWay { kByElements = 0, kByHalves = 1, kByNeighbours = 2 };
template <bool BF16, bool E8, int WAY>
__global__ void __launch_bounds__(kAppendThreads, 4) topkv_append_kernel(const AppendParams p) {
  __shared__ __align__(16) float2 s_turn[kAppendPairs];
  __shared__ int64_t s_place[kAppendThreads];  // offset of the token's page row in the slab, -1: left out
  __shared__ int s_position[kAppendThreads];
  const int tid = threadIdx.x;
  pdl_wait_prior_grid();
  pdl_release_next_grid();
  const int64_t t0 = (int64_t)blockIdx.x * p.tokens;
  const int n = (int)min((int64_t)p.tokens, p.num_rows - t0);
  // The request of the CTA's first row: all offsets are looked at side by side, which takes one access where a
  // search by halves takes one after the other.
  int r0 = (int)min(t0, (int64_t)p.R);
  if (p.cu != nullptr) {
    r0 = 0;
    for (int i = 0; i < p.R; i += kAppendThreads)
      r0 += __syncthreads_count(i + tid < p.R && p.cu[min(i + tid, p.R - 1) + 1] <= t0);
  }
  if (tid < n) {
    const int64_t t = t0 + tid;
    int r = p.cu != nullptr ? r0 : (int)min(t, (int64_t)p.R);
    int64_t behind = 1;  // rows of the request from this one on
    if (p.cu != nullptr) {
      while (r < p.R && p.cu[r + 1] <= t) ++r;
      behind = r < p.R ? p.cu[r + 1] - t : 0;
      if (r < p.R && p.cu[r] > t) r = p.R;  // before the first request's rows
    }
    int64_t place = -1;
    int position = 0;
    if (r < p.R) {
      const int s = p.sl[r];
      const int64_t i = s - behind;
      if (s < 0 || s > (int64_t)p.maxp * p.P || (s > 0 && i < 0)) {
        raise_error(kErrTable);
      } else if (s > 0) {
        const int j = (int)i / p.P, page = p.bt[(int64_t)r * p.maxp + j];
        if (page < 0 || page >= p.num_pages)
          raise_error(kErrTable);
        else
          place = (int64_t)page * p.S_page + ((int)i - j * p.P) * p.S_tok;
        position = p.positions != nullptr ? p.positions[t] : (int)i;
      }
    }
    s_place[tid] = place;
    s_position[tid] = position;
  }
  __syncthreads();
  for (int e = tid; e < n * p.half; e += kAppendThreads) {
    const int k = e / p.half, j = e - k * p.half;
    const uint64_t a = (uint64_t)(int64_t)s_position[k] * p.turns[j];
    float sine, cosine;
    sincospif((float)(int32_t)(a >> 32) * 0x1p-31f, &sine, &cosine);
    s_turn[e] = make_float2(cosine * p.scale, sine * p.scale);
  }
  __syncthreads();

  if constexpr (WAY != kByElements) {
    constexpr bool kPairs = WAY == kByNeighbours;
    const int chunks = p.D / 8, first = p.first / 8, turned = kPairs ? p.half / 4 : p.half / 8;
    // items of a row: chunks of pairs that turn (halves: two chunks each), then the others
    const int items = turned + chunks - p.half / 4;
    const int step = kAppendThreads / items, item = tid % items;
    int row0 = tid / items;
    if (row0 >= step) return;
    const bool turns = item < turned;
    int c0, c1 = 0;
    if (turns) {
      c0 = first + item;
      c1 = c0 + turned;
    } else {
      c0 = item - turned;
      if (c0 >= first) c0 += p.half / 4;
    }
    const bool two = turns && !kPairs;
    const int by = step * gridDim.y;
    // Rows of all the CTA's tokens behind each other, kAhead of them at a time, so that their loads run together.
    constexpr int kAhead = kPairs ? 4 : 2;
    int k = 0, row = row0 + blockIdx.y * step;
    auto settle = [&] {  // to a row that exists, of a token that has a place; k == n: none is left
      for (;;) {
        while (k < n && row >= p.rows) {
          row -= p.rows;
          ++k;
        }
        if (k >= n || s_place[k] >= 0) return;
        row += by;
      }
    };
    settle();
    while (k < n) {
      uint4 a[kAhead], b[kAhead];
      int at_k[kAhead], at_row[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        at_k[u] = k;
        at_row[u] = row;
        if (k < n) {
          const uint8_t* src = append_from(p, t0 + k, row);
          a[u] = *reinterpret_cast<const uint4*>(src + c0 * 16);
          if (!kPairs && two) b[u] = *reinterpret_cast<const uint4*>(src + c1 * 16);
          row += by;
          settle();
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        if (at_k[u] >= n) break;
        const AppendTo to = append_to<E8>(p, t0 + at_k[u], at_row[u], s_place[at_k[u]]);
        const bool keys = at_row[u] < p.Hq + p.H;
        const float2* cs = s_turn + at_k[u] * p.half + (kPairs ? item * 4 : item * 8);
        if (!(turns && keys) && !(E8 && to.narrow)) {  // as it is
          *reinterpret_cast<uint4*>(to.p + c0 * 16) = a[u];
          if (!kPairs && two) *reinterpret_cast<uint4*>(to.p + c1 * 16) = b[u];
          continue;
        }
        float x[8], y[8];
        unpack8<BF16>(a[u], x);
        if (!kPairs && two) {
          unpack8<BF16>(b[u], y);
          if (keys) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float2 c = cs[i];
              const float v = x[i] * c.x - y[i] * c.y;
              y[i] = x[i] * c.y + y[i] * c.x;
              x[i] = v;
            }
          }
          append_store8<BF16, E8>(to, c1 * 8, y);
        } else if (turns && keys) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 c = cs[i];
            const float v = x[2 * i] * c.x - x[2 * i + 1] * c.y;
            x[2 * i + 1] = x[2 * i] * c.y + x[2 * i + 1] * c.x;
            x[2 * i] = v;
          }
        }
        append_store8<BF16, E8>(to, c0 * 8, x);
      }
    }
  } else {
    // items of a row: pairs, then the elements that stay
    const int items = p.half + p.D - 2 * p.half;
    for (int64_t e = tid + (int64_t)blockIdx.y * kAppendThreads; e < (int64_t)n * p.rows * items; e += (int64_t)kAppendThreads * gridDim.y) {
      const int k = (int)(e / ((int64_t)p.rows * items)), rest = (int)(e - (int64_t)k * p.rows * items);
      const int row = rest / items, item = rest - row * items;
      if (s_place[k] < 0) continue;
      const uint8_t* src = append_from(p, t0 + k, row);
      const AppendTo to = append_to<E8>(p, t0 + k, row, s_place[k]);
      if (item < p.half) {
        const int d0 = p.first + (p.pairs ? 2 * item : item), d1 = d0 + (p.pairs ? 1 : p.half);
        float x = load_io<BF16>(src + 2 * d0), y = load_io<BF16>(src + 2 * d1);
        if (row < p.Hq + p.H) {
          const float2 cs = s_turn[k * p.half + item];
          const float v = x * cs.x - y * cs.y;
          y = x * cs.y + y * cs.x;
          x = v;
        }
        append_store1<BF16, E8>(to, d0, x);
        append_store1<BF16, E8>(to, d1, y);
      } else {
        int d = item - p.half;
        if (d >= p.first) d += 2 * p.half;
        append_store1<BF16, E8>(to, d, load_io<BF16>(src + 2 * d));
      }
    }
  }
}

}  // namespace topkv

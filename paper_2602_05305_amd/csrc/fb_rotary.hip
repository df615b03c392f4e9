// Rotary positions of a block's queries and keys, and appending to the paged cache with the rotation on the way (gfx950).
//
// Pair j of a row at position p turns by the angle a = p * inv_freq[j], p the position on the pair's axis:
//   x -> x cos a - y sin a,  y -> x sin a + y cos a        (inverse: -a, the transposed operator, which is the gradient)
// inv_freq is taken as the exact number its fp32 value is.  The angle in turns is p * (inv_freq / 2 pi) in 64 bits, of which only the
// fraction goes on in 32: at p = 2^20 an angle in 32 bits is off by 0.06, the one here by 1e-7, at 2^31 by 8e-7.  Products and sums are fp32, a
// bf16 result is rounded once.
//
// What bounds it: HBM, one read and one write of every element; below some 10 MB the launch and two dependent memory round trips.
//   * A workgroup belongs to one of the three tensors (its strides are scalars: looked up by lane they were vector loads, and more rows to a
//     thread made the pass slower, 193 -> 268 us at 8 x 4096 tokens of 32 / 8 heads) and has some tokens and a range of their heads.  Angles
//     do not depend on the head: a thread to an angle, once for all heads of the range, into LDS (64-bit products and a sine for
//     every element instead would be the bound).
//   * A thread owns V = 16 bytes / element pairs, that is both members of each, so a call may be in place; it asks for its rows before it
//     computes angles.
//   * Lanes run along a row first, then along the tokens, then the heads: reads of a token-major row and writes of [B,H,Bq,d] are both whole
//     128-byte lines.
#include "fb_kernels.h"

namespace fb {
namespace {

constexpr int kMinTokens = 4;       // of a workgroup: at 64 pairs one angle for each of the 256 threads
constexpr double kInvTwoPi = 0.15915494309189533577;

template <typename T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int V = 4;
};
template <>
struct Vec<__bf16> {
  static constexpr int V = 8;
};

// V elements at an address of the element's alignment (16 bytes on the usual paths; the hardware takes any)
template <typename T>
struct Pack {
  T x[Vec<T>::V];
};

template <typename T>
__device__ __forceinline__ Pack<T> load_pack(const T* at) {
  Pack<T> r;
  __builtin_memcpy(&r, at, sizeof(r));
  return r;
}
template <typename T>
__device__ __forceinline__ void store_pack(T* at, const Pack<T>& r) {
  __builtin_memcpy(at, &r, sizeof(r));
}
template <typename T>
__device__ __forceinline__ Pack<T> load_aligned(const T* at) {
  return *(const Pack<T>*)__builtin_assume_aligned(at, 16);
}
template <typename T>
__device__ __forceinline__ void store_aligned(T* at, const Pack<T>& r) {
  *(Pack<T>*)__builtin_assume_aligned(at, 16) = r;
}

// A thread's two packs, pairs j0 .. j0 + V - 1.  Halves: the pairs' first members, from j0, and their second ones, from j0 + pairs.  Flat: the
// elements 2 j0 .. 2 j0 + 2 V - 1 (adjacent members, or elements that no pair covers).  Mixed: each of its own, where the pairs end inside.
enum SlotKind : int { kSlotHalves, kSlotFlat, kSlotMixed };

// A workgroup: ROWS rows (token x head), a slot to a thread.  (More slots to a thread: 8 x 4096 tokens of 32 / 8 heads, head_dim 128, 1 / 2 / 4 / 8
// 157 / 162 / 169 / 192 us; a plain copy of as many bytes 150.  Non-temporal stores 164.)
template <typename T, int D>
struct TCfg {
  static constexpr int V = Vec<T>::V, SLOTS = D / (2 * V), ROWS = 256 / SLOTS;
};

template <typename T, int D>
__global__ __launch_bounds__(256) void rotate_rows_kernel(const RotateParams p) {
  using C = TCfg<T, D>;
  constexpr int V = C::V;
  __shared__ __align__(16) float cos_s[C::ROWS][D / 2 + 4], sin_s[C::ROWS][D / 2 + 4];      // (one head: a token to a row)
  __shared__ long long dst_s[C::ROWS];                                    // paged: element offset of head 0's row in the pools, or -1
  const uint32_t wg = blockIdx.x;
  const int which = (wg >= p.part[1].first_wg ? 1 : 0) + (wg >= p.part[2].first_wg ? 1 : 0);      // uniform
  const RotatePart& part = p.part[which];
  const int tid = threadIdx.x, slot = tid % C::SLOTS, row = tid / C::SLOTS;
  const uint32_t local = wg - part.first_wg, group = fastdiv(local, part.div_groups);
  const int tokens = 1 << part.tokens_log2, t = row & (tokens - 1);
  const uint32_t token0 = group << part.tokens_log2, head0 = (local - group * part.div_groups.d) * (uint32_t)(C::ROWS >> part.tokens_log2);

  // ---- this thread's rows
  const uint32_t token = token0 + t;
  bool ok = token < p.tokens;
  const uint32_t b = fastdiv(ok ? token : 0u, p.div_block), i = (ok ? token : 0u) - b * p.div_block.d;
  const bool paged = part.paged != 0;
  if (paged && p.counts != nullptr) ok = ok && (int)i < p.counts[b];      // this token does not go into the cache
  const uint32_t h = head0 + (uint32_t)(row >> part.tokens_log2);
  const bool live = ok && h < (uint32_t)part.heads;
  Pack<T> a, c;
  const int pairs = part.turned ? p.pairs : 0, j0 = slot * V;
  const SlotKind kind = p.adjacent || j0 >= pairs ? kSlotFlat : j0 + V <= pairs ? kSlotHalves : kSlotMixed;
  if (live) {
    const T* at = (const T*)part.src + b * part.s_batch + i * part.s_row + h * part.s_head;
    if (kind == kSlotFlat) {
      a = load_aligned(at + 2 * j0);
      c = load_aligned(at + 2 * j0 + V);
    } else if (kind == kSlotHalves) {
      a = load_aligned(at + j0);
      c = load_pack(at + j0 + pairs);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = j0 + e;
        a.x[e] = at[j < pairs ? j : 2 * j];
        c.x[e] = at[j < pairs ? j + pairs : 2 * j + 1];
      }
    }
  }

  // ---- angles of the workgroup's tokens; where the tokens go in the cache
  const int left = (int)min((uint32_t)tokens, p.tokens - token0);
  for (int x = tid; x < left * pairs; x += 256) {
    const int t2 = (int)fastdiv((uint32_t)x, p.div_pairs), j = x - t2 * pairs;
    const uint32_t tok = token0 + t2, b2 = fastdiv(tok, p.div_block), i2 = tok - b2 * p.div_block.d;
    const double f = (double)p.inv_freq[j] * kInvTwoPi;
    int pos;
    if (p.positions != nullptr) {
      int axis = 0;
      while (axis + 1 < p.n_axes && j >= p.axis_end[axis]) ++axis;
      pos = p.positions[b2 * p.position_stride + (long long)i2 * p.n_axes + axis];
    } else {
      pos = (int)((uint32_t)p.offset + (uint32_t)(p.first != nullptr ? p.first[b2] : 0) + i2);
    }
    const double turns = (double)pos * f;
    float s, co;
    sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &co);
    cos_s[t2][j] = co;
    sin_s[t2][j] = p.inverse ? -s : s;
  }
  if (paged && tid < left) {
    const uint32_t tok = token0 + tid, b2 = fastdiv(tok, p.div_block), i2 = tok - b2 * p.div_block.d;
    const int len = max(p.lens[b2], 0), count = min(max(p.counts != nullptr ? p.counts[b2] : (int)p.div_block.d, 0), (int)p.div_block.d);
    const long long at = (long long)len + i2;
    long long dst = -1;
    if ((int)i2 < count && at < p.capacity) {
      const uint32_t page_i = fastdiv((uint32_t)at, p.div_page);
      const int page = p.block_table[(size_t)b2 * p.max_pages + page_i];
      if (page >= 0 && page < p.num_pages)
        dst = ((long long)page * part.heads * (int)p.div_page.d + (int)((uint32_t)at - page_i * p.div_page.d)) * D;
    }
    dst_s[tid] = dst;
    if (p.lens_out != nullptr && i2 == 0 && head0 == 0 && which == 1) {
      const long long end = (long long)len + count;
      p.lens_out[b2] = (int)(end < p.capacity ? end : p.capacity > len ? p.capacity : len);
    }
  }
  __syncthreads();

  if (!live) return;
  T* at = (T*)part.dst;
  if (paged) {
    if (dst_s[t] < 0) return;
    at += dst_s[t] + (long long)h * (int)p.div_page.d * D;
  } else {
    at += b * part.d_batch + i * part.d_row + h * part.d_head;
  }
  if (j0 < pairs) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (kind != kSlotHalves && j0 + e >= pairs) continue;
      const float co = cos_s[t][j0 + e], s = sin_s[t][j0 + e];
      if (p.adjacent) {
        // pair e of the slot: elements 2 e, 2 e + 1 of the two packs in a row
        T& xr = 2 * e < V ? a.x[(2 * e) % V] : c.x[(2 * e) % V];
        T& yr = 2 * e < V ? a.x[(2 * e + 1) % V] : c.x[(2 * e + 1) % V];
        const float x = (float)xr, y = (float)yr;
        xr = (T)(x * co - y * s);
        yr = (T)(x * s + y * co);
      } else {
        const float x = (float)a.x[e], y = (float)c.x[e];
        a.x[e] = (T)(x * co - y * s);
        c.x[e] = (T)(x * s + y * co);
      }
    }
  }
  if (kind == kSlotFlat) {
    store_aligned(at + 2 * j0, a);
    store_aligned(at + 2 * j0 + V, c);
  } else if (kind == kSlotHalves) {
    store_aligned(at + j0, a);
    store_pack(at + j0 + pairs, c);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int j = j0 + e;
      at[j < pairs ? j : 2 * j] = a.x[e];
      at[j < pairs ? j + pairs : 2 * j + 1] = c.x[e];
    }
  }
}

template <typename T, int D>
hipError_t launch_typed(const RotateParams& p, hipStream_t s) {
  using C = TCfg<T, D>;
  RotateParams q = p;
  q.div_pairs = make_fastdiv((uint32_t)(p.pairs > 0 ? p.pairs : 1));
  long long grid = 0;
  for (RotatePart& part : q.part) {
    part.first_wg = (uint32_t)grid;
    part.div_groups = make_fastdiv(1);
    if (part.heads == 0) continue;
    // heads of a workgroup: a power of two, so many that kMinTokens tokens are left, and that the last group is not half idle
    int heads = 1;
    while (heads < part.heads && 2 * heads * kMinTokens <= C::ROWS) heads *= 2;
    while (heads > 4 && (part.heads - 1) % heads < heads / 2) heads /= 2;
    part.tokens_log2 = 0;
    while ((heads << (part.tokens_log2 + 1)) <= C::ROWS) ++part.tokens_log2;
    part.div_groups = make_fastdiv((uint32_t)((part.heads + heads - 1) / heads));
    grid += (long long)((p.tokens + (1u << part.tokens_log2) - 1) >> part.tokens_log2) * part.div_groups.d;
    if (grid >= (1ll << 31)) return hipErrorInvalidValue;
  }
  hipLaunchKernelGGL((rotate_rows_kernel<T, D>), dim3((unsigned)grid), dim3(256), 0, s, q);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateParams& p, int D, bool is_bf16, hipStream_t s) {
  if (is_bf16) return D == 64 ? launch_typed<__bf16, 64>(p, s) : launch_typed<__bf16, 128>(p, s);
  return D == 64 ? launch_typed<float, 64>(p, s) : launch_typed<float, 128>(p, s);
}

}  // namespace fb

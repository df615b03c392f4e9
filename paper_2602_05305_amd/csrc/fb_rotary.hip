// Rotary positions of a block's queries and keys, and appending to the paged cache with the rotation on the way (gfx950).
//
// Pair j of a row at position p turns by the angle a = p * inv_freq[j], p the position on the pair's axis:
//   x -> x cos a - y sin a,  y -> x sin a + y cos a        (inverse: -a, the transposed operator, which is the gradient)
// inv_freq is taken as the exact number its fp32 value is.  The angle in turns is p * (inv_freq / 2 pi) in 64 bits, of which only the
// fraction goes on in 32: at p = 2^20 an angle in 32 bits is off by 0.06, the one here by 1e-7, at 2^31 by 8e-7.  Products and sums are fp32, a
// bf16 result is rounded once.
//
// What bounds it: HBM, one read and one write of every element; below some 10 MB the launch and two dependent memory round trips.
//   * A workgroup has kTokens tokens and a range of their heads.  The angles do not depend on the head: one thread to an angle, once for all heads
//     of the range, into LDS (64-bit products and a sine for every element instead would be the bound).
//   * A thread owns V = 16 bytes / element pairs, that is both members of each, so a call may be in place; it asks for its rows before it
//     computes angles.
//   * Lanes run along a row first, then along the tokens, then the heads: reads of a token-major row and writes of [B,H,Bq,d] are both whole
//     128-byte lines.
#include "fb_kernels.h"

namespace fb {
namespace {

constexpr int kTokens = 4;          // at 64 pairs one angle for each of the 256 threads
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

// Where the two packs of slot c start: pair j = V c + e has its members at first + e and second + e (halves), or the pack pair
// holds pairs next to each other (adjacent, and what no pair covers).
enum SlotKind : int { kSlotHalves, kSlotFlat, kSlotMixed };

// ITEMS: slots of a thread.
template <typename T, int D, int ITEMS>
__global__ __launch_bounds__(256) void rotate_rows_kernel(const RotateParams p) {
  constexpr int V = Vec<T>::V, SLOTS = D / (2 * V), RPP = 256 / SLOTS;    // slots of a row, rows (token x head) of a pass over the workgroup
  constexpr int HEADS = ITEMS * RPP / kTokens;                           // heads of a workgroup
  __shared__ float cos_s[kTokens][D / 2 + 4], sin_s[kTokens][D / 2 + 4];
  __shared__ long long dst_s[kTokens];                                    // paged: element offset of head 0's row in the pools, or -1
  const int tid = threadIdx.x, slot = tid % SLOTS, row = tid / SLOTS;
  const uint32_t group = blockIdx.x / p.head_groups, head0 = (blockIdx.x - group * p.head_groups) * HEADS;
  const uint32_t token0 = group * kTokens;

  // ---- this thread's rows
  const int t = row % kTokens;
  const uint32_t token = token0 + t;
  const bool token_ok = token < p.tokens;
  const uint32_t b = fastdiv(token_ok ? token : 0u, p.div_block), i = (token_ok ? token : 0u) - b * p.div_block.d;
  bool kept = true;                                                      // paged: this token goes into the cache
  if (p.counts != nullptr) kept = (int)i < p.counts[b];
  Pack<T> a[ITEMS], c[ITEMS];
  const int pairs = p.pairs, j0 = slot * V;
  // kind of the slot in a rotated row; a row that is only moved is flat
  const SlotKind kind = p.adjacent || j0 >= pairs ? kSlotFlat : j0 + V <= pairs ? kSlotHalves : kSlotMixed;
  auto part_of = [&](uint32_t head, uint32_t& h) -> int {
    h = head;
    int k = 0;
    while (k < 2 && h >= (uint32_t)p.part[k].heads) h -= (uint32_t)p.part[k++].heads;
    return k;
  };
  bool live[ITEMS];
#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    uint32_t h;
    const uint32_t head = head0 + (u * RPP + row) / kTokens;
    const int k = part_of(head, h);
    const RotatePart& part = p.part[k];
    live[u] = token_ok && h < (uint32_t)part.heads && (kept || !part.paged);
    if (!live[u]) continue;
    const T* src = (const T*)part.src + b * part.s_batch + h * part.s_head + i * part.s_row;
    const SlotKind kd = part.turned ? kind : kSlotFlat;
    if (kd == kSlotFlat) {
      a[u] = load_aligned(src + 2 * j0);
      c[u] = load_aligned(src + 2 * j0 + V);
    } else if (kd == kSlotHalves) {
      a[u] = load_aligned(src + j0);
      c[u] = load_pack(src + j0 + pairs);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = j0 + e;
        a[u].x[e] = src[j < pairs ? j : 2 * j];
        c[u].x[e] = src[j < pairs ? j + pairs : 2 * j + 1];
      }
    }
  }

  // ---- angles of the workgroup's tokens; where the tokens go in the cache
  for (int x = tid; x < kTokens * pairs; x += 256) {
    const int t2 = x / pairs, j = x - t2 * pairs;
    const uint32_t tok = token0 + t2;
    if (tok >= p.tokens) break;
    const uint32_t b2 = fastdiv(tok, p.div_block), i2 = tok - b2 * p.div_block.d;
    const double f = (double)p.inv_freq[j] * kInvTwoPi;
    int pos;
    if (p.positions != nullptr) {
      int axis = 0;
      while (axis + 1 < p.n_axes && j >= p.axis_end[axis]) ++axis;
      pos = p.positions[b2 * p.position_stride + (long long)i2 * p.n_axes + axis];
    } else {
      pos = p.offset + (p.first != nullptr ? p.first[b2] : 0) + (int)i2;
    }
    const double turns = (double)pos * f;
    float s, co;
    sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &co);
    cos_s[t2][j] = co;
    sin_s[t2][j] = p.inverse ? -s : s;
  }
  if (p.block_table != nullptr && tid < kTokens && token0 + tid < p.tokens) {
    const uint32_t tok = token0 + tid, b2 = fastdiv(tok, p.div_block), i2 = tok - b2 * p.div_block.d;
    const int len = max(p.lens[b2], 0), count = min(max(p.counts != nullptr ? p.counts[b2] : (int)p.div_block.d, 0), (int)p.div_block.d);
    const long long at = (long long)len + i2;
    long long dst = -1;
    if ((int)i2 < count && at < p.capacity) {
      const uint32_t page_i = fastdiv((uint32_t)at, p.div_page);
      const int page = p.block_table[(size_t)b2 * p.max_pages + page_i];
      if (page >= 0 && page < p.num_pages)
        dst = ((long long)page * p.part[1].heads * (int)p.div_page.d + (int)((uint32_t)at - page_i * p.div_page.d)) * D;
    }
    dst_s[tid] = dst;
    if (p.lens_out != nullptr && i2 == 0 && head0 == 0) {
      const long long end = (long long)len + count;
      p.lens_out[b2] = (int)(end < p.capacity ? end : p.capacity > len ? p.capacity : len);
    }
  }
  __syncthreads();

#pragma unroll
  for (int u = 0; u < ITEMS; ++u) {
    if (!live[u]) continue;
    uint32_t h;
    const int k = part_of(head0 + (u * RPP + row) / kTokens, h);
    const RotatePart& part = p.part[k];
    long long at;
    if (part.paged) {
      if (dst_s[t] < 0) continue;
      at = dst_s[t] + (long long)h * (int)p.div_page.d * D;
    } else {
      at = b * part.d_batch + h * part.d_head + i * part.d_row;
    }
    T* dst = (T*)part.dst + at;
    const SlotKind kd = part.turned ? kind : kSlotFlat;
    if (part.turned && j0 < pairs) {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        if (j0 + e >= pairs) continue;
        const float co = cos_s[t][j0 + e], s = sin_s[t][j0 + e];
        if (p.adjacent) {
          // pair e of the slot: elements 2 e, 2 e + 1 of the two packs in a row
          T& xr = 2 * e < V ? a[u].x[(2 * e) % V] : c[u].x[(2 * e) % V];
          T& yr = 2 * e < V ? a[u].x[(2 * e + 1) % V] : c[u].x[(2 * e + 1) % V];
          const float x = (float)xr, y = (float)yr;
          xr = (T)(x * co - y * s);
          yr = (T)(x * s + y * co);
        } else {
          const float x = (float)a[u].x[e], y = (float)c[u].x[e];
          a[u].x[e] = (T)(x * co - y * s);
          c[u].x[e] = (T)(x * s + y * co);
        }
      }
    }
    if (kd == kSlotFlat) {
      store_aligned(dst + 2 * j0, a[u]);
      store_aligned(dst + 2 * j0 + V, c[u]);
    } else if (kd == kSlotHalves) {
      store_aligned(dst + j0, a[u]);
      store_pack(dst + j0 + pairs, c[u]);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int j = j0 + e;
        dst[j < pairs ? j : 2 * j] = a[u].x[e];
        dst[j < pairs ? j + pairs : 2 * j + 1] = c[u].x[e];
      }
    }
  }
}

template <typename T, int D, int ITEMS>
hipError_t launch_items(const RotateParams& p, hipStream_t s) {
  constexpr int HEADS = ITEMS * (256 / (D / (2 * Vec<T>::V))) / kTokens;
  RotateParams q = p;
  const int heads = p.part[0].heads + p.part[1].heads + p.part[2].heads;
  q.head_groups = (uint32_t)((heads + HEADS - 1) / HEADS);
  const long long grid = (long long)((p.tokens + kTokens - 1) / kTokens) * q.head_groups;
  if (grid >= (1ll << 31)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((rotate_rows_kernel<T, D, ITEMS>), dim3((unsigned)grid), dim3(256), 0, s, q);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_typed(const RotateParams& p, hipStream_t s) {
  return launch_items<T, D, 1>(p, s);
}

}  // namespace

hipError_t launch_rotate(const RotateParams& p, int D, bool is_bf16, hipStream_t s) {
  if (is_bf16) return D == 64 ? launch_typed<__bf16, 64>(p, s) : launch_typed<__bf16, 128>(p, s);
  return D == 64 ? launch_typed<float, 64>(p, s) : launch_typed<float, 128>(p, s);
}

}  // namespace fb

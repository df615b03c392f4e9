// Second launch of a refresh step, or of an external pass, over a shared prefix (bf16, gfx950): folds the split partials of the first
// launch (Eq. 5), streams a sequence's own pages, computes the block-internal attention (Eq. 7) and merges (Eq. 8-9), all for up to 32 rows
// of one KV head of one sequence to a workgroup (finish_rows: 32, or fewer where the workgroups would be few).
//
// What bounds it: HBM over the own keys where there are many; else the latency of a chain of four memory round trips (length, page, keys,
// partials), which is why it is one kernel: passes of their own write the own partials and read them back, and each adds a launch.
//   * A wavefront is by itself until the end: it loads tiles of 8 KB of keys and as much of values straight into its own LDS stage, waits
//     for its own loads and computes all 32 rows with them, no workgroup barrier.  The four wavefronts take every fourth tile; eight of them to
//     a CU (two workgroups) keep 128 KB in flight, three times what HBM asks of a CU, so a wavefront does not load ahead.
//   * The block's own keys, at most 32, are one tile, the last wavefront's, which then takes none of the others: a second set of accumulators
//     for it (255 registers instead of 206) made four wavefronts of own keys no faster than three.
//   * Row groups of the same KV head come next to each other on one XCD, whose L2 serves the second and later readings of the keys.
//   * At the end the wavefronts' sums meet in LDS, 64 columns at a time (so that it fits where the stages were).  A group of 8
//     threads folds the split partials of a row, several groups where the workgroup has few rows, each every n-th split; groups of a wavefront
//     meet in registers.  Cycle stamps, batch 64, one row of 32 / 8 heads, head_dim 128, us: length and page 0.5, first tile 2.2, partials 0.4
//     (16 splits 1.6), the end 1.8 (2.9 with LDS reads one after the other); own keys spread to 512, 67 MB, 8 at the median and 12 for the longest.
// Tiles, rotations and register layouts are those of the streaming kernel (fb_stream_bf16.hip); sums and statistics are fp32, weights
// are rounded to bf16 for the value product, as there.
#include "fb_kernels.h"
#include "fb_rows_bf16.h"

namespace fb {
namespace {

constexpr int kWaves = 4, kBlockWave = kWaves - 1;

template <int D>
struct NCfg {
  static constexpr int ROWB = D * 2, CPR = ROWB / 16;
  static constexpr int KT = 8192 / ROWB, NKB = KT / 32;       // keys of a tile
  static constexpr int OPB = KT * ROWB, STAGE = 2 * OPB;
  static constexpr int NLOAD = OPB / 1024;
  static constexpr int NKS = D / 16, NDB = D / 32;
  static constexpr int RS = 64 + 4;                           // floats of a row of 64 columns in LDS
  static constexpr int RECS = kWaves + 1;                     // wavefronts, split partials
  static constexpr int RING = kWaves * STAGE, REC = RECS * 32 * RS * 4;
  static constexpr int STAT = RING > REC ? RING : REC;        // then (m, l) of every record's rows
  static constexpr int LDS = STAT + RECS * 32 * 8;
  static_assert(2 * LDS <= 160 * 1024, "two workgroups to a CU");
  __device__ static __forceinline__ int rot_k(int row) { return D == 128 ? row : (row >> 1); }
  __device__ static __forceinline__ int rot_v(int row) { return D == 128 ? 4 * row : 4 * (row >> 1); }
};

template <int NDB>
struct FinAcc {
  float m, l;
  f32x16 o[NDB];
  __device__ __forceinline__ void init() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int i = 0; i < NDB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
  }
};

// What a thread folds of a row's split partials: 8 columns of each 64, log2-domain reference, sum.
template <int NH>
struct Folded {
  f32x4 a[NH], b[NH];
  float m, l;
};
// With the lanes across: of both sides the same row, one after the other.
enum Across { kAcross32, kAcross16, kAcross8 };
template <int NH, Across ACROSS>
__device__ __forceinline__ void fold_lanes(Folded<NH>& f) {
  auto both = [](float x, float& lo, float& hi) __attribute__((always_inline)) {
    if constexpr (ACROSS == kAcross8) {
      lo = x;
      hi = turn16<8>(x);
    } else if constexpr (ACROSS == kAcross16) {
      const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      lo = __uint_as_float(r[0]);
      hi = __uint_as_float(r[1]);
    } else {
      const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      lo = __uint_as_float(r[0]);
      hi = __uint_as_float(r[1]);
    }
  };
  float m0, m1, lo, hi;
  both(f.m, m0, m1);
  f.m = fmaxf(m0, m1);
  const float mu = f.m == -INFINITY ? 0.f : f.m, w0 = __builtin_amdgcn_exp2f(m0 - mu), w1 = __builtin_amdgcn_exp2f(m1 - mu);
  auto fold = [&](float x) __attribute__((always_inline)) {
    both(x, lo, hi);
    return fmaf(hi, w1, lo * w0);
  };
  f.l = fold(f.l);
#pragma unroll
  for (int half = 0; half < NH; ++half)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f.a[half][i] = fold(f.a[half][i]);
      f.b[half][i] = fold(f.b[half][i]);
    }
}

template <int D>
__global__ __launch_bounds__(256, 2) void shared_finish_kernel(const FinishParams p) {
  using C = NCfg<D>;
  extern __shared__ __align__(16) unsigned char lds[];
  const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));

  // ---- workgroup -> (row group, KV head, sequence)
  const uint32_t j8 = blockIdx.x >> 3, jq = fastdiv(j8, p.div_rowtiles), unit = jq * 8 + (blockIdx.x & 7);
  if (unit >= (uint32_t)(p.B * p.Hkv)) return;                // workgroup-uniform
  const int row0 = (int)(j8 - jq * p.div_rowtiles.d) * p.wg_rows;
  int b = (int)fastdiv(unit, p.div_hkv);
  const int kvh = (int)(unit - (uint32_t)b * p.div_hkv.d);
  if (p.order != nullptr) b = sload(p.order, b);
  const int valid = min(p.wg_rows, p.G * p.Bq - row0);
  const size_t grow0 = (size_t)(b * p.Hq + kvh * p.G) * p.Bq + row0;
  // the first tile's page is asked for along with the length, used or not
  int nkeys = 0;
  int32_t page = 0;
  if (p.own_keys > 0) {
    const int32_t* table = p.block_table + (size_t)b * p.max_pages;
    page = sload(table, min((int)fastdiv((uint32_t)(wave * C::KT), p.div_page), p.max_pages - 1));
    nkeys = min(p.own_keys, max(0, sload(p.prefix_lens, b)));
  }

  bf16x8 qreg[C::NKS];
  {
    const unsigned char* q = (const unsigned char*)p.q + (grow0 + min(l32, valid - 1)) * C::ROWB + h * 16;
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) qreg[ks] = *(const bf16x8*)(q + ks * 32);
  }
  unsigned char* stage = lds + wave * C::STAGE;
  const uint32_t stage_at = (uint32_t)(uintptr_t)stage;
  uint32_t kaddr[C::NKS], vaddr[C::NDB];
#pragma unroll
  for (int ks = 0; ks < C::NKS; ++ks) kaddr[ks] = (uint32_t)(l32 * C::ROWB + ((2 * ks + h + C::rot_k(l32)) & (C::CPR - 1)) * 16);
  {
    const int i16 = lane & 15, blk1 = (lane >> 4) & 1, rrow = 4 * h + (i16 >> 2);
#pragma unroll
    for (int db = 0; db < C::NDB; ++db)
      vaddr[db] = (uint32_t)(C::OPB + rrow * C::ROWB + ((4 * db + 2 * blk1 + ((i16 & 3) >> 1) + C::rot_v(rrow)) & (C::CPR - 1)) * 16 + (i16 & 1) * 8);
  }

  // direct-to-LDS load j: LDS chunk 64 j + lane is row ROWS1 j + lane / CPR, position lane % CPR, and holds the row's chunk (position - rotation).
  // Rotations come round in j, so the offsets of PK loads of keys and one of values are enough; the rest is in the scalar address.
  constexpr int ROWS1 = 64 / C::CPR, PK = D == 128 ? 4 : 2;
  const int lrow = lane / C::CPR, lpc = lane % C::CPR;
  uint32_t off_k[PK];
#pragma unroll
  for (int j = 0; j < PK; ++j) off_k[j] = (uint32_t)(lrow * C::ROWB + ((lpc - C::rot_k(ROWS1 * j + lrow)) & (C::CPR - 1)) * 16);
  const uint32_t off_v = (uint32_t)(lrow * C::ROWB + ((lpc - C::rot_v(lrow)) & (C::CPR - 1)) * 16);

  // one tile of this wavefront: nvalid of its keys exist
  auto tile = [&](FinAcc<C::NDB>& acc, const unsigned char* kt, const unsigned char* vt, int nvalid) __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");        // the last tile's reads have left the stage
    const bool ragged = nvalid < C::KT;                       // wavefront-uniform
    if (!ragged) {
#pragma unroll
      for (int j = 0; j < C::NLOAD; ++j) dma16(kt + j * 1024, off_k[j % PK], stage_at + j * 1024);
#pragma unroll
      for (int j = 0; j < C::NLOAD; ++j) dma16(vt + j * 1024, off_v, stage_at + C::OPB + j * 1024);
    } else {
      // rows past the end read the last key (their scores are masked)
#pragma unroll
      for (int j = 0; j < C::NLOAD; ++j) {
        const int r = ROWS1 * j + lrow, back = max(r - (nvalid - 1), 0) * C::ROWB;
        dma16(kt, (uint32_t)(off_k[j % PK] + j * 1024 - back), stage_at + j * 1024);
      }
#pragma unroll
      for (int j = 0; j < C::NLOAD; ++j) {
        const int r = ROWS1 * j + lrow, back = max(r - (nvalid - 1), 0) * C::ROWB;
        dma16(vt, (uint32_t)(off_v + j * 1024 - back), stage_at + C::OPB + j * 1024);
      }
    }
    wait_vm<C::NLOAD>();                                      // the keys are there
    f32x16 s[C::NKB];
#pragma unroll
    for (int kb = 0; kb < C::NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks)
#pragma unroll
      for (int kb = 0; kb < C::NKB; ++kb) {
        const bf16x8 a = *(const bf16x8*)(stage + kaddr[ks] + kb * 32 * C::ROWB);
        s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qreg[ks], s[kb], 0, 0, 0);
      }
    // s[kb][r]: row lane % 32, key 32 kb + 8 (r / 4) + 4 h + r % 4
    if (ragged) {
      asm volatile("" ::: "memory");                          // a branch, not a select for every score
#pragma unroll
      for (int kb = 0; kb < C::NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * kb + 8 * (r / 4) + 4 * h + (r % 4) >= nvalid) s[kb][r] = -INFINITY;
    }
    float tmax = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < C::NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) tmax = fmaxf(tmax, s[kb][r]);
    tmax = max_halves(tmax * p.scale_log2);
    const float m_new = tmax > acc.m + 8.f ? tmax : acc.m;    // moves rarely: weights stay below 2^8
    const float m_use = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(acc.m - m_use);
    bf16x8 pb[2 * C::NKB];
    float lsum = 0.f;
#pragma unroll
    for (int kb = 0; kb < C::NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(fmaf(s[kb][r], p.scale_log2, -m_use));
        lsum += w;
        pb[2 * kb + r / 8][r % 8] = (__bf16)w;
      }
    acc.l = acc.l * alpha + lsum;
    acc.m = m_new;
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int db = 0; db < C::NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc.o[db][r] *= alpha;
    }
    wait_vm<0>();
    if (ragged) {
      // value rows past the end: a weight of 0 must not meet an infinity or NaN of the duplicated last key
      for (int c = nvalid * C::CPR + lane; c < C::KT * C::CPR; c += 64) *(f32x4*)(stage + C::OPB + c * 16) = f32x4{0.f, 0.f, 0.f, 0.f};
      // other lanes of the wavefront read them: LDS keeps the order by itself, the compiler is told
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
#pragma unroll
    for (int t = 0; t < 2 * C::NKB; ++t)
#pragma unroll
      for (int db = 0; db < C::NDB; ++db) {
        const unsigned char* at = stage + vaddr[db] + 16 * t * C::ROWB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(at + 8 * C::ROWB));
        const s16x8 both = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        acc.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), pb[t], acc.o[db], 0, 0, 0);
      }
  };

  FinAcc<C::NDB> acc;
  acc.init();
  const bool step = p.k_block != nullptr;                     // uniform
  const int nown = step ? kWaves - 1 : kWaves;                // wavefronts for the own keys
  if (step && wave == kBlockWave) {
    const size_t off = (size_t)(b * p.Hkv + kvh) * p.Bq * C::ROWB;
    tile(acc, (const unsigned char*)p.k_block + off, (const unsigned char*)p.v_block + off, p.Bq);
  }
  const int ntiles = (nkeys + C::KT - 1) / C::KT;
  for (int t = wave; t < ntiles && wave < nown; t += nown) {
    const int k0 = t * C::KT, slot = (int)fastdiv((uint32_t)k0, p.div_page);
    page = min(max(page, 0), p.num_pages - 1);                // clamped into the pool
    const size_t off = (((size_t)page * p.Hkv + kvh) * p.div_page.d + (k0 - slot * (int)p.div_page.d)) * C::ROWB;
    const int k1 = min(k0 + nown * C::KT, nkeys - 1);       // the next tile's page, or the last one again
    page = sload(p.block_table + (size_t)b * p.max_pages, (int)fastdiv((uint32_t)k1, p.div_page));
    tile(acc, (const unsigned char*)p.k_pool + off, (const unsigned char*)p.v_pool + off, nkeys - k0);
  }

  // ---- records of 64 columns: [wavefronts: own keys][block][groups of splits][32 rows]
  float* rec = (float*)lds;
  float2* stat = (float2*)(lds + C::STAT);
  const int part = threadIdx.x & 7, group = threadIdx.x >> 3;
  const int rv_log2 = valid <= 1 ? 0 : 32 - __builtin_clz(valid - 1), rv = 1 << rv_log2, slices = 32 >> rv_log2;      // rows rounded up; groups to a row
  const int row = group & (rv - 1), slice = group >> rv_log2;
  auto put = [&](const FinAcc<C::NDB>& acc, int at, int half) __attribute__((always_inline)) {
#pragma unroll
    for (int d2 = 0; d2 < 2; ++d2)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // static register indices
          if constexpr (D == 128) v[i] = half ? acc.o[2 + d2][4 * q4 + i] : acc.o[d2][4 * q4 + i];
          else v[i] = acc.o[d2][4 * q4 + i];
        }
        *(f32x4*)(rec + (at * 32 + l32) * C::RS + 32 * d2 + 8 * q4 + 4 * h) = v;
      }
    if (half == 0) {
      const float l = sum_halves(acc.l);
      if (h == 0) stat[at * 32 + l32] = make_float2(acc.m, l);
    }
  };
  // this group's split partials, of all columns in one memory round trip
  constexpr int NH = D / 64;
  Folded<NH> f;
  f.m = -INFINITY;
  f.l = 0.f;
#pragma unroll
  for (int half = 0; half < NH; ++half) f.a[half] = f.b[half] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (row < valid) {
    constexpr int CH = 12 / NH;                               // splits in a round trip
    for (int s0 = slice; s0 < p.nsplit; s0 += slices * CH) {
      f32x4 oa[CH][NH], ob[CH][NH];
      float mv[CH], lv[CH], cm = f.m;
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        const int s = s0 + c * slices;
        mv[c] = -INFINITY;
        lv[c] = 0.f;
#pragma unroll
        for (int half = 0; half < NH; ++half) oa[c][half] = ob[c][half] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (s < p.nsplit) {
          const size_t g = (size_t)s * p.rows + grow0 + row;
          mv[c] = p.ws_m[g];
          lv[c] = p.ws_l[g];
#pragma unroll
          for (int half = 0; half < NH; ++half) {
            const float* o = p.ws_o + g * D + 64 * half + 8 * part;
            oa[c][half] = *(const f32x4*)o;
            ob[c][half] = *(const f32x4*)(o + 4);
          }
        }
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) cm = fmaxf(cm, mv[c]);
      if (cm == -INFINITY) continue;
      const float back = __builtin_amdgcn_exp2f(f.m - cm);
      float w[CH];
#pragma unroll
      for (int c = 0; c < CH; ++c) w[c] = __builtin_amdgcn_exp2f(mv[c] - cm);
      f.m = cm;
      f.l *= back;
#pragma unroll
      for (int c = 0; c < CH; ++c) f.l = fmaf(lv[c], w[c], f.l);
#pragma unroll
      for (int half = 0; half < NH; ++half)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f.a[half][i] *= back;
          f.b[half][i] *= back;
#pragma unroll
          for (int c = 0; c < CH; ++c) {
            f.a[half][i] = fmaf(oa[c][half][i], w[c], f.a[half][i]);
            f.b[half][i] = fmaf(ob[c][half][i], w[c], f.b[half][i]);
          }
        }
    }
  }
  // groups of a wavefront that have the same row: lanes 32, 16, 8 across; what is left goes through LDS, at most kWaves to a row
  if (rv_log2 <= 2) fold_lanes<NH, kAcross32>(f);
  if (rv_log2 <= 1) fold_lanes<NH, kAcross16>(f);
  if (rv_log2 == 0) fold_lanes<NH, kAcross8>(f);
  const int inside = max(0, 3 - rv_log2), nslots = slices >> inside, slot = slice >> inside;
  const bool writes = (slice & ((1 << inside) - 1)) == 0;
  const int nw = ntiles > 0 ? nown : 0;
  // a thread of the end: row `group`, 8 columns of each 64; weights of the slots and of the wavefronts
  float ws[kWaves], ww[kWaves], wblk = 0.f, wext = 0.f, M = -INFINITY, adj = 0.f;
#pragma unroll
  for (int half = 0; half < NH; ++half) {
    __syncthreads();                                          // the stages, or the records of the first 64 columns, have been read
    put(acc, wave, half);
    if (writes) {
      const int at = kWaves * 32 + slot * rv + row;
      *(f32x4*)(rec + at * C::RS + 8 * part) = f.a[half];
      *(f32x4*)(rec + at * C::RS + 8 * part + 4) = f.b[half];
      if (part == 0 && half == 0) stat[at] = make_float2(f.m, f.l);
    }
    __syncthreads();
    if (group < valid) {
      const size_t g = grow0 + group;
      const int col = 64 * half + 8 * part;
      // (what is not there is read in the place of the first one and left out below: reads in front of the branches overlap)
      auto slot_at = [&](int i) { return kWaves * 32 + (i < nslots ? i : 0) * rv + group; };
      auto wave_at = [&](int i) { return (i < nw ? i : 0) * 32 + group; };
      if (half == 0) {
        float2 ss[kWaves], sw[kWaves];
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          ss[i] = stat[slot_at(i)];
          sw[i] = stat[wave_at(i)];
        }
        const float2 sb = stat[kBlockWave * 32 + group];
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          if (i < nslots) M = fmaxf(M, ss[i].x);
          if (i < nw) M = fmaxf(M, sw[i].x);
        }
        const float Mu = M == -INFINITY ? 0.f : M;
        float l = 0.f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          ws[i] = __builtin_amdgcn_exp2f(ss[i].x - Mu);
          if (i < nslots) l = fmaf(ss[i].y, ws[i], l);
        }
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
          ww[i] = __builtin_amdgcn_exp2f(sw[i].x - Mu);
          if (i < nw) l = fmaf(sw[i].y, ww[i], l);
        }
        // the partial, in natural-log units: m is rounded when converted, o is rescaled to the reference that consumers recover from it
        float m_nat = -INFINITY, L = -INFINITY;
        if (l > 0.f) {
          m_nat = M * kLn2;
          adj = __builtin_amdgcn_exp2f(M - m_nat * kLog2e);
          L = (M + log2f(l)) * kLn2;
        }
        if (part == 0) {
          p.m[g] = m_nat;
          p.lse[g] = L;
        }
        if (step) {
          const float M2 = fmaxf(M, sb.x), M2u = M2 == -INFINITY ? 0.f : M2;
          wext = __builtin_amdgcn_exp2f(M - M2u);
          wblk = __builtin_amdgcn_exp2f(sb.x - M2u);
          const float den = l * wext + sb.y * wblk, inv = den > 0.f ? 1.f / den : 0.f;
          wext *= inv;
          wblk *= inv;
          if (part == 0 && p.lse_out != nullptr) p.lse_out[g] = den > 0.f ? (M2 + log2f(den)) * kLn2 : -INFINITY;
        }
      }
      f32x4 va[2 * kWaves + 1], vb[2 * kWaves + 1], ta = {0.f, 0.f, 0.f, 0.f}, tb = ta;
#pragma unroll
      for (int i = 0; i <= 2 * kWaves; ++i) {
        const float* o = rec + (i < kWaves ? slot_at(i) : i < 2 * kWaves ? wave_at(i - kWaves) : kBlockWave * 32 + group) * C::RS + 8 * part;
        va[i] = *(const f32x4*)o;
        vb[i] = *(const f32x4*)(o + 4);
      }
#pragma unroll
      for (int i = 0; i < 2 * kWaves; ++i)
        if (i < kWaves ? i < nslots : i - kWaves < nw) {
          const float w = i < kWaves ? ws[i % kWaves] : ww[i % kWaves];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            ta[j] = fmaf(va[i][j], w, ta[j]);
            tb[j] = fmaf(vb[i][j], w, tb[j]);
          }
        }
      *(f32x4*)(p.o + g * D + col) = ta * adj;
      *(f32x4*)(p.o + g * D + col + 4) = tb * adj;
      if (step) {
        float r[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          r[j] = ta[j] * wext + va[2 * kWaves][j] * wblk;
          r[4 + j] = tb[j] * wext + vb[2 * kWaves][j] * wblk;
        }
        const u32x4 pk = {pack_bf16x2(r[0], r[1]), pack_bf16x2(r[2], r[3]), pack_bf16x2(r[4], r[5]), pack_bf16x2(r[6], r[7])};
        *(u32x4*)((__bf16*)p.out + g * D + col) = pk;
      }
    }
  }
}

template <int D>
hipError_t launch_finish(const FinishParams& p, hipStream_t s) {
  using C = NCfg<D>;
  FinishParams q = p;
  const int rowtiles = (p.G * p.Bq + p.wg_rows - 1) / p.wg_rows;
  q.div_rowtiles = make_fastdiv((uint32_t)rowtiles);
  q.div_hkv = make_fastdiv((uint32_t)p.Hkv);
  q.div_page = make_fastdiv((uint32_t)(p.page_size > 0 ? p.page_size : 1));
  const long long grid = ((long long)p.B * p.Hkv + 7) / 8 * 8 * rowtiles;
  if (grid >= (1ll << 31) || p.wg_rows < 1 || p.wg_rows > 32 || (p.k_block != nullptr && (p.Bq > kFinishBlock || p.out == nullptr))) return hipErrorInvalidValue;
  static LdsLimit lim;
  hipError_t e = raise_lds_limit(shared_finish_kernel<D>, C::LDS, lim, C::LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(shared_finish_kernel<D>, dim3((unsigned)grid), dim3(256), C::LDS, s, q);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_shared_finish(const FinishParams& p, int D, hipStream_t s) {
  return D == 64 ? launch_finish<64>(p, s) : launch_finish<128>(p, s);
}

}  // namespace fb

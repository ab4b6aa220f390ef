// What the kernels that go over a paged 4-bit cache by tiles of 32 tokens share: the
// copies of a tile into LDS, its codes as operands of the matrix instructions, the
// softmax of its scores, and which tokens rows see.
#pragma once

#include "kv_cache.h"
#include "mfma_tile.h"

namespace sph {

// Where references start, in binades: finite, so that differences with it are no NaN,
// and below any score that fp32 holds.
constexpr float kNoScore = -3.402823466e38f;
constexpr float kLate = 8.0f;
constexpr float kLn2 = 0.693147180559945f;

// Tiles of 32 tokens go from memory straight into a ring of LDS stages that is the
// wave's own: as many as the ring holds are in flight at no cost in registers, and
// no wave waits for another.  A stage is the codes of both blocks as they are
// stored, then the scales of both.
template <int D>
struct Stage {
  static constexpr int kCodes = 32 * D;                               // bytes
  static constexpr int kBytes = (34 * D + 255) / 256 * 256;
  static constexpr int kCodeCopies = kCodes / 1024;                   // a wave copies 64 x 16 bytes,
  static constexpr int kScaleCopies = (2 * D + 255) / 256;            // scales 64 x 4
  static constexpr int kCopies = kCodeCopies + kScaleCopies;
};

// A lane's share of a stage: codes, and the scale bytes of its keys (one, two for D
// 256) and of its values (four tokens).
template <int D>
struct KvKeys {
  uint32_t c[2][D / 32], s[2];
};
template <int D>
struct KvValues {
  uint32_t c[2][D / 32], s[2];
};

// Pages of a tile's two blocks, -1 for one that no row of the wave sees or the
// table does not name.
struct KvPages {
  int page[2];
};
__device__ __forceinline__ KvPages tile_pages(const KvArgs& a, const KvSession& ses, int pos, int end) {
  KvPages p;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int at = pos + b * kKvBlock;
    const uint32_t i = (uint32_t)at >> a.page_shift, last = a.max_pages - 1;
    // (read wherever it is, so that the load need not wait for the session's length;
    // the constant address space makes it a scalar one)
    const int page = ((const __attribute__((address_space(4))) int32_t*)ses.table)[i < last ? i : last];
    p.page[b] = at < end && i <= last && (unsigned)page < (unsigned)a.n_pages ? page : -1;
  }
  return p;
}

// Copies of one tile into the stage `to`.  A block that does not exist is copied
// from page 0 and not used.  lane16: the lane's 16 bytes (kept apart from the base,
// which stays scalar); the offset operand counts for both sides.
template <int D, int AUX>
__device__ __forceinline__ void copy_with(uint8_t* to, const KvArgs& a, int head, int pos, const KvPages& pages,
                                          uint32_t& lane16, uint32_t lane) {
  const uint8_t* blk[2];
  asm volatile("" : "+v"(lane16));
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int page = pages.page[b];
    blk[b] = scalar_ptr(kv_block<D>(a, page < 0 ? 0 : page, head, page < 0 ? 0 : pos + b * kKvBlock));
    lds_void_t* at = (lds_void_t*)(to + b * 16 * D);
    __builtin_amdgcn_global_load_lds(blk[b] + lane16, at, 16, 0, AUX);
    if constexpr (D >= 128) __builtin_amdgcn_global_load_lds(blk[b] + lane16, at, 16, 1024, AUX);
    if constexpr (D >= 256) {
      __builtin_amdgcn_global_load_lds(blk[b] + lane16, at, 16, 2048, AUX);
      __builtin_amdgcn_global_load_lds(blk[b] + lane16, at, 16, 3 * 1024, AUX);
    }
  }
  lds_void_t* at = (lds_void_t*)(to + Stage<D>::kCodes);
  if constexpr (D == 256) {  // 256 bytes of either block
    const uint32_t lane4 = lane16 / 4 + 16 * D;
    __builtin_amdgcn_global_load_lds(blk[0] + lane4, at, 4, 0, AUX);
    __builtin_amdgcn_global_load_lds(blk[1] + lane4, (lds_void_t*)(to + Stage<D>::kCodes + 256), 4, 0, AUX);
  } else {                   // D bytes of either; for D 64 the last half of the lanes repeat the first
    const uint32_t in = lane * 4 % (2 * D);
    const uint64_t b0 = reinterpret_cast<uint64_t>(blk[0]), b1 = reinterpret_cast<uint64_t>(blk[1]);
    const uint64_t base = in < D ? b0 : b1;
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint8_t*>(base) + (16 * D + in % D), at, 4, 0, AUX);
  }
}

// Codes that one workgroup alone reads go past the caches as a stream (192 sessions
// with 16 rows of a head 166 -> 148 us, with 20 rows 183 -> 169); where tiles of
// rows read the same ones they meet in L2.
template <int D>
__device__ __forceinline__ void copy_tile(uint8_t* to, const KvArgs& a, int head, int pos, const KvPages& pages,
                                          uint32_t& lane16, uint32_t lane, bool alone) {
  if (alone) copy_with<D, 2>(to, a, head, pos, pages, lane16, lane);
  else copy_with<D, 0>(to, a, head, pos, pages, lane16, lane);
}

// At most N of the wave's newest copies may still be on their way.
template <int N>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// Reads of a stage end with their own wait: the compiler would make them wait for
// every copy in flight.  at_c, at_s: LDS addresses of the lane's codes and scales.
template <int D>
__device__ __forceinline__ void read_codes(uint32_t (&c)[2][D / 32], uint32_t& s0, uint32_t& s1, uint32_t at_c,
                                           uint32_t at_s, bool bytes) {
  if constexpr (D == 64) {
    u32x2_t x, y;
    if (bytes)
      asm volatile("ds_read_b64 %0, %4\n ds_read_b64 %1, %4 offset:1024\n ds_read_u8 %2, %5\n"
                   "ds_read_u8 %3, %5 offset:64\n s_waitcnt lgkmcnt(0)"
                   : "=&v"(x), "=&v"(y), "=&v"(s0), "=&v"(s1) : "v"(at_c), "v"(at_s) : "memory");
    else
      asm volatile("ds_read_b64 %0, %4\n ds_read_b64 %1, %4 offset:1024\n ds_read_b32 %2, %5\n"
                   "ds_read_b32 %3, %5 offset:64\n s_waitcnt lgkmcnt(0)"
                   : "=&v"(x), "=&v"(y), "=&v"(s0), "=&v"(s1) : "v"(at_c), "v"(at_s) : "memory");
    c[0][0] = x[0], c[0][1] = x[1], c[1][0] = y[0], c[1][1] = y[1];
  } else if constexpr (D == 128) {
    u32x4_t x, y;
    if (bytes)
      asm volatile("ds_read_b128 %0, %4\n ds_read_b128 %1, %4 offset:2048\n ds_read_u8 %2, %5\n"
                   "ds_read_u8 %3, %5 offset:128\n s_waitcnt lgkmcnt(0)"
                   : "=&v"(x), "=&v"(y), "=&v"(s0), "=&v"(s1) : "v"(at_c), "v"(at_s) : "memory");
    else
      asm volatile("ds_read_b128 %0, %4\n ds_read_b128 %1, %4 offset:2048\n ds_read_b32 %2, %5\n"
                   "ds_read_b32 %3, %5 offset:128\n s_waitcnt lgkmcnt(0)"
                   : "=&v"(x), "=&v"(y), "=&v"(s0), "=&v"(s1) : "v"(at_c), "v"(at_s) : "memory");
#pragma unroll
    for (int e = 0; e < 4; ++e) c[0][e] = x[e], c[1][e] = y[e];
  } else {
    u32x4_t x, y, z, w;
    if (bytes) {
      uint32_t t0, t1;  // the second group's bytes
      asm volatile("ds_read_b128 %0, %8\n ds_read_b128 %1, %8 offset:16\n ds_read_b128 %2, %8 offset:4096\n"
                   "ds_read_b128 %3, %8 offset:4112\n ds_read_u8 %4, %9\n ds_read_u8 %5, %9 offset:256\n"
                   "ds_read_u8 %6, %9 offset:16\n ds_read_u8 %7, %9 offset:272\n s_waitcnt lgkmcnt(0)"
                   : "=&v"(x), "=&v"(y), "=&v"(z), "=&v"(w), "=&v"(s0), "=&v"(s1), "=&v"(t0), "=&v"(t1)
                   : "v"(at_c), "v"(at_s) : "memory");
      s0 |= t0 << 8;
      s1 |= t1 << 8;
    } else {
      asm volatile("ds_read_b128 %0, %6\n ds_read_b128 %1, %6 offset:16\n ds_read_b128 %2, %6 offset:4096\n"
                   "ds_read_b128 %3, %6 offset:4112\n ds_read_b32 %4, %7\n ds_read_b32 %5, %7 offset:256\n"
                   "s_waitcnt lgkmcnt(0)"
                   : "=&v"(x), "=&v"(y), "=&v"(z), "=&v"(w), "=&v"(s0), "=&v"(s1) : "v"(at_c), "v"(at_s) : "memory");
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) c[0][e] = x[e], c[0][4 + e] = y[e], c[1][e] = z[e], c[1][4 + e] = w[e];
  }
}

__device__ __forceinline__ float max_over_groups(float x) {  // of lanes n, n + 16, n + 32, n + 48
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_over_groups(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  bf16x2_t r;
  r[0] = (__bf16)lo;
  r[1] = (__bf16)hi;
  return __builtin_bit_cast(uint32_t, r);
}

// What a wave keeps for its MT tiles of 16 rows: lane l the outputs of row n at
// dimensions (4 g + e) D/16 + c in o[m][c][e], the reference and sum of its weights.
template <int D, int MT>
struct Rows {
  f32x4_t o[MT][D / 16];
  float top[MT], sum[MT];  // sums of the lane's own tokens
};

// Queries as the second operand of the first product: tile m, step j.  Where the
// outputs alone are 128 registers they come from LDS.
template <int D, int MT, bool LDS>
struct Queries {
  bf16x8_t r[LDS ? 1 : MT][LDS ? 1 : D / 32];
  const u32x4_t* l;  // LDS [row groups][MT][D / 32][64 lanes]
  uint32_t own;      // the lane's first
  __device__ __forceinline__ bf16x8_t at(int m, int j) const {
    if constexpr (LDS) return __builtin_bit_cast(bf16x8_t, l[own + (m * (D / 32) + j) * 64]);
    else return r[m][j];
  }
};

// Scores of 32 tokens: lane l has row n against tokens 4 g + e of both blocks.
template <int D, int MT, bool LDS>
__device__ __forceinline__ void take_keys(f32x4_t (&sc)[MT][2], const KvKeys<D>& k, Queries<D, MT, LDS>& q) {
  // (read again for every tile: kept in registers they would cost what LDS saves)
  if constexpr (LDS) asm volatile("" : "+v"(q.own));
#pragma unroll
  for (int m = 0; m < MT; ++m) sc[m][0] = sc[m][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    bf16x8_t kf[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float s = e8m0_operand(D == 256 ? (k.s[b] >> (8 * (j / 4))) & 0xFFu : k.s[b]);
      const uint32_t c = k.c[b][j];
      const u32x4_t x{fp4_pair<0>(c, s), fp4_pair<1>(c, s), fp4_pair<2>(c, s), fp4_pair<3>(c, s)};
      kf[b] = __builtin_bit_cast(bf16x8_t, x);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const bf16x8_t qf = q.at(m, j);
      sc[m][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0], qf, sc[m][0], 0, 0, 0);
      sc[m][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[1], qf, sc[m][1], 0, 0, 0);
    }
  }
}

// What the lane's rows do not see of 32 tokens from t0: row n of tile m, at
// position pos[m], sees `window` tokens up to its own.
template <int MT>
__device__ __forceinline__ void mask_scores(f32x4_t (&sc)[MT][2], const int (&pos)[MT], int window, int t0, int g) {
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int most = pos[m] < 0 ? 0 : pos[m] + 1;
    const int span = window > 0 && window < most ? window : most;  // its tokens, up to pos
    const int from = t0 + 4 * g - (pos[m] - span + 1);
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sc[m][b][e] = (uint32_t)(from + b * kKvBlock + e) < (uint32_t)span ? sc[m][b][e] : -INFINITY;
  }
}

// Tokens that do not exist: what their bytes say is anything, and zero times it
// has to be zero.
template <int D>
__device__ __forceinline__ void clear_values(KvValues<D>& v, const int (&held)[2], int g) {
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * g + i >= held[b]) {
        v.s[b] &= ~(0xFFu << (8 * i));
        if constexpr (D == 64) v.c[b][i >> 1] &= ~(0xFFFFu << (16 * (i & 1)));
        else if constexpr (D == 128) v.c[b][i] = 0u;
        else v.c[b][2 * i] = v.c[b][2 * i + 1] = 0u;
      }
}

// Weights of 32 tokens as the second operand of the second product, in bf16 (its
// sums stay in fp32: an output is off by about the rounding of a bf16).  They are
// taken against a reference that is at most kLate binades below the row's largest
// score so far, so that they stay below 2^kLate: lanes look at their own scores
// and exchange them only when one goes past that, which is rare after the first
// tiles.  A score past fp32 makes the row NaN (infinity less itself), one below it
// weighs nothing.  The reference is a rounded product, weights are exact against it: their
// largest is 2^(half a step of it) at most, in range up to references of 2^30 binades.
template <int D, int MT>
__device__ __forceinline__ void take_weights(bf16x8_t (&p)[MT], Rows<D, MT>& w, const f32x4_t (&sc)[MT][2],
                                             float scale_log2) {
  float most[MT];
  bool late = false;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    most[m] = sc[m][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most[m] = fmaxf(most[m], sc[m][i >> 2][i & 3]);
    late = late || fmaf(most[m], scale_log2, -w.top[m]) > kLate;
  }
  if (__any(late)) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const float t = fmaxf(w.top[m], max_over_groups(most[m]) * scale_log2);
      const float f = __builtin_amdgcn_exp2f(w.top[m] - t) + (t - t);
      w.sum[m] *= f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) w.o[m][c] *= f;
      w.top[m] = t;
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    float e8[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e8[i] = __builtin_amdgcn_exp2f(fmaf(sc[m][i >> 2][i & 3], scale_log2, -w.top[m]));
      w.sum[m] += e8[i];
    }
    const u32x4_t x{pack_bf16(e8[0], e8[1]), pack_bf16(e8[2], e8[3]), pack_bf16(e8[4], e8[5]), pack_bf16(e8[6], e8[7])};
    p[m] = __builtin_bit_cast(bf16x8_t, x);
  }
}

// The second product: columns 2 c, 2 c + 1 of the lane's part are a byte of each
// of its eight tokens.
template <int D, int MT>
__device__ __forceinline__ void take_values(Rows<D, MT>& w, const KvValues<D>& v, const bf16x8_t (&p)[MT]) {
  float s[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) s[b][i] = e8m0_operand_at(v.s[b], i);
#pragma unroll
  for (int c = 0; c < D / 32; ++c) {
    uint32_t x8[8];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = i * (D / 32) + c;  // byte of the lane's D/8
        x8[4 * b + i] = fp4_pair_at(v.c[b][at / 4], s[b][i], at % 4);
      }
    u32x4_t x, y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = __builtin_amdgcn_perm(x8[2 * i + 1], x8[2 * i], 0x05040100u);
      y[i] = __builtin_amdgcn_perm(x8[2 * i + 1], x8[2 * i], 0x07060302u);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      w.o[m][2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), p[m], w.o[m][2 * c], 0, 0, 0);
      w.o[m][2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, y), p[m], w.o[m][2 * c + 1], 0, 0, 0);
    }
  }
}

// A workgroup is 4 waves, WT of which (4 or 2) share the tokens of the same rows
// while 4 / WT have rows of their own, or 8 that share the tokens of one group of rows.
constexpr int waves_in(int wt) { return wt == 8 ? 8 : 4; }
// Waves of a SIMD that the registers leave room for, and the stages of a ring.
constexpr int waves_of(int d, int mt, int wt) {
  return wt == 8 ? (d == 128 ? 4 : 2) : d * mt <= 128 ? 4 : (mt < 4 && d * mt <= 256 ? 3 : 2);
}
constexpr bool queries_in_lds(int d, int mt) { return d * mt >= 512; }
constexpr int stages_of(int d, int wt) { return d == 64 ? 4 : (d == 128 && wt < 8 ? 3 : 2); }
// LDS of a workgroup: rings and queries, in their place the waves' outputs.
constexpr int attend_lds(int d, int mt, int wt) {
  const int nw = waves_in(wt);
  const int run = nw * stages_of(d, wt) * ((34 * d + 255) / 256 * 256) +
                  (queries_in_lds(d, mt) ? nw / wt * mt * (d / 32) * 1024 : 0);
  const int end = nw * (64 * d + 128 * mt);
  return run > end ? run : end;
}
constexpr int resident(int d, int mt, int wt) {  // workgroups of a CU
  const int by_lds = 160 * 1024 / attend_lds(d, mt, wt), by_waves = waves_of(d, mt, wt) * 4 / waves_in(wt);
  return by_lds < by_waves ? by_lds : by_waves;
}
// Tokens that rows r_lo ... r_hi of a session see (lo ... hi - 1, lo down to a whole
// tile) and those that all of them see.  base: position of row 0, from -kKvMost on;
// window below kKvMost (kv_window), so that nothing passes 32 bits.
struct KvSpan {
  int lo, hi, all_lo, all_hi;
};
__host__ __device__ __forceinline__ KvSpan kv_span(int base, int r_lo, int r_hi, int window) {
  KvSpan t{0, base + r_hi + 1, 0, base + r_lo + 1};
  if (window > 0) {
    t.lo = base + r_lo - window + 1;
    t.all_lo = base + r_hi - window + 1;
  }
  t.lo = t.lo > 0 ? t.lo & ~31 : 0;
  t.hi = t.hi > 0 ? t.hi : 0;  // rows before the first token see none, and name no page
  t.all_hi = t.all_hi > 0 ? t.all_hi : 0;
  return t;
}
// The tokens of one share of them; the last takes what is left.
struct KvShare {
  int from, to;
};
__host__ __device__ __forceinline__ KvShare kv_share(const KvSpan& t, int split, int splits, int chunk) {
  KvShare r;
  r.from = t.lo + split * chunk;
  r.to = split == splits - 1 ? t.hi : (r.from + chunk < t.hi ? r.from + chunk : t.hi);
  return r;
}

}  // namespace sph

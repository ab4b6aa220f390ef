// Attention of every session's last rows over its paged 4-bit cache.
//
//   o[r, h] = sum_j p_j V[j, h / G],  p = softmax_j(scale q[r, h] . K[j, h / G])
//   over the positions j that row r sees: j <= pos(r) = len - rows + r and, with
//   a window, j > pos(r) - window.
//
// The rows of all G query heads of one key/value head are one matrix of R G
// rows.  A wave takes MT tiles of 16 of them and walks over 32 tokens at a time:
//   S^T = K Q^T     (tokens x rows) 16x16x32 products, K from registers
//   O^T += V^T P^T  (dimensions x rows), P from the registers of S
// Both products contract over an axis whose order is free as long as the two
// operands agree, so codes go from memory to registers in the order they are
// stored and are never exchanged between lanes: lane l = 16 g + n reads
//   K  token n of the block, dimensions g D/4 ... (row n of the first operand)
//   V  tokens 4 g ... 4 g + 3, part n (row n of V^T for D/16 products)
// and the scores that lane l receives, row n of the tile against tokens
// 4 g ... 4 g + 3 of both blocks, are its operand of the second product.  A
// lane's outputs are D/4 neighbouring values of one row.
#include "kv_cache.h"
#include "mfma_tile.h"

namespace sph {

struct AttendArgs {
  KvArgs kv;
  const uint16_t* q;     // bf16 [M][q_heads][D]
  int64_t q_row, q_head;
  uint16_t* out;         // bf16 [M][q_heads][D]
  int64_t o_row, o_head;
  float* lse;            // fp32 [M][q_heads] or null
  int group;             // query heads of a key/value head
  int window;            // 0: none
  float scale, scale_log2;
  float late;            // kLate binades of weight, as a difference of raw scores
  bool q_aligned, o_aligned;
  int tiles;             // blocks of rows of a session and head
  int splits, chunk;     // shares of the tokens, tokens of one
  float2* part_ml;       // [rows x heads][splits]: maximum of the raw scores, sum
  float* part_o;         // [rows x heads][splits][D]
};

constexpr float kNoScore = -1.0e30f;  // finite, also times a scale: differences with it are no NaN
constexpr float kLate = 8.0f;
constexpr float kLn2 = 0.693147180559945f;

// A lane's share of 32 tokens: codes, the scale bytes of its keys (one, two for D
// 256) and of its values (four tokens).
template <int D>
struct KvTile {
  uint32_t k[2][D / 32], v[2][D / 32];
  uint32_t ks[2], vs[2];
};

// Pages of a tile's two blocks, -1 for one that no row of the wave sees or the
// table does not name.
struct KvPages {
  int page[2];
};
__device__ __forceinline__ KvPages tile_pages(const KvArgs& a, const KvSession& ses, int pos, int end) {
  KvPages p;
#pragma unroll
  for (int b = 0; b < 2; ++b) p.page[b] = pos + b * kKvBlock < end ? kv_page(a, ses, pos + b * kKvBlock) : -1;
  return p;
}

template <int N>
__device__ __forceinline__ void load_words(uint32_t (&r)[N], const uint8_t* p) {
  if constexpr (N == 2) {
    const u32x2_t x = *reinterpret_cast<const u32x2_t*>(p);
    r[0] = x[0], r[1] = x[1];
  } else {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p + 16 * i);
#pragma unroll
      for (int e = 0; e < 4; ++e) r[4 * i + e] = x[e];
    }
  }
}

// A block that does not exist is read from page 0 and not used.
template <int D>
__device__ __forceinline__ void load_tile(KvTile<D>& t, const KvArgs& a, int head, int pos, const KvPages& pages,
                                          uint32_t lane) {
  const uint32_t g = lane >> 4, n = lane & 15;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int page = pages.page[b];
    const uint8_t* blk = scalar_ptr(kv_block<D>(a, page < 0 ? 0 : page, head, page < 0 ? 0 : pos + b * kKvBlock));
    load_words(t.k[b], blk + (n * (D / 2) + g * (D / 8)));
    load_words(t.v[b], blk + (KvLayout<D>::kValues + lane * (D / 8)));
    constexpr uint32_t KS = KvLayout<D>::kKeyScales;
    if constexpr (D == 64) t.ks[b] = blk[KS + (g >> 1) * kKvBlock + n];
    else if constexpr (D == 128) t.ks[b] = blk[KS + g * kKvBlock + n];
    else t.ks[b] = blk[KS + 2 * g * kKvBlock + n] | ((uint32_t)blk[KS + (2 * g + 1) * kKvBlock + n] << 8);
    t.vs[b] = *reinterpret_cast<const uint32_t*>(blk + (KvLayout<D>::kValueScales + n * D / 512 * kKvBlock + 4 * g));
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

// 32 tokens from position t0.  MASK: some of them are not for all of the rows:
// held[b] tokens of either block exist, row n of tile m stands at pos[m].
template <int D, int MT, bool MASK>
__device__ __forceinline__ void take_tile(Rows<D, MT>& w, KvTile<D>& cur, const bf16x8_t (&q)[MT][D / 32],
                                          const AttendArgs& a, int t0, const int (&held)[2], const int (&pos)[MT],
                                          int g) {
  constexpr int KJ = D / 32;  // steps of the first product
  constexpr int VC = D / 16;  // products of the second
  if constexpr (MASK) {
    // tokens that do not exist: what their bytes say is anything, and zero times
    // it has to be zero
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (4 * g + i >= held[b]) {
          cur.vs[b] &= ~(0xFFu << (8 * i));
          if constexpr (D == 64) cur.v[b][i >> 1] &= ~(0xFFFFu << (16 * (i & 1)));
          else if constexpr (D == 128) cur.v[b][i] = 0u;
          else cur.v[b][2 * i] = cur.v[b][2 * i + 1] = 0u;
        }
  }

  // scores: lane l has row n against tokens 4 g + e of both blocks
  f32x4_t sc[MT][2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
#pragma unroll
    for (int m = 0; m < MT; ++m) sc[m][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      const float ks = e8m0_operand(D == 256 ? (cur.ks[b] >> (8 * (j / 4))) & 0xFFu : cur.ks[b]);
      const uint32_t c = cur.k[b][j];
      const u32x4_t x{fp4_pair<0>(c, ks), fp4_pair<1>(c, ks), fp4_pair<2>(c, ks), fp4_pair<3>(c, ks)};
      const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, x);
#pragma unroll
      for (int m = 0; m < MT; ++m)
        sc[m][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[m][j], sc[m][b], 0, 0, 0);
    }
  }
  if constexpr (MASK) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int in = 4 * g + e, j = t0 + b * kKvBlock + in;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          const bool sees = in < held[b] && j <= pos[m] && (a.window <= 0 || j > pos[m] - a.window);
          sc[m][b][e] = sees ? sc[m][b][e] : -INFINITY;
        }
      }
  }

  // Weights are taken against a reference that is at most kLate binades below the
  // row's largest score so far (so that weights stay below 2^kLate): lanes look
  // at their own scores and exchange them only when one goes past that, which is
  // rare after the first tiles.
  float most[MT];
  bool late = false;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    most[m] = sc[m][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) most[m] = fmaxf(most[m], sc[m][i >> 2][i & 3]);
    late = late || most[m] > w.top[m] + a.late;
  }
  if (__any(late)) {
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const float t = fmaxf(w.top[m], max_over_groups(most[m]));
      const float f = __builtin_amdgcn_exp2f((w.top[m] - t) * a.scale_log2);
      w.sum[m] *= f;
#pragma unroll
      for (int c = 0; c < VC; ++c) w.o[m][c] *= f;
      w.top[m] = t;
    }
  }
  // P rounded to bf16 for the second product (its sums stay in fp32: an output is
  // off by about the rounding of a bf16)
  bf16x8_t p[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const float off = w.top[m] * a.scale_log2;
    float e8[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e8[i] = __builtin_amdgcn_exp2f(fmaf(sc[m][i >> 2][i & 3], a.scale_log2, -off));
      w.sum[m] += e8[i];
    }
    const u32x4_t x{pack_bf16(e8[0], e8[1]), pack_bf16(e8[2], e8[3]), pack_bf16(e8[4], e8[5]), pack_bf16(e8[6], e8[7])};
    p[m] = __builtin_bit_cast(bf16x8_t, x);
  }

  float vs[2][4];
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) vs[b][i] = e8m0_operand((cur.vs[b] >> (8 * i)) & 0xFFu);
  // columns 2 c, 2 c + 1 of the lane's part: a byte of each of its eight tokens
#pragma unroll
  for (int c = 0; c < VC / 2; ++c) {
    uint32_t x8[8];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = i * (D / 32) + c;  // byte of the lane's D/8
        x8[4 * b + i] = fp4_pair_at(cur.v[b][at / 4], vs[b][i], at % 4);
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

// A workgroup is 4 waves: WT of them share the tokens of the same rows, 4 / WT
// have rows of their own.
#ifndef WPE
#define WPE(D, MT) ((D) * (MT) <= 128 ? 3 : (D) * (MT) <= 256 ? 2 : 1)
#endif
template <int D, int MT, int WT>
__global__ __launch_bounds__(256, WPE(D, MT)) void k_kv_attend(AttendArgs a) {
  constexpr int WR = 4 / WT;
  constexpr int KJ = D / 32;   // steps of the first product
  constexpr int VC = D / 16;   // products of the second
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wt = wave % WT, wr = wave / WT;

  const int units = a.kv.heads * a.kv.n_sessions;
  const int unit = blockIdx.x % units;
  const int rest = blockIdx.x / units;
  const int split = rest % a.splits;
  const int tile = a.tiles - 1 - rest / a.splits;  // rows that see most come first
  const int head = unit % a.kv.heads, s = unit / a.kv.heads;
  const KvSession ses = kv_session(a.kv, s);
  const int G = a.group, total = a.kv.R * G, live = ses.rows * G;
  const int base = ses.len - ses.rows;
  const int row0 = (tile * WR + wr) * 16 * MT;     // the wave's first of total rows

  // rows: fq = r G + query head; those past the session's see nothing
  bf16x8_t q[MT][KJ];
  int pos[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int fq = row0 + m * 16 + n;
    const int r = fq / G;
    pos[m] = fq < live ? base + r : -1;
    const uint16_t* p = a.q + ((int64_t)s * a.kv.R + r) * a.q_row + (int64_t)(head * G + fq - r * G) * a.q_head + g * (D / 4);
#pragma unroll
    for (int j = 0; j < KJ; ++j) {
      u32x4_t x{0u, 0u, 0u, 0u};
      if (fq < live) {
        if (a.q_aligned) {
          x = *reinterpret_cast<const u32x4_t*>(p + 8 * j);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = (uint32_t)p[8 * j + 2 * i] | ((uint32_t)p[8 * j + 2 * i + 1] << 16);
        }
      }
      q[m][j] = __builtin_bit_cast(bf16x8_t, x);
    }
  }

  // tokens that the wave's rows see, and those that all of them see
  const int last_row = (row0 + 16 * MT < live ? row0 + 16 * MT : live) - 1;
  int lo = 0, hi = 0, all_lo = 0, all_hi = 0;
  if (row0 < live) {
    const int r_lo = row0 / G, r_hi = last_row / G;
    hi = base + r_hi + 1;
    all_hi = base + r_lo + 1;
    if (a.window > 0) {
      lo = base + r_lo - a.window + 1;
      all_lo = base + r_hi - a.window + 1;
    }
    lo = lo > 0 ? lo & ~31 : 0;
  }
  // the share of this workgroup; the last takes what is left
  const int from = lo + split * a.chunk;
  const int to = split == a.splits - 1 ? hi : (from + a.chunk < hi ? from + a.chunk : hi);

  Rows<D, MT> w;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    w.top[m] = kNoScore;
    w.sum[m] = 0.0f;
#pragma unroll
    for (int c = 0; c < VC; ++c) w.o[m][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // The wave's tiles from `start` on, STEP tokens apart.  Those that all its rows
  // see whole, from `whole` to `part`, come first, then the others: the order of
  // tokens is free.  A wave that finds a page missing takes all as the latter.
  constexpr int STEP = 32 * WT;
  const int start = from + 32 * wt;
  int whole = start + (all_lo > start ? (all_lo - start + STEP - 1) / STEP * STEP : 0);
  int part = whole + ((all_hi < to ? all_hi : to) - whole + STEP - 32) / STEP * STEP;
  if (part > whole) {
    bool missing = false;
    for (int c = (whole >> a.kv.page_shift) + lane; c <= (part - STEP + 31) >> a.kv.page_shift; c += 64)
      missing = missing || kv_page(a.kv, ses, c << a.kv.page_shift) < 0;
    if (__any(missing)) part = whole;
  }
  if (part <= whole) whole = part = start;
  const int n_whole = (part - whole) / STEP, n_head = (whole - start) / STEP;
  const int n_tiles = n_whole + n_head + (to > part ? (to - part + STEP - 1) / STEP : 0);
  auto place = [&](int k) {
    if (k >= n_tiles) return to;
    return k < n_whole ? whole + k * STEP : (k < n_whole + n_head ? start : part - n_head * STEP) + (k - n_whole) * STEP;
  };

  // codes are asked for one tile ahead, pages two
  KvTile<D> next;
  KvPages here = tile_pages(a.kv, ses, place(0), to);
  if (n_tiles > 0) load_tile<D>(next, a.kv, head, place(0), here, lane);
  KvPages ahead = tile_pages(a.kv, ses, place(1), to);
  int k = 0;
  for (; k < n_whole; ++k) {
    KvTile<D> cur = next;
    const KvPages after = tile_pages(a.kv, ses, place(k + 2), to);
    if (k + 1 < n_tiles) load_tile<D>(next, a.kv, head, place(k + 1), ahead, lane);
    const int held[2] = {kKvBlock, kKvBlock};
    take_tile<D, MT, false>(w, cur, q, a, 0, held, pos, g);
    here = ahead;
    ahead = after;
  }
  for (; k < n_tiles; ++k) {
    KvTile<D> cur = next;
    const int t0 = place(k);
    const KvPages after = tile_pages(a.kv, ses, place(k + 2), to);
    if (k + 1 < n_tiles) load_tile<D>(next, a.kv, head, place(k + 1), ahead, lane);
    int held[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int left = to - t0 - b * kKvBlock;
      held[b] = here.page[b] < 0 ? 0 : (left < kKvBlock ? left : kKvBlock);
    }
    take_tile<D, MT, true>(w, cur, q, a, t0, held, pos, g);
    here = ahead;
    ahead = after;
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) w.sum[m] = sum_over_groups(w.sum[m]);

  // lane l holds row n, dimensions (4 g + e) D/16 + c = w.o[m][c][e]
  __shared__ float s_ml[WT > 1 ? 4 * MT * 16 * 2 : 1];
  __shared__ float s_o[WT > 1 ? 4 * D * 16 : 1];
  if constexpr (WT > 1) {
    if (g == 0)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        s_ml[((wave * MT + m) * 16 + n) * 2] = w.top[m];
        s_ml[((wave * MT + m) * 16 + n) * 2 + 1] = w.sum[m];
      }
    __syncthreads();
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    float t = w.top[m], l = w.sum[m];
    constexpr int PER = WT > 1 ? (D / 4) / WT : D / 4;  // values a lane ends with
    float y[PER];
    int d0;  // its first dimension
    if constexpr (WT > 1) {
      t = kNoScore;
#pragma unroll
      for (int k = 0; k < WT; ++k) t = fmaxf(t, s_ml[(((wr * WT + k) * MT + m) * 16 + n) * 2]);
      l = 0.0f;
#pragma unroll
      for (int k = 0; k < WT; ++k) {
        const float* ml = &s_ml[(((wr * WT + k) * MT + m) * 16 + n) * 2];
        l += ml[1] * __builtin_amdgcn_exp2f((ml[0] - t) * a.scale_log2);
      }
      const float f = __builtin_amdgcn_exp2f((w.top[m] - t) * a.scale_log2);
      if (m > 0) __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VC; ++c) s_o[((wave * 4 + e) * VC + c) * 64 + lane] = w.o[m][c][e] * f;
      __syncthreads();
      // wave wt of WT sums its share of the (e, c) pairs over the WT waves
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        float x = 0.0f;
#pragma unroll
        for (int k = 0; k < WT; ++k) x += s_o[((wr * WT + k) * 4 * VC + wt * PER + i) * 64 + lane];
        y[i] = x;
      }
      d0 = g * (D / 4) + wt * PER;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VC; ++c) y[e * VC + c] = w.o[m][c][e];
      d0 = g * (D / 4);
    }
    const int fq = row0 + m * 16 + n;
    if (fq >= live) l = 0.0f;  // rows that are none
    if (fq < total) {
      const int r = fq / G, hq = head * G + fq - r * G;
      const int64_t row = (int64_t)s * a.kv.R + r;
      if (a.splits == 1) {
        const float f = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t* dst = a.out + row * a.o_row + hq * a.o_head + d0;
#pragma unroll
        for (int i = 0; i < PER; i += 2) {
          const uint32_t w = pack_bf16(l == 0.0f ? 0.0f : y[i] * f, l == 0.0f ? 0.0f : y[i + 1] * f);
          if (a.o_aligned) {
            *reinterpret_cast<uint32_t*>(dst + i) = w;
          } else {
            dst[i] = (uint16_t)w;
            dst[i + 1] = (uint16_t)(w >> 16);
          }
        }
        if (a.lse && g == 0 && (WT == 1 || wt == 0))
          a.lse[row * (a.kv.heads * G) + hq] = l == 0.0f ? -INFINITY : fmaf(t, a.scale, __builtin_amdgcn_logf(l) * kLn2);
      } else {
        const int64_t at = (row * (a.kv.heads * G) + hq) * a.splits + split;
        if (g == 0 && (WT == 1 || wt == 0)) a.part_ml[at] = make_float2(t, l);
        if (!(l == 0.0f)) {
#pragma unroll
          for (int i = 0; i < PER; i += 4)
            *reinterpret_cast<f32x4_t*>(a.part_o + at * D + d0 + i) = f32x4_t{y[i], y[i + 1], y[i + 2], y[i + 3]};
        }
      }
    }
  }
}

// The shares of a row joined: a workgroup a row and head, D/4 lanes for a share,
// the shares in turns; sums in an order that is always the same.
template <int D>
__global__ __launch_bounds__(256) void k_kv_join(AttendArgs a) {
  constexpr int LPS = D / 4, TURNS = 256 / LPS;  // 16, 32 or 64 lanes
  __shared__ float s_l[TURNS];
  __shared__ f32x4_t s_o[256];
  const int d4 = threadIdx.x % LPS, turn = threadIdx.x / LPS;
  const int64_t i = blockIdx.x;
  const int heads = a.kv.heads * a.group;
  const int64_t row = i / heads;
  const int hq = (int)(i - row * heads);
  const float2* ml = a.part_ml + i * a.splits;
  const float* part = a.part_o + i * a.splits * D + d4 * 4;
  float t = kNoScore;
  for (int k = threadIdx.x & 63; k < a.splits; k += 64) t = fmaxf(t, ml[k].x);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) t = fmaxf(t, __shfl_xor(t, o, 64));
  float l = 0.0f;
  f32x4_t y{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int k = turn; k < a.splits; k += TURNS) {
    const float2 x = ml[k];
    const bool some = !(x.y == 0.0f);  // shares without a token left their place unwritten
    const float f = some ? __builtin_amdgcn_exp2f((x.x - t) * a.scale_log2) : 0.0f;
    f32x4_t o{0.0f, 0.0f, 0.0f, 0.0f};
    if (some) o = *reinterpret_cast<const f32x4_t*>(part + (int64_t)k * D);
    l += some ? x.y * f : 0.0f;
    y += o * f;
  }
  s_o[threadIdx.x] = y;
  if (d4 == 0) s_l[turn] = l;
  __syncthreads();
  if (turn != 0) return;
#pragma unroll
  for (int k = 1; k < TURNS; ++k) {
    y += s_o[k * LPS + d4];
    l += s_l[k];
  }
  const float f = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* dst = a.out + row * a.o_row + hq * a.o_head + d4 * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e) dst[e] = (uint16_t)pack_bf16(l == 0.0f ? 0.0f : y[e] * f, 0.0f);
  if (a.lse && d4 == 0)
    a.lse[i] = l == 0.0f ? -INFINITY : fmaf(t, a.scale, __builtin_amdgcn_logf(l) * kLn2);
}

namespace {

struct Plan {
  int mt, wt, tiles, splits, chunk;
};

// How rows and tokens are shared out.  R G rows of one head: up to 16 MT in a
// workgroup whose four waves share the tokens, or 64 MT with rows a wave.
Plan plan_of(int d, int64_t units, int64_t rows, int64_t span) {
  Plan p;
#ifndef M64
#define M64 4
#endif
#ifndef M128
#define M128 2
#endif
#ifndef M256
#define M256 1
#endif
  const int most = d == 64 ? M64 : (d == 128 ? M128 : M256);
  p.mt = 1;
  while (p.mt < most && rows > 16 * p.mt) p.mt *= 2;
  p.wt = 4;
  while (p.wt > 1 && rows > 16 * p.mt * (4 / p.wt)) p.wt /= 2;
  const int per = 16 * p.mt * (4 / p.wt);
  p.tiles = (int)((rows + per - 1) / per);
#ifndef BLOCKS
#define BLOCKS 512
#endif
  // as many workgroups as the chip holds at a time, with 256 tokens at least
  int64_t splits = 1;
  if (units * p.tiles > 0) splits = BLOCKS / (units * p.tiles);
  const int64_t least = 256;
  if (splits > (span + least - 1) / least) splits = (span + least - 1) / least;
  if (splits < 1) splits = 1;
  int64_t chunk = ((span + splits - 1) / splits + 127) / 128 * 128;
  if (chunk < 128) chunk = 128;
  p.chunk = (int)chunk;
  p.splits = (int)((span + chunk - 1) / chunk);
  if (p.splits < 1) p.splits = 1;
  return p;
}

int64_t span_of(int64_t max_len, int64_t rows, int64_t window) {
  return window > 0 && window + rows + 31 < max_len ? window + rows + 31 : max_len;
}

template <int D, int MT, int WT>
void launch_one(const AttendArgs& a, int64_t blocks, hipStream_t s) {
  launch_kernel(k_kv_attend<D, MT, WT>, dim3((unsigned)blocks), dim3(256), 0, s, a);
}

template <int D, int MT>
void launch_waves(const Plan& p, const AttendArgs& a, int64_t blocks, hipStream_t s) {
  if (p.wt == 4) launch_one<D, MT, 4>(a, blocks, s);
  else if (p.wt == 2) launch_one<D, MT, 2>(a, blocks, s);
  else launch_one<D, MT, 1>(a, blocks, s);
}

template <int D>
void launch_tiles(const Plan& p, const AttendArgs& a, int64_t blocks, hipStream_t s) {
  constexpr int M = D == 64 ? M64 : (D == 128 ? M128 : M256);
  if (p.mt == M) launch_waves<D, M>(p, a, blocks, s);
  else if constexpr (M > 1) {
    if (p.mt == 1) launch_one<D, 1, 4>(a, blocks, s);
    else if constexpr (M > 2) launch_one<D, 2, 4>(a, blocks, s);
  }
}

}  // namespace

// Workspace: the shares' maxima and sums, then their outputs.
size_t kv_attend_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads,
                         int64_t max_len, int64_t window) {
  const Plan p = plan_of(d, n_sessions * heads, R * (q_heads / heads), span_of(max_len, R, window));
  if (p.splits <= 1) return 0;
  const size_t n = (size_t)n_sessions * R * q_heads * p.splits;
  return (n * 8 + 255) / 256 * 256 + n * d * 4;
}

hipError_t launch_kv_attend(int d, const KvArgs& kv, const AttendCall& c, void* workspace, hipStream_t s) {
  if (kv.n_sessions <= 0 || kv.R <= 0) return hipSuccess;
  AttendArgs a{};
  a.kv = kv;
  a.q = static_cast<const uint16_t*>(c.q);
  a.q_row = c.q_row;
  a.q_head = c.q_head;
  a.out = static_cast<uint16_t*>(c.out);
  a.o_row = c.o_row;
  a.o_head = c.o_head;
  a.lse = c.lse;
  a.group = c.q_heads / kv.heads;
  a.window = c.window;
  a.scale = c.scale;
  a.scale_log2 = c.scale * 1.44269504088896f;
  a.late = kLate / a.scale_log2;
  a.q_aligned = c.q_row % 8 == 0 && c.q_head % 8 == 0 && (reinterpret_cast<uintptr_t>(c.q) & 15) == 0;
  a.o_aligned = c.o_row % 2 == 0 && c.o_head % 2 == 0 && (reinterpret_cast<uintptr_t>(c.out) & 3) == 0;
  const int64_t units = (int64_t)kv.n_sessions * kv.heads;
  const Plan p = plan_of(d, units, (int64_t)kv.R * a.group, span_of(c.max_len, kv.R, c.window));
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.chunk = p.chunk;
  const int64_t rows = (int64_t)kv.n_sessions * kv.R * c.q_heads;
  if (p.splits > 1) {
    a.part_ml = static_cast<float2*>(workspace);
    a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + ((size_t)rows * p.splits * 8 + 255) / 256 * 256);
  }
  const int64_t blocks = units * p.tiles * p.splits;
  if (blocks > 0x7FFFFFFF || rows > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (d == 64) launch_tiles<64>(p, a, blocks, s);
  else if (d == 128) launch_tiles<128>(p, a, blocks, s);
  else if (d == 256) launch_tiles<256>(p, a, blocks, s);
  else return hipErrorInvalidValue;
  if (p.splits > 1) {
    const dim3 grid((unsigned)rows);
    if (d == 64) launch_kernel(k_kv_join<64>, grid, dim3(256), 0, s, a);
    else if (d == 128) launch_kernel(k_kv_join<128>, grid, dim3(256), 0, s, a);
    else launch_kernel(k_kv_join<256>, grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sph

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
  bool q_aligned, o_aligned;
  int tiles;             // blocks of rows of a session and head
  int splits, chunk;     // shares of the tokens, tokens of one
  float2* part_ml;       // [rows x heads][splits]: maximum of the raw scores, sum
  float* part_o;         // [rows x heads][splits][D]
};

constexpr float kNoScore = -1.0e30f;  // finite, also times a scale: differences with it are no NaN
constexpr float kLn2 = 0.693147180559945f;

template <int D>
struct KvTile {  // a lane's share of 32 tokens
  uint32_t k[2][D / 32], v[2][D / 32];
  uint32_t ks[2], vs[2];  // scale bytes: keys' D/128 (at least one), values' four
  int held[2];            // tokens of either block that exist
};

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

template <int D>
__device__ __forceinline__ void load_tile(KvTile<D>& t, const KvArgs& a, const KvSession& ses, int head,
                                          int pos, int end, int lane) {
  const int g = lane >> 4, n = lane & 15;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int p0 = pos + b * kKvBlock;
    int page = p0 < end ? kv_page(a, ses, p0) : -1;
    const int left = ses.len - p0;
    t.held[b] = page < 0 ? 0 : (left < kKvBlock ? left : kKvBlock);
    // a block that does not exist is read from page 0 and not used
    const uint8_t* blk = kv_block<D>(a, page < 0 ? 0 : page, head, page < 0 ? 0 : p0);
    load_words(t.k[b], blk + n * (D / 2) + g * (D / 8));
    load_words(t.v[b], blk + KvLayout<D>::kValues + lane * (D / 8));
    const uint8_t* ks = blk + KvLayout<D>::kKeyScales + n;
    if constexpr (D == 64) t.ks[b] = ks[(g >> 1) * kKvBlock];
    else if constexpr (D == 128) t.ks[b] = ks[g * kKvBlock];
    else t.ks[b] = ks[2 * g * kKvBlock] | ((uint32_t)ks[(2 * g + 1) * kKvBlock] << 8);
    t.vs[b] = *reinterpret_cast<const uint32_t*>(blk + KvLayout<D>::kValueScales + n * D / 512 * kKvBlock + 4 * g);
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

// A workgroup is 4 waves: WT of them share the tokens of the same rows, 4 / WT
// have rows of their own.
template <int D, int MT, int WT>
__global__ __launch_bounds__(256) void k_kv_attend(AttendArgs a) {
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

  f32x4_t o[MT][VC];
  float top[MT], sum[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    top[m] = kNoScore;
    sum[m] = 0.0f;
#pragma unroll
    for (int c = 0; c < VC; ++c) o[m][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  }

  int t0 = from + 32 * wt;
  KvTile<D> next;
  if (t0 < to) load_tile<D>(next, a.kv, ses, head, t0, to, lane);
  for (; t0 < to; t0 += 32 * WT) {
    KvTile<D> cur = next;
    if (t0 + 32 * WT < to) load_tile<D>(next, a.kv, ses, head, t0 + 32 * WT, to, lane);

    const bool whole = cur.held[0] == kKvBlock && cur.held[1] == kKvBlock && t0 >= all_lo &&
                       t0 + 32 <= all_hi && t0 + 32 <= to;
    if (!whole) {
      // tokens that do not exist: what their bytes say is anything, and zero
      // times it has to be zero
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * g + i >= cur.held[b]) {
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
        const uint32_t w = cur.k[b][j];
        const u32x4_t x{fp4_pair<0>(w, ks), fp4_pair<1>(w, ks), fp4_pair<2>(w, ks), fp4_pair<3>(w, ks)};
        const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, x);
#pragma unroll
        for (int m = 0; m < MT; ++m)
          sc[m][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, q[m][j], sc[m][b], 0, 0, 0);
      }
    }
    if (!whole) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int in = 4 * g + e, j = t0 + b * kKvBlock + in;
          const bool exists = in < cur.held[b] && j < to;
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const bool sees = exists && j <= pos[m] && (a.window <= 0 || j > pos[m] - a.window);
            sc[m][b][e] = sees ? sc[m][b][e] : -INFINITY;
          }
        }
    }

    // running maximum and sum; P rounded to bf16 for the second product (its
    // sums stay in fp32: an output is off by about the rounding of a bf16)
    bf16x8_t p[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      float t = top[m];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) t = fmaxf(t, sc[m][b][e]);
      t = max_over_groups(t);
      if (__any(t > top[m])) {
        const float f = __builtin_amdgcn_exp2f((top[m] - t) * a.scale_log2);
        sum[m] *= f;
#pragma unroll
        for (int c = 0; c < VC; ++c) o[m][c] *= f;
        top[m] = t;
      }
      const float off = t * a.scale_log2;
      float e8[8];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          e8[4 * b + e] = __builtin_amdgcn_exp2f(fmaf(sc[m][b][e], a.scale_log2, -off));
          sum[m] += e8[4 * b + e];
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
      uint32_t w[8];
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int at = i * (D / 32) + c;  // byte of the lane's D/8
          const uint32_t word = cur.v[b][at / 4] >> (8 * (at % 4));
          w[4 * b + i] = fp4_pair<0>(word, vs[b][i]);
        }
      u32x4_t x, y;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100u);
        y[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302u);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        o[m][2 * c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), p[m], o[m][2 * c], 0, 0, 0);
        o[m][2 * c + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, y), p[m], o[m][2 * c + 1], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) sum[m] = sum_over_groups(sum[m]);

  // lane l holds row n, dimensions (4 g + e) D/16 + c = o[m][c][e]
  __shared__ float s_ml[WT > 1 ? 4 * MT * 16 * 2 : 1];
  __shared__ float s_o[WT > 1 ? 4 * D * 16 : 1];
  if constexpr (WT > 1) {
    if (g == 0)
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        s_ml[((wave * MT + m) * 16 + n) * 2] = top[m];
        s_ml[((wave * MT + m) * 16 + n) * 2 + 1] = sum[m];
      }
    __syncthreads();
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    float t = top[m], l = sum[m];
    constexpr int PER = WT > 1 ? (D / 4) / WT : D / 4;  // values a lane ends with
    float y[PER];
    int d0;  // its first dimension
    if constexpr (WT > 1) {
      t = kNoScore;
#pragma unroll
      for (int w = 0; w < WT; ++w) t = fmaxf(t, s_ml[(((wr * WT + w) * MT + m) * 16 + n) * 2]);
      l = 0.0f;
#pragma unroll
      for (int w = 0; w < WT; ++w) {
        const float* ml = &s_ml[(((wr * WT + w) * MT + m) * 16 + n) * 2];
        l += ml[1] * __builtin_amdgcn_exp2f((ml[0] - t) * a.scale_log2);
      }
      const float f = __builtin_amdgcn_exp2f((top[m] - t) * a.scale_log2);
      if (m > 0) __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VC; ++c) s_o[((wave * 4 + e) * VC + c) * 64 + lane] = o[m][c][e] * f;
      __syncthreads();
      // wave wt of WT sums its share of the (e, c) pairs over the WT waves
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        float x = 0.0f;
#pragma unroll
        for (int w = 0; w < WT; ++w) x += s_o[((wr * WT + w) * 4 * VC + wt * PER + i) * 64 + lane];
        y[i] = x;
      }
      d0 = g * (D / 4) + wt * PER;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < VC; ++c) y[e * VC + c] = o[m][c][e];
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

// The shares of a row joined, in the order of its tokens: a wave a row and head.
template <int D>
__global__ __launch_bounds__(256) void k_kv_join(AttendArgs a, int64_t rows) {
  const int lane = threadIdx.x & 63;
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (i >= rows) return;
  const int heads = a.kv.heads * a.group;
  const int64_t row = i / heads;
  const int hq = (int)(i - row * heads);
  const float2* ml = a.part_ml + i * a.splits;
  float t = kNoScore, l = 0.0f;
  for (int k = 0; k < a.splits; ++k) t = fmaxf(t, ml[k].x);
  constexpr int PER = D / 64;
  float y[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) y[e] = 0.0f;
  for (int k = 0; k < a.splits; ++k) {
    const float2 x = ml[k];
    if (x.y == 0.0f) continue;
    const float f = __builtin_amdgcn_exp2f((x.x - t) * a.scale_log2);
    l += x.y * f;
    const float* o = a.part_o + (i * a.splits + k) * D + lane * PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) y[e] += o[e] * f;
  }
  const float f = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* dst = a.out + row * a.o_row + hq * a.o_head + lane * PER;
#pragma unroll
  for (int e = 0; e < PER; ++e) dst[e] = (uint16_t)pack_bf16(l == 0.0f ? 0.0f : y[e] * f, 0.0f);
  if (a.lse && lane == 0)
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
  const int most = d == 256 ? 2 : 4;
  if (rows > 16 * most) {
    p.mt = most;
    p.wt = 1;
  } else {
    p.mt = rows <= 16 ? 1 : (rows <= 32 ? 2 : 4);
    p.wt = 4;
  }
  const int per = 16 * p.mt * (4 / p.wt);
  p.tiles = (int)((rows + per - 1) / per);
  // as many workgroups as the chip holds at a time, with 256 tokens at least
  int64_t splits = 1;
  if (units * p.tiles > 0) splits = 1024 / (units * p.tiles);
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

template <int D>
void launch_tiles(const Plan& p, const AttendArgs& a, int64_t blocks, hipStream_t s) {
  if constexpr (D == 256) {
    if (p.wt == 1) launch_one<D, 2, 1>(a, blocks, s);
    else if (p.mt == 1) launch_one<D, 1, 4>(a, blocks, s);
    else launch_one<D, 2, 4>(a, blocks, s);
  } else {
    if (p.wt == 1) launch_one<D, 4, 1>(a, blocks, s);
    else if (p.mt == 1) launch_one<D, 1, 4>(a, blocks, s);
    else if (p.mt == 2) launch_one<D, 2, 4>(a, blocks, s);
    else launch_one<D, 4, 4>(a, blocks, s);
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
  if (blocks > 0x7FFFFFFF || (rows + 3) / 4 > 0x7FFFFFFF) return hipErrorInvalidValue;
  if (d == 64) launch_tiles<64>(p, a, blocks, s);
  else if (d == 128) launch_tiles<128>(p, a, blocks, s);
  else if (d == 256) launch_tiles<256>(p, a, blocks, s);
  else return hipErrorInvalidValue;
  if (p.splits > 1) {
    const dim3 grid((unsigned)((rows + 3) / 4));
    if (d == 64) launch_kernel(k_kv_join<64>, grid, dim3(256), 0, s, a, rows);
    else if (d == 128) launch_kernel(k_kv_join<128>, grid, dim3(256), 0, s, a, rows);
    else launch_kernel(k_kv_join<256>, grid, dim3(256), 0, s, a, rows);
  }
  return hipGetLastError();
}

}  // namespace sph

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
//
// Few rows are bound by the codes' stream (64 users' single tokens, 1 to 8192 held:
// 285 MB in 52 us, 5.5 TB/s), windows by the conversion of codes and the softmax: of
// the clocks of 256 sessions with 64 rows a head (650 us, 845 TFLOP/s) vector
// instructions take 58% and the matrix cores work in 38%, and the two waves of a
// SIMD that the registers leave room for hardly overlap them.  A prompt's chunk of 4099
// rows behind 11902 tokens, 128 dimensions, runs 0.99 PFLOP/s.
#include <array>

#include "kv_tile.h"

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
  float scale_log2;      // of a raw score, to binades of weight
  float binade;          // one of them as a difference of scores (ln 2, but for scale_log2's rounding)
  bool q_aligned, o_aligned;
  int order;             // sessions that a round of workgroups holds (0: as they come, see session_at)
  int tiles;             // blocks of rows of a session and head
  int splits, chunk;     // shares of the tokens, tokens of one
  float2* part_ml;       // [rows x heads][splits]: reference of the weights, their sum
  float* part_o;         // [rows x heads][splits][D]
};

// Session at place p of the order in which workgroups are started: the longest
// first, so that none starts late and goes on alone.  Where all workgroups are
// resident from the start, a round of the CUs descends and the next ascends, so that
// a CU's sessions add up alike.  Ranks are counted by one thread a session, so that more
// of them start as they come (single tokens of 1 to 8192 held: 256 sessions 180 us,
// 257 208; alike or not, 300 are 9% over the floor of their bytes).
constexpr int kOrdered = 256;
__device__ __forceinline__ int session_at(const AttendArgs& a, int p) {
  __shared__ __align__(16) uint32_t s_key[kOrdered];
  __shared__ int s_found;
  const int n = a.kv.n_sessions, t = threadIdx.x;
  const int round = p / a.order, first = round * a.order;
  const int last = first + a.order < n ? first + a.order - 1 : n - 1;
  const int rank = round & 1 ? first + last - p : p;
  uint32_t key = 0;
  if (t < n) {  // (ties go to the first)
    const int len = kv_length(a.kv, a.kv.slots ? a.kv.slots[t] : t);
    key = (uint32_t)(len < (1 << 23) ? len : (1 << 23)) << 8 | (uint32_t)(kOrdered - 1 - t);
  }
  if (t < kOrdered) s_key[t] = key;
  __syncthreads();
  if (t < n) {
    int above = 0;
    const u32x4_t* keys = reinterpret_cast<const u32x4_t*>(s_key);
#pragma unroll 8
    for (int j = 0; j < (n + 3) / 4; ++j) {
      const u32x4_t k = keys[j];
      above += (k[0] > key) + (k[1] > key) + (k[2] > key) + (k[3] > key);
    }
    if (above == rank) s_found = t;
  }
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(s_found);
}

template <int D, int MT, int WT>
__global__ __launch_bounds__(64 * waves_in(WT), waves_of(D, MT, WT)) void k_kv_attend(AttendArgs a) {
  constexpr int NS = stages_of(D, WT);
  constexpr int NW = waves_in(WT);
  constexpr int WR = NW / WT;
  constexpr int KJ = D / 32;   // steps of the first product
  constexpr int VC = D / 16;   // products of the second
  constexpr bool QL = queries_in_lds(D, MT);
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wt = wave % WT, wr = wave / WT;

  const int units = a.kv.heads * a.kv.n_sessions;
  const int unit = blockIdx.x % units;
  const int rest = blockIdx.x / units;
  const int split = rest % a.splits;
  const int tile = a.tiles - 1 - rest / a.splits;  // rows that see most come first
  const int head = unit % a.kv.heads;
  const int s = a.order > 0 ? session_at(a, unit / a.kv.heads) : unit / a.kv.heads;
  const KvSession ses = kv_session(a.kv, s);
  const int G = a.group, total = a.kv.R * G, live = ses.rows * G;
  const int base = ses.len - ses.rows;
  const int row0 = (tile * WR + wr) * 16 * MT;     // the wave's first of total rows

  // rows: fq = r G + query head; those past the session's see nothing
  extern __shared__ __align__(16) uint8_t smem[];  // rings, then queries of each group of rows
  u32x4_t* s_q = reinterpret_cast<u32x4_t*>(smem + NW * NS * Stage<D>::kBytes);
  Queries<D, MT, QL> q;
  q.l = s_q;
  q.own = wr * (MT * KJ * 64) + lane;
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
      // (waves that share rows share the work of it)
      if (fq < live && (!QL || j % WT == wt)) {
        if (a.q_aligned) {
          x = *reinterpret_cast<const u32x4_t*>(p + 8 * j);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = (uint32_t)p[8 * j + 2 * i] | ((uint32_t)p[8 * j + 2 * i + 1] << 16);
        }
      }
      if constexpr (!QL) q.r[m][j] = __builtin_bit_cast(bf16x8_t, x);
      else if (j % WT == wt) s_q[((wr * MT + m) * KJ + j) * 64 + lane] = x;
    }
  }
  // tokens that the wave's rows see, and those that all of them see
  const int last_row = (row0 + 16 * MT < live ? row0 + 16 * MT : live) - 1;
  KvSpan seen{0, 0, 0, 0};
  if (row0 < live) seen = kv_span(base, row0 / G, last_row / G, a.window);
  const int all_lo = seen.all_lo, all_hi = seen.all_hi;
  const KvShare share = kv_share(seen, split, a.splits, a.chunk);
  const int from = share.from, to = share.to;

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
  // tokens is free.
  constexpr int STEP = 32 * WT;
  const int start = from + 32 * wt;
  int whole = start + (all_lo > start ? (all_lo - start + STEP - 1) / STEP * STEP : 0);
  int part = whole + ((all_hi < to ? all_hi : to) - whole + STEP - 32) / STEP * STEP;
  if (part <= whole) whole = part = start;
  const int n_whole = (part - whole) / STEP, n_head = (whole - start) / STEP;
  const int n_tiles = n_whole + n_head + (to > part ? (to - part + STEP - 1) / STEP : 0);
  auto place = [&](int k) {
    if (k >= n_tiles) return to;
    return k < n_whole ? whole + k * STEP : (k < n_whole + n_head ? start : part - n_head * STEP) + (k - n_whole) * STEP;
  };

  uint8_t* ring = smem + wave * (NS * Stage<D>::kBytes);
  uint32_t lane16 = lane * 16;
  const bool alone = WT >= 4 && a.tiles == 1;
  const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void_t*)ring;
  // the lane's places in a stage: keys token n of a block, values as they lie
  const uint32_t key_at = n * (D / 2) + g * (D / 8), value_at = KvLayout<D>::kValues + lane * (D / 8);
  const uint32_t ks_at = Stage<D>::kCodes + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g) * kKvBlock + n;
  const uint32_t vs_at = Stage<D>::kCodes + D / 2 + n * D / 512 * kKvBlock + 4 * g;
  uint32_t none = 0;  // of the tiles in flight, the next in the low bits: blocks without a page
  auto none_of = [](const KvPages& p) { return (uint32_t)(p.page[0] < 0) | ((uint32_t)(p.page[1] < 0) << 1); };
#pragma unroll
  for (int i = 0; i < NS - 1; ++i)
    if (i < n_tiles) {
      const KvPages pages = tile_pages(a.kv, ses, place(i), to);
      none |= none_of(pages) << (2 * i);
      copy_tile<D>(ring + i * Stage<D>::kBytes, a.kv, head, place(i), pages, lane16, lane, alone);
    }
  if constexpr (QL) __syncthreads();
  else  // here, not in the loop: the compiler's wait would be for all copies in flight
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int j = 0; j < KJ; ++j) asm volatile("" : "+v"(q.r[m][j]));
  KvPages ahead = tile_pages(a.kv, ses, place(NS - 1), to);
  int k = 0, stage = 0, fill = NS - 1;  // stages read and written next
  KvKeys<D> keys;
  KvValues<D> values;
  f32x4_t sc[MT][2];
  bf16x8_t p[MT];
  // asks for the tile NS - 1 ahead, waits for this one, and scores it
  auto begin = [&] {
    const KvPages after = tile_pages(a.kv, ses, place(k + NS), to);
    if (k + NS - 1 < n_tiles) {
      none |= none_of(ahead) << (2 * (NS - 1));
      copy_tile<D>(ring + fill * Stage<D>::kBytes, a.kv, head, place(k + NS - 1), ahead, lane16, lane, alone);
      wait_copies<(NS - 1) * Stage<D>::kCopies>();
    } else if (NS > 2 && k + 2 == n_tiles) {
      wait_copies<Stage<D>::kCopies>();
    } else if (NS > 3 && k + 3 == n_tiles) {
      wait_copies<2 * Stage<D>::kCopies>();
    } else {
      wait_copies<0>();
    }
    ahead = after;
    const uint32_t at = ring_at + stage * Stage<D>::kBytes;
    read_codes<D>(keys.c, keys.s[0], keys.s[1], at + key_at, at + ks_at, true);
    take_keys(sc, keys, q);
    read_codes<D>(values.c, values.s[0], values.s[1], at + value_at, at + vs_at, false);
    if (none & 3) {  // no such tokens: no weight, and values that zero times is zero
#pragma unroll
      for (int b = 0; b < 2; ++b)
        if ((none >> b) & 1) {
          values.s[b] = 0u;
#pragma unroll
          for (int m = 0; m < MT; ++m) sc[m][b] = f32x4_t{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
        }
    }
    none >>= 2;
    stage = stage + 1 == NS ? 0 : stage + 1;
    fill = fill + 1 == NS ? 0 : fill + 1;
  };
  for (; k < n_whole; ++k) {
    begin();
    take_weights(p, w, sc, a.scale_log2);
    take_values(w, values, p);
  }
  for (; k < n_tiles; ++k) {
    const int t0 = place(k);
    begin();
    mask_scores(sc, pos, a.window, t0, g);
    take_weights(p, w, sc, a.scale_log2);
    if (t0 + 32 > ses.len) {
      const int held[2] = {ses.len - t0, ses.len - t0 - kKvBlock};
      clear_values(values, held, g);
    }
    take_values(w, values, p);
  }
#pragma unroll
  for (int m = 0; m < MT; ++m) w.sum[m] = sum_over_groups(w.sum[m]);

  // lane l holds row n, dimensions (4 g + e) D/16 + c = w.o[m][c][e]
  // (what the rows are is worked out again: kept since the start it would be spilled
  // around the loop, and waited for here; 192 sessions with 20 rows of a head 175 -> 163 us)
  int heads_of = G, row_first = row0;
  asm volatile("" : "+s"(heads_of), "+s"(row_first));
  // (in what were rings)
  float* s_o = reinterpret_cast<float*>(smem);       // NW x 16 D
  float* s_ml = reinterpret_cast<float*>(smem) + NW * 16 * D;
  __syncthreads();
  if (g == 0)
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      s_ml[((wave * MT + m) * 16 + n) * 2] = w.top[m];
      s_ml[((wave * MT + m) * 16 + n) * 2 + 1] = w.sum[m];
    }
  __syncthreads();
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    constexpr int PER = D / 4 / WT;  // values a lane ends with
    float t = kNoScore, l = 0.0f;
#pragma unroll
    for (int k = 0; k < WT; ++k) t = fmaxf(t, s_ml[(((wr * WT + k) * MT + m) * 16 + n) * 2]);
#pragma unroll
    for (int k = 0; k < WT; ++k) {
      const float* ml = &s_ml[(((wr * WT + k) * MT + m) * 16 + n) * 2];
      l += ml[1] * __builtin_amdgcn_exp2f(ml[0] - t);
    }
    const float f = __builtin_amdgcn_exp2f(w.top[m] - t);
    if (m > 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int c = 0; c < VC; ++c) s_o[((wave * 4 + e) * VC + c) * 64 + lane] = w.o[m][c][e] * f;
    __syncthreads();
    // wave wt of WT sums its share of the (e, c) pairs over the WT waves
    float y[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      float x = 0.0f;
#pragma unroll
      for (int k = 0; k < WT; ++k) x += s_o[((wr * WT + k) * 4 * VC + wt * PER + i) * 64 + lane];
      y[i] = x;
    }
    const int d0 = g * (D / 4) + wt * PER;  // the first of them
    const int fq = row_first + m * 16 + n;
    if (fq >= live) l = 0.0f;  // rows that are none
    if (fq < total) {
      const int r = fq / heads_of, hq = head * heads_of + fq - r * heads_of;
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
        if (a.lse && g == 0 && wt == 0)
          a.lse[row * (a.kv.heads * G) + hq] = l == 0.0f ? -INFINITY : fmaf(t, a.binade, __builtin_amdgcn_logf(l) * kLn2);
      } else {
        const int64_t at = (row * (a.kv.heads * G) + hq) * a.splits + split;
        if (g == 0 && wt == 0) a.part_ml[at] = make_float2(t, l);
        if (!(l == 0.0f)) {
#pragma unroll
          for (int i = 0; i < PER; i += 4)
            *reinterpret_cast<f32x4_t*>(a.part_o + at * D + d0 + i) = f32x4_t{y[i], y[i + 1], y[i + 2], y[i + 3]};
        }
      }
    }
  }
}

// The shares of a row joined.  D/4 lanes take a share, TURNS groups of them the
// shares of one row and head in turns, each eight at a time so that all their
// loads are on their way together; sums in an order that is always the same.
template <int D, int TURNS>
__global__ __launch_bounds__(256) void k_kv_join(AttendArgs a, int64_t rows) {
  constexpr int LPS = D / 4, PER = 256 / LPS / TURNS;  // rows of a workgroup
  __shared__ float s_l[256 / LPS];
  __shared__ f32x4_t s_o[TURNS > 1 ? 256 : 1];
  const int d4 = threadIdx.x % LPS, turn = threadIdx.x / LPS % TURNS;
  const int64_t want = (int64_t)blockIdx.x * PER + threadIdx.x / (LPS * TURNS);
  const int64_t i = want < rows ? want : rows - 1;
  const float2* ml = a.part_ml + i * a.splits;
  const float* part = a.part_o + i * a.splits * D + d4 * 4;
  float top = kNoScore, l = 0.0f;
  f32x4_t y{0.0f, 0.0f, 0.0f, 0.0f};
  for (int k0 = turn; k0 < a.splits; k0 += 8 * TURNS) {
    float2 x[8];
    f32x4_t o[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = k0 + u * TURNS;
      const bool in = k < a.splits;
      x[u] = in ? ml[k] : make_float2(kNoScore, 0.0f);
      // shares without a token left their place unwritten: read, not used
      if (in) o[u] = *reinterpret_cast<const f32x4_t*>(part + (int64_t)k * D);
    }
    float t = top;
#pragma unroll
    for (int u = 0; u < 8; ++u) t = fmaxf(t, x[u].x);
    const float f = __builtin_amdgcn_exp2f(top - t);
    l *= f;
    y *= f;
    top = t;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (x[u].y == 0.0f) continue;
      const float e = __builtin_amdgcn_exp2f(x[u].x - top);
      l += x[u].y * e;
      y += o[u] * e;
    }
  }
  if constexpr (TURNS > 1) {
    __shared__ float s_top[256 / LPS];
    s_o[threadIdx.x] = y;
    if (d4 == 0) {
      s_l[turn] = l;
      s_top[turn] = top;
    }
    __syncthreads();
    if (turn != 0) return;
    float t = top;
#pragma unroll
    for (int k = 1; k < TURNS; ++k) t = fmaxf(t, s_top[k]);
    y = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    l = 0.0f;
#pragma unroll
    for (int k = 0; k < TURNS; ++k) {
      const float e = __builtin_amdgcn_exp2f(s_top[k] - t);
      y += s_o[k * LPS + d4] * e;
      l += s_l[k] * e;
    }
    top = t;
  }
  if (want >= rows) return;
  const int heads = a.kv.heads * a.group;
  const int64_t row = i / heads;
  const int hq = (int)(i - row * heads);
  const float f = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* dst = a.out + row * a.o_row + hq * a.o_head + d4 * 4;
  const uint32_t lo = l == 0.0f ? 0u : pack_bf16(y[0] * f, y[1] * f), hi = l == 0.0f ? 0u : pack_bf16(y[2] * f, y[3] * f);
  if (a.o_aligned) {
    *reinterpret_cast<uint32_t*>(dst) = lo;
    *reinterpret_cast<uint32_t*>(dst + 2) = hi;
  } else {
    dst[0] = (uint16_t)lo, dst[1] = (uint16_t)(lo >> 16);
    dst[2] = (uint16_t)hi, dst[3] = (uint16_t)(hi >> 16);
  }
  if (a.lse && d4 == 0)
    a.lse[i] = l == 0.0f ? -INFINITY : fmaf(top, a.binade, __builtin_amdgcn_logf(l) * kLn2);
}

template <int D>
void launch_join(const AttendArgs& a, int64_t rows, hipStream_t s) {
  constexpr int ALL = 256 / (D / 4);
  if (a.splits <= 8)
    launch_kernel(k_kv_join<D, 1>, dim3((unsigned)((rows + ALL - 1) / ALL)), dim3(256), 0, s, a, rows);
  else
    launch_kernel(k_kv_join<D, ALL>, dim3((unsigned)rows), dim3(256), 0, s, a, rows);
}

namespace {

// Whether workgroups start by their sessions' lengths (shares of a window are alike):
// where there are more of them than CUs, and where the longest takes long enough,
// turns of its waves, for the 2 us of ranking that each spends (208 sessions of 762
// tokens each 22 -> 27 us).  64 users of 1 to 8192 tokens 79 -> 68 us, 128 with heads
// of 256 up to 4096 87 -> 69, 256 with 64 heads up to 16384 714 -> 650.
bool by_length(int64_t n_sessions, int64_t blocks, int64_t turns) {
  return n_sessions > 1 && n_sessions <= kOrdered && blocks > kCUs && turns >= 16;
}

// How the rows of one head and the tokens of a session are shared out.
struct Plan {
  int mt, wt;          // tiles of 16 rows of a wave, waves that share the tokens of the same rows
  int tiles;           // workgroups for all rows of a head
  int splits, chunk;   // shares of the tokens, tokens of one
};

// heads: of keys and values; group: query heads of one of those; R rows of a session,
// which has max_len tokens at most.
Plan account(int d, int64_t n_sessions, int64_t heads, int64_t R, int64_t group, int64_t max_len, int64_t window) {
  const int64_t rows = R * group, units = n_sessions * heads;
  // Row tiles of a wave and waves that share its rows: many rows share the conversion
  // of the codes (a long prompt of 128 dimensions, us: 1450 with {2, 1}, 1215 with
  // {4, 4}), few make more workgroups (sliding window, 64 dimensions: 82 and 67).
  // Eight waves a session end a long one sooner where few rows need few registers (64
  // users' single tokens 57 -> 51), and share 256 dimensions' conversion among 32 rows,
  // which leave room for no second workgroup anyway (prompts 153 -> 126).
  static constexpr int kNarrow[][2] = {{1, 4}, {2, 4}, {4, 4}, {2, 2}};
  static constexpr int kMiddle[][2] = {{1, 4}, {2, 4}, {4, 4}, {2, 2}, {1, 8}};
  static constexpr int kWide[][2] = {{1, 4}, {1, 2}, {2, 8}};
  const int(*shapes)[2] = d == 64 ? kNarrow : d == 128 ? kMiddle : kWide;
  Plan best{};
  double least = 0;
  for (int i = 0; i < (d == 128 ? 5 : d == 64 ? 4 : 3); ++i) {
    const int mt = shapes[i][0], wt = shapes[i][1], waves = waves_in(wt);
    const int per = 16 * mt * (waves / wt);
    const int64_t tiles = (rows + per - 1) / per, blocks = units * tiles, step = 32 * wt;
    const int64_t slots = (int64_t)kCUs * resident(d, mt, wt);
    // tokens that a workgroup's rows see
    const int64_t wide = window + (per < rows ? per : rows) / group + 32;
    const int64_t span = window > 0 && wide < max_len ? wide : max_len;
    // A rough account in microseconds.  A workgroup starts and ends in about 5 and
    // joins its waves' outputs; a tile of a wave is the issue of its instructions (a
    // third more for what does not overlap) times the waves that share a SIMD, or a
    // wave's own latencies; joining shares costs a launch and the partial outputs'
    // way out and back.
    const double issue = (4.0 * (0.9 * d + 20 + 36 * mt) + (32.0 + d / 2.0) * mt) * 1.35 / 2100;
    auto workgroup = [&](int64_t n, int64_t tokens) {  // n of them at a time
      const double beside = (double)((n + kCUs - 1) / kCUs * (waves / 4));
      const double tile = beside * issue > issue + 0.7 ? beside * issue : issue + 0.7;
      return 5.0 + 1.5 * mt + (double)((tokens + step - 1) / step) * tile;
    };
    static constexpr int kShares[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 80, 96, 128};
    for (const int64_t n : kShares) {
      if (n > 1 && n * step > span + step - 1) break;
      const int64_t chunk = ((span + n - 1) / n + step - 1) / step * step;
      const int64_t all = blocks * n, last = all % slots;
      double t = (double)(all / slots) * workgroup(slots, chunk) + (last > 0 ? workgroup(last, chunk) : 0.0);
      // (tiles of rows see less and less: the last ones fill the gaps)
      if (tiles > 1 && all > slots) t = ((double)all / (double)slots + 0.1) * workgroup(slots, chunk);
      const bool ordered = n == 1 && window == 0 && by_length(n_sessions, all, chunk / step);
      if (ordered) {
        // Sessions may be all alike or very different, which is half of the work and the
        // longest alone.
        const double load = all > slots ? (double)all / (double)slots * workgroup(slots, chunk / 2) : workgroup(all, chunk / 2);
        const double alone = workgroup(1, chunk);
        t = 0.5 * (t + (load > alone ? load : alone));
      }
      if (n > 1) t += 6.0 + (double)(units * rows * n) * (d * 8 + 16) / 4e6;
      if (best.mt == 0 || t < 0.97 * least) {
        least = t;
        best = Plan{mt, wt, (int)tiles, (int)((span + chunk - 1) / chunk), (int)chunk};
      }
    }
  }
  if (best.splits < 1) best.splits = 1;
  return best;
}

// The account takes 1 us of the host: a layer's workspace query, its call and the next
// layers' ask for the same sizes.
Plan plan_of(int d, int64_t n_sessions, int64_t heads, int64_t R, int64_t group, int64_t max_len, int64_t window) {
  thread_local std::array<int64_t, 7> sizes{};
  thread_local Plan plan{};
  const std::array<int64_t, 7> want{d, n_sessions, heads, R, group, max_len, window};
  if (sizes != want) {
    plan = account(d, n_sessions, heads, R, group, max_len, window);
    sizes = want;
  }
  return plan;
}

template <int D, int MT, int WT>
hipError_t launch_one(const AttendArgs& a, int64_t blocks, hipStream_t s) {
  constexpr size_t lds = attend_lds(D, MT, WT);
  static std::atomic<uint64_t> done{0};
  const hipError_t e = set_lds_limit_once(done, reinterpret_cast<const void*>(k_kv_attend<D, MT, WT>), lds);
  if (e != hipSuccess) return e;
  launch_kernel(k_kv_attend<D, MT, WT>, dim3((unsigned)blocks), dim3(64 * waves_in(WT)), (uint32_t)lds, s, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_tiles(const Plan& p, const AttendArgs& a, int64_t blocks, hipStream_t s) {
  if (p.mt == 1 && p.wt == 4) return launch_one<D, 1, 4>(a, blocks, s);
  if constexpr (D == 256)
    return p.wt == 8 ? launch_one<D, 2, 8>(a, blocks, s) : launch_one<D, 1, 2>(a, blocks, s);
  if constexpr (D == 128)
    if (p.wt == 8) return launch_one<D, 1, 8>(a, blocks, s);
  if constexpr (D < 256) {
    if (p.wt == 2) return launch_one<D, 2, 2>(a, blocks, s);
    if (p.mt == 2) return launch_one<D, 2, 4>(a, blocks, s);
    return launch_one<D, 4, 4>(a, blocks, s);
  }
}

}  // namespace

int64_t kv_window(int64_t window, int64_t most) { return window < most ? window : 0; }

void kv_attend_span(int base, int r_lo, int r_hi, int window, int split, int splits, int chunk, int span[6]) {
  const KvSpan t = kv_span(base, r_lo, r_hi, window);
  const KvShare share = kv_share(t, split, splits, chunk);
  const int out[6] = {t.lo, t.hi, t.all_lo, t.all_hi, share.from, share.to};
  for (int i = 0; i < 6; ++i) span[i] = out[i];
}

// Workspace: the shares' maxima and sums, then their outputs.
size_t kv_attend_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads,
                         int64_t max_len, int64_t window) {
  const Plan p = plan_of(d, n_sessions, heads, R, q_heads / heads, max_len, window);
  if (p.splits <= 1) return 0;
  const size_t n = (size_t)n_sessions * R * q_heads * p.splits;
  return (n * 8 + 255) / 256 * 256 + n * d * 4;
}

void kv_attend_shape(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len,
                     int64_t window, int shape[5]) {
  const Plan p = plan_of(d, n_sessions, heads, R, q_heads / heads, max_len, window);
  const int out[5] = {p.mt, p.wt, p.tiles, p.splits, p.chunk};
  for (int i = 0; i < 5; ++i) shape[i] = out[i];
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
  a.scale_log2 = c.scale * 1.44269504088896f;
  a.binade = (float)((double)c.scale / a.scale_log2);
  a.q_aligned = c.q_row % 8 == 0 && c.q_head % 8 == 0 && (reinterpret_cast<uintptr_t>(c.q) & 15) == 0;
  a.o_aligned = c.o_row % 2 == 0 && c.o_head % 2 == 0 && (reinterpret_cast<uintptr_t>(c.out) & 3) == 0;
  const int64_t units = (int64_t)kv.n_sessions * kv.heads;
  const Plan p = plan_of(d, kv.n_sessions, kv.heads, kv.R, a.group, c.max_len, c.window);
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.chunk = p.chunk;
  const int64_t rows = (int64_t)kv.n_sessions * kv.R * c.q_heads;
  if (p.splits > 1) {
    a.part_ml = static_cast<float2*>(workspace);
    a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + ((size_t)rows * p.splits * 8 + 255) / 256 * 256);
  }
  const int64_t blocks = units * p.tiles * p.splits;
  if (p.splits == 1 && c.window == 0 && by_length(kv.n_sessions, blocks, p.chunk / (32 * p.wt))) {
    const int per = kCUs / kv.heads;
    const bool at_once = p.tiles == 1 && blocks <= (int64_t)kCUs * resident(d, p.mt, p.wt);
    a.order = at_once && per > 0 ? per : kv.n_sessions;
  }
  const hipError_t e = d == 64    ? launch_tiles<64>(p, a, blocks, s)
                       : d == 128 ? launch_tiles<128>(p, a, blocks, s)
                       : d == 256 ? launch_tiles<256>(p, a, blocks, s)
                                  : hipErrorInvalidValue;
  if (e != hipSuccess) return e;
  if (p.splits > 1) {
    if (d == 64) launch_join<64>(a, rows, s);
    else if (d == 128) launch_join<128>(a, rows, s);
    else launch_join<256>(a, rows, s);
  }
  return hipGetLastError();
}

}  // namespace sph

// What each held token receives of the attention of a call's rows:
//
//   w[j] += sum_{r, h} exp(scale q[r, h] . K[j, h / G] - lse[r, h])
//   over the rows r that see j (kv_attend.hip), lse the log-sum-exp of their scores.
//
// A wave owns TT tiles of 32 tokens and goes over the key/value heads; every tile of 16
// of the R G rows is multiplied with the tokens' keys,
//   S^T = K Q^T   (tokens x rows) 16x16x32 products,
// lane l = 16 g + n holding row n against tokens 4 g ... 4 g + 3 of each block.  Weights
// of one token stay apart by lanes and are added up over the rows and heads in
// registers; the 16 lanes meet once, at the end.  Every token is one wave's (or one
// wave's of each part of the heads and rows, joined in their order), so that sums do
// not depend on timing and nothing is added atomically.
//
// Up to 64 rows of a head (k_weigh_few) the keys of all heads stream through rings of
// LDS stages: 256 sessions' windows of four rows over 8192 tokens read their keys at
// 5.2 TB/s (226 us), 64 at 4.7.  Sessions of 5 to 8192 tokens leave CUs idle (busy 62%): a
// workgroup's tokens are as many for all.  A window masks what rows do not see, its keys
// are read all the same: four rows of 32 sessions of 65536 tokens take 223 us with a window
// of 1024, 239 without.
// More rows (k_weigh_many) pass a head's keys held as operands in registers, those that see
// none of them left out (330 us in place of 700 for prompts when the keys' conversion and the
// spilled registers around it were in the loop): 0.92 PFLOP/s where sessions are alike.  There vector instructions
// take 57% of the clocks and the matrix cores 34%, and the two do not overlap on a SIMD,
// though one product stands beside four vector instructions in the loop: what is left is
// an exponential, a multiply-add and an addition for each score.
#include "kv_tile.h"

namespace sph {

struct WeighArgs {
  KvArgs kv;
  const uint16_t* q;  // bf16 [M][q_heads][D]
  int64_t q_row, q_head;
  const float* lse;   // [M][q_heads]
  float* w;           // [n_slots][ld_w]
  int64_t ld_w;
  int group;          // query heads of a key/value head
  int window;         // 0: none
  int fresh;          // the rows' own tokens start at zero
  float scale_log2;
  bool q_aligned;
  int groups;         // workgroups along the tokens of a session
  int parts;          // shares of the heads and rows, `by_rows` of them for one head
  int by_rows, heads_each;
  float* part;        // [n_sessions][parts][groups x tokens of a workgroup]
};

constexpr float kLog2e = 1.44269504088896f;
constexpr int weigh_tiles(int d) { return d == 256 ? 2 : 4; }          // of 32 tokens, of a wave
constexpr int weigh_tokens(int d) { return 4 * 32 * weigh_tiles(d); }  // of a workgroup

// What a workgroup does of a call: tokens `at` x TOKENS ... of a session for some heads
// and tiles of rows.
struct WeighShare {
  int h0, h1, phase, step;
  bool whole;  // all of them
};
__device__ __forceinline__ WeighShare weigh_share(const WeighArgs& a, int part, int at) {
  // tokens past those that max_len promised have no place among the parts
  const bool whole = a.parts == 1 || at >= a.groups;
  WeighShare w;
  w.whole = whole;
  w.h0 = whole ? 0 : part / a.by_rows * a.heads_each;
  w.h1 = whole ? a.kv.heads : (w.h0 + a.heads_each < a.kv.heads ? w.h0 + a.heads_each : a.kv.heads);
  w.step = whole ? 1 : a.by_rows;
  w.phase = whole ? 0 : part % a.by_rows;
  if (whole && part > 0) w.h1 = 0;
  return w;
}

// Tiles of 16 rows that see any of tokens t0 ... t1 - 1.
__device__ __forceinline__ void rows_that_see(const KvSession& ses, int G, int window, int t0, int t1, int* rt0, int* rt1) {
  const int base = ses.len - ses.rows;
  const int first = t0 > base ? t0 - base : 0;
  const int64_t out = (int64_t)t1 - 1 + window - base;  // the first past all tokens' windows
  const int past = window > 0 && out < ses.rows ? (int)out : ses.rows;
  *rt0 = (int)((int64_t)first * G / 16);
  *rt1 = past > first && t0 < ses.len ? (int)(((int64_t)past * G + 15) / 16) : 0;
}

// Over the 16 rows of a lane group; lane n then has values n, n + 16 ... of 8 TT: value
// v is token v / 4 * 16 + 4 g + v % 4 of the wave's.
template <int TT>
__device__ __forceinline__ void give_weights(const WeighArgs& a, const KvSession& ses, int s, int slot, int part, bool whole,
                                             int t0, int tokens, f32x4_t (&acc)[TT][2], int g, int n) {
  float out[TT / 2];
#pragma unroll
  for (int i = 0; i < TT * 8; ++i) {
    float x = acc[i / 8][i / 4 % 2][i % 4];
    x += __uint_as_float(dpp_u32<0x128>(__float_as_uint(x)));  // row_ror 8, 4, 2, 1
    x += __uint_as_float(dpp_u32<0x124>(__float_as_uint(x)));
    x += __uint_as_float(dpp_u32<0x122>(__float_as_uint(x)));
    x += __uint_as_float(dpp_u32<0x121>(__float_as_uint(x)));
    if (n == i % 16) out[i / 16] = x;
  }
#pragma unroll
  for (int i = 0; i < TT / 2; ++i) {
    const int v = i * 16 + n;
    const int j = t0 + v / 4 * 16 + 4 * g + v % 4;
    if (j >= ses.len) continue;
    if (whole) {
      float* w = a.w + slot * a.ld_w + j;
      *w = (a.fresh && j >= ses.len - ses.rows ? 0.0f : *w) + out[i];
    } else {
      a.part[((int64_t)s * a.parts + part) * ((int64_t)a.groups * tokens) + j] = out[i];
    }
  }
}

// Adds the weights of two blocks' scores against a tile of rows.
__device__ __forceinline__ void add_weights(f32x4_t (&acc)[2], const f32x4_t (&sc)[2], float scale_log2, float l) {
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[b][e] += __builtin_amdgcn_exp2f(fmaf(sc[b][e], scale_log2, -l));
}
// The same where the row sees `span` tokens from `from` tokens before the lane's first.
__device__ __forceinline__ void add_seen(f32x4_t (&acc)[2], const f32x4_t (&sc)[2], float scale_log2, float l, int from,
                                         int span, const int (&page)[2]) {
#pragma unroll
  for (int b = 0; b < 2; ++b)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float p = __builtin_amdgcn_exp2f(fmaf(sc[b][e], scale_log2, -l));
      const bool sees = (uint32_t)(from + 16 * b + e) < (uint32_t)span && page[b] >= 0;
      acc[b][e] += sees ? p : 0.0f;
    }
}

// Few rows: the keys of all heads stream through the wave's ring of LDS stages, heads in
// the outer and tiles of tokens in the inner loop, as in kv_attend.hip without values.
template <int D>
struct KeyStage {
  static constexpr int kCodes = 16 * D;                       // bytes: both blocks' codes, then their scales,
  static constexpr int kBytes = kCodes + 256;                 // which a copy of all lanes brings
  static constexpr int kCopies = (D == 64 ? 1 : D / 64) + 1;  // 64 x 16 bytes of codes, 64 x 4 of scales
};
template <int D>
__device__ __forceinline__ void copy_keys(uint8_t* to, const KvArgs& a, int head, int pos, const KvPages& pages, uint32_t lane) {
  const uint8_t* blk[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const int page = pages.page[b];
    blk[b] = scalar_ptr(kv_block<D>(a, page < 0 ? 0 : page, head, page < 0 ? 0 : pos + b * kKvBlock));
  }
  const uint64_t b0 = reinterpret_cast<uint64_t>(blk[0]), b1 = reinterpret_cast<uint64_t>(blk[1]);
  if constexpr (D == 64) {  // 512 bytes of either block
    const uint64_t base = lane < 32 ? b0 : b1;
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint8_t*>(base) + lane % 32 * 16, (lds_void_t*)to, 16, 0, 2);
  } else {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      lds_void_t* at = (lds_void_t*)(to + b * 8 * D);
      __builtin_amdgcn_global_load_lds(blk[b] + lane * 16, at, 16, 0, 2);
      if constexpr (D == 256) __builtin_amdgcn_global_load_lds(blk[b] + lane * 16, at, 16, 1024, 2);
    }
  }
  // D/2 bytes of scales of either (lanes past them repeat the others)
  const uint32_t in = lane * 4 % D;
  const uint64_t base = in < D / 2 ? b0 : b1;
  __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint8_t*>(base) + (16 * D + in % (D / 2)), (lds_void_t*)(to + 16 * D), 4, 0, 2);
}

// A lane's keys of a stage; ends with its own wait.
template <int D>
__device__ __forceinline__ void read_keys(KvKeys<D>& k, uint32_t at_c, uint32_t at_s) {
  if constexpr (D == 64) {
    u32x2_t x, y;
    asm volatile("ds_read_b64 %0, %4\n ds_read_b64 %1, %4 offset:512\n ds_read_u8 %2, %5\n"
                 "ds_read_u8 %3, %5 offset:32\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(x), "=&v"(y), "=&v"(k.s[0]), "=&v"(k.s[1]) : "v"(at_c), "v"(at_s) : "memory");
    k.c[0][0] = x[0], k.c[0][1] = x[1], k.c[1][0] = y[0], k.c[1][1] = y[1];
  } else if constexpr (D == 128) {
    u32x4_t x, y;
    asm volatile("ds_read_b128 %0, %4\n ds_read_b128 %1, %4 offset:1024\n ds_read_u8 %2, %5\n"
                 "ds_read_u8 %3, %5 offset:64\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(x), "=&v"(y), "=&v"(k.s[0]), "=&v"(k.s[1]) : "v"(at_c), "v"(at_s) : "memory");
#pragma unroll
    for (int e = 0; e < 4; ++e) k.c[0][e] = x[e], k.c[1][e] = y[e];
  } else {
    u32x4_t x, y, z, w;
    uint32_t t0, t1;  // the second group's bytes
    asm volatile("ds_read_b128 %0, %8\n ds_read_b128 %1, %8 offset:16\n ds_read_b128 %2, %8 offset:2048\n"
                 "ds_read_b128 %3, %8 offset:2064\n ds_read_u8 %4, %9\n ds_read_u8 %5, %9 offset:128\n"
                 "ds_read_u8 %6, %9 offset:16\n ds_read_u8 %7, %9 offset:144\n s_waitcnt lgkmcnt(0)"
                 : "=&v"(x), "=&v"(y), "=&v"(z), "=&v"(w), "=&v"(k.s[0]), "=&v"(k.s[1]), "=&v"(t0), "=&v"(t1)
                 : "v"(at_c), "v"(at_s) : "memory");
    k.s[0] |= t0 << 8;
    k.s[1] |= t1 << 8;
#pragma unroll
    for (int e = 0; e < 4; ++e) k.c[0][e] = x[e], k.c[0][4 + e] = y[e], k.c[1][e] = z[e], k.c[1][4 + e] = w[e];
  }
}

// What of the queries of a head a workgroup holds in LDS: operands [MT][D / 32][64 lanes]
// of 16 bytes, then the rows' log-sum-exp [MT][16].
template <int D, int MT>
struct QueryStage {
  static constexpr int kChunks = MT * (D / 32);
  static constexpr int kBytes = kChunks * 1024 + 256;
  static constexpr int kCopies = (kChunks + 3) / 4 + 1;  // of each of four waves
};
constexpr int weigh_waves(int d, int mt) { return d * mt <= 128 ? 4 : d * mt <= 256 ? 3 : 2; }

template <int D, int MT>
__global__ __launch_bounds__(256, weigh_waves(D, MT)) void k_weigh_few(WeighArgs a) {
  constexpr int TT = weigh_tiles(D), KJ = D / 32, TOKENS = weigh_tokens(D), NS = TT;  // (a head's tiles are the ring's stages)
  using Q = QueryStage<D, MT>;
  __shared__ __align__(16) uint8_t smem[4 * NS * KeyStage<D>::kBytes + 2 * Q::kBytes];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int part_of = blockIdx.x % a.parts;
  const int rest = blockIdx.x / a.parts;
  const int s = (rest + rest / a.kv.n_sessions) % a.kv.n_sessions;  // (a session's groups of tokens on all XCDs)
  const KvSession ses = kv_session(a.kv, s);
  const int G = a.group, live = ses.rows * G, base = ses.len - ses.rows;
  const int slot = a.kv.slots ? a.kv.slots[s] : s;
  if (live <= 0) return;
  uint8_t* ring = smem + wave * (NS * KeyStage<D>::kBytes);
  uint8_t* queries = smem + 4 * NS * KeyStage<D>::kBytes;
  const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void_t*)ring;
  const uint32_t key_at = n * (D / 2) + g * (D / 8);
  const uint32_t ks_at = KeyStage<D>::kCodes + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g) * kKvBlock + n;

  // rows: fq = r G + query head of the key/value head's; those past the session's are
  // its last, of no weight
  int row_at[MT], head_at[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int fq = m * 16 + n < live ? m * 16 + n : live - 1;
    row_at[m] = fq / G;
    head_at[m] = fq - row_at[m] * G;
  }
  // A wave's share of a head's queries, on their way into LDS: a lane's 16 bytes are the
  // ones that it reads.
  auto fetch_queries = [&](int head, int buffer) {
    uint8_t* to = queries + buffer * Q::kBytes;
#pragma unroll
    for (int i = 0; i < (Q::kChunks + 3) / 4; ++i) {
      const int chunk = Q::kChunks < 4 ? wave % Q::kChunks : i * 4 + wave, m = chunk / KJ, j = chunk % KJ;
      int r = row_at[0], in = head_at[0];
#pragma unroll
      for (int k = 1; k < MT; ++k)
        if (m == k) r = row_at[k], in = head_at[k];
      const uint16_t* p = a.q + ((int64_t)s * a.kv.R + r) * a.q_row + (int64_t)(head * G + in) * a.q_head + g * (D / 4) + 8 * j;
      if (a.q_aligned) {
        __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint8_t*>(p), (lds_void_t*)(to + chunk * 1024), 16, 0, 0);
      } else {
        u32x4_t x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = (uint32_t)p[2 * e] | ((uint32_t)p[2 * e + 1] << 16);
        *reinterpret_cast<u32x4_t*>(to + chunk * 1024 + lane * 16) = x;
      }
    }
    int r = row_at[0], in = head_at[0];  // lane g 16 + n: row n of tile g
#pragma unroll
    for (int k = 1; k < MT; ++k)
      if (g == k) r = row_at[k], in = head_at[k];
    const float* p = a.lse + ((int64_t)s * a.kv.R + r) * (a.kv.heads * G) + head * G + in;
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint8_t*>(p), (lds_void_t*)(to + Q::kChunks * 1024), 4, 0, 0);
  };

  for (int at = rest / a.kv.n_sessions; at * TOKENS < ses.len; at += a.groups) {
    const WeighShare share = weigh_share(a, part_of, at);
    const int t0 = at * TOKENS + wave * (32 * TT), t1 = t0 + 32 * TT;
    if (share.h0 >= share.h1) continue;
    KvPages pages[TT];
    bool whole = true;  // every row sees every token
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      pages[t] = tile_pages(a.kv, ses, t0 + 32 * t, ses.len);
      whole = whole && pages[t].page[0] >= 0 && pages[t].page[1] >= 0;
    }
    whole = whole && base >= t1 - 1 && (a.window == 0 || t0 > ses.len - 1 - a.window);
    int from[MT], span[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const int pos = base + row_at[m], most = pos < 0 || m * 16 + n >= live ? 0 : pos + 1;
      span[m] = a.window > 0 && a.window < most ? a.window : most;
      from[m] = t0 + 4 * g - (pos - span[m] + 1);
    }
    f32x4_t acc[TT][2];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t][0] = acc[t][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    __syncthreads();  // the queries of the tokens before are read
    fetch_queries(share.h0, 0);
#pragma unroll
    for (int t = 0; t < NS - 1; ++t) copy_keys<D>(ring + t * KeyStage<D>::kBytes, a.kv, share.h0, t0 + 32 * t, pages[t], lane);
    for (int head = share.h0; head < share.h1; ++head) {
      constexpr int C = KeyStage<D>::kCopies;
      const bool more = head + 1 < share.h1;
      const int buffer = (head - share.h0) & 1;
      wait_copies<(NS - 1) * C>();  // the queries are older than those of the tiles
      __syncthreads();
      if (more) fetch_queries(head + 1, buffer ^ 1);
      const uint8_t* held = queries + buffer * Q::kBytes;
      u32x4_t qf[MT][KJ];
      float l[MT];
      bool dead = false;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        // (what a row sees is compared for every head: kept, the answers would be spilled)
        asm volatile("" : "+v"(from[m]), "+v"(span[m]));
#pragma unroll
        for (int j = 0; j < KJ; ++j) qf[m][j] = *reinterpret_cast<const u32x4_t*>(held + (m * KJ + j) * 1024 + lane * 16);
        const float x = *reinterpret_cast<const float*>(held + Q::kChunks * 1024 + (m * 16 + n) * 4);
        const bool is = m * 16 + n < live;
        dead = dead || (is && x == -INFINITY);  // a row that sees nothing
        l[m] = is && x != -INFINITY ? x * kLog2e : INFINITY;  // no weight of finite scores
      }
      const bool alive = whole && !__any(dead);
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int next = t + NS - 1;
        if (next < TT) copy_keys<D>(ring + next * KeyStage<D>::kBytes, a.kv, head, t0 + 32 * next, pages[next], lane);
        else if (more)
          copy_keys<D>(ring + (next - TT) * KeyStage<D>::kBytes, a.kv, head + 1, t0 + 32 * (next - TT), pages[next - TT], lane);
        if (more) {
          if (a.q_aligned && t < TT - 1) wait_copies<(NS - 1) * C + Q::kCopies>();
          else wait_copies<(NS - 1) * C>();
        } else if (t == 0) {
          wait_copies<(NS - 1) * C>();
        } else if (t + 2 < TT) {
          wait_copies<2 * C>();
        } else if (t + 1 < TT) {
          wait_copies<C>();
        } else {
          wait_copies<0>();
        }
        KvKeys<D> keys;
        const uint32_t stage = ring_at + t * KeyStage<D>::kBytes;
        read_keys<D>(keys, stage + key_at, stage + ks_at);
        // (a key that is no number would weigh on rows that are none)
        bool numbers = keys.s[0] != 255u && keys.s[1] != 255u;
        if constexpr (D == 256)
          numbers = (keys.s[0] & 255u) != 255u && keys.s[0] >> 8 != 255u && (keys.s[1] & 255u) != 255u && keys.s[1] >> 8 != 255u;
        const bool all = alive && __all(numbers);
        f32x4_t sc[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m) sc[m][0] = sc[m][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < KJ; ++j) {
          bf16x8_t kf[2];
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const float x = e8m0_operand(D == 256 ? (keys.s[b] >> (8 * (j / 4))) & 0xFFu : keys.s[b]);
            const uint32_t c = keys.c[b][j];
            const u32x4_t y{fp4_pair<0>(c, x), fp4_pair<1>(c, x), fp4_pair<2>(c, x), fp4_pair<3>(c, x)};
            kf[b] = __builtin_bit_cast(bf16x8_t, y);
          }
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            const bf16x8_t q = __builtin_bit_cast(bf16x8_t, qf[m][j]);
            sc[m][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[0], q, sc[m][0], 0, 0, 0);
            sc[m][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[1], q, sc[m][1], 0, 0, 0);
          }
        }
        if (all) {
#pragma unroll
          for (int m = 0; m < MT; ++m) add_weights(acc[t], sc[m], a.scale_log2, l[m]);
        } else {
#pragma unroll
          for (int m = 0; m < MT; ++m)
            add_seen(acc[t], sc[m], a.scale_log2, l[m], from[m] + 32 * t, l[m] == INFINITY ? 0 : span[m], pages[t].page);
        }
      }
    }
    give_weights<TT>(a, ses, s, slot, part_of, share.whole, t0, TOKENS, acc, g, n);
  }
}

// Many rows: a head's keys stay in registers as operands while its tiles of rows pass.
template <int D>
__global__ __launch_bounds__(256, 2) void k_weigh_many(WeighArgs a) {
  constexpr int TT = weigh_tiles(D), KJ = D / 32, TOKENS = weigh_tokens(D);
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int part_of = blockIdx.x % a.parts;
  const int rest = blockIdx.x / a.parts;
  const int s = (rest + rest / a.kv.n_sessions) % a.kv.n_sessions;  // (a session's groups of tokens on all XCDs)
  const KvSession ses = kv_session(a.kv, s);
  const int G = a.group, live = ses.rows * G, base = ses.len - ses.rows;
  const int slot = a.kv.slots ? a.kv.slots[s] : s;

  for (int at = rest / a.kv.n_sessions; at * TOKENS < ses.len; at += a.groups) {
    const WeighShare share = weigh_share(a, part_of, at);
    if (share.h0 >= share.h1) continue;
    const int t0 = at * TOKENS + wave * (32 * TT), t1 = t0 + 32 * TT;
    int pages[TT][2];
    bool paged = true;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const KvPages p = tile_pages(a.kv, ses, t0 + 32 * t, ses.len);
      pages[t][0] = p.page[0], pages[t][1] = p.page[1];
      paged = paged && p.page[0] >= 0 && p.page[1] >= 0;
    }
    int rt0, rt1;
    rows_that_see(ses, G, a.window, t0, t1, &rt0, &rt1);
    rt0 += share.phase;
    // A lane's row goes 16 x step further each time; one past the session's is its last.
    const int step = share.step, far_r = 16 * step / G, far_in = 16 * step - far_r * G;
    const int first_r = (rt0 * 16 + n) / G, first_in = rt0 * 16 + n - first_r * G;
    const int64_t heads = (int64_t)a.kv.heads * G;
    const int last_r = (live - 1) / G, last_in = live - 1 - last_r * G;

    f32x4_t acc[TT][2];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t][0] = acc[t][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int head = share.h0; head < share.h1 && rt0 < rt1; ++head) {
      const uint16_t* q0 = a.q + (int64_t)s * a.kv.R * a.q_row + (int64_t)head * G * a.q_head + g * (D / 4);
      const float* l0 = a.lse + (int64_t)s * a.kv.R * heads + head * G;
      int r = first_r, in = first_in, fq = rt0 * 16 + n;
      struct Fetched {
        u32x4_t q[KJ];
        float l;
      };
      Fetched even, odd;
      auto fetch = [&](Fetched& f) {
        const int at_r = fq < live ? r : last_r, at_in = fq < live ? in : last_in;
        const uint16_t* p = q0 + at_r * a.q_row + at_in * a.q_head;
        if (a.q_aligned) {
#pragma unroll
          for (int j = 0; j < KJ; ++j) f.q[j] = *reinterpret_cast<const u32x4_t*>(p + 8 * j);
        } else {
#pragma unroll
          for (int j = 0; j < KJ; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) f.q[j][i] = (uint32_t)p[8 * j + 2 * i] | ((uint32_t)p[8 * j + 2 * i + 1] << 16);
        }
        f.l = l0[at_r * heads + at_in];
      };
      fetch(even);
      bf16x8_t k[TT][2][KJ];
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int page = pages[t][b];
          const uint8_t* blk = kv_block<D>(a.kv, page < 0 ? 0 : page, head, page < 0 ? 0 : t0 + 32 * t + 16 * b);
          const uint32_t* codes = reinterpret_cast<const uint32_t*>(blk + n * (D / 2) + g * (D / 8));
          const uint8_t* sc = blk + KvLayout<D>::kKeyScales + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g) * kKvBlock + n;
#pragma unroll
          for (int j = 0; j < KJ; ++j) {
            const float x = e8m0_operand(sc[j / 4 * kKvBlock]);
            const uint32_t w = codes[j];
            const u32x4_t y{fp4_pair<0>(w, x), fp4_pair<1>(w, x), fp4_pair<2>(w, x), fp4_pair<3>(w, x)};
            k[t][b][j] = __builtin_bit_cast(bf16x8_t, y);
          }
        }
      // tile rt of the rows, with the next on its way
      auto take = [&](int rt, const Fetched& now, Fetched& next) {
        const bool dead = now.l == -INFINITY || fq >= live;  // the row sees nothing, or is none
        const float l = now.l * kLog2e;
        const int pos = base + r;
        const int low_pos = __builtin_amdgcn_readlane(pos, 0), high_pos = __builtin_amdgcn_readlane(pos, 15);
        const bool whole = paged && low_pos >= t1 - 1 && (a.window == 0 || t0 > high_pos - a.window) && !__any(dead);
        r += far_r;
        in += far_in;
        fq += 16 * step;
        if (in >= G) {
          in -= G;
          ++r;
        }
        if (rt + step < rt1) fetch(next);
        f32x4_t sc[2][2];
        auto score = [&](int t) {
          f32x4_t(&x)[2] = sc[t & 1];
          x[0] = x[1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int j = 0; j < KJ; ++j) {
            const bf16x8_t q = __builtin_bit_cast(bf16x8_t, now.q[j]);
            x[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][0][j], q, x[0], 0, 0, 0);
            x[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][1][j], q, x[1], 0, 0, 0);
          }
        };
        score(0);
        if (whole) {  // the products of the next tile beside the weights of this one
#pragma unroll
          for (int t = 0; t < TT; ++t) {
            if (t + 1 < TT) score(t + 1);
            add_weights(acc[t], sc[t & 1], a.scale_log2, l);
#pragma unroll
            for (int i = 0; i < 2 * KJ; ++i) {
              __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);                // a product,
              __builtin_amdgcn_sched_group_barrier(0x2, 16 / (2 * KJ) > 0 ? 16 / (2 * KJ) : 1, 0);  // vector instructions,
              __builtin_amdgcn_sched_group_barrier(0x400, 8 / (2 * KJ) > 0 ? 8 / (2 * KJ) : 1, 0);  // exponentials
            }
          }
        } else {
          const int most = pos < 0 || dead ? 0 : pos + 1;
          const int span = a.window > 0 && a.window < most ? a.window : most;
          const int from = t0 + 4 * g - (pos - span + 1);
#pragma unroll
          for (int t = 0; t < TT; ++t) {
            if (t > 0) score(t);
            add_seen(acc[t], sc[t & 1], a.scale_log2, l, from + 32 * t, span, pages[t]);
          }
        }
      };
      for (int rt = rt0; rt < rt1; rt += 2 * step) {
        take(rt, even, odd);
        if (rt + step < rt1) take(rt + step, odd, even);
      }
    }
    give_weights<TT>(a, ses, s, slot, part_of, share.whole, t0, TOKENS, acc, g, n);
  }
}

// The parts of a token's sum, in their order.
__global__ __launch_bounds__(256) void k_weigh_join(WeighArgs a, int tokens) {
  const int s = blockIdx.x % a.kv.n_sessions, j = blockIdx.x / a.kv.n_sessions * 256 + threadIdx.x;
  const KvSession ses = kv_session(a.kv, s);
  if (j >= tokens || j >= ses.len || ses.rows <= 0) return;
  const float* part = a.part + (int64_t)s * a.parts * tokens + j;
  float x = 0.0f;
#pragma unroll 8
  for (int k = 0; k < a.parts; ++k) x += part[(int64_t)k * tokens];
  float* w = a.w + (a.kv.slots ? a.kv.slots[s] : s) * a.ld_w + j;
  *w = (a.fresh && j >= ses.len - ses.rows ? 0.0f : *w) + x;
}

namespace {

// How a call's tokens, heads and rows are shared out.
struct WeighPlan {
  int mt;  // row tiles of a wave at a time, 0: keys in registers for many
  int groups, by_rows, heads_each, parts;
  int tokens;
};
WeighPlan weigh_plan(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t group, int64_t max_len) {
  WeighPlan p{};
  const int64_t tiles = (R * group + 15) / 16;
  p.mt = tiles > (d == 256 ? 2 : 4) ? 0 : tiles > 2 ? 4 : (int)tiles;
  p.tokens = weigh_tokens(d);
  p.groups = (int)((max_len + p.tokens - 1) / p.tokens);
  // (a workgroup goes on to further groups of tokens)
  const int64_t most_groups = (1 << 22) / n_sessions > 1 ? (1 << 22) / n_sessions : 1;
  if (p.groups > most_groups) p.groups = (int)most_groups;
  const int64_t units = n_sessions * p.groups, want = (p.mt == 0 ? 16 : 2) * kCUs;
  p.by_rows = 1;
  p.heads_each = (int)heads;
  p.parts = 1;
  if (units < want) {
    const int64_t need = (want + units - 1) / units;
    p.heads_each = (int)(need < heads ? (heads + need - 1) / need : 1);
    const int64_t by_heads = (heads + p.heads_each - 1) / p.heads_each;
    // what shares a head's rows converts its keys once each: worth it from eight tiles on
    const int64_t most = p.mt == 0 ? tiles / 8 : 1;
    p.by_rows = (int)(need / by_heads < most ? need / by_heads : most);
    if (p.by_rows < 1) p.by_rows = 1;
    p.parts = (int)by_heads * p.by_rows;
  }
  return p;
}

template <int D>
void launch_weigh(int mt, dim3 grid, const WeighArgs& a, hipStream_t s) {
  if (mt == 1) launch_kernel(k_weigh_few<D, 1>, grid, dim3(256), 0, s, a);
  else if (mt == 2) launch_kernel(k_weigh_few<D, 2>, grid, dim3(256), 0, s, a);
  else if (mt == 0) launch_kernel(k_weigh_many<D>, grid, dim3(256), 0, s, a);
  else if constexpr (D < 256) launch_kernel(k_weigh_few<D, 4>, grid, dim3(256), 0, s, a);
}

}  // namespace

size_t kv_weigh_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len) {
  const WeighPlan p = weigh_plan(d, n_sessions, R, heads, q_heads / heads, max_len);
  return p.parts == 1 ? 0 : (size_t)n_sessions * p.parts * p.groups * p.tokens * 4;
}

hipError_t launch_kv_weigh(int d, const KvArgs& kv, const WeighCall& c, void* workspace, hipStream_t s) {
  WeighArgs a{};
  a.kv = kv;
  a.q = static_cast<const uint16_t*>(c.q);
  a.q_row = c.q_row;
  a.q_head = c.q_head;
  a.lse = c.lse;
  a.w = c.weights;
  a.ld_w = c.ld_weights;
  a.group = c.q_heads / kv.heads;
  a.window = c.window;
  a.fresh = c.fresh;
  a.scale_log2 = c.scale * kLog2e;
  a.q_aligned = c.q_row % 8 == 0 && c.q_head % 8 == 0 && (reinterpret_cast<uintptr_t>(c.q) & 15) == 0;
  const WeighPlan p = weigh_plan(d, kv.n_sessions, kv.R, kv.heads, a.group, c.max_len);
  a.groups = p.groups;
  a.parts = p.parts;
  a.by_rows = p.by_rows;
  a.heads_each = p.heads_each;
  a.part = static_cast<float*>(workspace);
  const dim3 grid((unsigned)((int64_t)kv.n_sessions * p.groups * p.parts));
  if (d == 64) launch_weigh<64>(p.mt, grid, a, s);
  else if (d == 128) launch_weigh<128>(p.mt, grid, a, s);
  else launch_weigh<256>(p.mt, grid, a, s);
  if (p.parts > 1) {
    const int tokens = p.groups * p.tokens;
    launch_kernel(k_weigh_join, dim3((unsigned)((int64_t)kv.n_sessions * (tokens / 256))), dim3(256), 0, s, a, tokens);
  }
  return hipGetLastError();
}

}  // namespace sph

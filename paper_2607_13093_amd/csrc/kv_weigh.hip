// What each held token receives of the attention of a call's rows:
//
//   w[j] += sum_{r, h} exp(scale q[r, h] . K[j, h / G] - lse[r, h])
//   over the rows r that see j (kv_attend.hip), lse the log-sum-exp of their scores.
//
// A wave owns TT tiles of 32 tokens and goes over the key/value heads: a head's
// codes become operands of the first product once, in registers, and every tile of 16
// of the R G rows is multiplied with them,
//   S^T = K Q^T   (tokens x rows) 16x16x32 products,
// lane l = 16 g + n holding row n against tokens 4 g ... 4 g + 3 of each block.  Weights
// of one token stay apart by lanes and are added up over the rows and heads in
// registers; the 16 lanes meet once, at the end.  Every token is one wave's (or one
// wave's of each part of the heads and rows, joined in their order), so that sums do
// not depend on timing and nothing is added atomically.
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
constexpr int kWeighTiles = 4;                                         // tiles of 32 tokens of a wave
constexpr int weigh_tiles(int d, bool many) { return many && d == 256 ? 2 : kWeighTiles; }
constexpr int weigh_tokens(int d, bool many) { return 4 * 32 * weigh_tiles(d, many); }  // of a workgroup

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

// A lane's query operand of row fq of a head, and the row's log-sum-exp in binades: q of
// a row that is none is 0.
template <int D>
__device__ __forceinline__ float fetch_query(const WeighArgs& a, u32x4_t (&q)[D / 32], int s, int head, int r, int in_group,
                                             bool in, int g) {
  const int64_t row = (int64_t)s * a.kv.R + r;
  const int hq = head * a.group + in_group;
  const uint16_t* p = a.q + row * a.q_row + (int64_t)hq * a.q_head + g * (D / 4);
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    u32x4_t x{0u, 0u, 0u, 0u};
    if (in) {
      if (a.q_aligned) {
        x = *reinterpret_cast<const u32x4_t*>(p + 8 * j);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (uint32_t)p[8 * j + 2 * i] | ((uint32_t)p[8 * j + 2 * i + 1] << 16);
      }
    }
    q[j] = x;
  }
  return in ? a.lse[row * (a.kv.heads * a.group) + hq] : -INFINITY;
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

constexpr int kKeyStages = 4;
constexpr int weigh_waves(int d, int mt) { return d * mt <= 128 ? 4 : d * mt <= 256 ? 3 : 2; }

template <int D, int MT>
__global__ __launch_bounds__(256, weigh_waves(D, MT)) void k_weigh_few(WeighArgs a) {
  constexpr int TT = kWeighTiles, KJ = D / 32, TOKENS = weigh_tokens(D, false), NS = kKeyStages;
  __shared__ __align__(16) uint8_t smem[4 * NS * KeyStage<D>::kBytes];
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int part_of = blockIdx.x % a.parts;
  const int rest = blockIdx.x / a.parts;
  const int s = rest % a.kv.n_sessions;
  const KvSession ses = kv_session(a.kv, s);
  const int G = a.group, live = ses.rows * G, base = ses.len - ses.rows;
  const int slot = a.kv.slots ? a.kv.slots[s] : s;
  uint8_t* ring = smem + wave * (NS * KeyStage<D>::kBytes);
  const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void_t*)ring;
  const uint32_t key_at = n * (D / 2) + g * (D / 8);
  const uint32_t ks_at = KeyStage<D>::kCodes + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g) * kKvBlock + n;

  for (int at = rest / a.kv.n_sessions; at * TOKENS < ses.len; at += a.groups) {
    const WeighShare share = weigh_share(a, part_of, at);
    const int t0 = at * TOKENS + wave * (32 * TT), t1 = t0 + 32 * TT;
    if (share.h0 >= share.h1) continue;
    KvPages pages[TT];
    bool paged = true;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      pages[t] = tile_pages(a.kv, ses, t0 + 32 * t, ses.len);
      paged = paged && pages[t].page[0] >= 0 && pages[t].page[1] >= 0;
    }
    int rt0, rt1;
    rows_that_see(ses, G, a.window, t0, t1, &rt0, &rt1);
    // groups of MT tiles, those of this part
    const int g0 = rt0 / MT + share.phase, g1 = rt1 > rt0 ? (rt1 + MT - 1) / MT : 0;

    f32x4_t acc[TT][2];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t][0] = acc[t][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    // units: heads x groups of tiles; each goes over the TT tiles of tokens
    int head = share.h0, rg = g0;
    int ahead_head = head, ahead_rg = rg;  // of the unit that the next copies are for
    if (g0 < g1) {
#pragma unroll
      for (int t = 0; t < NS - 1; ++t) copy_keys<D>(ring + t * KeyStage<D>::kBytes, a.kv, head, t0 + 32 * t, pages[t], lane);
    }
    while (g0 < g1 && head < share.h1) {
      ahead_rg = rg + share.step;
      ahead_head = head;
      if (ahead_rg >= g1) {
        ahead_rg = g0;
        ++ahead_head;
      }
      const bool more = ahead_head < share.h1;
      u32x4_t qf[MT][KJ];
      float l[MT];
      int from[MT], span[MT];
      bool whole = paged;
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int fq = (rg * MT + m) * 16 + n;
        const int r = fq / G;
        l[m] = fetch_query<D>(a, qf[m], s, head, r, fq - r * G, fq < live, g);
      }
#pragma unroll
      for (int m = 0; m < MT; ++m) {
        const int low = (rg * MT + m) * 16, high = low + 15 < live ? low + 15 : live - 1;
        const int r = (low + n) / G, pos = base + r;
        const bool dead = l[m] == -INFINITY;  // the row sees nothing
        whole = whole && low + 16 <= live && base + low / G >= t1 - 1 && (a.window == 0 || t0 > base + high / G - a.window) &&
                !__any(dead);
        const int most = pos < 0 || dead ? 0 : pos + 1;
        span[m] = a.window > 0 && a.window < most ? a.window : most;
        from[m] = t0 + 4 * g - (pos - span[m] + 1);
        l[m] *= kLog2e;
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        constexpr int C = KeyStage<D>::kCopies;
        const int next = t + NS - 1;
        static_assert(NS == TT, "a unit's tiles are the ring's stages");
        if (next < TT) {
          copy_keys<D>(ring + next * KeyStage<D>::kBytes, a.kv, head, t0 + 32 * next, pages[next], lane);
          wait_copies<(NS - 1) * C>();
        } else if (more) {
          copy_keys<D>(ring + (next - TT) * KeyStage<D>::kBytes, a.kv, ahead_head, t0 + 32 * (next - TT), pages[next - TT], lane);
          wait_copies<(NS - 1) * C>();
        } else if (t == 1) {
          wait_copies<2 * C>();
        } else if (t == 2) {
          wait_copies<C>();
        } else {
          wait_copies<0>();
        }
        KvKeys<D> keys;
        const uint32_t stage = ring_at + t * KeyStage<D>::kBytes;
        read_keys<D>(keys, stage + key_at, stage + ks_at);
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
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          if (whole) add_weights(acc[t], sc[m], a.scale_log2, l[m]);
          else add_seen(acc[t], sc[m], a.scale_log2, l[m], from[m] + 32 * t, span[m], pages[t].page);
        }
      }
      head = ahead_head;
      rg = ahead_rg;
    }
    give_weights<TT>(a, ses, s, slot, part_of, share.whole, t0, TOKENS, acc, g, n);
  }
}

// Many rows: a head's keys stay in registers as operands while its tiles of rows pass.
template <int D>
__global__ __launch_bounds__(256, 2) void k_weigh_many(WeighArgs a) {
  constexpr int TT = weigh_tiles(D, true), KJ = D / 32, TOKENS = weigh_tokens(D, true);
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int part_of = blockIdx.x % a.parts;
  const int rest = blockIdx.x / a.parts;
  const int s = rest % a.kv.n_sessions;
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
    // a lane's row goes 16 x step further each time
    const int step = share.step, far_r = 16 * step / G, far_in = 16 * step - far_r * G;
    const int first_r = (rt0 * 16 + n) / G, first_in = rt0 * 16 + n - first_r * G;

    f32x4_t acc[TT][2];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t][0] = acc[t][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int head = share.h0; head < share.h1 && rt0 < rt1; ++head) {
      int r = first_r, in = first_in;
      u32x4_t next[KJ];
      float next_l = fetch_query<D>(a, next, s, head, r, in, rt0 * 16 + n < live, g);
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
      for (int rt = rt0; rt < rt1; rt += step) {
        bf16x8_t q[KJ];
#pragma unroll
        for (int j = 0; j < KJ; ++j) q[j] = __builtin_bit_cast(bf16x8_t, next[j]);
        const float l = next_l * kLog2e;
        const int pos = base + r;
        r += far_r;
        in += far_in;
        if (in >= G) in -= G, ++r;
        if (rt + step < rt1) next_l = fetch_query<D>(a, next, s, head, r, in, (rt + step) * 16 + n < live, g);
        const int low = rt * 16, high = low + 15 < live ? low + 15 : live - 1;
        const bool dead = l == -INFINITY;  // the row sees nothing
        const bool whole = paged && low + 16 <= live && base + low / G >= t1 - 1 &&
                           (a.window == 0 || t0 > base + high / G - a.window) && !__any(dead);
        const int most = pos < 0 || dead ? 0 : pos + 1;
        const int span = a.window > 0 && a.window < most ? a.window : most;
        const int from = t0 + 4 * g - (pos - span + 1);
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          f32x4_t sc[2];
          sc[0] = sc[1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
          for (int j = 0; j < KJ; ++j) {
            sc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][0][j], q[j], sc[0], 0, 0, 0);
            sc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[t][1][j], q[j], sc[1], 0, 0, 0);
          }
          if (whole) add_weights(acc[t], sc, a.scale_log2, l);
          else add_seen(acc[t], sc, a.scale_log2, l, from + 32 * t, span, pages[t]);
        }
      }
    }
    give_weights<TT>(a, ses, s, slot, part_of, share.whole, t0, TOKENS, acc, g, n);
  }
}

// The parts of a token's sum, in their order.
__global__ __launch_bounds__(256) void k_weigh_join(WeighArgs a, int tokens) {
  const int s = blockIdx.x % a.kv.n_sessions, j = blockIdx.x / a.kv.n_sessions * 256 + threadIdx.x;
  const KvSession ses = kv_session(a.kv, s);
  if (j >= tokens || j >= ses.len) return;
  const float* part = a.part + (int64_t)s * a.parts * tokens + j;
  float x = 0.0f;
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
  p.tokens = weigh_tokens(d, p.mt == 0);
  p.groups = (int)((max_len + p.tokens - 1) / p.tokens);
  // (a workgroup goes on to further groups of tokens)
  const int64_t most_groups = (1 << 22) / n_sessions > 1 ? (1 << 22) / n_sessions : 1;
  if (p.groups > most_groups) p.groups = (int)most_groups;
  const int64_t units = n_sessions * p.groups, want = (p.mt == 0 ? 8 : 2) * kCUs;
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

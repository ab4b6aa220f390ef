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
constexpr int weigh_tiles(int d) { return d == 256 ? 2 : 4; }
constexpr int weigh_tokens(int d) { return 4 * 32 * weigh_tiles(d); }  // of a workgroup

template <int D>
__global__ __launch_bounds__(256, 2) void k_kv_weigh(WeighArgs a) {
  constexpr int TT = weigh_tiles(D), KJ = D / 32, TOKENS = weigh_tokens(D);
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int part_of = blockIdx.x % a.parts;
  const int rest = blockIdx.x / a.parts;
  const int s = rest % a.kv.n_sessions;
  const KvSession ses = kv_session(a.kv, s);
  const int G = a.group, live = ses.rows * G, base = ses.len - ses.rows;
  const int slot = a.kv.slots ? a.kv.slots[s] : s;

  for (int at = rest / a.kv.n_sessions; at * TOKENS < ses.len; at += a.groups) {
    // tokens past those that max_len promised have no place among the parts
    const bool whole_call = a.parts == 1 || at >= a.groups;
    if (whole_call && part_of > 0) continue;
    const int h0 = whole_call ? 0 : part_of / a.by_rows * a.heads_each;
    const int h1 = whole_call ? a.kv.heads : (h0 + a.heads_each < a.kv.heads ? h0 + a.heads_each : a.kv.heads);
    const int step = whole_call ? 1 : a.by_rows, phase = whole_call ? 0 : part_of % a.by_rows;

    const int t0 = at * TOKENS + wave * (32 * TT), t1 = t0 + 32 * TT;
    int pages[TT][2];
    bool paged = true;
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const KvPages p = tile_pages(a.kv, ses, t0 + 32 * t, ses.len);
      pages[t][0] = p.page[0], pages[t][1] = p.page[1];
      paged = paged && p.page[0] >= 0 && p.page[1] >= 0;
    }
    // tiles of rows that see any of the tokens
    const int first_row = t0 > base ? t0 - base : 0;
    const int64_t out_row = (int64_t)t1 - 1 + a.window - base;  // the first past all tokens' windows
    const int past_row = a.window > 0 && out_row < ses.rows ? (int)out_row : ses.rows;
    int rt0 = (int)((int64_t)first_row * G / 16), rt1 = past_row > first_row ? (int)(((int64_t)past_row * G + 15) / 16) : 0;
    if (t0 >= ses.len) rt1 = 0;
    rt0 += phase;

    f32x4_t acc[TT][2];
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[t][0] = acc[t][1] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    uint32_t c[TT][2][KJ], cs[TT][2];
    auto fetch_keys = [&](int head) {
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int page = pages[t][b];
          const uint8_t* blk = kv_block<D>(a.kv, page < 0 ? 0 : page, head, page < 0 ? 0 : t0 + 32 * t + 16 * b);
          const uint8_t* codes = blk + n * (D / 2) + g * (D / 8);
          if constexpr (D == 64) {
            const u32x2_t x = *reinterpret_cast<const u32x2_t*>(codes);
            c[t][b][0] = x[0], c[t][b][1] = x[1];
          } else {
#pragma unroll
            for (int i = 0; i < KJ; i += 4) {
              const u32x4_t x = *reinterpret_cast<const u32x4_t*>(codes + 4 * i);
#pragma unroll
              for (int e = 0; e < 4; ++e) c[t][b][i + e] = x[e];
            }
          }
          const uint8_t* sc = blk + KvLayout<D>::kKeyScales + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g) * kKvBlock + n;
          cs[t][b] = sc[0];
          if constexpr (D == 256) cs[t][b] |= (uint32_t)sc[kKvBlock] << 8;
        }
    };
    u32x4_t qn[KJ];
    float ln = 0.0f;
    auto fetch_rows = [&](int head, int rt) {
      const int fq = rt * 16 + n;
      const int r = fq / G, hq = head * G + fq - r * G;
      const int64_t row = (int64_t)s * a.kv.R + r;
      const bool in = fq < live;
      const uint16_t* p = a.q + row * a.q_row + (int64_t)hq * a.q_head + g * (D / 4);
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        u32x4_t x{0u, 0u, 0u, 0u};
        if (in) {
          if (a.q_aligned) {
            x = *reinterpret_cast<const u32x4_t*>(p + 8 * j);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (uint32_t)p[8 * j + 2 * i] | ((uint32_t)p[8 * j + 2 * i + 1] << 16);
          }
        }
        qn[j] = x;
      }
      ln = in ? a.lse[row * (a.kv.heads * G) + hq] : -INFINITY;
    };

    if (rt0 < rt1 && h0 < h1) {
      fetch_keys(h0);
      fetch_rows(h0, rt0);
    }
    for (int head = h0; head < h1 && rt0 < rt1; ++head) {
      bf16x8_t k[TT][2][KJ];
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int j = 0; j < KJ; ++j) {
            const float x = e8m0_operand(D == 256 ? (cs[t][b] >> (8 * (j / 4))) & 0xFFu : cs[t][b]);
            const uint32_t w = c[t][b][j];
            const u32x4_t y{fp4_pair<0>(w, x), fp4_pair<1>(w, x), fp4_pair<2>(w, x), fp4_pair<3>(w, x)};
            k[t][b][j] = __builtin_bit_cast(bf16x8_t, y);
          }
      if (head + 1 < h1) fetch_keys(head + 1);  // on its way while the rows are taken
      for (int rt = rt0; rt < rt1; rt += step) {
        bf16x8_t q[KJ];
#pragma unroll
        for (int j = 0; j < KJ; ++j) q[j] = __builtin_bit_cast(bf16x8_t, qn[j]);
        const float l = ln * kLog2e;
        if (rt + step < rt1) fetch_rows(head, rt + step);
        else if (head + 1 < h1) fetch_rows(head + 1, rt0);
        const int low = rt * 16, high = low + 15 < live ? low + 15 : live - 1;
        const int low_pos = base + low / G, high_pos = base + high / G;
        const bool dead = l == -INFINITY;  // the row sees nothing
        const bool whole = paged && low + 16 <= live && low_pos >= t1 - 1 && (a.window == 0 || t0 > high_pos - a.window) &&
                           !__any(dead);
        const int pos = base + (low + n) / G, most = pos < 0 || dead ? 0 : pos + 1;
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
          if (whole) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[t][b][e] += __builtin_amdgcn_exp2f(fmaf(sc[b][e], a.scale_log2, -l));
          } else {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(fmaf(sc[b][e], a.scale_log2, -l));
                const bool sees = (uint32_t)(from + 32 * t + 16 * b + e) < (uint32_t)span && pages[t][b] >= 0;
                acc[t][b][e] += sees ? p : 0.0f;
              }
          }
        }
      }
    }

    // over the 16 rows of a lane group; lane n keeps values n and, of 32, n + 16
    float out[(TT * 8 + 15) / 16];
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
    for (int i = 0; i < (TT * 8 + 15) / 16; ++i) {
      const int v = i * 16 + n;
      const int j = t0 + v / 4 * 16 + 4 * g + v % 4;
      if (j >= ses.len) continue;
      if (whole_call) {
        float* w = a.w + slot * a.ld_w + j;
        *w = (a.fresh && j >= base ? 0.0f : *w) + out[i];
      } else {
        a.part[((int64_t)s * a.parts + part_of) * ((int64_t)a.groups * TOKENS) + j] = out[i];
      }
    }
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
  int groups, by_rows, heads_each, parts;
};
WeighPlan weigh_plan(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t group, int64_t max_len) {
  WeighPlan p{};
  p.groups = (int)((max_len + weigh_tokens(d) - 1) / weigh_tokens(d));
  // (a workgroup goes on to further groups of tokens)
  const int64_t most_groups = (1 << 22) / n_sessions > 1 ? (1 << 22) / n_sessions : 1;
  if (p.groups > most_groups) p.groups = (int)most_groups;
  const int64_t units = n_sessions * p.groups, want = 2 * kCUs;  // two workgroups of a CU are resident
  p.by_rows = 1;
  p.heads_each = (int)heads;
  p.parts = 1;
  if (units < want) {
    const int64_t need = (want + units - 1) / units;
    p.heads_each = (int)(need < heads ? (heads + need - 1) / need : 1);
    const int64_t by_heads = (heads + p.heads_each - 1) / p.heads_each;
    const int64_t tiles = (R * group + 15) / 16;
    // a tile of rows is worth its keys' conversion from four on
    const int64_t most = tiles / 4 > 1 ? tiles / 4 : 1;
    p.by_rows = (int)(need / by_heads < most ? (need / by_heads > 1 ? need / by_heads : 1) : most);
    p.parts = (int)by_heads * p.by_rows;
  }
  return p;
}

}  // namespace

size_t kv_weigh_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len) {
  const WeighPlan p = weigh_plan(d, n_sessions, R, heads, q_heads / heads, max_len);
  return p.parts == 1 ? 0 : (size_t)n_sessions * p.parts * p.groups * weigh_tokens(d) * 4;
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
  if (d == 64) launch_kernel(k_kv_weigh<64>, grid, dim3(256), 0, s, a);
  else if (d == 128) launch_kernel(k_kv_weigh<128>, grid, dim3(256), 0, s, a);
  else launch_kernel(k_kv_weigh<256>, grid, dim3(256), 0, s, a);
  if (p.parts > 1) {
    const int tokens = p.groups * weigh_tokens(d);
    launch_kernel(k_weigh_join, dim3((unsigned)((int64_t)kv.n_sessions * (tokens / 256))), dim3(256), 0, s, a, tokens);
  }
  return hipGetLastError();
}

}  // namespace sph

// Rows of keys and values into the paged 4-bit cache, and back.
//
// 32 values share a scale 2^e with e = floor(log2 m) - 2, m their largest
// magnitude rounded to two significant bits (ties to even): the least e for
// which no value rounds past 6, the largest E2M1 magnitude (at most 125).  A code is the
// nearest E2M1 value of x 2^-e, ties to even.
//
// Bound by memory: 8 prompts of 2048 to 4096 tokens with 8 heads of 128 are written
// in 25.6 us and read back in 24.6, 5.2 TB/s in and out, a copy's rate; a window's
// rows (64 x 5) take a launch's 3.5 us.
#include "kv_cache.h"

namespace sph {

struct KvRows {
  uint16_t* p;      // bf16 [M][heads][D], rows and heads apart by
  int64_t row, head;
  bool aligned;     // 16-byte loads and stores are possible
};

__device__ __forceinline__ u32x4_t load_octet(const KvRows& x, int64_t row, int head, int d) {
  const uint16_t* p = x.p + row * x.row + head * x.head + d;
  if (x.aligned) return *reinterpret_cast<const u32x4_t*>(p);
  u32x4_t v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
  return v;
}

__device__ __forceinline__ void store_octet(const KvRows& x, int64_t row, int head, int d, u32x4_t v) {
  uint16_t* p = x.p + row * x.row + head * x.head + d;
  if (x.aligned) {
    *reinterpret_cast<u32x4_t*>(p) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p[2 * i] = (uint16_t)v[i];
    p[2 * i + 1] = (uint16_t)(v[i] >> 16);
  }
}

// Largest magnitude of a lane's eight bf16 values, as bf16 bits (infinities and
// NaN are the largest: 0x7F80 and above).
__device__ __forceinline__ uint32_t octet_top(u32x4_t v) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = v[i] & 0x7FFFu, hi = (v[i] >> 16) & 0x7FFFu;
    m = m > lo ? m : lo;
    m = m > hi ? m : hi;
  }
  return m;
}
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {  // of four neighbouring lanes
  uint32_t o = dpp_u32<0xB1>(m);                            // quad_perm 1,0,3,2
  m = m > o ? m : o;
  o = dpp_u32<0x4E>(m);                                     // quad_perm 2,3,0,1
  return m > o ? m : o;
}

// Scale byte of a group whose largest magnitude has the bits `top`.
__device__ __forceinline__ uint32_t group_scale(uint32_t top) {
  const int e = (int)((top + 0x1Fu + ((top >> 6) & 1u)) >> 7) - 2;  // biased, of the rounded top
  // infinities and what would round to 2^128 saturate: 6 2^126 is no bf16
  return e < 0 ? 0u : (e < 252 ? (uint32_t)e : 252u);
}

// Eight codes, the first in the low bits.  Values past 6 steps (infinities)
// saturate; a NaN's code is whatever the conversion gives: its token answers
// NaN by its keys' scales.
template <int BYTE>
__device__ __forceinline__ uint32_t pair_codes(uint32_t c, uint32_t pair, float s) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, pair), s, BYTE);
}
__device__ __forceinline__ uint32_t octet_codes(u32x4_t v, uint32_t scale) {
  const float s = e8m0_operand(scale);
  return pair_codes<3>(pair_codes<2>(pair_codes<1>(pair_codes<0>(0u, v[0], s), v[1], s), v[2], s), v[3], s);
}

// Byte of the values' codes of part n of token t in its block.
template <int D>
__device__ __forceinline__ int value_at(int t, int n) {
  return KvLayout<D>::kValues + (((t >> 2) * 16 + n) * 4 + (t & 3)) * (D / 32);
}

// A workgroup takes 16 tokens of a block of one head, D/8 lanes a token, eight
// values of keys and of values a lane: what it writes is contiguous, so lines
// are written whole by one workgroup where a prompt fills them.
template <int D>
__global__ __launch_bounds__(2 * D) void k_kv_append(KvArgs a, KvRows k, KvRows v) {
  constexpr int LPT = D / 8;  // lanes per token: 8, 16 or 32, neighbours in one wave
  const int s = blockIdx.z, head = blockIdx.y;
  const KvSession ses = kv_session(a, s);
  const int first = ses.len - ses.rows;  // position of row 0
  const int t = threadIdx.x / LPT, o = threadIdx.x % LPT;
  const int pos = ((first >> 4) + (int)blockIdx.x) * kKvBlock + t;
  const int r = pos - first;
  // lanes of one token agree on all of this
  const bool mine = pos >= 0 && r >= 0 && r < ses.rows;
  const int page = mine ? kv_page(a, ses, pos) : -1;
  if (page < 0) return;
  const int64_t row = (int64_t)s * a.R + r;
  const u32x4_t kx = load_octet(k, row, head, o * 8), vx = load_octet(v, row, head, o * 8);
  const uint32_t ktop = quad_max(octet_top(kx)), vtop = quad_max(octet_top(vx));
  uint32_t worst = ktop > vtop ? ktop : vtop;
#pragma unroll
  for (int x = 4; x < LPT; x <<= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)worst, x, 64);
    worst = worst > y ? worst : y;
  }
  uint32_t ks = group_scale(ktop);
  const uint32_t vs = group_scale(vtop);
  const uint32_t kc = octet_codes(kx, ks), vc = octet_codes(vx, vs);
  // A token with an infinity or a NaN gets NaN scales for its keys: rows that see
  // it answer NaN, and its values, which a matrix product also gives to rows that
  // do not see it (times zero), stay finite.
  if (worst >= 0x7F80u) ks = 255u;
  uint8_t* b = kv_block<D>(a, page, head, pos);
  *reinterpret_cast<uint32_t*>(b + t * (D / 2) + o * 4) = kc;
  if constexpr (D == 64) {  // an octet is two parts
    *reinterpret_cast<uint16_t*>(b + value_at<D>(t, 2 * o)) = (uint16_t)vc;
    *reinterpret_cast<uint16_t*>(b + value_at<D>(t, 2 * o + 1)) = (uint16_t)(vc >> 16);
  } else {                  // or one, or half of one
    constexpr int OPP = D / 128;
    *reinterpret_cast<uint32_t*>(b + value_at<D>(t, o / OPP) + o % OPP * 4) = vc;
  }
  if (o % 4 == 0) {
    b[KvLayout<D>::kKeyScales + o / 4 * kKvBlock + t] = (uint8_t)ks;
    b[KvLayout<D>::kValueScales + o / 4 * kKvBlock + t] = (uint8_t)vs;
  }
}

// The same rows back as the values that they stand for (those below 2^-126 to
// within that); zeros where there is no row, or no page.
template <int D>
__global__ __launch_bounds__(2 * D) void k_kv_read(KvArgs a, KvRows k, KvRows v) {
  constexpr int LPT = D / 8;
  const int s = blockIdx.z, head = blockIdx.y;
  const KvSession ses = kv_session(a, s);
  const int first = ses.len - ses.rows;
  const int t = threadIdx.x / LPT, o = threadIdx.x % LPT;
  const int pos = ((first >> 4) + (int)blockIdx.x) * kKvBlock + t;
  const int r = pos - first;
  if (r < 0 || r >= a.R) return;
  const int page = pos >= 0 && r < ses.rows ? kv_page(a, ses, pos) : -1;
  const int64_t row = (int64_t)s * a.R + r;
  u32x4_t kx{0u, 0u, 0u, 0u}, vx{0u, 0u, 0u, 0u};
  if (page >= 0) {
    const uint8_t* b = kv_block<D>(a, page, head, pos);
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(b + t * (D / 2) + o * 4);
    uint32_t vc;
    if constexpr (D == 64) {
      vc = *reinterpret_cast<const uint16_t*>(b + value_at<D>(t, 2 * o)) |
           ((uint32_t)*reinterpret_cast<const uint16_t*>(b + value_at<D>(t, 2 * o + 1)) << 16);
    } else {
      constexpr int OPP = D / 128;
      vc = *reinterpret_cast<const uint32_t*>(b + value_at<D>(t, o / OPP) + o % OPP * 4);
    }
    const float ks = e8m0_operand(b[KvLayout<D>::kKeyScales + o / 4 * kKvBlock + t]);
    const float vs = e8m0_operand(b[KvLayout<D>::kValueScales + o / 4 * kKvBlock + t]);
    kx = u32x4_t{fp4_pair<0>(kc, ks), fp4_pair<1>(kc, ks), fp4_pair<2>(kc, ks), fp4_pair<3>(kc, ks)};
    vx = u32x4_t{fp4_pair<0>(vc, vs), fp4_pair<1>(vc, vs), fp4_pair<2>(vc, vs), fp4_pair<3>(vc, vs)};
  }
  store_octet(k, row, head, o * 8, kx);
  store_octet(v, row, head, o * 8, vx);
}

namespace {
KvRows rows_of(const void* p, int64_t row, int64_t head) {
  KvRows x{static_cast<uint16_t*>(const_cast<void*>(p)), row, head, false};
  x.aligned = row % 8 == 0 && head % 8 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
  return x;
}

template <int D>
void launch_rows(bool append, const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t s) {
  // R rows that start anywhere in a block of 16
  const dim3 grid((a.R + 14) / 16 + 1, a.heads, a.n_sessions);
  if (append)
    launch_kernel(k_kv_append<D>, grid, dim3(2 * D), 0, s, a, k, v);
  else
    launch_kernel(k_kv_read<D>, grid, dim3(2 * D), 0, s, a, k, v);
}
}  // namespace

hipError_t launch_kv_rows(bool append, int d, const KvArgs& a, const void* k, int64_t k_row,
                          int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                          hipStream_t s) {
  if (a.n_sessions <= 0 || a.R <= 0) return hipSuccess;
  const KvRows kr = rows_of(k, k_row, k_head), vr = rows_of(v, v_row, v_head);
  if (d == 64) launch_rows<64>(append, a, kr, vr, s);
  else if (d == 128) launch_rows<128>(append, a, kr, vr, s);
  else if (d == 256) launch_rows<256>(append, a, kr, vr, s);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace sph

// The paged 4-bit key/value cache as the kernels see it: the block layout, the
// E2M1 conversions, and where a session's rows lie.
#pragma once

#include "sph_internal.h"

namespace sph {

typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// A block of 16 tokens of one head of D values is 17 D bytes:
//   keys' codes    16 rows of D/2 bytes, a token each
//   values' codes  [4 quads of tokens][16 parts][4 tokens][D/32 bytes]: part n
//                  is values n D/16 ... of a token
//   keys' scales   [D/32 groups][16 tokens] bytes
//   values' scales the same
// Lane l = 16 g + n of a wave then reads its operands of the matrix
// instructions as D/8 contiguous bytes of either codes: of the keys token n,
// dimensions g D/4 ...; of the values tokens 4 g ... 4 g + 3, part n, which is a
// column of V^T for each of D/16 products (see kv_attend.hip).  A token of its
// own is still whole words in all four, so that appending one writes no byte of
// another.
constexpr int kKvBlock = 16;  // tokens
constexpr int kKvMost = 1 << 30;  // tokens of a session, so that positions and shares stay in 32 bits
template <int D>
struct KvLayout {
  static constexpr int kBytes = 17 * D;
  static constexpr int kValues = 8 * D;                // offsets in a block
  static constexpr int kKeyScales = 16 * D;
  static constexpr int kValueScales = 16 * D + D / 2;
};

// Where calls on a layer find its pages, and the sessions of a call: session s
// is slot slots[s] (s if null) and has rows[s] rows (R if null), the last ones
// of its lens[slot] tokens.
struct KvArgs {
  uint8_t* pool;        // the layer's pages, page_stride bytes apart
  int64_t page_stride;
  int n_pages;
  const int32_t* table; // [n_slots][ld_table]
  int64_t ld_table;
  int max_pages;        // entries of a slot
  const int32_t* lens;
  const int32_t* rows;
  const int32_t* slots;
  int n_slots;
  int n_sessions;
  int R;
  int heads;            // key/value heads
  int page_shift;       // log2 of the tokens of a page
};

// A page pool's upkeep: the whole cache, not one layer.
struct PagesArgs {
  uint8_t* pool;        // layer_stride bytes from layer to layer
  int64_t layer_stride, page_stride, page_bytes;
  int layers;
  int n_pages;
  int32_t* table;       // [n_slots][ld_table], -1 where there is no page
  int64_t ld_table;
  int max_pages;
  int32_t* lens;
  int32_t* refs;        // [n_pages]
  int n_slots;
  int page_shift;
};

struct AttendCall {
  const void* q;
  int64_t q_row, q_head;
  int q_heads;
  float scale;
  int window;
  int64_t max_len;
  void* out;
  int64_t o_row, o_head;
  float* lse;
};

struct WeighCall {
  const void* q;
  int64_t q_row, q_head;
  int q_heads;
  const float* lse;
  float scale;
  int window;
  int64_t max_len;
  int fresh;
  float* weights;          // [n_slots][ld_weights]
  int64_t ld_weights;
};

struct EvictCall {
  const float* weights;    // [n_slots][ld_weights]
  int64_t ld_weights;
  const int32_t* keep;     // [n_slots]
  int first, recent;
  float* weights_out;      // may be weights
  int64_t ld_out;
  int32_t* kept;           // [n_slots][ld_kept] or null
  int64_t ld_kept;
};

// Launchers (return the HIP launch status); d: the head size, 64, 128 or 256.
hipError_t launch_kv_rows(bool append, int d, const KvArgs& a, const void* k, int64_t k_row,
                          int64_t k_head, const void* v, int64_t v_row, int64_t v_head,
                          hipStream_t s);
size_t kv_attend_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads,
                         int64_t max_len, int64_t window);
// How such a call is shared out: row tiles of a wave, waves that share its rows,
// workgroups for the rows of a head, shares of the tokens, tokens of a share.
void kv_attend_shape(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len,
                     int64_t window, int shape[5]);
// What such a call's window comes to where no session holds more than `most` tokens:
// one that leaves none of them out is none (0).
int64_t kv_window(int64_t window, int64_t most);
// Tokens that a wave's rows see (some, all of them) and those of one share: lo, hi,
// all_lo, all_hi, from, to.
void kv_attend_span(int base, int r_lo, int r_hi, int window, int split, int splits, int chunk, int span[6]);
hipError_t launch_kv_attend(int d, const KvArgs& kv, const AttendCall& c, void* workspace, hipStream_t s);

constexpr int kShareSessions = 2048;  // of a plan
bool kv_share_fits(int64_t n_sessions, int64_t R, int64_t q_heads);
size_t kv_share_bytes(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len);
size_t kv_share_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len);
hipError_t launch_share_plan(int d, const KvArgs& kv, int q_heads, int window, int64_t max_len, void* plan, hipStream_t s);
hipError_t launch_attend_shared(int d, const KvArgs& kv, const AttendCall& c, void* plan, void* workspace, hipStream_t s);

size_t kv_weigh_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len);
hipError_t launch_kv_weigh(int d, const KvArgs& kv, const WeighCall& c, void* workspace, hipStream_t s);

size_t pages_grow_scratch(int64_t n_pages, int64_t n_slots);
size_t pages_compact_scratch(int64_t n_pages);
hipError_t launch_pages_grow(const PagesArgs& a, const int32_t* add, int32_t* status, void* workspace, hipStream_t s);
hipError_t launch_pages_trim(const PagesArgs& a, const int32_t* kept, hipStream_t s);
hipError_t launch_pages_fork(const PagesArgs& a, const int32_t* parents, const int32_t* children, int n, hipStream_t s);
hipError_t launch_pages_copy(const PagesArgs& a, const int32_t* src, const int32_t* dst, int64_t n, hipStream_t s);
hipError_t launch_pages_compact(const PagesArgs& a, int32_t* table_out, int64_t ld_out, int32_t* refs_out,
                                int32_t* live_out, void* workspace, hipStream_t s);
// most: tokens that a row of the table names
size_t pages_evict_scratch(int64_t n_slots, int64_t most);
hipError_t launch_pages_evict(int d, int heads, int64_t most, const PagesArgs& p, const EvictCall& c, void* workspace,
                              hipStream_t s);

struct KvSession {
  const int32_t* table;  // its page row
  int len;               // tokens held
  int rows;              // its rows, at positions len - rows ...
};

// A slot out of range holds nothing; lengths are cut to what a page row can
// name, row counts to [0, R].
__device__ __forceinline__ int kv_length(const KvArgs& a, int slot) {
  const int64_t named = (int64_t)a.max_pages << a.page_shift, most = named < kKvMost ? named : kKvMost;
  const int len = (unsigned)slot < (unsigned)a.n_slots ? a.lens[slot] : 0;
  return len < 0 ? 0 : (len > most ? (int)most : len);
}
__device__ __forceinline__ KvSession kv_session(const KvArgs& a, int s) {
  const int slot = a.slots ? a.slots[s] : s;
  KvSession r;
  r.table = a.table + ((unsigned)slot < (unsigned)a.n_slots ? slot : 0) * a.ld_table;
  r.len = kv_length(a, slot);
  const int n = a.rows ? a.rows[s] : a.R;
  r.rows = n < 0 ? 0 : (n > a.R ? a.R : n);
  return r;
}

// Page of a position (>= 0), or -1 where the row names none.
__device__ __forceinline__ int kv_page(const KvArgs& a, const KvSession& s, int pos) {
  const int i = pos >> a.page_shift;
  const int p = i < a.max_pages ? s.table[i] : -1;
  return (unsigned)p < (unsigned)a.n_pages ? p : -1;
}

template <int D>
__device__ __forceinline__ uint8_t* kv_block(const KvArgs& a, int page, int head, int pos) {
  const int in_page = (pos & ((1 << a.page_shift) - 1)) / kKvBlock;
  const int per_head = (1 << a.page_shift) / kKvBlock;
  return a.pool + page * a.page_stride + (int64_t)(head * per_head + in_page) * KvLayout<D>::kBytes;
}

// An E8M0 byte as the fp32 whose exponent field the conversions use (byte 0 is
// 2^-127, byte 255 NaN).
__device__ __forceinline__ float e8m0_operand(uint32_t byte) { return __uint_as_float(byte << 23); }

// The same for a byte of a word, number a constant: one instruction with the byte
// selected by its operand (the compiler makes two of three of them a shift and a mask).
__device__ __forceinline__ float e8m0_operand_at(uint32_t word, int byte) {
  uint32_t r;
  const uint32_t by = 23;
#define SPH_BYTE(N)                                                                                  \
  asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_" #N \
      : "=v"(r) : "v"(by), "v"(word))
  switch (byte) {
    case 0: SPH_BYTE(0); break;
    case 1: SPH_BYTE(1); break;
    case 2: SPH_BYTE(2); break;
    default: SPH_BYTE(3); break;
  }
#undef SPH_BYTE
  return __uint_as_float(r);
}

// Two E2M1 codes of a byte as bf16: exact, values below 2^-126 to within 2^-126.
template <int BYTE>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, BYTE));
}

// The same for a byte number that unrolling makes a constant.
__device__ __forceinline__ uint32_t fp4_pair_at(uint32_t codes, float scale, int byte) {
  switch (byte) {
    case 0: return fp4_pair<0>(codes, scale);
    case 1: return fp4_pair<1>(codes, scale);
    case 2: return fp4_pair<2>(codes, scale);
    default: return fp4_pair<3>(codes, scale);
  }
}

}  // namespace sph

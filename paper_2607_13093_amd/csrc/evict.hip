// Eviction: every slot keeps a number of its tokens, those that received the most
// attention, and the kept ones move together, in order, in every layer and head.
//
// One workgroup a slot chooses them: a search for the weight that the last kept
// token has, a digit of its order at a time, then one pass that numbers the kept
// tokens and notes where each lies.  Whole pages behind the new length are given
// back.  Pages that other slots hold too lie at the front of a row and stay as they
// are, so that nothing moves out of them or into them.
//
// Tokens only ever move down, so they move in place: a workgroup takes one slot,
// layer and head and goes up its blocks, a chunk at a time; all of a chunk is read
// before any of it is written, and what later chunks read lies above it.
#include "kv_cache.h"

namespace sph {

struct EvictSlot {
  int32_t start, len;  // first token that moves, tokens kept (start == len: none moves)
};

struct EvictArgs {
  PagesArgs p;
  EvictCall c;
  int heads, block_bytes;
  int most;          // tokens that a row of the table names
  int64_t* from;     // [n_slots][most]: where the token to come to a place lies
  EvictSlot* slots;  // [n_slots]
};

// A weight's place in the order of all: NaN below -infinity, -0 beside 0.
__device__ __forceinline__ uint32_t order_of(float w) {
  const uint32_t u = __float_as_uint(w);
  if (w != w) return 0u;
  if (w == 0.0f) return 0x80000000u;
  return (int32_t)u < 0 ? ~u : u | 0x80000000u;
}

constexpr int kChoose = 1024;  // threads that choose a slot's tokens
constexpr int kLook = 4;       // tokens a thread looks at in a turn

__global__ __launch_bounds__(kChoose) void k_evict_choose(EvictArgs a) {
  __shared__ uint32_t s_bins[16][256];
  __shared__ int s_sure[64], s_tie[64];
  __shared__ int s_shared, s_start, s_digit, s_need;
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const PagesArgs& p = a.p;
  int32_t* row = p.table + (int64_t)s * p.ld_table;
  const float* w = a.c.weights + s * a.c.ld_weights;
  float* w_out = a.c.weights_out + s * a.c.ld_out;
  int32_t* kept = a.c.kept ? a.c.kept + s * a.c.ld_kept : nullptr;
  int64_t* from = a.from + (int64_t)s * a.most;

  const int held_len = p.lens[s];
  const int len = held_len < 0 ? 0 : (held_len < a.most ? held_len : a.most);
  const int held = (len + (1 << p.page_shift) - 1) >> p.page_shift;
  if (threadIdx.x == 0) {
    s_shared = 0;
    s_start = len;
  }
  __syncthreads();
  int last = 0;  // pages up to the last that others hold too
  for (int c = threadIdx.x; c < held; c += kChoose) {
    const int page = row[c];
    if ((unsigned)page < (unsigned)p.n_pages && p.refs[page] > 1) last = c + 1;
  }
  if (last) atomicMax(&s_shared, last);
  __syncthreads();
  const int64_t fixed = (int64_t)s_shared << p.page_shift;
  int front = fixed > a.c.first ? (fixed < len ? (int)fixed : len) : (a.c.first < len ? a.c.first : len);
  const int back = len - front > a.c.recent ? len - a.c.recent : front;
  const int must = front + len - back;
  const int want = a.c.keep[s];
  const int n = want < must ? must : (want < len ? want : len);
  int need = n - must;  // of the tokens from front to back

  // the weight of the last that is kept, and how many of that weight are
  uint32_t least = 0;
  if (need > 0 && n < len) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 16 * 256; i += kChoose) s_bins[0][i] = 0;
      __syncthreads();
      for (int j = front + threadIdx.x; j < back; j += kChoose) {
        const uint32_t x = order_of(w[j]);
        if (shift == 24 || (x ^ least) >> (shift + 8) == 0) atomicAdd(&s_bins[wave][(x >> shift) & 255], 1u);
      }
      __syncthreads();
      if (threadIdx.x < 256) {
        uint32_t t = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += s_bins[k][threadIdx.x];
        s_bins[0][threadIdx.x] = t;
      }
      __syncthreads();
      if (wave == 0) {  // lane l: digits 255 - 4 l ... down
        int t[4], all = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) all += t[k] = s_bins[0][255 - 4 * lane - k];
        int before = all;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const int y = __shfl_up(before, o, 64);
          if (lane >= o) before += y;
        }
        before -= all;
        if (before < need && need <= before + all) {
          int k = 0;
          while (k < 3 && need > before + t[k]) before += t[k++];
          s_digit = 255 - 4 * lane - k;
          s_need = need - before;
        }
      }
      __syncthreads();
      least |= (uint32_t)s_digit << shift;
      need = s_need;
      __syncthreads();
    }
  }

  // numbers of the kept ones, in order; equal weights are kept from the first on
  int sure_before = 0, tie_before = 0;
  for (int at = 0; at < len; at += kLook * kChoose) {
    float x[kLook];
    uint64_t sure[kLook], tie[kLook];
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      const int j = at + i * kChoose + threadIdx.x;
      x[i] = j < len ? w[j] : 0.0f;
      bool is_sure = n == len && j < len, is_tie = false;
      if (j < front || (j >= back && j < len)) is_sure = true;
      else if (j < len && n < len && need > 0) {
        const uint32_t o = order_of(x[i]);
        is_sure = o > least;
        is_tie = o == least;
      }
      sure[i] = __ballot(is_sure);
      tie[i] = __ballot(is_tie);
      if (lane == 0) {
        s_sure[i * 16 + wave] = __popcll(sure[i]);
        s_tie[i * 16 + wave] = __popcll(tie[i]);
      }
    }
    __syncthreads();
    int ns = s_sure[lane], nt = s_tie[lane];
    const int ms = ns, mt = nt;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(ns, o, 64), z = __shfl_up(nt, o, 64);
      if (lane >= o) ns += y, nt += z;
    }
    const int all_sure = __shfl(ns, 63, 64), all_tie = __shfl(nt, 63, 64);
    ns -= ms;
    nt -= mt;
    const uint64_t below = (uint64_t(1) << lane) - 1;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      const int j = at + i * kChoose + threadIdx.x;
      const int t = tie_before + __shfl(nt, i * 16 + wave, 64) + __popcll(tie[i] & below);
      const int to = sure_before + __shfl(ns, i * 16 + wave, 64) + __popcll(sure[i] & below) + (t < need ? t : need);
      const bool stays = (sure[i] >> lane & 1) || ((tie[i] >> lane & 1) && t < need);
      if (stays) {
        const int page = row[j >> p.page_shift];
        const int in_page = j & ((1 << p.page_shift) - 1);
        from[to] = (unsigned)page < (unsigned)p.n_pages
                       ? (page * p.page_stride + (in_page / kKvBlock) * a.block_bytes) | (in_page % kKvBlock)
                       : -1;
        w_out[to] = x[i];
        if (kept) kept[to] = j;
      } else if (j < len) {
        atomicMin(&s_start, j);
      }
    }
    sure_before += all_sure;
    tie_before += all_tie;
    __syncthreads();  // the counts are free, the row and these weights read
  }
  for (int j = n + threadIdx.x; j < len; j += kChoose) w_out[j] = 0.0f;
  const int stay = (n + (1 << p.page_shift) - 1) >> p.page_shift;
  for (int c = stay + threadIdx.x; c < held; c += kChoose) {
    const int page = row[c];
    if ((unsigned)page < (unsigned)p.n_pages) atomicSub(&p.refs[page], 1);
    row[c] = -1;
  }
  if (threadIdx.x == 0) {
    a.slots[s] = EvictSlot{s_start < n ? s_start : n, n};
    if (n < len) p.lens[s] = n;
  }
}

// One block of 16 tokens on its way: lane l = 16 g + n has 16-byte pieces of keys,
// the codes of its part of four values, and scale bytes of token n.
template <int D>
struct MovedBlock {
  static constexpr int kKeys = D == 256 ? 2 : 1, kScales = D == 256 ? 4 : 2, kPart = D / 32;
  u32x4_t k[kKeys];
  uint64_t v[4];      // kPart bytes each
  uint8_t s[kScales]; // keys', then values'

  static __device__ __forceinline__ int key_token(int lane, int i) { return (i * 64 + lane) / (D / 32); }
  static __device__ __forceinline__ bool key_lane(int lane) { return D >= 128 || lane < 32; }
  // byte among the scales of a block, its token being lane % 16
  static __device__ __forceinline__ int scale_at(int lane, int i) { return i * 64 + lane; }

  // from: where the block's tokens lie, `held` of them
  __device__ __forceinline__ void read(const uint8_t* base, const int64_t* from, int held, int lane) {
    auto place = [&](int t) { return t < held ? from[t] : -1; };
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      k[i] = u32x4_t{0u, 0u, 0u, 0u};
      const int64_t f = key_lane(lane) ? place(key_token(lane, i)) : -1;
      if (f >= 0)
        k[i] = *reinterpret_cast<const u32x4_t*>(base + (f & ~15) + (f & 15) * (D / 2) + (i * 64 + lane) % (D / 32) * 16);
    }
    const int part = lane & 15;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int64_t f = place(lane / 16 * 4 + t);
      v[t] = 0;
      if (f >= 0) {
        const uint8_t* at = base + (f & ~15) + 8 * D + (((f & 15) >> 2) * 16 + part) * (D / 8) + (f & 3) * kPart;
        if constexpr (D == 64) v[t] = *reinterpret_cast<const uint16_t*>(at);
        else if constexpr (D == 128) v[t] = *reinterpret_cast<const uint32_t*>(at);
        else v[t] = *reinterpret_cast<const uint64_t*>(at);
      }
    }
    const int64_t f = place(lane & 15);
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      const int b = scale_at(lane, i);
      s[i] = 0;
      if (f >= 0 && b < D) s[i] = base[(f & ~15) + 16 * D + b / 16 * 16 + (f & 15)];
    }
  }
  // tokens past `held` stay as they are
  __device__ __forceinline__ void write(uint8_t* block, int held, int lane) const {
#pragma unroll
    for (int i = 0; i < kKeys; ++i)
      if (key_lane(lane) && key_token(lane, i) < held) *reinterpret_cast<u32x4_t*>(block + (i * 64 + lane) * 16) = k[i];
    uint8_t* at = block + 8 * D + lane * (D / 8);
    const int mine = held - lane / 16 * 4;  // of the lane's four tokens
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (t < mine) {
        if constexpr (D == 64) *reinterpret_cast<uint16_t*>(at + t * kPart) = (uint16_t)v[t];
        else if constexpr (D == 128) *reinterpret_cast<uint32_t*>(at + t * kPart) = (uint32_t)v[t];
        else *reinterpret_cast<uint64_t*>(at + t * kPart) = v[t];
      }
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      const int b = scale_at(lane, i);
      if (b < D && (lane & 15) < held) block[16 * D + b] = s[i];
    }
  }
};

constexpr int kMoveWaves = 8, kMoveBlocks = 2;  // waves of a workgroup, blocks of a wave at a time

template <int D>
__global__ __launch_bounds__(64 * kMoveWaves) void k_evict_move(EvictArgs a, int64_t units) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const PagesArgs& p = a.p;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int head = (int)(u % a.heads);
    const int64_t rest = u / a.heads;
    const int layer = (int)(rest % p.layers), slot = (int)(rest / p.layers);
    const EvictSlot at = a.slots[slot];
    const int32_t* row = p.table + (int64_t)slot * p.ld_table;
    const int64_t* from = a.from + (int64_t)slot * a.most;
    const int per_head = (1 << p.page_shift) / kKvBlock;
    uint8_t* base = p.pool + layer * p.layer_stride + (int64_t)head * per_head * a.block_bytes;
    for (int first = at.start & ~(kKvBlock - 1); first < at.len; first += kMoveWaves * kMoveBlocks * kKvBlock) {
      MovedBlock<D> b[kMoveBlocks];
      const int mine = first + wave * kMoveBlocks * kKvBlock;
#pragma unroll
      for (int i = 0; i < kMoveBlocks; ++i) b[i].read(base, from + mine + i * kKvBlock, at.len - mine - i * kKvBlock, lane);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // read, in every wave, before any of it is written
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kMoveBlocks; ++i) {
        const int t = mine + i * kKvBlock;
        const int page = t < at.len ? row[t >> p.page_shift] : -1;
        if ((unsigned)page < (unsigned)p.n_pages)
          b[i].write(base + page * p.page_stride + ((t & ((1 << p.page_shift) - 1)) / kKvBlock) * a.block_bytes, at.len - t, lane);
      }
    }
  }
}

size_t pages_evict_scratch(int64_t n_slots, int64_t most) {
  if (n_slots * most > int64_t(1) << 56) return ~size_t(0);  // (more than there is)
  return (size_t)n_slots * sizeof(EvictSlot) + 255 + (size_t)n_slots * most * 8;
}

hipError_t launch_pages_evict(int d, int heads, int64_t most, const PagesArgs& p, const EvictCall& c, void* workspace,
                              hipStream_t s) {
  EvictArgs a{};
  a.p = p;
  a.c = c;
  a.heads = heads;
  a.block_bytes = 17 * d;
  a.most = (int)most;
  a.slots = static_cast<EvictSlot*>(workspace);
  a.from = reinterpret_cast<int64_t*>(static_cast<uint8_t*>(workspace) + ((size_t)p.n_slots * sizeof(EvictSlot) + 255) / 256 * 256);
  launch_kernel(k_evict_choose, dim3((unsigned)p.n_slots), dim3(kChoose), 0, s, a);
  const int64_t units = (int64_t)p.n_slots * p.layers * heads;
  const dim3 grid((unsigned)(units < (1 << 20) ? units : (1 << 20)));
  if (d == 64) launch_kernel(k_evict_move<64>, grid, dim3(64 * kMoveWaves), 0, s, a, units);
  else if (d == 128) launch_kernel(k_evict_move<128>, grid, dim3(64 * kMoveWaves), 0, s, a, units);
  else launch_kernel(k_evict_move<256>, grid, dim3(64 * kMoveWaves), 0, s, a, units);
  return hipGetLastError();
}

}  // namespace sph

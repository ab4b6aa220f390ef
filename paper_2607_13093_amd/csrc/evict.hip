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
//
// Moving is bound by memory: 64 slots of up to 4096 tokens in 16 layers, 2.2 GB read
// and written in 445 us, 5.0 TB/s, a copy's rate.  Where a quarter of the tokens stays,
// the lines that hold them are read nearly whole (a value's codes lie between those of
// three other tokens): 569 MB kept and written in 197 us.  Where slots, layers and heads are
// few a unit's chunks follow one another: half of 16384 tokens of one layer takes 116 us with
// one head and 125 with eight, 188 in 32 layers, choosing 27 of it (one workgroup's latency, 9
// for 700 tokens).
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
constexpr int kLook = 4;       // tokens of a thread that are numbered at a time
constexpr int kBins = 2048;    // of a digit of 11 bits; three digits are an order

// Sum over the threads before this one, and over all.  For kChoose threads.
__device__ __forceinline__ int threads_before(int x, int* all, int* s_wave) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int y = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int z = __shfl_up(y, o, 64);
    if (lane >= o) y += z;
  }
  if (lane == 63) s_wave[wave] = y;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int n = s_wave[k];
    if (k < wave) before += n;
    total += n;
  }
  *all = total;
  return before + y - x;
}

// The tokens of a slot.  KEPT: weights that a thread holds in registers, all of a slot
// of up to 1024 KEPT tokens; longer ones are read once more for each digit.
template <int KEPT>
__device__ __forceinline__ void choose_tokens(const EvictArgs& a, int len, int held) {
  __shared__ uint32_t s_bins[kBins];
  constexpr int kCounts = KEPT > 0 ? KEPT * 16 : 64;  // of 64 tokens each
  __shared__ int s_sure[kCounts], s_tie[kCounts], s_wave[16];
  __shared__ int s_shared, s_start, s_digit, s_need;
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const PagesArgs& p = a.p;
  int32_t* row = p.table + (int64_t)s * p.ld_table;
  const float* w = a.c.weights + s * a.c.ld_weights;
  float* w_out = a.c.weights_out + s * a.c.ld_out;
  int32_t* kept = a.c.kept ? a.c.kept + s * a.c.ld_kept : nullptr;
  int64_t* from = a.from + (int64_t)s * a.most;

  float mine[KEPT > 0 ? KEPT : 1];
#pragma unroll
  for (int i = 0; i < KEPT; ++i) {
    const int j = i * kChoose + threadIdx.x;
    mine[i] = j < len ? w[j] : 0.0f;
  }
  uint32_t order[KEPT > 0 ? KEPT : 1];
#pragma unroll
  for (int i = 0; i < KEPT; ++i) order[i] = order_of(mine[i]);
  const int want = a.c.keep[s];
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
  for (int i = threadIdx.x; i < kBins; i += kChoose) s_bins[i] = 0;
  __syncthreads();
  const int64_t fixed = (int64_t)s_shared << p.page_shift;
  const int front = fixed > a.c.first ? (fixed < len ? (int)fixed : len) : (a.c.first < len ? a.c.first : len);
  const int back = len - front > a.c.recent ? len - a.c.recent : front;
  const int must = front + len - back;
  const int n = want < must ? must : (want < len ? want : len);
  int need = n - must;  // of the tokens from front to back

  // the weight of the last that is kept, and how many of that weight are
  uint32_t least = 0;
  if (need > 0 && n < len) {
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {
      const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bits = digit == 2 ? 10 : 11;
      auto count = [&](int j, uint32_t o) {
        if (j >= front && j < back && (digit == 0 || (o ^ least) >> (shift + bits) == 0))
          atomicAdd(&s_bins[(o >> shift) & ((1 << bits) - 1)], 1u);
      };
      if constexpr (KEPT > 0) {
#pragma unroll
        for (int i = 0; i < KEPT; ++i)
          if (i * kChoose < back) count(i * kChoose + threadIdx.x, order[i]);
      } else {
        for (int j0 = front; j0 < back; j0 += 8 * kChoose) {
          float x[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int j = j0 + i * kChoose + threadIdx.x;
            x[i] = j < back ? w[j] : 0.0f;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) count(j0 + i * kChoose + threadIdx.x, order_of(x[i]));
        }
      }
      __syncthreads();
      // a thread's two digits, from the largest down
      const int top = kBins - 1 - 2 * threadIdx.x;
      const int t0 = s_bins[top], t1 = s_bins[top - 1];
      int all = 0;
      const int before = threads_before(t0 + t1, &all, s_wave);
      s_bins[top] = s_bins[top - 1] = 0;  // for the next
      if (before < need && need <= before + t0 + t1) {
        const bool first = need <= before + t0;
        s_digit = first ? top : top - 1;
        s_need = need - before - (first ? 0 : t0);
      }
      __syncthreads();
      least |= (uint32_t)s_digit << shift;
      need = s_need;
    }
  }

  // numbers of the kept ones, in order; equal weights are kept from the first on
  auto is_sure = [&](int j, uint32_t o) {
    return j < len && (n == len || j < front || j >= back || (need > 0 && o > least));
  };
  auto is_tie = [&](int j, uint32_t o) { return n < len && need > 0 && j >= front && j < back && o == least; };
  const uint64_t below = (uint64_t(1) << lane) - 1;
  int start = len;  // the first that goes
  // token j of weight x, with `sure` certain and `tie` equal ones before its 64
  auto give = [&](int j, float x, uint32_t o, int page, int sure_before, int tie_before) {
    const bool sure = is_sure(j, o), tie = is_tie(j, o);
    const uint64_t sures = __ballot(sure), ties = __ballot(tie);
    const int t = tie_before + __popcll(ties & below);
    const int to = sure_before + __popcll(sures & below) + (t < need ? t : need);
    if (sure || (tie && t < need)) {
      const int in_page = j & ((1 << p.page_shift) - 1);
      from[to] = (unsigned)page < (unsigned)p.n_pages
                     ? (page * p.page_stride + (in_page / kKvBlock) * a.block_bytes) | (in_page % kKvBlock)
                     : -1;
      w_out[to] = x;
      if (kept) kept[to] = j;
    } else if (j < start) {
      start = j;
    }
  };
  auto number_of = [&](const int* s_count, int* all) {  // this lane's sum of the counts before, in their order
    int x = s_count[lane];
    const int its = x;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o, 64);
      if (lane >= o) x += y;
    }
    *all = __builtin_amdgcn_readlane(x, 63);
    return x - its;
  };
  if constexpr (KEPT > 0) {
    int page[KEPT];
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
      const int j = i * kChoose + threadIdx.x;
      page[i] = j < len ? row[j >> p.page_shift] : -1;
    }
#pragma unroll
    for (int i = 0; i < KEPT; ++i) {
      const int j = i * kChoose + threadIdx.x;
      const uint64_t sures = __ballot(is_sure(j, order[i])), ties = __ballot(is_tie(j, order[i]));
      if (lane == 0) {
        s_sure[i * 16 + wave] = __popcll(sures);
        s_tie[i * 16 + wave] = __popcll(ties);
      }
    }
    __syncthreads();
    int sure_before = 0, tie_before = 0;
#pragma unroll
    for (int k = 0; k < KEPT / 4; ++k) {  // (64 counts are four turns of the 16 waves)
      int all_sure = 0, all_tie = 0;
      const int ns = number_of(s_sure + 64 * k, &all_sure), nt = number_of(s_tie + 64 * k, &all_tie);
#pragma unroll
      for (int i = 4 * k; i < 4 * k + 4; ++i) {
        const int at = i % 4 * 16 + wave;
        if (i * kChoose < len)
          give(i * kChoose + threadIdx.x, mine[i], order[i], page[i], sure_before + __builtin_amdgcn_readlane(ns, at),
               tie_before + __builtin_amdgcn_readlane(nt, at));
      }
      sure_before += all_sure;
      tie_before += all_tie;
    }
  } else {
    int sure_before = 0, tie_before = 0;
    for (int at = 0; at < len; at += kLook * kChoose) {
      float x[kLook];
      int page[kLook];
#pragma unroll
      for (int i = 0; i < kLook; ++i) {
        const int j = at + i * kChoose + threadIdx.x;
        x[i] = j < len ? w[j] : 0.0f;
        page[i] = j < len ? row[j >> p.page_shift] : -1;
      }
#pragma unroll
      for (int i = 0; i < kLook; ++i) {
        const int j = at + i * kChoose + threadIdx.x;
        const uint64_t sures = __ballot(is_sure(j, order_of(x[i]))), ties = __ballot(is_tie(j, order_of(x[i])));
        if (lane == 0) {
          s_sure[i * 16 + wave] = __popcll(sures);
          s_tie[i * 16 + wave] = __popcll(ties);
        }
      }
      __syncthreads();  // (these weights are read too, and may be written over)
      int all_sure = 0, all_tie = 0;
      const int ns = number_of(s_sure, &all_sure), nt = number_of(s_tie, &all_tie);
#pragma unroll
      for (int i = 0; i < kLook; ++i)
        give(at + i * kChoose + threadIdx.x, x[i], order_of(x[i]), page[i],
             sure_before + __builtin_amdgcn_readlane(ns, i * 16 + wave), tie_before + __builtin_amdgcn_readlane(nt, i * 16 + wave));
      sure_before += all_sure;
      tie_before += all_tie;
      __syncthreads();  // the counts are free
    }
  }
  if (start < len) atomicMin(&s_start, start);
  __syncthreads();  // the row and all weights are read
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

// (16384 tokens 72 us where weights were read again for each of four digits, and numbered
// 4096 at a time)
__global__ __launch_bounds__(kChoose) void k_evict_choose(EvictArgs a) {
  const PagesArgs& p = a.p;
  const int held_len = p.lens[blockIdx.x];
  const int len = held_len < 0 ? 0 : (held_len < a.most ? held_len : a.most);
  const int held = (len + (1 << p.page_shift) - 1) >> p.page_shift;
  if (len <= 4 * kChoose) choose_tokens<4>(a, len, held);
  else if (len <= 8 * kChoose) choose_tokens<8>(a, len, held);
  else if (len <= 16 * kChoose) choose_tokens<16>(a, len, held);
  else choose_tokens<0>(a, len, held);
}

// One block of 16 tokens on its way: lane l = 16 g + n has 16-byte pieces of keys,
// the codes of its part of four values, and scale bytes of token n.
template <int D>
struct MovedBlock {
  static constexpr int kKeys = D == 256 ? 2 : 1, kScales = D == 256 ? 4 : 2, kPart = D / 32;
  u32x4_t k[kKeys];
  typename std::conditional<D == 256, uint64_t, uint32_t>::type v[4];  // kPart bytes each
  uint32_t s[kScales];  // bytes: keys', then values'
  uint32_t none;        // pieces of tokens that are none: keys', four values', scales'

  static __device__ __forceinline__ int key_token(int lane, int i) { return (i * 64 + lane) / (D / 32); }
  static __device__ __forceinline__ bool key_lane(int lane) { return D >= 128 || lane < 32; }
  // byte among the scales of a block, its token being lane % 16
  static __device__ __forceinline__ int scale_at(int lane, int i) { return i * 64 + lane; }

  // where the block's tokens lie, `held` of them: of the lane's pieces of keys, its four
  // tokens' values and its scales' token; -1 for what is none
  struct Places {
    int64_t k[kKeys], v[4], s;
  };
  static __device__ __forceinline__ Places places(const int64_t* from, int held, int lane) {
    Places f;
    auto place = [&](int t) {
      const int64_t x = from[t < held ? t : 0];
      return t < held ? x : -1;
    };
#pragma unroll
    for (int i = 0; i < kKeys; ++i) f.k[i] = place(key_token(lane, i));
#pragma unroll
    for (int t = 0; t < 4; ++t) f.v[t] = place(lane / 16 * 4 + t);
    f.s = place(lane & 15);
    return f;
  }
  // (loads of every lane, from the first block where a token is none, so that nothing waits
  // for a branch)
  __device__ __forceinline__ void read(const uint8_t* base, const Places& f, int lane) {
    auto block = [&](int64_t x) { return base + (x < 0 ? 0 : x & ~int64_t(15)); };
    auto token = [&](int64_t x) { return (int)x & 15; };
    none = (f.s < 0 ? 64u : 0u);
#pragma unroll
    for (int i = 0; i < kKeys; ++i) none |= f.k[i] < 0 ? 1u << i : 0u;
#pragma unroll
    for (int t = 0; t < 4; ++t) none |= f.v[t] < 0 ? 4u << t : 0u;
#pragma unroll
    for (int i = 0; i < kKeys; ++i)
      k[i] = *reinterpret_cast<const u32x4_t*>(block(f.k[i]) + token(f.k[i]) * (D / 2) + (i * 64 + lane) % (D / 32) * 16);
    const int part = lane & 15;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint8_t* at = block(f.v[t]) + 8 * D + ((token(f.v[t]) >> 2) * 16 + part) * (D / 8) + (token(f.v[t]) & 3) * kPart;
      if constexpr (D == 64) v[t] = *reinterpret_cast<const uint16_t*>(at);
      else if constexpr (D == 128) v[t] = *reinterpret_cast<const uint32_t*>(at);
      else v[t] = *reinterpret_cast<const uint64_t*>(at);
    }
#pragma unroll
    for (int i = 0; i < kScales; ++i) s[i] = block(f.s)[16 * D + scale_at(lane, i) % D / 16 * 16 + token(f.s)];
  }
  // Waits for the loads; a token that is none is zeros.
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      asm volatile("" : "+v"(k[i]));
      if (none >> i & 1) k[i] = u32x4_t{0u, 0u, 0u, 0u};
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      asm volatile("" : "+v"(v[t]));
      if (none >> (2 + t) & 1) v[t] = 0;
    }
#pragma unroll
    for (int i = 0; i < kScales; ++i) {
      asm volatile("" : "+v"(s[i]));
      if (none >> 6 & 1) s[i] = 0;
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
      if (b < D && (lane & 15) < held) block[16 * D + b] = (uint8_t)s[i];
    }
  }
};

// Waves of a workgroup, a block of tokens each at a time: two where there are many
// workgroups, which leaves more of them room (8192 units of 64 dimensions: 2.2 GB in 442 us,
// 5.0 TB/s, 482 with eight waves), eight where few have to take a slot's tokens faster
// (1024 units of 128 dimensions 43 -> 38 us; 43 again with sixteen).  Two blocks a wave cost registers and
// starts: 527 us.
constexpr int64_t kManyUnits = 4096;

template <int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_evict_move(EvictArgs a, int64_t units) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const PagesArgs& p = a.p;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int head = (int)(u % a.heads);
    const int64_t rest = u / a.heads;
    const int layer = (int)(rest % p.layers), slot = (int)(rest / p.layers);
    const EvictSlot at = a.slots[slot];
    // (read as constants, by scalar loads, which the vector loads on their way do not hold up)
    const auto* row = (const __attribute__((address_space(4))) int32_t*)(p.table + (int64_t)slot * p.ld_table);
    const int64_t* from = a.from + (int64_t)slot * a.most;
    const int per_head = (1 << p.page_shift) / kKvBlock;
    uint8_t* base = p.pool + layer * p.layer_stride + (int64_t)head * per_head * a.block_bytes;
    // A chunk's places are asked for two chunks ahead, its tokens one ahead.
    constexpr int CHUNK = WAVES * kKvBlock;
    using Block = MovedBlock<D>;
    struct Chunk {
      Block b;
      typename Block::Places f;
    };
    if (at.start >= at.len) continue;
    auto ask = [&](int t, Chunk& x) { x.f = Block::places(from + (t < at.len ? t : 0), at.len - t, lane); };
    auto move = [&](int t, Chunk& now, Chunk& next) {
      // (asked for before: loads end in their order)
      ask(t + 2 * CHUNK, now);
      next.b.read(base, next.f, lane);
      now.b.arrive();
      __syncthreads();  // read, in every wave, before any of it is written
      const int page = t < at.len ? row[t >> p.page_shift] : -1;
      if ((unsigned)page < (unsigned)p.n_pages)
        now.b.write(base + page * p.page_stride + ((t & ((1 << p.page_shift) - 1)) / kKvBlock) * a.block_bytes, at.len - t, lane);
    };
    const int first = at.start & ~(kKvBlock - 1), mine = wave * kKvBlock;
    Chunk x, y;
    ask(first + mine, x);
    ask(first + mine + CHUNK, y);
    x.b.read(base, x.f, lane);
    for (int t0 = first; t0 < at.len; t0 += 2 * CHUNK) {
      move(t0 + mine, x, y);
      if (t0 + CHUNK < at.len) move(t0 + mine + CHUNK, y, x);
    }
    __syncthreads();  // (the next unit's tokens are other bytes, but its waves may not run ahead of these)
  }
}

template <int D>
void launch_move(const EvictArgs& a, int64_t units, hipStream_t s) {
  const dim3 grid((unsigned)(units < (1 << 20) ? units : (1 << 20)));
  if (units >= kManyUnits) launch_kernel(k_evict_move<D, 2>, grid, dim3(128), 0, s, a, units);
  else launch_kernel(k_evict_move<D, 8>, grid, dim3(512), 0, s, a, units);
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
  if (d == 64) launch_move<64>(a, units, s);
  else if (d == 128) launch_move<128>(a, units, s);
  else launch_move<256>(a, units, s);
  return hipGetLastError();
}

}  // namespace sph

// Upkeep of a page pool: growing, trimming, forking, copying and compacting.
//
// A page is free when its count of references is zero; there is no list of
// free pages.  What is handed out are the lowest free pages, to sessions in
// their order, so that the same calls give the same tables on every run; all
// counts are integers, whose atomic sums do not depend on their order.
//
// Tables and counts are a few hundred kilobytes: these calls are bound by launches
// and by dependent loads (growth 7.9 us of one workgroup for 256 sessions and 65536
// pages).  Copies of pages run at a copy's rate: 1.14 GB moved in 499 us, 4.6 TB/s in
// and out; 248 shared last pages in 32 layers 106 us.
#include "kv_cache.h"

namespace sph {

constexpr int kChunkPages = 4096;              // pages a workgroup looks at: 64 words of 64
constexpr int kChunkWords = kChunkPages / 64;

__device__ __forceinline__ int pages_up(int n, int shift) { return (int)(((int64_t)n + (1 << shift) - 1) >> shift); }

// Words of 64 pages, a bit for each with (want_free) no reference or a
// reference, and their number, by 1024 threads.
__device__ __forceinline__ void chunk_bits(const int32_t* refs, int n_pages, int chunk, bool want_free,
                                           uint64_t* words, int32_t* counts) {
  __shared__ int s_n;
  if (threadIdx.x == 0) s_n = 0;
  __syncthreads();
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < kChunkPages / 1024; ++i) {
    const int w = i * 16 + wave;
    const int64_t p = (int64_t)chunk * kChunkPages + w * 64 + lane;
    const bool in = p < n_pages;
    const int r = in ? refs[p] : 0;
    const uint64_t m = __ballot(in && (want_free ? r <= 0 : r > 0));
    if (lane == 0) {
      words[(int64_t)chunk * kChunkWords + w] = m;
      atomicAdd(&s_n, __popcll(m));
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) counts[chunk] = s_n;
}

// Sums of counts[0 .. chunk) and of all, by a workgroup.
__device__ __forceinline__ void chunk_base(const int32_t* counts, int chunks, int chunk, int* before, int* all) {
  __shared__ int s_before, s_all;
  if (threadIdx.x == 0) s_before = s_all = 0;
  __syncthreads();
  int b = 0, t = 0;
  for (int i = threadIdx.x; i < chunks; i += blockDim.x) {
    const int c = counts[i];
    t += c;
    if (i < chunk) b += c;
  }
  if (b) atomicAdd(&s_before, b);
  if (t) atomicAdd(&s_all, t);
  __syncthreads();
  *before = s_before;
  *all = s_all;
  __syncthreads();
}

// Exclusive sums of the 64 words' counts of a chunk into s_rank[0 .. 64], by one
// wave; ends with a barrier of the workgroup.
__device__ __forceinline__ void word_ranks(const uint64_t* words, int base, int* s_rank) {
  if (threadIdx.x < 64) {
    int n = __popcll(words[threadIdx.x]), x = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(x, o, 64);
      if ((int)threadIdx.x >= o) x += y;
    }
    s_rank[threadIdx.x] = base + x - n;
  }
  __syncthreads();
}

// ---- growing -------------------------------------------------------------

struct GrowScratch {
  uint64_t* words;     // free pages
  int32_t* counts;     // of each chunk
  int32_t* first;      // [slots + 1]: ranks of the pages that a session gets
  int32_t* pair;       // [slots]: the session's copied page among the pairs, or -1
  int32_t* src;        // [slots]
  int32_t* dst;
  int32_t* head;       // pairs, sessions with too short a row
};

// Sums of pages stop at 2^31 - 1, more than any pool has free.
__device__ __forceinline__ uint32_t add_pages(uint32_t a, uint32_t b) {
  return a + b < 0x7FFFFFFFu ? a + b : 0x7FFFFFFFu;
}

// What the sessions need, with the state as it was before the call, by 1024
// threads: first[s], the pages of the sessions before s, and the shared pages that
// are to be copied, in pairs pair[s].
__device__ __forceinline__ void grow_needs(const PagesArgs& a, const int32_t* add, const GrowScratch& w, int32_t* first) {
  __shared__ uint32_t s_need[16];
  __shared__ int s_pair[16], s_short;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) s_short = 0;
  uint32_t need0 = 0;
  int pair0 = 0;
  __syncthreads();
  for (int at = 0; at < a.n_slots; at += 1024) {
    const int s = at + threadIdx.x;
    uint32_t need = 0;
    int source = -1;
    if (s < a.n_slots) {
      const int64_t len = a.lens[s] > 0 ? a.lens[s] : 0, more = add[s] > 0 ? add[s] : 0;
      const int64_t page = int64_t(1) << a.page_shift;
      const int64_t have = (len + page - 1) >> a.page_shift, want = (len + more + page - 1) >> a.page_shift;
      if (want > a.max_pages || len + more > kKvMost) {
        atomicAdd(&s_short, 1);
      } else {
        need = (uint32_t)(want - have);
        if (more > 0 && (len & (page - 1))) {  // a page partly filled: is it another's too?
          const int p = a.table[(int64_t)s * a.ld_table + (len >> a.page_shift)];
          if ((unsigned)p < (unsigned)a.n_pages && a.refs[p] > 1) source = p;
        }
        need += source >= 0;
      }
    }
    uint32_t x = need;
    int y = source >= 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t u = (uint32_t)__shfl_up((int)x, o, 64);
      const int v = __shfl_up(y, o, 64);
      if (lane >= o) x = add_pages(x, u), y += v;
    }
    if (lane == 63) s_need[wave] = x, s_pair[wave] = y;
    __syncthreads();
    uint32_t before = need0, all = 0;
    int pairs = pair0, all_pairs = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i < wave) before = add_pages(before, s_need[i]), pairs += s_pair[i];
      all = add_pages(all, s_need[i]);
      all_pairs += s_pair[i];
    }
    if (s < a.n_slots) {
      first[s] = (int)(before + x - need);  // (of no use where a sum stopped: no page is given out then)
      const int k = pairs + y - 1;
      w.pair[s] = source >= 0 ? k : -1;
      if (source >= 0) w.src[k] = source;
    }
    need0 = add_pages(need0, all);
    pair0 += all_pairs;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    first[a.n_slots] = (int)need0;
    w.head[0] = pair0;
    w.head[1] = s_short;
  }
}

// Session that gets the free page of rank k: first[s] <= k < first[s + 1].
__device__ __forceinline__ int session_of(const int32_t* first, int n, int k) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= k) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Page `page` is the k-th that session s gets.  (lens as before the call)
__device__ __forceinline__ void give_page(const PagesArgs& a, const GrowScratch& w, int s, int k, int page) {
  int col = pages_up(a.lens[s] > 0 ? a.lens[s] : 0, a.page_shift) + k;
  const int pair = w.pair[s];
  if (pair >= 0) {
    col -= 1;  // the shared page's place is the first
    if (k == 0) w.dst[pair] = page;
  }
  a.table[(int64_t)s * a.ld_table + col] = page;
  a.refs[page] = 1;
}

// Sizes and decisions: workgroups of chunks look for free pages, one more adds up
// what the sessions need.
__global__ __launch_bounds__(1024) void k_grow_plan(PagesArgs a, const int32_t* add, GrowScratch w, int chunks) {
  if ((int)blockIdx.x < chunks) chunk_bits(a.refs, a.n_pages, blockIdx.x, true, w.words, w.counts);
  else grow_needs(a, add, w, w.first);
}

// Free page of rank k goes to the session whose share of the ranks holds k.
__global__ __launch_bounds__(256) void k_grow_apply(PagesArgs a, const int32_t* add, GrowScratch w, int chunks,
                                                    int32_t* status) {
  __shared__ int s_rank[kChunkWords];
  int before, all;
  chunk_base(w.counts, chunks, blockIdx.x, &before, &all);
  const int total = w.first[a.n_slots], too_short = w.head[1];
  const bool fits = total <= all && too_short == 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    status[0] = total > all ? total - all : 0;
    status[1] = too_short;
  }
  if (!fits) return;
  for (int s = blockIdx.x * 256 + threadIdx.x; s < a.n_slots; s += gridDim.x * 256) {
    if (w.pair[s] >= 0) atomicSub(&a.refs[w.src[w.pair[s]]], 1);
  }
  if (before < total) {
    word_ranks(w.words + (int64_t)blockIdx.x * kChunkWords, before, s_rank);
    const int lane = threadIdx.x & 63;
    for (int i = threadIdx.x >> 6; i < kChunkWords; i += 4) {
      const uint64_t m = w.words[(int64_t)blockIdx.x * kChunkWords + i];
      const int rank = s_rank[i] + __popcll(m & ((uint64_t(1) << lane) - 1));
      if (!((m >> lane) & 1) || rank >= total) continue;
      const int s = session_of(w.first, a.n_slots, rank);
      give_page(a, w, s, rank - w.first[s], blockIdx.x * kChunkPages + i * 64 + lane);
    }
  }
}

// All of that by one workgroup, for pools and tables that fit its LDS: it looks at
// pages from the lowest on until there are enough free ones, which a pool that is
// not nearly full has among its first.  (One launch less, 3.7 us of the host's time:
// 256 sessions giving back and taking 8 rows in 65536 pages 18.3 -> 14.8 us.)
constexpr int kOnePages = 131072, kOneSlots = 4096;
__global__ __launch_bounds__(1024) void k_grow_one(PagesArgs a, const int32_t* add, GrowScratch w, int32_t* status) {
  constexpr int kWords = kOnePages / 64, kLook = 16;  // words of 64 pages; pages a thread looks at in a turn
  __shared__ uint64_t s_words[kWords];
  __shared__ int s_rank[kWords], s_first[kOneSlots + 1], s_wave[16], s_found;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (threadIdx.x == 0) s_found = 0;
  int r[kLook];
  auto look = [&](int words) {
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      const int64_t p = (int64_t)words * 64 + i * 1024 + threadIdx.x;
      r[i] = p < a.n_pages ? a.refs[p] : 1;
    }
  };
  look(0);  // on their way while the needs are added up
  grow_needs(a, add, w, s_first);
  __syncthreads();
  const int total = s_first[a.n_slots], too_short = w.head[1];
  int words = 0;  // looked at
  while (s_found < total && words * 64 < a.n_pages) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kLook; ++i) {
      const uint64_t m = __ballot(r[i] <= 0);
      if (lane == 0 && words + i * 16 + wave < kWords) s_words[words + i * 16 + wave] = m;
      n += __popcll(m);
    }
    __syncthreads();  // (s_found was read)
    if (lane == 0) atomicAdd(&s_found, n);
    words += kLook * 16;
    __syncthreads();
    if (s_found < total && words * 64 < a.n_pages) look(words);
  }
  const int found = s_found;
  if (threadIdx.x == 0) {
    status[0] = total > found ? total - found : 0;
    status[1] = too_short;
    if (total > found || too_short) w.head[0] = 0;  // nothing to copy
  }
  if (total > found || too_short) return;
  words = words < kWords ? words : kWords;
  // free pages before each word: two words a thread
  const int at = threadIdx.x * 2;
  const int n0 = at < words ? __popcll(s_words[at]) : 0, n1 = at + 1 < words ? __popcll(s_words[at + 1]) : 0;
  int x = n0 + n1;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  if (lane == 63) s_wave[wave] = x;
  __syncthreads();
  for (int i = 0; i < wave; ++i) x += s_wave[i];
  if (at < kWords) {
    s_rank[at] = x - n0 - n1;
    s_rank[at + 1] = x - n1;
  }
  for (int s = threadIdx.x; s < a.n_slots; s += 1024)
    if (w.pair[s] >= 0) atomicSub(&a.refs[w.src[w.pair[s]]], 1);
  __syncthreads();
  for (int k = threadIdx.x; k < total; k += 1024) {
    int lo = 0, hi = words;  // the last word with rank <= k
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_rank[mid] <= k) lo = mid;
      else hi = mid;
    }
    uint64_t m = s_words[lo];
    for (int i = k - s_rank[lo]; i > 0; --i) m &= m - 1;
    const int s = session_of(s_first, a.n_slots, k);
    give_page(a, w, s, k - s_first[s], lo * 64 + __ffsll((unsigned long long)m) - 1);
  }
  __syncthreads();
  for (int s = threadIdx.x; s < a.n_slots; s += 1024) {
    if (add[s] > 0) a.lens[s] = (a.lens[s] > 0 ? a.lens[s] : 0) + add[s];
  }
}

constexpr int kPiece = 16384;  // bytes that a workgroup copies at a time

__device__ __forceinline__ void copy_pieces(const PagesArgs& a, const int32_t* src, const int32_t* dst,
                                            int64_t pairs, int block, int blocks) {
  const int pieces = (int)((a.page_bytes + kPiece - 1) / kPiece);
  const int64_t items = pairs * a.layers * pieces;
  for (int64_t it = block; it < items; it += blocks) {
    const int piece = (int)(it % pieces);
    const int64_t rest = it / pieces;
    const int64_t layer = rest % a.layers, k = rest / a.layers;
    const int s = src[k], d = dst[k];
    if ((unsigned)s >= (unsigned)a.n_pages || (unsigned)d >= (unsigned)a.n_pages || s == d) continue;
    const uint8_t* from = a.pool + layer * a.layer_stride + s * a.page_stride;
    uint8_t* to = a.pool + layer * a.layer_stride + d * a.page_stride;
    u32x4_t v[kPiece / 4096];
#pragma unroll
    for (int i = 0; i < kPiece / 4096; ++i) {
      const int64_t at = (int64_t)piece * kPiece + i * 4096 + threadIdx.x * 16;
      if (at < a.page_bytes) v[i] = *reinterpret_cast<const u32x4_t*>(from + at);
    }
#pragma unroll
    for (int i = 0; i < kPiece / 4096; ++i) {
      const int64_t at = (int64_t)piece * kPiece + i * 4096 + threadIdx.x * 16;
      if (at < a.page_bytes) *reinterpret_cast<u32x4_t*>(to + at) = v[i];
    }
  }
}

// Lengths last, the workgroups before read them; then the shared pages' copies.
__global__ __launch_bounds__(256) void k_grow_finish(PagesArgs a, const int32_t* add, GrowScratch w,
                                                     const int32_t* status) {
  if (status[0] != 0 || status[1] != 0) return;
  for (int s = blockIdx.x * 256 + threadIdx.x; s < a.n_slots; s += gridDim.x * 256)
    if (add[s] > 0) a.lens[s] = (a.lens[s] > 0 ? a.lens[s] : 0) + add[s];
  copy_pieces(a, w.src, w.dst, w.head[0], blockIdx.x, gridDim.x);
}
__global__ __launch_bounds__(256) void k_grow_copy(PagesArgs a, GrowScratch w) {
  copy_pieces(a, w.src, w.dst, w.head[0], blockIdx.x, gridDim.x);
}

__global__ __launch_bounds__(256) void k_pages_copy(PagesArgs a, const int32_t* src, const int32_t* dst, int64_t n) {
  copy_pieces(a, src, dst, n, blockIdx.x, gridDim.x);
}

// ---- trimming and forking -------------------------------------------------

__device__ __forceinline__ void release(const PagesArgs& a, int32_t* row, int from, int to) {
  for (int c = from + threadIdx.x; c < to; c += blockDim.x) {
    const int p = row[c];
    if ((unsigned)p < (unsigned)a.n_pages) atomicSub(&a.refs[p], 1);
    row[c] = -1;
  }
}

__device__ __forceinline__ int held_pages(const PagesArgs& a, int len) {
  const int n = pages_up(len > 0 ? len : 0, a.page_shift);
  return n < a.max_pages ? n : a.max_pages;
}

__global__ __launch_bounds__(64) void k_pages_trim(PagesArgs a, const int32_t* kept) {
  const int s = blockIdx.x;
  const int len = a.lens[s], keep = kept[s] > 0 ? kept[s] : 0;
  if (len <= keep) return;
  release(a, a.table + (int64_t)s * a.ld_table, held_pages(a, keep), held_pages(a, len));
  __syncthreads();
  if (threadIdx.x == 0) a.lens[s] = keep;
}

// A child gives back what it holds and takes its parent's row.
__global__ __launch_bounds__(256) void k_pages_fork(PagesArgs a, const int32_t* parents, const int32_t* children) {
  const int p = parents[blockIdx.x], c = children[blockIdx.x];
  if ((unsigned)p >= (unsigned)a.n_slots || (unsigned)c >= (unsigned)a.n_slots || p == c) return;
  const int len = a.lens[p], mine = a.lens[c];
  int32_t* row = a.table + (int64_t)c * a.ld_table;
  const int32_t* from = a.table + (int64_t)p * a.ld_table;
  const int held = held_pages(a, len);
  release(a, row, 0, held_pages(a, mine));
  __syncthreads();
  for (int i = threadIdx.x; i < a.max_pages; i += 256) {
    const int page = i < held ? from[i] : -1;
    if ((unsigned)page < (unsigned)a.n_pages) atomicAdd(&a.refs[page], 1);
    row[i] = page;
  }
  __syncthreads();
  if (threadIdx.x == 0) a.lens[c] = len;
}

// ---- compacting -------------------------------------------------------------

struct CompactScratch {
  uint64_t* words;   // live pages
  int32_t* counts;
  int32_t* ranks;    // live pages before each word
  int32_t* holes;    // free pages below the number of live ones, ascending
  int32_t* movers;   // live pages from there on, ascending
  int32_t* refs;     // the movers' counts
};

__global__ __launch_bounds__(1024) void k_compact_plan(PagesArgs a, CompactScratch w) {
  chunk_bits(a.refs, a.n_pages, blockIdx.x, false, w.words, w.counts);
}

// Live pages before page p, by the words of its chunk (ranks not needed).
__device__ __forceinline__ int live_before(const CompactScratch& w, int p, int* s_x) {
  const int chunk = p / kChunkPages;
  int n = 0;
  for (int i = threadIdx.x; i < chunk; i += blockDim.x) n += w.counts[i];
  const int word = (p % kChunkPages) / 64;
  for (int i = threadIdx.x; i <= word; i += blockDim.x) {
    uint64_t m = w.words[(int64_t)chunk * kChunkWords + i];
    if (i == word) m &= (uint64_t(1) << (p & 63)) - 1;
    n += __popcll(m);
  }
  if (threadIdx.x == 0) *s_x = 0;
  __syncthreads();
  if (n) atomicAdd(s_x, n);
  __syncthreads();
  return *s_x;
}

__global__ __launch_bounds__(256) void k_compact_lists(PagesArgs a, CompactScratch w, int chunks, int32_t* refs_out,
                                                       int32_t* live_out) {
  __shared__ int s_rank[kChunkWords], s_x;
  int before, live;
  chunk_base(w.counts, chunks, blockIdx.x, &before, &live);
  // live pages below the first `live` places stay; live == n_pages: all do
  const int stay = live < a.n_pages ? live_before(w, live, &s_x) : live;
  word_ranks(w.words + (int64_t)blockIdx.x * kChunkWords, before, s_rank);
  if (blockIdx.x == 0 && threadIdx.x == 0) *live_out = live;
  const int lane = threadIdx.x & 63;
  for (int i = threadIdx.x >> 6; i < kChunkWords; i += 4) {
    const int64_t word = (int64_t)blockIdx.x * kChunkWords + i;
    if (lane == 0) w.ranks[word] = s_rank[i];
    const uint64_t m = w.words[word];
    const int64_t page = word * 64 + lane;
    if (page >= a.n_pages) continue;
    const bool is_live = (m >> lane) & 1;
    const int rank = s_rank[i] + __popcll(m & ((uint64_t(1) << lane) - 1));
    const int r = is_live ? a.refs[page] : 0;
    if (page >= live) {
      if (is_live) {
        w.movers[rank - stay] = (int)page;
        w.refs[rank - stay] = r;
      }
      refs_out[page] = 0;
    } else if (is_live) {
      refs_out[page] = r;
    } else {
      w.holes[page - rank] = (int)page;
    }
  }
}

__global__ __launch_bounds__(256) void k_compact_move(PagesArgs a, CompactScratch w, int32_t* table_out,
                                                      int64_t ld_out, int32_t* refs_out, const int32_t* live_out) {
  __shared__ int s_x;
  const int live = *live_out;
  const int stay = live < a.n_pages ? live_before(w, live, &s_x) : live;
  const int movers = live - stay;
  const int64_t entries = (int64_t)a.n_slots * a.max_pages, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < movers; i += step) refs_out[w.holes[i]] = w.refs[i];
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += step) {
    const int64_t s = i / a.max_pages, c = i - s * a.max_pages;
    int p = a.table[s * a.ld_table + c];
    if (p >= live && p < a.n_pages) {
      const uint64_t m = w.words[p / 64];
      if ((m >> (p & 63)) & 1)
        p = w.holes[w.ranks[p / 64] + __popcll(m & ((uint64_t(1) << (p & 63)) - 1)) - stay];
    }
    table_out[s * ld_out + c] = p;
  }
  copy_pieces(a, w.movers, w.holes, movers, blockIdx.x, gridDim.x);
}

// ---- host -------------------------------------------------------------------

namespace {

struct Carve {  // pieces of a workspace, 256-byte aligned
  uint8_t* p;
  size_t n = 0;
  template <class T>
  T* take(size_t count) {
    T* r = reinterpret_cast<T*>(p + n);
    n += (count * sizeof(T) + 255) / 256 * 256;
    return r;
  }
};

int chunks_of(int64_t n_pages) { return (int)((n_pages + kChunkPages - 1) / kChunkPages); }

GrowScratch grow_scratch(Carve& c, int64_t n_pages, int64_t n_slots) {
  const size_t k = (size_t)chunks_of(n_pages);
  GrowScratch w;
  w.words = c.take<uint64_t>(k * kChunkWords);
  w.counts = c.take<int32_t>(k);
  w.first = c.take<int32_t>((size_t)n_slots + 1);
  w.pair = c.take<int32_t>((size_t)n_slots);
  w.src = c.take<int32_t>((size_t)n_slots);
  w.dst = c.take<int32_t>((size_t)n_slots);
  w.head = c.take<int32_t>(2);
  return w;
}

CompactScratch compact_scratch(Carve& c, int64_t n_pages) {
  const size_t k = (size_t)chunks_of(n_pages);
  CompactScratch w;
  w.words = c.take<uint64_t>(k * kChunkWords);
  w.counts = c.take<int32_t>(k);
  w.ranks = c.take<int32_t>(k * kChunkWords);
  w.holes = c.take<int32_t>((size_t)n_pages);
  w.movers = c.take<int32_t>((size_t)n_pages);
  w.refs = c.take<int32_t>((size_t)n_pages);
  return w;
}

// Workgroups of a launch that copies up to `pairs` pages: no more than the chip
// holds at a time, each goes on to the next piece.
unsigned copy_blocks(const PagesArgs& a, int64_t pairs) {
  const double n = (double)pairs * a.layers * ((a.page_bytes + kPiece - 1) / kPiece);
  return (unsigned)(n < 1 ? 1 : (n > 2048 ? 2048 : n));
}

}  // namespace

size_t pages_grow_scratch(int64_t n_pages, int64_t n_slots) {
  Carve c{nullptr};
  grow_scratch(c, n_pages, n_slots);
  return c.n;
}
size_t pages_compact_scratch(int64_t n_pages) {
  Carve c{nullptr};
  compact_scratch(c, n_pages);
  return c.n;
}

hipError_t launch_pages_grow(const PagesArgs& a, const int32_t* add, int32_t* status, void* workspace, hipStream_t s) {
  Carve c{static_cast<uint8_t*>(workspace)};
  const GrowScratch w = grow_scratch(c, a.n_pages, a.n_slots);
  if (a.n_pages <= kOnePages && a.n_slots <= kOneSlots) {
    launch_kernel(k_grow_one, dim3(1), dim3(1024), 0, s, a, add, w, status);
    launch_kernel(k_grow_copy, dim3(copy_blocks(a, a.n_slots)), dim3(256), 0, s, a, w);
    return hipGetLastError();
  }
  const int chunks = chunks_of(a.n_pages);
  launch_kernel(k_grow_plan, dim3(chunks + 1), dim3(1024), 0, s, a, add, w, chunks);
  launch_kernel(k_grow_apply, dim3(chunks), dim3(256), 0, s, a, add, w, chunks, status);
  launch_kernel(k_grow_finish, dim3(copy_blocks(a, a.n_slots)), dim3(256), 0, s, a, add, w,
                (const int32_t*)status);
  return hipGetLastError();
}

hipError_t launch_pages_trim(const PagesArgs& a, const int32_t* kept, hipStream_t s) {
  if (a.n_slots <= 0) return hipSuccess;
  launch_kernel(k_pages_trim, dim3(a.n_slots), dim3(64), 0, s, a, kept);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesArgs& a, const int32_t* parents, const int32_t* children, int n, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  launch_kernel(k_pages_fork, dim3(n), dim3(256), 0, s, a, parents, children);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const PagesArgs& a, const int32_t* src, const int32_t* dst, int64_t n, hipStream_t s) {
  if (n <= 0) return hipSuccess;
  launch_kernel(k_pages_copy, dim3(copy_blocks(a, n)), dim3(256), 0, s, a, src, dst, n);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PagesArgs& a, int32_t* table_out, int64_t ld_out, int32_t* refs_out,
                                int32_t* live_out, void* workspace, hipStream_t s) {
  Carve c{static_cast<uint8_t*>(workspace)};
  const CompactScratch w = compact_scratch(c, a.n_pages);
  const int chunks = chunks_of(a.n_pages);
  launch_kernel(k_compact_plan, dim3(chunks), dim3(1024), 0, s, a, w);
  launch_kernel(k_compact_lists, dim3(chunks), dim3(256), 0, s, a, w, chunks, refs_out, live_out);
  launch_kernel(k_compact_move, dim3(copy_blocks(a, a.n_pages)), dim3(256), 0, s, a, w, table_out, ld_out, refs_out,
                (const int32_t*)live_out);
  return hipGetLastError();
}

}  // namespace sph

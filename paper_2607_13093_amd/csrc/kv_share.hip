// Attention of sessions that hold pages in common: what sessions' rows of the table
// name alike from the start on is read once for all of them.
//
// A plan, made on the device from the tables, cuts the sessions' tokens into
// segments: ranges that a set of sessions holds on the same pages, and what each session
// holds alone.  Sessions are sorted by their rows of the table, a level at a time: those
// of a group whose next page is the same form a group of the next level, and share
// what they all name alike from there on.  So every row is the rows' end of a path of
// segments, some levels long, and its softmax the join of its segments' parts:
//   l_k = sum_j exp2(x_j - t_k),  o_k = sum_j exp2(x_j - t_k) V_j   over segment k
//   out = sum_k exp2(t_k - t) o_k / sum_k exp2(t_k - t) l_k,  t = max_k t_k
// Long segments are cut into shares of their tokens, which are parts too.
//
// The parts are computed as in kv_attend.hip, by workgroups that go over a list of
// items, a share of a segment for a tile of the rows of all its sessions each: many
// rows on a shared segment, so that its codes are converted once for 64 rows, few on
// a session's own.  One launch takes both kinds, the shared first, from a queue, so
// that what own tokens wait for memory hides behind the products of shared ones; a second
// joins the parts.
//
// 16 windows of five rows on one document of 65504 tokens: 129 us (0.67 PFLOP/s; the
// plain call, which reads and converts the document 16 times, 185): vector instructions
// 47% of the clocks, matrix cores 28%, one after the other, CUs busy 86%.  256 windows of
// eight rows behind one prompt of 4096: 501 us, 57% and 35%, bound by issue; the plain
// call, whose tiles of 64 rows are as full, 448.  The plan takes 16 us for two sessions and
// 30 for 256, once for all layers.  Most calls are faster by the plain call: beside a plan
// that is there already, 40 of 45 (15 of them share nothing: 1.4 times as long at the
// median, 2.0 at most): every row's parts go out in fp32 and come back for the join, and
// few rows run at the occupancy of many.
#include "kv_tile.h"

namespace sph {

constexpr int kShareLevels = 3;             // segments of a path that are shared, at most
constexpr int kShareLooks = kShareLevels + 2;  // groups of groups that are looked at
constexpr int kShareStep = 128;   // tokens that shares are multiples of
constexpr int kShareLeast = 256;  // and at least
// Tokens whose reading a segment has to save: a part of every row costs about as much.
constexpr int kShareWorth = 256;
// us of an item beside its tokens and outputs, where another hides the rest.  This and the
// other constants of the account of time are fitted: with them its choice of a length is
// within 3% of the best of the sixteen that it tries (one row of 32 sessions on 2037 tokens,
// five of 16 on 65504, eight of 256 on 4096, a tree of six times eight sessions).
constexpr double kShareItem = 4.0;
constexpr int64_t kShareRoom = int64_t(1) << 30;  // bytes of all rows' parts, where two of each fit

// Tokens from ... to - 1 of `members` sessions from place `first` of the order.
struct ShareSeg {
  int32_t first, members, from, to;
};

// A session of the order: its rows at positions base ..., its row of the table.
struct SharePlace {
  int32_t session, slot, base, rows;
};

// An item: tile `tile` of the rows of such sessions over such tokens, on the pages of
// row `slot`, which holds `len` of them; place `part` of each row's parts.
struct ShareItem {
  int32_t first, members, tile, from, to, part;
  int32_t flags;  // 1: no other tile reads the tokens, 2: a tile of few rows
  int32_t slot;
};

struct ShareHead {
  uint32_t key;   // of the sizes that the plan is for
  int32_t items;
  int32_t next;   // the next item that a workgroup takes, zero between calls
  int32_t shared; // segments that several sessions hold
};

// Sizes of a plan, from a call's.
struct ShareSizes {
  int levels, parts;  // segments of a path that are shared at most, parts of a row
  int extra;          // parts beyond one for each segment of a path
  int mt[2], wt;      // row tiles of a wave on segments of many rows and of few (own ones), waves that share them
  int rows[2];        // of a tile of an item
  int slots;          // workgroups that run at a time
  float us[2];        // of one of them for a token of an item
  float item_us[2];   // and for an item, its outputs' way out and back with it
  float read_us;      // for a token's way from memory, all workgroups at it
  int cap;            // items at most
};

struct SharePlanArgs {
  KvArgs kv;
  ShareSizes z;
  int group, window;
  uint32_t key;
  ShareHead* head;
  SharePlace* order; // [S]: sessions, those of a segment side by side
  int32_t* parts;    // [S]: parts of a session's rows
  ShareItem* items;  // [cap]
};

constexpr int kPlanThreads = 1024;

// Sum of x over the threads before this one; all: over all.  For 1024 threads.
__device__ __forceinline__ int sum_before(int x, int* all) {
  __shared__ int s_wave[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int y = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int z = __shfl_up(y, o, 64);
    if (lane >= o) y += z;
  }
  __syncthreads();  // (a call before this one is read)
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

// Keys in ascending order, no two alike, n a power of two.  Up to 256 each is counted
// into its place by four threads, one step; more are merged in log2(n)^2 / 2.
__device__ __forceinline__ void sort_keys(uint64_t* key, int n) {
  __syncthreads();
  if (n <= kPlanThreads / 4) {
    const int i = threadIdx.x >> 2, quarter = threadIdx.x & 3;
    const uint64_t mine = i < n ? key[i] : 0;
    int below = 0;
    if (i < n) {
#pragma unroll 8
      for (int k = 2 * quarter; k < n; k += 8) {
        typedef uint64_t u64x2_t __attribute__((ext_vector_type(2)));
        const u64x2_t two = *reinterpret_cast<const u64x2_t*>(key + k);
        below += (two[0] < mine) + (two[1] < mine);
      }
    }
    below += __shfl_xor(below, 1, 64);
    below += __shfl_xor(below, 2, 64);
    __syncthreads();
    if (i < n && quarter == 0) key[below] = mine;
    __syncthreads();
    return;
  }
  for (int size = 2; size <= n; size <<= 1)
    for (int gap = size >> 1; gap > 0; gap >>= 1) {
      __syncthreads();
      for (int i = threadIdx.x; i < n / 2; i += kPlanThreads) {
        const int lo = i / gap * (2 * gap) + i % gap, hi = lo + gap;
        const uint64_t a = key[lo], b = key[hi];
        if ((a > b) == ((lo & size) == 0)) {
          key[lo] = b;
          key[hi] = a;
        }
      }
    }
  __syncthreads();
}

// The rows of the table of a level's groups, in LDS but for the table.
struct Alike {
  const uint64_t* key;
  const int32_t *slot, *depth;
  int32_t* alike;
  const uint16_t *group, *first;
  const int32_t* table;
  int64_t ld_table;
  int max_pages;
};

// Each session's row against its group's first from the place after `depth` on, up to
// alike[group], which is lowered to the first place where they differ.  A wave takes M
// sessions at a time, 256 COLS places of each, four a lane, so that their loads are on their
// way together.  (Places from `c` on are compared, those before are alike.)
template <int M, int COLS>
__device__ __forceinline__ void compare_rows(const Alike& a, int S) {
  typedef int32_t places_t __attribute__((ext_vector_type(4), aligned(4)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  for (int at0 = wave; at0 < S; at0 += 16 * M) {
    // lane m looks up session m
    const int at = at0 + 16 * lane;
    const bool in = lane < M && at < S;
    const int group = a.group[in ? at : at0], lead = a.first[group];
    const int64_t row_x = a.slot[(int)(a.key[lead] & 4095)] * a.ld_table, row_y = a.slot[(int)(a.key[in ? at : at0] & 4095)] * a.ld_table;
    const int begin = in && at != lead ? a.depth[at] + 1 : kKvMost;
    uint32_t open = (uint32_t)__ballot(in && at != lead);
    int c = begin;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const int z = __shfl_xor(c, o, 64);
      c = z < c ? z : c;
    }
    c = __builtin_amdgcn_readfirstlane(c);
    const int32_t *x[M], *y[M];
    auto of_lane = [](int64_t v, int m) {
      return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), m) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane((int)v, m));
    };
#pragma unroll
    for (int m = 0; m < M; ++m) {
      x[m] = a.table + of_lane(row_x, m);
      y[m] = a.table + of_lane(row_y, m);
    }
    while (open) {
      places_t p[M][COLS], q[M][COLS];
      int col[COLS];  // the last places of a row again for those past it
#pragma unroll
      for (int i = 0; i < COLS; ++i) {
        const int64_t to = (int64_t)c + i * 256 + lane * 4;
        col[i] = to < a.max_pages - 4 ? (int)to : a.max_pages - 4;
      }
      const int ends = *(volatile const int32_t*)&a.alike[group];  // at most a row's places
      int end[M];
#pragma unroll
      for (int m = 0; m < M; ++m) {
        end[m] = open >> m & 1 ? __builtin_amdgcn_readlane(ends, m) : 0;
#pragma unroll
        for (int i = 0; i < COLS; ++i)
          if (c + i * 256 < end[m]) {
            p[m][i] = *reinterpret_cast<const places_t*>(x[m] + col[i]);
            q[m][i] = *reinterpret_cast<const places_t*>(y[m] + col[i]);
          }
      }
#pragma unroll
      for (int m = 0; m < M; ++m) {
        int differs = kKvMost;
#pragma unroll
        for (int i = COLS - 1; i >= 0; --i)
          if (c + i * 256 < end[m]) {
            const places_t d = p[m][i] ^ q[m][i];
            const uint64_t others = __ballot((d[0] | d[1] | d[2] | d[3]) != 0);
            if (others) {
              const int mine = col[i] + (d[0] ? 0 : d[1] ? 1 : d[2] ? 2 : 3);
              differs = __builtin_amdgcn_readlane(mine, __builtin_ctzll(others));
            }
          }
        // (one lane: 64 atomics on one place take 64 turns, 45 us for 196 sessions)
        if (differs != kKvMost && lane == 0) atomicMin(&a.alike[__builtin_amdgcn_readlane(group, m)], differs);
        if (differs != kKvMost || c + COLS * 256 >= end[m]) open &= ~(1u << m);
      }
      c += COLS * 256;
    }
  }
}
// The same where rows have fewer than four places: a session a thread.
__device__ __forceinline__ void compare_short_rows(const Alike& a, int S) {
  for (int at = threadIdx.x; at < S; at += kPlanThreads) {
    const int group = a.group[at];
    const int32_t *x = a.table + a.slot[(int)(a.key[a.first[group]] & 4095)] * a.ld_table, *y = a.table + a.slot[(int)(a.key[at] & 4095)] * a.ld_table;
#pragma nounroll
    for (int c = a.depth[at] + 1; c < a.max_pages; ++c)
      if (x[c] != y[c]) {
        atomicMin(&a.alike[group], c);
        break;
      }
  }
}

// 50 bytes a session, and as many segments as two sessions each can have
constexpr int plan_lds(int n2) { return 50 * n2 + 16 + kShareLevels * n2 / 2 * (int)sizeof(ShareSeg); }
static_assert(plan_lds(kShareSessions) + 1024 <= 160 * 1024, "LDS of a plan");

__global__ __launch_bounds__(kPlanThreads, 4) void k_share_plan(SharePlanArgs a, int n2) {
  extern __shared__ __align__(16) uint8_t smem[];
  ShareSeg* segs = reinterpret_cast<ShareSeg*>(smem);          // [3 n2 / 2] those that several sessions hold
  uint64_t* key = reinterpret_cast<uint64_t*>(segs + kShareLevels * n2 / 2);  // [n2] by place: group, page, session
  int32_t* limit = reinterpret_cast<int32_t*>(key + n2);       // [n2] by session: pages that may be shared
  int32_t* slot = limit + n2;                                  // by session: its row of the table
  int32_t* base = slot + n2;                                   // by session: position of its first row
  int32_t* length = base + n2;                                 // by session
  int32_t* page0 = length + n2;                                // by session: its first page; later parts and items before a segment's
  int32_t* depth = page0 + n2;                                 // by place: pages that its group names alike
  int32_t* start = depth + n2;                                 // by place: those in segments
  int32_t* alike = start + n2;                                 // by group: pages named alike
  int32_t* low = alike + n2;                                   // by group: least position of a first row
  uint16_t* count = reinterpret_cast<uint16_t*>(low + n2);     // by place: parts so far
  uint16_t* group = count + n2;                                // by place
  uint16_t* first = group + n2;                                // [n2 + 1] by group: its first place
  __shared__ int s_segs, s_longest, s_ends[kShareLooks];  // segments up to the end of each level
  __shared__ float s_us[16];
  const int S = a.kv.n_sessions, shift = a.kv.page_shift, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto row_of = [&](int at) { return a.kv.table + (int64_t)slot[(int)(key[at] & 4095)] * a.kv.ld_table; };

  if (threadIdx.x == 0) s_segs = s_longest = 0;
  __syncthreads();
  int longest = 0;
  for (int s = threadIdx.x; s < n2; s += kPlanThreads) {
    int n = 0, at = 0, b = 0, p0 = -1, len = 0;
    if (s < S) {
      const int mine = a.kv.slots ? a.kv.slots[s] : s;
      at = (unsigned)mine < (unsigned)a.kv.n_slots ? mine : 0;
      p0 = a.kv.table[at * a.kv.ld_table];  // (beside the lengths)
      const KvSession ses = kv_session(a.kv, s);
      len = ses.len;
      b = ses.len - ses.rows;
      n = b > 0 ? b : 0;  // all its rows see those
      longest = ses.len > longest ? ses.len : longest;
    }
    limit[s] = n >> shift;
    slot[s] = at;
    base[s] = b;
    length[s] = len;
    page0[s] = p0;
    depth[s] = start[s] = count[s] = 0;
    group[s] = 0;
    key[s] = s < S ? (uint64_t)s : ~uint64_t(0);
  }
  if (longest > 0) atomicMax(&s_longest, longest);
  __syncthreads();
  longest = s_longest;

  const int RG = a.kv.R * a.group, row_shift[2] = {__ffs(a.z.rows[0]) - 1, __ffs(a.z.rows[1]) - 1};
  auto kind_of = [&](int members) { return members == 1 || members * RG <= a.z.rows[1]; };  // 1: few rows
  auto tiles_of = [&](int members, int kind) { return (int)(((uint32_t)members * RG + a.z.rows[kind] - 1) >> row_shift[kind]); };
  // Whether tokens are read once for tiles of all members' rows, with a part more for each of
  // them, or beside each session's own: shared unless this account has it take twice as long.
  // (16 tokens that 32 sessions of eight rows and 4931 tokens hold in common, four layers:
  // shared 248 us, left to the sessions 202.  With 1, 1.5 or 3 for the factor calls took as long
  // as with two.  The account leaves out what the parts cost the join and the sessions' own
  // items: of 30 calls with a segment, sharing none at all was more than 3% faster in 11, most
  // where the common part is short or rows are few (53.6 -> 41.8 us), and slower in 9 (344 -> 546).)
  auto worth = [&](int members, int tokens) {
    const int kind = kind_of(members);
    const float n = (float)tokens, shared = (float)tiles_of(members, kind) * (n * a.z.us[kind] + a.z.item_us[kind]) + n * a.z.read_us;
    return shared < 2.0f * n * (float)members * ((float)tiles_of(1, 1) * a.z.us[1] + a.z.read_us);
  };

  // (loops that are not unrolled: run once, code costs its way from memory)
  int groups = 1, levels = 0;
#pragma nounroll
  for (int level = 0; level < kShareLooks && S > 1; ++level) {
    for (int at = threadIdx.x; at < S; at += kPlanThreads) {
      const int s = (int)(key[at] & 4095), d = depth[at];
      const int page = d >= limit[s] ? -1 : level == 0 ? page0[s] : row_of(at)[d];
      const bool valid = (unsigned)page < (unsigned)a.kv.n_pages;
      key[at] = (uint64_t)group[at] << 44 | (valid ? (uint64_t)page << 12 : uint64_t(1) << 43 | (uint64_t)s << 12) | (uint64_t)s;
    }
    sort_keys(key, n2);
    // groups of the level: places whose keys are alike but for the session
    const int each = (n2 + kPlanThreads - 1) / kPlanThreads, mine = threadIdx.x * each;
    int starts = 0;
    for (int i = mine; i < mine + each && i < S; ++i) starts += i == 0 || key[i] >> 12 != key[i - 1] >> 12;
    int id = sum_before(starts, &groups);
    if (groups == S) break;  // no two alike
    for (int i = mine; i < mine + each && i < S; ++i) {
      if (i == 0 || key[i] >> 12 != key[i - 1] >> 12) first[id++] = (uint16_t)i;
      group[i] = (uint16_t)(id - 1);
    }
    if (threadIdx.x == 0) first[groups] = (uint16_t)S;
    for (int g = threadIdx.x; g < groups; g += kPlanThreads) alike[g] = low[g] = kKvMost;
    __syncthreads();
    for (int at = threadIdx.x; at < S; at += kPlanThreads) {
      const int s = (int)(key[at] & 4095);
      atomicMin(&alike[group[at]], limit[s]);
      if (a.window > 0) atomicMin(&low[group[at]], base[s]);
    }
    __syncthreads();
    // pages named alike by a group's first session and each of the others
    const Alike all{key, slot, depth, alike, group, first, a.kv.table, a.kv.ld_table, a.kv.max_pages};
    if (a.kv.max_pages < 4) compare_short_rows(all, S);
    else if (S <= 16) compare_rows<1, 4>(all, S);
    else if (S <= 64) compare_rows<4, 2>(all, S);
    else compare_rows<8, 1>(all, S);
    __syncthreads();
    // segments of the level, in the order of their groups
    const int before = s_segs;
    int made = 0;
    for (int g0 = 0; g0 < groups; g0 += kPlanThreads) {
      const int g = g0 + threadIdx.x;
      bool take = false;
      int from = 0, to = 0, members = 0;
      if (g < groups) {
        members = first[g + 1] - first[g];
        from = start[first[g]] << shift;
        to = alike[g] << shift;
        take = members > 1 && count[first[g]] < a.z.levels && (int64_t)(to - from) * (members - 1) >= kShareWorth &&
               worth(members, to - from);
      }
      int all = 0;
      const int at = sum_before(take ? 1 : 0, &all);
      if (take) {
        int seen = from;
        if (a.window > 0) {
          const int64_t lowest = (int64_t)low[g] - a.window + 1;
          if (lowest > seen) seen = lowest < to ? (int)lowest & ~(kKvBlock - 1) : to;
        }
        segs[before + made + at] = ShareSeg{first[g], members, seen, to};
      }
      if (g < groups) low[g] = take;
      made += all;
    }
    __syncthreads();
    for (int at = threadIdx.x; at < S; at += kPlanThreads) {
      const int g = group[at];
      if (first[g + 1] - first[g] == 1) limit[(int)(key[at] & 4095)] = 0;  // nothing further
      else depth[at] = alike[g];
      // (what is not worth a segment of its own is left to those of smaller groups)
      if (low[g]) {
        start[at] = alike[g];
        ++count[at];
      }
    }
    if (threadIdx.x == 0) s_segs = s_ends[level] = before + made;
    levels = level + 1;
    __syncthreads();
  }
  const int shared = s_segs;
  // What sessions hold alone, the longest first.
  for (int at = threadIdx.x; at < S; at += kPlanThreads) {
    const int s = (int)(key[at] & 4095);
    int from = start[at] << shift;
    count[at] = 0;
    if (a.window > 0) {
      const int64_t lowest = (int64_t)base[s] - a.window + 1;
      if (lowest > from) from = (int)lowest & ~(kKvBlock - 1);
    }
    alike[at] = from;
    low[at] = length[s] > from ? length[s] : from;
    a.order[at] = SharePlace{s, slot[s], base[s], length[s] - base[s]};
    limit[at] = s;
  }
  __syncthreads();
  for (int at = threadIdx.x; at < n2; at += kPlanThreads)
    key[at] = at < S ? (uint64_t)(uint32_t)(kKvMost - (low[at] - alike[at])) << 12 | (uint64_t)at : ~uint64_t(0);
  sort_keys(key, n2);

  // Shares: each wave tries a length, in time, and what all items then take, an item's own
  // time with their tokens'.
  const int room = a.z.extra > 0 ? (longest + a.z.extra - 1) / a.z.extra : longest;
  auto chunk_of = [&](int kind, int candidate) {
    const float us = __builtin_amdgcn_exp2f(2.0f + 0.42f * candidate);  // 4 ... 315
    const float c = us / a.z.us[kind];
    int n = c < (float)longest ? (int)c : longest;
    n = n > room ? n : room;
    n = n > kShareLeast ? n : kShareLeast;
    return (n + kShareStep - 1) / kShareStep * kShareStep;
  };
  {
    const float heads = (float)a.kv.heads / (float)a.z.slots;
    float load = 0.0f, longest_us = 0.0f;
    const int chunk[2] = {chunk_of(0, wave), chunk_of(1, wave)};
#pragma nounroll
    for (int own = 0; own < 2; ++own) {
      const int n = own ? S : shared;
      float us = 0.0f, items = 0.0f, most = 0.0f;
      for (int i = lane; i < n; i += 64) {
        const ShareSeg t = own ? ShareSeg{i, 1, alike[i], low[i]} : segs[i];
        const int kind = kind_of(t.members), c = chunk[kind], its = t.to - t.from;
        const float k = (float)tiles_of(t.members, kind), shares = (float)((uint32_t)(its + c - 1) / (uint32_t)c);
        us += k * ((float)its * a.z.us[kind] + shares * a.z.item_us[kind]);
        items += k * shares;
        most = fmaxf(most, (float)(its < c ? its : c) * a.z.us[kind] + a.z.item_us[kind]);
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        us += __shfl_xor(us, o, 64);
        items += __shfl_xor(items, o, 64);
        most = fmaxf(most, __shfl_xor(most, o, 64));
      }
      load += us * heads;
      // Rounds of items: a last one that is not full has CUs with one workgroup, which is
      // done sooner.
      const float rounds = items * heads, full = floorf(rounds);
      const float last = rounds > full ? 0.4f + 0.65f * (rounds - full) : 0.0f;
      longest_us = fmaxf(longest_us, most * (full + last));
    }
    if (lane == 0) s_us[wave] = fmaxf(load, longest_us);
  }
  __syncthreads();
  int best = 0;
#pragma unroll
  for (int k = 1; k < 16; ++k) best = s_us[k] < s_us[best] ? k : best;
  const int chunk[2] = {chunk_of(0, best), chunk_of(1, best)};

  // Parts of each segment, level by level along the paths, and the items, one a
  // thread, which looks for its segment in the sums of them.
  int32_t *before = page0, *part_of = base;  // of up to n2 segments
  int made = 0;
#pragma nounroll
  for (int level = 0; level <= levels; ++level) {
    const bool own = level == levels;
    const int lo = own || level == 0 ? 0 : s_ends[level - 1], hi = own ? S : s_ends[level];
    auto segment = [&](int i) {
      if (!own) return segs[i];
      const int at = (int)(key[i] & 4095);
      return ShareSeg{at, 1, alike[at], low[at]};
    };
    int sum = 0;
    for (int i0 = lo; i0 < hi; i0 += kPlanThreads) {
      const int i = i0 + threadIdx.x;
      int n = 0, shares = 0, all = 0;
      ShareSeg t{0, 0, 0, 0};
      if (i < hi) {
        t = segment(i);
        const int kind = kind_of(t.members);
        const uint32_t c = chunk[kind];
        shares = (uint32_t)(t.to - t.from + c - 1) / c;
        n = tiles_of(t.members, kind) * shares;
        part_of[i - lo] = count[t.first];
      }
      const int at = sum + sum_before(n, &all);
      if (i < hi) before[i - lo] = at;
      sum += all;
      if (own) {
        if (i < hi) count[t.first] = (uint16_t)(count[t.first] + shares);
      } else {  // (a segment's members by a wave)
        const int mine = hi - i0 - wave * 64 < 64 ? hi - i0 - wave * 64 : 64;
        for (int k = 0; k < mine; ++k) {
          const int from = __builtin_amdgcn_readlane(t.first, k), m = __builtin_amdgcn_readlane(t.members, k);
          const int more_parts = __builtin_amdgcn_readlane(shares, k);
          for (int x = lane; x < m; x += 64) count[from + x] = (uint16_t)(count[from + x] + more_parts);
        }
      }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < sum; x += kPlanThreads) {
      int i = 0, past = hi - lo;  // the last segment with before <= x (one without items has the next one's)
      while (past - i > 1) {
        const int mid = (i + past) >> 1;
        if (before[mid] <= x) i = mid;
        else past = mid;
      }
      const ShareSeg t = segment(lo + i);
      const int kind = kind_of(t.members);
      const uint32_t c = chunk[kind], nt = tiles_of(t.members, kind), rest = x - before[i];
      const uint32_t share = rest / nt, tile = rest - share * nt;
      const int64_t to = (int64_t)t.from + (int64_t)(share + 1) * c;
      if (made + x < a.z.cap)
        a.items[made + x] = ShareItem{t.first, t.members, (int)tile, (int)(t.from + share * c), to < t.to ? (int)to : t.to,
                                      (int)(part_of[i] + share), (nt == 1 ? 1 : 0) | (kind ? 2 : 0), slot[limit[t.first]]};
    }
    made += sum;
    __syncthreads();
  }
  for (int at = threadIdx.x; at < S; at += kPlanThreads) a.parts[limit[at]] = count[at];
  if (threadIdx.x == 0) *a.head = ShareHead{a.key, made, 0, shared};
}

// Division by a number that is the same for all: by its reciprocal, one short at most.
struct Divisor {
  uint32_t d, r;
};
inline Divisor divisor_of(uint32_t d) { return Divisor{d, d == 1 ? 0xFFFFFFFFu : (uint32_t)((uint64_t(1) << 32) / d)}; }
__device__ __forceinline__ uint32_t divide(uint32_t n, const Divisor& d, uint32_t* rest) {
  uint32_t q = __umulhi(n, d.r), x = n - q * d.d;
  if (x >= d.d) {
    x -= d.d;
    ++q;
  }
  *rest = x;
  return q;
}

struct ShareArgs {
  KvArgs kv;
  const uint16_t* q;
  int64_t q_row, q_head;
  uint16_t* out;
  int64_t o_row, o_head;
  float* lse;
  int group, window;
  Divisor of_rows, of_group;  // by the rows of a session and head, and by group
  float scale_log2, binade;
  bool q_aligned, o_aligned;
  uint32_t key;
  ShareHead* head;
  const SharePlace* order;
  const int32_t* n_parts;
  const ShareItem* items;
  int cap;
  int parts;        // places of a row
  float2* part_ml;  // [rows x heads][parts]: reference of the weights, their sum
  float* part_o;    // [rows x heads][parts][D]
};

// A row of an item: number fq of its sessions' rows.
struct ShareRow {
  int session, r, in_group;  // in_group: query head of the key/value head's
  bool is, live;             // live: it is one of the session's rows
  int pos;
};
__device__ __forceinline__ ShareRow share_row(const ShareArgs& a, const ShareItem& it, int fq) {
  ShareRow w;
  uint32_t x, in;
  const int member = (int)divide((uint32_t)fq, a.of_rows, &x);
  w.r = (int)divide(x, a.of_group, &in);
  w.in_group = (int)in;
  const int at = it.first + member;
  w.is = member < it.members && (unsigned)at < (unsigned)a.kv.n_sessions;
  const SharePlace p = a.order[w.is ? at : 0];
  w.is = w.is && (unsigned)p.session < (unsigned)a.kv.n_sessions;
  w.session = w.is ? p.session : 0;
  w.live = w.is && w.r < p.rows;
  w.pos = p.base + w.r;
  return w;
}

// The parts of an item's rows for one key/value head.
template <int D, int MT, int WT>
__device__ __forceinline__ void share_item(const ShareArgs& a, const ShareItem& it, int head, uint8_t* smem) {
  constexpr int NS = stages_of(D, WT);
  constexpr int NW = waves_in(WT);
  constexpr int WR = NW / WT;
  constexpr int KJ = D / 32;   // steps of the first product
  constexpr int VC = D / 16;   // products of the second
  constexpr bool QL = queries_in_lds(D, MT);
  const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wt = wave % WT, wr = wave / WT;
  const int G = a.group;
  // of each row: its place among all parts (-1: none), whether it is one of its session's
  __shared__ int s_row[WR * MT * 16][2];
  {
    // pages of a row of the table; all of its tokens up to it.to are held
    KvSession ses;
    ses.table = a.kv.table + ((unsigned)it.slot < (unsigned)a.kv.n_slots ? it.slot : 0) * a.kv.ld_table;
    const int row0 = (it.tile * WR + wr) * 16 * MT;  // the wave's first

    // Without a window the first tiles are known before the rows are: they come while
    // those are looked up.  (The rows may see fewer of them: waits are for the newest.)
    constexpr int STEP = 32 * WT;
    int from = it.from > 0 ? it.from & ~(kKvBlock - 1) : 0;
    uint8_t* ring = smem + wave * (NS * Stage<D>::kBytes);
    uint32_t lane16 = lane * 16;
    const bool alone = WT >= 4 && (it.flags & 1);
    uint32_t none = 0;  // of the tiles in flight, the next in the low bits: blocks without a page
    auto none_of = [](const KvPages& p) { return (uint32_t)(p.page[0] < 0) | ((uint32_t)(p.page[1] < 0) << 1); };
    if (a.window == 0) {
#pragma unroll
      for (int i = 0; i < NS - 1; ++i) {
        const int at = from + 32 * wt + i * STEP;
        if (at < it.to) {
          const KvPages pages = tile_pages(a.kv, ses, at, it.to);
          none |= none_of(pages) << (2 * i);
          copy_tile<D>(ring + i * Stage<D>::kBytes, a.kv, head, at, pages, lane16, lane, alone);
        }
      }
    }

    u32x4_t* s_q = reinterpret_cast<u32x4_t*>(smem + NW * NS * Stage<D>::kBytes);
    Queries<D, MT, QL> q;
    q.l = s_q;
    q.own = wr * (MT * KJ * 64) + lane;
    int pos[MT];
    int low = kKvMost, high = -1;  // of the rows that are
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const ShareRow w = share_row(a, it, row0 + m * 16 + n);
      const bool live = w.live;
      if (g == 0 && wt == 0) {
        s_row[(wr * MT + m) * 16 + n][0] = w.is ? (w.session * a.kv.R + w.r) * (a.kv.heads * G) + head * G + w.in_group : -1;
        s_row[(wr * MT + m) * 16 + n][1] = live;
      }
      pos[m] = live ? w.pos : -1;
      if (live) {
        low = w.pos < low ? w.pos : low;
        high = w.pos > high ? w.pos : high;
      }
      const uint16_t* p = a.q + ((int64_t)w.session * a.kv.R + w.r) * a.q_row + (int64_t)(head * G + w.in_group) * a.q_head + g * (D / 4);
#pragma unroll
      for (int j = 0; j < KJ; ++j) {
        u32x4_t x{0u, 0u, 0u, 0u};
        // (waves that share rows share the work of it)
        if (live && (!QL || j % WT == wt)) {
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
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const int x = __shfl_xor(low, o, 64), y = __shfl_xor(high, o, 64);
      low = x < low ? x : low;
      high = y > high ? y : high;
    }
    low = __builtin_amdgcn_readfirstlane(low);
    high = __builtin_amdgcn_readfirstlane(high);
    const int to = it.to < high + 1 ? it.to : high + 1;
    int all_lo = 0;
    const int all_hi = low < 0 ? 0 : low + 1;
    if (a.window > 0) {
      const int64_t first = (int64_t)low - a.window + 1;
      if (first > from) from = (int)first & ~(kKvBlock - 1);
      all_lo = high - a.window + 1;
    }

    Rows<D, MT> w;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      w.top[m] = kNoScore;
      w.sum[m] = 0.0f;
#pragma unroll
      for (int c = 0; c < VC; ++c) w.o[m][c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // The wave's tiles as in kv_attend.hip: those that all its rows see whole first.
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

    const uint32_t ring_at = (uint32_t)(uintptr_t)(lds_void_t*)ring;
    // the lane's places in a stage: keys token n of a block, values as they lie
    const uint32_t key_at = n * (D / 2) + g * (D / 8), value_at = KvLayout<D>::kValues + lane * (D / 8);
    const uint32_t ks_at = Stage<D>::kCodes + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g) * kKvBlock + n;
    const uint32_t vs_at = Stage<D>::kCodes + D / 2 + n * D / 512 * kKvBlock + 4 * g;
    if (a.window > 0) {
#pragma unroll
      for (int i = 0; i < NS - 1; ++i)
        if (i < n_tiles) {
          const KvPages pages = tile_pages(a.kv, ses, place(i), to);
          none |= none_of(pages) << (2 * i);
          copy_tile<D>(ring + i * Stage<D>::kBytes, a.kv, head, place(i), pages, lane16, lane, alone);
        }
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
      if (t0 + 32 > it.to) {
        const int held[2] = {it.to - t0, it.to - t0 - kKvBlock};
        clear_values(values, held, g);
      }
      take_values(w, values, p);
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) w.sum[m] = sum_over_groups(w.sum[m]);

    // the waves' outputs, in what were rings
    constexpr int VP = VC / WT;  // of its D/16 columns of outputs, those that a wave ends with
    f32x4_t* s_o = reinterpret_cast<f32x4_t*>(smem);   // [NW][VC][64 lanes]
    float* s_ml = reinterpret_cast<float*>(smem) + NW * 16 * D;
    wait_copies<0>();  // tiles that no row saw
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
      for (int c = 0; c < VC; ++c) s_o[(wave * VC + c) * 64 + lane] = w.o[m][c] * f;
      __syncthreads();
      f32x4_t y[VP];
#pragma unroll
      for (int i = 0; i < VP; ++i) {
        y[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < WT; ++k) y[i] += s_o[((wr * WT + k) * VC + wt * VP + i) * 64 + lane];
      }
      const int row = s_row[(wr * MT + m) * 16 + n][0];
      if (row >= 0 && (unsigned)it.part < (unsigned)a.parts) {
        if (!s_row[(wr * MT + m) * 16 + n][1]) l = 0.0f;
        const int64_t at = (int64_t)row * a.parts + it.part;
        if (g == 0 && wt == 0) a.part_ml[at] = make_float2(t, l);
        if (!(l == 0.0f)) {
#pragma unroll
          for (int i = 0; i < VP; ++i)
            *reinterpret_cast<f32x4_t*>(a.part_o + at * D + ((g * VC) + wt * VP + i) * 4) = y[i];
        }
      }
    }
  }
}

constexpr int share_lds(int d, int mt, int own_mt, int wt) {
  return attend_lds(d, mt, wt) > attend_lds(d, own_mt, wt) ? attend_lds(d, mt, wt) : attend_lds(d, own_mt, wt);
}
constexpr int share_waves(int d, int mt, int wt) { return waves_of(d, mt, wt) < 2 ? waves_of(d, mt, wt) : 2; }
constexpr int share_resident(int d, int mt, int own_mt, int wt) {  // workgroups of a CU
  const int by_lds = 160 * 1024 / share_lds(d, mt, own_mt, wt), by_waves = share_waves(d, mt, wt) * 4 / waves_in(wt);
  return by_lds < by_waves ? by_lds : by_waves;
}

// Workgroups take an item and head at a time, in the order of the list: the shared
// segments' first, bound by the matrix cores and the softmax, beside which the sessions'
// own tokens come from memory, the longest first.  MT, OWN: row tiles of a wave on
// either.
template <int D, int MT, int OWN, int WT>
__global__ __launch_bounds__(64 * waves_in(WT), share_waves(D, MT, WT)) void k_share_parts(ShareArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];  // rings, then queries of each group of rows
  __shared__ int s_next;
  if (a.head->key != a.key) return;
  const int items = a.head->items < a.cap ? a.head->items : a.cap;
  const int units = items * a.kv.heads;
  int unit = blockIdx.x;
  while (unit < units) {
    if (threadIdx.x == 0) s_next = gridDim.x + atomicAdd(&a.head->next, 1);
    const int head = unit % a.kv.heads;
    const auto* x8 = (const __attribute__((address_space(4))) int32_t*)(a.items + unit / a.kv.heads);
    const ShareItem it{x8[0], x8[1], x8[2], x8[3], x8[4], x8[5], x8[6], x8[7]};
    if (OWN == MT || !(it.flags & 2)) share_item<D, MT, WT>(a, it, head, smem);
    else share_item<D, OWN, WT>(a, it, head, smem);
    __syncthreads();  // the outputs in LDS are read, the next unit is known
    unit = __builtin_amdgcn_readfirstlane(s_next);
    __syncthreads();
  }
}

// A row's parts joined, in their order, by D/16 lanes a row and head.  Parts hold
// outputs in the order of the lanes that made them: value ((4 g + e) D/16 + c) of a row at
// (g D/16 + c) 4 + e; a lane takes four c of one g.
// TURNS groups of lanes take the parts of a row in turns.
template <int D, int TURNS>
__global__ __launch_bounds__(256) void k_share_join(ShareArgs a, int64_t rows) {
  constexpr int LPS = D / 16, PER = 256 / LPS / TURNS;  // rows of a workgroup
  __shared__ float s_l[256 / LPS], s_top[256 / LPS];
  __shared__ f32x4_t s_y[TURNS > 1 ? 4 * 256 : 1];
  const int lane = threadIdx.x % LPS, turn = threadIdx.x / LPS % TURNS;
  const int64_t want = (int64_t)blockIdx.x * PER + threadIdx.x / (LPS * TURNS);
  const int64_t i = want < rows ? want : rows - 1;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.head->next = 0;  // for the next call
  const int heads = a.kv.heads * a.group;
  const int64_t row = i / heads;
  const int hq = (int)(i - row * heads);
  const int session = (int)(row / a.kv.R);
  const bool planned = a.head->key == a.key;
  int n = planned ? a.n_parts[session] : 0;
  n = n < a.parts ? n : a.parts;
  const float2* ml = a.part_ml + i * a.parts;
  const float* part = a.part_o + i * a.parts * D + lane * 16;
  float top = kNoScore, l = planned ? 0.0f : NAN;
  f32x4_t y[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) y[c] = f32x4_t{l, l, l, l};
  for (int k0 = turn; k0 < n; k0 += 2 * TURNS) {
    float2 x[2];
    f32x4_t o[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k = k0 + u * TURNS;
      x[u] = k < n ? ml[k] : make_float2(kNoScore, 0.0f);
      // parts without a token left their place unwritten: read, not used
      if (k < n) {
#pragma unroll
        for (int c = 0; c < 4; ++c) o[u][c] = *reinterpret_cast<const f32x4_t*>(part + (int64_t)k * D + 4 * c);
      }
    }
    const float t = fmaxf(fmaxf(top, x[0].x), x[1].x);
    const float f = __builtin_amdgcn_exp2f(top - t);
    l *= f;
#pragma unroll
    for (int c = 0; c < 4; ++c) y[c] *= f;
    top = t;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (x[u].y == 0.0f) continue;
      const float e = __builtin_amdgcn_exp2f(x[u].x - top);
      l += x[u].y * e;
#pragma unroll
      for (int c = 0; c < 4; ++c) y[c] += o[u][c] * e;
    }
  }
  if constexpr (TURNS > 1) {
    const int group = threadIdx.x / LPS;
    if (lane == 0) {
      s_l[group] = l;
      s_top[group] = top;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) s_y[c * 256 + threadIdx.x] = y[c];
    __syncthreads();
    if (turn != 0) return;
    float t = top;
#pragma unroll
    for (int k = 1; k < TURNS; ++k) t = fmaxf(t, s_top[group + k]);
    l = 0.0f;
#pragma unroll
    for (int c = 0; c < 4; ++c) y[c] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < TURNS; ++k) {
      const float e = __builtin_amdgcn_exp2f(s_top[group + k] - t);
      l += s_l[group + k] * e;
#pragma unroll
      for (int c = 0; c < 4; ++c) y[c] += s_y[c * 256 + threadIdx.x + k * LPS] * e;
    }
    top = t;
  }
  if (want >= rows) return;
  const float f = l == 0.0f ? 0.0f : 1.0f / l;
  const int g = lane / (LPS / 4), c0 = lane % (LPS / 4) * 4;
  uint16_t* dst = a.out + row * a.o_row + hq * a.o_head;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint16_t* at = dst + (4 * g + e) * LPS + c0;
    const uint32_t lo = l == 0.0f ? 0u : pack_bf16(y[0][e] * f, y[1][e] * f), hi = l == 0.0f ? 0u : pack_bf16(y[2][e] * f, y[3][e] * f);
    if (a.o_aligned) {
      *reinterpret_cast<uint32_t*>(at) = lo;
      *reinterpret_cast<uint32_t*>(at + 2) = hi;
    } else {
      at[0] = (uint16_t)lo, at[1] = (uint16_t)(lo >> 16);
      at[2] = (uint16_t)hi, at[3] = (uint16_t)(hi >> 16);
    }
  }
  if (a.lse && lane == 0)
    a.lse[i] = l == 0.0f ? -INFINITY : fmaf(top, a.binade, __builtin_amdgcn_logf(l) * kLn2);
}

namespace {

ShareSizes share_sizes(int d, int64_t S, int64_t R, int64_t heads, int64_t group, int64_t max_len) {
  ShareSizes z{};
  const int64_t RG = R * group;
  // Shared segments: as many rows a tile as the registers hold; own ones: as many as there are.
  z.mt[0] = d == 256 ? 2 : 4;
  z.wt = d == 256 ? 8 : 4;
  z.mt[1] = RG <= 16 ? 1 : d == 256 || RG <= 32 ? 2 : 4;
  // Parts of a row beyond one for each segment, so that few rows can be cut often; for more
  // rows than kShareRoom has places for, fewer segments too, at least a shared one and the
  // row's own (four prompts of 4095 rows of 64 heads of 256 dimensions behind 4096 tokens: 2.2 GB
  // for 6.5, 9.8 ms either way; eight of 1000 rows in two branches 1.1 for 3.2, 5.9 ms for 6.5).
  const int64_t rows = S * RG * heads, shares = (max_len + kShareLeast - 1) / kShareLeast;
  const int64_t places = kShareRoom / (rows * (8 + 4 * d));
  if (S * RG > 65536) {  // prompts: nothing to cut
    z.levels = 1;
    z.extra = 0;
  } else {
    z.levels = kShareLevels;
    const int64_t most = (1 << 18) / rows;
    z.extra = (int)(most < 2 ? 2 : most > 56 ? 56 : most);
    if (z.extra > shares) z.extra = (int)shares;
  }
  if (z.levels > places - 1) z.levels = places > 2 ? (int)places - 1 : 1;
  if (z.extra > places - 1 - z.levels) z.extra = places - 1 > z.levels ? (int)places - 1 - z.levels : 0;
  z.parts = z.levels + 1 + z.extra;
  for (int k = 0; k < 2; ++k) z.rows[k] = 16 * z.mt[k];
  z.slots = kCUs * (d == 64 ? share_resident(64, 4, 4, 4) : d == 128 ? share_resident(128, 4, 4, 4) : share_resident(256, 2, 2, 8));
  // A token of a tile of rows: the issue of its instructions, vector ones and products one
  // after the other, on a SIMD that two waves share (4096 tokens for 64 rows of 128
  // dimensions: two workgroups 84 us).
  for (int k = 0; k < 2; ++k)
    z.us[k] = (float)((4.0 * (0.9 * d + 20 + 36 * z.mt[k]) + (32.0 + d / 2.0) * z.mt[k]) * 1.85 / 2100 * 2 / (32 * z.wt));
  z.read_us = (float)(17.0 / 16 * d * z.slots / 5.5e6);  // at 5.5 TB/s
  // an item, and half of its outputs' way out and back, at 4 TB/s
  for (int k = 0; k < 2; ++k) z.item_us[k] = (float)(kShareItem + (double)z.rows[k] * (d * 4 + 8) * z.slots / 4e6);
  // A level's segments have a tile more each than their rows fill, and shares.
  const int64_t wide = (S * RG + z.rows[0] - 1) / z.rows[0] + S / 2 + 1, own = S * ((RG + z.rows[1] - 1) / z.rows[1]);
  z.cap = (int)((z.levels * wide + own) * (1 + z.extra));
  return z;
}

// Which calls a plan is for.
uint32_t share_key(int d, const KvArgs& a, int group, int window, int extra) {
  uint32_t h = 2166136261u;
  for (const uint32_t x : {(uint32_t)d, (uint32_t)a.heads, (uint32_t)a.n_sessions, (uint32_t)a.R, (uint32_t)group,
                           (uint32_t)window, (uint32_t)a.page_shift, (uint32_t)a.max_pages, (uint32_t)extra, 0x5348u})
    h = (h ^ x) * 16777619u;
  return h;
}

struct SharePlaces {
  size_t order, parts, items, all;
};
SharePlaces share_places(const ShareSizes& z, int64_t S) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  SharePlaces p{};
  p.order = up(sizeof(ShareHead));
  p.parts = p.order + up(S * sizeof(SharePlace));
  p.items = p.parts + up(S * 4);
  p.all = p.items + up(z.cap * sizeof(ShareItem));
  return p;
}

template <int D, int MT, int OWN, int WT>
hipError_t launch_parts(const ShareArgs& a, int slots, hipStream_t s) {
  constexpr size_t lds = share_lds(D, MT, OWN, WT);
  static std::atomic<uint64_t> done{0};
  const hipError_t e = set_lds_limit_once(done, reinterpret_cast<const void*>(k_share_parts<D, MT, OWN, WT>), lds);
  if (e != hipSuccess) return e;
  const int64_t most = (int64_t)a.cap * a.kv.heads;
  launch_kernel(k_share_parts<D, MT, OWN, WT>, dim3((unsigned)(most < slots ? most : slots)), dim3(64 * waves_in(WT)),
                (uint32_t)lds, s, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_own(int own, const ShareArgs& a, int slots, hipStream_t s) {
  if constexpr (D == 256) return own == 1 ? launch_parts<D, 2, 1, 8>(a, slots, s) : launch_parts<D, 2, 2, 8>(a, slots, s);
  else
    return own == 1 ? launch_parts<D, 4, 1, 4>(a, slots, s)
           : own == 2 ? launch_parts<D, 4, 2, 4>(a, slots, s)
                      : launch_parts<D, 4, 4, 4>(a, slots, s);
}

// (2560 rows of up to 35 parts of 128 dimensions: 13.1 us by one group of lanes a row)
template <int D>
void launch_share_join(const ShareArgs& a, int64_t rows, hipStream_t s) {
  constexpr int ALL = 256 / (D / 16);  // groups of lanes of a workgroup
  if (a.parts <= 6) launch_kernel(k_share_join<D, 1>, dim3((unsigned)((rows + ALL - 1) / ALL)), dim3(256), 0, s, a, rows);
  else launch_kernel(k_share_join<D, 8>, dim3((unsigned)((rows * 8 + ALL - 1) / ALL)), dim3(256), 0, s, a, rows);
}

}  // namespace

bool kv_share_fits(int64_t n_sessions, int64_t R, int64_t q_heads) {
  return n_sessions <= kShareSessions && n_sessions * R * q_heads <= (int64_t(1) << 26);
}

size_t kv_share_bytes(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len) {
  return share_places(share_sizes(d, n_sessions, R, heads, q_heads / heads, max_len), n_sessions).all;
}

size_t kv_share_scratch(int d, int64_t n_sessions, int64_t R, int64_t heads, int64_t q_heads, int64_t max_len) {
  const ShareSizes z = share_sizes(d, n_sessions, R, heads, q_heads / heads, max_len);
  const size_t n = (size_t)n_sessions * R * q_heads * z.parts;
  return (n * 8 + 255) / 256 * 256 + n * d * 4;
}

hipError_t launch_share_plan(int d, const KvArgs& kv, int q_heads, int window, int64_t max_len, void* plan, hipStream_t s) {
  SharePlanArgs a{};
  a.kv = kv;
  a.group = q_heads / kv.heads;
  a.window = window;
  a.z = share_sizes(d, kv.n_sessions, kv.R, kv.heads, a.group, max_len);
  a.key = share_key(d, kv, a.group, window, a.z.extra);
  const SharePlaces p = share_places(a.z, kv.n_sessions);
  uint8_t* base = static_cast<uint8_t*>(plan);
  a.head = reinterpret_cast<ShareHead*>(base);
  a.order = reinterpret_cast<SharePlace*>(base + p.order);
  a.parts = reinterpret_cast<int32_t*>(base + p.parts);
  a.items = reinterpret_cast<ShareItem*>(base + p.items);
  int n2 = 2;
  while (n2 < kv.n_sessions) n2 *= 2;
  static std::atomic<uint64_t> done{0};
  const hipError_t e = set_lds_limit_once(done, reinterpret_cast<const void*>(k_share_plan), plan_lds(kShareSessions));
  if (e != hipSuccess) return e;
  launch_kernel(k_share_plan, dim3(1), dim3(kPlanThreads), (uint32_t)plan_lds(n2), s, a, n2);
  return hipGetLastError();
}

hipError_t launch_attend_shared(int d, const KvArgs& kv, const AttendCall& c, void* plan, void* workspace, hipStream_t s) {
  ShareArgs a{};
  a.kv = kv;
  a.q = static_cast<const uint16_t*>(c.q);
  a.q_row = c.q_row;
  a.q_head = c.q_head;
  a.out = static_cast<uint16_t*>(c.out);
  a.o_row = c.o_row;
  a.o_head = c.o_head;
  a.lse = c.lse;
  a.group = c.q_heads / kv.heads;
  a.of_rows = divisor_of((uint32_t)(kv.R * a.group));
  a.of_group = divisor_of((uint32_t)a.group);
  a.window = c.window;
  a.scale_log2 = c.scale * 1.44269504088896f;
  a.binade = (float)((double)c.scale / a.scale_log2);
  a.q_aligned = c.q_row % 8 == 0 && c.q_head % 8 == 0 && (reinterpret_cast<uintptr_t>(c.q) & 15) == 0;
  a.o_aligned = c.o_row % 2 == 0 && c.o_head % 2 == 0 && (reinterpret_cast<uintptr_t>(c.out) & 3) == 0;
  const ShareSizes z = share_sizes(d, kv.n_sessions, kv.R, kv.heads, a.group, c.max_len);
  const SharePlaces p = share_places(z, kv.n_sessions);
  uint8_t* base = static_cast<uint8_t*>(plan);
  a.key = share_key(d, kv, a.group, c.window, z.extra);
  a.head = reinterpret_cast<ShareHead*>(base);
  a.order = reinterpret_cast<const SharePlace*>(base + p.order);
  a.n_parts = reinterpret_cast<const int32_t*>(base + p.parts);
  a.parts = z.parts;
  const int64_t rows = (int64_t)kv.n_sessions * kv.R * c.q_heads;
  a.part_ml = static_cast<float2*>(workspace);
  a.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + ((size_t)rows * z.parts * 8 + 255) / 256 * 256);
  a.cap = z.cap;
  a.items = reinterpret_cast<const ShareItem*>(base + p.items);
  const hipError_t e = d == 64    ? launch_own<64>(z.mt[1], a, z.slots, s)
                       : d == 128 ? launch_own<128>(z.mt[1], a, z.slots, s)
                                  : launch_own<256>(z.mt[1], a, z.slots, s);
  if (e != hipSuccess) return e;
  if (d == 64) launch_share_join<64>(a, rows, s);
  else if (d == 128) launch_share_join<128>(a, rows, s);
  else launch_share_join<256>(a, rows, s);
  return hipGetLastError();
}

}  // namespace sph

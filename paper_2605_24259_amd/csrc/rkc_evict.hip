// rkc_evict.hip -- eviction from a paged cache by the account of its slots.
//
// Kept are the protected first slots, recent ones, and of the others those of the largest account.  One workgroup decides
// for a head of a sequence of up to 16,384 slots, one for each tile of that many in longer ones (evict_round): the account of the last slot to be kept is found 8 bits of its
// 32-bit order at a time, by counts of the digits in LDS (whole numbers: their order does not matter); ties go to the
// lowest slots, and prefix sums pair the gaps in front of the new end with the kept slots behind it.  A second kernel moves their
// keys and values.  Sources lie behind the new end and targets before it, so that the moves need no order among
// each other, and what is kept in place is not touched: the least that can be moved.
#include "rkc_cache_dev.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kItems = 16, kTile = kThreads * kItems, kMoves = 128, kCopies = 16;

struct evict_args {
  rkc_cache c;
  rkc_eviction e;
  int32_t *gaps, *from, *count;  // scratch: [row][most], [row][most], [row]
  int most;
  int parts;        // tiles of the longest sequence; where more than one:
  uint32_t* hist;   // [2][row][part][2 classes][kBins]: digit counts of each tile, of odd and even rounds
  int32_t* tally;   // [row][part][4]: of each tile, see evict_round
  uint32_t* state;  // [4][row][4]: after each round the order so far, how many are left, whether among recent ones
};

constexpr int kBins = 2048;  // 11 bits

// The account's order in whole numbers above 0; NaN lowest, both zeros alike.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 1;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}

// Sum over the lower lanes and this one, by shifts within rows of 16 and broadcasts of rows' last lanes.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += moved<0x111, 0xf>(x);  // row_shr:1
  x += moved<0x112, 0xf>(x);
  x += moved<0x114, 0xf>(x);
  x += moved<0x118, 0xf>(x);
  x += moved<0x142, 0xa>(x);  // row_bcast:15
  x += moved<0x143, 0xc>(x);  // row_bcast:31
  return x;
}

// Number of the lower lanes whose bit is set.
__device__ __forceinline__ int lower(uint64_t m) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0)); }

// A head of a sequence: what is kept of it in number, and where its accounts and positions are.
struct Head {
  int s, h, len, held, now, recent_from;
  bool ok, recents;
  const float* w;
  const int32_t* pos;
  float* w_out;
  int32_t* pos_out;
  __device__ int pos_at(int j) const { return pos ? pos[j] : j; }
};

__device__ __forceinline__ Head load_head(const evict_args& g, int row) {
  const rkc_eviction& e = g.e;
  Head x;
  x.s = row / g.c.kv_heads, x.h = row % g.c.kv_heads;
  x.len = word(e.d_length, x.s);
  x.ok = x.len >= 0 && x.len <= e.max_len;
  x.held = e.d_protect ? min(x.len, max(0, word(e.d_protect, x.s))) : 0;
  x.now = min(x.len, max(x.held, max(0, word(e.d_budget, x.s))));
  x.recents = e.d_recent_from != nullptr;
  x.recent_from = x.recents ? word(e.d_recent_from, x.s) : 0x7fffffff;
  const int64_t at = x.s * e.weight_seq_stride + x.h * e.weight_head_stride;
  x.w = e.d_weight + at, x.pos = e.d_pos ? e.d_pos + at : nullptr;
  x.w_out = e.d_weight_out + at, x.pos_out = e.d_pos_out + at;
  return x;
}

// A tile of a head's slots, of a workgroup of N threads: a thread has slots tid, tid + N, ... of it.
template <int N> struct Tile {
  static constexpr int kSlots = N * kItems;
  float wt[kItems];
  int ps[kItems];
  uint32_t open, recent;  // bit i: slot i of the thread is behind the protected ones; is recent
  int base;
  __device__ __forceinline__ int slot(int i) const { return base + i * N + (int)threadIdx.x; }
  __device__ __forceinline__ void load(const Head& x, int tile) {
    base = tile * kSlots, open = recent = 0;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = slot(i);
      wt[i] = 0.f, ps[i] = j;
      if (base + i * N >= x.len) continue;
      if (j < x.len) {
        wt[i] = x.w[j];
        if (x.pos) ps[i] = x.pos[j];
      }
    }
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      if (base + i * N >= x.len) continue;
      const int j = slot(i);
      const bool in = j >= x.held && j < x.len;
      open |= (in ? 1u : 0u) << i;
      recent |= (in && x.recents && ps[i] >= x.recent_from ? 1u : 0u) << i;
    }
  }
  // Bits of the slots that stay whatever comes, with those above the last order T, and of those that tie with it.
  __device__ __forceinline__ void judge(const Head& x, bool among_recent, bool any, uint32_t T, uint32_t& keep, uint32_t& tie) const {
    const uint32_t in = among_recent ? recent : open & ~recent;
    keep = among_recent ? 0 : recent, tie = 0;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      if (base + i * N >= x.len) continue;
      const uint32_t key = order_of(wt[i]);
      if (slot(i) < x.held) keep |= 1u << i;
      if (any && (in >> i & 1)) {
        if (key > T) keep |= 1u << i;
        if (key == T) tie |= 1u << i;
      }
    }
  }
};

// Counts of runs of 64 slots (of two kinds), then what lies before each in the tile; the last entry: the tile's.
template <int N> struct Runs { uint32_t n[2][kItems * N / 64 + 1]; };
template <int N> __device__ __forceinline__ void runs_before(Runs<N>& table) {
  constexpr int kRuns = kItems * N / 64, K = kRuns / 64;
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
  __syncthreads();
  if (wave < 2) {
    uint32_t x[K], sum = 0;
#pragma unroll
    for (int k = 0; k < K; k++) x[k] = sum, sum += table.n[wave][lane * K + k];
    const uint32_t to = wave_scan(sum);
#pragma unroll
    for (int k = 0; k < K; k++) table.n[wave][lane * K + k] = to - sum + x[k];
    if (lane == 63) table.n[wave][kRuns] = to;
  }
  __syncthreads();
}

// The lowest `left` of a tile's ties stay.
template <int N> __device__ __forceinline__ void keep_ties(Runs<N>& table, uint32_t tie, uint32_t left, uint32_t& keep) {
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < kItems; i++) {
    const uint64_t m = __ballot(tie >> i & 1);
    if (lane == 0) table.n[0][i * (N / 64) + wave] = __popcll(m), table.n[1][i * (N / 64) + wave] = 0;
  }
  runs_before(table);
#pragma unroll
  for (int i = 0; i < kItems; i++) {
    const uint64_t m = __ballot(tie >> i & 1);
    if ((tie >> i & 1) && table.n[0][i * (N / 64) + wave] + lower(m) < left) keep |= 1u << i;
  }
  __syncthreads();
}

// Lists a tile's gaps before the new end and its kept slots behind it, from places gap0 and from0 on, and writes what
// stays; gap_at, if given: the gaps of the only tile.
template <int N> __device__ __forceinline__ void list_moves(const evict_args& g, int row, const Head& x, const Tile<N>& t, uint32_t keep, Runs<N>& table, int gap0, int from0, uint16_t* gap_at) {
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < kItems; i++) {
    const int j = t.slot(i);
    const bool kept = keep >> i & 1;
    const uint64_t gap = __ballot(j < x.now && !kept), src = __ballot(j >= x.now && j < x.len && kept);
    if (lane == 0) table.n[0][i * (N / 64) + wave] = __popcll(gap), table.n[1][i * (N / 64) + wave] = __popcll(src);
  }
  runs_before(table);
  int32_t* gaps = g.gaps + (int64_t)row * g.most;
  int32_t* from = g.from + (int64_t)row * g.most;
#pragma unroll
  for (int i = 0; i < kItems; i++) {
    const int j = t.slot(i);
    if (t.base + i * N >= x.now) continue;
    const bool kept = keep >> i & 1, is_gap = j < x.now && !kept;
    const int at = gap0 + table.n[0][i * (N / 64) + wave] + lower(__ballot(is_gap));
    if (is_gap) gaps[at] = j;
    if (is_gap && gap_at) gap_at[at] = (uint16_t)j;
    if (j < x.now && kept) x.w_out[j] = t.wt[i], x.pos_out[j] = t.ps[i];
  }
  if (gap_at) __syncthreads();
#pragma unroll
  for (int i = 0; i < kItems; i++) {
    const int j = t.slot(i);
    if (t.base + i * N >= x.len) continue;
    const bool is_src = j >= x.now && j < x.len && (keep >> i & 1);
    const int at = from0 + table.n[1][i * (N / 64) + wave] + lower(__ballot(is_src));
    if (is_src) from[at] = j;
    if (is_src && gap_at) {
      const int to = gap_at[at];
      x.w_out[to] = t.wt[i], x.pos_out[to] = t.ps[i];
    }
  }
}

// Sequences of at most one tile: one workgroup decides for a head, whose accounts stay in its registers: one read of
// them, up to four counts of a digit.  Four waves where the sequences are of up to 4,096 slots, as barriers of sixteen
// cost more than they save (8 heads of up to 1,280 slots: 9.1 us instead of 13.6).  Bound by latency and by the LDS
// additions of the counts: 27 to 30 us for 256 heads of 5,000 to 16,384.  (A copy of the counts for each lane left no room for
// as many waves: 39 us.)
template <int N> __global__ __launch_bounds__(N) void evict_choose(const evict_args g) {
  // counts of 256 digits, a copy for each of 16 lanes: at most 4 lanes of an addition meet in a word, whatever the digits
  __shared__ __attribute__((aligned(16))) uint32_t hist[256 * kCopies];
  uint16_t* const gap_at = (uint16_t*)hist;  // later: the gaps, at most half of the slots
  static_assert(sizeof(hist) >= N * kItems / 2 * sizeof(uint16_t), "gaps");
  __shared__ Runs<N> table;
  __shared__ uint32_t found[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const Head x = load_head(g, blockIdx.x);
  if (!x.ok) {
    if (tid == 0) {
      g.count[blockIdx.x] = 0;
      if (x.h == 0) flag(g.c, x.s, RKC_CS_LENGTH);
    }
    return;
  }
  if (tid == 0 && x.h == 0) g.e.d_length_out[x.s] = x.now;
  if (x.now == x.len) {
    for (int j = tid; j < x.len; j += N) x.w_out[j] = x.w[j], x.pos_out[j] = x.pos_at(j);
    if (tid == 0) g.count[blockIdx.x] = 0;
    return;
  }
  Tile<N> t;
  t.load(x, 0);
  int K = x.now - x.held;  // to be kept of the slots behind the protected ones
  bool among_recent = false;  // the choice is among the recent ones; else they stay, and it is among the others
  if (x.recents) {
    if (tid == 0) found[0] = 0;
    __syncthreads();
    const uint32_t n = wave_scan(__popc(t.recent));
    if (lane == 63 && n) atomicAdd(&found[0], n);
    __syncthreads();
    among_recent = (int)found[0] >= K;
    if (!among_recent) K -= found[0];
    __syncthreads();
  }
  // The order of the last slot to be kept, 8 bits at a time from the top; `left`: how many of those that agree with
  // it so far are to be kept.
  uint32_t T = 0, left = K, same = 0;
  const uint32_t in = among_recent ? t.recent : t.open & ~t.recent;
  if (K > 0) {
#pragma unroll
    for (int b = 24; b >= 0; b -= 8) {
      // all of them are: lower bits do not matter (few slots: 9.1 us instead of 11.8; many seldom end early, 27.8 for 26.4)
      if (N == 256 && left == same) break;
      for (int k = tid; k < 256 * kCopies / 4; k += N) ((u32x4*)hist)[k] = u32x4{0, 0, 0, 0};
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kItems; i++) {
        if (i * N >= x.len) continue;
        const uint32_t key = order_of(t.wt[i]);
        if ((in >> i & 1) && (b == 24 || (key ^ T) >> b >> 8 == 0)) atomicAdd(&hist[(key >> b & 255) * kCopies + (lane & (kCopies - 1))], 1u);
      }
      __syncthreads();
      constexpr int Q = 1024 / N;
      uint32_t n[Q];
#pragma unroll
      for (int k = 0; k < Q; k++) {
        const u32x4 x4 = ((const u32x4*)hist)[k * N + tid];  // a quarter of a digit's copies
        n[k] = x4[0] + x4[1] + x4[2] + x4[3];
        n[k] += (uint32_t)dpp<0xb1>((int)n[k]);  // quad_perm [1,0,3,2]
        n[k] += (uint32_t)dpp<0x4e>((int)n[k]);  // quad_perm [2,3,0,1]
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < Q; k++)
        if ((tid & 3) == 0) hist[k * (N / 4) + (tid >> 2)] = n[k];
      __syncthreads();
      if (wave == 0) {  // lane l: digits 255 - 4 l and the three below
        const u32x4 y = ((const u32x4*)hist)[63 - lane];
        const uint32_t mine = y[0] + y[1] + y[2] + y[3], to = wave_scan(mine);
        uint32_t above = to - mine;
        if (above < left && left <= to) {
          int d = 3;
          while (above + y[d] < left) above += y[d--];
          found[0] = (63 - lane) * 4 + d, found[1] = left - above, found[2] = y[d];
        }
      }
      __syncthreads();
      T |= found[0] << b, left = found[1], same = found[2];
    }
  }
  uint32_t keep, tie;
  const bool all = left == same;  // then T itself is to be kept: orders are above 0
  t.judge(x, among_recent, K > 0, all && T ? T - 1 : T, keep, tie);
  if (!all) keep_ties(table, tie, left, keep);
  list_moves(g, blockIdx.x, x, t, keep, table, 0, 0, gap_at);
  if (tid == 0) g.count[blockIdx.x] = table.n[0][kItems * N / 64];
}

// Longer sequences: a workgroup for each tile of a head, and a launch for each step, which reads what the tiles of the
// step before wrote, as one workgroup would take a tile after the other (8 heads of 65,536 slots 145 us a call instead of
// 78).  Every workgroup adds up the counts of all its head's tiles, 8 KB each, so that what is read grows with the square
// of the length: 4 x 32 KB a head and round at 65,536 slots, 4,096 x 32 MB at 2^26.
// Rounds 0, 1 and 2 count 11, 11 and 10 bits of the order; round 3 tallies each tile (ties, those of them before the new end,
// kept slots without ties before and behind it); round 4 lists and writes.
template <int ROUND>
__global__ __launch_bounds__(kThreads) void evict_round(const evict_args g) {
  constexpr int kShift[5] = {21, 10, 0, 0, 0};
  __shared__ __attribute__((aligned(16))) uint32_t hist[2 * kBins];
  __shared__ Runs<kThreads> table;
  __shared__ uint32_t sums[kWaves], found[3], told[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int row = blockIdx.x / g.parts, part = blockIdx.x % g.parts;
  const Head x = load_head(g, row);
  const int tiles = (x.len + kTile - 1) / kTile, rows = gridDim.x / g.parts;
  if (!x.ok || x.len == 0) {
    if (ROUND == 0 && part == 0 && tid == 0) {
      g.count[row] = 0;
      if (x.h == 0 && x.ok) g.e.d_length_out[x.s] = 0;
      if (x.h == 0 && !x.ok) flag(g.c, x.s, RKC_CS_LENGTH);
    }
    return;
  }
  if (part >= tiles) return;
  if (ROUND == 0 && part == 0 && tid == 0 && x.h == 0) g.e.d_length_out[x.s] = x.now;
  Tile<kThreads> t;
  if (x.now == x.len) {  // nothing goes
    if (ROUND == 4) {
      t.load(x, part);
#pragma unroll
      for (int i = 0; i < kItems; i++)
        if (t.slot(i) < x.len) x.w_out[t.slot(i)] = t.wt[i], x.pos_out[t.slot(i)] = t.ps[i];
      if (part == 0 && tid == 0) g.count[row] = 0;
    }
    return;
  }
  t.load(x, part);
  // [row][part][class][bin] of the round before, and of this one
  const uint32_t* before = g.hist + ((int64_t)(((ROUND + 1) & 1) * rows + row) * g.parts) * 2 * kBins;
  uint32_t* mine = g.hist + ((int64_t)((ROUND & 1) * rows + row) * g.parts + part) * 2 * kBins;
  uint32_t T = 0, left = x.now - x.held;
  bool among_recent = false;
  if (ROUND > 1) {
    const uint32_t* st = g.state + (int64_t)((ROUND - 2) * rows + row) * 4;
    T = st[0], left = st[1], among_recent = st[2];
  }
  uint32_t same = 0;
  if (ROUND >= 1 && ROUND <= 3) {
    // the digit of the round before: thread i has bins 2047 - 2 i and 2046 - 2 i
    auto sum_of = [&](int cls) {
      uint2 n = {0, 0};
      for (int p = 0; p < tiles; p++) {
        const uint2 y = *(const uint2*)(before + ((int64_t)p * 2 + cls) * kBins + kBins - 2 - 2 * tid);
        n.x += y.x, n.y += y.y;
      }
      return n;
    };
    auto scan = [&](uint32_t v, uint32_t& all) {  // inclusive, over the workgroup
      const uint32_t inc = wave_scan(v);
      __syncthreads();
      if (lane == 63) sums[wave] = inc;
      __syncthreads();
      uint32_t low = 0;
      all = 0;
#pragma unroll
      for (int k = 0; k < kWaves; k++) low += k < wave ? sums[k] : 0, all += sums[k];
      return low + inc;
    };
    uint32_t all;
    if (ROUND == 1 && x.recents) {
      const uint2 n = sum_of(1);
      scan(n.x + n.y, all);
      among_recent = all >= left;
      if (!among_recent) left -= all;
    }
    if (left > 0) {
      const uint2 n = sum_of(among_recent ? 1 : 0);
      const uint32_t to = scan(n.x + n.y, all);
      const uint32_t above = to - n.x - n.y;
      if (above < left && left <= to) {
        const bool high = above + n.y >= left;
        found[0] = kBins - 2 - 2 * tid + high, found[1] = left - above - (high ? 0 : n.y), found[2] = high ? n.y : n.x;
      }
      __syncthreads();
      T |= found[0] << kShift[ROUND - 1], left = found[1], same = found[2];
    }
    if (part == 0 && tid == 0) {
      uint32_t* st = g.state + (int64_t)((ROUND - 1) * rows + row) * 4;
      st[0] = T, st[1] = left, st[2] = among_recent;
    }
  }
  if (ROUND <= 2) {
    for (int k = tid; k < 2 * kBins / 4; k += kThreads) ((u32x4*)hist)[k] = u32x4{0, 0, 0, 0};
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const uint32_t key = order_of(t.wt[i]);
      const bool in = (t.open >> i & 1) && (ROUND == 0 || (key ^ T) >> kShift[ROUND ? ROUND - 1 : 0] == 0);
      const uint32_t bin = (t.recent >> i & 1) * kBins + (key >> kShift[ROUND] & (ROUND == 2 ? 1023 : 2047));
      const uint64_t all = __ballot(in);
      if (!all) continue;
      // those that agree with the first one are added at once: many accounts are zero
      const int first = __builtin_ctzll(all);
      const bool alike = in && bin == (uint32_t)__builtin_amdgcn_readlane((int)bin, first);
      const uint64_t m = __ballot(alike);
      if (lane == first) atomicAdd(&hist[bin], (uint32_t)__popcll(m));
      if (in && !alike) atomicAdd(&hist[bin], 1u);
    }
    __syncthreads();
    for (int k = tid; k < 2 * kBins / 4; k += kThreads) ((u32x4*)mine)[k] = ((const u32x4*)hist)[k];
    return;
  }
  uint32_t keep, tie;
  if (ROUND == 4) {
    const uint32_t* st = g.state + (int64_t)(2 * rows + row) * 4;
    T = st[0], left = st[1], among_recent = st[2];
  }
  t.judge(x, among_recent, left > 0, T, keep, tie);
  int32_t* tally = g.tally + (int64_t)row * g.parts * 4;
  if (ROUND == 3) {
    uint32_t n[4] = {};
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const bool front = t.slot(i) < x.now;
      n[0] += tie >> i & 1, n[1] += front && (tie >> i & 1);
      n[2] += front && (keep >> i & 1), n[3] += !front && (keep >> i & 1);
    }
    if (tid < 4) told[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const uint32_t all = wave_scan(n[k]);
      if (lane == 63) atomicAdd(&told[k], all);
    }
    __syncthreads();
    if (tid < 4) tally[part * 4 + tid] = told[tid];
    return;
  }
  // round 4: what lies before this tile
  int ties = 0, gap0 = 0, from0 = 0, total = 0;
  for (int p = 0; p < tiles; p++) {
    const int4 y = *(const int4*)(tally + p * 4);
    const int stay = max(0, min(y.x, (int)left - ties)), front = min(stay, y.y);
    const int gaps = max(0, min(kTile, x.now - p * kTile)) - y.z - front, from = y.w + stay - front;
    if (p < part) gap0 += gaps, from0 += from;
    if (p == part) same = (uint32_t)max(0, (int)left - ties);
    ties += y.x, total += gaps;
  }
  if (part == 0 && tid == 0) g.count[row] = total;
  keep_ties(table, tie, same, keep);
  list_moves(g, row, x, t, keep, table, gap0, from0, nullptr);
}

// Moves the keys and values of up to kMoves slots of a head of a sequence, 16 bytes a lane.  Bound by the copy: 256 heads
// of 5,000 to 16,384 slots of 128 elements down to half move 0.69 GB in 158 us, 4.4 TB/s read and written.
__global__ __launch_bounds__(256) void evict_move(const evict_args g, int chunks) {
  const rkc_cache& c = g.c;
  const int row = blockIdx.x / chunks, first = blockIdx.x % chunks * kMoves, n = min(g.count[row] - first, kMoves);
  if (n <= 0) return;
  const int H = c.kv_heads, s = row / H, h = row % H, per = c.head_dim / 8, shift = 31 - __builtin_clz(c.page_tokens);
  const int32_t* table = c.d_block_table + (int64_t)s * c.max_pages;
  const int32_t* gaps = g.gaps + (int64_t)row * g.most + first;
  const int32_t* from = g.from + (int64_t)row * g.most + first;
  for (int x = threadIdx.x; x < n * per; x += 256) {
    const int i = x / per, e = x % per * 8, to = gaps[i], at = from[i];
    bool bad = false;
    auto page = [&](int t) {
      const int id = table[t >> shift];
      const bool out = (uint32_t)id >= (uint32_t)c.n_blocks;
      bad |= out;
      return (int64_t)(out ? 0 : id);
    };
    const int64_t pt = page(to), pf = page(at);
    const int in_page = c.page_tokens - 1;
    uint16_t* k = (uint16_t*)c.d_k + h * c.k_head_stride + e;
    uint16_t* v = (uint16_t*)c.d_v + h * c.v_head_stride + e;
    if (g.parts > 1 && e == 0) {  // of the only tile, evict_choose has written them
      const int64_t o = s * g.e.weight_seq_stride + h * g.e.weight_head_stride;
      g.e.d_weight_out[o + to] = g.e.d_weight[o + at], g.e.d_pos_out[o + to] = g.e.d_pos ? g.e.d_pos[o + at] : at;
    }
    if (bad) {  // a block that is another sequence's must not be written in its place
      flag(c, s, RKC_CS_BLOCK);
      continue;
    }
    const u32x4 a = *(const u32x4*)(k + pf * c.k_block_stride + (at & in_page) * c.k_slot_stride);
    const u32x4 b = *(const u32x4*)(v + pf * c.v_block_stride + (at & in_page) * c.v_slot_stride);
    *(u32x4*)(k + pt * c.k_block_stride + (to & in_page) * c.k_slot_stride) = a;
    *(u32x4*)(v + pt * c.v_block_stride + (to & in_page) * c.v_slot_stride) = b;
  }
}

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

// Lays the scratch out from `base` on; its size.
size_t lay_out(const rkc_cache* c, const rkc_eviction* e, char* base, evict_args* g) {
  const size_t rows = (size_t)c->n_seqs * c->kv_heads, most = (size_t)e->max_len / 2 + 1;
  const size_t parts = e->max_len > kTile ? ((size_t)e->max_len + kTile - 1) / kTile : 1;
  size_t at = 0;
  auto take = [&](size_t n) {
    char* p = base + at;
    at += up(n);
    return p;
  };
  g->most = (int)most, g->parts = (int)parts;
  g->gaps = (int32_t*)take(rows * most * 4), g->from = (int32_t*)take(rows * most * 4), g->count = (int32_t*)take(rows * 4);
  if (parts > 1) {
    g->hist = (uint32_t*)take(2 * rows * parts * 2 * kBins * 4);
    g->tally = (int32_t*)take(rows * parts * 16), g->state = (uint32_t*)take(4 * rows * 16);
  }
  return at;
}

}  // namespace

extern "C" {

size_t rkc_evict_scratch_bytes(const rkc_cache* c, const rkc_eviction* e) {
  if (!c || !e || c->n_seqs < 1 || c->kv_heads < 1 || e->max_len < 0) return 0;
  evict_args g;
  return lay_out(c, e, nullptr, &g);
}

rkc_status rkc_evict(const rkc_cache* c, const rkc_eviction* e, void* stream) {
  if (rkc_status st = rkc_cache_check(c)) return st;
  if (!e) return RKC_E_NULL;
  if (e->max_len < 0 || e->reserved || e->max_len > RKC_MAX_CACHE_LEN || e->max_len > (int64_t)c->max_pages * c->page_tokens) return RKC_E_RANGE;
  const int64_t far = (int64_t)1 << 40;
  if (e->weight_seq_stride < 0 || e->weight_head_stride < 0 || e->weight_seq_stride > far || e->weight_head_stride > far) return RKC_E_RANGE;
  if (c->n_seqs == 0) return RKC_OK;
  if (!e->d_length || !e->d_budget || !e->d_weight || !e->d_weight_out || !e->d_pos_out || !e->d_length_out) return RKC_E_NULL;
  for (const void* p : {(const void*)e->d_length, (const void*)e->d_budget, (const void*)e->d_protect, (const void*)e->d_recent_from,
                        (const void*)e->d_weight, (const void*)e->d_pos, (const void*)e->d_weight_out, (const void*)e->d_pos_out,
                        (const void*)e->d_length_out})
    if ((uintptr_t)p & 3) return RKC_E_ALIGN;
  if (e->d_weight_out == e->d_weight || e->d_pos_out == e->d_pos) return RKC_E_RANGE;
  for (const int32_t* p : {e->d_length, e->d_budget, e->d_protect, e->d_recent_from})
    if (e->d_length_out == p) return RKC_E_RANGE;
  if (rkc_shared(e->max_len, c->n_seqs, e->weight_seq_stride, c->kv_heads, e->weight_head_stride)) return RKC_E_RANGE;
  if (rkc_shared(c->head_dim, c->n_blocks, c->k_block_stride, c->page_tokens, c->k_slot_stride, c->kv_heads, c->k_head_stride) ||
      rkc_shared(c->head_dim, c->n_blocks, c->v_block_stride, c->page_tokens, c->v_slot_stride, c->kv_heads, c->v_head_stride))
    return RKC_E_RANGE;
  const size_t need = rkc_evict_scratch_bytes(c, e);
  if (!e->d_scratch || e->scratch_bytes < need) return RKC_E_SCRATCH;
  if ((uintptr_t)e->d_scratch & 255) return RKC_E_ALIGN;
  const size_t rows = (size_t)c->n_seqs * c->kv_heads;
  evict_args g = {};
  g.c = *c, g.e = *e;
  lay_out(c, e, (char*)e->d_scratch, &g);
  const int64_t chunks = (e->max_len / 2 + kMoves - 1) / kMoves;
  if (!rkc_fits((int64_t)rows * g.parts, kThreads) || !rkc_fits((int64_t)rows * chunks, 256)) return RKC_E_UNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  const dim3 block(kThreads), one((unsigned)rows), tiles((unsigned)(rows * g.parts));
  if (e->max_len <= 256 * kItems) {
    evict_choose<256><<<one, dim3(256), 0, s>>>(g);
  } else if (g.parts == 1) {
    evict_choose<kThreads><<<one, block, 0, s>>>(g);
  } else {
    evict_round<0><<<tiles, block, 0, s>>>(g);
    evict_round<1><<<tiles, block, 0, s>>>(g);
    evict_round<2><<<tiles, block, 0, s>>>(g);
    evict_round<3><<<tiles, block, 0, s>>>(g);
    evict_round<4><<<tiles, block, 0, s>>>(g);
  }
  if (chunks) evict_move<<<dim3((unsigned)(rows * chunks)), dim3(256), 0, s>>>(g, (int)chunks);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

}  // extern "C"

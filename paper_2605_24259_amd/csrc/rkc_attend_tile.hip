// rkc_attend_tile.hip -- attention of many rows over a paged cache (chunks of prompts, larger trees).
//
// out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m) in one pass over the slots, m the running maximum of a row's scores.
// A workgroup of W waves holds R W packed rows (rows x query heads of one key/value head), R of them in each wave as the
// columns of its matrix products, and goes over the slots that any of them sees in tiles of 64 (32 at 256 elements a
// head).  K and V of up to three tiles ahead are on their way from memory into LDS, past the registers.  Tiles that
// every row sees skip the masks, waves whose rows see nothing of a tile skip it.
//   D = 64, 128:   4 waves of 32 rows, 32x32x16 products, a barrier a tile
//   D = 128, more than 128 packed rows where they fill the card (rkc_attend_plan): 8 waves of 32 rows in two groups that
//                  multiply and weigh in turns (in_turns)
//   D = 256:       8 waves of 16 rows, 16x16x32 products, in turns as well (a wave of 32 rows would hold 128 registers of
//                  outputs, 64 of queries and 16 of scores, of the 256 that two waves a SIMD have; that form is not built)
// What bounds it: matrix products and the exponentials between them.  2,048 rows of 32 heads over 32,768 slots (8 heads of
// 128 elements): 1,040 us, 1,020 TFLOP/s, 0.86 of a large matrix product's rate; 1,311 us with a cap, of which the matrix
// units are at work for 0.36 and the vector units' issue is taken for 0.65, so that the two hardly overlap.  At 256 elements
// a head 2,048 rows of 16 heads over 16,384 slots: 680 us, 760 TFLOP/s.  32 trees of 64 rows over 8,192 slots: 345 us, 790
// TFLOP/s.
#include <type_traits>

#include "rkc_cache_dev.h"
#include "rkc_tiles.h"

namespace {

template <int R> struct Acc;
template <> struct Acc<32> { typedef f32x16 t; };
template <> struct Acc<16> { typedef f32x4 t; };

template <typename T, int D, int W, int R>
__global__ __launch_bounds__(64 * W, D == 64 ? 3 : 2) void attend_tile(const rkc_cache c, const rkc_attention a, const rkc_plan pl) {
  typedef typename Vec8<T>::t V8;
  // R rows a wave: products of R x R, A elements a lane; tiles of BK slots, kAhead of them on their way
  typedef typename Acc<R>::t acc;
  constexpr int A = R * R / 64, kRows = R * W, kThreads = 64 * W;
  constexpr int BK = D == 256 ? 32 : 64, kAhead = W == 8 ? 3 : 1, CH = D / 8;
  constexpr int KT = BK / R, KC = D * R / 512, DB = D / R, NP = KT * A / 8;  // score blocks, key operands, output blocks, weight operands
  constexpr int P = BK * CH / kThreads;  // 16-byte pieces of K, and of V, per thread
  constexpr int kTile = BK * D;
  __shared__ __attribute__((aligned(16))) T lds[(kAhead + 1) * 2 * kTile];  // K and V of each tile
  __shared__ uint64_t lines[RKC_MAX_TREE_ROWS][4];
  __shared__ int depths[RKC_MAX_TREE_ROWS], lim[W][2];

  const int H = c.kv_heads, G = a.q_heads / H;
  // Heads first: with 8 of them each XCD has one, and its cache that head's keys and values for the row tiles of a
  // sequence, which are neighbours; the rows that see most go first.  (All heads on each XCD: trees 397 us instead of
  // 334, documents 57 instead of 49; sequences before row tiles: 455 and 62.)
  const int h = blockIdx.x % H, split = blockIdx.x / H % pl.splits, b = blockIdx.x / (H * pl.splits);
  const int qt = pl.tiles - 1 - b % pl.tiles, s = pl.sorted ? seq_of_rank(c, a, b / pl.tiles) : b / pl.tiles;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), grp = lane / R, col = lane % R;
  // which rows are the wave's: neighbours work in turns on one SIMD, also where a tile is not full
  const int part = W == 8 ? (wave & 3) * 2 + (wave >> 2) : wave;
  const Seq q = load_seq(c, a, s);
  if (!q.ok) {
    if (split == 0 && h == 0 && qt == 0 && tid == 0) flag(c, s, RKC_CS_LENGTH);
    return;
  }
  const int M = q.n * G, m0 = qt * kRows;
  if (m0 >= M) return;
  const int last = (min(M, m0 + kRows) - 1) / G;
  const int c0 = split * pl.chunk, c1 = min(rows_end(a, q, s, last), c0 + pl.chunk);
  if (split && c0 >= c1) return;
  const int32_t* table = c.d_block_table + (int64_t)s * c.max_pages;
  const int shift = 31 - __builtin_clz(c.page_tokens), in_page = c.page_tokens - 1;

  const int m = min(m0 + R * part + col, M - 1), qi = m / G, qh = h * G + m % G;
  const bool mine = m0 + R * part + col < M, rows = m0 + R * part < M;
  const Scale f = load_scale(a);
  Row row = load_row(a, q, s, qi);
  const float slope = a.d_slope ? a.d_slope[qh] * kLog2e / f.post : 0.f;
  V8 qf[KC];
  {
    const T* p = (const T*)a.d_q + (q.row0 + qi) * a.q_row_stride + qh * a.q_head_stride + grp * 8;
#pragma unroll
    for (int k = 0; k < KC; k++) {
      qf[k] = *(const V8*)(p + 512 / R * k);
      if (f.negate) qf[k] = negated(qf[k]);
    }
  }
  const bool tree = a.d_parent != nullptr, drafts = tree && c1 > q.base;
  if (drafts || (tree && a.d_slope)) {
    tree_lines(c, a, q, s, h == 0 && qt == 0, lines, depths);  // of a cut sequence, only parts that reach the tree come here
    row.pos = q.base + depths[qi];
  }
  // slots that all of the wave's rows see, and slots that any of them, and of the workgroup's, sees
  int all_from = 0, any_from = 0;
  if (a.d_row_start) all_from = wave_max(row.start), any_from = wave_min(row.start);
  const int all_to = uni(row.end), pre = uni(row.prefix);  // a wave's first lane has its first row
  const int any_to = tree ? q.len : max(pre, __builtin_amdgcn_readlane(row.end, R - 1));
  if (lane == 0) lim[wave][0] = any_from, lim[wave][1] = any_to;
  __syncthreads();
  int g_any_from = lim[0][0], g_any_to = lim[0][1];
#pragma unroll
  for (int k = 1; k < W; k++) g_any_from = min(g_any_from, lim[k][0]), g_any_to = max(g_any_to, lim[k][1]);
  g_any_from = uni(g_any_from), g_any_to = uni(g_any_to);
  const int end = min(c1, g_any_to);

  const Pool kp = k_pool(c, h), vp = v_pool(c, h);

  float top = -kInf, sum = 0.f, lift = 0.f;  // lift: what all scores of a tile and lane are to lose yet
  acc o[DB];
#pragma unroll
  for (int d = 0; d < DB; d++)
#pragma unroll
    for (int k = 0; k < A; k++) o[d][k] = 0.f;

  const rkc_tiles<BK> tiles(c0, end, pre, g_any_from);
  const int n_tiles = tiles.n;
  auto slot_of = [&](int i) { return tiles.slot(i); };
  bool bad = false;
  // this thread's pieces of a tile: a wave's pieces of one load lie in 16 slots of one page
  const int lane_run = uni(tid / CH & ~15);
  auto key_in = [](int r, int c) { return R == 32 ? tile_at<D>(r, c) : keys16_at<D>(r, c); };
  auto val_in = [](int r, int c) { return R == 32 ? tile_at<D>(r, c) : vals16_at<D>(r, c); };
  // Of a piece in its run; the chunk is the one that the tile's layout has at its place.  A thread's pieces lie whole runs
  // apart, and the layouts repeat after 16 rows.
  static_assert(kThreads / CH % 16 == 0, "runs");
  const uint32_t r = threadIdx.x / CH;
  const uint32_t k_off = (r & 15) * kp.slot + (key_in(r, tid % CH) - r * D) * 2, v_off = (r & 15) * vp.slot + (val_in(r, tid % CH) - r * D) * 2;
  int page[P];  // of the next tile to be loaded
  auto run_of = [&](int t0, int p) {  // a run behind the end stands for the first one
    const int at = t0 + lane_run + p * kThreads / CH;
    return at < end ? at : t0;
  };
  auto look_up = [&](int i) {
    const int t0 = slot_of(i);
#pragma unroll
    for (int p = 0; p < P; p++) page[p] = page_of(table, shift, run_of(t0, p));
  };
  auto load = [&](int i, int buf) {
    const int t0 = slot_of(i);
    T* to = lds + buf * 2 * kTile + wave * 64 * 8;
#pragma unroll
    for (int p = 0; p < P; p++) {
      const int at = run_of(t0, p) & in_page;
      const int block = block_of(c, page[p], bad);
      dma(fixed(run_at(kp, block, at)) + k_off, to + p * kThreads * 8);
      dma(fixed(run_at(vp, block, at)) + v_off, to + kTile + p * kThreads * 8);
    }
  };
  // byte offsets of a lane's first key and first values of a tile; the others differ by an exclusive or (chunks along
  // a row) and by whole rows.  Element e = 4 x + y of a score block is slot 4 * (64 / R) x + 4 grp + y of its R.
  const int vi = lane & 15, vr = 4 * grp + (vi >> 2), vc = R == 32 ? (lane >> 4 & 1) * 2 + ((vi & 3) >> 1) : (vi & 3) >> 1, ve = (vi & 1) * 4;
  const int key_at = 2 * key_in(col, grp), val_at = 2 * (kTile + val_in(vr, vc) + ve);
  // whether any of the wave's rows sees anything of a tile, and whether all see all of it
  auto sees = [&](int t0) { return rows && ((t0 + BK > any_from && t0 < any_to) || t0 < pre); };
  auto keys = [&](int ka, int u, int k) { return *(const V8*)((const char*)lds + (ka ^ k * (1024 / R)) + 2 * R * D * u); };
  // values of the 512 / R slots of weight operand i, columns R d .. R d + R - 1
  auto vals = [&](int va, int i, int d) {
    const char* at = (const char*)lds + i * (512 / R) * 2 * D;
    const int x = va ^ d * 2 * R;
    if constexpr (R == 32) return read_tr2<T>(at + x, at + (x ^ 32) + 16 * D);
    else return read_tr2<T>(at + x, at + x + 32 * D);
  };
  auto scores = [&](acc(&sc)[KT], int buf) {
    const int ka = here(buf * 4 * kTile + key_at);
#pragma unroll
    for (int u = 0; u < KT; u++)
#pragma unroll
      for (int k = 0; k < A; k++) sc[u][k] = 0.f;
#pragma unroll
    for (int k = 0; k < KC; k++)
#pragma unroll
      for (int u = 0; u < KT; u++) sc[u] = mma(keys(ka, u, k), qf[k], sc[u]);
  };
  auto slot_in = [](int u, int k) { return R * u + (k & 3) + 256 / R * (k >> 2); };  // less 4 grp
  // cap, distance, masks, and the maximum that the weights refer to
  auto fold = [&](acc(&sc)[KT], uint32_t(&seen)[BK / 32], int t0) {
    const bool whole = t0 + BK <= pre || (t0 >= all_from && t0 + BK <= all_to);
    if (a.softcap > 0.f) cap_all(sc, f);
    if (a.d_slope && t0 + BK <= all_to) {  // all slots lie before all rows: the part that is the same for a row's slots waits
      lift = slope * (float)(row.pos - t0 - 4 * grp) * f.post;
#pragma unroll
      for (int u = 0; u < KT; u++)
#pragma unroll
        for (int k = 0; k < A; k++) sc[u][k] = __builtin_fmaf(slope, (float)slot_in(u, k), sc[u][k]);
    } else if (a.d_slope) {
      lift = 0.f;
      const int base_at = here(q.base - t0 - 4 * grp);
      const float far = (float)(here(row.pos - t0) - 4 * grp);
#pragma unroll
      for (int u = 0; u < KT; u++)
#pragma unroll
        for (int k = 0; k < A; k++) {
          const int j = slot_in(u, k);
          float gap = far - (float)j;
          if (drafts && t0 + BK > q.base) {
            const int i = j - base_at, d = depths[max(0, min(i, RKC_MAX_TREE_ROWS - 1))];
            gap = i >= 0 ? (float)(row.pos - q.base - d) : gap;
          }
          sc[u][k] = __builtin_fmaf(-slope, fabsf(gap), sc[u][k]);
        }
    }
#pragma unroll
    for (int x = 0; x < BK / 32; x++) seen[x] = 0xffffffff;
    if (!whole) {
#pragma unroll
      for (int x = 0; x < BK / 32; x++) {
        const int j0 = t0 + 32 * x;
        seen[x] = seen_of(row, j0, drafts ? line_window(lines[qi], 4, j0 - q.base) : 0) >> 4 * grp;
      }
#pragma unroll
      for (int u = 0; u < KT; u++)
#pragma unroll
        for (int k = 0; k < A; k++) sc[u][k] = masked(sc[u][k], seen[slot_in(u, k) / 32], slot_in(u, k) % 32);
    }
    float most = -kInf;
#pragma unroll
    for (int u = 0; u < KT; u++)
#pragma unroll
      for (int k = 0; k < A; k++) most = fmaxf(most, sc[u][k]);
    most = most * f.post - lift;
    most = R == 32 ? max32(most) : max32(max16(most));
    // weights up to 2^8 are let stand: the maximum moves, and the outputs are rescaled, in few tiles only
    if (__any(most > top + (8.f + kRoom<T>))) {
      const float now = fmaxf(top, most - kRoom<T>), by = now == -kInf ? 1.f : ex2(top - now);
      top = now, sum *= by;
#pragma unroll
      for (int d = 0; d < DB; d++) o[d] *= by;
    }
  };
  // Weight operand i.  The products' operands have the cache's type: the weights are rounded to it here, their sum is not.
  auto weights = [&](const acc(&sc)[KT], int i) {
    const float mx = (top == -kInf ? 0.f : top) + lift;
    f32x8 p;
#pragma unroll
    for (int k = 0; k < 8; k++) p[k] = ex2(__builtin_fmaf(sc[(8 * i + k) / A][(8 * i + k) % A], f.post, -mx));
    sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    return __builtin_convertvector(p, V8);
  };

  // One tile after the other, all waves in the same step of it.
  auto go_over = [&](auto with_care) {
    constexpr bool careful = decltype(with_care)::value;
    // kAhead tiles are on their way while one is worked on
    rkc_first_tiles<kAhead>(n_tiles, look_up, load);
    int buf = 0;
    for (int i = 0; i < n_tiles; i++) {
      const int t0 = slot_of(i);
      if constexpr (W == 4) {
        // of a CU's workgroups those that have most left go first (2 prompts of 4,096 tokens, 16 heads of 64 elements: 122 us
        // instead of 132)
        const int left = n_tiles - i;
        if (left >= 24) __builtin_amdgcn_s_setprio(3);
        else if (left >= 16) __builtin_amdgcn_s_setprio(2);
        else if (left >= 8) __builtin_amdgcn_s_setprio(1);
        else __builtin_amdgcn_s_setprio(0);
      }
      if (i + kAhead <= n_tiles) dma_barrier<2 * P * (kAhead - 1)>();
      else dma_barrier<0>();
      if (i + kAhead < n_tiles) load(i + kAhead, buf ? buf - 1 : kAhead);
      if (i + kAhead + 1 < n_tiles) look_up(i + kAhead + 1);
      T* tile_v = lds + buf * 2 * kTile + kTile;
      const int va = here(buf * 4 * kTile + val_at);
      bool hurt = false;
      if (t0 + BK > end || careful) {  // what lies behind the last slot that a row sees must not enter a product
        for (int k = tid; k < BK * CH; k += kThreads) {
          const int j = t0 + k / CH;
          V8* v = (V8*)(tile_v + 8 * k);
          if (j >= end || (j < g_any_from && j >= pre)) *v = __builtin_bit_cast(V8, u32x4{0, 0, 0, 0});
          else if constexpr (careful) hurt |= any_hurt<T>(__builtin_bit_cast(u32x4, *v));
        }
        if constexpr (careful) hurt = __syncthreads_or(hurt);
        else __syncthreads();
      }
      acc sc[KT];
      uint32_t seen[BK / 32];
      if (sees(t0)) {
        scores(sc, buf);
        fold(sc, seen, t0);
      }
      if constexpr (careful) if (hurt) {  // the same for the whole workgroup
        if (sees(t0)) {
#pragma unroll
          for (int d = 0; d < DB; d++) {
            acc n;
#pragma unroll
            for (int k = 0; k < A; k++) n[k] = 0.f;
#pragma unroll 1
            for (int x = 0; x < NP; x++) {
              const int j0 = 512 / R * x;
              const uint32_t bits = (BK > 32 && j0 >= 32 ? seen[BK / 32 - 1] : seen[0]) >> (j0 & 31);
              V8 by, vt = vals(va, x, d);
#pragma unroll
              for (int k = 0; k < 8; k++) by[k] = (T)(bits >> ((k & 3) + 256 / R * (k >> 2)) & 1 ? 1.f : 0.f);
              n = mma(strip<T>(vt), by, n);
            }
#pragma unroll
            for (int k = 0; k < A; k++) o[d][k] += hurt_by(n[k]);
          }
        }
        __syncthreads();
        for (int k = tid; k < kTile / 8; k += kThreads) {
          V8 v = *(const V8*)(tile_v + 8 * k);
          strip<T>(v);
          *(V8*)(tile_v + 8 * k) = v;
        }
        __syncthreads();
      }
      if (sees(t0)) {
#pragma unroll
        for (int x = 0; x < NP; x++) {
          const V8 pb = weights(sc, x);
#pragma unroll
          for (int d = 0; d < DB; d++) o[d] = mma(vals(va, x, d), pb, o[d]);
        }
      }
      buf = buf == kAhead ? 0 : buf + 1;
    }
  };

  // Two waves to a SIMD in turns: while one multiplies (the next tile's scores and this one's outputs), the other
  // works on its scores.  Steps are numbered over the workgroup; the second four waves are one step behind.  Step
  // 2 i needs tile i and leaves the place of tile i - 2 to tile i + 2.
  auto in_turns = [&] {
    static_assert(W != 8 || kAhead == 3, "four places");
    const bool behind = wave >= 4;
    rkc_first_tiles<2>(n_tiles, look_up, load);
    auto even = [&](int i) {
      if (i + 1 < n_tiles) dma_barrier<2 * P>();
      else dma_barrier<0>();
      if (i + 2 < n_tiles) load(i + 2, i + 2 & 3);
      if (i + 3 < n_tiles) look_up(i + 3);
      __builtin_amdgcn_sched_barrier(0);
    };
    auto odd = [&] {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    acc sc[KT];
    V8 pb[NP];
    bool had = false;  // weights of the tile before are there
    auto outputs = [&](int i) {
      const int va = here((i & 3) * 4 * kTile + val_at);
#pragma unroll
      for (int x = 0; x < NP; x++)
#pragma unroll
        for (int d = 0; d < DB; d++) o[d] = mma(vals(va, x, d), pb[x], o[d]);
    };
    auto multiply = [&](int i) {
      const bool has = i < n_tiles && sees(slot_of(i));
      if (has && had) {
        scores(sc, i & 3);
        outputs(i - 1);
        // operands a few products ahead of their use
        {
          __builtin_amdgcn_sched_group_barrier(0x100, 12, 0);
#pragma unroll
          for (int k = 0; k < KT * KC + NP * DB; k++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          }
        }
      } else if (has) {
        scores(sc, i & 3);
      } else if (had) {
        outputs(i - 1);
      }
      had = has;
      __builtin_amdgcn_sched_barrier(0);
    };
    auto weigh = [&](int i) {
      const int t0 = slot_of(i);
      if (had) {
        uint32_t seen[BK / 32];
        fold(sc, seen, t0);
#pragma unroll
        for (int x = 0; x < NP; x++) pb[x] = weights(sc, x);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    // What lies behind the last slot that a row sees must not enter a product: zeroed by the second waves at step 2 i,
    // the first ones multiply with it from step 2 i + 2 on.
    auto blank = [&](int i) {
      const int t0 = slot_of(i);
      if (t0 + BK <= end) return;
      T* tile_v = lds + (i & 3) * 2 * kTile + kTile;
      for (int k = tid - kThreads / 2; k < BK * CH; k += kThreads / 2) {
        const int j = t0 + k / CH;
        if (j >= end || (j < g_any_from && j >= pre)) *(u32x4*)(tile_v + 8 * k) = u32x4{0, 0, 0, 0};
      }
    };
    if (!behind) {
      for (int i = 0; i <= n_tiles; i++) {
        even(i);
        multiply(i);
        odd();
        if (i < n_tiles) weigh(i);
      }
    } else {
      even(0);
      if (n_tiles) blank(0);
      for (int i = 0; i <= n_tiles; i++) {
        odd();
        multiply(i);
        if (i < n_tiles) {
          even(i + 1);
          if (i + 1 < n_tiles) blank(i + 1);
          weigh(i);
        }
      }
    }
    __syncthreads();
  };
  if constexpr (W == 8) in_turns();
  else go_over(std::false_type());
  // A value that is not finite reaches rows that do not see its slot, through a weight of zero.  That shows in the
  // outputs, and then all is done once more with care.
  float odd = 0.f;  // stays 0 unless an output is not finite
#pragma unroll
  for (int d = 0; d < DB; d++)
#pragma unroll
    for (int k = 0; k < A; k++) odd = __builtin_fmaf(o[d][k], 0.f, odd);
  if (__syncthreads_or(odd != 0.f)) {
    top = -kInf, sum = 0.f;
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int k = 0; k < A; k++) o[d][k] = 0.f;
    go_over(std::true_type());
  }
  if (bad) flag(c, s, RKC_CS_BLOCK);

  sum = R == 32 ? sum32(sum) : sum32(sum16(sum));
  if (!mine) return;
  typedef T T4 __attribute__((ext_vector_type(4)));
  if (pl.splits == 1) {
    const float by = 1.f / sum;
    T* to = (T*)a.d_out + (q.row0 + qi) * a.out_row_stride + qh * a.out_head_stride + 4 * grp;
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int k = 0; k < A / 4; k++) {
        f32x4 x = f32x4{o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]} * by;
        if (sum == 0.f) x = f32x4{0.f, 0.f, 0.f, 0.f};
        *(T4*)(to + R * d + 256 / R * k) = __builtin_convertvector(x, T4);
      }
    if (grp == 0) a.d_lse[(int64_t)(q.row0 + qi) * a.q_heads + qh] = sum == 0.f ? -kInf : kLn2 * (top + lg2(sum));
  } else {
    const int64_t at = ((int64_t)((s * H + h) * pl.tiles + qt) * pl.splits + split) * kRows + R * part + col;
    float* to = (float*)((char*)a.d_scratch + pl.part_at) + at * D + 4 * grp;
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int k = 0; k < A / 4; k++) *(f32x4*)(to + R * d + 256 / R * k) = f32x4{o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]};
    float* st = (float*)((char*)a.d_scratch + pl.stat_at) + at * 2;
    if (grp == 0) st[0] = top, st[1] = sum;
  }
}

template <typename T, int D, int W, int R>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  attend_tile<T, D, W, R><<<dim3(p->units * p->splits), dim3(64 * W), 0, s>>>(*c, *a, *p);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

template <typename T>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  if (c->head_dim == 256) return go<T, 256, 8, 16>(c, a, p, s);
  if (c->head_dim == 128) return p->rows == 256 ? go<T, 128, 8, 32>(c, a, p, s) : go<T, 128, 4, 32>(c, a, p, s);
  return go<T, 64, 4, 32>(c, a, p, s);
}

}  // namespace

rkc_status rkc_attend_tile(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  return c->dtype == RKC_BF16 ? go<__bf16>(c, a, p, s) : go<_Float16>(c, a, p, s);
}

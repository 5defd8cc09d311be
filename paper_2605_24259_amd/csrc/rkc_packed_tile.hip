// rkc_packed_tile.hip -- attention of many rows over a paged cache in 4 bits (chunks of prompts, larger trees).
//
// out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m) in one pass over the slots, m the running maximum of a row's scores.
// A workgroup of W waves holds 32 W packed rows (rows x query heads of one key/value head), 32 of them in each wave as the
// columns of its matrix products, and goes over the slots that any of them sees in tiles of 64 (32 at 256 elements a
// head).  A tile's codes and scales are loaded ahead into registers, a thread's part of it each, and converted once for all
// waves into 16 bits in LDS, while the tile before is worked on.  Tiles that every row sees skip the masks, waves whose rows see
// nothing of a tile skip it.
//   128 rows: 4 waves, a barrier a tile (go_over)
//   256 rows: 8 waves in two groups that multiply and weigh in turns (in_turns), at 128 and 256 elements a head
// A marked slot's scores are NaN by its key's first scale, and so only the rows that see it; values are always finite.
// The products take 16-bit operands: the matrix units' own products of 4 bits cut what lies 2^13 below the largest of 16
// neighbouring products, which a score of 32 bits must not lose.
// What bounds it: without a cap a step's products wait for their operands from LDS (1,500 cycles of the 1,040 that the matrix
// units need), and the weights take as long beside them: 2,048 rows of 32 heads over 32,768 slots (8 heads of 128 elements)
// 939 us, 1,134 TFLOP/s, 0.92 of a large matrix product's rate; with a cap the weights' instructions, 1,147 us.  At 256
// elements 2,048 rows of 16 heads over 16,384 slots take 632 us, 816 TFLOP/s; two prompts of 4,096 tokens, 16 heads of 64, 100 us.
#include <type_traits>

#include "rkc_packed_dev.h"
#include "rkc_tiles.h"

namespace {

template <typename T, int D, int W>
__global__ __launch_bounds__(64 * W, D == 64 ? 3 : D == 256 && W == 4 ? 1 : 2) void packed_tile(const rkc_cache c, const rkc_attention a, const rkc_plan pl) {
  typedef typename Vec8<T>::t V8;
  // 32 rows a wave: products of 32 x 32, A elements a lane; tiles of BK slots
  typedef f32x16 acc;
  constexpr int A = 16, kRows = 32 * W, kThreads = 64 * W;
  constexpr int BK = D == 256 ? 32 : 64;
  constexpr int KT = BK / 32, KC = D / 16, DB = D / 32, NP = KT * 2;  // score blocks, key operands, output blocks, weight operands
  constexpr int E = BK * D / kThreads, PER = D / E, NC = E / 8;  // elements of a key, and of a value, per thread; threads of a slot; dwords
  constexpr int kTile = BK * D;
  __shared__ __attribute__((aligned(16))) T lds[2 * 2 * kTile];  // K and V of two tiles
  __shared__ uint64_t lines[RKC_MAX_TREE_ROWS][4];
  __shared__ int depths[RKC_MAX_TREE_ROWS], lim[W][2];

  const int H = c.kv_heads, G = a.q_heads / H;
  // Heads first: with 8 of them each XCD has one, and its cache that head's keys and values for the row tiles of a
  // sequence, which are neighbours; the rows that see most go first.  (Heads last: 40 trees over 700 to 8,192 slots 274 us instead
  // of 217, two prompts of 4,096 tokens in documents 152 instead of 130.  Sequences before row tiles: 24 chunks of up to 512 rows 226
  // instead of 183, the documents 150; but two whole prompts, 16 heads of 64 elements, 91 instead of 102.)
  const int h = blockIdx.x % H, split = blockIdx.x / H % pl.splits, b = blockIdx.x / (H * pl.splits);
  const int qt = pl.tiles - 1 - b % pl.tiles, s = pl.sorted ? seq_of_rank(c, a, b / pl.tiles) : b / pl.tiles;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), grp = lane / 32, col = lane % 32;
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

  const int m = min(m0 + 32 * part + col, M - 1), qi = m / G, qh = h * G + m % G;
  const bool mine = m0 + 32 * part + col < M, rows = m0 + 32 * part < M;
  const Scale f = load_scale(a);
  Row row = load_row(a, q, s, qi);
  const float slope = a.d_slope ? a.d_slope[qh] * kLog2e / f.post : 0.f;
  V8 qf[KC];
  {
    const T* p = (const T*)a.d_q + (q.row0 + qi) * a.q_row_stride + qh * a.q_head_stride + grp * 8;
#pragma unroll
    for (int k = 0; k < KC; k++) {
      qf[k] = *(const V8*)(p + 16 * k);
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
  const int any_to = tree ? q.len : max(pre, __builtin_amdgcn_readlane(row.end, 31));
  if (lane == 0) lim[wave][0] = any_from, lim[wave][1] = any_to;
  __syncthreads();
  int g_any_from = lim[0][0], g_any_to = lim[0][1];
#pragma unroll
  for (int k = 1; k < W; k++) g_any_from = min(g_any_from, lim[k][0]), g_any_to = max(g_any_to, lim[k][1]);
  g_any_from = uni(g_any_from), g_any_to = uni(g_any_to);
  const int end = min(c1, g_any_to);

  const Codes held = codes_of<D>(c, h);

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
  // this thread's part of a tile: a wave's parts lie in 16 slots of one page
  static_assert(64 / PER <= 16, "runs");
  const int lane_run = uni(tid / PER & ~15);
  // What follows from the thread's number is found anew where it is used, where 256 registers are not enough to keep it.
  auto self = [&] { return D == 256 && W == 8 ? here(tid) : tid; };
  typedef uint32_t codes_t __attribute__((ext_vector_type(NC)));
  codes_t kf, vf;   // of the next tile
  uint32_t ks, vs;
  int page;         // of the one behind it
  auto run_of = [&](int t0) {  // a run behind the end stands for the first one
    const int at = t0 + lane_run;
    return at < end ? at : t0;
  };
  auto look_up = [&](int i) { page = page_of(table, shift, run_of(slot_of(i))); };
  auto load = [&](int i) {
    const int at = run_of(slot_of(i)) & in_page;
    const char* b = held.base + (uint64_t)(uint32_t)block_of(c, page, bad) * held.block;
    const char* kb = b + at * (D / 2);
    const char* sb = b + held.key_scales + at * (D / 32);
    const int t = self() & (16 * PER - 1), c_off = t * (E / 2), s_off = t / PER * (D / 32) + t % PER * E / 32;
    kf = from_global<codes_t>(kb, c_off), vf = from_global<codes_t>(kb + held.values, c_off);
    ks = from_global<uint8_t>(sb, s_off), vs = from_global<uint8_t>(sb + (held.value_scales - held.key_scales), s_off);
  };
  // byte offset of this thread's part in a tile
  auto put_at = [&] {
    const int t = self();
    return 2 * tile_at<D>(t / PER, t % PER * NC);
  };
  auto put_keys = [&](int buf) {
    const int at = here(put_at() + buf * 4 * kTile);
    const float f = scale_float(ks);
#pragma unroll
    for (int k = 0; k < NC; k++) *(u32x4*)((char*)lds + (at ^ k << 4)) = unpack8<T>(kf[k], f);
  };
  // a scale that nobody wrote may be anything: what no row sees is to be finite
  auto put_values = [&](int buf, const codes_t& codes, uint32_t scale) {
    const int at = here(put_at() + 2 * kTile + buf * 4 * kTile);
    const float f = scale_float(min(scale, (uint32_t)kTopScale<T>));
#pragma unroll
    for (int k = 0; k < NC; k++) *(u32x4*)((char*)lds + (at ^ k << 4)) = unpack8<T>(codes[k], f);
  };
  // Byte offsets of a lane's first key and first values of a tile; the others differ by an exclusive or (chunks along a row) and
  // by whole rows.  Element e = 4 x + y of a score block is slot 8 x + 4 grp + y of its 32.
  auto key_at = [&] {
    const int t = self() & 63;
    return 2 * tile_at<D>(t % 32, t / 32);
  };
  auto val_at = [&] {
    const int t = self() & 63, i = t & 15;
    return 2 * (kTile + tile_at<D>(4 * (t / 32) + (i >> 2), (t >> 4 & 1) * 2 + ((i & 3) >> 1)) + (i & 1) * 4);
  };
  // whether any of the wave's rows sees anything of a tile, and whether all see all of it
  auto sees = [&](int t0) { return rows && ((t0 + BK > any_from && t0 < any_to) || t0 < pre); };
  auto keys = [&](int ka, int u, int k) { return *(const V8*)((const char*)lds + (ka ^ k * 32) + 64 * D * u); };
  // values of the 16 slots of weight operand i, columns 32 d .. 32 d + 31
  auto vals = [&](int va, int i, int d) {
    const char* at = (const char*)lds + i * 32 * D;
    const int x = va ^ d * 64;
    return read_tr2<T>(at + x, at + (x ^ 32) + 16 * D);
  };
  auto scores = [&](acc(&sc)[KT], int buf) {
    const int ka = here(buf * 4 * kTile + key_at());
#pragma unroll
    for (int u = 0; u < KT; u++)
#pragma unroll
      for (int k = 0; k < A; k++) sc[u][k] = 0.f;
#pragma unroll
    for (int k = 0; k < KC; k++)
#pragma unroll
      for (int u = 0; u < KT; u++) sc[u] = mma(keys(ka, u, k), qf[k], sc[u]);
  };
  // A cap without a distance stays -1 / (exp(2 y) + 1), half of tanh(y) less a half: the exponent's factor and the maximum take
  // up the rest, which saves an operation a score.
  const bool short_cap = a.softcap > 0.f && !f.far && !a.d_slope;
  const float times = short_cap ? 2.f * f.post : f.post, plus = short_cap ? f.post : 0.f;
  auto each = [](acc(&sc)[KT], auto f) {
#pragma unroll
    for (int u = 0; u < KT; u++)
#pragma unroll
      for (int k = 0; k < A; k++) sc[u][k] = f(sc[u][k]);
  };
  auto slot_in = [](int u, int k) { return 32 * u + (k & 3) + 8 * (k >> 2); };  // less 4 grp
  // cap, distance, masks, and the maximum that the weights refer to
  auto fold = [&](acc(&sc)[KT], int t0) {
    const bool whole = t0 + BK <= pre || (t0 >= all_from && t0 + BK <= all_to);
    if (short_cap) {
      each(sc, [&](float y) { return ex2(y * f.pre); });
      each(sc, [&](float y) { return __builtin_amdgcn_rcpf(-1.f - y); });
    } else if (a.softcap > 0.f) {
      cap_all(sc, f);
    }
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
    if (!whole) {
      uint32_t seen[BK / 32];
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
    most = __builtin_fmaf(most, times, plus) - lift;
    most = max32(most);
    // weights up to 2^8 are let stand: the maximum moves, and the outputs are rescaled, in few tiles only
    if (__any(most > top + (8.f + kRoom<T>))) {
      const float now = fmaxf(top, most - kRoom<T>), by = now == -kInf ? 1.f : ex2(top - now);
      top = now, sum *= by;
#pragma unroll
      for (int d = 0; d < DB; d++) o[d] *= by;
    }
  };
  // Weight operand i.  The products' operands have the cache's type: the weights are rounded to it here, their sum is not.  (As the sum
  // of two operands, with a second product each, outputs are as near as 16 bits can be: 0.0017 of their size off, root mean square,
  // instead of 0.0021 to 0.0023 in bfloat16.  But the products are what bounds the kernel: 2,048 rows of 32 heads over 32,768 slots 1,330 us
  // instead of 970, with a cap 1,556 instead of 1,187; 40 trees over 700 to 8,192 slots 277 instead of 216.)
  auto weights = [&](const acc(&sc)[KT], int i) {
    const float mx = (top == -kInf ? 0.f : top) + lift - plus;
    f32x8 p;
#pragma unroll
    for (int k = 0; k < 8; k++) p[k] = ex2(__builtin_fmaf(sc[(8 * i + k) / A][(8 * i + k) % A], times, -mx));
    sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    return __builtin_convertvector(p, V8);
  };

  // One tile after the other, all waves in the same step of it.
  auto go_over = [&] {
    if (n_tiles > 0) {
      look_up(0);
      load(0);
      if (n_tiles > 1) look_up(1);
      put_keys(0), put_values(0, vf, vs);
      if (n_tiles > 1) load(1);
      if (n_tiles > 2) look_up(2);
    }
    for (int i = 0; i < n_tiles; i++) {
      const int t0 = slot_of(i), buf = i & 1;
      if constexpr (D < 256) {
        // of a CU's workgroups those that have most left go first (2 prompts of 4,096 tokens, 16 heads of 64 elements: 102 us
        // instead of 114)
        const int left = n_tiles - i;
        if (left >= 24) __builtin_amdgcn_s_setprio(3);
        else if (left >= 16) __builtin_amdgcn_s_setprio(2);
        else if (left >= 8) __builtin_amdgcn_s_setprio(1);
        else __builtin_amdgcn_s_setprio(0);
      }
      __syncthreads();  // tile i is in LDS, and no wave reads tile i - 1 any more
      const int va = here(buf * 4 * kTile + val_at());
      acc sc[KT];
      const bool has = sees(t0);
      if (has) scores(sc, buf);
      if (has) {
        fold(sc, t0);
#pragma unroll
        for (int x = 0; x < NP; x++) {
          const V8 pb = weights(sc, x);
#pragma unroll
          for (int d = 0; d < DB; d++) o[d] = mma(vals(va, x, d), pb, o[d]);
        }
      }
      if (i + 1 < n_tiles) {
        put_keys(buf ^ 1), put_values(buf ^ 1, vf, vs);
        if (i + 2 < n_tiles) load(i + 2);
        if (i + 3 < n_tiles) look_up(i + 3);
      }
    }
  };

  // Two waves to a SIMD in turns: while one multiplies (a tile's scores and the outputs of the one before), the other works on
  // its scores.  The second four waves are one step behind.  A tile's keys are read in the two steps from step 2 i on, its
  // values in the two behind them; so while tile i is multiplied, the keys of tile i + 1 and the values of tile i are put.
  auto in_turns = [&] {
    const bool behind = wave >= 4;
    // Where a tile is converted and put, and the one behind it loaded: behind a step's products, which wait for LDS rather than
    // for the wave's instructions; the loads, in scalar instructions for the most part, go with the weights unless a cap makes
    // those the longer part (exchanged, 3 % slower without a cap and with one).  At 256 elements a head, where some
    // registers are kept in memory and are waited for behind the loads, all of it goes before the weights (637 us for 2,048 rows
    // of 16 heads over 16,384 slots, 857 behind the products).
    constexpr bool early = D == 256;
    const bool with_products = a.softcap > 0.f;
    codes_t held_v;
    uint32_t held_s;
    auto take = [&](int i) {
      if (i < n_tiles) load(i);
      if (i + 1 < n_tiles) look_up(i + 1);
    };
    auto put = [&](int i) {
      if (i + 1 < n_tiles) put_keys(i + 1 & 1);
      if (i < n_tiles) put_values(i & 1, held_v, held_s);
      held_v = vf, held_s = vs;
      if (early) take(i + 2);
    };
    if (n_tiles) {
      look_up(0);
      take(0);
      put_keys(0);
      held_v = vf, held_s = vs;
      take(1);
    }
    auto step = [&] {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    acc sc[KT];
    V8 pb[NP];
    bool had = false;  // weights of the tile before are there
    auto outputs = [&](int i) {
      const int va = here((i & 1) * 4 * kTile + val_at());
#pragma unroll
      for (int x = 0; x < NP; x++)
#pragma unroll
        for (int d = 0; d < DB; d++) o[d] = mma(vals(va, x, d), pb[x], o[d]);
    };
    // Operands a few products ahead of their use: one read a key, two a value (12 ahead and two of either: 2,048 rows over 32,768
    // slots 989 us instead of 975, 16 ahead 1,213).
    auto feed = [](int keys, int values) {
      __builtin_amdgcn_sched_group_barrier(0x100, D == 256 ? 12 : 6, 0);
#pragma unroll
      for (int k = 0; k < keys + values; k++) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (D < 256 && k < keys) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        else __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
    };
    auto multiply = [&](int i) {
      const bool has = i < n_tiles && sees(slot_of(i));
      if (has && had) {
        scores(sc, i & 1);
        outputs(i - 1);
        feed(KT * KC, NP * DB);
      } else if (has) {
        scores(sc, i & 1);
        feed(KT * KC, 0);
      } else if (had) {
        outputs(i - 1);
        feed(0, NP * DB);
      }
      had = has;
      __builtin_amdgcn_sched_barrier(0);
    };
    auto weigh = [&](int i) {
      if (!early) {
        if (!with_products && i + 2 < n_tiles) load(i + 2);
        if (i + 3 < n_tiles) look_up(i + 3);
      }
      if (had) {
        fold(sc, slot_of(i));
#pragma unroll
        for (int x = 0; x < NP; x++) pb[x] = weights(sc, x);
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    // products at a higher priority: the other wave of the SIMD has instructions for every cycle
    auto turn = [&](int i) {
      step();
      __builtin_amdgcn_s_setprio(2);
      multiply(i);
      if (!early && i < n_tiles) {
        put(i);
        if (with_products && i + 2 < n_tiles) load(i + 2);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    if (!behind) {
      for (int i = 0; i <= n_tiles; i++) {
        turn(i);
        step();
        if (i < n_tiles) {
          if (early) put(i);
          weigh(i);
        }
      }
    } else {
      step();
      if (early && n_tiles) put(0);
      for (int i = 0; i <= n_tiles; i++) {
        turn(i);
        if (i < n_tiles) {
          step();
          if (early && i + 1 < n_tiles) put(i + 1);
          weigh(i);
        }
      }
    }
    __syncthreads();
  };
  if constexpr (W == 8) in_turns();
  else go_over();
  if (bad) flag(c, s, RKC_CS_BLOCK);

  sum = sum32(sum);
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
        *(T4*)(to + 32 * d + 8 * k) = __builtin_convertvector(x, T4);
      }
    if (grp == 0) a.d_lse[(int64_t)(q.row0 + qi) * a.q_heads + qh] = sum == 0.f ? -kInf : kLn2 * (top + lg2(sum));
  } else {
    const int64_t at = ((int64_t)((s * H + h) * pl.tiles + qt) * pl.splits + split) * kRows + 32 * part + col;
    float* to = (float*)((char*)a.d_scratch + pl.part_at) + at * D + 4 * grp;
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int k = 0; k < A / 4; k++) *(f32x4*)(to + 32 * d + 8 * k) = f32x4{o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]};
    float* st = (float*)((char*)a.d_scratch + pl.stat_at) + at * 2;
    if (grp == 0) st[0] = top, st[1] = sum;
  }
}

template <typename T, int D, int W>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  packed_tile<T, D, W><<<dim3(p->units * p->splits), dim3(64 * W), 0, s>>>(*c, *a, *p);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

template <typename T>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  if (c->head_dim == 256) return p->rows == 256 ? go<T, 256, 8>(c, a, p, s) : go<T, 256, 4>(c, a, p, s);
  if (c->head_dim == 128) return p->rows == 256 ? go<T, 128, 8>(c, a, p, s) : go<T, 128, 4>(c, a, p, s);
  return go<T, 64, 4>(c, a, p, s);
}

}  // namespace

rkc_status rkc_packed_tile(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  return c->dtype == RKC_BF16 ? go<__bf16>(c, a, p, s) : go<_Float16>(c, a, p, s);
}

// rkc_weigh.hip -- the account of a cache: how much attention each of its slots received.
//
// weight_j = decay * before_j + sum over rows of exp(x_j - lse).  Softmax sums are given, so slots are independent: a
// wave holds the keys of 32 slots in registers as columns of 16x16x32 products, with those of its next 32 on their way,
// and goes over the packed rows, whose queries lie in LDS, 16 at a time; a lane adds up the weights of its slot's column
// in 32 bits, in a fixed order.  One read of the keys; no atomics.  What bounds it: the read of the keys, with the
// products and an exponential for every row and slot in between (32 rows of 32 heads, 8 heads of 128 elements: 32
// sequences of 8,192 slots 146 us, 3.9 TB/s, 470 TFLOP/s; 8 of 6,000 to 16,384 60 us, 3.6 TB/s).  Four workgroups a CU
// hide the latency between those: with the lines of trees always in LDS there was room for three, 178 us instead of 146.
// Of more than 128 packed rows the queries are staged anew for each turn of 128 slots, behind two barriers each, and bound
// it: 1,024 rows of 32 heads over each of two prompts of 8,192 slots 318 us, 405 TFLOP/s; a whole prompt of 4,096 tokens,
// which has 128 workgroups, 1,036 us, 66 TFLOP/s of what its rows see.
#include "rkc_cache_dev.h"

namespace {

constexpr int kThreads = 256, kRuns = 2, kSlots = 16 * kRuns, kTurn = kThreads / 64 * kSlots;
constexpr int kBlock = 128;  // packed rows whose queries, masks and sums lie in LDS at a time
static_assert(kThreads == RKC_MAX_TREE_ROWS, "tree_lines");
constexpr int kTreeBytes = RKC_MAX_TREE_ROWS * 36;  // lines and depths

struct RowIn {
  int start, end, pos, line;
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 2 : 4) void weigh(const rkc_cache c, const rkc_attention a, int chunks, int turns) {
  typedef typename Vec8<T>::t V8;
  constexpr int KC = D / 32;
  __shared__ __attribute__((aligned(16))) T rows_q[kBlock * D];
  __shared__ __attribute__((aligned(16))) float lse2[kBlock], slopes[kBlock];
  __shared__ RowIn in[kBlock];
  extern __shared__ __attribute__((aligned(16))) char of_trees[];  // kTreeBytes where there are trees
  uint64_t(*const lines)[4] = (uint64_t(*)[4])of_trees;
  int* const depths = (int*)(of_trees + RKC_MAX_TREE_ROWS * 32);

  const int H = c.kv_heads, G = a.q_heads / H;
  const int h = blockIdx.x % H, part = blockIdx.x / H % chunks, s = blockIdx.x / (H * chunks);
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), quad = lane >> 4, col = lane & 15;
  const Seq q = load_seq(c, a, s);
  if (!q.ok) {
    if (part == 0 && h == 0 && tid == 0) flag(c, s, RKC_CS_LENGTH);
    return;
  }
  const int w0 = part * turns * kTurn;
  if (w0 >= q.len) return;
  const int n_turns = min(turns, (q.len - w0 + kTurn - 1) / kTurn), M = q.n * G;
  const int32_t* table = c.d_block_table + (int64_t)s * c.max_pages;
  const int shift = 31 - __builtin_clz(c.page_tokens), in_page = c.page_tokens - 1;
  const Pool kp = k_pool(c, h);
  const uint32_t k_off = col * kp.slot + quad * 16;
  bool bad = false;
  V8 next[kRuns][KC];
  auto load = [&](int turn) {
#pragma unroll
    for (int u = 0; u < kRuns; u++) {
      const int at = min(w0 + turn * kTurn + wave * kSlots + 16 * u, (q.len - 1) & ~15);
      const char* kb = run_at(kp, block_of(c, page_of(table, shift, at), bad), at & in_page);
#pragma unroll
      for (int k = 0; k < KC; k++) next[u][k] = *(const V8*)(kb + k_off + 64 * k);
    }
  };
  load(0);
  const bool tree = a.d_parent != nullptr;
  const bool drafts = tree && w0 + n_turns * kTurn > q.base;
  if (drafts || (tree && a.d_slope)) tree_lines(c, a, q, s, h == 0, lines, depths);  // only parts that reach the tree come here
  const int pre = a.d_prefix ? max(0, min(word(a.d_prefix, s), tree ? q.base : q.len)) : 0;
  const Scale sc = load_scale(a);

  // queries, sums and masks of up to kBlock packed rows from row mb on
  int rows = 0, all_from = 0, all_to = 0, any_from = 0, any_to = 0;  // what all of them see, and what any sees
  auto stage = [&](int mb) {
    __syncthreads();
    rows = min(kBlock, M - mb);
    const int rows_up = (rows + 15) & ~15;
    for (int x = tid; x < rows_up * (D / 8); x += kThreads) {
      const int r = x / (D / 8), m = min(mb + r, M - 1), qi = m / G;
      V8 v = *(const V8*)((const T*)a.d_q + (q.row0 + qi) * a.q_row_stride + (h * G + m - qi * G) * a.q_head_stride + x % (D / 8) * 8);
      *(V8*)(rows_q + keys16_at<D>(r, x % (D / 8))) = sc.negate ? negated(v) : v;
    }
    if (tid < rows_up) {
      const int m = mb + tid;
      RowIn r = {0x7fffffff, 0, 0, 0};
      float z = kInf, sl = 0.f;
      if (m < M) {
        const int qi = m / G, qh = h * G + m - qi * G;
        const Row w = load_row(a, q, s, qi);
        const float lse = a.d_lse[(int64_t)(q.row0 + qi) * a.q_heads + qh];
        z = lse == -kInf ? kInf : lse * kLog2e;  // a row that saw nothing gave nothing
        if (a.d_slope) sl = a.d_slope[qh] * kLog2e / sc.post;
        r.start = w.start, r.end = w.end, r.line = qi;
        r.pos = tree && a.d_slope ? q.base + depths[qi] : w.pos;
      }
      in[tid] = r, lse2[tid] = z, slopes[tid] = sl;
    }
    __syncthreads();
    all_from = any_from = 0;
    if (a.d_row_start) {
      const int e0 = lane < rows ? lane : 0, e1 = lane + 64 < rows ? lane + 64 : 0;
      all_from = wave_max(max(in[e0].start, in[e1].start)), any_from = wave_min(min(in[e0].start, in[e1].start));
    }
    all_to = uni(in[0].end), any_to = tree ? q.len : uni(in[rows - 1].end);
  };
  if (M > 0 && M <= kBlock) stage(0);

  for (int turn = 0; turn < n_turns; turn++) {
    const int t0 = w0 + turn * kTurn + wave * kSlots;
    V8 kf[kRuns][KC];
#pragma unroll
    for (int u = 0; u < kRuns; u++)
#pragma unroll
      for (int k = 0; k < KC; k++) kf[u][k] = next[u][k];
    if (turn + 1 < n_turns) load(turn + 1);
    float acc[kRuns] = {};
    for (int mb = 0; mb < M; mb += kBlock) {
      if (M > kBlock) stage(mb);
      if (!((t0 + kSlots > any_from && t0 < any_to) || t0 < pre) || t0 >= q.len) continue;
      const bool whole = t0 + kSlots <= pre || (t0 >= all_from && t0 + kSlots <= all_to);
      for (int m0 = 0; m0 < rows; m0 += 16) {
        const int rm = m0 + quad * 4;  // rows of this lane's four elements of a product
        V8 qf[KC];
#pragma unroll
        for (int k = 0; k < KC; k++) qf[k] = *(const V8*)(rows_q + keys16_at<D>(m0 + col, 4 * k + quad));
        const f32x4 z = *(const f32x4*)(lse2 + rm);  // rows behind the last one have a sum of infinity
        f32x4 x[kRuns];
#pragma unroll
        for (int u = 0; u < kRuns; u++) {
          x[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < KC; k++) x[u] = mma16(qf[k], kf[u][k], x[u]);
        }
        if (a.softcap > 0.f) cap_all(x, sc);
        if (a.d_slope) {
          const f32x4 sl = *(const f32x4*)(slopes + rm);
#pragma unroll
          for (int u = 0; u < kRuns; u++) {
            int j = t0 + 16 * u + col;
            if (drafts && j >= q.base) j = q.base + depths[min(j - q.base, RKC_MAX_TREE_ROWS - 1)];
#pragma unroll
            for (int e = 0; e < 4; e++) x[u][e] = __builtin_fmaf(-sl[e], fabsf((float)(in[rm + e].pos - j)), x[u][e]);
          }
        }
#pragma unroll
        for (int u = 0; u < kRuns; u++)
#pragma unroll
          for (int e = 0; e < 4; e++) x[u][e] = ex2(__builtin_fmaf(x[u][e], sc.post, -z[e]));
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 4; e++) {
            const RowIn r = in[rm + e];
#pragma unroll
            for (int u = 0; u < kRuns; u++) {
              const int j = t0 + 16 * u + col;
              bool see = (j >= r.start && j < r.end) || j < pre;
              if (drafts && j >= q.base) {
                const int d = min(j - q.base, RKC_MAX_TREE_ROWS - 1);
                see |= lines[r.line][d >> 6] >> (d & 63) & 1;
              }
              x[u][e] = see && z[e] != kInf ? x[u][e] : 0.f;
            }
          }
        }
#pragma unroll
        for (int u = 0; u < kRuns; u++) acc[u] += (x[u][0] + x[u][1]) + (x[u][2] + x[u][3]);
      }
    }
#pragma unroll
    for (int u = 0; u < kRuns; u++) {
      const float got = sum32(sum16(acc[u]));
      const int j = t0 + 16 * u + col;
      if (quad == 0 && j < q.len) {
        const int64_t at = s * a.weight_seq_stride + h * a.weight_head_stride + j;
        a.d_weight[at] = (a.d_weight_in ? a.decay * a.d_weight_in[at] : 0.f) + got;
      }
    }
  }
  if (bad) flag(c, s, RKC_CS_BLOCK);
}

struct Cut {
  int turns, chunks;
  int64_t workgroups;
};

// A workgroup keeps its queries for as many turns as leave four workgroups a CU, at most for one turn per 8 packed
// rows: few rows are staged quickly, and short turns even out sequences of unlike length.
Cut cut_of(const rkc_cache* c, const rkc_attention* a) {
  const int64_t units = (int64_t)c->n_seqs * c->kv_heads, all = units * ((a->max_len + kTurn - 1) / kTurn);
  const int64_t most = (int64_t)a->max_rows * (a->q_heads / c->kv_heads) / 8;
  int64_t turns = all / (4 * 256);
  turns = turns > most ? most : turns;
  turns = turns > 16 ? 16 : turns < 2 ? 2 : turns;
  const int chunks = (int)((a->max_len + turns * kTurn - 1) / (turns * kTurn));
  return {(int)turns, chunks, units * chunks};
}

template <typename T>
rkc_status go(const rkc_cache* c, const rkc_attention* a, hipStream_t s) {
  const Cut cut = cut_of(c, a);
  const int lds = a->d_parent ? kTreeBytes : 0;
  const dim3 grid((unsigned)cut.workgroups), block(kThreads);
  if (c->head_dim == 64) weigh<T, 64><<<grid, block, lds, s>>>(*c, *a, cut.chunks, cut.turns);
  else if (c->head_dim == 128) weigh<T, 128><<<grid, block, lds, s>>>(*c, *a, cut.chunks, cut.turns);
  else weigh<T, 256><<<grid, block, lds, s>>>(*c, *a, cut.chunks, cut.turns);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

}  // namespace

bool rkc_weigh_fits(const rkc_cache* c, const rkc_attention* a) { return rkc_fits(cut_of(c, a).workgroups, kThreads); }

extern "C" rkc_status rkc_weigh(const rkc_cache* c, const rkc_attention* a, void* stream) {
  if (rkc_status st = rkc_attention_check(c, a, true)) return st;
  if (c->n_seqs == 0 || a->max_len == 0) return RKC_OK;
  if (!rkc_weigh_fits(c, a)) return RKC_E_UNSUPPORTED;
  return c->dtype == RKC_BF16 ? go<__bf16>(c, a, (hipStream_t)stream) : go<_Float16>(c, a, (hipStream_t)stream);
}

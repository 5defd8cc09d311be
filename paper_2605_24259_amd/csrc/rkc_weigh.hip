// rkc_weigh.hip -- the account of a cache: how much attention each of its slots received.
//
// Softmax sums are given, so slots are independent: a wave holds the keys of 64 slots (32 at 256 elements a head) in
// registers as columns of 16x16x32 products and goes over the packed rows 16 at a time; a lane adds up the
// weights of its slot's column in 32 bits, in a fixed order.  One read of the keys; no atomics.
#include "rkc_cache_dev.h"

namespace {

constexpr int kThreads = 256, kBlock = 128;  // packed rows whose masks and sums lie in LDS at a time
static_assert(kThreads == RKC_MAX_TREE_ROWS, "tree_lines");

struct RowIn {
  float lse2, slope;
  int start, end, pos, line;
};

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void weigh(const rkc_cache c, const rkc_attention a, int chunks) {
  typedef typename Vec8<T>::t V8;
  constexpr int KC = D / 32, NS = D == 256 ? 2 : 4, kSlots = 16 * NS;
  __shared__ RowIn in[kBlock];
  __shared__ uint64_t lines[RKC_MAX_TREE_ROWS][4];
  __shared__ int depths[RKC_MAX_TREE_ROWS];

  const int H = c.kv_heads, G = a.q_heads / H;
  const int h = blockIdx.x % H, part = blockIdx.x / H % chunks, s = blockIdx.x / (H * chunks);
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), quad = lane >> 4, col = lane & 15;
  const Seq q = load_seq(c, a, s);
  if (!q.ok) {
    if (part == 0 && h == 0 && tid == 0) flag(c, s, RKC_CS_LENGTH);
    return;
  }
  const int w0 = part * 4 * kSlots, t0 = w0 + wave * kSlots;
  if (w0 >= q.len) return;
  const int M = q.n * G;
  const int32_t* table = c.d_block_table + (int64_t)s * c.max_pages;
  const int shift = 31 - __builtin_clz(c.page_tokens), in_page = c.page_tokens - 1;
  V8 kf[NS][KC];
  bool bad = false;
  const T* kp = (const T*)c.d_k + h * c.k_head_stride;
#pragma unroll
  for (int u = 0; u < NS; u++) {
    const int at = min(t0 + 16 * u, (q.len - 1) & ~15);
    const T* kb = kp + (int64_t)page_of(c, table, shift, at, bad) * c.k_block_stride + (at & in_page) * c.k_slot_stride + (int)(col * (int)c.k_slot_stride) + quad * 8;
#pragma unroll
    for (int k = 0; k < KC; k++) kf[u][k] = *(const V8*)(kb + 32 * k);
  }
  if (bad) flag(c, s, RKC_CS_BLOCK);
  const bool tree = a.d_parent != nullptr;
  const bool drafts = tree && w0 + 4 * kSlots > q.base;
  if (drafts || (tree && a.d_slope)) tree_lines(c, a, q, s, part == 0 && h == 0, lines, depths);
  const int pre = a.d_prefix ? max(0, min(word(a.d_prefix, s), tree ? q.base : q.len)) : 0;
  const Scale sc = load_scale(a);
  float acc[NS] = {};

  for (int mb = 0; mb < M; mb += kBlock) {
    __syncthreads();
    if (tid < kBlock) {
      const int m = mb + tid;
      RowIn r = {kInf, 0.f, 0x7fffffff, 0, 0, 0};
      if (m < M) {
        const int qi = m / G, qh = h * G + m % G;
        const Row w = load_row(a, q, s, qi);
        const float lse = a.d_lse[(int64_t)(q.row0 + qi) * a.q_heads + qh];
        r.lse2 = lse == -kInf ? kInf : lse * kLog2e;  // a row that saw nothing gave nothing
        r.slope = a.d_slope ? a.d_slope[qh] * kLog2e / sc.post : 0.f;
        r.start = w.start, r.end = w.end, r.line = qi;
        r.pos = tree && a.d_slope ? q.base + depths[qi] : w.pos;
      }
      in[tid] = r;
    }
    __syncthreads();
    const int rows = min(kBlock, M - mb);
    // what all rows of the block see, and what any sees
    const int e0 = lane < rows ? lane : 0, e1 = lane + 64 < rows ? lane + 64 : 0;
    const int all_from = wave_max(max(in[e0].start, in[e1].start)), all_to = wave_min(min(in[e0].end, in[e1].end));
    const int any_from = wave_min(min(in[e0].start, in[e1].start)), any_to = tree ? q.len : wave_max(max(in[e0].end, in[e1].end));
    if (!((t0 + kSlots > any_from && t0 < any_to) || t0 < pre) || t0 >= q.len) continue;
    const bool whole = t0 + kSlots <= pre || (t0 >= all_from && t0 + kSlots <= all_to);
    for (int m0 = 0; m0 < rows; m0 += 16) {
      const int m = min(mb + m0 + col, M - 1), qi = m / G, qh = h * G + m % G;
      const T* p = (const T*)a.d_q + (q.row0 + qi) * a.q_row_stride + qh * a.q_head_stride + quad * 8;
      V8 qf[KC];
#pragma unroll
      for (int k = 0; k < KC; k++) {
        qf[k] = *(const V8*)(p + 32 * k);
        if (sc.negate) qf[k] = negated(qf[k]);
      }
#pragma unroll
      for (int u = 0; u < NS; u++) {
        f32x4 x = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KC; k++) x = mma16(qf[k], kf[u][k], x);
        const int j = t0 + 16 * u + col;
#pragma unroll
        for (int e = 0; e < 4; e++) {
          const RowIn& r = in[m0 + quad * 4 + e];  // rows behind the last one have a sum of infinity
          float y = x[e];
          if (a.softcap > 0.f) y = capped(y, sc);
          if (a.d_slope) {
            const int at = drafts && j >= q.base ? q.base + depths[min(j - q.base, RKC_MAX_TREE_ROWS - 1)] : j;
            y -= r.slope * fabsf((float)(r.pos - at));
          }
          y = ex2(y * sc.post - r.lse2);
          if (!whole) {
            bool see = (j >= r.start && j < r.end) || j < pre;
            if (drafts && j >= q.base) {
              const int d = min(j - q.base, RKC_MAX_TREE_ROWS - 1);
              see |= lines[r.line][d >> 6] >> (d & 63) & 1;
            }
            y = see && r.lse2 != kInf ? y : 0.f;
          }
          acc[u] += y;
        }
      }
    }
  }
#pragma unroll
  for (int u = 0; u < NS; u++) {
    const float got = sum32(sum16(acc[u]));
    const int j = t0 + 16 * u + col;
    if (quad == 0 && j < q.len) {
      const int64_t at = s * a.weight_seq_stride + h * a.weight_head_stride + j;
      a.d_weight[at] = (a.d_weight_in ? a.decay * a.d_weight_in[at] : 0.f) + got;
    }
  }
}

template <typename T>
rkc_status go(const rkc_cache* c, const rkc_attention* a, hipStream_t s) {
  const int slots = c->head_dim == 256 ? 128 : 256, chunks = (a->max_len + slots - 1) / slots;
  if ((int64_t)c->n_seqs * c->kv_heads * chunks > 0x7fffffff) return RKC_E_UNSUPPORTED;
  const dim3 grid(c->n_seqs * c->kv_heads * chunks), block(kThreads);
  if (c->head_dim == 64) weigh<T, 64><<<grid, block, 0, s>>>(*c, *a, chunks);
  else if (c->head_dim == 128) weigh<T, 128><<<grid, block, 0, s>>>(*c, *a, chunks);
  else weigh<T, 256><<<grid, block, 0, s>>>(*c, *a, chunks);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

}  // namespace

extern "C" rkc_status rkc_weigh(const rkc_cache* c, const rkc_attention* a, void* stream) {
  if (rkc_status st = rkc_attention_check(c, a, true)) return st;
  if (c->n_seqs == 0 || a->max_len == 0) return RKC_OK;
  return c->dtype == RKC_BF16 ? go<__bf16>(c, a, (hipStream_t)stream) : go<_Float16>(c, a, (hipStream_t)stream);
}

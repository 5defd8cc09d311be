// rkc_attend_few.hip -- attention of few rows over a paged cache (decode steps, small trees).
//
// out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m), x the masked and capped scores, m their running maximum.  Up to 16
// packed rows (rows x query heads of one key/value head) are the columns of a 16x16x32 matrix product, so every key and
// value is read once for all of them; what bounds the kernel is that read: 5.9 TB/s of K and V with 5 sequences of
// 250,000 to 262,144 slots, 8 heads of 128 elements (887 us), 4.4 TB/s with 64 of 1 to 4,096 slots (123 us), where
// workgroups begin and end more often.
// A workgroup takes a chunk of one sequence's slots for one head, its four waves (eight, see rkc_attend_plan) take 32 slots at a time:
//   K goes from memory straight into the product's operand (a lane holds 8 elements of its slot's key),
//   V goes through the wave's own 32-slot tile in LDS, from where it is read transposed (no barriers; its bank
//   conflicts are 0.04 of the LDS cycles of long sequences, 0.16 of those of many short ones),
//   both for the next 32 slots are in flight while these are worked on.
// Waves keep maxima, sums and outputs of their own (32 bits) and join them once at the end; chunks are joined by a
// second kernel where a sequence has more than one.
// Weights go into the second product as two operands each, rounded and the rest, as the matrix units wait for the read
// anyway: outputs are as near to the formula's as with weights in 32 bits (4 sequences of up to 1,280 slots in float16:
// 4.8e-5, with rounded weights alone up to 1.5 times as far), at the same time (898 us of 5 long ones, 899 without).
// Heads of 256 elements leave a wave a SIMD: 4.6 TB/s of 5 sequences of 125,000 to 131,072 slots, 8 heads (1,141 us).
#include "rkc_cache_dev.h"
#include "rkc_tiles.h"

namespace {

template <typename T, int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves, D <= 128 ? 2 : 1) void attend_few(const rkc_cache c, const rkc_attention a, const rkc_plan pl) {
  typedef typename Vec8<T>::t V8;
  constexpr int KC = D / 32, DB = D / 16, VP = D / 16;  // key operands, output blocks, 16-byte pieces of V per lane
  constexpr int kTile = 32 * D;                         // elements of a wave's V tile
  constexpr int kJoin = 16 * D * 4;                // bytes of a wave's output tile at the join
  constexpr int kLds = kTile * 2 > kJoin ? kTile * 2 : kJoin;
  __shared__ __attribute__((aligned(16))) char lds[kWaves * kLds];
  __shared__ float stat[kWaves][16][2], total[16];

  const int H = c.kv_heads, G = a.q_heads / H;
  // The parts of a sequence are neighbours, turned by a number of their own in each: XCDs take workgroups in turn, and
  // an XCD would else have the same parts of every sequence, the last ones of short sequences being empty (64 sequences
  // of 1 to 4,096 slots in 8 parts: 123 us instead of 159).
  const int u = blockIdx.x / pl.splits, h = u % H, s = u / H, split = (blockIdx.x % pl.splits + (u * 0x9e3779b1u >> 16)) % pl.splits;
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), quad = lane >> 4, col = lane & 15;
  const Seq q = load_seq(c, a, s);
  if (!q.ok) {
    if (split == 0 && h == 0 && threadIdx.x == 0) flag(c, s, RKC_CS_LENGTH);
    return;
  }
  const int M = q.n * G;
  if (!M) return;
  const int c0 = split * pl.chunk, c1 = min(q.len, c0 + pl.chunk);
  if (split && c0 >= q.len) return;
  const int32_t* table = c.d_block_table + (int64_t)s * c.max_pages;
  const int shift = 31 - __builtin_clz(c.page_tokens), in_page = c.page_tokens - 1;

  const Scale f = load_scale(a);
  const int mine_m = min(col, M - 1), qi = mine_m / G, qh = h * G + mine_m % G;
  Row row = load_row(a, q, s, qi);
  const float slope = a.d_slope ? a.d_slope[qh] * kLog2e / f.post : 0.f;
  V8 qf[KC];
  {
    const T* p = (const T*)a.d_q + (q.row0 + qi) * a.q_row_stride + qh * a.q_head_stride + quad * 8;
#pragma unroll
    for (int k = 0; k < KC; k++) {
      qf[k] = *(const V8*)(p + 32 * k);
      if (f.negate) qf[k] = negated(qf[k]);
    }
  }
  // a tree's rows are at most 16 here: lines as bits of a register, walked through the lanes' parents
  uint32_t line = 0;
  int depth_of = 0;  // depth of row `lane`
  if (a.d_parent && c1 > q.base) {
    int par = -1;
    if (lane < q.n) {
      par = a.d_parent[q.row0 + lane];
      if (par < -1 || par >= lane) {
        flag(c, s, RKC_CS_PARENT);
        par = -1;
      }
    }
    uint32_t mine = lane < 32 ? 1u << lane : 0;
    for (int at = par; __any(at >= 0);) {
      const int up = __shfl(par, at & 63);
      if (at >= 0) mine |= 1u << at, at = up;
    }
    depth_of = __popc(mine) - 1;
    line = (uint32_t)__shfl((int)mine, qi);
    row.pos = q.base + __shfl(depth_of, qi);
  } else if (a.d_parent && a.d_slope) {
    // distances need the rows' depths in every chunk
    int par = lane < q.n ? a.d_parent[q.row0 + lane] : -1;
    if (par < -1 || par >= lane) par = -1;
    int d = 0;
    for (int at = par; __any(at >= 0);) {
      const int up = __shfl(par, at & 63);
      if (at >= 0) d++, at = up;
    }
    row.pos = q.base + __shfl(d, qi);
  }
  // slots that all rows see, and slots that any sees
  const int all_from = wave_max(row.start), all_to = wave_min(row.end), any_from = wave_min(row.start), all_pre = uni(row.prefix);
  int any_to = wave_max(max(row.end, row.prefix));
  if (a.d_parent) any_to = q.len;
  const int end = min(c1, any_to);  // of what is looked at here: a chunk is a multiple of 32 slots

  const Pool kp = k_pool(c, h), vp = v_pool(c, h);
  T* tile = (T*)(lds + wave * kLds);

  float top = -kInf, sum = 0.f;
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; d++) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

  const rkc_tiles<32> tiles(c0, end, all_pre, any_from);
  const int n_tiles = tiles.n;
  auto slot_of = [&](int i) { return tiles.slot(i); };
  V8 kf[2][KC];
  u32x4 vf[VP];
  bool bad = false;
  int page[2];  // of the next tile to be loaded: two runs of 16 slots, each within a page
  auto run_of = [&](int t0, int u) { return u && t0 + 16 >= end ? t0 : t0 + 16 * u; };  // one behind the end repeats the first
  auto look_up = [&](int i) {
    const int t0 = slot_of(i);
#pragma unroll
    for (int u = 0; u < 2; u++) page[u] = page_of(table, shift, run_of(t0, u));
  };
  constexpr int RP = 512 / D;  // rows of a piece of V: 64 lanes of 16 bytes
  const uint32_t k_off = col * kp.slot + quad * 16, v_off = lane / (D / 8) * vp.slot + lane % (D / 8) * 16;
  auto load = [&](int i) {
    const int t0 = slot_of(i);
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int at = run_of(t0, u) & in_page;
      const int block = block_of(c, page[u], bad);
      const char* kb = fixed(run_at(kp, block, at));
      const char* vb = run_at(vp, block, at);
#pragma unroll
      for (int k = 0; k < KC; k++) kf[u][k] = *(const V8*)(kb + k_off + 64 * k);
#pragma unroll
      for (int p = 0; p < VP / 2; p++) vf[u * (VP / 2) + p] = *(const u32x4*)(fixed(vb + p * RP * vp.slot) + v_off);
    }
  };
  // byte offsets in the tile: of this lane's piece of V, and of its first values for a product
  const int put_at = 2 * vals16_at<D>(lane / (D / 8), lane % (D / 8));
  const int val_at = 2 * (vals16_at<D>(quad * 4 + (col >> 2), (col & 3) >> 1) + (col & 1) * 4);

  // A tile that all rows see is multiplied as it is.  An infinity in it would meet the rest of a weight, which may be zero or
  // negative, and come out as NaN: an output that is not finite has the wave go over its tiles once more, all looked through.
  for (bool careful = false;; careful = true) {
    int i = wave;
    if (i < n_tiles) {
      look_up(i);
      load(i);
      if (i + kWaves < n_tiles) look_up(i + kWaves);
    }
    for (; i < n_tiles; i += kWaves) {
      const int t0 = slot_of(i);
      f32x4 sc[2];
#pragma unroll
      for (int u = 0; u < 2; u++) {
        sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KC; k++) sc[u] = mma16(kf[u][k], qf[k], sc[u]);
      }
      const bool whole = t0 + 32 <= all_pre || (t0 >= all_from && t0 + 32 <= all_to);
      bool hurt = false;
      const int pa = here(put_at), va = here(val_at);
      auto put = [&](int p, u32x4 x) { *(u32x4*)((char*)tile + ((pa ^ vals16_x<D>(p * RP) << 4) + p * RP * 2 * D)) = x; };
      if (whole && !careful) {
#pragma unroll
        for (int p = 0; p < VP; p++) put(p, vf[p]);
      } else {
#pragma unroll
        for (int p = 0; p < VP; p++) {
          const int j = t0 + p * RP + lane / (D / 8);
          u32x4 x = vf[p];
          if (j >= end || (j < any_from && j >= all_pre)) x = u32x4{0, 0, 0, 0};  // no row sees it
          hurt |= any_hurt<T>(x);
          put(p, x);
        }
        hurt = __any(hurt);
      }
      uint32_t seen = 0xffffffff;
      if (a.softcap > 0.f) cap_all(sc, f);
      if (a.d_slope) {
        const float far = (float)(here(row.pos - t0) - quad * 4);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          float gap = far - (float)(16 * (e >> 2) + (e & 3));
          if (a.d_parent && t0 + 32 > q.base) {
            const int at = t0 + quad * 4 + 16 * (e >> 2) + (e & 3) - q.base, d = __shfl(depth_of, at & 63);
            gap = at >= 0 ? (float)(row.pos - q.base - d) : gap;
          }
          sc[e >> 2][e & 3] = __builtin_fmaf(-slope, fabsf(gap), sc[e >> 2][e & 3]);
        }
      }
      if (!whole) {
        const int from = t0 - q.base;
        const uint32_t drafted = from >= 32 || from <= -32 ? 0 : from >= 0 ? line >> from : line << -from;
        seen = seen_of(row, t0, drafted) >> 4 * quad;
#pragma unroll
        for (int e = 0; e < 8; e++) sc[e >> 2][e & 3] = masked(sc[e >> 2][e & 3], seen, 16 * (e >> 2) + (e & 3));
      }
      auto vals = [&](int d) { return read_tr2<T>((const char*)tile + (va ^ d << 5), (const char*)tile + (va ^ d << 5) + 32 * D); };
      if (pl.keep) {
        float* to = (float*)((char*)a.d_scratch + pl.score_at) + (int64_t)(s * H + h) * (a.max_rows * G) * pl.wide + (int64_t)t0 * (a.max_rows * G) + 32 * col + quad * 4;
        if (col < M) *(f32x4*)to = sc[0] * f.post, *(f32x4*)(to + 16) = sc[1] * f.post;
      }
      if (i + kWaves < n_tiles) {
        load(i + kWaves);
        if (i + 2 * kWaves < n_tiles) look_up(i + 2 * kWaves);
      }
      float most = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])),
                         fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])));
      most = max32(max16(most)) * f.post;
      // weights up to 2^8 are let stand: the maximum moves, and the outputs are rescaled, in few tiles only
      if (__any(most > top + (8.f + kRoom<T>))) {
        const float now = fmaxf(top, most - kRoom<T>), by = now == -kInf ? 1.f : ex2(top - now);
        top = now, sum *= by;
#pragma unroll
        for (int d = 0; d < DB; d++) o[d] *= by;
      }
      const float m = top == -kInf ? 0.f : top;
      f32x8 p;
#pragma unroll
      for (int e = 0; e < 8; e++) p[e] = ex2(__builtin_fmaf(sc[e >> 2][e & 3], f.post, -m));
      sum += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      // the products' operands have the cache's type: a weight is the sum of two of them, with at least twice its bits
      const V8 pb = __builtin_convertvector(p, V8), pr = __builtin_convertvector(p - __builtin_convertvector(pb, f32x8), V8);
      if (hurt) {
        V8 by;
#pragma unroll
        for (int e = 0; e < 8; e++) by[e] = (T)(seen >> (16 * (e >> 2) + (e & 3)) & 1 ? 1.f : 0.f);
#pragma unroll
        for (int d = 0; d < DB; d++) {
          V8 vt = vals(d);
          const f32x4 n = mma16(strip<T>(vt), by, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int k = 0; k < 4; k++) o[d][k] += hurt_by(n[k]);
        }
        for (int k = lane; k < kTile / 8; k += 64) {
          V8 v = *(const V8*)(tile + 8 * k);
          strip<T>(v);
          *(V8*)(tile + 8 * k) = v;
        }
      }
#pragma unroll
      for (int d = 0; d < DB; d++) {
        const V8 vt = vals(d);
        o[d] = mma16(vt, pr, mma16(vt, pb, o[d]));
      }
    }
    if (careful) break;
    float odd = 0.f;  // stays 0 unless an output is not finite
#pragma unroll
    for (int d = 0; d < DB; d++)
#pragma unroll
      for (int k = 0; k < 4; k++) odd = __builtin_fmaf(o[d][k], 0.f, odd);
    if (!__any(odd != 0.f)) break;
    top = -kInf, sum = 0.f;
#pragma unroll
    for (int d = 0; d < DB; d++) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  if (bad) flag(c, s, RKC_CS_BLOCK);

  // join the waves; one that saw nothing of a row has a sum of 0
  sum = sum32(sum16(sum));
  if (quad == 0) stat[wave][col][0] = top, stat[wave][col][1] = sum;
  __syncthreads();
  float m_all = -kInf, l_all = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; w++) m_all = fmaxf(m_all, stat[w][col][0]);
#pragma unroll
  for (int w = 0; w < kWaves; w++) l_all += stat[w][col][1] == 0.f ? 0.f : stat[w][col][1] * ex2(stat[w][col][0] - m_all);
  {
    const float by = ex2(top - m_all);
    float* to = (float*)(lds + wave * kLds) + col * D + quad * 4;
    // 16 rows of D floats: rotated so that the rows' 16-byte pieces do not share banks
#pragma unroll
    for (int d = 0; d < DB; d++) *(f32x4*)(to + 16 * ((d + col) % DB)) = sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[d] * by;
  }
  const int unit = s * H + h;
  if (wave == 0 && quad == 0) {
    total[col] = l_all;
    if (pl.splits > 1) {
      float* st = (float*)((char*)a.d_scratch + pl.stat_at) + ((int64_t)(unit * pl.splits + split) * pl.rows + col) * 2;
      st[0] = m_all, st[1] = l_all;
    } else if (col < M) {
      a.d_lse[(int64_t)(q.row0 + qi) * a.q_heads + qh] = l_all == 0.f ? -kInf : kLn2 * (m_all + lg2(l_all));
    }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < M * (D / 4); x += 64 * kWaves) {
    const int m = x / (D / 4), b = x % (D / 4), d = b >> 2;
    const float* from = (const float*)lds + m * D + 16 * ((d + m) % DB) + (b & 3) * 4;
    f32x4 y = *(const f32x4*)from;
#pragma unroll
    for (int w = 1; w < kWaves; w++) y += *(const f32x4*)((const char*)from + w * kLds);
    if (pl.splits == 1) {
      const float l = total[m];
      const float by = l == 0.f ? 0.f : 1.f / l;
      T* to = (T*)a.d_out + (q.row0 + m / G) * a.out_row_stride + (h * G + m % G) * a.out_head_stride + b * 4;
      typedef T T4 __attribute__((ext_vector_type(4)));
      *(T4*)to = __builtin_convertvector(y * by, T4);
    } else {
      *(f32x4*)((float*)((char*)a.d_scratch + pl.part_at) + ((int64_t)(unit * pl.splits + split) * pl.rows + m) * D + b * 4) = y;
    }
  }
}

template <typename T, int D, int W>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  attend_few<T, D, W><<<dim3(p->units * p->splits), dim3(64 * W), 0, s>>>(*c, *a, *p);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

template <typename T, int D>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  if constexpr (D <= 128) {
    if (p->waves == 8) return go<T, D, 8>(c, a, p, s);
  }
  return go<T, D, 4>(c, a, p, s);
}

template <typename T>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  return c->head_dim == 64 ? go<T, 64>(c, a, p, s) : c->head_dim == 128 ? go<T, 128>(c, a, p, s) : go<T, 256>(c, a, p, s);
}

}  // namespace

rkc_status rkc_attend_few(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  return c->dtype == RKC_BF16 ? go<__bf16>(c, a, p, s) : go<_Float16>(c, a, p, s);
}

// rkc_packed.hip -- attention over a paged cache in 4 bits: C ABI, choice of kernel, and the kernel of few rows (decode steps,
// small trees).
//
// out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m), x the masked and capped scores, m their running maximum.  16 packed
// rows (rows x query heads of one key/value head) are the columns of a 16x16x32 matrix product, and a workgroup has one or two
// blocks of 16, so that every key and value is read and converted once for all of them.  What bounds the kernel is that read:
// 5.3 TB/s with 5 sequences of 250,000 to 262,144 slots, 8 heads of 128 elements (266 us; the 16-bit cache's 896), 4.7 TB/s
// with 64 of 1 to 8,192 (62 us).  With two blocks two waves a SIMD are left, and the vector units' work on the scores counts
// as much (32 packed rows over 40 sequences of 700 to 8,192 slots: 2.7 TB/s, 81 us).
// A workgroup takes a chunk of one sequence's slots for one head, its waves take 32 slots at a time:
//   K  a lane has a quarter of its slot's key (head_dim / 4 elements), which it makes the product's operand of by the
//      conversion of two codes an instruction with the scale in it (exact, but for float16 below 2^-24);
//   V  likewise a quarter of a slot's value, converted and put into the wave's own tile in LDS, from where it is read
//      transposed (no barriers);
// both for the next 32 slots are in flight while these are worked on.
// A marked slot's scores are NaN by its key's first scale, and so only the rows that see it; values are always finite, so that
// one that a row does not see meets a weight of zero and gives zero.
#include <type_traits>

#include "rkc_packed_dev.h"
#include "rkc_tiles.h"

namespace {

// The sequence of rank r by length, the longest first, of at most 64, as seq_of_rank finds it, in three instructions a sequence:
// lengths and lanes in one number, so that none are alike.
__device__ __forceinline__ int seq_by_length(const rkc_cache& c, const rkc_attention& a, int r) {
  const int lane = threadIdx.x & 63;
  const uint32_t key = lane < c.n_seqs ? (uint32_t)a.d_length[lane] << 6 | (63 - lane) : 0;
  int rank = 0;
#pragma unroll 8
  for (int k = 0; k < c.n_seqs; k++) rank += (uint32_t)__builtin_amdgcn_readlane((int)key, k) > key;
  return uni(__builtin_ctzll(__ballot(lane < c.n_seqs && rank == r)));
}

template <typename T, int D, int kWaves, int NB>
__global__ __launch_bounds__(64 * kWaves, D == 256 && NB == 2 ? 1 : 2) void packed_few(const rkc_cache c, const rkc_attention a, const rkc_plan pl) {
  typedef typename Vec8<T>::t V8;
  constexpr int kRows = 16 * NB;           // NB blocks of packed rows, a lane's column of each
  constexpr int KC = D / 32, DB = D / 16;  // dwords of codes in a quarter of a slot, and key operands; output blocks
  constexpr int NS = D == 256 ? 2 : 1;     // scales of a quarter
  constexpr int kTile = 32 * D;            // elements of a wave's V tile
  constexpr int kJoin = 16 * D * 4;        // bytes of a wave's outputs of a block at the join
  constexpr int kLds = kTile * 2 > kJoin ? kTile * 2 : kJoin;
  __shared__ __attribute__((aligned(16))) char lds[kWaves * kLds];
  __shared__ float stat[kWaves][kRows][2], total[kRows];

  const int H = c.kv_heads, G = a.q_heads / H;
  // The parts of a sequence are neighbours, turned by a number of their own in each: XCDs take workgroups in turn, and
  // an XCD would else have the same parts of every sequence, the last ones of short sequences being empty.
  // Row tiles of the same part are eight workgroups apart: on one XCD, whose cache has what the first of them read.
  const int x = blockIdx.x / (8 * pl.tiles) * 8 + blockIdx.x % 8, qt = blockIdx.x / 8 % pl.tiles;
  const int rank = x / pl.splits / H, h = x / pl.splits % H;
  if (rank >= c.n_seqs) return;
  // Of whole sequences the longer half goes first, from the longest on, and the other from the shortest on: a CU's second
  // workgroup then is the shorter, the longer its first one is.
  const int half = (c.n_seqs + 1) / 2, s = pl.sorted ? seq_by_length(c, a, rank < half ? rank : c.n_seqs - 1 - (rank - half)) : rank;
  const int u = s * H + h, split = (x % pl.splits + (u * 0x9e3779b1u >> 16)) % pl.splits;
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), quad = lane >> 4, col = lane & 15;
  const Seq q = load_seq(c, a, s);
  if (!q.ok) {
    if (split == 0 && h == 0 && qt == 0 && threadIdx.x == 0) flag(c, s, RKC_CS_LENGTH);
    return;
  }
  const int m0 = qt * kRows, M = q.n * G - m0;  // rows yet to be had by this tile and those behind it
  if (M <= 0) return;
  const int c0 = split * pl.chunk, c1 = min(q.len, c0 + pl.chunk);
  if (split && c0 >= q.len) return;
  const int32_t* table = c.d_block_table + (int64_t)s * c.max_pages;
  const int shift = 31 - __builtin_clz(c.page_tokens), in_page = c.page_tokens - 1;

  const Scale f = load_scale(a);
  int qi[NB], qh[NB];
  Row row[NB];
  float slope[NB];
  V8 qf[NB][KC];  // a quarter of the rows' queries, as the keys'
#pragma unroll
  for (int n = 0; n < NB; n++) {
    const int m = min(16 * n + col, M - 1);
    qi[n] = (m0 + m) / G, qh[n] = h * G + (m0 + m) % G;
    row[n] = load_row(a, q, s, qi[n]);
    slope[n] = a.d_slope ? a.d_slope[qh[n]] * kLog2e / f.post : 0.f;
    const T* p = (const T*)a.d_q + (q.row0 + qi[n]) * a.q_row_stride + qh[n] * a.q_head_stride + quad * (D / 4);
#pragma unroll
    for (int k = 0; k < KC; k++) {
      qf[n][k] = *(const V8*)(p + 8 * k);
      if (f.negate) qf[n][k] = negated(qf[n][k]);
    }
  }
  // a tree's rows are at most 32 here: lines as bits of a register, walked through the lanes' parents
  uint32_t line[NB] = {};
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
#pragma unroll
    for (int n = 0; n < NB; n++) line[n] = (uint32_t)__shfl((int)mine, qi[n]), row[n].pos = q.base + __shfl(depth_of, qi[n]);
  } else if (a.d_parent && a.d_slope) {
    // distances need the rows' depths in every chunk
    int par = lane < q.n ? a.d_parent[q.row0 + lane] : -1;
    if (par < -1 || par >= lane) par = -1;
    int d = 0;
    for (int at = par; __any(at >= 0);) {
      const int up = __shfl(par, at & 63);
      if (at >= 0) d++, at = up;
    }
#pragma unroll
    for (int n = 0; n < NB; n++) row[n].pos = q.base + __shfl(d, qi[n]);
  }
  // slots that all rows see, and slots that any sees
  int first = row[0].start, last = row[0].start, least = row[0].end, most_end = max(row[0].end, row[0].prefix);
#pragma unroll
  for (int n = 1; n < NB; n++) {
    first = min(first, row[n].start), last = max(last, row[n].start);
    least = min(least, row[n].end), most_end = max(most_end, row[n].end);
  }
  const int all_from = wave_max(last), all_to = wave_min(least), any_from = wave_min(first), all_pre = uni(row[0].prefix);
  int any_to = wave_max(most_end);
  if (a.d_parent) any_to = q.len;
  const int end = min(c1, any_to);  // of what is looked at here: a chunk is a multiple of 32 slots

  const Codes held = codes_of<D>(c, h);
  T* tile = (T*)(lds + wave * kLds);

  float top[NB], sum[NB];
  f32x4 o[NB][DB];
#pragma unroll
  for (int n = 0; n < NB; n++) {
    top[n] = -kInf, sum[n] = 0.f;
#pragma unroll
    for (int d = 0; d < DB; d++) o[n][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  const rkc_tiles<32> tiles(c0, end, all_pre, any_from);
  const int n_tiles = tiles.n;
  auto slot_of = [&](int i) { return tiles.slot(i); };
  typedef uint32_t codes_t __attribute__((ext_vector_type(KC)));
  codes_t kf[2], vf[2];
  uint32_t ks[2], vs[2];  // scales: a byte, or two
  bool bad = false;
  int page[2];  // of the next tile to be loaded: two runs of 16 slots, each within a page
  auto run_of = [&](int t0, int u) { return u && t0 + 16 >= end ? t0 : t0 + 16 * u; };  // one behind the end repeats the first
  auto look_up = [&](int i) {
    const int t0 = slot_of(i);
#pragma unroll
    for (int u = 0; u < 2; u++) page[u] = page_of(table, shift, run_of(t0, u));
  };
  // a lane's quarter of a key, and of a value: slot and which
  const int v_slot = lane >> 2, v_quad = lane & 3;
  const uint32_t k_off = col * (D / 2) + quad * (D / 8), v_off = lane * (D / 8);
  const uint32_t ks_off = col * (D / 32) + quad * (D / 32) / 4 * (D >= 128) + (D == 64 ? quad >> 1 : 0);
  const uint32_t vs_off = v_slot * (D / 32) + v_quad * (D / 32) / 4 * (D >= 128) + (D == 64 ? v_quad >> 1 : 0);
  typedef typename std::conditional<NS == 2, uint16_t, uint8_t>::type scales_t;
  auto load = [&](int i) {
    const int t0 = slot_of(i);
#pragma unroll
    for (int u = 0; u < 2; u++) {
      const int at = run_of(t0, u) & in_page;
      const char* b = held.base + (uint64_t)(uint32_t)block_of(c, page[u], bad) * held.block;
      const char* kb = b + at * (D / 2);
      const char* sb = b + held.key_scales + at * (D / 32);
      kf[u] = from_global<codes_t>(kb, k_off), vf[u] = from_global<codes_t>(kb + held.values, v_off);
      ks[u] = from_global<scales_t>(sb, ks_off), vs[u] = from_global<scales_t>(sb + (held.value_scales - held.key_scales), vs_off);
    }
  };
  auto scale_k = [](uint32_t s, int k) { return scale_float(NS == 2 ? s >> 8 * (k / 4) & 255 : s); };
  // byte offsets in the tile: of this lane's quarter of a value, and of its first values for a product
  const int val_at = 2 * (vals16_at<D>(quad * 4 + (col >> 2), (col & 3) >> 1) + (col & 1) * 4);
  const int put_at = 2 * vals16_at<D>(v_slot, v_quad * KC);

  int i = wave;
  if (i < n_tiles) {
    look_up(i);
    load(i);
    if (i + kWaves < n_tiles) look_up(i + kWaves);
  }
  for (; i < n_tiles; i += kWaves) {
    const int t0 = slot_of(i);
    f32x4 sc[NB][2];
    const int pa = here(put_at), va = here(val_at);
#pragma unroll
    for (int u = 0; u < 2; u++) {
#pragma unroll
      for (int n = 0; n < NB; n++) sc[n][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KC; k++) {
        const V8 key = __builtin_bit_cast(V8, unpack8<T>(kf[u][k], scale_k(ks[u], k)));
#pragma unroll
        for (int n = 0; n < NB; n++) sc[n][u] = mma16(key, qf[n][k], sc[n][u]);
      }
      // a scale that nobody wrote may be anything: what no row sees is to be finite
#pragma unroll
      for (int k = 0; k < KC; k++) {
        const uint32_t b = NS == 2 ? vs[u] >> 8 * (k / 4) & 255 : vs[u];
        *(u32x4*)((char*)tile + ((pa ^ k << 4) + u * 16 * 2 * D)) = unpack8<T>(vf[u][k], scale_float(min(b, (uint32_t)kTopScale<T>)));
      }
    }
    const bool whole = t0 + 32 <= all_pre || (t0 >= all_from && t0 + 32 <= all_to);
    auto vals = [&](int d) { return read_tr2<T>((const char*)tile + (va ^ d << 5), (const char*)tile + (va ^ d << 5) + 32 * D); };
    if (i + kWaves < n_tiles) {
      load(i + kWaves);
      if (i + 2 * kWaves < n_tiles) look_up(i + 2 * kWaves);
    }
    V8 pb[NB], pr[NB];
#pragma unroll
    for (int n = 0; n < NB; n++) {
      if (a.softcap > 0.f) cap_all(sc[n], f);
      if (a.d_slope) {
        const float far = (float)(here(row[n].pos - t0) - quad * 4);
#pragma unroll
        for (int e = 0; e < 8; e++) {
          float gap = far - (float)(16 * (e >> 2) + (e & 3));
          if (a.d_parent && t0 + 32 > q.base) {
            const int at = t0 + quad * 4 + 16 * (e >> 2) + (e & 3) - q.base, d = __shfl(depth_of, at & 63);
            gap = at >= 0 ? (float)(row[n].pos - q.base - d) : gap;
          }
          sc[n][e >> 2][e & 3] = __builtin_fmaf(-slope[n], fabsf(gap), sc[n][e >> 2][e & 3]);
        }
      }
      if (!whole) {
        const int from = t0 - q.base;
        const uint32_t drafted = from >= 32 || from <= -32 ? 0 : from >= 0 ? line[n] >> from : line[n] << -from;
        const uint32_t seen = seen_of(row[n], t0, drafted) >> 4 * quad;
#pragma unroll
        for (int e = 0; e < 8; e++) sc[n][e >> 2][e & 3] = masked(sc[n][e >> 2][e & 3], seen, 16 * (e >> 2) + (e & 3));
      }
      float most = fmaxf(fmaxf(fmaxf(sc[n][0][0], sc[n][0][1]), fmaxf(sc[n][0][2], sc[n][0][3])),
                         fmaxf(fmaxf(sc[n][1][0], sc[n][1][1]), fmaxf(sc[n][1][2], sc[n][1][3])));
      most = max32(max16(most)) * f.post;
      // weights up to 2^8 are let stand: the maximum moves, and the outputs are rescaled, in few tiles only
      if (__any(most > top[n] + (8.f + kRoom<T>))) {
        const float now = fmaxf(top[n], most - kRoom<T>), by = now == -kInf ? 1.f : ex2(top[n] - now);
        top[n] = now, sum[n] *= by;
#pragma unroll
        for (int d = 0; d < DB; d++) o[n][d] *= by;
      }
      const float m = top[n] == -kInf ? 0.f : top[n];
      f32x8 p;
#pragma unroll
      for (int e = 0; e < 8; e++) p[e] = ex2(__builtin_fmaf(sc[n][e >> 2][e & 3], f.post, -m));
      sum[n] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      // The products' operands have 16 bits.  Of one block a weight is the sum of two of them, with at least twice its bits, as the
      // matrix units wait for the read anyway; of two it is rounded, as in the kernel of many rows (as the sum of two, 32 packed rows
      // over 40 sequences of 700 to 8,192 slots 90 us instead of 84, 96 of them 190 instead of 166).
      pb[n] = __builtin_convertvector(p, V8);
      if (NB == 1) pr[n] = __builtin_convertvector(p - __builtin_convertvector(pb[n], f32x8), V8);
    }
#pragma unroll
    for (int d = 0; d < DB; d++) {
      const V8 vt = vals(d);
#pragma unroll
      for (int n = 0; n < NB; n++) {
        o[n][d] = mma16(vt, pb[n], o[n][d]);
        if (NB == 1) o[n][d] = mma16(vt, pr[n], o[n][d]);
      }
    }
  }

  if (bad) flag(c, s, RKC_CS_BLOCK);

  // join the waves, a block of rows after the other; one that saw nothing of a row has a sum of 0
  const int unit = u * pl.tiles + qt;
#pragma unroll
  for (int n = 0; n < NB; n++) {
    sum[n] = sum32(sum16(sum[n]));
    if (quad == 0) stat[wave][16 * n + col][0] = top[n], stat[wave][16 * n + col][1] = sum[n];
  }
#pragma unroll
  for (int n = 0; n < NB; n++) {
    if (16 * n >= M) break;
    __syncthreads();  // of the first block: the sums are there; of the others: the one before is written
    float m_all = -kInf, l_all = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; w++) m_all = fmaxf(m_all, stat[w][16 * n + col][0]);
#pragma unroll
    for (int w = 0; w < kWaves; w++) l_all += stat[w][16 * n + col][1] == 0.f ? 0.f : stat[w][16 * n + col][1] * ex2(stat[w][16 * n + col][0] - m_all);
    {
      const float by = ex2(top[n] - m_all);
      float* to = (float*)(lds + wave * kLds) + col * D + quad * 4;
      // 16 rows of D floats: rotated so that the rows' 16-byte pieces do not share banks
#pragma unroll
      for (int d = 0; d < DB; d++) *(f32x4*)(to + 16 * ((d + col) % DB)) = sum[n] == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[n][d] * by;
    }
    if (wave == 0 && quad == 0) {
      total[16 * n + col] = l_all;
      if (pl.splits > 1) {
        float* st = (float*)((char*)a.d_scratch + pl.stat_at) + ((int64_t)(unit * pl.splits + split) * pl.rows + 16 * n + col) * 2;
        st[0] = m_all, st[1] = l_all;
      } else if (16 * n + col < M) {
        a.d_lse[(int64_t)(q.row0 + qi[n]) * a.q_heads + qh[n]] = l_all == 0.f ? -kInf : kLn2 * (m_all + lg2(l_all));
      }
    }
    __syncthreads();
    for (int y4 = threadIdx.x; y4 < min(16, M - 16 * n) * (D / 4); y4 += 64 * kWaves) {
      const int r = y4 / (D / 4), m = 16 * n + r, b = y4 % (D / 4), d = b >> 2;
      const float* from = (const float*)lds + r * D + 16 * ((d + r) % DB) + (b & 3) * 4;
      f32x4 y = *(const f32x4*)from;
#pragma unroll
      for (int w = 1; w < kWaves; w++) y += *(const f32x4*)((const char*)from + w * kLds);
      if (pl.splits == 1) {
        const float l = total[m];
        const float by = l == 0.f ? 0.f : 1.f / l;
        T* to = (T*)a.d_out + (q.row0 + (m0 + m) / G) * a.out_row_stride + (h * G + (m0 + m) % G) * a.out_head_stride + b * 4;
        typedef T T4 __attribute__((ext_vector_type(4)));
        *(T4*)to = __builtin_convertvector(y * by, T4);
      } else {
        *(f32x4*)((float*)((char*)a.d_scratch + pl.part_at) + ((int64_t)(unit * pl.splits + split) * pl.rows + m) * D + b * 4) = y;
      }
    }
  }
}

template <typename T, int D, int W, int NB>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  packed_few<T, D, W, NB><<<dim3(rkc_packed_few_workgroups(p)), dim3(64 * W), 0, s>>>(*c, *a, *p);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

template <typename T, int D>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  if (p->rows == 32) return go<T, D, 4, 2>(c, a, p, s);
  if constexpr (D <= 128) {
    if (p->waves == 8) return go<T, D, 8, 1>(c, a, p, s);
  }
  return go<T, D, 4, 1>(c, a, p, s);
}

template <typename T>
rkc_status go(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  return c->head_dim == 64 ? go<T, 64>(c, a, p, s) : c->head_dim == 128 ? go<T, 128>(c, a, p, s) : go<T, 256>(c, a, p, s);
}

}  // namespace

rkc_status rkc_packed_few(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  return c->dtype == RKC_BF16 ? go<__bf16>(c, a, p, s) : go<_Float16>(c, a, p, s);
}

// How a sequence is cut for one of the kernels.  That of few rows has 16 rows a workgroup or tiles of 32.  In the other 256 rows a
// workgroup halve what is converted and read of LDS per product, where such tiles, counted with 256 slots each, are twice the card's
// CUs: fewer leave CUs idle.  A sequence is cut where sequences, heads and row tiles do not fill the card a few times over.
static rkc_plan cut_plan(const rkc_cache* c, const rkc_attention* a, bool few) {
  rkc_plan p = {};
  const int64_t G = a->q_heads / c->kv_heads, M = a->max_rows * G;
  p.few = few;
  const int64_t wide = (int64_t)c->n_seqs * c->kv_heads * ((M + 255) / 256) * ((a->max_len + 255) / 256);
  p.rows = p.few ? (M <= 16 ? 16 : 32) : M <= 128 || c->head_dim == 64 || wide < 512 ? 128 : 256;
  p.tiles = (int)((M + p.rows - 1) / p.rows);
  if (p.tiles < 1) p.tiles = 1;
  const int64_t units = (int64_t)c->n_seqs * c->kv_heads * p.tiles;
  p.units = (int)units;
  // Workgroups wanted: of few rows ten a CU (5 sequences of 250,000 to 262,144 slots, 8 heads: 268 us, with four 307), of heads
  // of 256 elements four (32 sequences of up to 8,192 slots, 4 heads: 53 us, with one 67); of many as many as a CU holds.
  const bool wide_head = c->head_dim == 256;
  const int64_t want = p.few ? (wide_head ? 4 : 10) * 256 : wide_head || p.rows == 256 ? 256 : 2 * 256, grain = p.few || wide_head ? 128 : 256;
  const int64_t cut = units ? (want + units - 1) / units : 1;
  int64_t chunk = (a->max_len + cut - 1) / cut;
  chunk = (chunk + grain - 1) / grain * grain;
  // Of few rows no less than four tiles a wave, and up to 512 slots of many none: starts and the join cost more than that saves.
  const int64_t least = p.few && !wide_head ? 512 : grain;
  if (chunk < least) chunk = least;
  if (!p.few && a->max_len <= 512 && (c->head_dim < 256 || units >= 32)) chunk = 512;
  // Whole sequences, by eight waves, need no second kernel for the join.  They pay where they are short, and longer ones where their
  // units fill rounds of the 512 workgroups that the card holds: one to three quarters, or several (8 heads of 128 elements, all of
  // 8,192 slots / of 1 to 8,192, in us:  384 units whole 93 / 55, in parts 100 / 62;  480 106 / 61 and 118 / 71;  512 112 / 64 and
  // 122 / 78;  1,280 262 / 147 and 269 / 155;  but 256 58 / 51 and 72 / 42;  320 89 / 58 and 83 / 55;  520 143 / 80 and 126 / 78;  768 162 / 114
  // and 171 / 104).  Between such rounds sequences of up to 4,096 slots are as fast either way or faster (520 77 / 45 and 73 / 47; 768
  // 84 / 62 and 96 / 59; 1,024 111 / 73 and 122 / 79).  A long sequence among short ones, which the host cannot see, takes 6 us for each
  // 1,000 slots if whole: one of 8,192 among 63 of 100 52 us, in parts 24; of more slots the odds get worse.
  const int64_t whole = M > 16 || wide_head ? -1 : (units >= 384 && units <= 512) || units >= 1280 ? 8192 : units > 512 ? 4096 : 1536;
  p.waves = a->max_len <= whole ? 8 : 4;
  if (p.waves == 8) chunk = a->max_len < 32 ? 32 : (a->max_len + 31) / 32 * 32;
  p.chunk = (int)chunk;
  p.splits = (int)((a->max_len + chunk - 1) / chunk);
  if (p.splits < 1) p.splits = 1;
  // More workgroups than the card holds at once: the longest go first, so that none starts late.  Whole sequences of few rows, two
  // a CU, are paired, long ones with short ones, but for short ones, where finding the order, 1.7 us, is more than it saves (64 of
  // 1 to 8,192 slots: 65 us, in the table's order 78, in parts 78).
  p.sorted = c->n_seqs > 1 && c->n_seqs <= 64 && (p.few ? p.splits == 1 && units > 256 && a->max_len > 1024 : units * p.splits > want);
  if (p.splits > 1) {
    const size_t rows = (size_t)units * p.splits * p.rows;
    p.part_at = 0;
    p.stat_at = rows * c->head_dim * 4;
    p.bytes = (p.stat_at + rows * 8 + 255) & ~(size_t)255;
  }
  return p;
}

// Nanoseconds of a plan's kernel where all sequences are as long as they may be: rounds of the workgroups that the card holds, each a
// start and so much for 128 slots.  Fitted to 118 sizes (1 to 64 sequences of 500 to 32,768 slots, 20 to 96 packed rows, both kernels).
static int64_t cost_of(const rkc_cache* c, const rkc_plan* p) {
  const int d = c->head_dim == 64 ? 0 : c->head_dim == 128 ? 1 : 2;
  static const int few[3][2] = {{7400, 750}, {8000, 1700}, {13000, 2000}}, many[3][2] = {{10000, 2400}, {8000, 4000}, {10000, 6400}};
  const int* of = p->few ? few[d] : many[d];
  const int64_t held = d == 2 ? 256 : 512, rounds = ((int64_t)p->units * p->splits + held - 1) / held;
  return rounds * (of[0] + (int64_t)of[1] * p->chunk / 128);
}

// Which kernel.  Up to 16 packed rows go to the one that reads the cache as fast as it can, more than 96, and trees of more than 32
// rows, to the one that keeps the matrix units busy.  Between, the first has a tile of 32 rows a workgroup and the second one of 128,
// a quarter of it empty or more, but reads the cache once: the cheaper by cost_of, a sixteenth in favour of the first, whose smaller parts
// even out unlike lengths.  (Few rows and many, in us: 64 packed rows of 8 heads of 128 elements, 4 sequences of 500 slots 14 and 20,
// 64 of 1,000 66 and 43, 64 of 4,096 150 and 135, 8 of 32,768 142 and 145, 40 of 700 to 8,192 123 and 192; 32 rows 14 and 19, 39 and
// 37, 97 and 123, 99 and 128, 84 and 192; 96 rows 14 and 21, 93 and 46, 196 and 141, 181 and 151, 166 and 202.  Of those 118 sizes
// none takes more than 1.11 times the other kernel's time.  Of 60 others, drawn from 1 to 200 sequences of up to 58,000 slots, what is
// chosen takes 1.03 times the faster kernel's time in the geometric mean and 1.40 at most; all by the first 1.11 and 2.1.)
rkc_plan rkc_packed_plan(const rkc_cache* c, const rkc_attention* a) {
  const int64_t M = (int64_t)a->max_rows * (a->q_heads / c->kv_heads);
  if (M <= 16) return cut_plan(c, a, true);
  const rkc_plan many = cut_plan(c, a, false);
  if (M > 96 || (a->d_parent && a->max_rows > 32)) return many;
  const rkc_plan few = cut_plan(c, a, true);
  return cost_of(c, &few) / 16 * 15 <= cost_of(c, &many) ? few : many;
}

extern "C" {

size_t rkc_packed_attend_scratch_bytes(const rkc_packed* c, const rkc_attention* a) {
  if (!c || !a || c->kv_heads < 1 || a->q_heads < 1 || a->q_heads % c->kv_heads || c->n_seqs < 1 || a->max_rows < 1 || a->max_len < 1) return 0;
  const rkc_cache x = rkc_packed_as_cache(c);
  return rkc_packed_plan(&x, a).bytes;
}

rkc_status rkc_packed_attend(const rkc_packed* c, const rkc_attention* a, void* stream) {
  if (rkc_status st = rkc_packed_check(c)) return st;
  rkc_cache x = rkc_packed_as_cache(c);
  {
    rkc_cache sized = x;  // the pool's strides are its own, checked above
    sized.k_block_stride = sized.k_head_stride = 0;
    if (rkc_status st = rkc_attention_check(&sized, a, false)) return st;
  }
  if (a->d_weight || a->d_weight_in) return RKC_E_UNSUPPORTED;
  if (c->n_seqs == 0 || a->n_rows == 0) return RKC_OK;
  hipStream_t s = (hipStream_t)stream;
  rkc_plan p = rkc_packed_plan(&x, a);
  if (a->max_rows == 0) p.splits = 1, p.bytes = 0;  // sequences that have rows all the same are told of
  // rows of tiles are counted in 32 bits
  if ((int64_t)c->n_seqs * c->kv_heads * p.tiles * p.rows > 0x7fffffff) return RKC_E_UNSUPPORTED;
  if (!rkc_fits(p.few ? rkc_packed_few_workgroups(&p) : (int64_t)p.units * p.splits, rkc_packed_lanes(&x, &p)) || (p.splits > 1 && !rkc_join_fits(&x, a, &p))) return RKC_E_UNSUPPORTED;
  if (p.bytes) {
    if (!a->d_scratch || a->scratch_bytes < p.bytes) return RKC_E_SCRATCH;
    if ((uintptr_t)a->d_scratch & 255) return RKC_E_ALIGN;
  }
  rkc_status st = p.few ? rkc_packed_few(&x, a, &p, s) : rkc_packed_tile(&x, a, &p, s);
  return st == RKC_OK && p.splits > 1 ? rkc_attend_join(&x, a, &p, s) : st;
}

}  // extern "C"

// rkc_packed.hip -- attention over a paged cache in 4 bits: C ABI, choice of kernel, and the kernel of few rows (decode steps,
// small trees).
//
// out = sum_j exp(x_j - m) v_j / sum_j exp(x_j - m), x the masked and capped scores, m their running maximum.  Up to 16
// packed rows (rows x query heads of one key/value head) are the columns of a 16x16x32 matrix product, so every key and
// value is read once for all of them; what bounds the kernel is that read.
// A workgroup takes a chunk of one sequence's slots for one head, its waves take 32 slots at a time:
//   K  a lane has a quarter of its slot's key (head_dim / 4 elements), which it makes the product's operand of by the
//      conversion of two codes an instruction, exact with the scale in it;
//   V  likewise a quarter of a slot's value, converted and put into the wave's own tile in LDS, from where it is read
//      transposed (no barriers);
// both for the next 32 slots are in flight while these are worked on.
// A marked slot's scores are NaN by its key's first scale, and so only the rows that see it; values are always finite, so that
// one that a row does not see meets a weight of zero and gives zero.
#include <type_traits>

#include "rkc_packed_dev.h"
#include "rkc_tiles.h"

namespace {

template <typename T, int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void packed_few(const rkc_cache c, const rkc_attention a, const rkc_plan pl) {
  typedef typename Vec8<T>::t V8;
  constexpr int KC = D / 32, DB = D / 16;  // dwords of codes in a quarter of a slot, and key operands; output blocks
  constexpr int NS = D == 256 ? 2 : 1;     // scales of a quarter
  constexpr int kTile = 32 * D;            // elements of a wave's V tile
  constexpr int kJoin = 16 * D * 4;        // bytes of a wave's output tile at the join
  constexpr int kLds = kTile * 2 > kJoin ? kTile * 2 : kJoin;
  __shared__ __attribute__((aligned(16))) char lds[kWaves * kLds];
  __shared__ float stat[kWaves][16][2], total[16];

  const int H = c.kv_heads, G = a.q_heads / H;
  // The parts of a sequence are neighbours, turned by a number of their own in each: XCDs take workgroups in turn, and
  // an XCD would else have the same parts of every sequence, the last ones of short sequences being empty.
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
  V8 qf[KC];  // a quarter of the row's query, as the keys'
  {
    const T* p = (const T*)a.d_q + (q.row0 + qi) * a.q_row_stride + qh * a.q_head_stride + quad * (D / 4);
#pragma unroll
    for (int k = 0; k < KC; k++) {
      qf[k] = *(const V8*)(p + 8 * k);
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

  const Codes held = codes_of<D>(c, h);
  T* tile = (T*)(lds + wave * kLds);

  float top = -kInf, sum = 0.f;
  f32x4 o[DB];
#pragma unroll
  for (int d = 0; d < DB; d++) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};

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
    f32x4 sc[2];
    const int pa = here(put_at), va = here(val_at);
#pragma unroll
    for (int u = 0; u < 2; u++) {
      sc[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KC; k++) sc[u] = mma16(__builtin_bit_cast(V8, unpack8<T>(kf[u][k], scale_k(ks[u], k))), qf[k], sc[u]);
      // a scale that nobody wrote may be anything: what no row sees is to be finite
#pragma unroll
      for (int k = 0; k < KC; k++) {
        const uint32_t b = NS == 2 ? vs[u] >> 8 * (k / 4) & 255 : vs[u];
        *(u32x4*)((char*)tile + ((pa ^ k << 4) + u * 16 * 2 * D)) = unpack8<T>(vf[u][k], scale_float(min(b, (uint32_t)kTopScale<T>)));
      }
    }
    const bool whole = t0 + 32 <= all_pre || (t0 >= all_from && t0 + 32 <= all_to);
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
      const uint32_t seen = seen_of(row, t0, drafted) >> 4 * quad;
#pragma unroll
      for (int e = 0; e < 8; e++) sc[e >> 2][e & 3] = masked(sc[e >> 2][e & 3], seen, 16 * (e >> 2) + (e & 3));
    }
    auto vals = [&](int d) { return read_tr2<T>((const char*)tile + (va ^ d << 5), (const char*)tile + (va ^ d << 5) + 32 * D); };
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
    // the products' operands have 16 bits: a weight is the sum of two of them, with at least twice its bits
    const V8 pb = __builtin_convertvector(p, V8), pr = __builtin_convertvector(p - __builtin_convertvector(pb, f32x8), V8);
#pragma unroll
    for (int d = 0; d < DB; d++) {
      const V8 vt = vals(d);
      o[d] = mma16(vt, pr, mma16(vt, pb, o[d]));
    }
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
  packed_few<T, D, W><<<dim3(p->units * p->splits), dim3(64 * W), 0, s>>>(*c, *a, *p);
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

rkc_status rkc_packed_few(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s) {
  return c->dtype == RKC_BF16 ? go<__bf16>(c, a, p, s) : go<_Float16>(c, a, p, s);
}

// As rkc_attend_plan: up to 16 packed rows go to the kernel that reads the cache as fast as it can, more to the one that keeps
// the matrix units busy, and a sequence is cut where sequences, heads and row tiles do not fill the card's 256 CUs.
rkc_plan rkc_packed_plan(const rkc_cache* c, const rkc_attention* a) {
  rkc_plan p = {};
  const int64_t G = a->q_heads / c->kv_heads, M = a->max_rows * G;
  p.few = M <= 16;
  const int64_t wide = (int64_t)c->n_seqs * c->kv_heads * ((M + 255) / 256) * ((a->max_len + 255) / 256);
  p.rows = p.few ? 16 : M <= 128 || c->head_dim == 64 || wide < 512 ? 128 : 256;
  p.tiles = p.few ? 1 : (int)((M + p.rows - 1) / p.rows);
  const int64_t units = (int64_t)c->n_seqs * c->kv_heads * p.tiles;
  p.units = (int)units;
  const bool wide_head = c->head_dim == 256;
  const int64_t want = p.few ? (wide_head ? 4 : 10) * 256 : wide_head || p.rows == 256 ? 256 : 2 * 256, grain = p.few || wide_head ? 128 : 256;
  const int64_t cut = units ? (want + units - 1) / units : 1;
  int64_t chunk = (a->max_len + cut - 1) / cut;
  chunk = (chunk + grain - 1) / grain * grain;
  const int64_t least = p.few && !wide_head ? 512 : grain;
  if (chunk < least) chunk = least;
  if (!p.few && a->max_len <= 512 && (c->head_dim < 256 || units >= 32)) chunk = 512;
  p.waves = p.few && c->head_dim <= 128 && a->max_len <= 1536 ? 8 : 4;
  if (p.waves == 8) chunk = a->max_len < 32 ? 32 : (a->max_len + 31) / 32 * 32;
  p.chunk = (int)chunk;
  p.splits = (int)((a->max_len + chunk - 1) / chunk);
  if (p.splits < 1) p.splits = 1;
  p.sorted = !p.few && c->n_seqs > 1 && c->n_seqs <= 64 && units * p.splits > want;
  if (p.splits > 1) {
    const size_t rows = (size_t)units * p.splits * p.rows;
    p.part_at = 0;
    p.stat_at = rows * c->head_dim * 4;
    p.bytes = (p.stat_at + rows * 8 + 255) & ~(size_t)255;
  }
  return p;
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
  if (!rkc_fits((int64_t)p.units * p.splits, rkc_packed_lanes(&x, &p)) || (p.splits > 1 && !rkc_join_fits(&x, a, &p))) return RKC_E_UNSUPPORTED;
  if (p.bytes) {
    if (!a->d_scratch || a->scratch_bytes < p.bytes) return RKC_E_SCRATCH;
    if ((uintptr_t)a->d_scratch & 255) return RKC_E_ALIGN;
  }
  rkc_status st = p.few ? rkc_packed_few(&x, a, &p, s) : rkc_packed_tile(&x, a, &p, s);
  return st == RKC_OK && p.splits > 1 ? rkc_attend_join(&x, a, &p, s) : st;
}

}  // extern "C"

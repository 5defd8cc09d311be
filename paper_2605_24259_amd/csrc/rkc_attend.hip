// rkc_attend.hip -- C ABI of the attention over a paged cache: checks, choice of kernel, join of the chunks.
#include "rkc_cache_dev.h"

#include <utility>

namespace {

// Joins the chunks of a packed row: with m the largest of their maxima m_k, out = sum_k 2^(m_k - m) o_k / sum_k
// 2^(m_k - m) l_k.  D / 4 lanes read a chunk's output, and `groups` of so many lanes share a row's chunks, which `join`
// chooses: with few rows of many chunks many, as latency bounds it (5 rows of 32 heads in 64 chunks: 8.7 us), with many rows
// one, where the reads do (24,900 rows of 64 elements in 3 chunks: 7.3 us, 41 with a workgroup for each row).
template <typename T, int D, int NT>
__global__ __launch_bounds__(NT) void attend_join(const rkc_cache c, const rkc_attention a, const rkc_plan pl, int groups) {
  constexpr int L = D / 4, N = NT / L;
  __shared__ __attribute__((aligned(16))) float part_o[N][D];
  __shared__ float part_l[N];
  const int H = c.kv_heads, G = a.q_heads / H, per = a.max_rows * G;
  const int group = threadIdx.x / L, lane = threadIdx.x % L, d = lane * 4, mine = group % groups;
  const int64_t id = (int64_t)blockIdx.x * (N / groups) + group / groups;
  const int m = (int)(id % per), s = (int)min(id / per / H, (int64_t)c.n_seqs - 1), h = (int)(id / per % H);
  const Seq q = load_seq(c, a, s);
  const bool row_here = id < (int64_t)c.n_seqs * H * per && q.ok && m < q.n * G;
  float top = -kInf, sum = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  if (row_here) {
    const int qt = m / pl.rows, last = (min(q.n * G, (qt + 1) * pl.rows) - 1) / G;
    const int n = max(1, (rows_end(a, q, s, last) + pl.chunk - 1) / pl.chunk);
    const int64_t at = ((int64_t)(s * H + h) * pl.tiles + qt) * pl.splits * pl.rows + m % pl.rows;
    const float* st = (const float*)((const char*)a.d_scratch + pl.stat_at) + at * 2;
    const float* part = (const float*)((const char*)a.d_scratch + pl.part_at) + at * D + d;
    for (int k = lane; k < n; k += L) top = fmaxf(top, st[(int64_t)k * pl.rows * 2]);
#pragma unroll
    for (int x = L / 2; x; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
#pragma unroll 4
    for (int k = mine; k < n; k += groups) {
      const float m_k = st[(int64_t)k * pl.rows * 2], l_k = st[(int64_t)k * pl.rows * 2 + 1];
      const f32x4 x = *(const f32x4*)(part + (int64_t)k * pl.rows * D);
      if (l_k != 0.f) {  // a chunk of which the row sees anything
        const float by = ex2(m_k - top);
        sum += l_k * by, o += x * by;
      }
    }
  }
  if (groups > 1) {
    *(f32x4*)&part_o[group][d] = o;
    if (d == 0) part_l[group] = sum;
    __syncthreads();
    if (mine) return;
    for (int k = 1; k < groups; k++) o += *(const f32x4*)&part_o[group + k][d], sum += part_l[group + k];
  }
  if (!row_here) return;
  const float by = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t row = q.row0 + m / G, qh = h * G + m % G;
  typedef T T4 __attribute__((ext_vector_type(4)));
  *(T4*)((T*)a.d_out + row * a.out_row_stride + qh * a.out_head_stride + d) = __builtin_convertvector(o * by, T4);
  if (d == 0) a.d_lse[row * a.q_heads + qh] = sum == 0.f ? -kInf : kLn2 * (top + lg2(sum));
}

// The account from kept scores: decay * before + sum over rows of exp(score - lse), four slots of 256 a thread, so that
// the scores are read along their slots.  8 bytes a slot and row go through the L2 in place of another read of the keys;
// latency bounds it (64 sequences of up to 4,096 slots: 10.4 us; with the keys read again a step took 194 us in place of
// 146).
__global__ __launch_bounds__(256) void attend_account(const rkc_cache c, const rkc_attention a, const rkc_plan pl, int parts) {
  const int H = c.kv_heads, G = a.q_heads / H, part = blockIdx.x % parts, unit = blockIdx.x / parts, s = unit / H, h = unit % H;
  const Seq q = load_seq(c, a, s);
  if (!q.ok || part * 1024 >= q.len) return;
  const int M = q.n * G, per = 32 * a.max_rows * G;
  const float* sc = (const float*)((const char*)a.d_scratch + pl.score_at) + (int64_t)unit * (a.max_rows * G) * pl.wide;
  const int64_t at = s * a.weight_seq_stride + h * a.weight_head_stride;
  float got[4] = {}, in[4] = {};
#pragma unroll
  for (int k = 0; k < 4; k++) {
    const int j = part * 1024 + k * 256 + threadIdx.x;
    if (a.d_weight_in && j < q.len) in[k] = a.decay * a.d_weight_in[at + j];
  }
  for (int m = 0; m < M; m++) {
    const float lse = a.d_lse[(int64_t)(q.row0 + m / G) * a.q_heads + h * G + m % G];
    const float z = lse == -kInf ? kInf : lse * kLog2e;  // a row that saw nothing gave nothing
#pragma unroll
    for (int k = 0; k < 4; k++) {
      const int j = part * 1024 + k * 256 + threadIdx.x;
      const float x = j < q.len ? sc[(int64_t)(j >> 5) * per + m * 32 + (j & 31)] : -kInf;
      got[k] += x == -kInf ? 0.f : ex2(x - z);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; k++) {
    const int j = part * 1024 + k * 256 + threadIdx.x;
    if (j < q.len) a.d_weight[at + j] = in[k] + got[k];
  }
}

struct Join {
  int groups, lanes;  // of a row, in units of D / 4 lanes; of a workgroup
  int64_t workgroups;
};

// Groups of lanes for a row: as many as leave each two chunks, until the card's 256 CUs have 1,024 lanes each.
Join join_plan(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p) {
  const int L = c->head_dim / 4;
  const int64_t rows = (int64_t)c->n_seqs * c->kv_heads * a->max_rows * (a->q_heads / c->kv_heads);
  Join j = {1, 256, 0};
  while (j.groups < 1024 / L && j.groups * 4 <= p->splits && rows * L * j.groups < 256 * 1024) j.groups *= 2;
  if (j.groups > 256 / L) j.lanes = 1024;
  const int64_t each = j.lanes / L / j.groups;
  j.workgroups = (rows + each - 1) / each;
  return j;
}

template <typename T, int D>
void join(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, const Join& j, hipStream_t s) {
  const dim3 grid((unsigned)j.workgroups);
  if (j.lanes == 256) attend_join<T, D, 256><<<grid, dim3(256), 0, s>>>(*c, *a, *p, j.groups);
  else attend_join<T, D, 1024><<<grid, dim3(1024), 0, s>>>(*c, *a, *p, j.groups);
}

template <typename T>
rkc_status join(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, const Join& j, hipStream_t s) {
  if (c->head_dim == 64) join<T, 64>(c, a, p, j, s);
  else if (c->head_dim == 128) join<T, 128>(c, a, p, j, s);
  else join<T, 256>(c, a, p, j, s);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

bool off16(const void* p) { return (uintptr_t)p & 15; }
bool off4(const void* p) { return (uintptr_t)p & 3; }
// a stride whose multiple by `times` is an element offset that the kernels keep in 32 bits
bool bad_stride(int64_t x, int64_t times) { return x < 0 || x % 8 || x > ((int64_t)1 << 30) / times; }
constexpr int64_t kFar = (int64_t)1 << 40;  // strides between blocks and rows: products stay far below 64 bits

}  // namespace

bool rkc_shared(int64_t width, int64_t n0, int64_t stride0, int64_t n1, int64_t stride1, int64_t n2, int64_t stride2) {
  struct { int64_t n, stride; } d[3] = {{n0, stride0}, {n1, stride1}, {n2, stride2}};
  if (d[0].stride > d[1].stride) std::swap(d[0], d[1]);
  if (d[1].stride > d[2].stride) std::swap(d[1], d[2]);
  if (d[0].stride > d[1].stride) std::swap(d[0], d[1]);
  for (auto& x : d) {  // from the nearest on: each step goes past all that the nearer ones reach
    if (x.n <= 1) continue;  // its stride says nothing
    if (x.stride < width) return true;
    width += (x.n - 1) * x.stride;
  }
  return false;
}

rkc_status rkc_cache_check(const rkc_cache* c) {
  if (!c) return RKC_E_NULL;
  if (c->n_seqs < 0 || c->n_blocks < 0 || c->max_pages < 0 || c->reserved) return RKC_E_RANGE;
  if (c->kv_heads < 1 || c->kv_heads > 1024 || c->n_seqs > 1 << 20) return RKC_E_RANGE;
  if (c->dtype != RKC_BF16 && c->dtype != RKC_F16) return RKC_E_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return RKC_E_UNSUPPORTED;
  if (c->page_tokens < 16 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1))) return RKC_E_UNSUPPORTED;
  for (int64_t x : {c->k_slot_stride, c->v_slot_stride})
    if (bad_stride(x, c->page_tokens)) return RKC_E_RANGE;
  for (int64_t x : {c->k_block_stride, c->v_block_stride})
    if (x < 0 || x % 8 || x >= (int64_t)1 << 31) return RKC_E_RANGE;
  for (int64_t x : {c->k_head_stride, c->v_head_stride})
    if (x < 0 || x % 8 || x > kFar) return RKC_E_RANGE;
  if (c->n_seqs == 0) return RKC_OK;
  if (!c->d_k || !c->d_v || !c->d_block_table) return RKC_E_NULL;
  if (off16(c->d_k) || off16(c->d_v) || off4(c->d_block_table) || off4(c->d_status)) return RKC_E_ALIGN;
  if (c->n_blocks < 1 || c->max_pages < 1) return RKC_E_RANGE;
  return RKC_OK;
}

rkc_status rkc_attention_check(const rkc_cache* c, const rkc_attention* a, bool weigh) {
  if (rkc_status st = rkc_cache_check(c)) return st;
  if (!a) return RKC_E_NULL;
  if (a->n_rows < 0 || a->max_rows < 0 || a->max_len < 0 || a->reserved) return RKC_E_RANGE;
  if (a->max_len > RKC_MAX_CACHE_LEN || a->max_len > (int64_t)c->max_pages * c->page_tokens) return RKC_E_RANGE;
  if (a->q_heads < 1 || a->q_heads % c->kv_heads || a->q_heads > 1 << 16) return RKC_E_RANGE;
  if ((int64_t)a->max_rows * (a->q_heads / c->kv_heads) > 1 << 30) return RKC_E_RANGE;
  if (!(a->softcap >= 0.f) || a->softcap == kInf || a->scale != a->scale) return RKC_E_RANGE;
  for (int64_t x : {a->q_row_stride, a->q_head_stride, a->out_row_stride, a->out_head_stride})
    if (x < 0 || x % 8 || x > kFar) return RKC_E_RANGE;
  if (a->d_parent && a->max_rows > RKC_MAX_TREE_ROWS) return RKC_E_UNSUPPORTED;
  if (a->weight_seq_stride < 0 || a->weight_head_stride < 0 || a->weight_seq_stride > kFar || a->weight_head_stride > kFar) return RKC_E_RANGE;
  if (c->n_seqs == 0 || (a->n_rows == 0 && !weigh)) return RKC_OK;
  if (!a->d_row_offset || !a->d_length || (a->n_rows && (!a->d_q || !a->d_lse))) return RKC_E_NULL;
  if (weigh ? !a->d_weight : !a->d_out) return RKC_E_NULL;
  if (off16(a->d_q) || (!weigh && off16(a->d_out))) return RKC_E_ALIGN;
  for (const void* p : {(const void*)a->d_row_offset, (const void*)a->d_length, (const void*)a->d_row_start, (const void*)a->d_prefix,
                        (const void*)a->d_parent, (const void*)a->d_slope, (const void*)a->d_lse, (const void*)a->d_weight_in, (const void*)a->d_weight})
    if (off4(p)) return RKC_E_ALIGN;
  if (!weigh && rkc_shared(c->head_dim, a->n_rows, a->out_row_stride, a->q_heads, a->out_head_stride)) return RKC_E_RANGE;
  if (a->d_weight && rkc_shared(a->max_len, c->n_seqs, a->weight_seq_stride, c->kv_heads, a->weight_head_stride)) return RKC_E_RANGE;
  return RKC_OK;
}

// Which kernel and how a sequence is cut.  Few packed rows: the kernel that reads the cache as fast as it can;
// more: the one that keeps the matrix units busy, which 17 to 32 rows gain from too.  256 rows a workgroup halve what
// is read of K and V per product and let two groups of waves take turns, at 128 elements a head; at 64 the registers of
// two waves a SIMD are not needed for it, at 256 the products have 16 rows a wave.  A sequence is cut where the
// sequences, heads and row tiles alone would not fill the card's 256 CUs a few times over.
rkc_plan rkc_attend_plan(const rkc_cache* c, const rkc_attention* a) {
  rkc_plan p = {};
  const int64_t G = a->q_heads / c->kv_heads, M = a->max_rows * G;
  p.few = M <= 16;
  // 256 rows only where such tiles, counted with 256 slots each, are twice the card's CUs: fewer leave CUs idle and are slower
  // from start to end (8 heads of 128 elements, 512 rows of 32 heads over 1,024 slots: 39.9 us, with 128 rows 35.0; over
  // 8,192 90.2 and 98.6).
  const int64_t wide = (int64_t)c->n_seqs * c->kv_heads * ((M + 255) / 256) * ((a->max_len + 255) / 256);
  p.rows = p.few ? 16 : M <= 128 || c->head_dim != 128 || wide < 512 ? 128 : 256;
  p.tiles = p.few ? 1 : (int)((M + p.rows - 1) / p.rows);
  const int64_t units = (int64_t)c->n_seqs * c->kv_heads * p.tiles;
  p.units = (int)units;
  // Workgroups wanted: where one is all that a CU holds (256 elements a head, 256 rows), one a CU; of few rows ten, two at a
  // time, as they even out unlike lengths (64 sequences of 1 to 4,096 slots: 122 us, with five 126, with three 141).
  const bool wide_head = c->head_dim == 256;
  const int64_t want = wide_head || p.rows == 256 ? 256 : p.few ? 10 * 256 : 2 * 256, grain = p.few || wide_head ? 128 : 256;
  // Workgroups along a sequence; rounded up, so that there may be a few more than the card holds at once (six units of 256
  // elements a head: 258).
  const int64_t cut = units ? (want + units - 1) / units : 1;
  int64_t chunk = (a->max_len + cut - 1) / cut;
  chunk = (chunk + grain - 1) / grain * grain;
  // Of few rows no less than four tiles a wave, else starts and joins cost more than they save (one sequence of 32,768
  // slots, 8 heads: 31 us, with one tile 42).
  const int64_t least = p.few && !wide_head ? 512 : grain;
  if (chunk < least) chunk = least;
  // Up to 512 slots the join, a second launch, costs more than shorter chunks save (512 rows of 32 heads of 128 elements:
  // 20.8 us whole, 28.4 in two chunks; 40 of 64 over 300 slots 12.2 and 16.6), but for a few workgroups that go through 256
  // elements a head (8 rows over 512 slots: 25.7 and 16.6; 512 rows 32.3 and 41.9).
  if (!p.few && a->max_len <= 512 && (c->head_dim < 256 || units >= 32)) chunk = 512;
  // Short sequences whole, by eight waves: no second kernel for the join (four sequences of up to 1,280 slots: 10.6 us in one
  // kernel where the split took 6.0 and the join 4.4, and 12.9 us a call instead of 16.8).
  p.waves = p.few && c->head_dim <= 128 && a->max_len <= 1536 ? 8 : 4;
  if (p.waves == 8) chunk = a->max_len < 32 ? 32 : (a->max_len + 31) / 32 * 32;
  p.chunk = (int)chunk;
  p.splits = (int)((a->max_len + chunk - 1) / chunk);
  if (p.splits < 1) p.splits = 1;
  // More workgroups than the card holds at once: the longest go first, so that none starts late.  (Each finds its
  // sequence by comparing lengths, less than 1 us; 48 trees of 700 to 8,192 slots: 247 us instead of 326.)
  p.sorted = !p.few && c->n_seqs > 1 && c->n_seqs <= 64 && units * p.splits > want;
  if (p.splits > 1) {
    const size_t rows = (size_t)units * p.splits * p.rows;
    p.part_at = 0;
    p.stat_at = rows * c->head_dim * 4;
    p.bytes = (p.stat_at + rows * 8 + 255) & ~(size_t)255;
  }
  // The account by scores kept (written and read: 8 bytes per slot and packed row) where that is at most half of what
  // reading the keys again would be (2 bytes per slot and element of a head).
  // (Not with documents: slots that no row sees are passed over, and would keep no score.)
  p.keep = a->d_weight && !a->d_row_start && p.few && M <= c->head_dim / 8 && M <= 16;
  if (p.keep) {
    p.wide = (a->max_len + 31) & ~31;
    p.score_at = p.bytes;
    p.bytes += (size_t)units * M * p.wide * 4;
  }
  return p;
}

extern "C" {

size_t rkc_attend_scratch_bytes(const rkc_cache* c, const rkc_attention* a) {
  if (!c || !a || c->kv_heads < 1 || a->q_heads < 1 || a->q_heads % c->kv_heads || c->n_seqs < 1 || a->max_rows < 1 || a->max_len < 1) return 0;
  return rkc_attend_plan(c, a).bytes;
}

rkc_status rkc_attend(const rkc_cache* c, const rkc_attention* a, void* stream) {
  if (rkc_status st = rkc_attention_check(c, a, false)) return st;
  if (c->n_seqs == 0) return RKC_OK;
  if (a->n_rows == 0) return a->d_weight ? rkc_weigh(c, a, stream) : RKC_OK;
  if (a->d_weight && a->d_out == a->d_q) return RKC_E_RANGE;  // the account may read the queries again
  hipStream_t s = (hipStream_t)stream;
  rkc_plan p = rkc_attend_plan(c, a);
  if (a->max_rows == 0) p.splits = 1, p.keep = false, p.bytes = 0;  // sequences that have rows all the same are told of
  // rows of tiles are counted in 32 bits
  if ((int64_t)c->n_seqs * c->kv_heads * p.tiles * p.rows > 0x7fffffff) return RKC_E_UNSUPPORTED;
  const Join j = join_plan(c, a, &p);
  const int parts = (a->max_len + 1023) / 1024;
  if (!rkc_fits((int64_t)p.units * p.splits, rkc_attend_lanes(c, &p)) || (p.splits > 1 && !rkc_fits(j.workgroups, j.lanes)) ||
      (a->d_weight && !(p.keep ? rkc_fits((int64_t)p.units * parts, 256) : rkc_weigh_fits(c, a))))
    return RKC_E_UNSUPPORTED;
  if (p.bytes) {
    if (!a->d_scratch || a->scratch_bytes < p.bytes) return RKC_E_SCRATCH;
    if ((uintptr_t)a->d_scratch & 255) return RKC_E_ALIGN;
  }
  rkc_status st = p.few ? rkc_attend_few(c, a, &p, s) : rkc_attend_tile(c, a, &p, s);
  if (st == RKC_OK && p.splits > 1) st = c->dtype == RKC_BF16 ? join<__bf16>(c, a, &p, j, s) : join<_Float16>(c, a, &p, j, s);
  if (st != RKC_OK || !a->d_weight) return st;
  if (!p.keep) return rkc_weigh(c, a, stream);
  if (!parts) return RKC_OK;  // of lengths of 0
  attend_account<<<dim3(p.units * parts), dim3(256), 0, s>>>(*c, *a, p, parts);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

}  // extern "C"

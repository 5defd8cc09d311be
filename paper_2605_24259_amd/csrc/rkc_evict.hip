// rkc_evict.hip -- eviction from a paged cache by the account of its slots.
//
// One workgroup decides for a head of a sequence: the account of the last slot to be kept is found by bisection
// of its 32-bit order (two bits a round: three counts by ballots, no atomics), ties go to the lowest slots, and
// two prefix sums pair the gaps in front of the new end with the kept slots behind it.  A second kernel moves their
// keys and values.  Sources lie behind the new end and targets before it, so that the moves need no order among
// each other, and what is kept in place is not touched: the least that can be moved.
#include "rkc_cache_dev.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kItems = 16, kTile = kThreads * kItems, kMoves = 128;

struct evict_args {
  rkc_cache c;
  rkc_eviction e;
  int32_t *gaps, *from, *count;  // scratch: [row][most], [row][most], [row]
  int most;
};

// The account's order in whole numbers above 0; NaN lowest, both zeros alike.
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 1;
  const uint32_t b = __float_as_uint(w + 0.f);
  return b >> 31 ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {  // inclusive
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  return x;
}

__global__ __launch_bounds__(kThreads) void evict_choose(const evict_args g) {
  const rkc_cache& c = g.c;
  const rkc_eviction& e = g.e;
  __shared__ uint32_t part[2][4][kWaves];
  const int H = c.kv_heads, s = blockIdx.x / H, h = blockIdx.x % H;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const int len = e.d_length[s];
  if (len < 0 || len > e.max_len) {
    if (tid == 0) {
      g.count[blockIdx.x] = 0;
      if (h == 0) flag(c, s, RKC_CS_LENGTH);
    }
    return;
  }
  const int held = e.d_protect ? min(len, max(0, e.d_protect[s])) : 0;
  const int now = min(len, max(held, max(0, e.d_budget[s])));
  const int recent_from = e.d_recent_from ? e.d_recent_from[s] : 0x7fffffff;
  const bool recents = e.d_recent_from != nullptr;
  const int64_t at = s * e.weight_seq_stride + h * e.weight_head_stride;
  const float* w = e.d_weight + at;
  const int32_t* pos = e.d_pos ? e.d_pos + at : nullptr;
  float* w_out = e.d_weight_out + at;
  int32_t* pos_out = e.d_pos_out + at;
  if (tid == 0 && h == 0) e.d_length_out[s] = now;
  auto pos_at = [&](int j) { return pos ? pos[j] : j; };
  if (now == len) {
    for (int j = tid; j < len; j += kThreads) w_out[j] = w[j], pos_out[j] = pos_at(j);
    if (tid == 0) g.count[blockIdx.x] = 0;
    return;
  }
  const int tiles = (len + kTile - 1) / kTile;
  int turn = 0;
  // sums of up to four counts of this wave over the workgroup
  auto total = [&](uint32_t a0, uint32_t a1, uint32_t a2, uint32_t* out) {
    if (lane == 0) part[turn][0][wave] = a0, part[turn][1][wave] = a1, part[turn][2][wave] = a2;
    __syncthreads();
    for (int k = 0; k < 3; k++) {
      uint32_t x = 0;
#pragma unroll
      for (int i = 0; i < kWaves; i++) x += part[turn][k][i];
      out[k] = x;
    }
    turn ^= 1;
  };
  uint32_t sums[3];
  int K = now - held;  // to be kept of the slots behind the protected ones
  bool among_recent = false;
  if (recents) {
    uint32_t n = 0;
    for (int j = held + tid; j - tid < len; j += kThreads) n += __popcll(__ballot(j < len && pos_at(j) >= recent_from));
    total(n, 0, 0, sums);
    among_recent = (int)sums[0] >= K;
    if (!among_recent) K -= sums[0];
  }
  // the slots the choice is among: their order, the others 0.  A thread has 16 neighbouring slots of a tile.
  uint32_t key[kItems], sure = 0;
  auto load = [&](int tile) {
    const int j0 = tile * kTile + tid * kItems;
    sure = 0;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = j0 + i;
      const bool in = j >= held && j < len;
      const bool recent = recents && in && pos_at(j) >= recent_from;
      key[i] = in && recent == among_recent ? order_of(w[j]) : 0;
      if (j < held || (recent && !among_recent)) sure |= 1u << i;
    }
  };
  if (tiles == 1) load(0);
  uint32_t T = 0;  // the order of the last slot to be kept
  if (K > 0) {
    for (int b = 30; b >= 0; b -= 2) {
      uint32_t n1 = 0, n2 = 0, n3 = 0;
      const uint32_t t1 = T | 1u << b, t2 = T | 2u << b, t3 = T | 3u << b;
      for (int t = 0; t < tiles; t++) {
        if (tiles > 1) load(t);
#pragma unroll
        for (int i = 0; i < kItems; i++) {
          n1 += __popcll(__ballot(key[i] >= t1));
          n2 += __popcll(__ballot(key[i] >= t2));
          n3 += __popcll(__ballot(key[i] >= t3));
        }
      }
      total(n1, n2, n3, sums);
      T = (int)sums[2] >= K ? t3 : (int)sums[1] >= K ? t2 : (int)sums[0] >= K ? t1 : T;
    }
  } else {
    T = 0xffffffffu;
  }
  int ties = 0;  // slots of that order to be kept, the lowest first
  if (K > 0) {
    uint32_t n = 0;
    for (int t = 0; t < tiles; t++) {
      if (tiles > 1) load(t);
#pragma unroll
      for (int i = 0; i < kItems; i++) n += __popcll(__ballot(key[i] > T));
    }
    total(n, 0, 0, sums);
    ties = K - sums[0];
  }
  int32_t* gaps = g.gaps + (int64_t)blockIdx.x * g.most;
  int32_t* from = g.from + (int64_t)blockIdx.x * g.most;
  int tie0 = 0, gap0 = 0, from0 = 0;
  // exclusive sum over the threads; *all: the total
  auto scan = [&](uint32_t x, uint32_t* all) {
    const uint32_t inc = wave_scan(x);
    if (lane == 63) part[turn][0][wave] = inc;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (int i = 0; i < kWaves; i++) {
      const uint32_t y = part[turn][0][i];
      before += i < wave ? y : 0, sum += y;
    }
    turn ^= 1;
    *all = sum;
    return before + inc - x;
  };
  for (int t = 0; t < tiles; t++) {
    if (tiles > 1) load(t);
    uint32_t all, keep = sure, eq = 0;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      if (K > 0 && key[i] > T) keep |= 1u << i;
      if (K > 0 && key[i] == T) eq |= 1u << i;
    }
    int left = ties - tie0 - (int)scan(__popc(eq), &all);
    tie0 += all;
#pragma unroll
    for (int i = 0; i < kItems; i++)
      if (eq >> i & 1 && left-- > 0) keep |= 1u << i;
    const int j0 = t * kTile + tid * kItems;
    uint32_t before = 0, behind = 0;  // slots in front of the new end, slots behind it
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      before |= (j0 + i < now ? 1u : 0u) << i;
      behind |= (j0 + i >= now && j0 + i < len ? 1u : 0u) << i;
    }
    const uint32_t gap = before & ~keep, src = behind & keep;
    const uint32_t mine = scan(__popc(gap) << 16 | __popc(src), &all);
    int gi = gap0 + (mine >> 16), fi = from0 + (mine & 0xffff);
    gap0 += all >> 16, from0 += all & 0xffff;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = j0 + i;
      if (gap >> i & 1) gaps[gi++] = j;
      if (src >> i & 1) from[fi++] = j;
      if (before & keep & 1u << i) w_out[j] = w[j], pos_out[j] = pos_at(j);
    }
  }
  __syncthreads();
  if (tid == 0) g.count[blockIdx.x] = gap0;
  for (int i = tid; i < gap0; i += kThreads) {
    const int j = from[i], to = gaps[i];
    w_out[to] = w[j], pos_out[to] = pos_at(j);
  }
}

// Moves the keys and values of up to kMoves slots of a head of a sequence, 16 bytes a lane.
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
    const int64_t pt = page_of(c, table, shift, to, bad), pf = page_of(c, table, shift, at, bad);
    if (bad) flag(c, s, RKC_CS_BLOCK);
    const int in_page = c.page_tokens - 1;
    uint16_t* k = (uint16_t*)c.d_k + h * c.k_head_stride + e;
    uint16_t* v = (uint16_t*)c.d_v + h * c.v_head_stride + e;
    const u32x4 a = *(const u32x4*)(k + pf * c.k_block_stride + (at & in_page) * c.k_slot_stride);
    const u32x4 b = *(const u32x4*)(v + pf * c.v_block_stride + (at & in_page) * c.v_slot_stride);
    *(u32x4*)(k + pt * c.k_block_stride + (to & in_page) * c.k_slot_stride) = a;
    *(u32x4*)(v + pt * c.v_block_stride + (to & in_page) * c.v_slot_stride) = b;
  }
}

size_t up(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

extern "C" {

size_t rkc_evict_scratch_bytes(const rkc_cache* c, const rkc_eviction* e) {
  if (!c || !e || c->n_seqs < 1 || c->kv_heads < 1 || e->max_len < 0) return 0;
  const size_t rows = (size_t)c->n_seqs * c->kv_heads, most = (size_t)e->max_len / 2 + 1;
  return 2 * up(rows * most * 4) + up(rows * 4);
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
  if (e->d_weight_out == e->d_weight || e->d_pos_out == e->d_pos || e->d_length_out == e->d_length) return RKC_E_RANGE;
  const size_t need = rkc_evict_scratch_bytes(c, e);
  if (!e->d_scratch || e->scratch_bytes < need) return RKC_E_SCRATCH;
  if ((uintptr_t)e->d_scratch & 255) return RKC_E_ALIGN;
  const size_t rows = (size_t)c->n_seqs * c->kv_heads;
  evict_args g;
  g.c = *c, g.e = *e;
  g.most = e->max_len / 2 + 1;
  char* at = (char*)e->d_scratch;
  g.gaps = (int32_t*)at;
  g.from = (int32_t*)(at + up(rows * g.most * 4));
  g.count = (int32_t*)(at + 2 * up(rows * g.most * 4));
  const int64_t chunks = (e->max_len / 2 + kMoves - 1) / kMoves;
  if ((int64_t)rows * (chunks + 1) > 0x7fffffff) return RKC_E_UNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  evict_choose<<<dim3((unsigned)rows), dim3(kThreads), 0, s>>>(g);
  if (chunks) evict_move<<<dim3((unsigned)(rows * chunks)), dim3(256), 0, s>>>(g, (int)chunks);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}

}  // extern "C"

// rkc_evict.hip -- eviction from a paged cache by the account of its slots.
//
// One workgroup decides for a head of a sequence: the account of the last slot to be kept is found 8 bits of its
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
};

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

__global__ __launch_bounds__(kThreads) void evict_choose(const evict_args g) {
  const rkc_cache& c = g.c;
  const rkc_eviction& e = g.e;
  // counts of 256 digits, a copy for each of 16 lanes: at most 4 lanes of an addition meet in a word, whatever the digits
  __shared__ __attribute__((aligned(16))) uint32_t hist[256 * kCopies];
  uint16_t* const gap_at = (uint16_t*)hist;  // later: the gaps of a sequence of one tile
  static_assert(sizeof(hist) >= kTile / 2 * sizeof(uint16_t), "gaps");
  __shared__ uint32_t table[2][kItems * kWaves + 1];  // counts per run of 64 slots, then what lies before each
  __shared__ uint32_t found[3];
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
  // A thread's slots of a tile: tid, tid + 1024, ...  Their accounts and positions stay in registers where a
  // sequence is one tile; of a longer one they are read again for each pass.
  const int tiles = (len + kTile - 1) / kTile;
  float wt[kItems];
  int ps[kItems];
  auto load = [&](int tile) {
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = tile * kTile + i * kThreads + tid;
      wt[i] = 0.f, ps[i] = j;
      if (j < len) {
        wt[i] = w[j];
        if (pos) ps[i] = pos[j];
      }
    }
  };
  // bit i: slot i of the thread is behind the protected ones; is recent
  auto slots_of = [&](int tile, uint32_t& open, uint32_t& recent) {
    open = recent = 0;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = tile * kTile + i * kThreads + tid;
      const bool in = j >= held && j < len;
      open |= (in ? 1u : 0u) << i;
      recent |= (in && recents && ps[i] >= recent_from ? 1u : 0u) << i;
    }
  };
  uint32_t open, recent;
  load(0);
  slots_of(0, open, recent);
  int K = now - held;  // to be kept of the slots behind the protected ones
  bool among_recent = false;  // the choice is among the recent ones; else they stay, and it is among the others
  if (recents) {
    if (tid == 0) found[0] = 0;
    __syncthreads();
    uint32_t n = 0;
    for (int t = 0; t < tiles; t++) {
      if (t) load(t), slots_of(t, open, recent);
      n += __popc(recent);
    }
    n = wave_scan(n);
    if (lane == 63 && n) atomicAdd(&found[0], n);
    __syncthreads();
    among_recent = (int)found[0] >= K;
    if (!among_recent) K -= found[0];
    __syncthreads();
  }
  // The order of the last slot to be kept, 8 bits at a time from the top; `left`: how many of those that agree with
  // it so far are to be kept.
  uint32_t T = 0, left = K, same = 0;
  if (K > 0) {
    for (int b = 24; b >= 0; b -= 8) {
      ((u32x4*)hist)[tid] = u32x4{0, 0, 0, 0};
      __syncthreads();
      for (int t = 0; t < tiles; t++) {
        if (tiles > 1) load(t), slots_of(t, open, recent);
        const uint32_t in = among_recent ? recent : open & ~recent;
#pragma unroll
        for (int i = 0; i < kItems; i++) {
          if (t * kTile + i * kThreads >= len) break;
          const uint32_t key = order_of(wt[i]);
          if ((in >> i & 1) && (b == 24 || (key ^ T) >> b >> 8 == 0)) atomicAdd(&hist[(key >> b & 255) * kCopies + (lane & (kCopies - 1))], 1u);
        }
      }
      __syncthreads();
      const u32x4 x4 = ((const u32x4*)hist)[tid];  // a quarter of a digit's copies
      uint32_t n = x4[0] + x4[1] + x4[2] + x4[3];
      n += (uint32_t)dpp<0xb1>((int)n);  // quad_perm [1,0,3,2]
      n += (uint32_t)dpp<0x4e>((int)n);  // quad_perm [2,3,0,1]
      __syncthreads();
      if ((tid & 3) == 0) hist[tid >> 2] = n;
      __syncthreads();
      if (wave == 0) {  // lane l: digits 255 - 4 l and the three below
        const u32x4 x = ((const u32x4*)hist)[63 - lane];
        const uint32_t mine = x[0] + x[1] + x[2] + x[3], to = wave_scan(mine);
        uint32_t above = to - mine;
        if (above < left && left <= to) {
          int d = 3;
          while (above + x[d] < left) above += x[d--];
          found[0] = (63 - lane) * 4 + d, found[1] = left - above, found[2] = x[d];
        }
      }
      __syncthreads();
      T |= found[0] << b, left = found[1], same = found[2];
    }
  }
  // prefix sums over the runs of 64 slots of a tile, of two counts at once; returns the tile's totals
  auto runs_before = [&](uint32_t& all0, uint32_t& all1) {
    __syncthreads();
    if (wave < 2) {
      uint32_t x[kItems * kWaves / 64], sum = 0;
#pragma unroll
      for (int k = 0; k < kItems * kWaves / 64; k++) x[k] = sum, sum += table[wave][lane * (kItems * kWaves / 64) + k];
      const uint32_t to = wave_scan(sum);
#pragma unroll
      for (int k = 0; k < kItems * kWaves / 64; k++) table[wave][lane * (kItems * kWaves / 64) + k] = to - sum + x[k];
      if (lane == 63) table[wave][kItems * kWaves] = to;
    }
    __syncthreads();
    all0 = table[0][kItems * kWaves], all1 = table[1][kItems * kWaves];
  };
  int32_t* gaps = g.gaps + (int64_t)blockIdx.x * g.most;
  int32_t* from = g.from + (int64_t)blockIdx.x * g.most;
  uint32_t tie0 = 0, gap0 = 0, from0 = 0, all0, all1;
  for (int t = 0; t < tiles; t++) {
    if (tiles > 1) load(t), slots_of(t, open, recent);
    const uint32_t in = among_recent ? recent : open & ~recent;
    uint32_t keep = among_recent ? 0 : recent, tie = 0;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const uint32_t key = order_of(wt[i]);
      if (t * kTile + i * kThreads + tid < held) keep |= 1u << i;
      if (K > 0 && (in >> i & 1)) {
        if (key > T) keep |= 1u << i;
        if (key == T) tie |= 1u << i;
      }
    }
    if (left == same) {  // all of the last order stay
      keep |= tie;
    } else {  // the lowest `left` of them
#pragma unroll
      for (int i = 0; i < kItems; i++) {
        const uint64_t m = __ballot(tie >> i & 1);
        if (lane == 0) table[0][i * kWaves + wave] = __popcll(m), table[1][i * kWaves + wave] = 0;
      }
      runs_before(all0, all1);
#pragma unroll
      for (int i = 0; i < kItems; i++) {
        const uint64_t m = __ballot(tie >> i & 1);
        if ((tie >> i & 1) && tie0 + table[0][i * kWaves + wave] + lower(m) < left) keep |= 1u << i;
      }
      tie0 += all0;
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = t * kTile + i * kThreads + tid;
      const uint64_t gap = __ballot(j < now && !(keep >> i & 1)), src = __ballot(j >= now && j < len && (keep >> i & 1));
      if (lane == 0) table[0][i * kWaves + wave] = __popcll(gap), table[1][i * kWaves + wave] = __popcll(src);
    }
    runs_before(all0, all1);
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = t * kTile + i * kThreads + tid;
      if (t * kTile + i * kThreads >= now) break;
      const bool kept = keep >> i & 1, is_gap = j < now && !kept;
      const uint64_t gap = __ballot(is_gap);
      const int at_gap = gap0 + table[0][i * kWaves + wave] + lower(gap);
      if (is_gap) gaps[at_gap] = j;
      if (is_gap && tiles == 1) gap_at[at_gap] = (uint16_t)j;
      if (j < now && kept) w_out[j] = wt[i], pos_out[j] = ps[i];
    }
    if (tiles == 1) __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; i++) {
      const int j = t * kTile + i * kThreads + tid;
      if (t * kTile + i * kThreads >= len) break;
      const bool is_src = j >= now && j < len && (keep >> i & 1);
      const uint64_t src = __ballot(is_src);
      const int at_src = from0 + table[1][i * kWaves + wave] + lower(src);
      if (is_src) from[at_src] = j;
      if (is_src && tiles == 1) {
        const int to = gap_at[at_src];
        w_out[to] = wt[i], pos_out[to] = ps[i];
      }
    }
    gap0 += all0, from0 += all1;
    __syncthreads();
  }
  if (tid == 0) g.count[blockIdx.x] = gap0;
  if (tiles > 1)
    for (int i = tid; i < (int)gap0; i += kThreads) {
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
    auto page = [&](int t) {
      const int id = table[t >> shift];
      const bool out = (uint32_t)id >= (uint32_t)c.n_blocks;
      bad |= out;
      return (int64_t)(out ? 0 : id);
    };
    const int64_t pt = page(to), pf = page(at);
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

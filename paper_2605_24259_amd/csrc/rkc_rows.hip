// rkc_rows.hip -- rows into a paged cache (norm, rotation, 4 bits) and back.
//
// store: y = x w / sqrt(mean(x^2) + eps) for each head of queries and keys, then pairs (a, b) -> (a cos t - b sin t,
// a sin t + b cos t) with t = frequency x position, in one pass over the rows.  What bounds it is the traffic, 2 bytes an
// element read and 2 (keys and values in 4 bits: 17/32) written: 13,400 rows of 48 heads of 128 elements 65 us over inputs that no
// cache has, 5.0 TB/s, 0.98 of a large copy's rate; 14,100 into 4 bits 72 us, 4.2 TB/s; and for a decode step's 64 rows a chain of loads,
// 4.8 and 5.6 us.
// A lane has 16 elements of a head: the two runs of 8 that turn into each other, so that a rotation needs no other lane.
// A workgroup has up to 16 rows, whose angles it finds once for all heads.
// read: the other way, a lane 8 elements of a head's key and value: 277,000 rows of 4 heads of 256 elements of 4 bits 283 us, 5.1 TB/s,
// a large copy's rate; 258,000 of 16 bits 407 us, 5.2 TB/s.
#include <type_traits>

#include "rkc_packed_dev.h"

namespace {

constexpr int kWaves = 4;
constexpr double kTurn = 6.283185307179586;                                          // 2 pi
constexpr double kTurnsHi = 0.15915494309189535, kTurnsLo = -9.839338337591243e-18;  // 1 / (2 pi) in two parts

// cos and sin of freq x position.  The product of 24 and 32 bits, the turns in it (with 1 / (2 pi) in two parts, so that what
// is left of a far position's angle keeps its bits) and the series over an eighth of a turn are in 64 bits, which this card
// multiplies as fast as 32: the error is a few units of 2^-53 of the angle's turn for any position.
__device__ __forceinline__ void cos_sin(int position, float freq, double& c, double& s) {
  const double p = (double)position * (double)freq, rest = __builtin_fma((double)position, (double)freq, -p);
  const double hi = p * kTurnsHi;
  const double lo = __builtin_fma(p, kTurnsHi, -hi) + __builtin_fma(p, kTurnsLo, rest * kTurnsHi);
  const double r = (hi - __builtin_rint(hi)) + lo, quarter = __builtin_rint(4.0 * r);
  const double x = __builtin_fma(-0.25, quarter, r) * kTurn, z = x * x;  // |x| <= pi / 4 and a little
  // Taylor's series; what is left out is below (pi / 4)^18 / 18!, 2e-18
  double a = 1.0, b = 1.0;
#pragma unroll
  for (int k = 8; k > 0; k--) {
    a = __builtin_fma(a * z, -1.0 / (2 * k * (2 * k + 1)), 1.0);  // sin x / x
    b = __builtin_fma(b * z, -1.0 / (2 * k * (2 * k - 1)), 1.0);  // cos x
  }
  a *= x;
  const int k = (int)quarter & 3;
  c = k & 1 ? a : b, s = k & 1 ? b : a;
  if (k == 1 || k == 2) c = -c;
  if (k >= 2) s = -s;
}

// The sequence of a row, by the whole wave: of 64 offsets at a time, how many are at most `row`.  Offsets out of order give
// some sequence that begins at the row or before it, whose end the caller checks.
__device__ __forceinline__ int seq_of(const int32_t* offset, int n_seqs, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = n_seqs;
  for (;;) {
    const int step = (n + 63) / 64;
    const bool in = lane * step < n;
    const uint64_t below = __ballot(in && offset[lo + (in ? lane * step : 0)] <= row);
    const int count = uni(~below ? __builtin_ctzll(~below) : 64);
    if (!count) return -1;
    lo += (count - 1) * step, n = min(step, n - (count - 1) * step);
    if (step == 1) return lo;
  }
}

// Where a row lies.  block < 0: the row is left alone, or (of a row to be stored) `known`: it has no block.
struct Place {
  int block, slot, in_page, known;
};

__device__ __forceinline__ void tell(int32_t* status, int s, int bit) {
  if (status && (threadIdx.x & 63) == 0) atomicOr(status + s, bit);
}

__device__ __forceinline__ bool out_of_limits(const rkc_rows& r, int r0, int r1, int len) {
  return r0 < 0 || r1 < r0 || r1 > r.n_rows || len < 0 || len > r.max_len || r1 - r0 > len;
}

// Sequences whose rows or length are out of their limits, by as many workgroups as they need: no row leads to one without rows, or
// whose offsets go back.  Last in the kernels, where it costs nothing (277,000 rows read 283 us; at their beginning 292).
template <typename C> __device__ __forceinline__ void tell_lengths(const C& c, const rkc_rows& r) {
  if (blockIdx.x > (uint32_t)(c.n_seqs - 1) / (64 * kWaves) || !c.d_status) return;
#pragma unroll 4
  for (int64_t s = blockIdx.x * 64 * kWaves + threadIdx.x; s < c.n_seqs; s += (int64_t)gridDim.x * 64 * kWaves)
    if (out_of_limits(r, r.d_row_offset[s], r.d_row_offset[s + 1], r.d_length[s])) atomicOr(c.d_status + s, RKC_CS_LENGTH);
}

template <typename C> __device__ __forceinline__ Place place_of(const C& c, const rkc_rows& r, int row, bool read) {
  Place p = {-1, 0, 0, 0};
  const int s = seq_of(r.d_row_offset, c.n_seqs, row);
  if (s < 0) return p;
  const int r0 = word(r.d_row_offset, s), r1 = word(r.d_row_offset, s + 1), len = word(r.d_length, s);
  if (row >= r1) return p;  // behind the last sequence
  if (out_of_limits(r, r0, r1, len)) return p;
  p.known = 1;
  p.slot = len - (r1 - row), p.in_page = p.slot & (c.page_tokens - 1);
  const int shift = 31 - __builtin_clz(c.page_tokens), id = word(c.d_block_table, (int64_t)s * c.max_pages + (p.slot >> shift));
  p.block = id;
  if ((uint32_t)id >= (uint32_t)c.n_blocks) {
    tell(c.d_status, s, RKC_CS_BLOCK);
    p.block = read ? 0 : -1;
  }
  return p;
}

// Of a head in a block, where it is.
struct Held {
  char* codes;   // keys' of the slot; values' are v_at further
  char* scales;  // keys' of the slot; values' are s_at further
  int v_at, s_at;
};
template <int D> __device__ __forceinline__ Held held_at(const rkc_packed& c, const Place& p, int h) {
  char* at = (char*)c.d_pool + (int64_t)p.block * c.block_stride + h * c.head_stride;
  const int n = code_bytes(c.page_tokens, D), m = scale_bytes(c.page_tokens, D);
  return {at + p.in_page * (D / 2), at + 2 * n + p.in_page * (D / 32), n, m};
}
template <typename T> __device__ __forceinline__ T* key_at(const rkc_cache& c, const Place& p, int h) {
  return (T*)c.d_k + p.block * c.k_block_stride + p.in_page * c.k_slot_stride + h * c.k_head_stride;
}
template <typename T> __device__ __forceinline__ T* value_at(const rkc_cache& c, const Place& p, int h) {
  return (T*)c.d_v + p.block * c.v_block_stride + p.in_page * c.v_slot_stride + h * c.v_head_stride;
}

template <int CTRL> __device__ __forceinline__ float swapped(float x) { return __uint_as_float(dpp<CTRL>(__float_as_uint(x))); }
template <int CTRL> __device__ __forceinline__ double swapped(double x) {
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint64_t y = (uint64_t)(uint32_t)dpp<CTRL>((int)(b >> 32)) << 32 | (uint32_t)dpp<CTRL>((int)b);
  return __builtin_bit_cast(double, y);
}
// Sum over L neighbouring lanes, in the same order in each.
template <int L, typename W> __device__ __forceinline__ W sum_of(W x) {
  x += swapped<0xb1>(x);                             // quad_perm [1,0,3,2]
  x += swapped<0x4e>(x);                             // quad_perm [2,3,0,1]
  if constexpr (L >= 8) x += swapped<0x141>(x);      // row_half_mirror
  if constexpr (L >= 16) x += swapped<0x140>(x);     // row_mirror
  return x;
}

// The largest over them.
template <int L> __device__ __forceinline__ float most_of(float x) {
  x = fmaxf(x, swapped<0xb1>(x));
  x = fmaxf(x, swapped<0x4e>(x));
  if constexpr (L >= 8) x = fmaxf(x, swapped<0x141>(x));
  if constexpr (L >= 16) x = fmaxf(x, swapped<0x140>(x));
  return x;
}

template <typename W> struct Pair { W c, s; };
template <typename T> struct Run { typename Vec8<T>::t a, b; };  // a lane's two runs of 8 elements

// 1 / sqrt(x): of the hardware, within a unit or two of the last place, in 32 bits, where the result is rounded to 16 behind it.
__device__ __forceinline__ float inverse_root(float x) { return __builtin_amdgcn_rsqf(x); }
__device__ __forceinline__ double inverse_root(double x) { return 1.0 / __builtin_sqrt(x); }
__device__ __forceinline__ float mad(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double mad(double a, double b, double c) { return __builtin_fma(a, b, c); }

// Norm and rotation of a lane's 16 elements.  W: 32 bits where the result is rounded to 16; 64 where it is rounded to 4,
// as an element next to a border between two codes goes by its last bits, and should be held alike wherever it is computed.
template <typename W, int L, int D, typename T>
__device__ __forceinline__ void norm_turn(const Run<T>& in, const float* w0, const float* w1, const rkc_rows& r, bool norm, bool turns, const Pair<W>* t, W (&y)[16]) {
#pragma unroll
  for (int k = 0; k < 8; k++) y[k] = (W)(float)in.a[k], y[8 + k] = (W)(float)in.b[k];
  if (norm) {
    W sum = 0;
#pragma unroll
    for (int k = 0; k < 16; k++) sum = mad(y[k], y[k], sum);
    W mean = sum_of<L>(sum) * (W)(1.0 / D) + (W)r.eps;
    if constexpr (std::is_same<W, float>::value && std::is_same<T, __bf16>::value) {
      // Squares past the range of 32 bits, or so far below one that bits are lost, which bfloat16 elements may have: the head, and eps
      // by the square, by the power of two that brings the largest element, or 2^-30 times the root of eps, to 1.
      if (__builtin_expect(!(mean >= 0x1p-100f && mean < kInf), 0)) {
        float most = 0.f;
#pragma unroll
        for (int k = 0; k < 16; k++) most = fmaxf(most, fabsf(y[k]));
        int e = __builtin_amdgcn_frexp_expf(most_of<L>(most));
        if (r.eps > 0.f) e = max(e, __builtin_amdgcn_frexp_expf(r.eps) / 2 - 30);
        sum = 0;
#pragma unroll
        for (int k = 0; k < 16; k++) y[k] = ldexpf(y[k], -e), sum = mad(y[k], y[k], sum);
        mean = sum_of<L>(sum) * (1.f / D) + ldexpf(r.eps, -2 * e);
      }
    }
    const W by = inverse_root(mean);
#pragma unroll
    for (int k = 0; k < 8; k++) y[k] = y[k] * by * (W)w0[k], y[8 + k] = y[8 + k] * by * (W)w1[k];
  }
  if (!turns) return;
  if (r.interleaved) {
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const W a = y[2 * k], b = y[2 * k + 1], c = t[k].c, s = t[k].s;
      y[2 * k] = mad(a, c, -(b * s)), y[2 * k + 1] = mad(a, s, b * c);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; k++) {
      const W a = y[k], b = y[8 + k], c = t[k].c, s = t[k].s;
      y[k] = mad(a, c, -(b * s)), y[8 + k] = mad(a, s, b * c);
    }
  }
}

template <typename T, typename W> __device__ __forceinline__ typename Vec8<T>::t rounded(const W* y) {
  f32x8 x;
#pragma unroll
  for (int k = 0; k < 8; k++) x[k] = (float)y[k];
  return __builtin_convertvector(x, typename Vec8<T>::t);
}

// A norm's weights into LDS, ones where there is none.
template <typename T, int D> __device__ __forceinline__ void weights(const rkc_rows& r, const void* norm, float* to) {
  for (int i = threadIdx.x; i < D; i += 64 * kWaves) to[i] = !norm ? 1.f : r.norm_f32 ? ((const float*)norm)[i] : (float)((const T*)norm)[i];
}

constexpr int rows_of(int D) { return D == 256 ? 8 : 16; }  // of a storing workgroup, at most
constexpr int kReadRows = 64, kReads = 2;                     // of a reading one; heads that a lane has on their way

template <typename T, int D, typename C>
__global__ __launch_bounds__(64 * kWaves, sizeof(C) == sizeof(rkc_packed) ? 3 : 4) void rows_store(const C c, const rkc_rows r, int per, int parts) {
  constexpr bool packed = sizeof(C) == sizeof(rkc_packed);
  typedef typename std::conditional<packed, double, float>::type W;  // of keys
  typedef typename Vec8<T>::t V8;
  constexpr int L = D / 16, N = 64 / L;  // lanes of a head, heads of a wave
  __shared__ __attribute__((aligned(16))) Pair<W> table[rows_of(D)][D / 2];
  __shared__ __attribute__((aligned(16))) float qw[D], kw[D];
  __shared__ Place place[rows_of(D)];
  __shared__ __attribute__((aligned(16))) float most[kWaves][N][D / 8];

  const int H = c.kv_heads, Q = r.d_q ? r.q_heads : 0;
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), l = lane % L, sub = lane / L;
  const int part = blockIdx.x % parts, row0 = blockIdx.x / parts * per, rows = min(per, r.n_rows - row0);
  // a lane's runs of 8 elements
  const int turning = r.n_freq / 8;
  const bool turns = l < turning;
  const int p0 = !turns ? 2 * l : r.interleaved ? 2 * l : l, p1 = !turns || r.interleaved ? 2 * l + 1 : turning + l;

  // of a wave at a time: N heads of queries, then of keys and values; those of the next time are on their way
  const int q_items = rows * Q, kv_items = rows * H, q_turns = (q_items + N - 1) / N, all = q_turns + (kv_items + N - 1) / N;
  const int step = parts * kWaves;
  struct Item {
    int i, h;
    bool in;
    Run<T> x, v;
  };
  auto fetch = [&](int turn) {
    Item t;
    const bool queries = turn < q_turns;
    const int item = (queries ? turn : turn - q_turns) * N + sub, n = queries ? q_items : kv_items, heads = queries ? Q : H;
    t.in = item < n, t.i = min(item, n - 1) / heads, t.h = min(item, n - 1) - t.i * heads;
    const T* from = queries ? (const T*)r.d_q + (row0 + t.i) * r.q_row_stride + t.h * r.q_head_stride
                            : (const T*)r.d_k + (row0 + t.i) * r.k_row_stride + t.h * r.k_head_stride;
    t.x = {*(const V8*)(from + 8 * p0), *(const V8*)(from + 8 * p1)};
    if (!queries) {
      const T* vf = (const T*)r.d_v + (row0 + t.i) * r.v_row_stride + t.h * r.v_head_stride;
      t.v = {*(const V8*)(vf + 16 * l), *(const V8*)(vf + 16 * l + 8)};
    }
    return t;
  };
  int turn = part * kWaves + wave;
  Item next;
  if (turn < all) next = fetch(turn);
  weights<T, D>(r, r.d_q_norm, qw), weights<T, D>(r, r.d_k_norm, kw);
  for (int i = wave; i < rows; i += kWaves) {
    const Place p = place_of(c, r, row0 + i, false);
    if (lane == 0) place[i] = p;
  }
  __syncthreads();
  for (int x = threadIdx.x; x < rows * r.n_freq; x += 64 * kWaves) {
    const int i = x / r.n_freq, j = x % r.n_freq;
    int at = place[i].slot;
    if (r.d_position) {
      const int axis = r.d_axis ? r.d_axis[j] : 0;
      at = r.d_position[(int64_t)((uint32_t)axis < (uint32_t)r.axes ? axis : 0) * r.n_rows + row0 + i];
    }
    double cs, sn;
    cos_sin(at, r.d_freq[j], cs, sn);
    table[i][j] = {(W)cs, (W)sn};
  }
  __syncthreads();

  for (; turn < all; turn += step) {
    const Item now = next;
    if (turn + step < all) next = fetch(turn + step);
    const Place p = place[now.i];
    const int i = now.i, h = now.h;
    if (turn < q_turns) {
      if (now.in && p.known) {
        Pair<float> t[8];
        if (turns) {
#pragma unroll
          for (int k = 0; k < 8; k++) t[k] = {(float)table[i][8 * l + k].c, (float)table[i][8 * l + k].s};
        }
        float y[16];
        norm_turn<float, L, D>(now.x, qw + 8 * p0, qw + 8 * p1, r, r.d_q_norm, turns, t, y);
        T* to = (T*)r.d_q_out + (row0 + i) * r.q_out_row_stride + h * r.q_out_head_stride;
        *(V8*)(to + 8 * p0) = rounded<T>(y), *(V8*)(to + 8 * p1) = rounded<T>(y + 8);
      }
      continue;
    }
    if (!now.in || p.block < 0) continue;  // the same for a head's lanes
    const Run<T> vin = now.v;
    W y[16];
    norm_turn<W, L, D>(now.x, kw + 8 * p0, kw + 8 * p1, r, r.d_k_norm, turns, &table[i][8 * l], y);
    if constexpr (!packed) {
      T* kt = key_at<T>(c, p, h);
      T* vt = value_at<T>(c, p, h);
      *(V8*)(kt + 8 * p0) = rounded<T>(y), *(V8*)(kt + 8 * p1) = rounded<T>(y + 8);
      *(V8*)(vt + 16 * l) = vin.a, *(V8*)(vt + 16 * l + 8) = vin.b;
    } else {
      float k0[8], k1[8], v0[8], v1[8], m0 = 0.f, m1 = 0.f, mv = 0.f;
      bool bad = false;
      auto finite = [&](float x) {
        const bool f = fabsf(x) < kInf;
        bad |= !f;
        return f ? x : 0.f;
      };
#pragma unroll
      for (int k = 0; k < 8; k++) {
        k0[k] = finite((float)y[k]), k1[k] = finite((float)y[8 + k]), v0[k] = finite((float)vin.a[k]), v1[k] = finite((float)vin.b[k]);
        m0 = fmaxf(m0, fabsf(k0[k])), m1 = fmaxf(m1, fabsf(k1[k])), mv = fmaxf(mv, fmaxf(fabsf(v0[k]), fabsf(v1[k])));
      }
      const bool mark = __ballot(bad) >> (lane - l) & ((1ull << L) - 1);
      // the largest of 32 keys: of the four runs of 8 in their block, which may be those of any lanes of the head
      most[wave][sub][p0] = m0, most[wave][sub][p1] = m1;
      __builtin_amdgcn_wave_barrier();
      const f32x4 a = *(const f32x4*)&most[wave][sub][p0 & ~3], b = *(const f32x4*)&most[wave][sub][p1 & ~3];
      __builtin_amdgcn_wave_barrier();
      const int e0 = scale_of<T>(fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]))), e1 = scale_of<T>(fmaxf(fmaxf(b[0], b[1]), fmaxf(b[2], b[3])));
      const int ev = scale_of<T>(fmaxf(mv, swapped<0xb1>(mv)));
      const Held to = held_at<D>(c, p, h);
      *(uint32_t*)(to.codes + 4 * p0) = pack8(k0, scale_float(e0));
      *(uint32_t*)(to.codes + 4 * p1) = pack8(k1, scale_float(e1));
      const uint32_t c0 = pack8(v0, scale_float(ev)), c1 = pack8(v1, scale_float(ev));
      *(uint64_t*)(to.codes + to.v_at + 8 * l) = (uint64_t)c1 << 32 | c0;
      if ((p0 & 3) == 0) to.scales[p0 >> 2] = (char)(mark && p0 == 0 ? kMark : e0);
      if ((p1 & 3) == 0) to.scales[p1 >> 2] = (char)e1;
      if ((l & 1) == 0) to.scales[to.s_at + (l >> 1)] = (char)ev;
    }
  }
  tell_lengths(c, r);
}

template <typename T, int D, typename C>
__global__ __launch_bounds__(64 * kWaves) void rows_read(const C c, const rkc_rows r, int per, int parts) {
  constexpr bool packed = sizeof(C) == sizeof(rkc_packed);
  constexpr int E = 8, L = D / E, N = 64 / L, U = kReads;  // elements of a lane, lanes of a head, heads of a wave, heads on their way
  __shared__ Place place[kReadRows];
  const int H = c.kv_heads, lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), l = lane % L, sub = lane / L;
  const int part = blockIdx.x % parts, row0 = blockIdx.x / parts * per, rows = min(per, r.n_rows - row0);
  for (int i = wave; i < rows; i += kWaves) {
    const Place p = place_of(c, r, row0 + i, true);
    if (lane == 0) place[i] = p;
  }
  __syncthreads();
  // a head's key and value of a row by L lanes, N of them at a time
  const int items = rows * H, step = parts * kWaves * N;
  for (int first = (part * kWaves + wave) * N + sub; first < items; first += U * step) {
    u32x4 x[U][2];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int item = min(first + u * step, items - 1), i = item / H, h = item - i * H;
      const Place p = place[i];
      if (p.block < 0) continue;
      if constexpr (packed) {
        const Held from = held_at<D>(c, p, h);
        const uint32_t k = *(const uint32_t*)(from.codes + E / 2 * l), v = *(const uint32_t*)(from.codes + from.v_at + E / 2 * l);
        const uint32_t ks = *(const uint8_t*)(from.scales + E * l / 32), vs = *(const uint8_t*)(from.scales + from.s_at + E * l / 32);
        const bool mark = *(const uint8_t*)from.scales == kMark;
        x[u][0] = unpack8<T>(k, scale_float(mark ? kMark : ks)), x[u][1] = unpack8<T>(v, scale_float(mark ? kMark : vs));
      } else {
        x[u][0] = *(const u32x4*)(key_at<T>(c, p, h) + 8 * l), x[u][1] = *(const u32x4*)(value_at<T>(c, p, h) + 8 * l);
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int item = first + u * step;
      if (item >= items) break;
      const int i = item / H, h = item - i * H;
      if (place[i].block < 0) continue;
      *(u32x4*)((T*)r.d_k + (row0 + i) * r.k_row_stride + h * r.k_head_stride + 8 * l) = x[u][0];
      *(u32x4*)((T*)r.d_v + (row0 + i) * r.v_row_stride + h * r.v_head_stride + 8 * l) = x[u][1];
    }
  }
  tell_lengths(c, r);
}

bool off16(const void* p) { return (uintptr_t)p & 15; }
bool off4(const void* p) { return (uintptr_t)p & 3; }
constexpr int64_t kFar = (int64_t)1 << 40;

// What both ways check; `cap`: slots of a sequence's pages.
rkc_status rows_check(const rkc_rows* r, int n_seqs, int64_t cap, int heads, int dim, bool read) {
  if (!r) return RKC_E_NULL;
  if (r->n_rows < 0 || r->max_len < 0 || r->max_len > RKC_MAX_CACHE_LEN || r->max_len > cap) return RKC_E_RANGE;
  for (int64_t x : {r->k_row_stride, r->k_head_stride, r->v_row_stride, r->v_head_stride})
    if (x < 0 || x % 8 || x > kFar) return RKC_E_RANGE;
  if (!read) {
    if (r->q_heads < 0 || r->q_heads > 1 << 16) return RKC_E_RANGE;
    if (r->n_freq < 0 || r->n_freq % 8 || r->n_freq > dim / 2) return RKC_E_RANGE;
    if ((r->interleaved | r->norm_f32) & ~1) return RKC_E_RANGE;
    if (!(r->eps >= 0.f) || r->eps == kInf) return RKC_E_RANGE;
    if (r->d_position && (r->axes < 1 || r->axes > RKC_MAX_AXES || (r->axes > 1 && !r->d_axis))) return RKC_E_RANGE;
    if (r->d_axis && !r->d_position) return RKC_E_RANGE;
    for (int64_t x : {r->q_row_stride, r->q_head_stride, r->q_out_row_stride, r->q_out_head_stride})
      if (x < 0 || x % 8 || x > kFar) return RKC_E_RANGE;
  }
  if (n_seqs == 0 || r->n_rows == 0) return RKC_OK;
  if (!r->d_row_offset || !r->d_length || !r->d_k || !r->d_v) return RKC_E_NULL;
  if (off16(r->d_k) || off16(r->d_v) || off4(r->d_row_offset) || off4(r->d_length)) return RKC_E_ALIGN;
  if (read) {
    if (rkc_shared(dim, r->n_rows, r->k_row_stride, heads, r->k_head_stride) || rkc_shared(dim, r->n_rows, r->v_row_stride, heads, r->v_head_stride))
      return RKC_E_RANGE;
    return RKC_OK;
  }
  if ((r->d_q && r->q_heads && !r->d_q_out) || (r->n_freq && !r->d_freq)) return RKC_E_NULL;
  for (const void* p : {(const void*)r->d_position, (const void*)r->d_axis, (const void*)r->d_freq})
    if (off4(p)) return RKC_E_ALIGN;
  for (const void* p : {r->d_q_norm, r->d_k_norm})
    if ((uintptr_t)p & (r->norm_f32 ? 3 : 1)) return RKC_E_ALIGN;
  if (r->d_q) {
    if (off16(r->d_q) || off16(r->d_q_out)) return RKC_E_ALIGN;
    if (rkc_shared(dim, r->n_rows, r->q_out_row_stride, r->q_heads, r->q_out_head_stride)) return RKC_E_RANGE;
    if (r->d_q == r->d_q_out && (r->q_row_stride != r->q_out_row_stride || r->q_head_stride != r->q_out_head_stride)) return RKC_E_RANGE;
  }
  return RKC_OK;
}

// Rows of a workgroup, and workgroups that share them: as many rows, up to `most`, as give its waves four turns and leave four
// workgroups a CU, and a few rows' heads over as many workgroups.  (13,400 rows of 48 heads of 128 elements stored over
// and over, their inputs in the last cache in part, 4 rows a workgroup: 60.7 us; 2 rows 72, 8 rows 63.6, 16 rows 71.)
// Reading, a workgroup has the rows whose heads its lanes take at once, twice: fewer rows are all start, and more keep their
// loads waiting for the stores before them (277,000 rows of 4 heads of 256 elements, 4 rows: 281 us; 2 rows 369, 8 rows 292,
// 64 rows 325; 157,000 of 8 heads of 64, 8 rows: 104; 4 rows 126, 16 rows 109).
struct Cut {
  int per, parts;
  int64_t workgroups;
};
Cut cut_of(int rows, int most, int64_t turns_of_a_row) {
  Cut k = {1, 1, 0};
  while (2 * k.per <= most && rows / (2 * k.per) >= 1024 && k.per * turns_of_a_row < 4 * kWaves) k.per *= 2;
  const int64_t waves = (turns_of_a_row + kWaves - 1) / kWaves;
  if (k.per == 1) k.parts = (int)(1024 / rows < 1 ? 1 : 1024 / rows < waves ? 1024 / rows : waves);
  k.workgroups = ((int64_t)rows + k.per - 1) / k.per * k.parts;
  return k;
}

template <typename T, int D, typename C> rkc_status go(const C* c, const rkc_rows* r, bool read, hipStream_t s) {
  const int Q = r->d_q ? r->q_heads : 0, H = c->kv_heads, n = 1024 / D, m = 512 / D, at_once = kReads * kWaves * m / H;
  const Cut k = read ? cut_of(r->n_rows, at_once < kReadRows ? at_once : kReadRows, (H + m - 1) / m)
                     : cut_of(r->n_rows, rows_of(D), (Q + n - 1) / n + (H + n - 1) / n);
  if (!rkc_fits(k.workgroups, 64 * kWaves)) return RKC_E_UNSUPPORTED;
  const dim3 grid((unsigned)k.workgroups), block(64 * kWaves);
  if (read) rows_read<T, D, C><<<grid, block, 0, s>>>(*c, *r, k.per, k.parts);
  else rows_store<T, D, C><<<grid, block, 0, s>>>(*c, *r, k.per, k.parts);
  return hipGetLastError() == hipSuccess ? RKC_OK : RKC_E_HIP;
}
template <typename T, typename C> rkc_status go(const C* c, const rkc_rows* r, bool read, hipStream_t s) {
  return c->head_dim == 64 ? go<T, 64>(c, r, read, s) : c->head_dim == 128 ? go<T, 128>(c, r, read, s) : go<T, 256>(c, r, read, s);
}
template <typename C> rkc_status rows(const C* c, const rkc_rows* r, bool read, void* s) {
  if (rkc_status st = rows_check(r, c->n_seqs, (int64_t)c->max_pages * c->page_tokens, c->kv_heads, c->head_dim, read)) return st;
  if (c->n_seqs == 0 || r->n_rows == 0) return RKC_OK;
  return c->dtype == RKC_BF16 ? go<__bf16>(c, r, read, (hipStream_t)s) : go<_Float16>(c, r, read, (hipStream_t)s);
}

}  // namespace

rkc_status rkc_packed_check(const rkc_packed* c) {
  if (!c) return RKC_E_NULL;
  if (c->n_seqs < 0 || c->n_blocks < 0 || c->max_pages < 0 || c->reserved) return RKC_E_RANGE;
  if (c->kv_heads < 1 || c->kv_heads > 1024 || c->n_seqs > 1 << 20) return RKC_E_RANGE;
  if (c->dtype != RKC_BF16 && c->dtype != RKC_F16) return RKC_E_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return RKC_E_UNSUPPORTED;
  if (c->page_tokens < 16 || c->page_tokens > 1024 || (c->page_tokens & (c->page_tokens - 1))) return RKC_E_UNSUPPORTED;
  if (c->block_stride < 0 || c->block_stride % 16 || c->block_stride >= (int64_t)1 << 32) return RKC_E_RANGE;
  if (c->head_stride < 0 || c->head_stride % 16 || c->head_stride > kFar) return RKC_E_RANGE;
  if (c->n_seqs == 0) return RKC_OK;
  if (!c->d_pool || !c->d_block_table) return RKC_E_NULL;
  if (off16(c->d_pool) || off4(c->d_block_table) || off4(c->d_status)) return RKC_E_ALIGN;
  if (c->n_blocks < 1 || c->max_pages < 1) return RKC_E_RANGE;
  return RKC_OK;
}

rkc_cache rkc_packed_as_cache(const rkc_packed* c) {
  rkc_cache x = {};
  x.n_seqs = c->n_seqs, x.n_blocks = c->n_blocks, x.max_pages = c->max_pages, x.page_tokens = c->page_tokens;
  x.kv_heads = c->kv_heads, x.head_dim = c->head_dim, x.dtype = c->dtype;
  x.d_block_table = c->d_block_table, x.d_status = c->d_status;
  x.d_k = x.d_v = c->d_pool;
  x.k_block_stride = c->block_stride, x.k_head_stride = c->head_stride;
  return x;
}

extern "C" {

rkc_status rkc_store(const rkc_cache* c, const rkc_rows* r, void* s) {
  if (rkc_status st = rkc_cache_check(c)) return st;
  // slots that share memory would be written by several rows
  if (c->n_seqs && (rkc_shared(c->head_dim, c->n_blocks, c->k_block_stride, c->page_tokens, c->k_slot_stride, c->kv_heads, c->k_head_stride) ||
                    rkc_shared(c->head_dim, c->n_blocks, c->v_block_stride, c->page_tokens, c->v_slot_stride, c->kv_heads, c->v_head_stride)))
    return RKC_E_RANGE;
  return rows(c, r, false, s);
}

rkc_status rkc_read(const rkc_cache* c, const rkc_rows* r, void* s) {
  if (rkc_status st = rkc_cache_check(c)) return st;
  return rows(c, r, true, s);
}

rkc_status rkc_packed_store(const rkc_packed* c, const rkc_rows* r, void* s) {
  if (rkc_status st = rkc_packed_check(c)) return st;
  if (c->n_seqs && rkc_shared((int64_t)c->page_tokens * (c->head_dim + c->head_dim / 16), c->n_blocks, c->block_stride, c->kv_heads, c->head_stride)) return RKC_E_RANGE;
  return rows(c, r, false, s);
}

rkc_status rkc_packed_read(const rkc_packed* c, const rkc_rows* r, void* s) {
  if (rkc_status st = rkc_packed_check(c)) return st;
  return rows(c, r, true, s);
}

}  // extern "C"

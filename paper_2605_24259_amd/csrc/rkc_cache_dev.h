// rkc_cache_dev.h -- what the kernels on a paged KV cache share: matrix instructions over both types, the
// layout of a tile in LDS, and what a row of a query sees.
//
// All of them compute scores transposed, S^T = K Q^T, so that a query row is a lane's column: its softmax
// statistics are one register per lane, a rescale of the output is one multiplication per register, and the
// probabilities come out of the first product in the layout in which the second one, O^T = V^T P^T, reads them.
// The sum over slots may take the slots in any order as long as V^T has the same: V goes through LDS and is
// read by transposing loads in that order.
#ifndef RKC_CACHE_DEV_H
#define RKC_CACHE_DEV_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rkc_cache.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kInf = __builtin_inff();

template <typename T> struct Vec8;
template <> struct Vec8<__bf16> { typedef bf16x8 t; };
template <> struct Vec8<_Float16> { typedef f16x8 t; };

__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return mma16(a, b, c); }
__device__ __forceinline__ f32x4 mma(f16x8 a, f16x8 b, f32x4 c) { return mma16(a, b, c); }
__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) { return mma32(a, b, c); }
__device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) { return mma32(a, b, c); }

// exp2 and log2 of the hardware (within one unit of the last place; below the smallest normal result: 0)
__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float lg2(float x) { return __builtin_amdgcn_logf(x); }

// Of lanes l and l ^ 16 (l ^ 32): both values, in an order that all lanes agree on up to a swap.
__device__ __forceinline__ void pair16(float x, float& a, float& b) {
  auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
}
__device__ __forceinline__ void pair32(float x, float& a, float& b) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]), b = __uint_as_float(r[1]);
}
__device__ __forceinline__ float max16(float x) { float a, b; pair16(x, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float max32(float x) { float a, b; pair32(x, a, b); return fmaxf(a, b); }
__device__ __forceinline__ float sum16(float x) { float a, b; pair16(x, a, b); return a + b; }
__device__ __forceinline__ float sum32(float x) { float a, b; pair32(x, a, b); return a + b; }

__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
// Minimum and maximum over the wave, by row permutations and swaps of rows.
template <int CTRL> __device__ __forceinline__ int dpp(int x) { return __builtin_amdgcn_mov_dpp(x, CTRL, 0xf, 0xf, true); }
template <typename Op> __device__ __forceinline__ int wave_all(int x, Op op) {
  x = op(x, dpp<0xb1>(x));   // quad_perm [1,0,3,2]
  x = op(x, dpp<0x4e>(x));   // quad_perm [2,3,0,1]
  x = op(x, dpp<0x141>(x));  // row_half_mirror
  x = op(x, dpp<0x140>(x));  // row_mirror
  auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = op((int)r[0], (int)r[1]);
  r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return uni(op((int)r[0], (int)r[1]));
}
__device__ __forceinline__ int wave_min(int x) { return wave_all(x, [](int a, int b) { return min(a, b); }); }
__device__ __forceinline__ int wave_max(int x) { return wave_all(x, [](int a, int b) { return max(a, b); }); }

// A tile of slots in LDS: rows of D elements in 16-byte chunks, the chunk's number xored with a number of
// the row so that neither a column of chunks over 16 rows (keys) nor 32 bytes of 4, 8 or 16 neighbouring rows
// (transposing reads of values) share banks.  Element offset of chunk `c` of row `r`.
// (The number is linear in the row's bits: of a sum of rows without a carry it is the exclusive or of theirs.)
template <int D> __device__ __forceinline__ constexpr int tile_x(int r) { return D == 64 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3); }
template <int D> __device__ __forceinline__ constexpr int tile_at(int r, int c) { return r * D + ((c ^ tile_x<D>(r)) << 3); }

// The same for products of 16 rows.  Keys, four chunks of 16 rows at a time: the number is the row's own.  Values, 32 bytes
// of 16 rows at a time: pairs of chunks stay together.
template <int D> __device__ __forceinline__ constexpr int keys16_at(int r, int c) { return r * D + ((c ^ (D == 64 ? r >> 1 & 7 : r & 15)) << 3); }
template <int D> __device__ __forceinline__ constexpr int vals16_x(int r) { return D == 64 ? (r >> 1 & 3) << 1 : (r & 7) << 1; }
template <int D> __device__ __forceinline__ constexpr int vals16_at(int r, int c) { return r * D + ((c ^ vals16_x<D>(r)) << 3); }

// Keeps the compiler from moving what follows from x out of a loop, where every element of a tile would cost a register.
__device__ __forceinline__ int here(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The same for a pointer in scalar registers, so that a load takes it from there with the lane's 32-bit offset.
__device__ __forceinline__ const char* fixed(const char* p) {
  asm volatile("" : "+s"(p));
  return p;
}

// 16 bytes a lane from memory into LDS, past the registers: lane l's go to `to` + 16 l.  The loads of a wave are done
// when its vector memory count says so (dma_barrier); what other waves loaded, behind the next barrier.
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void glb_void;
__device__ __forceinline__ void dma(const char* from, void* to) {
  __builtin_amdgcn_global_load_lds((glb_void*)from, (lds_void*)to, 16, 0, 0);
}
// Waits for this wave's loads but the last N, and its LDS accesses, then for the workgroup.
template <int N> __device__ __forceinline__ void dma_barrier() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// 4 slots x 16 columns, transposed within each 16 lanes: lane i gets column i of the 4 slots whose addresses
// lanes 4 s .. 4 s + 3 give (8 bytes each).
__device__ __forceinline__ s16x4 read_tr(const void* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p);
}

template <typename T> __device__ __forceinline__ typename Vec8<T>::t read_tr2(const void* a, const void* b) {
  const s16x4 x = read_tr(a), y = read_tr(b);
  const s16x8 z = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(typename Vec8<T>::t, z);
}

// Values that are not finite must not reach the rows that do not see their slot, where a product would meet them
// with a weight of zero.  Tiles that have such values and are not seen whole (`hurt`) are multiplied with them
// replaced by zeros, and once more with a code in their place against "seen" in place of the weights; the counts
// in that sum say what the rows get.
template <typename T> struct Bits;
template <> struct Bits<__bf16> { static constexpr uint16_t e = 0x7f80; };  // the exponent's bits
template <> struct Bits<_Float16> { static constexpr uint16_t e = 0x7c00; };

// Weights are exp2(score - top), and top lies this far below the row's maximum when it is set: with 16-bit floats of 5
// bits of exponent, the many small weights of a long row would else fall among the numbers without a leading one and
// lose bits there.  Up to 2^8 more is let stand until the maximum moves, 2^14 in all.
template <typename T> constexpr float kRoom = 0.f;
template <> inline constexpr float kRoom<_Float16> = 6.f;

template <typename T> __device__ __forceinline__ bool any_hurt(u32x4 x) {
  bool bad = false;
  constexpr uint32_t m = Bits<T>::e;
#pragma unroll
  for (int k = 0; k < 4; k++) bad |= (x[k] & m) == m || (x[k] & m << 16) == m << 16;
  return bad;
}

// Zeroes what is not finite in v; returns 1 for each NaN, 128 for each infinity, 16384 for each negative one.
template <typename T> __device__ __forceinline__ typename Vec8<T>::t strip(typename Vec8<T>::t& v) {
  s16x8 b = __builtin_bit_cast(s16x8, v);
  typename Vec8<T>::t code;
#pragma unroll
  for (int k = 0; k < 8; k++) {
    const uint16_t w = (uint16_t)b[k];
    const bool bad = (w & Bits<T>::e) == Bits<T>::e;
    code[k] = (T)(!bad ? 0.f : (w & 0x7fff) != Bits<T>::e ? 1.f : w >> 15 ? 16384.f : 128.f);
    if (bad) b[k] = 0;
  }
  v = __builtin_bit_cast(typename Vec8<T>::t, b);
  return code;
}

// What a sum of codes over at most 64 slots adds to an output.
__device__ __forceinline__ float hurt_by(float codes) {
  const int n = (int)codes;
  float x = n & 127 ? __builtin_nanf("") : 0.f;
  if (n >> 7 & 127) x += kInf;
  if (n >> 14) x -= kInf;
  return x;
}

// A word that no kernel of the call writes, at an address that is the same for the wave: loaded as a scalar, also behind
// barriers, where the compiler must otherwise expect it to have changed.
template <typename T> __device__ __forceinline__ T word(const T* p, int64_t i) {
  return ((const __attribute__((address_space(4))) T*)p)[i];
}

// ------------------------------------------------------------------------------------------------------------
// What a row sees.  Slots [start, end) and [0, prefix), and of a tree's drafted slots those of `line`.
struct Row {
  int start, end, prefix;
  int pos;  // position that distances are counted from
};

struct Seq {
  int row0, n, len, base;  // base: the slot of the first row
  bool ok;
};

// Reads and checks a sequence's row range and length.
__device__ __forceinline__ Seq load_seq(const rkc_cache& c, const rkc_attention& a, int s) {
  Seq q;
  const int r0 = word(a.d_row_offset, s), r1 = word(a.d_row_offset, s + 1);
  q.row0 = r0, q.n = r1 - r0, q.len = word(a.d_length, s), q.base = q.len - q.n;
  q.ok = r0 >= 0 && r1 >= r0 && r1 <= a.n_rows && q.n <= a.max_rows && q.len >= 0 && q.len <= a.max_len && q.n <= q.len;
  return q;
}

__device__ __forceinline__ void flag(const rkc_cache& c, int s, int bit) {
  if (c.d_status) atomicOr(c.d_status + s, bit);
}

__device__ __forceinline__ Row load_row(const rkc_attention& a, const Seq& q, int s, int i) {
  Row r;
  r.start = a.d_row_start ? max(0, a.d_row_start[q.row0 + i]) : 0;
  if (a.d_parent) r.start = min(r.start, q.base);  // drafted slots are seen by `line` alone, also behind a later start
  r.end = a.d_parent ? q.base : q.base + i + 1;
  r.prefix = a.d_prefix ? max(0, min(word(a.d_prefix, s), a.d_parent ? q.base : q.len)) : 0;
  r.pos = q.base + i;
  return r;
}

// The sequence of rank r by length, the longest first, of at most 64: found by each wave for itself.
__device__ __forceinline__ int seq_of_rank(const rkc_cache& c, const rkc_attention& a, int r) {
  const int lane = threadIdx.x & 63, len = lane < c.n_seqs ? a.d_length[lane] : (int)0x80000000;
  int rank = 0;
  for (int k = 0; k < c.n_seqs; k++) {
    const int other = __builtin_amdgcn_readlane(len, k);
    rank += other > len || (other == len && k < lane);
  }
  return uni(__builtin_ctzll(__ballot(lane < c.n_seqs && rank == r)));
}

// Lines of a tree of at most RKC_MAX_TREE_ROWS rows, by a workgroup of as many threads or more: every row joins the line
// of the row that its own line ends at, until all end at a root.  On return depths holds the rows' depths.
__device__ __forceinline__ void tree_lines(const rkc_cache& c, const rkc_attention& a, const Seq& q, int s, bool tell, uint64_t (*lines)[4], int* depths) {
  const int tid = threadIdx.x;
  uint64_t w[4] = {};
  int up = -1;
  if (tid < q.n) {
    up = a.d_parent[q.row0 + tid];
    if (up < -1 || up >= tid) {
      if (tell) flag(c, s, RKC_CS_PARENT);
      up = -1;
    }
#pragma unroll
    for (int k = 0; k < 4; k++) w[k] = tid >> 6 == k ? 1ull << (tid & 63) : 0;
  }
  for (int reach = 1;; reach *= 2) {
    if (tid < RKC_MAX_TREE_ROWS) {
#pragma unroll
      for (int k = 0; k < 4; k++) lines[tid][k] = w[k];
      depths[tid] = up;
    }
    __syncthreads();
    if (reach >= q.n) break;
    if (up >= 0) {
#pragma unroll
      for (int k = 0; k < 4; k++) w[k] |= lines[up][k];
      up = depths[up];
    }
    __syncthreads();
  }
  if (tid < RKC_MAX_TREE_ROWS) depths[tid] = __popcll(w[0]) + __popcll(w[1]) + __popcll(w[2]) + __popcll(w[3]) - 1;
  __syncthreads();
}

// Bits of `line` (bit d: drafted row d) for the 32 slots from t0 on.
__device__ __forceinline__ uint32_t line_window(const uint64_t* line, int words, int from) {
  if (from <= -32 || from >= 64 * words) return 0;
  if (from < 0) return (uint32_t)(line[0] << -from);
  const int w = from >> 6, sh = from & 63;
  uint64_t x = line[w] >> sh;
  if (sh > 32 && w + 1 < words) x |= line[w + 1] << (64 - sh);
  return (uint32_t)x;
}

// The end of the slots that the tile's rows up to `last` see.
__device__ __forceinline__ int rows_end(const rkc_attention& a, const Seq& q, int s, int last) {
  if (a.d_parent) return q.len;
  const int pre = a.d_prefix ? max(0, min(word(a.d_prefix, s), q.len)) : 0;
  return max(pre, q.base + last + 1);
}

// Bits of 32 slots from number `lo` of them on.
__device__ __forceinline__ uint32_t bits_from(int lo) { return (uint32_t)(0xffffffffull << max(0, min(lo, 32))); }

// Which of the 32 slots from j0 on a row sees, `line` being what it sees of drafted ones.
__device__ __forceinline__ uint32_t seen_of(const Row& r, int j0, uint32_t line) {
  return (bits_from(r.start - j0) & ~bits_from(r.end - j0)) | ~bits_from(r.prefix - j0) | line;
}

// x where bit k of m is set, else -inf: two instructions.
__device__ __forceinline__ float masked(float x, uint32_t m, int k) {
  const uint32_t all = (uint32_t)((int32_t)(m << (31 - k)) >> 31);
  return __uint_as_float((__float_as_uint(x) & all) | (0xff800000u & ~all));
}

// Memory of slot t's 16 neighbours: base + page x block + (t in its page) x slot, all in bytes; uniform.
struct Pool {
  const char* base;
  uint32_t block, slot;
};
__device__ __forceinline__ Pool k_pool(const rkc_cache& c, int h) {
  return {(const char*)c.d_k + 2 * h * c.k_head_stride, 2 * (uint32_t)c.k_block_stride, 2 * (uint32_t)c.k_slot_stride};
}
__device__ __forceinline__ Pool v_pool(const rkc_cache& c, int h) {
  return {(const char*)c.d_v + 2 * h * c.v_head_stride, 2 * (uint32_t)c.v_block_stride, 2 * (uint32_t)c.v_slot_stride};
}
__device__ __forceinline__ const char* run_at(const Pool& p, int page, int in_page) {
  return p.base + (uint64_t)(uint32_t)page * p.block + (uint32_t)in_page * p.slot;
}

// Block of the page that slot t, the same for the wave, lies in, as the table has it: to be looked up ahead of its use.
__device__ __forceinline__ int page_of(const int32_t* table, int shift, int t) { return word(table, t >> shift); }
// The block itself; 0 for an id outside the pool, which `bad` remembers.
__device__ __forceinline__ int block_of(const rkc_cache& c, int id, bool& bad) {
  const bool out = (uint32_t)id >= (uint32_t)c.n_blocks;
  bad |= out;
  return out ? 0 : id;
}

// The factors of a score: x = raw, or capped; then x - slope * distance; weights are exp2(x * post - maximum).
// The scale, or the cap, stays out of the scores until the exponent takes it up; a negative scale goes into the
// queries' signs, so that the maximum of the scores is that of the products.
struct Scale {
  float pre, post;
  bool negate, far;
};

__device__ __forceinline__ float uni_float(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

__device__ __forceinline__ Scale load_scale(const rkc_attention& a) {
  Scale s;
  s.negate = a.scale < 0.f;
  const float by = fabsf(a.scale);
  s.pre = uni_float(a.softcap > 0.f ? by / a.softcap * (2.f * kLog2e) : 1.f);
  s.far = a.softcap > 256.f;
  s.post = uni_float(fmaxf((a.softcap > 0.f ? a.softcap : by) * kLog2e, 1e-30f));  // above 0: what is masked stays -inf
  return s;
}

// tanh(y) of a lane's scores, x * pre = 2 y log2(e), by 1 - 2 / (exp(2 y) + 1).  That is off by 2^-23 of the cap, which
// of a cap past 256 would be too much of a small score: there, a score with |y| up to 0.8 takes a polynomial in y^2 of least
// relative error on that range (6e-8; 3e-7 with the roundings of 32 bits), whatever the scores beside it are: those are
// other rows', or of slots that nothing sees.  (For all caps it is the slower form: 2,048 rows over 32,768 slots 1,430 us
// instead of 1,320.)
__device__ __forceinline__ float cap_by_exp(float y2) { return 1.f - 2.f * __builtin_amdgcn_rcpf(ex2(y2) + 1.f); }
__device__ __forceinline__ float cap_small(float z) {
  const float t = z * z;
  float y = __builtin_fmaf(t, -0.00435528671f, 0.0190932825f);
  y = __builtin_fmaf(y, t, -0.0531143062f);
  y = __builtin_fmaf(y, t, 0.13321048f);
  y = __builtin_fmaf(y, t, -0.333326757f);
  return z * __builtin_fmaf(y, t, 0.99999994f);
}
template <typename V, int N> __device__ __forceinline__ void cap_all(V (&x)[N], const Scale& s) {
  constexpr int A = sizeof(V) / 4;
  constexpr float kSmall = 1.6f * kLog2e, kHalf = 0.5f * kLn2;
  auto each = [&](auto cap) {
#pragma unroll
    for (int u = 0; u < N; u++)
#pragma unroll
      for (int k = 0; k < A; k++) x[u][k] = cap(x[u][k]);
  };
  if (!s.far) {
    each([&](float y) { return cap_by_exp(y * s.pre); });
    return;
  }
  float most = 0.f;
  each([&](float y) { return most = fmaxf(most, fabsf(y)), y; });
  if (__any(most * s.pre > kSmall)) {
    // a small one's result is below kSmall, so that what is not small yet is told from it: few registers at a time
    each([&](float y) { return y * s.pre; });
    each([&](float y) { return fabsf(y) <= kSmall ? cap_small(y * kHalf) : y; });
    each([&](float y) { return fabsf(y) <= kSmall ? y : cap_by_exp(y); });
  } else {
    each([&](float y) { return cap_small(y * (s.pre * kHalf)); });
  }
}

template <typename V> __device__ __forceinline__ V negated(V v) {
  u32x4 b = __builtin_bit_cast(u32x4, v);
  return __builtin_bit_cast(V, b ^ 0x80008000u);
}

}  // namespace

// Host side: what every call checks.
rkc_status rkc_cache_check(const rkc_cache* c);
// Whether rows of `width` elements that lie apart by three strides, of so many each, share elements: what is written
// must not.
bool rkc_shared(int64_t width, int64_t n0, int64_t stride0, int64_t n1, int64_t stride1, int64_t n2 = 1, int64_t stride2 = 0);
rkc_status rkc_attention_check(const rkc_cache* c, const rkc_attention* a, bool weigh);
// Whether so many workgroups can be launched: the runtime counts a launch's lanes in 32 bits.  Asked of every launch of a
// call before the first one.
inline bool rkc_fits(int64_t workgroups, int lanes) { return workgroups <= 0x7fffffff && workgroups * lanes <= 0xffffffffll; }
bool rkc_weigh_fits(const rkc_cache* c, const rkc_attention* a);

// Entry of the two attention kernels: one for up to 16 packed rows (rows x query heads of a key/value head) of a
// sequence, one for tiles of 128 or 256; chunk: slots per workgroup, splits: workgroups along a sequence.
struct rkc_plan {
  bool few;
  int units;   // sequences x key/value heads x row tiles
  int tiles;   // row tiles per sequence and head
  int rows;    // packed rows of a tile
  int waves;   // of a workgroup, where few
  int chunk, splits;
  bool sorted;  // long sequences first
  size_t part_at, stat_at, bytes;  // scratch: partial outputs, their maxima and sums, in all
  bool keep;        // scores are kept for the account: [unit][32 slots][packed row][slot], in units of log2
  int wide;         // slots of a unit
  size_t score_at;
};
rkc_plan rkc_attend_plan(const rkc_cache* c, const rkc_attention* a);
// Lanes of a workgroup of the kernel that the plan takes.
inline int rkc_attend_lanes(const rkc_cache* c, const rkc_plan* p) { return 64 * (p->few ? p->waves : p->rows == 256 || c->head_dim == 256 ? 8 : 4); }
rkc_status rkc_attend_few(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s);
rkc_status rkc_attend_tile(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s);
// The join of a plan's parts, and whether it can be launched.
bool rkc_join_fits(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p);
rkc_status rkc_attend_join(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s);

#endif

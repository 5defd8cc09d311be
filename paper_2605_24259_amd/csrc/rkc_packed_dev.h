// rkc_packed_dev.h -- what the kernels on a cache of 4 bits share: where things lie, and the 4 bits themselves.
#ifndef RKC_PACKED_DEV_H
#define RKC_PACKED_DEV_H

#include "rkc_cache_dev.h"
#include "rkc_packed.h"

namespace {

// Bytes of a head's keys (or values) in a block, and of their scales.
__device__ __forceinline__ constexpr int code_bytes(int page, int D) { return page * D / 2; }
__device__ __forceinline__ constexpr int scale_bytes(int page, int D) { return page * D / 32; }

// The largest scale's byte: 6 times it is finite, 8 times it is not (bfloat16: 2^125; float16: 2^13).
template <typename T> constexpr int kTopScale = 252;
template <> inline constexpr int kTopScale<_Float16> = 140;
constexpr int kMark = 255;  // of a key's first scale: the head of this slot is not a number

// Byte of the least scale with which `most` is at most 7: a mantissa past 1.75 carries into the exponent.
template <typename T> __device__ __forceinline__ int scale_of(float most) {
  return max(1, min((int)((__float_as_uint(most) + 0x1fffffu) >> 23) - 2, kTopScale<T>));
}

// A scale as the conversions take it, which look at its exponent alone; 255 makes NaN of all.
__device__ __forceinline__ float scale_float(uint32_t b) { return __uint_as_float(b << 23); }

// Of a head of a cache of 4 bits as rkc_packed_as_cache has it: a block's keys' codes; values' codes and both scales lie behind.
struct Codes {
  const char* base;
  uint32_t block;
  int values, key_scales, value_scales;  // bytes from the keys' codes on
};
template <int D> __device__ __forceinline__ Codes codes_of(const rkc_cache& c, int h) {
  const int n = code_bytes(c.page_tokens, D);
  return {(const char*)c.d_k + h * c.k_head_stride, (uint32_t)c.k_block_stride, n, 2 * n, 2 * n + scale_bytes(c.page_tokens, D)};
}

// Memory at a lane's offset from a pointer in scalar registers, told to be global: a load of any memory would be waited for
// with those of LDS.
template <typename V> __device__ __forceinline__ V from_global(const char* p, uint32_t offset) {
  return *(const __attribute__((address_space(1))) V*)((const __attribute__((address_space(1))) char*)fixed(p) + (uint32_t)here((int)offset));
}

// Two codes of a byte as T, times the scale: exact, as a scaled code has two bits of mantissa; but for what float16 has no number for,
// odd multiples of 2^-25 and less, which are rounded to the nearest (halves to even): off by 2^-25 at most.
template <int BYTE> __device__ __forceinline__ uint32_t unpack2(__bf16, uint32_t codes, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, BYTE));
}
template <int BYTE> __device__ __forceinline__ uint32_t unpack2(_Float16, uint32_t codes, float s) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, BYTE));
}
template <typename T> __device__ __forceinline__ u32x4 unpack8(uint32_t codes, float s) {
  return u32x4{unpack2<0>(T(), codes, s), unpack2<1>(T(), codes, s), unpack2<2>(T(), codes, s), unpack2<3>(T(), codes, s)};
}

// Eight elements as codes: rounded to nearest, halves to even, past 7 scales held as 6.
__device__ __forceinline__ uint32_t pack8(const float (&x)[8], float s) {
  uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
}

}  // namespace

// Host side.
rkc_status rkc_packed_check(const rkc_packed* c);
// The cache as the attention's shared code takes it: its counts, table and status, the pool as the keys.
rkc_cache rkc_packed_as_cache(const rkc_packed* c);
rkc_plan rkc_packed_plan(const rkc_cache* c, const rkc_attention* a);
inline int rkc_packed_lanes(const rkc_cache* c, const rkc_plan* p) { return 64 * (p->few ? p->waves : p->rows == 256 ? 8 : 4); }
// Workgroups of the kernel of few rows: eight at a time for each row tile.
inline int64_t rkc_packed_few_workgroups(const rkc_plan* p) {
  const int64_t n = (int64_t)p->units / p->tiles * p->splits;
  return p->tiles == 1 ? n : (n + 7) / 8 * 8 * p->tiles;
}
rkc_status rkc_packed_few(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s);
rkc_status rkc_packed_tile(const rkc_cache* c, const rkc_attention* a, const rkc_plan* p, hipStream_t s);

#endif

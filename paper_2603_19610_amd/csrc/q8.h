// The 8-bit cache rows that several sources write or read (gfx950).
//
// A row x of D values is D e4m3 codes and one exponent byte e, and stands for
// code * 2^(e - 127).  e is the smallest number in [1, 254] with
// max |x_i| <= 448 * 2^(e - 127) over the finite x_i: a power of two, so the
// scaling is exact, the codes are one rounding of the row (half a step, 2^-4 of
// the value), and the conversion to bf16 takes a key row's power in by itself.
// A factor max / 448 instead would use the codes' range a little better, at no
// gain in a floating type's relative error, for 4 bytes a row.
#pragma once

#include "common.h"

namespace pvlm {

// One side (K or V) of a cache and both of it, padded (table == NULL:
// [B][Hkv][n_cap][D] codes, [B][Hkv][n_cap] exponents) or paged
// ([n_pages][Hkv][1 << shift][D] and [n_pages][Hkv][1 << shift]).
struct Q8Cache {
  uint8_t* kc;
  uint8_t* ke;
  uint8_t* vc;
  uint8_t* ve;
  const int32_t* table;  // [B][max_pages]
  int64_t n_pages, n_cap;
  int max_pages, shift;
};

// Row index (in rows of D codes) of logical row `row` of layer l, sequence b,
// KV head g; -1 where its page entry lies outside the pool.
__device__ __forceinline__ int64_t q8_row(const Q8Cache& c, int l, int B, int b, int Hkv, int g, int64_t row) {
  if (!c.table) return (((int64_t)l * B + b) * Hkv + g) * c.n_cap + row;
  const int pg = c.table[(int64_t)b * c.max_pages + (row >> c.shift)];
  if (pg < 0 || pg >= c.n_pages) return -1;
  return (((l * c.n_pages + pg) * Hkv + g) << c.shift) + (row & ((1 << c.shift) - 1));
}

// The exponent byte of a row whose largest finite magnitude is `top`:
// 448 = 1.75 * 2^8.  At most 247 (a finite top is below 2^128).
__device__ __forceinline__ int q8_exponent(float top) {
  const uint32_t u = __float_as_uint(top);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
  return e < 1 ? 1 : e;
}
// 2^(127 - e) and 2^(e - 127), e in [1, 253] and [1, 254]
__device__ __forceinline__ float q8_scale(int e) { return __uint_as_float((uint32_t)(254 - e) << 23); }
__device__ __forceinline__ float q8_unit(uint32_t e) { return __uint_as_float(e << 23); }

// |x| of a finite x, else 0
__device__ __forceinline__ float finite_abs(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? __uint_as_float(u) : 0.f;
}
// x, or NaN for an infinity: e4m3 has none, and a row that held one stays visible as such
__device__ __forceinline__ float inf_to_nan(float x) {
  return (__float_as_uint(x) & 0x7fffffffu) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : x;
}
// 0x80 in every byte of w that is a NaN code (0x7f or 0xff)
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// Four codes, nearest even (|x| <= 448, or NaN, which gives 0x7f whatever its sign).
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  return (uint32_t)w & ~nan_codes(w);
}

// What every call checks of a cache's pointers and capacity: 16-byte vectors of
// codes, 4-byte groups of exponents, and blocks of 32 rows that a read may
// take whole.
inline pvlm_status check_q8(const void* kc, const void* ke, const void* vc, const void* ve, int64_t n_cap) {
  if (!kc || !ke || !vc || !ve) return PVLM_ERR_NULL;
  if (n_cap < 32 || n_cap % 32 != 0 || n_cap > ((int64_t)1 << 30)) return PVLM_ERR_SHAPE;
  if (((uintptr_t)kc | (uintptr_t)vc) % 16 != 0 || ((uintptr_t)ke | (uintptr_t)ve) % 4 != 0)
    return PVLM_ERR_UNSUPPORTED;
  return PVLM_OK;
}
// A page pool's geometry as a cache's.
inline pvlm_status q8_pages(int page_size, int max_pages, int64_t n_pages, const int32_t* table, Q8Cache* c) {
  if (!table) return PVLM_ERR_NULL;
  const int shift = page_shift_of(page_size);
  if (shift < 0 || max_pages < 1 || n_pages < 1 || n_pages > INT32_MAX) return PVLM_ERR_SHAPE;
  c->table = table;
  c->n_pages = n_pages;
  c->max_pages = max_pages;
  c->shift = shift;
  c->n_cap = (int64_t)max_pages << shift;
  return PVLM_OK;
}

}  // namespace pvlm

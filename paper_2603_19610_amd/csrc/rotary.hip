// Rotary embedding of rows by position and the append of their keys and values by
// slot (gfx950), to a bf16 or fp32 cache and to a 4-bit one (ParallelVLM Sec. 2.2;
// Sec. 4.2, Parallel Decoding): pvlm_rope_append's operation for models that pair
// neighbouring elements, rotate part of a head or scale their frequencies, for
// rows of ragged sequences, and for rows that are slices of one projection's.
//
// Row n turns pair i of each q and k head by the angle p_n * f_i.  The frequencies
// are the host's (float64, at most 128, in the kernel's arguments), the angles
// reach 1e5 rad, and they, their sines and cosines and the rotation are float64,
// as pvlm_rope_append's are; a result is rounded to fp32 and then to its type.
//
// One workgroup a row (and, where there are few rows, a part of its heads): one
// wave takes the angles once for all heads, then D / 8 lanes take a head, eight
// values each.  A slot names a row of the cache whatever lays it out: padded,
// paged or ragged rows are one kernel, with one 64-bit division for a row.
//
// A prompt's rows are bound by memory: 12800 rows of 64 q and 2 x 8 K/V heads of 128,
// 524 MB, take 104 us to a bf16 cache (5.0 TB/s; a large copy 5.1) and 102 to a
// 4-bit one.  A step's few rows are bound by one launch and its chain of loads,
// angle and store: 6 rows of 28 + 2 x 4 heads 3.5 us, 16 rows to a 4-bit cache 3.9.
#include <cmath>

#include "q4.h"

namespace pvlm {
namespace {

constexpr int kMaxPairs = 128;

struct RotArgs {
  const void* q_in;
  const void* k_in;
  const void* v_in;
  const int32_t* pos;
  const int64_t* slots;
  void* q_out;
  void* k_cache;  // (codes of a 4-bit cache)
  void* v_cache;
  uint8_t* ke;
  uint8_t* ve;
  int32_t* status;
  int64_t N, q_stride, k_stride, v_stride, block, n_slots;
  double mscale;
  int Hq, Hkv, D, R, s0, s01, mrope, rows;  // rows: heads of a workgroup
  double freq[kMaxPairs];
};

// Four or eight consecutive values of a row to fp32, and four from it.
template <typename E, int N>
__device__ __forceinline__ void load_n(const void* p, size_t at, float* x) {
  if constexpr (sizeof(E) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + at + i);
      x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
  } else if constexpr (N == 8) {
    float y[8];
    bf16x8_to_f32(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at), y);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = y[i];
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + at);
    x[0] = __uint_as_float(u.x << 16), x[1] = __uint_as_float(u.x & 0xffff0000u);
    x[2] = __uint_as_float(u.y << 16), x[3] = __uint_as_float(u.y & 0xffff0000u);
  }
}
template <typename E>
__device__ __forceinline__ void store4(void* p, size_t at, const float* x) {
  if constexpr (sizeof(E) == 4)
    *reinterpret_cast<float4*>(static_cast<float*>(p) + at) = make_float4(x[0], x[1], x[2], x[3]);
  else
    *reinterpret_cast<uint64_t*>(static_cast<uint16_t*>(p) + at) = pack_bf16x4(x[0], x[1], x[2], x[3]);
}
// Eight values as they are, bit for bit.
template <typename E>
__device__ __forceinline__ void copy8(void* dst, size_t to, const void* src, size_t at) {
  constexpr int W = sizeof(E) / 2;
  const uint4* s = reinterpret_cast<const uint4*>(static_cast<const E*>(src) + at);
  uint4* d = reinterpret_cast<uint4*>(static_cast<E*>(dst) + to);
#pragma unroll
  for (int i = 0; i < W; ++i) d[i] = s[i];
}

// To fp32, by a rounding of its own: left to itself the compiler joins it with the one
// to bf16 that follows in some of the kernels and not in others, and the 4-bit rows
// would not be those of the bf16 cache.
__device__ __forceinline__ float to_f32(double x) {
  float f = static_cast<float>(x);
  asm("" : "+v"(f));
  return f;
}

// E: the rows' type (float, or uint16_t for bf16).  Q4: into a 4-bit cache (bf16 rows).  INTER: a pair is elements
// (2 i, 2 i + 1), else (i, i + R / 2).
template <typename E, bool Q4, bool INTER>
__global__ void __launch_bounds__(256) rotary_append_kernel(RotArgs a) {
  __shared__ double s_cos[kMaxPairs], s_sin[kMaxPairs];
  __shared__ __align__(16) float s_row[Q4 && !INTER ? 2048 : 4];
  const int64_t n = blockIdx.x;
  const int64_t slot = a.slots[n];
  if (slot < 0) return;  // a row of padding
  if (slot >= a.n_slots) {
    if (blockIdx.y == 0 && threadIdx.x == 0) dev_flag(a.status, PVLM_DEV_RANGE);
    return;
  }
  if (threadIdx.x < a.R / 2) {
    const int i = threadIdx.x;
    const int axis = a.mrope ? (i < a.s0 ? 0 : (i < a.s01 ? 1 : 2)) : 0;
    double s, c;
    sincos((double)a.pos[axis * a.N + n] * a.freq[i], &s, &c);
    s_cos[i] = c * a.mscale;
    s_sin[i] = s * a.mscale;
  }
  __syncthreads();
  const int LPR = a.D / 8, RPP = 256 / LPR;
  const int hl = threadIdx.x / LPR, u = threadIdx.x - hl * LPR;
  if (hl >= RPP) return;
  const int64_t blk = slot / a.block, r = slot - blk * a.block;
  const int heads = a.Hq + 2 * a.Hkv, h1 = min((int)(blockIdx.y + 1) * a.rows, heads);
  // where the lane's values of a head lie: 4 + 4 of a rotated half, or 8 in a row
  const bool turns = 8 * u < a.R;
  const int at0 = !INTER && turns ? 4 * u : 8 * u, at1 = !INTER && turns ? a.R / 2 + 4 * u : 8 * u + 4;
  for (int h = blockIdx.y * a.rows + hl; h < h1; h += RPP) {
    const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
    const int g = is_q ? h : is_k ? h - a.Hq : h - a.Hq - a.Hkv;
    const void* in = is_q ? a.q_in : is_k ? a.k_in : a.v_in;
    const size_t from = (size_t)(n * (is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride)) + (size_t)g * a.D;
    const int64_t row = (blk * a.Hkv + g) * a.block + r;  // of the cache
    if (!is_q && !is_k) {  // values are appended as they are
      if constexpr (Q4) {
        float x[8];
        int e;
        load_n<E, 8>(in, from + 8 * u, x);
        const uint32_t codes = q4_encode(x, e);
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.v_cache) + row * (a.D / 2) + 4 * u) = codes;
        if (u % 4 == 0) a.ve[row * (a.D / 32) + u / 4] = (uint8_t)e;
      } else {
        copy8<E>(a.v_cache, (size_t)row * a.D + 8 * u, in, from + 8 * u);
      }
      continue;
    }
    float x[8];
    if (turns) {
      load_n<E, 4>(in, from + at0, x);
      load_n<E, 4>(in, from + at1, x + 4);
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const double c = s_cos[4 * u + p], s = s_sin[4 * u + p];
        const int i = INTER ? 2 * p : p, j = INTER ? 2 * p + 1 : 4 + p;
        const double x1 = x[i], x2 = x[j];
        x[i] = to_f32(x1 * c - x2 * s);
        x[j] = to_f32(x2 * c + x1 * s);
      }
    } else if constexpr (Q4) {
      load_n<E, 8>(in, from + 8 * u, x);
    } else {
      copy8<E>(is_q ? a.q_out : a.k_cache, is_q ? ((size_t)n * a.Hq + g) * a.D + 8 * u : (size_t)row * a.D + 8 * u, in,
               from + 8 * u);
      continue;
    }
    if (is_q || !Q4) {
      void* out = is_q ? a.q_out : a.k_cache;
      const size_t to = is_q ? ((size_t)n * a.Hq + g) * a.D : (size_t)row * a.D;
      store4<E>(out, to + at0, x);
      store4<E>(out, to + at1, x + 4);
      continue;
    }
    if constexpr (Q4) {
      // a key is rounded to bf16 first: the codes are those of the row that a bf16 cache would hold
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = bf16_to_f32(f32_to_bf16(x[i]));
      if constexpr (!INTER) {  // to lanes of eight in a row; a head's lanes are one wave's
        float* mine = s_row + hl * a.D;
        *reinterpret_cast<float4*>(mine + at0) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(mine + at1) = make_float4(x[4], x[5], x[6], x[7]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const float4 lo = *reinterpret_cast<const float4*>(mine + 8 * u), hi = *reinterpret_cast<const float4*>(mine + 8 * u + 4);
        __builtin_amdgcn_wave_barrier();
        x[0] = lo.x, x[1] = lo.y, x[2] = lo.z, x[3] = lo.w;
        x[4] = hi.x, x[5] = hi.y, x[6] = hi.z, x[7] = hi.w;
      }
      int e;
      const uint32_t codes = q4_encode(x, e);
      *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(a.k_cache) + row * (a.D / 2) + 4 * u) = codes;
      if (u % 4 == 0) a.ke[row * (a.D / 32) + u / 4] = (uint8_t)e;
    }
  }
}

// ------------------------------------------------------------------ host --
bool positive(double x) { return std::isfinite(x) && x > 0.0; }

// The frequencies of R / 2 pairs; PVLM_ERR_SHAPE for parameters that have none.
pvlm_status frequencies(const pvlm_rotary& p, double* f) {
  const int R = p.rot_dim;
  if (R < 8 || R % 8 != 0 || R > 2 * kMaxPairs || !(p.base > 1.0 && p.base < 1e300) || !positive(p.mscale))
    return PVLM_ERR_SHAPE;
  const bool parts = p.scaling == PVLM_ROPE_PARTS || p.scaling == PVLM_ROPE_YARN;
  if (p.scaling != PVLM_ROPE_UNSCALED && p.scaling != PVLM_ROPE_LINEAR && !parts) return PVLM_ERR_SHAPE;
  if (p.scaling != PVLM_ROPE_UNSCALED && !positive(p.factor)) return PVLM_ERR_SHAPE;
  if (parts && !(positive(p.orig_ctx) && positive(p.alpha) && std::isfinite(p.beta) && p.beta > p.alpha))
    return PVLM_ERR_SHAPE;
  const double two_pi = 6.283185307179586476925, ln_base = std::log(p.base);
  double lo = 0.0, hi = 1.0;
  if (p.scaling == PVLM_ROPE_YARN) {
    lo = std::floor(R / 2 * std::log(p.orig_ctx / (two_pi * p.beta)) / ln_base);
    hi = std::ceil(R / 2 * std::log(p.orig_ctx / (two_pi * p.alpha)) / ln_base);
    if (lo < 0.0) lo = 0.0;
    if (hi > R - 1) hi = R - 1;
  }
  for (int i = 0; i < R / 2; ++i) {
    const double w = std::exp(-2.0 * i / R * ln_base);
    double keep = 1.0;  // how much of the frequency is not scaled
    if (p.scaling == PVLM_ROPE_LINEAR) keep = 0.0;
    if (p.scaling == PVLM_ROPE_PARTS) keep = (p.orig_ctx * w / two_pi - p.alpha) / (p.beta - p.alpha);
    if (p.scaling == PVLM_ROPE_YARN) keep = 1.0 - (i - lo) / (hi - lo > 0.001 ? hi - lo : 0.001);
    keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
    f[i] = p.scaling == PVLM_ROPE_UNSCALED ? w : w * keep + w / p.factor * (1.0 - keep);
  }
  return PVLM_OK;
}

pvlm_status rotary_run(pvlm_dtype dt, bool q4, int64_t N, int Hq, int Hkv, int D, const pvlm_rotary* rot,
                       const int32_t* pos, const void* q_in, int64_t q_stride, const void* k_in, int64_t k_stride,
                       const void* v_in, int64_t v_stride, const int64_t* slots, int64_t n_blocks, int64_t block,
                       void* q_out, void* k, uint8_t* ke, void* v, uint8_t* ve, int32_t* status, hipStream_t stream) {
  if (!rot || !pos || !q_in || !k_in || !v_in || !slots || !q_out || !k || !v || (q4 && (!ke || !ve)))
    return PVLM_ERR_NULL;
  if (q4 ? dt != PVLM_BF16 || (D != 64 && D != 128) : dt != PVLM_BF16 && dt != PVLM_F32) return PVLM_ERR_UNSUPPORTED;
  if (N < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || D < 8 || D % 8 != 0 || D > 2 * kMaxPairs) return PVLM_ERR_SHAPE;
  // one workgroup of 256 a row, in a launch of fewer than 2^32 work-items
  if (N > (((int64_t)1 << 32) - 256) / 256 || (int64_t)Hq + 2 * (int64_t)Hkv > 65536) return PVLM_ERR_SHAPE;
  if (block < 1 || block > ((int64_t)1 << 30) || n_blocks < 1 || n_blocks > INT32_MAX) return PVLM_ERR_SHAPE;
  const int64_t most = (int64_t)1 << 40;
  if (q_stride < (int64_t)Hq * D || k_stride < (int64_t)Hkv * D || v_stride < (int64_t)Hkv * D || q_stride > most ||
      k_stride > most || v_stride > most)
    return PVLM_ERR_SHAPE;
  if (rot->layout != PVLM_ROPE_HALF && rot->layout != PVLM_ROPE_INTERLEAVED) return PVLM_ERR_SHAPE;
  if (rot->rot_dim > D) return PVLM_ERR_SHAPE;
  RotArgs a;
  const pvlm_status st = frequencies(*rot, a.freq);
  if (st != PVLM_OK) return st;
  const int32_t* s = rot->sections;
  a.mrope = s[0] != 0 || s[1] != 0 || s[2] != 0;
  if (a.mrope && (s[0] < 0 || s[1] < 0 || s[2] < 0 || (int64_t)s[0] + s[1] + s[2] != rot->rot_dim / 2))
    return PVLM_ERR_SHAPE;
  if ((q_stride | k_stride | v_stride) % 8 != 0) return PVLM_ERR_UNSUPPORTED;
  if (((uintptr_t)q_in | (uintptr_t)k_in | (uintptr_t)v_in | (uintptr_t)q_out | (uintptr_t)k | (uintptr_t)v) % 16 != 0 ||
      (q4 && ((uintptr_t)ke | (uintptr_t)ve) % 4 != 0) || (uintptr_t)slots % 8 != 0)
    return PVLM_ERR_UNSUPPORTED;
  a.s0 = s[0];
  a.s01 = s[0] + s[1];
  a.q_in = q_in;
  a.k_in = k_in;
  a.v_in = v_in;
  a.pos = pos;
  a.slots = slots;
  a.q_out = q_out;
  a.k_cache = k;
  a.v_cache = v;
  a.ke = ke;
  a.ve = ve;
  a.status = status;
  a.N = N;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.block = block;
  a.n_slots = n_blocks * block;
  a.mscale = rot->mscale;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.D = D;
  a.R = rot->rot_dim;
  // A workgroup takes a pass of its lanes over the heads, or all heads where the
  // device is full without (it has the angles once then).
  const int heads = Hq + 2 * Hkv, pass = 256 / (D / 8), passes = (heads + pass - 1) / pass;
  const bool split = N * passes <= 1024;
  a.rows = split ? pass : heads;
  const bool inter = rot->layout == PVLM_ROPE_INTERLEAVED;
  const auto kernel =
      q4 ? (inter ? rotary_append_kernel<uint16_t, true, true> : rotary_append_kernel<uint16_t, true, false>)
      : dt == PVLM_BF16
          ? (inter ? rotary_append_kernel<uint16_t, false, true> : rotary_append_kernel<uint16_t, false, false>)
          : (inter ? rotary_append_kernel<float, false, true> : rotary_append_kernel<float, false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)N, split ? passes : 1), dim3(256), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

}  // namespace
}  // namespace pvlm

using namespace pvlm;

extern "C" pvlm_status pvlm_rotary_freqs(const pvlm_rotary* rot, double* freqs) {
  if (!rot || !freqs) return PVLM_ERR_NULL;
  return frequencies(*rot, freqs);
}

extern "C" pvlm_status pvlm_rotary_append(pvlm_dtype dt, int64_t N, int Hq, int Hkv, int D, const pvlm_rotary* rot,
                                          const int32_t* pos, const void* q_in, int64_t q_stride, const void* k_in,
                                          int64_t k_stride, const void* v_in, int64_t v_stride, const int64_t* slots,
                                          int64_t n_blocks, int64_t block_rows, void* q_out, void* k_cache,
                                          void* v_cache, int32_t* status, hipStream_t stream) {
  return rotary_run(dt, false, N, Hq, Hkv, D, rot, pos, q_in, q_stride, k_in, k_stride, v_in, v_stride, slots, n_blocks,
                    block_rows, q_out, k_cache, nullptr, v_cache, nullptr, status, stream);
}

extern "C" pvlm_status pvlm_rotary_append_q4(pvlm_dtype dt, int64_t N, int Hq, int Hkv, int D, const pvlm_rotary* rot,
                                             const int32_t* pos, const void* q_in, int64_t q_stride, const void* k_in,
                                             int64_t k_stride, const void* v_in, int64_t v_stride,
                                             const int64_t* slots, int64_t n_blocks, int64_t block_rows, void* q_out,
                                             uint8_t* k_codes, uint8_t* k_exps, uint8_t* v_codes, uint8_t* v_exps,
                                             int32_t* status, hipStream_t stream) {
  return rotary_run(dt, true, N, Hq, Hkv, D, rot, pos, q_in, q_stride, k_in, k_stride, v_in, v_stride, slots, n_blocks,
                    block_rows, q_out, k_codes, k_exps, v_codes, v_exps, status, stream);
}

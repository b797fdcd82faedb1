// Writing a 4-bit KV cache from a prefill's and reading it back as the draft's
// compact cache [V*, X] (gfx950; ParallelVLM Sec. 4.2, Stage I).  The row format is
// that of q4.h; rows are appended in rotary.hip.
//
// Both are streams, bound by memory: every row is read once and written once.
// Quantise: a lane has eight values, four lanes a block, whose maximum stays in the
// vector unit (28 layers of 4 heads and 6432 bf16 rows, 467 MB: 84 us, 5.5 TB/s; a
// large copy on the same card 5.1).  Gather: a lane reads eight codes and writes a
// whole 16 bytes of bf16 (28 layers of 787 rows, 57 MB: 14 us, 4.1 TB/s, where the
// start and the end of a launch are 3 us).
#include "q4.h"

namespace pvlm {
namespace {

// -------------------------------------------------------------- quantise --
struct QuantArgs {
  const void* k;
  const void* v;
  const int32_t* len;
  int32_t* status;
  Q4Cache c;
  int64_t src_cap;
  int B, Hkv;
};

template <typename E>
__device__ __forceinline__ void load8(const void* p, size_t at, float (&x)[8]) {
  if constexpr (sizeof(E) == 2) {
    bf16x8_to_f32(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at), x);
  } else {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 u = f[0], w = f[1];
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
    x[4] = w.x, x[5] = w.y, x[6] = w.z, x[7] = w.w;
  }
}

// grid: x = row blocks, y = KV head, z = layer * B + sequence.
template <typename E, int D>
__global__ void __launch_bounds__(256) quantize_q4_kernel(QuantArgs a) {
  constexpr int LPR = D / 8, RPP = 256 / LPR;
  const int lb = blockIdx.z, l = lb / a.B, b = lb - l * a.B, g = blockIdx.y;
  const int64_t r = (int64_t)blockIdx.x * RPP + threadIdx.x / LPR;
  const int j = threadIdx.x % LPR;
  const int64_t most = a.src_cap < a.c.n_cap ? a.src_cap : a.c.n_cap;
  int64_t n = a.len[b];
  if (n < 0 || n > most) {
    if (lb == b && g == 0 && blockIdx.x == 0 && threadIdx.x == 0) dev_flag(a.status, PVLM_DEV_RANGE);
    n = n < 0 ? 0 : most;
  }
  if (r >= n) return;
  const int64_t row = q4_row(a.c, l, a.B, b, a.Hkv, g, r);
  if (row < 0) {
    if (j == 0) dev_flag(a.status, PVLM_DEV_RANGE);
    return;
  }
  const size_t at = (((size_t)lb * a.Hkv + g) * a.src_cap + r) * D + 8 * j;
  float xk[8], xv[8];
  load8<E>(a.k, at, xk);
  load8<E>(a.v, at, xv);
  int ek, ev;
  const uint32_t ck = q4_encode(xk, ek), cv = q4_encode(xv, ev);
  *reinterpret_cast<uint32_t*>(a.c.kc + row * (D / 2) + 4 * j) = ck;
  *reinterpret_cast<uint32_t*>(a.c.vc + row * (D / 2) + 4 * j) = cv;
  if (j % 4 == 0) {
    a.c.ke[row * (D / 32) + j / 4] = (uint8_t)ek;
    a.c.ve[row * (D / 32) + j / 4] = (uint8_t)ev;
  }
}

// ---------------------------------------------------------------- gather --
struct GatherArgs {
  Q4Cache c;
  const int32_t* idx;
  const int32_t* kk;
  const int32_t* tail_begin;
  const int32_t* tail_len;
  void* kd;
  void* vd;
  uint8_t* kde;
  uint8_t* vde;
  int32_t* status;
  int64_t dst_cap;
  int B, Hkv, k_cap, fill;
};

enum { kCopy = 0, kToBf16 = 1, kToF32 = 2 };

// A lane's eight codes into the destination row at element `at`.
template <int TO>
__device__ __forceinline__ void put8(void* dst, size_t at, uint32_t codes, uint32_t e) {
  if constexpr (TO == kCopy) {
    *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(dst) + at / 2) = codes;
  } else {
    const float unit = __uint_as_float(e << 23);
    if constexpr (TO == kToBf16) {
      uint4 o;
      o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 0));
      o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 1));
      o.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 2));
      o.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, 3));
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(dst) + at) = o;
    } else {
      const auto p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0);
      const auto q = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1);
      const auto r = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2);
      const auto s = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
      float4* o = reinterpret_cast<float4*>(static_cast<float*>(dst) + at);
      o[0] = make_float4(p[0], p[1], q[0], q[1]);
      o[1] = make_float4(r[0], r[1], s[0], s[1]);
    }
  }
}

// grid: x = destination row blocks, y = KV head, z = layer * B + sequence.
template <int TO, int D>
__global__ void __launch_bounds__(256) gather_q4_kernel(GatherArgs a) {
  constexpr int LPR = D / 8, RPP = 256 / LPR;
  const int lb = blockIdx.z, l = lb / a.B, b = lb - l * a.B, g = blockIdx.y;
  const int64_t r = (int64_t)blockIdx.x * RPP + threadIdx.x / LPR;
  const int j = threadIdx.x % LPR;
  int64_t kb = a.kk[b], tb = a.tail_begin[b], tl = a.tail_len[b];
  const int64_t k_most = a.k_cap < a.dst_cap ? a.k_cap : a.dst_cap;
  const int64_t kb0 = kb, tb0 = tb, tl0 = tl;
  kb = kb < 0 ? 0 : kb > k_most ? k_most : kb;
  tb = tb < 0 ? 0 : tb > a.c.n_cap ? a.c.n_cap : tb;
  const int64_t t_most = a.c.n_cap - tb < a.dst_cap - kb ? a.c.n_cap - tb : a.dst_cap - kb;
  tl = tl < 0 ? 0 : tl > t_most ? t_most : tl;
  if ((kb != kb0 || tb != tb0 || tl != tl0) && blockIdx.x == 0 && g == 0 && lb == b && threadIdx.x == 0)
    dev_flag(a.status, PVLM_DEV_RANGE);
  if (r >= a.dst_cap) return;
  int64_t row = -1;
  if (r < kb + tl) {
    const int64_t src = r < kb ? a.idx[(int64_t)b * a.k_cap + r] : tb + (r - kb);
    if (src >= 0 && src < a.c.n_cap) row = q4_row(a.c, l, a.B, b, a.Hkv, g, src);
    if (row < 0 && j == 0) dev_flag(a.status, PVLM_DEV_RANGE);
  }
  if (row < 0 && !a.fill) return;
  uint32_t ck = 0, cv = 0;
  uint8_t ek = 0, ev = 0;
  if (row >= 0) {
    ck = *reinterpret_cast<const uint32_t*>(a.c.kc + row * (D / 2) + 4 * j);
    cv = *reinterpret_cast<const uint32_t*>(a.c.vc + row * (D / 2) + 4 * j);
    ek = a.c.ke[row * (D / 32) + j / 4];
    ev = a.c.ve[row * (D / 32) + j / 4];
  }
  const int64_t drow = ((int64_t)lb * a.Hkv + g) * a.dst_cap + r;
  put8<TO>(a.kd, (size_t)drow * D + 8 * j, ck, ek);
  put8<TO>(a.vd, (size_t)drow * D + 8 * j, cv, ev);
  if (TO == kCopy && j % 4 == 0) {
    a.kde[drow * (D / 32) + j / 4] = ek;
    a.vde[drow * (D / 32) + j / 4] = ev;
  }
}

// ------------------------------------------------------------------ host --
// Grid of a stacked call: rows of `rpp` a workgroup, KV heads, layers * B.
pvlm_status stacked_grid(int n_layers, int B, int Hkv, int64_t rows, int rpp, dim3* grid) {
  if (n_layers < 1 || B < 1 || Hkv < 1 || rows < 0 || rows > ((int64_t)1 << 30)) return PVLM_ERR_SHAPE;
  const int64_t x = (rows + rpp - 1) / rpp, z = (int64_t)n_layers * B;
  if (z > 65535 || Hkv > 65535 || x * 256 > ((int64_t)1 << 32) - 256) return PVLM_ERR_SHAPE;
  *grid = dim3((unsigned)x, (unsigned)Hkv, (unsigned)z);
  return PVLM_OK;
}

pvlm_status quantize_run(pvlm_dtype dt, int n_layers, int B, int Hkv, int D, int64_t src_cap, const void* k_src,
                         const void* v_src, const int32_t* len, const Q4Cache& c, int32_t* status,
                         hipStream_t stream) {
  if (!k_src || !v_src || !len) return PVLM_ERR_NULL;
  if ((dt != PVLM_BF16 && dt != PVLM_F32) || (D != 64 && D != 128)) return PVLM_ERR_UNSUPPORTED;
  if (src_cap < 1) return PVLM_ERR_SHAPE;
  pvlm_status st = check_q4(c.kc, c.ke, c.vc, c.ve, c.n_cap);
  if (st != PVLM_OK) return st;
  if (((uintptr_t)k_src | (uintptr_t)v_src) % 16 != 0) return PVLM_ERR_UNSUPPORTED;
  dim3 grid;
  st = stacked_grid(n_layers, B, Hkv, src_cap < c.n_cap ? src_cap : c.n_cap, 2048 / D, &grid);
  if (st != PVLM_OK) return st;
  if (src_cap > ((int64_t)1 << 30)) return PVLM_ERR_SHAPE;
  QuantArgs a{k_src, v_src, len, status, c, src_cap, B, Hkv};
  const auto kernel = dt == PVLM_BF16 ? (D == 128 ? quantize_q4_kernel<uint16_t, 128> : quantize_q4_kernel<uint16_t, 64>)
                                      : (D == 128 ? quantize_q4_kernel<float, 128> : quantize_q4_kernel<float, 64>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

pvlm_status gather_run(pvlm_dtype to, int n_layers, int B, int Hkv, int D, const Q4Cache& c, const int32_t* idx,
                       const int32_t* k, int32_t k_cap, const int32_t* tail_begin, const int32_t* tail_len,
                       int64_t dst_cap, int fill, void* k_dst, uint8_t* k_dst_exp, void* v_dst, uint8_t* v_dst_exp,
                       int32_t* status, hipStream_t stream) {
  if (!k || !tail_begin || !tail_len || !k_dst || !v_dst) return PVLM_ERR_NULL;
  if (k_cap > 0 && !idx) return PVLM_ERR_NULL;
  if ((to != PVLM_E2M1 && to != PVLM_BF16 && to != PVLM_F32) || (D != 64 && D != 128)) return PVLM_ERR_UNSUPPORTED;
  if (k_cap < 0) return PVLM_ERR_SHAPE;
  pvlm_status st = check_q4(c.kc, c.ke, c.vc, c.ve, c.n_cap);
  if (st != PVLM_OK) return st;
  if (to == PVLM_E2M1) {
    st = check_q4(k_dst, k_dst_exp, v_dst, v_dst_exp, dst_cap);
    if (st != PVLM_OK) return st;
  } else if (((uintptr_t)k_dst | (uintptr_t)v_dst) % 16 != 0) {
    return PVLM_ERR_UNSUPPORTED;
  }
  dim3 grid;
  st = stacked_grid(n_layers, B, Hkv, dst_cap, 2048 / D, &grid);
  if (st != PVLM_OK) return st;
  if (dst_cap == 0) return PVLM_OK;
  GatherArgs a{c, idx, k, tail_begin, tail_len, k_dst, v_dst, k_dst_exp, v_dst_exp, status, dst_cap, B, Hkv, k_cap, fill};
  const auto kernel = to == PVLM_E2M1   ? (D == 128 ? gather_q4_kernel<kCopy, 128> : gather_q4_kernel<kCopy, 64>)
                      : to == PVLM_BF16 ? (D == 128 ? gather_q4_kernel<kToBf16, 128> : gather_q4_kernel<kToBf16, 64>)
                                        : (D == 128 ? gather_q4_kernel<kToF32, 128> : gather_q4_kernel<kToF32, 64>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

Q4Cache padded(const uint8_t* kc, const uint8_t* ke, const uint8_t* vc, const uint8_t* ve, int64_t n_cap) {
  return Q4Cache{const_cast<uint8_t*>(kc), const_cast<uint8_t*>(ke), const_cast<uint8_t*>(vc),
                 const_cast<uint8_t*>(ve), nullptr, 0, n_cap, 0, 0};
}

}  // namespace
}  // namespace pvlm

using namespace pvlm;

extern "C" pvlm_status pvlm_quantize_kv_q4(pvlm_dtype dt, int n_layers, int B, int Hkv, int D, int64_t src_cap,
                                           const void* k_src, const void* v_src, const int32_t* len, int64_t n_cap,
                                           uint8_t* k_codes, uint8_t* k_exps, uint8_t* v_codes, uint8_t* v_exps,
                                           int32_t* status, hipStream_t stream) {
  return quantize_run(dt, n_layers, B, Hkv, D, src_cap, k_src, v_src, len,
                      padded(k_codes, k_exps, v_codes, v_exps, n_cap), status, stream);
}

extern "C" pvlm_status pvlm_quantize_kv_q4_paged(pvlm_dtype dt, int n_layers, int B, int Hkv, int D, int page_size,
                                                 int max_pages, int64_t n_pages, int64_t src_cap, const void* k_src,
                                                 const void* v_src, const int32_t* len, const int32_t* page_table,
                                                 uint8_t* k_codes, uint8_t* k_exps, uint8_t* v_codes, uint8_t* v_exps,
                                                 int32_t* status, hipStream_t stream) {
  Q4Cache c = padded(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  return quantize_run(dt, n_layers, B, Hkv, D, src_cap, k_src, v_src, len, c, status, stream);
}

extern "C" pvlm_status pvlm_gather_kv_q4(pvlm_dtype dst_dt, int n_layers, int B, int Hkv, int D, int64_t n_cap,
                                         const uint8_t* k_codes, const uint8_t* k_exps, const uint8_t* v_codes,
                                         const uint8_t* v_exps, const int32_t* idx, const int32_t* k, int32_t k_cap,
                                         const int32_t* tail_begin, const int32_t* tail_len, int64_t dst_cap, int fill,
                                         void* k_dst, uint8_t* k_dst_exps, void* v_dst, uint8_t* v_dst_exps,
                                         int32_t* status, hipStream_t stream) {
  return gather_run(dst_dt, n_layers, B, Hkv, D, padded(k_codes, k_exps, v_codes, v_exps, n_cap), idx, k, k_cap,
                    tail_begin, tail_len, dst_cap, fill, k_dst, k_dst_exps, v_dst, v_dst_exps, status, stream);
}

extern "C" pvlm_status pvlm_gather_kv_q4_paged(pvlm_dtype dst_dt, int n_layers, int B, int Hkv, int D, int page_size,
                                               int max_pages, int64_t n_pages, const uint8_t* k_codes,
                                               const uint8_t* k_exps, const uint8_t* v_codes, const uint8_t* v_exps,
                                               const int32_t* page_table, const int32_t* idx, const int32_t* k,
                                               int32_t k_cap, const int32_t* tail_begin, const int32_t* tail_len,
                                               int64_t dst_cap, int fill, void* k_dst, uint8_t* k_dst_exps, void* v_dst,
                                               uint8_t* v_dst_exps, int32_t* status, hipStream_t stream) {
  Q4Cache c = padded(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  return gather_run(dst_dt, n_layers, B, Hkv, D, c, idx, k, k_cap, tail_begin, tail_len, dst_cap, fill, k_dst, k_dst_exps,
                    v_dst, v_dst_exps, status, stream);
}

// Writing an 8-bit KV cache and reading it back (gfx950): the rotated append of
// new rows, the rows of a 16- or 32-bit cache, and the draft's compact cache
// [V*, X] of kept rows (ParallelVLM Sec. 2.2; Sec. 4.2, Parallel Decoding and
// Stage I).  The row format is that of q8.h.
//
// All three are streams: every row is read once and written once by a few
// neighbouring lanes (8 values each; 16 codes each in the gather), whose
// maximum is a reduction over at most 16 lanes that stays in the vector unit.  They
// are bound by HBM where there are rows enough, by a launch's latency else (one
// MI355X, kernel times):
//   append    80 heads of 12800 prompt rows, 0.5 GB: 97 us, 5.1 TB/s; 6 rows: 3.5 us
//   quantise  28 layers of 6432 rows, 4 heads, 0.55 GB: 95 us, 5.8 TB/s; from fp32,
//             0.92 GB: 163 us, 5.7 TB/s; one layer of 787 rows: 3 us
//   gather    80 layers, 1510 rows kept, to bf16, 0.74 GB: 148 to 164 us, 4.5 to
//             5.0 TB/s; to fp32, 1.24 GB: 396 us, 3.1 TB/s (stores of 8 and 16 bytes
//             a lane, 32 and 64 apart); 28 layers, 0.045 GB, copied: 10 us, 4.5 TB/s
#include "q8.h"

namespace pvlm {
namespace {

// Maximum over the LPR (8 or 16) neighbouring lanes of a row.
template <int LPR>
__device__ __forceinline__ float row_max(float x) {
  x = fmaxf(x, lane_xor1(x));
  x = fmaxf(x, lane_xor2(x));
  x = fmaxf(x, lane_mirror8(x));
  if constexpr (LPR == 16) x = fmaxf(x, lane_xor8(x));
  return x;
}

// Codes of a lane's 8 values of a row, and the row's exponent.
template <int LPR>
__device__ __forceinline__ uint2 encode(const float (&x)[8], int& e) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(x[i]));
  e = q8_exponent(row_max<LPR>(top));
  const float f = q8_scale(e);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = inf_to_nan(x[i]) * f;
  return make_uint2(e4m3x4(y[0], y[1], y[2], y[3]), e4m3x4(y[4], y[5], y[6], y[7]));
}

__device__ __forceinline__ void bf16x4(uint2 u, float* x) {
  x[0] = __uint_as_float(u.x << 16);
  x[1] = __uint_as_float(u.x & 0xffff0000u);
  x[2] = __uint_as_float(u.y << 16);
  x[3] = __uint_as_float(u.y & 0xffff0000u);
}

// ---------------------------------------------------------------- append --
struct AppendArgs {
  const uint16_t* q_in;
  const uint16_t* k_in;
  const uint16_t* v_in;
  const int32_t* pos;
  const int32_t* ctx_len;
  uint16_t* q_out;
  int32_t* status;
  Q8Cache c;
  double log2_base;
  int B, T, Hq, Hkv, s0, s01, mrope, rows;  // rows of one workgroup
};

// One workgroup per (b, t) and `rows` of its q, k and v rows.  The angles reach
// 1e5 rad, so they, their sines and cosines and the rotation are taken in
// float64, as pvlm_rope_append does; one wave takes them once for all rows.  A
// lane holds the pairs 4 j .. 4 j + 3 of a row.  A key is rounded to bf16
// before it is quantised: the codes are those of the row that a bf16 cache
// would hold.
template <int D>
__global__ void __launch_bounds__(256) append_q8_kernel(AppendArgs a) {
  constexpr int H = D / 2, LPR = D / 8, RPP = 256 / LPR;
  __shared__ double s_cos[H], s_sin[H];
  const int64_t bt = blockIdx.x;
  const int b = (int)(bt / a.T), t = (int)(bt - (int64_t)b * a.T);
  const int heads = a.Hq + 2 * a.Hkv;
  int ctx = a.ctx_len[b];
  if (ctx < 0 || (int64_t)ctx + a.T > a.c.n_cap) {
    if (t == 0 && blockIdx.y == 0 && threadIdx.x == 0) dev_flag(a.status, PVLM_DEV_RANGE);
    ctx = ctx < 0 ? 0 : (int)(a.c.n_cap - a.T);
  }
  if (threadIdx.x < H) {
    const int i = threadIdx.x;
    const int axis = a.mrope ? (i < a.s0 ? 0 : (i < a.s01 ? 1 : 2)) : 0;
    const double p = (double)a.pos[((int64_t)axis * a.B + b) * a.T + t];
    sincos(p * exp2(-2.0 * i / D * a.log2_base), &s_sin[i], &s_cos[i]);
  }
  __syncthreads();
  const int j = threadIdx.x % LPR;
  const int h1 = min((int)(blockIdx.y + 1) * a.rows, heads);
  for (int h = blockIdx.y * a.rows + threadIdx.x / LPR; h < h1; h += RPP) {
    const bool is_q = h < a.Hq, is_k = !is_q && h < a.Hq + a.Hkv;
    const int g = is_q ? h : is_k ? h - a.Hq : h - a.Hq - a.Hkv;
    const uint16_t* in = is_q ? a.q_in : is_k ? a.k_in : a.v_in;
    const size_t at = ((size_t)bt * (is_q ? a.Hq : a.Hkv) + g) * D + 4 * j;
    float x[8];
    bf16x4(*reinterpret_cast<const uint2*>(in + at), x);
    bf16x4(*reinterpret_cast<const uint2*>(in + at + H), x + 4);
    if (is_q || is_k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double cs = s_cos[4 * j + i], sn = s_sin[4 * j + i], x1 = x[i], x2 = x[4 + i];
        x[i] = bf16_to_f32(f32_to_bf16(static_cast<float>(x1 * cs - x2 * sn)));
        x[4 + i] = bf16_to_f32(f32_to_bf16(static_cast<float>(x2 * cs + x1 * sn)));
      }
    }
    if (is_q) {
      *reinterpret_cast<uint64_t*>(a.q_out + at) = pack_bf16x4(x[0], x[1], x[2], x[3]);
      *reinterpret_cast<uint64_t*>(a.q_out + at + H) = pack_bf16x4(x[4], x[5], x[6], x[7]);
      continue;
    }
    int e;
    const uint2 codes = encode<LPR>(x, e);
    const int64_t row = q8_row(a.c, 0, a.B, b, a.Hkv, g, (int64_t)ctx + t);
    if (row < 0) {
      if (j == 0) dev_flag(a.status, PVLM_DEV_RANGE);
      continue;
    }
    uint8_t* dst = (is_k ? a.c.kc : a.c.vc) + row * D + 4 * j;
    *reinterpret_cast<uint32_t*>(dst) = codes.x;
    *reinterpret_cast<uint32_t*>(dst + H) = codes.y;
    if (j == 0) (is_k ? a.c.ke : a.c.ve)[row] = (uint8_t)e;
  }
}

// -------------------------------------------------------------- quantise --
struct QuantArgs {
  const void* k;
  const void* v;
  const int32_t* len;
  int32_t* status;
  Q8Cache c;
  int64_t src_cap;
  int B, Hkv;
};

template <typename E>
__device__ __forceinline__ void load8(const void* p, size_t at, float (&x)[8]) {
  if constexpr (sizeof(E) == 2) {
    const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
    bf16x4(make_uint2(u.x, u.y), x);
    bf16x4(make_uint2(u.z, u.w), x + 4);
  } else {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    const float4 u = f[0], w = f[1];
    x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
    x[4] = w.x, x[5] = w.y, x[6] = w.z, x[7] = w.w;
  }
}

// grid: x = row blocks, y = KV head, z = layer * B + sequence.
template <typename E, int D>
__global__ void __launch_bounds__(256) quantize_kernel(QuantArgs a) {
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
  const int64_t row = q8_row(a.c, l, a.B, b, a.Hkv, g, r);
  if (row < 0) {
    if (j == 0) dev_flag(a.status, PVLM_DEV_RANGE);
    return;
  }
  const size_t at = (((size_t)lb * a.Hkv + g) * a.src_cap + r) * D + 8 * j;
  float xk[8], xv[8];
  load8<E>(a.k, at, xk);
  load8<E>(a.v, at, xv);
  int ek, ev;
  const uint2 ck = encode<LPR>(xk, ek), cv = encode<LPR>(xv, ev);
  *reinterpret_cast<uint2*>(a.c.kc + row * D + 8 * j) = ck;
  *reinterpret_cast<uint2*>(a.c.vc + row * D + 8 * j) = cv;
  if (j == 0) {
    a.c.ke[row] = (uint8_t)ek;
    a.c.ve[row] = (uint8_t)ev;
  }
}

// ---------------------------------------------------------------- gather --
struct GatherArgs {
  Q8Cache c;
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

// A lane's 16 codes into the destination row at element `at`.
template <int TO>
__device__ __forceinline__ void put16(void* dst, size_t at, uint4 codes, uint32_t e) {
  if constexpr (TO == kCopy) {
    *reinterpret_cast<uint4*>(static_cast<uint8_t*>(dst) + at) = codes;
  } else {
    const float unit = q8_unit(e);
    const uint32_t w[4] = {codes.x, codes.y, codes.z, codes.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
      if constexpr (TO == kToBf16)  // exact but for results under 2^-126
        *reinterpret_cast<uint64_t*>(static_cast<uint16_t*>(dst) + at + 4 * i) =
            pack_bf16x4(lo[0] * unit, lo[1] * unit, hi[0] * unit, hi[1] * unit);
      else
        *reinterpret_cast<float4*>(static_cast<float*>(dst) + at + 4 * i) =
            make_float4(lo[0] * unit, lo[1] * unit, hi[0] * unit, hi[1] * unit);
    }
  }
}

// grid: x = destination row blocks, y = KV head, z = layer * B + sequence.
template <int TO, int D>
__global__ void __launch_bounds__(256) gather_q8_kernel(GatherArgs a) {
  constexpr int LPR = D / 16, RPP = 256 / LPR;
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
    if (src >= 0 && src < a.c.n_cap) row = q8_row(a.c, l, a.B, b, a.Hkv, g, src);
    if (row < 0 && j == 0) dev_flag(a.status, PVLM_DEV_RANGE);
  }
  if (row < 0 && !a.fill) return;
  uint4 ck = make_uint4(0u, 0u, 0u, 0u), cv = ck;
  uint8_t ek = 0, ev = 0;
  if (row >= 0) {
    ck = *reinterpret_cast<const uint4*>(a.c.kc + row * D + 16 * j);
    cv = *reinterpret_cast<const uint4*>(a.c.vc + row * D + 16 * j);
    ek = a.c.ke[row];
    ev = a.c.ve[row];
  }
  const int64_t drow = ((int64_t)lb * a.Hkv + g) * a.dst_cap + r;
  put16<TO>(a.kd, (size_t)drow * D + 16 * j, ck, ek);
  put16<TO>(a.vd, (size_t)drow * D + 16 * j, cv, ev);
  if (TO == kCopy && j == 0) {
    a.kde[drow] = ek;
    a.vde[drow] = ev;
  }
}

// ------------------------------------------------------------------ host --
pvlm_status append_run(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, double base,
                       const int32_t* sections, const int32_t* pos, const void* q_in, const void* k_in,
                       const void* v_in, const int32_t* ctx_len, void* q_out, const Q8Cache& c,
                       int32_t* status, hipStream_t stream) {
  if (!pos || !q_in || !k_in || !v_in || !ctx_len || !q_out) return PVLM_ERR_NULL;
  if (dt != PVLM_BF16 || (D != 64 && D != 128)) return PVLM_ERR_UNSUPPORTED;
  if (B < 1 || T < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || c.n_cap < T || !(base > 1.0 && base < 1e300))
    return PVLM_ERR_SHAPE;
  const pvlm_status st = check_q8(c.kc, c.ke, c.vc, c.ve, c.n_cap);
  if (st != PVLM_OK) return st;
  if (((uintptr_t)q_in | (uintptr_t)k_in | (uintptr_t)v_in | (uintptr_t)q_out) % 8 != 0) return PVLM_ERR_UNSUPPORTED;
  const int64_t heads = (int64_t)Hq + 2 * (int64_t)Hkv, bt = (int64_t)B * T;
  // one launch of fewer than 2^32 work-items, one workgroup of 256 per (b, t) at least
  if (heads > 65536 || bt > (((int64_t)1 << 32) - 256) / 256) return PVLM_ERR_SHAPE;
  AppendArgs a;
  a.mrope = sections != nullptr;
  a.s0 = a.s01 = D / 2;
  if (sections) {
    if (sections[0] < 0 || sections[1] < 0 || sections[2] < 0 || sections[0] + sections[1] + sections[2] != D / 2)
      return PVLM_ERR_SHAPE;
    a.s0 = sections[0];
    a.s01 = sections[0] + sections[1];
  }
  a.q_in = static_cast<const uint16_t*>(q_in);
  a.k_in = static_cast<const uint16_t*>(k_in);
  a.v_in = static_cast<const uint16_t*>(v_in);
  a.pos = pos;
  a.ctx_len = ctx_len;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.status = status;
  a.c = c;
  a.log2_base = std::log2(base);
  a.B = B;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  // A workgroup takes a pass of 256 lanes over the heads, or all of them where the
  // device is full without (it has the angles once then).  6 rows of 28 + 8 heads:
  // 3.7 us split, 4.7 in one; a prompt's rows fill the device either way.
  const int pass = 2048 / D, passes = (int)((heads + pass - 1) / pass);
  const bool split = bt * passes <= 1024;
  a.rows = split ? pass : (int)heads;
  hipLaunchKernelGGL(D == 128 ? append_q8_kernel<128> : append_q8_kernel<64>, dim3((unsigned)bt, split ? passes : 1),
                     dim3(256), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

// Grid of a stacked call: rows of `rpp` a workgroup, KV heads, layers * B.
pvlm_status stacked_grid(int n_layers, int B, int Hkv, int64_t rows, int rpp, dim3* grid) {
  if (n_layers < 1 || B < 1 || Hkv < 1 || rows < 0 || rows > ((int64_t)1 << 30)) return PVLM_ERR_SHAPE;
  const int64_t x = (rows + rpp - 1) / rpp, z = (int64_t)n_layers * B;
  if (z > 65535 || Hkv > 65535 || x * 256 > ((int64_t)1 << 32) - 256) return PVLM_ERR_SHAPE;
  *grid = dim3((unsigned)x, (unsigned)Hkv, (unsigned)z);
  return PVLM_OK;
}

pvlm_status quantize_run(pvlm_dtype dt, int n_layers, int B, int Hkv, int D, int64_t src_cap, const void* k_src,
                         const void* v_src, const int32_t* len, const Q8Cache& c, int32_t* status,
                         hipStream_t stream) {
  if (!k_src || !v_src || !len) return PVLM_ERR_NULL;
  if ((dt != PVLM_BF16 && dt != PVLM_F32) || (D != 64 && D != 128)) return PVLM_ERR_UNSUPPORTED;
  if (src_cap < 1) return PVLM_ERR_SHAPE;
  pvlm_status st = check_q8(c.kc, c.ke, c.vc, c.ve, c.n_cap);
  if (st != PVLM_OK) return st;
  if (((uintptr_t)k_src | (uintptr_t)v_src) % 16 != 0) return PVLM_ERR_UNSUPPORTED;
  dim3 grid;
  st = stacked_grid(n_layers, B, Hkv, src_cap < c.n_cap ? src_cap : c.n_cap, 2048 / D, &grid);
  if (st != PVLM_OK) return st;
  if (src_cap > ((int64_t)1 << 30)) return PVLM_ERR_SHAPE;
  QuantArgs a{k_src, v_src, len, status, c, src_cap, B, Hkv};
  const auto kernel = dt == PVLM_BF16 ? (D == 128 ? quantize_kernel<uint16_t, 128> : quantize_kernel<uint16_t, 64>)
                                      : (D == 128 ? quantize_kernel<float, 128> : quantize_kernel<float, 64>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

pvlm_status gather_run(pvlm_dtype to, int n_layers, int B, int Hkv, int D, const Q8Cache& c, const int32_t* idx,
                       const int32_t* k, int32_t k_cap, const int32_t* tail_begin, const int32_t* tail_len,
                       int64_t dst_cap, int fill, void* k_dst, uint8_t* k_dst_exp, void* v_dst, uint8_t* v_dst_exp,
                       int32_t* status, hipStream_t stream) {
  if (!k || !tail_begin || !tail_len || !k_dst || !v_dst) return PVLM_ERR_NULL;
  if (k_cap > 0 && !idx) return PVLM_ERR_NULL;
  if ((to != PVLM_E4M3 && to != PVLM_BF16 && to != PVLM_F32) || (D != 64 && D != 128)) return PVLM_ERR_UNSUPPORTED;
  if (k_cap < 0) return PVLM_ERR_SHAPE;
  pvlm_status st = check_q8(c.kc, c.ke, c.vc, c.ve, c.n_cap);
  if (st != PVLM_OK) return st;
  if (to == PVLM_E4M3) {
    st = check_q8(k_dst, k_dst_exp, v_dst, v_dst_exp, dst_cap);
    if (st != PVLM_OK) return st;
  } else if (((uintptr_t)k_dst | (uintptr_t)v_dst) % 16 != 0) {
    return PVLM_ERR_UNSUPPORTED;
  }
  dim3 grid;
  st = stacked_grid(n_layers, B, Hkv, dst_cap, 4096 / D, &grid);
  if (st != PVLM_OK) return st;
  if (dst_cap == 0) return PVLM_OK;
  GatherArgs a{c, idx, k, tail_begin, tail_len, k_dst, v_dst, k_dst_exp, v_dst_exp, status, dst_cap, B, Hkv, k_cap, fill};
  const auto kernel = to == PVLM_E4M3   ? (D == 128 ? gather_q8_kernel<kCopy, 128> : gather_q8_kernel<kCopy, 64>)
                      : to == PVLM_BF16 ? (D == 128 ? gather_q8_kernel<kToBf16, 128> : gather_q8_kernel<kToBf16, 64>)
                                        : (D == 128 ? gather_q8_kernel<kToF32, 128> : gather_q8_kernel<kToF32, 64>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

Q8Cache padded(const uint8_t* kc, const uint8_t* ke, const uint8_t* vc, const uint8_t* ve, int64_t n_cap) {
  return Q8Cache{const_cast<uint8_t*>(kc), const_cast<uint8_t*>(ke), const_cast<uint8_t*>(vc),
                 const_cast<uint8_t*>(ve), nullptr, 0, n_cap, 0, 0};
}

}  // namespace
}  // namespace pvlm

using namespace pvlm;

extern "C" pvlm_status pvlm_rope_append_q8(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int64_t n_cap,
                                           double base, const int32_t* sections, const int32_t* pos,
                                           const void* q_in, const void* k_in, const void* v_in,
                                           const int32_t* ctx_len, void* q_out, uint8_t* k_codes,
                                           uint8_t* k_exps, uint8_t* v_codes, uint8_t* v_exps, int32_t* status,
                                           hipStream_t stream) {
  return append_run(dt, B, T, Hq, Hkv, D, base, sections, pos, q_in, k_in, v_in, ctx_len, q_out,
                    padded(k_codes, k_exps, v_codes, v_exps, n_cap), status, stream);
}

extern "C" pvlm_status pvlm_rope_append_q8_paged(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int page_size,
                                                 int max_pages, int64_t n_pages, double base,
                                                 const int32_t* sections, const int32_t* pos, const void* q_in,
                                                 const void* k_in, const void* v_in, const int32_t* page_table,
                                                 const int32_t* ctx_len, void* q_out, uint8_t* k_codes,
                                                 uint8_t* k_exps, uint8_t* v_codes, uint8_t* v_exps,
                                                 int32_t* status, hipStream_t stream) {
  Q8Cache c = padded(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  return append_run(dt, B, T, Hq, Hkv, D, base, sections, pos, q_in, k_in, v_in, ctx_len, q_out, c, status, stream);
}

extern "C" pvlm_status pvlm_quantize_kv(pvlm_dtype dt, int n_layers, int B, int Hkv, int D, int64_t src_cap,
                                        const void* k_src, const void* v_src, const int32_t* len, int64_t n_cap,
                                        uint8_t* k_codes, uint8_t* k_exps, uint8_t* v_codes, uint8_t* v_exps,
                                        int32_t* status, hipStream_t stream) {
  return quantize_run(dt, n_layers, B, Hkv, D, src_cap, k_src, v_src, len,
                      padded(k_codes, k_exps, v_codes, v_exps, n_cap), status, stream);
}

extern "C" pvlm_status pvlm_quantize_kv_paged(pvlm_dtype dt, int n_layers, int B, int Hkv, int D, int page_size,
                                              int max_pages, int64_t n_pages, int64_t src_cap, const void* k_src,
                                              const void* v_src, const int32_t* len, const int32_t* page_table,
                                              uint8_t* k_codes, uint8_t* k_exps, uint8_t* v_codes,
                                              uint8_t* v_exps, int32_t* status, hipStream_t stream) {
  Q8Cache c = padded(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  return quantize_run(dt, n_layers, B, Hkv, D, src_cap, k_src, v_src, len, c, status, stream);
}

extern "C" pvlm_status pvlm_gather_kv_q8(pvlm_dtype dst_dt, int n_layers, int B, int Hkv, int D, int64_t n_cap,
                                         const uint8_t* k_codes, const uint8_t* k_exps, const uint8_t* v_codes,
                                         const uint8_t* v_exps, const int32_t* idx, const int32_t* k, int32_t k_cap,
                                         const int32_t* tail_begin, const int32_t* tail_len, int64_t dst_cap, int fill,
                                         void* k_dst, uint8_t* k_dst_exps, void* v_dst, uint8_t* v_dst_exps,
                                         int32_t* status, hipStream_t stream) {
  return gather_run(dst_dt, n_layers, B, Hkv, D, padded(k_codes, k_exps, v_codes, v_exps, n_cap), idx, k, k_cap,
                    tail_begin, tail_len, dst_cap, fill, k_dst, k_dst_exps, v_dst, v_dst_exps, status, stream);
}

extern "C" pvlm_status pvlm_gather_kv_q8_paged(pvlm_dtype dst_dt, int n_layers, int B, int Hkv, int D, int page_size,
                                               int max_pages, int64_t n_pages, const uint8_t* k_codes,
                                               const uint8_t* k_exps, const uint8_t* v_codes, const uint8_t* v_exps,
                                               const int32_t* page_table, const int32_t* idx, const int32_t* k,
                                               int32_t k_cap, const int32_t* tail_begin, const int32_t* tail_len,
                                               int64_t dst_cap, int fill, void* k_dst, uint8_t* k_dst_exps, void* v_dst,
                                               uint8_t* v_dst_exps, int32_t* status, hipStream_t stream) {
  Q8Cache c = padded(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  return gather_run(dst_dt, n_layers, B, Hkv, D, c, idx, k, k_cap, tail_begin, tail_len, dst_cap, fill, k_dst, k_dst_exps,
                    v_dst, v_dst_exps, status, stream);
}

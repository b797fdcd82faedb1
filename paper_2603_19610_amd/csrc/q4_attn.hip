// Verify attention with fused per-token attention mass over a 4-bit cache (gfx950):
// pvlm_verify_attn's operation (ParallelVLM Sec. 2.2, Sec. 4.2; the mass of Sec. 3,
// Challenge 2) on rows in the format of q4.h, for T = 1 (a decode step) to 32 rows.
//
// Mathematics.  With K_i and V_i the values that the rows stand for:
//   s_i = scale <q, K_i>     P_i = softmax(s)_i over visible i
//   out = sum_i P_i V_i      mass_i = sum over rows of P_i
//  * Both products run on bf16 with fp32 sums: K_i and V_i are bf16 values (two
//    significant bits and a power of two), so their conversion rounds nothing.
//  * P is rounded to bf16 for the second product, half a step being 2^-9 to 2^-8
//    of a term of a result that is rounded to bf16 itself; the row is divided by
//    the sum of what was rounded.  lse and mass use the unrounded sum.
//  * One pass over a share with a running reference and sum in fp32; shares are
//    joined by the combine kernel.  The mass needs every row's sum first, so K is
//    read a second time.  Every order of summation is fixed.  No workgroup waits
//    for another.
//
// Launches, all on the caller's stream: partial, combine, and with the mass a third.
#include "q4.h"
#include "q4_plan.h"

namespace pvlm {
namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr double kLog2e = 1.4426950408889634;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();
// A wave's running reference may trail its row maximum by this much (log2 domain):
// O is rescaled only when a block's maximum exceeds it, which few blocks do.
// Probabilities then reach 2^24 in a type of bf16's range.
constexpr float kRefSlack = 24.f;

struct Q4Args : QShape {
  const uint16_t* q;
  Q4Cache c;
  const int32_t* ctx_len;
  int Hq, G, R;
  unsigned g_magic;  // row / G == row * g_magic >> 20 for row < 640 (2^20 / G + 1; G <= 640)
  int RTT;
  float sl2;         // scale * log2(e)
  float4* stats;     // [record][tile][16] of a row: log2-domain reference, sum, sum of the rounded, unused
  uint32_t* nan;     // [record] the values hold a NaN that not every row sees
  float2* rows;      // [B][Hkv][RTT * 16] maximum and inverse sum, for the mass
  float* opart;      // [record][tile][16][D] sums of P . V relative to that reference
  uint16_t* out;
  float* lse;
  float* mass;
  int32_t* status;
  int MG, GW, chunk;
};

// ------------------------------------------------------------ the shares --
// A wave's way to its share of the tokens, from the lengths on the device (the
// shares themselves: q8_plan.h).
typedef const __attribute__((address_space(4))) int32_t* ConstInts;  // (uniform loads go through the scalar cache)
__device__ __forceinline__ int uniform_load(const int32_t* p, int64_t i) { return ((ConstInts)(uintptr_t)p)[i]; }

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ int wave_scan(int x) {
#define PVLM_SCAN(ctrl, rows) x += __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, false)
  PVLM_SCAN(0x111, 0xf);  // row_shr:1, 2, 4, 8: within 16 lanes
  PVLM_SCAN(0x112, 0xf);
  PVLM_SCAN(0x114, 0xf);
  PVLM_SCAN(0x118, 0xf);
  PVLM_SCAN(0x142, 0xa);  // lane 15 of a row to the next: rows 1 and 3
  PVLM_SCAN(0x143, 0xc);  // lane 31 to rows 2 and 3
#undef PVLM_SCAN
  return x;
}

// The lengths of 64 sequences, one a lane, for q8_find.
struct Wave {
  const int32_t* ctx_len;
  int lane, ctx, raw, u, upto;
  __device__ __forceinline__ explicit Wave(const int32_t* lengths) : ctx_len(lengths), lane(threadIdx.x & 63) {}
  __device__ __forceinline__ void load(const QShape& a, int b0) {
    const bool here = b0 + lane < a.B;
    ctx = here ? clamp_ctx(a, ctx_len[b0 + lane]) : 0;
    raw = here ? units_of(a, ctx) : 0;
  }
  __device__ __forceinline__ void sum(int align) {
    u = aligned(raw, align);
    upto = wave_scan(u);
  }
  __device__ __forceinline__ int last() const { return __builtin_amdgcn_readlane(upto, 63); }
  __device__ __forceinline__ int ahead(int x) const { return __builtin_amdgcn_readlane(upto - u, x); }
  __device__ __forceinline__ int ctx_of(int x) const { return __builtin_amdgcn_readlane(ctx, x); }
  __device__ __forceinline__ int reaching(const QShape& a, int b0, int before, int at) const {
    const uint64_t m = __ballot(b0 + lane < a.B && (before + upto) * a.HR > at);
    return m ? __builtin_ctzll(m) : -1;
  }
};

struct Piece : QPiece {
  // false where the share is empty
  __device__ __forceinline__ bool first(const QShape& a, const int32_t* ctx_len) {
    return begin(a, q8_find<true>(a, Wave(ctx_len), blockIdx.x, 0), blockIdx.x);
  }
  // false where the share ends
  __device__ __forceinline__ bool next(const QShape& a, const int32_t* ctx_len) {
    return advance(a, [&](int x) { return __builtin_amdgcn_readfirstlane(clamp_ctx(a, uniform_load(ctx_len, x))); });
  }
};

// The page-table entry of token t (0 in a padded cache), and the row index (in
// rows) of the unit that t opens.  An entry outside the pool sets bad and is
// clamped into it.
__device__ __forceinline__ int page_entry(const Q8Cache& c, int b, int t) {
  return c.table ? uniform_load(c.table, (int64_t)b * c.max_pages + (t >> c.shift)) : 0;
}
__device__ __forceinline__ int64_t unit_row(const Q8Cache& c, int Hkv, int b, int g, int t, int page, bool& bad) {
  if (!c.table) return ((int64_t)b * Hkv + g) * c.n_cap + t;
  if (page < 0 || page >= c.n_pages) {
    bad = true;
    page = page < 0 ? 0 : (int)(c.n_pages - 1);
  }
  return (((int64_t)page * Hkv + g) << c.shift) + (t & ((1 << c.shift) - 1));
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int row_t(const Q4Args& a, int row) { return (int)((unsigned)row * a.g_magic >> 20); }

// Eight codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8 to_bf16(uint32_t w, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ float unit_of(uint32_t e) { return __uint_as_float(e << 23); }

// A lane's part of a 16-token tile of K or V: with n = lane & 15 and gq = lane >> 4,
// D / 4 consecutive values of row n from value (D / 4) gq on, D / 32 words of eight
// codes, within one block of 32.  A wave's loads of a tile are then one run of
// memory, and word ks is an operand of the 16x16x32 product over values
// (D / 4) gq + 8 ks + j: the order of the sum over d is free, so long as the queries
// have it too.
template <int D>
struct Codes {
  uint32_t w[D / 32];
  uint32_t e;
};
template <int D>
__device__ __forceinline__ void load_codes(const uint8_t* codes, const uint8_t* exps, int64_t row0, int n, int gq,
                                           Codes<D>& x) {
  const uint8_t* p = codes + row0 * (D / 2) + (n * (D / 2) + gq * (D / 8));
  if constexpr (D == 128) {
    const uintx4 v = *reinterpret_cast<const uintx4*>(p);
    x.w[0] = v[0], x.w[1] = v[1], x.w[2] = v[2], x.w[3] = v[3];
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x.w[0] = v.x, x.w[1] = v.y;
  }
  x.e = exps[row0 * (D / 32) + (n * (D / 32) + gq * (D / 32) / 4)];
}

template <int D>
struct Query {
  bf16x8 s[D / 32];
};
template <int D>
__device__ __forceinline__ void load_query(const Q4Args& a, int b, int g, int row, int gq, Query<D>& q) {
  const int r = min(row, a.R - 1), t = row_t(a, r), h = g * a.G + r - t * a.G;
  const bf16x8* src = reinterpret_cast<const bf16x8*>(a.q + (((size_t)b * a.T + t) * a.Hq + h) * D + gq * (D / 4));
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) q.s[ks] = src[ks];
}

// Maximum over the four lanes l, l^16, l^32, l^48.
__device__ __forceinline__ float rows4_maximum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// ---------------------------------------------------- values through LDS --
// P . V wants eight tokens' values of one column in a lane, where a lane has
// consecutive values of one token: a wave writes a unit of 32 tokens to LDS as bf16
// rows of its own and reads them transposed.  Nobody else touches them, and a
// wave's LDS operations run in order, so nothing waits but for data.
// Chunk c (16 bytes) of row r lies at chunk c ^ swz(r): a transposed read takes
// the same two chunks of eight rows at a time, a write one chunk of eight rows.
template <int D>
struct Lay {
  static constexpr int kUnit = 32 * D * 2;
  static __device__ __forceinline__ int swz(int r) { return D == 128 ? (r & 7) << 1 : (r >> 1 & 3) << 1; }
};
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s4* lds_s4;

template <int D>
__device__ __forceinline__ void put_values(uint32_t lds, int tt, const Codes<D>& x, int n, int gq) {
  const float unit = unit_of(x.e);
  const uint32_t row = lds + (16 * tt + n) * D * 2;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
    *(__attribute__((address_space(3))) bf16x8*)(row + (((gq * (D / 32) + c) ^ Lay<D>::swz(n)) << 4)) = to_bf16(x.w[c], unit);
}

// O += P . V over the unit in LDS; P holds tokens 4 gq + {0..3, 16..19}.
template <int D, int TPW, int S>
__device__ __forceinline__ void weigh(uint32_t lds, const bf16x8 (&P)[TPW][S], int u, floatx4 (&O)[TPW][D / 16], int n,
                                      int gq) {
  const int row = 4 * gq + n / 4;
  const uint32_t at = lds + row * D * 2 + 8 * (n & 1);
  const int sw = Lay<D>::swz(row), c0 = n >> 1 & 1;
#pragma unroll
  for (int jd = 0; jd < D / 16; ++jd) {
    const uint32_t p = at + (((2 * jd + c0) ^ sw) << 4);
    const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)p);
    const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(p + 16 * D * 2));
    const bf16x8 v = __builtin_bit_cast(bf16x8, (s8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
    for (int x = 0; x < TPW; ++x) O[x][jd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P[x][u], v, O[x][jd], 0, 0, 0);
  }
}

// -------------------------------------------------------- partial kernel --
template <int D, int RT>
struct PartShape {
  static constexpr int TPW = q4_waves(RT).tpw, RW = q4_waves(RT).rw, TW = q4_waves(RT).tw;
  static constexpr int kWaves = RW * TW, kThreads = kWaves * 64;
  static constexpr int NB = TPW == 3 ? 1 : 2;  // units of 32 tokens that a wave takes at a time
  static constexpr int kLds = kWaves * Lay<D>::kUnit;
};

template <int D, int RT>
__global__ void __launch_bounds__((PartShape<D, RT>::kThreads)) __attribute__((amdgpu_waves_per_eu(2, 2)))
q4_part_kernel(Q4Args a) {
  typedef PartShape<D, RT> S_;
  constexpr int TPW = S_::TPW, TW = S_::TW, NB = S_::NB, DPL = D / 16, BT = 32 * NB;
  extern __shared__ __align__(1024) char s_values[];  // [wave][32][D] bf16; then a tile's O, [wave][16][D] fp32
  __shared__ float s_ref[S_::kWaves][16], s_z[S_::kWaves][16], s_zt[S_::kWaves][16];
  __shared__ uint32_t s_nan[S_::kWaves];

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && w == 0)
    for (int b = threadIdx.x; b < a.B; b += 64)
      if (a.ctx_len[b] < 0 || a.ctx_len[b] > a.max_ctx) dev_flag(a.status, PVLM_DEV_RANGE);
  Piece p;
  if (!p.first(a, a.ctx_len)) return;
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int tw = w % TW, rw = w / TW;
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_addr(s_values)) + w * Lay<D>::kUnit;
  bool bad_page = false;
  do {
    const int tile0 = p.rg * RT + rw * TPW;  // of the KV head's
    Query<D> q[TPW];
    int lim[TPW];
    float ref[TPW], z[TPW];
    floatx4 O[TPW][DPL], zt[TPW];
#pragma unroll
    for (int x = 0; x < TPW; ++x) {
      const int row = (tile0 + x) * 16 + n;
      load_query<D>(a, p.b, p.g, row, gq, q[x]);
      lim[x] = rw * TPW + x < RT && row < a.R ? min(p.c1 - 1, p.ctx + row_t(a, row)) : -1;
      ref[x] = kNegInf;
      z[x] = 0.f;
      zt[x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int jd = 0; jd < DPL; ++jd) O[x][jd] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    uint32_t nan = 0;
    Codes<D> kc[NB][2], vc[NB][2];
    auto load = [&](int tb) {
#pragma unroll
      for (int u = 0; u < NB; ++u) {
        const int t = min(tb + 32 * u, (p.c1 - 1) & ~31);
        const int64_t r = unit_row(a.c, a.Hkv, p.b, p.g, t, page_entry(a.c, p.b, t), bad_page);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) load_codes<D>(a.c.kc, a.c.ke, r + 16 * tt, n, gq, kc[u][tt]);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) load_codes<D>(a.c.vc, a.c.ve, r + 16 * tt, n, gq, vc[u][tt]);
      }
    };
    auto block = [&](int tb, bool tail) {
      floatx4 S[TPW][2 * NB];
#pragma unroll
      for (int j = 0; j < 2 * NB; ++j) {
        const float unit = unit_of(kc[j / 2][j % 2].e);
#pragma unroll
        for (int x = 0; x < TPW; ++x) S[x][j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < D / 32; ++ks) {
          const bf16x8 k = to_bf16(kc[j / 2][j % 2].w[ks], unit);
#pragma unroll
          for (int x = 0; x < TPW; ++x) S[x][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[x].s[ks], S[x][j], 0, 0, 0);
        }
      }
      if (tail) {
#pragma unroll
        for (int x = 0; x < TPW; ++x)
#pragma unroll
          for (int j = 0; j < 8 * NB; ++j)
            if (tb + 16 * (j / 4) + 4 * gq + j % 4 > lim[x]) S[x][j / 4][j % 4] = kNegInf;
#pragma unroll
        for (int u = 0; u < NB; ++u)
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            // rows past the piece become zeros (their probabilities are 0, and 0 times what
            // an unwritten row holds may be NaN), and so do NaN of rows that not every query
            // row sees: the record's flag has the combine kernel look for them
            const int t = tb + 32 * u + 16 * tt + n;
            const bool past = t >= p.c1, hidden = t > p.ctx && vc[u][tt].e == 255;
            if (hidden && !past) nan = 1;
            if (past || hidden) {
              vc[u][tt].e = 127;
#pragma unroll
              for (int c = 0; c < D / 32; ++c) vc[u][tt].w[c] = 0;
            }
          }
      }
      bf16x8 P[TPW][NB];
#pragma unroll
      for (int x = 0; x < TPW; ++x) {
        float m = kNegInf;
#pragma unroll
        for (int j = 0; j < 8 * NB; ++j) m = fmaxf(m, S[x][j / 4][j % 4]);
        m *= a.sl2;
        if (__any(m > ref[x] + kRefSlack)) {  // the first block, and seldom after it
          const float nm = fmaxf(ref[x], rows4_maximum(m));
          const float al = ref[x] == kNegInf ? 0.f : fast_exp2(ref[x] - nm);
          z[x] *= al;
          ref[x] = nm;
          floatx4 f;
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = __shfl(al, 4 * gq + i, 64);
          zt[x] = zt[x] * f;
#pragma unroll
          for (int jd = 0; jd < DPL; ++jd) O[x][jd] = O[x][jd] * f;
        }
        const float r = ref[x] == kNegInf ? 0.f : ref[x];  // no visible token yet: P = 0
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8 * NB; ++j) {
          const float e = fast_exp2(fmaf(S[x][j / 4][j % 4], a.sl2, -r));
          sum += e;
          P[x][j / 8][j % 8] = static_cast<__bf16>(e);
        }
        z[x] += sum;
      }
      bf16x8 ones;
#pragma unroll
      for (int j = 0; j < 8; ++j) ones[j] = static_cast<__bf16>(1.f);
#pragma unroll
      for (int u = 0; u < NB; ++u) {
#pragma unroll
        for (int x = 0; x < TPW; ++x) zt[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P[x][u], ones, zt[x], 0, 0, 0);
        asm volatile("" ::: "memory");  // (the wave's LDS operations keep their order)
        put_values<D>(lds, 0, vc[u][0], n, gq);
        put_values<D>(lds, 1, vc[u][1], n, gq);
        asm volatile("" ::: "memory");
        weigh<D, TPW, NB>(lds, P, u, O, n, gq);
        asm volatile("" ::: "memory");
      }
    };
    const int whole = min(p.c1 - 1, p.ctx);  // the last token that every row sees
    for (int tb = p.c0 + BT * tw; tb < p.c1; tb += BT * TW) {
      load(tb);
      block(tb, __builtin_amdgcn_readfirstlane(tb + BT - 1 - whole) > 0);
    }
    // The token waves' results joined: a tile at a time, through LDS (position
    // DPL n + jd of a row holds column 16 jd + n).
    const int rec = p.group(a) + blockIdx.x;
    const bool any = __any(nan);
    if (lane == 0) s_nan[w] = any;
#pragma unroll
    for (int x = 0; x < TPW; ++x) {
      __syncthreads();
      const float zz = rows4_sum(z[x]);
      if (gq == 0) s_ref[w][n] = ref[x], s_z[w][n] = zz;
      if (n == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) s_zt[w][4 * gq + i] = zt[x][i];
      float* mine = reinterpret_cast<float*>(s_values) + w * 16 * D;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int h = 0; h < DPL / 4; ++h)
          *reinterpret_cast<float4*>(mine + (4 * gq + i) * D + DPL * n + 4 * h) =
              make_float4(O[x][4 * h][i], O[x][4 * h + 1][i], O[x][4 * h + 2][i], O[x][4 * h + 3][i]);
      __syncthreads();
      const int tile = rw * TPW + x;
      if (tile < RT) {
        for (int i = tw * 64 + lane; i < 16 * D / 4; i += TW * 64) {
          const int r = i / (D / 4), c = i % (D / 4);
          if ((p.rg * RT + tile) * 16 + r >= a.R) continue;
          float M = kNegInf;
#pragma unroll
          for (int k = 0; k < TW; ++k) M = fmaxf(M, s_ref[rw * TW + k][r]);
          const float base = M == kNegInf ? 0.f : M;
          float Z = 0.f, Zt = 0.f;
          floatx4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < TW; ++k) {
            const int v = rw * TW + k;
            if (s_z[v][r] == 0.f) continue;  // nothing that the row sees
            const float f = fast_exp2(s_ref[v][r] - base);
            Z += s_z[v][r] * f;
            Zt += s_zt[v][r] * f;
            const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(s_values) + (v * 16 + r) * D + 4 * c);
            o[0] = fmaf(y.x, f, o[0]), o[1] = fmaf(y.y, f, o[1]), o[2] = fmaf(y.z, f, o[2]), o[3] = fmaf(y.w, f, o[3]);
          }
          const size_t at = ((size_t)rec * RT + tile) * 16 + r;
          *reinterpret_cast<float4*>(a.opart + at * D + 4 * c) = make_float4(o[0], o[1], o[2], o[3]);
          if (c == 0) a.stats[at] = make_float4(M, Z, Zt, 0.f);
        }
      }
    }
    if (threadIdx.x == 0) {
      uint32_t any_wave = 0;
      for (int k = 0; k < S_::kWaves; ++k) any_wave |= s_nan[k];
      a.nan[rec] = any_wave;
    }
    __syncthreads();
  } while (p.next(a, a.ctx_len));
  if (bad_page && lane == 0) dev_flag(a.status, PVLM_DEV_RANGE);
}

// -------------------------------------------------------- combine kernel --
// A wave joins a row's records: their references and sums a lane each, then the
// partial results weighted by exp2(record's reference - row maximum).
constexpr int kCombineWaves = 4;

template <int D>
__global__ void __launch_bounds__(kCombineWaves * 64) q4_combine_kernel(Q4Args a, int RT) {
  constexpr int C = D / 64, DPL = D / 16, kU = 8;
  const int lane = threadIdx.x & 63;
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * kCombineWaves + (threadIdx.x >> 6));
  if (id >= a.B * a.Hkv * a.R) return;
  const int bg = id / a.R, row = id - bg * a.R, b = bg / a.Hkv, g = bg - b * a.Hkv;
  const Shares s = q8_find<false>(a, Wave(a.ctx_len), 0, b);
  const int rg = row / (16 * RT), tile = row / 16 - rg * RT;
  const Holders h = holders(a, s.per, s.align, s.before, b, g * a.RG + rg, s.ctx);
  const size_t at = ((size_t)h.rec * RT + tile) * 16 + row % 16, step = (size_t)RT * 16;
  float m = kNegInf, z = 0.f, zt = 0.f, o[C];
  bool nan = false;
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.f;
  for (int s0 = 0; s0 < h.count; s0 += 64) {
    const int cnt = min(64, h.count - s0);
    float4 st = make_float4(kNegInf, 0.f, 0.f, 0.f);
    if (lane < cnt) {
      st = a.stats[at + (s0 + lane) * step];
      nan |= a.nan[h.rec + s0 + lane] != 0 && st.y != 0.f;
    }
    const float M = fmaxf(m, warp_max(st.y != 0.f ? st.x : kNegInf)), r = M == kNegInf ? 0.f : M;
    const float f = z != 0.f ? fast_exp2(m - r) : 0.f, e = st.y != 0.f ? fast_exp2(st.x - r) : 0.f;
    z = (z != 0.f ? z * f : 0.f) + warp_sum(st.y != 0.f ? st.y * e : 0.f);
    zt = zt * f + warp_sum(st.y != 0.f ? st.z * e : 0.f);
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] *= f;
    m = M;
    for (int k0 = 0; k0 < cnt; k0 += kU) {
      float v[kU][C], wgt[kU];
#pragma unroll
      for (int k = 0; k < kU; ++k) {
        const int i = min(k0 + k, cnt - 1);
        const float* src = a.opart + (at + (s0 + i) * step) * D + C * lane;
#pragma unroll
        for (int c = 0; c < C; ++c) v[k][c] = src[c];
        wgt[k] = __shfl(e, i, 64);
      }
#pragma unroll
      for (int k = 0; k < kU; ++k)
        if (k0 + k < cnt)  // (a weight of 0 too: NaN stays)
#pragma unroll
          for (int c = 0; c < C; ++c) o[c] = fmaf(v[k][c], wgt[k], o[c]);
    }
  }
  const int t = row_t(a, row), head = g * a.G + row - t * a.G;
  const float inv = 1.f / zt;
  const bool look = __any(nan);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int pos = C * lane + c, col = 16 * (pos % DPL) + pos / DPL;
    float y = o[c] * inv;
    if (look)  // the values past the context that the row sees, whose NaN counted as 0
      for (int j = s.ctx + 1; j <= s.ctx + t; ++j) {
        bool flagged_before;  // by the partial kernel
        const int64_t vr = unit_row(a.c, a.Hkv, b, g, j & ~31, page_entry(a.c, b, j), flagged_before) + (j & 31);
        if (a.c.ve[vr * (D / 32) + col / 32] == 255) y = __uint_as_float(0x7fc00000u);
      }
    a.out[(((size_t)b * a.T + t) * a.Hq + head) * D + col] = f32_to_bf16(y);
  }
  if (lane == 0) {
    if (a.lse) a.lse[((size_t)b * a.Hq + head) * a.T + t] = (m + __log2f(z)) * kLn2;
    if (a.mass) a.rows[(size_t)bg * a.RTT * 16 + row] = make_float2(m, 1.f / z);
  }
}

// ----------------------------------------------------------- mass kernel --
// A workgroup takes a run of a sequence's tokens and every query row: its waves
// hold the queries of a set of row tiles each (GW sets at a time), with the rows on
// the M side, so that a lane's scores of a token sum up in the lane.  A row's maximum
// and inverse sum are kept apart: a probability's exponent is rounded at its
// distance from the maximum, which is nothing where the mass is.
template <int D, int MT>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) q4_mass_kernel(Q4Args a) {
  __shared__ float s_mass[8][512];
  const int b = blockIdx.y;
  const int64_t t0 = (int64_t)blockIdx.x * a.chunk;
  const int ctx = clamp_ctx(a, __builtin_amdgcn_readfirstlane(uniform_load(a.ctx_len, b)));
  const int N = ctx + a.T;
  float* mass = a.mass + (size_t)b * a.c.n_cap;
  const int64_t t_end = min(t0 + a.chunk, a.c.n_cap);
  if (t0 >= N) {
    for (int64_t t = t0 + threadIdx.x; t < t_end; t += 512) mass[t] = 0.f;
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int gw = w % a.GW, tw = w / a.GW, TW = 8 / a.GW;
  const int c0 = (int)t0, c1 = min((int)t_end, N);
  bool bad_page = false;
  for (int set = gw; set < a.Hkv * a.MG; set += a.GW) {
    const int g = set / a.MG, tile0 = (set - g * a.MG) * MT;
    Query<D> q[MT];
    float top[MT][4], inv[MT][4];
#pragma unroll
    for (int x = 0; x < MT; ++x) {
      load_query<D>(a, b, g, (tile0 + x) * 16 + n, gq, q[x]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = (tile0 + x) * 16 + 4 * gq + i;
        const float2 s = a.rows[((size_t)b * a.Hkv + g) * a.RTT * 16 + min(row, a.R - 1)];
        top[x][i] = row < a.R ? s.x : __builtin_huge_valf();
        inv[x][i] = row < a.R ? s.y : 0.f;
      }
    }
    for (int t = c0 + 16 * tw; t < c1; t += 16 * TW) {
      const int unit = t & ~31;
      const int64_t r = unit_row(a.c, a.Hkv, b, g, unit, page_entry(a.c, b, unit), bad_page) + (t - unit);
      Codes<D> kc;
      load_codes<D>(a.c.kc, a.c.ke, r, n, gq, kc);
      const float u = unit_of(kc.e);
      floatx4 S[MT];
#pragma unroll
      for (int x = 0; x < MT; ++x) S[x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) {
        const bf16x8 k = to_bf16(kc.w[ks], u);
#pragma unroll
        for (int x = 0; x < MT; ++x) S[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[x].s[ks], k, S[x], 0, 0, 0);
      }
      float sum = 0.f;
      if (__builtin_amdgcn_readfirstlane(t + 15 - ctx) > 0) {
#pragma unroll
        for (int x = 0; x < MT; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int row = (tile0 + x) * 16 + 4 * gq + i;
            if (row < a.R && t + n <= ctx + row_t(a, row)) sum += fast_exp2(fmaf(S[x][i], a.sl2, -top[x][i])) * inv[x][i];
          }
      } else {
#pragma unroll
        for (int x = 0; x < MT; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum = fmaf(fast_exp2(fmaf(S[x][i], a.sl2, -top[x][i])), inv[x][i], sum);
      }
      sum = rows4_sum(sum);
      if (gq == 0) {
        float* at = &s_mass[gw][t - c0 + n];
        *at = set == gw ? sum : *at + sum;
      }
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < (int)(t_end - t0); i += 512) {
    float sum = 0.f;
    if (c0 + i < c1)
      for (int k = 0; k < a.GW; ++k) sum += s_mass[k][i];
    mass[t0 + i] = sum;
  }
  if (bad_page && lane == 0) dev_flag(a.status, PVLM_DEV_RANGE);
}

// ------------------------------------------------------------------ host --
typedef void (*Q4Kernel)(Q4Args);
struct PartKernel {
  Q4Kernel fn;
  int threads, lds;
};
template <int D, int RT>
PartKernel part() {
  return {q4_part_kernel<D, RT>, PartShape<D, RT>::kThreads, PartShape<D, RT>::kLds};
}
template <int D>
PartKernel pick_part(int RT) {
  switch (RT) {
    case 1: return part<D, 1>();
    case 2: return part<D, 2>();
    case 3: return part<D, 3>();
    case 4: return part<D, 4>();
    case 5: return part<D, 5>();
    case 6: return part<D, 6>();
    case 7: return part<D, 7>();
    case 8: return part<D, 8>();
    default: return part<D, 9>();
  }
}
template <int D>
Q4Kernel pick_mass(int MT) {
  switch (MT) {
    case 1: return q4_mass_kernel<D, 1>;
    case 2: return q4_mass_kernel<D, 2>;
    case 3: return q4_mass_kernel<D, 3>;
    case 4: return q4_mass_kernel<D, 4>;
    default: return q4_mass_kernel<D, 5>;
  }
}

pvlm_status verify_q4_run(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int64_t max_ctx, float scale,
                          const void* q, const Q4Cache& c, const int32_t* ctx_len, void* out, float* mass, float* lse,
                          void* ws, size_t ws_bytes, int32_t* status, hipStream_t stream) {
  if (!q || !ctx_len || !out) return PVLM_ERR_NULL;
  if (dt != PVLM_BF16) return PVLM_ERR_UNSUPPORTED;
  if (!(scale > 0.f) || !std::isfinite(scale)) return PVLM_ERR_SHAPE;
  pvlm_status st = check_verify_q4(B, T, Hq, Hkv, D, c.n_cap, max_ctx);
  if (st != PVLM_OK) return st;
  st = check_q4(c.kc, c.ke, c.vc, c.ve, c.n_cap);
  if (st != PVLM_OK) return st;
  if ((uintptr_t)q % 16 != 0) return PVLM_ERR_UNSUPPORTED;
  DeviceInfo di;
  st = device_info(&di, stream);
  if (st != PVLM_OK) return st;
  Q4Split p;
  split_verify_q4(B, T, Hq, Hkv, D, max_ctx, di.cus, &p);
  if (!ws || ws_bytes < p.bytes || (uintptr_t)ws % 16 != 0) return PVLM_ERR_WORKSPACE;
  char* wsb = static_cast<char*>(ws);
  Q4Args a;
  a.q = static_cast<const uint16_t*>(q);
  a.c = c;
  a.ctx_len = ctx_len;
  a.B = B;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = p.G;
  a.R = p.R;
  a.g_magic = (1u << 20) / (unsigned)p.G + 1u;
  a.RTT = p.RTT;
  a.RG = p.RG;
  a.HR = Hkv * p.RG;
  a.max_ctx = (int)max_ctx;
  a.wgs = p.wgs;
  a.sl2 = (float)((double)scale * kLog2e);
  a.stats = reinterpret_cast<float4*>(wsb + p.off_stats);
  a.nan = reinterpret_cast<uint32_t*>(wsb + p.off_nan);
  a.rows = reinterpret_cast<float2*>(wsb + p.off_rows);
  a.opart = reinterpret_cast<float*>(wsb + p.off_opart);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.mass = mass;
  a.status = status;
  a.MG = p.MG;
  a.GW = p.GW;
  a.chunk = p.chunk;
  const PartKernel k = D == 128 ? pick_part<128>(p.RT) : pick_part<64>(p.RT);
  PVLM_HIP(allow_dynamic_lds(reinterpret_cast<const void*>(k.fn), k.lds));
  hipLaunchKernelGGL(k.fn, dim3(p.wgs), dim3(k.threads), k.lds, stream, a);
  PVLM_LAUNCHED();
  const int rows = B * Hkv * p.R;
  hipLaunchKernelGGL(D == 128 ? q4_combine_kernel<128> : q4_combine_kernel<64>,
                     dim3((rows + kCombineWaves - 1) / kCombineWaves), dim3(kCombineWaves * 64), 0, stream, a, p.RT);
  PVLM_LAUNCHED();
  if (mass) {
    const unsigned chunks = (unsigned)((c.n_cap + p.chunk - 1) / p.chunk);
    hipLaunchKernelGGL(D == 128 ? pick_mass<128>(p.MT) : pick_mass<64>(p.MT), dim3(chunks, B), dim3(512), 0, stream, a);
    PVLM_LAUNCHED();
  }
  return PVLM_OK;
}

Q4Cache view(const uint8_t* kc, const uint8_t* ke, const uint8_t* vc, const uint8_t* ve, int64_t n_cap) {
  return Q4Cache{const_cast<uint8_t*>(kc), const_cast<uint8_t*>(ke), const_cast<uint8_t*>(vc),
                 const_cast<uint8_t*>(ve), nullptr, 0, n_cap, 0, 0};
}

}  // namespace
}  // namespace pvlm

using namespace pvlm;

extern "C" size_t pvlm_verify_attn_q4_workspace_size(int B, int T, int Hq, int Hkv, int D, int64_t n_cap,
                                                     int64_t max_ctx) {
  DeviceInfo di;
  if (check_verify_q4(B, T, Hq, Hkv, D, n_cap, max_ctx) != PVLM_OK || device_info(&di) != PVLM_OK) return 0;
  Q4Split p;
  split_verify_q4(B, T, Hq, Hkv, D, max_ctx, di.cus, &p);
  return p.bytes;
}

extern "C" pvlm_status pvlm_verify_attn_q4(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int64_t n_cap,
                                           int64_t max_ctx, float scale, const void* q, const uint8_t* k_codes,
                                           const uint8_t* k_exps, const uint8_t* v_codes, const uint8_t* v_exps,
                                           const int32_t* ctx_len, void* out, float* mass, float* lse, void* ws,
                                           size_t ws_bytes, int32_t* status, hipStream_t stream) {
  return verify_q4_run(dt, B, T, Hq, Hkv, D, max_ctx, scale, q, view(k_codes, k_exps, v_codes, v_exps, n_cap), ctx_len,
                       out, mass, lse, ws, ws_bytes, status, stream);
}

extern "C" pvlm_status pvlm_verify_attn_q4_paged(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int page_size,
                                                 int max_pages, int64_t n_pages, int64_t max_ctx, float scale,
                                                 const void* q, const uint8_t* k_codes, const uint8_t* k_exps,
                                                 const uint8_t* v_codes, const uint8_t* v_exps,
                                                 const int32_t* page_table, const int32_t* ctx_len, void* out,
                                                 float* mass, float* lse, void* ws, size_t ws_bytes,
                                                 int32_t* status, hipStream_t stream) {
  Q4Cache c = view(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  return verify_q4_run(dt, B, T, Hq, Hkv, D, max_ctx, scale, q, c, ctx_len, out, mass, lse, ws, ws_bytes, status, stream);
}

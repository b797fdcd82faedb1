// Verify attention with fused per-token attention mass over an 8-bit cache
// (gfx950): pvlm_verify_attn's operation (ParallelVLM Sec. 2.2, Sec. 4.2; the
// mass of Sec. 3, Challenge 2) on rows in the format of q8.h, for T = 1 (a
// decode step) to 32 rows.
//
// Mathematics.  With K_i = ck_i 2^(ek_i - 127) and V_i likewise:
//   s_i = scale <q, ck_i> 2^(ek_i - 127)     P_i = softmax(s)_i over visible i
//   out = sum_i (P_i 2^(ev_i - 127)) cv_i    mass_i = sum over rows of P_i
//  * Both products run on bf16 with fp32 sums: codes become bf16 exactly, a
//    key's with its row's power of two taken in by the conversion.  (The 8-bit
//    matrix instructions align an instruction's products to the largest of them
//    and lose up to 2^-14 of it, measured against float64; bf16 ones 2^-21.)
//  * P is rounded to bf16 after its row's unit 2^(ev - 127) is taken in: half a
//    step, 2^-8 of each term, of a result that is rounded to bf16 itself.
//  * One pass over a chunk with a running maximum and sum in fp32; the chunks'
//    (maximum, sum) and fp32 O partials are joined by the finish kernel.  The
//    mass needs every row's log-sum-exp first, so K is read a second time.
//    Every order of summation is fixed.  No workgroup waits for another.
#include "q8.h"
#include "q8_plan.h"

namespace pvlm {
namespace {

typedef int intx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kPageSlots = 512;  // page-table entries a workgroup stages in LDS
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();
// A wave's running reference may trail its row maximum by this much (log2
// domain): O is rescaled only when a block's maximum exceeds it.
constexpr float kRefSlack = 8.f;
constexpr int kFinWaves = kFinThreads / 64;

struct QArgs {
  const uint16_t* q;
  Q8Cache c;
  const int32_t* ctx_len;
  int B, T, Hq, Hkv, G, R;
  unsigned g_magic;  // row / G == row * g_magic >> 20 for row < 640 (2^20 / G + 1; G <= 640)
  int RTT, RG;
  int max_ctx;
  int splits, chunk, units;
  float sl2;         // scale * log2(e)
  float* mpart;      // [B][Hkv * RG][n_cap] mass of one workgroup's rows
  float2* stats;     // [B * Hkv * RTT][splits][16] (log2-domain maximum, sum) of a chunk's rows
  float* opart;      // [B * Hkv * RTT][splits][16][D] chunk sums relative to that maximum
  uint16_t* out;
  float* lse;
  float* mass;
  int32_t* status;
  int mass_wgs, mass_per, mass_rows;  // finish kernel: workgroups that sum the mass, of a sequence, rows of one
};

struct Unit {
  int split, bg, b, g, rg, ctx, N, c0, c1;
};

__device__ __forceinline__ int seq_ctx(const QArgs& a, int b, bool flag) {
  const int ctx = a.ctx_len[b];
  if (ctx >= 0 && ctx <= a.max_ctx) return ctx;
  if (flag) dev_flag(a.status, PVLM_DEV_RANGE);
  return ctx < 0 ? 0 : a.max_ctx;
}

// Workgroup i runs on XCD i % 8; consecutive units, whose row groups read the
// same cache rows, go to one XCD and share its L2 (a matter of speed only).
__device__ __forceinline__ bool decode_unit(const QArgs& a, Unit& u) {
  const int per = gridDim.x / 8;
  const int lg = ((int)blockIdx.x % 8) * per + (int)blockIdx.x / 8;
  if (lg >= a.units) return false;
  u.rg = lg % a.RG;
  const int cs = lg / a.RG;
  u.split = cs % a.splits;
  u.bg = cs / a.splits;
  u.g = u.bg % a.Hkv;
  u.b = u.bg / a.Hkv;
  u.ctx = seq_ctx(a, u.b, u.split == 0 && threadIdx.x == 0);
  u.N = u.ctx + a.T;
  u.c0 = u.split * a.chunk;
  u.c1 = min(u.c0 + a.chunk, u.N);
  return u.c0 < u.N;
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int row_t(const QArgs& a, int row) { return (int)((unsigned)row * a.g_magic >> 20); }

// ------------------------------------------------------------ cache rows --
// Rows of (b, g): row r of the chunk lies at index base + r (padded), or in
// page `pages[...]` of the pool.  Entries are checked once, when they are
// staged (every thread takes part); one outside the pool is flagged and
// clamped into it.
struct Rows {
  int64_t base;            // padded: row index of logical row 0; paged: of the head's row 0 in pool page 0
  int64_t page_rows;       // rows between pages, all heads
  const int32_t* table;
  const int32_t* staged;   // LDS copy from logical page page0, where the chunk's entries fit
  int64_t n_pages;
  int shift, page0;
  bool paged, in_lds;
};

__device__ __forceinline__ Rows rows_setup(const QArgs& a, const Unit& u, int32_t* s_pages) {
  Rows v;
  v.paged = a.c.table != nullptr;
  if (!v.paged) {
    v.base = ((int64_t)u.b * a.Hkv + u.g) * a.c.n_cap;
    v.page_rows = 0;
    v.table = nullptr;
    v.staged = nullptr;
    v.n_pages = 0;
    v.shift = v.page0 = 0;
    v.in_lds = false;
    return v;
  }
  v.shift = a.c.shift;
  v.base = (int64_t)u.g << v.shift;
  v.page_rows = (int64_t)a.Hkv << v.shift;
  v.table = a.c.table + (int64_t)u.b * a.c.max_pages;
  v.staged = s_pages;
  v.n_pages = a.c.n_pages;
  v.page0 = u.c0 >> v.shift;
  const int p1 = (u.c1 - 1) >> v.shift;
  v.in_lds = p1 - v.page0 < kPageSlots;
  for (int pg = v.page0 + threadIdx.x; pg <= p1; pg += (int)blockDim.x) {
    int e = v.table[pg];
    if (e < 0 || e >= v.n_pages) {
      dev_flag(a.status, PVLM_DEV_RANGE);
      e = e < 0 ? 0 : (int)(v.n_pages - 1);
    }
    if (v.in_lds) s_pages[pg - v.page0] = e;
  }
  __syncthreads();
  return v;
}

__device__ __forceinline__ int64_t row_index(const Rows& v, int r) {
  if (!v.paged) return v.base + r;
  int pg;
  if (v.in_lds) {
    pg = v.staged[(r >> v.shift) - v.page0];
  } else {
    pg = v.table[r >> v.shift];
    pg = pg < 0 ? 0 : pg >= v.n_pages ? (int)(v.n_pages - 1) : pg;
  }
  return v.base + pg * v.page_rows + (r & ((1 << v.shift) - 1));
}

// --------------------------------------------------------------- layouts --
// Tokens are the M side of the score tiles and query rows the N side.  A block
// is 64 tokens: tile tt holds tokens 4 n + tt, so lane (n, gq) = (lane & 15,
// lane >> 4), which owns rows 4 gq .. 4 gq + 3 of each tile's result, gets the
// 16 consecutive tokens 16 gq + 4 i + tt: the order P.V wants for its A
// operand, and one 16-byte read of their exponents.  The exponents of a
// lane's four key rows are one 4-byte word.
//
// LDS holds a stage's codes as lines of 256 bytes (2 rows at D = 128, 4 at 64):
// 16-byte chunk c of row r lies at position ((r mod rows-per-line) * CH + c) ^
// key(r) of its line.  K's key is (r / 4) mod 16: the 16 rows 4 n + tt of an
// operand read fall on 16 positions.  V's key spreads the 8 consecutive rows
// of a transposed read over the positions.
template <int D>
struct Lay {
  static constexpr int CH = D / 16, LR = 256 / D, ST = kQStageBytes / D, DPL = D / 16;
  static __device__ __forceinline__ int kkey(int line) { return (line * LR >> 2) & 15; }
  static __device__ __forceinline__ int vkey(int line) {
    if constexpr (D == 128) return (line & 3) | ((line >> 1) & 4);
    else return line & 3;
  }
  static __device__ __forceinline__ int at(int r, int c, int key) {
    return (r / LR) * 256 + ((((r % LR) * CH + c) ^ key) << 4);
  }
};

// One 16-byte piece of a stage: piece i of the LDS image, as (row, chunk).
template <int D, bool IS_K>
__device__ __forceinline__ void piece(int i, int& row, int& chunk) {
  typedef Lay<D> L;
  const int line = i >> 4, p = (i & 15) ^ (IS_K ? L::kkey(line) : L::vkey(line));
  row = line * L::LR + p / L::CH;
  chunk = p % L::CH;
}

// ---------------------------------------------------------------- operands --
// A lane's d range of a row: 32 values at D = 128, 16 at 64, of which k-step s
// takes values 8 s .. 8 s + 7 (the same assignment on both sides).
template <int D>
struct Query {
  bf16x8 s[D / 32];
};

template <int D>
__device__ __forceinline__ void load_query(const QArgs& a, int b, int g, int row, int gq, Query<D>& q) {
  const int r = min(row, a.R - 1), t = row_t(a, r), h = g * a.G + r - t * a.G;
  const bf16x8* src = reinterpret_cast<const bf16x8*>(a.q + (((size_t)b * a.T + t) * a.Hq + h) * D + D / 4 * gq);
#pragma unroll
  for (int s = 0; s < D / 32; ++s) q.s[s] = src[s];
}

// Eight codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8 to_bf16(uint32_t lo, uint32_t hi, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, unit, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, unit, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, unit, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, unit, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Scores of one block against a row tile: S[tt][i] is token 16 gq + 4 i + tt.
template <int D>
__device__ __forceinline__ void scores(const char* kb, uint32_t exps, int r0, int n, int gq, const Query<D>& q,
                                       floatx4 (&S)[4]) {
  typedef Lay<D> L;
  constexpr int NC = D / 64;  // 16-byte chunks of a lane's range
  uint4 k[4][NC];
#pragma unroll
  for (int tt = 0; tt < 4; ++tt) {
    const int r = r0 + 4 * n + tt, key = L::kkey(r / L::LR);
#pragma unroll
    for (int c = 0; c < NC; ++c) k[tt][c] = *reinterpret_cast<const uint4*>(kb + L::at(r, NC * gq + c, key));
  }
#pragma unroll
  for (int tt = 0; tt < 4; ++tt) S[tt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
      const float unit = q8_unit((exps >> (8 * tt)) & 0xffu);
      S[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16(k[tt][c].x, k[tt][c].y, unit), q.s[2 * c], S[tt], 0, 0, 0);
      S[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16(k[tt][c].z, k[tt][c].w, unit), q.s[2 * c + 1], S[tt], 0, 0, 0);
    }
}

// Eight consecutive tokens (rows r .. r + 7 of the lane group) of column 16 jd + n.
template <int D>
__device__ __forceinline__ intx2 read_v(const char* vb, int r, int jd, int n) {
  typedef Lay<D> L;
  typedef __attribute__((address_space(3))) intx2* lds_v2;
  const int row = r + n / 2;
  const uint32_t at = lds_addr(vb) + L::at(row, jd, L::vkey(row / L::LR)) + 8 * (n & 1);
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2)at);
}
// O += P' . V over one block.  P'[j] is token 16 gq + j.
template <int D>
__device__ __forceinline__ void weigh(const char* vb, int r0, int n, int gq, const float (&P)[16],
                                      floatx4 (&O)[D / 16]) {
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {
    bf16x8 pa;
#pragma unroll
    for (int j = 0; j < 8; ++j) pa[j] = static_cast<__bf16>(P[8 * ks + j]);
#pragma unroll
    for (int jd = 0; jd < D / 16; ++jd) {
      const intx2 v = read_v<D>(vb, r0 + 16 * gq + 8 * ks, jd, n);
      O[jd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa, to_bf16(v[0], v[1], 1.f), O[jd], 0, 0, 0);
    }
  }
}
// The same for a block in which some rows see less than others: a NaN value
// (0 times it is NaN) must not reach the rows that do not see it.  NaN codes
// count as 0 in the product, and a second one, of the rows' visibility with
// the NaN positions, says which results they belong to.  `seen` has bit j for
// token 16 gq + j.
template <int D>
__device__ __forceinline__ void weigh_masked(const char* vb, int r0, int n, int gq, const float (&P)[16],
                                             uint32_t seen, floatx4 (&O)[D / 16]) {
  bf16x8 pa[2], va[2];
#pragma unroll
  for (int ks = 0; ks < 2; ++ks)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      pa[ks][j] = static_cast<__bf16>(P[8 * ks + j]);
      va[ks][j] = static_cast<__bf16>((seen >> (8 * ks + j)) & 1 ? 1.f : 0.f);
    }
#pragma unroll
  for (int jd = 0; jd < D / 16; ++jd) {
    floatx4 hit = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const intx2 v = read_v<D>(vb, r0 + 16 * gq + 8 * ks, jd, n);
      const uint32_t b0 = nan_codes(v[0]), b1 = nan_codes(v[1]);
      // a NaN byte's mask, and 0x38 (1.0) in its place
      const intx2 clean = {(int)(v[0] & ~(b0 | (b0 - (b0 >> 7)))), (int)(v[1] & ~(b1 | (b1 - (b1 >> 7))))};
      const intx2 one = {(int)((b0 >> 7) * 0x38u), (int)((b1 >> 7) * 0x38u)};
      O[jd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa[ks], to_bf16(clean[0], clean[1], 1.f), O[jd], 0, 0, 0);
      hit = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[ks], to_bf16(one[0], one[1], 1.f), hit, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) O[jd][i] = hit[i] > 0.f ? __uint_as_float(0x7fc00000u) : O[jd][i];
  }
}

// log2-sum-exp of row n of a row tile over its nsp chunks, the lane groups
// taking the chunks in turn (+inf for padding rows: their probabilities are 0).
__device__ __forceinline__ void join(float& m, float& z, float m2, float z2) {
  const float M = fmaxf(m, m2), r = M == kNegInf ? 0.f : M;
  // (a sum of 0 belongs to a chunk in which the row sees nothing; NaN passes)
  z = (z != 0.f ? z * fast_exp2(m - r) : 0.f) + (z2 != 0.f ? z2 * fast_exp2(m2 - r) : 0.f);
  m = M;
}
__device__ __forceinline__ float tile_lse(const QArgs& a, int tile, bool real, int nsp, int n, int gq) {
  const float2* st = a.stats + (size_t)tile * a.splits * 16 + n;
  float M = kNegInf, Z = 0.f;
  for (int s = gq; s < nsp; s += 4) {
    const float2 v = st[(size_t)s * 16];
    join(M, Z, v.x, v.y);
  }
  join(M, Z, lane_xor16(M), lane_xor16(Z));
  join(M, Z, lane_xor32(M), lane_xor32(Z));
  return real ? M + __log2f(Z) : __builtin_huge_valf();
}

// Sums of a block's probabilities over the 16 rows (lanes n) of a tile, token
// `lane` of the block into dst[lane]: each step a lane keeps half of its values,
// chosen by one bit of n, and adds its partner's copy of that half.
__device__ __forceinline__ void rows_to_lds(const float (&p)[16], float* dst, int lane) {
  const bool h8 = lane & 8, h4 = lane & 4, h2 = lane & 2, h1 = lane & 1;
  float a8[8], a4[4], a2[2];
#pragma unroll
  for (int k = 0; k < 8; ++k) a8[k] = (h8 ? p[8 + k] : p[k]) + lane_xor8(h8 ? p[k] : p[8 + k]);
#pragma unroll
  for (int k = 0; k < 4; ++k) a4[k] = (h4 ? a8[4 + k] : a8[k]) + lane_mirror8(h4 ? a8[k] : a8[4 + k]);
#pragma unroll
  for (int k = 0; k < 2; ++k) a2[k] = (h2 ? a4[2 + k] : a4[k]) + lane_xor2(h2 ? a4[k] : a4[2 + k]);
  dst[lane] = (h1 ? a2[1] : a2[0]) + lane_xor1(h1 ? a2[0] : a2[1]);
}

// -------------------------------------------------------- partial kernel --
template <int D, int RT>
struct Shape {
  static constexpr int TW = RT <= 2 ? 2 : 1;  // waves sharing a row tile's tokens
  static constexpr int kThreads = RT * TW * 64;
  static constexpr int ST = kQStageBytes / D, NB = ST / 64 / TW;  // tokens of a stage, blocks of it per wave
  static constexpr int kStage = 2 * kQStageBytes + 2 * ST;        // K codes, V codes, their exponents
};

// A stage's codes and exponents into LDS.  Rows past the chunk repeat its last
// one; exponents are read in groups of four rows, which never leave a block of
// 32 (capacities and pages are whole blocks).
template <int D, bool WITH_V>
__device__ __forceinline__ void load_stage(const QArgs& a, const Rows& v, int t0, int c1, char* s) {
  constexpr int ST = kQStageBytes / D;
  for (int i = threadIdx.x; i < kQStageBytes / 16; i += (int)blockDim.x) {
    int row, chunk;
    piece<D, true>(i, row, chunk);
    *reinterpret_cast<uint4*>(s + 16 * i) =
        *reinterpret_cast<const uint4*>(a.c.kc + row_index(v, min(t0 + row, c1 - 1)) * D + 16 * chunk);
    if constexpr (WITH_V) {
      piece<D, false>(i, row, chunk);
      *reinterpret_cast<uint4*>(s + kQStageBytes + 16 * i) =
          *reinterpret_cast<const uint4*>(a.c.vc + row_index(v, min(t0 + row, c1 - 1)) * D + 16 * chunk);
    }
  }
  for (int i = threadIdx.x; i < ST / 4; i += (int)blockDim.x) {
    const int64_t at = row_index(v, min(t0 + 4 * i, (c1 - 1) & ~3));
    *reinterpret_cast<uint32_t*>(s + 2 * kQStageBytes + 4 * i) = *reinterpret_cast<const uint32_t*>(a.c.ke + at);
    if constexpr (WITH_V)
      *reinterpret_cast<uint32_t*>(s + 2 * kQStageBytes + ST + 4 * i) = *reinterpret_cast<const uint32_t*>(a.c.ve + at);
  }
}

template <int D, int RT>
__global__ void __launch_bounds__((Shape<D, RT>::kThreads)) q8_part_kernel(QArgs a) {
  typedef Shape<D, RT> S_;
  constexpr int DPL = D / 16, TW = S_::TW, ST = S_::ST, NB = S_::NB;
  __shared__ int32_t s_pages[kPageSlots];
  __shared__ __align__(256) char s_stage[S_::kStage];

  Unit u;
  if (!decode_unit(a, u)) return;
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rows rows = rows_setup(a, u, s_pages);
  const int nst = (u.c1 - u.c0 + ST - 1) / ST;

  const int rt = w / TW, tw = w % TW, gt = u.rg * RT + rt;  // row tile of the KV head
  const bool live = gt < a.RTT;
  const int row = gt * 16 + n;
  const int lim = row < a.R ? min(u.c1 - 1, u.ctx + row_t(a, row)) : -1;  // last token the lane's row sees
  const int vis_all = min(u.c1 - 1, u.ctx);                               // row 0 sees the least
  Query<D> q;
  load_query<D>(a, u.b, u.g, row, gq, q);
  float ref = kNegInf, z = 0.f;
  floatx4 O[DPL];
#pragma unroll
  for (int jd = 0; jd < DPL; ++jd) O[jd] = floatx4{0.f, 0.f, 0.f, 0.f};

  for (int s = 0; s < nst; ++s) {
    __syncthreads();
    load_stage<D, true>(a, rows, u.c0 + s * ST, u.c1, s_stage);
    __syncthreads();
    for (int x = 0; x < NB; ++x) {
      const int r0 = (tw * NB + x) * 64, tb = u.c0 + s * ST + r0;
      if (tb >= u.c1 || !live) break;
      const char *kb = s_stage, *vb = s_stage + kQStageBytes, *eb = s_stage + 2 * kQStageBytes;
      const uint32_t ke = *reinterpret_cast<const uint32_t*>(eb + r0 + 4 * n);
      const uint4 ve4 = *reinterpret_cast<const uint4*>(eb + ST + r0 + 16 * gq);
      const uint32_t ve[4] = {ve4.x, ve4.y, ve4.z, ve4.w};
      floatx4 S[4];
      scores<D>(kb, ke, r0, n, gq, q, S);
      const bool tail = tb + 63 > vis_all;
      uint32_t seen = 0xffffu;
      if (tail) {
        const int off = lim - tb - 16 * gq;  // the lane's token j is visible iff j <= off
        seen = off < 0 ? 0u : off >= 15 ? 0xffffu : (2u << off) - 1u;
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((seen >> (4 * i + tt)) & 1)) S[tt][i] = kNegInf;
      }
      float mx = kNegInf;
#pragma unroll
      for (int tt = 0; tt < 4; ++tt) mx = fmaxf(fmaxf(mx, fmaxf(S[tt][0], S[tt][1])), fmaxf(S[tt][2], S[tt][3]));
      mx = rows4_max(mx) * a.sl2;
      if (__any(mx > ref + kRefSlack)) {  // the first block, and seldom after it
        const float nm = fmaxf(ref, mx);
        const float al = ref == kNegInf ? 0.f : fast_exp2(ref - nm);
        z *= al;
        ref = nm;
        floatx4 f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = __shfl(al, 4 * gq + i, 64);
#pragma unroll
        for (int jd = 0; jd < DPL; ++jd) O[jd] = O[jd] * f;
      }
      const float r = ref == kNegInf ? 0.f : ref;  // no visible token yet: P = 0
      float P[16];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
          const float p = fast_exp2(fmaf(S[tt][i], a.sl2, -r));
          z += p;
          P[4 * i + tt] = p * q8_unit((ve[i] >> (8 * tt)) & 0xffu);
        }
      if (!tail) {
        weigh<D>(vb, r0, n, gq, P, O);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (!((seen >> j) & 1)) P[j] = 0.f;  // (an unwritten row's exponent may be anything)
        weigh_masked<D>(vb, r0, n, gq, P, seen, O);
      }
    }
  }

  z = rows4_sum(z);
  if constexpr (TW > 1) {  // the second token wave's sums join the first's
    floatx4* xo = reinterpret_cast<floatx4*>(s_stage) + rt * (DPL * 64 + 64);
    static_assert(RT * (DPL * 64 + 64) * 16 <= S_::kStage, "the exchange fits the stage");
    __syncthreads();
    if (tw == 1) {
#pragma unroll
      for (int jd = 0; jd < DPL; ++jd) xo[jd * 64 + lane] = O[jd];
      xo[DPL * 64 + lane] = floatx4{ref, z, 0.f, 0.f};
    }
    __syncthreads();
    if (tw == 1) return;
    const floatx4 o = xo[DPL * 64 + lane];
    const float M = fmaxf(ref, o[0]), r = M == kNegInf ? 0.f : M;
    const float f0 = z != 0.f ? fast_exp2(ref - r) : 0.f, f1 = o[1] != 0.f ? fast_exp2(o[0] - r) : 0.f;
    z = z * f0 + o[1] * f1;
    ref = M;
    floatx4 g0, g1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g0[i] = __shfl(f0, 4 * gq + i, 64);
      g1[i] = __shfl(f1, 4 * gq + i, 64);
    }
#pragma unroll
    for (int jd = 0; jd < DPL; ++jd) O[jd] = O[jd] * g0 + xo[jd * 64 + lane] * g1;
  }
  if (!live) return;
  const size_t rec = (size_t)(u.bg * a.RTT + gt) * a.splits + u.split;
  if (gq == 0) a.stats[rec * 16 + n] = make_float2(ref, z);
  // position DPL n + jd of a stored row holds column 16 jd + n
  float* op = a.opart + rec * 16 * D;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int h = 0; h < DPL / 4; ++h)
      *reinterpret_cast<float4*>(op + (4 * gq + i) * D + DPL * n + 4 * h) =
          make_float4(O[4 * h][i], O[4 * h + 1][i], O[4 * h + 2][i], O[4 * h + 3][i]);
}

// ----------------------------------------------------------- mass kernel --
// The partial kernel's units again, every row's log-sum-exp known.
template <int D, int RT>
__global__ void __launch_bounds__((Shape<D, RT>::kThreads)) q8_mass_kernel(QArgs a) {
  typedef Shape<D, RT> S_;
  constexpr int TW = S_::TW, ST = S_::ST, NB = S_::NB;
  __shared__ int32_t s_pages[kPageSlots];
  __shared__ __align__(256) char s_stage[S_::kStage];
  __shared__ float s_sum[RT][ST];

  Unit u;
  if (!decode_unit(a, u)) return;
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Rows rows = rows_setup(a, u, s_pages);
  const int nst = (u.c1 - u.c0 + ST - 1) / ST;
  const int rt = w / TW, tw = w % TW, gt = u.rg * RT + rt;
  const int row = gt * 16 + n;
  const int lim = row < a.R ? min(u.c1 - 1, u.ctx + row_t(a, row)) : -1;
  Query<D> q;
  load_query<D>(a, u.b, u.g, row, gq, q);
  const float lse = tile_lse(a, u.bg * a.RTT + min(gt, a.RTT - 1), row < a.R, (u.N + a.chunk - 1) / a.chunk, n, gq);
  float* mp = a.mpart + ((size_t)u.bg * a.RG + u.rg) * a.c.n_cap;
  for (int s = 0; s < nst; ++s) {
    __syncthreads();
    load_stage<D, false>(a, rows, u.c0 + s * ST, u.c1, s_stage);
    __syncthreads();
    for (int x = 0; x < NB; ++x) {
      const int r0 = (tw * NB + x) * 64, tb = u.c0 + s * ST + r0;
      if (tb >= u.c1) break;
      const uint32_t ke = *reinterpret_cast<const uint32_t*>(s_stage + 2 * kQStageBytes + r0 + 4 * n);
      floatx4 S[4];
      scores<D>(s_stage, ke, r0, n, gq, q, S);
      const int off = lim - tb - 16 * gq;
      float P[16];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
          P[4 * i + tt] = 4 * i + tt <= off ? fast_exp2(fmaf(S[tt][i], a.sl2, -lse)) : 0.f;
      rows_to_lds(P, &s_sum[rt][r0], lane);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < ST; i += (int)blockDim.x) {
      const int t = u.c0 + s * ST + i;
      if (t < u.c1) {
        float sum = s_sum[0][i];
#pragma unroll
        for (int k = 1; k < RT; ++k) sum += s_sum[k][i];
        mp[t] = sum;
      }
    }
  }
}

// --------------------------------------------------------- finish kernel --
// One wave per row of O: the sum over its chunks of the partials weighted by
// exp2(chunk maximum - row maximum) / row sum, and the row's log-sum-exp.
template <int D>
__device__ __forceinline__ void combine_row(const QArgs& a, int64_t id) {
  constexpr int LPR = D / 4, SG = 64 / LPR;  // lanes of a row, chunks side by side
  if (id >= (int64_t)a.B * a.Hkv * a.R) return;
  const int lane = threadIdx.x & 63, sg = lane / LPR, col = lane % LPR;
  const int bg = (int)(id / a.R), row = (int)(id - (int64_t)bg * a.R);
  const int b = bg / a.Hkv, g = bg - b * a.Hkv;
  const int nsp = (seq_ctx(a, b, false) + a.T + a.chunk - 1) / a.chunk;
  const size_t rec = ((size_t)bg * a.RTT + row / 16) * a.splits * 16 + row % 16;
  const float2* st = a.stats + rec;
  const float* op = a.opart + rec * D + 4 * col;
  float M = kNegInf, Z = 0.f;
  for (int s = lane; s < nsp; s += 64) join(M, Z, st[(size_t)s * 16].x, st[(size_t)s * 16].y);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) join(M, Z, __shfl_xor(M, o, 64), __shfl_xor(Z, o, 64));
  const float r = M == kNegInf ? 0.f : M, inv = 1.f / Z;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = sg; s < nsp; s += SG) {
    const float2 v = st[(size_t)s * 16];
    const float wt = v.y != 0.f ? fast_exp2(v.x - r) * inv : 0.f;
    const float4 p = *reinterpret_cast<const float4*>(op + (size_t)s * 16 * D);
    if (v.y != 0.f) {
      acc[0] = fmaf(wt, p.x, acc[0]);
      acc[1] = fmaf(wt, p.y, acc[1]);
      acc[2] = fmaf(wt, p.z, acc[2]);
      acc[3] = fmaf(wt, p.w, acc[3]);
    }
  }
#pragma unroll
  for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] += __shfl_xor(acc[k], o, 64);
  const int t = row_t(a, row), h = g * a.G + row - t * a.G;
  if (sg == 0) {
    constexpr int DPL = D / 16;
    uint16_t* o = a.out + (((size_t)b * a.T + t) * a.Hq + h) * D;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int at = 4 * col + k;
      o[16 * (at % DPL) + at / DPL] = f32_to_bf16(acc[k]);
    }
  }
  if (a.lse && lane == 0) a.lse[((size_t)b * a.Hq + h) * a.T + t] = (M + __log2f(Z)) * kLn2;
}

// The mass of every cache row: the sum of its KV heads' and row groups'
// partials in order (0 past the sequence).
__device__ __forceinline__ void sum_mass(const QArgs& a, int id) {
  const int P = a.Hkv * a.RG;
  const int b = id / a.mass_per;
  const int64_t t0 = (int64_t)(id - b * a.mass_per) * a.mass_rows;
  const int N = seq_ctx(a, b, false) + a.T;
  const float* mp = a.mpart + (size_t)b * P * a.c.n_cap;
  float* mass = a.mass + (size_t)b * a.c.n_cap;
  for (int64_t t = t0 + threadIdx.x; t < min(t0 + a.mass_rows, a.c.n_cap); t += kFinThreads) {
    float sum = 0.f;
    if (t < N)
      for (int p = 0; p < P; ++p) sum += mp[(size_t)p * a.c.n_cap + t];
    mass[t] = sum;
  }
}

template <int D>
__global__ void __launch_bounds__(kFinThreads) q8_finish_kernel(QArgs a) {
  const int id = blockIdx.x;
  if (id < a.mass_wgs) sum_mass(a, id);
  else combine_row<D>(a, (int64_t)(id - a.mass_wgs) * kFinWaves + (threadIdx.x >> 6));
}

// ------------------------------------------------------------------ host --
typedef void (*QKernel)(QArgs);
struct QKernels {
  QKernel part, mass, finish;
  int threads;
};

template <int D>
QKernels pick(int RT) {
#define PVLM_Q8_RT(n) \
  case n: return {q8_part_kernel<D, n>, q8_mass_kernel<D, n>, q8_finish_kernel<D>, Shape<D, n>::kThreads};
  switch (RT) {
    PVLM_Q8_RT(1)
    PVLM_Q8_RT(2)
    PVLM_Q8_RT(3)
    PVLM_Q8_RT(4)
    PVLM_Q8_RT(5)
    PVLM_Q8_RT(6)
    PVLM_Q8_RT(7)
    PVLM_Q8_RT(8)
    default:
    PVLM_Q8_RT(9)
  }
#undef PVLM_Q8_RT
}

pvlm_status verify_q8_run(int B, int T, int Hq, int Hkv, int D, int64_t max_ctx, float scale, const void* q,
                          const Q8Cache& c, const int32_t* ctx_len, void* out, float* mass, float* lse, void* ws,
                          size_t ws_bytes, int32_t* status, hipStream_t stream) {
  if (!q || !ctx_len || !out) return PVLM_ERR_NULL;
  if (!(scale > 0.f) || !std::isfinite(scale)) return PVLM_ERR_SHAPE;
  pvlm_status st = check_verify_q8(B, T, Hq, Hkv, D, c.n_cap, max_ctx);
  if (st != PVLM_OK) return st;
  st = check_q8(c.kc, c.ke, c.vc, c.ve, c.n_cap);
  if (st != PVLM_OK) return st;
  if ((uintptr_t)q % 16 != 0) return PVLM_ERR_UNSUPPORTED;
  DeviceInfo di;
  st = device_info(&di, stream);
  if (st != PVLM_OK) return st;
  QSplit p;
  split_verify_q8(B, T, Hq, Hkv, D, c.n_cap, max_ctx, di.cus, &p);
  if (!ws || ws_bytes < p.bytes || (uintptr_t)ws % 16 != 0) return PVLM_ERR_WORKSPACE;
  char* wsb = static_cast<char*>(ws);
  QArgs a;
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
  a.max_ctx = (int)max_ctx;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.units = B * Hkv * p.RG * p.splits;
  a.sl2 = scale * kLog2e;
  a.mpart = reinterpret_cast<float*>(wsb + p.off_mpart);
  a.stats = reinterpret_cast<float2*>(wsb + p.off_stats);
  a.opart = reinterpret_cast<float*>(wsb + p.off_opart);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.mass = mass;
  a.status = status;
  a.mass_rows = (int)mass_rows(B, c.n_cap);
  a.mass_per = (int)mass_workgroups(c.n_cap, a.mass_rows);
  a.mass_wgs = mass ? B * a.mass_per : 0;
  const QKernels k = D == 128 ? pick<128>(p.RT) : pick<64>(p.RT);
  const dim3 grid((a.units + 7) / 8 * 8);
  hipLaunchKernelGGL(k.part, grid, dim3(k.threads), 0, stream, a);
  PVLM_LAUNCHED();
  if (mass) {
    hipLaunchKernelGGL(k.mass, grid, dim3(k.threads), 0, stream, a);
    PVLM_LAUNCHED();
  }
  const int combine_wgs = (int)(((int64_t)B * Hkv * p.R + kFinWaves - 1) / kFinWaves);
  hipLaunchKernelGGL(k.finish, dim3(a.mass_wgs + combine_wgs), dim3(kFinThreads), 0, stream, a);
  PVLM_LAUNCHED();
  return PVLM_OK;
}

Q8Cache view(const uint8_t* kc, const uint8_t* ke, const uint8_t* vc, const uint8_t* ve, int64_t n_cap) {
  return Q8Cache{const_cast<uint8_t*>(kc), const_cast<uint8_t*>(ke), const_cast<uint8_t*>(vc),
                 const_cast<uint8_t*>(ve), nullptr, 0, n_cap, 0, 0};
}

}  // namespace
}  // namespace pvlm

using namespace pvlm;

extern "C" size_t pvlm_verify_attn_q8_workspace_size(int B, int T, int Hq, int Hkv, int D, int64_t n_cap,
                                                     int64_t max_ctx) {
  DeviceInfo di;
  if (check_verify_q8(B, T, Hq, Hkv, D, n_cap, max_ctx) != PVLM_OK || device_info(&di) != PVLM_OK) return 0;
  QSplit p;
  split_verify_q8(B, T, Hq, Hkv, D, n_cap, max_ctx, di.cus, &p);
  return p.bytes;
}

extern "C" pvlm_status pvlm_verify_attn_q8(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int64_t n_cap,
                                           int64_t max_ctx, float scale, const void* q, const uint8_t* k_codes,
                                           const uint8_t* k_exps, const uint8_t* v_codes, const uint8_t* v_exps,
                                           const int32_t* ctx_len, void* out, float* mass, float* lse, void* ws,
                                           size_t ws_bytes, int32_t* status, hipStream_t stream) {
  if (dt != PVLM_BF16) return PVLM_ERR_UNSUPPORTED;
  return verify_q8_run(B, T, Hq, Hkv, D, max_ctx, scale, q, view(k_codes, k_exps, v_codes, v_exps, n_cap), ctx_len,
                       out, mass, lse, ws, ws_bytes, status, stream);
}

extern "C" pvlm_status pvlm_verify_attn_q8_paged(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int page_size,
                                                 int max_pages, int64_t n_pages, int64_t max_ctx, float scale,
                                                 const void* q, const uint8_t* k_codes, const uint8_t* k_exps,
                                                 const uint8_t* v_codes, const uint8_t* v_exps,
                                                 const int32_t* page_table, const int32_t* ctx_len, void* out,
                                                 float* mass, float* lse, void* ws, size_t ws_bytes,
                                                 int32_t* status, hipStream_t stream) {
  Q8Cache c = view(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  if (dt != PVLM_BF16) return PVLM_ERR_UNSUPPORTED;
  return verify_q8_run(B, T, Hq, Hkv, D, max_ctx, scale, q, c, ctx_len, out, mass, lse, ws, ws_bytes, status, stream);
}

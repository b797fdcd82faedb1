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
// Launches, all on the caller's stream: partial; combine, unless the shares are whole
// groups; and the mass.
//
// What bounds it.  A row is 68 bytes (D = 128) where bf16 has 256, so the bytes pass in a
// fraction of the time that both products' matrix instructions, the conversions and
// the exponentials take:
//  * 16 sequences of one row, 28 / 4 heads, 2048 to 16384 tokens (89 MB): partial 22 us,
//    4.0 TB/s; combine 4.
//  * 9 rows of 64 / 8 heads over 12800 tokens (14 MB): partial 20.5, combine 5, mass 11, of
//    which 3 to 5 each are the start, the joins and the end.
//  * 17 rows of 64 / 8 heads over 132096 tokens (145 MB): partial 110 (matrix instructions
//    39 % of the cycles, vector ones 57), mass 75 (25 and 65), combine 6.
// Vector and matrix instructions of different waves run side by side, so what is left of
// a SIMD's time is where its two waves want the same pipe.
#include <type_traits>

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
  const int32_t* n_new;  // rows of q that a sequence has, or NULL: T each
  int Hq, G, R;
  unsigned g_magic;  // row / G == row * g_magic >> 20 for row < 640 (2^20 / G + 1; G <= 640)
  int RTT;
  float sl2;         // scale * log2(e)
  float4* stats;     // [record][row tile][16] of a row: log2-domain reference, sum, sum of the rounded, unused
  uint32_t* nan;     // [record] the values hold a NaN that not every row sees
  float2* rows;      // [B][Hkv][R] maximum and inverse sum, for the mass
  float* opart;      // [record][row tile][16][D] sums of P . V relative to that reference
  uint16_t* out;
  float* lse;
  float* mass;
  int32_t* status;
  int per_share, MG, GW, chunk, chunks;
};

// ------------------------------------------------------------ the shares --
// A wave's way to its share of the tokens, from the lengths on the device (the
// shares themselves: q8_plan.h).
typedef const __attribute__((address_space(4))) int32_t* ConstInts;  // (uniform loads go through the scalar cache)
__device__ __forceinline__ int uniform_load(const int32_t* p, int64_t i) { return ((ConstInts)(uintptr_t)p)[i]; }

// The rows of q that sequence b has, and the tokens that they see: those behind them in
// q and in the cache may hold anything.  The shares are counted as if there were T.
__device__ __forceinline__ int rows_of(const Q4Args& a, int b) {
  if (!a.n_new) return a.T;
  const int n = __builtin_amdgcn_readfirstlane(uniform_load(a.n_new, b));
  return n < 0 ? 0 : n < a.T ? n : a.T;
}
__device__ __forceinline__ int tokens_of(int ctx, int rows) { return rows ? ctx + rows : 0; }

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
  __device__ __forceinline__ explicit Wave(const int32_t* lengths) : ctx_len(lengths), lane(threadIdx.x & 63) {
    asm volatile("" : "+v"(lane));  // (its addresses, made before a loop over pieces, would spill)
  }
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
  __device__ __forceinline__ bool first(const QShape& a, const int32_t* ctx_len, int share) {
    return begin(a, q8_find<true>(a, Wave(ctx_len), share, 0), share);
  }
  // All of group `group`, where a share is a group.
  __device__ __forceinline__ void whole(const QShape& a, const int32_t* ctx_len, int group) {
    b = group / a.Hkv;
    g = group - b * a.Hkv;
    rg = before = c0 = 0;
    align = 1;
    ctx = __builtin_amdgcn_readfirstlane(clamp_ctx(a, uniform_load(ctx_len, b)));
    left = per = units_of(a, ctx);
    set(a);
  }
  // false where the share ends
  __device__ __forceinline__ bool next(const QShape& a, const int32_t* ctx_len) {
    return advance(a, [&](int x) { return __builtin_amdgcn_readfirstlane(clamp_ctx(a, uniform_load(ctx_len, x))); });
  }
};

// Where the rows of one (sequence, KV head) lie: row t of a paged cache in page
// table[t >> shift], of a padded one behind `first` (its table is any word: the
// page's number then counts for nothing).  An entry outside the pool sets bad and is
// clamped into it.
struct Rows {
  const int32_t* table;
  int64_t first, page_rows;
  uint32_t n_pages;
  int shift, mask;
  __device__ __forceinline__ Rows(const Q4Cache& c, const int32_t* any, int Hkv, int b, int g) {
    const bool paged = c.table != nullptr;
    table = paged ? c.table + (int64_t)b * c.max_pages : any;
    shift = paged ? c.shift : 31;
    mask = paged ? (1 << c.shift) - 1 : 0x7fffffff;
    first = paged ? (int64_t)g << c.shift : ((int64_t)b * Hkv + g) * c.n_cap;
    page_rows = paged ? (int64_t)Hkv << c.shift : 0;
    n_pages = paged ? (uint32_t)c.n_pages : 0xffffffffu;
  }
  // The page that row t lies in, and the row's number of the cache's.  (Apart, so that a
  // loop can have the entry before it is wanted.)
  __device__ __forceinline__ int entry(int t) const { return uniform_load(table, t >> shift); }
  __device__ __forceinline__ int64_t at(int t, int entry, bool& bad) const {
    uint32_t page = (uint32_t)entry;
    if (page >= n_pages) {
      bad |= n_pages != 0xffffffffu;
      page = entry < 0 ? 0 : n_pages - 1;
    }
    return (int64_t)page * page_rows + first + (t & mask);
  }
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
// The factor of sums that go to a reference -x above their own.  They reach 2^kRefSlack and
// more, so one under 2^-126 still counts, and the instruction's would be 0 there: the
// square of half the way is subnormal, off by 2^-150 at most.  (Otherwise parts whose
// probabilities are 2^-102 of the row's largest are lost.)
__device__ __forceinline__ float shift_exp2(float x) {
  const float h = fast_exp2(0.5f * x);
  return h * h;
}
__device__ __forceinline__ int row_t(const Q4Args& a, int row) { return (int)((unsigned)row * a.g_magic >> 20); }

// Eight codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8 to_bf16(uint32_t w, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, unit, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A lane's part of a 16-token tile of K or V: with n = lane & 15 and gq = lane >> 4,
// D / 4 consecutive values of row n from value (D / 4) gq on, D / 32 words of eight
// codes, within one block of 32.  A wave's loads of a tile are then one run of
// memory, and word ks is an operand of the 16x16x32 product over values
// (D / 4) gq + 8 ks + j: the order of the sum over d is free, so long as the queries
// have it too.
// Its exponent is a byte of the word that is loaded (a byte load's result the compiler
// masks where it arrives, and so waits for it there).
template <int D>
struct Codes {
  uint32_t w[D / 32];
  uint32_t e;
};
template <int D>
struct LaneOf {  // a lane's place in a tile
  uint32_t codes, exps, shift;  // (unsigned: an address is then a scalar base and this)
  __device__ __forceinline__ LaneOf(int n, int gq)
      : codes(n * (D / 2) + gq * (D / 8)),
        exps(n * (D / 32) & ~3),
        shift(8 * ((n * (D / 32) + gq * (D / 32) / 4) & 3)) {}
  __device__ __forceinline__ uint32_t exponent(uint32_t e) const { return __builtin_amdgcn_ubfe(e, shift, 8); }
  __device__ __forceinline__ float unit(uint32_t e) const { return __uint_as_float(exponent(e) << 23); }
};
// A pointer that the wave's lanes have in common, in scalar registers.  (The compiler adds
// the lane's offset in the vector unit all the same, a 64-bit addition for each load,
// but right before it: left to itself it adds it ahead of the loop, and keeps 64 bits of
// every address a lane.)
typedef const __attribute__((address_space(1))) uint8_t* Global;
__device__ __forceinline__ Global scalar(const uint8_t* p) {
  const uint64_t u = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)u), hi = __builtin_amdgcn_readfirstlane((int)(u >> 32));
  return (Global)((uint64_t)hi << 32 | lo);
}
template <int D>
__device__ __forceinline__ void load_codes(const uint8_t* codes, const uint8_t* exps, int64_t row0, const LaneOf<D>& at,
                                           Codes<D>& x) {
  typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
  const words v = *(const __attribute__((address_space(1))) words*)(scalar(codes + row0 * (D / 2)) + at.codes);
#pragma unroll
  for (int i = 0; i < D / 32; ++i) x.w[i] = v[i];
  x.e = *(const __attribute__((address_space(1))) uint32_t*)(scalar(exps + row0 * (D / 32)) + at.exps);
}

template <int D>
struct Query {
  bf16x8 s[D / 32];
};
// (In place of a row that the sequence does not have, its last one: what q holds there
// reaches nothing, not even the references, which a wave's rows move together.)
template <int D>
__device__ __forceinline__ void load_query(const Q4Args& a, int b, int g, int row, int gq, int n_rows, Query<D>& q) {
  const int r = min(row, a.R - 1), tr = row_t(a, r), h = g * a.G + r - tr * a.G, t = min(tr, max(n_rows, 1) - 1);
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
// Rows lie 32 bytes more than their length apart, and rows whose number has bit 2 set
// hold every two 16-byte chunks in the other order: a transposed read (the same 32
// bytes of eight rows at a time, 256 bytes) and a write (the same chunk of eight rows at
// a time, 128 bytes) then fall on distinct banks, and every address is the lane's first
// (of the even chunks or the odd ones) and a constant.  (In one order the writes had
// conflicts, 13 % of the kernel's cycles: 9 rows over 12800 tokens 21.9 us for 21.2.)
template <int D>
struct Lay {
  static constexpr int kRow = 2 * D + 32, kHalf = 16 * kRow, kUnit = 2 * kHalf;
  static __device__ __forceinline__ uint32_t swap(int row) { return (row & 4) * 4; }
};
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s4* lds_s4;

// `put`, `odd`: LDS addresses of the lane's chunk 0 and, less 16, 1 in rows 0 .. 15 of the
// wave's unit.
template <int D>
__device__ __forceinline__ void put_values(uint32_t put, uint32_t odd, int tt, const Codes<D>& x, float unit) {
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
    *(__attribute__((address_space(3))) bf16x8*)((c % 2 ? odd : put) + tt * Lay<D>::kHalf + 16 * c) = to_bf16(x.w[c], unit);
}

// O += P . V over the unit in LDS; P holds tokens 4 gq + {0..3, 16..19}, `get` is the
// lane's first address: of sixteen lanes each takes 8 bytes of row 4 gq + n / 4, and
// receives column n of the four rows.  AHEAD operands are under way while the matrix
// instructions of earlier ones run (the compiler, left to itself, waits for each alone).
template <int D, int TPW, int AHEAD>
__device__ __forceinline__ void weigh(uint32_t get, const bf16x8 (&P)[TPW], floatx4 (&O)[TPW][D / 16]) {
  constexpr int N = D / 16;
  s4 lo[AHEAD], hi[AHEAD];
  auto read = [&](int j) {
    lo[j % AHEAD] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(get + 32 * j));
    hi[j % AHEAD] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(get + 32 * j + Lay<D>::kHalf));
  };
#pragma unroll
  for (int j = 0; j < AHEAD - 1; ++j) read(j);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (j + AHEAD - 1 < N) read(j + AHEAD - 1);
    __builtin_amdgcn_sched_barrier(0);
    const s8 both = __builtin_shufflevector(lo[j % AHEAD], hi[j % AHEAD], 0, 1, 2, 3, 4, 5, 6, 7);
    const bf16x8 v = __builtin_bit_cast(bf16x8, both);
#pragma unroll
    for (int x = 0; x < TPW; ++x) O[x][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P[x], v, O[x][j], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// ------------------------------------------------------------- a result --
// C columns of a row of the result, from the sums relative to its reference m: positions
// C part .. of a stored row, of which position (D / 16) n + jd is column 16 jd + n.
// `look`: the values hold a NaN that not every row sees.  Those past the context that
// this row sees counted as 0 and are looked for here.  A row that the sequence does not
// have is 0, its log-sum-exp -inf, and it has no part in the mass.
template <int D, int C>
__device__ __forceinline__ void put_row(const Q4Args& a, int b, int g, int row, int ctx, const Rows& rows, int part,
                                        const float (&o)[C], float m, float z, float zt, bool look) {
  constexpr int DPL = D / 16;
  const int t = row_t(a, row), head = g * a.G + row - t * a.G;
  const float inv = 1.f / zt;
  const bool real = t < rows_of(a, b);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int pos = C * part + c, col = 16 * (pos % DPL) + pos / DPL;
    float y = real ? o[c] * inv : 0.f;
    if (look && real) {
      for (int j = ctx + 1; j <= ctx + t; ++j) {
        bool flagged_before = false;  // by the loads of the row
        const int64_t r = rows.at(j, rows.table[j >> rows.shift], flagged_before);
        if (a.c.ve[r * (D / 32) + col / 32] == 255) y = __uint_as_float(0x7fc00000u);
      }
    }
    a.out[(((size_t)b * a.T + t) * a.Hq + head) * D + col] = f32_to_bf16(y);
  }
  if (part == 0) {
    if (a.lse) a.lse[((size_t)b * a.Hq + head) * a.T + t] = real ? (m + __log2f(z)) * kLn2 : kNegInf;
    if (a.mass) a.rows[((size_t)b * a.Hkv + g) * a.R + row] = real ? make_float2(m, 1.f / z) : make_float2(-kNegInf, 0.f);
  }
}

// -------------------------------------------------------- partial kernel --
// A workgroup's eight waves hold the same set of row tiles, TPW of them, and take its
// tokens in turn, a unit of 32 at a time, with the next unit's loads on their way.
constexpr int kAhead = 3;  // operands of P . V read ahead
// A lane's sum of this many units goes to its place in LDS: beside one large
// probability a running sum of all of a long share would round small ones away.
constexpr int kSumUnits = 16;

// SINGLE: every group is one share, and the workgroup writes the results.  (A kernel of
// its own: that path's registers cost the other one 7 %.)
template <int D, int TPW, bool SINGLE>
__global__ void __launch_bounds__(kQ4Waves * 64)
__attribute__((amdgpu_waves_per_eu(kQ4Waves / 4, kQ4Waves / 4))) q4_part_kernel(Q4Args a) {
  constexpr int DPL = D / 16, TW = kQ4Waves;
  extern __shared__ __align__(1024) char s_values[];  // [wave][32][D] bf16; then a tile's O, [wave][16][D] fp32
  __shared__ float s_ref[TW][16], s_z[TW][16], s_zt[TW][16];
  __shared__ uint32_t s_nan[TW];
  __shared__ float s_sum[SINGLE ? 1 : TW][TPW][64];  // (a single share's sums are short)

  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && w == 0)
    for (int b = threadIdx.x; b < a.B; b += 64)
      if (a.ctx_len[b] < 0 || a.ctx_len[b] > a.max_ctx || (a.n_new && (a.n_new[b] < 0 || a.n_new[b] > a.T)))
        dev_flag(a.status, PVLM_DEV_RANGE);
  // The sets of row tiles of a share read the same tokens at about the same time:
  // they are neighbours on one die (workgroup i runs on die i mod 8), whose L2 has
  // what the first of them read.
  const int wgs = gridDim.x, id = blockIdx.x, whole8 = wgs & ~7;
  const int place = id < whole8 ? (id & 7) * (whole8 >> 3) + (id >> 3) : id;
  const int share = place / a.per_share;
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_addr(s_values)) + w * Lay<D>::kUnit;

  const LaneOf<D> place_of(n, gq);
  const uint32_t put = lds + n * Lay<D>::kRow + gq * (D / 2) + Lay<D>::swap(n), odd = put - 2 * Lay<D>::swap(n);
  const uint32_t get = lds + (4 * gq + n / 4) * Lay<D>::kRow + (8 * (n & 3) ^ Lay<D>::swap(4 * gq));
  bool bad_page = false;
  for (int rg = place - share * a.per_share; rg * TPW < a.RTT; rg += a.per_share) {
    Piece p;
    if constexpr (SINGLE) p.whole(a, a.ctx_len, share);
    else if (!p.first(a, a.ctx_len, share)) break;
    do {
      const int tile0 = rg * TPW;  // of the KV head's
      const Rows rows(a.c, a.ctx_len, a.Hkv, p.b, p.g);
      const int n_rows = rows_of(a, p.b), end = min(p.c1, tokens_of(p.ctx, n_rows));  // (may be c0 or before it)
      Query<D> q[TPW];
      int lim[TPW];
      float ref[TPW], z[TPW];
      floatx4 O[TPW][DPL], zt[TPW];
      int first = tile0 * 16 + n;
      asm volatile("" : "+v"(first));  // (as the share's addresses)
#pragma unroll
      for (int x = 0; x < TPW; ++x) {
        const int row = first + 16 * x;
        load_query<D>(a, p.b, p.g, row, gq, n_rows, q[x]);
        lim[x] = row < a.R ? min(end - 1, p.ctx + row_t(a, row)) : -1;
        ref[x] = kNegInf;
        z[x] = 0.f;
        if constexpr (!SINGLE) s_sum[w][x][lane] = 0.f;
        zt[x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int jd = 0; jd < DPL; ++jd) O[x][jd] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
      uint32_t nan = 0;
      // The next unit (past the piece, its last one) and its page.
      Codes<D> kc[2], vc[2];
      int page;
      auto unit = [&](int t) { return min(t, (max(end, 1) - 1) & ~31); };
      auto load = [&](int t) {
        const int64_t row = rows.at(unit(t), page, bad_page);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) load_codes<D>(a.c.kc, a.c.ke, row + 16 * tt, place_of, kc[tt]);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) load_codes<D>(a.c.vc, a.c.ve, row + 16 * tt, place_of, vc[tt]);
        page = rows.entry(unit(t + 32 * TW));
      };
      // The unit of tokens t0 .. t0 + 31; TAIL: some row does not see all of them.
      auto block = [&](int t0, auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        if constexpr (TAIL) {
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            // rows past its tokens become zeros (their probabilities are 0, and 0 times what
            // an unwritten row holds may be NaN), and so do NaN of rows that not every query
            // row sees: the record's flag has the rows looked at that see them
            const int t = t0 + 16 * tt + n;
            const bool past = t >= end, hidden = t > p.ctx && place_of.exponent(vc[tt].e) == 255;
            if (hidden && !past) nan = 1;
            if (past || hidden) {
              vc[tt].e = 0;
#pragma unroll
              for (int c = 0; c < D / 32; ++c) vc[tt].w[c] = 0;
            }
          }
        }
        // (the values' conversion runs beside the matrix instructions of the scores)
        asm volatile("" ::: "memory");  // (the wave's LDS operations keep their order)
        put_values<D>(put, odd, 0, vc[0], place_of.unit(vc[0].e));
        put_values<D>(put, odd, 1, vc[1], place_of.unit(vc[1].e));
        floatx4 S[TPW][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float scale = place_of.unit(kc[j].e);
#pragma unroll
          for (int x = 0; x < TPW; ++x) S[x][j] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int ks = 0; ks < D / 32; ++ks) {
            const bf16x8 k = to_bf16(kc[j].w[ks], scale);
#pragma unroll
            for (int x = 0; x < TPW; ++x) S[x][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[x].s[ks], S[x][j], 0, 0, 0);
          }
        }
        asm volatile("" ::: "memory");
        if (t0 + 32 * TW < end) load(t0 + 32 * TW);
        if constexpr (TAIL) {
#pragma unroll
          for (int x = 0; x < TPW; ++x)
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (t0 + 16 * (j / 4) + 4 * gq + j % 4 > lim[x]) S[x][j / 4][j % 4] = kNegInf;
        }
        bf16x8 P[TPW];
#pragma unroll
        for (int x = 0; x < TPW; ++x) {
          float m = kNegInf;  // (the maximum that passes NaN on: the other one has every operand canonicalised first)
#pragma unroll
          for (int j = 0; j < 8; ++j) m = __builtin_elementwise_maximum(m, S[x][j / 4][j % 4]);
          m *= a.sl2;
          if (__any(m > ref[x] + kRefSlack)) {  // the first unit, and seldom after it
            const float nm = fmaxf(ref[x], rows4_maximum(m));
            const float al = ref[x] == kNegInf ? 0.f : shift_exp2(ref[x] - nm);
            z[x] *= al;
            if constexpr (!SINGLE) s_sum[w][x][lane] *= al;
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
          for (int j = 0; j < 8; ++j) {
            const float e = fast_exp2(fmaf(S[x][j / 4][j % 4], a.sl2, -r));
            sum += e;
            P[x][j] = static_cast<__bf16>(e);
          }
          z[x] += sum;
        }
        bf16x8 ones;
#pragma unroll
        for (int j = 0; j < 8; ++j) ones[j] = static_cast<__bf16>(1.f);
        weigh<D, TPW, kAhead>(get, P, O);
#pragma unroll
        for (int x = 0; x < TPW; ++x) zt[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P[x], ones, zt[x], 0, 0, 0);
        asm volatile("" ::: "memory");
      };
      // (two loops: in one, the compiler has every unit go through the tail's selections)
      int t = p.c0 + 32 * w;
      page = rows.entry(unit(t));
      if (t < end) load(t);
      for (int left = kSumUnits; t + 31 <= min(end - 1, p.ctx); t += 32 * TW) {
        block(t, std::false_type{});
        if (!SINGLE && --left == 0) {
          left = kSumUnits;
#pragma unroll
          for (int x = 0; x < TPW; ++x) s_sum[SINGLE ? 0 : w][x][lane] += z[x], z[x] = 0.f;
        }
      }
      for (; t < end; t += 32 * TW) block(t, std::true_type{});
      // The token waves' results joined: a tile at a time, through LDS (position
      // DPL n + jd of a row holds column 16 jd + n).
      const int rec = p.group(a) + share;
      int tid = threadIdx.x;
      asm volatile("" : "+v"(tid));  // (addresses of the results, made before the loop, would spill)
      const bool any = __any(nan);
      if (lane == 0) s_nan[w] = any;
#pragma unroll
      for (int x = 0; x < TPW; ++x) {
        __syncthreads();
        const float zz = rows4_sum(SINGLE ? z[x] : z[x] + s_sum[SINGLE ? 0 : w][x][lane]);
        if (gq == 0) s_ref[w][n] = ref[x], s_z[w][n] = zz;
        if (n == 0)
#pragma unroll
          for (int i = 0; i < 4; ++i) s_zt[w][4 * gq + i] = zt[x][i];
        float* mine = reinterpret_cast<float*>(s_values) + w * (Lay<D>::kUnit / 4);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int h = 0; h < DPL / 4; ++h)
            *reinterpret_cast<float4*>(mine + (4 * gq + i) * D + DPL * n + 4 * h) =
                make_float4(O[x][4 * h][i], O[x][4 * h + 1][i], O[x][4 * h + 2][i], O[x][4 * h + 3][i]);
        __syncthreads();
        for (int i = tid; i < 16 * D / 4; i += TW * 64) {
          const int r = i / (D / 4), c = i % (D / 4), row = (tile0 + x) * 16 + r;
          if (row >= a.R) continue;
          // (everything is read first: a branch for each wave would wait for its reads alone)
          float M = kNegInf, ref_k[TW], z_k[TW], zt_k[TW];
          float4 o_k[TW];
#pragma unroll
          for (int k = 0; k < TW; ++k) {
            ref_k[k] = s_ref[k][r], z_k[k] = s_z[k][r], zt_k[k] = s_zt[k][r];
            const float* theirs = reinterpret_cast<const float*>(s_values) + k * (Lay<D>::kUnit / 4);
            o_k[k] = *reinterpret_cast<const float4*>(theirs + r * D + 4 * c);
          }
#pragma unroll
          for (int k = 0; k < TW; ++k) M = fmaxf(M, ref_k[k]);
          const float base = M == kNegInf ? 0.f : M;
          float Z = 0.f, Zt = 0.f;
          floatx4 o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < TW; ++k) {
            const bool seen = z_k[k] != 0.f;  // (else the wave has nothing that the row sees)
            const float f = shift_exp2(ref_k[k] - base);
            Z = seen ? fmaf(z_k[k], f, Z) : Z;
            Zt = seen ? fmaf(zt_k[k], f, Zt) : Zt;
            o[0] = seen ? fmaf(o_k[k].x, f, o[0]) : o[0];
            o[1] = seen ? fmaf(o_k[k].y, f, o[1]) : o[1];
            o[2] = seen ? fmaf(o_k[k].z, f, o[2]) : o[2];
            o[3] = seen ? fmaf(o_k[k].w, f, o[3]) : o[3];
          }
          const size_t at = (size_t)rec * a.RTT * 16 + row;
          if constexpr (SINGLE) {
            uint32_t any_wave = 0;
#pragma unroll
            for (int k = 0; k < TW; ++k) any_wave |= s_nan[k];
            float y[4] = {o[0], o[1], o[2], o[3]};
            put_row<D, 4>(a, p.b, p.g, row, p.ctx, rows, c, y, M, Z, Zt, any_wave != 0);
          } else {
            if (c == 0) a.stats[at] = make_float4(M, Z, Zt, 0.f);
            *reinterpret_cast<float4*>(a.opart + at * D + 4 * c) = make_float4(o[0], o[1], o[2], o[3]);
          }
        }
      }
      if (!SINGLE && threadIdx.x == 0 && rg == 0) {
        uint32_t any_wave = 0;
        for (int k = 0; k < TW; ++k) any_wave |= s_nan[k];
        a.nan[rec] = any_wave;
      }
      __syncthreads();
    } while (!SINGLE && p.next(a, a.ctx_len));
  }
  if (bad_page && lane == 0) dev_flag(a.status, PVLM_DEV_RANGE);
}

// --------------------------------------------------------------- combine --
// A wave joins a row's records: their references and sums a lane each, then the
// partial results weighted by exp2(record's reference - row maximum).
template <int D>
__device__ __forceinline__ void combine_row(const Q4Args& a, int id) {
  constexpr int C = D / 64, kU = 8;
  const int lane = threadIdx.x & 63;
  const int bg = id / a.R, row = id - bg * a.R, b = bg / a.Hkv, g = bg - b * a.Hkv;
  const Shares s = q8_find<false>(a, Wave(a.ctx_len), 0, b);
  const Holders h = holders(a, s.per, s.align, s.before, b, g, s.ctx);
  const size_t step = (size_t)a.RTT * 16, at = h.rec * step + row;
  float m = kNegInf, z = 0.f, zt = 0.f, o[C];
  bool nan = false;
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.f;
  for (int s0 = 0; s0 < h.count; s0 += 64) {
    const int cnt = min(64, h.count - s0);
    float v[kU][C];
    auto load = [&](int k0) {
#pragma unroll
      for (int k = 0; k < kU; ++k) {
        const float* src = a.opart + (at + (s0 + min(k0 + k, cnt - 1)) * step) * D + C * lane;
#pragma unroll
        for (int c = 0; c < C; ++c) v[k][c] = src[c];
      }
    };
    load(0);  // (beside the statistics)
    float4 st = make_float4(kNegInf, 0.f, 0.f, 0.f);
    if (lane < cnt) {
      st = a.stats[at + (s0 + lane) * step];
      nan |= a.nan[h.rec + s0 + lane] != 0 && st.y != 0.f;
    }
    const float M = fmaxf(m, warp_max(st.y != 0.f ? st.x : kNegInf)), r = M == kNegInf ? 0.f : M;
    const float f = z != 0.f ? shift_exp2(m - r) : 0.f, e = st.y != 0.f ? shift_exp2(st.x - r) : 0.f;
    z = (z != 0.f ? z * f : 0.f) + warp_sum(st.y != 0.f ? st.y * e : 0.f);
    zt = zt * f + warp_sum(st.y != 0.f ? st.z * e : 0.f);
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] *= f;
    m = M;
    for (int k0 = 0; k0 < cnt; k0 += kU) {
      if (k0 > 0) load(k0);
#pragma unroll
      for (int k = 0; k < kU; ++k) {
        const float wgt = __shfl(e, min(k0 + k, cnt - 1), 64);
        if (k0 + k < cnt)  // (a weight of 0 too: NaN stays)
#pragma unroll
          for (int c = 0; c < C; ++c) o[c] = fmaf(v[k][c], wgt, o[c]);
      }
    }
  }
  const Rows rows(a.c, a.ctx_len, a.Hkv, b, g);
  put_row<D, C>(a, b, g, row, s.ctx, rows, lane, o, m, z, zt, __any(nan));
}

constexpr int kCombineWaves = 4;
template <int D>
__global__ void __launch_bounds__(kCombineWaves * 64) q4_combine_kernel(Q4Args a) {
  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * kCombineWaves + (threadIdx.x >> 6));
  if (id < a.B * a.Hkv * a.R) combine_row<D>(a, id);
}

// ----------------------------------------------------------------- mass --
// A run of a sequence's tokens and every query row: the waves hold the queries of a set
// of row tiles each (GW sets at a time), with the rows on the M side, so that a lane's
// scores of a token sum up in the lane.  A row's maximum and inverse sum are kept
// apart: a probability's exponent is rounded at its distance from the maximum, which
// is nothing where the mass is.
template <int D, int MT>
__device__ __forceinline__ void mass_run(const Q4Args& a, int64_t item, float (*s_mass)[kQ4MassRun]) {
  const int b = (int)(item / a.chunks);
  const int64_t t0 = (item - (int64_t)b * a.chunks) * a.chunk;
  const int ctx = __builtin_amdgcn_readfirstlane(clamp_ctx(a, uniform_load(a.ctx_len, b)));
  const int n_rows = rows_of(a, b), N = tokens_of(ctx, n_rows);
  float* mass = a.mass + (size_t)b * a.c.n_cap;
  const int64_t t_end = min(t0 + a.chunk, a.c.n_cap);
  if (t0 >= N) {
    for (int64_t t = t0 + threadIdx.x; t < t_end; t += 512) mass[t] = 0.f;
    return;
  }
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int gw = w % a.GW, tw = w / a.GW, TW = 8 / a.GW;
  const LaneOf<D> place_of(n, gq);
  const int c0 = (int)t0, c1 = min((int)t_end, N);
  bool bad_page = false;
  for (int set = gw; set < a.Hkv * a.MG; set += a.GW) {
    const int g = set / a.MG, tile0 = (set - g * a.MG) * MT;
    const Rows rows(a.c, a.ctx_len, a.Hkv, b, g);
    // (a tile is loaded one ahead, its page two; past the run, the last one again)
    auto tile = [&](int t) { return min(t, (c1 - 1) & ~15); };
    Codes<D> kc;
    int page = rows.entry(tile(c0 + 16 * tw));
    auto load = [&](int t) {
      load_codes<D>(a.c.kc, a.c.ke, rows.at(tile(t), page, bad_page), place_of, kc);
      page = rows.entry(tile(t + 16 * TW));
    };
    load(c0 + 16 * tw);
    Query<D> q[MT];
    float top[MT][4], inv[MT][4];
#pragma unroll
    for (int x = 0; x < MT; ++x) {
      load_query<D>(a, b, g, (tile0 + x) * 16 + n, gq, n_rows, q[x]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = (tile0 + x) * 16 + 4 * gq + i;
        const float2 r = a.rows[((size_t)b * a.Hkv + g) * a.R + min(row, a.R - 1)];
        top[x][i] = row < a.R ? r.x : __builtin_huge_valf();
        inv[x][i] = row < a.R ? r.y : 0.f;
      }
    }
    for (int t = c0 + 16 * tw; t < c1; t += 16 * TW) {
      const float u = place_of.unit(kc.e);
      floatx4 S[MT];
#pragma unroll
      for (int x = 0; x < MT; ++x) S[x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ks = 0; ks < D / 32; ++ks) {
        const bf16x8 k = to_bf16(kc.w[ks], u);
#pragma unroll
        for (int x = 0; x < MT; ++x) S[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[x].s[ks], k, S[x], 0, 0, 0);
      }
      load(t + 16 * TW);
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
  __syncthreads();
  if (bad_page && lane == 0) dev_flag(a.status, PVLM_DEV_RANGE);
}

// (Registers for four waves a SIMD with up to three row tiles a wave, two with more.)
template <int D, int MT>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(MT <= 3 ? 4 : 2, MT <= 3 ? 4 : 2)))
q4_mass_kernel(Q4Args a) {
  __shared__ float s_mass[8][kQ4MassRun];
  for (int64_t item = blockIdx.x; item < (int64_t)a.chunks * a.B; item += gridDim.x) mass_run<D, MT>(a, item, s_mass);
}

// ------------------------------------------------------------------ host --
typedef void (*Q4Kernel)(Q4Args);
template <int D, bool SINGLE>
Q4Kernel pick_part(int RT) {
  return RT == 1 ? q4_part_kernel<D, 1, SINGLE> : RT == 2 ? q4_part_kernel<D, 2, SINGLE> : q4_part_kernel<D, 3, SINGLE>;
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
                          const void* q, const Q4Cache& c, const int32_t* ctx_len, const int32_t* n_new, void* out,
                          float* mass, float* lse, void* ws, size_t ws_bytes, int32_t* status, hipStream_t stream) {
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
  a.n_new = n_new;
  a.B = B;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = p.G;
  a.R = p.R;
  a.g_magic = (1u << 20) / (unsigned)p.G + 1u;
  a.RTT = p.RTT;
  a.RG = 1;
  a.HR = Hkv;
  a.max_ctx = (int)max_ctx;
  a.wgs = p.shares;
  a.per_share = p.per_share;
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
  a.chunks = (int)((c.n_cap + p.chunk - 1) / p.chunk);
  const Q4Kernel part = p.single ? (D == 128 ? pick_part<128, true>(p.RT) : pick_part<64, true>(p.RT))
                                 : (D == 128 ? pick_part<128, false>(p.RT) : pick_part<64, false>(p.RT));
  const int lds = kQ4Waves * (D == 128 ? Lay<128>::kUnit : Lay<64>::kUnit);
  PVLM_HIP(allow_dynamic_lds(reinterpret_cast<const void*>(part), lds));
  hipLaunchKernelGGL(part, dim3(p.shares * p.per_share), dim3(kQ4Waves * 64), lds, stream, a);
  PVLM_LAUNCHED();
  if (!p.single) {
    const int rows = B * Hkv * p.R;
    hipLaunchKernelGGL(D == 128 ? q4_combine_kernel<128> : q4_combine_kernel<64>,
                       dim3((rows + kCombineWaves - 1) / kCombineWaves), dim3(kCombineWaves * 64), 0, stream, a);
    PVLM_LAUNCHED();
  }
  if (mass) {
    // on a stream with a budget, one workgroup for each of its compute units
    const int64_t items = (int64_t)a.chunks * B, most = di.budgeted ? di.cus : (int64_t)1 << 22;
    hipLaunchKernelGGL(D == 128 ? pick_mass<128>(p.MT) : pick_mass<64>(p.MT),
                       dim3((unsigned)(items < most ? items : most)), dim3(512), 0, stream, a);
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

extern "C" pvlm_status pvlm_verify_attn_q4_ragged(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int64_t n_cap,
                                                  int64_t max_ctx, float scale, const void* q, const uint8_t* k_codes,
                                                  const uint8_t* k_exps, const uint8_t* v_codes, const uint8_t* v_exps,
                                                  const int32_t* ctx_len, const int32_t* n_new, void* out, float* mass,
                                                  float* lse, void* ws, size_t ws_bytes, int32_t* status,
                                                  hipStream_t stream) {
  return verify_q4_run(dt, B, T, Hq, Hkv, D, max_ctx, scale, q, view(k_codes, k_exps, v_codes, v_exps, n_cap), ctx_len,
                       n_new, out, mass, lse, ws, ws_bytes, status, stream);
}

extern "C" pvlm_status pvlm_verify_attn_q4(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int64_t n_cap,
                                           int64_t max_ctx, float scale, const void* q, const uint8_t* k_codes,
                                           const uint8_t* k_exps, const uint8_t* v_codes, const uint8_t* v_exps,
                                           const int32_t* ctx_len, void* out, float* mass, float* lse, void* ws,
                                           size_t ws_bytes, int32_t* status, hipStream_t stream) {
  return pvlm_verify_attn_q4_ragged(dt, B, T, Hq, Hkv, D, n_cap, max_ctx, scale, q, k_codes, k_exps, v_codes, v_exps,
                                    ctx_len, nullptr, out, mass, lse, ws, ws_bytes, status, stream);
}

extern "C" pvlm_status pvlm_verify_attn_q4_ragged_paged(
    pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int page_size, int max_pages, int64_t n_pages, int64_t max_ctx,
    float scale, const void* q, const uint8_t* k_codes, const uint8_t* k_exps, const uint8_t* v_codes,
    const uint8_t* v_exps, const int32_t* page_table, const int32_t* ctx_len, const int32_t* n_new, void* out,
    float* mass, float* lse, void* ws, size_t ws_bytes, int32_t* status, hipStream_t stream) {
  Q4Cache c = view(k_codes, k_exps, v_codes, v_exps, 0);
  const pvlm_status st = q8_pages(page_size, max_pages, n_pages, page_table, &c);
  if (st != PVLM_OK) return st;
  return verify_q4_run(dt, B, T, Hq, Hkv, D, max_ctx, scale, q, c, ctx_len, n_new, out, mass, lse, ws, ws_bytes, status,
                       stream);
}

extern "C" pvlm_status pvlm_verify_attn_q4_paged(pvlm_dtype dt, int B, int T, int Hq, int Hkv, int D, int page_size,
                                                 int max_pages, int64_t n_pages, int64_t max_ctx, float scale,
                                                 const void* q, const uint8_t* k_codes, const uint8_t* k_exps,
                                                 const uint8_t* v_codes, const uint8_t* v_exps,
                                                 const int32_t* page_table, const int32_t* ctx_len, void* out,
                                                 float* mass, float* lse, void* ws, size_t ws_bytes,
                                                 int32_t* status, hipStream_t stream) {
  return pvlm_verify_attn_q4_ragged_paged(dt, B, T, Hq, Hkv, D, page_size, max_pages, n_pages, max_ctx, scale, q,
                                          k_codes, k_exps, v_codes, v_exps, page_table, ctx_len, nullptr, out, mass, lse,
                                          ws, ws_bytes, status, stream);
}

// Verify attention with fused per-token attention mass over an 8-bit cache
// (gfx950): pvlm_verify_attn's operation (ParallelVLM Sec. 2.2, Sec. 4.2; the
// mass of Sec. 3, Challenge 2) on rows in the format of q8.h, for T = 1 (a
// decode step) to 32 rows.
//
// Mathematics.  With K_i = ck_i 2^(ek_i - 127) and V_i likewise:
//   s_i = scale <q, K_i>     P_i = softmax(s)_i over visible i
//   out = sum_i P_i V_i      mass_i = sum over rows of P_i
//  * Both products run on bf16 with fp32 sums: K_i and V_i are bf16 values (four
//    significant bits and a power of two), so their conversion rounds nothing.
//    (The 8-bit matrix instructions align an instruction's products to the
//    largest of them and lose up to 2^-14 of it, measured against float64; bf16
//    ones 2^-21.)
//  * P is rounded to bf16 for the second product, half a step being 2^-9 to 2^-8
//    of a term of a result that is rounded to bf16 itself; the row is divided by
//    the sum of what was rounded.  lse and mass use the unrounded sum.
//  * One pass over a chunk with a running maximum and sum in fp32; the chunks'
//    (maximum, sum) and fp32 O partials are joined by the finish kernel.  The
//    mass needs every row's sum first, so K is read a second time.
//    Every order of summation is fixed.  No workgroup waits for another.
//
// Three launches (two without the mass), all on the caller's stream:
//   partial  waves that convert a block of 64 tokens from memory to bf16 in LDS,
//            once for all row tiles, beside waves that hold a tile of 16 rows
//   mass     the same shares of the tokens, K alone, up to three tiles a wave
//   finish   a wave or a workgroup joins a row's records; others sum the mass
// What bounds them, and what they measured (one MI355X, D = 128, kernel times
// under the profiler, which slows the longer ones by up to a tenth):
//   memory: 16 sequences of one token, 84 MB of each of K and V: partial 37.5 us,
//     4.5 TB/s.  4 sequences of 9 tokens, 117 MB each: partial 54 to 59 us, 4.0 to
//     4.3 TB/s; mass (K again) 41 to 43 us, 2.8 TB/s.
//   instructions, with many rows: 136 rows a head over 132K tokens, 136 MB each:
//     partial 112 to 121 us (0.6 PFLOP/s), mass 69 to 75 us (0.5 PFLOP/s).  Of a
//     SIMD's cycles 37 % are matrix instructions, 48 % vector ones, of LDS's 43 %
//     reads and writes; barriers keep the waves too close in step for more of each.
//   partial results, with few rows over few tokens: 72 rows a head over 12800 tokens
//     write and read 18 MB of them beside 26 MB of cache (partial 19 us, mass 13,
//     finish 7).
//   latency in small calls: a launch that waits for the lengths, then for its
//     first blocks (all compute units ask at once), then for its stores takes
//     4 to 8 us.
#include "q8.h"
#include "q8_plan.h"

namespace pvlm {
namespace {

typedef uint32_t uintx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr double kLog2e = 1.4426950408889634;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNegInf = -__builtin_huge_valf();
// A wave's running reference may trail its row maximum by this much (log2
// domain): O is rescaled only when a block's maximum exceeds it, which a few
// blocks in a thousand do (with 8, one in six of a workgroup of 45 rows and one
// in three of 72).  Probabilities then reach 2^24 in a type of bf16's range.
constexpr float kRefSlack = 24.f;
constexpr int kFinWaves = kFinThreads / 64;

struct QArgs : QShape {
  const uint16_t* q;
  Q8Cache c;
  const int32_t* ctx_len;
  int Hq, G, R;
  unsigned g_magic;  // row / G == row * g_magic >> 20 for row < 640 (2^20 / G + 1; G <= 640)
  int RTT;
  float sl2;         // scale * log2(e)
  float* mpart;      // [B][HR][waves][mrows] mass of one wave's rows
  int64_t mrows;     // max_ctx + T in whole units
  float2* stats;     // [record][tile][token wave][16] (log2-domain maximum, sum) of rows
  float* zt;         // the same sums of the probabilities as P . V takes them, rounded to bf16
  uint32_t* nan;     // [record][CW] the values hold a NaN that not every row sees
  float* opart;      // [record][tile][token wave][16][D] sums of P . V relative to that maximum
  uint16_t* out;
  float* lse;
  float* mass;
  int32_t* status;
  int mass_wgs, mass_per, mass_rows;  // finish kernel: workgroups that sum the mass, of a sequence, rows of one
};

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
  __device__ __forceinline__ explicit Wave(const QArgs& a) : ctx_len(a.ctx_len), lane(threadIdx.x & 63) {}
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
  __device__ __forceinline__ bool first(const QArgs& a) {
    return begin(a, q8_find<true>(a, Wave(a), blockIdx.x, 0), blockIdx.x);
  }
  // false where the share ends
  __device__ __forceinline__ bool next(const QArgs& a) {
    return advance(a, [&](int x) { return __builtin_amdgcn_readfirstlane(clamp_ctx(a, uniform_load(a.ctx_len, x))); });
  }
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int row_t(const QArgs& a, int row) { return (int)((unsigned)row * a.g_magic >> 20); }

// ------------------------------------------------------------- the blocks --
// The page-table entry of token t (0 in a padded cache), and the row index (in
// rows of codes) of the unit that t opens.  An entry outside the pool sets bad
// and is clamped into it.
__device__ __forceinline__ int page_entry(const QArgs& a, int b, int t) {
  return a.c.table ? uniform_load(a.c.table, (int64_t)b * a.c.max_pages + (t >> a.c.shift)) : 0;
}
__device__ __forceinline__ int64_t unit_row(const QArgs& a, int b, int g, int t, int page, bool& bad) {
  if (!a.c.table) return ((int64_t)b * a.Hkv + g) * a.c.n_cap + t;
  if (page < 0 || page >= a.c.n_pages) {
    bad = true;
    page = page < 0 ? 0 : (int)(a.c.n_pages - 1);
  }
  return (((int64_t)page * a.Hkv + g) << a.c.shift) + (t & ((1 << a.c.shift) - 1));
}

// LDS holds a block of 64 tokens as bf16 rows, of K and of V: 16-byte chunk c
// of row r lies at chunk c ^ swz(r) of the row.  swz is linear in the bits of r
// mod 16, and these are placed so that what LDS serves at a time falls on distinct
// banks (its conflict counter is then 0; r mod 16 in place of swz: a third of the
// LDS cycles were conflicts):
//   a read of K, 256 bytes: chunk 4 ks of rows 0-3 and 12-15, chunk 4 ks + 1 of
//     rows 4-11, or the other way round;
//   a read of V, 256 bytes: eight rows' same two chunks;
//   a write, 128 bytes: four even chunks of two rows that differ in bit 2.
template <int D>
struct Lay {
  static constexpr int CH = D / 8, kSide = 64 * D * 2;  // chunks of a row, bytes of a block's K or V
  // Where a lane's reads of a block begin: K's chunk gq of row n (the others are
  // 4 ks chunks and 16 tt rows on), and V's 8 bytes of row 4 gq + n / 4 (32 jd
  // bytes, and 16 and 32 rows on).  Chunks differ by an exclusive or of the
  // address: blocks start at multiples of 256 bytes.
  static constexpr __host__ __device__ int swz(int r) {
    const int m = D == 128 ? r : r >> 1 & 7;  // (two rows of D = 64 fill the banks)
    return (m << 1 & 6) ^ (D == 128 ? (r & 4 ? 9 : 0) ^ (r & 8) : (r & 4 ? 1 : 0) ^ (r & 8 ? 4 : 0));
  }
  static __device__ __forceinline__ uint32_t k_lane(int n, int gq) { return n * D * 2 + ((gq ^ swz(n)) << 4); }
  static __device__ __forceinline__ uint32_t k_at(uint32_t lane, int ks, int tt) { return (lane ^ (ks << 6)) + tt * 32 * D; }
  static __device__ __forceinline__ uint32_t v_lane(int n, int gq) {
    const int row = 4 * gq + n / 4;
    return row * D * 2 + ((((n >> 1) & 1) ^ swz(row)) << 4) + 8 * (n & 1);
  }
  static __device__ __forceinline__ uint32_t v_at(uint32_t lane, int jd, int rows) { return (lane ^ (jd << 5)) + rows * D * 2; }
};

template <typename T>
__device__ __forceinline__ T lds_read(uint32_t at) {
  return *(const __attribute__((address_space(3))) T*)at;
}
__device__ __forceinline__ void lds_write(uint32_t at, bf16x8 x) { *(__attribute__((address_space(3))) bf16x8*)at = x; }

// Eight codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8 to_bf16(uint32_t lo, uint32_t hi, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, unit, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, unit, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, unit, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, unit, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// What a converting wave does: one side (K or V) of the workgroup's blocks, from
// memory through registers into LDS as bf16, a row's power of two taken in.  Each
// conversion happens once for all row tiles.  A wave takes half a block (one
// unit) at a time: of a round's 2 TW halves those from number `first` on, CW apart.
// DEPTH halves are on their way at any time, by ordinary loads that the compiler
// waits for one half at a time.  For a round, LDS has two slots of ROUND bytes: one
// barrier a round hands a filled one over and an emptied one back.
//
// Rows past the piece become zeros (their tokens' probabilities are 0, and 0
// times what an unwritten row holds may be NaN).  So do NaN values of rows that
// not every query row sees; the record's flag has the finish kernel look for
// them.
template <int D, int TW, int CW, int DEPTH, int ROUND, int BLOCK, bool IS_V>
__device__ __forceinline__ void convert_share(const QArgs& a, Piece p, int first, uint32_t ring) {
  constexpr int PER = 2 * TW / CW;  // halves of a round
  // Lanes of a row, and rows of a lane: consecutive ones, whose exponents it reads
  // at once.  Eight neighbouring lanes write rows that differ in bit 2 (see Lay).
  constexpr int LPR = D / 16, NI = D / 32;
  const int lane = threadIdx.x & 63, c = lane % LPR, q = lane / LPR;
  const uint32_t row0 = NI * (D == 128 ? q ^ (c >> 2) : (q & ~3) | (q & 1) << 1 | (q >> 1 & 1));
  const uint32_t at_codes = row0 * D + 16 * c;
  const uint8_t* codes = IS_V ? a.c.vc : a.c.kc;
  const uint8_t* exps = IS_V ? a.c.ve : a.c.ke;
  const uint32_t lds0 = row0 * D * 2 + (((2 * c) ^ Lay<D>::swz(row0)) << 4);

  uintx4 v[DEPTH][NI];
  uint32_t e[DEPTH];
  int tb[DEPTH], c1[DEPTH], ctx[DEPTH], last_of[DEPTH];  // its tokens; its record if it is its piece's last, else -1
  int t0 = p.c0 + 32 * first, x = 0, total = 0;
  bool more = true, bad_page = false;
  // vmcnt(0): nothing of another path is under way (the compiler would wait for it at every half)
  __builtin_amdgcn_s_waitcnt(0x0f70);
  // The next half's unit (past the piece, the piece's last; of a whole unit every
  // row may be read), and its page entry, which is then there when it is wanted.
  int unit, page;
  auto find_unit = [&] {
    unit = min(t0, (p.c1 - 1) & ~31);
    page = page_entry(a, p.b, unit);
  };
  // (always loads, so that the compiler knows how many loads are under way: past
  // the share, rows of its last piece again)
  auto issue = [&](int k) {
    const int64_t r = unit_row(a, p.b, p.g, unit, page, bad_page);
    const uint8_t *src = codes + r * D, *src_e = exps + r;
#pragma unroll
    for (int i = 0; i < NI; ++i) v[k][i] = *reinterpret_cast<const uintx4*>(src + at_codes + i * D);
    if constexpr (NI == 4) e[k] = *reinterpret_cast<const uint32_t*>(src_e + row0);
    else e[k] = *reinterpret_cast<const uint16_t*>(src_e + row0);
    if (!more) return;
    tb[k] = t0;
    c1[k] = p.c1;
    ctx[k] = p.ctx;
    last_of[k] = -1;
    ++total;
    t0 += 32 * CW;
    if (++x == PER) {
      x = 0;
      if (t0 - 32 * first >= p.c1) {
        last_of[k] = (p.group(a) + blockIdx.x) * CW + first;
        Piece next = p;
        more = next.next(a);
        if (more) {
          p = next;
          t0 = p.c0 + 32 * first;
        }
      }
    }
    find_unit();
  };
  find_unit();
  uint32_t bad = 0;
  auto convert = [&](int k, uint32_t at) {
    const int whole = IS_V ? min(c1[k] - 1, ctx[k]) : c1[k] - 1;
    if (__builtin_amdgcn_readfirstlane(tb[k] + 31 - whole) > 0) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int t = tb[k] + (int)row0 + i;
        if (t >= c1[k]) {
          v[k][i] = uintx4{0, 0, 0, 0};
          e[k] = (e[k] & ~(0xffu << 8 * i)) | 127u << 8 * i;
        }
        if (IS_V && t > ctx[k])
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t m = nan_codes(v[k][i][j]);
            bad |= m;
            v[k][i][j] &= ~(m | (m - (m >> 7)));
          }
      }
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const float unit = q8_unit((e[k] >> (8 * i)) & 0xffu);
      lds_write((at ^ (Lay<D>::swz(i) << 4)) + i * D * 2, to_bf16(v[k][i][0], v[k][i][1], unit));
      lds_write((at ^ ((Lay<D>::swz(i) ^ 1) << 4)) + i * D * 2, to_bf16(v[k][i][2], v[k][i][3], unit));
    }
    if (IS_V && last_of[k] >= 0) {
      const bool any = __any(bad);
      if (lane == 0) a.nan[last_of[k]] = any;
      bad = 0;
    }
  };
  // (one loop body and no way out of its middle, for the same reason)
  int done = -DEPTH;
  do {
#pragma unroll
    for (int k = 0; k < DEPTH; ++k) {
      const bool now = done >= 0 && done < total;
      const int half = done % PER * CW + first;
      if (now) convert(k, ring + lds0 + (done / PER % 2) * ROUND + half / 2 * BLOCK + half % 2 * 32 * D * 2);
      issue(k);
      ++done;
      if (now && done % PER == 0) lds_sync();  // the round is there; every wave is done with the one before
    }
  } while (done < total);
  if (bad_page && lane == 0) dev_flag(a.status, PVLM_DEV_RANGE);
}

// ---------------------------------------------------------------- operands --
// Tokens are the M side of 16-row score tiles and query rows the N side (lane
// (n, gq) = (lane & 15, lane >> 4) owns row n and tokens 16 tt + 4 gq + i of tile
// tt), which is the layout P . V needs as its A operand.
template <int D>
struct Query {
  bf16x8 s[D / 32];  // chunk 4 ks + gq of the row
};

template <int D>
__device__ __forceinline__ void load_query(const QArgs& a, int b, int g, int row, int gq, Query<D>& q) {
  const int r = min(row, a.R - 1), t = row_t(a, r), h = g * a.G + r - t * a.G;
  const bf16x8* src = reinterpret_cast<const bf16x8*>(a.q + (((size_t)b * a.T + t) * a.Hq + h) * D) + gq;
#pragma unroll
  for (int ks = 0; ks < D / 32; ++ks) q.s[ks] = src[4 * ks];
}

// Maximum over the four lanes l, l^16, l^32, l^48; NaN if one is.
__device__ __forceinline__ float rows4_maximum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __builtin_elementwise_maximum(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Scores of a block (its K at LDS address k plus the lane's offset) against a
// wave's row tiles.  AHEAD operand reads of LDS are under way while the matrix
// instructions of earlier ones run (the compiler, left to itself, waits for each
// read alone).
template <int D, int TPW, int AHEAD>
__device__ __forceinline__ void scores(uint32_t k, const Query<D> (&q)[TPW], floatx4 (&S)[TPW][4]) {
  constexpr int N = D / 8;  // operands: chunk 4 ks + gq of the rows of tile tt, number 4 ks + tt
  bf16x8 kr[AHEAD];
#pragma unroll
  for (int j = 0; j < AHEAD - 1; ++j) kr[j] = lds_read<bf16x8>(Lay<D>::k_at(k, j / 4, j % 4));
#pragma unroll
  for (int x = 0; x < TPW; ++x)
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) S[x][tt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int m = j + AHEAD - 1;
    if (m < N) kr[m % AHEAD] = lds_read<bf16x8>(Lay<D>::k_at(k, m / 4, m % 4));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < TPW; ++x)
      S[x][j % 4] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kr[j % AHEAD], q[x].s[j / 4], S[x][j % 4], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// O += P . V over a block; P[h] holds tokens 32 h + 4 gq + {0..3, 16..19}.
// Transposed LDS reads: each 16 lanes fetch 16 columns of four rows (lane n the
// 8 bytes of row n / 4, columns 4 (n mod 4) on) and lane n receives column n.
template <int D, int AHEAD>
__device__ __forceinline__ void weigh(uint32_t v, const bf16x8 (&P)[2], floatx4 (&O)[D / 16]) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  typedef short s8 __attribute__((ext_vector_type(8)));
  typedef __attribute__((address_space(3))) s4* lds_s4;
  constexpr int N = D / 8;  // operands: columns 16 jd + n of tokens 32 h on, number 2 jd + h
  s4 lo[AHEAD], hi[AHEAD];
  auto read = [&](int j) {
    lo[j % AHEAD] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)Lay<D>::v_at(v, j / 2, j % 2 * 32));
    hi[j % AHEAD] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)Lay<D>::v_at(v, j / 2, j % 2 * 32 + 16));
  };
#pragma unroll
  for (int j = 0; j < AHEAD - 1; ++j) read(j);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (j + AHEAD - 1 < N) read(j + AHEAD - 1);
    __builtin_amdgcn_sched_barrier(0);
    const s8 b = __builtin_shufflevector(lo[j % AHEAD], hi[j % AHEAD], 0, 1, 2, 3, 4, 5, 6, 7);
    O[j / 2] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P[j % 2], __builtin_bit_cast(bf16x8, b), O[j / 2], 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// (maximum, sum) of two sets of scores.  A sum of 0 belongs to one of which the
// row sees nothing; NaN passes.
__device__ __forceinline__ void join(float& m, float& z, float m2, float z2) {
  const float M = fmaxf(m, m2), r = M == kNegInf ? 0.f : M;
  z = (z != 0.f ? z * fast_exp2(m - r) : 0.f) + (z2 != 0.f ? z2 * fast_exp2(m2 - r) : 0.f);
  m = M;
}
// Maximum of row n of a wave's tiles over a group's records, and the inverse of its
// sum, the lane groups taking the records in turn, with many loads in flight
// (padding rows: +inf, their probabilities are 0).  The two apart, and not their
// log-sum-exp: a probability's exponent is then rounded at its distance from the
// maximum, which is nothing where the mass is.
template <int RT, int TPW>
__device__ __forceinline__ void tile_sums(const QArgs& a, const Holders& h, int tile0, int tiles, const bool (&real)[TPW],
                                         int n, int gq, float (&top)[TPW], float (&inv)[TPW]) {
  // records of every tile in flight: a group has dozens, and a round trip takes a
  // microsecond (42 rows over 6432 tokens, 102 records: 14.4 us, with four 17.5)
  constexpr int kU = 16;
  constexpr int TW = q8_waves(RT).tw;
  const int cnt = TW * h.count;
  const float2* st = a.stats + (size_t)h.rec * RT * TW * 16 + n;
  float M[TPW], Z[TPW];
#pragma unroll
  for (int x = 0; x < TPW; ++x) M[x] = kNegInf, Z[x] = 0.f;
  for (int s0 = gq; s0 < cnt; s0 += 4 * kU) {
    float2 v[kU][TPW];
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const int s = min(s0 + 4 * j, cnt - 1);
      const float2* r = st + (size_t)(s / TW * RT * TW + s % TW) * 16;
#pragma unroll
      for (int x = 0; x < TPW; ++x) v[j][x] = r[min(tile0 + x, tiles - 1) * TW * 16];
    }
#pragma unroll
    for (int x = 0; x < TPW; ++x) {
      float m = M[x];
#pragma unroll
      for (int j = 0; j < kU; ++j) m = fmaxf(m, v[j][x].x);
      const float r = m == kNegInf ? 0.f : m;
      float z = Z[x] != 0.f ? Z[x] * fast_exp2(M[x] - r) : 0.f;
#pragma unroll
      for (int j = 0; j < kU; ++j)
        z += v[j][x].y != 0.f && s0 + 4 * j < cnt ? v[j][x].y * fast_exp2(v[j][x].x - r) : 0.f;
      M[x] = m;
      Z[x] = z;
    }
  }
#pragma unroll
  for (int x = 0; x < TPW; ++x) {
    join(M[x], Z[x], lane_xor16(M[x]), lane_xor16(Z[x]));
    join(M[x], Z[x], lane_xor32(M[x]), lane_xor32(Z[x]));
    top[x] = real[x] ? M[x] : __builtin_huge_valf();
    inv[x] = real[x] ? 1.f / Z[x] : 0.f;
  }
}

// Sum over the 16 rows (lanes n) of the value with number n (lane & 15): each
// step a lane keeps half of its values, chosen by one bit of n, and adds its
// partner's copy of that half.
__device__ __forceinline__ float row_sums(const float (&p)[16], int lane) {
  const bool h8 = lane & 8, h4 = lane & 4, h2 = lane & 2, h1 = lane & 1;
  float a8[8], a4[4], a2[2];
#pragma unroll
  for (int k = 0; k < 8; ++k) a8[k] = (h8 ? p[8 + k] : p[k]) + lane_xor8(h8 ? p[k] : p[8 + k]);
#pragma unroll
  for (int k = 0; k < 4; ++k) a4[k] = (h4 ? a8[4 + k] : a8[k]) + lane_mirror8(h4 ? a8[k] : a8[4 + k]);
#pragma unroll
  for (int k = 0; k < 2; ++k) a2[k] = (h2 ? a4[2 + k] : a4[k]) + lane_xor2(h2 ? a4[k] : a4[2 + k]);
  return (h1 ? a2[1] : a2[0]) + lane_xor1(h1 ? a2[0] : a2[1]);
}

// -------------------------------------------------------- partial kernel --
template <int D, int RT>
struct PartShape {
  static constexpr int TW = q8_waves(RT).tw, CW = q8_waves(RT).cw;
  static constexpr int kCompute = RT * TW, kThreads = (kCompute + 2 * CW) * 64;
  // waves of a SIMD; two at least, so that a wave's registers are all of one kind
  static constexpr int kPerEu = kThreads <= 512 ? 2 : (kThreads + 255) / 256;
  static constexpr int kBlock = 2 * Lay<D>::kSide, kRound = TW * kBlock, kLds = 2 * kRound;
  // halves of blocks, of 16 registers (D = 128), that a converting wave has on their way
  static constexpr int kDepth = 4 * (128 / D);
};

// A computing wave's state: a row tile against the tokens of its blocks, with AHEAD
// operands read ahead.
template <int D, int AHEAD>
struct PartWave {
  static constexpr int DPL = D / 16;
  Query<D> q[1];
  int lim;  // last token that the lane's row sees
  float ref;
  float z, over;  // the sum of the row's probabilities, and what its rounding added to that
  floatx4 O[DPL], zt;

  __device__ __forceinline__ void begin(const QArgs& a, const Piece& p, int tile, bool here, int n, int gq) {
    const int row = tile * 16 + n;
    load_query<D>(a, p.b, p.g, row, gq, q[0]);
    lim = here && row < a.R ? min(p.c1 - 1, p.ctx + row_t(a, row)) : -1;
    ref = kNegInf;
    z = over = 0.f;
    zt = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int jd = 0; jd < DPL; ++jd) O[jd] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // The block of tokens tb .. tb + 63, K and V at LDS addresses k and v (with the lane's offsets).  TAIL: some row
  // does not see all of them.
  template <bool TAIL>
  __device__ __forceinline__ void block(const QArgs& a, uint32_t k, uint32_t v, int tb, int gq) {
    floatx4 S[1][4];
    scores<D, 1, AHEAD>(k, q, S);
    if constexpr (TAIL) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (16 * (j / 4) + j % 4 > lim - tb - 4 * gq) S[0][j / 4][j % 4] = kNegInf;
    }
    float m = kNegInf;  // (the maximum that passes NaN on: the other one has every operand canonicalised first)
#pragma unroll
    for (int j = 0; j < 16; ++j) m = __builtin_elementwise_maximum(m, S[0][j / 4][j % 4]);
    m = rows4_maximum(m) * a.sl2;
    if (__any(m > ref + kRefSlack)) {  // the first block, and seldom after it
      const float nm = fmaxf(ref, m);
      const float al = ref == kNegInf ? 0.f : fast_exp2(ref - nm);
      z *= al;
      over *= al;
      ref = nm;
      floatx4 f;
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __shfl(al, 4 * gq + i, 64);
      zt = zt * f;
#pragma unroll
      for (int jd = 0; jd < DPL; ++jd) O[jd] = O[jd] * f;
    }
    bf16x8 ones, P[2];
#pragma unroll
    for (int j = 0; j < 8; ++j) ones[j] = static_cast<__bf16>(1.f);
    const float r = ref == kNegInf ? 0.f : ref;  // no visible token yet: P = 0
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float e = fast_exp2(fmaf(S[0][j / 4][j % 4], a.sl2, -r));
      sum += e;
      P[j / 8][j % 8] = static_cast<__bf16>(e);
    }
    // Kahan's sum over the blocks: beside one large term, thousands of small ones
    // would each be rounded away (a log-sum-exp 6e-6 off over 132K tokens)
    sum -= over;
    const float old = z;
    z += sum;
    over = (z - old) - sum;
#pragma unroll
    for (int h = 0; h < 2; ++h) zt = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P[h], ones, zt, 0, 0, 0);
    weigh<D, AHEAD>(v, P, O);
  }

  __device__ __forceinline__ void end(const QArgs& a, size_t rec, int tile, int n, int gq) {
    const float zz = rows4_sum(z - over);
    if (gq == 0) a.stats[rec * 16 + n] = make_float2(ref, zz);
    if (n == 0) *reinterpret_cast<floatx4*>(a.zt + rec * 16 + 4 * gq) = zt;
    // position DPL n + jd of a stored row holds column 16 jd + n
    float* op = a.opart + rec * 16 * D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (tile * 16 + 4 * gq + i < a.R)
#pragma unroll
        for (int h = 0; h < DPL / 4; ++h)
          *reinterpret_cast<float4*>(op + (4 * gq + i) * D + DPL * n + 4 * h) =
              make_float4(O[4 * h][i], O[4 * h + 1][i], O[4 * h + 2][i], O[4 * h + 3][i]);
  }
};

template <int D, int RT>
__global__ void __launch_bounds__((PartShape<D, RT>::kThreads))
__attribute__((amdgpu_waves_per_eu(PartShape<D, RT>::kPerEu, PartShape<D, RT>::kPerEu))) q8_part_kernel(QArgs a) {
  typedef PartShape<D, RT> S_;
  constexpr int TW = S_::TW;
  extern __shared__ __align__(1024) char s_ring[];  // [2][TW][K, V][64][D]

  Piece p;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && w == 0)
    for (int b = threadIdx.x; b < a.B; b += 64)
      if (a.ctx_len[b] < 0 || a.ctx_len[b] > a.max_ctx) dev_flag(a.status, PVLM_DEV_RANGE);
  if (!p.first(a)) return;
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr(s_ring));
  if (w >= S_::kCompute) {
    const int x = w - S_::kCompute;
    if (x < S_::CW) convert_share<D, TW, S_::CW, S_::kDepth, S_::kRound, S_::kBlock, false>(a, p, x, ring);
    else convert_share<D, TW, S_::CW, S_::kDepth, S_::kRound, S_::kBlock, true>(a, p, x - S_::CW, ring + Lay<D>::kSide);
    return;
  }
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int tw = w % TW, tile = w / TW;  // its blocks, and its tile
  const uint32_t k0 = ring + tw * S_::kBlock + Lay<D>::k_lane(n, gq);
  const uint32_t v0 = ring + tw * S_::kBlock + Lay<D>::kSide + Lay<D>::v_lane(n, gq);
  uint32_t slot = 0;
  do {
    const int tile_g = p.rg * RT + tile;  // of the KV head's; one past its rows is idle
    const bool here = tile_g < a.RTT;
    PartWave<D, S_::kPerEu == 4 ? 4 : 8> v;  // (by a wave's registers: 128 or 168)
    v.begin(a, p, tile_g, here, n, gq);
    // the wave's rounds whose block every row sees whole, then the others (two
    // loops with their test at the end: joined, or with the test ahead, the
    // compiler copies all of O in every round)
    const int rounds = __builtin_amdgcn_readfirstlane((p.c1 - p.c0 + 64 * TW - 1) / (64 * TW));
    const int whole = __builtin_amdgcn_readfirstlane(
        here ? (min(p.c1 - 1, p.ctx) - (64 * tw + 63) - p.c0 + 64 * TW) / (64 * TW) : 0);
    int s = 0;
    if (whole > 0) {
      do {
        lds_sync();
        v.template block<false>(a, k0 + slot, v0 + slot, 0, gq);
        slot = S_::kRound - slot;
      } while (++s < whole);
    }
    if (s < rounds) {
      do {
        lds_sync();
        const int tb = p.c0 + 64 * (s * TW + tw);
        if (tb < p.c1 && here) v.template block<true>(a, k0 + slot, v0 + slot, tb, gq);
        slot = S_::kRound - slot;
      } while (++s < rounds);
    }
    if (here) v.end(a, ((size_t)(p.group(a) + blockIdx.x) * RT + tile) * TW + tw, tile_g, n, gq);
  } while (p.next(a));
}

// ----------------------------------------------------------- mass kernel --
// The partial kernel's shares again, every row's maximum and sum known.
template <int D, int RT>
struct MassShape {
  static constexpr int TPW = q8_mass_waves(RT).tpw, RW = q8_mass_waves(RT).rw, TW = q8_mass_waves(RT).tw;
  static constexpr int CW = q8_mass_waves(RT).cw, kCompute = RW * TW, kThreads = (kCompute + CW) * 64;
  static constexpr int kBlock = Lay<D>::kSide, kRound = TW * kBlock, kLds = 2 * kRound;
  static constexpr int kDepth = 8 * (128 / D);
};

template <int D, int RT>
__global__ void __launch_bounds__((MassShape<D, RT>::kThreads)) __attribute__((amdgpu_waves_per_eu(2, 2)))
q8_mass_kernel(QArgs a) {
  typedef MassShape<D, RT> S_;
  constexpr int TPW = S_::TPW, TW = S_::TW;
  extern __shared__ __align__(1024) char s_ring[];  // [2][TW][64][D]

  Piece p;
  if (!p.first(a)) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr(s_ring));
  if (w >= S_::kCompute) {
    convert_share<D, TW, S_::CW, S_::kDepth, S_::kRound, S_::kBlock, false>(a, p, w - S_::kCompute, ring);
    return;
  }
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int tw = w % TW, rw = w / TW, t_first = rw * TPW;
  const uint32_t k0 = ring + tw * S_::kBlock + Lay<D>::k_lane(n, gq);
  const int token = 16 * (n / 4) + 4 * gq + n % 4;  // of a block, whose sum the lane gets
  uint32_t slot = 0;
  do {
    const int tiles = min(RT, a.RTT - p.rg * RT);
    const Holders h = holders(a, p.per, p.align, p.before, p.b, p.g * a.RG + p.rg, p.ctx);
    Query<D> q[TPW];
    int lim[TPW];
    float top[TPW], inv[TPW];
    bool real[TPW];
#pragma unroll
    for (int x = 0; x < TPW; ++x) {
      const int row = (p.rg * RT + t_first + x) * 16 + n;
      real[x] = t_first + x < tiles && row < a.R;
      load_query<D>(a, p.b, p.g, row, gq, q[x]);
      lim[x] = real[x] ? min(p.c1 - 1, p.ctx + row_t(a, row)) : -1;
    }
    tile_sums<RT, TPW>(a, h, t_first, tiles, real, n, gq, top, inv);
    const int vis_all = min(p.c1 - 1, p.ctx);
    float* mp = a.mpart + ((size_t)p.group(a) * S_::RW + rw) * a.mrows;
    for (int t0 = p.c0; t0 < p.c1; t0 += 64 * TW) {
      lds_sync();
      const uint32_t k = k0 + slot;
      slot = S_::kRound - slot;
      const int tb = t0 + 64 * tw;
      if (__builtin_amdgcn_readfirstlane(tb - p.c1) >= 0) continue;
      floatx4 S[TPW][4];
      scores<D, TPW, 8>(k, q, S);
      if (__builtin_amdgcn_readfirstlane(tb + 63 - vis_all) > 0) {
#pragma unroll
        for (int x = 0; x < TPW; ++x)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (16 * (j / 4) + j % 4 > lim[x] - tb - 4 * gq) S[x][j / 4][j % 4] = kNegInf;
      }
      // (NaN scores of padding rows, whose q is a real row's, make a token's sum NaN that the real row makes so)
      float sum[16];
#pragma unroll
      for (int x = 0; x < TPW; ++x)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float e = fast_exp2(fmaf(S[x][j / 4][j % 4], a.sl2, -top[x]));
          sum[j] = x ? fmaf(e, inv[x], sum[j]) : e * inv[x];
        }
      const float m = row_sums(sum, lane);
      if (tb + token < p.c1) mp[tb + token] = m;
    }
  } while (p.next(a));
}

// --------------------------------------------------------- finish kernel --
// A row of O: the sum over its records of the partials weighted by
// exp2(record's maximum - row maximum), over the rounded probabilities' sum, and
// the row's log-sum-exp.  Dividing by the sum of what P . V took in, and not of
// the unrounded probabilities, leaves a row that one token dominates with the
// rounding of its result alone.
//
// D / 4 lanes take a record, four columns each.  Every such set joins its own
// records (kU in flight: the kernel is bound by these round trips), then the
// sets of a wave and, with WPR waves a row, the waves through LDS.
struct RowSum {
  float m, z, zt;
  floatx4 o;
  bool nan;  // a record's values hold a NaN that not every row sees
};
__device__ __forceinline__ void join(RowSum& a, float m, float z, float zt, floatx4 o, bool nan) {
  a.nan |= nan;
  const float M = fmaxf(a.m, m), r = M == kNegInf ? 0.f : M;
  const float f = a.z != 0.f ? fast_exp2(a.m - r) : 0.f, g = z != 0.f ? fast_exp2(m - r) : 0.f;
  a.z = (a.z != 0.f ? a.z * f : 0.f) + (z != 0.f ? z * g : 0.f);
  a.zt = a.zt * f + zt * g;
  a.o = a.o * f + o * g;
  a.m = M;
}

template <int D, int RT, int WPR>
__device__ __forceinline__ void combine_rows(const QArgs& a, int wg, RowSum (*s_row)[D / 4]) {
  constexpr int LPR = D / 4, SG = 64 / LPR, TW = q8_waves(RT).tw, CW = q8_waves(RT).cw, kU = 8;
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane % LPR;
  const int id = wg * (kFinWaves / WPR) + w / WPR;  // (fewer than 2^22 rows)
  const bool row_here = id < a.B * a.Hkv * a.R;
  RowSum t{kNegInf, 0.f, 0.f, floatx4{0.f, 0.f, 0.f, 0.f}, false};
  int b = 0, g = 0, row = 0, ctx = 0;
  if (row_here) {
    const int bg = __builtin_amdgcn_readfirstlane(id / a.R);
    row = id - bg * a.R;
    b = bg / a.Hkv;
    g = bg - b * a.Hkv;
    const Shares s_ = q8_find<false>(a, Wave(a), 0, b);
    ctx = s_.ctx;
    const int rg = row / (16 * RT), tile = row / 16 - rg * RT;
    const Holders h = holders(a, s_.per, s_.align, s_.before, b, g * a.RG + rg, s_.ctx);
    const size_t rec = ((size_t)h.rec * RT + tile) * TW * 16 + row % 16;
    const int cnt = h.count * TW, sets = SG * WPR;
    for (int s0 = lane / LPR + SG * (w % WPR); s0 < cnt; s0 += kU * sets) {
      float2 v[kU];
      float zt[kU];
      uint32_t nan[kU];
      floatx4 o[kU];
#pragma unroll
      for (int j = 0; j < kU; ++j) {
        const int s = min(s0 + j * sets, cnt - 1);
        const size_t i = rec + (size_t)(s / TW * RT * TW + s % TW) * 16;
#pragma unroll
        for (int c = 0; c < CW; ++c) {
          const uint32_t x = a.nan[(h.rec + s / TW) * CW + c];
          nan[j] = c ? nan[j] | x : x;
        }
        v[j] = a.stats[i];
        zt[j] = a.zt[i];
        o[j] = *reinterpret_cast<const floatx4*>(a.opart + i * D + 4 * col);
      }
      float m = t.m;
#pragma unroll
      for (int j = 0; j < kU; ++j) m = fmaxf(m, v[j].x);
      const float r = m == kNegInf ? 0.f : m, f = t.z != 0.f ? fast_exp2(t.m - r) : 0.f;
      t.z = t.z != 0.f ? t.z * f : 0.f;
      t.zt *= f;
      t.o = t.o * f;
      t.m = m;
#pragma unroll
      for (int j = 0; j < kU; ++j)
        if (s0 + j * sets < cnt && v[j].y != 0.f) {  // (0: nothing that the row sees)
          const float e = fast_exp2(v[j].x - r);
          t.z = fmaf(v[j].y, e, t.z);
          t.zt = fmaf(zt[j], e, t.zt);
          t.nan |= nan[j] != 0;
          t.o = t.o + o[j] * e;
        }
    }
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
      floatx4 y;
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = __shfl_xor(t.o[k], o, 64);
      join(t, __shfl_xor(t.m, o, 64), __shfl_xor(t.z, o, 64), __shfl_xor(t.zt, o, 64), y, __shfl_xor(t.nan, o, 64));
    }
  }
  if constexpr (WPR > 1) {
    if (lane < LPR) s_row[w][lane] = t;
    __syncthreads();
    if (w % WPR) return;
    for (int k = 1; k < WPR; ++k) {
      const RowSum y = s_row[w + k][col];
      join(t, y.m, y.z, y.zt, y.o, y.nan);
    }
  }
  if (!row_here || lane >= LPR) return;
  const int tt = row_t(a, row), head = g * a.G + row - tt * a.G;
  constexpr int DPL = D / 16;
  if (t.nan) {  // the values past the context that the row sees, whose NaN codes counted as 0
    for (int j = ctx + 1; j <= ctx + tt; ++j) {
      bool flagged_before;  // by the partial kernel
      const int64_t r = unit_row(a, b, g, j & ~31, page_entry(a, b, j), flagged_before) + (j & 31);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = 4 * col + k;
        if ((a.c.vc[r * D + 16 * (c % DPL) + c / DPL] & 0x7f) == 0x7f) t.o[k] = __uint_as_float(0x7fc00000u);
      }
    }
  }
  const float inv = 1.f / t.zt;
  uint16_t* o = a.out + (((size_t)b * a.T + tt) * a.Hq + head) * D;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int c = 4 * col + k;
    o[16 * (c % DPL) + c / DPL] = f32_to_bf16(t.o[k] * inv);
  }
  if (a.lse && lane == 0) a.lse[((size_t)b * a.Hq + head) * a.T + tt] = (t.m + __log2f(t.z)) * kLn2;
}

// The mass of every cache row: the sum of its groups' and waves' partials in
// order (0 past the sequence).
template <int RT>
__device__ __forceinline__ void sum_mass(const QArgs& a, int id) {
  const int P = a.HR * q8_mass_waves(RT).rw;
  const int b = id / a.mass_per;
  const int64_t t0 = (int64_t)(id - b * a.mass_per) * a.mass_rows;
  const int N = clamp_ctx(a, a.ctx_len[b]) + a.T;
  const float* mp = a.mpart + (size_t)b * P * a.mrows;
  float* mass = a.mass + (size_t)b * a.c.n_cap;
  for (int64_t t = t0 + threadIdx.x; t < min(t0 + a.mass_rows, a.c.n_cap); t += kFinThreads) {
    constexpr int kU = 8;  // partials in flight
    float sum = 0.f;
    if (t < N)
      for (int p0 = 0; p0 < P; p0 += kU) {
        float v[kU];
#pragma unroll
        for (int j = 0; j < kU; ++j) v[j] = mp[(size_t)min(p0 + j, P - 1) * a.mrows + t];
#pragma unroll
        for (int j = 0; j < kU; ++j)
          if (p0 + j < P) sum += v[j];
      }
    mass[t] = sum;
  }
}

template <int D, int RT, int WPR>
__global__ void __launch_bounds__(kFinThreads) q8_finish_kernel(QArgs a) {
  __shared__ RowSum s_row[WPR > 1 ? kFinWaves : 1][D / 4];
  const int id = blockIdx.x;
  if (id < a.mass_wgs) sum_mass<RT>(a, id);
  else combine_rows<D, RT, WPR>(a, id - a.mass_wgs, s_row);
}

// ------------------------------------------------------------------ host --
typedef void (*QKernel)(QArgs);
struct QKernels {
  QKernel part, mass, finish[2];  // finish: one wave, or a workgroup, for a row
  int part_threads, mass_threads, part_lds, mass_lds;
};

template <int D, int RT>
QKernels kernels() {
  return {q8_part_kernel<D, RT>,
          q8_mass_kernel<D, RT>,
          {q8_finish_kernel<D, RT, 1>, q8_finish_kernel<D, RT, kFinWaves>},
          PartShape<D, RT>::kThreads,
          MassShape<D, RT>::kThreads,
          PartShape<D, RT>::kLds,
          MassShape<D, RT>::kLds};
}
template <int D>
QKernels pick(int RT) {
  switch (RT) {
    case 1: return kernels<D, 1>();
    case 2: return kernels<D, 2>();
    case 3: return kernels<D, 3>();
    case 4: return kernels<D, 4>();
    case 5: return kernels<D, 5>();
    case 6: return kernels<D, 6>();
    case 7: return kernels<D, 7>();
    case 8: return kernels<D, 8>();
    case 9: return kernels<D, 9>();
    default: return kernels<D, 10>();
  }
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
  a.HR = Hkv * p.RG;
  a.max_ctx = (int)max_ctx;
  a.wgs = p.wgs;
  a.sl2 = (float)((double)scale * kLog2e);
  a.mpart = reinterpret_cast<float*>(wsb + p.off_mpart);
  a.mrows = p.mrows;
  a.stats = reinterpret_cast<float2*>(wsb + p.off_stats);
  a.zt = reinterpret_cast<float*>(wsb + p.off_zt);
  a.nan = reinterpret_cast<uint32_t*>(wsb + p.off_nan);
  a.opart = reinterpret_cast<float*>(wsb + p.off_opart);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.mass = mass;
  a.status = status;
  a.mass_rows = (int)mass_rows(B, c.n_cap);
  a.mass_per = (int)mass_workgroups(c.n_cap, a.mass_rows);
  a.mass_wgs = mass ? B * a.mass_per : 0;
  const QKernels k = D == 128 ? pick<128>(p.RT) : pick<64>(p.RT);
  PVLM_HIP(allow_dynamic_lds(reinterpret_cast<const void*>(k.part), k.part_lds));
  hipLaunchKernelGGL(k.part, dim3(p.wgs), dim3(k.part_threads), k.part_lds, stream, a);
  PVLM_LAUNCHED();
  if (mass) {
    PVLM_HIP(allow_dynamic_lds(reinterpret_cast<const void*>(k.mass), k.mass_lds));
    hipLaunchKernelGGL(k.mass, dim3(p.wgs), dim3(k.mass_threads), k.mass_lds, stream, a);
    PVLM_LAUNCHED();
  }
  // a wave joins 16 records (8 at D = 64: 32) in one round of loads
  const bool wide = p.recs * q8_waves(p.RT).tw > (size_t)B * a.HR * 2 * 16;
  const int per_wg = wide ? 1 : kFinWaves, row_count = B * Hkv * p.R;
  hipLaunchKernelGGL(k.finish[wide], dim3(a.mass_wgs + (row_count + per_wg - 1) / per_wg), dim3(kFinThreads), 0, stream,
                     a);
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

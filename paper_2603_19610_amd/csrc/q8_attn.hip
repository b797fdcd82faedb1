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

__device__ __forceinline__ int64_t uniform64(int64_t x) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}

struct QArgs {
  const uint16_t* q;
  Q8Cache c;
  const int32_t* ctx_len;
  int B, T, Hq, Hkv, G, R;
  unsigned g_magic;  // row / G == row * g_magic >> 20 for row < 640 (2^20 / G + 1; G <= 640)
  int RTT, RG, HR;   // HR = Hkv * RG, the groups of a sequence
  int max_ctx, wgs;
  float sl2;         // scale * log2(e)
  float* mpart;      // [B][HR][waves][n_cap] mass of one wave's rows
  float2* stats;     // [record][tile][token wave][16] (log2-domain maximum, sum) of rows
  float* zt;         // the same sums of the probabilities as P . V takes them, rounded to bf16
  float* opart;      // [record][tile][token wave][16][D] sums of P . V relative to that maximum
  uint16_t* out;
  float* lse;
  float* mass;
  int32_t* status;
  int mass_wgs, mass_per, mass_rows;  // finish kernel: workgroups that sum the mass, of a sequence, rows of one
};

typedef const __attribute__((address_space(4))) int32_t* ConstInts;  // (uniform loads go through the scalar cache)
__device__ __forceinline__ int uniform_load(const int32_t* p, int64_t i) { return ((ConstInts)(uintptr_t)p)[i]; }

__device__ __forceinline__ int clamp_ctx(const QArgs& a, int ctx) { return ctx < 0 ? 0 : min(ctx, a.max_ctx); }
__device__ __forceinline__ int units_of(const QArgs& a, int ctx) { return (ctx + a.T + kQUnit - 1) / kQUnit; }

// Where the groups lie in the row of units.  Every wave finds its place from
// the lengths: sequence b's first group begins at HR * before.
struct Shares {
  int per;     // units of a workgroup
  int before;  // units (of one group each) of the sequences ahead of b
  int b, ctx;
};
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

// The sequence that holds the first unit of share wg (b = B: none), or sequence `seq`.
template <bool FIND_UNIT>
__device__ __forceinline__ Shares find(const QArgs& a, int wg, int seq) {
  const int lane = threadIdx.x & 63;
  Shares s;
  int total = 0, ctx = 0, u = 0, upto = 0;
  auto load = [&](int b0) {
    const bool here = b0 + lane < a.B;
    ctx = here ? clamp_ctx(a, a.ctx_len[b0 + lane]) : 0;
    u = here ? units_of(a, ctx) : 0;
    upto = wave_scan(u);
  };
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    load(b0);
    total += __builtin_amdgcn_readlane(upto, 63);
  }
  s.per = max((total * a.HR + a.wgs - 1) / a.wgs, kQMinUnits);
  s.before = 0;
  s.b = a.B;
  s.ctx = 0;
  // (wg * per stays within 32 bits: per exceeds total / wgs by less than one, or is the least share of few units)
  const int at = wg * s.per;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    if (a.B > 64) load(b0);
    int hit = seq - b0;
    if constexpr (FIND_UNIT) {
      const uint64_t m = __ballot(b0 + lane < a.B && (s.before + upto) * a.HR > at);
      hit = m ? __builtin_ctzll(m) : -1;
    }
    if (hit >= 0 && hit < 64) {
      s.before += __builtin_amdgcn_readlane(upto - u, hit);
      s.b = b0 + hit;
      s.ctx = __builtin_amdgcn_readlane(ctx, hit);
      break;
    }
    s.before += __builtin_amdgcn_readlane(upto, 63);
  }
  return s;
}

// A workgroup's share as pieces of groups, one after the other.
struct Piece {
  int b, g, rg, ctx;     // group: sequence, KV head, share of its row tiles
  int c0, c1;            // its tokens (c0 opens a unit)
  int left;              // units of the share from c0 on
  int before, per;       // units of the sequences ahead of b; of a share
  __device__ __forceinline__ void set(const QArgs& a) {
    const int N = ctx + a.T, u = c0 / kQUnit + left;
    c1 = __builtin_amdgcn_readfirstlane(u > N / kQUnit ? N : u * kQUnit);
  }
  // false where the share is empty
  __device__ __forceinline__ bool first(const QArgs& a) {
    const Shares s = find<true>(a, blockIdx.x, 0);
    if (s.b >= a.B) return false;
    b = s.b;
    ctx = s.ctx;
    before = s.before;
    per = left = s.per;
    const int u = units_of(a, ctx), off = (int)blockIdx.x * per - before * a.HR;
    const int hr = __builtin_amdgcn_readfirstlane(off / u);
    g = __builtin_amdgcn_readfirstlane(hr / a.RG);
    rg = hr - g * a.RG;
    c0 = __builtin_amdgcn_readfirstlane((off - hr * u) * kQUnit);
    set(a);
    return true;
  }
  // false where the share ends
  __device__ __forceinline__ bool next(const QArgs& a) {
    left -= (c1 - c0 + kQUnit - 1) / kQUnit;
    if (left <= 0) return false;
    if (++rg == a.RG) {
      rg = 0;
      if (++g == a.Hkv) {
        g = 0;
        before += units_of(a, ctx);
        if (++b == a.B) return false;
        ctx = __builtin_amdgcn_readfirstlane(clamp_ctx(a, uniform_load(a.ctx_len, b)));
      }
    }
    c0 = 0;
    set(a);
    return true;
  }
  __device__ __forceinline__ int group(const QArgs& a) const { return (b * a.Hkv + g) * a.RG + rg; }
};

// The workgroups that hold pieces of a group (hr = g * RG + rg), and its first record.
struct Holders {
  int rec, count;
};
__device__ __forceinline__ Holders holders(const QArgs& a, int per, int before, int b, int hr, int ctx) {
  const int u = units_of(a, ctx), start = before * a.HR + hr * u;
  const int w0 = start / per, w1 = (start + u - 1) / per;
  return {b * a.HR + hr + w0, w1 - w0 + 1};
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int row_t(const QArgs& a, int row) { return (int)((unsigned)row * a.g_magic >> 20); }

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
  static constexpr int CH = D / 16, LR = 256 / D;  // chunks of a row, rows of a line
  static __device__ __forceinline__ int kkey(int line) { return (line * LR >> 2) & 15; }
  static __device__ __forceinline__ int vkey(int line) {
    if constexpr (D == 128) return (line & 3) | ((line >> 1) & 4);
    else return line & 3;
  }
  // Where a lane's reads of a block begin (of K's chunk NC gq of row 4 n, and of
  // V's first column pair of rows 16 gq + ...), from the block's own start.  The
  // others differ by a few bits of the position, so by an exclusive or of the
  // address (blocks start at multiples of 256 bytes), and by whole lines.
  static constexpr int NC = D / 64;  // 16-byte chunks of a lane's part of a key row
  static __device__ __forceinline__ uint32_t k_lane(int n, int gq) {
    const int line = 4 * n / LR;
    return line * 256 + ((NC * gq ^ kkey(line)) << 4);
  }
  static __device__ __forceinline__ uint32_t k_at(uint32_t first, int tt, int c) {
    return (first ^ (((tt % LR) * CH + c) << 4)) + tt / LR * 256;
  }
  static __device__ __forceinline__ uint32_t v_lane(int n, int gq) {
    const int row = 16 * gq + n / 2, line = row / LR;
    return line * 256 + ((((row % LR) * CH) ^ vkey(line)) << 4) + 8 * (n & 1);
  }
  // rows 8 ks on, column 16 jd + n: 8 ks rows are 8 / LR lines, which change V's key at D = 64
  static __device__ __forceinline__ uint32_t v_at(uint32_t first, int ks, int jd) {
    const int key = D == 128 ? 0 : vkey(8 * ks / LR);
    return (first ^ ((jd ^ key) << 4)) + ks * (8 / LR) * 256;
  }
};

template <typename T>
__device__ __forceinline__ T lds_read(uint32_t at) {
  return *(const __attribute__((address_space(3))) T*)at;
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

// Maximum over the four lanes l, l^16, l^32, l^48; NaN if one is.
__device__ __forceinline__ float rows4_maximum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __builtin_elementwise_maximum(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __builtin_elementwise_maximum(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Eight codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8 to_bf16(uint32_t lo, uint32_t hi, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, unit, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, unit, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, unit, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, unit, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Scores of one block against a wave's row tiles: S[x][tt][i] is token
// 16 gq + 4 i + tt.  The keys are converted once for all tiles.
template <int D, int TPW>
__device__ __forceinline__ void scores(uint32_t k_first, uint32_t exps, const Query<D> (&q)[TPW], floatx4 (&S)[TPW][4]) {
  constexpr int NC = Lay<D>::NC;
  uintx4 k[4][NC];
#pragma unroll
  for (int tt = 0; tt < 4; ++tt)
#pragma unroll
    for (int c = 0; c < NC; ++c) k[tt][c] = lds_read<uintx4>(Lay<D>::k_at(k_first, tt, c));
#pragma unroll
  for (int x = 0; x < TPW; ++x)
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) S[x][tt] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
      const float unit = q8_unit((exps >> (8 * tt)) & 0xffu);
      const bf16x8 k0 = to_bf16(k[tt][c].x, k[tt][c].y, unit), k1 = to_bf16(k[tt][c].z, k[tt][c].w, unit);
#pragma unroll
      for (int x = 0; x < TPW; ++x) {
        S[x][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, q[x].s[2 * c], S[x][tt], 0, 0, 0);
        S[x][tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, q[x].s[2 * c + 1], S[x][tt], 0, 0, 0);
      }
    }
}

// Eight consecutive tokens (rows 16 gq + 8 ks on) of column 16 jd + n.
template <int D>
__device__ __forceinline__ intx2 read_v(uint32_t v_first, int ks, int jd) {
  typedef __attribute__((address_space(3))) intx2* lds_v2;
  return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_v2)Lay<D>::v_at(v_first, ks, jd));
}

// Two columns' operands of a block, as codes.
struct VPair {
  intx2 v[4];
};
template <int D>
__device__ __forceinline__ VPair read_pair(uint32_t v_first, int pair) {
  VPair p;
#pragma unroll
  for (int i = 0; i < 4; ++i) p.v[i] = read_v<D>(v_first, i & 1, 2 * pair + i / 2);
  return p;
}

// O += P' . V over one block; P'[ks] holds tokens 16 gq + 8 ks + j.  The next
// two columns are read while two are multiplied; the barriers keep the compiler
// from reading all of them at once, for which there are no registers.
//
// MASKED: of the tokens that not every row sees, NaN codes count as 0 (0 times
// NaN would be NaN for rows that do not see them); mask has 0xff in the bytes
// of those tokens.  Returns whether there were any: the finish kernel then
// gives the rows that see them their NaN.
template <int D, bool MASKED>
__device__ __forceinline__ uint32_t weigh(uint32_t v_first, const bf16x8 (&P)[2], VPair cur,
                                          const uint32_t (&mask)[4], floatx4 (&O)[D / 16]) {
  uint32_t bad = 0;
#pragma unroll
  for (int pair = 0; pair < D / 32; ++pair) {
    VPair next;
    if (pair + 1 < D / 32) next = read_pair<D>(v_first, pair + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t v0 = cur.v[i][0], v1 = cur.v[i][1];
      if constexpr (MASKED) {
        const uint32_t b0 = nan_codes(v0) & mask[2 * (i & 1)], b1 = nan_codes(v1) & mask[2 * (i & 1) + 1];
        bad |= b0 | b1;
        v0 &= ~(b0 | (b0 - (b0 >> 7)));
        v1 &= ~(b1 | (b1 - (b1 >> 7)));
      }
      const bf16x8 b = to_bf16(v0, v1, 1.f);
      const int jd = 2 * pair + i / 2;
      O[jd] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(P[i & 1], b, O[jd], 0, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    cur = next;
  }
  return bad;
}

// (maximum, sum) of two sets of scores.  A sum of 0 belongs to one of which the
// row sees nothing; NaN passes.
__device__ __forceinline__ void join(float& m, float& z, float m2, float z2) {
  const float M = fmaxf(m, m2), r = M == kNegInf ? 0.f : M;
  z = (z != 0.f ? z * fast_exp2(m - r) : 0.f) + (z2 != 0.f ? z2 * fast_exp2(m2 - r) : 0.f);
  m = M;
}
// log2-sum-exp of row n of a wave's tiles over a group's records, the lane
// groups taking them in turn, with many loads in flight (+inf for padding rows:
// their probabilities are 0).
template <int RT, int TPW>
__device__ __forceinline__ void tile_lse(const QArgs& a, const Holders& h, int tile0, int tiles, const bool (&real)[TPW],
                                         int n, int gq, float (&lse)[TPW]) {
  constexpr int kU = TPW == 1 ? 8 : 4;  // records of every tile in flight
  const int cnt = 2 * h.count;  // (of a tile that one wave has the first of every two)
  const float2* st = a.stats + (size_t)h.rec * RT * 2 * 16 + n;
  float M[TPW], Z[TPW];
#pragma unroll
  for (int x = 0; x < TPW; ++x) M[x] = kNegInf, Z[x] = 0.f;
  for (int s0 = gq; s0 < cnt; s0 += 4 * kU) {
    float2 v[kU][TPW];
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      const int s = min(s0 + 4 * j, cnt - 1);
      const float2* r = st + (size_t)(s / 2 * RT * 2 + s % 2) * 16;
#pragma unroll
      for (int x = 0; x < TPW; ++x) {
        const int tile = min(tile0 + x, tiles - 1);
        v[j][x] = tile < q8_full_tiles(RT) && s % 2 ? make_float2(kNegInf, 0.f) : r[tile * 2 * 16];
      }
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
    lse[x] = real[x] ? M[x] + __log2f(Z[x]) : __builtin_huge_valf();
  }
}

// Sum over the 16 rows (lanes n) of a block's values, of token `lane` of the
// block: each step a lane keeps half of its values, chosen by one bit of n, and
// adds its partner's copy of that half.
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

// ------------------------------------------------------------------ ring --
// A stage is 128 tokens' codes and exponents.  The loading waves copy stages
// into an LDS ring by global->LDS loads of 1 KB (16 bytes a lane, in LDS order:
// the lanes fetch permuted chunks), so loads stay in flight behind the other
// waves' arithmetic.  One barrier a stage hands a landed slot over and an
// emptied one back.
template <int D>
struct Ring {
  static constexpr int ST = 128, KB = ST * D;          // tokens of a stage, bytes of its codes (K or V)
  static constexpr int NI = KB / 1024;                 // load instructions for them
  static constexpr int kSide = KB + 256;               // ... and exponents (ST bytes; a load writes 256)
  static constexpr int RPI = 1024 / D, IPU = 32 / RPI; // rows of an instruction, instructions of a unit
};

// Loads as inline asm: the compiler neither counts them nor waits for them; the
// loading wave, which issues no other vector memory operation (but to flag an
// error, which only makes a wait longer), counts them itself.  An LDS load may
// not directly follow the scalar write of M0 that gives its LDS address (one
// wait state, hence the s_nop).
__device__ __forceinline__ void lds_load16(int64_t base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" : : "s"(lds), "v"(p) : "memory", "m0");
}
// Wait until at most `stages` later stages' loads (N each) are in flight.
template <int N, int MOST>
__device__ __forceinline__ void wait_stage(int stages) {
  static_assert(MOST * N < 64, "vmcnt holds 6 bits");
  if constexpr (MOST == 0) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  } else {
    if (stages >= MOST) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N * MOST) : "memory");
    else wait_stage<N, MOST - 1>(stages);
  }
}

// The row index (in rows of codes) of the unit that token t opens.  A page entry
// outside the pool is flagged and clamped into it.
__device__ __forceinline__ int64_t unit_row(const QArgs& a, int b, int g, int t) {
  if (!a.c.table) return ((int64_t)b * a.Hkv + g) * a.c.n_cap + t;
  int pg = uniform_load(a.c.table, (int64_t)b * a.c.max_pages + (t >> a.c.shift));
  if (pg < 0 || pg >= a.c.n_pages) {
    dev_flag(a.status, PVLM_DEV_RANGE);
    pg = pg < 0 ? 0 : (int)(a.c.n_pages - 1);
  }
  return (((int64_t)pg * a.Hkv + g) << a.c.shift) + (t & ((1 << a.c.shift) - 1));
}

// One side (K or V) of the stage at token t0 into LDS.  Rows past the piece repeat its last one;
// exponents are read in groups of four rows, which never leave a unit.
template <int D, bool IS_K>
__device__ __forceinline__ void issue_stage(const QArgs& a, const Piece& p, int t0, const uint32_t (&off)[IS_K ? 2 : 1][Ring<D>::IPU],
                                            uint32_t lds, int lane) {
  typedef Ring<D> R_;
  typedef Lay<D> L;
  const uint8_t* codes = IS_K ? a.c.kc : a.c.vc;
  const uint8_t* exps = IS_K ? a.c.ke : a.c.ve;
  const int last = p.c1 - 1;
  int64_t row[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) row[u] = unit_row(a, p.b, p.g, min(t0 + 32 * u, last & ~31));
  const bool whole = t0 + R_::ST <= p.c1;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int64_t base = uniform64((int64_t)(uintptr_t)(codes + row[u] * D));
#pragma unroll
    for (int i = 0; i < R_::IPU; ++i) {
      uint32_t o = off[IS_K ? u & 1 : 0][i];
      if (!whole) {  // (offsets are row * D + 16 * chunk, rows counted from the unit)
        const int most = max(0, last - (t0 + 32 * u));
        const int at = t0 + 32 * u > last ? (last & 31) : min((int)(o / D), most);
        o = at * D + o % D;
      }
      lds_load16(base, o, lds + (u * R_::IPU + i) * 1024);
    }
  }
  // lane l: rows 4 l .. 4 l + 3 (lanes past the stage repeat)
  const int l = lane & 31, u = l >> 3;
  const int64_t r = u == 0 ? row[0] : u == 1 ? row[1] : u == 2 ? row[2] : row[3];
  lds_load4(exps + r + 4 * (l & 7), lds + R_::KB);
}

// What a loading wave does: every stage of the workgroup's share, kSlots - 1
// stages ahead, in STRIDE bytes a slot.
template <int D, bool IS_K, int SLOTS, int STRIDE>
__device__ __forceinline__ void load_share(const QArgs& a, Piece p, char* ring) {
  typedef Ring<D> R_;
  typedef Lay<D> L;
  const int lane = threadIdx.x & 63;
  // offsets of a lane's pieces in a unit; K's order repeats every two units, V's every one
  uint32_t off[IS_K ? 2 : 1][R_::IPU];
#pragma unroll
  for (int u = 0; u < (IS_K ? 2 : 1); ++u)
#pragma unroll
    for (int i = 0; i < R_::IPU; ++i) {
      const int line = (32 * u + i * R_::RPI) / L::LR + lane / 16;
      const int at = (lane & 15) ^ (IS_K ? L::kkey(line) : L::vkey(line));
      off[u][i] = (line * L::LR - 32 * u + at / L::CH) * D + 16 * (at % L::CH);
    }
  const uint32_t base = __builtin_amdgcn_readfirstlane(lds_addr(ring));
  __builtin_amdgcn_s_setprio(3);  // the loads go out before the other waves' arithmetic
  __builtin_amdgcn_s_waitcnt(0);  // the counts start from zero
  int issued = 0, t0 = p.c0;
  bool more = true;
  auto issue = [&]() {
    issue_stage<D, IS_K>(a, p, t0, off, base + (issued % SLOTS) * STRIDE, lane);
    ++issued;
    t0 += R_::ST;
    if (t0 >= p.c1) {
      more = p.next(a);
      t0 = p.c0;
    }
  };
  for (int s = 0; s < SLOTS - 1 && more; ++s) issue();
  for (int s = 0; s < issued; ++s) {
    wait_stage<R_::NI + 1, SLOTS - 2>(issued - 1 - s);
    lds_sync();  // stage s has landed; every wave is done with stage s - 1
    if (more) issue();
  }
}

// -------------------------------------------------------- partial kernel --
template <int D>
struct PartRing {
  static constexpr int kSlots = D == 128 ? 4 : 8, kStride = 2 * Ring<D>::kSide, kLds = kSlots * kStride;
};

// A computing wave's tile and blocks.  Wave w runs on SIMD w mod 4, the loading
// waves on SIMDs 2 and 3 of three that hold ten others: waves of whole tiles
// are placed first on those, then on 0 and 1 (RT = 6: 2 + 2 half tiles a SIMD).
struct Role {
  int tile, block, blocks;
};
template <int RT>
__device__ __forceinline__ Role role(int w) {
  constexpr int full = q8_full_tiles(RT);
  constexpr int order[8] = {2, 3, 0, 1, 6, 7, 4, 5};
  int ahead = 0;  // waves of whole tiles before w
#pragma unroll
  for (int k = 0; k < full; ++k) {
    if (order[k] == w) return {k, 0, 2};
    ahead += order[k] < w;
  }
  return {full + (w - ahead) / 2, (w - ahead) % 2, 1};
}

// A wave's state: a row tile against the tokens of its blocks.
template <int D>
struct PartWave {
  static constexpr int DPL = D / 16;
  Query<D> q[1];
  int lim;  // last token that the lane's row sees
  int ctx;  // last token that every row sees
  float ref, z;
  floatx4 O[DPL], zt;
  uint32_t bad;  // a NaN value that not every row sees
  uint32_t k_lane, v_lane;

  __device__ __forceinline__ void begin(const QArgs& a, const Piece& p, int tile, int n, int gq) {
    ctx = p.ctx;
    bad = 0;
    k_lane = Lay<D>::k_lane(n, gq);
    v_lane = Lay<D>::v_lane(n, gq);
    const int row = tile * 16 + n;
    load_query<D>(a, p.b, p.g, row, gq, q[0]);
    lim = row < a.R ? min(p.c1 - 1, p.ctx + row_t(a, row)) : -1;
    ref = kNegInf;
    z = 0.f;
    zt = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int jd = 0; jd < DPL; ++jd) O[jd] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // The block of tokens tb .. tb + 63, block x of the stage at LDS address `at`.  TAIL: some row does not see all of them.
  template <bool TAIL>
  __device__ __forceinline__ void block(const QArgs& a, uint32_t at, int tb, int x, int n, int gq) {
    typedef Ring<D> R_;
    const uint32_t kb = at + x * 64 * D, vb = kb + R_::kSide, eb = at + R_::KB + x * 64;
    const uint32_t ke = lds_read<uint32_t>(eb + 4 * n);
    const uintx4 ve = lds_read<uintx4>(eb + R_::kSide + 16 * gq);
    floatx4 S1[1][4];
    scores<D, 1>(kb + k_lane, ke, q, S1);
    floatx4(&S)[4] = S1[0];
    if constexpr (TAIL) {  // the lane's token j is visible iff j <= lim - tb - 16 gq
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (j > lim - tb - 16 * gq) S[j % 4][j / 4] = kNegInf;
    }
    float mx = kNegInf;  // (the maximum that passes NaN on: the other one has every operand canonicalised first)
#pragma unroll
    for (int j = 0; j < 16; ++j) mx = __builtin_elementwise_maximum(mx, S[j / 4][j % 4]);
    mx = rows4_maximum(mx) * a.sl2;
    if (__any(mx > ref + kRefSlack)) {  // the first block, and seldom after it
      const float nm = fmaxf(ref, mx);
      const float al = ref == kNegInf ? 0.f : fast_exp2(ref - nm);
      z *= al;
      ref = nm;
      floatx4 f;
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = __shfl(al, 4 * gq + i, 64);
      zt = zt * f;
#pragma unroll
      for (int jd = 0; jd < DPL; ++jd) O[jd] = O[jd] * f;
    }
    const VPair v0 = read_pair<D>(vb + v_lane, 0);
    bf16x8 ones;
#pragma unroll
    for (int j = 0; j < 8; ++j) ones[j] = static_cast<__bf16>(1.f);
    const float r = ref == kNegInf ? 0.f : ref;  // no visible token yet: P = 0
    bf16x8 pz[2], pv[2];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float e = fast_exp2(fmaf(S[j % 4][j / 4], a.sl2, -r));
      z += e;
      pz[j / 8][j % 8] = static_cast<__bf16>(e);
      float y = e * q8_unit((ve[j / 4] >> (8 * (j % 4))) & 0xffu);
      if constexpr (TAIL)
        if (j > lim - tb - 16 * gq) y = 0.f;  // (an unwritten row's exponent may be anything)
      pv[j / 8][j % 8] = static_cast<__bf16>(y);
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) zt = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pz[ks], ones, zt, 0, 0, 0);
    uint32_t mask[4] = {0u, 0u, 0u, 0u};
    if constexpr (TAIL) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int o = ctx - tb - 16 * gq - 4 * k;  // tokens 4 k + j, j <= o, are seen by every row
        mask[k] = o >= 3 ? 0u : o < 0 ? ~0u : ~0u << (8 * (o + 1));
      }
    }
    bad |= weigh<D, TAIL>(vb + v_lane, pv, v0, mask, O);
  }

  __device__ __forceinline__ void end(const QArgs& a, size_t rec, int tile, int n, int gq) {
    const bool nan = __any(bad);
    const float zz = rows4_sum(z);
    rec *= 16;
    if (gq == 0) a.stats[rec + n] = make_float2(ref, zz);
    // (a negative sum: the rows' values hold a NaN that not every row sees)
    if (n == 0) *reinterpret_cast<floatx4*>(a.zt + rec + 4 * gq) = nan ? -zt : zt;
    // position DPL n + jd of a stored row holds column 16 jd + n
    float* op = a.opart + rec * D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (tile * 16 + 4 * gq + i < a.R)
#pragma unroll
        for (int h = 0; h < DPL / 4; ++h)
          *reinterpret_cast<float4*>(op + (4 * gq + i) * D + DPL * n + 4 * h) =
              make_float4(O[4 * h][i], O[4 * h + 1][i], O[4 * h + 2][i], O[4 * h + 3][i]);
  }
};

template <int RT>
struct PartShape {
  static constexpr int kCompute = q8_part_waves(RT), kThreads = (kCompute + 2) * 64;
  // waves of a SIMD; two at least, so that a wave's registers are all of one kind
  static constexpr int kPerEu = kCompute <= 6 ? 2 : 3;
};

template <int D, int RT>
__global__ void __launch_bounds__((PartShape<RT>::kThreads))
__attribute__((amdgpu_waves_per_eu(PartShape<RT>::kPerEu, PartShape<RT>::kPerEu))) q8_part_kernel(QArgs a) {
  typedef Ring<D> R_;
  typedef PartRing<D> P_;
  constexpr int kCompute = PartShape<RT>::kCompute;
  extern __shared__ __align__(1024) char s_ring[];  // [slot][K, V][codes, exponents]

  Piece p;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (blockIdx.x == 0 && w == 0)
    for (int b = threadIdx.x; b < a.B; b += 64)
      if (a.ctx_len[b] < 0 || a.ctx_len[b] > a.max_ctx) dev_flag(a.status, PVLM_DEV_RANGE);
  if (!p.first(a)) return;
  if (w == kCompute) {
    load_share<D, true, P_::kSlots, P_::kStride>(a, p, s_ring);
    return;
  }
  if (w == kCompute + 1) {
    load_share<D, false, P_::kSlots, P_::kStride>(a, p, s_ring + R_::kSide);
    return;
  }
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const Role my = role<RT>(w);
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr(s_ring));
  int slot = 0;
  do {
    const int tile = p.rg * RT + my.tile;  // of the KV head
    const bool live = tile < a.RTT;
    PartWave<D> v;
    v.begin(a, p, tile, n, gq);
    // the wave's stages whose blocks every row sees whole, then the others (two
    // loops with their test at the end: joined, or with the test ahead, the
    // compiler copies all of O in every round)
    const int nst = __builtin_amdgcn_readfirstlane((p.c1 - p.c0 + R_::ST - 1) / R_::ST);
    const int last = 64 * (my.block + my.blocks) - 1;  // of the wave's tokens in a stage
    const int whole = __builtin_amdgcn_readfirstlane(live ? (min(p.c1 - 1, p.ctx) - last - p.c0 + R_::ST) / R_::ST : 0);
    auto stage = [&]() {
      lds_sync();
      const uint32_t at = ring + slot * P_::kStride;
      slot = slot + 1 == P_::kSlots ? 0 : slot + 1;
      return at;
    };
    int s = 0;
    if (whole > 0) {
      do {
        const uint32_t at = stage();
        int x = 0;
        do v.template block<false>(a, at, 0, my.block + x, n, gq);
        while (++x < my.blocks);
      } while (++s < whole);
    }
    if (s < nst) {
      do {
        const uint32_t at = stage();
        if (live) {
          int x = 0;
          do {
            const int tb = p.c0 + s * R_::ST + 64 * (my.block + x);
            if (tb < p.c1) v.template block<true>(a, at, tb, my.block + x, n, gq);
          } while (++x < my.blocks);
        }
      } while (++s < nst);
    }
    if (live) v.end(a, ((size_t)(p.group(a) + blockIdx.x) * RT + my.tile) * 2 + my.block, tile, n, gq);
  } while (p.next(a));
}

// ----------------------------------------------------------- mass kernel --
// The partial kernel's shares again, every row's log-sum-exp known.
template <int D>
struct MassRing {
  static constexpr int kSlots = D == 128 ? 4 : 8, kStride = Ring<D>::kSide, kLds = kSlots * kStride;
};

template <int RT>
struct MassShape {
  static constexpr int TPW = q8_mass_tiles(RT), RW = q8_mass_rows(RT), kCompute = 2 * RW, kThreads = (kCompute + 1) * 64;
};

template <int D, int RT>
__global__ void __launch_bounds__((MassShape<RT>::kThreads)) __attribute__((amdgpu_waves_per_eu(2, 2)))
q8_mass_kernel(QArgs a) {
  typedef Ring<D> R_;
  typedef MassRing<D> P_;
  constexpr int TPW = MassShape<RT>::TPW, RW = MassShape<RT>::RW, kCompute = MassShape<RT>::kCompute;
  extern __shared__ __align__(1024) char s_ring[];

  Piece p;
  if (!p.first(a)) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (w == kCompute) {
    load_share<D, true, P_::kSlots, P_::kStride>(a, p, s_ring);
    return;
  }
  const int lane = threadIdx.x & 63, n = lane & 15, gq = lane >> 4;
  const int tw = w % 2, rw = w / 2, t_first = rw * TPW;
  const uint32_t ring = __builtin_amdgcn_readfirstlane(lds_addr(s_ring)), k_lane = Lay<D>::k_lane(n, gq);
  int slot = 0;
  do {
    const int tiles = min(RT, a.RTT - p.rg * RT);
    const Holders h = holders(a, p.per, p.before, p.b, p.g * a.RG + p.rg, p.ctx);
    Query<D> q[TPW];
    int lim[TPW];
    float lse[TPW];
    bool real[TPW];
#pragma unroll
    for (int x = 0; x < TPW; ++x) {
      const int row = (p.rg * RT + t_first + x) * 16 + n;
      real[x] = t_first + x < tiles && row < a.R;
      load_query<D>(a, p.b, p.g, row, gq, q[x]);
      lim[x] = real[x] ? min(p.c1 - 1, p.ctx + row_t(a, row)) : -1;
    }
    tile_lse<RT, TPW>(a, h, t_first, tiles, real, n, gq, lse);
    const int vis_all = min(p.c1 - 1, p.ctx);
    float* mp = a.mpart + ((size_t)p.group(a) * RW + rw) * a.c.n_cap;
    for (int t0 = p.c0; t0 < p.c1; t0 += R_::ST) {
      lds_sync();
      const uint32_t at = ring + slot * P_::kStride;
      slot = slot + 1 == P_::kSlots ? 0 : slot + 1;
      const int tb = t0 + 64 * tw;
      if (__builtin_amdgcn_readfirstlane(tb - p.c1) >= 0) continue;
      const uint32_t ke = lds_read<uint32_t>(at + R_::KB + 64 * tw + 4 * n);
      floatx4 S[TPW][4];
      scores<D, TPW>(at + tw * 64 * D + k_lane, ke, q, S);
      if (__builtin_amdgcn_readfirstlane(tb + 63 - vis_all) > 0) {
#pragma unroll
        for (int x = 0; x < TPW; ++x)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j > lim[x] - tb - 16 * gq) S[x][j % 4][j / 4] = kNegInf;
      }
      // (NaN scores of padding rows, whose q is a real row's, make a token's sum NaN that the real row makes so)
      float sum[16];
#pragma unroll
      for (int x = 0; x < TPW; ++x)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float e = fast_exp2(fmaf(S[x][j % 4][j / 4], a.sl2, -lse[x]));
          sum[j] = x ? sum[j] + e : e;
        }
      const float m = row_sums(sum, lane);
      if (tb + lane < p.c1) mp[tb + lane] = m;
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
  constexpr int LPR = D / 4, SG = 64 / LPR, kU = 8;
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
    const Shares s_ = find<false>(a, 0, b);
    ctx = s_.ctx;
    const int rg = row / (16 * RT), tile = row / 16 - rg * RT;
    const Holders h = holders(a, s_.per, s_.before, b, g * a.RG + rg, s_.ctx);
    const int tw = tile < q8_full_tiles(RT) ? 1 : 2;  // records of a tile in each of the group's
    const size_t rec = ((size_t)h.rec * RT + tile) * 2 * 16 + row % 16;
    const int cnt = h.count * tw, sets = SG * WPR;
    for (int s0 = lane / LPR + SG * (w % WPR); s0 < cnt; s0 += kU * sets) {
      float2 v[kU];
      float zt[kU];
      floatx4 o[kU];
#pragma unroll
      for (int j = 0; j < kU; ++j) {
        const int s = min(s0 + j * sets, cnt - 1);
        const size_t i = rec + (size_t)(tw == 1 ? 2 * RT * s : s / 2 * RT * 2 + s % 2) * 16;
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
          t.zt = fmaf(fabsf(zt[j]), e, t.zt);
          t.nan |= zt[j] < 0.f;
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
      const int64_t r = unit_row(a, b, g, j & ~31) + (j & 31);
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
  const int P = a.HR * q8_mass_rows(RT);
  const int b = id / a.mass_per;
  const int64_t t0 = (int64_t)(id - b * a.mass_per) * a.mass_rows;
  const int N = clamp_ctx(a, a.ctx_len[b]) + a.T;
  const float* mp = a.mpart + (size_t)b * P * a.c.n_cap;
  float* mass = a.mass + (size_t)b * a.c.n_cap;
  for (int64_t t = t0 + threadIdx.x; t < min(t0 + a.mass_rows, a.c.n_cap); t += kFinThreads) {
    constexpr int kU = 8;  // partials in flight
    float sum = 0.f;
    if (t < N)
      for (int p0 = 0; p0 < P; p0 += kU) {
        float v[kU];
#pragma unroll
        for (int j = 0; j < kU; ++j) v[j] = mp[(size_t)min(p0 + j, P - 1) * a.c.n_cap + t];
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
  return {q8_part_kernel<D, RT>, q8_mass_kernel<D, RT>, {q8_finish_kernel<D, RT, 1>, q8_finish_kernel<D, RT, kFinWaves>}, PartShape<RT>::kThreads,
          MassShape<RT>::kThreads, PartRing<D>::kLds, MassRing<D>::kLds};
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
    default: return kernels<D, 9>();
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
  a.stats = reinterpret_cast<float2*>(wsb + p.off_stats);
  a.zt = reinterpret_cast<float*>(wsb + p.off_zt);
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
  const bool wide = p.recs * 2 > (size_t)B * a.HR * 2 * 16;
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

// Launch plan of verify attention over an 8-bit cache: how its row tiles and
// tokens are spread over workgroups, and where the workspace's areas lie.  Plain
// C++, so that the plan can be run over all sizes without a GPU, and with it the
// arithmetic by which the kernels find their shares.
#pragma once

#include "verify_plan.h"

namespace pvlm {

// The tokens of every group (sequence, KV head, share of its query rows) are
// counted in units of 32 (a page holds whole ones), all groups in a row, and
// every workgroup takes an equal share of that row, whatever the lengths are:
// a ragged batch keeps no compute unit idle, and a workgroup may end one
// group and begin the next (unless the shares are enough for every group to begin
// its own).  The shares follow from the lengths on the device.
constexpr int kQUnit = 32;
constexpr int kQMinUnits = 2;  // least share: one 64-token block
constexpr int kQMaxRT = 10;    // 16-row tiles of a workgroup

// The waves of a workgroup: RW for its row tiles, with TPW tiles each, times TW
// for as many blocks of 64 tokens at a time (a round), and CW that convert K's
// halves of these blocks and CW for V's.
struct QWaves {
  int tpw, rw, tw, cw;
};
// The partial kernel's: sixteen waves, four a SIMD, at most.  With few tiles the
// conversion bounds a round, and every half has a wave of its own (3 tiles, 117 MB
// of each of K and V: 55 us, with two halves a wave 60).  Two tiles a wave, which
// read a block once for both, are two a SIMD or spill: 9 tiles over 132K tokens
// took 126 to 146 us where one, at that step, took 124 to 128 (now 112 to 121).
constexpr QWaves q8_waves(int RT) { return {1, RT, RT <= 6 ? 2 : 1, RT <= 4 ? 4 : 2}; }
// The mass kernel's, with K alone and no results to hold: up to three tiles a
// wave, which sum their rows together, and two waves a SIMD.
constexpr QWaves q8_mass_waves(int RT) {
  const int rw = (RT + 2) / 3;
  return {(RT + rw - 1) / rw, rw, rw <= 3 ? 2 : 1, 2};
}

struct QSplit {
  int G, R;         // query heads of a KV head, and its query rows G * T
  int RTT, RG, RT;  // their 16-row tiles, the workgroups that share them, and the tiles of one
  int wgs;          // workgroups of the partial and mass kernels
  size_t recs;      // partial results of RT tiles: group x of workgroup w is number x + w
  int64_t mrows;    // tokens of a row of mass partials: no sequence has more
  size_t off_mpart, off_stats, off_zt, off_nan, off_opart, bytes;
};

// What the shares follow from, beside the lengths.
struct QShape {
  int B, T, Hkv, RG;  // RG: workgroups that share a KV head's row tiles
  int HR;             // Hkv * RG, the groups of a sequence
  int wgs, max_ctx;
};

#if defined(__HIPCC__)
#define PVLM_Q8_FN __host__ __device__ __forceinline__
#else
#define PVLM_Q8_FN inline
#endif

// A value that a wave's lanes have in common, held once for the wave.
PVLM_Q8_FN int q8_uniform(int x) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_readfirstlane(x);
#else
  return x;
#endif
}

PVLM_Q8_FN int clamp_ctx(const QShape& a, int ctx) { return ctx < 0 ? 0 : ctx < a.max_ctx ? ctx : a.max_ctx; }
PVLM_Q8_FN int units_of(const QShape& a, int ctx) { return (ctx + a.T + kQUnit - 1) / kQUnit; }
PVLM_Q8_FN int aligned(int units, int align) { return align == 1 ? units : (units + align - 1) / align * align; }

// Where the groups lie in the row of units.  Every wave finds its place from
// the lengths: sequence b's first group begins at HR * before.  Where the shares
// are enough for it, every group begins a share of its own (align = per; its units
// count as a multiple of that): a share that ends one group and begins another
// takes a round and the statistics of both (72 rows over 12800 tokens, 8 groups:
// mass kernel 15.8 us, aligned 13.0).
struct Shares {
  int per;     // units of a workgroup
  int align;   // what a group's units are rounded up to a multiple of
  int before;  // units (of one group each) of the sequences ahead of b
  int b, ctx;
};

// The sequence that holds the first unit of share wg (b = B: none), or sequence
// `seq`.  Wave holds 64 sequences at a time, one a lane: load(a, b0) those from
// b0 on; sum(align) adds their units up, to last() in all, ahead(lane) before a
// lane's; reaching(a, b0, before, at) is the first lane whose groups end past
// unit `at` of the row (-1: none); ctx_of(lane) its length.
template <bool FIND_UNIT, typename Wave>
PVLM_Q8_FN Shares q8_find(const QShape& a, Wave w, int wg, int seq) {
  Shares s;
  int total = 0;
  auto add_up = [&](int b0, int align) {
    if (b0 > 0 || a.B > 64) w.load(a, b0);
    w.sum(align);
  };
  w.load(a, 0);
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    add_up(b0, 1);
    total += w.last();
  }
  s.per = (total * a.HR + a.wgs - 1) / a.wgs;
  if (s.per < kQMinUnits) s.per = kQMinUnits;
  s.align = 1;
  if (a.B * a.HR <= a.wgs) {  // (so the sums below stay under wgs shares and as many units of rounding)
    int sum = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
      add_up(b0, s.per);
      sum += w.last();
    }
    if ((int64_t)sum * a.HR <= (int64_t)a.wgs * s.per) s.align = s.per;
  }
  s.before = 0;
  s.b = a.B;
  s.ctx = 0;
  // (wg * per stays within 32 bits: per exceeds total / wgs by less than one, or is the least share of few units)
  const int at = wg * s.per;
  for (int b0 = 0; b0 < a.B; b0 += 64) {
    add_up(b0, s.align);
    int hit = seq - b0;
    if constexpr (FIND_UNIT) hit = w.reaching(a, b0, s.before, at);
    if (hit >= 0 && hit < 64) {
      s.before += w.ahead(hit);
      s.b = b0 + hit;
      s.ctx = w.ctx_of(hit);
      break;
    }
    s.before += w.last();
  }
  return s;
}

// A workgroup's share as pieces of groups, one after the other.
struct QPiece {
  int b, g, rg, ctx;     // group: sequence, KV head, share of its row tiles
  int c0, c1;            // its tokens (c0 opens a unit)
  int left;              // units of the share from c0 on
  int before, per, align;  // units of the sequences ahead of b; of a share; see Shares
  PVLM_Q8_FN void set(const QShape& a) {
    const int N = ctx + a.T, u = c0 / kQUnit + left;
    c1 = q8_uniform(u > N / kQUnit ? N : u * kQUnit);
  }
  // The first piece of share wg, with that share's Shares; false where it is empty.
  PVLM_Q8_FN bool begin(const QShape& a, const Shares& s, int wg) {
    if (s.b >= a.B) return false;
    b = s.b;
    ctx = s.ctx;
    before = s.before;
    per = s.per;
    align = s.align;
    const int units = units_of(a, ctx), u = aligned(units, align), off = wg * per - before * a.HR;
    const int hr = q8_uniform(off / u);
    g = q8_uniform(hr / a.RG);
    rg = hr - g * a.RG;
    const int from = q8_uniform(off - hr * u);
    left = align == 1 || per < units - from ? per : units - from;
    c0 = from * kQUnit;
    set(a);
    return true;
  }
  // The next piece, `ctx_of(b)` giving a sequence's length; false where the share
  // ends.  (A share that is aligned holds one piece.)
  template <typename F>
  PVLM_Q8_FN bool advance(const QShape& a, F ctx_of) {
    left -= (c1 - c0 + kQUnit - 1) / kQUnit;
    if (left <= 0) return false;
    if (++rg == a.RG) {
      rg = 0;
      if (++g == a.Hkv) {
        g = 0;
        before += units_of(a, ctx);
        if (++b == a.B) return false;
        ctx = ctx_of(b);
      }
    }
    c0 = 0;
    set(a);
    return true;
  }
  PVLM_Q8_FN int group(const QShape& a) const { return (b * a.Hkv + g) * a.RG + rg; }
};

// The workgroups that hold pieces of a group (hr = g * RG + rg), and its first record.
struct Holders {
  int rec, count;
};
PVLM_Q8_FN Holders holders(const QShape& a, int per, int align, int before, int b, int hr, int ctx) {
  const int u = aligned(units_of(a, ctx), align), start = before * a.HR + hr * u;
  const int w0 = start / per, w1 = (start + u - 1) / per;
  return {b * a.HR + hr + w0, w1 - w0 + 1};
}

inline pvlm_status check_verify_q8(int B, int T, int Hq, int Hkv, int D, int64_t n_cap, int64_t max_ctx) {
  const pvlm_status st = check_verify(PVLM_BF16, B, T, Hq, Hkv, D, n_cap, max_ctx);
  if (st != PVLM_OK) return st;
  if (n_cap % 32 != 0) return PVLM_ERR_SHAPE;
  // the finish kernel has 64 work-items for each row, in one launch of fewer than 2^32
  if ((int64_t)B * Hq * T > ((int64_t)1 << 22)) return PVLM_ERR_SHAPE;
  // units are counted in 32 bits (at most 4 workgroups share 40 tiles)
  const int64_t units = (max_ctx + T + kQUnit - 1) / kQUnit;
  return (int64_t)B * Hkv * 4 * units > INT32_MAX - 65536 ? PVLM_ERR_SHAPE : PVLM_OK;
}

// The plan for arguments that check_verify_q8 takes, on `cus` compute units (a
// workgroup's ring takes most of a unit's LDS).  It grows with `cus`, so the
// bytes planned for the whole device are enough under every budget.
inline void split_verify_q8(int B, int T, int Hq, int Hkv, int D, int64_t, int64_t max_ctx, int cus, QSplit* p) {
  p->G = Hq / Hkv;
  p->R = p->G * T;
  p->RTT = (p->R + 15) / 16;
  p->RG = (p->RTT + kQMaxRT - 1) / kQMaxRT;
  p->RT = (p->RTT + p->RG - 1) / p->RG;
  const int64_t groups = (int64_t)B * Hkv * p->RG;
  const int64_t units = groups * ((max_ctx + T + kQUnit - 1) / kQUnit);
  const int64_t shares = (units + kQMinUnits - 1) / kQMinUnits;
  p->wgs = (int)(shares < cus ? shares : cus);
  p->recs = (size_t)(groups + p->wgs);
  const size_t rows = p->recs * p->RT * q8_waves(p->RT).tw * 16;
  p->mrows = (max_ctx + T + 31) / 32 * 32;
  p->off_mpart = kSyncRegion;  // (the region at the start is other calls')
  p->off_stats = align_up(p->off_mpart + 4 * (size_t)groups * q8_mass_waves(p->RT).rw * p->mrows, 256);
  p->off_zt = align_up(p->off_stats + 8 * rows, 256);
  p->off_nan = align_up(p->off_zt + 4 * rows, 256);
  p->off_opart = align_up(p->off_nan + 4 * p->recs * q8_waves(p->RT).cw, 256);
  p->bytes = align_up(p->off_opart + 4 * rows * D, 256);
}

}  // namespace pvlm

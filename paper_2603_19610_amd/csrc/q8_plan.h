// Launch plan of verify attention over an 8-bit cache: how its row tiles and
// tokens are spread over workgroups, and where the workspace's areas lie.  Plain
// C++, so that the plan can be run over all sizes without a GPU.
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
// took 126 to 146 us where one took 124 to 128.
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
  size_t off_mpart, off_stats, off_zt, off_nan, off_opart, bytes;
};

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
inline void split_verify_q8(int B, int T, int Hq, int Hkv, int D, int64_t n_cap, int64_t max_ctx, int cus,
                            QSplit* p) {
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
  p->off_mpart = kSyncRegion;  // (the region at the start is other calls')
  p->off_stats = align_up(p->off_mpart + 4 * (size_t)groups * q8_mass_waves(p->RT).rw * n_cap, 256);
  p->off_zt = align_up(p->off_stats + 8 * rows, 256);
  p->off_nan = align_up(p->off_zt + 4 * rows, 256);
  p->off_opart = align_up(p->off_nan + 4 * p->recs * q8_waves(p->RT).cw, 256);
  p->bytes = align_up(p->off_opart + 4 * rows * D, 256);
}

}  // namespace pvlm

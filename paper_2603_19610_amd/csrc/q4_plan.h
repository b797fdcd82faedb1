// Launch plan of attention over a 4-bit cache: how its row tiles and tokens are
// spread over workgroups and waves, and where the workspace's areas lie.  Plain C++,
// so that the plan can be run over all sizes without a GPU.  The shares of the
// tokens are those of the 8-bit cache's plan.
#pragma once

#include "q8_plan.h"

namespace pvlm {

constexpr int kQ4MaxRT = 9;   // 16-row tiles of a workgroup of the partial kernel
constexpr int kQ4MassRT = 5;  // and of a wave of the mass kernel, which holds their queries

// The waves of a partial workgroup: RW for its row tiles, with TPW tiles each, times
// TW, which take its blocks of tokens in turn.
struct Q4Waves {
  int tpw, rw, tw;
};
constexpr Q4Waves q4_waves(int RT) {
  return RT <= 3 ? Q4Waves{RT, 1, 8} : RT == 4 ? Q4Waves{2, 2, 4} : RT <= 6 ? Q4Waves{3, 2, 4} : RT <= 8 ? Q4Waves{2, 4, 2} : Q4Waves{3, 3, 2};
}

struct Q4Split {
  int G, R;           // query heads of a KV head, and its query rows G * T
  int RTT, RG, RT;    // their 16-row tiles, the workgroups that share them, and the tiles of one
  int wgs;            // workgroups of the partial kernel
  size_t recs;        // partial results of RT tiles: group x of workgroup w is number x + w
  int MG, MT;         // mass kernel: a KV head's tiles as MG sets of MT
  int GW;             // its waves that take sets in turn; 8 / GW share the tokens
  int chunk;          // tokens of a mass workgroup
  size_t off_stats, off_nan, off_rows, off_opart, bytes;
};

inline pvlm_status check_verify_q4(int B, int T, int Hq, int Hkv, int D, int64_t n_cap, int64_t max_ctx) {
  const pvlm_status st = check_verify_q8(B, T, Hq, Hkv, D, n_cap, max_ctx);
  if (st != PVLM_OK) return st;
  // units are counted in 32 bits (at most 5 workgroups share 40 tiles)
  const int64_t units = (max_ctx + T + kQUnit - 1) / kQUnit;
  if ((int64_t)B * Hkv * 5 * units > INT32_MAX - 65536) return PVLM_ERR_SHAPE;
  // the mass kernel has 512 work-items for each 32 rows or more, in one launch of fewer than 2^32
  return B > 65535 || n_cap / 32 > (((int64_t)1 << 32) - 512) / 512 ? PVLM_ERR_SHAPE : PVLM_OK;
}

// The plan for arguments that check_verify_q4 takes, on `cus` compute units.  It grows
// with `cus`, so the bytes planned for the whole device are enough under every budget.
inline void split_verify_q4(int B, int T, int Hq, int Hkv, int D, int64_t max_ctx, int cus, Q4Split* p) {
  p->G = Hq / Hkv;
  p->R = p->G * T;
  p->RTT = (p->R + 15) / 16;
  p->RG = (p->RTT + kQ4MaxRT - 1) / kQ4MaxRT;
  p->RT = (p->RTT + p->RG - 1) / p->RG;
  const int64_t groups = (int64_t)B * Hkv * p->RG;
  const int64_t rows = max_ctx + T;
  const int64_t units = groups * ((rows + kQUnit - 1) / kQUnit);
  const int64_t shares = (units + kQMinUnits - 1) / kQMinUnits;
  p->wgs = (int)(shares < cus ? shares : cus);
  p->recs = (size_t)(groups + p->wgs);
  p->MG = (p->RTT + kQ4MassRT - 1) / kQ4MassRT;
  p->MT = (p->RTT + p->MG - 1) / p->MG;
  p->GW = 8;
  while (p->GW > Hkv * p->MG) p->GW /= 2;
  // two workgroups a compute unit, of at least one token tile for each of a workgroup's waves
  const int least = 16 * (8 / p->GW) > 32 ? 16 * (8 / p->GW) : 32;
  p->chunk = 512;
  while (p->chunk > least && (rows + p->chunk - 1) / p->chunk * B < 2 * cus) p->chunk /= 2;
  const size_t stats = p->recs * p->RT * 16;
  p->off_stats = kSyncRegion;  // (the region at the start is other calls')
  p->off_nan = align_up(p->off_stats + 16 * stats, 256);
  p->off_rows = align_up(p->off_nan + 4 * p->recs, 256);
  p->off_opart = align_up(p->off_rows + 8 * (size_t)B * Hkv * p->RTT * 16, 256);
  p->bytes = align_up(p->off_opart + 4 * stats * D, 256);
}

}  // namespace pvlm

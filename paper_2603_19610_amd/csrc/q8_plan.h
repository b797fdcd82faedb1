// Launch plan of verify attention over an 8-bit cache: how its row tiles and
// tokens are split over workgroups, and where the workspace's areas lie.  Plain
// C++, so that the plan can be run over all sizes without a GPU.
#pragma once

#include "verify_plan.h"

namespace pvlm {

// A stage of the partial and mass kernels: 16 KB of K codes and 16 KB of V codes.
constexpr int kQStageBytes = 16384;
constexpr int kQMaxRT = 9;  // 16-row tiles of a workgroup
inline int q8_stage_rows(int D) { return kQStageBytes / D; }

struct QSplit {
  int G, R;            // query heads of a KV head, and its query rows G * T
  int RTT, RG, RT;     // their 16-row tiles, the workgroups that share them, and the tiles of one
  int chunk, splits;   // tokens of a workgroup, and the chunks of the longest sequence
  size_t off_mpart, off_stats, off_opart, bytes;
};

inline pvlm_status check_verify_q8(int B, int T, int Hq, int Hkv, int D, int64_t n_cap, int64_t max_ctx) {
  const pvlm_status st = check_verify(PVLM_BF16, B, T, Hq, Hkv, D, n_cap, max_ctx);
  if (st != PVLM_OK) return st;
  if (n_cap % 32 != 0) return PVLM_ERR_SHAPE;
  // launches of fewer than 2^32 work-items: at most 704 for each 16-row tile
  // and 64 for each row
  return (int64_t)B * Hq * T > ((int64_t)1 << 22) ? PVLM_ERR_SHAPE : PVLM_OK;
}

// The plan for arguments that check_verify_q8 takes, on `cus` compute units.  A
// workgroup's ring takes most of a unit's LDS, so one of them runs on each; the
// tokens of a KV head are cut into as many chunks of whole stages as its share
// of the units.  Fewer units never make more chunks, so the bytes planned for
// the whole device are enough under every budget.
inline void split_verify_q8(int B, int T, int Hq, int Hkv, int D, int64_t n_cap, int64_t max_ctx, int cus,
                            QSplit* p) {
  p->G = Hq / Hkv;
  p->R = p->G * T;
  p->RTT = (p->R + 15) / 16;
  p->RG = (p->RTT + kQMaxRT - 1) / kQMaxRT;
  p->RT = (p->RTT + p->RG - 1) / p->RG;
  const int64_t groups = (int64_t)B * Hkv * p->RG, rows = q8_stage_rows(D);
  const int64_t stages = (max_ctx + T + rows - 1) / rows;
  const int64_t most = cus > groups ? cus / groups : 1;
  const int64_t per = (stages + most - 1) / most;
  p->chunk = (int)(per * rows);
  p->splits = (int)((stages + per - 1) / per);
  const size_t tiles = (size_t)B * Hkv * p->RTT;
  p->off_mpart = kSyncRegion;  // (the region at the start is other calls')
  p->off_stats = align_up(p->off_mpart + 4 * (size_t)groups * n_cap, 256);
  p->off_opart = align_up(p->off_stats + 128 * tiles * p->splits, 256);
  p->bytes = align_up(p->off_opart + 64 * tiles * p->splits * D, 256);
}

}  // namespace pvlm

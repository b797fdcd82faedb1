// Launch plan of attention over a 4-bit cache: how its row tiles and tokens are
// spread over workgroups and waves, and where the workspace's areas lie.  Plain C++,
// so that the plan can be run over all sizes without a GPU.  The shares of the
// tokens are those of the 8-bit cache's plan.
#pragma once

#include "q8_plan.h"

namespace pvlm {

constexpr int kQ4RowTiles = 3;  // 16-row tiles of a partial workgroup, which each of its waves holds
constexpr int kQ4Waves = 8;      // its waves, which take the tokens in turn
constexpr int kQ4Single = 1024;  // most rows that one workgroup takes of a group by itself
constexpr int kQ4MassRun = 512; // most tokens that a mass workgroup takes at a time
constexpr int kQ4MassRT = 3;    // row tiles of a wave of the mass kernel, which holds their queries

struct Q4Split {
  int G, R;          // query heads of a KV head, and its query rows G * T
  int RTT, RG, RT;   // their 16-row tiles, as RG sets of RT
  int shares;        // equal shares of the tokens (see q8_plan.h, a KV head being one group)
  int per_share;     // workgroups of a share, which take its sets of row tiles in turn
  bool single;       // every group is a share of its own
  size_t recs;       // partial results of RTT tiles: group x of share w is number x + w
  int MG, MT;        // mass kernel: a KV head's tiles as MG sets of MT
  int GW;            // its waves that take sets in turn; 8 / GW share the tokens
  int chunk;         // tokens that a mass workgroup takes at a time
  size_t off_stats, off_nan, off_rows, off_opart, bytes;
};

// (The shares are counted as the 8-bit call's, within its limits.)
inline pvlm_status check_verify_q4(int B, int T, int Hq, int Hkv, int D, int64_t n_cap, int64_t max_ctx) {
  return check_verify_q8(B, T, Hq, Hkv, D, n_cap, max_ctx);
}

// The plan for arguments that check_verify_q4 takes, on `cus` compute units.  It grows
// with `cus`, so the bytes planned for the whole device are enough under every budget.
inline void split_verify_q4(int B, int T, int Hq, int Hkv, int D, int64_t max_ctx, int cus, Q4Split* p) {
  p->G = Hq / Hkv;
  p->R = p->G * T;
  p->RTT = (p->R + 15) / 16;
  p->RG = (p->RTT + kQ4RowTiles - 1) / kQ4RowTiles;
  p->RT = (p->RTT + p->RG - 1) / p->RG;
  const int64_t groups = (int64_t)B * Hkv;
  const int64_t rows = max_ctx + T;
  const int64_t units = groups * ((rows + kQUnit - 1) / kQUnit);
  p->per_share = p->RG < cus ? p->RG : cus;
  const int64_t most = cus / p->per_share, shares = (units + kQMinUnits - 1) / kQMinUnits;
  // Few tokens: a workgroup for each group writes the results, and nothing is combined.
  // (Us a call in a graph, one workgroup a group against shares.  One row of 28 / 4
  // heads: 4.8 and 12.3 at 30 tokens, 6.3 and 9.9 at 500, 8.2 and 10.5 at 1000; 9 rows of 64 / 8:
  // 11.5 and 16.1, 14.2 and 16.8, 17.2 and 18.6; 6 rows of 28 / 4: 16.8 and 16.6 at 1000.)
  p->single = rows <= kQ4Single && groups <= most;
  p->shares = (int)(p->single ? groups : shares < most ? shares : most);
  p->recs = (size_t)(groups + p->shares);
  // Up to five tiles in one set: a run has its queries and sums to load but once.  (Us a
  // call in a graph, one set against two.  Five tiles: 28.3 and 29.7 over 2000 tokens of 8
  // heads, 34.7 and 42.0 over 12800, 49 and 57 over 40000, but 124 and 113 over 132096; four
  // tiles: 29.2 and 33.7 over 12800 of 8 heads, 32.8 and 33.4 over 40000 of 4, 25.6 and 23.8 over 6432.)
  p->MG = p->RTT <= 5 ? 1 : (p->RTT + kQ4MassRT - 1) / kQ4MassRT;
  p->MT = (p->RTT + p->MG - 1) / p->MG;
  p->GW = 8;
  while (p->GW > Hkv * p->MG) p->GW /= 2;
  // The batch's tokens over two workgroups a compute unit, in one round of them if 512
  // tokens each are enough (131K tokens in 517 runs of 256 took two: 87 us; in
  // 486 of 272: 75 us); a token tile for each of a workgroup's waves at least.
  const int step = 16 * (8 / p->GW), slots = p->MT <= 3 ? 2 * cus : cus;
  int64_t chunk = (rows * B + slots - 1) / slots;
  while (chunk < kQ4MassRun && (rows + chunk - 1) / chunk * B > slots) chunk += step;
  chunk = (chunk + step - 1) / step * step;
  p->chunk = (int)(chunk < 32 ? 32 : chunk < kQ4MassRun ? chunk : kQ4MassRun);
  const size_t stats = p->recs * p->RTT * 16;
  p->off_stats = kSyncRegion;  // (the region at the start is other calls')
  p->off_nan = align_up(p->off_stats + 16 * stats, 256);
  p->off_rows = align_up(p->off_nan + 4 * p->recs, 256);
  p->off_opart = align_up(p->off_rows + 8 * (size_t)groups * p->R, 256);
  p->bytes = align_up(p->off_opart + 4 * stats * D, 256);
}

}  // namespace pvlm

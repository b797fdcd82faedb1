// Runs the 4-bit attention's plan over its sizes without a GPU.
//   q4_plan_check areas  the workspace's areas follow each other inside it, a workspace
//                        sized for the whole device holds under every budget, and the
//                        shares' arithmetic stays within 32 bits
//   q4_plan_check waves  tiles, waves and token runs are what the kernels are compiled
//                        for, and hold every row and token
// Prints the first failures and their number.
#include <cstdio>
#include <cstring>

#include "q4_plan.h"

using namespace pvlm;

struct Call {
  int B, T, Hq, Hkv, D;
  int64_t n_cap, ctx;
};

template <typename F>
static long each_plan(F bad) {
  const int64_t ctxs[] = {0, 1, 31, 62, 63, 333, 1300, 6432, 16384, 70000, 131072, 1 << 20};
  long n = 0, fail = 0;
  for (int D : {64, 128})
    for (int Hkv : {1, 2, 3, 4, 5, 8, 16, 256})
      for (int G : {1, 4, 5, 7, 8, 20})
        for (int T : {1, 2, 5, 9, 17, 32})
          for (int B : {1, 2, 7, 64, 65, 300})
            for (int64_t ctx : ctxs) {
              const Call c{B, T, G * Hkv, Hkv, D, (ctx + T + 31) / 32 * 32, ctx};
              if (check_verify_q4(c.B, c.T, c.Hq, c.Hkv, c.D, c.n_cap, c.ctx) != PVLM_OK) continue;
              for (int cus : {256, 104, 8, 1}) {
                Q4Split p;
                split_verify_q4(c.B, c.T, c.Hq, c.Hkv, c.D, c.ctx, cus, &p);
                ++n;
                if (bad(c, cus, p) && fail++ < 10)
                  std::printf("B %d T %d heads %d/%d D %d ctx %ld, %d units: RT %d RG %d shares %d chunk %d\n", B, T,
                              c.Hq, Hkv, D, (long)ctx, cus, p.RT, p.RG, p.shares, p.chunk);
              }
            }
  std::printf("%ld plans, %ld failures\n", n, fail);
  return n ? fail : 1;
}

static bool bad_areas(const Call& c, int cus, const Q4Split& p) {
  Q4Split whole;
  split_verify_q4(c.B, c.T, c.Hq, c.Hkv, c.D, c.ctx, 256, &whole);
  const size_t rows = p.recs * p.RTT * 16, groups = (size_t)c.B * c.Hkv;
  const size_t at[] = {kSyncRegion, p.off_stats, p.off_nan, p.off_rows, p.off_opart, p.bytes};
  const size_t need[] = {0, 16 * rows, 4 * p.recs, 8 * groups * p.R, 4 * rows * c.D};
  for (int i = 0; i < 5; ++i)
    if (at[i] % 16 || at[i] + need[i] > at[i + 1]) return true;
  const int64_t units = (int64_t)groups * ((c.ctx + c.T + kQUnit - 1) / kQUnit);
  if (units + p.shares > INT32_MAX || p.shares * p.per_share > cus) return true;
  return p.bytes > whole.bytes;
}

static bool bad_waves(const Call& c, int, const Q4Split& p) {
  if (p.RT < 1 || p.RT > kQ4RowTiles || p.RT * p.RG < p.RTT || (p.RG - 1) * p.RT >= p.RTT) return true;
  if (p.per_share < 1 || p.per_share > p.RG || p.shares < 1) return true;
  if (p.single && (p.shares != c.B * c.Hkv || c.ctx + c.T > kQ4Single)) return true;
  if (p.MT < 1 || p.MT > 5 || p.MT * p.MG < p.RTT || (p.MG - 1) * p.MT >= p.RTT) return true;
  if (p.GW < 1 || p.GW > 8 || 8 % p.GW || p.GW > c.Hkv * p.MG) return true;
  return p.chunk < 32 || p.chunk > kQ4MassRun || p.chunk % 16 || p.chunk < 16 * (8 / p.GW);
}

int main(int argc, char** argv) {
  const char* what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "areas")) return each_plan(bad_areas) != 0;
  if (!std::strcmp(what, "waves")) return each_plan(bad_waves) != 0;
  return 2;
}

// Runs the 8-bit verify's plan over its sizes without a GPU.
//   q8_plan_check areas    the workspace's areas follow each other inside it, and
//                          a workspace sized for the whole device holds under
//                          every budget
//   q8_plan_check shares   the workgroups' shares hold every unit of every group
//                          once, and no two pieces the same record
//   q8_plan_check waves    a workgroup's waves, and the waves of a SIMD, within
//                          what the kernels are compiled for
// Prints the first failures and their number.
#include <cstdio>
#include <cstring>
#include <random>
#include <set>
#include <utility>
#include <vector>

#include "q8_plan.h"

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
    for (int Hkv : {1, 2, 4, 5, 8, 16})
      for (int G : {1, 4, 5, 7, 8, 20})
        for (int T : {1, 2, 5, 9, 17, 32})
          for (int B : {1, 2, 7, 64, 65, 300})
            for (int64_t ctx : ctxs) {
              const Call c{B, T, G * Hkv, Hkv, D, (ctx + T + 31) / 32 * 32, ctx};
              if (check_verify_q8(c.B, c.T, c.Hq, c.Hkv, c.D, c.n_cap, c.ctx) != PVLM_OK) continue;
              for (int cus : {256, 104, 8, 1}) {
                QSplit p;
                split_verify_q8(c.B, c.T, c.Hq, c.Hkv, c.D, c.n_cap, c.ctx, cus, &p);
                ++n;
                if (bad(c, cus, p) && fail++ < 10)
                  std::printf("B %d T %d heads %d/%d D %d ctx %ld, %d units: RT %d RG %d wgs %d\n", B, T, c.Hq, Hkv, D,
                              (long)ctx, cus, p.RT, p.RG, p.wgs);
              }
            }
  std::printf("%ld plans, %ld failures\n", n, fail);
  return n ? fail : 1;
}

static bool bad_areas(const Call& c, int, const QSplit& p) {
  QSplit whole;
  split_verify_q8(c.B, c.T, c.Hq, c.Hkv, c.D, c.n_cap, c.ctx, 256, &whole);
  const size_t rows = p.recs * p.RT * q8_waves(p.RT).tw * 16, groups = (size_t)c.B * c.Hkv * p.RG;
  const size_t at[] = {kSyncRegion, p.off_mpart, p.off_stats, p.off_zt, p.off_nan, p.off_opart, p.bytes};
  const size_t need[] = {0, 4 * groups * q8_mass_waves(p.RT).rw * (size_t)c.n_cap, 8 * rows, 4 * rows,
                         4 * p.recs * q8_waves(p.RT).cw, 4 * rows * c.D};
  for (int i = 0; i < 6; ++i)
    if (at[i] % 16 || at[i] + need[i] > at[i + 1]) return true;
  return p.bytes > whole.bytes;
}

// The device's arithmetic (find, Piece, holders) over random lengths.
static bool bad_shares(const Call& c, int cus, const QSplit& p) {
  if (c.ctx > 20000 || c.B * c.Hkv * p.RG > 2500) return false;
  std::mt19937 rng(c.B * 131 + c.T + (int)c.ctx * 7 + cus);
  const int HR = c.Hkv * p.RG;
  std::vector<int> units(c.B);
  long total = 0;
  for (int b = 0; b < c.B; ++b) {
    const int len = rng() % 3 ? (int)(rng() % (c.ctx + 1)) : (int)c.ctx;
    units[b] = (len + c.T + kQUnit - 1) / kQUnit;
    total += units[b];
  }
  long per = (total * HR + p.wgs - 1) / p.wgs;
  if (per < kQMinUnits) per = kQMinUnits;
  // groups begin shares of their own where these are enough
  std::vector<int> real = units;
  long rounded = 0;
  for (int u : units) rounded += (u + per - 1) / per * per;
  const bool aligned = c.B * HR <= p.wgs && rounded * HR <= p.wgs * per;
  if (aligned)
    for (int& u : units) u = (int)((u + per - 1) / per * per);
  std::set<long> records;
  std::vector<long> first(c.B * HR, -1), count(c.B * HR, 0);
  long done = 0;
  for (int w = 0; w < p.wgs; ++w) {
    const long at = w * per;
    if (at > INT32_MAX) return true;
    long before = 0;
    int b = 0;
    while (b < c.B && (before + units[b]) * HR <= at) before += units[b++];
    if (b == c.B) continue;
    long off = at - before * HR, left = per;
    int hr = (int)(off / units[b]);
    off -= (long)hr * units[b];
    if (aligned && real[b] - off < left) left = real[b] - off;
    if (left <= 0) return true;
    const long share = left;
    while (left > 0) {
      const long here = left < units[b] - off ? left : units[b] - off, group = (long)b * HR + hr;
      if (at + share - left != before * HR + (long)hr * units[b] + off) return true;
      const long rec = group + w;
      if (rec >= (long)p.recs || !records.insert(rec).second) return true;
      if (first[group] < 0) first[group] = w;
      // what the kernels that read the records take for the group's holders
      const long start = before * HR + (long)hr * units[b];
      if (start / per != first[group] || (start + units[b] - 1) / per < w) return true;
      ++count[group];
      done += here;
      left -= here;
      off = 0;
      if (here < units[b] && left <= 0) break;
      if (++hr == HR) {
        hr = 0;
        before += units[b];
        if (++b == c.B) break;
      }
    }
  }
  long before = 0;
  for (int b = 0; b < c.B; ++b) {
    for (int hr = 0; hr < HR; ++hr) {
      const long start = before * HR + (long)hr * units[b];
      if (count[(long)b * HR + hr] != (start + units[b] - 1) / per - start / per + 1) return true;
    }
    before += units[b];
  }
  return done != total * HR;
}

static bool bad_waves(const Call&, int, const QSplit& p) {
  if (p.RT < 1 || p.RT > kQMaxRT || p.RT * p.RG < p.RTT) return true;
  const QWaves w = q8_waves(p.RT), m = q8_mass_waves(p.RT);
  if (w.tpw != 1 || w.rw != p.RT || 2 * w.tw % w.cw || w.rw * w.tw + 2 * w.cw > 16) return true;
  return m.tpw > 3 || m.rw * m.tpw < p.RT || (m.rw - 1) * m.tpw >= p.RT || 2 * m.tw % m.cw || m.rw * m.tw + m.cw > 8;
}

int main(int argc, char** argv) {
  const char* what = argc > 1 ? argv[1] : "";
  if (!std::strcmp(what, "areas")) return each_plan(bad_areas) != 0;
  if (!std::strcmp(what, "shares")) return each_plan(bad_shares) != 0;
  if (!std::strcmp(what, "waves")) return each_plan(bad_waves) != 0;
  return 2;
}

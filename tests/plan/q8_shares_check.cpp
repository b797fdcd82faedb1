// Runs the arithmetic by which the 8-bit verify's kernels find their shares
// (q8_find, QPiece, holders: the functions that the kernels are built from, in
// their own types) over sizes and lengths without a GPU, and checks what the kernels
// rely on:
//   every group's tokens 0 .. N - 1 are held by pieces that follow each other, each
//   opening a unit; every piece ends a block of its group or its group; records are
//   within the workspace and no two pieces have the same one; a group's holders
//   are the workgroups that hold it, and its first record the first of them.
//   q8_shares_check ragged    sizes of all kinds, random lengths
//   q8_shares_check extremes  the largest unit counts that a call is taken for
//   q8_shares_check workspace a workspace goes by the longest context, not by the cache's capacity
//   q8_shares_check planted   one length counted a token long: has to fail
// Built with a check of signed overflow: an index past 32 bits ends the run.
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>
#include <vector>

#include "q8_plan.h"

using namespace pvlm;

// 64 lanes of a wave, as arrays.
struct HostWave {
  const std::vector<int32_t>* lens;
  int ctx[64], raw[64], u[64], upto[64];
  void load(const QShape& a, int b0) {
    for (int i = 0; i < 64; ++i) {
      const bool here = b0 + i < a.B;
      ctx[i] = here ? clamp_ctx(a, (*lens)[b0 + i]) : 0;
      raw[i] = here ? units_of(a, ctx[i]) : 0;
    }
  }
  void sum(int align) {
    int run = 0;
    for (int i = 0; i < 64; ++i) {
      u[i] = aligned(raw[i], align);
      run += u[i];
      upto[i] = run;
    }
  }
  int last() const { return upto[63]; }
  int ahead(int i) const { return upto[i] - u[i]; }
  int ctx_of(int i) const { return ctx[i]; }
  int reaching(const QShape& a, int b0, int before, int at) const {
    for (int i = 0; i < 64; ++i)
      if (b0 + i < a.B && (before + upto[i]) * a.HR > at) return i;
    return -1;
  }
};

static long g_runs = 0, g_fail = 0;
static bool g_plant = false;

static const char* wrong(const QShape& a, const QSplit& p, const std::vector<int32_t>& lens) {
  struct Group {
    int64_t end = 0;  // tokens held so far
    int pieces = 0, first_rec = -1, last_wg = -1;
  };
  std::vector<Group> groups((size_t)a.B * a.HR);
  std::vector<bool> taken(p.recs, false);
  auto length = [&](int b) -> int64_t {  // what the call's documentation says a length outside its range counts as
    const int64_t x = lens[b];
    return (x < 0 ? 0 : x > a.max_ctx ? a.max_ctx : x) + (g_plant && b == a.B / 2);
  };
  HostWave w;
  w.lens = &lens;
  for (int wg = 0; wg < a.wgs; ++wg) {
    QPiece q;
    if (!q.begin(a, q8_find<true>(a, w, wg, 0), wg)) continue;
    int64_t units = 0;
    do {
      if (q.b < 0 || q.b >= a.B || q.g < 0 || q.g >= a.Hkv || q.rg < 0 || q.rg >= a.RG) return "group";
      if (q.ctx != length(q.b)) return "length";
      const int64_t N = length(q.b) + a.T;
      const int gr = q.group(a);
      if (gr != (q.b * a.Hkv + q.g) * a.RG + q.rg) return "group number";
      Group& x = groups[gr];
      if (q.c0 != x.end || q.c0 % kQUnit || q.c1 <= q.c0 || q.c1 > N) return "piece";
      if (q.c1 < N && q.c1 % kQUnit) return "end";
      const int64_t rec = (int64_t)gr + wg;
      if (rec >= (int64_t)p.recs || taken[rec]) return "record";
      taken[rec] = true;
      x.end = q.c1;
      if (x.pieces++ == 0) x.first_rec = (int)rec;
      x.last_wg = wg;
      units += (q.c1 - q.c0 + kQUnit - 1) / kQUnit;
    } while (q.advance(a, [&](int b) { return clamp_ctx(a, lens[b]); }));
    if (units > q.per) return "share";
  }
  for (int b = 0; b < a.B; ++b) {
    if (b > 200 && b < a.B - 200) continue;  // (the search is quadratic in B)
    const Shares s = q8_find<false>(a, w, 0, b);
    if (s.b != b || s.ctx != length(b)) return "sequence";
    for (int hr = 0; hr < a.HR; ++hr) {
      const Group& x = groups[(size_t)b * a.HR + hr];
      const Holders h = holders(a, s.per, s.align, s.before, b, hr, s.ctx);
      if (h.rec != x.first_rec || h.count != x.pieces) return "holders";
      if (h.rec + h.count - 1 != b * a.HR + hr + x.last_wg) return "last holder";
    }
  }
  for (int b = 0; b < a.B; ++b)
    for (int hr = 0; hr < a.HR; ++hr)
      if (groups[(size_t)b * a.HR + hr].end != length(b) + a.T) return "tokens";
  return nullptr;
}

static void run(int B, int T, int G, int Hkv, int64_t max_ctx, int cus, std::mt19937& rng, int kind) {
  const int64_t n_cap = (max_ctx + T + 31) / 32 * 32;
  if (check_verify_q8(B, T, G * Hkv, Hkv, 128, n_cap, max_ctx) != PVLM_OK) return;
  QSplit p;
  split_verify_q8(B, T, G * Hkv, Hkv, 128, n_cap, max_ctx, cus, &p);
  QShape a;
  a.B = B;
  a.T = T;
  a.Hkv = Hkv;
  a.RG = p.RG;
  a.HR = Hkv * p.RG;
  a.wgs = p.wgs;
  a.max_ctx = (int)max_ctx;
  std::vector<int32_t> lens(B);
  for (int b = 0; b < B; ++b) {
    const int64_t r = (int64_t)(rng() % (uint64_t)(max_ctx + 1));
    lens[b] = (int32_t)(kind == 0 ? max_ctx : kind == 1 ? 0 : kind == 2 ? r : rng() % 4 ? r / 64 : max_ctx);
    if (kind == 3 && rng() % 16 == 0) lens[b] = rng() % 2 ? -5 : INT32_MAX;  // outside the range: clamped
  }
  ++g_runs;
  const char* why = wrong(a, p, lens);
  if (why && g_fail++ < 10)
    std::printf("%s: B %d T %d G %d Hkv %d max_ctx %ld, %d units, lengths %d\n", why, B, T, G, Hkv, (long)max_ctx, cus,
                kind);
}

int main(int argc, char** argv) {
  const char* what = argc > 1 ? argv[1] : "";
  std::mt19937 rng(11);
  g_plant = !std::strcmp(what, "planted");
  if (!std::strcmp(what, "ragged") || g_plant) {
    const int64_t ctxs[] = {0, 1, 31, 62, 63, 333, 1300, 6432, 16384, 70000, 131072, 1 << 20};
    for (int Hkv : {1, 2, 5, 8, 16})
      for (int G : {1, 20})
        for (int T : {1, 9, 32})
          for (int B : {1, 2, 7, 64, 65, 200, 700})
            for (int64_t ctx : ctxs)
              for (int cus : {256, 104, 8})
                for (int kind = 0; kind < 4; ++kind)
                  if (B * Hkv * ctx < (int64_t)1 << 27 || kind == 3) run(B, T, G, Hkv, ctx, cus, rng, kind);
  } else if (!std::strcmp(what, "extremes")) {
    // B * Hkv * 4 * units just under the limit, with one and with four shares of a KV head's rows
    struct Case {
      int B, Hkv;
    };
    for (const Case& c : {Case{1, 15}, Case{15, 1}, Case{1, 255}, Case{3, 85}, Case{64, 8}, Case{65, 8}, Case{257, 4},
                          Case{1024, 8}, Case{3000, 2}, Case{4096, 1}})
      for (int T : {1, 32})
        for (int G : {1, 20}) {
          const int64_t most = ((int64_t)INT32_MAX - 65536) / ((int64_t)c.B * c.Hkv * 4) * kQUnit - T;
          const int64_t ctx = most < ((int64_t)1 << 30) - 32 - T ? most : ((int64_t)1 << 30) - 32 - T;
          for (int cus : {256, 8, 1})
            for (int kind = 0; kind < 4; ++kind) {
              const long before = g_runs;
              run(c.B, T, G, c.Hkv, ctx, cus, rng, kind);
              if (g_runs == before && (int64_t)c.B * c.Hkv * G * T <= 1 << 22) {
                std::printf("refused: B %d Hkv %d T %d G %d\n", c.B, c.Hkv, T, G);
                ++g_fail;
              }
            }
        }
  } else if (!std::strcmp(what, "workspace")) {
    for (int B : {1, 4, 64})
      for (int T : {1, 9, 32})
        for (int64_t ctx : {0, 31, 787, 16384})
          for (int64_t n_cap : {32768, 131072, 1 << 30}) {
            QSplit tight, wide;
            split_verify_q8(B, T, 64, 8, 128, (ctx + T + 31) / 32 * 32, ctx, 256, &tight);
            split_verify_q8(B, T, 64, 8, 128, n_cap, ctx, 256, &wide);
            ++g_runs;
            g_fail += tight.bytes != wide.bytes;
          }
  } else {
    return 2;
  }
  std::printf("%ld plans, %ld failures\n", g_runs, g_fail);
  return g_runs && !g_fail ? 0 : 1;
}

// The shares of pdattn_decode_tree's CTAs over many batches: every key tile of every unit belongs to exactly one piece, the first and
// last piece of a cut unit have at least kTreeMinCut tiles and the others two, and a CTA leaves at most one piece that continues a unit and one that begins one
// without ending it.  Built and run by tests/test_tree_sparse_cpu.py.
#include <cstdint>
#include <cstdio>
#include <random>
#include <vector>

#include "partition.h"

using pdattn::kTreeMinCut;
using pdattn::kTreeStart;

struct Seq {
  int units;
  int64_t tiles;
};
struct At {
  int s, u, t;
  bool operator<(const At& o) const { return s != o.s ? s < o.s : u != o.u ? u < o.u : t < o.t; }
};

static bool check(const std::vector<Seq>& q, int ctas) {
  int64_t total = 0, units = 0;
  for (auto& x : q) total += x.units * (x.tiles + kTreeStart), units += x.units;
  ctas = pdattn::tree_shares(total, units, ctas);
  auto locate = [&](int64_t x) {
    if (x >= total) return At{static_cast<int>(q.size()), 0, 0};
    int64_t before = 0;
    int s = 0;
    for (; before + q[s].units * (q[s].tiles + kTreeStart) <= x; ++s) before += q[s].units * (q[s].tiles + kTreeStart);
    At a{s, 0, 0};
    pdattn::tree_cut(x - before, q[s].tiles, &a.u, &a.t);
    if (a.u >= q[s].units) a = At{s + 1, 0, 0};
    return a;
  };
  std::vector<std::vector<int64_t>> done(q.size());
  for (size_t s = 0; s < q.size(); ++s) done[s].assign(q[s].units, 0);
  for (int c = 0; c < ctas; ++c) {
    At a = locate(total * c / ctas);
    const At end = locate(total * (c + 1) / ctas);
    int slot[2] = {0, 0};
    while (a.s < static_cast<int>(q.size()) && a < end) {
      if (a.u >= q[a.s].units) {
        a = At{a.s + 1, 0, 0};
        continue;
      }
      const int64_t tiles = q[a.s].tiles, te = a.s == end.s && a.u == end.u ? end.t : tiles;
      if (done[a.s][a.u] != a.t || (te <= a.t && tiles > 0) || te > tiles) return false;
      if (te - a.t < tiles) {
        if (te - a.t < (a.t == 0 || te == tiles ? kTreeMinCut : 2)) return false;
        ++slot[a.t > 0 ? 0 : 1];
      }
      done[a.s][a.u] = te == tiles ? -1 : te;       // -1: complete (also a unit without tiles)
      a = te == tiles ? At{a.s, a.u + 1, 0} : At{a.s, a.u, static_cast<int>(te)};
    }
    if (slot[0] > 1 || slot[1] > 1) return false;
  }
  for (auto& x : done)
    for (auto d : x)
      if (d != -1) return false;
  return true;
}

int main() {
  std::mt19937 r(1);
  for (int i = 0; i < 20000; ++i) {
    std::vector<Seq> q(1 + r() % (i % 3 ? 6 : 300));
    const int64_t top = i % 7 == 0 ? 1 << 22 : i % 5 == 0 ? 700 : 30;
    for (auto& x : q) x = Seq{static_cast<int>(r() % 20), static_cast<int64_t>(r() % top)};
    const int ctas = i % 4 == 0 ? 1 + r() % 148 : 148;
    if (!check(q, ctas)) {
      std::fprintf(stderr, "batch %d\n", i);
      return 1;
    }
  }
  std::puts("tree_cut_check: ok");
  return 0;
}

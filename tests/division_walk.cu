// Walks the division of the attention kernels' work on the host: every stretch of a launch, with the code that the kernels run.  Each step of each
// tile has to be met exactly once, each partial result written once and found by the join in its place, inside the workspace.
// Arguments: first and last group size.  Prints what is wrong; exit status 1 if anything is.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <tuple>
#include <vector>

#include "attention_join.cuh"
#include "attention_tc.cuh"

namespace vscan {          // of the library's host side; nothing is launched here
std::atomic<uint64_t> g_launches;
thread_local int g_last_cuda_error;
}

using namespace vscan::kv;
using FlatShape = TileShape<256, 64, 64, 4>;      // the CUDA-core kernel's

struct Step { int b, head, tile, u0, u1, units, n_rows, first; };
struct Walk { std::vector<Step> pieces; Boundary cut; };
struct Case { std::vector<int> rows, keys; int kv_heads, group, tile_rows, causal, ctas, head_dim; };

static int g_wrong = 0;
static void wrong(const Case& c, const char* kernel, const char* what, const Step& s) {
  if (++g_wrong <= 40)
    printf("%s: group %d, %d rows a tile, causal %d, %d CTAs, %zu sequences (first: %d rows, %d keys): %s: sequence %d head %d tile %d steps %d..%d of %d\n",
           kernel, c.group, c.tile_rows, c.causal, c.ctas, c.rows.size(), c.rows[0], c.keys[0], what, s.b, s.head, s.tile, s.u0, s.u1, s.units);
}

// Which sequence a stretch starts in, as the kernels find it
template <typename S, typename P>
static TcStretch place(const P& p, const std::vector<long long>& weight, long long total, int ctas, int k) {
  TcStretch st = stretch_of<S>(p, total, ctas, k);
  long long at = 0;
  for (int b = 0; b < p.batch; ++b) {
    if (at <= st.begin && st.begin < at + weight[b]) { st.b = b; st.seq0 = at; break; }
    at += weight[b];
  }
  return st;
}

template <typename S, typename P, typename F>
static void check(const Case& c, const char* kernel, P& p, F walk) {
  std::vector<long long> weight;
  long long total = 0;
  for (int b = 0; b < p.batch; ++b) {
    weight.push_back(tc_sequence_at<S>(p, b).weight * p.kv_heads);
    total += weight.back();
  }
  std::map<std::tuple<int, int, int>, std::vector<int>> met;     // of each tile: how often each step
  for (int b = 0; b < p.batch; ++b) {
    const long long rows = static_cast<long long>(c.rows[b]) * c.group;
    for (long long t = 0; t * c.tile_rows < rows; ++t) {
      const long long last = (std::min((t + 1) * c.tile_rows, rows) - 1) / c.group, m = c.keys[b];
      const long long seen = c.causal ? std::min(std::max(m - c.rows[b] + last + 1, 0ll), m) : m;
      for (int h = 0; h < c.kv_heads; ++h)
        met[{b, h, static_cast<int>(t)}].assign(std::max((seen + S::kKeys - 1) / S::kKeys, 1ll), 0);
    }
  }
  std::vector<Walk> all(c.ctas);
  std::vector<Boundary> cuts(c.ctas);
  std::vector<Step> slot(2 * c.ctas, Step{-1, 0, 0, 0, 0, 0, 0, 0});
  std::vector<int> joined(2 * c.ctas, 0);
  for (int k = 0; k < c.ctas; ++k) {
    all[k].cut = Boundary{};
    walk(place<S>(p, weight, total, c.ctas, k), all[k]);
    cuts[k] = all[k].cut;
    for (const Step& s : all[k].pieces) {
      auto it = met.find({s.b, s.head, s.tile});
      if (it == met.end()) { wrong(c, kernel, "no such tile", s); continue; }
      if (s.units != static_cast<int>(it->second.size()) || s.u0 < 0 || s.u1 > s.units) { wrong(c, kernel, "steps that are not there", s); continue; }
      for (int u = s.u0; u < s.u1; ++u) ++it->second[u];
      if (s.u0 == 0 && s.u1 == s.units) continue;
      Step& to = slot[2 * k + (s.u0 == 0)];
      if (to.b >= 0) wrong(c, kernel, "a partial result over another", s);
      to = s;
    }
  }
  for (const auto& [at, steps] : met)
    for (size_t u = 0; u < steps.size(); ++u)
      if (steps[u] != 1) wrong(c, kernel, steps[u] ? "a step twice" : "a step not met",
                               Step{std::get<0>(at), std::get<1>(at), std::get<2>(at), static_cast<int>(u), static_cast<int>(u) + 1, static_cast<int>(steps.size()), 0, 0});
  // the join, from the boundaries
  p.boundary = cuts.data();
  const size_t stride = partial_floats(p.tile_rows, p.head_dim);
  std::vector<float> base(1);
  p.partial = base.data();
  for (int k = 0; k < c.ctas; ++k) {
    Boundary bd;
    Pieces pc;
    if (!cut_at(p, k, bd, pc)) continue;
    int u = 0, units = -1;
    for (int i = 0; i < pc.n; ++i) {
      const long long at = (reinterpret_cast<long long>(pc.at(i)) - reinterpret_cast<long long>(base.data())) / static_cast<long long>(stride * 4);
      const Step none = {bd.b, bd.head, bd.tile, k, i, pc.n, 0, 0};
      if (at < 0 || at >= 2 * c.ctas) { wrong(c, kernel, "the join reads outside the workspace", none); break; }
      const Step& s = slot[at];
      if (s.b != bd.b || s.head != bd.head || s.tile != bd.tile || s.u0 != u || s.n_rows != bd.rows || s.first != bd.first) {
        wrong(c, kernel, "the join reads what is not its tile's", none);
        break;
      }
      ++joined[at];
      u = s.u1;
      units = s.units;
    }
    if (u != units) wrong(c, kernel, "the join ends before the tile does", Step{bd.b, bd.head, bd.tile, 0, u, units, 0, 0});
  }
  for (int i = 0; i < 2 * c.ctas; ++i)
    if (slot[i].b >= 0 && joined[i] != 1) wrong(c, kernel, "a partial result that is not joined once", slot[i]);
}

static std::vector<int32_t> offsets(const std::vector<int>& n) {
  std::vector<int32_t> o = {0};
  for (int x : n) o.push_back(o.back() + x);
  return o;
}

static void check_case(const Case& c) {
  const auto rows = offsets(c.rows), keys = offsets(c.keys);
  PromptParams p = {};
  p.row_offset = rows.data(); p.kv_offset = keys.data();
  p.rows = rows.back(); p.kv_rows = keys.back(); p.max_q_len = *std::max_element(c.rows.begin(), c.rows.end());
  p.batch = static_cast<int>(c.rows.size()); p.kv_heads = c.kv_heads; p.group = c.group; p.q_heads = c.kv_heads * c.group; p.causal = c.causal;
  Case now = c;
  // 5th-generation tensor cores: two tiles of whole tokens, or one
  for (int tiles : {2, 1}) {
    now.tile_rows = p.tile_rows = tiles * (128 / c.group) * c.group;
    p.head_dim = tiles == 2 ? 128 : 256;
    check<PtShape>(now, "prompt", p, [&](const TcStretch& st, Walk& w) {
      PtPlanner plan = {st};
      PtPiece pc;
      Boundary cut;
      while (plan.next(p, pc, cut)) {
        if (pc.b >= p.batch || plan.st.b >= p.batch) { wrong(now, "prompt", "behind the last sequence", Step{pc.b, pc.head, pc.tile, pc.u0, pc.u1, pc.units, 0, 0}); return; }
        w.pieces.push_back({pc.b, pc.head, pc.tile, pc.u0, pc.u1, pc.units, pc.n_rows, pc.first});
        if (pc.u0 > 0) w.cut = cut;
      }
    });
  }
  now.tile_rows = p.tile_rows = 64;
  check<FlatShape>(now, "flat", p, [&](TcStretch st, Walk& w) {
    TcPiece pc;
    while (tc_next<FlatShape>(p, st, pc)) {
      w.pieces.push_back({pc.b, pc.head, pc.tile, pc.u0, pc.u1, pc.units, pc.n_rows, pc.q.s.first});
      if (pc.u0 > 0) w.cut = {pc.seg0, pc.seg1, st.quota, pc.b, pc.head, pc.tile, pc.q.s.first, pc.n_rows, 0};
    }
  });
  // over the cache
  std::vector<int32_t> lens(c.keys.begin(), c.keys.end());
  AttnParams a = p;
  a.kv_len = lens.data();
  a.block_size = 16; a.shift = 4; a.max_blocks = *std::max_element(c.keys.begin(), c.keys.end()) / 16 + 1;
  now.tile_rows = a.tile_rows = kTcRows;
  a.head_dim = 128;
  check<TcShape>(now, "cache", a, [&](TcStretch st, Walk& w) {
    TcPiece pc;
    while (tc_next<TcShape>(a, st, pc)) {
      w.pieces.push_back({pc.b, pc.head, pc.tile, pc.u0, pc.u1, pc.units, pc.n_rows, pc.q.s.first});
      if (pc.u0 > 0) w.cut = {pc.seg0, pc.seg1, st.quota, pc.b, pc.head, pc.tile, pc.q.s.first, pc.n_rows, 0};
    }
  });
}

int main(int argc, char** argv) {
  const int g0 = argc > 1 ? atoi(argv[1]) : 1, g1 = argc > 2 ? atoi(argv[2]) : 64;
  for (int group = g0; group <= g1; ++group)
    for (int causal = 1; causal >= 0; --causal) {
      std::mt19937 rng(group * 2 + causal);
      auto upto = [&](int n) { return static_cast<int>(rng() % (n + 1)); };
      check_case({{2000, 2000, 2000, 2000}, {2000, 2000, 2000, 2000}, 8, group, 0, causal, 148, 0});
      check_case({{6000}, {6000}, 4, group, 0, causal, 148, 0});
      check_case({{300, 300}, {300, 300}, 3, group, 0, causal, 148, 0});
      check_case({{20, 130, 70}, {5020, 2130, 9070}, 4, group, 0, causal, 148, 0});
      for (int n = 0; n < 6; ++n) {
        Case c = {{}, {}, 1 + upto(7), group, 0, causal, n % 3 ? 148 : 1 + upto(295), 0};
        for (int b = 0, batch = 1 + upto(n % 2 ? 60 : 5); b < batch; ++b) {
          const int rows = upto(5) == 0 ? 0 : 1 + upto(n % 2 ? 90 : 1200), kind = upto(3);
          c.rows.push_back(rows);
          c.keys.push_back(kind == 0 ? rows : kind == 1 ? upto(rows) : rows + upto(n % 2 ? 300 : 6000));      // kind 1: rows that see nothing
        }
        if (*std::max_element(c.rows.begin(), c.rows.end()) > 0) check_case(c);
      }
    }
  if (g_wrong) printf("%d wrong\n", g_wrong);
  return g_wrong != 0;
}

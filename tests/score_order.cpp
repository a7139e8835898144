// The bar of the scores' join, walked on the host with the kernels' own rules: a set of which a logit may be taken has to be one whose logits were stored.
// Run by tests/test_score_order.py.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "score_order.hpp"

using namespace gensor;

static int failures = 0;
static long crossed = 0, walked = 0;

static void check(bool ok, const char* what, double x = 0, double y = 0) {
  if (!ok && ++failures < 20) std::printf("%s: %.9g %.9g\n", what, x, y);
}

static float nth_of(const std::vector<float>& x, int n) {
  return nth_reached(n, [&](uint32_t least) {
    int reach = 0;
    for (float v : x) reach += (uint32_t)(rank_key(v, 0) >> 32) >= least;
    return reach;
  });
}

// One token: pieces of whole sets, the bar of those before, and everything that a piece has not stored replaced by a number above all logits.
static void walk(const std::vector<float>& z, int set, int sets_a_piece, int top, int groups) {
  const int V = (int)z.size();
  const float stale = 3e38f;
  std::vector<uint64_t> best;
  float bar = NAN;
  for (int first = 0; first < V; first += set * sets_a_piece) {
    const int rows = std::min(set * sets_a_piece, V - first), sets = (rows + set - 1) / set;
    std::vector<float> maxima(sets, -INFINITY), most(groups, -INFINITY), logits((size_t)sets * set, stale);
    for (int s = 0; s < sets; ++s) {
      for (int i = first + s * set; i < std::min(first + (s + 1) * set, V); ++i) maxima[s] = std::max(maxima[s], z[i]);
      most[s % groups] = std::max(most[s % groups], maxima[s]);
      if (set_is_stored(maxima[s], bar))
        for (int i = 0; i < set; ++i) logits[s * set + i] = first + s * set + i < V ? z[first + s * set + i] : -INFINITY;
    }
    int above = 0;
    for (float m : most) above += m > bar;
    const float least = least_wanted(bar, above >= top, [&]() { return nth_of(most, top); });
    if (bar == bar) {
      check(!(least <= bar), "the bar fell", least, bar);
      crossed += above >= top && nth_of(most, top) <= bar;
    }
    for (int s = 0; s < sets; ++s) {
      if (!(maxima[s] >= least)) continue;
      check(set_is_stored(maxima[s], bar), "not stored", maxima[s], bar);
      for (int i = 0; i < set && first + s * set + i < V; ++i)
        if (logits[s * set + i] >= least) best.push_back(rank_key(logits[s * set + i], first + s * set + i));
    }
    std::sort(best.begin(), best.end(), std::greater<uint64_t>());
    if ((int)best.size() > top) best.resize(top);
    bar = (int)best.size() == top ? key_value(best.back()) : NAN;
    ++walked;
  }
  std::vector<int> order(V);
  for (int i = 0; i < V; ++i) order[i] = i;
  std::stable_sort(order.begin(), order.end(), [&](int x, int y) { return z[x] > z[y]; });
  for (int r = 0; r < top; ++r) {
    check(key_entry(best[r]) == order[r], "entry", key_entry(best[r]), order[r]);
    check(key_value(best[r]) == z[order[r]], "value", key_value(best[r]), z[order[r]]);
  }
}

int main() {
  // ---- the order, the number above, the number that so many reach
  std::vector<float> line = {-INFINITY, -3.402823466e38f, -1.f, -1.17549435e-38f, -1.4e-45f, 0.f, 1.4e-45f, 1.17549435e-38f, 0.99999994f, 1.f, 3.402823466e38f, INFINITY};
  for (size_t i = 0; i < line.size(); ++i) {
    check(key_value(rank_key(line[i], 7)) == line[i] && key_entry(rank_key(line[i], 7)) == 7, "key", line[i]);
    check(rank_key(line[i], 5) > rank_key(line[i], 6) && rank_key(line[i], 2147483647) > 0, "lower entry first", line[i]);
    if (i) check(rank_key(line[i], 9) > rank_key(line[i - 1], 3), "order", line[i]);
    if (i + 1 < line.size()) check(next_above(line[i]) == std::nextafter(line[i], INFINITY), "above", line[i], next_above(line[i]));
  }
  check(rank_key(-0.f, 1) == rank_key(0.f, 1) && next_above(-0.f) == 1.4e-45f, "minus zero");
  check(next_above(INFINITY) != next_above(INFINITY) && next_above(NAN) != next_above(NAN), "above infinity");
  check(least_wanted(INFINITY, false, []() { return 0.f; }) != least_wanted(INFINITY, false, []() { return 0.f; }), "nothing is above infinity");
  check(least_wanted(-INFINITY, false, []() { return 0.f; }) == -3.402823466e38f && least_wanted(NAN, false, []() { return 2.f; }) == 2.f, "bars");
  check(least_wanted(5.f, true, []() { return 4.f; }) == next_above(5.f) && least_wanted(5.f, true, []() { return 6.f; }) == 6.f, "the larger one");
  check(least_wanted(5.f, true, []() { return -INFINITY; }) == next_above(5.f), "none that reach");

  std::mt19937 g(7);
  for (int n = 0; n < 300; ++n) {
    std::vector<float> x(64);
    std::normal_distribution<float> d(n % 3 == 0 ? 0.f : n % 3 == 1 ? 100.f : -100.f, n % 2 ? 1.f : 0.01f);
    for (float& v : x) v = d(g);
    std::vector<float> sorted = x;
    std::sort(sorted.begin(), sorted.end(), std::greater<float>());
    for (int k : {1, 8, 64}) {
      const float r = nth_of(x, k);
      check(r <= sorted[k - 1] && r >= sorted[k - 1] - std::fabs(sorted[k - 1]) * (1.f / 1024), "nth", r, sorted[k - 1]);
    }
    check(nth_of(x, 65) == -INFINITY, "fewer than that");
  }

  // ---- whole tokens
  struct Spread { float mean, width; bool even; };
  for (const Spread& s : {Spread{100.f, 0.005f, true}, Spread{-100.f, 0.005f, true}, Spread{100.f, 0.1f, false}, Spread{20.f, 0.2f, false}, Spread{-20.f, 0.2f, false}, Spread{0.f, 2.f, false}})
    for (int top : {1, 8, 40, 64})
      for (int n = 0; n < 40; ++n) {
        std::vector<float> z(9000 + 37 * n);
        std::uniform_real_distribution<float> u(s.mean - s.width, s.mean + s.width);
        std::normal_distribution<float> d(s.mean, s.width);
        for (float& v : z) v = s.even ? u(g) : d(g);
        if (n % 8 == 7)
          for (float& v : z) v = s.mean + std::round((v - s.mean) / s.width) * s.width / 64;        // many equal ones
        walk(z, n % 2 ? 32 : 16, n % 3 == 0 ? 8 : n % 3 == 1 ? 64 : 130, top, top > 24 ? 256 : 64);
      }
  std::printf("%ld pieces, the cut number at or below the bar in %ld, %d failures\n", walked, crossed, failures);
  return failures != 0 || crossed < 100;
}

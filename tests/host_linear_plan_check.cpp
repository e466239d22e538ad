// Host-only check of the linear attention planner (plan.cpp), built with g++ and the address and undefined-behaviour
// sanitizers by tests/test_linear_plan_host.py.  Randomized calls (0 to 2^31 - 1 tokens, empty sequences, 1 to 128 KV heads,
// 1 to 16 query heads each, states in place, forked, fresh and not kept) are planned, and the plan is carried out with a
// number for a state (every token adds its own) in the order of the launches: sums, scans, items.
//   - every token of every query head belongs to exactly one item, whose state before it is the sum of its sequence's source
//     and earlier tokens;
//   - a destination gets its sequence's whole sum from exactly one item, no other item of that launch reads it;
//   - the workspace is read where it was written, its parts are within linear_most_parts, whatever the query heads;
//   - sequences without tokens cost nothing unless their state moves, and change nothing about the others' work.
// `self-test` plants mistakes into plans and expects the checks to reject each of them.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <random>
#include <vector>

#include "../paper_2608_11152_amd/csrc/kvp_plan.h"

using kvp::LinearItem;
using kvp::LinearPlan;

#define EXPECT(c, ...)                                    \
  do {                                                    \
    if (!(c)) {                                           \
      if (!g_quiet) {                                     \
        std::fprintf(stderr, "check failed: " __VA_ARGS__); \
        std::fprintf(stderr, "\n");                       \
      }                                                   \
      return false;                                       \
    }                                                     \
  } while (0)

static bool g_quiet = false;
static std::mt19937_64 rng;

static int64_t between(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }

struct Call {
  std::vector<int32_t> cu, src, dst;
  int Hkv = 1, G = 1, D = 64, slots = 0;
  int size() const { return (int)src.size(); }
  int32_t n(int i) const { return cu[i + 1] - cu[i]; }
};

static LinearPlan plan_of(const Call& c) {
  LinearPlan P;
  kvp::plan_linear(c.cu.data(), c.size(), c.Hkv, c.D, c.G, c.src.data(), c.dst.data(), &P);
  return P;
}

// The sum of the numbers of tokens [a, b): token t counts t + 1 (modulo 2^64).
static uint64_t tokens(int64_t a, int64_t b) { return (uint64_t)(a + 1 + b) * (uint64_t)(b - a) / 2; }
static uint64_t slot_value(int slot) { return slot < 0 ? 0 : 0x9e3779b97f4a7c15ull * (uint64_t)(slot + 1); }

static bool check(const Call& c, const LinearPlan& P) {
  const int64_t most = kvp::linear_most_parts(c.cu.data(), c.size(), c.Hkv, c.D);
  EXPECT(P.parts >= 0 && P.parts <= most, "%d parts, %lld promised", P.parts, (long long)most);
  std::vector<uint64_t> part(P.parts, 0);
  std::vector<char> written(P.parts, 0);
  auto slot = [&](int s) { return -2 - s; };
  for (const LinearItem& it : P.sums) {
    EXPECT(slot(it.dst) >= 0 && slot(it.dst) < P.parts && !written[slot(it.dst)], "sum into part %d", slot(it.dst));
    EXPECT(it.n > 0, "a sum of %d tokens", it.n);
    written[slot(it.dst)] = 1;
    part[slot(it.dst)] = tokens(it.t0, (int64_t)it.t0 + it.n);
  }
  for (const auto& s : P.scans) {
    EXPECT(s.n >= 1 && s.part >= 0 && s.part + s.n <= P.parts, "scan of parts %d + %d", s.part, s.n);
    EXPECT(s.src >= -1 && s.src < c.slots, "scan from slot %d", s.src);
    uint64_t S = slot_value(s.src);
    if (s.src >= 0) {
      EXPECT(!written[s.part], "part %d is written twice", s.part);
      part[s.part] = S;
      written[s.part] = 1;
    }
    for (int i = 1; i < s.n; ++i) {
      EXPECT(written[s.part + i], "part %d has no sum", s.part + i);
      part[s.part + i] = S += part[s.part + i];
    }
  }
  struct Use {
    int writers = 0;
    int readers_apart = 0;  // items that read it and do not write it
  };
  std::map<int, Use> use;
  std::map<int, int> seq_of;                         // first token -> sequence with tokens
  for (int i = 0; i < c.size(); ++i)
    if (c.n(i) > 0) seq_of[c.cu[i]] = i;
  std::vector<std::vector<const LinearItem*>> work(c.size());
  std::vector<const LinearItem*> empty;
  for (const LinearItem& it : P.items) {
    EXPECT(it.n >= 0 && it.g0 >= 0 && it.gn >= 1 && it.g0 + it.gn <= c.G, "item heads %d + %d", it.g0, it.gn);
    EXPECT(it.dst >= -1 && it.dst < c.slots && it.src < c.slots, "item slots");
    if (it.src <= -2) EXPECT(slot(it.src) < P.parts && written[slot(it.src)], "item reads part %d", slot(it.src));
    if (it.dst >= 0) ++use[it.dst].writers;
    if (it.src >= 0 && it.src != it.dst) ++use[it.src].readers_apart;
    if (it.n == 0) {
      empty.push_back(&it);
      continue;
    }
    auto s = seq_of.upper_bound(it.t0);
    EXPECT(s != seq_of.begin(), "item in no sequence");
    work[(--s)->second].push_back(&it);
  }
  for (const auto& u : use)
    EXPECT(u.second.writers <= 1 && (u.second.writers == 0 || u.second.readers_apart == 0),
           "slot %d: %d writers, %d other readers", u.first, u.second.writers, u.second.readers_apart);
  for (int i = 0; i < c.size(); ++i) {
    if (c.n(i) == 0) {
      if (c.dst[i] >= 0 && c.dst[i] != c.src[i]) {
        bool found = false;
        for (const LinearItem* it : empty) found |= it->src == c.src[i] && it->dst == c.dst[i];
        EXPECT(found, "sequence %d does not hand its state on", i);
      }
      continue;
    }
    std::map<int32_t, int> heads;  // first token of a part -> query heads done
    std::map<int32_t, int32_t> length;  // and its tokens
    int64_t covered = 0;
    bool kept = false;
    for (const LinearItem* it : work[i]) {
      const uint64_t before = it->src <= -2 ? part[slot(it->src)] : slot_value(it->src);
      EXPECT(before == slot_value(c.src[i]) + tokens(c.cu[i], it->t0), "the state before token %d", it->t0);
      EXPECT(it->t0 >= c.cu[i] && (int64_t)it->t0 + it->n <= c.cu[i + 1], "item beyond its sequence");
      EXPECT(it->g0 == heads[it->t0] || it->gn == c.G, "heads %d of token %d out of turn", it->g0, it->t0);
      heads[it->t0] += it->gn;
      EXPECT(length.emplace(it->t0, it->n).first->second == it->n, "parts of two lengths at token %d", it->t0);
      if (it->g0 == 0) covered += it->n;
      if (it->dst >= 0) {
        EXPECT(it->dst == c.dst[i] && it->t0 + it->n == c.cu[i + 1] && !kept, "slot %d is not what item keeps", it->dst);
        kept = true;
      }
    }
    for (const auto& h : heads) EXPECT(h.second == c.G, "%d of %d query heads", h.second, c.G);
    EXPECT(covered == c.n(i), "%lld of %d tokens", (long long)covered, c.n(i));
    EXPECT(kept == (c.dst[i] >= 0), "the state of sequence %d", i);
  }
  return true;
}

static bool alone(const Call& c, const LinearPlan& P) {
  size_t moved = 0, empty = 0;
  Call d = c;
  d.cu = {0};
  d.src.clear(), d.dst.clear();
  for (int i = 0; i < c.size(); ++i) {
    if (c.n(i) == 0) {
      moved += c.dst[i] >= 0 && c.dst[i] != c.src[i];
      continue;
    }
    d.cu.push_back(c.cu[i + 1]);
    d.src.push_back(c.src[i]);
    d.dst.push_back(c.dst[i]);
  }
  for (const LinearItem& it : P.items) empty += it.n == 0;
  EXPECT(empty == moved, "%zu items without tokens, %zu states move", empty, moved);
  const LinearPlan Q = plan_of(d);
  EXPECT(Q.items.size() + empty == P.items.size() && Q.parts == P.parts && Q.sums.size() == P.sums.size(),
         "%zu items and %d parts, without the empty sequences %zu and %d", P.items.size(), P.parts, Q.items.size(), Q.parts);
  return true;
}

static Call random_call() {
  Call c;
  c.D = between(0, 1) ? 128 : 64;
  c.Hkv = 1 << between(0, 7);
  if (between(0, 3) == 0) c.Hkv = (int)between(1, 128);
  c.G = 1 << between(0, 4);
  const int B = (int)between(1, between(0, 1) ? 6 : 300);
  const int64_t hi = 1ll << between(0, 20);
  const int kinds = (int)between(0, 2);  // tokens for all, some, few
  int64_t at = 0;
  c.cu.push_back(0);
  for (int i = 0; i < B; ++i) {
    const bool idle = kinds > 0 && between(0, kinds == 1 ? 2 : 20) > 0;
    at += idle ? 0 : between(kinds == 0 ? 1 : 0, hi);
    c.cu.push_back((int32_t)std::min<int64_t>(at, INT32_MAX));
  }
  if (between(0, 9) == 0) c.cu.back() = INT32_MAX;
  c.slots = 2 * B + 1;
  for (int i = 0; i < B; ++i) {
    const int k = (int)between(0, 4);  // in place, fresh, fork, not kept, handed nowhere
    c.src.push_back(k == 0 ? i : k == 1 ? -1 : k == 2 || k == 3 ? 2 * B : -1);
    c.dst.push_back(k == 3 || k == 4 ? -1 : i);
  }
  return c;
}

static int64_t g_parts = 0, g_split = 0;

static bool run(const Call& c) {
  const LinearPlan P = plan_of(c);
  g_parts += P.parts;
  for (const LinearItem& it : P.items) g_split += it.gn < c.G;
  return check(c, P) && alone(c, P);
}

static bool self_test() {
  int planted = 0, rejected = 0;
  g_quiet = true;
  for (int k = 0; k < 3000; ++k) {
    const Call c = random_call();
    LinearPlan P = plan_of(c);
    if (P.items.empty()) continue;
    LinearItem& it = P.items[between(0, (int64_t)P.items.size() - 1)];
    switch (between(0, 8)) {
      case 0: it = P.items.back(), P.items.pop_back(); break;
      case 1: if (it.n == 0) continue; it.t0 += 1; break;
      case 2: if (it.n == 0) continue; it.n -= 1; break;
      case 3: if (it.src == -1) continue; it.src = -1; break;
      case 4: if (it.dst == -1) continue; it.dst = -1; break;
      case 5: if (it.n == 0 || it.gn == 1) continue; it.gn /= 2; break;
      case 6: if (P.sums.empty()) continue; P.sums.pop_back(); break;
      case 7:  // (two parts from zeros are what they were)
        if (P.scans.empty() || (P.scans.back().src < 0 && P.scans.back().n <= 2)) continue;
        P.scans.pop_back();
        break;
      case 8: P.parts = (int)kvp::linear_most_parts(c.cu.data(), c.size(), c.Hkv, c.D) + 1; break;
    }
    ++planted;
    rejected += !(check(c, P) && alone(c, P));
  }
  std::printf("self-test: %d of %d planted mistakes rejected\n", rejected, planted);
  return planted > 500 && rejected == planted;
}

int main(int argc, char** argv) {
  if (argc > 1 && !std::strcmp(argv[1], "self-test")) return self_test() ? 0 : 1;
  const int iters = argc > 1 ? std::atoi(argv[1]) : 200;
  rng.seed(argc > 2 ? std::strtoull(argv[2], nullptr, 10) : 12345);
  for (int k = 0; k < iters; ++k)
    if (!run(random_call())) {
      std::fprintf(stderr, "call %d\n", k);
      return 1;
    }
  if (g_parts == 0 || g_split == 0) return 1;
  std::printf("ok: %d plans checked, %lld parts, %lld items of shared-out heads\n", iters, (long long)g_parts,
              (long long)g_split);
  return 0;
}

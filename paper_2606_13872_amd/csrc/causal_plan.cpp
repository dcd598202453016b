// Work items of causal attention over packed sequences (host only, plain C++).
//
// An item costs its steps (64-key or 64-token LDS tiles); items are launched longest first, so that the
// short ones fill the compute units that long ones leave (a causal prompt's items differ by as much as its
// length). K/V heads are innermost: item i runs on XCD i % 8, so with 8 heads (or a multiple, or 1, 2, 4) an XCD
// streams the K and V of one of them through its L2. Where a launch has few, long items, they are cut into
// pieces whose partial sums a second kernel adds up: the launch is replayed on 256 compute units for a few
// lengths of the pieces and the one that ends first is taken.
#include "sra_causal.h"

#include <algorithm>
#include <functional>
#include <queue>

namespace sra {

namespace {

// Costs in steps of a forward item (64 keys x 256 rows). A dQ step computes three products to the
// forward's two, a dK/dV step four; both run at one wave per SIMD.
constexpr double kStepCost[3] = {1.0, 1.5, 2.0};
constexpr double kItemCost = 2.5;      // an item's loads before the first product and its epilogue
constexpr double kCombineCost = 3.5;   // the combine launch
constexpr double kSlotCost[3] = {0.25, 0.25, 0.5};  // writing and reading the partial results of one piece
constexpr int kMaxSplit = 32;
constexpr size_t kSplitItems = 2048;   // launches of more items are not cut (eight rounds of 256)

struct Unit {
  CausalItem it;
  int32_t steps;
  double cost() const { return steps * kStepCost[it.kind]; }
};

int pieces_of(const Unit& u, double cap) {
  if (cap <= 0 || u.cost() <= cap || u.steps < 4) return 1;
  const int n = int(u.cost() / cap) + 1;
  return std::min({n, kMaxSplit, u.steps / 2});
}

// When the last of the launch's pieces ends, launched longest first on 256 compute units.
double replay(const std::vector<Unit>& units, double cap) {
  std::vector<double> c;
  bool split = false;
  for (const Unit& u : units) {
    const int n = pieces_of(u, cap);
    split |= n > 1;
    for (int i = 0; i < n; ++i) {
      const int steps = u.steps * (i + 1) / n - u.steps * i / n;
      c.push_back(kItemCost + steps * kStepCost[u.it.kind] + (n > 1 ? kSlotCost[u.it.kind] : 0.0));
    }
  }
  std::sort(c.begin(), c.end(), std::greater<double>());
  std::priority_queue<double, std::vector<double>, std::greater<double>> cu;
  for (int i = 0; i < kNumCus; ++i) cu.push(0.0);
  double end = 0;
  for (double x : c) {
    const double t = cu.top() + x;
    cu.pop();
    cu.push(t);
    end = std::max(end, t);
  }
  return end + (split ? kCombineCost : 0.0);
}

double choose_cap(const std::vector<Unit>& units) {
  if (units.empty() || units.size() > kSplitItems) return 0;
  double total = 0;
  for (const Unit& u : units) total += u.cost();
  double best_cap = 0, best = replay(units, 0);
  for (double f : {2.0, 1.4, 1.0, 0.8, 0.65, 0.5, 0.4, 0.33, 0.25}) {
    const double cap = std::max(f * total / kNumCus, 4.0);
    const double t = replay(units, cap);
    if (t < 0.97 * best) best = t, best_cap = cap;
  }
  return best_cap;
}

// Appends the units' items, cut where `cap` says, longest first.
void emit(const std::vector<Unit>& units, double cap, std::vector<CausalItem>* items,
          std::vector<CausalItem>* combine, int32_t slots[3]) {
  std::vector<std::pair<double, CausalItem>> out;
  for (const Unit& u : units) {
    const int n = pieces_of(u, cap);
    if (n > 1) {
      CausalItem c = u.it;
      c.lo = slots[u.it.kind];
      c.hi = n;
      combine->push_back(c);
    }
    for (int i = 0; i < n; ++i) {
      CausalItem x = u.it;
      const int a = u.steps * i / n, b = u.steps * (i + 1) / n;
      if (u.it.kind == kDkv) {
        x.lo = a;
        x.hi = b;
      } else {
        x.lo = 64 * a;
        x.hi = std::min(64 * b, u.it.hi);
      }
      if (n > 1) x.slot = ++slots[u.it.kind];
      out.emplace_back((b - a) * kStepCost[u.it.kind], x);
    }
  }
  std::stable_sort(out.begin(), out.end(), [](const auto& a, const auto& b) { return a.first > b.first; });
  for (auto& x : out) items->push_back(x.second);
}

}  // namespace

void build_causal_tables(CausalTables* t) {
  const int32_t G = t->heads / t->kv_heads;
  std::vector<Unit> fwd, dq, dkv;
  int32_t q0 = 0, k0 = 0;
  for (int32_t b = 0; b < t->batch; ++b) {
    const int32_t nq = t->nq[b], nk = t->nk[b];
    const int32_t rows = nq * G;
    for (int32_t r = 0; r < rows; r += kCausalTile) {
      const int32_t len = std::min(kCausalTile, rows - r);
      const int32_t keys = std::max(0, (r + len - 1) / G + nk - nq + 1);  // seen by the last row
      for (int32_t h = 0; h < t->kv_heads; ++h) {
        const CausalItem it{kForward, h, r, len, q0, nq, k0, nk, 0, keys, 0, b};
        fwd.push_back({it, (keys + 63) / 64});
        if (t->backward) {
          dq.push_back(fwd.back());
          dq.back().it.kind = kDq;
        }
      }
    }
    if (t->backward)
      for (int32_t k = 0; k < nk; k += kCausalTile) {
        CausalItem it{kDkv, 0, k, std::min(kCausalTile, nk - k), q0, nq, k0, nk, 0, 0, 0, b};
        it.hi = G * causal_tiles(it).n;
        for (it.kvh = 0; it.kvh < t->kv_heads; ++it.kvh) dkv.push_back({it, it.hi});
      }
    q0 += nq;
    k0 += nk;
  }
  int32_t slots[3] = {0, 0, 0};
  emit(fwd, choose_cap(fwd), &t->fwd, &t->fwd_combine, slots);
  if (dq.size() + dkv.size() <= kSplitItems) {  // few items: both kinds together, each fills the other's gaps
    std::vector<Unit> both(dkv);
    both.insert(both.end(), dq.begin(), dq.end());
    emit(both, choose_cap(both), &t->grad, &t->grad_combine, slots);
  } else {  // many: one kind after the other, so that an XCD streams one kind of rows at a time
    emit(dkv, 0, &t->grad, &t->grad_combine, slots);
    emit(dq, 0, &t->grad, &t->grad_combine, slots);
  }
  t->fwd_slots = slots[kForward];
  t->q_slots = slots[kDq];
  t->kv_slots = slots[kDkv];
}

}  // namespace sra

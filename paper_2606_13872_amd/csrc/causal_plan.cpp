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

// Costs in steps of a forward item (64 keys x 256 rows; 1.75 us at head_dim 128, measured, as the others are). A
// dQ step computes three products to the forward's two, a dK/dV step four.
constexpr double kStepCost[3] = {1.0, 1.5, 1.85};
constexpr double kItemCost[3] = {2.9, 4.5, 6.0};  // an item's loads before the first product, diagonal and epilogue
constexpr double kSlotCost[3] = {2.2, 2.2, 4.5};  // writing the 32-bit partial results of a piece
constexpr double kCombineCost = 3.0;              // the combine launch,
constexpr double kCombineSlot = 0.025;            // and reading a piece's results there
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
  double combine = 0;
  for (const Unit& u : units) {
    const int n = pieces_of(u, cap);
    if (n > 1) combine += n * kCombineSlot * (u.it.kind == kDkv ? 2 : 1);
    for (int i = 0; i < n; ++i) {
      const int steps = u.steps * (i + 1) / n - u.steps * i / n;
      c.push_back(kItemCost[u.it.kind] + steps * kStepCost[u.it.kind] + (n > 1 ? kSlotCost[u.it.kind] : 0.0));
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
  return end + (combine > 0 ? kCombineCost + combine : 0.0);
}

double choose_cap(const std::vector<Unit>& units) {
  if (units.empty() || units.size() > kSplitItems) return 0;
  double total = 0;
  for (const Unit& u : units) total += u.cost();
  double best_cap = 0, best = replay(units, 0);
  for (double f : {2.0, 1.7, 1.4, 1.2, 1.0, 0.9, 0.8, 0.7, 0.6, 0.5, 0.4, 0.3, 0.2}) {
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
  int64_t n = 0;
  for (int32_t nq : t->nq) n += (int64_t(nq) * G + kCausalTile - 1) / kCausalTile * t->kv_heads;
  // Launches that are not cut anyway take larger forward items.
  t->fwd_tile = n > int64_t(kSplitItems) ? fwd_large_tile(t->head_dim) : kCausalTile;
  std::vector<Unit> fwd, dq, dkv;
  int32_t q0 = 0, k0 = 0;
  for (int32_t b = 0; b < t->batch; ++b) {
    const int32_t nq = t->nq[b], nk = t->nk[b];
    const int32_t rows = nq * G;
    auto row_items = [&](CausalKind kind, int32_t tile, std::vector<Unit>* out) {
      for (int32_t r = 0; r < rows; r += tile) {
        const int32_t len = std::min(tile, rows - r);
        const int32_t keys = std::max(0, (r + len - 1) / G + nk - nq + 1);  // seen by the last row
        for (int32_t h = 0; h < t->kv_heads; ++h)
          out->push_back({CausalItem{kind, h, r, len, q0, nq, k0, nk, 0, keys, 0, b}, (keys + 63) / 64});
      }
    };
    row_items(kForward, t->fwd_tile, &fwd);
    if (t->backward) row_items(kDq, kCausalTile, &dq);
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

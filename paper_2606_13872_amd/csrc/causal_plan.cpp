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

namespace sra {

namespace {

// Costs in steps of a forward item (64 keys x 256 rows; 1.75 us at head_dim 128, measured, as the others are). A
// dQ step computes three products to the forward's two, a dK/dV step four.
constexpr double kStepCost[3] = {1.0, 1.5, 1.85};
constexpr double kItemCost[3] = {2.9, 4.5, 6.0};  // an item's loads before the first product, diagonal and epilogue
constexpr double kSlotCost[3] = {2.2, 2.2, 4.5};  // writing the 32-bit partial results of a piece
constexpr double kCombineCost = 3.0;              // the combine launch,
constexpr double kCombineSlot = 0.025;            // and reading a piece's results there
// A step of a large forward item (384 or 512 rows) to one of 256 rows: 0.93 times the work's share.
constexpr double large_step(int head_dim) { return 0.93 * fwd_large_tile(head_dim) / kCausalTile; }
// Steps of 64 head dims take 0.6 times as long, what does not depend on them is worth more of them.
constexpr double fixed_cost(int head_dim) { return head_dim == 128 ? 1.0 : 1.7; }
constexpr int kMaxSplit = 32;
constexpr size_t kSplitItems = 2048;   // launches of more items are not cut (eight rounds of 256)

struct Unit {
  CausalItem it;
  int32_t steps;
  double step;  // cost of one
  double cost() const { return steps * step; }
};

int pieces_of(const Unit& u, double cap) {
  if (cap <= 0 || u.cost() <= cap || u.steps < 4) return 1;
  const int n = int(u.cost() / cap) + 1;
  return std::min({n, kMaxSplit, u.steps / 2});
}

// When the last of the launch's pieces ends, launched longest first on 256 compute units.
double replay(const std::vector<Unit>& units, double cap, double fixed) {
  std::vector<double> c;
  c.reserve(units.size() * 2);
  double combine = 0;
  for (const Unit& u : units) {
    const int n = pieces_of(u, cap);
    if (n > 1) combine += n * kCombineSlot * (u.it.kind == kDkv ? 2 : 1);
    for (int i = 0; i < n; ++i) {
      const int steps = u.steps * (i + 1) / n - u.steps * i / n;
      c.push_back(fixed * kItemCost[u.it.kind] + steps * u.step + (n > 1 ? kSlotCost[u.it.kind] : 0.0));
    }
  }
  std::sort(c.begin(), c.end(), std::greater<double>());
  double heap[kNumCus] = {};  // when each compute unit is free; the first is the least
  double end = 0;
  for (double x : c) {
    const double t = heap[0] + x;
    int i = 0;
    for (int k; (k = 2 * i + 1) < kNumCus; i = k) {
      if (k + 1 < kNumCus && heap[k + 1] < heap[k]) ++k;
      if (heap[k] >= t) break;
      heap[i] = heap[k];
    }
    heap[i] = t;
    end = std::max(end, t);
  }
  return end + (combine > 0 ? fixed * kCombineCost + combine : 0.0);
}

// The cost from which on items are cut (0: none is), and when the launch then ends.
double choose_cap(const std::vector<Unit>& units, double fixed, double* end) {
  double total = 0;
  for (const Unit& u : units) total += u.cost();
  double best_cap = 0, best = replay(units, 0, fixed);
  for (double f : {2.0, 1.5, 1.2, 1.1, 1.0, 0.8, 0.65, 0.5, 0.35}) {
    const double cap = std::max(f * total / kNumCus, 4.0);
    const double t = replay(units, cap, fixed);
    if (t < 0.97 * best) best = t, best_cap = cap;
  }
  if (end) *end = best;
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
      out.emplace_back((b - a) * u.step, x);
    }
  }
  std::stable_sort(out.begin(), out.end(), [](const auto& a, const auto& b) { return a.first > b.first; });
  for (auto& x : out) items->push_back(x.second);
}

}  // namespace

void build_causal_tables(CausalTables* t) {
  const int32_t G = t->heads / t->kv_heads;
  const double fixed = fixed_cost(t->head_dim);
  // Items of `tile` rows or keys each, K/V heads innermost.
  auto units = [&](CausalKind kind, int32_t tile, double step) {
    std::vector<Unit> out;
    int32_t q0 = 0, k0 = 0;
    for (int32_t b = 0; b < t->batch; ++b) {
      const int32_t nq = t->nq[b], nk = t->nk[b], n = kind == kDkv ? nk : nq * G;
      for (int64_t at = 0; at < n; at += tile) {
        const int32_t r = int32_t(at);
        CausalItem it{kind, 0, r, std::min(tile, n - r), q0, nq, k0, nk, 0, 0, 0, b};
        int32_t steps;
        if (kind == kDkv) {
          steps = it.hi = G * causal_tiles(it).n;
        } else {
          it.hi = std::max(0, (r + it.len - 1) / G + nk - nq + 1);  // keys seen by the last row
          steps = (it.hi + 63) / 64;
        }
        for (it.kvh = 0; it.kvh < t->kv_heads; ++it.kvh) out.push_back({it, steps, step});
      }
      q0 += nq;
      k0 += nk;
    }
    return out;
  };
  int32_t slots[3] = {0, 0, 0};
  std::vector<Unit> fwd = units(kForward, kCausalTile, kStepCost[kForward]);
  double cap = 0, end = 0;
  t->fwd_tile = fwd_large_tile(t->head_dim);
  if (fwd.size() <= kSplitItems) {  // larger items, or these, cut or not: whichever end first
    cap = choose_cap(fwd, fixed, &end);
    if (end <= replay(units(kForward, t->fwd_tile, large_step(t->head_dim)), 0, fixed)) t->fwd_tile = kCausalTile;
  }
  if (t->fwd_tile != kCausalTile) {
    fwd = units(kForward, t->fwd_tile, large_step(t->head_dim));
    cap = 0;
  }
  emit(fwd, cap, &t->fwd, &t->fwd_combine, slots);
  if (t->backward) {
    std::vector<Unit> dkv = units(kDkv, kCausalTile, kStepCost[kDkv]), dq = units(kDq, kCausalTile, kStepCost[kDq]);
    if (dq.size() + dkv.size() <= kSplitItems) {  // few items: both kinds together, each fills the other's gaps
      dkv.insert(dkv.end(), dq.begin(), dq.end());
      emit(dkv, choose_cap(dkv, fixed, nullptr), &t->grad, &t->grad_combine, slots);
    } else {  // many: one kind after the other, so that an XCD streams one kind of rows at a time
      emit(dkv, 0, &t->grad, &t->grad_combine, slots);
      emit(dq, 0, &t->grad, &t->grad_combine, slots);
    }
  }
  t->fwd_slots = slots[kForward];
  t->q_slots = slots[kDq];
  t->kv_slots = slots[kDkv];
}

}  // namespace sra

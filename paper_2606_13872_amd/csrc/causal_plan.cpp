// Work items of causal attention over packed sequences (host only, plain C++).
//
// An item costs its steps (64-key or 64-token LDS tiles); items are launched longest first, so that the
// short ones fill the compute units that long ones leave (a causal prompt's items differ by as much as its
// length). K/V heads are innermost: item i runs on XCD i % 8, so with 8 heads (or a multiple, or 1, 2, 4) an XCD
// streams the K and V of one of them through its L2. Where a launch has few, long items, they are cut into
// pieces whose partial sums a second kernel adds up: the launch is replayed on 256 compute units for a few sizes and
// lengths of the pieces and the one that ends first is taken.
#include "sra_causal.h"

#include <algorithm>
#include <functional>
#include <limits>

namespace sra {

namespace {

// Costs of a kind of items, in steps of its launch's unit.
struct Cost {
  double step;            // 64 keys (dK/dV: 64 tokens)
  double item;            // its loads before the first product, diagonal and epilogue
  double slot;            // writing the 32-bit partial results of a piece
  double combine, part;   // the combine launch, and reading a piece's results there
};
// Forward, in steps of 256 rows (1.4 us at head_dim 128, 1.05 at 64 where power does not bound them). Fitted to 44
// sets of lengths, each with the items of 128 and of 256 rows cut at six lengths: what is chosen by them is 1.6 % slower
// than the best of the twelve on average, 15 % at most (items of 256 rows alone: 20 and 70 %).
constexpr Cost kSmallForward = {0.62, 4.2, 0.2, 2.75, 0.009};  // 128 rows
constexpr Cost kForwardCost = {1.0, 5.9, 1.7, 2.75, 0.009};    // 256 rows
// A step of a large item (384 or 512 rows) to one of 256 rows: 0.93 times the work's share.
constexpr double large_step(int head_dim) { return 0.93 * fwd_large_tile(head_dim) / kCausalTile; }
constexpr int kSmallTile = kCausalTile / 2;
// Backward, in the same way (1.75 and 1.05 us): a dQ step computes three products to the forward's two, a dK/dV step
// four. Fitted with pairs of 256 and 128 keys and rows: 2 to 3 % slower than the best on average.
constexpr Cost kDkvCost = {1.77, 7.2, 4.3, 1.5, 0.012}, kSmallDkv = {1.75, 5.5, 2.2, 1.5, 0.012};
constexpr Cost kDqCost = {1.2, 8.8, 1.8, 1.5, 0.006}, kSmallDq = {1.14, 5.4, 0.9, 1.5, 0.006};
constexpr int kMaxSplit = 32;
constexpr size_t kSplitItems = 2048;   // launches of more items are not cut (eight rounds of 256)
// Launches of 256 rows or keys that end later are not tried with 128: what they may gain (1 to 3 %) is less than planning
// them costs a caller who has other lengths in each step.
constexpr double kSmallEnd = 128;

// An item of K/V head 0, uncut; those of the other heads are like it.
struct Unit {
  CausalItem it;
  int32_t steps;
  const Cost* each;
  double cost() const { return steps * each->step; }
};

int pieces_of(const Unit& u, double cap) {
  if (cap <= 0 || u.cost() <= cap || u.steps < 4) return 1;
  const int n = int(u.cost() / cap) + 1;
  return std::min({n, kMaxSplit, u.steps / 2});
}

// When the last of the launch's pieces ends, launched longest first on 256 compute units; `limit` if not before that.
double replay(const std::vector<Unit>& units, int32_t heads, double cap, double limit) {
  std::vector<double> c;
  c.reserve(units.size() * 2);
  double combine = 0, sum = 0;
  for (const Unit& u : units) {
    const int n = pieces_of(u, cap);
    if (n > 1) combine = std::max(combine, u.each->combine);
    for (int i = 0; i < n; ++i) {
      const int steps = u.steps * (i + 1) / n - u.steps * i / n;
      c.push_back(u.each->item + steps * u.each->step + (n > 1 ? u.each->slot : 0.0));
      sum += c.back();
    }
    if (n > 1) combine += n * u.each->part * heads;
  }
  if (sum * heads / kNumCus + combine >= limit) return limit;
  std::sort(c.begin(), c.end(), std::greater<double>());
  double heap[kNumCus] = {};  // when each compute unit is free; the first is the least
  double end = 0;
  for (double x : c)
    for (int32_t h = 0; h < heads; ++h) {
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
  return std::min(end + combine, limit);
}

// Sets `cap`, the cost from which on items are cut (0: none is), and `end`, when the launch then ends, if that is
// before *end.
bool choose_cap(const std::vector<Unit>& units, int32_t heads, double* cap, double* end) {
  double total = 0, best = *end;
  for (const Unit& u : units) total += heads * u.cost();
  auto consider = [&](double c, double least) {
    const double t = replay(units, heads, c, least * best);
    if (t < least * best) best = t, *cap = c;
  };
  consider(0, 1.0);
  for (double f : {2.0, 1.5, 1.2, 1.1, 1.0, 0.8, 0.65, 0.5, 0.35}) consider(std::max(f * total / kNumCus, 4.0), 0.97);
  const bool better = best < *end;
  *end = best;
  return better;
}

// Appends the units' items, cut where `cap` says, longest first.
void emit(const std::vector<Unit>& units, int32_t heads, double cap, std::vector<CausalItem>* items,
          std::vector<CausalItem>* combine, int32_t slots[3]) {
  std::vector<std::pair<double, CausalItem>> out;
  for (const Unit& u : units) {
    const int n = pieces_of(u, cap);
    CausalItem c = u.it;
    for (c.kvh = 0; c.kvh < heads; ++c.kvh) {
      if (n > 1) {
        c.lo = slots[c.kind];
        c.hi = n;
        combine->push_back(c);
      }
      for (int i = 0; i < n; ++i) {
        CausalItem x = c;
        const int a = u.steps * i / n, b = u.steps * (i + 1) / n;
        if (c.kind == kDkv) {
          x.lo = a;
          x.hi = b;
        } else {
          x.lo = 64 * a;
          x.hi = std::min(64 * b, u.it.hi);
        }
        if (n > 1) x.slot = ++slots[c.kind];
        out.emplace_back((b - a) * u.each->step, x);
      }
    }
  }
  std::stable_sort(out.begin(), out.end(), [](const auto& a, const auto& b) { return a.first > b.first; });
  for (auto& x : out) items->push_back(x.second);
}

}  // namespace

void build_causal_tables(CausalTables* t) {
  const int32_t G = t->heads / t->kv_heads;
  // Items of `tile` rows or keys each.
  auto units = [&](CausalKind kind, int32_t tile, const Cost& each) {
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
        out.push_back({it, steps, &each});
      }
      q0 += nq;
      k0 += nk;
    }
    return out;
  };
  const int32_t heads = t->kv_heads;
  auto few = [&](size_t n) { return n * heads <= kSplitItems; };
  int32_t slots[3] = {0, 0, 0};
  Cost large = kForwardCost;
  large.step = large_step(t->head_dim);
  std::vector<Unit> fwd = units(kForward, t->fwd_tile = fwd_large_tile(t->head_dim), large);
  double cap = 0;
  // larger items, or items of 256 or 128 rows, cut or not: whichever end first
  std::vector<Unit> less = units(kForward, kCausalTile, kForwardCost);
  if (few(less.size())) {
    double end = replay(fwd, heads, 0, std::numeric_limits<double>::infinity());
    for (int32_t tile : {kCausalTile, kSmallTile}) {
      if (tile == kSmallTile) {
        if (end > kSmallEnd) break;
        less = units(kForward, kSmallTile, kSmallForward);
      }
      if (choose_cap(less, heads, &cap, &end)) {
        fwd = std::move(less);
        t->fwd_tile = tile;
      }
    }
  }
  emit(fwd, heads, cap, &t->fwd, &t->fwd_combine, slots);
  if (t->backward) {
    std::vector<Unit> dkv = units(kDkv, kCausalTile, kDkvCost), dq = units(kDq, kCausalTile, kDqCost);
    if (few(dq.size() + dkv.size())) {  // both kinds together, each fills the other's gaps
      std::vector<Unit> best;
      double end = std::numeric_limits<double>::infinity();
      for (int i = 0; i < 3; ++i) {  // items of 256 or 128, cut or not: whichever end first
        if (i > 0 && end > kSmallEnd) break;
        if (i == 1) dkv = units(kDkv, kSmallTile, kSmallDkv);
        if (i == 2) dq = units(kDq, kSmallTile, kSmallDq);
        std::vector<Unit> both = dkv;
        both.insert(both.end(), dq.begin(), dq.end());
        if (choose_cap(both, heads, &cap, &end)) best = std::move(both);
      }
      emit(best, heads, cap, &t->grad, &t->grad_combine, slots);
    } else {  // many: one kind after the other, so that an XCD streams one kind of rows at a time
      emit(dkv, heads, 0, &t->grad, &t->grad_combine, slots);
      emit(dq, heads, 0, &t->grad, &t->grad_combine, slots);
    }
  }
  t->fwd_slots = slots[kForward];
  t->q_slots = slots[kDq];
  t->kv_slots = slots[kDkv];
}

}  // namespace sra

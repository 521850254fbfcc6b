// A model of the ring of tiles of the attention over 4-bit caches, on the host: the loading warps, the copies under
// way, the multiplying warps with the walk of k_ring4.cuh and the warp that joins, in random order, over barriers that
// count phases and answer a parity wait as the hardware does.  Now and then a copy is held back for as long as anything
// else can go on.  Checked: a step reads its own tile, whole, from begin to end; every warp ends.
//   walk    the kernel's walk: no wrong read, no stop;
//   short   the same walk without its wait for the slot's last tile: the model has to find wrong reads or a stop.
// Prints one line per class and exits non-zero on any mismatch.  Test code only.
#include <cstdio>
#include <random>
#include <vector>

#include "k_ring4.cuh"

using bkv::Ring4;
using bkv::RingWalk;

namespace {

struct Bar {
  int count, arrived = 0, bytes = 0, phase = 0;  // phase: number of the running one
  explicit Bar(int n) : count(n) {}
  void settle() {
    if (arrived == count && bytes == 0) {
      ++phase;
      arrived = 0;
    }
  }
  void arrive(int expect = 0) {
    ++arrived;
    bytes += expect;
    settle();
  }
  void land() {
    --bytes;
    settle();
  }
  bool passes(int parity) const { return (phase & 1) != parity; }
};

// What an agent waits for, one after another.
struct Wait {
  Bar* bar;
  int parity;
};

template <typename R>
struct Model {
  const std::vector<int>& steps;  // of each segment
  bool whole;                     // with the wait for the slot's last tile
  std::mt19937& rng;
  std::vector<Bar> full, empty, jfull, qfull;
  Bar jempty{1};
  std::vector<std::vector<int>> holds;  // [slot][loader]: the tile that landed there, -1 while one is under way
  struct Copy {
    int slot, loader, tile;
  };
  std::vector<Copy> copies;
  struct Loader {
    int seg = 0, tile = 0, all = 0;  // all: tiles of the segments before and of this one
    bool done = false;
  };
  std::vector<Loader> loaders{3};
  struct Warp {
    RingWalk<R> at;
    int state = 0, seg = 0, busy = 0;
    explicit Warp(int i) : at(i) {}
  };
  std::vector<Warp> warps;
  int join_seg = 0, join_state = 0;
  bool join_done = false;
  long long wrong = 0;

  Model(const std::vector<int>& s, bool w, std::mt19937& r) : steps(s), whole(w), rng(r) {
    for (int i = 0; i < R::kSlots; ++i) {
      full.emplace_back(3);
      empty.emplace_back(R::kPart);
      holds.push_back(std::vector<int>(3, -2));
    }
    jfull.emplace_back(R::kWarps);
    for (int i = 0; i < 2; ++i) qfull.emplace_back(1);
    for (int i = 0; i < R::kWarps; ++i) warps.emplace_back(i);
  }

  bool load(int i) {
    Loader& l = loaders[i];
    while (l.seg < static_cast<int>(steps.size()) && l.tile * R::kPart >= steps[l.seg]) {
      l.tile = 0;
      ++l.seg;
    }
    if (l.seg == static_cast<int>(steps.size())) {
      l.done = true;
      return true;
    }
    const int slot = l.all % R::kSlots, turn = l.all / R::kSlots;
    if (turn > 0 && !empty[slot].passes((turn - 1) & 1)) return false;
    full[slot].arrive(1);
    holds[slot][i] = -1;
    copies.push_back({slot, i, l.all});
    if (i == 0)
      for (int x = steps[l.seg] - l.tile * R::kPart; x < R::kPart; ++x) empty[slot].arrive();
    ++l.tile;
    ++l.all;
    return true;
  }

  void look(const Warp& w) {
    const int tile = w.at.tiles + w.at.step / R::kPart;
    for (int x : holds[w.at.slot])
      if (x != tile) {
        ++wrong;
        break;
      }
  }

  bool work(Warp& w) {
    switch (w.state) {
      case 0:  // a segment begins
        if (w.seg == static_cast<int>(steps.size())) {
          w.state = 9;
          return true;
        }
        if (!qfull[w.seg & 1].passes((w.seg >> 1) & 1)) return false;
        w.at.begin();
        w.state = 1;
        return true;
      case 1:  // a step's tile
        if (w.at.step >= steps[w.seg]) {
          w.state = 3;
          return true;
        }
        {
          const auto used = [&](int s, int parity) { return !whole || empty[s].passes(parity); };
          const auto landed = [&](int s, int parity) { return full[s].passes(parity); };
          bool ok = w.at.there(used, landed), waited = true;
          w.at.await([&](int s, int parity) { waited = waited && used(s, parity); },
                     [&](int s, int parity) { waited = waited && landed(s, parity); });
          if (ok != waited) ++wrong;
          if (!ok) return false;
        }
        look(w);
        w.busy = rng() % 4;
        w.state = 2;
        return true;
      case 2:
        if (w.busy-- > 0) return true;
        look(w);
        empty[w.at.slot].arrive();
        w.at.next();
        w.state = 1;
        return true;
      case 3:  // the segment's sums
        if (w.seg >= 1 && !jempty.passes((w.seg - 1) & 1)) return false;
        w.at.end(steps[w.seg]);
        jfull[0].arrive();
        ++w.seg;
        w.state = 0;
        return true;
      default: return false;
    }
  }

  bool join() {  // queries of segment join_seg, then the sums of the one before
    const int n = static_cast<int>(steps.size());
    if (join_state == 0) {
      if (join_seg < n) qfull[join_seg & 1].arrive();
      join_state = 1;
      return true;
    }
    if (join_seg > 0) {
      if (!jfull[0].passes((join_seg - 1) & 1)) return false;
      jempty.arrive();
    }
    if (join_seg == n) join_done = true;
    ++join_seg;
    join_state = 0;
    return true;
  }

  // False where everybody waits for ever.
  bool run() {
    int late = -1;  // a copy that lands only when nothing else moves
    const int agents = 3 + R::kWarps + 1 + 1;
    std::vector<int> order(agents);
    for (;;) {
      bool all = copies.empty() && join_done;
      for (auto& l : loaders) all = all && l.done;
      for (auto& w : warps) all = all && w.state == 9;
      if (all) return true;
      // agents in a random order until one moves
      for (int i = 0; i < agents; ++i) {
        const int j = rng() % (i + 1);
        order[i] = order[j];
        order[j] = i;
      }
      bool moved = false;
      for (int a : order) {
        if (a < 3) moved = !loaders[a].done && load(a);
        else if (a < 3 + R::kWarps) moved = work(warps[a - 3]);
        else if (a == 3 + R::kWarps) moved = !join_done && join();
        else {
          const int free = static_cast<int>(copies.size()) - (late >= 0);
          if (free > 0) {
            int c = rng() % free;
            if (late >= 0 && c >= late) ++c;
            if (late < 0 && rng() % 8 == 0) {
              late = c;
              moved = true;
            } else {
              land(c);
              if (late > c) --late;
              moved = true;
            }
          }
        }
        if (moved) break;
      }
      if (!moved) {
        if (late < 0) return false;
        land(late);
        late = -1;
      }
    }
  }
  void land(int c) {
    const Copy x = copies[c];
    copies.erase(copies.begin() + c);
    holds[x.slot][x.loader] = x.tile;
    full[x.slot].land();
  }
};

template <typename R>
bool check(const char* name) {
  std::mt19937 rng(11);
  long long wrong[2] = {}, stopped[2] = {};
  for (int run = 0; run < 300; ++run) {
    std::vector<int> steps(1 + rng() % 8);
    // long segments, segments of a few steps, empty ones
    const int most = run % 3 == 0 ? 200 : run % 3 == 1 ? 30 : 3;
    for (int& s : steps) s = rng() % (most + 1);
    if (run % 5 == 0) steps.resize(steps.size() + 20, 1);
    for (int w = 0; w < 2; ++w) {
      Model<R> m(steps, w == 0, rng);
      if (!m.run()) ++stopped[w];
      wrong[w] += m.wrong;
    }
  }
  std::printf("%s walk: %lld wrong reads, %lld stops; short: %lld, %lld\n", name, wrong[0], stopped[0], wrong[1],
              stopped[1]);
  return wrong[0] == 0 && stopped[0] == 0 && wrong[1] + stopped[1] > 0;
}

}  // namespace

int main() {
  using namespace bkv;
  bool ok = check<Ring4<128, 1>>("128, one block:");
  ok = check<Ring4<128, 2>>("128, two blocks:") && ok;
  ok = check<Ring4<64, 1>>("64, one block:") && ok;
  ok = check<Ring4<64, 2>>("64, two blocks:") && ok;
  return ok ? 0 : 1;
}

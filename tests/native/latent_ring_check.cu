// Model of one stage of the latent kernel's ring, on the CPU: two load warps that fill it for one tile
// after the other, the products that give it back group by group, and barriers that tell their phases
// apart by parity only, as mbarriers do. The lists of waits are the kernel's own (topkv_latent.cuh).
// Every order in which the three can take their steps is followed, for every mixture of tiles loaded
// by tensor copies and by rows; a wait that lets a warp pass before the release it stands for is a fault.
// Built with nvcc and run by tests/test_latent_ring_host.py; needs no GPU.
#include <cstdio>
#include <set>
#include <tuple>
#include <vector>

#include "topkv_latent.cuh"

constexpr int kTiles = 6;

// waits(by_rows, i, half, groups): group of a warp's i-th wait for a tile, -1 behind the last.
template <typename Waits>
static int faults(const Waits& waits) {
  int found = 0;
  for (int groups = 1; groups <= 4; ++groups)
    for (int paths = 0; paths < 1 << kTiles; ++paths) {  // bit j: tile j comes by rows
      using State = std::tuple<int, int, int, int, int>;  // tile and next wait of each warp, groups released in all
      std::set<State> known;
      std::vector<State> open;
      auto reach = [&](const State& s) {
        if (known.insert(s).second) open.push_back(s);
      };
      reach({0, 0, 0, 0, 0});
      bool early = false;
      while (!open.empty()) {
        int tile[2], next[2], released;
        std::tie(tile[0], next[0], tile[1], next[1], released) = open.back();
        open.pop_back();
        for (int h = 0; h < 2; ++h) {
          if (tile[h] == kTiles) continue;
          int t[2] = {tile[0], tile[1]}, n[2] = {next[0], next[1]};
          const int v = tile[h] == 0 ? -1 : waits(paths >> tile[h] & 1, next[h], h, groups);
          if (v < 0) {  // all waits passed: the warp loads and goes on to the next tile
            ++t[h];
            n[h] = 0;
          } else {
            const int phase = tile[h] - 1;                                           // waits for the release of the tile before
            const int complete = released / groups + (released % groups > v ? 1 : 0);  // phases of this barrier so far
            if ((complete & 1) == (phase & 1)) continue;                             // the parity says: not yet
            if (complete < tile[h]) early = true;
            ++n[h];
          }
          reach({t[0], n[0], t[1], n[1], released});
        }
        // products of a tile need all of it loaded, and end group by group
        if (released / groups < std::min(tile[0], tile[1])) reach({tile[0], next[0], tile[1], next[1], released + 1});
      }
      if (early) ++found;
      if (!known.count({kTiles, 0, kTiles, 0, kTiles * groups})) return -1;  // nothing may hang
    }
  return found;
}

int main() {
  const int kernel = faults([](bool by_rows, int i, int half, int groups) {
    return by_rows ? topkv::rows_await(i, groups) : topkv::pieces_await(i, half, groups);
  });
  // the model itself: waiting for the last group alone is not enough once a tile came by tensor copies
  const int last_only = faults([](bool by_rows, int i, int half, int groups) {
    return by_rows ? (i == 0 ? groups - 1 : -1) : topkv::pieces_await(i, half, groups);
  });
  std::printf("kernel %d, last group only %d\n", kernel, last_only);
  return kernel == 0 && last_only > 0 ? 0 : 1;
}

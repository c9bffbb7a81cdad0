// A model of the recurrence's scan over tiles (csrc/glr.h) under limited residency: R of G
// workgroups run at once, the others start as those end, in any order.  A workgroup
// takes turns b, b + G, ..; turn i takes the next tile of column i % columns, publishes
// the tile's map, waits until the nearest eight tiles before it show, in every column that
// its 64 lanes look at, a state and all maps after it, and publishes its state.  Which
// columns those are is the kernels' own glr_channel.  Prints the first setting in which
// every running workgroup waits for a tile that none of them holds.
#include <stdio.h>

#include <random>
#include <set>
#include <vector>

#include "layer.h"

enum Word { kNone, kMap, kState };

static bool finishes(int groups, int resident, int D, int tiles, unsigned seed) {
  const int cols = (D + 63) / 64, turns = tiles * cols;
  std::mt19937 rng(seed);
  std::vector<int> next(cols, 0);
  std::vector<std::vector<Word>> words(cols, std::vector<Word>(tiles, kNone));
  std::vector<std::set<int>> sees(cols);
  for (int c = 0; c < cols; ++c)
    for (int lane = 0; lane < 64; ++lane) sees[c].insert((int)hagdn::glr_channel((uint32_t)(c * 64 + lane), (uint32_t)D) / 64);
  struct Group {
    long turn;
    int col, tile;  // tile -1: about to take one
  };
  std::vector<Group> running;
  int started = 0;
  for (; started < groups && started < resident; ++started) running.push_back({started, 0, -1});
  auto ready = [&](const Group &g) {
    if (g.tile == 0) return true;
    for (int j = g.tile - 1; j >= 0 && j >= g.tile - 8; --j) {
      bool all_states = true;
      for (int c : sees[g.col]) {
        if (words[c][j] == kNone) return false;
        all_states &= words[c][j] == kState;
      }
      if (all_states) return true;
    }
    return false;
  };
  while (!running.empty()) {
    std::vector<size_t> able;
    for (size_t i = 0; i < running.size(); ++i)
      if (running[i].tile < 0 || ready(running[i])) able.push_back(i);
    if (able.empty()) return false;
    const size_t i = able[rng() % able.size()];
    Group &g = running[i];
    if (g.tile < 0 && g.turn < turns) {
      g.col = (int)(g.turn % cols);
      g.tile = next[g.col]++;
      if (g.tile >= tiles) return false;
      words[g.col][g.tile] = kMap;
    } else if (g.tile >= 0) {
      words[g.col][g.tile] = kState;
      g.tile = -1;
      g.turn += groups;
    } else if (started < groups) {
      g = {started++, 0, -1};
    } else {
      running.erase(running.begin() + (long)i);
    }
  }
  for (int c = 0; c < cols; ++c)
    if (next[c] != tiles) return false;
  return true;
}

int main() {
  for (int D : {1, 33, 64, 65, 128, 130, 447, 448, 705, 4630})
    for (int groups : {1, 3, 32, 512})
      for (int resident : {1, 2, 7, 40, 512})
        for (int tiles : {2, 9, 235}) {
          const int cols = (D + 63) / 64, grid = groups < tiles * cols ? groups : tiles * cols;
          for (unsigned seed = 0; seed < 3; ++seed)
            if (!finishes(grid, resident, D, tiles, seed)) {
              printf("no progress: %d channels, %d tiles, %d workgroups, %d at once, order %u\n", D, tiles, grid, resident, seed);
              return 1;
            }
        }
  puts("every wait ends");
  return 0;
}

// Forks and compactions through their C entry points, with the kernels of k12_pool.hip run on
// the CPU (on_host.h): every buffer is an allocation of its own and of no byte
// more than the header asks for, so that AddressSanitizer sees an access beyond it.  Results
// against the rules carried out one row at a time.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <random>

#include "hagdn.h"

#include "api_mixer.cpp"
#include "k12_pool.hip"

namespace hagdn {
int set_error(int code, const char *msg) {
  fprintf(stderr, "error %d: %s\n", code, msg);
  return code;
}
int device_cus() { return 256; }
hipError_t launch_conv_forward(const ConvArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_conv_backward(const ConvArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_conv_step(const ConvStepArgs &, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_ssm_forward(const SsmArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_ssm_backward(const SsmArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_ssm_step(const SsmStepArgs &, bool, bool, hipStream_t) { return hipErrorNoDevice; }
}  // namespace hagdn

#define CHECK(cond)                                                   \
  do {                                                                \
    if (!(cond)) {                                                    \
      fprintf(stderr, "line %d: %s\n", __LINE__, #cond);              \
      exit(1);                                                        \
    }                                                                 \
  } while (0)

typedef std::vector<int32_t> Ints;

// Pools of rows that say which slot they were in.
struct Pools {
  size_t row_bytes[2] = {8, 20};
  std::vector<Ints> rows;
  explicit Pools(int S) : rows(2) {
    for (int p = 0; p < 2; ++p)
      for (int s = 0; s < S; ++s) rows[p].insert(rows[p].end(), row_bytes[p] / 4, 1000 * s + p);
    for (Ints &r : rows) r.shrink_to_fit();
  }
  void copy(int dst, int src) {
    for (int p = 0; p < 2; ++p) {
      const size_t n = row_bytes[p] / 4;
      std::copy_n(rows[p].begin() + (long)(src * n), n, rows[p].begin() + (long)(dst * n));
    }
  }
};

static void fork(int N, int M, int S, int kind, std::mt19937 &rng) {
  Ints slots(N), parents(M), all(std::max(N, S));
  for (size_t i = 0; i < all.size(); ++i) all[i] = (int)i;
  std::shuffle(all.begin(), all.end(), rng);  // some beyond the pools where N > S
  std::copy_n(all.begin(), N, slots.begin());
  for (int &p : parents) p = kind == 0 ? 0 : (int)(rng() % N);
  if (kind == 2) {
    for (int &p : parents)
      if (rng() % 5 == 0) p = rng() % 2 ? -1 : N;
    for (int &s : slots)
      if (rng() % 5 == 0) s = -1;
  }
  Pools got(S), want(S);
  const auto at = [&](int p) { return p >= 0 && p < N && slots[p] >= 0 && slots[p] < S ? slots[p] : -1; };
  std::vector<bool> kept(S), seen(S);
  for (int p : parents)
    if (at(p) >= 0) kept[at(p)] = true;
  Ints new_slots;
  int next = 0;
  bool full = false;
  for (int p : parents) {
    const int s = at(p);
    int to = s;
    if (s >= 0 && seen[s]) {
      while (next < S && kept[next]) ++next;
      to = next < S ? next++ : -1;
      full |= to < 0;
      if (to >= 0) want.copy(to, s);
    } else if (s >= 0) {
      seen[s] = true;
    }
    new_slots.push_back(to);
  }
  Ints out(M);
  const size_t bytes = hagdn_pool_workspace_size(S);
  void *ws = malloc(bytes), *pools[2] = {got.rows[0].data(), got.rows[1].data()};
  memset(ws, 0x5a, bytes);
  printf("fork of %d sequences into %d children, %d slots, form %d\n", N, M, S, kind);
  fflush(stdout);
  CHECK(hagdn_pool_fork(pools, got.row_bytes, 2, slots.data(), N, parents.data(), M, S, out.data(), ws, bytes, nullptr) == HAGDN_OK);
  CHECK(*static_cast<int *>(ws) == (full ? HAGDN_DEV_POOL_FULL : HAGDN_DEV_OK));
  CHECK(out == new_slots);
  CHECK(got.rows == want.rows);
  free(ws);
}

static void compact(int N, int S, std::mt19937 &rng) {
  Ints table(N), all(S);
  for (int s = 0; s < S; ++s) all[s] = s;
  std::shuffle(all.begin(), all.end(), rng);
  std::copy_n(all.begin(), N, table.begin());
  for (int &s : table)
    if (rng() % 3 == 0) s = rng() % 2 ? -1 : S;
  if (N > 4) table[3] = table[1];
  Pools got(S), want(S);
  Ints live, moved(S, -1), after;
  for (int s : table)
    if (s >= 0 && s < S && moved[s] < 0) live.push_back(s), moved[s] = s;
  std::sort(live.begin(), live.end());
  int hole = 0;
  for (int s : live)
    if (s >= (int)live.size()) {
      while (std::binary_search(live.begin(), live.end(), hole)) ++hole;
      want.copy(hole, s);
      moved[s] = hole++;
    }
  for (int s : table) after.push_back(s >= 0 && s < S ? moved[s] : s);
  Ints out(N);
  const size_t bytes = hagdn_pool_workspace_size(S);
  void *ws = malloc(bytes), *pools[2] = {got.rows[0].data(), got.rows[1].data()};
  printf("compaction of %d of %d slots\n", (int)live.size(), S);
  fflush(stdout);
  CHECK(hagdn_pool_compact(pools, got.row_bytes, 2, table.data(), N, S, out.data(), ws, bytes, nullptr) == HAGDN_OK);
  CHECK(out == after);
  CHECK(got.rows == want.rows);
  free(ws);
}

int main() {
  std::mt19937 rng(1);
  // plans in LDS, up to 4096 slots and children, and in memory, with and without enough free
  // slots; the children of one sequence, of all, and some of none
  const int cases[][3] = {{1, 5, 3}, {8, 8, 20}, {40, 4096, 4096}, {3, 4097, 4096}, {3000, 4096, 4097}, {3000, 4500, 6000},
                          {1, 5000, 100}, {100, 5000, 100}, {200, 4097, 1}, {2000, 9000, 5000}};
  for (const auto &c : cases)
    for (int kind = 0; kind < 3; ++kind) fork(c[0], c[1], c[2], kind, rng);
  for (const auto &c : {std::pair<int, int>{3, 9}, {700, 4096}, {4097, 4097}, {2500, 5000}}) compact(c.first, c.second, rng);
  puts("pool plans passed");
  return 0;
}

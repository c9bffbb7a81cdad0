// Kernels without matrix instructions on the CPU: stands in for hip/hip_runtime.h, device.h and
// prefill.h where a kernel's source is compiled for the host (test_pool_plans.py).  A thread is a
// context of its own that runs up to the next barrier or ballot, workgroups run one after another;
// LDS is static memory, so that the sanitizers see every access.
#pragma once

#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <algorithm>
#include <functional>
#include <vector>

#define __global__
#define __host__
#define __device__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static

typedef int hipError_t;
typedef struct ihipStream_t *hipStream_t;
constexpr hipError_t hipSuccess = 0, hipErrorNoDevice = 100;
inline hipError_t hipGetLastError() { return hipSuccess; }
inline const char *hipGetErrorString(hipError_t) { return "no device"; }

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {}
};
inline dim3 threadIdx, blockIdx, blockDim, gridDim;
using std::max;
using std::min;

namespace on_host {
enum State { kReady, kAtGroup, kAtWave, kDone };
struct Fiber {
  ucontext_t context;
  State state;
  std::vector<char> stack = std::vector<char>(1 << 16);
};
inline std::vector<Fiber> fibers;
inline ucontext_t scheduler;
inline unsigned current;
inline bool votes[1024];
inline std::function<void()> body;

inline void wait(State at) {
  Fiber &f = fibers[current];
  f.state = at;
  swapcontext(&f.context, &scheduler);
}
inline void enter() {
  body();
  wait(kDone);
}
// Runs the threads of a wave that can go on, until each waits or has ended; whether all did so in
// one place.
inline bool run_wave(unsigned first, State &place) {
  for (;;) {
    for (unsigned t = first; t < first + 64; ++t) {
      if (fibers[t].state != kReady) continue;
      current = t;
      threadIdx = dim3(t);
      swapcontext(&scheduler, &fibers[t].context);
    }
    place = fibers[first].state;
    for (unsigned t = first; t < first + 64; ++t)
      if (fibers[t].state != place) return false;
    if (place != kAtWave) return true;
    for (unsigned t = first; t < first + 64; ++t) fibers[t].state = kReady;
  }
}
template <typename F> void launch(dim3 grid, dim3 block, F f) {
  gridDim = grid;
  blockDim = block;
  body = f;
  fibers.resize(1024);
  for (unsigned b = 0; b < grid.x; ++b) {
    blockIdx = dim3(b);
    for (unsigned t = 0; t < block.x; ++t) {
      Fiber &n = fibers[t];
      n.state = kReady;
      getcontext(&n.context);
      n.context.uc_stack.ss_sp = n.stack.data();
      n.context.uc_stack.ss_size = n.stack.size();
      n.context.uc_link = nullptr;
      makecontext(&n.context, enter, 0);
    }
    for (State all = kReady; all != kDone;) {
      for (unsigned t = 0; t < block.x; t += 64) {
        State place;
        if (!run_wave(t, place) || (t > 0 && place != all)) {
          fprintf(stderr, "threads of workgroup %u wait in different places\n", b);
          exit(1);
        }
        all = place;
      }
      for (unsigned t = 0; t < block.x && all == kAtGroup; ++t) fibers[t].state = kReady;
    }
  }
}
}  // namespace on_host
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) on_host::launch(grid, block, [&] { kernel(__VA_ARGS__); })

inline void __syncthreads() { on_host::wait(on_host::kAtGroup); }
inline void __threadfence() {}
inline uint64_t __ballot(bool v) {
  const unsigned first = threadIdx.x / 64 * 64;
  on_host::votes[threadIdx.x] = v;
  on_host::wait(on_host::kAtWave);
  uint64_t bits = 0;
  for (unsigned i = 0; i < 64; ++i) bits |= (uint64_t)on_host::votes[first + i] << i;
  on_host::wait(on_host::kAtWave);
  return bits;
}
inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
inline int atomicMin(int *p, int v) {
  const int old = *p;
  *p = min(old, v);
  return old;
}

namespace hagdn {
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
inline int lane_id() { return (int)(threadIdx.x & 63); }
constexpr int kPreGateSoftplus = 2;
}  // namespace hagdn

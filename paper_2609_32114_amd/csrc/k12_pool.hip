// k12_pool.hip -- copies between rows of state pools, and the plans that say which rows a
// fork or a compaction moves.  Copies are bound by HBM: every moved byte is read once and
// written once, all pools of a call in one launch.  A beam search's step over 24 pools (303 MB)
// 59 us, 131 states of 1 MiB in four layers to the front (some 800 MB) 148, 5.1 to 5.4 TB/s.
#include "device.h"
#include "mixer.h"
#include "prefill.h"

namespace hagdn {

// Calls f with a value of a pool's access type.
template <typename F> __device__ __forceinline__ void with_unit(int unit, F f) {
  switch (unit) {
    case 16: f(u32x4{}); break;
    case 8: f(uint64_t{}); break;
    case 4: f(uint32_t{}); break;
    case 2: f(uint16_t{}); break;
    default: f(uint8_t{}); break;
  }
}

constexpr int kPieces = 8;  // units a thread moves at once, at most

// Row of entry i, or -1: none (a null table: row i).
__device__ __forceinline__ int row_of(const int32_t *table, int rows, int i) {
  const int r = table ? table[i] : i;
  return r >= 0 && r < rows ? r : -1;
}

// The pool that piece `at` of an entry lies in, and the piece's place there; `each` units to a piece.
__device__ __forceinline__ int find_pool(const PoolCopyArgs &a, uint32_t each, uint64_t &at) {
  for (int p = 0;; ++p) {
    const uint64_t here = (a.pools[p].units + each - 1) / each;
    if (at < here || p + 1 == a.count) return p;
    at -= here;
  }
}

// Rows that no other entry of the call writes or reads: a workgroup moves `span` units of one
// row after another.  A source outside its rows gives zeros.
__global__ __launch_bounds__(256) void pool_move_kernel(PoolCopyArgs a, uint32_t span, uint64_t pieces) {
  const int n = a.moves ? a.moves[0] : a.n;
  for (uint64_t item = blockIdx.x; item < pieces * n; item += gridDim.x) {
    const int i = (int)(item / pieces);
    uint64_t at = item - (uint64_t)i * pieces;
    const Pool &pool = a.pools[find_pool(a, span, at)];
    const int dst = a.moves ? a.moves[1 + 2 * i] : row_of(a.dst, a.dst_rows, i);
    const int src = a.moves ? a.moves[2 + 2 * i] : row_of(a.src, a.src_rows, i);
    if (dst < 0) continue;
    const uint64_t units = pool.units, first = at * span + threadIdx.x, end = min(units, (at + 1) * span);
    with_unit(pool.unit, [&](auto u) {
      using U = decltype(u);
      const U *from = static_cast<const U *>(pool.from) + (src < 0 ? 0 : (uint64_t)src * units);
      U *to = static_cast<U *>(pool.to) + (uint64_t)dst * units;
      U v[kPieces] = {};
      if (src >= 0) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
          if (first + k * 256 < end) v[k] = __builtin_nontemporal_load(from + first + k * 256);
      }
#pragma unroll
      for (int k = 0; k < kPieces; ++k)
        if (first + k * 256 < end) __builtin_nontemporal_store(v[k], to + first + k * 256);
    });
  }
}

// Rows of the same pools, as if all were read before any is written: a workgroup has a span
// of units of every entry's row, all of them in registers between its loads and its stores.
// 88 rows of 20 pools (242 MB) 61 us.
template <int THREADS> __global__ __launch_bounds__(THREADS) void pool_shuffle_kernel(PoolCopyArgs a, uint32_t width, uint64_t spans) {
  for (uint64_t item = blockIdx.x; item < spans; item += gridDim.x) {
    uint64_t at = item;
    const Pool &pool = a.pools[find_pool(a, width, at)];
    const uint64_t units = pool.units, first = at * width;
    with_unit(pool.unit, [&](auto u) {
      using U = decltype(u);
      U *rows = static_cast<U *>(pool.to), v[kPieces] = {};
      // unit k of this thread: its entry, and where in the row it lies
      const auto entry = [&](int k, uint64_t &col) {
        const uint32_t e = k * THREADS + threadIdx.x, i = e / width;  // n x width <= THREADS x kPieces
        col = first + (e - i * width);
        return i < (uint32_t)a.n && col < units ? (int)i : -1;
      };
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        uint64_t col;
        const int i = entry(k, col);
        if (i < 0 || row_of(a.dst, a.dst_rows, i) < 0) continue;
        const int src = row_of(a.src, a.src_rows, i);
        if (src >= 0) v[k] = rows[(uint64_t)src * units + col];
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        uint64_t col;
        const int i = entry(k, col);
        const int dst = i < 0 ? -1 : row_of(a.dst, a.dst_rows, i);
        if (dst >= 0) rows[(uint64_t)dst * units + col] = v[k];
      }
      __syncthreads();
    });
  }
}

// Exclusive prefix sums of one flag a thread over a workgroup of 1024, and their total.
__device__ __forceinline__ int prefix(bool flag, int (&waves)[16], int &total) {
  const uint64_t bits = __ballot(flag);
  const int wave = threadIdx.x >> 6;
  __syncthreads();  // the last call's sums have been read
  if (lane_id() == 0) waves[wave] = __popcll(bits);
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    before += w < wave ? waves[w] : 0;
    total += waves[w];
  }
  return before + __popcll(bits & ((1ull << lane_id()) - 1));
}

// The workgroup's stores and atomics in memory are done and seen by all of it.
__device__ __forceinline__ void settle() {
  __threadfence();
  __syncthreads();
}

// The slot that child i's parent is in, or -1.
__device__ __forceinline__ int parent_slot(const PoolPlanArgs &a, int i) {
  const int p = a.parents[i];
  return p >= 0 && p < a.N ? row_of(a.slots, a.num_slots, p) : -1;
}

// Plans of up to kSmallPlan slots and children are made in LDS: 256 children over 320 slots 4.6
// us instead of 14, 512 slots compacted 4.7 instead of 19.
constexpr int kSmallPlan = 4096;
constexpr int kNobody = 0x7fffffff;

// mark[slot]: the first child that goes on from the parent there, or none.  That child
// stays; the k-th of the others gets the k-th slot without a mark.
__global__ __launch_bounds__(1024) void pool_small_fork_kernel(PoolPlanArgs a) {
  __shared__ int sWaves[16], sMark[kSmallPlan], sSource[kSmallPlan], sFree[kSmallPlan];
  const int t = threadIdx.x;
  for (int i = t; i < a.num_slots; i += 1024) sMark[i] = kNobody;
  for (int i = t; i < a.M; i += 1024) sSource[i] = parent_slot(a, i);
  __syncthreads();
  for (int i = t; i < a.M; i += 1024)
    if (sSource[i] >= 0) atomicMin(&sMark[sSource[i]], i);
  __syncthreads();
  int free_slots = 0, moves = 0, total;
  for (int base = 0; base < a.num_slots; base += 1024) {
    const int i = base + t;
    const bool free_slot = i < a.num_slots && sMark[i] == kNobody;
    const int k = free_slots + prefix(free_slot, sWaves, total);
    if (free_slot) sFree[k] = i;
    free_slots += total;
  }
  __syncthreads();
  for (int base = 0; base < a.M; base += 1024) {
    const int i = base + t, s = i < a.M ? sSource[i] : -1;
    const bool moved = s >= 0 && sMark[s] != i;
    const int k = moves + prefix(moved, sWaves, total);
    const int to = !moved ? s : k < free_slots ? sFree[k] : -1;
    if (i < a.M) a.out[i] = to;
    if (moved && to >= 0) {
      a.moves[1 + 2 * k] = to;
      a.moves[2 + 2 * k] = s;
    }
    moves += total;
  }
  if (t == 0) {
    a.moves[0] = min(moves, free_slots);
    *a.status = moves > free_slots ? kDevPoolFull : 0;
  }
}

// mark[slot]: the slot that its state is in afterwards.
__global__ __launch_bounds__(1024) void pool_small_compact_kernel(PoolPlanArgs a) {
  __shared__ int sWaves[16], sMark[kSmallPlan], sFree[kSmallPlan];
  const int t = threadIdx.x;
  for (int i = t; i < a.num_slots; i += 1024) sMark[i] = -1;
  __syncthreads();
  for (int i = t; i < a.N; i += 1024) {
    const int s = row_of(a.slots, a.num_slots, i);
    if (s >= 0) sMark[s] = s;
  }
  __syncthreads();
  int live = 0, holes = 0, moves = 0, total;
  for (int base = 0; base < a.num_slots; base += 1024) {
    prefix(base + t < a.num_slots && sMark[base + t] >= 0, sWaves, total);
    live += total;
  }
  for (int base = 0; base < live; base += 1024) {  // free slots among the first `live`
    const int i = base + t;
    const bool hole = i < live && sMark[i] < 0;
    const int k = holes + prefix(hole, sWaves, total);
    if (hole) sFree[k] = i;
    holes += total;
  }
  __syncthreads();
  for (int base = live; base < a.num_slots; base += 1024) {  // as many states lie beyond them
    const int i = base + t;
    const bool moved = i < a.num_slots && sMark[i] >= 0;
    const int k = moves + prefix(moved, sWaves, total);
    if (moved) {
      sMark[i] = sFree[k];
      a.moves[1 + 2 * k] = sFree[k];
      a.moves[2 + 2 * k] = i;
    }
    moves += total;
  }
  __syncthreads();
  for (int i = t; i < a.N; i += 1024) {
    const int s = row_of(a.slots, a.num_slots, i);
    a.out[i] = s >= 0 ? sMark[s] : a.slots[i];
  }
  if (t == 0) {
    a.moves[0] = moves;
    *a.status = 0;
  }
}

// The same plans of any size, with their tables in memory.
__global__ __launch_bounds__(1024) void pool_fork_plan_kernel(PoolPlanArgs a) {
  __shared__ int sWaves[16];
  const int t = threadIdx.x;
  const auto source = [&](int i) { return parent_slot(a, i); };
  for (int i = t; i < a.num_slots; i += 1024) a.mark[i] = kNobody;
  settle();
  for (int i = t; i < a.M; i += 1024) {
    const int s = source(i);
    if (s >= 0) atomicMin(a.mark + s, i);
  }
  settle();
  int moves = 0, total;
  for (int base = 0; base < a.M; base += 1024) {  // the sources, in the children's order
    const int i = base + t, s = i < a.M ? source(i) : -1;
    const bool moved = s >= 0 && a.mark[s] != i;
    const int k = moves + prefix(moved, sWaves, total);
    if (moved && k < a.num_slots) a.moves[2 + 2 * k] = s;  // more than the slots are counted, not carried out
    moves += total;
  }
  int free_slots = 0;
  for (int base = 0; base < a.num_slots && free_slots < moves; base += 1024) {  // the free slots, in their order
    const int i = base + t;
    const bool free_slot = i < a.num_slots && a.mark[i] == kNobody;
    const int k = free_slots + prefix(free_slot, sWaves, total);
    if (free_slot && k < moves) a.moves[1 + 2 * k] = i;
    free_slots += total;
  }
  settle();
  const int done = min(moves, free_slots);
  int seen = 0;
  for (int base = 0; base < a.M; base += 1024) {  // the children's slots
    const int i = base + t, s = i < a.M ? source(i) : -1;
    const bool moved = s >= 0 && a.mark[s] != i;
    const int k = seen + prefix(moved, sWaves, total);
    if (i < a.M) a.out[i] = !moved ? s : k < done ? a.moves[1 + 2 * k] : -1;
    seen += total;
  }
  if (t == 0) {
    a.moves[0] = done;
    *a.status = moves > done ? kDevPoolFull : 0;
  }
}

__global__ __launch_bounds__(1024) void pool_compact_plan_kernel(PoolPlanArgs a) {
  __shared__ int sWaves[16];
  const int t = threadIdx.x;
  for (int i = t; i < a.num_slots; i += 1024) a.mark[i] = -1;
  settle();
  for (int i = t; i < a.N; i += 1024) {
    const int s = row_of(a.slots, a.num_slots, i);
    if (s >= 0) a.mark[s] = s;
  }
  settle();
  int live = 0, total;
  for (int base = 0; base < a.num_slots; base += 1024) {
    prefix(base + t < a.num_slots && a.mark[base + t] >= 0, sWaves, total);
    live += total;
  }
  int holes = 0, moves = 0;
  for (int base = 0; base < live; base += 1024) {  // free slots among the first `live`
    const int i = base + t;
    const bool hole = i < live && a.mark[i] < 0;
    const int k = holes + prefix(hole, sWaves, total);
    if (hole) a.moves[1 + 2 * k] = i;
    holes += total;
  }
  settle();
  for (int base = live; base < a.num_slots; base += 1024) {  // as many states lie beyond them
    const int i = base + t;
    const bool moved = i < a.num_slots && a.mark[i] >= 0;
    const int k = moves + prefix(moved, sWaves, total);
    if (moved) {
      a.moves[2 + 2 * k] = i;
      a.mark[i] = a.moves[1 + 2 * k];
    }
    moves += total;
  }
  settle();
  for (int i = t; i < a.N; i += 1024) {
    const int s = row_of(a.slots, a.num_slots, i);
    a.out[i] = s >= 0 ? a.mark[s] : a.slots[i];
  }
  if (t == 0) {
    a.moves[0] = moves;
    *a.status = 0;
  }
}

hipError_t launch_pool_fork_plan(const PoolPlanArgs &a, hipStream_t s) {
  if (a.num_slots <= kSmallPlan && a.M <= kSmallPlan) hipLaunchKernelGGL(pool_small_fork_kernel, dim3(1), dim3(1024), 0, s, a);
  else hipLaunchKernelGGL(pool_fork_plan_kernel, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}
hipError_t launch_pool_compact_plan(const PoolPlanArgs &a, hipStream_t s) {
  if (a.num_slots <= kSmallPlan) hipLaunchKernelGGL(pool_small_compact_kernel, dim3(1), dim3(1024), 0, s, a);
  else hipLaunchKernelGGL(pool_compact_plan_kernel, dim3(1), dim3(1024), 0, s, a);
  return hipGetLastError();
}

// Long rows go 32 KiB (of 16-byte units) at a time; calls that move little in as many pieces as
// give every CU four workgroups, of one unit a thread at least.  (One row of 144 KiB in pieces
// of 32 KiB 6.6 us, 4.2 in pieces of 4 KiB.)
hipError_t launch_pool_copy(const PoolCopyArgs &a, bool in_place, int cus, hipStream_t s) {
  const uint64_t most = 16ull * (cus > 0 ? cus : 256);  // workgroups
  uint64_t units = 0;                                   // of one entry
  for (int p = 0; p < a.count; ++p) units += a.pools[p].units;
  const auto pieces = [&](uint64_t span) {
    uint64_t n = 0;
    for (int p = 0; p < a.count; ++p) n += (a.pools[p].units + span - 1) / span;
    return n;
  };
  const uint64_t share = (units * (in_place ? 1 : (uint64_t)a.n) + most / 4 - 1) / (most / 4);
  if (!in_place) {
    const uint32_t span = (uint32_t)(share < 256 ? 256 : share > 256 * kPieces ? 256 * kPieces : (share + 255) / 256 * 256);
    const uint64_t each = pieces(span), items = each * (uint64_t)a.n;
    hipLaunchKernelGGL(pool_move_kernel, dim3((unsigned)(items < most ? items : most)), dim3(256), 0, s, a, span, each);
    return hipGetLastError();
  }
  const bool many = a.n > 256 * kPieces;
  const uint32_t widest = (many ? 1024u : 256u) * kPieces / (uint32_t)a.n;  // n <= kMaxMovesInPlace
  const uint32_t least = (256 + (uint32_t)a.n - 1) / (uint32_t)a.n;         // a unit a thread
  const uint32_t width = (uint32_t)(share < least ? (least < widest ? least : widest) : share < widest ? share : widest);
  const uint64_t spans = pieces(width);
  const dim3 grid((unsigned)(spans < most ? spans : most));
  if (many) hipLaunchKernelGGL((pool_shuffle_kernel<1024>), grid, dim3(1024), 0, s, a, width, spans);
  else hipLaunchKernelGGL((pool_shuffle_kernel<256>), grid, dim3(256), 0, s, a, width, spans);
  return hipGetLastError();
}

}  // namespace hagdn

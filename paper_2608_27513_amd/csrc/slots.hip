// Slots of a state pool as the pages of its cache (damp_serving.h): counts of
// their holders, copies, and compaction.
//
// The copies move whole slots, num_v_heads * tile_stride contiguous bytes (a
// multiple of 128) in each layer, and are bound by memory: a source is read
// once and written once for each of its copies, 16 bytes a lane, past the
// caches on both sides (what is copied is used much later, if at all): 8 slots
// of 14.8 MB into 4 each take 98 us, 5.9 TB/s (117 us through the caches and
// four words a lane, 111 with the words, 106 with two).
//
// The counts are kept by one workgroup each: pools have tens to thousands of
// slots, and the launch is what such a call costs.
#include "internal.hpp"

namespace damp {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = kThreads * 16;  // bytes of a workgroup's piece of a slot
constexpr int kPlanThreads = 1024;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct PoolView {
  uint8_t* base;
  uint64_t slot_bytes;   // bytes of one slot in one layer
  uint64_t layer_bytes;
  int32_t num_slots;
};

PoolView view_of(const damp_pool* pool, int32_t layer) {
  PoolView v;
  v.slot_bytes = pool->tile_stride * static_cast<uint64_t>(pool->num_v_heads);
  v.layer_bytes = v.slot_bytes * static_cast<uint64_t>(pool->num_slots);
  v.base = layer_base(pool, layer < 0 ? 0 : layer);
  v.num_slots = pool->num_slots;
  return v;
}

// One piece of a slot in one layer into `fan` others.
__device__ __forceinline__ void copy_piece(const PoolView& v, uint64_t layer, int from,
                                           const int32_t* to, int fan, uint64_t piece) {
  uint8_t* base = v.base + layer * v.layer_bytes;
  const uint64_t at = piece * kChunk + threadIdx.x * 16;
  if (at >= v.slot_bytes) return;
  const u32x4 w = __builtin_nontemporal_load(
      reinterpret_cast<const u32x4*>(base + from * v.slot_bytes + at));
  for (int j = 0; j < fan; ++j) {
    const int d = to[j];
    if (d < 0 || d >= v.num_slots) continue;
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(base + d * v.slot_bytes + at));
  }
}

__global__ __launch_bounds__(kThreads) void fork_kernel(const PoolView v, const int32_t* src,
                                                        const int32_t* dst, int fan, int pieces) {
  const int i = blockIdx.x / pieces;
  const int from = src[i];
  if (from < 0 || from >= v.num_slots) return;
  copy_piece(v, blockIdx.y, from, dst + static_cast<size_t>(i) * fan, fan, blockIdx.x % pieces);
}

// How many threads before this one are told `yes`, and how many in all; for
// two questions at once. Threads of a workgroup of kPlanThreads.
struct Counts {
  int a, b;
};
__device__ __forceinline__ int popc(uint64_t x) { return static_cast<int>(__popcll(x)); }
__device__ __forceinline__ Counts count_before(bool yes_a, bool yes_b, Counts& all) {
  __shared__ Counts wave[kPlanThreads / 64];
  const int lane = threadIdx.x & 63;
  const uint64_t a = __builtin_amdgcn_ballot_w64(yes_a), b = __builtin_amdgcn_ballot_w64(yes_b);
  const uint64_t below = (uint64_t{1} << lane) - 1;
  if (lane == 0) wave[threadIdx.x >> 6] = {popc(a), popc(b)};
  __syncthreads();
  Counts n = {popc(a & below), popc(b & below)};
  all = {0, 0};
#pragma unroll
  for (int i = 0; i < kPlanThreads / 64; ++i) {
    const Counts w = wave[i];
    if (i < static_cast<int>(threadIdx.x >> 6)) {
      n.a += w.a;
      n.b += w.b;
    }
    all.a += w.a;
    all.b += w.b;
  }
  __syncthreads();
  return n;
}

__global__ __launch_bounds__(kPlanThreads) void alloc_kernel(int32_t* refs, int num_slots,
                                                             int32_t* out, int n) {
  int taken = 0;
  for (int s0 = 0; s0 < num_slots && taken < n; s0 += kPlanThreads) {
    const int s = s0 + static_cast<int>(threadIdx.x);
    const bool free_slot = s < num_slots && refs[s] <= 0;
    Counts all;
    const int at = taken + count_before(free_slot, false, all).a;
    if (free_slot && at < n) {
      out[at] = s;
      refs[s] = 1;
    }
    taken += all.a;
  }
  for (int i = taken + static_cast<int>(threadIdx.x); i < n; i += kPlanThreads) out[i] = -1;
}

__global__ __launch_bounds__(kPlanThreads) void count_kernel(int32_t* refs, int num_slots,
                                                             const int32_t* slots, int n, int by) {
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int s = slots[i];
    if (s >= 0 && s < num_slots) atomicAdd(&refs[s], by);
  }
  if (by > 0) return;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int s = slots[i];
    if (s >= 0 && s < num_slots) atomicMax(&refs[s], 0);
  }
}

// moves[0] = M, then from[M] at moves[4 ..] and to[M] num_slots entries on.
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(int32_t* refs, int num_slots,
                                                            int32_t* map, int32_t* live,
                                                            int32_t* moves) {
  int32_t* from = moves + 4;
  int32_t* to = from + num_slots;
  const int t = threadIdx.x;
  const int first = t < num_slots ? refs[t] : 0;  // the first slots' counts are read once
  auto count_of = [&](int s) { return s < kPlanThreads ? first : refs[s]; };
  int n = 0;  // live slots
  for (int s0 = 0; s0 < num_slots; s0 += kPlanThreads)
    n += __syncthreads_count(s0 + t < num_slots && count_of(s0 + t) > 0);
  int moved = 0, holes = 0;
  for (int s0 = 0; s0 < num_slots; s0 += kPlanThreads) {
    const int s = s0 + t;
    const bool inside = s < num_slots;
    const bool is_live = inside && count_of(s) > 0;
    const bool moves_down = is_live && s >= n, hole = inside && !is_live && s < n;
    Counts all;
    const Counts at = count_before(moves_down, hole, all);
    if (moves_down) from[moved + at.a] = s;
    if (hole) to[holes + at.b] = s;
    if (inside) map[s] = is_live ? s : -1;
    moved += all.a;
    holes += all.b;
  }
  __syncthreads();
  for (int i = t; i < moved; i += kPlanThreads) {
    const int a = from[i], b = to[i];
    map[a] = b;
    refs[b] = refs[a];
    refs[a] = 0;
  }
  if (t == 0) {
    moves[0] = moved;
    live[0] = n;
  }
}

__global__ __launch_bounds__(kThreads) void move_kernel(const PoolView v, const int32_t* moves,
                                                        int pieces, int layers) {
  const int32_t* from = moves + 4;
  const int32_t* to = from + v.num_slots;
  const uint64_t all = static_cast<uint64_t>(moves[0]) * pieces * layers;
  for (uint64_t w = blockIdx.x; w < all; w += gridDim.x) {
    const uint64_t piece = w % pieces, rest = w / pieces;
    const int i = static_cast<int>(rest / layers);
    copy_piece(v, rest % layers, from[i], to + i, 1, piece);
  }
}

damp_status counts(const char* name, int32_t* refs, int32_t num_slots, const int32_t* slots,
                   int32_t n, int by, void* stream) {
  clear_error();
  if (num_slots <= 0 || n < 0)
    return fail(DAMP_ERR_INVALID_ARG, "%s: num_slots = %d, n = %d", name, num_slots, n);
  if (n == 0) return DAMP_OK;
  if (!refs || !slots) return fail(DAMP_ERR_INVALID_ARG, "%s: a required pointer is NULL", name);
  hipLaunchKernelGGL(count_kernel, dim3(1), dim3(kPlanThreads), 0, as_stream(stream), refs,
                     num_slots, slots, n, by);
  return check_launch(name);
}

}  // namespace
}  // namespace damp

extern "C" {

damp_status damp_slots_alloc(int32_t* refs, int32_t num_slots, int32_t* out, int32_t n,
                             void* stream) {
  using namespace damp;
  clear_error();
  const char* name = "damp_slots_alloc";
  if (num_slots <= 0 || n < 0)
    return fail(DAMP_ERR_INVALID_ARG, "%s: num_slots = %d, n = %d", name, num_slots, n);
  if (n == 0) return DAMP_OK;
  if (!refs || !out) return fail(DAMP_ERR_INVALID_ARG, "%s: a required pointer is NULL", name);
  hipLaunchKernelGGL(alloc_kernel, dim3(1), dim3(kPlanThreads), 0, as_stream(stream), refs,
                     num_slots, out, n);
  return check_launch(name);
}

damp_status damp_slots_retain(int32_t* refs, int32_t num_slots, const int32_t* slots, int32_t n,
                              void* stream) {
  return damp::counts("damp_slots_retain", refs, num_slots, slots, n, 1, stream);
}

damp_status damp_slots_release(int32_t* refs, int32_t num_slots, const int32_t* slots, int32_t n,
                               void* stream) {
  return damp::counts("damp_slots_release", refs, num_slots, slots, n, -1, stream);
}

damp_status damp_slots_fork(const damp_pool* pool, int32_t layer, const int32_t* src,
                            const int32_t* dst, int32_t n, int32_t fan, void* stream) {
  using namespace damp;
  clear_error();
  const char* name = "damp_slots_fork";
  damp_status st = check_pool(pool);
  if (st != DAMP_OK) return st;
  if (layer < -1 || layer >= pool->num_layers)
    return fail(DAMP_ERR_INVALID_ARG, "%s: layer %d outside [-1, %d)", name, layer,
                pool->num_layers);
  if (n < 0 || fan < 0 || static_cast<int64_t>(n) * fan > INT32_MAX)
    return fail(DAMP_ERR_INVALID_ARG, "%s: n = %d, fan = %d", name, n, fan);
  if (n == 0 || fan == 0) return DAMP_OK;
  if (!src || !dst) return fail(DAMP_ERR_INVALID_ARG, "%s: a required pointer is NULL", name);
  const PoolView v = view_of(pool, layer);
  const uint64_t pieces = (v.slot_bytes + kChunk - 1) / kChunk;
  const int layers = layer < 0 ? pool->num_layers : 1;
  if (pieces * n > INT32_MAX || layers > 65535)
    return fail(DAMP_ERR_INVALID_ARG, "%s: too many bytes for one call", name);
  if (slots_checked()) {
    st = debug_check_slots(pool, dst, n * fan, as_stream(stream), name);
    if (st == DAMP_OK)
      st = check_slots_apart(pool, src, n, dst, n * fan, false, as_stream(stream), name);
    if (st != DAMP_OK) return st;
  }
  hipLaunchKernelGGL(fork_kernel, dim3(static_cast<uint32_t>(pieces * n), layers), dim3(kThreads),
                     0, as_stream(stream), v, src, dst, fan, static_cast<int>(pieces));
  return check_launch(name);
}

size_t damp_slots_compact_workspace_bytes(const damp_pool* pool) {
  if (damp::check_pool(pool) != DAMP_OK) return 0;
  return (4 + 2 * static_cast<size_t>(pool->num_slots)) * sizeof(int32_t);
}

damp_status damp_slots_compact(const damp_pool* pool, int32_t* refs, int32_t* map, int32_t* live,
                               void* workspace, size_t workspace_bytes, void* stream) {
  using namespace damp;
  clear_error();
  const char* name = "damp_slots_compact";
  damp_status st = check_pool(pool);
  if (st != DAMP_OK) return st;
  if (!refs || !map || !live)
    return fail(DAMP_ERR_INVALID_ARG, "%s: a required pointer is NULL", name);
  const size_t need = damp_slots_compact_workspace_bytes(pool);
  if (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
    return fail(DAMP_ERR_INVALID_ARG, "%s: needs %zu bytes of 16-byte aligned workspace", name,
                need);
  const PoolView v = view_of(pool, -1);
  const uint64_t pieces = (v.slot_bytes + kChunk - 1) / kChunk;
  if (pieces > INT32_MAX)
    return fail(DAMP_ERR_INVALID_ARG, "%s: too many bytes in a slot", name);
  int32_t* moves = static_cast<int32_t*>(workspace);
  hipStream_t s = as_stream(stream);
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, refs, pool->num_slots, map,
                     live, moves);
  // a move goes from above the live slots into a hole among them: at most half
  const uint64_t most = pieces * pool->num_layers * static_cast<uint64_t>(pool->num_slots / 2);
  const uint32_t grid = static_cast<uint32_t>(most < 4096 ? most : 4096);
  if (grid > 0)
    hipLaunchKernelGGL(move_kernel, dim3(grid), dim3(kThreads), 0, s, v, moves,
                       static_cast<int>(pieces), pool->num_layers);
  return check_launch(name);
}

}  // extern "C"

// Verification of drafted tokens (damp_serving.h): which drafts stand, and
// the next token drawn from what the target has over the draft.
//
// One row of V weights is summed and searched for each request (its first
// refused draft's, or the one after its last), so the row's bytes bound the
// operator. A row is cut into tiles, one workgroup each; weights are whole
// numbers of 2^-40, so the tiles' sums are exact in any order. A second kernel
// finds the tile in which the running sum passes the drawn threshold and
// scans that tile again.
#include "device.hpp"
#include "internal.hpp"

namespace damp {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 4096;  // tokens of a tile
constexpr int kMaxDrafts = 1024;

struct VerifyParams {
  const void* p;
  const void* q;
  const int32_t* tokens;
  const int32_t* lens;
  const float* u;
  int32_t* accepted;
  int32_t* out;
  uint64_t* sums;  // [B, tiles]
  int32_t K, V, tiles;
};

template <typename T>
__device__ __forceinline__ float prob(const T* row, int x) {
  if constexpr (sizeof(T) == 4) return row[x];
  else return bf16_to_f32(row[x]);
}

// floor(2^40 min(max(y, 0), 1)), in two exact steps of 20 bits each.
__device__ __forceinline__ uint64_t fix40(float y) {
  y = y > 0.0f ? fminf(y, 1.0f) : 0.0f;
  const float up = y * 1048576.0f;
  const uint32_t hi = static_cast<uint32_t>(up);
  const uint32_t lo = static_cast<uint32_t>((up - static_cast<float>(hi)) * 1048576.0f);
  return (static_cast<uint64_t>(hi) << 20) + lo;
}

template <typename T>
__device__ __forceinline__ uint64_t weight(const T* p, const T* q, int x) {
  const uint64_t a = fix40(prob(p, x));
  if (!q) return a;
  const uint64_t b = fix40(prob(q, x));
  return a > b ? a - b : 0;
}

// The drafts of request b that stand; every thread receives the number.
template <typename T>
__device__ int drafts_that_stand(const VerifyParams& v, int b, int& n) {
  __shared__ int first;
  n = v.lens ? min(max(v.lens[b], 0), v.K) : v.K;
  if (threadIdx.x == 0) first = n;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int x = v.tokens[static_cast<size_t>(b) * v.K + i];
    bool stands = x >= 0 && x < v.V;
    if (stands) {
      const size_t row = static_cast<size_t>(b) * v.K + i;
      const T* p = static_cast<const T*>(v.p) + (row + b) * v.V;
      const T* q = static_cast<const T*>(v.q) + row * v.V;
      // the product of two fp32 numbers is exact in double
      stands = static_cast<double>(v.u[row + b]) * static_cast<double>(prob(q, x)) <
               static_cast<double>(prob(p, x));
    }
    if (!stands) atomicMin(&first, i);
  }
  __syncthreads();
  return first;
}

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(static_cast<unsigned long long>(x), m, 64);
  return x;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_sums(const VerifyParams v) {
  __shared__ uint64_t part[kThreads / 64];
  const int b = blockIdx.y, t = threadIdx.x;
  int n;
  const int a = drafts_that_stand<T>(v, b, n);
  const T* p = static_cast<const T*>(v.p) + (static_cast<size_t>(b) * (v.K + 1) + a) * v.V;
  const T* q = a < n ? static_cast<const T*>(v.q) + (static_cast<size_t>(b) * v.K + a) * v.V
                     : nullptr;
  const int x0 = blockIdx.x * kTile, x1 = min(x0 + kTile, v.V);
  uint64_t s = 0;
  for (int x = x0 + t; x < x1; x += kThreads) s += weight(p, q, x);
  s = wave_sum_u64(s);
  if ((t & 63) == 0) part[t >> 6] = s;
  __syncthreads();
  if (t == 0)
    v.sums[static_cast<size_t>(b) * v.tiles + blockIdx.x] =
        (part[0] + part[1]) + (part[2] + part[3]);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_draw(const VerifyParams v) {
  __shared__ uint64_t before[kThreads];
  __shared__ uint64_t rest;
  __shared__ int found;
  const int b = blockIdx.x, t = threadIdx.x;
  int n;
  const int a = drafts_that_stand<T>(v, b, n);
  const T* p = static_cast<const T*>(v.p) + (static_cast<size_t>(b) * (v.K + 1) + a) * v.V;
  const T* q = a < n ? static_cast<const T*>(v.q) + (static_cast<size_t>(b) * v.K + a) * v.V
                     : nullptr;
  if (t == 0) {
    const uint64_t* sums = v.sums + static_cast<size_t>(b) * v.tiles;
    uint64_t total = 0;
    for (int i = 0; i < v.tiles; ++i) total += sums[i];
    const float u = v.u[static_cast<size_t>(b) * (v.K + 1) + v.K];
    const uint32_t r = u > 0.0f ? min(static_cast<uint32_t>(fminf(u, 1.0f) * 16777216.0f), 0xffffffu)
                                : 0u;
    uint64_t left = (total >> 24) * r + (((total & 0xffffffu) * r) >> 24);
    int tile = -1;
    if (total > 0)
      for (tile = 0; left >= sums[tile]; ++tile) left -= sums[tile];
    rest = left;
    found = tile;
  }
  __syncthreads();
  const int tile = found;
  int next = -1;
  if (tile >= 0) {
    // thread t sums its run of the tile's tokens; the run that the threshold
    // falls into is walked by its thread
    const int run = kTile / kThreads;
    const int x0 = tile * kTile + t * run, x1 = min(x0 + run, v.V);
    uint64_t s = 0;
    for (int x = x0; x < x1; ++x) s += weight(p, q, x);
    before[t] = s;
    __syncthreads();
    uint64_t sum = 0;
    for (int i = 0; i < t; ++i) sum += before[i];
    if (rest >= sum && rest < sum + s) {
      uint64_t left = rest - sum;
      for (int x = x0; x < x1; ++x) {
        const uint64_t w = weight(p, q, x);
        if (left < w) {
          next = x;
          break;
        }
        left -= w;
      }
      found = next;
    }
    __syncthreads();
    next = found;
  }
  if (t == 0) v.accepted[b] = a;
  for (int i = t; i <= v.K; i += kThreads)
    v.out[static_cast<size_t>(b) * (v.K + 1) + i] =
        i < a ? v.tokens[static_cast<size_t>(b) * v.K + i] : (i == a ? next : -1);
}

}  // namespace
}  // namespace damp

extern "C" {

size_t damp_verify_workspace_bytes(int32_t B, int32_t V) {
  if (B <= 0 || B > 65535 || V <= 0 || V > (1 << 22)) return 0;
  const size_t tiles = (static_cast<size_t>(V) + damp::kTile - 1) / damp::kTile;
  return static_cast<size_t>(B) * tiles * sizeof(uint64_t);
}

damp_status damp_verify_drafts(const void* p, const void* q, int32_t dtype, const int32_t* tokens,
                               const int32_t* lens, const float* u, int32_t B, int32_t K, int32_t V,
                               int32_t* accepted, int32_t* out, void* workspace,
                               size_t workspace_bytes, void* stream) {
  using namespace damp;
  clear_error();
  const char* name = "damp_verify_drafts";
  if (B < 0 || B > 65535) return fail(DAMP_ERR_INVALID_ARG, "%s: B = %d outside [0, 65535]", name, B);
  if (K < 0 || K > kMaxDrafts)
    return fail(DAMP_ERR_INVALID_ARG, "%s: K = %d outside [0, %d]", name, K, kMaxDrafts);
  if (V < 1 || V > (1 << 22))
    return fail(DAMP_ERR_INVALID_ARG, "%s: V = %d outside [1, 2^22]", name, V);
  if (dtype != DAMP_DT_FP32 && dtype != DAMP_DT_BF16)
    return fail(DAMP_ERR_INVALID_ARG, "%s: dtype must be FP32 or BF16", name);
  if (B == 0) return DAMP_OK;
  if (!p || !u || !accepted || !out || (K > 0 && (!q || !tokens)))
    return fail(DAMP_ERR_INVALID_ARG, "%s: a required pointer is NULL", name);
  const size_t need = damp_verify_workspace_bytes(B, V);
  if (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
    return fail(DAMP_ERR_INVALID_ARG, "%s: needs %zu bytes of 16-byte aligned workspace", name,
                need);
  VerifyParams v;
  v.p = p;
  v.q = q;
  v.tokens = tokens;
  v.lens = lens;
  v.u = u;
  v.accepted = accepted;
  v.out = out;
  v.sums = static_cast<uint64_t*>(workspace);
  v.K = K;
  v.V = V;
  v.tiles = (V + kTile - 1) / kTile;
  hipStream_t s = as_stream(stream);
  if (dtype == DAMP_DT_FP32) {
    hipLaunchKernelGGL(verify_sums<float>, dim3(v.tiles, B), dim3(kThreads), 0, s, v);
    hipLaunchKernelGGL(verify_draw<float>, dim3(B), dim3(kThreads), 0, s, v);
  } else {
    hipLaunchKernelGGL(verify_sums<uint16_t>, dim3(v.tiles, B), dim3(kThreads), 0, s, v);
    hipLaunchKernelGGL(verify_draw<uint16_t>, dim3(B), dim3(kThreads), 0, s, v);
  }
  return check_launch(name);
}

}  // extern "C"

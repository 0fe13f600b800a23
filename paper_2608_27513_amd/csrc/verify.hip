// Verification of drafted tokens (damp_serving.h): which drafts stand, and
// the next token drawn from what the target has over the draft.
//
// The scheme is the published rejection sampling of speculative decoding
// (Leviathan, Kalman and Matias, 2023; Chen et al., 2023), decided exactly.
//
// One row of V weights is summed and searched for each request (its first
// refused draft's, or the one after its last), so the row's bytes, of p and
// after a refusal of q, bound the operator; short rows are bound by the chain
// lens -> tokens -> their probabilities -> the row.
//
// Weights are whole numbers of 2^-40, so sums are exact in any order. A wave
// takes 64 vectors of 16 bytes of the row (a "piece") at a time and leaves the
// piece's sum; the last workgroup of a request to finish (a ticket, so nothing
// waits) runs over the sums to the piece that the drawn threshold falls into
// and scans that one again. The largest rows are read once by many workgroups
// and the rest of the work is a few kilobytes, in one launch: 128 requests of
// 151001 fp32 tokens take 30 us (110 MB, 3.7 TB/s), one of 32000 6.6 us, which
// is the launch and two chains of dependent loads. Twice the pieces in flight, by
// a second set of registers, is slower (36.6 us against 30.7, side by side).
#include <algorithm>

#include "device.hpp"
#include "internal.hpp"

namespace damp {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxDrafts = 1024;
constexpr int kTickets = 65536;
constexpr int kAhead = 4;  // pieces of a wave in flight

struct VerifyParams {
  const void* p;
  const void* q;
  const int32_t* tokens;
  const int32_t* lens;
  const float* u;
  int32_t* accepted;
  int32_t* out;
  uint32_t* tickets;  // [65536], zero between calls; a request's is at b * spacing
  uint64_t* sums;     // [B, pieces]
  int32_t K, V;
  int32_t pieces;  // of a row
  int32_t steps;   // pieces of a wave
  int32_t spacing;
};

template <typename T>
constexpr int vec() {
  return 16 / static_cast<int>(sizeof(T));
}

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return bf16_to_f32(x); }

// vec<T>() values from x on, zero from V on. Rows start anywhere (V is any
// number), which wide loads may do here.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
  T v[vec<T>()];
};
template <typename T>
__device__ __forceinline__ Vec<T> load_vec(const T* row, int x, int V) {
  Vec<T> r;
  if (x + vec<T>() <= V) {
    r = *reinterpret_cast<const Vec<T>*>(row + x);
  } else {
#pragma unroll
    for (int i = 0; i < vec<T>(); ++i) {
      r.v[i] = 0;
      if (x + i < V) r.v[i] = row[x + i];
    }
  }
  return r;
}

// floor(2^40 min(max(y, 0), 1)) (0 for NaN) as hi 2^20 + lo, in exact steps of
// 20 bits.
__device__ __forceinline__ void fix40(float y, int& hi, int& lo) {
  const float up = __builtin_amdgcn_fmed3f(y, 0.0f, 1.0f) * 1048576.0f;
  const float whole = floorf(up);
  hi = static_cast<int>(whole);
  lo = static_cast<int>((up - whole) * 1048576.0f);
}

// A uniform number cut to [0, 1 - 2^-24], NaN to 0. (fmaxf gives its other
// operand for a NaN.)
__device__ __forceinline__ float uniform(float u) {
  return fminf(fmaxf(u, 0.0f), 1.0f - 0x1p-24f);
}

// The weight of a token as hi 2^20 + lo (lo may be negative).
__device__ __forceinline__ void weight(float p, float q, int& hi, int& lo) {
  int hp, lp, hq, lq;
  fix40(p, hp, lp);
  fix40(q, hq, lq);
  const bool over = hp > hq || (hp == hq && lp > lq);
  hi = over ? hp - hq : 0;
  lo = over ? lp - lq : 0;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_i32(int x) {
  return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false);
}
// Sum over a wave, in lane 63.
__device__ __forceinline__ int wave_sum_i32(int x) {
  x += dpp_i32<0x111, 0xf>(x);
  x += dpp_i32<0x112, 0xf>(x);
  x += dpp_i32<0x114, 0xf>(x);
  x += dpp_i32<0x118, 0xf>(x);
  x += dpp_i32<0x142, 0xa>(x);
  x += dpp_i32<0x143, 0xc>(x);
  return x;
}
// Sum over the lanes before this one.
__device__ __forceinline__ uint64_t wave_before_u64(uint64_t x) {
  const int lane = threadIdx.x & 63;
  unsigned long long s = x;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const unsigned long long y = __shfl_up(s, m, 64);
    if (lane >= m) s += y;
  }
  return s - x;
}

template <typename T, bool REFUSED>
__device__ __forceinline__ uint64_t vec_weight(const Vec<T>& p, const Vec<T>& q, int i) {
  int hi, lo;
  if constexpr (REFUSED) weight(widen(p.v[i]), widen(q.v[i]), hi, lo);
  else fix40(widen(p.v[i]), hi, lo);
  return (static_cast<uint64_t>(hi) << 20) + static_cast<uint64_t>(static_cast<int64_t>(lo));
}

// The sums of this wave's pieces.
template <typename T, bool REFUSED>
__device__ __forceinline__ void sum_pieces(const VerifyParams& v, const T* p, const T* q,
                                           uint64_t* sums, int piece0) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < v.steps; s0 += kAhead) {
    Vec<T> pv[kAhead], qv[kAhead];
    const int piece = piece0 + s0;
    if (s0 + kAhead <= v.steps && (piece + kAhead) * 64 * vec<T>() <= v.V) {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        const int x = ((piece + s) * 64 + lane) * vec<T>();
        pv[s] = *reinterpret_cast<const Vec<T>*>(p + x);
        if constexpr (REFUSED) qv[s] = *reinterpret_cast<const Vec<T>*>(q + x);
      }
    } else {
#pragma unroll
      for (int s = 0; s < kAhead; ++s) {
        const int x = ((piece + s) * 64 + lane) * vec<T>();
        const int end = s0 + s < v.steps ? v.V : 0;
        pv[s] = load_vec(p, x, end);
        if constexpr (REFUSED) qv[s] = load_vec(q, x, end);
      }
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      if (s0 + s >= v.steps || piece + s >= v.pieces) break;
      int hi = 0, lo = 0;
#pragma unroll
      for (int i = 0; i < vec<T>(); ++i) {
        int h, l;
        if constexpr (REFUSED) weight(widen(pv[s].v[i]), widen(qv[s].v[i]), h, l);
        else fix40(widen(pv[s].v[i]), h, l);
        hi += h;  // at most 2^9 weights of 2^20
        lo += l;
      }
      hi = wave_sum_i32(hi);
      lo = wave_sum_i32(lo);
      if (lane == 63)
        __hip_atomic_store(&sums[piece + s],
                           (static_cast<uint64_t>(hi) << 20) + static_cast<int64_t>(lo),
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
}

// The token in which the running sum passes `left`, in the piece that it does.
template <typename T, bool REFUSED>
__device__ __forceinline__ void draw_in_piece(const VerifyParams& v, const T* p, const T* q,
                                              int piece, uint64_t left, int* next) {
  const int x = (piece * 64 + (threadIdx.x & 63)) * vec<T>();
  const Vec<T> pv = load_vec(p, x, v.V);
  Vec<T> qv = pv;
  if constexpr (REFUSED) qv = load_vec(q, x, v.V);
  uint64_t s = 0;
#pragma unroll
  for (int i = 0; i < vec<T>(); ++i) s += vec_weight<T, REFUSED>(pv, qv, i);
  uint64_t before = wave_before_u64(s);
  if (left < before || left >= before + s) return;
  int at = 0;
  bool found = false;
#pragma unroll
  for (int i = 0; i < vec<T>(); ++i) {
    before += vec_weight<T, REFUSED>(pv, qv, i);
    if (!found && left < before) {
      found = true;
      at = x + i;
    }
  }
  *next = at;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void verify_kernel(const VerifyParams v) {
  __shared__ int first, last, found_piece, next;
  __shared__ uint64_t found_left, wave_total[kWaves];
  const int b = blockIdx.y, t = threadIdx.x, lane = t & 63, wave = t >> 6;

  // ---- the drafts that stand
  const int n = v.lens ? min(max(v.lens[b], 0), v.K) : v.K;
  if (t == 0) {
    first = n;
    next = -1;
  }
  __syncthreads();
  for (int i = t; i < n; i += kThreads) {
    const int x = v.tokens[static_cast<size_t>(b) * v.K + i];
    bool stands = x >= 0 && x < v.V;
    if (stands) {
      const size_t row = static_cast<size_t>(b) * v.K + i;
      const float px = widen(static_cast<const T*>(v.p)[(row + b) * v.V + x]);
      const float qx = widen(static_cast<const T*>(v.q)[row * v.V + x]);
      // the product of two fp32 numbers is exact in double
      stands = static_cast<double>(uniform(v.u[row + b])) * static_cast<double>(qx) <
               static_cast<double>(px);
    }
    if (!stands) atomicMin(&first, i);
  }
  __syncthreads();
  const int a = first;
  const bool refused = a < n;
  const T* p = static_cast<const T*>(v.p) + (static_cast<size_t>(b) * (v.K + 1) + a) * v.V;
  const T* q = static_cast<const T*>(v.q) + (static_cast<size_t>(b) * v.K + a) * v.V;

  // ---- the sums of this workgroup's pieces
  uint64_t* sums = v.sums + static_cast<size_t>(b) * v.pieces;
  const int piece0 = (static_cast<int>(blockIdx.x) * kWaves + wave) * v.steps;
  if (refused) sum_pieces<T, true>(v, p, q, sums, piece0);
  else sum_pieces<T, false>(v, p, q, sums, piece0);
  // The sums go through agent-scope atomic stores and loads, which pass the
  // L2 of their XCD, so they are in order with the ticket as soon as the stores
  // are acknowledged. A release fence would do, but writes back the whole L2
  // for each workgroup (270 us against 30 at 128 requests of 151001 tokens).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (t == 0) {
    const uint32_t ticket =
        __hip_atomic_fetch_add(&v.tickets[b * v.spacing], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    last = ticket == gridDim.x - 1;
    if (last)
      __hip_atomic_store(&v.tickets[b * v.spacing], 0u, __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!last) return;

  // ---- the last of a request: the piece that the threshold falls into
  const int each = (v.pieces + kThreads - 1) / kThreads;
  const int i0 = min(t * each, v.pieces), i1 = min(i0 + each, v.pieces);
  auto sum_of = [&](int i) {
    return __hip_atomic_load(&sums[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  uint64_t s = 0;
  for (int i = i0; i < i1; ++i) s += sum_of(i);
  uint64_t before = wave_before_u64(s);
  if (lane == 63) wave_total[wave] = before + s;
  if (t == 0) found_piece = -1;
  __syncthreads();
  uint64_t total = 0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    if (i < wave) before += wave_total[i];
    total += wave_total[i];
  }
  const uint32_t r = static_cast<uint32_t>(
      uniform(v.u[static_cast<size_t>(b) * (v.K + 1) + v.K]) * 16777216.0f);
  const uint64_t threshold = (total >> 24) * r + (((total & 0xffffffu) * r) >> 24);
  if (threshold >= before && threshold < before + s) {
    uint64_t left = threshold - before;
    int i = i0;
    for (; i + 1 < i1; ++i) {
      const uint64_t w = sum_of(i);
      if (left < w) break;
      left -= w;
    }
    found_piece = i;
    found_left = left;
  }
  __syncthreads();
  if (wave == 0 && found_piece >= 0) {
    if (refused) draw_in_piece<T, true>(v, p, q, found_piece, found_left, &next);
    else draw_in_piece<T, false>(v, p, q, found_piece, found_left, &next);
  }
  __syncthreads();
  if (t == 0) v.accepted[b] = a;
  for (int i = t; i <= v.K; i += kThreads)
    v.out[static_cast<size_t>(b) * (v.K + 1) + i] =
        i < a ? v.tokens[static_cast<size_t>(b) * v.K + i] : (i == a ? next : -1);
}

// Pieces of a wave: as few as make kWorkgroups workgroups, four on each of 256
// CUs. Each first follows the chain of dependent loads to its row and ends with
// an atomic, so more of them cost more than the loads that they add (64
// requests of 131072 bf16 tokens: 512 / 1024 / 1536 / 2048 take 15.5 / 16.0 /
// 17.6 / 17.5 us, 128 of 151001 fp32 tokens 34.9 / 30.3 / 30.1 / 30.2).
constexpr int kWorkgroups = 1024;
// Tickets of different requests in lines of their own, as far as there is room
// (16 requests of 128000 tokens: 9.8 us against 30 side by side).
constexpr int kTicketLine = 32;

template <typename T>
void launch(VerifyParams v, int B, hipStream_t s) {
  v.pieces = (v.V + 64 * vec<T>() - 1) / (64 * vec<T>());
  const int64_t waves = static_cast<int64_t>(v.pieces) * B;
  const int64_t steps = (waves + kWorkgroups * kWaves - 1) / (kWorkgroups * kWaves);
  v.steps = static_cast<int32_t>(steps < v.pieces ? steps : v.pieces);
  const int blocks = (v.pieces + kWaves * v.steps - 1) / (kWaves * v.steps);
  v.spacing = std::min(kTickets / B, kTicketLine);
  hipLaunchKernelGGL(verify_kernel<T>, dim3(blocks, B), dim3(kThreads), 0, s, v);
}

// Tickets have one place whatever B is: a workspace may serve any batch.
constexpr size_t kTicketBytes = kTickets * sizeof(uint32_t);

}  // namespace
}  // namespace damp

extern "C" {

size_t damp_verify_workspace_bytes(int32_t B, int32_t V) {
  if (B <= 0 || B > 65535 || V <= 0 || V > (1 << 22)) return 0;
  const size_t pieces = (static_cast<size_t>(V) + 255) / 256;
  return damp::kTicketBytes + static_cast<size_t>(B) * pieces * sizeof(uint64_t);
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
  const uintptr_t at = reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(q);
  if (at % (dtype == DAMP_DT_FP32 ? 4 : 2) != 0)
    return fail(DAMP_ERR_INVALID_ARG, "%s: p and q must be aligned to their type", name);
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
  v.tickets = static_cast<uint32_t*>(workspace);
  v.sums = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(workspace) + kTicketBytes);
  v.K = K;
  v.V = V;
  if (dtype == DAMP_DT_FP32) launch<float>(v, B, as_stream(stream));
  else launch<uint16_t>(v, B, as_stream(stream));
  return check_launch(name);
}

}  // extern "C"

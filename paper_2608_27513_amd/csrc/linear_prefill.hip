// Linear attention with one decay a head over packed prompts, on the matrix
// cores.
//
// A request's tokens are taken in chunks of C = 64. With L_i the sum of the
// log-decays of a chunk's tokens up to i, and S the state before it,
//   o_i = scale (exp(L_i) S^T q_i + sum_{j <= i} exp(L_i - L_j) (q_i . k_j) v_j)
//   S'  = exp(L_C) S + sum_j k_j (exp(L_C - L_j) v_j)^T
// which are four products: K Q^T, S^T Q^T, V^T P^T (P the decayed, causal
// scores) and K^T (D V).
//
// A workgroup owns up to 128 columns of the state of one (request, value
// head), 32 columns a wave, in accumulators for its whole run of tokens. All
// products are 32x32x16 bf16 instructions, whose results hold column n of a
// lane in the order that the next product wants its operand: with
//   k slots (lane half h, j = 0 .. 7)  <->  rows 16 s + 4 h + j (+ 4 if j > 3)
// the state's accumulators are S^T's operand and the scores' are P^T's without
// leaving the lane. The state's rows are key channels in an order that makes
// these 8 rows 8 neighbouring channels (the middle two quads of every 16 are
// swapped), so that K and Q are read as they are; K^T and V^T come through
// transposing LDS reads.
//
// q, k, v are bf16 and enter as they are. What is fp32 (S, P, D V) enters as
// a sum of bf16 parts, x = x1 + x2 (+ x3), each the rounding of what the
// parts before it leave: three parts hold all 24 bits (the state, and o in
// fp32), two hold 16 (for o in bf16, whose own rounding is 2^-8: with three, 423
// us against 368 at 32768 tokens, 164 against 150 for eleven packed prompts).
//
// Log-decays are summed in double, in units of log2: their differences stay
// good to fp32 however far the sum has run. A log-decay below -1000 counts as
// that (its factor is 0 in fp32 either way), so -inf makes no inf - inf. Where
// log-decays are positive a chunk ends before their sum passes kMostGrowth (one
// token alone may): a factor over more tokens would lose digits, and leave fp32
// where what it multiplies is 0 or tiny. The factor of a segment has an exponent
// of its own for the same reason.
//
// q, k, v and o set the floor: memory, as 4 d_k d_v operations a token and head
// are few beside their bytes. What bounds the kernel is the issue of vector and matrix
// instructions and the waits between them: at 32768 tokens, 32 heads of 128 and
// o in bf16, 372 us in three launches (130 + 11 + 235 at their fastest in a
// profile, 136 + 12 + 245 at the median there), 185 TFLOP/s of the recurrence's
// operations and 2.2 TB/s of the floor's bytes, the third launch with its matrix
// units busy 37% and its vector issue 41% of the time, 1.6 waves a SIMD. Tried
// and not kept: the parts of the next step placed between the products of this
// one (the same time), a fourth wave that repeats a score tile to avoid the
// branch (slower).
//
// Where there are fewer requests and heads than the device has room for, the
// tokens are cut into segments: a first pass leaves the state that each
// segment adds, a second runs over the segments to the state before each,
// and the third works on all segments at once.
#include <algorithm>

#include "device.hpp"
#include "linear.hpp"

namespace damp {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 64;
constexpr int kBufferConfig = 0x00020000;  // raw 32-bit buffer (gfx9 family)
constexpr uint32_t kNowhere = 0x80000000u;  // past the end of every buffer here
constexpr float kLeastLog = -1000.0f;
constexpr double kLog2e = 1.4426950408889634;
constexpr double kMostGrowth = 16.0;  // log2; exponents below it are good to 2^-21 in fp32

struct PromptParams {
  LinearParams l;
  const int32_t* seq_start;
  const int32_t* seq_len;
  float* seg_states;  // [B, segments, HV, dk, dv]
  float2* seg_decays;  // [B, segments, HV]: x 2^y, 1 <= x <= 2
  int32_t n_tokens;
  int32_t max_len;
  int32_t seg_len;   // tokens, a multiple of kChunk
  int32_t segments;  // of the longest request
};

// One number of a request, the same in every lane, and in a scalar register:
// what buffers are described by has to be.
__device__ __forceinline__ int of_request(const int32_t* numbers, int b) {
  return __builtin_amdgcn_readfirstlane(numbers[b]);
}

// First token and length of request b, within the token axis and max_len.
__device__ __forceinline__ void request_range(const PromptParams& p, int b, int& start, int& len) {
  start = of_request(p.seq_start, b);
  const bool inside = start >= 0 && start <= p.n_tokens;
  len = inside ? min(min(of_request(p.seq_len, b), p.max_len), p.n_tokens - start) : 0;
  len = __builtin_amdgcn_readfirstlane(max(len, 0));
  if (!inside) start = 0;
}

__device__ __forceinline__ int segments_of(const PromptParams& p, int len) {
  return len > 0 ? (len - 1) / p.seg_len + 1 : 1;
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Eight values as PARTS bf16 vectors that add up to them; x keeps what the last
// part was rounded from.
template <int PARTS>
__device__ __forceinline__ void split8(float (&x)[8], u32x4 (&out)[PARTS]) {
#pragma unroll
  for (int n = 0; n < PARTS; ++n) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
      if (n + 1 < PARTS) {
        x[2 * j] -= bf16_lo(w[j]);
        x[2 * j + 1] -= bf16_hi(w[j]);
      }
    }
    out[n] = w;
  }
}

typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Four tokens of one column per lane, from rows of 16-bit values in LDS: each
// lane gives the place of four columns of one token.
__device__ __forceinline__ uint2 read_columns(const uint16_t* at) {
  return __builtin_bit_cast(
      uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at));
}
__device__ __forceinline__ bf16x8 read_columns8(const uint16_t* at, int step) {
  const uint2 a = read_columns(at), b = read_columns(at + step);
  const u32x4 w = {a.x, a.y, b.x, b.y};
  return __builtin_bit_cast(bf16x8, w);
}

// An offset into a buffer, past its end where `in` is false; as a select.
__device__ __forceinline__ uint32_t offset_if(bool in, uint32_t at) {
  asm("" : "+v"(at));
  return in ? at : kNowhere;
}

// The rows from `row0` on of a chunk as a buffer: reads of rows past `rows`
// give zeros and writes to them are dropped. row_bytes * 64 < 2^31.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const void* base, int64_t row0,
                                                          int64_t row_bytes, int rows) {
  // (a clamp is a vector instruction: back into a scalar register)
  const int n = __builtin_amdgcn_readfirstlane(max(min(rows, kChunk), 0));
  return __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(static_cast<const uint8_t*>(base)) + row0 * row_bytes, 0,
      n * static_cast<int>(row_bytes), kBufferConfig);
}

// One head's state.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t state_buffer(const float* state,
                                                               const LinearParams& p) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(state), 0, p.dk * p.dv * 4,
                                           kBufferConfig);
}

// Sum over the lanes up to this one (zeros come in from below).
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_f64(double x) {
  const uint64_t w = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(w), CTRL, ROWS, 0xf, false);
  const uint32_t hi =
      __builtin_amdgcn_update_dpp(0, static_cast<int>(w >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double wave_scan_f64(double x) {
  x += dpp_f64<0x111, 0xf>(x);  // row_shr 1, 2, 4, 8
  x += dpp_f64<0x112, 0xf>(x);
  x += dpp_f64<0x114, 0xf>(x);
  x += dpp_f64<0x118, 0xf>(x);
  x += dpp_f64<0x142, 0xa>(x);  // the last lane of each row of 16 into the next
  x += dpp_f64<0x143, 0xc>(x);  // the last lane of the first half into the second
  return x;
}

// 2^x with fp32's digits however large |x| is.
__device__ __forceinline__ float exp2_f32(double x) {
  const double whole = floor(x);
  return ldexpf(__builtin_amdgcn_exp2f(static_cast<float>(x - whole)), static_cast<int>(whole));
}

// 2^x in double, by the series of e^y to y^9 at |y| <= ln(2) / 2 (7e-12 of it is
// left out). A loop: its constants would be kept in registers otherwise.
__constant__ const double kInverseFactorial[10] = {
    1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880};
__device__ __forceinline__ double exp2_f64(double x) {
  const double whole = __builtin_rint(x), y = (x - whole) * 0.6931471805599453;
  double sum = 0.0;
#pragma clang loop unroll(disable)
  for (int n = 9; n >= 0; --n) sum = fma(sum, y, kInverseFactorial[n]);
  return ldexp(sum, static_cast<int>(whole));
}

// PARTS = 0: the first pass, which leaves the state of each segment but the
// last from a zero start. PARTS = 2 or 3: outputs, with so many parts of S
// and P.
template <int DK, int NW, int PARTS>
__global__ __launch_bounds__(64 * NW, DK <= 128 ? 2 : 1) void prompt_chunks(const PromptParams pp) {
  const LinearParams& p = pp.l;
  constexpr bool kOut = PARTS > 0;
  constexpr int NT = 64 * NW;
  constexpr int KT = DK / 32;             // state tiles of a wave
  constexpr int QS = DK + 8;              // row of Q in LDS, 16-bit values
  // rows of K 20 words of the 64 banks apart: 16 rows side by side and 4 rows
  // of 16 columns both spread over (nearly) all of them; rows of V 16 apart
  constexpr int KS = DK + 40, VS = 32 * NW + 32;
  constexpr int KV = 64 * (DK / 8) / NT;  // 16-byte loads of a thread for K (and Q)
  constexpr int VV = 4;                   // and for V
  constexpr int NP = kOut ? PARTS : 1;

  __shared__ __attribute__((aligned(16))) uint16_t kt[kChunk * KS];
  __shared__ __attribute__((aligned(16))) uint16_t qt[kOut ? kChunk * QS : 8];
  __shared__ __attribute__((aligned(16))) uint16_t vt[kChunk * VS];
  __shared__ u32x4 pt[kOut ? 3 * 2 * NP * 64 : 1];
  __shared__ float2 logs[2][kChunk];  // L_i as a multiple of 2^-6 and the rest
  __shared__ __attribute__((aligned(16))) float to_end[2][kChunk];
  __shared__ float from_start[2][kChunk];  // times the scale
  __shared__ float chunk_decay[2];
  __shared__ int chunk_len[2];

  // Branches from here on go by scalars. In a branch that only some lanes or
  // waves take, the compiler may save a register before the others are back,
  // which then lose it: seen with states of 256 channels, whose accumulators
  // crowd the rest out of the vector registers.
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const int half = lane >> 5, n32 = lane & 31;
  const int blocks_v = (p.dv + 32 * NW - 1) / (32 * NW);
  const int nx = p.HV * blocks_v;
  // heads that share keys on one XCD (workgroups go to the 8 XCDs in turn)
  const int x = nx % 8 == 0 ? (blockIdx.x % 8) * (nx / 8) + blockIdx.x / 8 : blockIdx.x;
  const int h = x / blocks_v, col0 = (x % blocks_v) * 32 * NW;
  const int b = blockIdx.y, seg = blockIdx.z;
  const int hk = h / (p.HV / p.HK);

  int start, len;
  request_range(pp, b, start, len);
  const int segs = segments_of(pp, len);
  if (seg >= (kOut ? segs : segs - 1)) return;
  const int64_t tok0 = static_cast<int64_t>(start) + static_cast<int64_t>(seg) * pp.seg_len;
  const int count = min(pp.seg_len, len - seg * pp.seg_len);

  const int from = of_request(p.slot_in, b), to = of_request(p.slot_out, b);
  const bool old = from >= 0 && from < p.num_slots;
  const bool keep = to >= 0 && to < p.num_slots;
  if (!old && from != DAMP_SLOT_ZERO) {  // padded request
    if constexpr (kOut) {
      const int w = min(p.dv - col0, 32 * NW);
      for (int64_t i = t; i < static_cast<int64_t>(count) * w; i += NT) {
        const size_t at = (static_cast<size_t>(tok0 + i / w) * p.HV + h) * p.dv + col0 + i % w;
        if (p.o_bf16) static_cast<uint16_t*>(p.o)[at] = 0;
        else static_cast<float*>(p.o)[at] = 0.0f;
      }
    }
    return;
  }

  const uint16_t* kb = p.k + hk * p.dk;
  const uint16_t* qb = p.q + hk * p.dk;
  const uint16_t* vb = p.v + static_cast<int64_t>(h) * p.dv + col0;
  const float* gb = p.g + h;

  // ---- the state before the first token
  const int col = col0 + 32 * wave + n32;
  const size_t tile = (static_cast<size_t>(b) * pp.segments * p.HV + h) * p.dk * p.dv;
  const size_t tile_step = static_cast<size_t>(p.HV) * p.dk * p.dv;
  // this lane's first row and column; rows and columns past the head are
  // past the buffer's end
  const uint32_t s_row = 4 * p.dv;
  const uint32_t s_at = offset_if(col < p.dv, 8 * half * s_row + 4 * col);
  f32x16 S[KT];
#pragma unroll
  for (int c = 0; c < KT; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) S[c][r] = 0.0f;
  if constexpr (kOut) {
    const float* src = nullptr;
    if (segs > 1)
      src = pp.seg_states + tile + seg * tile_step;
    else if (old)
      src = reinterpret_cast<const float*>(p.layer_base + from * p.slot_stride + h * p.tile_stride);
    if (src) {
      const auto sbuf = state_buffer(src, p);
#pragma unroll
      for (int c = 0; c < KT; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          S[c][r] = __uint_as_float(
              __builtin_amdgcn_raw_buffer_load_b32(sbuf, s_at + s_row * (32 * c + 16 * (r / 8) + r % 8), 0, 0));
    }
  }

  // ---- loads of a chunk: rows past the end and columns past the head are zero
  const int64_t k_row = 2 * p.k_stride, q_row = 2 * p.q_stride, v_row = 2 * p.v_stride;
  const int64_t o_row = static_cast<int64_t>(p.HV) * p.dv * (p.o_bf16 ? 2 : 4);
  constexpr int kRows = NT / (DK / 8), vRows = 16;  // rows that one load instruction spans
  const int k8 = t % (DK / 8), v8 = t % (4 * NW);
  const uint32_t k_at =
      offset_if(8 * k8 < p.dk, t / (DK / 8) * static_cast<uint32_t>(k_row) + 16 * k8);
  const uint32_t q_at =
      offset_if(8 * k8 < p.dk, t / (DK / 8) * static_cast<uint32_t>(q_row) + 16 * k8);
  const uint32_t v_at =
      offset_if(col0 + 8 * v8 < p.dv, t / (4 * NW) * static_cast<uint32_t>(v_row) + 16 * v8);
  u32x4 kr[KV], qr[kOut ? KV : 1], vr[VV];
  // load i of a thread: K, Q, then V
  constexpr int kLoads = (kOut ? 2 : 1) * KV + VV;
  struct Rows {
    __amdgpu_buffer_rsrc_t k, q, v;
  };
  auto rows = [&](int first) {
    return Rows{rows_of(kb, tok0 + first, k_row, count - first),
                rows_of(qb, tok0 + first, q_row, count - first),
                rows_of(vb, tok0 + first, v_row, count - first)};
  };
  auto load = [&](const Rows& from, int i) {
    if (i < KV) {
      kr[i] = __builtin_amdgcn_raw_buffer_load_b128(
          from.k, k_at + i * kRows * static_cast<uint32_t>(k_row), 0, 0);
    } else if (kOut && i < 2 * KV) {
      qr[i - KV] = __builtin_amdgcn_raw_buffer_load_b128(
          from.q, q_at + (i - KV) * kRows * static_cast<uint32_t>(q_row), 0, 0);
    } else {
      const int j = i - (kOut ? 2 : 1) * KV;
      vr[j] = __builtin_amdgcn_raw_buffer_load_b128(
          from.v, v_at + j * vRows * static_cast<uint32_t>(v_row), 0, 0);
    }
  };

  // ---- decays of a chunk, by the last wave, one chunk ahead of their use
  const bool decays = wave == NW - 1;
  float gr = 0.0f;
  double run_log = 0.0;  // of the segment so far
  const int64_t g_row = 4 * p.g_stride;
  auto load_g = [&](int first) {
    // one decay a head is a row of no length: its buffer ends behind the number
    const int rows = __builtin_amdgcn_readfirstlane(max(min(count - first, kChunk), 0));
    const auto gbuf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(gb)) + (tok0 + first) * g_row, 0,
        rows > 0 ? (rows - 1) * static_cast<int>(g_row) + 4 : 0, kBufferConfig);
    gr = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(
        gbuf, offset_if(lane < rows, lane * static_cast<uint32_t>(g_row)), 0, 0));
  };
  // Returns the chunk's tokens, of those that its rows hold.
  float owed = 0.0f;  // what growing chunks' factors were rounded by, relative
  auto scan_g = [&](int to_buf) {
    const double s = wave_scan_f64(static_cast<double>(gr < kLeastLog ? kLeastLog : gr) * kLog2e);
    double all = __shfl(s, 63, 64);
    int n = kChunk;
    float left = exp2_f32(all - s), whole = exp2_f32(all);
    // (once a chunk's factor has been rounded so, all later ones make up for it)
    if (__builtin_amdgcn_ballot_w64(gr > 0.0f || owed != 0.0f) != 0) {
      const double growth = wave_scan_f64(static_cast<double>(gr > 0.0f ? gr : 0.0f) * kLog2e);
      const uint64_t past = __builtin_amdgcn_ballot_w64(!(growth <= kMostGrowth));
      if (past != 0) {
        n = max(static_cast<int>(__builtin_ctzll(past)), 1);
        all = __shfl(s, n - 1, 64);
        // the rows past the chunk's tokens add nothing to the state
        left = lane < n ? exp2_f32(all - s) : 0.0f;
      }
      // what grows carries the rounding of every factor since: each makes up
      // for those before it
      const double exact = exp2_f64(all) * (1.0 + owed);
      whole = static_cast<float>(exact);
      owed = static_cast<float>(exact - whole) * __builtin_amdgcn_rcpf(whole);
      owed = fabsf(owed) < 0x1p-20f ? owed : 0.0f;  // of 0, of an infinity: nothing
    }
    run_log += all;
    const double coarse = __builtin_rint(s * 64.0) * 0.015625;
    logs[to_buf][lane] = make_float2(static_cast<float>(coarse), static_cast<float>(s - coarse));
    to_end[to_buf][lane] = left;
    from_start[to_buf][lane] = exp2_f32(s) * p.scale;
    chunk_decay[to_buf] = whole;
    chunk_len[to_buf] = n;
    return n;
  };

  auto stage = [&] {
#pragma unroll
    for (int i = 0; i < KV; ++i) {
      const int row = t / (DK / 8) + kRows * i;
      *reinterpret_cast<u32x4*>(kt + row * KS + 8 * k8) = kr[i];
      if constexpr (kOut) *reinterpret_cast<u32x4*>(qt + row * QS + 8 * k8) = qr[i];
    }
#pragma unroll
    for (int i = 0; i < VV; ++i)
      *reinterpret_cast<u32x4*>(vt + (t / (4 * NW) + vRows * i) * VS + 8 * v8) = vr[i];
  };

  int n = kChunk;  // tokens of the chunk
  if (count > 0) {
    const Rows head = rows(0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load(head, i);
    if (decays) {
      load_g(0);
      scan_g(0);
    }
    stage();
    __syncthreads();  // the first chunk is there
    n = __builtin_amdgcn_readfirstlane(chunk_len[0]);
    if (decays) load_g(n);
    // (past the end the buffers are empty and their loads give zeros)
    const Rows next = rows(n);
#pragma unroll
    for (int i = 0; i < (kOut ? KV : kLoads); ++i) load(next, i);
  }
  int buf = 0, next_n = kChunk;
  for (int first = 0; first < count; first += n, n = next_n, buf ^= 1) {
    const bool more = first + n < count;
    const float all = chunk_decay[buf];
    const bool whole = PARTS != 2 || (seg == segs - 1 && keep);
    f32x16 O[2];
    if constexpr (kOut) {
      const Rows soon = rows(first + n);
      // ---- scores of tiles (tokens j, tokens i): (0, 0), (0, 1), (1, 1)
      for (int w = wave; w < 3; w += NW) {
        const int jt = w >> 1, it = (w + 1) >> 1;
        f32x16 A;
#pragma unroll
        for (int r = 0; r < 16; ++r) A[r] = 0.0f;
#pragma unroll
        for (int s = 0; s < DK / 16; ++s) {
          const bf16x8 ka = *reinterpret_cast<const bf16x8*>(kt + (32 * jt + n32) * KS + 16 * s + 8 * half);
          const bf16x8 qa = *reinterpret_cast<const bf16x8*>(qt + (32 * it + n32) * QS + 16 * s + 8 * half);
          A = mfma(ka, qa, A);
        }
        const int i = 32 * it + n32;
        const float2 li = logs[buf][i];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          float y[8];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const int j = 32 * jt + 16 * s + 8 * (r / 4) + 4 * half + r % 4;
            const float2 lj = logs[buf][j];
            float a = A[8 * s + r] * p.scale;
            a *= __builtin_amdgcn_exp2f((li.x - lj.x) + (li.y - lj.y));
            asm("" : "+v"(a));  // all of it before the mask: no branch for each value
            y[r] = j <= i ? a : 0.0f;
          }
          u32x4 part[NP];
          split8<NP>(y, part);
#pragma unroll
          for (int n = 0; n < NP; ++n)
            pt[((w * 2 + s) * NP + n) * 64 + lane] = part[n];
        }
      }
      // ---- S^T Q^T, then its decay from the chunk's start
#pragma unroll
      for (int it = 0; it < 2; ++it)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[it][r] = 0.0f;
#pragma unroll
      for (int e = 0; e < 2 * KT; ++e) {  // 16 channels each; Q and V of the next chunk on the way
#pragma unroll
        for (int i = KV + e * (KV + VV) / (2 * KT); i < KV + (e + 1) * (KV + VV) / (2 * KT); ++i)
          load(soon, i);
        float y[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) y[r] = S[e / 2][8 * (e % 2) + r];
        u32x4 part[NP];
        split8<NP>(y, part);
#pragma unroll
        for (int it = 0; it < 2; ++it) {
          const bf16x8 qa =
              *reinterpret_cast<const bf16x8*>(qt + (32 * it + n32) * QS + 16 * e + 8 * half);
#pragma unroll
          for (int n = 0; n < NP; ++n)
            O[it] = mfma(__builtin_bit_cast(bf16x8, part[n]), qa, O[it]);
        }
      }
#pragma unroll
      for (int it = 0; it < 2; ++it) {
        const float d = from_start[buf][32 * it + n32];
#pragma unroll
        for (int r = 0; r < 16; ++r) O[it][r] *= d;
      }
    }

    // ---- V^T: lane n32 of a wave holds its column, 8 tokens of each 16
    const int tr_row = 4 * half + (lane % 16) / 4, tr_col = 16 * ((lane / 16) & 1);
    bf16x8 va[4];
#pragma unroll
    for (int s = 0; s < 4; ++s)
      va[s] = read_columns8(vt + (16 * s + tr_row) * VS + 32 * wave + tr_col + 4 * (lane & 3),
                            8 * VS);
    // ---- S = exp(L_C) S + K^T (D V)
    // the state's row order: the quads of 16 channels as 0 2 1 3
    const int k_quad = 4 * (((lane & 1) << 1) | ((lane >> 1) & 1));
#pragma unroll
    for (int c = 0; c < KT; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) S[c][r] *= all;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const float4 d0 = *reinterpret_cast<const float4*>(to_end[buf] + 16 * s + 4 * half);
      const float4 d1 = *reinterpret_cast<const float4*>(to_end[buf] + 16 * s + 4 * half + 8);
      const u32x4 w = __builtin_bit_cast(u32x4, va[s]);
      float y[8] = {bf16_lo(w[0]) * d0.x, bf16_hi(w[0]) * d0.y, bf16_lo(w[1]) * d0.z,
                    bf16_hi(w[1]) * d0.w, bf16_lo(w[2]) * d1.x, bf16_hi(w[2]) * d1.y,
                    bf16_lo(w[3]) * d1.z, bf16_hi(w[3]) * d1.w};
      auto k_columns = [&](int c) {
        return read_columns8(kt + (16 * s + tr_row) * KS + 32 * c + tr_col + k_quad, 8 * KS);
      };
      u32x4 part[2];
      split8<2>(y, part);
#pragma unroll
      for (int c = 0; c < KT; ++c) {
        const bf16x8 ka = k_columns(c);
#pragma unroll
        for (int n = 0; n < 2; ++n) S[c] = mfma(ka, __builtin_bit_cast(bf16x8, part[n]), S[c]);
      }
      if (whole) {
        u32x4 third;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          third[j] = pack_bf16x2(y[2 * j] - bf16_lo(part[1][j]), y[2 * j + 1] - bf16_hi(part[1][j]));
#pragma unroll
        for (int c = 0; c < KT; ++c)
          S[c] = mfma(k_columns(c), __builtin_bit_cast(bf16x8, third), S[c]);
      }
    }

    // ---- the next decays; then P is there, and K, Q and V have been read
    if (decays && more) load_g(first + n + scan_g(buf ^ 1));
    __syncthreads();
    if (more) stage();
    next_n = more ? __builtin_amdgcn_readfirstlane(chunk_len[buf ^ 1]) : kChunk;
    const Rows ahead = rows(first + n + next_n);
    if constexpr (!kOut) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) load(ahead, i);
    } else {
      // ---- O += V^T P^T, the loads of the chunk after next between
#pragma unroll
      for (int m = 0; m < 6 * NP; ++m) {
        const int x = m / NP, n = m % NP;
        const int it = x < 2 ? 0 : 1, s = x < 2 ? x : x - 2;  // tile (s / 2, it)
        const int w = (s >> 1) + it;
        O[it] = mfma(va[s], __builtin_bit_cast(bf16x8, pt[((w * 2 + (s & 1)) * NP + n) * 64 + lane]),
                     O[it]);
#pragma unroll
        for (int i = m * KV / (6 * NP); i < (m + 1) * KV / (6 * NP); ++i) load(ahead, i);
      }
      const auto obuf = rows_of(static_cast<uint8_t*>(p.o) + (static_cast<int64_t>(h) * p.dv + col0) *
                                                                 (p.o_bf16 ? 2 : 4),
                                tok0 + first, o_row, min(count - first, n));
#pragma unroll
      for (int it = 0; it < 2; ++it) {
        const uint32_t row_at = (32 * it + n32) * static_cast<uint32_t>(o_row);
        const f32x16& y = O[it];
        if (p.o_bf16) {
          // a lane's four columns and those of the lane 32 on make 16 bytes
#pragma unroll
          for (int r4 = 0; r4 < 4; r4 += 2) {
            const int c = 32 * wave + 8 * (r4 + half);
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const auto x = __builtin_amdgcn_permlane32_swap(
                  pack_bf16x2(y[4 * r4 + 2 * e], y[4 * r4 + 2 * e + 1]),
                  pack_bf16x2(y[4 * r4 + 4 + 2 * e], y[4 * r4 + 5 + 2 * e]), false, false);
              w[e] = x[0];
              w[2 + e] = x[1];
            }
            __builtin_amdgcn_raw_buffer_store_b128(
                w, obuf, col0 + c < p.dv ? row_at + 2 * c : kNowhere, 0, 0);
          }
        } else {
#pragma unroll
          for (int r4 = 0; r4 < 4; ++r4) {
            const int c = 32 * wave + 8 * r4 + 4 * half;
            const u32x4 w = {__float_as_uint(y[4 * r4]), __float_as_uint(y[4 * r4 + 1]),
                             __float_as_uint(y[4 * r4 + 2]), __float_as_uint(y[4 * r4 + 3])};
            __builtin_amdgcn_raw_buffer_store_b128(
                w, obuf, col0 + c < p.dv ? row_at + 4 * c : kNowhere, 0, 0);
          }
        }
      }
    }
    if (more) __syncthreads();  // the next chunk is there
  }

  // ---- the state after the last token
  float* dst = nullptr;
  if constexpr (kOut) {
    if (seg == segs - 1 && keep)
      dst = reinterpret_cast<float*>(p.layer_base + to * p.slot_stride + h * p.tile_stride);
  } else {
    dst = pp.seg_states + tile + seg * tile_step;
    if (decays && col0 == 0) {
      const double whole = floor(fmin(fmax(run_log, -4096.0), 4096.0));
      pp.seg_decays[(static_cast<size_t>(b) * pp.segments + seg) * p.HV + h] = make_float2(
          __builtin_amdgcn_exp2f(static_cast<float>(run_log - whole)), static_cast<float>(whole));
    }
  }
  if (dst) {
    const auto sbuf = state_buffer(dst, p);
#pragma unroll
    for (int c = 0; c < KT; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(S[c][r]), sbuf,
                                              s_at + s_row * (32 * c + 16 * (r / 8) + r % 8), 0, 0);
  }
}

// The state before each segment of a request, in the place of what the
// segment adds: X_0 = S_in, X_{s+1} = decay_s X_s + added_s.
__global__ __launch_bounds__(256) void prompt_states(const PromptParams pp) {
  const LinearParams& p = pp.l;
  const int h = blockIdx.x, b = blockIdx.y;
  int start, len;
  request_range(pp, b, start, len);
  const int segs = segments_of(pp, len);
  const int from = p.slot_in[b];
  const bool old = from >= 0 && from < p.num_slots;
  const int at = (blockIdx.z * 256 + threadIdx.x) * 4;
  if (segs < 2 || at >= p.dk * p.dv || (!old && from != DAMP_SLOT_ZERO)) return;
  float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (old)
    x = *reinterpret_cast<const float4*>(p.layer_base + from * p.slot_stride + h * p.tile_stride +
                                         static_cast<size_t>(at) * 4);
  const size_t step = static_cast<size_t>(p.HV) * p.dk * p.dv;
  float* state = pp.seg_states + static_cast<size_t>(b) * pp.segments * step +
                 static_cast<size_t>(h) * p.dk * p.dv + at;
  const float2* decay = pp.seg_decays + static_cast<size_t>(b) * pp.segments * p.HV + h;
  for (int s = 0; s < segs; ++s) {
    float4* place = reinterpret_cast<float4*>(state + s * step);
    const bool last = s == segs - 1;
    const float4 add = last ? x : *place;
    const float2 d = last ? make_float2(0.0f, 0.0f) : decay[static_cast<size_t>(s) * p.HV];
    const int e = static_cast<int>(d.y);
    *place = x;
    x.x = fmaf(d.x, ldexpf(x.x, e), add.x);
    x.y = fmaf(d.x, ldexpf(x.y, e), add.y);
    x.z = fmaf(d.x, ldexpf(x.z, e), add.z);
    x.w = fmaf(d.x, ldexpf(x.w, e), add.w);
  }
}

// Tokens of a segment. The lengths are on the device; the host knows that B
// requests share n_tokens and none is longer than max_len. Segments are as
// long as leave every CU its two workgroups, at least kLeastSegment tokens (a
// request of up to kUncut is not cut: the two other launches would cost more),
// and no shorter than the finest cut, which goes by B and max_len alone. More
// tokens never make shorter segments, so the workspace for n_tokens = max_len,
// the least there can be, has room for all of a B and max_len. Measured on 256
// CUs, in us, with kWorkgroups = 512 / 1024 / 2048 / 4096: one request of 32768
// tokens and 32 heads 373 / 389 / 418 / 465; eleven of 0 to 4096 tokens 152 /
// 150 / 184 / 185; sixteen of 2000 and 64 columns 151 / 175 / 185 / 203. One of
// 200 tokens whole 19, in two 25; one of 500 in segments of 128 / 256: 27 / 37.
constexpr int kWorkgroups = 512;
constexpr int kMostWorkgroups = 4096;
constexpr int kLeastSegment = 128, kUncut = 256;

struct Split {
  int32_t seg_len, segments;
};

Split split_of(const damp_pool* pool, int32_t B, int64_t n_tokens, int32_t max_len) {
  const int64_t heads = static_cast<int64_t>(pool->num_v_heads) * ((pool->layout.d_v + 127) / 128);
  const int64_t longest = (static_cast<int64_t>(max_len) + kChunk - 1) / kChunk;
  const int64_t finest = (longest * B * heads + kMostWorkgroups - 1) / kMostWorkgroups;
  const int64_t wanted = ((n_tokens / kChunk + B) * heads + kWorkgroups - 1) / kWorkgroups;
  const int64_t seg = std::min<int64_t>(
      std::max<int64_t>({finest * kChunk, wanted * kChunk,
                         max_len <= kUncut ? kUncut : kLeastSegment}),
      1 << 30);
  return {static_cast<int32_t>(seg),
          static_cast<int32_t>(std::max<int64_t>((max_len + seg - 1) / seg, 1))};
}

size_t workspace_bytes_of(const damp_pool* pool, int32_t B, const Split& s) {
  if (s.segments < 2) return 0;
  const size_t tiles = static_cast<size_t>(B) * s.segments * pool->num_v_heads;
  return tiles * (static_cast<size_t>(pool->layout.d_k) * pool->layout.d_v * sizeof(float) + sizeof(float2));
}

template <int DK, int NW>
void launch(const PromptParams& p, int B, hipStream_t s) {
  const int nx = p.l.HV * ((p.l.dv + 32 * NW - 1) / (32 * NW));
  if (p.segments > 1) {
    hipLaunchKernelGGL((prompt_chunks<DK, NW, 0>), dim3(nx, B, p.segments - 1), dim3(64 * NW), 0, s,
                       p);
    hipLaunchKernelGGL(prompt_states, dim3(p.l.HV, B, (p.l.dk * p.l.dv + 1023) / 1024), dim3(256),
                       0, s, p);
  }
  if (p.l.o_bf16)
    hipLaunchKernelGGL((prompt_chunks<DK, NW, 2>), dim3(nx, B, p.segments), dim3(64 * NW), 0, s, p);
  else
    hipLaunchKernelGGL((prompt_chunks<DK, NW, 3>), dim3(nx, B, p.segments), dim3(64 * NW), 0, s, p);
}

// Two waves where the head has no columns for four: 16 requests of 2000 tokens,
// 32 heads of 64, take 151 us against 155, with keys of 128 channels 194 against
// 218.
template <int DK>
void launch(const PromptParams& p, int B, hipStream_t s) {
  if (p.l.dv <= 64) launch<DK, 2>(p, B, s);
  else launch<DK, 4>(p, B, s);
}

}  // namespace
}  // namespace damp

extern "C" {

size_t damp_linear_prefill_workspace_bytes(const damp_pool* pool, int32_t B, int32_t max_len) {
  using namespace damp;
  if (check_pool(pool) != DAMP_OK || B <= 0 || B > 65535 || max_len < 0) return 0;
  return workspace_bytes_of(pool, B, split_of(pool, B, max_len, max_len));
}

damp_status damp_linear_prefill(const damp_pool* pool, int32_t layer, const int32_t* slot_in,
                                const int32_t* slot_out, int32_t B, int64_t n_tokens,
                                int32_t max_len, const int32_t* seq_start, const int32_t* seq_len,
                                int32_t num_k_heads, const uint16_t* q, int64_t q_stride,
                                const uint16_t* k, int64_t k_stride, const uint16_t* v,
                                int64_t v_stride, const float* g, int64_t g_stride, float scale,
                                void* o, int32_t o_dtype, void* workspace, size_t workspace_bytes,
                                void* stream) {
  using namespace damp;
  clear_error();
  const char* name = "damp_linear_prefill";
  hipStream_t s = as_stream(stream);
  if (n_tokens < 0 || n_tokens > INT32_MAX)
    return fail(DAMP_ERR_INVALID_ARG, "%s: n_tokens = %lld outside [0, 2^31)", name,
                static_cast<long long>(n_tokens));
  if (max_len < 0 || max_len > n_tokens)
    return fail(DAMP_ERR_INVALID_ARG, "%s: max_len = %d outside [0, n_tokens = %lld]", name,
                max_len, static_cast<long long>(n_tokens));
  if (B > 0 && (!seq_start || !seq_len))
    return fail(DAMP_ERR_INVALID_ARG, "%s: seq_start or seq_len is NULL", name);
  PromptParams p;
  damp_status st = linear_params(name, pool, layer, slot_in, slot_out, B, n_tokens, num_k_heads, q,
                                 q_stride, k, k_stride, v, v_stride, g, g_stride, scale, o,
                                 o_dtype, s, &p.l);
  if (st != DAMP_OK || B == 0) return st;
  // a chunk's rows are addressed with 31 bits
  constexpr int64_t kMost = (int64_t{1} << 31) / kChunk / 4 - 8;
  if (q_stride > 2 * kMost || k_stride > 2 * kMost || v_stride > 2 * kMost || g_stride > kMost ||
      static_cast<int64_t>(p.l.HV) * p.l.dv > kMost)
    return fail(DAMP_ERR_INVALID_ARG, "%s: a token's row is too long", name);
  const Split split = split_of(pool, B, n_tokens, max_len);
  const size_t need = workspace_bytes_of(pool, B, split_of(pool, B, max_len, max_len));
  if (need > 0 && (!workspace || workspace_bytes < need ||
                   reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
    return fail(DAMP_ERR_INVALID_ARG, "%s: needs %zu bytes of 16-byte aligned workspace", name,
                need);
  p.seq_start = seq_start;
  p.seq_len = seq_len;
  p.n_tokens = static_cast<int32_t>(n_tokens);
  p.max_len = max_len;
  p.seg_len = split.seg_len;
  p.segments = split.segments;
  p.seg_states = static_cast<float*>(workspace);
  p.seg_decays = reinterpret_cast<float2*>(
      p.seg_states + static_cast<size_t>(B) * split.segments * p.l.HV * p.l.dk * p.l.dv);
  if (p.l.dk <= 64) launch<64>(p, B, s);
  else if (p.l.dk <= 128) launch<128>(p, B, s);
  else launch<256>(p, B, s);
  return check_launch(name);
}

}  // extern "C"

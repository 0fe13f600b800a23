// Linear attention with one decay a head, one token per request: the checks
// that both entry points share, and the decode kernel.
//
//   S' = exp(g) S + k v^T,   o = scale * S'^T q
//
// The state is read once and written once (8 d_k d_v bytes a head against
// 4 d_k d_v operations), so memory bounds the kernel: 196 us at 256 requests
// of 32 heads of 128 x 128, 5.5 TB/s, where a large copy reaches 5.1. A
// workgroup owns W columns of one (request, value head) tile: the columns of a
// state do not depend on each other, the rows meet only in o. Thread t holds
// four neighbouring columns of the rows t / (W / 4) + i RG, up to 128 rows in
// flight before the first is used; o is summed over rows by lane exchanges and
// one LDS pass over the four waves.
#include "device.hpp"
#include "linear.hpp"

namespace damp {

namespace {

// With DAMP_CHECK_SLOTS set: a slot that one request writes is written and
// read by no other.
damp_status check_linear_slots(const char* name, const damp_pool* pool, const int32_t* slot_in,
                               const int32_t* slot_out, int32_t B, hipStream_t stream) {
  damp_status st = debug_check_slots(pool, slot_out, B, stream, name);
  if (st != DAMP_OK || slot_in == slot_out || !slots_checked()) return st;
  return check_slots_apart(pool, slot_in, B, slot_out, B, true, stream, name);
}

}  // namespace

damp_status linear_params(const char* name, const damp_pool* pool, int32_t layer,
                          const int32_t* slot_in, const int32_t* slot_out, int32_t B, int64_t rows,
                          int32_t num_k_heads, const uint16_t* q, int64_t q_stride,
                          const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride,
                          const float* g, int64_t g_stride, float scale, void* o, int32_t o_dtype,
                          hipStream_t stream, LinearParams* p) {
  damp_status st = check_pool(pool);
  if (st != DAMP_OK) return st;
  const int32_t dk = pool->layout.d_k, dv = pool->layout.d_v, HV = pool->num_v_heads;
  if (layer < 0 || layer >= pool->num_layers)
    return fail(DAMP_ERR_INVALID_ARG, "%s: layer %d outside [0, %d)", name, layer,
                pool->num_layers);
  if (B < 0 || B > 65535) return fail(DAMP_ERR_INVALID_ARG, "%s: B = %d outside [0, 65535]", name, B);
  if (num_k_heads <= 0 || HV % num_k_heads != 0)
    return fail(DAMP_ERR_INVALID_ARG, "%s: num_v_heads %d is not a multiple of num_k_heads %d",
                name, HV, num_k_heads);
  if (o_dtype != DAMP_DT_FP32 && o_dtype != DAMP_DT_BF16)
    return fail(DAMP_ERR_INVALID_ARG, "%s: o_dtype must be FP32 or BF16", name);
  if (pool->layout.kind != DAMP_STATE_FP32 || dk % 8 != 0 || dv % 8 != 0 || dk > 256 || dv > 256)
    return fail(DAMP_ERR_UNSUPPORTED,
                "%s: needs an FP32 pool with d_k and d_v multiples of 8 up to 256", name);
  if (reinterpret_cast<uintptr_t>(pool->base) % 16 != 0)
    return fail(DAMP_ERR_INVALID_ARG, "%s: pool base is not 16-byte aligned", name);
  if (B == 0) return DAMP_OK;
  if (!slot_in) return fail(DAMP_ERR_INVALID_ARG, "%s: slot_in is NULL", name);
  if (rows > 0) {
    if (!q || !k || !v || !g || !o)
      return fail(DAMP_ERR_INVALID_ARG, "%s: a required pointer is NULL", name);
    const uintptr_t at = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k) |
                         reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(o);
    if (at % 16 != 0 || reinterpret_cast<uintptr_t>(g) % 4 != 0)
      return fail(DAMP_ERR_INVALID_ARG, "%s: q, k, v and o must be 16-byte aligned, g 4-byte", name);
    const int64_t kq = static_cast<int64_t>(num_k_heads) * dk, vo = static_cast<int64_t>(HV) * dv;
    if (q_stride < kq || k_stride < kq || v_stride < vo || (q_stride | k_stride | v_stride) % 8 != 0)
      return fail(DAMP_ERR_INVALID_ARG,
                  "%s: token distances of q, k, v must be multiples of 8 and hold a token's heads",
                  name);
    if (g_stride != 0 && g_stride < HV)
      return fail(DAMP_ERR_INVALID_ARG, "%s: g_stride %lld is neither 0 nor >= %d", name,
                  static_cast<long long>(g_stride), HV);
    // byte offsets are 64-bit in the kernels
    const int64_t most = INT64_MAX / 4 / rows;
    if (q_stride > most || k_stride > most || v_stride > most || g_stride > most || vo > most)
      return fail(DAMP_ERR_INVALID_ARG, "%s: operands span more than 2^63 bytes", name);
  }
  if (!slot_out) slot_out = slot_in;
  st = check_linear_slots(name, pool, slot_in, slot_out, B, stream);
  if (st != DAMP_OK) return st;
  p->layer_base = layer_base(pool, layer);
  p->tile_stride = pool->tile_stride;
  p->slot_stride = pool->tile_stride * static_cast<uint64_t>(HV);
  p->slot_in = slot_in;
  p->slot_out = slot_out;
  p->q = q;
  p->k = k;
  p->v = v;
  p->g = g;
  p->o = o;
  p->q_stride = q_stride;
  p->k_stride = k_stride;
  p->v_stride = v_stride;
  p->g_stride = g_stride;
  p->scale = scale;
  p->num_slots = pool->num_slots;
  p->HK = num_k_heads;
  p->HV = HV;
  p->dk = dk;
  p->dv = dv;
  p->o_bf16 = o_dtype == DAMP_DT_BF16;
  return DAMP_OK;
}

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kBufferConfig = 0x00020000;  // raw 32-bit buffer (gfx9 family)

template <int W, bool STREAM>
__global__ __launch_bounds__(256) void linear_update_kernel(const LinearParams p) {
  constexpr int C4 = W / 4;      // lanes of a row
  constexpr int RG = 256 / C4;   // rows side by side
  constexpr int U = 128 / RG;    // rows of a thread in one pass over 128
  constexpr int kLoad = STREAM ? 2 : 0;        // non-temporal
  constexpr int kStore = STREAM ? 2 | 16 : 0;  // non-temporal, device scope
  __shared__ float2 kq[256];
  __shared__ float red[4][W];

  const int t = threadIdx.x;
  const int h = blockIdx.x, b = blockIdx.y;
  const int cg = t % C4, rg = t / C4;
  const int col = blockIdx.z * W + 4 * cg;
  const bool in_row = col < p.dv;
  const int hk = h / (p.HV / p.HK);
  // in scalar registers, as what buffers are described by has to be
  const int from = __builtin_amdgcn_readfirstlane(p.slot_in[b]);
  const int to = __builtin_amdgcn_readfirstlane(p.slot_out[b]);
  const bool old = from >= 0 && from < p.num_slots;
  const bool keep = to >= 0 && to < p.num_slots;
  const size_t o_at = (static_cast<size_t>(b) * p.HV + h) * p.dv;

  if (!old && from != DAMP_SLOT_ZERO) {  // padded request
    const int c = blockIdx.z * W + t;
    if (t < W && c < p.dv) {
      if (p.o_bf16) static_cast<uint16_t*>(p.o)[o_at + c] = 0;
      else static_cast<float*>(p.o)[o_at + c] = 0.0f;
    }
    return;
  }
  // one tile as a buffer: rows and columns past the head are past its end, and
  // so is all of a state that is not read or kept
  const int bytes = p.dk * p.dv * 4;
  const auto src = __builtin_amdgcn_make_buffer_rsrc(
      p.layer_base + (old ? from : 0) * p.slot_stride + h * p.tile_stride, 0, old ? bytes : 0,
      kBufferConfig);
  const auto dst = __builtin_amdgcn_make_buffer_rsrc(
      p.layer_base + (keep ? to : 0) * p.slot_stride + h * p.tile_stride, 0, keep ? bytes : 0,
      kBufferConfig);
  const uint32_t row = 4 * p.dv;
  const uint32_t at = in_row ? 4 * col : 0x80000000u;

  // the operands
  const float g = p.g[b * p.g_stride + h];
  uint16_t k_w = 0, q_w = 0;
  if (t < p.dk) {
    k_w = p.k[b * p.k_stride + hk * p.dk + t];
    q_w = p.q[b * p.q_stride + hk * p.dk + t];
  }
  float vv[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (in_row) {
    const uint2 w = *reinterpret_cast<const uint2*>(p.v + b * p.v_stride + h * p.dv + col);
    vv[0] = bf16_lo(w.x);
    vv[1] = bf16_hi(w.x);
    vv[2] = bf16_lo(w.y);
    vv[3] = bf16_hi(w.y);
  }

  float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  float a = 0.0f;
  for (int r0 = 0; r0 < p.dk; r0 += 128) {
    u32x4 x[U];
#pragma unroll
    for (int i = 0; i < U; ++i)
      x[i] = __builtin_amdgcn_raw_buffer_load_b128(src, at + (r0 + rg + RG * i) * row, 0, kLoad);
    if (r0 == 0) {  // behind the first loads of the state
      kq[t] = make_float2(bf16_to_f32(k_w), bf16_to_f32(q_w));
      a = expf(g);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int r = r0 + rg + RG * i;
      if (r >= p.dk) break;
      const float2 w = kq[r];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float y = fmaf(w.x, vv[j], a * __uint_as_float(x[i][j]));
        acc[j] = fmaf(w.y, y, acc[j]);
        x[i][j] = __float_as_uint(y);
      }
      __builtin_amdgcn_raw_buffer_store_b128(x[i], dst, at + r * row, 0, kStore);
    }
  }
#pragma unroll
  for (int m = C4; m < 64; m <<= 1)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], m, 64);
  if ((t & 63) < C4)
#pragma unroll
    for (int j = 0; j < 4; ++j) red[t >> 6][4 * cg + j] = acc[j];
  __syncthreads();
  const int c = blockIdx.z * W + t;
  if (t < W && c < p.dv) {
    const float o = p.scale * ((red[0][t] + red[1][t]) + (red[2][t] + red[3][t]));
    if (p.o_bf16) static_cast<uint16_t*>(p.o)[o_at + c] = f32_to_bf16(o);
    else static_cast<float*>(p.o)[o_at + c] = o;
  }
}

template <int W, bool STREAM>
void launch(const LinearParams& p, int B, hipStream_t s) {
  hipLaunchKernelGGL((linear_update_kernel<W, STREAM>), dim3(p.HV, B, (p.dv + W - 1) / W),
                     dim3(256), 0, s, p);
}

// Fewer tiles than CUs: 32 columns each, for the shorter chain of loads (one
// request of 32 heads: 3.4 us against 4.0 with 128). Otherwise the whole row,
// up to 128 columns. States of 128 MB and more whose rows are wider than 32
// columns pass by the caches (256 requests: 196 against 211 us; 64 requests, 134
// MB: 50.9 against 53.5); smaller ones may still be there from the step before
// (32 requests: 21.7 us against 26.6).
constexpr int64_t kFewTiles = 256;
constexpr int64_t kStreamBytes = int64_t{128} << 20;

void launch(const LinearParams& p, int B, hipStream_t s) {
  const int64_t tiles = static_cast<int64_t>(B) * p.HV;
  const bool stream = tiles * p.dk * p.dv * 4 >= kStreamBytes;
  if (p.dv <= 32 || tiles < kFewTiles) launch<32, false>(p, B, s);
  else if (p.dv <= 64 && stream) launch<64, true>(p, B, s);
  else if (p.dv <= 64) launch<64, false>(p, B, s);
  else if (stream) launch<128, true>(p, B, s);
  else launch<128, false>(p, B, s);
}

}  // namespace
}  // namespace damp

extern "C" damp_status damp_linear_update(const damp_pool* pool, int32_t layer,
                                          const int32_t* slot_in, const int32_t* slot_out,
                                          int32_t B, int32_t num_k_heads, const uint16_t* q,
                                          int64_t q_stride, const uint16_t* k, int64_t k_stride,
                                          const uint16_t* v, int64_t v_stride, const float* g,
                                          int64_t g_stride, float scale, void* o, int32_t o_dtype,
                                          void* stream) {
  using namespace damp;
  clear_error();
  const char* name = "damp_linear_update";
  hipStream_t s = as_stream(stream);
  LinearParams p;
  damp_status st = linear_params(name, pool, layer, slot_in, slot_out, B, B, num_k_heads, q,
                                 q_stride, k, k_stride, v, v_stride, g, g_stride, scale, o,
                                 o_dtype, s, &p);
  if (st != DAMP_OK || B == 0) return st;
  launch(p, B, s);
  return check_launch(name);
}

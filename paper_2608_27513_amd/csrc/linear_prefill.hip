// Linear attention with one decay a head over packed prompts.
#include "device.hpp"
#include "linear.hpp"

namespace damp {
namespace {

struct PromptParams {
  LinearParams l;
  const int32_t* seq_start;
  const int32_t* seq_len;
  int32_t n_tokens;
  int32_t max_len;
};

// First token and length of request b, within the token axis and max_len.
__device__ __forceinline__ void request_range(const PromptParams& p, int b, int& start, int& len) {
  start = p.seq_start[b];
  const bool inside = start >= 0 && start <= p.n_tokens;
  len = inside ? min(min(p.seq_len[b], p.max_len), p.n_tokens - start) : 0;
  len = max(len, 0);
  if (!inside) start = 0;
}

// The recurrence token by token: a workgroup owns 32 columns of one (request,
// value head) state in registers, 8 lanes a row.
__global__ __launch_bounds__(256) void prompt_recurrent(const PromptParams pp) {
  const LinearParams& p = pp.l;
  __shared__ float red[2][4][32];
  const int t = threadIdx.x;
  const int h = blockIdx.x, b = blockIdx.y;
  const int cg = t % 8, rg = t / 8;
  const int col = blockIdx.z * 32 + 4 * cg;
  const bool in_row = col < p.dv;
  const int hk = h / (p.HV / p.HK);
  const int from = p.slot_in[b], to = p.slot_out[b];
  const bool old = from >= 0 && from < p.num_slots;
  const bool keep = to >= 0 && to < p.num_slots;
  const bool padded = !old && from != DAMP_SLOT_ZERO;
  int start, len;
  request_range(pp, b, start, len);

  const float* src = reinterpret_cast<const float*>(
      p.layer_base + (old ? from : 0) * p.slot_stride + h * p.tile_stride);
  float x[8][4];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = rg + 32 * i;
    float4 w = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (old && in_row && r < p.dk)
      w = *reinterpret_cast<const float4*>(src + static_cast<size_t>(r) * p.dv + col);
    x[i][0] = w.x;
    x[i][1] = w.y;
    x[i][2] = w.z;
    x[i][3] = w.w;
  }
  for (int tok = 0; tok < len; ++tok) {
    const int64_t at = static_cast<int64_t>(start) + tok;
    const float a = expf(p.g[at * p.g_stride + h]);
    float vv[4] = {0.0f, 0.0f, 0.0f, 0.0f}, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (in_row)
#pragma unroll
      for (int j = 0; j < 4; ++j) vv[j] = bf16_to_f32(p.v[at * p.v_stride + h * p.dv + col + j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = rg + 32 * i;
      if (r >= p.dk) break;
      const float kr = bf16_to_f32(p.k[at * p.k_stride + hk * p.dk + r]);
      const float qr = bf16_to_f32(p.q[at * p.q_stride + hk * p.dk + r]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[i][j] = fmaf(kr, vv[j], a * x[i][j]);
        acc[j] = fmaf(qr, x[i][j], acc[j]);
      }
    }
#pragma unroll
    for (int m = 8; m < 64; m <<= 1)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += __shfl_xor(acc[j], m, 64);
    if ((t & 63) < 8)
#pragma unroll
      for (int j = 0; j < 4; ++j) red[tok & 1][t >> 6][4 * cg + j] = acc[j];
    __syncthreads();
    const int c = blockIdx.z * 32 + t;
    if (t < 32 && c < p.dv) {
      const float(&w)[4][32] = red[tok & 1];
      const float o = padded ? 0.0f : p.scale * ((w[0][t] + w[1][t]) + (w[2][t] + w[3][t]));
      const size_t o_at = (static_cast<size_t>(at) * p.HV + h) * p.dv + c;
      if (p.o_bf16) static_cast<uint16_t*>(p.o)[o_at] = f32_to_bf16(o);
      else static_cast<float*>(p.o)[o_at] = o;
    }
  }
  if (padded || !keep || !in_row) return;
  float* dst = reinterpret_cast<float*>(p.layer_base + to * p.slot_stride + h * p.tile_stride);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int r = rg + 32 * i;
    if (r < p.dk)
      *reinterpret_cast<float4*>(dst + static_cast<size_t>(r) * p.dv + col) =
          make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
  }
}

}  // namespace
}  // namespace damp

extern "C" {

size_t damp_linear_prefill_workspace_bytes(const damp_pool* pool, int32_t B, int32_t max_len) {
  (void)pool;
  (void)B;
  (void)max_len;
  return 0;
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
  const size_t need = damp_linear_prefill_workspace_bytes(pool, B, max_len);
  if (need > 0 && (!workspace || workspace_bytes < need ||
                   reinterpret_cast<uintptr_t>(workspace) % 16 != 0))
    return fail(DAMP_ERR_INVALID_ARG, "%s: needs %zu bytes of 16-byte aligned workspace", name,
                need);
  p.seq_start = seq_start;
  p.seq_len = seq_len;
  p.n_tokens = static_cast<int32_t>(n_tokens);
  p.max_len = max_len;
  hipLaunchKernelGGL(prompt_recurrent, dim3(p.l.HV, B, (p.l.dv + 31) / 32), dim3(256), 0, s, p);
  return check_launch(name);
}

}  // extern "C"

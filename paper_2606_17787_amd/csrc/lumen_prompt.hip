// Causal attention over packed sequences for MI355X (gfx950), as specified in
// include/lumen_attn.h (lumen_attn_prompt).

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "lumen_attn.h"
#include "lumen_attn_common.h"

namespace {

using namespace lumen_attn_detail;

struct PromptArgs {
  Rows q, k, v;
  const int32_t *cu_q, *cu_k;
  int32_t num_seqs;
  int64_t num_q, num_k;
  int32_t q_heads, kv_heads;
  float scale_log2;  // scale * log2(e)
  uint16_t *out;
  int32_t *status;
};

// One wavefront per (query, head), a key at a time.
template <int D, bool kBf16>
__global__ __launch_bounds__(kWave) void prompt_kernel(PromptArgs a) {
  constexpr int kE = D / 64;
  const int s = blockIdx.y, lane = threadIdx.x;
  const int64_t q0 = a.cu_q[s], q1 = a.cu_q[s + 1];
  const int64_t k0 = a.cu_k[s], k1 = a.cu_k[s + 1];
  if (q0 < 0 || q1 < q0 || q1 > a.num_q || k0 < 0 || k1 < k0 || k1 > a.num_k) {
    record_wave(a.status, LUMEN_ERR_RANGE);
    return;
  }
  const int64_t items = (q1 - q0) * a.q_heads;
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
    const int64_t n = i / a.q_heads;
    const int hq = int(i - n * a.q_heads), h = hq / (a.q_heads / a.kv_heads);
    const uint16_t *q = a.q.base + (q0 + n) * a.q.token + hq * a.q.head;
    float x[kE], o[kE];
    for (int e = 0; e < kE; ++e) {
      x[e] = value<kBf16>(q[lane * kE + e]) * a.scale_log2;
      o[e] = 0.0f;
    }
    float m = -INFINITY, l = 0.0f;
    const int64_t last = n + (k1 - k0) - (q1 - q0);
    for (int64_t j = 0; j <= last; ++j) {
      const uint16_t *k = a.k.base + (k0 + j) * a.k.token + h * a.k.head;
      const uint16_t *v = a.v.base + (k0 + j) * a.v.token + h * a.v.head;
      float d = 0.0f;
      for (int e = 0; e < kE; ++e) d += x[e] * value<kBf16>(k[lane * kE + e]);
      for (int b = 1; b < kWave; b <<= 1) d += __shfl_xor(d, b);
      const float mn = fmaxf(m, d);
      const float c = exp2f(m - mn), p = exp2f(d - mn);
      m = mn;
      l = l * c + p;
      for (int e = 0; e < kE; ++e)
        o[e] = o[e] * c + p * value<kBf16>(v[lane * kE + e]);
    }
    uint16_t *out = a.out + ((q0 + n) * a.q_heads + hq) * D;
    for (int e = 0; e < kE; ++e)
      out[lane * kE + e] = rounded<kBf16>(last >= 0 ? o[e] / l : 0.0f);
  }
}

}  // namespace

extern "C" int lumen_attn_prompt(
    const lumen_attn_rows *q, const lumen_attn_rows *k,
    const lumen_attn_rows *v, int32_t dtype, const int32_t *d_cu_q,
    const int32_t *d_cu_k, int32_t num_seqs, int64_t num_q_tokens,
    int64_t num_k_tokens, int32_t num_q_heads, int32_t num_kv_heads,
    int32_t head_dim, float scale, void *d_out, int32_t *d_status,
    lumen_stream_t stream) {
  int st = check_dtype(dtype);
  if (st != LUMEN_OK) return st;
  if (num_seqs < 0 || num_q_tokens < 0 || num_k_tokens < 0 || num_q_heads < 1 ||
      num_kv_heads < 1 || num_q_heads % num_kv_heads || !(scale > 0.0f) ||
      !(scale < INFINITY) || (!d_cu_k && num_q_tokens != num_k_tokens))
    return LUMEN_ERR_INVALID_ARG;
  if ((head_dim != 64 && head_dim != 128) || num_q_tokens > INT32_MAX ||
      num_k_tokens > INT32_MAX)
    return LUMEN_ERR_UNSUPPORTED;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if (num_seqs > LUMEN_ATTN_MAX_REQS) return LUMEN_ERR_TOO_MANY;
  if ((st = check_rows(q, num_q_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(k, num_k_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(v, num_k_tokens)) != LUMEN_OK) return st;
  if (num_seqs > 0 && !d_cu_q) return LUMEN_ERR_INVALID_ARG;
  if (num_q_tokens > 0 && !d_out) return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_out, 16) || !aligned(d_cu_q, 4) || !aligned(d_cu_k, 4))
    return LUMEN_ERR_MISALIGNED;
  if (num_seqs == 0) return LUMEN_OK;
  (void)hipGetLastError();
  PromptArgs a{rows_of(q, 0), rows_of(k, 0), rows_of(v, 0), d_cu_q,
               d_cu_k ? d_cu_k : d_cu_q, num_seqs, num_q_tokens, num_k_tokens,
               num_q_heads, num_kv_heads, scale * 1.44269504088896341f,
               static_cast<uint16_t *>(d_out), d_status};
  const bool bf = dtype == LUMEN_ATTN_BF16;
  void (*kernel)(PromptArgs) =
      head_dim == 64 ? (bf ? prompt_kernel<64, true> : prompt_kernel<64, false>)
                     : (bf ? prompt_kernel<128, true> : prompt_kernel<128, false>);
  int64_t blocks = num_q_tokens * num_q_heads;
  if (blocks < 1) blocks = 1;  // the bounds are still checked
  if (blocks > 65536) blocks = 65536;
  hipLaunchKernelGGL(kernel, dim3(unsigned(blocks), unsigned(num_seqs)),
                     dim3(kWave), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

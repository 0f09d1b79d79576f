// The weights that new tokens' attention gives the places of a 16-bit paged KV cache,
// added up by place, for MI355X (gfx950), as specified in include/lumen_paged.h
// (lumen_paged_weigh).

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "lumen_attn_tiles.h"
#include "lumen_paged.h"
#include "lumen_paged_common.h"

namespace {

using namespace lumen_paged_detail;

constexpr int kPlaces = 64;  // of a wavefront
constexpr int kWaves = 4, kThreads = kWaves * kWave;

struct WeighArgs : Call {
  const float *lse;
  float *weights;  // of the layer
  int32_t chunks;  // of kWaves * kPlaces places, of a request at most
};

// A wavefront takes 64 places of a request and a KV head, holds their keys as the
// left operand of 32x32x16 products, and goes over the query rows that see them, 32
// at a time: scores^T = K Q^T, queries across, so that a lane has one query's lse.
// Its weights are added up by place in 32 bits, and over the lanes at the end.
template <int D, bool kBf16>
__global__ __launch_bounds__(kThreads, 2) void weigh_kernel(WeighArgs a) {
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int64_t items = int64_t(a.num_reqs) * a.chunks * a.kv_heads;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t rest = item / a.kv_heads;
    const int h = int(item - rest * a.kv_heads);
    const int r = int(rest / a.chunks), chunk = int(rest - int64_t(r) * a.chunks);
    Request q;
    int err = request(a, r, &q);
    if (chunk == 0 && h == 0 && wave == 0) record_wave(a.status, err);
    const int place0 = (chunk * kWaves + wave) * kPlaces;
    const int n = q.n < a.cap ? q.n : a.cap;
    if (q.m == 0 || place0 >= n) continue;
    // ---- the places: the lane's own, and the keys of two of them as fragments
    const int place = place0 + lane;
    int64_t block = 0;
    int at = 0;
    bool in = place < n;
    err = LUMEN_OK;
    if (in) {
      const int page = int(uint32_t(place) / uint32_t(a.block_size));
      block = a.bt[int64_t(r) * a.bt_cols + page];
      at = place - page * a.block_size;
      in = block >= 0 && block < a.num_blocks;
      if (!in) err = LUMEN_ERR_BLOCK_ID;
    }
    record_wave(a.status, err);
    const uint64_t live = __ballot(in);
    if (live == 0) continue;
    const int64_t offset = block * a.page + int64_t(at) * a.slot_bytes;
    const uint8_t *const kb = a.k + int64_t(h) * a.head_bytes + 16 * half;
    frag8 k[2][D / 16];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int64_t from = __shfl(offset, t * 32 + col);
      const bool there = live >> (t * 32 + col) & 1;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        k[t][i] = frag8{0, 0, 0, 0, 0, 0, 0, 0};
        if (there) k[t][i] = *reinterpret_cast<const frag8 *>(kb + from + 32 * i);
      }
    }
    f32x16 sum[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[t][i] = 0.0f;
    // ---- the rows, from the first that sees place0 on
    const int behind = q.n - q.m, rows = q.m * a.group;
    const int first = place0 > behind ? (place0 - behind) * a.group : 0;
    for (int row0 = first / 32 * 32; row0 < rows; row0 += 32) {
      const int row = row0 + col < rows ? row0 + col : rows - 1;
      const int tok = row / a.group;
      const int head = h * a.group + (row - tok * a.group);
      const uint16_t *p = a.q.base + (int64_t(q.q0) + tok) * a.q.token +
                          int64_t(head) * a.q.head + 8 * half;
      frag8 x[D / 16];
#pragma unroll
      for (int i = 0; i < D / 16; ++i) x[i] = *reinterpret_cast<const frag8 *>(p + 16 * i);
      const float lse = a.lse[(int64_t(q.q0) + tok) * a.q_heads + head];
      // a query that saw nothing adds nothing
      const float shift = lse == -INFINITY ? INFINITY : lse * 1.44269504088896341f;
      f32x16 sc[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[t][i] = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) sc[t] = mfma<kBf16>(k[t][i], x[i], sc[t]);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sc[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i], a.scale_log2, -shift));
      }
      if (row0 + 31 >= rows || behind + row0 / a.group < place0 + kPlaces - 1) {
        const int to = behind + tok - place0;
        const uint64_t sees = row0 + col >= rows ? 0
                              : to >= kPlaces - 1 ? ~uint64_t(0)
                              : to < 0            ? 0
                                                  : (uint64_t(2) << to) - 1;
        const uint64_t mine = sees >> (4 * half);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(uint32_t(mine >> (32 * t)) >> (8 * (i / 4) + i % 4) & 1)) sc[t][i] = 0.0f;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[t][i] += sc[t][i];
    }
    // ---- over the queries' lanes: each step halves the places that a lane holds
    float s[32];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[16 * t + i] = sum[t][i];
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      const bool high = lane & o;
#pragma unroll
      for (int i = 0; i < o; ++i) {
        const float send = high ? s[i] : s[i + o];
        s[i] = (high ? s[i + o] : s[i]) + __shfl_xor(send, o);
      }
    }
    // the lane's place: element col of the list above
    const int mine = (col / 16) * 32 + (col % 16 / 4) * 8 + 4 * half + col % 4;
    const int64_t word = (block * a.kv_heads + h) * a.block_size + at;
    const int64_t to = __shfl(word, mine);
    if (live >> mine & 1) a.weights[to] += s[0];
  }
}

// Workgroups of a launch at most: more than run at once, and few enough that their
// threads are counted in 32 bits.
constexpr int64_t kMostGroups = 1 << 22;

}  // namespace

extern "C" {

size_t lumen_paged_weigh_workspace_bytes(const lumen_kv_layout *, int32_t, int32_t, int64_t,
                                         int32_t, int32_t) {
  return 0;
}

int lumen_paged_weigh(const lumen_kv_layout *layout, int32_t layer, const void *d_cache,
                      const int32_t *d_block_tables, int32_t bt_cols, const int32_t *d_lens,
                      const int32_t *d_cu, int32_t num_reqs, const lumen_attn_rows *q,
                      int64_t num_tokens, int32_t max_new, int32_t dtype, int32_t num_q_heads,
                      float scale, const float *d_lse, void *d_ledger, void *d_workspace,
                      size_t workspace_bytes, int32_t *d_status, lumen_stream_t stream) {
  Pages pages;
  int st = check_pages(layout, layer, 1, &pages);
  if (st != LUMEN_OK) return st;
  if ((st = check_dtype(dtype)) != LUMEN_OK) return st;
  if ((st = check_scale(scale)) != LUMEN_OK) return st;
  if ((st = check_queries(layout, bt_cols, num_reqs, num_tokens, max_new, num_q_heads)) !=
      LUMEN_OK)
    return st;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if ((st = check_rows(q, num_tokens)) != LUMEN_OK) return st;
  if (num_reqs == 0 || num_tokens == 0) return LUMEN_OK;
  if (!d_lens || !d_cu || !d_lse || (!d_block_tables && bt_cols > 0) ||
      ((!d_cache || !d_ledger) && layout->num_blocks > 0))
    return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_cache, 16) || !aligned(d_workspace, 16) || !aligned(d_lens, 4) ||
      !aligned(d_cu, 4) || !aligned(d_block_tables, 4) || !aligned(d_lse, 4) ||
      !aligned(d_ledger, 4))
    return LUMEN_ERR_MISALIGNED;
  if (lumen_paged_weigh_workspace_bytes(layout, bt_cols, num_reqs, num_tokens, max_new,
                                        num_q_heads) > (d_workspace ? workspace_bytes : 0))
    return LUMEN_ERR_INVALID_ARG;
  (void)hipGetLastError();
  WeighArgs a;
  static_cast<Call &>(a) =
      call_of(layout, pages, layer, d_cache, d_block_tables, bt_cols, d_lens, d_cu, num_reqs, q,
              num_tokens, max_new, num_q_heads, scale, d_status);
  a.lse = d_lse;
  a.weights = static_cast<float *>(d_ledger) + 2 * layer * ledger_words(layout);
  a.chunks = (a.cap + kWaves * kPlaces - 1) / (kWaves * kPlaces);
  if (a.chunks < 1) a.chunks = 1;  // which looks at the requests
  int64_t groups = int64_t(num_reqs) * a.chunks;
  groups = groups < kMostGroups / a.kv_heads ? groups * a.kv_heads : kMostGroups;
  const bool bf = dtype == LUMEN_ATTN_BF16;
  const auto kernel = layout->head_dim == 64 ? (bf ? weigh_kernel<64, true> : weigh_kernel<64, false>)
                                             : (bf ? weigh_kernel<128, true> : weigh_kernel<128, false>);
  hipLaunchKernelGGL(kernel, dim3(unsigned(groups)), dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

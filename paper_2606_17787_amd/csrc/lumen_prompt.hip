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
  int32_t heads_per_tile;
  float scale_log2;  // scale * log2(e)
  uint16_t *out;
  int32_t *status;
};

// 16-bit fragments of the matrix instructions, and their products.
typedef short frag8 __attribute__((ext_vector_type(8)));
typedef short frag4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <bool kBf16>
__device__ __forceinline__ f32x16 mfma(frag8 a, frag8 b, f32x16 c) {
  if constexpr (kBf16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(
        __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(
        __builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * kWave;
constexpr int kKeys = 64;  // keys of a tile
constexpr float kSlack = 8.0f;
constexpr int kMfma = 0x8, kDsRead = 0x100;  // of sched_group_barrier

template <int D>
__device__ __forceinline__ int swizzle_k(int row) {
  return D == 128 ? row & 15 : (row >> 1) & 7;
}
template <int D>
__device__ __forceinline__ int swizzle_v(int row) {
  // 0, 4, 10, 14 for the four rows that one transposing read takes
  return D == 128 ? (row & 3) * 4 + ((row & 2) ? 2 : 0) : (row & 3) * 2;
}

// Sum over the wavefront's lanes, the same in all of them.
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);  // row_shr 1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, true);  // row_bcast 15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, true);  // row_bcast 31
  return __builtin_amdgcn_readlane(x, 63);
}

// Sequences a thread looks at when there are more than a wavefront's lanes.
constexpr int kPer = (LUMEN_ATTN_MAX_REQS + kThreads - 1) / kThreads;

// The `rank`-th query tile in the order of falling work: tile t of a sequence
// with `behind` keys before its first query sees about (t + 1) tiles of keys
// more than behind, its level; tiles of one level are in the order of their
// sequences' threads.  Hardware starts workgroups in order, so the long ones
// start first and the short ones fill the end.  The level is found by
// bisection over the number of tiles at or above it, a sum over the sequences:
// on one wavefront's lanes (every wavefront for itself) up to 64 sequences,
// on the workgroup's threads above.  False: there are fewer tiles.
__device__ bool find_tile(const PromptArgs &a, int tile_tokens, uint32_t rank,
                          uint32_t *lds, int *seq, int *tile) {
  const bool narrow = a.num_seqs <= kWave;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int me = narrow ? lane : tid, step = narrow ? kWave : kThreads;
  uint32_t n[kPer], off[kPer], top = 0;
  int err = LUMEN_OK;
  for (int i = 0; i < kPer; ++i) {
    n[i] = off[i] = 0;
    const int s = me + i * step;
    if (s >= a.num_seqs || (narrow && i)) continue;
    const int64_t q0 = a.cu_q[s], q1 = a.cu_q[s + 1];
    const int64_t k0 = a.cu_k[s], k1 = a.cu_k[s + 1];
    if (q0 < 0 || q1 < q0 || q1 > a.num_q || k0 < 0 || k1 < k0 || k1 > a.num_k) {
      err = LUMEN_ERR_RANGE;
      continue;
    }
    n[i] = uint32_t((q1 - q0 + tile_tokens - 1) / tile_tokens);
    const int64_t behind = (k1 - k0) - (q1 - q0);
    off[i] = behind > 0 ? uint32_t(behind) / uint32_t(tile_tokens) : 0u;
    top = n[i] && n[i] + off[i] > top ? n[i] + off[i] : top;
  }
  if (blockIdx.x == 0) record_wave(a.status, err);
  const auto total = [&](uint32_t x) {
    x = wave_sum(x);
    if (narrow) return x;
    __syncthreads();
    if (lane == 0) lds[wave] = x;
    __syncthreads();
    x = 0;
    for (int w = 0; w < kWaves; ++w) x += lds[w];
    return x;
  };
  // tiles at level j or above
  const auto above = [&](uint32_t j) {
    uint32_t c = 0;
    for (int i = 0; i < kPer; ++i) {
      if (narrow && i) break;
      const uint32_t last = n[i] + off[i];
      const uint32_t x = last >= j ? last - j + 1 : 0;
      c += x < n[i] ? x : n[i];
    }
    return total(c);
  };
  if (rank >= above(1)) return false;
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t t = __shfl_xor(top, o);
    top = t > top ? t : top;
  }
  if (!narrow) {
    __syncthreads();
    if (lane == 0) lds[wave] = top;
    __syncthreads();
    for (int w = 0; w < kWaves; ++w) top = lds[w] > top ? lds[w] : top;
  }
  uint32_t lo = 1, hi = top, before = 0;  // above(lo) > rank >= above(hi + 1)
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    const uint32_t c = above(mid);
    if (c > rank) {
      lo = mid;
    } else {
      hi = mid - 1;
      before = c;
    }
  }
  rank -= before;  // of the tiles at level lo, in thread order
  uint32_t mine = 0;
  for (int i = 0; i < kPer; ++i) mine += off[i] < lo && lo <= off[i] + n[i];
  uint32_t upto = mine;  // inclusive over the lanes
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t u = __shfl_up(upto, o);
    if (lane >= o) upto += u;
  }
  if (!narrow) {
    __syncthreads();
    if (lane == kWave - 1) lds[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += lds[w];
  }
  uint32_t left = rank - (upto - mine);
  const bool found = rank < upto && rank >= upto - mine;
  int s = 0, t = 0;
  if (found)
    for (int i = 0; i < kPer; ++i)
      if (off[i] < lo && lo <= off[i] + n[i] && left-- == 0) {
        s = me + i * step;
        t = int(lo - 1 - off[i]);
      }
  if (narrow) {
    const int at = __ffsll(static_cast<unsigned long long>(__ballot(found))) - 1;
    *seq = __builtin_amdgcn_readlane(s, at);
    *tile = __builtin_amdgcn_readlane(t, at);
  } else {
    __syncthreads();
    if (found) lds[0] = uint32_t(s), lds[1] = uint32_t(t);
    __syncthreads();
    *seq = __builtin_amdgcn_readfirstlane(int(lds[0]));
    *tile = __builtin_amdgcn_readfirstlane(int(lds[1]));
    __syncthreads();
  }
  return true;
}

// A workgroup takes 256 query rows of one KV head: 8 wavefronts of 32
// consecutive tokens of one query head each, kHeads of them of different
// heads of the group.
template <int D, bool kBf16>
__global__ __launch_bounds__(kThreads) void prompt_kernel(PromptArgs a) {
  constexpr int kChunks = D / 8;              // 16-byte chunks of a row
  constexpr int kTile = kKeys * D;            // elements of a K or V tile
  constexpr int kIssues = kKeys * kChunks / kThreads;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[2][2][kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;

  // ---- the unit: sequence, tokens, heads
  const int gp = a.heads_per_tile;
  const int groups = a.q_heads / gp;
  const int tile_tokens = 32 * kWaves / gp;
  const int hg = int(blockIdx.x % unsigned(groups));
  int s, tile;
  if (!find_tile(a, tile_tokens, blockIdx.x / unsigned(groups),
                 reinterpret_cast<uint32_t *>(lds), &s, &tile))
    return;
  const int64_t q0 = a.cu_q[s], q1 = a.cu_q[s + 1];
  const int64_t k0 = a.cu_k[s], k1 = a.cu_k[s + 1];
  const int nq = int(q1 - q0), nk = int(k1 - k0), behind = nk - nq;
  const int t0 = tile * tile_tokens;
  const int hq = hg * gp + wave % gp;
  const int hk = hg * gp / (a.q_heads / a.kv_heads);
  const int w0 = t0 + wave / gp * 32;  // the wavefront's first token
  const int tok = w0 + col;
  const bool here = w0 < nq;
  const int limit = tok + behind;  // last key that the lane's query sees
  const int tile_end = t0 + tile_tokens < nq ? t0 + tile_tokens : nq;
  const int steps = tile_end + behind > 0 ? (tile_end + behind + kKeys - 1) / kKeys : 0;
  const int wave_end = (w0 + 32 < nq ? w0 + 32 : nq) + behind;
  const int wave_steps = here && wave_end > 0 ? (wave_end + kKeys - 1) / kKeys : 0;

  // ---- Q: the lane's query, as the right operand (k = 8 * half + j)
  frag8 q[D / 16];
  {
    const int t = tok < nq ? tok : nq - 1;
    const uint16_t *p = a.q.base + (q0 + t) * a.q.token + hq * a.q.head + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      q[i] = *reinterpret_cast<const frag8 *>(p + 16 * i);
  }

  // the queries are here before the first tile's loads, which the compiler does
  // not count, so that no wait for them is left in the loop
  __builtin_amdgcn_s_waitcnt(0x0f70);

  const uint16_t *kb = a.k.base + k0 * a.k.token + hk * a.k.head;
  const uint16_t *vb = a.v.base + k0 * a.v.token + hk * a.v.head;
  const uint32_t lds_at = uint32_t(__builtin_amdgcn_readfirstlane(
      int(reinterpret_cast<uintptr_t>(LDS_PTR(uint16_t, lds))) + wave * kWave * 16));
  const auto load = [&](int step, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kIssues; ++i) {
      const int at = i * kThreads + wave * 64;
      const int row = (at + lane) / kChunks, pos = (at + lane) % kChunks;
      int key = step * kKeys + row;
      key = key < nk ? key : nk - 1;  // rows past the end repeat the last key
      const uint32_t to = lds_at + (buf * 2 * kTile + i * kThreads * 8) * 2;
      load_to_lds<false>(kb + int64_t(key) * a.k.token + 8 * (pos ^ swizzle_k<D>(row)),
                         to);
      load_to_lds<false>(vb + int64_t(key) * a.v.token + 8 * (pos ^ swizzle_v<D>(row)),
                         to + kTile * 2);
    }
  };

  f32x16 o[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  if (steps > 0) load(0, 0);
  for (int step = 0; step < steps; ++step) {
    const int buf = step & 1;
    wait_loads<0>();
    lds_barrier();
    if (step + 1 < steps) load(step + 1, buf ^ 1);
    if (step >= wave_steps) continue;
    // ---- scores, keys down and queries across
    f32x16 sc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[t][i] = 0.0f;
    // the second half's keys are read while the first half's products run
    frag8 k[D / 16];
    const auto key_row = [&](int t, int i) __attribute__((always_inline)) {
      const int row = t * 32 + col;
      return *reinterpret_cast<const frag8 *>(
          &lds[buf][0][row * D + 8 * ((2 * i + half) ^ swizzle_k<D>(row))]);
    };
#pragma unroll
    for (int i = 0; i < D / 16; ++i) k[i] = key_row(0, i);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      sc[0] = mfma<kBf16>(k[i], q[i], sc[0]);
      k[i] = key_row(1, i);
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i) sc[1] = mfma<kBf16>(k[i], q[i], sc[1]);
    __builtin_amdgcn_sched_group_barrier(kDsRead, D / 16, 0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
      __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(kMfma, D / 16, 0);
    if (step * kKeys + kKeys - 1 > w0 + behind) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = step * kKeys + t * 32 + 8 * (i / 4) + 4 * half + i % 4;
          if (key > limit) sc[t][i] = -INFINITY;
        }
    }
    // ---- running maximum: moved only when a score passes it by kSlack
    float top = -INFINITY;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[t][i]);
    float ta, tb;
    both<32>(top, &ta, &tb);
    top = fmaxf(ta, tb) * a.scale_log2;
    if (__any(top > m + kSlack)) {
      const float mn = fmaxf(m, top);
      const float c = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= c;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= c;
    }
    const float ms = m == -INFINITY ? 0.0f : m;
    frag8 p[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x =
            __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i], a.scale_log2, -ms));
        l += x;
        p[2 * t + i / 8][i % 8] = short(rounded<kBf16>(x));
      }
    // ---- weighted values
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        frag8 v;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int row = ks * 16 + 8 * b + 4 * half + ((lane & 15) >> 2);
          const int at = d * 32 + (lane & 16) + 4 * (lane & 3);
          const frag4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(
              frag4, &lds[buf][1][row * D + 8 * ((at >> 3) ^ swizzle_v<D>(row)) +
                                  (at & 7)]));
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * b + i] = x[i];
        }
        o[d] = mfma<kBf16>(v, p[ks], o[d]);
      }
  }
  if (!here) return;
  float la, lb;
  both<32>(l, &la, &lb);
  l = la + lb;
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  uint16_t *out = a.out + ((q0 + tok) * a.q_heads + hq) * D;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      uint32_t w[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int i = 8 * g + 2 * b;
        w[b] = uint32_t(rounded<kBf16>(o[d][i] * inv)) |
               uint32_t(rounded<kBf16>(o[d][i + 1] * inv)) << 16;
      }
      const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
      const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
      if (tok < nq)
        *reinterpret_cast<uint4 *>(out + d * 32 + 16 * g + 8 * half) =
            uint4{x[0], y[0], x[1], y[1]};
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
               num_q_heads, num_kv_heads, 0, scale * 1.44269504088896341f,
               static_cast<uint16_t *>(d_out), d_status};
  const bool bf = dtype == LUMEN_ATTN_BF16;
  void (*kernel)(PromptArgs) =
      head_dim == 64 ? (bf ? prompt_kernel<64, true> : prompt_kernel<64, false>)
                     : (bf ? prompt_kernel<128, true> : prompt_kernel<128, false>);
  const int group = num_q_heads / num_kv_heads;
  a.heads_per_tile = group % 8 == 0   ? 8
                     : group % 4 == 0 ? 4
                     : group % 2 == 0 ? 2
                                      : 1;
  // at most a part-filled tile for each sequence beside the full ones
  const int tile = 32 * kWaves / a.heads_per_tile;
  int64_t blocks = (num_q_tokens / tile + num_seqs) *
                   (num_q_heads / a.heads_per_tile);
  if (blocks > INT32_MAX) return LUMEN_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(kernel, dim3(unsigned(blocks)), dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

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
  uint32_t slots;  // workgroups that run at once, a set of heads; 0: no tile is cut
  float scale_log2;  // scale * log2(e)
  uint16_t *out;
  int32_t *status;
  float *parts;  // [max_parts][part_floats]
  uint32_t max_parts;  // parts of cut tiles, times sets of heads
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

// Tiles of at least this many keys may be cut: shorter parts would cost more to
// start and to join than they save.
constexpr int kMinPartKeys = 512;
// Keys of a call from which on tiles may be cut: below, the second launch that
// joins them costs what it saves.
constexpr int kCutKeys = 2048;

// A part of a query tile's keys: tile `tile` of sequence `seq`, part `part` of
// `parts`, each of `levels` levels; `first` is its tile's first part's place in
// the order of all parts.
struct Part {
  int seq, tile, part, parts, levels;
  uint32_t first;
};

// The order of work.  Tile t of a sequence with `behind` keys before its first
// query sees about (t + 1) tiles of keys more than behind: its level.  Tiles go
// by falling level, those of one level in the order of their sequences' threads,
// so that the long ones start first and the short ones fill the end.  A tile of
// more than `cut` levels, what a workgroup's slot has to do on average, goes as
// ceil(level / size) equal parts, where `size` is half of that (and at least
// kMinPartKeys): few long rows then fill the chip as many short ones do.  The
// level of a rank is found by bisection over the number of parts at or above it,
// a sum over the sequences: on one wavefront's lanes (every wavefront for itself)
// up to 64 sequences, on the workgroup's threads above.
template <int kThreads>
struct Finder {
  static constexpr int kPer = (LUMEN_ATTN_MAX_REQS + kThreads - 1) / kThreads;
  uint32_t n[kPer], off[kPer], top, cut, size;
  float inv_size;
  bool narrow;
  int me, step, lane, wave;
  uint32_t *lds;

  __device__ __forceinline__ uint32_t total(uint32_t x) const {
    x = wave_sum(x);
    if (narrow) return x;
    __syncthreads();
    if (lane == 0) lds[wave] = x;
    __syncthreads();
    x = 0;
    for (int w = 0; w < kThreads / kWave; ++w) x += lds[w];
    return x;
  }
  // x / size, exact for x below 2^23 (levels are at most 2^22)
  __device__ __forceinline__ uint32_t over_size(uint32_t x) const {
    uint32_t a = uint32_t(float(x) * inv_size);
    a -= a * size > x;
    return a + ((a + 1) * size <= x);
  }
  __device__ __forceinline__ uint32_t parts_at(uint32_t level) const {
    return level <= cut ? 1u : over_size(level + size - 1);
  }
  // parts of the tiles of levels 1 to m, all of them cut into parts of `size`
  __device__ __forceinline__ uint32_t parts_to(uint32_t m) const {
    const uint32_t a = over_size(m), b = m - a * size;
    return size * (a * (a + 1) / 2) + b * (a + 1);
  }
  // parts at level j or above
  __device__ __forceinline__ uint32_t above(uint32_t j) const {
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (narrow && i) break;
      const uint32_t last = n[i] + off[i], from = j - 1 > off[i] ? j - 1 : off[i];
      if (last <= from) continue;
      if (top <= cut) {  // nothing is cut
        c += last - from;
        continue;
      }
      const uint32_t whole = last < cut ? last : cut;  // levels up to here
      if (from < whole) c += whole - from;
      if (last > cut) c += parts_to(last) - parts_to(from > cut ? from : cut);
    }
    return total(c);
  }

  // `slots`: workgroups that run at once, for one set of heads; 0: no cuts
  __device__ void look(const PromptArgs &a, int tile_tokens, uint32_t slots,
                       uint32_t *scratch) {
    const int tid = threadIdx.x;
    narrow = a.num_seqs <= kWave;
    lane = tid & (kWave - 1), wave = tid / kWave;
    me = narrow ? lane : tid, step = narrow ? kWave : kThreads;
    lds = scratch;
    top = 0, cut = 0x7fffffffu, size = 1;
    int err = LUMEN_OK;
    uint64_t work = 0;
#pragma unroll
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
      n[i] = uint32_t(q1 - q0 + tile_tokens - 1) / uint32_t(tile_tokens);
      const int64_t behind = (k1 - k0) - (q1 - q0);
      off[i] = behind > 0 ? uint32_t(behind) / uint32_t(tile_tokens) : 0u;
      top = n[i] && n[i] + off[i] > top ? n[i] + off[i] : top;
      work += uint64_t(n[i]) * off[i] + uint64_t(n[i]) * (n[i] + 1) / 2;
    }
    if (blockIdx.x == 0) record_wave(a.status, err);
    if (slots) {
      // in two pieces, so that sums over the threads stay in 32 bits
      const uint64_t low = total(uint32_t(work) & 0x3fffffu);
      const uint64_t all = low + (uint64_t(total(uint32_t(work >> 22))) << 22);
      // held to 2^22, which no level passes
      const float share = fminf(float(all) / float(slots), 4194304.0f);
      const uint32_t least = uint32_t((kMinPartKeys + tile_tokens - 1) / tile_tokens);
      cut = uint32_t(share) + 1;
      size = cut / 2 + 1;
      size = size > least ? size : least;
      cut = cut > size ? cut : size;
    }
    inv_size = 1.0f / float(size);
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t t = __shfl_xor(top, o);
      top = t > top ? t : top;
    }
    if (!narrow) {
      __syncthreads();
      if (lane == 0) lds[wave] = top;
      __syncthreads();
      for (int w = 0; w < kThreads / kWave; ++w) top = lds[w] > top ? lds[w] : top;
    }
    top = __builtin_amdgcn_readfirstlane(top);
  }

  // The part of place `rank`; false where there are fewer.
  __device__ bool find(uint32_t rank, Part *out) {
    if (top == 0 || rank >= above(1)) return false;
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
    rank -= before;  // among the parts at level lo, in thread order
    const uint32_t parts = parts_at(lo);
    const uint32_t index = parts == 1 ? rank : rank / parts;  // the tile among those
    uint32_t mine = 0;
#pragma unroll
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
    uint32_t left = index - (upto - mine);
    const bool found = index < upto && index >= upto - mine;
    int s = 0, t = 0;
    if (found) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (off[i] < lo && lo <= off[i] + n[i] && left-- == 0) {
          s = me + i * step;
          t = int(lo - 1 - off[i]);
        }
    }
    if (narrow) {
      const int at = __ffsll(static_cast<unsigned long long>(__ballot(found))) - 1;
      out->seq = __builtin_amdgcn_readlane(s, at);
      out->tile = __builtin_amdgcn_readlane(t, at);
    } else {
      __syncthreads();
      if (found) lds[0] = uint32_t(s), lds[1] = uint32_t(t);
      __syncthreads();
      out->seq = __builtin_amdgcn_readfirstlane(int(lds[0]));
      out->tile = __builtin_amdgcn_readfirstlane(int(lds[1]));
      __syncthreads();
    }
    out->part = int(rank - index * parts);
    out->parts = int(parts);
    out->levels = parts == 1 ? int(lo) : int((lo + parts - 1) / parts);
    out->first = before + index * parts;
    return true;
  }
};

// Floats of a part's result: the lanes' sums, then their maxima and sums.
constexpr int part_floats(int D, int waves) { return waves * kWave * (D / 2 + 2); }

// What a lane's query is, and how its result is written.
struct Row {
  int tok, nq;      // of the sequence
  int64_t q0;       // of the sequence's first query
  int hq, half;
};

template <int D, bool kBf16>
__device__ __forceinline__ void write_row(const PromptArgs &a, const Row &r,
                                          const f32x16 *o, float l) {
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  uint16_t *out = a.out + ((r.q0 + r.tok) * a.q_heads + r.hq) * D;
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
      const uint32_t x0 = x[0], y0 = y[0], x1 = x[1], y1 = y[1];
      if (r.tok < r.nq)
        *reinterpret_cast<uint4 *>(out + d * 32 + 16 * g + 8 * r.half) =
            uint4{x0, y0, x1, y1};
    }
}

// A workgroup takes 32 * kWaves query rows of one KV head: a wavefront 32
// consecutive tokens of one query head, heads_per_tile of them different heads
// of the group.
template <int D, bool kBf16, int kWaves>
__global__ __launch_bounds__(kWaves *kWave, 2) void prompt_kernel(PromptArgs a) {
  constexpr int kThreads = kWaves * kWave;
  constexpr int kChunks = D / 8;              // 16-byte chunks of a row
  constexpr int kTile = kKeys * D;            // elements of a K or V tile
  constexpr int kIssues = kKeys * kChunks / kThreads;
  // tiles in LDS: kStages - 1 under way while one is used
  constexpr int kStages = kWaves == 8 ? 4 : 2;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[kStages][2][kTile];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = lane & 31, half = lane >> 5;

  // ---- the unit: sequence, tokens, heads
  const int gp = a.heads_per_tile;
  const int groups = a.q_heads / gp;
  const int tile_tokens = 32 * kWaves / gp;
  const int hg = int(blockIdx.x % unsigned(groups));
  Part p;
  {
    Finder<kThreads> finder;
    finder.look(a, tile_tokens, a.slots, reinterpret_cast<uint32_t *>(lds));
    if (!finder.find(blockIdx.x / unsigned(groups), &p)) return;
  }
  const int s = p.seq, tile = p.tile;
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
  // the part's keys, in steps of kKeys: [first_step, steps)
  const auto steps_to = [](int keys) { return keys > 0 ? (keys + kKeys - 1) / kKeys : 0; };
  int steps = steps_to(tile_end + behind), first_step = 0;
  if (p.parts > 1) {
    const int part_keys = p.levels * tile_tokens;
    first_step = steps_to(p.part * part_keys);
    const int stop = steps_to((p.part + 1) * part_keys);
    if (p.part + 1 < p.parts && stop < steps) steps = stop;
  }
  const int wave_end = (w0 + 32 < nq ? w0 + 32 : nq) + behind;
  int wave_steps = here ? steps_to(wave_end) : 0;
  wave_steps = wave_steps < steps ? wave_steps : steps;

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

#pragma unroll
  for (int i = 0; i < kStages - 1; ++i)
    if (first_step + i < steps) load(first_step + i, i);
  int buf = 0;
  for (int step = first_step; step < steps; ++step) {
    const int behind_it = steps - 1 - step;  // tiles loaded after this one
    if (kStages > 3 && behind_it >= 2)
      wait_loads<2 * 2 * kIssues>();
    else if (kStages > 2 && behind_it >= 1)
      wait_loads<2 * kIssues>();
    else
      wait_loads<0>();
    lds_barrier();
    const int now = buf;
    buf = buf + 1 < kStages ? buf + 1 : 0;
    if (step + kStages - 1 < steps)
      load(step + kStages - 1, now ? now - 1 : kStages - 1);
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
          &lds[now][0][row * D + 8 * ((2 * i + half) ^ swizzle_k<D>(row))]);
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
    frag8 pr[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x =
            __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i], a.scale_log2, -ms));
        l += x;
        pr[2 * t + i / 8][i % 8] = short(rounded<kBf16>(x));
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
              frag4, &lds[now][1][row * D + 8 * ((at >> 3) ^ swizzle_v<D>(row)) +
                                  (at & 7)]));
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * b + i] = x[i];
        }
        o[d] = mfma<kBf16>(v, pr[ks], o[d]);
      }
  }
  float la, lb;
  both<32>(l, &la, &lb);
  l = la + lb;
  if (p.parts > 1) {
    if (blockIdx.x >= a.max_parts) return;  // only where sequences share queries
    float *part = a.parts + int64_t(blockIdx.x) * part_floats(D, kWaves);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4 *>(part + ((d * 4 + i) * kThreads + tid) * 4) =
            float4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    part[kThreads * (D / 2) + tid] = m;
    part[kThreads * (D / 2 + 1) + tid] = l;
    return;
  }
  if (!here) return;
  write_row<D, kBf16>(a, Row{tok, nq, q0, hq, half}, o, l);
}

// Puts the parts of cut tiles together, in their order: a workgroup for a tile
// and set of heads, with the lanes' places of prompt_kernel.
template <int D, bool kBf16, int kWaves>
__global__ __launch_bounds__(kWaves *kWave, 2) void prompt_join_kernel(PromptArgs a) {
  constexpr int kThreads = kWaves * kWave;
  __shared__ uint32_t lds[kWaves + 2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int gp = a.heads_per_tile, groups = a.q_heads / gp;
  const int tile_tokens = 32 * kWaves / gp;
  const int hg = int(blockIdx.x % unsigned(groups));
  Finder<kThreads> finder;
  Part p;
  finder.look(a, tile_tokens, a.slots, lds);
  // parts of cut tiles come first, and each has at least two: the workgroup
  // takes the tiles that start at its two places
  for (uint32_t rank = blockIdx.x / unsigned(groups) * 2, end = rank + 2; rank < end;
       ++rank) {
    if (finder.top <= finder.cut || rank >= finder.above(finder.cut + 1)) return;
    if (!finder.find(rank, &p) || p.first != rank) continue;
    if ((uint64_t(rank) + p.parts) * groups > a.max_parts) return;
    const int64_t q0 = a.cu_q[p.seq];
    const Row r{p.tile * tile_tokens + wave / gp * 32 + (lane & 31),
                int(a.cu_q[p.seq + 1] - q0), q0, hg * gp + wave % gp, lane >> 5};
    f32x16 o[D / 32];
    float m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    for (int c = 0; c < p.parts; ++c) {
      const float *part =
          a.parts + (int64_t(rank + c) * groups + hg) * part_floats(D, kWaves);
      const float pm = part[kThreads * (D / 2) + tid];
      const float pl = part[kThreads * (D / 2 + 1) + tid];
      const float mn = fmaxf(m, pm);
      const float c0 = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      const float c1 = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(pm - mn);
      m = mn;
      l = l * c0 + pl * c1;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 x =
              *reinterpret_cast<const float4 *>(part + ((d * 4 + i) * kThreads + tid) * 4);
          o[d][4 * i] = o[d][4 * i] * c0 + x.x * c1;
          o[d][4 * i + 1] = o[d][4 * i + 1] * c0 + x.y * c1;
          o[d][4 * i + 2] = o[d][4 * i + 2] * c0 + x.z * c1;
          o[d][4 * i + 3] = o[d][4 * i + 3] * c0 + x.w * c1;
        }
    }
    write_row<D, kBf16>(a, r, o, l);
  }
}

// ------------------------------------------------------------ host side

// Grid and workspace of a call.
struct PromptPlan {
  int waves, heads_per_tile, tile_tokens, groups;
  int slots;      // workgroups that run at once, for one set of heads
  int64_t tiles;  // at most, for one set of heads
  int64_t parts;  // of cut tiles at most, for one set of heads; 0: none is cut
  size_t bytes;
};

// The workspace is sized for the largest device of this architecture, so that
// its size needs no device.
constexpr int kMaxUnits = 256;

PromptPlan prompt_plan(int32_t num_seqs, int64_t num_q, int64_t num_k,
                       int32_t q_heads, int32_t kv_heads, int32_t head_dim, int cus) {
  PromptPlan p;
  // Waves of a workgroup.
  p.waves = 8;
  const int group = q_heads / kv_heads;
  p.heads_per_tile = p.waves;
  while (group % p.heads_per_tile) p.heads_per_tile /= 2;
  p.tile_tokens = 32 * p.waves / p.heads_per_tile;
  p.groups = q_heads / p.heads_per_tile;
  p.slots = (cus < kMaxUnits ? cus : kMaxUnits) * 8 / p.waves / p.groups;
  // at most a part-filled tile for each sequence beside the full ones
  p.tiles = num_q / p.tile_tokens + num_seqs;
  p.parts = 0;
  if (num_k >= kCutKeys) {
    // a cut tile of `level` levels has less than 2 * level / size parts, and size
    // is more than half a slot's share of all levels (its float's rounding is
    // far less than the 1 added to each half)
    p.parts = int64_t(p.slots) * 4;
    const int64_t most = p.tiles * (num_k / kMinPartKeys + 2);
    if (p.parts > most) p.parts = most;
  }
  p.bytes = size_t(p.parts) * p.groups * part_floats(head_dim, p.waves) * sizeof(float);
  return p;
}

struct PromptKernels {
  void (*main)(PromptArgs);
  void (*join)(PromptArgs);
};

template <int D, int kWaves>
PromptKernels prompt_kernels(bool bf16) {
  return bf16 ? PromptKernels{prompt_kernel<D, true, kWaves>, prompt_join_kernel<D, true, kWaves>}
              : PromptKernels{prompt_kernel<D, false, kWaves>, prompt_join_kernel<D, false, kWaves>};
}

int check_prompt(int32_t num_seqs, int64_t num_q, int64_t num_k, int32_t q_heads,
                 int32_t kv_heads, int32_t head_dim) {
  if (num_seqs < 0 || num_q < 0 || num_k < 0 || q_heads < 1 || kv_heads < 1 ||
      q_heads % kv_heads)
    return LUMEN_ERR_INVALID_ARG;
  if ((head_dim != 64 && head_dim != 128) || num_q > LUMEN_ATTN_MAX_TOKENS ||
      num_k > LUMEN_ATTN_MAX_TOKENS)
    return LUMEN_ERR_UNSUPPORTED;
  return num_seqs > LUMEN_ATTN_MAX_REQS ? LUMEN_ERR_TOO_MANY : LUMEN_OK;
}

}  // namespace

extern "C" {

size_t lumen_attn_prompt_workspace_bytes(int32_t num_seqs, int64_t num_q_tokens,
                                         int64_t num_k_tokens, int32_t num_q_heads,
                                         int32_t num_kv_heads, int32_t head_dim) {
  if (check_prompt(num_seqs, num_q_tokens, num_k_tokens, num_q_heads, num_kv_heads,
                   head_dim) != LUMEN_OK)
    return 0;
  return prompt_plan(num_seqs, num_q_tokens, num_k_tokens, num_q_heads, num_kv_heads,
                     head_dim, kMaxUnits).bytes;
}

int lumen_attn_prompt(const lumen_attn_rows *q, const lumen_attn_rows *k,
                      const lumen_attn_rows *v, int32_t dtype,
                      const int32_t *d_cu_q, const int32_t *d_cu_k,
                      int32_t num_seqs, int64_t num_q_tokens,
                      int64_t num_k_tokens, int32_t num_q_heads,
                      int32_t num_kv_heads, int32_t head_dim, float scale,
                      void *d_out, void *d_workspace, size_t workspace_bytes,
                      int32_t *d_status, lumen_stream_t stream) {
  int st = check_dtype(dtype);
  if (st != LUMEN_OK) return st;
  if (!(scale > 0.0f) || !(scale < INFINITY) ||
      (!d_cu_k && num_q_tokens != num_k_tokens))
    return LUMEN_ERR_INVALID_ARG;
  if ((st = check_prompt(num_seqs, num_q_tokens, num_k_tokens, num_q_heads,
                         num_kv_heads, head_dim)) != LUMEN_OK)
    return st;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if ((st = check_rows(q, num_q_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(k, num_k_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(v, num_k_tokens)) != LUMEN_OK) return st;
  if (num_seqs > 0 && !d_cu_q) return LUMEN_ERR_INVALID_ARG;
  if (num_q_tokens > 0 && !d_out) return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_out, 16) || !aligned(d_workspace, 16) || !aligned(d_cu_q, 4) ||
      !aligned(d_cu_k, 4))
    return LUMEN_ERR_MISALIGNED;
  if (num_seqs == 0) return LUMEN_OK;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  PromptPlan p = prompt_plan(num_seqs, num_q_tokens, num_k_tokens, num_q_heads,
                             num_kv_heads, head_dim, cus);
  if (!d_workspace) p.parts = 0;
  if (p.parts && workspace_bytes < p.bytes) return LUMEN_ERR_INVALID_ARG;
  if ((p.tiles + p.parts) * p.groups > INT32_MAX) return LUMEN_ERR_UNSUPPORTED;
  (void)hipGetLastError();
  PromptArgs a;
  a.q = rows_of(q, 0);
  a.k = rows_of(k, 0);
  a.v = rows_of(v, 0);
  a.cu_q = d_cu_q;
  a.cu_k = d_cu_k ? d_cu_k : d_cu_q;
  a.num_seqs = num_seqs;
  a.num_q = num_q_tokens;
  a.num_k = num_k_tokens;
  a.q_heads = num_q_heads;
  a.kv_heads = num_kv_heads;
  a.heads_per_tile = p.heads_per_tile;
  a.slots = p.parts ? uint32_t(p.slots) : 0u;
  a.scale_log2 = scale * 1.44269504088896341f;
  a.out = static_cast<uint16_t *>(d_out);
  a.status = d_status;
  a.parts = static_cast<float *>(d_workspace);
  a.max_parts = uint32_t(p.parts * p.groups);
  const bool bf = dtype == LUMEN_ATTN_BF16;
  const PromptKernels kernels =
      p.waves == 4 ? (head_dim == 64 ? prompt_kernels<64, 4>(bf) : prompt_kernels<128, 4>(bf))
                   : (head_dim == 64 ? prompt_kernels<64, 8>(bf) : prompt_kernels<128, 8>(bf));
  const dim3 threads(unsigned(p.waves * kWave));
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(kernels.main, dim3(unsigned((p.tiles + p.parts) * p.groups)),
                     threads, 0, s, a);
  if (p.parts)
    hipLaunchKernelGGL(kernels.join, dim3(unsigned((p.parts + 1) / 2 * p.groups)),
                       threads, 0, s, a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

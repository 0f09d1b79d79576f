// Causal attention over packed sequences for MI355X (gfx950), as specified in
// include/lumen_attn.h (lumen_attn_prompt).

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "lumen_attn.h"
#include "lumen_attn_common.h"
#include "lumen_attn_tiles.h"

namespace {

using namespace lumen_attn_detail;

// A workgroup's work: queries [t0, t0 + tile) of a sequence against its keys'
// steps [first, last).
struct Unit {
  int32_t q0, nq, k0, nk;  // the sequence; nq 0: no work
  int32_t t0, first, last;
  int32_t place;  // of its result among the parts, or -1: it is the whole
};

// A tile that was cut: its first unit, and how many there are.
struct Cut {
  int32_t unit, parts;
};

struct PromptArgs {
  Rows q, k, v;
  const int32_t *cu_q, *cu_k;
  int32_t num_seqs;
  int64_t num_q, num_k;
  int32_t q_heads, kv_heads;
  int32_t heads_per_tile, tile_tokens;
  float scale_log2;
  uint16_t *out;
  int32_t *status;
  // the plan; units is NULL where the kernel finds its unit itself
  Unit *units;
  int32_t num_units;  // room, for one set of heads
  int32_t slots;      // workgroups that run at once, for one set of heads
  int32_t *num_cuts;
  Cut *cuts;
  int32_t max_parts;  // room, for one set of heads; 0: no tile is cut
  float *parts;       // [max_parts][sets of heads][part_floats]
};

constexpr int kKeys = 64;  // keys of a tile

// Tiles are cut into parts of at least this many keys: shorter ones would cost
// more to start and to join than they save (3 sequences around 40 queries behind up
// to 5,000 keys, 8 query heads over one: 30 us, 33 with 256 and 35 with 1,024; 2 of
// 128 behind up to 16,384, 32 over 8: 68, 68 and 71).
constexpr int kMinPartKeys = 512;
// Keys of a call from which on tiles may be cut, in all its sequences: their own
// lengths are on the device.  With 2,048, 4,096 and 8,192, 2 sequences around 100
// queries behind up to 3,500 keys take 28, 63 and 63 us, one prompt of 2,048 tokens
// 41, 38 and 39 (8 query heads over 2), 64 of 32 21, 17 and 17, where nothing is cut:
// what the plan and the join cost a call is less than what long keys do uncut.
constexpr int kCutKeys = 2048;

__device__ __forceinline__ int steps_to(int keys) {
  return keys > 0 ? (keys + kKeys - 1) / kKeys : 0;
}

// One sequence of a call.
struct Sequence {
  int64_t q0, k0;
  int nq, nk;
  int tiles;  // of queries
};

__device__ __forceinline__ bool sequence(const PromptArgs &a, int s, Sequence *out) {
  const int64_t q0 = a.cu_q[s], q1 = a.cu_q[s + 1];
  const int64_t k0 = a.cu_k[s], k1 = a.cu_k[s + 1];
  *out = Sequence{q0, k0, 0, 0, 0};
  if (q0 < 0 || q1 < q0 || q1 > a.num_q || k0 < 0 || k1 < k0 || k1 > a.num_k)
    return false;
  out->nq = int(q1 - q0);
  out->nk = int(k1 - k0);
  out->tiles = (out->nq + a.tile_tokens - 1) / a.tile_tokens;
  return true;
}

// The whole tile `t` of a sequence.
__device__ __forceinline__ Unit whole_tile(const PromptArgs &a, const Sequence &s, int t) {
  const int t0 = t * a.tile_tokens;
  const int end = t0 + a.tile_tokens < s.nq ? t0 + a.tile_tokens : s.nq;
  return Unit{int(s.q0), s.nq, int(s.k0), s.nk, t0, 0, steps_to(end + s.nk - s.nq), -1};
}

// The `rank`-th tile, sequence by sequence: for calls whose tiles all run at
// once, so that their order does not matter.
__device__ __forceinline__ Unit find_tile(const PromptArgs &a, int rank) {
  const int lane = threadIdx.x & (kWave - 1);
  int err = LUMEN_OK;
  for (int base = 0; base < a.num_seqs; base += kWave) {
    Sequence s{0, 0, 0, 0, 0};
    if (base + lane < a.num_seqs && !sequence(a, base + lane, &s)) err = LUMEN_ERR_RANGE;
    if (blockIdx.x == 0) record_wave(a.status, err);
    int upto = s.tiles;  // inclusive over the lanes
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const uint64_t past = __ballot(rank < upto);
    if (past && blockIdx.x) {  // the first workgroup looks at every sequence
      const int at = __ffsll(static_cast<unsigned long long>(past)) - 1;
      const Sequence found{__builtin_amdgcn_readlane(int(s.q0), at),
                           __builtin_amdgcn_readlane(int(s.k0), at),
                           __builtin_amdgcn_readlane(s.nq, at),
                           __builtin_amdgcn_readlane(s.nk, at), 0};
      const int before = __builtin_amdgcn_readlane(upto - s.tiles, at);
      return whole_tile(a, found, rank - before);
    }
    if (past) {
      const int at = __ffsll(static_cast<unsigned long long>(past)) - 1;
      const int seq = base + at, tile = rank - __builtin_amdgcn_readlane(upto - s.tiles, at);
      for (int i = base + kWave + lane; i < a.num_seqs; i += kWave) {
        Sequence rest;
        if (!sequence(a, i, &rest)) err = LUMEN_ERR_RANGE;
      }
      record_wave(a.status, err);
      Sequence found;
      sequence(a, seq, &found);
      return whole_tile(a, found, tile);
    }
    rank -= __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return Unit{0, 0, 0, 0, 0, 0, 0, -1};
}

// The plan: every tile by falling work, so that the long ones start first and
// the short ones fill the end.  A part is three quarters of the steps that a
// workgroup's slot has to do on average, at least kMinPartKeys, and tiles of
// more than twice that are cut into equal parts of at most a part, so that few
// long rows fill the chip as many short ones do.  (Smaller parts balance better
// and cost more to join: 5 suffixes of 1,237 tokens behind up to 11,003 take 153
// us, against 164 with a half and 175 with the whole average; 8 of 300 behind up
// to 5,000 take 110, 113 and 114; 2 of 128 behind up to 16,384 take 68, 78 and
// 58.)  One workgroup: tiles are counted by work into kPlanThreads bins, the bins are
// summed from the top, and each tile takes the next place of its bin.  Which of
// two tiles of a bin comes first changes nothing but that order.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void prompt_plan_kernel(PromptArgs a) {
  __shared__ int tiles_to[LUMEN_ATTN_MAX_REQS];  // inclusive, over the sequences
  __shared__ uint32_t bins[kPlanThreads];
  __shared__ uint64_t wave_work[kPlanThreads / kWave];
  __shared__ int64_t wave_tiles[kPlanThreads / kWave];
  __shared__ int top, cuts, parts_used;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int per = (a.num_seqs + kPlanThreads - 1) / kPlanThreads;
  int err = LUMEN_OK, longest = 0;
  int64_t mine = 0;
  uint64_t work = 0;
  Sequence s;
  if (tid == 0) top = cuts = parts_used = 0;
  bins[tid] = 0;
  for (int i = tid * per; i < (tid + 1) * per && i < a.num_seqs; ++i) {
    if (!sequence(a, i, &s)) err = LUMEN_ERR_RANGE;
    mine += s.tiles;
    tiles_to[i] = int(mine < a.num_units ? mine : a.num_units);
    // steps of the sequence's tiles, and of its last one
    const int seen = s.nk < s.nq ? s.nk : s.nq;  // queries that see a key
    const int64_t n = (seen + a.tile_tokens - 1) / a.tile_tokens + (s.nk < s.nq);
    work += uint64_t(n * (s.nk - seen) + a.tile_tokens * n * (n + 1) / 2) / kKeys + n;
    const int last = s.tiles ? steps_to(s.nk) : 0;
    longest = last > longest ? last : longest;
  }
  int64_t upto = mine;
  uint64_t sum = work;
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
    sum += __shfl_xor(sum, o);
    const int y = __shfl_xor(longest, o);
    longest = y > longest ? y : longest;
  }
  if (lane == kWave - 1) wave_tiles[wave] = upto;
  if (lane == 0) wave_work[wave] = sum;
  __syncthreads();
  if (lane == 0) atomicMax(&top, longest);
  int64_t before = upto - mine, all = 0;
  sum = 0;
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    if (w < wave) before += wave_tiles[w];
    all += wave_tiles[w];
    sum += wave_work[w];
  }
  // held to the room there is: more tiles are possible only where sequences
  // share queries
  const int tiles = int(all < a.num_units ? all : a.num_units);
  for (int i = tid * per; i < (tid + 1) * per && i < a.num_seqs; ++i) {
    const int64_t to = tiles_to[i] + before;
    tiles_to[i] = int(to < a.num_units ? to : a.num_units);
  }
  __syncthreads();
  // more steps than this: a cut into parts of `part` steps or a little less
  const uint64_t share = sum / uint32_t(a.slots);
  const int most = share < 0x1fffffff ? int(share * 3 / 4) + 1 : 0x1fffffff;
  const int part = most > kMinPartKeys / kKeys ? most : kMinPartKeys / kKeys;
  const int whole = a.max_parts ? 2 * part : 0x7fffffff;
  // a bin of work, the most in bin 0
  const float scale = float(kPlanThreads - 1) / float(top + 1);
  const auto bin_of = [&](int steps) {
    return kPlanThreads - 1 - int(float(steps) * scale);
  };
  const auto tile_at = [&](int i, int *parts) {
    int lo = 0, hi = a.num_seqs - 1;  // the first sequence with tiles_to > i
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (tiles_to[mid] > i)
        hi = mid;
      else
        lo = mid + 1;
    }
    Sequence q;
    sequence(a, lo, &q);
    const Unit u = whole_tile(a, q, i - (lo ? tiles_to[lo - 1] : 0));
    *parts = u.last > whole ? (u.last + part - 1) / part : 1;
    return u;
  };
  for (int i = tid; i < tiles; i += kPlanThreads) {
    int parts;
    const Unit u = tile_at(i, &parts);
    atomicAdd(&bins[bin_of(u.last / parts)], uint32_t(parts));
  }
  __syncthreads();
  // exclusive sums of the bins
  uint32_t bin = bins[tid], run = bin;
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t x = __shfl_up(run, o);
    if (lane >= o) run += x;
  }
  if (lane == kWave - 1) wave_tiles[wave] = run;
  __syncthreads();
  for (int w = 0; w < wave; ++w) run += uint32_t(wave_tiles[w]);
  bins[tid] = run - bin;
  uint32_t total = 0;
  for (int w = 0; w < kPlanThreads / kWave; ++w) total += uint32_t(wave_tiles[w]);
  __syncthreads();
  for (int i = tid; i < tiles; i += kPlanThreads) {
    int parts;
    Unit u = tile_at(i, &parts);
    const uint32_t at = atomicAdd(&bins[bin_of(u.last / parts)], uint32_t(parts));
    // more units, or parts, than there is room for are possible only where
    // sequences share queries
    if (at + uint32_t(parts) > uint32_t(a.num_units)) {
      // places of it that there are hold no unit
      for (uint32_t x = at; x < uint32_t(a.num_units); ++x) a.units[x].nq = 0;
      continue;
    }
    if (parts == 1) {
      a.units[at] = u;
      continue;
    }
    const int place = atomicAdd(&parts_used, parts);
    const bool room = place + parts <= a.max_parts;
    if (room) a.cuts[atomicAdd(&cuts, 1)] = Cut{int(at), parts};
    const int steps = u.last;
    for (int c = 0; c < parts; ++c) {
      Unit x = u;
      if (room) {
        x.first = int(int64_t(steps) * c / parts);
        x.last = int(int64_t(steps) * (c + 1) / parts);
        x.place = place + c;
      } else if (c) {
        x.nq = 0;
      }
      a.units[at + c] = x;
    }
  }
  for (uint32_t i = total + tid; i < uint32_t(a.num_units); i += kPlanThreads)
    a.units[i].nq = 0;
  __syncthreads();
  if (tid == 0) *a.num_cuts = cuts;
  record_wave(a.status, err);
}

// Floats of a part's result: the lanes' sums, then their maxima and sums.
constexpr int part_floats(int D, int waves) { return waves * kWave * (D / 2 + 2); }

// What a lane's query is, and how its result is written.
struct Row {
  int tok, nq;      // of the sequence
  int64_t q0;       // of the sequence's first query
  int hq, half;
  bool sees;        // a key
};

// 32 elements of it from element 32 * d on: zeros where it sees no key.  The sum
// of the weights of one that does is 0 only if every score is -infinity: the row
// is NaN then, as the formula has it.
template <int D, bool kBf16>
__device__ __forceinline__ void write_row(const PromptArgs &a, const Row &r, int d,
                                          const f32x16 &o, float l) {
  const float inv = r.sees ? 1.0f / l : 0.0f;
  uint16_t *out = a.out + ((r.q0 + r.tok) * a.q_heads + r.hq) * D + d * 32;
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    uint32_t w[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int i = 8 * g + 2 * b;
      w[b] = uint32_t(rounded<kBf16>(o[i] * inv)) |
             uint32_t(rounded<kBf16>(o[i + 1] * inv)) << 16;
    }
    const auto x = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const uint32_t x0 = x[0], y0 = y[0], x1 = x[1], y1 = y[1];
    if (r.tok < r.nq)
      *reinterpret_cast<uint4 *>(out + 16 * g + 8 * r.half) = uint4{x0, y0, x1, y1};
  }
}

template <int D, int kWaves>
struct PromptShape {
  static constexpr int kThreads = kWaves * kWave;
  static constexpr int kChunks = D / 8;    // 16-byte chunks of a row
  static constexpr int kTile = kKeys * D;  // elements of a K or V tile
  // tiles in LDS: kStages - 1 under way while one is used; two workgroups of
  // four wavefronts share a compute unit's 160 KB
  static constexpr int kStages = kWaves == 8 ? 4 : 2;
};

// Infinities and NaN of a tile in LDS become 0; the rows that had some are set in
// `rows`, a bit each.
template <int D, bool kBf16, int kThreads>
__device__ __forceinline__ void clear_nonfinite(uint16_t *tile, uint32_t *rows, int tid) {
  uint32_t *w = reinterpret_cast<uint32_t *>(tile);
#pragma unroll 1
  for (int i = tid; i < kKeys * D / 2; i += kThreads) {
    const uint32_t x = w[i];
    const uint32_t keep = (not_finite16<kBf16>(x) ? 0u : 0xffffu) |
                          (not_finite16<kBf16>(x >> 16) ? 0u : 0xffff0000u);
    if (keep != 0xffffffffu) {
      w[i] = x & keep;
      const int row = i / (D / 2);
      atomicOr(&rows[row / 32], 1u << (row % 32));
    }
  }
}

// One workgroup's tile, or part of one: 32 * kWaves query rows of one KV head,
// a wavefront 32 consecutive tokens of one query head, heads_per_tile of them
// different heads of the group.
//
// A step is 64 keys: scores^T = K Q^T and sums^T = V^T P^T by 32x32x16 products,
// queries across, so that a lane has one query's maximum and sum, and the
// weights come out in the order in which they go in again.  K and V come
// straight into LDS, kStages steps in turn, their 16-byte chunks permuted by row
// so that neither the reads of K nor the transposing reads of V meet in a bank.
// Weights are 2^(s - m) with m at most kSlack under the running maximum, so that
// the sums are rescaled only now and then; they are rounded to the inputs' type
// for the products, their sum is taken before that in 32 bits.
//
// Bound by the matrix units and the power they draw, the vector unit close behind
// (32 exponentials and about 150 other instructions a wavefront and step, against
// 32 products): one prompt of 16,384 tokens, 32 query heads over 8, D 128, takes
// 1.92 to 2.17 ms on one card and another, 1.01 to 1.15 PFLOP/s (a large library
// product: 1.37), with the units busy 56% of the cycles at 1.7 GHz.  Letting half of
// the wavefronts lag behind by half a step, so that products meet exponentials, or
// giving them priority changed nothing.  Short sequences lose to the tiles' ragged
// ends and few steps: 24 of 384 or so take 126 us, 0.62 PFLOP/s.
//
// A value that is masked for some of a wavefront's queries has the weight 0 for
// them in the products, which keeps it out unless it is an infinity or NaN.
// Where a sum comes out as one, nothing is written and the call returns true:
// the tile is then done again with kApart, where such values are taken out of
// the products and the rows that had some, found on the way, are added to the
// queries that see them.  A prompt of 16,384 tokens (32 query heads over 8, D 128)
// takes 4.6 ms instead of 2.1 with a NaN in an early value, and 43 with an
// infinity in every second one.
template <int D, bool kBf16, int kWaves, bool kApart>
__device__ __forceinline__ bool prompt_tile(const PromptArgs &a, const int tid,
                                            uint16_t *lds, bool *not_finite,
                                            uint32_t (*bad_rows)[2]) {
  using S = PromptShape<D, kWaves>;
  constexpr int kThreads = S::kThreads, kChunks = S::kChunks, kTile = S::kTile;
  constexpr int kStages = S::kStages, kStageBytes = 2 * kTile * 2;
  constexpr int kIssues = kKeys * kChunks / kThreads;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;

  // ---- the unit: sequence, tokens, heads
  const int gp = a.heads_per_tile;
  const int groups = a.q_heads / gp;
  const int hg = int(blockIdx.x % unsigned(groups));
  const int rank = int(blockIdx.x / unsigned(groups));
  Unit u;
  if (a.units) {  // by scalar loads
    const auto *from = CONSTANT_PTR(int32_t, a.units + rank);
    u = Unit{from[0], from[1], from[2], from[3], from[4], from[5], from[6], from[7]};
  } else {
    u = find_tile(a, rank);
    for (int32_t *x : {&u.q0, &u.nq, &u.k0, &u.nk, &u.t0, &u.first, &u.last, &u.place})
      *x = __builtin_amdgcn_readfirstlane(*x);
  }
  if (u.nq == 0) return false;
  const int64_t q0 = u.q0, k0 = u.k0;
  const int nq = u.nq, nk = u.nk, t0 = u.t0, behind = nk - nq;
  const int hq = hg * gp + wave % gp;
  const int hk = hg * gp / (a.q_heads / a.kv_heads);
  const int w0 = t0 + wave / gp * 32;  // the wavefront's first token
  const int tok = w0 + col;
  const bool here = w0 < nq;
  const int limit = tok + behind;  // last key that the lane's query sees
  const int first_step = u.first, steps = u.last;
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
  // the lane's piece of each load: its key in the tile, its chunk, and both as
  // an offset from the tile's first key
  const auto row_of = [&](int i) { return (i * kThreads + tid) / kChunks; };
  const auto chunk_k = [&](int i) { return 16 * ((tid % kChunks) ^ swizzle_k<D>(row_of(i))); };
  const auto chunk_v = [&](int i) { return 16 * ((tid % kChunks) ^ swizzle_v<D>(row_of(i))); };
  const uint32_t token_k = uint32_t(a.k.token) * 2, token_v = uint32_t(a.v.token) * 2;
  uint32_t from_k[kIssues], from_v[kIssues];
#pragma unroll
  for (int i = 0; i < kIssues; ++i) {
    from_k[i] = row_of(i) * token_k + chunk_k(i);
    from_v[i] = row_of(i) * token_v + chunk_v(i);
  }
  const auto load = [&](int step, int buf) __attribute__((always_inline)) {
    const uint16_t *kt = kb + int64_t(step) * kKeys * a.k.token;
    const uint16_t *vt = vb + int64_t(step) * kKeys * a.v.token;
    const uint32_t to = lds_at + buf * kStageBytes;
    const int last = nk - 1 - step * kKeys;
    if (last >= kKeys - 1) {
#pragma unroll
      for (int i = 0; i < kIssues; ++i) {
        load_to_lds(kt, from_k[i], to + i * kThreads * 16);
        load_to_lds(vt, from_v[i], to + i * kThreads * 16 + kTile * 2);
      }
    } else {  // rows past the end repeat the last key
#pragma unroll
      for (int i = 0; i < kIssues; ++i) {
        const uint32_t row = row_of(i) < last ? row_of(i) : last;
        load_to_lds(kt, row * token_k + chunk_k(i), to + i * kThreads * 16);
        load_to_lds(vt, row * token_v + chunk_v(i), to + i * kThreads * 16 + kTile * 2);
      }
    }
  };

  // where the lane reads in a tile; the other chunks' places differ in those
  // bits of the address that count chunks
  const auto *lds_bytes = LDS_PTR(const char, lds);
  const uint32_t read_k = col * D * 2 + 16 * (half ^ swizzle_k<D>(col));
  const int tr_row = 4 * half + ((lane & 15) >> 2);
  const uint32_t read_v = kTile * 2 + tr_row * D * 2 +
                          16 * ((((lane & 16) >> 3) | ((lane & 2) >> 1)) ^ swizzle_v<D>(tr_row)) +
                          8 * (lane & 1);

  f32x16 o[D / 32];
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  if constexpr (kApart)  // of this step and the next, in turn
    if (tid < 4) bad_rows[tid / 2][tid % 2] = 0;
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
    if constexpr (kApart) {
      clear_nonfinite<D, kBf16, kThreads>(lds + now * 2 * kTile + kTile,
                                          bad_rows[step & 1], tid);
      lds_barrier();
      if (tid < 2) bad_rows[~step & 1][tid] = 0;
    }
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
    const uint32_t stage = now * kStageBytes;
    const auto key_row = [&](int t, int i) __attribute__((always_inline)) {
      return *reinterpret_cast<const __attribute__((address_space(3))) frag8 *>(
          lds_bytes + ((read_k ^ (32 * i)) + stage) + t * 32 * D * 2);
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
    const float ms = m == -INFINITY ? 0.0f : m - lift<kBf16>();
    frag8 pr[4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float x =
            __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i], a.scale_log2, -ms));
        l += x;  // before the rounding, which the products need
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
          const frag4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) frag4 *)(
                  lds_bytes + ((read_v ^ (64 * d)) + stage) + (ks * 16 + 8 * b) * D * 2));
#pragma unroll
          for (int i = 0; i < 4; ++i) v[4 * b + i] = x[i];
        }
        o[d] = mfma<kBf16>(v, pr[ks], o[d]);
      }
    if constexpr (kApart) {
      uint64_t rows = uniform(uint64_t(bad_rows[step & 1][1]) << 32 | bad_rows[step & 1][0]);
#pragma unroll 1
      for (; rows; rows &= rows - 1) {
        const int key = step * kKeys + __builtin_ctzll(rows);
        if (key >= nk) break;  // a copy of the last key
        add_nonfinite<D, kBf16>(vb + int64_t(key) * a.v.token + 4 * half,
                                key <= limit, o);
      }
    }
  }
  if constexpr (!kApart) {
    float z = 0.0f;  // NaN if any sum is not finite
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) z = __builtin_fmaf(o[d][i], 0.0f, z);
    const bool any = __any(z != z);
    if (lane == 0) not_finite[wave] = any;
    lds_barrier();
    bool again = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) again |= not_finite[w];
    if (__builtin_amdgcn_readfirstlane(again)) return true;
  }
  float la, lb;
  both<32>(l, &la, &lb);
  l = la + lb;
  if (u.place >= 0) {
    float *part = a.parts + (int64_t(u.place) * groups + hg) * part_floats(D, kWaves);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4 *>(part + ((d * 4 + i) * kThreads + tid) * 4) =
            float4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    part[kThreads * (D / 2) + tid] = m;
    part[kThreads * (D / 2 + 1) + tid] = l;
  } else if (here) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
      write_row<D, kBf16>(a, Row{tok, nq, q0, hq, half, limit >= 0}, d, o[d], l);
  }
  return false;
}

template <int D, bool kBf16, int kWaves>
__global__ __launch_bounds__(kWaves *kWave, 2) void prompt_kernel(PromptArgs a) {
  using S = PromptShape<D, kWaves>;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[S::kStages * 2 * S::kTile];
  __shared__ bool not_finite[kWaves];
  __shared__ uint32_t bad_rows[2][kKeys / 32];
  if (!prompt_tile<D, kBf16, kWaves, false>(a, threadIdx.x, lds, not_finite, bad_rows)) return;
  // from the arguments on, so that nothing is kept for this in the first loop
  auto *args = __builtin_amdgcn_kernarg_segment_ptr();
  int tid = threadIdx.x;
  asm volatile("" : "+s"(args));
  asm volatile("" : "+v"(tid));
  uint64_t words[sizeof(PromptArgs) / 8];
#pragma unroll
  for (unsigned i = 0; i < sizeof(PromptArgs) / 8; ++i)
    words[i] = CONSTANT_PTR(uint64_t, args)[i];
  PromptArgs again;
  static_assert(sizeof(words) == sizeof(again));
  __builtin_memcpy(&again, words, sizeof(again));
  prompt_tile<D, kBf16, kWaves, true>(again, tid, lds, not_finite, bad_rows);
}

// Puts the parts of cut tiles together, in their order: a workgroup for 32
// elements of a tile's rows of a set of heads, with the lanes' places of
// prompt_kernel.  A tile of few rows over long keys may have tens of parts:
// their loads do not wait for one another.
template <int D, bool kBf16, int kWaves>
__global__ __launch_bounds__(kWaves *kWave, 2) void prompt_join_kernel(PromptArgs a) {
  constexpr int kThreads = kWaves * kWave;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int gp = a.heads_per_tile, groups = a.q_heads / gp;
  const int items = *a.num_cuts * groups * (D / 32);
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int d = item % (D / 32), hg = item / (D / 32) % groups;
    const Cut cut = a.cuts[item / (D / 32) / groups];
    const Unit u = a.units[cut.unit];
    const int tok = u.t0 + wave / gp * 32 + (lane & 31);
    const Row r{tok, u.nq, u.q0, hg * gp + wave % gp, lane >> 5, tok + u.nk - u.nq >= 0};
    const int64_t apart = int64_t(groups) * part_floats(D, kWaves);
    const float *part = a.parts + (int64_t(u.place) * groups + hg) * part_floats(D, kWaves);
    const float *ms = part + kThreads * (D / 2) + tid, *ls = ms + kThreads;
    const float *os = part + (d * 4 * kThreads + tid) * 4;
    float m = -INFINITY, l = 0.0f;
#pragma unroll 8
    for (int c = 0; c < cut.parts; ++c) m = fmaxf(m, ms[c * apart]);
    f32x16 o;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = 0.0f;
    // no key of any part is seen: all sums are 0
    const float shift = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
    for (int c = 0; c < cut.parts; ++c) {
      const float w = __builtin_amdgcn_exp2f(ms[c * apart] - shift);
      l = __builtin_fmaf(ls[c * apart], w, l);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 x =
            *reinterpret_cast<const float4 *>(os + c * apart + i * kThreads * 4);
        o[4 * i] = __builtin_fmaf(x.x, w, o[4 * i]);
        o[4 * i + 1] = __builtin_fmaf(x.y, w, o[4 * i + 1]);
        o[4 * i + 2] = __builtin_fmaf(x.z, w, o[4 * i + 2]);
        o[4 * i + 3] = __builtin_fmaf(x.w, w, o[4 * i + 3]);
      }
    }
    write_row<D, kBf16>(a, r, d, o, l);
  }
}

// ------------------------------------------------------------ host side

// Grid and workspace of a call.
struct PromptPlan {
  int waves, heads_per_tile, tile_tokens, groups;
  int slots;        // workgroups that run at once, for one set of heads
  int64_t tiles;    // at most, for one set of heads
  int64_t parts;    // of cut tiles at most, for one set of heads; 0: none is cut
  bool planned;     // by a kernel before
  size_t units_at, cuts_at, parts_at, bytes;
};

// The workspace is sized for the largest device of this architecture, so that
// its size needs no device.
constexpr int kMaxUnits = 256;

// Wavefronts of a workgroup. Eight share a tile of keys among twice the queries
// and keep two more tiles under way: 1.92 ms against 1.96 for one prompt of
// 16,384 tokens (32 query heads over 8, D 128), 142 us against 149 for 4,096,
// 83 against 84 for 8 x 2,048 tokens of 8 heads over one. Four, of which two
// workgroups run on a compute unit, leave fewer lanes idle at the ends of
// sequences and spread few tiles better: 101 us against 122 for 64 prompts of
// 256 tokens, 89 against 100 for 8 of 1,024, 59 against 62 for one of 2,048,
// 154 against 160 for 5 around 1,237 tokens of 8 heads over one behind up to 11,003.
int prompt_waves(int32_t num_seqs, int64_t num_q, int32_t q_heads) {
  const bool long_ones = num_q >= int64_t(num_seqs) * 2048;
  const bool many = num_q * q_heads / (8 * 32) >= 2 * kMaxUnits;
  return long_ones && many ? 8 : 4;
}

PromptPlan prompt_plan(int32_t num_seqs, int64_t num_q, int64_t num_k,
                       int32_t q_heads, int32_t kv_heads, int32_t head_dim, int cus) {
  PromptPlan p;
  p.waves = prompt_waves(num_seqs, num_q, q_heads);
  const int group = q_heads / kv_heads;
  p.heads_per_tile = p.waves;
  while (group % p.heads_per_tile) p.heads_per_tile /= 2;
  p.tile_tokens = 32 * p.waves / p.heads_per_tile;
  p.groups = q_heads / p.heads_per_tile;
  const auto slots = [&](int units) {
    const int n = units * 8 / p.waves / p.groups;
    return n < 1 ? 1 : n;
  };
  p.slots = slots(cus < kMaxUnits ? cus : kMaxUnits);
  // at most a part-filled tile for each sequence beside the full ones
  p.tiles = num_q / p.tile_tokens + num_seqs;
  p.parts = 0;
  if (num_k >= kCutKeys) {
    // a cut tile has less than twice its steps over `part`'s parts, and `part`
    // is at least three quarters of a slot's share of all steps
    p.parts = int64_t(p.slots) * 4;
    const int64_t most = p.tiles * (num_k / kMinPartKeys + 2);
    if (p.parts > most) p.parts = most;
  }
  // Without a plan every workgroup looks its tile up, 64 sequences at a time: 9.3 us
  // against 14.8 with one for 8 prompts around 216 tokens (4 query heads over 2), 17
  // against 20 for 128 of 12 (32 over 8), but 49 against 40 for 400 of 4 and 155
  // against 82 for 1,000 of 2.  The same for every device, as the workspace's size is:
  // a small device takes a call's few tiles without a plan too, in another order.
  p.planned = p.parts > 0 || p.tiles > slots(kMaxUnits);
  const auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
  p.units_at = 256;  // the number of cuts stands first
  p.cuts_at = p.units_at + up(size_t(p.tiles + p.parts) * sizeof(Unit));
  p.parts_at = p.cuts_at + up(size_t(p.parts / 2 + 1) * sizeof(Cut));
  p.bytes = !p.planned ? 0
                       : p.parts_at + size_t(p.parts) * p.groups *
                                          part_floats(head_dim, p.waves) * sizeof(float);
  return p;
}

// A grid of more threads than a launch takes.
bool too_many_threads(const PromptPlan &p) {
  return (p.tiles + p.parts) * p.groups * p.waves * kWave > int64_t(UINT32_MAX);
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
  const PromptPlan p = prompt_plan(num_seqs, num_q_tokens, num_k_tokens, num_q_heads,
                                   num_kv_heads, head_dim, kMaxUnits);
  return too_many_threads(p) ? 0 : p.bytes;
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
  if (check_scale(scale) != LUMEN_OK || (!d_cu_k && num_q_tokens != num_k_tokens))
    return LUMEN_ERR_INVALID_ARG;
  if ((st = check_prompt(num_seqs, num_q_tokens, num_k_tokens, num_q_heads,
                         num_kv_heads, head_dim)) != LUMEN_OK)
    return st;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if ((st = check_rows(q, num_q_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(k, num_k_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(v, num_k_tokens)) != LUMEN_OK) return st;
  // a tile's rows are within 32 bits of its first
  if (num_k_tokens > 1 && (k->token_stride > LUMEN_ATTN_MAX_STRIDE ||
                           v->token_stride > LUMEN_ATTN_MAX_STRIDE))
    return LUMEN_ERR_UNSUPPORTED;
  if (num_seqs > 0 && !d_cu_q) return LUMEN_ERR_INVALID_ARG;
  if (num_q_tokens > 0 && !d_out) return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_out, 16) || !aligned(d_workspace, 16) || !aligned(d_cu_q, 4) ||
      !aligned(d_cu_k, 4))
    return LUMEN_ERR_MISALIGNED;
  if (num_seqs == 0) return LUMEN_OK;
  if (too_many_threads(prompt_plan(num_seqs, num_q_tokens, num_k_tokens, num_q_heads,
                                   num_kv_heads, head_dim, kMaxUnits)))
    return LUMEN_ERR_UNSUPPORTED;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  const PromptPlan p = prompt_plan(num_seqs, num_q_tokens, num_k_tokens, num_q_heads,
                                   num_kv_heads, head_dim, cus);
  if (p.planned && (!d_workspace || workspace_bytes < p.bytes))
    return LUMEN_ERR_INVALID_ARG;
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
  a.tile_tokens = p.tile_tokens;
  a.scale_log2 = scale_log2(scale);
  a.out = static_cast<uint16_t *>(d_out);
  a.status = d_status;
  char *ws = static_cast<char *>(d_workspace);
  a.units = p.planned ? reinterpret_cast<Unit *>(ws + p.units_at) : nullptr;
  a.num_units = int32_t(p.tiles + p.parts);
  a.slots = p.slots;
  a.num_cuts = reinterpret_cast<int32_t *>(ws);
  a.cuts = reinterpret_cast<Cut *>(ws + p.cuts_at);
  a.max_parts = int32_t(p.parts);
  a.parts = reinterpret_cast<float *>(ws + p.parts_at);
  const bool bf = dtype == LUMEN_ATTN_BF16;
  const PromptKernels kernels =
      p.waves == 4 ? (head_dim == 64 ? prompt_kernels<64, 4>(bf) : prompt_kernels<128, 4>(bf))
                   : (head_dim == 64 ? prompt_kernels<64, 8>(bf) : prompt_kernels<128, 8>(bf));
  const dim3 threads(unsigned(p.waves * kWave));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.planned)
    hipLaunchKernelGGL(prompt_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  hipLaunchKernelGGL(kernels.main, dim3(unsigned((p.tiles + p.parts) * p.groups)),
                     threads, 0, s, a);
  if (p.parts) {
    int64_t items = p.parts / 2 * p.groups * (head_dim / 32);
    if (items > 4 * cus) items = 4 * cus;
    hipLaunchKernelGGL(kernels.join, dim3(unsigned(items < 1 ? 1 : items)), threads, 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

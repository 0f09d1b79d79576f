// Attention of new tokens over a 16-bit paged KV cache for MI355X (gfx950), as
// specified in include/lumen_paged.h (lumen_paged_attend).

#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>
#include <stdint.h>

#include "lumen_attn_tiles.h"
#include "lumen_paged.h"
#include "lumen_paged_common.h"

namespace {

using namespace lumen_paged_detail;

// A workgroup's work: query rows [row0, row0 + tile) of a request against steps
// [first, last) of its places.  Row i is head i % group of a KV head's query heads,
// for new token i / group.
struct Unit {
  int32_t q0, m, r, n;  // the request's queries and places; m 0: no work
  int32_t row0, first, last;
  int32_t place;  // of its result among the parts, or -1: it is the whole
};

// A tile that was cut: its first unit, and how many there are.
struct Cut {
  int32_t unit, parts;
};

struct AttendArgs : Call {
  uint16_t *out;
  float *lse;
  // the plan; units is NULL where the kernel finds its unit itself
  int32_t tile_rows;
  Unit *units;
  int32_t num_units;  // room, for one KV head
  int32_t slots;      // workgroups that run at once, for one KV head
  int32_t *num_cuts;
  Cut *cuts;
  int32_t max_parts;  // room, for one KV head; 0: no tile is cut
  float *parts;       // [max_parts][kv_heads][part_floats]
};

constexpr int kKeys = 64;  // places of a step

__device__ __forceinline__ int steps_to(int places) {
  return places > 0 ? int((uint32_t(places) + kKeys - 1) / kKeys) : 0;
}

__device__ __forceinline__ int tiles_of(const AttendArgs &a, const Request &q) {
  return (q.m * a.group + a.tile_rows - 1) / a.tile_rows;
}

// Places that the rows up to `end` see at most, of those that the table has.
__device__ __forceinline__ int seen_to(const AttendArgs &a, const Request &q, int end) {
  const int rows = q.m * a.group;
  const int tok = quotient(a.by_group, (end < rows ? end : rows) - 1);
  const int to = q.n - q.m + tok + 1;
  return to < a.cap ? to : a.cap;
}

// The whole tile `t` of a request.
__device__ __forceinline__ Unit whole_tile(const AttendArgs &a, const Request &q, int r, int t) {
  const int row0 = t * a.tile_rows;
  return Unit{q.q0, q.m, r, q.n, row0, 0, steps_to(seen_to(a, q, row0 + a.tile_rows)), -1};
}

// The `rank`-th tile, request by request: for calls whose tiles all run at once,
// so that their order does not matter.  The first workgroup looks at every request,
// for its errors.
__device__ __forceinline__ Unit find_tile(const AttendArgs &a, int rank) {
  const int lane = threadIdx.x & (kWave - 1);
  int err = LUMEN_OK;
  Unit found{0, 0, 0, 0, 0, 0, 0, -1};
  bool have = false;
  for (int base = 0; base < a.num_reqs; base += kWave) {
    Request q{0, 0, 0};
    if (base + lane < a.num_reqs) {
      const int e = request(a, base + lane, &q);
      err = e < err ? e : err;
    }
    const int tiles = tiles_of(a, q);
    int upto = tiles;  // inclusive over the lanes
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    const uint64_t past = __ballot(rank < upto);
    if (past && !have) {
      const int at = __ffsll(static_cast<unsigned long long>(past)) - 1;
      const Request p{__builtin_amdgcn_readlane(q.q0, at), __builtin_amdgcn_readlane(q.m, at),
                      __builtin_amdgcn_readlane(q.n, at)};
      found = whole_tile(a, p, base + at,
                         rank - __builtin_amdgcn_readlane(upto - tiles, at));
      have = true;
      if (blockIdx.x) break;
    }
    rank -= __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  if (blockIdx.x == 0) record_wave(a.status, err);
  return found;
}

// Tiles are cut into parts of at least this many places where the parts of all run at
// once, and at least an eighth of the longest up to twice as many; of at least twice as
// many elsewhere.  With 256 and 512 throughout single tokens (32 query heads over 8) of 1
// request with 2,000 places take 22.7 and 26.2 us, with 16,000 55.8 and 40.5, of 4 around
// 1,500 26.5 and 36.7, of 16 with 2,000 47.3 and 39.3; with 1,024 the first two take 51.1
// and 41.5.
constexpr int kMinPartKeys = 256;

// The plan: every tile by falling work, so that the long ones start first and the
// short ones fill the end; tiles that are long beside a workgroup slot's share of
// all steps are cut into equal parts, so that few long rows fill the chip as many
// short ones do.  One workgroup: tiles are counted by work into kPlanThreads bins,
// the bins are summed from the top, and each tile takes the next place of its bin.
// Which of two tiles of a bin comes first changes nothing but that order.
constexpr int kPlanThreads = 1024;
__global__ __launch_bounds__(kPlanThreads) void attend_plan_kernel(AttendArgs a) {
  __shared__ int tiles_to[LUMEN_ATTN_MAX_REQS];  // inclusive, over the requests
  __shared__ uint32_t bins[kPlanThreads];
  __shared__ uint64_t wave_work[kPlanThreads / kWave];
  __shared__ int64_t wave_tiles[kPlanThreads / kWave];
  __shared__ int top, cuts, parts_used;
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int per = (a.num_reqs + kPlanThreads - 1) / kPlanThreads;
  int err = LUMEN_OK, longest = 0;
  int64_t mine = 0;
  uint64_t work = 0;
  Request q;
  if (tid == 0) top = cuts = parts_used = 0;
  bins[tid] = 0;
  for (int i = tid * per; i < (tid + 1) * per && i < a.num_reqs; ++i) {
    const int e = request(a, i, &q);
    err = e < err ? e : err;
    const int count = tiles_of(a, q);
    mine += count;
    tiles_to[i] = int(mine < a.num_units ? mine : a.num_units);
    if (count == 0) continue;
    // steps of the request's tiles: those of the first and the last, on average.  Past
    // the table's places the tiles are all alike, more than that average: as many as the
    // last has, so that there are no more parts than there is room for
    const int last = whole_tile(a, q, i, count - 1).last;
    work += q.n > a.cap ? uint64_t(count) * uint32_t(last)
                        : uint64_t(count) * uint32_t(whole_tile(a, q, i, 0).last + last + 1) / 2;
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
  // held to the room there is: more tiles are possible only where requests share
  // queries
  const int tiles = int(all < a.num_units ? all : a.num_units);
  for (int i = tid * per; i < (tid + 1) * per && i < a.num_reqs; ++i) {
    const int64_t to = tiles_to[i] + before;
    tiles_to[i] = int(to < a.num_units ? to : a.num_units);
  }
  __syncthreads();
  // More steps than twice `part`: a cut into parts of `part` steps or a little less.
  // At 5/8 of a share no part is long when the last ones run, at 1/2 even work is cut
  // that needs no cut.  For 1/2, 5/8, 3/4 and 1: 64 requests around 4,096 places with 5
  // tokens each 255, 242, 253 and 295 us, chunks of 512 among 96 requests 128, 124, 128
  // and 139, a chunk of 2,048 behind 14,336 592, 511, 511 and 511.  A cut from 1.5 times
  // `part` on would cost the chunks 4 % and the long one 28 %.
  const uint64_t share = sum / uint32_t(a.slots);
  const int most = share < 0x1fffffff ? int(share * 5 / 8) + 1 : 0x1fffffff;
  constexpr int kMinPart = kMinPartKeys / kKeys;
  const int eighth = share < kMinPart ? top / 8 : 2 * kMinPart;
  const int least = eighth < kMinPart ? kMinPart : eighth < 2 * kMinPart ? eighth : 2 * kMinPart;
  const int part = most > least ? most : least;
  const int whole = a.max_parts ? 2 * part : 0x7fffffff;
  // a bin of work, the most in bin 0
  const float scale = float(kPlanThreads - 1) / float(top + 1);
  const auto bin_of = [&](int steps) {
    return kPlanThreads - 1 - int(float(steps) * scale);
  };
  const auto tile_at = [&](int i, int *parts) {
    int lo = 0, hi = a.num_reqs - 1;  // the first request with tiles_to > i
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (tiles_to[mid] > i)
        hi = mid;
      else
        lo = mid + 1;
    }
    Request p;
    request(a, lo, &p);
    const Unit u = whole_tile(a, p, lo, i - (lo ? tiles_to[lo - 1] : 0));
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
    // more units, or parts, than there is room for are possible only where requests
    // share queries
    if (at + uint32_t(parts) > uint32_t(a.num_units)) {
      // places of it that there are hold no unit
      for (uint32_t x = at; x < uint32_t(a.num_units); ++x) a.units[x].m = 0;
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
        x.m = 0;
      }
      a.units[at + c] = x;
    }
  }
  for (uint32_t i = total + tid; i < uint32_t(a.num_units); i += kPlanThreads)
    a.units[i].m = 0;
  __syncthreads();
  if (tid == 0) *a.num_cuts = cuts;
  record_wave(a.status, err);
}

// Floats of a part's result: the lanes' sums, then their maxima and sums of weights.
constexpr int part_floats(int D, int waves) { return waves * kWave * (D / 2 + 3); }

// What a lane's query is, and where its result goes.
struct Row {
  bool here;     // it is a row of the request
  int64_t at;    // packed token * q_heads + query head
  int half;
};

__device__ __forceinline__ Row row_of(const AttendArgs &a, const Unit &u, int h, int row,
                                      int half) {
  int head;
  const int tok = quotient(a.by_group, row, &head);
  return Row{row < u.m * a.group,
             (int64_t(u.q0) + tok) * a.q_heads + h * a.group + head, half};
}

// 32 elements of it from element 32 * d on.  m is -infinity where the row has seen
// no place: it is zeros.  Where it has, the sum of the weights is 0 only if every
// score is -infinity (m is then -FLT_MAX): the row is NaN, as the formula has it.
template <int D, bool kBf16>
__device__ __forceinline__ void write_row(const AttendArgs &a, const Row &r, int d,
                                          const f32x16 &o, float m, float l) {
  const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
  uint16_t *out = a.out + r.at * D + d * 32;
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
    if (r.here)
      *reinterpret_cast<uint4 *>(out + 16 * g + 8 * r.half) = uint4{x0, y0, x1, y1};
  }
}

// The log of the weights' sum: they were taken times 2^(lift - m).
template <bool kBf16>
__device__ __forceinline__ void write_lse(const AttendArgs &a, const Row &r, float m, float l) {
  if (a.lse && r.here && r.half == 0)
    a.lse[r.at] = m == -INFINITY ? m
                                 : (m - lift<kBf16>() + __builtin_amdgcn_logf(l)) *
                                       0.693147180559945309f;
}

template <int D, int kWaves>
struct TileShape {
  static constexpr int kThreads = kWaves * kWave;
  static constexpr int kChunks = D / 8;    // 16-byte chunks of a row
  static constexpr int kTile = kKeys * D;  // elements of a K or V tile
  // tiles in LDS: kStages - 1 under way while one is used; two workgroups of
  // four wavefronts share a compute unit's 160 KB
  static constexpr int kStages = kWaves == 8 ? 4 : 2;
};

// The sum of eight fp16 values and c, in 32 bits.
__device__ __forceinline__ float add_all(frag8 x, float c) {
  typedef short pair16 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 8; i += 2)
    c = __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, pair16{x[i], x[i + 1]}),
                               f16x2{_Float16(1.0f), _Float16(1.0f)}, c, false);
  return c;
}

constexpr int kRound = 128;    // steps whose rows are looked up at a time
constexpr int kEntries = 1024; // runs of rows among them

// One workgroup's tile, or part of one: 32 * kWaves query rows of one KV head, a
// wavefront 32 of them.
//
// A step is 64 places: scores^T = K Q^T and sums^T = V^T P^T by 32x32x16 products,
// queries across, so that a lane has one query's maximum and sum, and the weights
// come out in the order in which they go in again.  K and V come straight into LDS,
// kStages steps in turn, their 16-byte chunks permuted by row (lumen_attn_tiles.h).
// Weights are 2^(s - m) with m at most kSlack under the running maximum, so that the
// sums are rescaled only now and then; they are rounded to the inputs' type for the
// products.  Their sum before that is lse's, and what bf16 rows are divided by.  fp16
// rows, whose outputs are eight times finer, are divided by the sum of the rounded
// weights, so that a weight that is most of its row leaves nothing of its rounding (in
// bf16 that would take a chunk of 2,048 tokens behind 14,336 from 518 to 533 us, for
// less than the rounding of its result).
//
// Where the rows of a step's places start is laid out in LDS for kRound steps at a
// time, an entry for each run of places that cannot leave its page (the largest power
// of two up to 16 that divides a page), and a bit for each place that counts.  Places
// that do not are read from a row of zeros.
//
// In steps with places that some of the tile's queries see and others do not, the
// weight 0 keeps a hidden value out of the products unless it is an infinity or NaN.
// Such values are taken out of the tile in LDS there, and the rows that had some are
// added to the queries that see them.
//
// Bound by the cache's bytes where a request has few new tokens: 256 of one around 2,048
// places (32 query heads over 8, D 128, bf16) take 500 us, 5.5 TB/s.  Bound by the
// products with the maxima, exponentials and roundings between them where it has many: a
// chunk of 2,048 behind 14,336 takes 492 to 515 us, 1.0 PFLOP/s.
template <int D, bool kBf16, int kWaves>
__global__ __launch_bounds__(kWaves *kWave, 2) void attend_kernel(AttendArgs a) {
  using S = TileShape<D, kWaves>;
  constexpr int kThreads = S::kThreads, kChunks = S::kChunks, kTile = S::kTile;
  constexpr int kStages = S::kStages, kStageBytes = 2 * kTile * 2;
  constexpr int kIssues = kKeys * kChunks / kThreads;
  __shared__ __attribute__((aligned(1024))) uint16_t lds[kStages * 2 * kTile];
  __shared__ uint64_t run_at[kEntries];  // bytes from the layer's K or V
  __shared__ uint64_t live_at[kRound];
  __shared__ uint32_t bad_rows[2];
  const int tid = threadIdx.x;
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;

  // ---- the unit
  const int h = int(blockIdx.x % unsigned(a.kv_heads));
  const int rank = int(blockIdx.x / unsigned(a.kv_heads));
  Unit u;
  if (a.units) {  // by scalar loads
    const auto *from = CONSTANT_PTR(int32_t, a.units + rank);
    u = Unit{from[0], from[1], from[2], from[3], from[4], from[5], from[6], from[7]};
  } else {
    u = find_tile(a, rank);
    for (int32_t *x : {&u.q0, &u.m, &u.r, &u.n, &u.row0, &u.first, &u.last, &u.place})
      *x = __builtin_amdgcn_readfirstlane(*x);
  }
  if (u.m == 0) return;
  const int rows = u.m * a.group;
  const int row = u.row0 + wave * 32 + col;
  const int wave_row = u.row0 + wave * 32;  // the wavefront's first
  const bool here = wave_row < rows;
  const int behind = u.n - u.m;
  const auto limit_of = [&](int x) __attribute__((always_inline)) {
    return behind + quotient(a.by_group, x < rows ? x : rows - 1);
  };
  const int limit = limit_of(row);              // last place that the lane's query sees
  const int wave_limit = limit_of(wave_row);    // that all of the wavefront's see
  const int tile_limit = limit_of(u.row0);      // that all of the tile's see
  const Request req{u.q0, u.m, u.n};
  const int end = seen_to(a, req, u.row0 + 32 * kWaves);  // of the tile's places
  const int wave_steps = here ? steps_to(seen_to(a, req, wave_row + 32)) : 0;

  // ---- Q: the lane's query, as the right operand (k = 8 * half + j)
  frag8 q[D / 16];
  {
    int head;
    const int tok = quotient(a.by_group, row < rows ? row : rows - 1, &head);
    const uint16_t *p = a.q.base + (int64_t(u.q0) + tok) * a.q.token +
                        int64_t(h * a.group + head) * a.q.head + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
      q[i] = *reinterpret_cast<const frag8 *>(p + 16 * i);
  }
  const uint8_t *const kb = a.k + int64_t(h) * a.head_bytes;
  const uint8_t *const vb = a.v + int64_t(h) * a.head_bytes;
  const uint32_t lds_at = uint32_t(__builtin_amdgcn_readfirstlane(
      int(reinterpret_cast<uintptr_t>(LDS_PTR(uint16_t, lds))) + wave * kWave * 16));
  // places of a run: the largest power of two up to 16 that divides a page
  const int low = a.block_size & -a.block_size;
  const int run_shift = low >= 16 ? 4 : __builtin_ctz(low);
  const int step_shift = 6 - run_shift;  // runs of a step
  const int round = kEntries >> step_shift < kRound ? kEntries >> step_shift : kRound;
  // the lane's piece of each load: its row in the step, and its chunk
  const auto row_in = [&](int i) { return (i * kThreads + tid) / kChunks; };
  const auto chunk_k = [&](int i) { return 16 * ((tid % kChunks) ^ swizzle_k<D>(row_in(i))); };
  const auto chunk_v = [&](int i) { return 16 * ((tid % kChunks) ^ swizzle_v<D>(row_in(i))); };
  const auto load = [&](int at, int buf) __attribute__((always_inline)) {
    const uint32_t to = lds_at + buf * kStageBytes;
    const uint64_t live = live_at[at];
    // all lookups first, so that one does not wait behind another's load
    const uint8_t *from_k[kIssues], *from_v[kIssues];
#pragma unroll
    for (int i = 0; i < kIssues; ++i) {
      const uint64_t run = run_at[(at << step_shift) + (row_in(i) >> run_shift)] +
                           uint32_t((row_in(i) & ((1 << run_shift) - 1)) * a.slot_bytes);
      from_k[i] = kb + run;
      from_v[i] = vb + run;
    }
    if (live != ~uint64_t(0)) {
#pragma unroll
      for (int i = 0; i < kIssues; ++i)
        if (!(live >> row_in(i) & 1))
          from_k[i] = from_v[i] = reinterpret_cast<const uint8_t *>(kZeroRow);
    }
#pragma unroll
    for (int i = 0; i < kIssues; ++i) {
      load_row(from_k[i] + chunk_k(i), to + i * kThreads * 16);
      load_row(from_v[i] + chunk_v(i), to + i * kThreads * 16 + kTile * 2);
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
  float m = -INFINITY, l = 0.0f, ls = 0.0f;  // ls: fp16's, of the rounded weights
  bool seen = false;
  int err = LUMEN_OK;

  for (int base = u.first; base < u.last; base += round) {
    const int count = u.last - base < round ? u.last - base : round;
    __syncthreads();  // the tables and tiles before are done with
    for (int i = tid; i < count * kKeys; i += kThreads) {
      const int place = base * kKeys + i;
      bool in = place < end;
      uint64_t at = 0;
      if (in) {
        int in_page;
        const int page = quotient(a.by_block, place, &in_page);
        const int32_t id = a.bt[int64_t(u.r) * a.bt_cols + page];
        in = id >= 0 && id < a.num_blocks;
        if (!in) err = LUMEN_ERR_BLOCK_ID;
        if (in) at = uint64_t(id) * a.page + uint64_t(in_page) * a.slot_bytes;
      }
      const uint64_t live = __ballot(in);
      if (lane == 0) live_at[i / kKeys] = live;
      if ((i & ((1 << run_shift) - 1)) == 0) run_at[i >> run_shift] = at;
    }
    if (tid < 2) bad_rows[tid] = 0;
    __syncthreads();
    // the queries are here before the first tile's loads, which the compiler does not
    // count, so that no wait for them is left in the loop
    __builtin_amdgcn_s_waitcnt(0x0f70);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i)
      if (i < count) load(i, i);
    int buf = 0;
    for (int at = 0; at < count; ++at) {
      const int step = base + at;
      const int behind_it = count - 1 - at;  // tiles loaded after this one
      if (kStages > 3 && behind_it >= 2)
        wait_loads<2 * 2 * kIssues>();
      else if (kStages > 2 && behind_it >= 1)
        wait_loads<2 * kIssues>();
      else
        wait_loads<0>();
      lds_barrier();
      const int now = buf;
      const bool border = step * kKeys + kKeys - 1 > tile_limit;
      if (border) {
        uint32_t *w = reinterpret_cast<uint32_t *>(lds + now * 2 * kTile + kTile);
#pragma unroll 1
        for (int i = tid; i < kTile / 2; i += kThreads) {
          const uint32_t x = w[i];
          const uint32_t keep = (not_finite16<kBf16>(x) ? 0u : 0xffffu) |
                                (not_finite16<kBf16>(x >> 16) ? 0u : 0xffff0000u);
          if (keep != 0xffffffffu) {
            w[i] = x & keep;
            const int place = i / (D / 2);
            atomicOr(&bad_rows[place / 32], 1u << (place % 32));
          }
        }
        lds_barrier();
      }
      buf = buf + 1 < kStages ? buf + 1 : 0;
      if (at + kStages - 1 < count) load(at + kStages - 1, now ? now - 1 : kStages - 1);
      uint64_t bad = 0;
      if (border) {
        bad = uniform(uint64_t(bad_rows[1]) << 32 | bad_rows[0]);
        if (bad) {
          lds_barrier();
          if (tid < 2) bad_rows[tid] = 0;
        }
      }
      if (step >= wave_steps) continue;
      // ---- scores, places down and queries across
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
      const uint64_t live = uniform(live_at[at]);
      if (live != ~uint64_t(0) || step * kKeys + kKeys - 1 > wave_limit) {
        const int to = limit - step * kKeys;
        const uint64_t sees =
            live & (to >= kKeys - 1 ? ~uint64_t(0) : to < 0 ? 0 : (uint64_t(2) << to) - 1);
        seen |= sees != 0;
        const uint64_t mine = sees >> (4 * half);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(uint32_t(mine >> (32 * t)) >> (8 * (i / 4) + i % 4) & 1)) sc[t][i] = -INFINITY;
      } else {
        seen = true;
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
        if constexpr (!kBf16) ls *= c;
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
      if constexpr (!kBf16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) ls = add_all(pr[i], ls);
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
#pragma unroll 1
      for (; bad; bad &= bad - 1) {
        const int p = __builtin_ctzll(bad);
        const uint64_t run = run_at[(at << step_shift) + (p >> run_shift)] +
                             uint32_t((p & ((1 << run_shift) - 1)) * a.slot_bytes);
        add_nonfinite<D, kBf16>(reinterpret_cast<const uint16_t *>(vb + run) + 4 * half,
                                step * kKeys + p <= limit, o);
      }
    }
  }
  float la, lb;
  both<32>(l, &la, &lb);
  l = la + lb;
  if constexpr (!kBf16) {
    both<32>(ls, &la, &lb);
    ls = la + lb;
  }
  if (seen && m == -INFINITY) m = -FLT_MAX;
  if (!here) {
  } else if (u.place >= 0) {
    float *part = a.parts + (int64_t(u.place) * a.kv_heads + h) * part_floats(D, kWaves);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4 *>(part + ((d * 4 + i) * kThreads + tid) * 4) =
            float4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    part[kThreads * (D / 2) + tid] = m;
    part[kThreads * (D / 2 + 1) + tid] = l;
    if constexpr (!kBf16) part[kThreads * (D / 2 + 2) + tid] = ls;
  } else {
    const Row r = row_of(a, u, h, row, half);
#pragma unroll
    for (int d = 0; d < D / 32; ++d) write_row<D, kBf16>(a, r, d, o[d], m, kBf16 ? l : ls);
    write_lse<kBf16>(a, r, m, l);
  }
  record_wave(a.status, err);
}

// Puts the parts of cut tiles together, in their order: a workgroup for 32
// elements of a tile's rows of a KV head, with the lanes' places of attend_kernel.
template <int D, bool kBf16, int kWaves>
__global__ __launch_bounds__(kWaves *kWave, 2) void attend_join_kernel(AttendArgs a) {
  constexpr int kThreads = kWaves * kWave;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int items = *a.num_cuts * a.kv_heads * (D / 32);
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int d = item % (D / 32), h = item / (D / 32) % a.kv_heads;
    const Cut cut = a.cuts[item / (D / 32) / a.kv_heads];
    const Unit u = a.units[cut.unit];
    if (u.row0 + wave * 32 >= u.m * a.group) continue;  // no rows of this wavefront
    const Row r = row_of(a, u, h, u.row0 + wave * 32 + (lane & 31), lane >> 5);
    const int64_t apart = int64_t(a.kv_heads) * part_floats(D, kWaves);
    const float *part = a.parts + (int64_t(u.place) * a.kv_heads + h) * part_floats(D, kWaves);
    const float *ms = part + kThreads * (D / 2) + tid, *sums = ms + kThreads;
    const float *os = part + (d * 4 * kThreads + tid) * 4;
    float m = -INFINITY, l = 0.0f, ls = 0.0f;
#pragma unroll 8
    for (int c = 0; c < cut.parts; ++c) m = fmaxf(m, ms[c * apart]);
    f32x16 o;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = 0.0f;
    // no place of any part is seen: all sums are 0
    const float shift = m == -INFINITY ? 0.0f : m;
#pragma unroll 4
    for (int c = 0; c < cut.parts; ++c) {
      const float w = __builtin_amdgcn_exp2f(ms[c * apart] - shift);
      l = __builtin_fmaf(sums[c * apart], w, l);
      if constexpr (!kBf16) ls = __builtin_fmaf(sums[c * apart + kThreads], w, ls);
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
    write_row<D, kBf16>(a, r, d, o, m, kBf16 ? l : ls);
    if (d == 0) write_lse<kBf16>(a, r, m, l);
  }
}

// ------------------------------------------------------------ host side

// Grid and workspace of a call.
struct AttendPlan {
  int waves, tile_rows;
  int slots;        // workgroups that run at once, for one KV head
  int64_t tiles;    // at most, for one KV head
  int64_t parts;    // of cut tiles at most, for one KV head; 0: none is cut
  bool planned;     // by a kernel before
  size_t units_at, cuts_at, parts_at, bytes;
};

// The workspace is sized for the largest device of this architecture, so that
// its size needs no device.
constexpr int kMaxUnits = 256;

// Places of a table row from which on tiles may be cut.  That takes two more kernels, of
// 10 to 19 us together (the plan 5.8 to 9.7, the join 4.6 to 9.1): single tokens of 1
// request with 1,100, 1,500 and 2,000 places take 23, 24 and 23 us with them and 28, 35
// and 44 without, of 16 requests 30 and 39 against 29 and 46 (1,100, 2,000), of 100
// requests with 2,000 each 172 against 170.  How many places the requests hold is not
// known here: 8 of around 230 take 11.8 us with a table of 480 places and 19 to 20 with
// one of 1,024 or more.
constexpr int kCutKeys = 1024;

// Wavefronts of a workgroup.  Eight share a tile of places among twice the rows and
// keep two more tiles under way, one workgroup a compute unit: a chunk of 2,048 tokens
// behind 14,336 (32 query heads over 8, D 128) takes 507 us against 543, a prompt of
// 4,096 157 against 173, 4 chunks of 2,048 behind 4,096 664 against 711.  Four leave
// fewer lanes idle and spread what does not fill the chip evenly: 405 against 419 for
// 3,000 behind 6,000 (12,000 rows a head: not looked at here), and at D 64, where three
// of them share a compute unit, 848 against 1,206 for 2,300 behind 30,000.
int attend_waves(const lumen_kv_layout *l, int32_t num_reqs, int64_t num_q, int group) {
  const int64_t rows = num_q * group;
  const bool long_ones = rows >= int64_t(num_reqs) * 4096;
  const bool many = rows / (8 * 32) * l->num_kv_heads >= kMaxUnits;
  return l->head_dim == 128 && long_ones && many ? 8 : 4;
}

AttendPlan attend_plan(const lumen_kv_layout *l, int64_t cap, int32_t num_reqs, int64_t num_q,
                       int32_t q_heads, int cus) {
  AttendPlan p;
  const int group = q_heads / l->num_kv_heads;
  p.waves = attend_waves(l, num_reqs, num_q, group);
  p.tile_rows = 32 * p.waves;
  const auto slots = [&](int units) {
    const int n = units * 8 / p.waves / l->num_kv_heads;
    return n < 1 ? 1 : n;
  };
  p.slots = slots(cus < kMaxUnits ? cus : kMaxUnits);
  // at most a part-filled tile for each request beside the full ones
  p.tiles = num_q * group / p.tile_rows + (num_reqs < num_q ? num_reqs : num_q);
  p.parts = 0;
  if (cap >= kCutKeys) {
    // a cut tile has fewer parts than one and a half times its steps over `part`; `part` is
    // at least five eighths of a slot's share of the steps as the plan counts them, and it
    // counts no less than three quarters of a request's: 3.2 for each slot
    p.parts = int64_t(p.slots) * 4;
    const int64_t most = p.tiles * (cap / kMinPartKeys + 2);
    if (p.parts > most) p.parts = most;
  }
  p.planned = p.parts > 0 || p.tiles > slots(kMaxUnits);
  const auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
  p.units_at = 256;  // the number of cuts stands first
  p.cuts_at = p.units_at + up(size_t(p.tiles + p.parts) * sizeof(Unit));
  p.parts_at = p.cuts_at + up(size_t(p.parts / 2 + 1) * sizeof(Cut));
  p.bytes = !p.planned ? 0
                       : p.parts_at + size_t(p.parts) * l->num_kv_heads *
                                          part_floats(l->head_dim, p.waves) * sizeof(float);
  return p;
}

// A grid of more threads than a launch takes.
bool too_many_threads(const AttendPlan &p, int32_t kv_heads) {
  return (p.tiles + p.parts) > int64_t(UINT32_MAX) / (int64_t(kv_heads) * p.waves * kWave);
}

struct AttendKernels {
  void (*main)(AttendArgs);
  void (*join)(AttendArgs);
};

template <int D, int kWaves>
AttendKernels attend_kernels(bool bf16) {
  return bf16 ? AttendKernels{attend_kernel<D, true, kWaves>, attend_join_kernel<D, true, kWaves>}
              : AttendKernels{attend_kernel<D, false, kWaves>,
                              attend_join_kernel<D, false, kWaves>};
}

}  // namespace

extern "C" {

size_t lumen_paged_attend_workspace_bytes(const lumen_kv_layout *layout, int32_t bt_cols,
                                          int32_t num_reqs, int64_t num_tokens, int32_t max_new,
                                          int32_t num_q_heads) {
  Pages pages;
  if (check_pages(layout, 0, 1, &pages) != LUMEN_OK ||
      check_queries(layout, bt_cols, num_reqs, num_tokens, max_new, num_q_heads) != LUMEN_OK)
    return 0;
  const AttendPlan p = attend_plan(layout, places_of(layout, bt_cols), num_reqs, num_tokens,
                                   num_q_heads, kMaxUnits);
  return too_many_threads(p, layout->num_kv_heads) ? 0 : p.bytes;
}

int lumen_paged_attend(const lumen_kv_layout *layout, int32_t layer, const void *d_cache,
                       const int32_t *d_block_tables, int32_t bt_cols, const int32_t *d_lens,
                       const int32_t *d_cu, int32_t num_reqs, const lumen_attn_rows *q,
                       int64_t num_tokens, int32_t max_new, int32_t dtype, int32_t num_q_heads,
                       float scale, void *d_out, float *d_lse, void *d_workspace,
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
  const int32_t kv_heads = layout->num_kv_heads;
  const int64_t cap = places_of(layout, bt_cols);
  if (too_many_threads(attend_plan(layout, cap, num_reqs, num_tokens, num_q_heads, kMaxUnits),
                       kv_heads))
    return LUMEN_ERR_UNSUPPORTED;
  if (num_reqs == 0 || num_tokens == 0) return LUMEN_OK;
  if (!d_lens || !d_cu || !d_out || (!d_block_tables && bt_cols > 0) ||
      (!d_cache && layout->num_blocks > 0))
    return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_cache, 16) || !aligned(d_out, 16) || !aligned(d_workspace, 16) ||
      !aligned(d_lens, 4) || !aligned(d_cu, 4) || !aligned(d_block_tables, 4) ||
      !aligned(d_lse, 4))
    return LUMEN_ERR_MISALIGNED;
  const size_t need = lumen_paged_attend_workspace_bytes(layout, bt_cols, num_reqs, num_tokens,
                                                         max_new, num_q_heads);
  if (need > (d_workspace ? workspace_bytes : 0)) return LUMEN_ERR_INVALID_ARG;
  // Workgroups read these while others write.  Queries in their results' place are read
  // and written by the same wavefront alone, in that order.
  const int32_t head_dim = layout->head_dim;
  const size_t heads = size_t(num_tokens) * size_t(num_q_heads);
  const size_t words = size_t(num_reqs) * sizeof(int32_t);
  const bool in_place = q->d_base == d_out &&
                        (num_q_heads == 1 || q->head_stride == head_dim) &&
                        (num_tokens == 1 || q->token_stride == int64_t(num_q_heads) * head_dim);
  const Span queries = span_of(q, num_tokens, num_q_heads, head_dim);
  if (overlap({{d_out, heads * size_t(head_dim) * 2},
               {d_lse, d_lse ? heads * sizeof(float) : 0},
               {d_workspace, need},
               {d_status, sizeof(int32_t)}},
              {{static_cast<const uint8_t *>(d_cache) + int64_t(layer) * 2 * pages.half,
                size_t(2 * pages.half)},
               {in_place ? nullptr : queries.at, in_place ? 0 : queries.bytes},
               {d_block_tables, words * size_t(bt_cols)},
               {d_lens, words},
               {d_cu, words + sizeof(int32_t)}}))
    return LUMEN_ERR_INVALID_ARG;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  const AttendPlan p = attend_plan(layout, cap, num_reqs, num_tokens, num_q_heads, cus);
  (void)hipGetLastError();
  AttendArgs a;
  static_cast<Call &>(a) =
      call_of(layout, pages, layer, d_cache, d_block_tables, bt_cols, d_lens, d_cu, num_reqs, q,
              num_tokens, max_new, num_q_heads, scale, d_status);
  a.out = static_cast<uint16_t *>(d_out);
  a.lse = d_lse;
  a.tile_rows = p.tile_rows;
  char *ws = static_cast<char *>(d_workspace);
  a.units = p.planned ? reinterpret_cast<Unit *>(ws + p.units_at) : nullptr;
  a.num_units = int32_t(p.tiles + p.parts);
  a.slots = p.slots;
  a.num_cuts = reinterpret_cast<int32_t *>(ws);
  a.cuts = reinterpret_cast<Cut *>(ws + p.cuts_at);
  a.max_parts = int32_t(p.parts);
  a.parts = reinterpret_cast<float *>(ws + p.parts_at);
  const bool bf = dtype == LUMEN_ATTN_BF16;
  const int D = layout->head_dim;
  const AttendKernels kernels = D == 64        ? attend_kernels<64, 4>(bf)
                                : p.waves == 4 ? attend_kernels<128, 4>(bf)
                                               : attend_kernels<128, 8>(bf);
  const dim3 threads(unsigned(p.waves * kWave));
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p.planned)
    hipLaunchKernelGGL(attend_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, a);
  hipLaunchKernelGGL(kernels.main, dim3(unsigned((p.tiles + p.parts) * kv_heads)), threads, 0, s,
                     a);
  if (p.parts) {
    int64_t items = p.parts / 2 * kv_heads * (D / 32);
    if (items > 4 * cus) items = 4 * cus;
    hipLaunchKernelGGL(kernels.join, dim3(unsigned(items < 1 ? 1 : items)), threads, 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

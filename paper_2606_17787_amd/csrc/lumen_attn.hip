// Serving operators for MI355X (gfx950): block tables and slot maps, the
// paged 4-bit KV cache's append, read-back and decode attention.
//
// The operations, the 4-bit row format and the errors are specified in
// include/lumen_attn.h.

#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>
#include <stdint.h>

#include "lumen_attn.h"
#include "lumen_attn_common.h"

namespace {

using namespace lumen_attn_detail;

// ---------------------------------------------------------------- slots

constexpr int kSlotThreads = 256;
// Consecutive tokens that a thread maps at a time, one page lookup after another
// (8 new tokens take 4.7 us with 2, 6.4 with 4 and 9.5 with 8; 1,024 prompts of
// 512 tokens 16.2, 16.8 and 16.1 with two workgroups a compute unit).
constexpr int kSlotTokens = 2;
constexpr uint32_t kHeld = 0x7fffffffu;  // token and page sums are held to this

// Sums of counts held to kHeld: associative, so any order of the scan gives
// the same.
__device__ __forceinline__ uint32_t add_held(uint32_t a, uint32_t b) {
  const uint32_t s = a + b;  // both at most 2^31 - 1
  return s < kHeld ? s : kHeld;
}

struct SlotArgs {
  const int32_t *start, *end, *have;
  int32_t num_reqs;
  int32_t *bt;
  int32_t bt_cols, block_size;
  int64_t num_blocks;
  const int32_t *free_ids;
  const int64_t *free_count;
  int64_t free_cap;
  int64_t *slots;
  int64_t num_slots;
  int32_t *cu, *lens;
  int64_t *free_left;
  int32_t *status;
};

struct SlotReq {
  uint32_t tokens;  // of the packed order
  uint32_t need;    // new pages it asks for
  int32_t first;    // its first new page
  bool range;       // refused with RANGE
};

// tokens >= 0; divided without the sign, in 32 bits
__device__ __forceinline__ int32_t pages_of(int32_t tokens, int32_t bs) {
  const uint32_t whole = uint32_t(tokens) / uint32_t(bs);
  return int32_t(whole + (whole * uint32_t(bs) != uint32_t(tokens)));
}

__device__ __forceinline__ SlotReq slot_req(const SlotArgs &a, int r) {
  const int32_t s = a.start[r], e = a.end[r], h = a.have ? a.have[r] : s;
  SlotReq q{0, 0, 0, true};
  if (s < 0 || e < s || h < 0) return q;
  q.tokens = uint32_t(e - s);
  const int32_t last = pages_of(e, a.block_size);
  q.first = pages_of(h, a.block_size);
  if (last > a.bt_cols) return q;
  q.range = false;
  q.need = last > q.first ? uint32_t(last - q.first) : 0u;
  return q;
}

// One launch, a memory-latency-bound one for a decode step: every workgroup
// scans the requests' token and page counts into LDS (no second launch, no
// wait for one), then the grid strides over the packed tokens and the new
// pages.  A token finds its request by bisection over the prefix in LDS; the
// page of a token that is new is read from the free list and not from the
// table, so the order in which workgroups write the table does not matter.
__global__ __launch_bounds__(kSlotThreads) void slots_kernel(SlotArgs a) {
  extern __shared__ uint32_t lds[];
  uint32_t *cu = lds;                      // [R + 1] packed token prefix
  uint32_t *base = lds + a.num_reqs + 1;   // [R + 1] new page prefix
  __shared__ uint32_t part[2][kSlotThreads / kWave];
  __shared__ uint32_t used;
  const int tid = threadIdx.x, R = a.num_reqs;
  const int per = (R + kSlotThreads - 1) / kSlotThreads;
  const int r0 = tid * per < R ? tid * per : R;
  const int r1 = r0 + per < R ? r0 + per : R;
  int err = LUMEN_OK;
  uint32_t t = 0, p = 0;
  for (int r = r0; r < r1; ++r) {
    const SlotReq q = slot_req(a, r);
    t = add_held(t, q.tokens);
    p = add_held(p, q.need);
    if (q.range) err = LUMEN_ERR_RANGE;
  }
  // inclusive scan over the wavefront's lanes, then over the wavefronts
  uint32_t ti = t, pi = p;
  for (int o = 1; o < kWave; o <<= 1) {
    const uint32_t tu = __shfl_up(ti, o), pu = __shfl_up(pi, o);
    if ((tid & (kWave - 1)) >= o) {
      ti = add_held(ti, tu);
      pi = add_held(pi, pu);
    }
  }
  if ((tid & (kWave - 1)) == kWave - 1) {
    part[0][tid / kWave] = ti;
    part[1][tid / kWave] = pi;
  }
  if (tid == 0) used = 0;
  __syncthreads();
  uint32_t tb = 0, pb = 0;
  for (int w = 0; w < tid / kWave; ++w) {
    tb = add_held(tb, part[0][w]);
    pb = add_held(pb, part[1][w]);
  }
  const uint32_t tx = __shfl_up(ti, 1), px = __shfl_up(pi, 1);
  if (tid & (kWave - 1)) {
    tb = add_held(tb, tx);
    pb = add_held(pb, px);
  }
  int64_t count64 = *a.free_count;
  if (count64 > a.free_cap) count64 = a.free_cap;
  if (count64 < 0) count64 = 0;
  // pages that can be granted: below kHeld, so that a held sum never is
  const uint32_t count = count64 < kHeld ? uint32_t(count64) : kHeld - 1;
  const bool first_wg = blockIdx.x == 0;
  uint32_t mine = 0;
  for (int r = r0; r < r1; ++r) {
    const SlotReq q = slot_req(a, r);
    cu[r] = tb;
    base[r] = pb;
    tb = add_held(tb, q.tokens);
    pb = add_held(pb, q.need);
    const bool got = !q.range && (q.need == 0 || pb <= count);
    if (got && q.need) mine = pb;
    if (!got && !q.range) err = err < LUMEN_ERR_CAPACITY ? err : LUMEN_ERR_CAPACITY;
    if (first_wg) {
      a.cu[r] = int32_t(cu[r]);
      a.lens[r] = got ? a.end[r] : a.start[r];
    }
  }
  if (tid == kSlotThreads - 1) {
    // the last thread's running sums are the totals: threads past the last
    // request carry them on
    cu[R] = tb;
    base[R] = pb;
  }
  if (mine) atomicMax(&used, mine);
  __syncthreads();
  const uint32_t total = cu[R];
  if (first_wg && tid == 0) {
    a.cu[R] = int32_t(total);
    *a.free_left = count64 - int64_t(used);
    if ((a.slots && int64_t(total) > a.num_slots) || total == kHeld)
      err = err < LUMEN_ERR_CAPACITY ? err : LUMEN_ERR_CAPACITY;
  }

  const int64_t grid = int64_t(gridDim.x) * kSlotThreads;
  const int64_t me = int64_t(blockIdx.x) * kSlotThreads + tid;
  // a thread's tokens are consecutive: the request is looked for once, the page
  // once each block_size tokens
  for (int64_t i0 = me * kSlotTokens; i0 < a.num_slots; i0 += grid * kSlotTokens) {
    int r = -1;
    uint32_t end = 0;          // of request r's tokens
    int32_t page = 0, pos = 0; // of the token
    int32_t id = -1;           // of the page, -1 where there is none
    for (int k = 0; k < kSlotTokens; ++k) {
      const int64_t i = i0 + k;
      if (i >= a.num_slots) break;
      int64_t slot = -1;
      if (i < int64_t(total)) {
        const uint32_t u = uint32_t(i);
        const bool other = u >= end;
        if (other) {
          int lo = r + 1, hi = R - 1;  // last r with cu[r] <= u
          while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (cu[mid] <= u)
              lo = mid;
            else
              hi = mid - 1;
          }
          r = lo;
          end = cu[r + 1];
          const uint32_t tok = uint32_t(a.start[r]) + (u - cu[r]);
          page = int32_t(tok / uint32_t(a.block_size));
          pos = int32_t(tok - uint32_t(page) * uint32_t(a.block_size));
        } else if (++pos == a.block_size) {
          pos = 0;
          ++page;
        }
        if (other || pos == 0) {
          const SlotReq q = slot_req(a, r);
          const uint32_t b = base[r];
          id = -1;
          if (!q.range && (q.need == 0 || add_held(b, q.need) <= count)) {
            // where nothing is new, every page is in the table
            id = q.need && page >= q.first
                     ? a.free_ids[count64 - 1 - b - (page - q.first)]
                     : a.bt[int64_t(r) * a.bt_cols + page];
            if (id < 0 || id >= a.num_blocks) {
              id = -1;
              err = err < LUMEN_ERR_BLOCK_ID ? err : LUMEN_ERR_BLOCK_ID;
            }
          }
        }
        if (id >= 0) slot = int64_t(id) * a.block_size + pos;
      }
      a.slots[i] = slot;
    }
  }
  // new pages: list places [0, used)
  for (int64_t i = me; i < int64_t(used); i += grid) {
    const uint32_t u = uint32_t(i);
    int lo = 0, hi = R - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (base[mid] <= u)
        lo = mid;
      else
        hi = mid - 1;
    }
    const SlotReq q = slot_req(a, lo);
    const int32_t id = a.free_ids[count64 - 1 - u];
    if (id >= 0 && id < a.num_blocks)
      a.bt[int64_t(lo) * a.bt_cols + q.first + int32_t(u - base[lo])] = id;
    else
      err = err < LUMEN_ERR_BLOCK_ID ? err : LUMEN_ERR_BLOCK_ID;
  }
  record_wave(a.status, err);
}

// ------------------------------------------------------- append and read

constexpr int kRowThreads = 256;

// What append and read need of the layer's part of the cache.
struct RowArgs {
  uint8_t *k, *v;  // K and V of the layer
  Rows rk, rv;
  const int64_t *slots;
  int64_t slot_limit;
  int32_t block_size, heads;
  int32_t block_shift;  // of block_size, or -1 where it is no power of two
  bool hnd;
  uint32_t tokens;
  uint32_t at_once;  // tokens that the grid takes at a time
  int32_t *status;
};

// A row's lanes: the same head of K or V for each of their tokens, so that a
// token costs no division and one multiplication of addresses.
template <int kRow, int kLanes>
struct RowLanes {
  uint32_t t;      // the first token
  int lane;        // in the row
  uint16_t *row;   // of token t, at the lane's 8 elements
  int64_t step;    // to the row of token t + at_once
  uint8_t *cached; // of slot 0, the row

  __device__ __forceinline__ explicit RowLanes(const RowArgs &a) {
    constexpr uint32_t kRows = kRowThreads / kLanes;
    const uint32_t per_token = 2u * uint32_t(a.heads);
    const uint32_t r = blockIdx.x * kRows + threadIdx.x / kLanes;
    t = r / per_token;
    lane = threadIdx.x % kLanes;
    const uint32_t kvh = r - t * per_token;
    const bool is_v = kvh >= uint32_t(a.heads);
    const uint32_t h = is_v ? kvh - a.heads : kvh;
    const Rows &rows = is_v ? a.rv : a.rk;
    row = rows.base + (int64_t(t) * rows.token + int64_t(h) * rows.head + lane * 8);
    step = int64_t(a.at_once) * rows.token;
    cached = (is_v ? a.v : a.k) + uint64_t(h) * (a.hnd ? a.block_size : 1) * kRow;
    if (t >= a.at_once) t = a.tokens;  // past the last whole token
  }
  __device__ __forceinline__ uint8_t *at(const RowArgs &a, int64_t slot) const {
    const uint32_t all = uint32_t(a.heads) * kRow;
    if (!a.hnd) return cached + uint64_t(slot) * all;
    const int64_t block = a.block_shift >= 0 ? slot >> a.block_shift
                          : slot <= UINT32_MAX
                              ? int64_t(uint32_t(slot) / uint32_t(a.block_size))
                              : slot / a.block_size;
    const uint32_t pos = uint32_t(slot - block * a.block_size);
    return cached + uint64_t(block) * a.block_size * all + pos * kRow;
  }
};

// x of the other lanes of a quarter, by data movement within its group of
// kGroup lanes: call it with o = 1, 2, 4 below kGroup and join as it goes.
template <int kLane>
__device__ __forceinline__ float across(float x) {
  // lanes swapped by 1, by 2, and mirrored in 8 (which of the other four it is
  // does not matter once each four are joined)
  constexpr int kControl = kLane == 1 ? 0xb1 : kLane == 2 ? 0x4e : 0x141;
  return __builtin_bit_cast(
      float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kControl, 0xf, 0xf,
                                         true));
}

// Quantises rows: D/8 lanes a row, 8 elements a lane (one 16-byte load, one
// dword of codes).  Memory-bound, 2*D bytes in and D/2 + 16 out a row, as long as
// its arithmetic stays under 100 or so instructions a load: 16,411 tokens of 8
// heads, D 128, take 18.7 to 20.7 us, 4.3 to 4.7 TB/s, and their reading back 16.5 to
// 16.9, 5.2 to 5.3 TB/s (a large library copy: 4.5 to 5.0).
template <int D, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void append4_kernel(RowArgs a) {
  constexpr int kLanes = D / 8;        // lanes of a row
  constexpr int kGroup = kLanes / 4;   // lanes of a quarter
  constexpr int kRow = D / 2 + 16;
  constexpr float kMost = float(LUMEN_ATTN_KV4_MAX);
  RowLanes<kRow, kLanes> r(a);
  int err = LUMEN_OK;
  for (uint32_t t = r.t; t < a.tokens; t += a.at_once, r.row += r.step) {
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.slot_limit) {
      if (slot >= 0) err = LUMEN_ERR_BLOCK_ID;
      continue;  // a whole row's lanes, and no lane reads another row's
    }
    float x[8];
    unpack8<kBf16>(*reinterpret_cast<const uint4 *>(r.row), x);
    bool nan = false;
#pragma unroll
    for (int k = 0; k < 8; k += 2) nan |= __builtin_isunordered(x[k], x[k + 1]);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __builtin_amdgcn_fmed3f(x[k], -kMost, kMost);
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) lo = fminf(lo, x[k]), hi = fmaxf(hi, x[k]);
    if (nan) hi = INFINITY;  // no element is: the quarter's sign of a NaN
    lo = fminf(lo, across<1>(lo)), hi = fmaxf(hi, across<1>(hi));
    if constexpr (kGroup > 2) lo = fminf(lo, across<2>(lo)), hi = fmaxf(hi, across<2>(hi));
    if constexpr (kGroup > 4) lo = fminf(lo, across<4>(lo)), hi = fmaxf(hi, across<4>(hi));
    const _Float16 ah = _Float16((hi - lo) * (1.0f / 15.0f));
    const float A = float(ah);
    const _Float16 bh = _Float16(lo - 64.0f * A);
    const float first = float(bh) + 64.0f * A;
    const float inv = A > 0.0f ? 1.0f / A : 0.0f;
    // held to 0..15 and added to 2^23, a code is rounded to nearest even and
    // stands in the lowest byte
    uint32_t c[8];
#pragma unroll
    for (int k = 0; k < 8; ++k)
      c[k] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_fmed3f((x[k] - first) * inv, 0.0f, 15.0f) + 8388608.0f);
    const auto bytes = [&](int k) {  // codes k, k + 2, k + 4, k + 6
      const uint32_t low = __builtin_amdgcn_perm(c[k + 2], c[k], 0x0c0c0400);
      const uint32_t high = __builtin_amdgcn_perm(c[k + 6], c[k + 4], 0x04000c0c);
      return low | high;
    };
    uint32_t codes = bytes(0) | bytes(1) << 4;
    uint32_t pair = bits(ah) | uint32_t(bits(bh)) << 16;
    if (hi == INFINITY) codes = 0, pair = 0x7e007e00u;
    uint8_t *row = r.at(a, slot);
    reinterpret_cast<uint32_t *>(row)[r.lane] = codes;
    if (r.lane % kGroup == 0)
      reinterpret_cast<uint32_t *>(row + D / 2)[r.lane / kGroup] = pair;
  }
  record_wave(a.status, err);
}

template <int D, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void read4_kernel(RowArgs a) {
  constexpr int kLanes = D / 8;
  constexpr int kGroup = kLanes / 4;
  constexpr int kRow = D / 2 + 16;
  RowLanes<kRow, kLanes> r(a);
  int err = LUMEN_OK;
  for (uint32_t t = r.t; t < a.tokens; t += a.at_once, r.row += r.step) {
    const int64_t slot = a.slots[t];
    uint4 raw{0, 0, 0, 0};
    if (slot >= 0 && slot < a.slot_limit) {
      const uint8_t *row = r.at(a, slot);
      const uint32_t codes = reinterpret_cast<const uint32_t *>(row)[r.lane];
      const uint32_t pair =
          reinterpret_cast<const uint32_t *>(row + D / 2)[r.lane / kGroup];
      const float A = float(half_of(pair)), B = float(half_of(pair >> 16));
      float x[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        x[k] = float(_Float16(
            A * float(64 + ((codes >> (4 * k)) & 15)) + B));
      raw = pack8<kBf16>(x);
    } else if (slot >= 0) {
      err = LUMEN_ERR_BLOCK_ID;
    }
    *reinterpret_cast<uint4 *>(r.row) = raw;
  }
  record_wave(a.status, err);
}

// --------------------------------------------------------------- decode

struct DecodeArgs {
  const uint8_t *k, *v;  // of the layer
  const int32_t *bt;
  int32_t bt_cols, block_size;
  int64_t num_blocks;
  const int32_t *lens;
  int32_t num_reqs, heads, group;
  bool hnd, bf16;
  Rows q;
  float scale_log2;
  uint16_t *out;
  int32_t *status;
  int32_t wg_heads, wg_blocks;  // heads and key blocks of a workgroup
  int32_t workers;              // workgroups of one set of heads
  int2 *spans;   // [num_reqs] the workers of a request's first and last unit
  float *parts;  // [sets of heads][workers][2][wg_heads][part_floats(D)]
};

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float float4v __attribute__((ext_vector_type(4)));

constexpr int kDecodeWaves = 8;
constexpr int kDecodeThreads = kDecodeWaves * kWave;
constexpr int kBlockKeys = 32;  // keys a wavefront takes at a time
constexpr int kSegments = kWave;
// A round's steps, tiles and blocks of 32 keys.
constexpr int kRoundSteps = 128, kTiles = 1024, kLive = 512, kLast = 256;
// A unit of work, in the workgroup's blocks.  Shorter ones share more evenly and cut
// more requests, whose parts the second kernel joins: with 1, 2, 4 and 8 of them 256
// requests around 2,048 tokens take 179, 180, 180 and 186 us, 512 around 4,096 of one
// KV head 118, 115, 118 and 124, 512 around 100 of 8 heads 51, 50, 52 and 59, four
// around 1,000 24, 21, 23 and 28.
constexpr int kUnitBlocks = 4;
constexpr int kQueries = 16;    // columns of a product
// Weights are 2^(s - m + kBias) with s - m at most kRise, rounded to 16-bit floats
// for the products with V; their own sum is taken before that, in 32 bits.  They
// stay under 2^14.  Where the maximum is not behind, one keeps its 11 bits down to
// 2^-20 of the largest and vanishes under 2^-31 of it, so that n such keys lose at
// most n * 2^-31 of the values' size.
constexpr float kRise = 8.0f, kBias = 6.0f;

template <int kE, bool kBf16>
__device__ __forceinline__ void store_out(uint16_t *to, const float *x) {
  if constexpr (kE == 4) {
    *reinterpret_cast<uint2 *>(to) =
        uint2{uint32_t(rounded<kBf16>(x[0])) | uint32_t(rounded<kBf16>(x[1])) << 16,
              uint32_t(rounded<kBf16>(x[2])) | uint32_t(rounded<kBf16>(x[3])) << 16};
  } else {
#pragma unroll
    for (int j = 0; j < kE; j += 8)
      *reinterpret_cast<uint4 *>(to + j) = pack8<kBf16>(x + j);
  }
}

// Floats of one partial result: kQueries rows of D sums, then a maximum and a
// sum for each.
constexpr int part_floats(int D) { return D * kQueries + 2 * kQueries; }

__device__ __forceinline__ half2v as_half2(uint32_t x) {
  return __builtin_bit_cast(half2v, x);
}

// Codes of four places in each 16-bit half of w (element i of the low half
// and of the high half in result i) as 64 + q: the code in bits 4..7 of a
// 16-bit float whose last place is 1/16 of its unit, 2^6 * (1 + q / 64).  `one`
// is kCodeOne, `mask` kCodeMask, in registers: an and-or takes no literals.
constexpr uint32_t kCodeMask = 0x00f000f0u, kCodeOne = 0x54005400u;
__device__ __forceinline__ void codes4(uint32_t w, uint32_t mask, uint32_t one,
                                       half2v *x) {
  x[0] = as_half2(((w << 4) & mask) | one);
  x[1] = as_half2((w & mask) | one);
  x[2] = as_half2(((w >> 4) & mask) | one);
  x[3] = as_half2(((w >> 8) & mask) | one);
}

// Maximum and sum over the four lanes of one query (l % 16).
__device__ __forceinline__ float quad_max(float x) {
  float a, b;
  both<16>(x, &a, &b);
  both<32>(fmaxf(a, b), &a, &b);
  return fmaxf(a, b);
}
__device__ __forceinline__ float quad_sum(float x) {
  float a, b;
  both<16>(x, &a, &b);
  both<32>(a + b, &a, &b);
  return a + b;
}

// What a row's sums are multiplied by.  m is -infinity where no key counted, and
// the row is zeros.  It is at least -FLT_MAX where one did: if the sum of the
// weights is 0 then, every score was -infinity, and the row is NaN as the formula
// has it.
__device__ __forceinline__ float inverse(float m, float l) {
  return m == -INFINITY ? 0.0f : 1.0f / l;
}

// Decode attention, bound by the cache's bytes: D/2 + 16 a row, read once.
//
// Work.  A workgroup takes wg_heads KV heads, those that lie side by side in a
// token-major page, times wg_blocks blocks of 32 keys: one head and one block
// a wavefront.  A worker, one a CU, takes an equal share of the requests' units
// of kUnitBlocks such steps, whatever the requests' lengths, so a share may
// start and end inside a request; its partial results go to d_workspace and
// decode4_join_kernel puts them together in a fixed order.
//
// Loads.  The rows of a step come straight into LDS, 16 bytes a lane in the
// order of their addresses, kStages steps in turn: what is in flight takes no
// registers, and each cache line is asked for once (a wavefront that reads its
// own head's 80 bytes out of each 640 makes the first-level cache fetch 1.5
// lines for 80 bytes: 2.2 TB/s).  Where a round's rows start, and which of its
// keys count, is laid out in LDS before the round, so that a step's addresses
// are one read and one addition.
//
// One block of 32 keys: scores^T = K Q^T and sums^T = V^T P^T by 16x16x32
// products of 16-bit floats, queries across (the heads of the group, up to 16).
// A lane reads its key's codes with one LDS load and holds them in the
// product's order at once, because the sum over head_dim may run in any order:
// lanes l / 16 take the four quarters of the row, each with one pair (A, B).
// The scores come out as the weights' operand goes in when the keys are taken
// in the same order again, so the weights never leave their lanes.  For V a
// lane holds D/16 consecutive elements of 8 keys, all of one quarter.  Values
// are exact: code and pair give the stored value by one fused multiply-add that
// rounds as the format says.
//
// Measured, D 128: 256 requests around 2,048 tokens, 32 query heads over 8, 181
// us, 4.9 TB/s; 512 around 4,096 of 8 over one, 118 us, 3.8 TB/s (a wavefront's own
// rows, 1,280 bytes of a page at a time); three of 100,000, 96 us, 4.1 TB/s (the join
// is 4.5 us of it).  D 256, 64 requests of 4,096 tokens, 32 query heads over 8: 126
// us, 4.8 TB/s, with two registers spilled where heads lie together.
//
// kPrivate: one head a workgroup, whose wavefronts load their own blocks' rows and
// wait for nobody else's.  Rows are not kept in caches (nt), also where a workgroup
// takes a part of the heads and shares lines with others: 64 requests around 2,048
// tokens, 64 query heads over 16, D 128, take 96 us, and 103 with rows kept; 32 at D
// 256 94 and 97; 64 of 32 over 32 176 both.
template <int D, bool kPrivate>
__global__ __launch_bounds__(kDecodeThreads, 2) void decode4_kernel(DecodeArgs a) {
  constexpr int kRow = D / 2 + 16;
  constexpr int kSteps = D / 32;  // products over head_dim
  constexpr int kE = D / 16;      // elements of V a lane holds of a key
  constexpr int kStages = D == 64 ? 4 : D == 128 ? 3 : 2;
  constexpr int kParts = kRow / 16;  // 16-byte pieces of a row
  constexpr int kIssues = 2 * kBlockKeys * kParts / kWave;
  constexpr int kStage = kDecodeWaves * 2 * kBlockKeys * kRow;  // bytes
  __shared__ __attribute__((aligned(16))) uint8_t ring[kStages * kStage];
  // of the steps of a round: where their tiles' rows start (bytes from the
  // layer's K), which keys of each block of 32 count, and the part of the round
  // that a step belongs to, with kLast in its last step
  __shared__ uint64_t tile_at[kTiles];
  __shared__ uint32_t live_keys[kLive];
  __shared__ int step_part[kRoundSteps];
  __shared__ float lds_m[kDecodeWaves][kQueries], lds_l[kDecodeWaves][kQueries];
  __shared__ uint64_t lds_scan[kDecodeWaves];
  __shared__ uint64_t lds_first;  // of the request that a share starts in
  __shared__ int lds_req;
  // the next kSegments parts of requests in the share: keys [key0, key1) of
  // request r, their steps' places in the round, and whether the request
  // starts (1) and ends (2) in it
  __shared__ uint32_t seg_key0[kSegments], seg_key1[kSegments];
  __shared__ int seg_end[kSegments + 1], seg_flags[kSegments];
  static_assert(kDecodeWaves / 2 * kE * 4 * kWave * int(sizeof(float)) <= kStage,
                "half of the wavefronts' sums fit a stage");

  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = lane & 15, quad = lane >> 4;
  const int worker = blockIdx.x % a.workers, set = blockIdx.x / a.workers;
  const int tiles = (a.group + kQueries - 1) / kQueries;
  const int h0 = set / tiles * a.wg_heads, g0 = set % tiles * kQueries;
  const int rows = a.group - g0 < kQueries ? a.group - g0 : kQueries;
  const int hi = wave % a.wg_heads, kbi = wave / a.wg_heads;
  const bool active = kbi < a.wg_blocks;
  const int step_keys = kBlockKeys * a.wg_blocks;
  const int unit_keys = step_keys * kUnitBlocks;
  int err = LUMEN_OK;
  uint32_t mask, one;  // not to be folded into literals again
  asm("s_mov_b32 %0, %1" : "=s"(mask) : "i"(kCodeMask));
  asm("v_mov_b32 %0, %1" : "=v"(one) : "i"(kCodeOne));

  // ---- the share: units [u0, u1) of all requests' units
  const int64_t cap = int64_t(a.bt_cols) * a.block_size;
  const auto length = [&](int r) __attribute__((always_inline)) {
    const int64_t len = a.num_blocks > 0 ? a.lens[r] : 0;
    return len < 0 ? int64_t(0) : len < cap ? len : cap;
  };
  const auto units_of = [&](int64_t len) __attribute__((always_inline)) {
    return len <= unit_keys ? 1u : uint32_t(len + unit_keys - 1) / uint32_t(unit_keys);
  };
  const int per = (a.num_reqs + kDecodeThreads - 1) / kDecodeThreads;
  const int ra = tid * per < a.num_reqs ? tid * per : a.num_reqs;
  const int rb = ra + per < a.num_reqs ? ra + per : a.num_reqs;
  uint64_t mine = 0;
  for (int r = ra; r < rb; ++r) {
    const int len = a.lens[r];
    if (len < 0 || len > cap) err = err < LUMEN_ERR_RANGE ? err : LUMEN_ERR_RANGE;
    if (len > 0 && a.num_blocks == 0) err = LUMEN_ERR_BLOCK_ID;
    mine += units_of(length(r));
  }
  uint64_t upto = mine;
  for (int o = 1; o < kWave; o <<= 1) {
    const uint64_t x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == kWave - 1) lds_scan[wave] = upto;
  __syncthreads();
  uint64_t total = 0;
  for (int w = 0; w < kDecodeWaves; ++w) {
    if (w < wave) upto += lds_scan[w];
    total += lds_scan[w];
  }
  total = uniform(total);
  const uint64_t shares = total < uint64_t(a.workers) ? total : uint64_t(a.workers);
  if (uint64_t(worker) >= shares) return;  // the whole workgroup
  const uint64_t u0 = total * worker / shares, u1 = total * (worker + 1) / shares;
  if (u0 >= upto - mine && u0 < upto) {
    uint64_t at = upto - mine;
    int r = ra;
    for (;; ++r) {
      const uint64_t c = units_of(length(r));
      if (u0 < at + c) break;
      at += c;
    }
    lds_req = r;
    lds_first = at;
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane(lds_req);
  uint64_t first = uniform(lds_first);  // first unit of request r

  // ---- the pieces of a step that this lane loads: 16 bytes c of the rows of K,
  // then of V, each (token, head, part) in the order of a token-major page
  const uint64_t page_bytes = uint64_t(a.block_size) * a.heads * kRow;
  const uint32_t slot_bytes = (a.hnd ? 1 : a.heads) * kRow;
  // A token's pieces are turned by a number of places that makes the same piece
  // of 16 tokens lie in 16 different sixteenths of the banks' 256 bytes.
  const int pieces = a.wg_heads * kParts;
  const int even = pieces & 15 ? pieces & -pieces : 16;  // gcd(pieces, 16)
  const auto turn = [&](int t) __attribute__((always_inline)) { return (t & 15) * even / 16; };
  // keys of a tile: the largest power of two up to 16 that divides a page
  const int low = a.block_size & -a.block_size;
  const int tile_shift = low >= 16 ? 4 : __builtin_ctz(low);
  int tile[kIssues];       // of the step, that the piece is in; below 0 of V
  uint32_t piece[kIssues]; // its place in a tile's rows of the heads
  const int64_t heads_at = int64_t(a.hnd ? h0 * a.block_size : h0) * kRow;
  const uint8_t *const k_at = a.k + heads_at, *const v_of = a.v + heads_at;
#pragma unroll
  for (int i = 0; i < kIssues; ++i) {
    const int half = kPrivate ? kBlockKeys * kParts : step_keys * pieces;
    int c = kPrivate ? i * kWave + lane : i * kDecodeThreads + tid;
    const bool is_v = c >= half;
    c = is_v ? c - half : c;
    c = c < half ? c : half - 1;  // lanes past the step's end repeat a piece
    int t = c / pieces;
    int x = c - t * pieces - turn(t);
    if (kPrivate) t += kbi * kBlockKeys;
    x = x < 0 ? x + pieces : x;
    tile[i] = t >> tile_shift | (is_v ? INT32_MIN : 0);
    piece[i] = (t & ((1 << tile_shift) - 1)) * slot_bytes + x * 16;
  }
  const auto address = [&](int i, int step_tile) __attribute__((always_inline)) {
    return (tile[i] < 0 ? v_of : k_at) + piece[i] + tile_at[step_tile + (tile[i] & 0xffff)];
  };
  const int step_tiles = step_keys >> tile_shift;
  int round = kTiles / step_tiles;  // steps
  round = round < kLive / a.wg_blocks ? round : kLive / a.wg_blocks;
  round = round < kRoundSteps ? round : kRoundSteps;
  // where the lane finds part `part` of its head's row of token t in a step
  const auto place = [&](int t, int part) __attribute__((always_inline)) {
    int x = hi * kParts + part + turn(t);
    x = x < pieces ? x : x - pieces;
    return uint32_t(t * pieces + x) * 16;
  };
  // offsets into a stage of what the lane reads: K of key n, the same for n + 16;
  // V of keys 4 quad + 0, 1 and + 2, 3, the same for + 16
  constexpr int kVBytes = kE / 2;  // of V's codes
  const int t0 = kPrivate ? 0 : (active ? kbi : 0) * kBlockKeys;
  uint32_t at_k[D == 256 ? 2 : 1], at_v[2], at_kp, at_vp[2];
  at_k[0] = place(t0 + n, quad * (D / 8) / 16) + quad * (D / 8) % 16;
  if constexpr (D == 256) at_k[1] = place(t0 + n, quad * 2 + 1);
  at_kp = place(t0 + n, kParts - 1) + quad * 4;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    at_v[j] = place(t0 + 4 * quad + 2 * j, n * kVBytes / 16) + n * kVBytes % 16;
    at_vp[j] = place(t0 + 4 * quad + 2 * j, kParts - 1) + n / 4 * 4;
  }
  // (turn() is the same for keys 2j and 2j + 1 wherever it is not 0: `even` is
  // at most 8 for any number of pieces of up to 8 heads)
  const uint32_t key_bytes = pieces * 16;
  const uint32_t v_at = (kPrivate ? kBlockKeys : step_keys) * key_bytes;
  constexpr int kOwn = 2 * kBlockKeys * kRow;  // bytes of a wavefront's block

  // ---- Q: 16-bit floats under a power of two of the row's own, which takes its
  // largest element to 2^13..2^14: bf16 has too wide a range for a 16-bit float, and
  // the products with the exact K need one.  Elements down to 2^-27 of the largest
  // keep all their bits; what smaller ones lose is under 2^-38 of the largest, far
  // less than the rounding of the scores' sums to 32 bits.
  half8v q[kSteps];
  float cq = 0.0f;
  uint4 raw[D == 256 ? 1 : kSteps];
  // (for D 256 there are no registers to hold a row as it is, so it is read
  // once more)
  constexpr bool kTwice = D == 256;
  const uint16_t *q_row = nullptr;
  const auto fetch_q = [&](int req) __attribute__((always_inline)) {
    const int row = (h0 + hi) * a.group + g0 + (n < rows ? n : 0);
    q_row = a.q.base + int64_t(req) * a.q.token + row * a.q.head + quad * (D / 4);
    if constexpr (!kTwice) {
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
        raw[i] = *reinterpret_cast<const uint4 *>(q_row + 8 * i);
    }
  };
  const auto take_q = [&]() __attribute__((always_inline)) {
    const auto part = [&](int i, float *x) __attribute__((always_inline)) {
      if constexpr (kTwice) raw[0] = *reinterpret_cast<const uint4 *>(q_row + 8 * i);
      a.bf16 ? unpack8<true>(raw[kTwice ? 0 : i], x) : unpack8<false>(raw[kTwice ? 0 : i], x);
    };
    float big = 0.0f, x[8];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      part(i, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) big = fmaxf(big, fabsf(x[j]));
    }
    big = quad_max(big);
    uint32_t e = __builtin_bit_cast(uint32_t, big) >> 23;  // NaN: not the maximum
    e = e == 255 ? 140 : e < 14 ? 14 : e;
    const float up = __builtin_bit_cast(float, (267 - e) << 23);  // to 2^13..2^14
    // Neither 0 (a masked key's -infinity times it would be NaN) nor infinite (a
    // score of 0 would): a score is at most 2^38 times it, so where it is held up
    // to 2^-126, for a row of zeros under a small scale, the scores stay below
    // 2^-88.
    cq = __builtin_amdgcn_fmed3f(a.scale_log2 * __builtin_bit_cast(float, (e - 13) << 23),
                                 0x1p-126f, FLT_MAX);
    if constexpr (kTwice) asm volatile("" ::: "memory");
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      part(i, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        q[i][2 * j] = _Float16(x[j] * up);
        q[i][2 * j + 1] = _Float16(x[j + 4] * up);
      }
    }
  };
  float4v o[kE];
  float m = -INFINITY, l = 0.0f;
  const auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kE; ++j) o[j] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    m = -INFINITY, l = 0.0f;
  };

  const auto use = [&](const uint8_t *stage, uint32_t live) __attribute__((always_inline)) {
    // everything the block reads, at once: one wait instead of one for each
    uint32_t kc[2][kSteps], kp[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t *row = stage + 16 * t * key_bytes;
      kp[t] = *reinterpret_cast<const uint32_t *>(row + at_kp);
      if constexpr (D == 64) {
        const uint2 x = *reinterpret_cast<const uint2 *>(row + at_k[0]);
        kc[t][0] = x.x, kc[t][1] = x.y;
      } else {
#pragma unroll
        for (int i = 0; i < kSteps; i += 4) {
          const uint4 x = *reinterpret_cast<const uint4 *>(row + at_k[i / 4]);
          kc[t][i] = x.x, kc[t][i + 1] = x.y, kc[t][i + 2] = x.z, kc[t][i + 3] = x.w;
        }
      }
    }
    uint32_t vc[8][kE >= 8 ? kE / 8 : 1], vp[8];  // V: the lane's elements of 8 keys
    const auto read_v = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint8_t *row = stage + v_at + ((j & 1) + (j & 4) * 4) * key_bytes;
        vp[j] = *reinterpret_cast<const uint32_t *>(row + at_vp[j / 2 % 2]);
        row += at_v[j / 2 % 2];
        if constexpr (D == 64) {
          vc[j][0] = *reinterpret_cast<const uint16_t *>(row);
        } else if constexpr (D == 128) {
          vc[j][0] = *reinterpret_cast<const uint32_t *>(row);
        } else {
          const uint2 x = *reinterpret_cast<const uint2 *>(row);
          vc[j][0] = x.x, vc[j][kE / 8 - 1] = x.y;
        }
      }
    };
    // for D 256 there are no registers to hold both at once
    if constexpr (D != 256) {
      read_v();
      __builtin_amdgcn_sched_barrier(0);
    }
    float4v s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      s[t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
      const half2v pair = as_half2(kp[t]);
      const half2v A = {pair[0], pair[0]}, B = {pair[1], pair[1]};
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        half2v x[4];
        codes4(kc[t][i], mask, one, x);
        half8v f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const half2v y = __builtin_elementwise_fma(x[j], A, B);
          f[2 * j] = y[0];
          f[2 * j + 1] = y[1];
        }
        s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f, q[i], s[t], 0, 0, 0);
      }
    }
    if constexpr (D == 256) {
      __builtin_amdgcn_sched_barrier(0);
      read_v();
    }
    if (live != 0xffffffffu) {
      // a key left out has no score, and no value either: its pair may be NaN
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = (live >> (4 * quad + (j < 4 ? j : 12 + j))) & 1;
        if (!in) s[j / 4][j % 4] = -INFINITY;
        if (!in) vp[j] = 0;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = fmaxf(top, s[j / 4][j % 4]);
    top = quad_max(top) * cq;
    m = fmaxf(m, -FLT_MAX);  // the block has a key that counts
    if (__any(top > m + kRise)) {
      const float mn = fmaxf(m, top);
      const float c = __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= c;
#pragma unroll
      for (int j = 0; j < kE; ++j) o[j] *= c;
    }
    const float shift = kBias - m;
    half8v p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = __builtin_amdgcn_exp2f(
          __builtin_fmaf(s[j / 4][j % 4], cq, shift));
      l += x;
      p[j] = _Float16(x);
    }
    half2v A[4], B[4];  // of keys 2j and 2j + 1 of the lane
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      A[j] = as_half2(__builtin_amdgcn_perm(vp[2 * j + 1], vp[2 * j], 0x05040100));
      B[j] = as_half2(__builtin_amdgcn_perm(vp[2 * j + 1], vp[2 * j], 0x07060302));
    }
#pragma unroll
    for (int w = 0; w < kE / 4; ++w) {  // four elements at a time
      half8v f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        half2v x[4];
        codes4(__builtin_amdgcn_perm(vc[2 * j + 1][w / 2], vc[2 * j][w / 2],
                                     w % 2 ? 0x07060302 : 0x05040100),
               mask, one, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const half2v y = __builtin_elementwise_fma(x[e], A[j], B[j]);
          f[e][2 * j] = y[0];
          f[e][2 * j + 1] = y[1];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o[4 * w + e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(f[e], p, o[4 * w + e],
                                                              0, 0, 0);
    }
  };

  const uint32_t ring_at = uint32_t(__builtin_amdgcn_readfirstlane(
      int(reinterpret_cast<uintptr_t>(LDS_PTR(uint8_t, ring))) +
      wave * (kPrivate ? kOwn : kWave * 16)));

  // ---- up to kSegments parts of requests at a time
  uint64_t u = u0;
  while (u < u1) {
    __syncthreads();  // the tables are used again
    if (wave == 0) {
      const int mine_r = r + lane;
      const int64_t len = mine_r < a.num_reqs ? length(mine_r) : 0;
      const uint64_t units = mine_r < a.num_reqs ? units_of(len) : 0;
      uint64_t at = units;  // inclusive over the lanes
      for (int d = 1; d < kWave; d <<= 1) {
        const uint64_t x = __shfl_up(at, d);
        if (lane >= d) at += x;
      }
      const uint64_t f = first + at - units;  // its first unit
      const uint64_t ua = f > u ? f : u, ub = f + units < u1 ? f + units : u1;
      uint32_t k0 = 0, k1 = 0;
      int steps = 0;
      if (ua < ub) {
        const int64_t end = int64_t(ub - f) * unit_keys;
        k0 = uint32_t(ua - f) * uint32_t(unit_keys);
        k1 = uint32_t(end < len ? end : len);
        if (k0 < k1) steps = int((k1 - k0 + step_keys - 1) / step_keys);
        if (a.spans && set == 0 && ua == f) {
          const uint64_t last = (f + units) * shares + total - 1;
          a.spans[mine_r] = int2{worker, int(last / total) - 1};
        }
      }
      int upto_step = steps;
      for (int d = 1; d < kWave; d <<= 1) {
        const int x = __shfl_up(upto_step, d);
        if (lane >= d) upto_step += x;
      }
      seg_key0[lane] = k0;
      seg_key1[lane] = k1;
      seg_end[lane] = upto_step;
      seg_flags[lane] = ua < ub ? (ua == f) | (ub == f + units) << 1 : -1;
      if (lane == kWave - 1) {
        seg_end[kSegments] = upto_step;
        lds_first = f + units;
      }
    }
    __syncthreads();
    const auto read = [](const int &x) __attribute__((always_inline)) { return __builtin_amdgcn_readfirstlane(x); };
    const int steps = read(seg_end[kSegments]);

    // The result of one part; `room` is a stage of the ring that is free.
    const auto finish = [&](int part, uint8_t *room) __attribute__((always_inline)) {
      l = quad_sum(l);
      // the wavefronts of one head together, in the first of them
      if (a.wg_blocks > 1) {
        auto &lds_o = *reinterpret_cast<float(*)[kDecodeWaves / 2][kE][4 * kWave]>(room);
        if (quad == 0) lds_m[wave][n] = m, lds_l[wave][n] = l;
        lds_barrier();
        float mm = m, ll = 0.0f;
        if (active) {
          for (int w = hi; w < a.wg_heads * a.wg_blocks; w += a.wg_heads)
            mm = fmaxf(mm, lds_m[w][n]);
          for (int w = hi; w < a.wg_heads * a.wg_blocks; w += a.wg_heads)
            ll += mm == -INFINITY ? 0.0f
                                  : lds_l[w][n] * __builtin_amdgcn_exp2f(lds_m[w][n] - mm);
        }
        const float c = mm == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mm);
        m = mm;
        l = ll;
#pragma unroll
        for (int j = 0; j < kE; ++j) o[j] *= c;
        for (int left = a.wg_blocks; left > 1;) {
          const int keep = (left + 1) / 2;
          if (kbi >= keep && kbi < left) {
#pragma unroll
            for (int j = 0; j < kE; ++j)
              *reinterpret_cast<float4v *>(
                  &lds_o[(kbi - keep) * a.wg_heads + hi][j][4 * lane]) = o[j];
          }
          lds_barrier();
          if (kbi < left - keep) {
#pragma unroll
            for (int j = 0; j < kE; ++j)
              o[j] += *reinterpret_cast<const float4v *>(
                  &lds_o[kbi * a.wg_heads + hi][j][4 * lane]);
          }
          lds_barrier();
          left = keep;
        }
      }
      const int flags = read(seg_flags[part]), req = r + part;
      if (kbi == 0 && n < rows) {
        if (flags == 3) {  // the whole request
          const float inv = inverse(m, l);
          uint16_t *out = a.out +
                          ((int64_t(req) * a.heads + h0 + hi) * a.group + g0 + n) * D +
                          4 * quad * kE;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float x[kE < 8 ? 8 : kE];
#pragma unroll
            for (int j = 0; j < kE; ++j) x[j] = o[j][i] * inv;
            uint16_t *to = out + i * kE;
            a.bf16 ? store_out<kE, true>(to, x) : store_out<kE, false>(to, x);
          }
        } else {
          // a share may end one request and start another: two places
          float *into = a.parts + (((int64_t(set) * a.workers + worker) * 2 + (flags & 1)) *
                                       a.wg_heads + hi) * part_floats(D);
          float *to = into + n * D + 4 * quad * kE;
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kE; j += 4)
              *reinterpret_cast<float4v *>(to + i * kE + j) =
                  float4v{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
          if (quad == 0) {
            into[D * kQueries + n] = m;
            into[D * kQueries + kQueries + n] = l;
          }
        }
      }
      clear();
    };
    // zeros for requests without keys, which have no steps
    for (int p = 0; p < kSegments && read(seg_flags[p]) >= 0; ++p)
      if (read(seg_end[p]) == (p ? read(seg_end[p - 1]) : 0))
        for (int i = tid; i < a.wg_heads * rows * (D / 8); i += kDecodeThreads) {
          const int head = i / (rows * (D / 8)), at = i - head * (rows * (D / 8));
          uint16_t *out =
              a.out + ((int64_t(r + p) * a.heads + h0 + head) * a.group + g0) * D;
          reinterpret_cast<uint4 *>(out)[at] = uint4{0, 0, 0, 0};
        }

    bool fresh = true;  // the next step starts a part
    clear();
    for (int base = 0; base < steps; base += round) {
      const int count = steps - base < round ? steps - base : round;
      // ---- the tables of the round's steps
      __syncthreads();  // those before are done with
      const auto part_of = [&](int step) __attribute__((always_inline)) {
        int lo = 0, hi = kSegments - 1;  // the first part that ends after `step`
        while (lo < hi) {
          const int mid = (lo + hi) / 2;
          if (seg_end[mid] > step)
            hi = mid;
          else
            lo = mid + 1;
        }
        return lo;
      };
      const auto key_of = [&](int part, int step) __attribute__((always_inline)) {
        const int before = part ? seg_end[part - 1] : 0;
        return seg_key0[part] + uint32_t(step - before) * uint32_t(step_keys);
      };
      for (int i = tid; i < count * step_tiles; i += kDecodeThreads) {
        const int step = i / step_tiles, part = part_of(base + step);
        uint32_t key = key_of(part, base + step) +
                       (uint32_t(i - step * step_tiles) << tile_shift);
        const uint32_t end = seg_key1[part];
        key = key < end ? key : (end - 1) >> tile_shift << tile_shift;
        const uint32_t page = key / uint32_t(a.block_size);
        int32_t id = a.bt[int64_t(r + part) * a.bt_cols + page];
        if (id < 0 || id >= a.num_blocks) id = 0;  // some block: its keys are left out
        tile_at[i] = uint32_t(id) * page_bytes +
                     uint64_t(key - page * uint32_t(a.block_size)) * slot_bytes;
      }
      for (int i = tid; i < count * a.wg_blocks * kBlockKeys; i += kDecodeThreads) {
        // two blocks a wavefront
        const int block = i / kBlockKeys, step = block / a.wg_blocks;
        const int part = part_of(base + step);
        const uint32_t key = key_of(part, base + step) +
                             uint32_t(i - step * a.wg_blocks * kBlockKeys);
        bool in = key < seg_key1[part];
        if (in) {
          const int32_t id =
              a.bt[int64_t(r + part) * a.bt_cols + key / uint32_t(a.block_size)];
          in = id >= 0 && id < a.num_blocks;
          if (!in) err = err < LUMEN_ERR_BLOCK_ID ? err : LUMEN_ERR_BLOCK_ID;
        }
        const uint64_t bits = __ballot(in);
        if ((lane & 31) == 0) live_keys[block] = uint32_t(bits >> (lane & 32));
      }
      for (int i = tid; i < count; i += kDecodeThreads) {
        const int part = part_of(base + i);
        step_part[i] = part | (seg_end[part] == base + i + 1 ? kLast : 0);
      }
      __syncthreads();

      // ---- the steps: kStages - 1 under way while one is used, over the ends
      // of requests too
      const uint8_t *from[kIssues];  // of the next start, a step ahead
      const auto prepare = [&](int i) __attribute__((always_inline)) {
        i = i < count ? i : count - 1;
#pragma unroll
        for (int c = 0; c < kIssues; ++c)
          from[c] = address(c, i * step_tiles);
      };
      const auto start = [&](int i, int stage) __attribute__((always_inline)) {
        if (i >= count) return;
        const uint32_t to = ring_at + stage * kStage;
#pragma unroll
        for (int c = 0; c < kIssues; ++c)
          load_to_lds(from[c], to + c * (kPrivate ? kWave : kDecodeThreads) * 16);
      };
      const auto live_of = [&](int i) __attribute__((always_inline)) {
        return active ? uint32_t(read(int(live_keys[i * a.wg_blocks + kbi]))) : 0u;
      };
      int part = read(step_part[0]);
      uint32_t live = live_of(0);
      if (fresh) {
        fetch_q(r + (part & (kLast - 1)));
        take_q();
        wait_loads<0>();
      }
#pragma unroll
      for (int i = 0; i < kStages - 1; ++i) {
        prepare(i);
        start(i, i);
      }
      prepare(kStages - 1);
      int stage = 0;
      for (int at = 0; at < count; ++at) {
        const int behind = count - 1 - at;  // started after this one
        if (kStages > 2 && behind >= kStages - 2)
          wait_loads<(kStages - 2) * kIssues>();
        else if (kStages > 3 && behind == 1)
          wait_loads<kIssues>();
        else
          wait_loads<0>();
        // everyone's loads of this step have come, and everyone is done with the
        // stage that the next start fills; a wavefront that reads only what it
        // loaded waits for itself alone, and runs ahead while others wait
        if constexpr (kPrivate)
          wait_lds();
        else
          lds_barrier();
        start(at + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
        prepare(at + kStages);
        const int next = at + 1 < count ? at + 1 : at;
        const int next_part = step_part[next];
        const int next_live = live_keys[next * a.wg_blocks + (active ? kbi : 0)];
        if (live) use(ring + stage * kStage + (kPrivate ? wave * kOwn : 0), live);
        fresh = part & kLast;
        if (fresh) {
          lds_barrier();  // this stage takes the sums
          finish(part & (kLast - 1), ring + stage * kStage);
        }
        part = read(next_part);
        live = active ? uint32_t(read(next_live)) : 0u;
        if (fresh && behind > 0) {
          fetch_q(r + (part & (kLast - 1)));
          take_q();
        }
        stage = stage + 1 < kStages ? stage + 1 : 0;
      }
      wait_loads<0>();
    }
    u = uniform(lds_first);
    first = u;
    r += kSegments;
  }
  record_wave(a.status, err);
}

// Partial results of requests that several workers shared, a workgroup for a
// (request, query head) in turn: its wavefronts take every kJoinWaves-th
// worker, two or four elements a lane, and wavefront 0 adds them up.
constexpr int kJoinWaves = 4;
template <int D, bool kBf16>
__global__ __launch_bounds__(kJoinWaves *kWave) void decode4_join_kernel(DecodeArgs a) {
  constexpr int kE = D / kWave;
  __shared__ float lds_o[kJoinWaves][D], lds_m[kJoinWaves], lds_l[kJoinWaves];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
  const int q_heads = a.heads * a.group;
  const int tiles = (a.group + kQueries - 1) / kQueries;
  const int64_t items = int64_t(a.num_reqs) * q_heads;
  for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
    const int r = int(i / q_heads), hq = int(i - int64_t(r) * q_heads);
    const int2 span = a.spans[r];
    if (span.x == span.y) continue;
    const int h = hq / a.group, g = hq - h * a.group;
    const int set = h / a.wg_heads * tiles + g / kQueries;
    const int hi = h % a.wg_heads, n = g % kQueries;
    float o[kE], m = -INFINITY, l = 0.0f;
    for (int e = 0; e < kE; ++e) o[e] = 0.0f;
    for (int w = span.x + wave; w <= span.y; w += kJoinWaves) {
      const float *part =
          a.parts + (((int64_t(set) * a.workers + w) * 2 + (w == span.x)) *
                         a.wg_heads + hi) * part_floats(D);
      const float pm = part[D * kQueries + n], pl = part[D * kQueries + kQueries + n];
      const float mn = fmaxf(m, pm);
      const float c0 = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - mn);
      const float c1 = mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(pm - mn);
      m = mn;
      l = l * c0 + pl * c1;
      for (int e = 0; e < kE; ++e)
        o[e] = o[e] * c0 + part[n * D + lane * kE + e] * c1;
    }
    __syncthreads();  // of the item before
    for (int e = 0; e < kE; ++e) lds_o[wave][lane * kE + e] = o[e];
    if (lane == 0) lds_m[wave] = m, lds_l[wave] = l;
    __syncthreads();
    if (wave > 0) continue;
    for (int w = 1; w < kJoinWaves; ++w) m = fmaxf(m, lds_m[w]);
    l = 0.0f;
    for (int e = 0; e < kE; ++e) o[e] = 0.0f;
    for (int w = 0; w < kJoinWaves; ++w) {
      const float c = m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(lds_m[w] - m);
      l += lds_l[w] * c;
      for (int e = 0; e < kE; ++e) o[e] += lds_o[w][lane * kE + e] * c;
    }
    const float inv = inverse(m, l);
    for (int e = 0; e < kE; ++e)
      a.out[i * D + lane * kE + e] = rounded<kBf16>(o[e] * inv);
  }
}

// ------------------------------------------------------------ host side

// The layer's K and V and the model's head_dim of a 4-bit layout.
struct Layer {
  int32_t head_dim;
  int64_t k, v;  // byte offsets into the cache
};

int check_layout(const lumen_kv_layout *l, int32_t layer, Layer *out) {
  if (!l || l->num_layers < 1 || l->num_kv_heads < 1 || l->block_size < 1 ||
      l->num_blocks < 0 || layer < 0 || layer >= l->num_layers)
    return LUMEN_ERR_INVALID_ARG;
  if (l->elem_bytes != 1 ||
      (l->head_dim != 48 && l->head_dim != 80 && l->head_dim != 144) ||
      (l->cache_order != LUMEN_CACHE_NHD && l->cache_order != LUMEN_CACHE_HND))
    return LUMEN_ERR_UNSUPPORTED;
  const int64_t page = int64_t(l->block_size) * l->num_kv_heads;
  if (page > INT32_MAX / l->head_dim) return LUMEN_ERR_UNSUPPORTED;
  int64_t half;
  if (__builtin_mul_overflow(page * l->head_dim, l->num_blocks, &half) ||
      half > INT64_MAX / 2 / l->num_layers)
    return LUMEN_ERR_INVALID_ARG;
  out->head_dim = (l->head_dim - 16) * 2;
  out->k = int64_t(layer) * 2 * half;
  out->v = out->k + half;
  return LUMEN_OK;
}

// Grid and workspace of a decode call on a device of `cus` compute units.
struct DecodePlan {
  int32_t wg_heads, wg_blocks;
  int32_t sets;     // sets of wg_heads KV heads, times tiles of 16 query heads
  int32_t workers;  // workgroups of one of them
  size_t parts_at, bytes;
};

// The workspace is sized for the largest device of this architecture, so that
// its size needs no device.
constexpr int kMaxUnits = 256;

DecodePlan decode_plan(const lumen_kv_layout *l, int32_t head_dim,
                       int32_t num_reqs, int32_t num_q_heads, int cus) {
  const int group = num_q_heads / l->num_kv_heads;
  DecodePlan p;
  // the most heads whose rows lie together, and blocks of keys for the rest of
  // the wavefronts: 256 requests around 2,048 tokens over 8 heads take 371 us with one
  // head a workgroup, 215 with 2, 191 with 4 and 180 with 8, 64 over 16 heads 198, 119,
  // 107 and 103.  (Eight short requests of 2 heads take 12.8 with one and 14.8 with
  // both.)
  p.wg_heads = 1;
  if (l->cache_order == LUMEN_CACHE_NHD)
    for (int d = 2; d <= kDecodeWaves; ++d)
      if (l->num_kv_heads % d == 0) p.wg_heads = d;
  p.wg_blocks = kDecodeWaves / p.wg_heads;
  p.sets = l->num_kv_heads / p.wg_heads * ((group + kQueries - 1) / kQueries);
  p.workers = (cus < kMaxUnits ? cus : kMaxUnits) / p.sets;  // one workgroup a CU
  if (p.workers < 1) p.workers = 1;
  p.parts_at = (size_t(num_reqs) * sizeof(int2) + 255) & ~size_t(255);
  p.bytes = p.parts_at + size_t(p.workers) * p.sets * 2 * p.wg_heads *
                             part_floats(head_dim) * sizeof(float);
  return p;
}

struct DecodeKernels {
  void (*main)(DecodeArgs);
  void (*join)(DecodeArgs);
};

template <int D>
DecodeKernels decode_kernels(bool bf16, bool one_head) {
  return {one_head ? decode4_kernel<D, true> : decode4_kernel<D, false>,
          bf16 ? decode4_join_kernel<D, true> : decode4_join_kernel<D, false>};
}

template <bool kAppend>
void (*row_kernel(int32_t head_dim, int32_t dtype))(RowArgs) {
  const bool bf = dtype == LUMEN_ATTN_BF16;
  if (kAppend)
    return head_dim == 64    ? (bf ? append4_kernel<64, true> : append4_kernel<64, false>)
           : head_dim == 128 ? (bf ? append4_kernel<128, true> : append4_kernel<128, false>)
                             : (bf ? append4_kernel<256, true> : append4_kernel<256, false>);
  return head_dim == 64    ? (bf ? read4_kernel<64, true> : read4_kernel<64, false>)
         : head_dim == 128 ? (bf ? read4_kernel<128, true> : read4_kernel<128, false>)
                           : (bf ? read4_kernel<256, true> : read4_kernel<256, false>);
}

template <bool kAppend>
int row_call(const lumen_kv_layout *layout, int32_t layer, void *d_cache,
             const lumen_attn_rows *k, const lumen_attn_rows *v, int32_t dtype,
             const int64_t *d_slots, int64_t num_tokens, int32_t *d_status,
             lumen_stream_t stream) {
  Layer at;
  int st = check_layout(layout, layer, &at);
  if (st != LUMEN_OK) return st;
  if ((st = check_dtype(dtype)) != LUMEN_OK) return st;
  if (num_tokens < 0) return LUMEN_ERR_INVALID_ARG;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if ((st = check_rows(k, num_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(v, num_tokens)) != LUMEN_OK) return st;
  if (num_tokens == 0) return LUMEN_OK;
  if (!d_slots || (!d_cache && layout->num_blocks > 0))
    return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_cache, 16) || !aligned(d_slots, 8)) return LUMEN_ERR_MISALIGNED;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  RowArgs a;
  a.k = static_cast<uint8_t *>(d_cache) + at.k;
  a.v = static_cast<uint8_t *>(d_cache) + at.v;
  a.slot_limit = layout->num_blocks * layout->block_size;
  a.block_size = layout->block_size;
  a.heads = layout->num_kv_heads;
  a.block_shift = a.block_size & (a.block_size - 1) ? -1 : __builtin_ctz(a.block_size);
  a.hnd = layout->cache_order == LUMEN_CACHE_HND;
  a.status = d_status;
  // rows are counted in 32 bits: a call over more of them is several launches
  const int64_t most = (int64_t(1) << 30) / (2 * a.heads);
  const int64_t step = most < 1 ? 1 : most;
  for (int64_t t = 0; t < num_tokens; t += step) {
    a.tokens = uint32_t(num_tokens - t < step ? num_tokens - t : step);
    a.rk = rows_of(k, t);
    a.rv = rows_of(v, t);
    a.slots = d_slots + t;
    const int64_t per_token = 2 * int64_t(a.heads), rows = a.tokens * per_token;
    const int per = kRowThreads / (at.head_dim / 8);
    // as many as run at once, and at least a token's
    const int64_t room = int64_t(cus) * (2048 / kRowThreads) * per;
    const int64_t taken = rows < room ? rows : room < per_token ? per_token : room;
    const int64_t blocks = (taken + per - 1) / per;
    a.at_once = uint32_t(blocks * per / per_token);
    hipLaunchKernelGGL(row_kernel<kAppend>(at.head_dim, dtype),
                       dim3(unsigned(blocks)), dim3(kRowThreads), 0,
                       static_cast<hipStream_t>(stream), a);
  }
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // namespace

extern "C" {

int lumen_attn_slots(const int32_t *d_start, const int32_t *d_end,
                     const int32_t *d_have, int32_t num_reqs,
                     int32_t *d_block_tables, int32_t bt_cols,
                     int32_t block_size, int64_t num_blocks,
                     const int32_t *d_free, const int64_t *d_free_count,
                     int64_t free_cap, int64_t *d_slots, int64_t num_slots,
                     int32_t *d_cu, int32_t *d_lens, int64_t *d_free_left,
                     int32_t *d_status, lumen_stream_t stream) {
  if (num_reqs < 0 || bt_cols < 0 || block_size < 1 || num_blocks < 0 ||
      free_cap < 0 || num_slots < 0)
    return LUMEN_ERR_INVALID_ARG;
  int st = check_status(d_status);
  if (st != LUMEN_OK) return st;
  if (num_reqs > LUMEN_ATTN_MAX_REQS) return LUMEN_ERR_TOO_MANY;
  if (!d_free_count || !d_cu || !d_free_left || (!d_free && free_cap > 0) ||
      (!d_slots && num_slots > 0))
    return LUMEN_ERR_INVALID_ARG;
  if (num_reqs > 0 && (!d_start || !d_end || !d_lens ||
                       (!d_block_tables && bt_cols > 0)))
    return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_slots, 8) || !aligned(d_free_count, 8) ||
      !aligned(d_free_left, 8) || !aligned(d_start, 4) || !aligned(d_end, 4) ||
      !aligned(d_have, 4) || !aligned(d_block_tables, 4) ||
      !aligned(d_free, 4) || !aligned(d_cu, 4) || !aligned(d_lens, 4))
    return LUMEN_ERR_MISALIGNED;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  SlotArgs a{d_start,  d_end,  d_have,       num_reqs, d_block_tables, bt_cols,
             block_size, num_blocks, d_free, d_free_count, free_cap, d_slots,
             num_slots, d_cu,  d_lens,       d_free_left, d_status};
  const int64_t per = int64_t(kSlotThreads) * kSlotTokens;
  int64_t blocks = num_slots / per + (num_slots % per != 0);
  // the new pages are at most this many, a thread each, on a workgroup for 16
  // requests at most: each scans all of them (pages alone of 1,024 prompts of 512
  // tokens: 9.5 us, and 8.4 with a workgroup for 2, 13.4 for 64; of 8 prompts of 8,192
  // 7.6, 4.4 and 7.6)
  const int64_t pages = (free_cap + kSlotThreads - 1) / kSlotThreads;
  const int64_t page_wgs = pages < num_reqs / 16 + 1 ? pages : num_reqs / 16 + 1;
  if (blocks < page_wgs) blocks = page_wgs;
  if (blocks < 1) blocks = 1;
  // more of them would scan the requests for too few tokens each (1,024 prompts of
  // 512 tokens: 16.2 us with 2 a compute unit, 14.6 with 4, 16.4 with 8)
  if (blocks > int64_t(cus) * 4) blocks = int64_t(cus) * 4;
  hipLaunchKernelGGL(slots_kernel, dim3(unsigned(blocks)), dim3(kSlotThreads),
                     2 * (size_t(num_reqs) + 1) * sizeof(uint32_t),
                     static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

int lumen_attn_append4(const lumen_kv_layout *layout, int32_t layer,
                       void *d_cache, const lumen_attn_rows *k,
                       const lumen_attn_rows *v, int32_t dtype,
                       const int64_t *d_slots, int64_t num_tokens,
                       int32_t *d_status, lumen_stream_t stream) {
  return row_call<true>(layout, layer, d_cache, k, v, dtype, d_slots,
                        num_tokens, d_status, stream);
}

int lumen_attn_read4(const lumen_kv_layout *layout, int32_t layer,
                     const void *d_cache, const int64_t *d_slots,
                     int64_t num_tokens, const lumen_attn_rows *k,
                     const lumen_attn_rows *v, int32_t dtype,
                     int32_t *d_status, lumen_stream_t stream) {
  return row_call<false>(layout, layer, const_cast<void *>(d_cache), k, v,
                         dtype, d_slots, num_tokens, d_status, stream);
}

size_t lumen_attn_decode4_workspace_bytes(const lumen_kv_layout *layout,
                                          int32_t num_reqs,
                                          int32_t num_q_heads) {
  Layer at;
  if (check_layout(layout, 0, &at) != LUMEN_OK || num_reqs < 0 ||
      num_reqs > LUMEN_ATTN_MAX_REQS || num_q_heads < 1 || num_q_heads > 65535 ||
      num_q_heads % layout->num_kv_heads)
    return 0;
  return decode_plan(layout, at.head_dim, num_reqs, num_q_heads, kMaxUnits).bytes;
}

int lumen_attn_decode4(const lumen_kv_layout *layout, int32_t layer,
                       const void *d_cache, const int32_t *d_block_tables,
                       int32_t bt_cols, const int32_t *d_lens,
                       int32_t num_reqs, const lumen_attn_rows *q,
                       int32_t dtype, int32_t num_q_heads, float scale,
                       void *d_out, void *d_workspace, size_t workspace_bytes,
                       int32_t *d_status, lumen_stream_t stream) {
  Layer at;
  int st = check_layout(layout, layer, &at);
  if (st != LUMEN_OK) return st;
  if ((st = check_dtype(dtype)) != LUMEN_OK) return st;
  if (num_reqs < 0 || bt_cols < 0 || num_q_heads < 1 ||
      num_q_heads % layout->num_kv_heads || check_scale(scale) != LUMEN_OK)
    return LUMEN_ERR_INVALID_ARG;
  if (num_q_heads > 65535) return LUMEN_ERR_UNSUPPORTED;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if (num_reqs > LUMEN_ATTN_MAX_REQS) return LUMEN_ERR_TOO_MANY;
  if ((st = check_rows(q, num_reqs)) != LUMEN_OK) return st;
  if (num_reqs == 0) return LUMEN_OK;
  if (!d_lens || !d_out || !d_workspace || (!d_block_tables && bt_cols > 0) ||
      (!d_cache && layout->num_blocks > 0) ||
      workspace_bytes < lumen_attn_decode4_workspace_bytes(layout, num_reqs,
                                                           num_q_heads))
    return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_cache, 16) || !aligned(d_out, 16) ||
      !aligned(d_workspace, 16) || !aligned(d_lens, 4) ||
      !aligned(d_block_tables, 4))
    return LUMEN_ERR_MISALIGNED;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  const DecodePlan plan =
      decode_plan(layout, at.head_dim, num_reqs, num_q_heads, cus);
  const int32_t bs = layout->block_size;
  const int64_t unit = int64_t(kBlockKeys) * plan.wg_blocks * kUnitBlocks;
  // no request can be shared: no results to join
  const bool shared = int64_t(bt_cols) * bs > unit;
  DecodeArgs a;
  a.k = static_cast<const uint8_t *>(d_cache) + at.k;
  a.v = static_cast<const uint8_t *>(d_cache) + at.v;
  a.bt = d_block_tables;
  a.bt_cols = bt_cols;
  a.block_size = bs;
  a.num_blocks = layout->num_blocks;
  a.lens = d_lens;
  a.num_reqs = num_reqs;
  a.heads = layout->num_kv_heads;
  a.group = num_q_heads / layout->num_kv_heads;
  a.hnd = layout->cache_order == LUMEN_CACHE_HND;
  a.q = rows_of(q, 0);
  a.scale_log2 = scale_log2(scale);
  a.out = static_cast<uint16_t *>(d_out);
  a.status = d_status;
  a.wg_heads = plan.wg_heads;
  a.wg_blocks = plan.wg_blocks;
  a.workers = plan.workers;
  a.bf16 = dtype == LUMEN_ATTN_BF16;
  a.spans = shared ? static_cast<int2 *>(d_workspace) : nullptr;
  a.parts = reinterpret_cast<float *>(static_cast<char *>(d_workspace) + plan.parts_at);
  const bool one = plan.wg_heads == 1;
  const DecodeKernels k = at.head_dim == 64    ? decode_kernels<64>(a.bf16, one)
                          : at.head_dim == 128 ? decode_kernels<128>(a.bf16, one)
                                               : decode_kernels<256>(a.bf16, one);
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(k.main, dim3(unsigned(plan.workers * plan.sets)),
                     dim3(kDecodeThreads), 0, s, a);
  if (shared) {
    int64_t items = int64_t(num_reqs) * num_q_heads;
    const int64_t most = int64_t(cus) * 8;
    hipLaunchKernelGGL(k.join, dim3(unsigned(items < most ? items : most)),
                       dim3(kJoinWaves * kWave), 0, s, a);
  }
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

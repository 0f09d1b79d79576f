// Serving operators for MI355X (gfx950): block tables and slot maps, the
// paged 4-bit KV cache's append, read-back and decode attention.
//
// The operations, the 4-bit row format and the errors are specified in
// include/lumen_attn.h.

#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include "lumen_attn.h"
#include "lumen_attn_common.h"

namespace {

using namespace lumen_attn_detail;

// ---------------------------------------------------------------- slots

constexpr int kSlotThreads = 256;
constexpr int kSlotTokens = 4;  // consecutive tokens a thread maps at a time
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

__device__ __forceinline__ int32_t pages_of(int32_t tokens, int32_t bs) {
  return int32_t((int64_t(tokens) + bs - 1) / bs);
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
  const uint32_t count = count64 < kHeld ? uint32_t(count64) : kHeld;
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
  for (int64_t i0 = me * kSlotTokens; i0 < a.num_slots; i0 += grid * kSlotTokens) {
    int r = -1;
    int32_t s = 0, first = 0;
    uint32_t b = 0;
    bool ok = false;
    for (int k = 0; k < kSlotTokens; ++k) {
      const int64_t i = i0 + k;
      if (i >= a.num_slots) break;
      int64_t slot = -1;
      if (i < int64_t(total)) {
        const uint32_t u = uint32_t(i);
        if (r < 0 || u >= cu[r + 1]) {
          int lo = r < 0 ? 0 : r + 1, hi = R - 1;  // last r with cu[r] <= u
          while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (cu[mid] <= u)
              lo = mid;
            else
              hi = mid - 1;
          }
          r = lo;
          const SlotReq q = slot_req(a, r);
          s = a.start[r];
          first = q.first;
          b = base[r];
          ok = !q.range && (q.need == 0 || add_held(b, q.need) <= count);
          if (q.need == 0) first = 0x7fffffff;  // every page is in the table
        }
        if (ok) {
          const int32_t tok = s + int32_t(u - cu[r]);
          const int32_t page = tok / a.block_size;
          const int32_t id =
              page >= first ? a.free_ids[count - 1 - b - uint32_t(page - first)]
                            : a.bt[int64_t(r) * a.bt_cols + page];
          if (id >= 0 && id < a.num_blocks)
            slot = int64_t(id) * a.block_size + (tok - page * a.block_size);
          else
            err = err < LUMEN_ERR_BLOCK_ID ? err : LUMEN_ERR_BLOCK_ID;
        }
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
    const int32_t id = a.free_ids[count - 1 - u];
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
  bool hnd;
  int64_t tokens;
  int32_t *status;
};

// Byte offset of the row of (slot, head).
__device__ __forceinline__ int64_t row_offset(int64_t slot, int32_t bs,
                                              int32_t h, int32_t heads,
                                              bool hnd, int32_t row) {
  if (!hnd) return (slot * heads + h) * row;
  const int64_t block = slot < 0x7fffffff
                            ? int64_t(uint32_t(slot) / uint32_t(bs))
                            : slot / bs;
  const int64_t pos = slot - block * bs;
  return ((block * heads + h) * bs + pos) * row;
}

// Quantises rows: D/8 lanes a row, 8 elements a lane (one 16-byte load, one
// dword of codes).  Memory-bound: 2*D bytes in and D/2 + 16 out a row.
template <int D, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void append4_kernel(RowArgs a) {
  constexpr int kLanes = D / 8;        // lanes of a row
  constexpr int kGroup = kLanes / 4;   // lanes of a quarter
  constexpr int kRow = D / 2 + 16;
  constexpr int kRows = kRowThreads / kLanes;
  const int lane = threadIdx.x % kLanes;
  const uint32_t per_token = 2u * uint32_t(a.heads);
  const uint32_t items = uint32_t(a.tokens) * per_token;
  int err = LUMEN_OK;
  for (uint32_t i = blockIdx.x * kRows + threadIdx.x / kLanes; i < items;
       i += gridDim.x * kRows) {
    const uint32_t t = i / per_token, kvh = i - t * per_token;
    const bool is_v = kvh >= uint32_t(a.heads);
    const int h = int(is_v ? kvh - a.heads : kvh);
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.slot_limit) {
      if (slot >= 0) err = LUMEN_ERR_BLOCK_ID;
      continue;  // a whole row's lanes, and no lane reads another row's
    }
    const Rows &src = is_v ? a.rv : a.rk;
    const uint4 raw = *reinterpret_cast<const uint4 *>(
        src.base + (int64_t(t) * src.token + int64_t(h) * src.head + lane * 8));
    float x[8];
    unpack8<kBf16>(raw, x);
    float lo = x[0], hi = x[0];
    bool nan = false;
    for (int k = 0; k < 8; ++k) {
      nan |= x[k] != x[k];
      x[k] = fminf(fmaxf(x[k], -float(LUMEN_ATTN_KV4_MAX)),
                   float(LUMEN_ATTN_KV4_MAX));
    }
    for (int k = 0; k < 8; ++k) {
      lo = fminf(k ? lo : x[0], x[k]);
      hi = fmaxf(k ? hi : x[0], x[k]);
    }
    int bad = nan;
    for (int o = 1; o < kGroup; o <<= 1) {
      lo = fminf(lo, __shfl_xor(lo, o));
      hi = fmaxf(hi, __shfl_xor(hi, o));
      bad |= __shfl_xor(bad, o);
    }
    const _Float16 ah = _Float16((hi - lo) * (1.0f / 15.0f));
    const float A = float(ah);
    const _Float16 bh = _Float16(lo - 64.0f * A);
    const float first = float(bh) + 64.0f * A;
    const float inv = A > 0.0f ? 1.0f / A : 0.0f;
    uint32_t codes = 0;
    for (int k = 0; k < 8; ++k) {
      const float q = rintf((x[k] - first) * inv);
      codes |= uint32_t(fminf(fmaxf(q, 0.0f), 15.0f)) << (4 * k);
    }
    uint32_t pair = bits(ah) | uint32_t(bits(bh)) << 16;
    if (bad) codes = 0, pair = 0x7e007e00u;
    uint8_t *row = (is_v ? a.v : a.k) +
                   row_offset(slot, a.block_size, h, a.heads, a.hnd, kRow);
    reinterpret_cast<uint32_t *>(row)[lane] = codes;
    if (lane % kGroup == 0)
      reinterpret_cast<uint32_t *>(row + D / 2)[lane / kGroup] = pair;
  }
  record_wave(a.status, err);
}

template <int D, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void read4_kernel(RowArgs a) {
  constexpr int kLanes = D / 8;
  constexpr int kGroup = kLanes / 4;
  constexpr int kRow = D / 2 + 16;
  constexpr int kRows = kRowThreads / kLanes;
  const int lane = threadIdx.x % kLanes;
  const uint32_t per_token = 2u * uint32_t(a.heads);
  const uint32_t items = uint32_t(a.tokens) * per_token;
  int err = LUMEN_OK;
  for (uint32_t i = blockIdx.x * kRows + threadIdx.x / kLanes; i < items;
       i += gridDim.x * kRows) {
    const uint32_t t = i / per_token, kvh = i - t * per_token;
    const bool is_v = kvh >= uint32_t(a.heads);
    const int h = int(is_v ? kvh - a.heads : kvh);
    const int64_t slot = a.slots[t];
    uint4 raw{0, 0, 0, 0};
    if (slot >= 0 && slot < a.slot_limit) {
      const uint8_t *row = (is_v ? a.v : a.k) + row_offset(slot, a.block_size, h,
                                                           a.heads, a.hnd, kRow);
      const uint32_t codes = reinterpret_cast<const uint32_t *>(row)[lane];
      const uint32_t pair =
          reinterpret_cast<const uint32_t *>(row + D / 2)[lane / kGroup];
      const float A = float(half_of(pair)), B = float(half_of(pair >> 16));
      float x[8];
      for (int k = 0; k < 8; ++k)
        x[k] = float(_Float16(
            A * float(64 + ((codes >> (4 * k)) & 15)) + B));
      raw = pack8<kBf16>(x);
    } else if (slot >= 0) {
      err = LUMEN_ERR_BLOCK_ID;
    }
    const Rows &dst = is_v ? a.rv : a.rk;
    *reinterpret_cast<uint4 *>(dst.base + (int64_t(t) * dst.token +
                                           int64_t(h) * dst.head + lane * 8)) =
        raw;
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
  bool hnd;
  Rows q;
  float scale_log2;  // scale * log2(e)
  uint16_t *out;
  int32_t *status;
};

// One wavefront per (request, query head), a key at a time.
template <int D, bool kBf16>
__global__ __launch_bounds__(kWave) void decode4_kernel(DecodeArgs a) {
  constexpr int kE = D / 64;  // elements a lane
  constexpr int kRow = D / 2 + 16;
  const int r = blockIdx.x, hq = blockIdx.y, lane = threadIdx.x;
  const int h = hq / a.group;
  const uint16_t *q = a.q.base + int64_t(r) * a.q.token + int64_t(hq) * a.q.head;
  float x[kE], o[kE];
  for (int e = 0; e < kE; ++e) {
    x[e] = value<kBf16>(q[lane * kE + e]) * a.scale_log2;
    o[e] = 0.0f;
  }
  const int len = a.lens[r];
  int err = len < 0 ? LUMEN_ERR_RANGE : LUMEN_OK;
  float m = -INFINITY, l = 0.0f;
  for (int t = 0; t < len; ++t) {
    const int page = t / a.block_size;
    if (page >= a.bt_cols) {
      err = err < LUMEN_ERR_RANGE ? err : LUMEN_ERR_RANGE;
      break;
    }
    const int32_t id = a.bt[int64_t(r) * a.bt_cols + page];
    if (id < 0 || id >= a.num_blocks) {
      err = err < LUMEN_ERR_BLOCK_ID ? err : LUMEN_ERR_BLOCK_ID;
      continue;
    }
    const int64_t off = row_offset(int64_t(id) * a.block_size + t % a.block_size,
                                   a.block_size, h, a.heads, a.hnd, kRow);
    float kv[2][kE];
    for (int w = 0; w < 2; ++w) {
      const uint8_t *row = (w ? a.v : a.k) + off;
      const uint32_t pair =
          reinterpret_cast<const uint32_t *>(row + D / 2)[lane / 16];
      for (int e = 0; e < kE; ++e) {
        const int n = lane * kE + e;
        const int code = (row[n / 2] >> (4 * (n & 1))) & 15;
        kv[w][e] = float(_Float16(float(half_of(pair)) * float(64 + code) +
                                  float(half_of(pair >> 16))));
      }
    }
    float s = 0.0f;
    for (int e = 0; e < kE; ++e) s += x[e] * kv[0][e];
    for (int b = 1; b < kWave; b <<= 1) s += __shfl_xor(s, b);
    const float mn = fmaxf(m, s);
    const float c = exp2f(m - mn), p = exp2f(s - mn);
    m = mn;
    l = l * c + p;
    for (int e = 0; e < kE; ++e) o[e] = o[e] * c + p * kv[1][e];
  }
  uint16_t *out = a.out + (int64_t(r) * a.heads * a.group + hq) * D;
  for (int e = 0; e < kE; ++e)
    out[lane * kE + e] = rounded<kBf16>(l > 0.0f || l != l ? o[e] / l : 0.0f);
  record_wave(a.status, err);
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
  a.hnd = layout->cache_order == LUMEN_CACHE_HND;
  a.status = d_status;
  // rows are counted in 32 bits: a call over more of them is several launches
  const int64_t most = (int64_t(1) << 30) / (2 * a.heads);
  const int64_t step = most < 1 ? 1 : most;
  for (int64_t t = 0; t < num_tokens; t += step) {
    a.tokens = num_tokens - t < step ? num_tokens - t : step;
    a.rk = rows_of(k, t);
    a.rv = rows_of(v, t);
    a.slots = d_slots + t;
    const int64_t rows = a.tokens * 2 * a.heads;
    const int per = kRowThreads / (at.head_dim / 8);
    int64_t blocks = (rows + per - 1) / per;
    if (blocks > int64_t(cus) * 32) blocks = int64_t(cus) * 32;
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
  // the new pages are at most this many, a thread each
  const int64_t pages = (free_cap + kSlotThreads - 1) / kSlotThreads;
  const int64_t page_wgs = pages < num_reqs / 16 + 1 ? pages : num_reqs / 16 + 1;
  if (blocks < page_wgs) blocks = page_wgs;
  if (blocks < 1) blocks = 1;
  if (blocks > int64_t(cus) * 2) blocks = int64_t(cus) * 2;
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
      num_reqs > LUMEN_ATTN_MAX_REQS || num_q_heads < 1 ||
      num_q_heads % layout->num_kv_heads)
    return 0;
  return 16;
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
      num_q_heads % layout->num_kv_heads || !(scale > 0.0f) ||
      !(scale < INFINITY))
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
  (void)hipGetLastError();
  DecodeArgs a{static_cast<const uint8_t *>(d_cache) + at.k,
               static_cast<const uint8_t *>(d_cache) + at.v,
               d_block_tables,
               bt_cols,
               layout->block_size,
               layout->num_blocks,
               d_lens,
               num_reqs,
               layout->num_kv_heads,
               num_q_heads / layout->num_kv_heads,
               layout->cache_order == LUMEN_CACHE_HND,
               rows_of(q, 0),
               scale * 1.44269504088896341f,
               static_cast<uint16_t *>(d_out),
               d_status};
  const bool bf = dtype == LUMEN_ATTN_BF16;
  void (*kernel)(DecodeArgs) =
      at.head_dim == 64    ? (bf ? decode4_kernel<64, true> : decode4_kernel<64, false>)
      : at.head_dim == 128 ? (bf ? decode4_kernel<128, true> : decode4_kernel<128, false>)
                           : (bf ? decode4_kernel<256, true> : decode4_kernel<256, false>);
  hipLaunchKernelGGL(kernel, dim3(unsigned(num_reqs), unsigned(num_q_heads)),
                     dim3(kWave), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

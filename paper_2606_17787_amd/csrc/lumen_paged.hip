// Filling a 16-bit paged KV cache and holding it to a budget, for MI355X
// (gfx950): append, evict and release, as specified in include/lumen_paged.h.

#include <hip/hip_runtime.h>

#include <stdint.h>

#include "lumen_paged.h"
#include "lumen_paged_common.h"

namespace {

using namespace lumen_paged_detail;

// ---------------------------------------------------------------- append

constexpr int kRowThreads = 256;

struct AppendArgs {
  uint8_t *k, *v;  // of the layer
  Rows rk, rv;
  const int64_t *slots;
  const int32_t *positions;
  int32_t *weights, *places;  // the ledger's words of the layer, or NULL
  int64_t slot_limit;
  int64_t page;
  int32_t slot_bytes, head_bytes;
  int32_t block_size, heads;
  uint32_t tokens;
  uint32_t at_once;  // tokens that the grid takes at a time
  int32_t *status;
};

// Rows of K and V as they are, 16 bytes a lane, D/8 lanes a row; a lane keeps its
// head of K or V for all of its tokens.  Bound by bytes: 4 D a token and head in
// and as many out.
template <int D>
__global__ __launch_bounds__(kRowThreads) void append_kernel(AppendArgs a) {
  constexpr uint32_t kLanes = D / 8, kRows = kRowThreads / kLanes;
  const uint32_t per_token = 2u * uint32_t(a.heads);
  const uint32_t r = blockIdx.x * kRows + threadIdx.x / kLanes;
  const int lane = threadIdx.x % kLanes;
  uint32_t t = r / per_token;
  const uint32_t kvh = r - t * per_token;
  const bool is_v = kvh >= uint32_t(a.heads);
  const uint32_t h = is_v ? kvh - a.heads : kvh;
  const Rows &rows = is_v ? a.rv : a.rk;
  const uint16_t *row = rows.base + (int64_t(t) * rows.token + int64_t(h) * rows.head + lane * 8);
  const int64_t step = int64_t(a.at_once) * rows.token;
  uint8_t *const cached = (is_v ? a.v : a.k) + int64_t(h) * a.head_bytes + lane * 16;
  if (t >= a.at_once) t = a.tokens;  // past the last whole token
  int err = LUMEN_OK;
  for (; t < a.tokens; t += a.at_once, row += step) {
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.slot_limit) {
      if (slot >= 0) err = LUMEN_ERR_BLOCK_ID;
      continue;
    }
    const uint4 x = *reinterpret_cast<const uint4 *>(row);
    const int64_t block = slot <= UINT32_MAX
                              ? int64_t(uint32_t(slot) / uint32_t(a.block_size))
                              : slot / a.block_size;
    const int32_t at = int32_t(slot - block * a.block_size);
    *reinterpret_cast<uint4 *>(cached + block * a.page + int64_t(at) * a.slot_bytes) = x;
    if (lane == 0 && a.weights) {
      const int64_t word = (block * a.heads + h) * a.block_size + at;
      if (is_v)
        a.places[word] = a.positions[t];
      else
        a.weights[word] = 0;
    }
  }
  record_wave(a.status, err);
}

// ----------------------------------------------------------------- evict

struct EvictArgs {
  uint8_t *cache;     // of the first layer
  uint32_t *ledger;   // of the first layer
  int64_t half, page; // bytes
  int64_t words;      // of a layer's weights
  int32_t slot_bytes, head_bytes;
  int32_t block_size, heads;
  int64_t num_blocks;
  const int32_t *bt;
  int32_t bt_cols;
  const int32_t *lens, *keep, *from;
  int32_t sinks, num_reqs;
  int32_t *left;
  int32_t *status;
  // the workspace, for each (layer, request, head): how many places move, and for
  // each 64 of its places which are kept and how many are before them
  int32_t *moves;
  uint64_t *kept;
  uint32_t *before;
  int32_t strips;    // 64 places each, of a request at most
  int32_t lds_keys;  // ranks that fit the workgroup's LDS
};

__device__ __forceinline__ bool protects(int32_t pos, int32_t sinks, int32_t from) {
  return pos < sinks || pos >= from;
}

// A weight's rank as a whole number: its order with -0 as 0, NaN at kNanRank.  Under
// it is kNoRank, for places that are not kept, above all ranks kAllRanks.
constexpr uint32_t kNoRank = 0, kNanRank = 1, kAllRanks = 0xffffffffu;
__device__ __forceinline__ uint32_t rank_of(uint32_t weight) {
  if ((weight & 0x7fffffffu) > 0x7f800000u) return kNanRank;
  if (weight == 0x80000000u) weight = 0;
  return weight & 0x80000000u ? ~weight : weight | 0x80000000u;
}

struct Item {
  int layer, r, h;
};

__device__ __forceinline__ Item item_of(const EvictArgs &a, int64_t i) {
  const int64_t lr = i / a.heads;
  const int layer = int(lr / a.num_reqs);
  return Item{layer, int(lr - int64_t(layer) * a.num_reqs), int(i - lr * a.heads)};
}

// Which places of one layer, request and head are kept.  Protected places are counted
// first: where they do not fill the budget, all of them are kept and the others are
// ranked, where they do, they are ranked alone.  The rank of the last one kept comes
// out of four counts over the ranks' bytes, from the highest on; the places of a
// wavefront's own stretch are then counted and written with what the wavefronts before
// it have.
template <int kThreads>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictArgs a) {
  constexpr int kWaves = kThreads / kWave;
  extern __shared__ uint32_t ranks[];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t wave_a[kWaves], wave_b[kWaves];
  __shared__ uint32_t digit, above;
  __shared__ int guarded;
  const int64_t id = blockIdx.x;
  const Item it = item_of(a, id);
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int n = a.lens[it.r], keep = a.keep[it.r];
  const bool first = it.layer == 0 && it.h == 0;
  int err = LUMEN_OK;
  bool alone = n < 0 || keep < 0 || int64_t(n) > int64_t(a.bt_cols) * a.block_size;
  if (alone) err = LUMEN_ERR_RANGE;
  const int32_t *table = a.bt + int64_t(it.r) * a.bt_cols;
  if (!alone && n > keep) {
    const int pages = (n - 1) / a.block_size + 1;
    int bad = 0;
    for (int p = tid; p < pages; p += kThreads)
      bad |= table[p] < 0 || table[p] >= a.num_blocks;
    if (__syncthreads_or(bad)) {
      alone = true;
      err = LUMEN_ERR_BLOCK_ID;
    }
  }
  if (first && tid == 0) {
    a.left[it.r] = !alone && n > keep ? keep : n;
    if (err) atomicMin(a.status, err);
  }
  if (alone || n <= keep || keep == 0) {
    if (tid == 0) a.moves[id] = 0;
    return;
  }
  const int32_t from = a.from[it.r];
  const uint32_t *weights = a.ledger + int64_t(it.layer) * 2 * a.words +
                            int64_t(it.h) * a.block_size;
  const auto word_of = [&](int i) __attribute__((always_inline)) {
    const int page = int(uint32_t(i) / uint32_t(a.block_size));
    return int64_t(table[page]) * a.heads * a.block_size + (i - page * a.block_size);
  };
  // the protected places are kept, or the ones kept are all among them
  int mine = 0;
  for (int i = tid; i < n; i += kThreads)
    mine += protects(int32_t(weights[word_of(i) + a.words]), a.sinks, from);
  if (tid == 0) guarded = 0;
  __syncthreads();
  for (int o = 1; o < kWave; o <<= 1) mine += __shfl_xor(mine, o);
  if (lane == 0) atomicAdd(&guarded, mine);
  __syncthreads();
  const bool among = guarded >= keep;
  const auto rank_at = [&](int i) __attribute__((always_inline)) {
    const int64_t word = word_of(i);
    const bool guard = protects(int32_t(weights[word + a.words]), a.sinks, from);
    if (guard != among) return guard ? kAllRanks : kNoRank;
    return rank_of(weights[word]);
  };
  const bool held = n <= a.lds_keys;
  if (held)
    for (int i = tid; i < n; i += kThreads) ranks[i] = rank_at(i);
  const auto rank = [&](int i) __attribute__((always_inline)) {
    return held ? ranks[i] : rank_at(i);
  };
  uint32_t last = 0, mask = 0, want = uint32_t(keep);
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kThreads) hist[i] = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
      const uint32_t x = rank(i);
      if ((x & mask) == last) atomicAdd(&hist[x >> shift & 255], 1u);
    }
    __syncthreads();
    if (wave == 0) {  // four digits a lane, the highest first
      uint32_t c[4], sum = 0;
      for (int j = 0; j < 4; ++j) sum += c[j] = hist[255 - (4 * lane + j)];
      uint32_t upto = sum;
      for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t x = __shfl_up(upto, o);
        if (lane >= o) upto += x;
      }
      uint32_t over = upto - sum;
      if (over < want && want <= upto)
        for (int j = 0; j < 4; ++j) {
          if (want <= over + c[j]) {
            digit = 255 - (4 * lane + j);
            above = over;
            break;
          }
          over += c[j];
        }
    }
    __syncthreads();
    last |= digit << shift;
    mask |= 255u << shift;
    want -= above;
  }
  // every place above `last` is kept, and the first `want` of those at it
  const int strips = (n + kWave - 1) / kWave;
  const int per = (strips + kWaves - 1) / kWaves;
  const int s0 = wave * per < strips ? wave * per : strips;
  const int s1 = s0 + per < strips ? s0 + per : strips;
  uint32_t more = 0, same = 0;
  for (int s = s0; s < s1; ++s) {
    const int i = s * kWave + lane;
    const uint32_t x = i < n ? rank(i) : 0;
    more += __popcll(__ballot(i < n && x > last));
    same += __popcll(__ballot(i < n && x == last));
  }
  if (lane == 0) wave_a[wave] = more, wave_b[wave] = same;
  __syncthreads();
  uint32_t kept_before = 0, same_before = 0;
  for (int w = 0; w < wave; ++w) {
    const uint32_t room = want > same_before ? want - same_before : 0;
    kept_before += wave_a[w] + (wave_b[w] < room ? wave_b[w] : room);
    same_before += wave_b[w];
  }
  uint64_t *kept = a.kept + id * a.strips;
  uint32_t *before = a.before + id * a.strips;
  for (int s = s0; s < s1; ++s) {
    const int i = s * kWave + lane;
    const uint32_t x = i < n ? rank(i) : 0;
    const uint64_t at = __ballot(i < n && x == last);
    const uint32_t nth = same_before + __popcll(at & ((uint64_t(1) << lane) - 1));
    const uint64_t bits = __ballot(i < n && (x > last || (x == last && nth < want)));
    if (lane == 0) {
      kept[s] = bits;
      before[s] = kept_before;
      if (s == keep / kWave)
        a.moves[id] = keep - int(kept_before + __popcll(bits & ((uint64_t(1) << keep % kWave) - 1)));
    }
    kept_before += __popcll(bits);
    same_before += __popcll(at);
  }
}

// The place of the n-th (from 0) set bit.
__device__ __forceinline__ int nth_bit(uint64_t bits, uint32_t n) {
  int at = 0;
#pragma unroll
  for (int width = 32; width; width >>= 1) {
    const uint32_t low = __popcll(bits & ((uint64_t(1) << width) - 1));
    if (n >= low) {
      n -= low;
      bits >>= width;
      at += width;
    }
  }
  return at;
}

// Moves what evict_select_kernel has chosen: a wavefront takes 64 moves, a lane
// finds the two places of one (the k-th place given up, the k-th one kept behind the
// budget) by bisection over the counts, and the rows go 16 bytes a lane.  No place
// is both read and written.
typedef uint32_t piece __attribute__((ext_vector_type(4)));  // 16 bytes of a row
constexpr int kMoveThreads = 256;
template <int D>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, int32_t parts) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes;  // rows at a time
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t id = blockIdx.x / unsigned(parts);
  const int part = int(blockIdx.x - id * parts);
  const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
  const int moves = __builtin_amdgcn_readfirstlane(a.moves[id]);
  const int waves = parts * (kMoveThreads / kWave);
  int c = part * (kMoveThreads / kWave) + wave;
  if (int64_t(c) * kWave >= moves) return;
  const Item it = item_of(a, id);
  const int keep = a.keep[it.r];
  const int n = a.lens[it.r], strips = (n + kWave - 1) / kWave, border = keep / kWave;
  const uint64_t *kept = a.kept + id * a.strips;
  const uint32_t *before = a.before + id * a.strips;
  const int32_t *table = a.bt + int64_t(it.r) * a.bt_cols;
  uint8_t *const k = a.cache + int64_t(it.layer) * 2 * a.half + int64_t(it.h) * a.head_bytes +
                     lane % kLanes * 16;
  uint32_t *const ledger = a.ledger + int64_t(it.layer) * 2 * a.words +
                           int64_t(it.h) * a.block_size;
  const uint32_t inside = uint32_t(keep - moves);  // kept places under `keep`
  for (; int64_t(c) * kWave < moves; c += waves) {
    const int m = c * kWave + lane;
    const int here = moves - c * kWave < kWave ? moves - c * kWave : kWave;
    const uint32_t nth = uint32_t(m < moves ? m : moves - 1);
    // the strip with the nth place given up: the last with at most nth before it
    int lo = 0, hi = border;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (uint32_t(mid) * kWave - before[mid] <= nth)
        lo = mid;
      else
        hi = mid - 1;
    }
    int to = lo * kWave + nth_bit(~kept[lo], nth - (uint32_t(lo) * kWave - before[lo]));
    to = to < keep ? to : keep - 1;  // (it is: the tables bound every access)
    lo = border, hi = strips - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (before[mid] <= inside + nth)
        lo = mid;
      else
        hi = mid - 1;
    }
    int src = lo * kWave + nth_bit(kept[lo], inside + nth - before[lo]);
    src = src < n ? src : n - 1;
    const auto bytes = [&](int place, int64_t *word) __attribute__((always_inline)) {
      const int page = int(uint32_t(place) / uint32_t(a.block_size));
      const int at = place - page * a.block_size;
      const int64_t block = table[page];
      *word = block * a.heads * a.block_size + at;
      return block * a.page + int64_t(at) * a.slot_bytes;
    };
    int64_t word_to, word_src;
    const int64_t byte_to = bytes(to, &word_to), byte_src = bytes(src, &word_src);
    if (m < moves) {
      ledger[word_to] = ledger[word_src];
      ledger[word_to + a.words] = ledger[word_src + a.words];
    }
    for (int i = 0; i < here; i += 4 * kRows) {  // four rows under way a lane
      piece x[4], y[4];
      int64_t to_row[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int row = i + u * kRows + lane / kLanes;  // below 64
        const int64_t from_row = __shfl(byte_src, row);
        to_row[u] = __shfl(byte_to, row);
        if (row < here) {
          x[u] = *reinterpret_cast<const piece *>(k + from_row);
          y[u] = *reinterpret_cast<const piece *>(k + a.half + from_row);
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i + u * kRows + lane / kLanes < here) {
          *reinterpret_cast<piece *>(k + to_row[u]) = x[u];
          *reinterpret_cast<piece *>(k + a.half + to_row[u]) = y[u];
        }
    }
  }
}

// A launch takes less than 2^32 threads.
constexpr int64_t kMostItems = UINT32_MAX / 1024;

struct EvictPlan {
  int32_t strips;
  size_t kept_at, before_at, bytes;
};

int evict_plan(const lumen_kv_layout *l, int32_t layers, int32_t bt_cols, int32_t num_reqs,
               EvictPlan *p) {
  if (bt_cols < 0 || num_reqs < 0) return LUMEN_ERR_INVALID_ARG;
  if (int64_t(bt_cols) * l->block_size > LUMEN_PAGED_MAX_PLACES) return LUMEN_ERR_UNSUPPORTED;
  int64_t items;
  if (__builtin_mul_overflow(int64_t(layers) * num_reqs, int64_t(l->num_kv_heads), &items) ||
      items > kMostItems)
    return LUMEN_ERR_UNSUPPORTED;
  p->strips = int32_t((int64_t(bt_cols) * l->block_size + kWave - 1) / kWave);
  const auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
  p->kept_at = up(size_t(items) * sizeof(int32_t));
  p->before_at = p->kept_at + up(size_t(items) * p->strips * sizeof(uint64_t));
  p->bytes = p->before_at + up(size_t(items) * p->strips * sizeof(uint32_t));
  return LUMEN_OK;
}

// --------------------------------------------------------------- release

constexpr int kReleaseThreads = 256;

struct ReleaseArgs {
  const int32_t *lens, *have;
  int32_t num_reqs;
  const int32_t *bt;
  int32_t bt_cols, block_size;
  int64_t num_blocks;
  int32_t *free_ids;
  const int64_t *free_count;
  int64_t free_cap;
  int64_t *free_now;
  int32_t *status;
};

__device__ __forceinline__ int32_t pages_of(int32_t places, int32_t bs) {
  const uint32_t whole = uint32_t(places) / uint32_t(bs);
  return int32_t(whole + (whole * uint32_t(bs) != uint32_t(places)));
}

// Every workgroup sums up the requests' pages in LDS (no second launch), then the
// grid strides over the pages that go back, each of which finds its request by
// bisection.
__global__ __launch_bounds__(kReleaseThreads) void release_kernel(ReleaseArgs a) {
  extern __shared__ int64_t upto[];  // pages of the requests up to each, with it
  __shared__ int64_t wave_sum[kReleaseThreads / kWave];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), R = a.num_reqs;
  const int per = (R + kReleaseThreads - 1) / kReleaseThreads;
  const int r0 = tid * per < R ? tid * per : R;
  const int r1 = r0 + per < R ? r0 + per : R;
  int err = LUMEN_OK;
  const auto pages = [&](int r, int32_t *first) {
    const int32_t n = a.lens[r], h = a.have[r];
    *first = 0;
    if (n < 0 || h < 0) {
      err = LUMEN_ERR_RANGE;
      return 0;
    }
    const int32_t last = pages_of(h, a.block_size);
    *first = pages_of(n, a.block_size);
    if (last <= *first) return 0;
    if (last > a.bt_cols) {
      err = LUMEN_ERR_RANGE;
      return 0;
    }
    return last - *first;
  };
  int64_t mine = 0;
  int32_t first;
  for (int r = r0; r < r1; ++r) {
    mine += pages(r, &first);
    upto[r] = mine;
  }
  int64_t sum = mine;
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t x = __shfl_up(sum, o);
    if (lane >= o) sum += x;
  }
  if (lane == kWave - 1) wave_sum[tid / kWave] = sum;
  __syncthreads();
  int64_t base = sum - mine, total = 0;
  for (int w = 0; w < kReleaseThreads / kWave; ++w) {
    if (w < tid / kWave) base += wave_sum[w];
    total += wave_sum[w];
  }
  for (int r = r0; r < r1; ++r) upto[r] += base;
  __syncthreads();
  int64_t count = *a.free_count;
  count = count < 0 ? 0 : count < a.free_cap ? count : a.free_cap;
  const int64_t room = a.free_cap - count;
  if (total > room) {
    total = room;
    err = err < LUMEN_ERR_CAPACITY ? err : LUMEN_ERR_CAPACITY;
  }
  if (blockIdx.x == 0 && tid == 0) *a.free_now = count + total;
  for (int64_t i = int64_t(blockIdx.x) * kReleaseThreads + tid; i < total;
       i += int64_t(gridDim.x) * kReleaseThreads) {
    int lo = 0, hi = R - 1;  // the first request with upto > i
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (upto[mid] > i)
        hi = mid;
      else
        lo = mid + 1;
    }
    const int32_t n = pages(lo, &first);
    const int64_t page = first + (i - (upto[lo] - n));
    const int32_t id = a.bt[int64_t(lo) * a.bt_cols + page];
    if (id < 0 || id >= a.num_blocks)
      err = err < LUMEN_ERR_BLOCK_ID ? err : LUMEN_ERR_BLOCK_ID;
    a.free_ids[count + i] = id;
  }
  record_wave(a.status, err);
}

}  // namespace

extern "C" {

int lumen_paged_append(const lumen_kv_layout *layout, int32_t layer, void *d_cache,
                       const lumen_attn_rows *k, const lumen_attn_rows *v,
                       const int64_t *d_slots, const int32_t *d_positions,
                       int64_t num_tokens, void *d_ledger, int32_t *d_status,
                       lumen_stream_t stream) {
  Pages p;
  int st = check_pages(layout, layer, 1, &p);
  if (st != LUMEN_OK) return st;
  if (num_tokens < 0 || !d_positions != !d_ledger) return LUMEN_ERR_INVALID_ARG;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if ((st = check_rows(k, num_tokens)) != LUMEN_OK) return st;
  if ((st = check_rows(v, num_tokens)) != LUMEN_OK) return st;
  if (num_tokens == 0) return LUMEN_OK;
  if (!d_slots || (!d_cache && layout->num_blocks > 0)) return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_cache, 16) || !aligned(d_slots, 8) || !aligned(d_positions, 4) ||
      !aligned(d_ledger, 4))
    return LUMEN_ERR_MISALIGNED;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  AppendArgs a;
  a.k = static_cast<uint8_t *>(d_cache) + int64_t(layer) * 2 * p.half;
  a.v = a.k + p.half;
  a.slot_limit = layout->num_blocks * layout->block_size;
  a.page = p.page;
  a.slot_bytes = p.slot;
  a.head_bytes = p.head;
  a.block_size = layout->block_size;
  a.heads = layout->num_kv_heads;
  a.weights = d_ledger ? static_cast<int32_t *>(d_ledger) + 2 * layer * ledger_words(layout)
                       : nullptr;
  a.places = d_ledger ? a.weights + ledger_words(layout) : nullptr;
  a.status = d_status;
  // rows are counted in 32 bits: a call over more of them is several launches
  const int64_t most = (int64_t(1) << 30) / (2 * a.heads);
  const int64_t step = most < 1 ? 1 : most;
  for (int64_t t = 0; t < num_tokens; t += step) {
    a.tokens = uint32_t(num_tokens - t < step ? num_tokens - t : step);
    a.rk = rows_of(k, t);
    a.rv = rows_of(v, t);
    a.slots = d_slots + t;
    a.positions = d_positions ? d_positions + t : nullptr;
    const int64_t per_token = 2 * int64_t(a.heads), rows = a.tokens * per_token;
    const int per = kRowThreads / (layout->head_dim / 8);
    // as many as run at once, and at least a token's
    const int64_t room = int64_t(cus) * (2048 / kRowThreads) * per;
    const int64_t taken = rows < room ? rows : room < per_token ? per_token : room;
    const int64_t blocks = (taken + per - 1) / per;
    a.at_once = uint32_t(blocks * per / per_token);
    hipLaunchKernelGGL(layout->head_dim == 64    ? append_kernel<64>
                       : layout->head_dim == 128 ? append_kernel<128>
                                                 : append_kernel<256>,
                       dim3(unsigned(blocks)), dim3(kRowThreads), 0,
                       static_cast<hipStream_t>(stream), a);
  }
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

size_t lumen_paged_evict_workspace_bytes(const lumen_kv_layout *layout, int32_t num_layers,
                                         int32_t bt_cols, int32_t num_reqs) {
  Pages p;
  EvictPlan plan;
  if (check_pages(layout, 0, num_layers, &p) != LUMEN_OK ||
      evict_plan(layout, num_layers, bt_cols, num_reqs, &plan) != LUMEN_OK ||
      num_reqs > LUMEN_ATTN_MAX_REQS)
    return 0;
  return plan.bytes;
}

int lumen_paged_evict(const lumen_kv_layout *layout, int32_t first_layer, int32_t num_layers,
                      void *d_cache, void *d_ledger, const int32_t *d_block_tables,
                      int32_t bt_cols, const int32_t *d_lens, const int32_t *d_keep,
                      const int32_t *d_recent_from, int32_t num_sinks, int32_t num_reqs,
                      int32_t *d_left, void *d_workspace, size_t workspace_bytes,
                      int32_t *d_status, lumen_stream_t stream) {
  Pages p;
  EvictPlan plan;
  int st = check_pages(layout, first_layer, num_layers, &p);
  if (st != LUMEN_OK) return st;
  if (num_layers < 1) return LUMEN_ERR_INVALID_ARG;
  if ((st = evict_plan(layout, num_layers, bt_cols, num_reqs, &plan)) != LUMEN_OK) return st;
  if ((st = check_status(d_status)) != LUMEN_OK) return st;
  if (num_reqs > LUMEN_ATTN_MAX_REQS) return LUMEN_ERR_TOO_MANY;
  if (num_reqs == 0) return LUMEN_OK;
  if (!d_lens || !d_keep || !d_recent_from || !d_left || !d_workspace ||
      (!d_block_tables && bt_cols > 0) ||
      ((!d_cache || !d_ledger) && layout->num_blocks > 0) || workspace_bytes < plan.bytes)
    return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_cache, 16) || !aligned(d_workspace, 16) || !aligned(d_ledger, 4) ||
      !aligned(d_block_tables, 4) || !aligned(d_lens, 4) || !aligned(d_keep, 4) ||
      !aligned(d_recent_from, 4) || !aligned(d_left, 4))
    return LUMEN_ERR_MISALIGNED;
  (void)hipGetLastError();
  EvictArgs a;
  a.words = ledger_words(layout);
  a.cache = static_cast<uint8_t *>(d_cache) + int64_t(first_layer) * 2 * p.half;
  a.ledger = static_cast<uint32_t *>(d_ledger) + int64_t(first_layer) * 2 * a.words;
  a.half = p.half;
  a.page = p.page;
  a.slot_bytes = p.slot;
  a.head_bytes = p.head;
  a.block_size = layout->block_size;
  a.heads = layout->num_kv_heads;
  a.num_blocks = layout->num_blocks;
  a.bt = d_block_tables;
  a.bt_cols = bt_cols;
  a.lens = d_lens;
  a.keep = d_keep;
  a.from = d_recent_from;
  a.sinks = num_sinks;
  a.num_reqs = num_reqs;
  a.left = d_left;
  a.status = d_status;
  char *ws = static_cast<char *>(d_workspace);
  a.moves = reinterpret_cast<int32_t *>(ws);
  a.kept = reinterpret_cast<uint64_t *>(ws + plan.kept_at);
  a.before = reinterpret_cast<uint32_t *>(ws + plan.before_at);
  a.strips = plan.strips;
  const int64_t cap = int64_t(bt_cols) * layout->block_size;
  const int64_t items = int64_t(num_layers) * num_reqs * a.heads;
  constexpr int kMost = 14336;  // ranks in 56 of a workgroup's 64 KB of LDS
  a.lds_keys = int32_t(cap < kMost ? cap : kMost);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cap <= 4096)
    hipLaunchKernelGGL(evict_select_kernel<256>, dim3(unsigned(items)), dim3(256),
                       size_t(a.lds_keys) * 4, s, a);
  else
    hipLaunchKernelGGL(evict_select_kernel<1024>, dim3(unsigned(items)), dim3(1024),
                       size_t(a.lds_keys) * 4, s, a);
  // a wavefront for 64 moves, of which a request has at most half its places
  int64_t parts = (cap / 2 + kMoveThreads - 1) / kMoveThreads;
  if (parts > 64) parts = 64;
  if (parts > int64_t(UINT32_MAX / kMoveThreads) / items) parts = UINT32_MAX / kMoveThreads / items;
  if (parts < 1) parts = 1;
  hipLaunchKernelGGL(layout->head_dim == 64    ? evict_move_kernel<64>
                     : layout->head_dim == 128 ? evict_move_kernel<128>
                                               : evict_move_kernel<256>,
                     dim3(unsigned(items * parts)), dim3(kMoveThreads), 0, s, a, int32_t(parts));
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

int lumen_paged_release(const int32_t *d_lens, const int32_t *d_have, int32_t num_reqs,
                        const int32_t *d_block_tables, int32_t bt_cols, int32_t block_size,
                        int64_t num_blocks, int32_t *d_free, const int64_t *d_free_count,
                        int64_t free_cap, int64_t *d_free_now, int32_t *d_status,
                        lumen_stream_t stream) {
  if (num_reqs < 0 || bt_cols < 0 || block_size < 1 || num_blocks < 0 || free_cap < 0)
    return LUMEN_ERR_INVALID_ARG;
  int st = check_status(d_status);
  if (st != LUMEN_OK) return st;
  if (num_reqs > LUMEN_ATTN_MAX_REQS) return LUMEN_ERR_TOO_MANY;
  if (!d_free_count || !d_free_now || (!d_free && free_cap > 0) ||
      (num_reqs > 0 && (!d_lens || !d_have || (!d_block_tables && bt_cols > 0))))
    return LUMEN_ERR_INVALID_ARG;
  if (!aligned(d_lens, 4) || !aligned(d_have, 4) || !aligned(d_block_tables, 4) ||
      !aligned(d_free, 4) || !aligned(d_free_count, 8) || !aligned(d_free_now, 8))
    return LUMEN_ERR_MISALIGNED;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  const ReleaseArgs a{d_lens,  d_have,       num_reqs, d_block_tables, bt_cols,    block_size,
                      num_blocks, d_free, d_free_count, free_cap,       d_free_now, d_status};
  // a thread a page, on a workgroup for 16 requests at most: each scans all of them
  const int64_t pages = int64_t(num_reqs) * bt_cols;
  int64_t blocks = (pages + kReleaseThreads - 1) / kReleaseThreads;
  if (blocks > num_reqs / 16 + 1) blocks = num_reqs / 16 + 1;
  if (blocks > cus) blocks = cus;
  if (blocks < 1) blocks = 1;
  hipLaunchKernelGGL(release_kernel, dim3(unsigned(blocks)), dim3(kReleaseThreads),
                     size_t(num_reqs) * sizeof(int64_t), static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

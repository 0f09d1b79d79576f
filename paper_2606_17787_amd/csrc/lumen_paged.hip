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

typedef uint32_t piece __attribute__((ext_vector_type(4)));  // 16 bytes of a row

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
  Divisor by_block;  // block_size
  uint32_t tokens;
  uint32_t at_once;  // tokens that the grid takes at a time
  int32_t *status;
};

// Rows of K and V as they are, 16 bytes a lane, D/8 lanes a row; a lane keeps its
// head of K or V for all of its tokens.  Bound by bytes: 4 D a token and head in
// and as many out.  For 16,411 tokens of 8 heads with D 128 the kernel takes 24.7 us, 5.5
// TB/s, of a pass's 30; for 256 it takes 3 of 4, the launch and two dependent reads.
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
  const auto store = [&](uint32_t tok, int64_t slot, const piece &x)
      __attribute__((always_inline)) {
    if (slot < 0 || slot >= a.slot_limit) {
      if (slot >= 0) err = LUMEN_ERR_BLOCK_ID;
      return;
    }
    int at;
    int64_t block;
    if (slot <= INT32_MAX) {
      block = quotient(a.by_block, int(slot), &at);
    } else {
      block = slot / a.block_size;
      at = int32_t(slot - block * a.block_size);
    }
    *reinterpret_cast<piece *>(cached + block * a.page + int64_t(at) * a.slot_bytes) = x;
    if (lane == 0 && a.weights) {
      const int64_t word = (block * a.heads + h) * a.block_size + at;
      if (is_v)
        a.places[word] = a.positions[tok];
      else
        a.weights[word] = 0;
    }
  };
  // two tokens at a time, their rows read beside their slots
  for (; t < a.tokens; t += 2 * a.at_once, row += 2 * step) {
    const bool two = a.tokens - t > a.at_once;
    const int64_t slot0 = a.slots[t], slot1 = two ? a.slots[t + a.at_once] : -1;
    const piece x0 = *reinterpret_cast<const piece *>(row);
    const piece x1 = *reinterpret_cast<const piece *>(two ? row + step : row);
    store(t, slot0, x0);
    store(t + a.at_once, slot1, x1);
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
  Divisor by_block;  // block_size
  int64_t num_blocks;
  const int32_t *bt;
  int32_t bt_cols;
  const int32_t *lens, *keep, *from;
  int32_t sinks, num_reqs;
  int32_t *left;
  int32_t *status;
  // the workspace, for each (layer, request, head): how many places move, and the
  // places given up and those that take them, the last first, or for each 64 of its
  // places which are kept and how many are before them
  int32_t *moves;
  uint16_t *lists;
  uint64_t *kept;
  uint32_t *before;
  int32_t strips;  // 64 places each, of a request at most
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

// Moves `count` places of one layer, request and head, at most 64: lane l knows where
// the l-th goes and where it is.  Rows of K and V go 16 bytes a lane, the ledger's
// words by the lane itself.  No place is both read and written.
template <int D>
__device__ __forceinline__ void move_places(const EvictArgs &a, const Item &it, int to, int src,
                                            int count) {
  constexpr int kLanes = D / 8, kRows = kWave / kLanes;  // rows at a time
  const int lane = threadIdx.x & (kWave - 1);
  const int32_t *table = a.bt + int64_t(it.r) * a.bt_cols;
  uint8_t *const k = a.cache + int64_t(it.layer) * 2 * a.half + int64_t(it.h) * a.head_bytes +
                     lane % kLanes * 16;
  uint32_t *const ledger = a.ledger + int64_t(it.layer) * 2 * a.words +
                           int64_t(it.h) * a.block_size;
  const auto bytes = [&](int place, int64_t *word) __attribute__((always_inline)) {
    int at;
    const int64_t block = table[quotient(a.by_block, place, &at)];
    *word = block * a.heads * a.block_size + at;
    return block * a.page + int64_t(at) * a.slot_bytes;
  };
  int64_t word_to, word_src;
  const int64_t byte_to = bytes(to, &word_to), byte_src = bytes(src, &word_src);
  if (lane < count) {
    ledger[word_to] = ledger[word_src];
    ledger[word_to + a.words] = ledger[word_src + a.words];
  }
  for (int i = 0; i < count; i += 4 * kRows) {  // four rows under way a lane
    piece x[4], y[4];
    int64_t to_row[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int row = i + u * kRows + lane / kLanes;  // below 64
      const int64_t from_row = __shfl(byte_src, row);
      to_row[u] = __shfl(byte_to, row);
      if (row < count) {
        x[u] = *reinterpret_cast<const piece *>(k + from_row);
        y[u] = *reinterpret_cast<const piece *>(k + a.half + from_row);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i + u * kRows + lane / kLanes < count) {
        *reinterpret_cast<piece *>(k + to_row[u]) = x[u];
        *reinterpret_cast<piece *>(k + a.half + to_row[u]) = y[u];
      }
  }
}

// What a workgroup does for one layer, request and head: which places are kept.
//
// Protected places are counted first: where they do not fill the budget, all of them
// are kept and the others are ranked, where they do, they are ranked alone.  The rank
// of the last one kept comes out of counts over the ranks' digits of 10 or 11 bits, from
// the highest on, until every rank left is kept.
//
// A thread holds the ranks of kPer places, one of each kThreads, for requests of up to
// kThreads * kPer; where kPer is 0 (longer ones), each pass reads them again.
//
// Where places move, the k-th place given up and the k-th one kept behind the budget
// belong together.  D is 0 where evict_move_kernel moves them; otherwise this
// workgroup does, with the two lists in LDS.
//
// Bound by vector instructions first, then by what comes one after the other in a
// workgroup: the table, the words, two or three digits' counts, the lists, the rows.  64
// requests of 2,064 places, 2,048 of them kept, in four layers of 8 heads: 41 us with the
// moves, for 34 MB of words and as many of rows; 1,780 vector instructions a wavefront are
// 57 thousand cycles a SIMD, 26 us of these.  16 prompts around 8,192 tokens to 1,024 in
// two layers: 76 us.
template <int kThreads, int kPer, int D>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(EvictArgs a) {
  constexpr int kWaves = kThreads / kWave;
  constexpr int kDigit = kThreads == 1024 ? 11 : 10, kBins = 1 << kDigit;
  constexpr int kOwn = kBins / kThreads;  // bins of a thread
  constexpr int kMostStrips = kPer ? kPer * kWaves : 1;
  // as many counts of a bin as keep lanes with the same digit from waiting for each other
  constexpr int kCopies = kThreads == 1024 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) uint32_t hist[kCopies][kBins];
  __shared__ uint32_t wave_a[kWaves], wave_b[kWaves];
  __shared__ uint32_t strip_more[kMostStrips], strip_same[kMostStrips];
  __shared__ uint16_t lists[2][D ? kThreads * kPer / 2 : 1];
  __shared__ uint32_t digit, above, inside;
  __shared__ int guarded, moved;
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
  const int32_t from = a.from[it.r];
  const uint32_t *weights = a.ledger + int64_t(it.layer) * 2 * a.words +
                            int64_t(it.h) * a.block_size;
  const int64_t block_words = int64_t(a.heads) * a.block_size;
  const auto page_of = [&](int i) __attribute__((always_inline)) {
    return quotient(a.by_block, i);
  };
  const auto word_of = [&](int i, int page, int32_t block) __attribute__((always_inline)) {
    return block * block_words + (i - page * a.block_size);
  };
  // ---- the weights and positions, and how many places are protected
  uint32_t held[kPer ? kPer : 1];
  bool guard[kPer ? kPer : 1];
  int mine = 0;
  if (!alone && n > keep) {
    bool bad = a.num_blocks == 0;
    if constexpr (kPer > 0) {
      if (!bad) {
        constexpr int kAtOnce = 4;
#pragma unroll
        for (int g = 0; g < kPer; g += kAtOnce) {
          if (g * kThreads >= n) break;
          int32_t block[kAtOnce], page[kAtOnce];
          uint32_t w[kAtOnce];
          int32_t pos[kAtOnce];
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j) {
            const int i = (g + j) * kThreads + tid, place = i < n ? i : n - 1;
            page[j] = page_of(place);
            block[j] = table[page[j]];
          }
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j) {
            const int i = (g + j) * kThreads + tid, place = i < n ? i : n - 1;
            const bool out = block[j] < 0 || block[j] >= a.num_blocks;
            bad |= out;
            const int64_t word = word_of(place, page[j], out ? 0 : block[j]);
            w[j] = weights[word];
            pos[j] = int32_t(weights[word + a.words]);
          }
#pragma unroll
          for (int j = 0; j < kAtOnce; ++j) {
            const int i = (g + j) * kThreads + tid;
            guard[g + j] = protects(pos[j], a.sinks, from);
            held[g + j] = rank_of(w[j]);
            mine += i < n && guard[g + j];
          }
        }
      }
    } else {
      const int pages = (n - 1) / a.block_size + 1;
      for (int p = tid; p < pages; p += kThreads)
        bad |= table[p] < 0 || table[p] >= a.num_blocks;
    }
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
  if constexpr (kPer == 0)
    for (int i = tid; i < n; i += kThreads)
      mine += protects(int32_t(weights[word_of(i, page_of(i), table[page_of(i)]) + a.words]),
                       a.sinks, from);
  if (tid == 0) guarded = 0;
#pragma unroll
  for (int b = 0; b < kOwn * kCopies; ++b) (&hist[0][0])[b * kThreads + tid] = 0;
  __syncthreads();
  for (int o = 1; o < kWave; o <<= 1) mine += __shfl_xor(mine, o);
  if (lane == 0) atomicAdd(&guarded, mine);
  __syncthreads();
  const bool among = guarded >= keep;
  if constexpr (kPer > 0) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (guard[j] != among) held[j] = guard[j] ? kAllRanks : kNoRank;
  }
  // calls f(i, rank, j) for the thread's places i: j of each kThreads
  const auto each = [&](const auto &f) __attribute__((always_inline)) {
    if constexpr (kPer > 0) {
#pragma unroll
      for (int j = 0; j < kPer; ++j)
        if (j * kThreads < n) f(j * kThreads + tid, held[j], j);
    } else {
      for (int j = 0; j * kThreads < n; ++j) {
        const int i = j * kThreads + tid;
        uint32_t rank = kNoRank;
        if (i < n) {
          const int64_t word = word_of(i, page_of(i), table[page_of(i)]);
          const bool g = protects(int32_t(weights[word + a.words]), a.sinks, from);
          rank = g != among ? (g ? kAllRanks : kNoRank) : rank_of(weights[word]);
        }
        f(i, rank, j);
      }
    }
  };
  // ---- the rank of the last place kept
  uint32_t last = 0, mask = 0, want = uint32_t(keep);
  for (int shift = 32 - kDigit; mask != 0xffffffffu; shift -= kDigit) {
    const int low = shift > 0 ? shift : 0;  // the last digit has fewer bits
    const uint32_t digits = (mask ? ~mask : 0xffffffffu) >> low;
    each([&](int i, uint32_t x, int) __attribute__((always_inline)) {
      if (i < n && (x & mask) == last) atomicAdd(&hist[tid % kCopies][x >> low & digits], 1u);
    });
    __syncthreads();
    // the thread's bins, the highest first
    uint32_t c[kOwn], sum = 0;
#pragma unroll
    for (int b = 0; b < kOwn; ++b) c[b] = 0;
#pragma unroll
    for (int y = 0; y < kCopies; ++y) {
      typedef uint32_t own __attribute__((ext_vector_type(kOwn)));
      own *const at = reinterpret_cast<own *>(&hist[y][kBins - kOwn * (tid + 1)]);
      const own x = *at;
#pragma unroll
      for (int b = 0; b < kOwn; ++b) c[b] += x[kOwn - 1 - b];
      *at = own(0);  // for the next digit
    }
#pragma unroll
    for (int b = 0; b < kOwn; ++b) sum += c[b];
    uint32_t upto = sum;
    for (int o = 1; o < kWave; o <<= 1) {
      const uint32_t x = __shfl_up(upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == kWave - 1) wave_a[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += wave_a[w];
    uint32_t over = upto - sum;
    if (over < want && want <= upto) {
#pragma unroll
      for (int b = 0; b < kOwn; ++b) {
        if (over < want && want <= over + c[b]) {
          digit = kBins - 1 - (kOwn * tid + b);
          above = over;
          inside = c[b];
        }
        over += c[b];
      }
    }
    __syncthreads();
    last |= digit << low;
    mask |= digits << low;
    want -= above;
    if (inside == want) break;  // all that are left are kept
  }
  // ---- every place above `last` is kept, and the first `want` of those at it
  const int strips = (n + kWave - 1) / kWave;
  const int half = (a.strips * kWave + 1) / 2;
  const auto to_at = [&](int m) __attribute__((always_inline)) -> uint16_t & {
    return D ? lists[0][m] : a.lists[id * 2 * half + m];
  };
  const auto src_at = [&](int m) __attribute__((always_inline)) -> uint16_t & {
    return D ? lists[1][m] : a.lists[id * 2 * half + half + m];
  };
  // What becomes of strip s, of whose places `more` and `same` are above and at `last`.
  const auto kept_of = [&](int s, uint64_t more, uint64_t same, uint32_t kept_before,
                           uint32_t same_before) __attribute__((always_inline)) {
    const uint64_t below = (uint64_t(1) << lane) - 1;
    const uint32_t nth = same_before + __popcll(same & below);
    const uint64_t bits = more | __ballot((same >> lane & 1) && nth < want);
    if (s == keep / kWave && lane == 0)
      moved = keep - int(kept_before + __popcll(bits & ((uint64_t(1) << keep % kWave) - 1)));
    if constexpr (kPer > 0) {
      const int i = s * kWave + lane;
      const int rank = int(kept_before + __popcll(bits & below));  // among the kept ones
      if (i < keep && !(bits >> lane & 1)) to_at(i - rank) = uint16_t(i);
      // the last of them first: how many are under the budget is not known yet
      if (i >= keep && bits >> lane & 1) src_at(keep - 1 - rank) = uint16_t(i);
    } else if (lane == 0) {
      a.kept[id * a.strips + s] = bits;
      a.before[id * a.strips + s] = kept_before;
    }
  };
  if constexpr (kPer > 0) {
    // strip j * kWaves + wave is the wavefront's j-th
    each([&](int i, uint32_t x, int j) __attribute__((always_inline)) {
      const uint64_t more = __ballot(i < n && (x & mask) > last);
      const uint64_t same = __ballot(i < n && (x & mask) == last);
      if (lane == 0) {
        strip_more[j * kWaves + wave] = __popcll(more);
        strip_same[j * kWaves + wave] = __popcll(same);
      }
    });
    __syncthreads();
    if (wave == 0) {  // what is before each strip
      uint32_t kept_before = 0, same_before = 0;
      for (int base = 0; base < strips; base += kWave) {
        const int s = base + lane;
        const uint32_t m = s < strips ? strip_more[s] : 0, e = s < strips ? strip_same[s] : 0;
        uint32_t same_to = e;
        for (int o = 1; o < kWave; o <<= 1) {
          const uint32_t x = __shfl_up(same_to, o);
          if (lane >= o) same_to += x;
        }
        const uint32_t b = same_before + same_to - e, room = want > b ? want - b : 0;
        const uint32_t k = m + (e < room ? e : room);
        uint32_t kept_to = k;
        for (int o = 1; o < kWave; o <<= 1) {
          const uint32_t x = __shfl_up(kept_to, o);
          if (lane >= o) kept_to += x;
        }
        if (s < strips) strip_more[s] = kept_before + kept_to - k, strip_same[s] = b;
        kept_before += __shfl(kept_to, kWave - 1);
        same_before += __shfl(same_to, kWave - 1);
      }
    }
    __syncthreads();
    each([&](int i, uint32_t x, int j) __attribute__((always_inline)) {
      const int s = j * kWaves + wave;
      const uint64_t more = __ballot(i < n && (x & mask) > last);
      const uint64_t same = __ballot(i < n && (x & mask) == last);
      if (s < strips) kept_of(s, more, same, strip_more[s], strip_same[s]);
    });
  } else {
    // a pass over the strips in order, kWaves at a time
    uint32_t kept_before = 0, same_before = 0;
    each([&](int i, uint32_t x, int j) __attribute__((always_inline)) {
      const uint64_t more = __ballot(i < n && (x & mask) > last);
      const uint64_t same = __ballot(i < n && (x & mask) == last);
      __syncthreads();
      if (lane == 0) wave_a[wave] = __popcll(more), wave_b[wave] = __popcll(same);
      __syncthreads();
      uint32_t k = kept_before, e = same_before;
      for (int w = 0; w < kWaves; ++w) {
        if (w == wave) {
          const int s = j * kWaves + wave;
          if (s < strips) kept_of(s, more, same, k, e);
        }
        const uint32_t room = want > e ? want - e : 0;
        k += wave_a[w] + (wave_b[w] < room ? wave_b[w] : room);
        e += wave_b[w];
      }
      kept_before = k;
      same_before = e;
    });
  }
  __syncthreads();
  if constexpr (D == 0) {
    if (tid == 0) a.moves[id] = moved;
  } else {
    const int moves = moved, per_wave = (moves + kWaves - 1) / kWaves;
    const int end = (wave + 1) * per_wave < moves ? (wave + 1) * per_wave : moves;
    for (int m = wave * per_wave; m < end; m += kWave) {
      const int count = end - m < kWave ? end - m : kWave;
      const int x = m + (lane < count ? lane : count - 1);
      move_places<D>(a, it, lists[0][x], lists[1][moves - 1 - x], count);
    }
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

// Moves what evict_select_kernel has chosen, 64 places a wavefront at a time.  With
// kLists their numbers are in the workspace; without, a lane finds them by bisection
// over the counts.
constexpr int kMoveThreads = 256;
template <int D, bool kLists>
__global__ __launch_bounds__(kMoveThreads) void evict_move_kernel(EvictArgs a, int32_t parts) {
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
  const int half = (a.strips * kWave + 1) / 2;
  const uint16_t *lists = a.lists + id * 2 * half;
  const uint32_t inside = uint32_t(keep - moves);  // kept places under `keep`
  for (; int64_t(c) * kWave < moves; c += waves) {
    const int count = moves - c * kWave < kWave ? moves - c * kWave : kWave;
    const int m = c * kWave + (lane < count ? lane : count - 1);
    int to, src;
    if constexpr (kLists) {
      to = lists[m];
      src = lists[half + moves - 1 - m];
    } else {
      const uint32_t nth = uint32_t(m);
      // the strip with the nth place given up: the last with at most nth before it
      int lo = 0, hi = border;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (uint32_t(mid) * kWave - before[mid] <= nth)
          lo = mid;
        else
          hi = mid - 1;
      }
      to = lo * kWave + nth_bit(~kept[lo], nth - (uint32_t(lo) * kWave - before[lo]));
      to = to < keep ? to : keep - 1;  // (it is: the tables bound every access)
      lo = border, hi = strips - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (before[mid] <= inside + nth)
          lo = mid;
        else
          hi = mid - 1;
      }
      src = lo * kWave + nth_bit(kept[lo], inside + nth - before[lo]);
      src = src < n ? src : n - 1;
    }
    move_places<D>(a, it, to, src, count);
  }
}

// A launch takes less than 2^32 threads.
constexpr int64_t kMostItems = UINT32_MAX / 1024;

// Places of a request up to which a thread of 1,024 holds its ranks: 16 prompts around
// 8,192 tokens take 114 us against 178 where each pass reads them again.
constexpr int kHeldPlaces = 1024 * 32;

// Counts of (layer, request, head) from which on their workgroups move the places
// themselves.  With fewer, the moves of one take longer than a second kernel over the
// whole chip.  In us, with the ledger's restoring copy, together against apart:
//     items              64       128       256       512
//     4,096 -> 1,024    35/37    46/54     67/100   115/180
//     16,000 -> 2,048   85/94   107/157
//     16,000 -> 8,000  159/114  188/181   291/323
//     32,000 -> 4,096  165/121  196/172   292/293
constexpr int kMovingItems = 128;

struct EvictPlan {
  int32_t strips;
  bool held, moving;
  size_t lists_at, before_at, bytes;
};

int evict_plan(const lumen_kv_layout *l, int32_t layers, int32_t bt_cols, int32_t num_reqs,
               EvictPlan *p) {
  if (bt_cols < 0 || num_reqs < 0) return LUMEN_ERR_INVALID_ARG;
  const int64_t cap = int64_t(bt_cols) * l->block_size;
  if (cap > LUMEN_PAGED_MAX_PLACES) return LUMEN_ERR_UNSUPPORTED;
  int64_t items;
  if (__builtin_mul_overflow(int64_t(layers) * num_reqs, int64_t(l->num_kv_heads), &items) ||
      items > kMostItems)
    return LUMEN_ERR_UNSUPPORTED;
  p->strips = int32_t((cap + kWave - 1) / kWave);
  p->held = cap <= kHeldPlaces;
  p->moving = p->held && items >= kMovingItems;
  const auto up = [](size_t n) { return (n + 255) & ~size_t(255); };
  const size_t strips = size_t(items) * p->strips;
  p->lists_at = up(size_t(items) * sizeof(int32_t));
  p->before_at = p->lists_at +
                 up(p->moving ? 0 : strips * (p->held ? kWave * sizeof(uint16_t) : sizeof(uint64_t)));
  p->bytes = p->before_at + up(p->held ? 0 : strips * sizeof(uint32_t));
  return LUMEN_OK;
}

// Threads, and how many places each holds, for requests of up to `cap` places: small
// workgroups share a compute unit, so that one counts while another waits.  With the
// ledger's restoring copy, 256 threads take 54 us for 64 requests of 2,064 places in
// four layers of 8 heads, 1,024 threads of 8 places 115 and of 32 places 175; for 8
// requests of 4,096 in eight layers 116, 118 and 132.  `cap` is what a table row has, for
// what the requests hold is not known here: these 64 take 51 us with a table of 2,064
// places, 112 with 8,192, 172 with 32,768 and 252 with 131,072.
template <int D>
void (*select_kernel(int64_t cap, int *threads))(EvictArgs) {
  *threads = cap <= 256 * 16 ? 256 : 1024;
  return cap <= 256 * 8    ? evict_select_kernel<256, 8, D>
         : cap <= 256 * 16 ? evict_select_kernel<256, 16, D>
         : cap <= 1024 * 8 ? evict_select_kernel<1024, 8, D>
                           : evict_select_kernel<1024, 32, D>;
}

template <bool kLists>
void (*move_kernel(int head_dim))(EvictArgs, int32_t) {
  return head_dim == 64    ? evict_move_kernel<64, kLists>
         : head_dim == 128 ? evict_move_kernel<128, kLists>
                           : evict_move_kernel<256, kLists>;
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
// bisection.  5 us for 64 requests and for 16 prompts' 7,000 pages: launch and latency.
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
  // workgroups read these while others write
  uint8_t *const cache = static_cast<uint8_t *>(d_cache) + int64_t(layer) * 2 * p.half;
  int32_t *const ledger =
      d_ledger ? static_cast<int32_t *>(d_ledger) + ledger_before(layout, layer) : nullptr;
  const size_t words = size_t(num_tokens) * sizeof(int32_t);
  if (overlap({{cache, size_t(2 * p.half)},
               {ledger, ledger ? size_t(2 * ledger_words(layout)) * sizeof(int32_t) : 0},
               {d_status, sizeof(int32_t)}},
              {{d_slots, 2 * words}, {d_positions, d_positions ? words : 0}}))
    return LUMEN_ERR_INVALID_ARG;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  AppendArgs a;
  a.k = cache;
  a.v = a.k + p.half;
  a.slot_limit = layout->num_blocks * layout->block_size;
  a.page = p.page;
  a.slot_bytes = p.slot;
  a.head_bytes = p.head;
  a.block_size = layout->block_size;
  a.by_block = divisor(a.block_size);
  a.heads = layout->num_kv_heads;
  a.weights = ledger;
  a.places = ledger ? ledger + ledger_words(layout) : nullptr;
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
  // workgroups read these while others write
  const size_t words = size_t(num_reqs) * sizeof(int32_t);
  const size_t ledger_bytes = size_t(2 * ledger_words(layout)) * sizeof(int32_t);
  uint8_t *const cache = static_cast<uint8_t *>(d_cache) + int64_t(first_layer) * 2 * p.half;
  uint8_t *const ledger = static_cast<uint8_t *>(d_ledger) + int64_t(first_layer) * ledger_bytes;
  if (overlap({{d_left, words},
               {d_status, sizeof(int32_t)},
               {d_workspace, plan.bytes},
               {cache, size_t(num_layers) * 2 * p.half},
               {ledger, size_t(num_layers) * ledger_bytes}},
              {{d_lens, words},
               {d_keep, words},
               {d_recent_from, words},
               {d_block_tables, words * size_t(bt_cols)}}))
    return LUMEN_ERR_INVALID_ARG;
  (void)hipGetLastError();
  EvictArgs a;
  a.words = ledger_words(layout);
  a.cache = cache;
  a.ledger = reinterpret_cast<uint32_t *>(ledger);
  a.half = p.half;
  a.page = p.page;
  a.slot_bytes = p.slot;
  a.head_bytes = p.head;
  a.block_size = layout->block_size;
  a.by_block = divisor(a.block_size);
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
  a.lists = reinterpret_cast<uint16_t *>(ws + plan.lists_at);
  a.kept = reinterpret_cast<uint64_t *>(ws + plan.lists_at);
  a.before = reinterpret_cast<uint32_t *>(ws + plan.before_at);
  a.strips = plan.strips;
  const int64_t cap = int64_t(bt_cols) * layout->block_size;
  const int64_t items = int64_t(num_layers) * num_reqs * a.heads;
  hipStream_t s = static_cast<hipStream_t>(stream);
  int threads = 1024;
  const int D = layout->head_dim;
  void (*select)(EvictArgs) = evict_select_kernel<1024, 0, 0>;
  if (plan.held)
    select = !plan.moving ? select_kernel<0>(cap, &threads)
             : D == 64    ? select_kernel<64>(cap, &threads)
             : D == 128   ? select_kernel<128>(cap, &threads)
                          : select_kernel<256>(cap, &threads);
  hipLaunchKernelGGL(select, dim3(unsigned(items)), dim3(unsigned(threads)), 0, s, a);
  if (!plan.moving) {
    // a wavefront for 64 moves, of which a request has at most half its places
    int64_t parts = (cap / 2 + kMoveThreads - 1) / kMoveThreads;
    if (parts > 64) parts = 64;
    if (parts > int64_t(UINT32_MAX / kMoveThreads) / items)
      parts = UINT32_MAX / kMoveThreads / items;
    if (parts < 1) parts = 1;
    const auto move = plan.held ? move_kernel<true>(D) : move_kernel<false>(D);
    hipLaunchKernelGGL(move, dim3(unsigned(items * parts)), dim3(kMoveThreads), 0, s, a,
                       int32_t(parts));
  }
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
  // workgroups read these while others write the list, its count or the status word
  const size_t words = size_t(num_reqs) * sizeof(int32_t);
  if (overlap({{d_free, size_t(free_cap) * sizeof(int32_t)},
               {d_free_now, sizeof(int64_t)},
               {d_status, sizeof(int32_t)}},
              {{d_lens, words},
               {d_have, words},
               {d_block_tables, words * size_t(bt_cols)},
               {d_free_count, sizeof(int64_t)}}))
    return LUMEN_ERR_INVALID_ARG;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  const ReleaseArgs a{d_lens,  d_have,       num_reqs, d_block_tables, bt_cols,    block_size,
                      num_blocks, d_free, d_free_count, free_cap,       d_free_now, d_status};
  // a thread a page; each workgroup scans all requests
  const int64_t pages = int64_t(num_reqs) * bt_cols;
  int64_t blocks = (pages + kReleaseThreads - 1) / kReleaseThreads;
  if (blocks > cus) blocks = cus;
  if (blocks < 1) blocks = 1;
  hipLaunchKernelGGL(release_kernel, dim3(unsigned(blocks)), dim3(kReleaseThreads),
                     size_t(num_reqs) * sizeof(int64_t), static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

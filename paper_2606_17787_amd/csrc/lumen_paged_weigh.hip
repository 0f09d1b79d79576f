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

constexpr int kWaves = 4, kThreads = kWaves * kWave;

struct WeighArgs : Call {
  const float *lse;
  float *weights;   // of the layer
  int32_t chunks;  // of a request's places at most
  int32_t chunk;   // weigh_few_kernel: places of one
};

// The sums of x[0..15] over the 32 lanes of a half: element i's in lanes i and i + 16
// of it.  Each step after the first adds two groups of lanes up and keeps half of the
// elements in each.
__device__ __forceinline__ float sum_by_lane(float *x, int lane) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float p, q;
    both<16>(x[i], &p, &q);
    x[i] = p + q;
  }
#pragma unroll
  for (int o = 8; o; o >>= 1) {
    const bool high = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      // (copies first: a choice among elements would be one by their number)
      const float low_one = x[i], high_one = x[i + o];
      const float send = high ? low_one : high_one;
      x[i] = (high ? high_one : low_one) + __shfl_xor(send, o);
    }
  }
  return x[0];
}

// The place, of 32 in a product's rows, that element i of half `half` is.
__device__ __forceinline__ int place_of(int i, int half) {
  return i / 4 * 8 + 4 * half + i % 4;
}

// What a query's scores are lowered by, in log2: one that saw nothing (lse
// -infinity) adds nothing.
__device__ __forceinline__ float shift_of(float lse) {
  return lse == -INFINITY ? INFINITY : lse * 1.44269504088896341f;
}

// Which of `count` places from place0 on a query sees that sees those up to `limit`.
__device__ __forceinline__ uint64_t sees_to(int limit, int place0) {
  const int to = limit - place0;
  return to >= 63 ? ~uint64_t(0) : to < 0 ? 0 : (uint64_t(2) << to) - 1;
}

// One place's slot: where its row of the keys starts, from the layer's, and its word
// of the ledger, for head 0; in is false where it does not count.
struct Slot {
  int64_t row, word;
  bool in;
};

__device__ __forceinline__ Slot slot_of(const Call &a, int r, int place, int n, int *err) {
  Slot s{0, 0, place < n};
  if (s.in) {
    int at;
    const int page = quotient(a.by_block, place, &at);
    const int64_t block = a.bt[int64_t(r) * a.bt_cols + page];
    s.in = block >= 0 && block < a.num_blocks;
    if (s.in) {
      s.row = block * a.page + int64_t(at) * a.slot_bytes;
      s.word = block * a.kv_heads * a.block_size + at;
    } else {
      *err = LUMEN_ERR_BLOCK_ID;
    }
  }
  return s;
}

// ------------------------------------------------- more than 128 query rows

constexpr int kGroups = 2;    // of four wavefronts
constexpr int kRows = 32 * kGroups;  // query rows of a tile
constexpr int kStages = 4;    // tiles in LDS
constexpr int kRound = 16;    // tiles whose lse is in LDS
constexpr int kChunk = 32 * kWaves;  // places of a workgroup

// A workgroup takes 128 places of a request and a KV head, a wavefront 32 of them,
// and holds their keys as the left operand of 32x32x16 products.  The query rows that
// see them come through LDS, 64 at a time and kStages tiles in turn, 32 for the first
// four wavefronts and 32 for the others, so that four of them share a SIMD: scores^T =
// K Q^T, queries across, so that a lane has one query's lse.  Its weights are added up
// by place in 32 bits, and over the lanes and the two groups at the end.  A tile's
// 16-byte chunks are permuted by row as attend's keys are.  Bound by the exponentials
// and sums, which take twice the cycles of the products they wait for: 2,048 tokens behind
// 6,144 places (32 query heads over 8, D 128) take 157 us, 0.77 PFLOP/s; with one group of
// wavefronts 201 against 169, and 167 with rows' addresses and ends looked at one by one.
template <int D, bool kBf16>
__global__ __launch_bounds__(kGroups *kThreads, 4) void weigh_kernel(WeighArgs a) {
  constexpr int kChunks = D / 8;
  constexpr int kAll = kGroups * kThreads;
  constexpr int kIssues = kRows * kChunks / kAll;
  constexpr int kTile = kRows * D * 2;  // bytes
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kStages * kTile];
  __shared__ float shifts[kRound * kRows], merged[kChunk];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const uint32_t lds_at = uint32_t(__builtin_amdgcn_readfirstlane(
      int(reinterpret_cast<uintptr_t>(LDS_PTR(uint8_t, lds))) + wave * kWave * 16));
  const auto *lds_bytes = LDS_PTR(const char, lds);
  const int group = wave / kWaves;  // of the wavefront
  const uint32_t read_q = (group * 32 + col) * D * 2 + 16 * (half ^ swizzle_k<D>(col));
  const int64_t items = int64_t(a.num_reqs) * a.chunks * a.kv_heads;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t rest = item / a.kv_heads;
    const int h = int(item - rest * a.kv_heads);
    const int r = int(rest / a.chunks), chunk = int(rest - int64_t(r) * a.chunks);
    Request q;
    int err = request(a, r, &q);
    if (chunk == 0 && h == 0 && wave == 0) record_wave(a.status, err);
    const int first_place = chunk * kChunk, place0 = first_place + wave % kWaves * 32;
    const int n = q.n < a.cap ? q.n : a.cap;
    if (q.m == 0 || first_place >= n) continue;
    // ---- the rows, from the first that sees a place of the workgroup's on
    const int behind = q.n - q.m, rows = q.m * a.group;
    const int first = (first_place > behind ? (first_place - behind) * a.group : 0) / kRows;
    const int tiles = (rows + kRows - 1) / kRows - first;
    const uint16_t *const qb = a.q.base + int64_t(q.q0) * a.q.token;
    const float *const lse = a.lse + int64_t(q.q0) * a.q_heads;
    // where each load of the next tile reads in the lane's row: it goes on by 64 rows with
    // one addition where whole tokens have as many, and with a few where they do not
    int next = first, head[kIssues];
    const uint16_t *from[kIssues];
    const auto chunk_of = [&](int i) __attribute__((always_inline)) {
      return 8 * ((tid % kChunks) ^ swizzle_k<D>((i * kAll + tid) / kChunks));
    };
    const auto row_at = [&](int x, int *hd) __attribute__((always_inline)) {
      const int tok = quotient(a.by_group, x, hd);
      return qb + int64_t(tok) * a.q.token + int64_t(h * a.group + *hd) * a.q.head;
    };
    int step_heads;
    const int step_toks = quotient(a.by_group, kRows, &step_heads);
    const int64_t step = step_toks * a.q.token + step_heads * a.q.head;
    const int64_t wrap = a.q.token - a.group * a.q.head;
    const uint16_t *const last = row_at(rows - 1, &head[0]);
#pragma unroll
    for (int i = 0; i < kIssues; ++i)
      from[i] = row_at(first * kRows + (i * kAll + tid) / kChunks, &head[i]) + chunk_of(i);
    const auto load_next = [&](int stage) __attribute__((always_inline)) {
      const uint32_t to = lds_at + stage * kTile;
      const int left = rows - next * kRows;
      ++next;
      if (left >= kRows) {
#pragma unroll
        for (int i = 0; i < kIssues; ++i) load_row(from[i], to + i * kAll * 16);
      } else {  // the last row again behind it
#pragma unroll
        for (int i = 0; i < kIssues; ++i)
          load_row((i * kAll + tid) / kChunks < left ? from[i] : last + chunk_of(i),
                   to + i * kAll * 16);
      }
#pragma unroll
      for (int i = 0; i < kIssues; ++i) from[i] += step;
      if (step_heads) {
#pragma unroll
        for (int i = 0; i < kIssues; ++i) {
          head[i] += step_heads;
          if (head[i] >= a.group) {
            head[i] -= a.group;
            from[i] += wrap;
          }
        }
      }
    };
    err = LUMEN_OK;
    const Slot slot = slot_of(a, r, place0 + col, n, &err);
    record_wave(a.status, err);
    frag8 k[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      k[i] = frag8{0, 0, 0, 0, 0, 0, 0, 0};
      if (slot.in)
        k[i] = *reinterpret_cast<const frag8 *>(a.k + int64_t(h) * a.head_bytes + slot.row +
                                                16 * half + 32 * i);
    }
    f32x16 sum;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.0f;
    for (int base = 0; base < tiles; base += kRound) {
      const int count = tiles - base < kRound ? tiles - base : kRound;
      __syncthreads();  // the tiles before are done with
      for (int i = tid; i < count * kRows; i += kAll) {
        const int x = (first + base) * kRows + i;
        int hd;
        const int tok = quotient(a.by_group, x < rows ? x : rows - 1, &hd);
        shifts[i] = shift_of(lse[int64_t(tok) * a.q_heads + h * a.group + hd]);
      }
      __syncthreads();
      // the keys are here before the first rows' loads, which the compiler does not
      // count, so that no wait for them is left in the loop
      __builtin_amdgcn_s_waitcnt(0x0f70);
#pragma unroll
      for (int i = 0; i < kStages - 1; ++i)
        if (i < count) load_next(i);
      int stage = 0;
      for (int at = 0; at < count; ++at) {
        const int tile = base + at, after = count - 1 - at;  // tiles loaded after this one
        if (after >= 2)
          wait_loads<2 * kIssues>();
        else if (after == 1)
          wait_loads<kIssues>();
        else
          wait_loads<0>();
        lds_barrier();
        if (at + kStages - 1 < count) load_next(stage ? stage - 1 : kStages - 1);
        const int row0 = (first + tile) * kRows + group * 32;
        const uint32_t in_stage = stage * kTile;
        f32x16 sc;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
          sc = mfma<kBf16>(k[i],
                           *reinterpret_cast<const __attribute__((address_space(3))) frag8 *>(
                               lds_bytes + ((read_q ^ (32 * i)) + in_stage)),
                           sc);
        const float shift = shifts[at * kRows + group * 32 + col];
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sc[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale_log2, -shift));
        if (row0 + 32 > rows || behind + quotient(a.by_group, row0 < rows ? row0 : rows - 1) < place0 + 31) {
          const int x = row0 + col;
          const uint64_t sees = x < rows ? sees_to(behind + quotient(a.by_group, x), place0) : 0;
          const uint32_t mine = uint32_t(sees) >> (4 * half);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (!(mine >> (i / 4 * 8 + i % 4) & 1)) sc[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[i] += sc[i];
        stage = stage + 1 < kStages ? stage + 1 : 0;
      }
    }
    float s[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = sum[i];
    const float total = sum_by_lane(s, lane);
    const int mine = place_of(col % 16, half);
    const int64_t word = __shfl(slot.word, mine) + int64_t(h) * a.block_size;
    const bool in = __shfl(int(slot.in), mine) && col < 16;
    __syncthreads();  // of the item before
    if (group && col < 16) merged[wave % kWaves * 32 + mine] = total;
    __syncthreads();
    if (!group && in) a.weights[word] += total + merged[wave % kWaves * 32 + mine];
  }
}

// ------------------------------------------------- up to 128 query rows

constexpr int kPlaces = 16 * kWaves;  // places of a step
constexpr int kEntries = 256;         // runs of places of a workgroup
constexpr int kMostPlaces16 = 1024;   // places of a workgroup

// The sum over a row of 16 lanes of s[i], for element i of 4 in the lanes with
// lane / 4 % 4 = i: two steps add mirrored lanes up and keep half of the elements in
// each, two more add what four lanes hold.
template <int kControl>
__device__ __forceinline__ float mirrored(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(
                                       0, __builtin_bit_cast(int, x), kControl, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum_of_four(const float *s, int lane) {
  const bool upper = lane & 8, odd = lane & 4;
  const float s0 = s[0], s1 = s[1], s2 = s[2], s3 = s[3];
  const float a = (upper ? s2 : s0) + mirrored<0x140>(upper ? s0 : s2);
  const float b = (upper ? s3 : s1) + mirrored<0x140>(upper ? s1 : s3);
  float c = (odd ? b : a) + mirrored<0x141>(odd ? a : b);
  c += mirrored<0x4e>(c);
  return c + mirrored<0xb1>(c);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));
template <bool kBf16>
__device__ __forceinline__ f32x4 mfma16(frag8 a, frag8 b, f32x4 c) {
  if constexpr (kBf16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
        __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(
        __builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A workgroup takes a stretch of a request's places for a KV head; each wavefront
// holds all of the request's query rows, in kTiles tiles of 16, as right operands of
// 16x16x32 products, and takes 16 of a step's 64 places.  The keys come through LDS,
// kStages steps in turn.  Where the places' rows start is laid out in LDS before, an
// entry for each run of places that cannot leave its page, as attend has it, and so are
// the weights that the places have; they are written back at the end.  Bound by the
// keys' bytes: 256 tokens behind around 2,048 places each (8 KV heads, D 128) take 310 us,
// 4.6 TB/s.  Writing the weights back is about 50 of them: each write is 64 bytes of
// another page.
template <int D, bool kBf16, int kTiles>
__global__ __launch_bounds__(kThreads, 2) void weigh_few_kernel(WeighArgs a) {
  constexpr int kChunks = D / 8;
  constexpr int kIssues = kPlaces * kChunks / kThreads;
  constexpr int kTile = kPlaces * D * 2;  // bytes
  __shared__ __attribute__((aligned(1024))) uint8_t lds[kStages * kTile];
  __shared__ float weights[kMostPlaces16];
  __shared__ int64_t run_row[kEntries];   // bytes from the layer's keys
  __shared__ int64_t run_word[kEntries];  // of the ledger
  __shared__ uint64_t live_at[kMostPlaces16 / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, quad = lane >> 4;
  const uint32_t lds_at = uint32_t(__builtin_amdgcn_readfirstlane(
      int(reinterpret_cast<uintptr_t>(LDS_PTR(uint8_t, lds))) + wave * kWave * 16));
  const auto *lds_bytes = LDS_PTR(const char, lds);
  const int my_row = wave * 16 + col;
  const uint32_t read_k = my_row * D * 2 + 16 * (quad ^ swizzle_k<D>(my_row));
  const int low = a.block_size & -a.block_size;
  const int run_shift = low >= 16 ? 4 : __builtin_ctz(low);
  const auto in_run = [&](int i) { return i & ((1 << run_shift) - 1); };
  const int64_t items = int64_t(a.num_reqs) * a.chunks * a.kv_heads;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const int64_t rest = item / a.kv_heads;
    const int h = int(item - rest * a.kv_heads);
    const int r = int(rest / a.chunks), chunk = int(rest - int64_t(r) * a.chunks);
    Request q;
    int err = request(a, r, &q);
    if (chunk == 0 && h == 0 && wave == 0) record_wave(a.status, err);
    const int first = chunk * a.chunk;
    const int n = q.n < a.cap ? q.n : a.cap;
    if (q.m == 0 || first >= n) continue;
    const int count = n - first < a.chunk ? n - first : a.chunk;
    const int steps = (count + kPlaces - 1) / kPlaces;
    __syncthreads();  // the item before is done with the tables and tiles
    // ---- the queries
    const int rows = q.m * a.group, behind = q.n - q.m;
    frag8 x[kTiles][D / 32];
    float shift[kTiles];
    int limit[kTiles];  // the last place that the lane's query sees
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int at = t * 16 + col, row = at < rows ? at : rows - 1;
      int head;
      const int tok = quotient(a.by_group, row, &head);
      head += h * a.group;
      const uint16_t *p = a.q.base + (int64_t(q.q0) + tok) * a.q.token +
                          int64_t(head) * a.q.head + 8 * quad;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) x[t][i] = *reinterpret_cast<const frag8 *>(p + 32 * i);
      shift[t] = shift_of(a.lse[(int64_t(q.q0) + tok) * a.q_heads + head]);
      limit[t] = at < rows ? behind + tok : -1;
    }
    // ---- where the places are
    err = LUMEN_OK;
    for (int i = tid; i < steps * kPlaces; i += kThreads) {
      const Slot s = slot_of(a, r, first + i, n, &err);
      const uint64_t live = __ballot(s.in);
      if (lane == 0) live_at[i / 64] = live;
      const int64_t word = s.word + int64_t(h) * a.block_size;
      if (in_run(i) == 0) {
        run_row[i >> run_shift] = s.row;
        run_word[i >> run_shift] = word;
      }
    }
    if (h == 0) record_wave(a.status, err);
    __syncthreads();
    const uint8_t *const kb = a.k + int64_t(h) * a.head_bytes;
    const auto load = [&](int step, int buf) __attribute__((always_inline)) {
      const int base = step * kPlaces;
      // all lookups first, so that one does not wait behind another's load
      const uint8_t *from[kIssues];
      const uint64_t live = live_at[step];
#pragma unroll
      for (int i = 0; i < kIssues; ++i) {
        const int place = base + (i * kThreads + tid) / kChunks;
        from[i] = kb + run_row[place >> run_shift] + int64_t(in_run(place)) * a.slot_bytes;
      }
      if (live != ~uint64_t(0)) {
#pragma unroll
        for (int i = 0; i < kIssues; ++i)
          if (!(live >> ((i * kThreads + tid) / kChunks) & 1))
            from[i] = reinterpret_cast<const uint8_t *>(kZeroRow);
      }
#pragma unroll
      for (int i = 0; i < kIssues; ++i)
        load_row(from[i] + 16 * ((tid % kChunks) ^ swizzle_k<D>((i * kThreads + tid) / kChunks)),
                 lds_at + buf * kTile + i * kThreads * 16);
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i)
      if (i < steps) load(i, i);
    // what the places weigh, beside the first keys
    for (int i = tid; i < steps * kPlaces; i += kThreads)
      weights[i] = live_at[i / 64] >> (i % 64) & 1
                       ? a.weights[run_word[i >> run_shift] + in_run(i)]
                       : 0.0f;
    // the compiler's own loads are here before the loop, so that no wait for them is
    // left in it
    __builtin_amdgcn_s_waitcnt(0x0f70);
    int buf = 0;
    for (int step = 0; step < steps; ++step) {
      const int after = steps - 1 - step;  // steps loaded after this one
      if (after >= 2)
        wait_loads<2 * kIssues>();
      else if (after == 1)
        wait_loads<kIssues>();
      else
        wait_loads<0>();
      lds_barrier();
      if (step + kStages - 1 < steps) load(step + kStages - 1, buf ? buf - 1 : kStages - 1);
      const int place0 = first + step * kPlaces + wave * 16;
      frag8 k[D / 32];
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        k[i] = *reinterpret_cast<const __attribute__((address_space(3))) frag8 *>(
            lds_bytes + ((read_k ^ (64 * i)) + buf * kTile));
      float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        if (t > 0 && t * 16 >= rows) break;
        f32x4 sc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < D / 32; ++i) sc = mfma16<kBf16>(k[i], x[t][i], sc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float y =
              __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i], a.scale_log2, -shift[t]));
          sum[i] += place0 + 4 * quad + i <= limit[t] ? y : 0.0f;
        }
      }
      const float total = sum_of_four(sum, lane);
      if (lane % 4 == 0)
        weights[step * kPlaces + wave * 16 + 4 * quad + lane / 4 % 4] += total;
      buf = buf + 1 < kStages ? buf + 1 : 0;
    }
    __syncthreads();
    for (int i = tid; i < count; i += kThreads)
      if (live_at[i / 64] >> (i % 64) & 1)
        a.weights[run_word[i >> run_shift] + in_run(i)] = weights[i];
  }
}

template <int kTiles>
void (*few_kernel(int head_dim, bool bf16))(WeighArgs) {
  if (head_dim == 64)
    return bf16 ? weigh_few_kernel<64, true, kTiles> : weigh_few_kernel<64, false, kTiles>;
  return bf16 ? weigh_few_kernel<128, true, kTiles> : weigh_few_kernel<128, false, kTiles>;
}

// Query rows up to which a wavefront holds them all (weigh_few_kernel, in 1, 4 or 8
// tiles of 16).  Of 16 prompts around 4,096 tokens 32, 64 and 128 rows take 41, 47 and 65
// us so and 93, 94 and 100 in weigh_kernel, of one with 16,384 tokens 128 rows take 22 and
// 22.  In 8 tiles always, 32 and 64 rows take 43 and 50 us, and 4 rows of 256 requests
// around 2,048 places 319 against 311.
constexpr int kFewRows = 128;

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
  // workgroups read these while others write
  float *const ledger = static_cast<float *>(d_ledger) + ledger_before(layout, layer);
  const size_t words = size_t(num_reqs) * sizeof(int32_t);
  if (overlap({{ledger, size_t(2 * ledger_words(layout)) * sizeof(float)},
               {d_status, sizeof(int32_t)}},
              {{static_cast<const uint8_t *>(d_cache) + int64_t(layer) * 2 * pages.half,
                size_t(2 * pages.half)},
               span_of(q, num_tokens, num_q_heads, layout->head_dim),
               {d_lse, size_t(num_tokens) * size_t(num_q_heads) * sizeof(float)},
               {d_block_tables, words * size_t(bt_cols)},
               {d_lens, words},
               {d_cu, words + sizeof(int32_t)}}))
    return LUMEN_ERR_INVALID_ARG;
  int cus = 0;
  if ((st = compute_units(&cus)) != LUMEN_OK) return st;
  (void)hipGetLastError();
  WeighArgs a;
  static_cast<Call &>(a) =
      call_of(layout, pages, layer, d_cache, d_block_tables, bt_cols, d_lens, d_cu, num_reqs, q,
              num_tokens, max_new, num_q_heads, scale, d_status);
  a.lse = d_lse;
  a.weights = ledger;
  const bool bf = dtype == LUMEN_ATTN_BF16;
  const int D = layout->head_dim;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const auto launch = [&](void (*kernel)(WeighArgs), int threads) {
    a.chunks = int32_t((uint32_t(a.cap) + uint32_t(a.chunk) - 1) / uint32_t(a.chunk));
    if (a.chunks < 1) a.chunks = 1;  // which looks at the requests
    int64_t groups = int64_t(num_reqs) * a.chunks;
    groups = groups < kMostGroups / a.kv_heads ? groups * a.kv_heads : kMostGroups;
    hipLaunchKernelGGL(kernel, dim3(unsigned(groups)), dim3(unsigned(threads)), 0, s, a);
  };
  const int64_t rows = int64_t(max_new) * a.group;
  if (rows <= kFewRows) {
    const int low = a.block_size & -a.block_size;
    a.chunk = kEntries * (low < 16 ? low : 16);
    if (a.chunk > kMostPlaces16) a.chunk = kMostPlaces16;
    // (The table's places count, which the requests need not fill: empty stretches cost
    // their launch.  One token behind 1,000 places with a table of 1,008, 8,192, 32,768 and
    // 131,072 places takes 5.9, 5.6, 8.2 and 12.9 us, 256 around 2,048 with 8,208, 32,768
    // and 131,072 310, 428 and 780.)
    // Smaller stretches where these would not fill the chip: one token behind 1,000 and
    // 16,384 places 5.7 and 11.2 us against 13.2 and 14.0, 32 tokens of 4 requests with
    // 8,000 places 25.7 against 28.6.  (256 requests around 2,048 places take 383 us in
    // stretches of 256, 331 of 512, 310 of 1,024 and 311 of 2,048.)
    while (a.chunk > kEntries &&
           int64_t(num_reqs) * a.kv_heads * ((int64_t(a.cap) + a.chunk - 1) / a.chunk) < 2 * cus)
      a.chunk /= 2;
    launch(rows <= 16 ? few_kernel<1>(D, bf) : rows <= 64 ? few_kernel<4>(D, bf)
                                                          : few_kernel<8>(D, bf),
           kThreads);
  } else {
    a.chunk = kChunk;
    launch(D == 64 ? (bf ? weigh_kernel<64, true> : weigh_kernel<64, false>)
                   : (bf ? weigh_kernel<128, true> : weigh_kernel<128, false>),
           kGroups * kThreads);
  }
  return hipGetLastError() == hipSuccess ? LUMEN_OK : LUMEN_ERR_HIP;
}

}  // extern "C"

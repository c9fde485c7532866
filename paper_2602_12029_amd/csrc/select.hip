// Choosing the blocks of its context that a request attends to: scores of all of them, and the highest.
//
// Score of block j for request r and KV head h: the largest over the group's query heads g of
//     (float(sum_c max(q_gc, 0) hi_jc + min(q_gc, 0) lo_jc) * s_j) * s_g
// on eight-bit codes (q of the query row with scale s_g, hi and lo of the block's summary with scale s_j).  The sum is a whole
// number below 2^24, so neither its order nor its grouping matters and every product is one float32 rounding: a choice is the
// same bits in every batch, split and run.  max and min of q side by side make it one product of 2 d terms on the matrix cores,
// v_mfma_i32_16x16x64_i8: A = 16 query rows' codes from LDS, B = 16 blocks' summaries straight from memory.
//
// Two launches.  Scoring: a workgroup per (range of a context, up to 64 query rows of the requests on it, KV head), HBM-bound
// by the summaries, which are read once for all of these.  Choice: a workgroup per (request, KV head), bound by the chain of its passes.
#include <algorithm>
#include <type_traits>

#include "kv_common.h"
#include "launch.h"

namespace psdev {

namespace {

typedef __attribute__((ext_vector_type(4))) int32_t i32x4;

struct SelectParams {
  const int32_t* blk;                  // the base layout's block array
  const ps_choice* choices;
  const ps_score_item* items;
  const void* q;
  const int8_t* summaries;
  const float* summary_scales;
  float* scores;
  int32_t* lists;                      // the selection's block array
  int64_t head_stride;
  int32_t num_q_heads, num_kv_heads, group;
};

constexpr int kRows = 64;              // query rows of an item, padded

// Codes of a query row, x[N] of 16 lanes each, four to a word, and its scale.  The largest magnitude is an integer maximum of
// the bits, which also shows what is not finite: counted as 0 (no number) or the largest finite one.
template <int N>
__device__ __forceinline__ float row16_codes(float (&x)[N], uint32_t (&codes)[N / 4]) {
  constexpr uint32_t kMagnitude = 0x7fffffffu, kMostBits = 0x7f7fffffu;
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) top = max(top, __float_as_uint(x[j]) & kMagnitude);
  if (__builtin_amdgcn_ballot_w64(top > kMostBits) != 0) {
    top = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      x[j] = x[j] == x[j] ? fminf(fmaxf(x[j], -kMost), kMost) : 0.f;
      top = max(top, __float_as_uint(x[j]) & kMagnitude);
    }
  }
  top = max(top, dpp_u32<kXor1>(0, top));
  top = max(top, dpp_u32<kXor2>(0, top));
  top = max(top, dpp_u32<kHalfMirror>(0, top));
  top = max(top, dpp_u32<kMirror>(0, top));
  const float scale = eight_bit_scale(__uint_as_float(top));
  eight_bit_codes<N>(x, scale, codes);
  return scale;
}

// Largest of a block's products with the rows of a request: a lane has the products with rows 4 kg + i of a tile, i = 0 .. 3, and the
// lanes 16 and 32 further on those of the other rows.  ROWS: a request's (1, 2: of v's first elements).
template <int ROWS>
__device__ __forceinline__ float rows_max(const float* v) {
  float m = v[0];
  if constexpr (ROWS >= 2) m = fmaxf(m, v[1]);
  if constexpr (ROWS >= 4) m = fmaxf(fmaxf(m, v[2]), v[3]);
  if constexpr (ROWS >= 8) {
    const auto swapped = __builtin_amdgcn_permlane16_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = fmaxf(__uint_as_float(swapped[0]), __uint_as_float(swapped[1]));
  }
  if constexpr (ROWS >= 16) {
    const auto swapped = __builtin_amdgcn_permlane32_swap(__float_as_uint(m), __float_as_uint(m), false, false);
    m = fmaxf(__uint_as_float(swapped[0]), __uint_as_float(swapped[1]));
  }
  return m;
}

// ROWS: rows of a request in a tile of 16, its group padded to a power of two; a group of more than 16 has tiles of its own
// (ROWS = 16) whose maxima are carried from one to the next.
// The query rows are the product's rows and the blocks its columns, so that the rows of a request lie in one lane's registers
// (the other way round the maxima took two DPP moves an element and more).  A wave takes two tiles of 16 blocks, and its chain is
// item, block ids, summaries; the query rows go the same way beside it, all under way before the codes are worked out.
// 64 / 128 / 256 blocks a workgroup, eight heads: 32 thousand blocks under three requests 24.1 / 20.1 / 20.7 us, 105 thousand under four
// 73.5 / 60.3 / 60.1, 8.7 thousand 10.6 / 9.7 / 10.6, 31 thousand under one 17.1 / 15.9 / 15.9; in rounds, four workgroups a compute unit,
// 22.6 / 70.4 / 10.9 / 15.4.  What bounds it is memory that is read 256 bytes a block at a time, blocks anywhere: 105 thousand blocks under
// one request 50 us, 4.2 TB/s, whether the loads cover whole 128-byte lines or halves of them, whatever the order of the heads.
template <int D, typename QT, int ROWS>
__global__ __launch_bounds__(256) void score_kernel(SelectParams p) {
  constexpr int kRowBytes = 2 * D, kLdsRow = kRowBytes + 16, kSteps = kRowBytes / 64, kPer = D / 16, NT = kPsScoreBlocks / 64;
  __shared__ __attribute__((aligned(16))) int8_t sm_q[kRows][kLdsRow];
  __shared__ __attribute__((aligned(16))) float sm_scale[kRows];
  const ps_score_item it = p.items[blockIdx.x / uint32_t(p.num_kv_heads)];
  const int h = int(blockIdx.x % uint32_t(p.num_kv_heads));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), n = lane & 15, kg = lane >> 4;
  const int tiles_per_request = ROWS == 16 ? (p.group + 15) >> 4 : 1;            // row tiles of a request, or
  constexpr int kRequests = 16 / ROWS;                                           // requests of a row tile
  const int row_tiles = ROWS == 16 ? it.n_req * tiles_per_request : (it.n_req + kRequests - 1) / kRequests;   // at most four
  // which request of the item and which head of its group a padded row is (padding: the last of them again, which changes no maximum)
  auto row_request = [&](int row) { return min(ROWS == 16 ? (row >> 4) / tiles_per_request : row / ROWS, it.n_req - 1); };
  auto row_head = [&](int row) { return min(ROWS == 16 ? row - 16 * tiles_per_request * ((row >> 4) / tiles_per_request) : row % ROWS, p.group - 1); };

  // this wave's blocks: lane l % (16 NT) has the l-th (past the end: the last again)
  const int first = 16 * NT * wave;
  const int id = p.blk[it.entry + min(first + lane % (16 * NT), it.num - 1)];
  // the query rows, 16 lanes to a row, 16 rows at a time
  struct alignas(sizeof(QT) * kPer) Piece { QT v[kPer]; };
  auto load_rows = [&](int pass) {
    const int row = 16 * pass + (int(threadIdx.x) >> 4);
    const int64_t r = p.choices[it.choice + row_request(row)].request;
    return *reinterpret_cast<const Piece*>(static_cast<const QT*>(p.q) + ((r * p.num_q_heads + h * p.group + row_head(row)) * D + n * kPer));
  };
  Piece raw = load_rows(0);
  const int64_t at = int64_t(id) * p.num_kv_heads + h;
  const float block_scale = p.summary_scales[at];
  i32x4 a[NT][kSteps];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int64_t tile_at = NT == 1 ? at : int64_t(__builtin_amdgcn_ds_bpermute((16 * t + n) << 2, id)) * p.num_kv_heads + h;
    const int8_t* row = p.summaries + tile_at * kRowBytes + 16 * kg;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) a[t][s] = *reinterpret_cast<const i32x4*>(row + 64 * s);
  }
  for (int pass = 0; pass < row_tiles; ++pass) {
    const int row = 16 * pass + (int(threadIdx.x) >> 4);
    float x[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      if constexpr (sizeof(QT) == 4) x[j] = raw.v[j];
      else x[j] = bf16_bits_to_f32(raw.v[j]);
    }
    if (pass + 1 < row_tiles) raw = load_rows(pass + 1);
    uint32_t codes[kPer / 4];
    const float scale = row16_codes<kPer>(x, codes);
#pragma unroll
    for (int j = 0; j < kPer / 4; ++j) {   // max(code, 0) and min(code, 0), byte by byte
      const uint32_t sign = (codes[j] >> 7) & 0x01010101u, negative = (sign << 8) - sign;
      *reinterpret_cast<uint32_t*>(&sm_q[row][n * kPer + 4 * j]) = codes[j] & ~negative;
      *reinterpret_cast<uint32_t*>(&sm_q[row][D + n * kPer + 4 * j]) = codes[j] & negative;
    }
    if (n == 0) sm_scale[row] = scale;
  }
  float sk[NT];   // of block n of every tile
#pragma unroll
  for (int t = 0; t < NT; ++t) sk[t] = NT == 1 ? block_scale : __int_as_float(__builtin_amdgcn_ds_bpermute((16 * t + n) << 2, __float_as_int(block_scale)));
  __syncthreads();

  constexpr int kOuts = ROWS < 4 ? 4 / ROWS : 1;   // requests that a lane has rows of
  float best[NT][kOuts];
  for (int rt = 0; rt < row_tiles; ++rt) {
    const bool carry = ROWS == 16 && rt % tiles_per_request != 0, last = ROWS != 16 || (rt + 1) % tiles_per_request == 0;
    const f32x4 sq = *reinterpret_cast<const f32x4*>(&sm_scale[16 * rt + 4 * kg]);
    i32x4 b[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) b[s] = *reinterpret_cast<const i32x4*>(&sm_q[16 * rt + n][64 * s + 16 * kg]);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      i32x4 dot = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[s], a[t][s], dot, 0, 0, 0);
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (float(dot[i]) * sk[t]) * sq[i];   // row 4 kg + i, block n
#pragma unroll
      for (int o = 0; o < kOuts; ++o) {
        const float m = rows_max<ROWS>(v + o * ROWS % 4);
        best[t][o] = carry ? fmaxf(best[t][o], m) : m;
      }
    }
    if (!last) continue;
#pragma unroll
    for (int o = 0; o < kOuts; ++o) {
      const int row = 16 * rt + 4 * kg + o * ROWS % 4;   // the first of a request's, or one that repeats what another lane stores
      if (ROWS > 4 && row % (ROWS == 16 ? 16 : ROWS) != 0) continue;
      if (ROWS != 16 && row / ROWS >= it.n_req) continue;
      const ps_choice* c = p.choices + it.choice + row_request(row);
      const int num = min(c->num, it.position + it.num);   // (a request may see less of the context)
      float* out = p.scores + 4 * (int64_t(c->scores) + int64_t(h) * ((c->num + 3) >> 2));
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int j = it.position + first + 16 * t + n;
        if (j < num) out[j] = best[t][o];
      }
    }
  }
}

// ---- choice ---------------------------------------------------------------------------------------------------------------
// A workgroup per (request, KV head).  Every position of the context gets a key: the order-preserving bits of its score (at least
// 0x007fffff, those of -inf), all ones where it is taken whatever its score, 0 where it is not to be listed.  The keys fall into
// 256 bins between the lowest and the highest; the bin with the need-th highest is settled by ranking its members against
// one another (by position where keys are equal) if they are few, else cut into bins again; what it gives up gets key 0, and the
// list is everything above its highest key or marked.  The first bins are even in the score itself: a float's bits put most
// scores into the few octaves at the top of their range.
//
// Nothing here is bound but by the chain of its steps: the keys stay in registers, PER a thread (0: in place of the scores, any
// number), waves meet by DPP rather than through LDS where they can, the members are ranked four at a time, and the block
// ids are fetched with the scores.  768 rows of up to 1900 positions 12.2 us with keys in LDS and exchanges by ds_bpermute, 6.8 now; 32 keys a
// thread, unrolled in every pass, were bound by fetching their instructions (32 rows of 8188, 34.8 us; sixteen waves to a row 14.2, 8.8 with
// the bins held and the block ids fetched early).
constexpr int kBins = 256, kFew = 256;
constexpr uint32_t kTaken = 0xffffffffu;

// order-preserving bits of a float, and back
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float((order >> 31) ? order ^ 0x80000000u : ~order); }

// over the wave, uniform
__device__ __forceinline__ uint32_t wave_min_u32(uint32_t x) {
  x = min(x, dpp_u32<kXor1>(x, x));
  x = min(x, dpp_u32<kXor2>(x, x));
  x = min(x, dpp_u32<kHalfMirror>(x, x));
  x = min(x, dpp_u32<kMirror>(x, x));
  x = min(x, dpp_u32<kBcast15, 0xa>(x, x));
  x = min(x, dpp_u32<kBcast31, 0xc>(x, x));
  return uint32_t(__builtin_amdgcn_readlane(int(x), 63));
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) { return ~wave_min_u32(~x); }
// over 4, 8 or 16 neighbouring lanes
template <int N>
__device__ __forceinline__ uint32_t few_min_u32(uint32_t x) {
  x = min(x, dpp_u32<kXor1>(x, x));
  x = min(x, dpp_u32<kXor2>(x, x));
  static_assert(N == 4 || N == 8 || N == 16, "");
  if constexpr (N >= 8) x = min(x, dpp_u32<kHalfMirror>(x, x));
  if constexpr (N == 16) x = min(x, dpp_u32<kMirror>(x, x));
  return uint32_t(__builtin_amdgcn_readfirstlane(int(x)));
}
// sum of the lanes up to and with this one
__device__ __forceinline__ uint32_t wave_prefix(uint32_t x) {
  x += dpp_u32<0x111>(0, x);   // row_shr 1, 2, 4, 8
  x += dpp_u32<0x112>(0, x);
  x += dpp_u32<0x114>(0, x);
  x += dpp_u32<0x118>(0, x);
  x += dpp_u32<kBcast15, 0xa>(0, x);
  x += dpp_u32<kBcast31, 0xc>(0, x);
  return x;
}

template <int THREADS, int PER>
__global__ __launch_bounds__(THREADS) void choose_kernel(SelectParams p) {
  constexpr int kWaves = THREADS / 64, kHeld = PER ? PER : 1;
  __shared__ uint32_t sm_bins[kBins], sm_low[kWaves], sm_high[kWaves], sm_count[kHeld * kWaves];
  __shared__ __attribute__((aligned(16))) uint64_t sm_few[kFew];
  __shared__ int32_t sm_ids[kFew];   // (their keys' rank decides: 1 taken, 0 not)
  __shared__ uint32_t sm_n, sm_top;
  const ps_choice c = p.choices[blockIdx.x / uint32_t(p.num_kv_heads)];
  const int h = int(blockIdx.x % uint32_t(p.num_kv_heads));
  const int tid = int(threadIdx.x), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int num = c.num;
  float* scores = p.scores + 4 * (int64_t(c.scores) + int64_t(h) * ((num + 3) >> 2));
  uint32_t* memory = reinterpret_cast<uint32_t*>(scores);   // PER = 0: the keys
  auto block_at = [&](int j) { return p.blk[j < c.num_root ? c.root_entry + j : c.prefix_entry + j - c.num_root]; };
  uint32_t key[kHeld];
  int32_t id[kHeld], slot[kHeld];
  uint32_t bin_at[kHeld];   // of the keys in question; the others: none
  // every position with its key, in any order
  auto each = [&](auto&& f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int u = 0; u < PER; ++u) f(u, u * THREADS + tid, key[u]);   // (past the end: 0)
    } else {
      for (int j = tid; j < num; j += THREADS) f(0, j, memory[j]);
    }
  };
  // lowest and highest of the workgroup; everybody gets both
  auto extent = [&](uint32_t& low, uint32_t& high) {
    low = wave_min_u32(low);
    high = wave_max_u32(high);
    if (lane == 0) {
      sm_low[wave] = low;
      sm_high[wave] = ~high;
    }
    __syncthreads();
    low = few_min_u32<kWaves>(sm_low[lane % kWaves]);
    high = ~few_min_u32<kWaves>(sm_high[lane % kWaves]);
  };

  uint32_t low = 0xffffffffu, high = 0;
  auto key_of = [&](float v, int j) {
    const uint32_t order = order_of(v == v ? v + 0.f : -__builtin_inff());   // (-0 counts as 0, and no number, from scales that are none, as the lowest)
    const bool open = j >= c.first && j < c.last && j != c.skip;
    if (open) {
      low = min(low, order);
      high = max(high, order);
    }
    return open ? order : j < num && j != c.skip ? kTaken : 0u;
  };
  if constexpr (PER > 0) {
    float v[kHeld];
#pragma unroll
    for (int u = 0; u < PER; ++u) v[u] = scores[min(u * THREADS + tid, num - 1)];
#pragma unroll
    for (int u = 0; u < PER; ++u) id[u] = block_at(min(u * THREADS + tid, num - 1));
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      key[u] = key_of(v[u], u * THREADS + tid);
      slot[u] = -1;
    }
  } else {
    for (int j = tid; j < num; j += THREADS) memory[j] = key_of(scores[j], j);
  }
  for (int i = tid; i < kBins; i += THREADS) {
    sm_bins[i] = 0;
    sm_few[i] = 0;
  }
  if (tid == 0) {
    sm_n = 0;
    sm_top = 0;
  }
  extent(low, high);

  uint32_t above = 0xfffffffeu;   // keys over this are listed
  int need = c.open;
  bool linear = true;
  while (need > 0) {
    // the candidates in question have keys in [low, high]
    const uint32_t range = high - low;
    const float bottom = value_of(low), width = value_of(high) - bottom;
    linear = linear && width < kMost && width > 0x1p-60f;   // (otherwise by the bits straight away)
    const float per_unit = linear ? float(kBins - 1) / width : 0.f;
    const int bits = range ? 32 - __builtin_clz(range) : 0, shift = bits > 8 ? bits - 8 : 0;
    auto bin_of = [&](uint32_t k) { return linear ? min(uint32_t((value_of(k) - bottom) * per_unit), uint32_t(kBins - 1)) : (k - low) >> shift; };
    each([&](int u, int, uint32_t k) {
      const uint32_t bin = k >= low && k <= high ? bin_of(k) : kTaken;
      bin_at[u] = bin;
      if (bin < uint32_t(kBins)) atomicAdd(&sm_bins[bin], 1u);
    });
    // (again, where they are not held)
    auto in = [&](int u, uint32_t k, uint32_t bin) { return PER > 0 ? bin_at[u] == bin : k >= low && k <= high && bin_of(k) == bin; };
    __syncthreads();
    // from the top: lane i of every wave holds bins 255 - 4 i .. 252 - 4 i
    uint32_t mine[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      mine[i] = sm_bins[kBins - 1 - 4 * lane - i];
      sum += mine[i];
    }
    const uint32_t upto = wave_prefix(sum);
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto >= uint32_t(need)));   // (never none: there are at least `need` candidates)
    uint32_t over = upto - sum, bin = 0, in_bin = 0;   // candidates above the bin, the bin, its candidates: by lane `at`
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (in_bin == 0 && over + mine[i] >= uint32_t(need)) {
        bin = uint32_t(kBins - 1 - 4 * lane - i);
        in_bin = mine[i];
      }
      if (in_bin == 0) over += mine[i];
    }
    over = uint32_t(__builtin_amdgcn_readlane(int(over), at));
    bin = uint32_t(__builtin_amdgcn_readlane(int(bin), at));
    in_bin = uint32_t(__builtin_amdgcn_readlane(int(in_bin), at));
    need -= int(over);
    if (in_bin <= uint32_t(kFew)) {
      each([&](int u, int j, uint32_t k) {
        if (in(u, k, bin)) {
          const uint32_t i = atomicAdd(&sm_n, 1u);
          sm_few[i] = uint64_t(k) << 32 | uint32_t(~j);
          if constexpr (PER > 0) slot[u] = int(i);
          atomicMax(&sm_top, k);
        }
      });
      __syncthreads();
      above = sm_top;
      if (tid < int(in_bin)) {
        const uint64_t own = sm_few[tid];
        int rank = 0;
        for (uint32_t i = 0; i < in_bin; i += 4) {   // (past the members: zeros)
#pragma unroll
          for (int e = 0; e < 4; ++e) rank += sm_few[i + e] > own;
        }
        if constexpr (PER > 0) sm_ids[tid] = rank < need;
        else memory[~uint32_t(own)] = rank < need ? kTaken : 0u;
      }
      __syncthreads();
      if constexpr (PER > 0) {
#pragma unroll
        for (int u = 0; u < PER; ++u)
          if (slot[u] >= 0) key[u] = sm_ids[slot[u]] ? kTaken : 0u;
      }
      break;
    }
    uint32_t bin_low = 0xffffffffu, bin_high = 0;
    each([&](int u, int, uint32_t k) {
      if (in(u, k, bin)) {
        bin_low = min(bin_low, k);
        bin_high = max(bin_high, k);
      }
    });
    __syncthreads();   // (the bins have been read)
    for (int i = tid; i < kBins; i += THREADS) sm_bins[i] = 0;
    extent(bin_low, bin_high);
    low = bin_low;
    high = bin_high;
    linear = false;
    if (low == high) {   // more equal ones than can be ranked: the first `need` of them, counted in order
      above = high;
      int before = 0;    // of the stretches in front
      auto stretch = [&](bool same) {   // THREADS positions in a row: is this thread's among the first `need`
        const uint64_t mask = __builtin_amdgcn_ballot_w64(same);
        __syncthreads();
        if (lane == 0) sm_low[wave] = uint32_t(__builtin_popcountll(mask));
        __syncthreads();
        int mine_at = before + int(__builtin_popcountll(mask & ((1ull << lane) - 1)));
        for (int w = 0; w < kWaves; ++w) {
          if (w < wave) mine_at += int(sm_low[w]);
          before += int(sm_low[w]);
        }
        return same && mine_at < need;
      };
      if constexpr (PER > 0) {
#pragma unroll
        for (int u = 0; u < PER; ++u) {
          const bool same = key[u] == high, first = stretch(same);
          if (same) key[u] = first ? kTaken : 0u;
        }
      } else {
        for (int j0 = 0; j0 < num; j0 += THREADS) {
          const int j = j0 + tid;
          const bool same = j < num && memory[j] == high, first = stretch(same);
          if (same) memory[j] = first ? kTaken : 0u;
        }
      }
      break;
    }
    __syncthreads();   // (sm_low and sm_high have been read)
  }
  __syncthreads();

  // the list, in ascending positions
  int32_t* list = p.lists + h * p.head_stride + c.list;
  const uint64_t in_front = (1ull << lane) - 1;
  if constexpr (PER > 0) {
    // counts of 64 positions in a row; every wave adds up those in front of its own
    uint64_t mask[kHeld];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      mask[u] = __builtin_amdgcn_ballot_w64(key[u] > above);
      if (lane == 0) sm_count[u * kWaves + wave] = uint32_t(__builtin_popcountll(mask[u]));
    }
    __syncthreads();
    constexpr int kMine = (PER * kWaves + 63) / 64;   // consecutive counts a lane has; a wave's are at the same place among them
    static_assert(kMine <= 4 && kWaves % 4 == 0 && (PER * kWaves) % kMine == 0, "");
    uint32_t sum = 0, part = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int e = kMine * lane + i;
      const uint32_t n = e < PER * kWaves ? sm_count[e] : 0;
      if (i < wave % kMine) part += n;
      sum += n;
    }
    part += wave_prefix(sum) - sum;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
      const uint32_t i = uint32_t(__builtin_amdgcn_readlane(int(part), (u * kWaves + wave) / kMine)) + uint32_t(__builtin_popcountll(mask[u] & in_front));
      if (((mask[u] >> lane) & 1) && i < uint32_t(c.count)) list[i] = id[u];
    }
  } else {
    // a stretch of positions per wave, counted, then written
    const int stretch = (num + 64 * kWaves - 1) / (64 * kWaves) * 64, begin = wave * stretch, end = min(num, begin + stretch);
    uint32_t count = 0;
    for (int j0 = begin; j0 < end; j0 += 64) count += uint32_t(__builtin_popcountll(__builtin_amdgcn_ballot_w64(j0 + lane < end && memory[j0 + lane] > above)));
    if (lane == 0) sm_low[wave] = count;
    __syncthreads();
    uint32_t base = 0;
    for (int w = 0; w < wave; ++w) base += sm_low[w];
    for (int j0 = begin; j0 < end; j0 += 64) {
      const int j = j0 + lane;
      const uint64_t mask = __builtin_amdgcn_ballot_w64(j < end && memory[j] > above);
      const uint32_t i = base + uint32_t(__builtin_popcountll(mask & in_front));
      if (((mask >> lane) & 1) && i < uint32_t(c.count)) list[i] = block_at(j);
      base += uint32_t(__builtin_popcountll(mask));
    }
  }
}

}  // namespace

int32_t launch_select_blocks(const ps_layout* base, const void* dev_tables, const ps_layout* sel, void* sel_tables, const void* q,
                             const int8_t* summaries, const float* summary_scales, float* scores, hipStream_t st) {
  const ps_geometry& g = base->geo;
  const ps_layout::selection& s = *sel->sel;
  int32_t* t = static_cast<int32_t*>(sel_tables);
  SelectParams p{};
  p.blk = static_cast<const int32_t*>(dev_tables) + base->off_blk;
  p.choices = reinterpret_cast<const ps_choice*>(t + s.off_choices);
  p.items = reinterpret_cast<const ps_score_item*>(t + s.off_score_items);
  p.q = q;
  p.summaries = summaries;
  p.summary_scales = summary_scales;
  p.scores = scores;
  p.lists = t + sel->off_blk;
  p.head_stride = sel->head_stride;
  p.num_q_heads = g.num_q_heads;
  p.num_kv_heads = g.num_kv_heads;
  p.group = g.num_q_heads / g.num_kv_heads;
  const int64_t n_items = int64_t(s.score_items.size() * 4 / sizeof(ps_score_item)), n_choices = int64_t(s.choices.size() * 4 / sizeof(ps_choice));
  if (n_items * g.num_kv_heads > kMaxWorkgroups || n_choices * g.num_kv_heads > kMaxWorkgroups / 4) return PS_ERR_UNSUPPORTED;   // (up to 1024 threads)
  const dim3 grid(unsigned(n_items * g.num_kv_heads));
#define PS_SCORE(D, T, ROWS) hipLaunchKernelGGL((score_kernel<D, T, ROWS>), grid, dim3(256), 0, st, p)
#define PS_SCORE_C(D, T)                                                                                                          \
  if (p.group == 1) PS_SCORE(D, T, 1); else if (p.group == 2) PS_SCORE(D, T, 2); else if (p.group <= 4) PS_SCORE(D, T, 4);         \
  else if (p.group <= 8) PS_SCORE(D, T, 8); else PS_SCORE(D, T, 16)
#define PS_SCORE_D(T) if (g.head_dim == 64) { PS_SCORE_C(64, T); } else if (g.head_dim == 128) { PS_SCORE_C(128, T); } else { PS_SCORE_C(256, T); }
  if (g.q_dtype == PS_F32) { PS_SCORE_D(float) } else { PS_SCORE_D(uint16_t) }
#undef PS_SCORE_D
#undef PS_SCORE_C
#undef PS_SCORE
  const dim3 rows(unsigned(n_choices * g.num_kv_heads));
  // Four keys a thread and as many waves as that takes; what sixteen waves do not hold so, eight and sixteen a thread; the rest in memory.
  // Scores and choice, 32 / 768 rows (256 from 4000 on), threads x keys: 875 positions 256x4 8.8 / 16.8 us, 256x8 9.8 / 17.8, 1024x4
  // 9.3 / 24.8; 1875 positions 512x4 9.1 / 28.3, 256x8 10.3 / 29.0, 1024x4 9.7 / 35.4; 4000 1024x4 9.6 / 21.7, 1024x8 11.1 / 23.0, 512x8
  // 10.0 / 22.1, 256x16 12.1 / 24.3; 8125 1024x8 13.1 / 23.9 (192 rows), 1024x16 18.1 / 32.6, in memory 18.4 / 31.5; 12500 1024x16 23.6 /
  // 35.9 (96 rows), in memory 28.4 / 40.5.
#define PS_CHOOSE(THREADS, PER) hipLaunchKernelGGL((choose_kernel<THREADS, PER>), rows, dim3(THREADS), 0, st, p)
  if (s.most_candidates <= 4 * 256) PS_CHOOSE(256, 4);
  else if (s.most_candidates <= 4 * 512) PS_CHOOSE(512, 4);
  else if (s.most_candidates <= 4 * 1024) PS_CHOOSE(1024, 4);
  else if (s.most_candidates <= 8 * 1024) PS_CHOOSE(1024, 8);
  else if (s.most_candidates <= 16 * 1024) PS_CHOOSE(1024, 16);
  else PS_CHOOSE(1024, 0);
#undef PS_CHOOSE
  return PS_OK;
}

}  // namespace psdev

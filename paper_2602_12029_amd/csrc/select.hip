// Choosing the blocks of its context that a request attends to: scores of all of them, and the highest.
//
// Score of block j for request r and KV head h: the largest over the group's query heads g of
//     (float(sum_c max(q_gc, 0) hi_jc + min(q_gc, 0) lo_jc) * s_j) * s_g
// on eight-bit codes (q of the query row with scale s_g, hi and lo of the block's summary with scale s_j).  The sum is a whole
// number below 2^24, so neither its order nor its grouping matters and every product is one float32 rounding: a choice is the
// same bits in every batch, split and run.  max and min of q side by side make it one product of 2 d terms on the matrix cores,
// v_mfma_i32_16x16x64_i8: A = 16 blocks' summaries straight from memory, B = 16 query rows' codes from LDS.
//
// Two launches.  Scoring: a workgroup per (range of a context, up to 64 query rows of the requests on it, KV head), HBM-bound
// by the summaries, which are read once for all of these.  Choice: a workgroup per (request, KV head) with the scores in registers:
// the K-th highest by histograms over ever narrower ranges, then the list in ascending order.
#include <algorithm>

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
constexpr float kMost = 0x1.fffffep127f;

__device__ __forceinline__ float row16_allreduce_max(float x) {
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true)));
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true)));
  x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true)));
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x140, 0xf, 0xf, true)));
}
// ... over aligned groups of COLS lanes of a 16-lane row
template <int COLS>
__device__ __forceinline__ float columns_max(float x) {
  if constexpr (COLS >= 2) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true)));
  if constexpr (COLS >= 4) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true)));
  if constexpr (COLS >= 8) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true)));
  if constexpr (COLS >= 16) x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x140, 0xf, 0xf, true)));
  return x;
}

// COLS: columns of a request in a tile of 16 rows, its group padded to a power of two; a group of more than 16 has tiles of its
// own (COLS = 16) whose maxima are carried from one to the next.
template <int D, typename QT, int COLS>
__global__ __launch_bounds__(256) void score_kernel(SelectParams p) {
  constexpr int kRowBytes = 2 * D, kLdsRow = kRowBytes + 16, kSteps = kRowBytes / 64, kPer = D / 16;
  __shared__ __attribute__((aligned(16))) int8_t sm_q[kRows][kLdsRow];
  __shared__ float sm_scale[kRows];
  const ps_score_item it = p.items[blockIdx.x];
  const int h = blockIdx.y;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), n = lane & 15, kg = lane >> 4;
  const int tiles_per_request = COLS == 16 ? (p.group + 15) >> 4 : 1;            // row tiles of a request, or
  constexpr int kRequests = 16 / COLS;                                           // requests of a row tile
  const int row_tiles = COLS == 16 ? it.n_req * tiles_per_request : (it.n_req + kRequests - 1) / kRequests;
  // which request of the item and which head of its group a padded row is; head >= group: none
  auto row_request = [&](int row) { return COLS == 16 ? (row >> 4) / tiles_per_request : row / COLS; };
  auto row_head = [&](int row) { return COLS == 16 ? row - 16 * tiles_per_request * row_request(row) : row % COLS; };

  // the query rows' codes: 16 lanes to a row
  for (int row = int(threadIdx.x) >> 4; row < 16 * row_tiles; row += 16) {
    const int req = row_request(row), head = row_head(row);
    const bool live = req < it.n_req && head < p.group;
    float x[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = 0.f;
    if (live) {
      const int64_t at = (int64_t(p.choices[it.choice + req].request) * p.num_q_heads + h * p.group + head) * D + n * kPer;
      const QT* src = static_cast<const QT*>(p.q) + at;
#pragma unroll
      for (int j = 0; j < kPer; ++j) {
        float v;
        if constexpr (sizeof(QT) == 4) v = src[j];
        else v = bf16_bits_to_f32(src[j]);
        x[j] = v == v ? fminf(fmaxf(v, -kMost), kMost) : 0.f;
      }
    }
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) top = fmaxf(top, fabsf(x[j]));
    float scale = row16_allreduce_max(top) * (1.f / 127.f);
    if (!(scale >= 0x1p-126f)) scale = 1.f;
#pragma unroll
    for (int j = 0; j < kPer; j += 4) {
      uint32_t hi = 0, lo = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int code = int(fminf(fmaxf(__builtin_rintf(x[j + i] / scale), -127.f), 127.f));
        hi |= uint32_t(max(code, 0) & 0xff) << (8 * i);
        lo |= uint32_t(min(code, 0) & 0xff) << (8 * i);
      }
      *reinterpret_cast<uint32_t*>(&sm_q[row][n * kPer + j]) = hi;
      *reinterpret_cast<uint32_t*>(&sm_q[row][D + n * kPer + j]) = lo;
    }
    if (n == 0) sm_scale[row] = scale;
  }
  __syncthreads();

  for (int t = wave; 16 * t < it.num; t += 4) {
    const int id = p.blk[it.entry + min(16 * t + n, it.num - 1)];
    const int64_t at = int64_t(id) * p.num_kv_heads + h;
    const int8_t* row = p.summaries + at * kRowBytes + 16 * kg;
    i32x4 a[kSteps];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) a[s] = *reinterpret_cast<const i32x4*>(row + 64 * s);
    const float block_scale = p.summary_scales[at];
    float sk[4];   // of the blocks this lane gets the products of: 4 kg + i
#pragma unroll
    for (int i = 0; i < 4; ++i) sk[i] = __int_as_float(__builtin_amdgcn_ds_bpermute((4 * kg + i) << 2, __float_as_int(block_scale)));
    float best[4];
    for (int rt = 0; rt < row_tiles; ++rt) {
      i32x4 dot = {0, 0, 0, 0};
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
        dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[s], *reinterpret_cast<const i32x4*>(&sm_q[16 * rt + n][64 * s + 16 * kg]), dot, 0, 0, 0);
      const int rowi = 16 * rt + n, req = row_request(rowi), head = row_head(rowi);
      const float sq = sm_scale[rowi];
      const bool carry = COLS == 16 && rt % tiles_per_request != 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = head < p.group ? (float(dot[i]) * sk[i]) * sq : -__builtin_inff();
        const float m = columns_max<COLS>(v);
        best[i] = carry ? fmaxf(best[i], m) : m;
      }
      if (COLS == 16 && (rt + 1) % tiles_per_request != 0) continue;
      if (n % COLS != 0 || req >= it.n_req) continue;
      const ps_choice* c = p.choices + it.choice + req;
      const int j = it.position + 16 * t + 4 * kg, num = min(c->num, it.position + it.num);   // (a request may see less of the context)
      float* out = p.scores + 4 * (int64_t(c->scores) + int64_t(h) * ((c->num + 3) >> 2));
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j + i < num) out[j + i] = best[i];
    }
  }
}

// ---- choice ---------------------------------------------------------------------------------------------------------------
// PER x 256 scores a workgroup holds in registers; 0: any number, read again in every round.
constexpr int kBins = 256;

template <int PER>
struct Scores {
  float v[PER];
  __device__ __forceinline__ Scores(const float* s, int num) {
#pragma unroll
    for (int u = 0; u < PER; ++u) v[u] = s[min(256 * u + int(threadIdx.x), num - 1)] + 0.f;   // (-0 counts as 0)
  }
  __device__ __forceinline__ float at(int u) const { return v[u]; }
};
template <>
struct Scores<0> {
  const float* s;
  int num;
  __device__ __forceinline__ Scores(const float* from, int n) : s(from), num(n) {}
  __device__ __forceinline__ float at(int u) const { return s[min(256 * u + int(threadIdx.x), num - 1)] + 0.f; }
};

// order-preserving bits of a float
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

template <int PER>
__global__ __launch_bounds__(256) void choose_kernel(SelectParams p) {
  constexpr int kMostRounds = PER ? PER : kPsSelectMostBlocks / 256;
  __shared__ uint32_t sm_bins[kBins], sm_low[4], sm_high[4];
  __shared__ uint16_t sm_count[4 * kMostRounds];      // chosen of 64 positions in a row (of them 64 at most)
  __shared__ uint32_t sm_base[4 * kMostRounds];
  const ps_choice c = p.choices[blockIdx.x / uint32_t(p.num_kv_heads)];
  const int h = int(blockIdx.x % uint32_t(p.num_kv_heads));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int rounds = (c.num + 255) >> 8;
  const Scores<PER> scores(p.scores + 4 * (int64_t(c.scores) + int64_t(h) * ((c.num + 3) >> 2)), c.num);
  auto each = [&](auto&& f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int u = 0; u < PER; ++u)
        if (u < rounds) f(u, 256 * u + int(threadIdx.x));
    } else {
      for (int u = 0; u < rounds; ++u) f(u, 256 * u + int(threadIdx.x));
    }
  };
  auto always = [&](int j) { return j < c.num && (j < c.first || j >= c.last) && j != c.skip; };
  auto open = [&](int j) { return j >= c.first && j < c.last && j != c.skip; };
  // lowest and highest of the workgroup; everybody gets both
  auto extent = [&](uint32_t low, uint32_t high, uint32_t& lowest, uint32_t& highest) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      low = min(low, uint32_t(__builtin_amdgcn_ds_bpermute((lane ^ m) << 2, int(low))));
      high = max(high, uint32_t(__builtin_amdgcn_ds_bpermute((lane ^ m) << 2, int(high))));
    }
    __syncthreads();
    if (lane == 0) {
      sm_low[wave] = low;
      sm_high[wave] = high;
    }
    __syncthreads();
    lowest = min(min(sm_low[0], sm_low[1]), min(sm_low[2], sm_low[3]));
    highest = max(max(sm_high[0], sm_high[1]), max(sm_high[2], sm_high[3]));
  };

  // Of the open positions those with order above `above` are taken, and `equal` of those with exactly that order, lowest first.
  uint32_t above = 0xffffffffu;
  int equal = 0, need = c.open;
  if (need > 0) {
    // the candidates still in question have orders in [low, high]; in every round they fall into 256 bins, and the one with
    // the need-th highest is looked at more closely.  The first round's bins are even in the score itself (a float's bits would put
    // most scores in the few octaves at the top of their range), the others' in the order.
    uint32_t low = 0xffffffffu, high = 0;
    each([&](int u, int j) {
      if (open(j)) {
        low = min(low, order_of(scores.at(u)));
        high = max(high, order_of(scores.at(u)));
      }
    });
    extent(low, high, low, high);
    bool linear = true;
    for (;;) {
      const uint32_t range = high - low;
      if (range == 0) {   // all the same: the first `need` of them
        above = low;
        equal = need;
        break;
      }
      auto value_of = [](uint32_t order) { return __uint_as_float((order >> 31) ? order ^ 0x80000000u : ~order); };
      const float bottom = value_of(low), width = value_of(high) - bottom;
      // (a width that overflows or is tiny: by order straight away)
      linear = linear && width < kMost && width > 0x1p-60f;
      const float per_unit = linear ? float(kBins - 1) / width : 0.f;
      const int bits = 32 - __builtin_clz(range), shift = bits > 8 ? bits - 8 : 0;
      auto bin_of = [&](float v) { return linear ? min(uint32_t((v - bottom) * per_unit), uint32_t(kBins - 1)) : (order_of(v) - low) >> shift; };
      __syncthreads();
      sm_bins[threadIdx.x] = 0;
      __syncthreads();
      each([&](int u, int j) {
        const float v = scores.at(u);
        const uint32_t o = order_of(v);
        if (open(j) && o >= low && o <= high) atomicAdd(&sm_bins[bin_of(v)], 1u);
      });
      __syncthreads();
      // from the top: lane i of every wave holds bins 255 - 4 i .. 252 - 4 i
      uint32_t mine[4], sum = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        mine[i] = sm_bins[kBins - 1 - 4 * lane - i];
        sum += mine[i];
      }
      uint32_t upto = sum;
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const uint32_t below = uint32_t(__builtin_amdgcn_ds_bpermute((lane - m) << 2, int(upto)));
        if (lane >= m) upto += below;
      }
      const uint64_t reached = __builtin_amdgcn_ballot_w64(upto >= uint32_t(need));
      const int at = __builtin_ctzll(reached);   // (never none: there are at least `need` candidates)
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
      // what is in the bin: its lowest and highest order
      uint32_t bin_low = 0xffffffffu, bin_high = 0;
      each([&](int u, int j) {
        const float v = scores.at(u);
        const uint32_t o = order_of(v);
        if (open(j) && o >= low && o <= high && bin_of(v) == bin) {
          bin_low = min(bin_low, o);
          bin_high = max(bin_high, o);
        }
      });
      extent(bin_low, bin_high, low, high);
      linear = false;
      if (in_bin == uint32_t(need)) {   // all of the bin
        above = low - 1;                // (an order is at least 0x007fffff, that of -inf)
        equal = 0;
        break;
      }
    }
  }

  // the list, in ascending positions
  const uint64_t before = (1ull << lane) - 1;
  if (equal > 0) {   // positions of that order, counted from the first
    each([&](int u, int j) {
      const uint64_t same = __builtin_amdgcn_ballot_w64(open(j) && order_of(scores.at(u)) == above);
      if (lane == 0) sm_count[4 * u + wave] = uint16_t(__builtin_popcountll(same));
    });
    __syncthreads();
    if (wave == 0) {
      uint32_t total = 0;
      for (int i0 = 0; i0 < 4 * rounds; i0 += 64) {
        const uint32_t own = i0 + lane < 4 * rounds ? sm_count[i0 + lane] : 0;
        uint32_t upto = own;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
          const uint32_t below = uint32_t(__builtin_amdgcn_ds_bpermute((lane - m) << 2, int(upto)));
          if (lane >= m) upto += below;
        }
        if (i0 + lane < 4 * rounds) sm_base[i0 + lane] = total + upto - own;
        total += uint32_t(__builtin_amdgcn_readlane(int(upto), 63));
      }
    }
    __syncthreads();
  }
  auto taken = [&](int u, int j) {
    const uint32_t o = order_of(scores.at(u));
    bool yes = always(j) || (open(j) && o > above && c.open > 0);
    if (equal > 0) {
      const bool same = open(j) && o == above;
      const uint64_t mask = __builtin_amdgcn_ballot_w64(same);
      yes |= same && int(sm_base[4 * u + wave]) + int(__builtin_popcountll(mask & before)) < equal;
    }
    return yes;
  };
  uint64_t chosen[PER ? PER : 1];
  each([&](int u, int j) {
    const uint64_t mask = __builtin_amdgcn_ballot_w64(taken(u, j));
    if constexpr (PER > 0) chosen[u] = mask;
    if (lane == 0) sm_count[4 * u + wave] = uint16_t(__builtin_popcountll(mask));
  });
  __syncthreads();   // (also: the first positions of the equal ones have been read where the masks are kept)
  int32_t* list = p.lists + h * p.head_stride + c.list;
  uint32_t total = 0;
  if constexpr (PER > 0) {
    if (wave == 0) {
      for (int i0 = 0; i0 < 4 * rounds; i0 += 64) {
        const uint32_t own = i0 + lane < 4 * rounds ? sm_count[i0 + lane] : 0;
        uint32_t upto = own;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
          const uint32_t below = uint32_t(__builtin_amdgcn_ds_bpermute((lane - m) << 2, int(upto)));
          if (lane >= m) upto += below;
        }
        if (i0 + lane < 4 * rounds) sm_base[i0 + lane] = total + upto - own;
        total += uint32_t(__builtin_amdgcn_readlane(int(upto), 63));
      }
    }
    __syncthreads();
    each([&](int u, int j) {
      const uint32_t at = sm_base[4 * u + wave] + uint32_t(__builtin_popcountll(chosen[u] & before));
      if (((chosen[u] >> lane) & 1) && at < uint32_t(c.count))
        list[at] = p.blk[j < c.num_root ? c.root_entry + j : c.prefix_entry + j - c.num_root];
    });
  } else {
    // (the masks are worked out again, round by round; every wave adds the counts in front of its own up)
    each([&](int u, int j) {
      const uint64_t mask = __builtin_amdgcn_ballot_w64(taken(u, j));
      uint32_t at = total;
      for (int w = 0; w < 4; ++w) {
        if (w < wave) at += sm_count[4 * u + w];
        total += sm_count[4 * u + w];
      }
      at += uint32_t(__builtin_popcountll(mask & before));
      if (((mask >> lane) & 1) && at < uint32_t(c.count))
        list[at] = p.blk[j < c.num_root ? c.root_entry + j : c.prefix_entry + j - c.num_root];
    });
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
  if (n_items > kMaxWorkgroups || g.num_kv_heads > 65535 || n_choices * g.num_kv_heads > kMaxWorkgroups) return PS_ERR_UNSUPPORTED;
  const dim3 grid(unsigned(n_items), unsigned(g.num_kv_heads));
#define PS_SCORE(D, T, COLS) hipLaunchKernelGGL((score_kernel<D, T, COLS>), grid, dim3(256), 0, st, p)
#define PS_SCORE_C(D, T)                                                                                                          \
  if (p.group == 1) PS_SCORE(D, T, 1); else if (p.group == 2) PS_SCORE(D, T, 2); else if (p.group <= 4) PS_SCORE(D, T, 4);         \
  else if (p.group <= 8) PS_SCORE(D, T, 8); else PS_SCORE(D, T, 16)
#define PS_SCORE_D(T) if (g.head_dim == 64) { PS_SCORE_C(64, T); } else if (g.head_dim == 128) { PS_SCORE_C(128, T); } else { PS_SCORE_C(256, T); }
  if (g.q_dtype == PS_F32) { PS_SCORE_D(float) } else { PS_SCORE_D(uint16_t) }
#undef PS_SCORE_D
#undef PS_SCORE_C
#undef PS_SCORE
  const dim3 rows(unsigned(n_choices * g.num_kv_heads));
#define PS_CHOOSE(PER) hipLaunchKernelGGL((choose_kernel<PER>), rows, dim3(256), 0, st, p)
  if (s.most_candidates <= 4 * 256) PS_CHOOSE(4);
  else if (s.most_candidates <= 8 * 256) PS_CHOOSE(8);
  else if (s.most_candidates <= 16 * 256) PS_CHOOSE(16);
  else if (s.most_candidates <= 32 * 256) PS_CHOOSE(32);
  else PS_CHOOSE(0);
#undef PS_CHOOSE
  return PS_OK;
}

}  // namespace psdev

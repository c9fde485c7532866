// Reading the paged pool: stored segments back into contiguous tensors, and the per-block summaries of the keys.
//
// Gather (the ingest the other way round): element (t, h, c) of a segment is code * scale of its tile (the value itself in bf16
// and float32 pools), in float32, rounded once to the destination's format.
//
// Summaries: per (block, KV head) the largest and the smallest key of every channel over the block's stored tokens, in eight
// bits each with one float32 scale: s = max |.| * (1 / 127) (1 where that is under the smallest normal number), code = round to
// nearest even of x / s.  For a query q, sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c is then (up to the eight bits) the largest
// product with q that a key of the block could have.  A key that is not a number is passed over, a channel with no other counts
// as 0, and an infinite one as the largest finite number.
//
// Both are streaming code, HBM-bound: one wavefront per piece of a (block, head[, K|V]) tile, eight elements a lane and load.
#include <algorithm>
#include <type_traits>

#include "kv_common.h"
#include "launch.h"

namespace psdev {

namespace {

// Eight consecutive elements of the pool, as they are stored and in float32.
template <int KVT>
struct Piece { u32x4 w[KVT == PS_F32 ? 2 : 1]; };
template <>
struct Piece<PS_FP8_E4M3> { u32x2 w[1]; };
template <int KVT>
__device__ __forceinline__ Piece<KVT> load_piece(const void* pool, int64_t elem) {
  Piece<KVT> r;
  if constexpr (KVT == PS_F32) {
    const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const float*>(pool) + elem);
    r.w[0] = stream_load(p);
    r.w[1] = stream_load(p + 1);
  } else if constexpr (KVT == PS_BF16) {
    r.w[0] = stream_load(reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(pool) + elem));
  } else {
    r.w[0] = stream_load(reinterpret_cast<const u32x2*>(static_cast<const uint8_t*>(pool) + elem));
  }
  return r;
}
template <int KVT>
__device__ __forceinline__ void widen_piece(const Piece<KVT>& r, float (&x)[8]) {
  if constexpr (KVT == PS_F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(r.w[j >> 2][j & 3]);
  } else if constexpr (KVT == PS_BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = bf16_bits_to_f32(r.w[0][j] & 0xffffu);
      x[2 * j + 1] = __uint_as_float(r.w[0][j] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(r.w[0][j], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(r.w[0][j], true);
      x[4 * j] = lo.x; x[4 * j + 1] = lo.y; x[4 * j + 2] = hi.x; x[4 * j + 3] = hi.y;
    }
  }
}

// ---- gather: a wave per `kLoads` x 64 pieces of a tile, `ppt` such parts a tile --------------------------------------------
// 239 thousand e4m3 tokens of eight heads of 128 to bf16: 255 us, 1468 MB at 5.8 TB/s.
template <int KVT, typename T>
__global__ __launch_bounds__(256) void gather_kernel(KvWriteParams p, T* __restrict__ dst_k, T* __restrict__ dst_v, int64_t s_tok, int64_t s_head,
                                                     int entry0, uint32_t num_tiles, uint32_t ppt) {
  constexpr int kLoads = 4;
  const int lane = threadIdx.x & 63;
  const uint64_t part = uint64_t(blockIdx.x) * 4 + uint32_t(__builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6));
  if (part >= uint64_t(num_tiles) * ppt) return;
  const uint32_t tile = ppt == 1 ? uint32_t(part) : uint32_t(part / ppt);
  // (heads inside K and V: the waves of a workgroup write neighbouring heads of the same tokens)
  const uint32_t heads = uint32_t(p.num_kv_heads);
  const int h = int(tile % heads), which = int(tile / heads % 2), e = entry0 + int(tile / (2 * heads));
  const int cpt = p.head_dim / 8;   // pieces of a token
  const int pieces = p.ent_valid[e] * cpt, c0 = int(part - uint64_t(tile) * ppt) * (64 * kLoads) + lane;
  if (c0 - lane >= pieces) return;  // behind the segment's end, or a block adopted from another layout
  const int id = p.blk[e];
  const int64_t src = int64_t(id) * p.s_block + int64_t(h) * p.s_head + int64_t(which) * p.s_kv;
  float scale = 1.f;
  if constexpr (KVT == PS_FP8_E4M3) scale = p.scales[(int64_t(id) * heads + h) * 2 + which];
  T* dst = (which ? dst_v : dst_k) + int64_t(p.ent_tok0[e]) * s_tok + int64_t(h) * s_head;
  Piece<KVT> raw[kLoads];
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int c = min(c0 + 64 * u, pieces - 1), tok = c / cpt;   // (past the end: the last piece again, not stored)
    raw[u] = load_piece<KVT>(p.kv, src + int64_t(tok) * p.s_tok + 8 * (c - tok * cpt));
  }
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const int c = c0 + 64 * u, tok = c / cpt;
    if (c >= pieces) continue;
    float x[8];
    widen_piece<KVT>(raw[u], x);
    if constexpr (KVT == PS_FP8_E4M3) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] *= scale;
    }
    T* at = dst + int64_t(tok) * s_tok + 8 * (c - tok * cpt);
    if constexpr (sizeof(T) == 4) {
      u32x4 a, b;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        a[j] = __float_as_uint(x[j]);
        b[j] = __float_as_uint(x[4 + j]);
      }
      stream_store(reinterpret_cast<u32x4*>(at), a);
      stream_store(reinterpret_cast<u32x4*>(at) + 1, b);
    } else {
      u32x4 a;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x2 b;
        b.x = (__bf16)x[2 * j];
        b.y = (__bf16)x[2 * j + 1];
        a[j] = __builtin_bit_cast(uint32_t, b);
      }
      stream_store(reinterpret_cast<u32x4*>(at), a);
    }
  }
}

// ---- summaries: a wave per (block, head), 64 / L tokens at a time, L = D / 8 lanes to a token --------------------------------
// Bound by the vector unit unless every element costs little: e4m3 codes are compared in pairs as float16, which holds them
// exactly; the comparisons are the three-operand ones (v_pk_maximum3_f16, v_maximum3_f32), which carry a NaN through and quiet
// nothing -- a wave that ends up with one goes over its tile again with those that pass over it.  One exchange of two
// registers' halves (v_permlane32_swap, v_permlane16_swap) and one maximum reduce the largest and the negated smallest together.
// What is left of the 16 values of eight channels is four a lane (eight where a token has 32 lanes), which share out the
// quantisation too.
// 249 thousand tiles of sixteen 128-wide e4m3 tokens: 166 us with float32 comparisons, exchanges by ds_bpermute of all sixteen
// values and a division for each; 144 with float16 pairs whose maxima quieted both their operands first; 121 now, 577 MB at 4.8 TB/s.
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;

template <int KVT>
struct Bounds {   // of eight channels: largest and smallest, as float32 or float16 pairs
  typedef std::conditional_t<KVT == PS_FP8_E4M3, f16x2, float> word;
  static constexpr int kWords = KVT == PS_FP8_E4M3 ? 4 : 8;
  word hi[kWords], lo[kWords];
  __device__ __forceinline__ Bounds() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      hi[i] = word(-__builtin_inff());
      lo[i] = word(__builtin_inff());
    }
  }
  static __device__ __forceinline__ void widen(const Piece<KVT>& r, word (&x)[kWords]) {
    if constexpr (KVT == PS_FP8_E4M3) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        x[2 * j] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(r.w[0][j], 1.f, false));
        x[2 * j + 1] = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(r.w[0][j], 1.f, true));
      }
    } else {
      widen_piece<KVT>(r, x);
    }
  }
  __device__ __forceinline__ void add(const Piece<KVT>& a, const Piece<KVT>& b) {   // a NaN stays
    word x[kWords], y[kWords];
    widen(a, x);
    widen(b, y);
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      hi[i] = __builtin_elementwise_maximum(__builtin_elementwise_maximum(hi[i], x[i]), y[i]);
      lo[i] = __builtin_elementwise_minimum(__builtin_elementwise_minimum(lo[i], x[i]), y[i]);
    }
  }
  __device__ __forceinline__ void add_numbers(const Piece<KVT>& a) {   // a NaN is passed over
    word x[kWords];
    widen(a, x);
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      hi[i] = __builtin_elementwise_max(hi[i], x[i]);
      lo[i] = __builtin_elementwise_min(lo[i], x[i]);
    }
  }
};

// a in one half of the lanes (or every other row of 16), b in the other, each the larger of its two
template <bool HALVES, typename W>
__device__ __forceinline__ W meet(W a, W b) {
  const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
  if constexpr (HALVES) {
    const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    return __builtin_elementwise_maximum(__builtin_bit_cast(W, uint32_t(r[0])), __builtin_bit_cast(W, uint32_t(r[1])));
  } else {
    const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    return __builtin_elementwise_maximum(__builtin_bit_cast(W, uint32_t(r[0])), __builtin_bit_cast(W, uint32_t(r[1])));
  }
}

// Lanes 0 .. 31 keep the largest, lanes 32 .. 63 the negated smallest: of a token's eight channels all (L = 32), else four, the first
// in even rows of 16 lanes.
template <int L, int KVT, int VALUES>
__device__ __forceinline__ void share_out(const Bounds<KVT>& m, float (&x)[VALUES]) {
  typedef typename Bounds<KVT>::word word;
  constexpr int kWords = Bounds<KVT>::kWords, kLeft = kWords * VALUES / 8;
  word left[kLeft];
  if constexpr (L == 32) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) left[i] = meet<true>(m.hi[i], word(-m.lo[i]));
  } else {
#pragma unroll
    for (int i = 0; i < kLeft; ++i)
      left[i] = meet<false>(meet<true>(m.hi[i], word(-m.lo[i])), meet<true>(m.hi[i + kLeft], word(-m.lo[i + kLeft])));
    if constexpr (L == 8) {
#pragma unroll
      for (int i = 0; i < kLeft; ++i)
        left[i] = __builtin_elementwise_maximum(left[i], __builtin_bit_cast(word, dpp_u32<kRor8>(0, __builtin_bit_cast(uint32_t, left[i]))));
    }
  }
#pragma unroll
  for (int i = 0; i < VALUES; ++i) {
    if constexpr (KVT == PS_FP8_E4M3) x[i] = float(left[i / 2][i & 1]);
    else x[i] = left[i];
  }
}

template <int D, int KVT>
__global__ __launch_bounds__(256) void summaries_kernel(KvWriteParams p, int8_t* __restrict__ summaries, float* __restrict__ summary_scales,
                                                        int entry0, uint32_t num_tiles) {
  constexpr int L = D / 8, kToks = 64 / L, kLoads = 4, kValues = L == 32 ? 8 : 4;
  const int lane = threadIdx.x & 63, c8 = lane & (L - 1);
  const uint32_t tile = blockIdx.x * 4u + uint32_t(__builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6));
  if (tile >= num_tiles) return;
  const int h = int(tile % uint32_t(p.num_kv_heads)), e = entry0 + int(tile / uint32_t(p.num_kv_heads));
  const int valid = p.ent_valid[e];
  if (valid <= 0) return;   // a block adopted from another layout, which has its summaries
  const int id = p.blk[e];
  const int64_t src = int64_t(id) * p.s_block + int64_t(h) * p.s_head + 8 * c8, lane_src = src + lane / L * p.s_tok;
  float kv_scale = 1.f;
  if constexpr (KVT == PS_FP8_E4M3) kv_scale = p.scales[(int64_t(id) * p.num_kv_heads + h) * 2];
  Bounds<KVT> m;
  int t0 = 0;
  for (; t0 + kLoads * kToks <= valid; t0 += kLoads * kToks) {
    Piece<KVT> raw[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) raw[u] = load_piece<KVT>(p.kv, lane_src + (t0 + u * kToks) * p.s_tok);
#pragma unroll
    for (int u = 0; u < kLoads; u += 2) m.add(raw[u], raw[u + 1]);
  }
  auto clamped = [&](int t) { return load_piece<KVT>(p.kv, src + int64_t(min(t + lane / L, valid - 1)) * p.s_tok); };   // (past the end: the last token again)
  for (; t0 < valid; t0 += 2 * kToks) m.add(clamped(t0), clamped(t0 + kToks));
  float x[kValues];
  share_out<L>(m, x);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < kValues; ++i) odd |= !(fabsf(x[i]) <= kMost);
  if (__builtin_amdgcn_ballot_w64(odd) != 0) {   // NaN or infinities among them
    Bounds<KVT> numbers;
    for (t0 = 0; t0 < valid; t0 += kToks) numbers.add_numbers(clamped(t0));
    share_out<L>(numbers, x);
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const float other = lane_xor(x[i], 32);      // (no number in a channel: -inf both ways)
      x[i] = x[i] == -__builtin_inff() && other == -__builtin_inff() ? 0.f : fminf(fmaxf(x[i], -kMost), kMost);
    }
  }
  // (a positive scale: the largest of the products is the product of the largest, rounded)
  const float sign = lane < 32 ? kv_scale : -kv_scale;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kValues; ++i) {
    x[i] *= sign;
    if constexpr (KVT == PS_FP8_E4M3) x[i] = fminf(fmaxf(x[i], -kMost), kMost);
    top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  }
  top = max(top, dpp_u32<kXor1>(0, top));
  top = max(top, dpp_u32<kXor2>(0, top));
  top = max(top, dpp_u32<kHalfMirror>(0, top));
  top = max(top, dpp_u32<kMirror>(0, top));
  top = max(top, dpp_u32<kBcast15, 0xa>(0, top));
  top = max(top, dpp_u32<kBcast31, 0xc>(0, top));
  const float scale = eight_bit_scale(__uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(top), 63))));
  uint32_t codes[kValues / 4];
  eight_bit_codes<kValues>(x, scale, codes);
  const int64_t at = int64_t(id) * p.num_kv_heads + h;
  int8_t* dst = summaries + at * (2 * D) + (lane < 32 ? 0 : D) + 8 * c8;
  if constexpr (L == 32) *reinterpret_cast<u32x2*>(dst) = u32x2{codes[0], codes[1]};
  else if (L == 16 || (lane & 8) == 0) *reinterpret_cast<uint32_t*>(dst + (lane & 16 ? 4 : 0)) = codes[0];
  if (lane == 0) summary_scales[at] = scale;
}

}  // namespace

int32_t launch_kv_gather(const ps_layout* lay, const void* dev_tables, int which, const void* kv, const float* scales, int dst_dtype,
                         void* dst_k, void* dst_v, int64_t s_tok, int64_t s_head, hipStream_t st) {
  const ps_geometry& g = lay->geo;
  int entry0 = 0;
  const int64_t entries = segment_entries(lay, which, &entry0), per_entry = int64_t(g.num_kv_heads) * 2;
  if (entries == 0) return PS_OK;
  if (g.head_dim % 8) return PS_ERR_UNSUPPORTED;
  const int64_t ppt = (int64_t(g.block_size) * (g.head_dim / 8) + 255) / 256;
  if (ppt > INT32_MAX / 256 || entries * per_entry > INT32_MAX) return PS_ERR_INVALID_ARG;
  const KvWriteParams p = make_write_params(lay, dev_tables, const_cast<void*>(kv), const_cast<float*>(scales));
  const int64_t step = entries_per_launch(entries, per_entry * ppt, 4);
  for (int64_t first = 0; first < entries; first += step) {
    const int64_t tiles = std::min(step, entries - first) * per_entry;
#define PS_GATHER(KVT, T)                                                                                                     \
  hipLaunchKernelGGL((gather_kernel<KVT, T>), dim3(unsigned((tiles * ppt + 3) / 4)), dim3(256), 0, st, p, static_cast<T*>(dst_k), \
                     static_cast<T*>(dst_v), s_tok, s_head, entry0 + int(first), uint32_t(tiles), uint32_t(ppt))
#define PS_GATHER_T(KVT) if (dst_dtype == PS_F32) PS_GATHER(KVT, float); else PS_GATHER(KVT, uint16_t)
    if (g.kv_dtype == PS_F32) { PS_GATHER_T(PS_F32); } else if (g.kv_dtype == PS_BF16) { PS_GATHER_T(PS_BF16); } else { PS_GATHER_T(PS_FP8_E4M3); }
#undef PS_GATHER_T
#undef PS_GATHER
  }
  return PS_OK;
}

int32_t launch_block_summaries(const ps_layout* lay, const void* dev_tables, int which, const void* kv, const float* scales,
                               int8_t* summaries, float* summary_scales, hipStream_t st) {
  const ps_geometry& g = lay->geo;
  int entry0 = 0;
  const int64_t entries = segment_entries(lay, which, &entry0);
  if (entries == 0) return PS_OK;
  if (entries * g.num_kv_heads > INT32_MAX) return PS_ERR_INVALID_ARG;
  const KvWriteParams p = make_write_params(lay, dev_tables, const_cast<void*>(kv), const_cast<float*>(scales));
  const int64_t step = entries_per_launch(entries, g.num_kv_heads, 4);
  for (int64_t first = 0; first < entries; first += step) {
    const int64_t tiles = std::min(step, entries - first) * g.num_kv_heads;
#define PS_SUMMARIES(D, KVT)                                                                                                  \
  hipLaunchKernelGGL((summaries_kernel<D, KVT>), dim3(unsigned((tiles + 3) / 4)), dim3(256), 0, st, p, summaries, summary_scales, \
                     entry0 + int(first), uint32_t(tiles))
#define PS_SUMMARIES_D(KVT) if (g.head_dim == 64) PS_SUMMARIES(64, KVT); else if (g.head_dim == 128) PS_SUMMARIES(128, KVT); else PS_SUMMARIES(256, KVT)
    if (g.kv_dtype == PS_F32) { PS_SUMMARIES_D(PS_F32); } else if (g.kv_dtype == PS_BF16) { PS_SUMMARIES_D(PS_BF16); } else { PS_SUMMARIES_D(PS_FP8_E4M3); }
#undef PS_SUMMARIES_D
#undef PS_SUMMARIES
  }
  return PS_OK;
}

}  // namespace psdev

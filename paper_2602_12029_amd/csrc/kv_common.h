// Pieces shared by the kernels that write and read the paged pool (kv_update.hip, rope.hip, kv_read.hip).
#pragma once
#include "device_common.h"

namespace psdev {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// Bulk K/V passes through these kernels once and is far larger than the caches: loads and stores are non-temporal,
// so the lines neither displace what the caches hold nor wait there for a reader that never comes.
template <typename V>
__device__ __forceinline__ V stream_load(const V* p) { return __builtin_nontemporal_load(p); }
template <typename V>
__device__ __forceinline__ void stream_store(V* p, V v) { __builtin_nontemporal_store(v, p); }

// e4m3fn code -> float32 (exact)
__device__ __forceinline__ float e4m3_to_f32(uint32_t code) {
  const uint32_t e = (code >> 3) & 0xf, m = code & 7;
  const float mag = e ? __uint_as_float(((e + 120u) << 23) | (m << 20)) : float(m) * 0x1p-9f;
  return (code & 0x80) ? -mag : mag;
}

// two float32 -> two e4m3fn codes in the low 16 bits (v_cvt_pk_fp8_f32: nearest even).  Inputs never reach the
// midpoint above 448 here (|x| <= tile maximum), so saturation behaviour is not relied upon.
__device__ __forceinline__ uint32_t f32x2_to_e4m3(float a, float b) {
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false)) & 0xffffu;
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) x = fmaxf(x, lane_xor(x, m));
  return x;
}

// x of another lane by a DPP control; lanes without one (and rows of 16 outside `ROWS`) get `none`
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t none, uint32_t x) {
  return uint32_t(__builtin_amdgcn_update_dpp(int(none), int(x), CTRL, ROWS, 0xf, false));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140, kRor8 = 0x128, kBcast15 = 0x142, kBcast31 = 0x143;

constexpr float kMost = 0x1.fffffep127f;   // the largest finite float32

// Eight-bit rows (block summaries, query rows that meet them): the scale of rows whose largest magnitude is `top`, and the codes,
// round to nearest even of x / scale, four to a word, of finite x of a whole wavefront.
// x / scale without a division per element: x times the instruction's reciprocal (one step off) is within 2^-15 of it (|x / scale|
// < 128), and adding 1.5 * 2^23 rounds to nearest even in place, the code in the low byte; where any of a wave's quotients lies within
// 2^-14 of half a step, the real division decides.
__device__ __forceinline__ float eight_bit_scale(float top) {
  const float scale = top * (1.f / 127.f);
  return scale >= 0x1p-126f ? scale : 1.f;
}
template <int N>
__device__ __forceinline__ void eight_bit_codes(const float (&x)[N], float scale, uint32_t (&codes)[N / 4]) {
  constexpr float kMagic = 12582912.f;
  const float rinv = __builtin_amdgcn_rcpf(scale);
  uint32_t byte[N];
  float off = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float y = __builtin_fmaf(x[j], rinv, kMagic);
    byte[j] = __float_as_uint(y);
    off = fmaxf(off, fabsf(__builtin_fmaf(x[j], rinv, kMagic - y)));
  }
  if (__builtin_amdgcn_ballot_w64(off > 0.5f - 0x1p-14f) != 0) {
#pragma unroll
    for (int j = 0; j < N; ++j) byte[j] = __float_as_uint(x[j] / scale + kMagic);
  }
#pragma unroll
  for (int j = 0; j < N; j += 4)
    codes[j / 4] = __builtin_amdgcn_perm(byte[j + 1], byte[j], 0x0c0c0400u) | __builtin_amdgcn_perm(byte[j + 3], byte[j + 2], 0x04000c0cu);
}

struct KvWriteParams {
  const int32_t* blk;        // concatenated block array
  const int32_t* ent_tok0;   // per entry: its first token in the ragged source of its kind
  const int32_t* ent_valid;  // per entry: tokens stored in the block
  const int32_t* ent_order;  // per entry position: the entry an ingest or stage-in takes there (shared kinds by physical block)
  const int32_t* dest;       // [R] block * B + slot of the token being appended, -1 = none
  void* kv;
  float* scales;
  int32_t num_kv_heads, head_dim, block_size;
  int64_t s_block, s_head, s_kv, s_tok;  // pool strides, elements
};

// Codes of x / scale, round to nearest even, for eight values a lane: exactly those of the correctly rounded float32 quotient,
// without a division per element.  With y the correctly rounded 1 / scale, q = x y is within two steps of the quotient; a
// correction q <- q - (q scale - x) y brings it within one, and by Markstein's theorem (IBM J. Res. Dev. 34, 1990: y correctly
// rounded, q within one step, the residual exact) the next one to the correctly rounded quotient.  The residual is written with
// this sign so that -0 keeps its own.  The residuals are exact where they do not underflow: from 2^-10 of the scale on, below
// which the code is 0 either way, so for any scale from 2^-90; the others, and infinities, are divided.  Quotients that were checked for the
// neighbourhood of a rounding boundary instead, and divided there, cost an ingest of 2.2 GB, often ties, 584 us, this 547.
struct E4m3Encoder {
  float scale, rinv;
  bool divide;   // uniform
  __device__ __forceinline__ explicit E4m3Encoder(float s) : scale(s), rinv(1.f / s), divide(!(s >= 0x1p-90f && s <= 0x1p120f)) {}
  __device__ __forceinline__ u32x2 operator()(const float (&x)[8]) const {
    float q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      q[j] = x[j] * rinv;
      q[j] = __builtin_fmaf(-__builtin_fmaf(q[j], scale, -x[j]), rinv, q[j]);
      q[j] = __builtin_fmaf(-__builtin_fmaf(q[j], scale, -x[j]), rinv, q[j]);
    }
    if (__builtin_expect(__builtin_amdgcn_readfirstlane(divide), 0)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = x[j] / scale;
    }
    u32x2 out;
    out[0] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), true));
    out[1] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false), true));
    return out;
  }
};

// The e4m3 tile that an appended token belongs to: its bytes, its scale, the token's slot.
struct E4m3Tile {
  uint8_t* at;
  float* scale;
  int slot;
};
__device__ __forceinline__ E4m3Tile e4m3_tile(const KvWriteParams& p, int dest, int h, int which) {
  const int id = dest / p.block_size;
  return {static_cast<uint8_t*>(p.kv) + int64_t(id) * p.s_block + int64_t(h) * p.s_head + int64_t(which) * p.s_kv,
          p.scales + (int64_t(id) * p.num_kv_heads + h) * 2 + which, dest % p.block_size};
}

// One token's row into its e4m3 tile by a wavefront, rows of 2^row_shift eight-element pieces, eight elements a lane (every token
// group of the wave holds the whole row x); old: the tile's scale.  The stored tokens of a tile whose scale has grown are
// rewritten 64 >> row_shift at a time, and four of those rounds are fetched together: a block of sixteen 128-wide tokens in one
// round trip (a byte at a time the launch was bound by the chain of those rewrites: 64 requests, eight heads, tokens of changing
// magnitude 8.5 -> 5.2 us).
__device__ __forceinline__ void append_e4m3x8_values(const KvWriteParams& p, const E4m3Tile& tile, float (&x)[8], float old, int row_shift) {
  const int lane = threadIdx.x & 63, slot = tile.slot;
  const int c = lane & ((1 << row_shift) - 1), tok0 = lane >> row_shift, toks = 64 >> row_shift;
  float amax = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) amax = fmaxf(amax, fmaxf(fabsf(x[2 * j]), fabsf(x[2 * j + 1])));
  amax = wave_max(amax);
  const float cand = amax / 448.f;
  float scale;
  auto encode = [](const float (&y)[8]) {
    u32x2 out;
    out[0] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true));
    out[1] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false), true));
    return out;
  };
  if (slot == 0) {
    scale = amax > 0.f ? cand : 1.f;
  } else {
    scale = fmaxf(old, cand);
    if (scale != old) {   // the tile's scale grew: re-encode what is stored, from the stored values
      for (int t0 = tok0; t0 < slot; t0 += 4 * toks) {
        u32x2 code[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (t0 + u * toks < slot) code[u] = *reinterpret_cast<const u32x2*>(tile.at + int64_t(t0 + u * toks) * p.s_tok + 8 * c);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (t0 + u * toks < slot) {
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = (e4m3_to_f32((code[u][j >> 2] >> (8 * (j & 3))) & 0xffu) * old) / scale;
            *reinterpret_cast<u32x2*>(tile.at + int64_t(t0 + u * toks) * p.s_tok + 8 * c) = encode(y);
          }
      }
    }
  }
  if (lane == 0) *tile.scale = scale;
  if (tok0 == 0) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = x[j] / scale;
    *reinterpret_cast<u32x2*>(tile.at + int64_t(slot) * p.s_tok + 8 * c) = encode(x);
  }
}

inline KvWriteParams make_write_params(const ps_layout* lay, const void* dev_tables, void* kv, float* scales) {
  const int32_t* t = static_cast<const int32_t*>(dev_tables);
  const ps_geometry& g = lay->geo;
  KvWriteParams p{};
  p.blk = t + lay->off_blk;
  p.ent_tok0 = t + lay->off_ent_tok0;
  p.ent_valid = t + lay->off_ent_valid;
  p.ent_order = t + lay->off_ent_order;
  p.dest = t + lay->off_dest;
  p.kv = kv;
  p.scales = scales;
  p.num_kv_heads = g.num_kv_heads;
  p.head_dim = g.head_dim;
  p.block_size = g.block_size;
  p.s_block = g.kv_stride_block;
  p.s_head = g.kv_stride_head;
  p.s_kv = g.kv_stride_kv;
  p.s_tok = g.kv_stride_tok;
  return p;
}

// Entries of the concatenated block array (prefixes, suffixes, roots) that a kind of segment has, and the first of them.
inline int64_t segment_entries(const ps_layout* lay, int which, int* entry0) {
  const int n_prefix = int(lay->prefix_blk.size()), n_suffix = int(lay->suffix_blk.size());
  *entry0 = which == 0 ? 0 : (which == 1 ? n_prefix : n_prefix + n_suffix);
  return which == 0 ? n_prefix : (which == 1 ? n_suffix : int64_t(lay->root_blk.size()));
}

}  // namespace psdev

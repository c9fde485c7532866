// Norm of queries and keys per head and rotation by position, on the way to the attention and into the paged cache.
//
// A row is one head of one token, x[d].  y = x * rsqrt(mean x^2 + eps) * w (y = x without weights), then the first `rot`
// elements turn pair by pair: (a, b) -> (a cos - b sin, a sin + b cos) by the angle position * radians[i] of pair i, whose
// elements are (i, i + rot/2) or (2i, 2i+1).  All of it in float32, rounded once: to the queries' format, to the pool's, or to
// e4m3 with the tile's scale.
//
// Angles.  position * radians in float32 is off by 2^-24 of the whole angle, 0.01 rad at position 200000.  The rates are
// therefore kept as 64-bit fixed-point fractions of a turn: position * rate modulo 2^64 is the angle modulo a turn, exact to
// 2^-64 turns a position, and its top 32 bits give a quarter and a remainder within an eighth of a turn, for which the Taylor
// series of sine and cosine to x^9 and x^10 are exact to float32 (next terms 2e-9 and 5e-10).  No table in memory, no library call.
//
// Every wave of the row kernels works the angles of its token out once, a pair a lane, and hands them over through LDS; the ingest
// does so once per workgroup for all heads of a block's tokens.
#include <algorithm>
#include <type_traits>

#include "kv_common.h"
#include "launch.h"

namespace psdev {

namespace {

// sine and cosine of `turn` / 2^32 turns
__device__ __forceinline__ void turn_sincos(uint32_t turn, float& s, float& c) {
  const uint32_t quarter = (turn + 0x20000000u) >> 30;
  const float x = float(int32_t(turn - (quarter << 30))) * 1.46291807926715968e-9f;   // 2 pi / 2^32; |x| <= pi / 4
  const float z = x * x;
  const float sp = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f);
  const float cp = __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f);
  const float sn = __builtin_fmaf(x * z, sp, x), cs = __builtin_fmaf(z, cp, 1.f);
  s = (quarter & 1) ? cs : sn;
  c = (quarter & 1) ? sn : cs;
  if (quarter & 2) s = -s;
  if ((quarter + 1) & 2) c = -c;
}

__device__ __forceinline__ uint32_t turn_of(int position, uint64_t rate) { return uint32_t((uint64_t(int64_t(position)) * rate) >> 32); }

// Sum over groups of L lanes; every lane of a group receives the same bits.
template <int L>
__device__ __forceinline__ float group_sum(float x) {
  static_assert(L == 8 || L == 16 || L == 32, "");
  if constexpr (L == 8) {
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xB1, 0xf, 0xf, true));   // quad_perm [1,0,3,2]
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4E, 0xf, 0xf, true));   // quad_perm [2,3,0,1]
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true));  // row_half_mirror
    return x;
  } else {
    x = row16_allreduce_sum(x);
    if constexpr (L == 32) x += lane_xor(x, 16);
    return x;
  }
}

// Eight consecutive elements of a row as they are stored.
template <typename T>
struct Raw8 { u32x4 w[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < int(sizeof(T)) / 2; ++i) r.w[i] = reinterpret_cast<const u32x4*>(p)[i];
  return r;
}
template <typename T>
__device__ __forceinline__ Raw8<T> stream_load8(const T* p) {
  Raw8<T> r;
#pragma unroll
  for (int i = 0; i < int(sizeof(T)) / 2; ++i) r.w[i] = stream_load(reinterpret_cast<const u32x4*>(p) + i);
  return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(r.w[j >> 2][j & 3]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = bf16_bits_to_f32(r.w[0][j] & 0xffffu);
      x[2 * j + 1] = bf16_bits_to_f32(r.w[0][j] >> 16);
    }
  }
}
// ... rounded to nearest even
template <typename T>
__device__ __forceinline__ Raw8<T> narrow8(const float (&x)[8]) {
  Raw8<T> r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (sizeof(T) == 4) {
      r.w[0][j] = __float_as_uint(x[j]);
      r.w[1][j] = __float_as_uint(x[4 + j]);
    } else {
      bf16x2 b;
      b.x = (__bf16)x[2 * j];
      b.y = (__bf16)x[2 * j + 1];
      r.w[0][j] = __builtin_bit_cast(uint32_t, b);
    }
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < int(sizeof(T)) / 2; ++i) reinterpret_cast<u32x4*>(p)[i] = r.w[i];
}
template <typename T>
__device__ __forceinline__ void stream_store8(T* p, const Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < int(sizeof(T)) / 2; ++i) stream_store(reinterpret_cast<u32x4*>(p) + i, r.w[i]);
}

// x * rsqrt(mean x^2 + eps) * w over a row of L lanes, eight elements each (v_rsq_f32: one float32 step, as the sum's own rounding)
template <int L>
__device__ __forceinline__ void norm8(float (&x)[8], const float (&w)[8], float eps) {
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(x[j], x[j], sum);
  const float mean = group_sum<L>(sum) * (1.f / (8 * L)) + eps;
  float inv = __builtin_amdgcn_rsqf(mean);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(mean < 0x1p-126f) != 0, 0))   // (the instruction takes those for 0; without an eps rows of 1e-19 have them)
    inv = mean < 0x1p-126f ? __builtin_amdgcn_rsqf(mean * 0x1p48f) * 0x1p24f : inv;
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] = (x[j] * inv) * w[j];
}

// The rotation of a row's elements 8 c8 .. 8 c8 + 7 (L lanes to a row), its pairs' cosines and sines in LDS, on a 16-byte boundary
// where pairs are halves.  All lanes of the wave come here.
template <int L>
__device__ __forceinline__ void rotate8(float (&x)[8], int c8, const float* cosines, const float* sines, int rot, bool neighbours) {
  const int c = 8 * c8, half = rot >> 1;
  if (neighbours) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + 2 * j < rot) {
        const float a = x[2 * j], b = x[2 * j + 1], co = cosines[(c >> 1) + j], si = sines[(c >> 1) + j];
        x[2 * j] = __builtin_fmaf(a, co, -(b * si));
        x[2 * j + 1] = __builtin_fmaf(a, si, b * co);
      }
    return;
  }
  // (half a multiple of 8: the partners of a lane's elements are all in one other lane of the row)
  const bool second = c >= half;
  float other[8];
  if (L == 16 && rot == 8 * L) {   // whole rows of 16 lanes: a rotation by 8 of them
#pragma unroll
    for (int j = 0; j < 8; ++j) other[j] = __uint_as_float(dpp_u32<kRor8>(0, __float_as_uint(x[j])));
  } else {
    const int lane = threadIdx.x & 63, from = c >= rot ? lane : second ? lane - (half >> 3) : lane + (half >> 3);
#pragma unroll
    for (int j = 0; j < 8; ++j) other[j] = __int_as_float(__builtin_amdgcn_ds_bpermute(from << 2, __float_as_int(x[j])));
  }
  if (c < rot) {
    const int i = second ? c - half : c;
    const uint32_t sign = second ? 0u : 0x80000000u;
#pragma unroll
    for (int j = 0; j < 8; j += 4) {
      const f32x4 co = *reinterpret_cast<const f32x4*>(cosines + i + j), si = *reinterpret_cast<const f32x4*>(sines + i + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float turned = __uint_as_float(__float_as_uint(si[e]) ^ sign);
        x[j + e] = __builtin_fmaf(x[j + e], co[e], other[j + e] * turned);
      }
    }
  }
}

// A wave's token: cosines and sines of its pairs into LDS, a pair a lane.
template <int D>
__device__ __forceinline__ void wave_angles(const RopeArgs& a, int position, float* cosines, float* sines) {
#pragma unroll
  for (int i0 = 0; i0 < D / 2; i0 += 64) {
    const int i = i0 + (int(threadIdx.x) & 63);
    if (i < (a.rot >> 1)) turn_sincos(turn_of(position, a.turns[i]), sines[i], cosines[i]);
  }
  wave_lds_order();
}

template <typename T>
__device__ __forceinline__ void load_weight(const void* weight, int c8, float (&w)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = 1.f;
  if (weight) widen8(load8(static_cast<const T*>(weight) + 8 * c8), w);
}

// ---- rows (queries of any number of tokens): one wave per (token, UNITS x 512 elements of its heads) ---------------------
// HBM-bound: 4576 tokens of 64 heads of 128 in bf16, 150 MB read and written, 30 us, 5.0 TB/s.
template <int D, typename T, int UNITS>
__global__ __launch_bounds__(256) void rope_rows_kernel(RopeArgs a, const T* __restrict__ src, int64_t s_row, int64_t s_head,
                                                        T* __restrict__ out, int64_t row0, int64_t num_waves, int heads, int groups) {
  constexpr int L = D / 8, kHeads = 64 / L;   // lanes of a head row, head rows a wave holds at a time
  __shared__ __attribute__((aligned(16))) float sm[4][2][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), c8 = lane & (L - 1);
  const int64_t id = int64_t(blockIdx.x) * 4 + wave;
  if (id >= num_waves) return;
  const int64_t t = row0 + id / groups;
  const int h0 = int(id % groups) * (kHeads * UNITS) + lane / L;
  Raw8<T> raw[UNITS];
#pragma unroll
  for (int u = 0; u < UNITS; ++u) raw[u] = load8(src + t * s_row + int64_t(min(h0 + u * kHeads, heads - 1)) * s_head + 8 * c8);
  float w[8];
  load_weight<T>(a.q_weight, c8, w);
  wave_angles<D>(a, a.positions[t], sm[wave][0], sm[wave][1]);
#pragma unroll
  for (int u = 0; u < UNITS; ++u) {
    float x[8];
    widen8(raw[u], x);
    if (a.q_weight) norm8<L>(x, w, a.eps);
    rotate8<L>(x, c8, sm[wave][0], sm[wave][1], a.rot, a.neighbours);
    const int h = h0 + u * kHeads;
    if (h < heads) store8(out + (t * heads + h) * D + 8 * c8, narrow8<T>(x));
  }
}

// ---- append: the step's token of a request, 64 lanes to eight-element pieces of its q, k and v rows ------------------------
// Bound by latency (position and rates, then the row, then the tile's scale): a wave per 512 elements of the token, or per
// (head, K|V) of an e4m3 pool, whose tile may have to be re-encoded.  Four tokens of 32 + 8 heads in bf16 3.0 us, 240 of 64 + 8 into e4m3
// tiles 5.8.
template <int D, int KVT, typename QT>
__global__ __launch_bounds__(256) void append_rope_kernel(RopeArgs a, KvWriteParams p, const QT* __restrict__ q, const void* __restrict__ new_k,
                                                          const void* __restrict__ new_v, int64_t s_row_q, int64_t s_head_q,
                                                          int64_t s_row_kv, int64_t s_head_kv, QT* __restrict__ q_out, int num_q_heads) {
  typedef std::conditional_t<KVT == PS_F32, float, uint16_t> T;
  constexpr int L = D / 8, kHeads = 64 / L;
  __shared__ __attribute__((aligned(16))) float sm[4][2][D / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), c8 = lane & (L - 1);
  const int r = blockIdx.x;
  const int nq = q ? (num_q_heads + kHeads - 1) / kHeads : 0;
  const int unit = int(blockIdx.y) * 4 + wave;
  if (unit < nq) {
    const int h = unit * kHeads + lane / L;
    const Raw8<QT> raw = load8(q + int64_t(r) * s_row_q + int64_t(min(h, num_q_heads - 1)) * s_head_q + 8 * c8);
    float w[8], x[8];
    load_weight<QT>(a.q_weight, c8, w);
    wave_angles<D>(a, a.positions[r], sm[wave][0], sm[wave][1]);
    widen8(raw, x);
    if (a.q_weight) norm8<L>(x, w, a.eps);
    rotate8<L>(x, c8, sm[wave][0], sm[wave][1], a.rot, a.neighbours);
    if (h < num_q_heads) store8(q_out + (int64_t(r) * num_q_heads + h) * D + 8 * c8, narrow8<QT>(x));
    return;
  }
  const int dest = p.dest[r];
  if (dest < 0) return;
  const int kv = unit - nq;
  if constexpr (KVT == PS_FP8_E4M3) {
    const int h = kv >> 1, which = kv & 1;
    if (h >= p.num_kv_heads) return;
    const T* src = static_cast<const T*>(which ? new_v : new_k) + int64_t(r) * s_row_kv + int64_t(h) * s_head_kv;
    const Raw8<T> raw = load8(src + 8 * c8);   // (every group of L lanes holds the whole row)
    const E4m3Tile tile = e4m3_tile(p, dest, h, which);
    const float old = *tile.scale;             // (of a fresh block: anything, and not used)
    float x[8];
    widen8(raw, x);
    if (which == 0) {
      float w[8];
      load_weight<T>(a.k_weight, c8, w);
      wave_angles<D>(a, a.positions[r], sm[wave][0], sm[wave][1]);
      if (a.k_weight) norm8<L>(x, w, a.eps);
      rotate8<L>(x, c8, sm[wave][0], sm[wave][1], a.rot, a.neighbours);
    }
    append_e4m3x8_values(p, tile, x, old, __builtin_ctz(L));
  } else {
    const int per = (p.num_kv_heads + kHeads - 1) / kHeads;
    const int which = kv >= per;
    const int h = (which ? kv - per : kv) * kHeads + lane / L;
    if (kv >= 2 * per) return;
    const T* src = static_cast<const T*>(which ? new_v : new_k) + int64_t(r) * s_row_kv + int64_t(min(h, p.num_kv_heads - 1)) * s_head_kv;
    Raw8<T> raw = load8(src + 8 * c8);
    if (which == 0) {
      float w[8], x[8];
      load_weight<T>(a.k_weight, c8, w);
      wave_angles<D>(a, a.positions[r], sm[wave][0], sm[wave][1]);
      widen8(raw, x);
      if (a.k_weight) norm8<L>(x, w, a.eps);
      rotate8<L>(x, c8, sm[wave][0], sm[wave][1], a.rot, a.neighbours);
      raw = narrow8<T>(x);
    }
    T* dst = static_cast<T*>(p.kv) + int64_t(dest / p.block_size) * p.s_block + int64_t(h) * p.s_head + int64_t(which) * p.s_kv +
             int64_t(dest % p.block_size) * p.s_tok;
    if (h < p.num_kv_heads) store8(dst + 8 * c8, raw);
  }
}

// ---- ingest: whole segments ------------------------------------------------------------------------------------------------
// A workgroup takes a pass of a block's tokens (PASS of them; all of an e4m3 block, whose tiles have a scale each) and works
// through its (head, K|V) tiles, WPT of its WAVES waves to a tile, CH eight-element pieces a lane.  HBM-bound.  The angles of the pass's
// tokens lie in LDS for all heads.  47 thousand tokens of eight heads of 128 in bf16 73 us (387 MB, 5.3 TB/s), 278 thousand into e4m3 tiles
// 315 (1713 MB, 5.4 TB/s; 440 at the two workgroups a compute unit that the registers gave without a bound, and with quotients
// that were checked and divided where in doubt).
template <int D, int KVT, int CH, int WPT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, CH <= 4 && KVT == PS_FP8_E4M3 ? 4 : 2) void ingest_rope_kernel(RopeArgs a, KvWriteParams p, const void* __restrict__ src_k, const void* __restrict__ src_v,
                                                          int64_t s_tok, int64_t s_head, int entry0, int passes, int tiles_per_team) {
  typedef std::conditional_t<KVT == PS_F32, float, uint16_t> T;
  constexpr int L = D / 8, kTeams = WAVES / WPT, kPass = CH * WPT * 64 / L;   // tokens the teams hold of a tile
  extern __shared__ __attribute__((aligned(16))) float angles[];                                      // [kPass][2][rot / 2]: cosines, sines
  __shared__ float sm_max[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6), c8 = lane & (L - 1);
  const int e = p.ent_order[entry0 + int(blockIdx.x) / passes];
  const int first = int(blockIdx.x) % passes * kPass;
  const int count = min(p.ent_valid[e] - first, kPass);   // tokens of this pass
  if (count <= 0) return;                                 // behind the segment's end, or a block adopted from another layout
  const int id = p.blk[e], tok0 = p.ent_tok0[e] + first, half = a.rot >> 1;
  const int team = wave / WPT, lane_tok = (wave % WPT) * (64 / L) + lane / L;   // token of the lane's first piece
  constexpr int kStep = WPT * 64 / L;
  const int num_tiles = 2 * p.num_kv_heads;
  auto fetch = [&](int tile, Raw8<T> (&raw)[CH]) {        // K tiles first, then V
    const int which = tile >= p.num_kv_heads, h = which ? tile - p.num_kv_heads : tile;
    const T* src = static_cast<const T*>(which ? src_v : src_k) + int64_t(tok0) * s_tok + int64_t(h) * s_head + 8 * c8;
#pragma unroll
    for (int i = 0; i < CH; ++i) raw[i] = stream_load8(src + int64_t(min(lane_tok + i * kStep, count - 1)) * s_tok);
  };
  int tile = int(blockIdx.y) * tiles_per_team * kTeams + team;
  const int tile_end = min(num_tiles, (int(blockIdx.y) + 1) * tiles_per_team * kTeams);
  Raw8<T> raw[CH];
  fetch(min(tile, num_tiles - 1), raw);
  if (int(blockIdx.y) * tiles_per_team * kTeams < p.num_kv_heads) {   // (V tiles alone need no angles)
    // a pair a lane, a token a wave
    for (int pair = lane; pair < half; pair += 64) {
      const uint64_t rate = a.turns[pair];
      for (int t = wave; t < count; t += WAVES) turn_sincos(turn_of(a.positions[tok0 + t], rate), angles[(2 * t + 1) * half + pair], angles[2 * t * half + pair]);
    }
    __syncthreads();
  }
  float w[8];
  load_weight<T>(a.k_weight, c8, w);
  // (a team without a tile of its own still meets the others of a WPT = 4 tile: there all waves are one team)
  for (; tile < tile_end; tile += kTeams) {
    const int which = tile >= p.num_kv_heads, h = which ? tile - p.num_kv_heads : tile;
    const int64_t at = int64_t(id) * p.s_block + int64_t(h) * p.s_head + int64_t(which) * p.s_kv + int64_t(first) * p.s_tok + 8 * c8;
    auto turned = [&](float (&x)[8], int i) {
      const int t = min(lane_tok + i * kStep, count - 1);
      if (a.k_weight) norm8<L>(x, w, a.eps);
      rotate8<L>(x, c8, angles + 2 * t * half, angles + (2 * t + 1) * half, a.rot, a.neighbours);
    };
    if constexpr (KVT == PS_FP8_E4M3) {
      float x[CH][8], amax = 0.f;
#pragma unroll
      for (int i = 0; i < CH; ++i) widen8(raw[i], x[i]);
      if (tile + kTeams < tile_end) fetch(tile + kTeams, raw);
      if (which == 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) turned(x[i], i);
      }
#pragma unroll
      for (int i = 0; i < CH; ++i)
        if (lane_tok + i * kStep < count) {
#pragma unroll
          for (int j = 0; j < 8; ++j) amax = fmaxf(amax, fabsf(x[i][j]));
        }
      amax = wave_max(amax);
      if constexpr (WPT > 1) {
        __syncthreads();                       // (the last tile's maxima have been read)
        if (lane == 0) sm_max[wave] = amax;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) amax = fmaxf(amax, sm_max[i]);
      }
      const float scale = amax > 0.f ? amax / 448.f : 1.f;
      if (lane == 0 && wave % WPT == 0) p.scales[(int64_t(id) * p.num_kv_heads + h) * 2 + which] = scale;
      const E4m3Encoder encode(scale);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int t = lane_tok + i * kStep;
        const u32x2 codes = encode(x[i]);
        if (t < count) stream_store(reinterpret_cast<u32x2*>(static_cast<uint8_t*>(p.kv) + at + int64_t(t) * p.s_tok), codes);
      }
    } else {
      float x[CH][8];
#pragma unroll
      for (int i = 0; i < CH; ++i) widen8(raw[i], x[i]);
      if (tile + kTeams < tile_end) fetch(tile + kTeams, raw);
      if (which == 0) {
#pragma unroll
        for (int i = 0; i < CH; ++i) turned(x[i], i);
      }
#pragma unroll
      for (int i = 0; i < CH; ++i) {
        const int t = lane_tok + i * kStep;
        if (t < count) stream_store8(static_cast<T*>(p.kv) + at + int64_t(t) * p.s_tok, narrow8<T>(x[i]));
      }
    }
  }
}

}  // namespace

int32_t launch_rope_rows(const RopeArgs& a, const ps_geometry& g, const void* src, int64_t s_row, int64_t s_head, int64_t num_rows,
                         void* out, hipStream_t st) {
  const int heads = g.num_q_heads, per = 512 / g.head_dim;   // head rows a wave holds at a time
  const int units = heads > 2 * per ? 4 : heads > per ? 2 : 1;
  const int groups = (heads + per * units - 1) / (per * units);
  const int64_t step = std::max<int64_t>(1, kMaxWorkgroups * 4 / groups);
  for (int64_t row0 = 0; row0 < num_rows; row0 += step) {
    const int64_t waves = std::min(step, num_rows - row0) * groups;
#define PS_ROWS(D, T, N)                                                                                                     \
  hipLaunchKernelGGL((rope_rows_kernel<D, T, N>), dim3(unsigned((waves + 3) / 4)), dim3(256), 0, st, a, static_cast<const T*>(src), \
                     s_row, s_head, static_cast<T*>(out), row0, waves, heads, groups)
#define PS_ROWS_N(D, T) if (units == 4) PS_ROWS(D, T, 4); else if (units == 2) PS_ROWS(D, T, 2); else PS_ROWS(D, T, 1)
#define PS_ROWS_D(T) if (g.head_dim == 64) { PS_ROWS_N(64, T); } else if (g.head_dim == 128) { PS_ROWS_N(128, T); } else { PS_ROWS_N(256, T); }
    if (g.q_dtype == PS_F32) { PS_ROWS_D(float) } else { PS_ROWS_D(uint16_t) }
#undef PS_ROWS_D
#undef PS_ROWS_N
#undef PS_ROWS
  }
  return PS_OK;
}

int32_t launch_append_rope(const ps_layout* lay, const void* dev_tables, const RopeArgs& a, const ps_token_rows& rows, void* q_out,
                           void* kv, float* scales, hipStream_t st) {
  const ps_geometry& g = lay->geo;
  const KvWriteParams p = make_write_params(lay, dev_tables, kv, scales);
  const int64_t per = 512 / g.head_dim;
  const int64_t kv_units = g.kv_dtype == PS_FP8_E4M3 ? 2 * int64_t(g.num_kv_heads) : 2 * ((g.num_kv_heads + per - 1) / per);
  const int64_t units = (rows.q ? (g.num_q_heads + per - 1) / per : 0) + kv_units;
  const int64_t wgs = (units + 3) / 4;
  if (wgs > 65535 || int64_t(lay->num_requests) > kMaxWorkgroups) return PS_ERR_UNSUPPORTED;
  const dim3 grid(unsigned(lay->num_requests), unsigned(wgs));
#define PS_APPEND(D, KVT, QT)                                                                                                \
  hipLaunchKernelGGL((append_rope_kernel<D, KVT, QT>), grid, dim3(256), 0, st, a, p, static_cast<const QT*>(rows.q), rows.k, rows.v, \
                     rows.q_stride_row, rows.q_stride_head, rows.kv_stride_row, rows.kv_stride_head, static_cast<QT*>(q_out), g.num_q_heads)
#define PS_APPEND_Q(D, KVT) if (g.q_dtype == PS_F32) PS_APPEND(D, KVT, float); else PS_APPEND(D, KVT, uint16_t)
#define PS_APPEND_D(KVT) if (g.head_dim == 64) { PS_APPEND_Q(64, KVT); } else if (g.head_dim == 128) { PS_APPEND_Q(128, KVT); } else { PS_APPEND_Q(256, KVT); }
  if (g.kv_dtype == PS_F32) { PS_APPEND_D(PS_F32) } else if (g.kv_dtype == PS_BF16) { PS_APPEND_D(PS_BF16) } else { PS_APPEND_D(PS_FP8_E4M3) }
#undef PS_APPEND_D
#undef PS_APPEND_Q
#undef PS_APPEND
  return PS_OK;
}

int32_t launch_ingest_rope(const ps_layout* lay, const void* dev_tables, int which, const RopeArgs& a, const void* src_k,
                           const void* src_v, int64_t s_tok, int64_t s_head, void* kv, float* scales, hipStream_t st) {
  const ps_geometry& g = lay->geo;
  int entry0 = 0;
  const int64_t entries = segment_entries(lay, which, &entry0);
  if (entries == 0) return PS_OK;
  const KvWriteParams p = make_write_params(lay, dev_tables, kv, scales);
  const bool e4m3 = g.kv_dtype == PS_FP8_E4M3;
  const int64_t pieces = int64_t(g.block_size) * g.head_dim / 8;   // of a tile, eight elements each
  // (e4m3: 2, 4 or 8 a lane of one wave, 8 a lane of four; else up to 4 a lane and as many passes as a block has.  Blocks of sixteen 64-wide
  // tokens, 150 thousand of them, with four a lane / two: bf16 one head 36.2 / 23.8 us, two 60.6 / 38.7, eight 127 / 107; e4m3 eight 139 / 97.  128-wide ones, 50 thousand, as two passes: one head bf16 17.6 / 14.4, float32 25.8 / 23.5, eight
  // heads 74.8 / 73.4 and 167.7 / 167.7, twice as many 140.0 / 140.8 and 325.7 / 329.8.)
  if (e4m3 && pieces > 2048) return PS_ERR_UNSUPPORTED;
  const int wpt = e4m3 && pieces > 512 ? 4 : 1, ch = e4m3 && pieces > 256 ? 8 : pieces > 128 && (e4m3 || g.num_kv_heads > 1) ? 4 : 2;
  const int pass_tokens = ch * wpt * 512 / g.head_dim;
  const int64_t passes = (g.block_size + pass_tokens - 1) / pass_tokens;
  const size_t lds = size_t(pass_tokens) * size_t(a.rot) * sizeof(float);
  const int waves = g.num_kv_heads == 1 && wpt == 1 ? 2 : 4;   // (one head has two tiles: 150 thousand float32 tokens 86.6 us with four waves, 65.6 with two)
  const int teams = waves / wpt, all = (2 * g.num_kv_heads + teams - 1) / teams;   // tiles a team would have alone
  // All tiles of a block in one workgroup, so that its angles are worked out once, where that gives four workgroups a compute
  // unit; a smaller batch has a block's tiles shared out over as many workgroups as that takes (rounded up from a quarter on).  Eight
  // heads, blocks of sixteen 128-wide tokens, one workgroup a block / two / four: 250 blocks bf16 12.6 / 11.3 / 9.0 us, e4m3 13.3 / 10.8 / 8.7;
  // 500 17.0 / 15.4 / 18.3, 17.4 / 13.8 / 16.0; 800 27.5 / 24.4 / 27.6, 22.1 / 20.1 / 22.3; 1000 30.0 / 29.3 / 33.4, 23.6 / 25.4 / 26.7; 3000 72.2 / 82.5 /
  // 90.8, 61.3 / 67.2 / 71.3.
  const int64_t wgs = entries * passes, most = 4 * kPsDefaultNumCus;
  const int parts = int(std::min<int64_t>(all, std::max<int64_t>(1, (most + wgs * 3 / 4) / wgs))), per_team = (all + parts - 1) / parts;
  const int64_t slices = (all + per_team - 1) / per_team;
  if (slices > 65535 || passes > INT32_MAX) return PS_ERR_UNSUPPORTED;
  const int64_t step = std::max<int64_t>(1, kMaxWorkgroups / passes);
  if (step * passes > INT32_MAX) return PS_ERR_UNSUPPORTED;
  for (int64_t first = 0; first < entries; first += step) {
    const dim3 grid(unsigned(std::min(step, entries - first) * passes), unsigned(slices));
#define PS_INGEST(D, KVT, CH, WPT, WAVES)                                                                                    \
  hipLaunchKernelGGL((ingest_rope_kernel<D, KVT, CH, WPT, WAVES>), grid, dim3(64 * WAVES), lds, st, a, p, src_k, src_v, s_tok, s_head, \
                     entry0 + int(first), int(passes), per_team)
#define PS_INGEST_W(D, KVT, CH) if (waves == 2) PS_INGEST(D, KVT, CH, 1, 2); else PS_INGEST(D, KVT, CH, 1, 4)
#define PS_INGEST_C(D, KVT) if (ch == 2) { PS_INGEST_W(D, KVT, 2); } else { PS_INGEST_W(D, KVT, 4); }
#define PS_INGEST_E(D) if (wpt == 4) PS_INGEST(D, PS_FP8_E4M3, 8, 4, 4); else if (ch == 8) { PS_INGEST_W(D, PS_FP8_E4M3, 8); } else { PS_INGEST_C(D, PS_FP8_E4M3) }
#define PS_INGEST_T(D) if (e4m3) { PS_INGEST_E(D) } else if (g.kv_dtype == PS_F32) { PS_INGEST_C(D, PS_F32) } else { PS_INGEST_C(D, PS_BF16) }
    if (g.head_dim == 64) { PS_INGEST_T(64); } else if (g.head_dim == 128) { PS_INGEST_T(128); } else { PS_INGEST_T(256); }
#undef PS_INGEST_T
#undef PS_INGEST_E
#undef PS_INGEST_C
#undef PS_INGEST_W
#undef PS_INGEST
  }
  return PS_OK;
}

}  // namespace psdev

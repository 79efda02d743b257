// Norm and rotation of queries and keys with the cache write, for gfx950.
//
// For every row (token) and head vector x of q and k: y = x w / sqrt(mean(x^2)
// + eps) (or y = x), the pairs of y's first rotary_dim dimensions turned by
// the row's angles, y' written to q_out or encoded into the row's cache slot;
// v is encoded into its slot as it is.  The cache's K tile is token-major, its
// V tile dims-major (one dimension's 16 tokens are contiguous).
//
// What bounds it: memory.  Every value is read once and written once: sixteen
// lanes hold one head vector, eight dimensions (16 bytes) each, so a wave
// loads and stores four heads in whole 256-byte rows.  The sum of squares
// crosses the sixteen lanes in the vector ALU; a pair (d, d + rotary_dim / 2)
// lies in two lanes, which exchange their raw bf16 (four words, not eight).
// A group of lanes takes several heads of one row, so that the row's cosines
// and sines are loaded once for them.
//
// V has to be turned from rows into columns.  Rows whose slots follow each
// other within a block form a run; one wave takes a run's rows of one head
// through LDS and writes each dimension's tokens together: whole 16-byte
// pieces where the run fills them (prompts), single values otherwise.
//
// With block scales (qk_norm_rope_append_scaled) K and V of a run are both a
// wave's: it has the run's values of one head in registers, takes the largest
// magnitude over its lanes, and with it the exponent of the block's scale.
// Earlier tokens of the block are encoded anew where the scale rises: a power of
// two apart, so that their values stay but where they fall below e4m3's normal
// range.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "common.h"

namespace dpool_rope {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kD = 128;
constexpr int kBS = 16;
constexpr int kWaves = 4;
constexpr float kE4M3Max = 448.0f;

struct RopeArgs {
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  const float* cos_sin;
  const int32_t* positions;
  const int64_t* slots;
  uint16_t* q_out;
  char* kc;
  char* vc;
  const float* k_scale;
  const float* v_scale;
  int64_t rows, n_positions, n_slots;  // n_slots: 16 * num_blocks
  int64_t q_stride, k_stride, v_stride;
  int64_t qk_groups;  // workgroups that take q and k; the others take v
  float eps;
  int32_t hq, hkv, rotary;
  uint8_t* k_exp;  // [num_blocks, Hkv] exponent bytes (block scales)
  uint8_t* v_exp;
};

__device__ __forceinline__ float lo_f32(int w) { return __uint_as_float((uint32_t)w << 16); }
__device__ __forceinline__ float hi_f32(int w) { return __uint_as_float((uint32_t)w & 0xffff0000u); }

__device__ __forceinline__ int pack_bf16(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(int, p);
}

// Four values to e4m3 codes: clamped (the conversion does not saturate), to nearest even.
// A NaN stays one, which fmin and fmax would make a number: the norm of a head with an
// infinity is NaN, and a -448 in its place would pass for a key.
__device__ __forceinline__ int pack_e4m3(float a, float b, float c, float d) {
  const auto cut = [](float x) { return x != x ? x : fminf(fmaxf(x, -kE4M3Max), kE4M3Max); };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(cut(a), cut(b), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(cut(c), cut(d), r, true);
}

// Sum over the sixteen lanes of a row of lanes, in every lane: rotations by 8, 4, 2 and 1
__device__ __forceinline__ float row_sum(float x) {
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x124, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x122, 0xf, 0xf, false));
  x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x121, 0xf, 0xf, false));
  return x;
}

__device__ __forceinline__ void unpack8(const i32x4& x, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = lo_f32(x[i]);
    f[2 * i + 1] = hi_f32(x[i]);
  }
}

// This lane's cosines and sines: eight pairs (halves), or four (neighbours), each used twice.
template <bool PAIRED>
struct Angles {
  float cs[PAIRED ? 4 : 8], sn[PAIRED ? 4 : 8];
};
template <bool PAIRED>
__device__ __forceinline__ void load_angles(const RopeArgs& a, int pos, int d0, Angles<PAIRED>& t) {
  const int half = a.rotary >> 1;
  const float* const row = a.cos_sin + (size_t)pos * a.rotary;
  const int p0 = PAIRED ? d0 / 2 : d0 < half ? d0 : d0 - half;
#pragma unroll
  for (int i = 0; i < (PAIRED ? 4 : 8); i += 4) {
    float4 c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
    if (d0 < a.rotary) {
      c = *(const float4*)(row + p0 + i);
      s = *(const float4*)(row + half + p0 + i);
    }
    t.cs[i] = c.x, t.cs[i + 1] = c.y, t.cs[i + 2] = c.z, t.cs[i + 3] = c.w;
    t.sn[i] = s.x, t.sn[i + 1] = s.y, t.sn[i + 2] = s.z, t.sn[i + 3] = s.w;
  }
}

// Norm and rotation of one head vector, dimensions d0 .. d0 + 8 of it in this lane
// (w may be null); every lane of the group of sixteen takes part.
template <bool PAIRED>
__device__ __forceinline__ void turn_head(const RopeArgs& a, const i32x4& x, const uint16_t* w, const Angles<PAIRED>& t,
                                          int d0, float (&z)[8]) {
  const int lane = threadIdx.x & 63, l = lane & 15, half = a.rotary >> 1;
  const bool turned = d0 < a.rotary;
  const int mate = (lane & 48) | ((d0 < half ? l + (half >> 3) : l - (half >> 3)) & 15);
  const float sign = d0 < half ? -1.f : 1.f;
  float y[8];
  unpack8(x, y);
  float inv = 1.f;
  if (w) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(y[e], y[e], ss);
    inv = 1.0f / sqrtf(row_sum(ss) * (1.0f / kD) + a.eps);
    float f[8];
    unpack8(*(const i32x4*)(w + d0), f);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = y[e] * inv * f[e];
  }
  if constexpr (PAIRED) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[2 * e] = turned ? y[2 * e] * t.cs[e] - y[2 * e + 1] * t.sn[e] : y[2 * e];
      z[2 * e + 1] = turned ? y[2 * e + 1] * t.cs[e] + y[2 * e] * t.sn[e] : y[2 * e + 1];
    }
  } else {
    i32x4 ox;
#pragma unroll
    for (int e = 0; e < 4; ++e) ox[e] = __shfl(x[e], mate);
    float o[8];
    unpack8(ox, o);
    if (w) {
      float f[8];
      unpack8(*(const i32x4*)(w + 8 * (mate & 15)), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] = o[e] * inv * f[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = turned ? y[e] * t.cs[e] + sign * o[e] * t.sn[e] : y[e];
  }
}

// HG: heads per group of sixteen lanes.  KEYS: k as well (else the queries only)
template <bool FP8, bool PAIRED, int HG, bool KEYS = true>
__device__ __forceinline__ void qk_part(const RopeArgs& a, int64_t group0 = 0) {
  const int lane = threadIdx.x & 63, l = lane & 15;
  const int H = a.hq + (KEYS ? a.hkv : 0);
  const int units = (H + HG - 1) / HG;  // per row
  const int64_t unit = (((int64_t)blockIdx.x - group0) * kWaves + (threadIdx.x >> 6)) * 4 + (lane >> 4);
  const int64_t r = unit / units;
  const bool live = r < a.rows;  // (exchanges below need every lane of a group, and a group is one unit's)
  const int64_t rc = live ? r : 0;
  const int h0 = (int)(unit - r * units) * HG;
  const int pos = a.positions[rc];
  const int64_t slot = a.slots[rc];
  if (!live || pos < 0 || pos >= a.n_positions) return;

  const int d0 = 8 * l;
  i32x4 x[HG];
#pragma unroll
  for (int i = 0; i < HG; ++i) {
    const int h = h0 + i;
    if (h < a.hq) x[i] = *(const i32x4*)(a.q + r * a.q_stride + h * kD + d0);
    else if (h < H) x[i] = *(const i32x4*)(a.k + r * a.k_stride + (h - a.hq) * kD + d0);
    else x[i] = i32x4{0, 0, 0, 0};
  }
  Angles<PAIRED> t;
  load_angles<PAIRED>(a, pos, d0, t);

#pragma unroll
  for (int i = 0; i < HG; ++i) {
    const int h = h0 + i;
    if (h >= H) break;
    const bool is_q = h < a.hq;
    float z[8];
    turn_head<PAIRED>(a, x[i], is_q ? a.q_weight : a.k_weight, t, d0, z);
    if (is_q) {
      const i32x4 p = {pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])};
      *(i32x4*)(a.q_out + (r * a.hq + h) * kD + d0) = p;
    } else if (slot >= 0 && slot < a.n_slots) {
      const int g = h - a.hq;
      const size_t at = (((size_t)(slot / kBS) * a.hkv + g) * kBS + slot % kBS) * kD + d0;
      if constexpr (FP8) {
        const float s = a.k_scale[g];
        const i32x2 p = {pack_e4m3(z[0] / s, z[1] / s, z[2] / s, z[3] / s),
                         pack_e4m3(z[4] / s, z[5] / s, z[6] / s, z[7] / s)};
        *(i32x2*)(a.kc + at) = p;
      } else {
        const i32x4 p = {pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]),
                         pack_bf16(z[6], z[7])};
        *(i32x4*)((uint16_t*)a.kc + at) = p;
      }
    }
  }
}

// Slot of row r if it goes into the cache, -1 otherwise
__device__ __forceinline__ int64_t cache_slot(const RopeArgs& a, int64_t r) {
  if (r < 0 || r >= a.rows) return -1;
  const int pos = a.positions[r];
  const int64_t slot = a.slots[r];
  return pos >= 0 && pos < a.n_positions && slot >= 0 && slot < a.n_slots ? slot : -1;
}

// One wave: the runs that start in a window of WIN rows, for head g.
template <bool FP8, int WIN>
__device__ __forceinline__ void v_part(const RopeArgs& a, uint32_t (*tile)[kD / 2]) {
  const int lane = threadIdx.x & 63, l = lane & 15;
  const int64_t unit = ((int64_t)blockIdx.x - a.qk_groups) * kWaves + (threadIdx.x >> 6);
  const int64_t win = unit / a.hkv;
  const int g = (int)(unit - win * a.hkv);
  const int64_t w0 = win * WIN;
  if (w0 >= a.rows) return;
  // lane i: row w0 - 1 + i
  const int64_t sl = lane <= WIN + kBS ? cache_slot(a, w0 - 1 + lane) : -1;
  const int64_t before = __shfl_up(sl, 1);
  const bool starts = sl >= 0 && (before < 0 || before + 1 != sl || sl % kBS == 0);
  const uint64_t start_bits = __ballot(lane >= 1 && starts);
  const uint64_t none_bits = __ballot(sl < 0);
  uint64_t todo = start_bits & (((1ull << WIN) - 1) << 1);
  const float scale = FP8 ? a.v_scale[g] : 1.f;
  while (todo) {
    const int f = __builtin_ctzll(todo);  // the run's first row is w0 - 1 + f
    todo &= todo - 1;
    const uint64_t ends = (start_bits | none_bits) & ~((2ull << f) - 1);
    const int len = min(ends ? __builtin_ctzll(ends) - f : 64 - f, kBS);
    const int64_t slot = __shfl(sl, f);
    const int64_t r0 = w0 - 1 + f;
    const int off = (int)(slot % kBS);
    const size_t at = (size_t)(slot / kBS) * a.hkv + g;
    // rows to LDS, four at a time
    for (int i = lane >> 4; i < len; i += 4)
      *(i32x4*)&tile[i][4 * l] = *(const i32x4*)(a.v + (r0 + i) * a.v_stride + g * kD + 8 * l);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // this lane's dimensions 2 lane and 2 lane + 1
    if constexpr (FP8) {
      char* const out = a.vc + at * (kBS * kD) + 2 * lane * kBS + off;
      if (len == kBS) {
        i32x4 c0, c1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x[4], y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int w = tile[4 * i + e][lane];
            x[e] = lo_f32(w) / scale;
            y[e] = hi_f32(w) / scale;
          }
          c0[i] = pack_e4m3(x[0], x[1], x[2], x[3]);
          c1[i] = pack_e4m3(y[0], y[1], y[2], y[3]);
        }
        *(i32x4*)out = c0;
        *(i32x4*)(out + kBS) = c1;
      } else {
        for (int i = 0; i < len;) {
          if ((off + i) % 4 == 0 && i + 4 <= len) {  // four tokens that one word holds
            float x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int w = tile[i + e][lane];
              x[e] = lo_f32(w) / scale;
              y[e] = hi_f32(w) / scale;
            }
            *(int*)(out + i) = pack_e4m3(x[0], x[1], x[2], x[3]);
            *(int*)(out + kBS + i) = pack_e4m3(y[0], y[1], y[2], y[3]);
            i += 4;
          } else {
            const int w = tile[i][lane];
            const int c = pack_e4m3(lo_f32(w) / scale, hi_f32(w) / scale, 0.f, 0.f);
            out[i] = (char)(c & 0xff);
            out[kBS + i] = (char)((c >> 8) & 0xff);
            ++i;
          }
        }
      }
    } else {
      uint16_t* const out = (uint16_t*)a.vc + at * (kBS * kD) + 2 * lane * kBS + off;
      if (len == kBS) {
        i32x4 c[4];  // dimension 2 lane, tokens 0-7 and 8-15, then 2 lane + 1
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t u = tile[2 * i][lane], w = tile[2 * i + 1][lane];
          c[i >> 2][i & 3] = (int)((u & 0xffff) | (w << 16));
          c[2 + (i >> 2)][i & 3] = (int)((u >> 16) | (w & 0xffff0000u));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) *(i32x4*)(out + 8 * i) = c[i];
      } else {
        for (int i = 0; i < len;) {
          if ((off + i) % 4 == 0 && i + 4 <= len) {
            const uint32_t w0 = tile[i][lane], w1 = tile[i + 1][lane], w2 = tile[i + 2][lane], w3 = tile[i + 3][lane];
            *(i32x2*)(out + i) = i32x2{(int)((w0 & 0xffff) | (w1 << 16)), (int)((w2 & 0xffff) | (w3 << 16))};
            *(i32x2*)(out + kBS + i) = i32x2{(int)((w0 >> 16) | (w1 & 0xffff0000u)), (int)((w2 >> 16) | (w3 & 0xffff0000u))};
            i += 4;
          } else {
            const uint32_t w = tile[i][lane];
            out[i] = (uint16_t)w;
            out[kBS + i] = (uint16_t)(w >> 16);
            ++i;
          }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the tile is read before the next run's rows
  }
}

// ------------------------------------------------------------------ block scales

// Largest value over the 64 lanes, in every lane: rotations within the rows of
// sixteen, then exchanges between them, all in the vector ALU
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x128, 0xf, 0xf, false)));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x124, 0xf, 0xf, false)));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x122, 0xf, 0xf, false)));
  x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x121, 0xf, 0xf, false)));
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// The exponent byte of the smallest power of two over which a magnitude is at
// most 448 = 1.75 * 2^8: its own exponent less 8, one more where its mantissa is
// above 1.75.  At most 246, so that 448 times it is finite in bf16.
__device__ __forceinline__ int need_byte(float a) {
  return min(max((int)((__float_as_uint(a) + 0x1fffffu) >> 23) - 8, 1), 246);
}
__device__ __forceinline__ float pow2_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }
// 1 over it (2^-127 has no exponent byte of its own; a begun block of byte 255 is NaN whatever its codes)
__device__ __forceinline__ float inverse_pow2_of(int byte) {
  return byte < 254 ? pow2_of(254 - byte) : __uint_as_float(0x00400000u);
}

__device__ __forceinline__ float finite_abs(float x) {
  const float b = fabsf(x);
  return b < INFINITY ? b : 0.f;  // (NaN too)
}

// Four values over a scale to e4m3 codes; `inv` is its inverse.  What is not
// finite becomes NaN: no code stands for an infinity, and the largest code of a
// block is as small as its scale.
__device__ __forceinline__ int encode4(float a, float b, float c, float d, float inv) {
  const auto cut = [inv](float x) {
    const float y = fminf(fmaxf(x * inv, -kE4M3Max), kE4M3Max);
    return fabsf(x) < INFINITY ? y : __builtin_nanf("");
  };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(cut(a), cut(b), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(cut(c), cut(d), r, true);
}

// Four codes times a power of two, as codes (a NaN stays one).
__device__ __forceinline__ int recode4(int w, float pow2) {
  const auto x = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, pow2, false);
  const auto y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, pow2, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], r, true);
}
// The factor of codes whose scale's byte rises from old to byte.
__device__ __forceinline__ float shrink(int old, int byte) { return pow2_of(max(127 + old - byte, 0)); }

// One wave: K (else V) of head g, for the runs of rows of one block that start in a window of WIN rows.
//
// Sixteen lanes hold a row, so four rows of a run are taken at a time.  K of up
// to four rows (single tokens, most drafts) stays in registers between the
// maximum and the codes; of longer runs it is computed again from the rows, which
// are in the caches by then: registers for sixteen rows (170 instead of 88) cost
// the queries' waves in the same launch their occupancy (nine prompts on 64/8
// heads, 12,677 rows, 500 MB: 175 us; 114 so).  Sharing the angles of a run's
// rows in LDS, or four heads of a row in one thread, came to 113 to 136.
template <bool PAIRED, int WIN>
__device__ __forceinline__ void scaled_part(const RopeArgs& a, int64_t unit, uint32_t (*tile)[kD / 2]) {
  const int lane = threadIdx.x & 63, l = lane & 15, sub = lane >> 4, d0 = 8 * l;
  const int64_t win = unit / (2 * a.hkv);
  const int head = (int)(unit - win * (2 * a.hkv));
  const bool keys = head < a.hkv;
  const int g = keys ? head : head - a.hkv;
  const int64_t w0 = win * WIN;
  if (w0 >= a.rows) return;
  const uint16_t* const src = (keys ? a.k : a.v) + g * kD + d0;
  const int64_t stride = keys ? a.k_stride : a.v_stride;
  uint8_t* const exps = keys ? a.k_exp : a.v_exp;
  // lane i: row w0 - 1 + i
  const int64_t row = w0 - 1 + lane;
  int pos = -1;
  int64_t sl = -1;
  if (lane <= WIN + kBS && row >= 0 && row < a.rows) {
    pos = a.positions[row];
    sl = a.slots[row];
  }
  // (with a window of one row the run, if there is one, starts there: its rows
  // are asked for together with their slots)
  i32x4 ahead = {0, 0, 0, 0};
  if (WIN == 1 && w0 + sub < a.rows) ahead = *(const i32x4*)(src + (w0 + sub) * stride);
  if (pos < 0 || pos >= a.n_positions || sl < 0 || sl >= a.n_slots) sl = -1;
  const int blk = sl < 0 ? -1 : (int)(sl / kBS);
  const int before = __shfl_up(blk, 1);
  const bool starts = blk >= 0 && blk != before;
  const uint64_t edges = __ballot(lane >= 1 && blk != before) | ~0ull << (WIN + kBS + 1);
  uint64_t todo = __ballot(lane >= 1 && starts) & (((1ull << WIN) - 1) << 1);
  while (todo) {
    const int f = __builtin_ctzll(todo);  // the run's first row is w0 - 1 + f
    todo &= todo - 1;
    const uint64_t ends = edges & ~((2ull << f) - 1);
    const int len = min(__builtin_ctzll(ends) - f, kBS);
    const int64_t r0 = w0 - 1 + f;
    const int off = (int)(__builtin_amdgcn_readlane((int)(sl & (kBS - 1)), f));
    const size_t at = (size_t)__builtin_amdgcn_readlane(blk, f) * a.hkv + g;
    const int slot = (int)(sl & (kBS - 1));  // of row w0 - 1 + lane in its block
    const int old = off > 0 ? exps[at] : 0;
    auto load_row = [&](int n) __attribute__((always_inline)) {
      return WIN == 1 && n < 4 ? ahead : *(const i32x4*)(src + (r0 + n) * stride);
    };
    if (keys) {
      char* const out = a.kc + at * (kBS * kD) + d0;
      float z[8];
      auto turned = [&](int n0) __attribute__((always_inline)) {  // z of row n0 + sub
        const int n = n0 + sub;
        const int p = __shfl(pos, f + n);
        i32x4 x = {0, 0, 0, 0};
        Angles<PAIRED> t{};
        if (n < len) {
          x = load_row(n);
          load_angles<PAIRED>(a, p, d0, t);
        }
        turn_head<PAIRED>(a, x, a.k_weight, t, d0, z);
        return n < len;
      };
      float top = 0.f;
      for (int n0 = 0; n0 < len; n0 += 4)
        if (turned(n0))
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_abs(z[e]));
      const int byte = max(need_byte(wave_max(top)), old);
      if (byte != old && off > 0) {
        const float p = shrink(old, byte);
        for (int n = sub; n < off; n += 4) {
          i32x2 c = *(const i32x2*)(out + n * kD);
          c[0] = recode4(c[0], p);
          c[1] = recode4(c[1], p);
          *(i32x2*)(out + n * kD) = c;
        }
      }
      const float inv = inverse_pow2_of(byte);
      for (int n0 = 0; n0 < len; n0 += 4) {
        const int at_slot = __shfl(slot, f + n0 + sub);
        if (len > 4) turned(n0);
        if (n0 + sub < len)
          *(i32x2*)(out + at_slot * kD) =
              i32x2{encode4(z[0], z[1], z[2], z[3], inv), encode4(z[4], z[5], z[6], z[7], inv)};
      }
      if (lane == 0) exps[at] = (uint8_t)byte;
    } else {
      // This lane's dimensions 2 lane and 2 lane + 1: sixteen tokens each, written
      // whole.  Slots that are not the run's keep their codes, those of earlier
      // tokens under the block's scale.
      i32x4* const out = (i32x4*)(a.vc + at * (kBS * kD) + 2 * lane * kBS);
      i32x4 c0 = {0, 0, 0, 0}, c1 = c0;
      if (len < kBS) {
        c0 = out[0];
        c1 = out[1];
      }
      float top = 0.f;
      for (int n = sub; n < len; n += 4) {
        const i32x4 x = load_row(n);
        *(i32x4*)&tile[n][4 * l] = x;
        float y[8];
        unpack8(x, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, finite_abs(y[e]));
      }
      const int byte = max(need_byte(wave_max(top)), old);
      const float inv = inverse_pow2_of(byte);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (byte != old && off > 0 && len < kBS) {
        const float p = shrink(old, byte);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = min(max(off - 4 * i, 0), 4);  // earlier tokens in this word
          const int m = k == 4 ? -1 : (1 << (8 * k)) - 1;
          c0[i] = (recode4(c0[i], p) & m) | (c0[i] & ~m);
          c1[i] = (recode4(c1[i], p) & m) | (c1[i] & ~m);
        }
      }
      if (len == kBS && off == 0) {
        // a whole block (its slots rise from 0 to 15)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x[4], y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int w = tile[4 * i + e][lane];
            x[e] = lo_f32(w);
            y[e] = hi_f32(w);
          }
          c0[i] = encode4(x[0], x[1], x[2], x[3], inv);
          c1[i] = encode4(y[0], y[1], y[2], y[3], inv);
        }
      } else {
        for (int n = 0; n < len; ++n) {
          const int to = __builtin_amdgcn_readlane(slot, f + n), sh = 8 * (to & 3);
          const int w = tile[n][lane];
          const int c = encode4(lo_f32(w), hi_f32(w), 0.f, 0.f, inv);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (i == to >> 2) {
              c0[i] = (c0[i] & ~(0xff << sh)) | ((c & 0xff) << sh);
              c1[i] = (c1[i] & ~(0xff << sh)) | (((c >> 8) & 0xff) << sh);
            }
          }
        }
      }
      out[0] = c0;
      out[1] = c1;
      if (lane == 0) exps[at] = (uint8_t)byte;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the tile is read before the next run's rows
    }
  }
}

template <bool PAIRED, int HG, int WIN>
__global__ __launch_bounds__(kWaves * 64) void qk_rope_scaled_kernel(RopeArgs a) {
  __shared__ uint32_t tile[kWaves][kBS][kD / 2];
  // K and V first: theirs are chains of dependent loads, quick while the memory
  // is idle (one such workgroup among every eight of the queries': 148 us for 114)
  const int64_t kv = (int64_t)gridDim.x - a.qk_groups;
  if ((int64_t)blockIdx.x < kv)
    scaled_part<PAIRED, WIN>(a, (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6), tile[threadIdx.x >> 6]);
  else
    qk_part<true, PAIRED, HG, false>(a, kv);
}

template <int HG, int WIN>
void launch_scaled(RopeArgs& a, bool paired, hipStream_t st) {
  const int64_t units = a.rows * ((a.hq + HG - 1) / HG);
  a.qk_groups = (units + 4 * kWaves - 1) / (4 * kWaves);
  const int64_t runs = (a.rows + WIN - 1) / WIN * (2 * a.hkv);
  const dim3 grid((unsigned)(a.qk_groups + (runs + kWaves - 1) / kWaves)), block(kWaves * 64);
  if (paired) hipLaunchKernelGGL((qk_rope_scaled_kernel<true, HG, WIN>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((qk_rope_scaled_kernel<false, HG, WIN>), grid, block, 0, st, a);
}

template <bool FP8, bool PAIRED, int HG, int WIN>
__global__ __launch_bounds__(kWaves * 64) void qk_rope_kernel(RopeArgs a) {
  __shared__ uint32_t tile[kWaves][kBS][kD / 2];
  if ((int64_t)blockIdx.x < a.qk_groups) qk_part<FP8, PAIRED, HG>(a);
  else v_part<FP8, WIN>(a, tile[threadIdx.x >> 6]);
}

template <int HG, int WIN>
void launch(RopeArgs& a, bool fp8, bool paired, hipStream_t st) {
  const int64_t units = a.rows * ((a.hq + a.hkv + HG - 1) / HG);
  a.qk_groups = (units + 4 * kWaves - 1) / (4 * kWaves);
  const int64_t v_units = (a.rows + WIN - 1) / WIN * a.hkv;
  const dim3 grid((unsigned)(a.qk_groups + (v_units + kWaves - 1) / kWaves)), block(kWaves * 64);
  if (fp8 && paired) hipLaunchKernelGGL((qk_rope_kernel<true, true, HG, WIN>), grid, block, 0, st, a);
  else if (fp8) hipLaunchKernelGGL((qk_rope_kernel<true, false, HG, WIN>), grid, block, 0, st, a);
  else if (paired) hipLaunchKernelGGL((qk_rope_kernel<false, true, HG, WIN>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((qk_rope_kernel<false, false, HG, WIN>), grid, block, 0, st, a);
}

}  // namespace dpool_rope

using namespace dpool_rope;

namespace {

// block: the scales of qk_norm_rope_append_scaled (k_exp, v_exp), else those of qk_norm_rope_append
int enqueue(const void* q, const void* k, const void* v, const void* q_weight, const void* k_weight, float eps,
            const float* cos_sin, const int32_t* positions, const int64_t* slots, void* q_out, void* k_blocks,
            void* v_blocks, const float* k_scale, const float* v_scale, bool block, uint8_t* k_exp, uint8_t* v_exp,
            const dp_qk_shape* sh, void* stream) {
  using dpool::fail;
  const char* const name = block ? "qk_norm_rope_append_scaled" : "qk_norm_rope_append";
  if (!sh) return fail(DP_EINVAL, "%s: null shape", name);
  if (sh->head_dim != kD) return fail(DP_ENOTSUP, "%s: head_dim %d (only 128)", name, sh->head_dim);
  if (sh->block_size != kBS) return fail(DP_ENOTSUP, "%s: block_size %d (only 16)", name, sh->block_size);
  if (block ? sh->kv_dtype != DP_KV_FP8_E4M3_BLOCK
            : sh->kv_dtype != DP_KV_BF16 && sh->kv_dtype != DP_KV_FP8_E4M3)
    return fail(DP_ENOTSUP, "%s: kv_dtype %d", name, sh->kv_dtype);
  if (sh->reserved != 0 || (sh->interleaved != 0 && sh->interleaved != 1))
    return fail(DP_EINVAL, "%s: reserved must be 0 and interleaved 0 or 1", name);
  if (sh->rotary_dim < 0 || sh->rotary_dim > kD || sh->rotary_dim % 16 != 0)
    return fail(DP_ENOTSUP, "%s: rotary_dim %d (a multiple of 16 up to 128)", name, sh->rotary_dim);
  if (sh->n_q_heads < (block ? 0 : 1) || sh->n_kv_heads <= 0 || sh->n_q_heads > 65536 || sh->n_kv_heads > 65536)
    return fail(DP_EINVAL, "%s: head counts out of range", name);
  if (sh->rows < 0 || sh->num_blocks <= 0 || sh->num_blocks > INT32_MAX || sh->n_positions <= 0 ||
      sh->n_positions > INT32_MAX)
    return fail(DP_EINVAL, "%s: rows, num_blocks or n_positions out of range", name);
  if (sh->rows > INT32_MAX / ((int64_t)sh->n_q_heads + 2 * (int64_t)sh->n_kv_heads))
    return fail(DP_EINVAL, "%s: too many rows", name);
  // (a row's heads lie next to each other, so rows closer than that would overlap)
  if (sh->q_stride < (int64_t)sh->n_q_heads * kD || sh->k_stride < (int64_t)sh->n_kv_heads * kD ||
      sh->v_stride < (int64_t)sh->n_kv_heads * kD || (sh->q_stride | sh->k_stride | sh->v_stride) % 8 != 0 ||
      std::max({sh->q_stride, sh->k_stride, sh->v_stride}) > INT64_MAX / 4 / std::max<int64_t>(sh->rows, 1))
    return fail(DP_EINVAL, "%s: strides must be multiples of 8 that hold a row's heads", name);
  if (sh->rows == 0) return DP_OK;
  if ((sh->n_q_heads && (!q || !q_out)) || !k || !v || !positions || !slots || !k_blocks || !v_blocks ||
      (sh->rotary_dim && !cos_sin))
    return fail(DP_EINVAL, "%s: null tensor pointer", name);
  const bool fp8 = sh->kv_dtype == DP_KV_FP8_E4M3;
  if (block && (!k_exp || !v_exp || k_exp == v_exp || k_blocks == v_blocks))
    return fail(DP_EINVAL, "%s: k_scale, v_scale and the two caches must be there, and apart", name);
  if (fp8 && (!k_scale || !v_scale))
    return fail(DP_EINVAL, "%s: e4m3 cache needs k_scale and v_scale", name);
  if (!fp8 && (k_scale || v_scale))
    return fail(DP_EINVAL, "%s: k_scale/v_scale must be NULL for a bf16 cache", name);
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_weight | (uintptr_t)k_weight | (uintptr_t)cos_sin |
       (uintptr_t)q_out | (uintptr_t)k_blocks | (uintptr_t)v_blocks) & 15)
    return fail(DP_EINVAL, "%s: q, k, v, weights, cos_sin, q_out and caches must be 16-byte aligned", name);
  if (((uintptr_t)positions | (uintptr_t)k_scale | (uintptr_t)v_scale) & 3 || (uintptr_t)slots & 7)
    return fail(DP_EINVAL, "%s: positions, slots and scales must be aligned to their elements", name);
  if (q_out && q_out == q && sh->q_stride != (int64_t)sh->n_q_heads * kD)
    return fail(DP_EINVAL, "%s: q_out may be q only where q_stride is n_q_heads * 128", name);
  if (q_out && (q_out == k || q_out == v)) return fail(DP_EINVAL, "%s: q_out must not be k or v", name);
  if ((q_weight || k_weight) && !(eps >= 0.0f && std::isfinite(eps)))
    return fail(DP_EINVAL, "%s: eps must be finite and >= 0", name);

  RopeArgs a;
  a.q = (const uint16_t*)q;
  a.k = (const uint16_t*)k;
  a.v = (const uint16_t*)v;
  a.q_weight = (const uint16_t*)q_weight;
  a.k_weight = (const uint16_t*)k_weight;
  a.cos_sin = cos_sin;
  a.positions = positions;
  a.slots = slots;
  a.q_out = (uint16_t*)q_out;
  a.kc = (char*)k_blocks;
  a.vc = (char*)v_blocks;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.rows = sh->rows;
  a.n_positions = sh->n_positions;
  a.n_slots = sh->num_blocks * kBS;
  a.q_stride = sh->q_stride;
  a.k_stride = sh->k_stride;
  a.v_stride = sh->v_stride;
  a.eps = eps;
  a.hq = sh->n_q_heads;
  a.hkv = sh->n_kv_heads;
  a.rotary = sh->rotary_dim;
  a.k_exp = k_exp;
  a.v_exp = v_exp;
  (void)hipGetLastError();
  // Heads per group of lanes, and rows whose runs one wave looks for.  Few rows
  // want many waves; many rows share cosines, and prompts' runs of sixteen want
  // windows of sixteen.  64/8 heads, bf16, us with (1, 1) / (2, 4) / (2, 16):
  // 256 single tokens 8.5 / 9.0 / 16.2; 256 trees of four 17.8 / 13.9 / 14.8;
  // 4,096 tokens of four prompts 84 / 51 / 43, as 4,096 single tokens 106 / 100 /
  // 114; 8,192 tokens of prompts 160 / 94 / 78 (5.4 TB/s; a large copy reaches 4.8).
  // The host sees rows and not their slots: thousands of single tokens pay for what
  // prompts gain.  Other head counts were not measured beside the rule.
  const bool paired = sh->interleaved == 1;
  hipStream_t st = (hipStream_t)stream;
  if (block) {
    // The same trade-off.  64/8 heads, us with (2, 1) / (8, 4) / (8, 16): 256 single
    // tokens 6.6 / 7.8 / 19; 512 in runs of five 8.4 / 7.9 / 12.9; 1,024 single
    // tokens 16.6 / 15.8 / 22.5, of prompts 20.6 / 11.2 / 12.5; 8,192 single tokens
    // 150 / 133 / 136, of prompts 154 / 81 / 58 (eight heads a group of lanes: more
    // loads in flight for a stream whose occupancy K's registers cut; with two 98).
    if (sh->rows < 512) launch_scaled<2, 1>(a, paired, st);
    else if (sh->rows < 4096) launch_scaled<8, 4>(a, paired, st);
    else launch_scaled<8, 16>(a, paired, st);
  } else if (sh->rows <= 256) launch<1, 1>(a, fp8, paired, st);
  else if (sh->rows < 4096) launch<2, 4>(a, fp8, paired, st);
  else launch<2, 16>(a, fp8, paired, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(DP_EIO, "%s: kernel launch failed: %s", name, hipGetErrorString(e));
  return DP_OK;
}

}  // namespace

extern "C" int qk_norm_rope_append(const void* q, const void* k, const void* v, const void* q_weight,
                                   const void* k_weight, float eps, const float* cos_sin, const int32_t* positions,
                                   const int64_t* slots, void* q_out, void* k_blocks, void* v_blocks,
                                   const float* k_scale, const float* v_scale, const dp_qk_shape* shape,
                                   void* stream) {
  return enqueue(q, k, v, q_weight, k_weight, eps, cos_sin, positions, slots, q_out, k_blocks, v_blocks, k_scale,
                 v_scale, false, nullptr, nullptr, shape, stream);
}

extern "C" int qk_norm_rope_append_scaled(const void* q, const void* k, const void* v, const void* q_weight,
                                          const void* k_weight, float eps, const float* cos_sin,
                                          const int32_t* positions, const int64_t* slots, void* q_out,
                                          void* k_blocks, void* v_blocks, uint8_t* k_scale, uint8_t* v_scale,
                                          const dp_qk_shape* shape, void* stream) {
  return enqueue(q, k, v, q_weight, k_weight, eps, cos_sin, positions, slots, q_out, k_blocks, v_blocks, nullptr,
                 nullptr, true, k_scale, v_scale, shape, stream);
}

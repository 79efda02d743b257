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

// HG: heads per group of sixteen lanes
template <bool FP8, bool PAIRED, int HG>
__device__ __forceinline__ void qk_part(const RopeArgs& a) {
  const int lane = threadIdx.x & 63, l = lane & 15;
  const int H = a.hq + a.hkv;
  const int units = (H + HG - 1) / HG;  // per row
  const int64_t unit = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * 4 + (lane >> 4);
  const int64_t r = unit / units;
  const bool live = r < a.rows;  // (exchanges below need every lane of a group, and a group is one unit's)
  const int64_t rc = live ? r : 0;
  const int h0 = (int)(unit - r * units) * HG;
  const int pos = a.positions[rc];
  const int64_t slot = a.slots[rc];
  if (!live || pos < 0 || pos >= a.n_positions) return;

  const int d0 = 8 * l, half = a.rotary >> 1;
  const bool turned = d0 < a.rotary;
  i32x4 x[HG];
#pragma unroll
  for (int i = 0; i < HG; ++i) {
    const int h = h0 + i;
    if (h < a.hq) x[i] = *(const i32x4*)(a.q + r * a.q_stride + h * kD + d0);
    else if (h < H) x[i] = *(const i32x4*)(a.k + r * a.k_stride + (h - a.hq) * kD + d0);
    else x[i] = i32x4{0, 0, 0, 0};
  }
  // this lane's cosines and sines: eight pairs (halves), or four (neighbours), each used twice
  float cs[PAIRED ? 4 : 8], sn[PAIRED ? 4 : 8];
  const float* const row = a.cos_sin + (size_t)pos * a.rotary;
  const int p0 = PAIRED ? d0 / 2 : d0 < half ? d0 : d0 - half;
#pragma unroll
  for (int i = 0; i < (PAIRED ? 4 : 8); i += 4) {
    float4 c = {1.f, 1.f, 1.f, 1.f}, s = {0.f, 0.f, 0.f, 0.f};
    if (turned) {
      c = *(const float4*)(row + p0 + i);
      s = *(const float4*)(row + half + p0 + i);
    }
    cs[i] = c.x, cs[i + 1] = c.y, cs[i + 2] = c.z, cs[i + 3] = c.w;
    sn[i] = s.x, sn[i + 1] = s.y, sn[i + 2] = s.z, sn[i + 3] = s.w;
  }
  const int mate = (lane & 48) | ((d0 < half ? l + (half >> 3) : l - (half >> 3)) & 15);
  const float sign = d0 < half ? -1.f : 1.f;

#pragma unroll
  for (int i = 0; i < HG; ++i) {
    const int h = h0 + i;
    if (h >= H) break;
    const bool is_q = h < a.hq;
    float y[8];
    unpack8(x[i], y);
    float inv = 1.f;
    const uint16_t* const w = is_q ? a.q_weight : a.k_weight;
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
    float z[8];
    if constexpr (PAIRED) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        z[2 * e] = turned ? y[2 * e] * cs[e] - y[2 * e + 1] * sn[e] : y[2 * e];
        z[2 * e + 1] = turned ? y[2 * e + 1] * cs[e] + y[2 * e] * sn[e] : y[2 * e + 1];
      }
    } else {
      i32x4 ox;
#pragma unroll
      for (int e = 0; e < 4; ++e) ox[e] = __shfl(x[i][e], mate);
      float o[8];
      unpack8(ox, o);
      if (w) {
        float f[8];
        unpack8(*(const i32x4*)(w + 8 * (mate & 15)), f);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = o[e] * inv * f[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = turned ? y[e] * cs[e] + sign * o[e] * sn[e] : y[e];
    }
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

extern "C" int qk_norm_rope_append(const void* q, const void* k, const void* v, const void* q_weight,
                                   const void* k_weight, float eps, const float* cos_sin, const int32_t* positions,
                                   const int64_t* slots, void* q_out, void* k_blocks, void* v_blocks,
                                   const float* k_scale, const float* v_scale, const dp_qk_shape* sh, void* stream) {
  using dpool::fail;
  if (!sh) return fail(DP_EINVAL, "qk_norm_rope_append: null shape");
  if (sh->head_dim != kD) return fail(DP_ENOTSUP, "qk_norm_rope_append: head_dim %d (only 128)", sh->head_dim);
  if (sh->block_size != kBS) return fail(DP_ENOTSUP, "qk_norm_rope_append: block_size %d (only 16)", sh->block_size);
  if (sh->kv_dtype != DP_KV_BF16 && sh->kv_dtype != DP_KV_FP8_E4M3)
    return fail(DP_ENOTSUP, "qk_norm_rope_append: kv_dtype %d", sh->kv_dtype);
  if (sh->reserved != 0 || (sh->interleaved != 0 && sh->interleaved != 1))
    return fail(DP_EINVAL, "qk_norm_rope_append: reserved must be 0 and interleaved 0 or 1");
  if (sh->rotary_dim < 0 || sh->rotary_dim > kD || sh->rotary_dim % 16 != 0)
    return fail(DP_ENOTSUP, "qk_norm_rope_append: rotary_dim %d (a multiple of 16 up to 128)", sh->rotary_dim);
  if (sh->n_q_heads <= 0 || sh->n_kv_heads <= 0 || sh->n_q_heads > 65536 || sh->n_kv_heads > 65536)
    return fail(DP_EINVAL, "qk_norm_rope_append: head counts out of range");
  if (sh->rows < 0 || sh->num_blocks <= 0 || sh->num_blocks > INT32_MAX || sh->n_positions <= 0 ||
      sh->n_positions > INT32_MAX)
    return fail(DP_EINVAL, "qk_norm_rope_append: rows, num_blocks or n_positions out of range");
  if (sh->rows > INT32_MAX / ((int64_t)sh->n_q_heads + 2 * (int64_t)sh->n_kv_heads))
    return fail(DP_EINVAL, "qk_norm_rope_append: too many rows");
  // (a row's heads lie next to each other, so rows closer than that would overlap)
  if (sh->q_stride < (int64_t)sh->n_q_heads * kD || sh->k_stride < (int64_t)sh->n_kv_heads * kD ||
      sh->v_stride < (int64_t)sh->n_kv_heads * kD || (sh->q_stride | sh->k_stride | sh->v_stride) % 8 != 0 ||
      std::max({sh->q_stride, sh->k_stride, sh->v_stride}) > INT64_MAX / 4 / std::max<int64_t>(sh->rows, 1))
    return fail(DP_EINVAL, "qk_norm_rope_append: strides must be multiples of 8 that hold a row's heads");
  if (sh->rows == 0) return DP_OK;
  if (!q || !k || !v || !positions || !slots || !q_out || !k_blocks || !v_blocks || (sh->rotary_dim && !cos_sin))
    return fail(DP_EINVAL, "qk_norm_rope_append: null tensor pointer");
  const bool fp8 = sh->kv_dtype == DP_KV_FP8_E4M3;
  if (fp8 && (!k_scale || !v_scale))
    return fail(DP_EINVAL, "qk_norm_rope_append: e4m3 cache needs k_scale and v_scale");
  if (!fp8 && (k_scale || v_scale))
    return fail(DP_EINVAL, "qk_norm_rope_append: k_scale/v_scale must be NULL for a bf16 cache");
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)q_weight | (uintptr_t)k_weight | (uintptr_t)cos_sin |
       (uintptr_t)q_out | (uintptr_t)k_blocks | (uintptr_t)v_blocks) & 15)
    return fail(DP_EINVAL, "qk_norm_rope_append: q, k, v, weights, cos_sin, q_out and caches must be 16-byte aligned");
  if (((uintptr_t)positions | (uintptr_t)k_scale | (uintptr_t)v_scale) & 3 || (uintptr_t)slots & 7)
    return fail(DP_EINVAL, "qk_norm_rope_append: positions, slots and scales must be aligned to their elements");
  if (q_out == q && sh->q_stride != (int64_t)sh->n_q_heads * kD)
    return fail(DP_EINVAL, "qk_norm_rope_append: q_out may be q only where q_stride is n_q_heads * 128");
  if (q_out == k || q_out == v) return fail(DP_EINVAL, "qk_norm_rope_append: q_out must not be k or v");
  if ((q_weight || k_weight) && !(eps >= 0.0f && std::isfinite(eps)))
    return fail(DP_EINVAL, "qk_norm_rope_append: eps must be finite and >= 0");

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
  if (sh->rows <= 256) launch<1, 1>(a, fp8, paired, st);
  else if (sh->rows < 4096) launch<2, 4>(a, fp8, paired, st);
  else launch<2, 16>(a, fp8, paired, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(DP_EIO, "qk_norm_rope_append: kernel launch failed: %s", hipGetErrorString(e));
  return DP_OK;
}

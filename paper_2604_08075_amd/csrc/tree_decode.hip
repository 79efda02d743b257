// Attention of drafted trees over the block-paged KV cache, for gfx950.
//
// For sequence s with T cached tokens, the last n of them drafted, query row
// i and head h (KV head g = h / G):
//     out = sum_t softmax_t(scale * q . K_t) V_t
// over the T - n committed tokens and the drafts whose bit is set in the
// row's mask.  K tiles are token-major, V tiles dims-major, as for decode.
//
// The (draft, head) pairs of a sequence and KV head form one list of columns,
// draft by draft; a workgroup takes the next 16 NC of them.  Its four waves
// take turns at the KV tiles (16 KiB: 32 tokens of bf16 or 64 of e4m3), each
// for all the columns:
//   * S^T = K Q^T with v_mfma_f32_16x16x32_bf16, K straight from memory in
//     operand layout.  The token behind each operand row is chosen so that a
//     lane's scores are the tokens that its operand of O^T += V^T P^T needs.
//   * online softmax in base 2 (scale * log2 e folded into one multiply-add);
//     the reference maximum of a column moves only when a score passes it by
//     2^kSlack, so the common path has no rescale.
//   * the denominator sums the rounded probabilities, so every output is a
//     convex combination of V rows.
// At the end the waves' sums meet in LDS under their common maximum.
//
// Masks: only tiles that reach past token T - n look at them.  There a value
// that is not finite must not leak into rows that do not see its token (0 times
// it is not 0), so V is made zero where it is not finite, and the few such
// values are added by hand to the columns that see them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <mutex>

#include "common.h"

namespace dpool_tree {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kD = 128;
constexpr int kBS = 16;
constexpr int kWaves = 4;
constexpr int kMaxBatch = 4096;
constexpr int kMaxWords = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;         // probabilities may reach 2^8 before the reference maximum moves
constexpr float kMinusBig = -3.0e38f;  // reference maximum of a column without a score (finite: no inf - inf)
constexpr int kPitch = kD + 4;         // floats of a column's sums in LDS

struct TreeArgs {
  const uint16_t* q;            // [total_q, Hq, 128] bf16
  const char* k;                // [num_blocks, Hkv, 16, 128]
  const char* v;                // [num_blocks, Hkv, 128, 16]
  const int32_t* block_tables;  // [B, max_blocks_per_seq]
  const int32_t* context_lens;  // [B]
  const int32_t* q_start;       // [B + 1]
  const uint32_t* mask;         // [total_q, 2 words]
  const float* k_scale;
  const float* v_scale;
  uint16_t* out;                // [total_q, Hq, 128] bf16
  float scale_log2;             // scale * log2(e)
  int32_t batch, hq, hkv, group, words;
  int32_t max_blocks, max_ctx, num_blocks_m1, total_q;
};

// Max over the four lanes li, li + 16, li + 32, li + 48
__device__ __forceinline__ float xor_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

__device__ __forceinline__ float xor_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

__device__ __forceinline__ uint16_t f32_to_bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

__device__ __forceinline__ int pack_bf16(float a, float b) {
  const bf16x2 p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(int, p);
}

__device__ __forceinline__ i32x4 fp8x8_to_bf16(int lo, int hi) {
  bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
  bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
  bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return i32x4{__builtin_bit_cast(int, a), __builtin_bit_cast(int, b), __builtin_bit_cast(int, c),
               __builtin_bit_cast(int, d)};
}

// What a tile needs to know of its sequence
struct Seq {
  int r0, n, T;
};

__device__ __forceinline__ Seq sequence(const TreeArgs& a, int s) {
  Seq q;
  q.r0 = min(max(a.q_start[s], 0), a.total_q);
  const int r1 = min(max(a.q_start[s + 1], q.r0), a.total_q);
  q.T = min(max(a.context_lens[s], 0), a.max_ctx);
  q.n = min(min(r1 - q.r0, q.T), 64 * a.words);
  return q;
}

template <bool FP8, int NC>
__global__ __launch_bounds__(kWaves * 64) void tree_kernel(TreeArgs a) {
  constexpr int COLS = 16 * NC;
  constexpr int KT = FP8 ? 64 : 32;   // tokens of a tile
  constexpr int KB = KT / kBS;        // blocks of a tile
  constexpr int M = KT / 16;          // row groups of a tile's scores
  constexpr size_t TB = FP8 ? 2048 : 4096;  // bytes of a (block, head) tile
  __shared__ float part[kWaves][COLS][kPitch];
  __shared__ float stat[kWaves][COLS][2];
  __shared__ uint32_t rows[COLS][2 * kMaxWords + 5];

  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int li = lane & 15, lj = lane >> 4;
  const int s = blockIdx.x, g = blockIdx.y, G = a.group;
  const Seq q = sequence(a, s);
  const int ncols = q.n * G, c0 = blockIdx.z * COLS;
  if (c0 >= ncols) return;
  const int pre = q.T - q.n;  // committed tokens
  const int nt = (q.T + KT - 1) / KT, nb = (q.T + kBS - 1) / kBS;
  const int32_t* const bt = a.block_tables + (size_t)s * a.max_blocks;

  float cmul = a.scale_log2, vsc = 1.0f;
  if constexpr (FP8) {
    cmul *= a.k_scale[g];
    vsc = a.v_scale[g];
  }
  // queries: chunk c of a column is 32 dimensions, eight of them this lane's
  // (e4m3: sixteen dimensions of two chunks lie together, as K's 16-byte loads have them)
  i32x4 qf[NC][4];
  int tok[NC];
#pragma unroll
  for (int b = 0; b < NC; ++b) {
    const int cc = min(c0 + 16 * b + li, ncols - 1);  // idle columns repeat the last one
    tok[b] = cc / G;
    const uint16_t* const p = a.q + ((size_t)(q.r0 + tok[b]) * a.hq + g * G + (cc - tok[b] * G)) * kD;
#pragma unroll
    for (int c = 0; c < 4; ++c)
      qf[b][c] = *(const i32x4*)(p + (FP8 ? 64 * (c >> 1) + 16 * lj + 8 * (c & 1) : 32 * c + 8 * lj));
  }

  // the rows' masks as a tile reads them: 64 set bits (committed tokens), the
  // drafts' bits, and clear ones past the last
  const int tok0 = c0 / G, n_rows = (min(c0 + COLS, ncols) - 1) / G - tok0 + 1;
  const int mw = 2 * a.words + 5;
  for (int i = tid; i < n_rows * mw; i += kWaves * 64) {
    const int r = i / mw, k = i - r * mw - 2;
    uint32_t x = k < 0 ? ~0u : 0u;
    if (k >= 0 && 32 * k < q.n) {
      x = a.mask[(size_t)(q.r0 + tok0 + r) * 2 * a.words + k];
      if (q.n < 32 * k + 32) x &= (1u << (q.n - 32 * k)) - 1;
    }
    rows[r][k + 2] = x;
  }
  __syncthreads();

  f32x4 acc[NC][8];
  float mc[NC], mlim[NC], lsum[NC];
#pragma unroll
  for (int b = 0; b < NC; ++b) {
    mc[b] = mlim[b] = kMinusBig;
    lsum[b] = 0.f;
#pragma unroll
    for (int nn = 0; nn < 8; ++nn) acc[b][nn] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  for (int j = w; j < nt; j += kWaves) {
    const int t0 = j * KT;
    // blocks of this lane's K and V values (past the sequence's end: its last block, masked below)
    const int kb = min(KB * j + (FP8 ? li >> 2 : li >> 3), nb - 1);
    const int vb = min(KB * j + (FP8 ? lj : lj >> 1), nb - 1);
    const size_t kt = (size_t)min(max(bt[kb], 0), a.num_blocks_m1) * a.hkv + g;
    const size_t vt = (size_t)min(max(bt[vb], 0), a.num_blocks_m1) * a.hkv + g;
    // K: operand row li of group m is token 8 (li / 4) + 4 m + li % 4 (e4m3: 16 (li / 4) + ...)
    const int krow = FP8 ? (li & 3) : 8 * ((li >> 2) & 1) + (li & 3);
    const char* const kp = a.k + kt * TB + (FP8 ? krow * 128 + 16 * lj : krow * 256 + 16 * lj);
    // V: operand row li of group nn is dimension 32 (nn / 2) + 8 (li / 4) + 4 (nn % 2) + li % 4
    const int vdim = 8 * (li >> 2) + (li & 3);
    const char* const vp = a.v + vt * TB + (FP8 ? vdim * 16 : vdim * 32 + 16 * (lj & 1));
    i32x4 kr[8], vr[8];
#pragma unroll
    for (int y = 0; y < 8; ++y)
      kr[y] = *(const i32x4*)(kp + (FP8 ? (y >> 1) * 512 + (y & 1) * 64 : (y >> 2) * 1024 + (y & 3) * 64));
#pragma unroll
    for (int y = 0; y < 8; ++y) vr[y] = *(const i32x4*)(vp + (32 * (y >> 1) + 4 * (y & 1)) * (FP8 ? 16 : 32));

    f32x4 z[NC][M];
#pragma unroll
    for (int b = 0; b < NC; ++b)
#pragma unroll
      for (int m = 0; m < M; ++m) z[b][m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        i32x4 kf;
        if constexpr (FP8) {
          const i32x4 x = kr[2 * m + (c >> 1)];
          kf = (c & 1) ? fp8x8_to_bf16(x[2], x[3]) : fp8x8_to_bf16(x[0], x[1]);
        } else {
          kf = kr[4 * m + c];
        }
#pragma unroll
        for (int b = 0; b < NC; ++b)
          z[b][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf),
                                                            __builtin_bit_cast(bf16x8, qf[b][c]), z[b][m], 0, 0, 0);
      }

    // this lane's tokens of the tile: t0 + 4 M lj + 4 m + e
    const int tl = t0 + 4 * M * lj;
    uint32_t odd = 0;  // this lane's tokens with a V value that is not finite
    uint32_t see[NC];
    const bool tail = t0 + KT > pre;
    if (tail) {
#pragma unroll
      for (int b = 0; b < NC; ++b) {
        const uint32_t* const mr = &rows[tok[b] - tok0][(tl - pre + 64) >> 5];
        const uint64_t two = (uint64_t)mr[1] << 32 | mr[0];
        see[b] = (uint32_t)(two >> ((tl - pre + 64) & 31)) & ((1u << (4 * M)) - 1);
#pragma unroll
        for (int x = 0; x < 4 * M; ++x)
          if (!((see[b] >> x) & 1)) z[b][x >> 2][x & 3] = -INFINITY;
      }
      // V: tokens past the end and values that are not finite become zero
#pragma unroll
      for (int y = 0; y < 8; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < (FP8 ? 4 : 2); ++h) {
            constexpr int BITS = FP8 ? 8 : 16;
            const uint32_t code = ((uint32_t)vr[y][e] >> (BITS * h)) & ((1u << BITS) - 1);
            const int x = (FP8 ? 4 : 2) * e + h;
            const bool inf = FP8 ? (code & 0x7f) == 0x7f : (code & 0x7f80) == 0x7f80;
            const bool in = tl + x < q.T;
            if (in && inf) odd |= 1u << x;
            if (!in || inf) vr[y][e] &= ~(int)(((1u << BITS) - 1) << (BITS * h));
          }
    }

    i32x4 p[NC][M / 2];
#pragma unroll
    for (int b = 0; b < NC; ++b) {
      float mx = z[b][0][0];
#pragma unroll
      for (int x = 1; x < 4 * M; ++x) mx = fmaxf(mx, z[b][x >> 2][x & 3]);
      if (__ballot(mx * cmul > mlim[b]) != 0) {
        const float m_new = fmaxf(mc[b], xor_max(mx) * cmul);
        if (m_new > mlim[b]) {
          const float alpha = __builtin_amdgcn_exp2f(mc[b] - m_new);
          mc[b] = m_new;
          mlim[b] = m_new + kSlack;
          lsum[b] *= alpha;
#pragma unroll
          for (int nn = 0; nn < 8; ++nn) acc[b][nn] *= alpha;
        }
      }
#pragma unroll
      for (int x = 0; x < 4 * M; x += 2) {
        float u = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][x >> 2][x & 3], cmul, -mc[b]));
        float v = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][x >> 2][(x & 3) + 1], cmul, -mc[b]));
        if (tail) {  // (a key scale of 0 makes -inf a NaN)
          if (!((see[b] >> x) & 1)) u = 0.f;
          if (!((see[b] >> (x + 1)) & 1)) v = 0.f;
        }
        const int r = pack_bf16(u, v);
        p[b][x >> 3][(x >> 1) & 3] = r;
        lsum[b] += __uint_as_float((uint32_t)r << 16) + __uint_as_float((uint32_t)r & 0xffff0000u);
      }
    }
#pragma unroll
    for (int nn = 0; nn < 8; ++nn)
#pragma unroll
      for (int h = 0; h < M / 2; ++h) {
        const i32x4 vf = FP8 ? fp8x8_to_bf16(vr[nn][2 * h], vr[nn][2 * h + 1]) : vr[nn];
#pragma unroll
        for (int b = 0; b < NC; ++b)
          acc[b][nn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, vf), __builtin_bit_cast(bf16x8, p[b][h]), acc[b][nn], 0, 0, 0);
      }

    // the values left out above, for the columns that see them
    if (tail) {
      for (int x = 0; x < KT; ++x) {
        const int src = x / (4 * M), bit = x % (4 * M);  // the row of lanes that holds token t0 + x
        const uint64_t who = __ballot(lj == src && ((odd >> bit) & 1));
        if (who == 0) continue;
        const int t = t0 + x;
        const size_t tile = ((size_t)min(max(bt[t / kBS], 0), a.num_blocks_m1) * a.hkv + g) * TB;
#pragma unroll
        for (int b = 0; b < NC; ++b) {
          // this column's probability of the token, from the lane that has it
          const uint32_t sees = __shfl(see[b], 16 * src + li);
          int pw = 0;
#pragma unroll
          for (int h = 0; h < M / 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (bit >> 1 == 4 * h + e) pw = p[b][h][e];
          pw = __shfl(pw, 16 * src + li);
          const float pr = (bit & 1) ? __uint_as_float((uint32_t)pw & 0xffff0000u)
                                     : __uint_as_float((uint32_t)pw << 16);
          if (!((sees >> bit) & 1)) continue;
#pragma unroll
          for (int nn = 0; nn < 8; ++nn)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int dim = 32 * (nn >> 1) + 8 * lj + 4 * (nn & 1) + e;
              float v;
              if constexpr (FP8) {
                const uint8_t c = *(const uint8_t*)(a.v + tile + dim * kBS + t % kBS);
                v = (c & 0x7f) == 0x7f ? NAN : 0.f;
              } else {
                const uint16_t c = *(const uint16_t*)(a.v + tile + (dim * kBS + t % kBS) * 2);
                v = (c & 0x7f80) == 0x7f80 ? __uint_as_float((uint32_t)c << 16) : 0.f;
              }
              if (v != 0.f) acc[b][nn][e] += pr * v;  // (true for NaN)
            }
        }
      }
    }
  }

  // fold the waves' sums
#pragma unroll
  for (int b = 0; b < NC; ++b) {
    const float l = xor_sum(lsum[b]);
    if (lj == 0) {
      stat[w][16 * b + li][0] = mc[b];
      stat[w][16 * b + li][1] = l;
    }
#pragma unroll
    for (int nn = 0; nn < 8; ++nn)
      *(f32x4*)&part[w][16 * b + li][32 * (nn >> 1) + 8 * lj + 4 * (nn & 1)] = acc[b][nn];
  }
  __syncthreads();
  for (int i = tid; i < COLS * 16; i += kWaves * 64) {
    const int col = i >> 4, d = (i & 15) * 8;
    if (c0 + col >= ncols) break;
    float m = stat[0][col][0];
#pragma unroll
    for (int k = 1; k < kWaves; ++k) m = fmaxf(m, stat[k][col][0]);
    float l = 0.f;
    f32x4 o0 = {0.f, 0.f, 0.f, 0.f}, o1 = o0;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
      const float f = __builtin_amdgcn_exp2f(stat[k][col][0] - m);
      l = __builtin_fmaf(stat[k][col][1], f, l);
      o0 += *(const f32x4*)&part[k][col][d] * f;
      o1 += *(const f32x4*)&part[k][col][d + 4] * f;
    }
    const float inv = l == 0.f ? 0.f : vsc / l;  // a row that sees no token: zeros
    const int cc = c0 + col, t = cc / G;
    const i32x4 o = {pack_bf16(o0[0] * inv, o0[1] * inv), pack_bf16(o0[2] * inv, o0[3] * inv),
                     pack_bf16(o1[0] * inv, o1[1] * inv), pack_bf16(o1[2] * inv, o1[3] * inv)};
    *(i32x4*)(a.out + ((size_t)(q.r0 + t) * a.hq + g * G + (cc - t * G)) * kD + d) = o;
  }
}

}  // namespace dpool_tree

using namespace dpool_tree;

namespace {

int check_shape(const dp_tree_shape* sh) {
  using dpool::fail;
  if (!sh) return fail(DP_EINVAL, "tree_decode_attention: null shape");
  if (sh->head_dim != kD) return fail(DP_ENOTSUP, "tree_decode_attention: head_dim %d (only 128)", sh->head_dim);
  if (sh->block_size != kBS) return fail(DP_ENOTSUP, "tree_decode_attention: block_size %d (only 16)", sh->block_size);
  if (sh->kv_dtype != DP_KV_BF16 && sh->kv_dtype != DP_KV_FP8_E4M3)
    return fail(DP_ENOTSUP, "tree_decode_attention: kv_dtype %d", sh->kv_dtype);
  if (sh->reserved != 0) return fail(DP_EINVAL, "tree_decode_attention: reserved must be 0");
  if (sh->batch < 0) return fail(DP_EINVAL, "tree_decode_attention: batch < 0");
  if (sh->batch > kMaxBatch) return fail(DP_ENOTSUP, "tree_decode_attention: batch above %d", kMaxBatch);
  if (sh->mask_words < 1 || sh->mask_words > kMaxWords)
    return fail(DP_ENOTSUP, "tree_decode_attention: mask_words %d (1 to %d)", sh->mask_words, kMaxWords);
  if (sh->n_kv_heads <= 0 || sh->n_q_heads <= 0 || sh->n_q_heads % sh->n_kv_heads != 0)
    return fail(DP_EINVAL, "tree_decode_attention: n_q_heads must be a positive multiple of n_kv_heads");
  if (sh->n_kv_heads > 65535 || sh->n_q_heads / sh->n_kv_heads > 1024)
    return fail(DP_ENOTSUP, "tree_decode_attention: n_kv_heads above 65535 or more than 1024 query heads to one");
  if (sh->max_blocks_per_seq <= 0 || sh->max_context_len < 0 ||
      (int64_t)sh->max_blocks_per_seq * kBS < sh->max_context_len || sh->num_blocks <= 0 ||
      sh->num_blocks > INT32_MAX)
    return fail(DP_EINVAL, "tree_decode_attention: need max_blocks_per_seq * 16 >= max_context_len and "
                           "0 < num_blocks <= INT32_MAX");
  if (sh->max_context_len > 1 << 30) return fail(DP_ENOTSUP, "tree_decode_attention: max_context_len above 2^30");
  if (sh->total_q < 0 || sh->total_q > INT32_MAX / 2)
    return fail(DP_EINVAL, "tree_decode_attention: total_q out of range");
  return DP_OK;
}

template <bool FP8>
void launch(const TreeArgs& a, int most, hipStream_t st) {
  const auto grid = [&](int cols) { return dim3(a.batch, a.hkv, (most + cols - 1) / cols); };
  if (most <= 16) hipLaunchKernelGGL((tree_kernel<FP8, 1>), grid(16), dim3(kWaves * 64), 0, st, a);
  else if (most <= 32) hipLaunchKernelGGL((tree_kernel<FP8, 2>), grid(32), dim3(kWaves * 64), 0, st, a);
  else hipLaunchKernelGGL((tree_kernel<FP8, 4>), grid(64), dim3(kWaves * 64), 0, st, a);
}

}  // namespace

extern "C" size_t tree_decode_workspace_size(const dp_tree_shape* sh) {
  if (check_shape(sh) != DP_OK) return 0;
  return 256;
}

extern "C" int tree_decode_attention(const void* q, const void* k_blocks, const void* v_blocks,
                                     const int32_t* block_tables, const int32_t* context_lens,
                                     const int32_t* q_start, const uint64_t* tree_mask, float scale,
                                     const float* k_scale, const float* v_scale, void* out, const dp_tree_shape* sh,
                                     void* workspace, size_t workspace_bytes, void* stream) {
  using dpool::fail;
  const int rc = check_shape(sh);
  if (rc != DP_OK) return rc;
  if (sh->batch == 0 || sh->total_q == 0) return DP_OK;
  if (!q || !k_blocks || !v_blocks || !block_tables || !context_lens || !q_start || !tree_mask || !out)
    return fail(DP_EINVAL, "tree_decode_attention: null tensor pointer");
  if (((uintptr_t)q | (uintptr_t)k_blocks | (uintptr_t)v_blocks | (uintptr_t)out) & 15)
    return fail(DP_EINVAL, "tree_decode_attention: q, k_blocks, v_blocks and out must be 16-byte aligned");
  if (((uintptr_t)block_tables | (uintptr_t)context_lens | (uintptr_t)q_start | (uintptr_t)k_scale |
       (uintptr_t)v_scale) & 3 || (uintptr_t)tree_mask & 7)
    return fail(DP_EINVAL, "tree_decode_attention: pointers must be aligned to their elements");
  const bool fp8 = sh->kv_dtype == DP_KV_FP8_E4M3;
  if (fp8 && (!k_scale || !v_scale))
    return fail(DP_EINVAL, "tree_decode_attention: e4m3 cache needs k_scale and v_scale");
  if (!fp8 && (k_scale || v_scale))
    return fail(DP_EINVAL, "tree_decode_attention: k_scale/v_scale must be NULL for a bf16 cache");
  if (!(scale > 0.0f) || !std::isfinite(scale))
    return fail(DP_EINVAL, "tree_decode_attention: scale must be finite and > 0");
  const size_t need = tree_decode_workspace_size(sh);
  if (!workspace || ((uintptr_t)workspace & 255))
    return fail(DP_EINVAL, "tree_decode_attention: workspace must be 256-byte aligned");
  if (workspace_bytes < need)
    return fail(DP_ENOMEM, "tree_decode_attention: workspace of %zu bytes, %zu needed", workspace_bytes, need);

  TreeArgs a;
  a.q = (const uint16_t*)q;
  a.k = (const char*)k_blocks;
  a.v = (const char*)v_blocks;
  a.block_tables = block_tables;
  a.context_lens = context_lens;
  a.q_start = q_start;
  a.mask = (const uint32_t*)tree_mask;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.out = (uint16_t*)out;
  a.scale_log2 = scale * kLog2e;
  a.batch = sh->batch;
  a.hq = sh->n_q_heads;
  a.hkv = sh->n_kv_heads;
  a.group = sh->n_q_heads / sh->n_kv_heads;
  a.words = sh->mask_words;
  a.max_blocks = sh->max_blocks_per_seq;
  a.max_ctx = sh->max_context_len;
  a.num_blocks_m1 = (int32_t)(sh->num_blocks - 1);
  a.total_q = (int32_t)sh->total_q;
  // columns of the longest possible tree
  const int most = (int)std::min<int64_t>(sh->total_q, 64 * sh->mask_words) * a.group;
  (void)hipGetLastError();
  if (fp8) launch<true>(a, most, (hipStream_t)stream);
  else launch<false>(a, most, (hipStream_t)stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(DP_EIO, "tree_decode_attention: kernel launch failed: %s", hipGetErrorString(e));
  return DP_OK;
}

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
constexpr int kMaxBatch = 4096;
constexpr int kMaxWords = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kSlack = 8.0f;         // probabilities may reach 2^8 before the reference maximum moves
constexpr float kMinusBig = -3.0e38f;  // reference maximum of a column without a score (finite: no inf - inf)
constexpr int kItemCost = 2;           // an item's start and end, in steps (for equal slices)
constexpr int kMinSlice = 4;           // steps of the smallest slice

// The item that a workgroup begins and does not finish
struct TreePiece {
  int32_t s, g, c0;
  int32_t last;  // the workgroup with its last piece; -1: none
};

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
  TreePiece* desc;              // [workgroups]
  float* stat;                  // [2 workgroups, columns, 2] reference maximum and sum
  float* part;                  // [2 workgroups, columns, 128]
};

// Max over the four lanes li, li + 16, li + 32, li + 48
__device__ __forceinline__ float xor_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}

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

// What an item needs to know of its sequence
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

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <bool FP8, int NW, int NC>
__global__ __launch_bounds__(NW * 64, 2) void tree_kernel(TreeArgs a) {
  constexpr int kThreads = NW * 64;
  constexpr int COLS = 16 * NC * NW;
  constexpr int SUB = FP8 ? 2 : 1;    // sub-tiles of 32 tokens in a step
  constexpr int KT = 32 * SUB;        // tokens of a step: 16 KiB of cache
  constexpr int KB = KT / kBS;        // blocks of a step
  constexpr int NP = 8 / NW;          // 16-byte pieces of K, and of V, a thread copies per step
  constexpr size_t TB = FP8 ? 2048 : 4096;  // bytes of a (block, head) tile
  struct Slot {
    char k[SUB][8192], v[SUB][8192];  // bf16: [32 tokens][128], [2 blocks][128 dims][16 tokens]
  };
  __shared__ __attribute__((aligned(16))) Slot slots[2];
  __shared__ uint32_t rows[COLS][2 * kMaxWords + 5];
  __shared__ uint64_t sums[NW];
  __shared__ uint64_t found_at;
  __shared__ int found;

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lj = lane >> 4;
  const int G = a.group;
  const int nwg = gridDim.x;
  // consecutive slices on one XCD (workgroups go to the eight in turn)
  const int wg = nwg % 8 == 0 ? (int)(blockIdx.x % 8) * (nwg / 8) + (int)(blockIdx.x / 8) : (int)blockIdx.x;

  // ---- this workgroup's slice of all units
  const auto item_units = [&](const Seq& q) { return (uint32_t)((q.T + KT - 1) / KT + kItemCost); };
  const auto items = [&](const Seq& q) { return (uint32_t)((q.n * G + COLS - 1) / COLS * a.hkv); };
  const int per_thread = (a.batch + kThreads - 1) / kThreads;
  const int s_lo = min(tid * per_thread, a.batch), s_hi = min(s_lo + per_thread, a.batch);
  uint64_t mine = 0;
  for (int s = s_lo; s < s_hi; ++s) {
    const Seq q = sequence(a, s);
    mine += (uint64_t)item_units(q) * items(q);
  }
  uint64_t upto = mine;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const uint64_t y = __shfl_up(upto, off);
    if (lane >= off) upto += y;
  }
  if (lane == 63) sums[w] = upto;
  if (tid == 0) found = -1;
  __syncthreads();
  uint64_t total = 0, before = 0;
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    if (k < w) before += sums[k];
    total += sums[k];
  }
  const uint64_t L = max((total + nwg - 1) / nwg, (uint64_t)kMinSlice);
  const uint64_t u_lo = wg * L, u_hi = min(u_lo + L, total);
  if (tid == 0) a.desc[wg].last = -1;
  upto += before;
  if (u_lo < u_hi && mine > 0 && upto - mine <= u_lo && u_lo < upto) {
    uint64_t at = upto - mine;
    for (int s = s_lo; s < s_hi; ++s) {
      const Seq q = sequence(a, s);
      const uint64_t u = (uint64_t)item_units(q) * items(q);
      if (u_lo < at + u) {
        found = s;
        found_at = at;
        break;
      }
      at += u;
    }
  }
  __syncthreads();
  if (u_lo >= u_hi) return;
  int s = __builtin_amdgcn_readfirstlane(found);
  uint64_t at = found_at;  // first unit of sequence s

  // ---- geometry of the copies: piece y = NP w + i of a step
  const int blk_w = w * KB / NW;  // the wave's pieces lie in one block
  int kdst[NP], vdst[NP];         // LDS; e4m3: the second half is 16 bytes on (K: exclusive or)
  uint32_t koff[NP], voff[NP];    // in the block's tile
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int y = NP * w + i;
    if constexpr (FP8) {
      const int tk = 8 * (y & 3) + (lane >> 3);
      const int f = (tk & 3) | (tk >> 3) << 2;
      kdst[i] = (y >> 2) * 8192 + tk * 256 + ((2 * (lane & 7)) ^ f) * 16;
      koff[i] = (8 * (y & 1) + (lane >> 3)) * 128 + (lane & 7) * 16;
      const int d = 64 * (y & 1) + lane;
      vdst[i] = (y >> 2) * 8192 + ((y >> 1) & 1) * 4096 + (d >> 5) * 1024 + ((2 * (d & 31)) ^ ((d >> 4) & 1) << 3) * 16;
      voff[i] = (y & 1) * 1024 + lane * 16;
    } else {
      const int tk = 4 * y + (lane >> 4);
      const int f = (tk & 3) | (tk >> 3) << 2;
      kdst[i] = tk * 256 + ((lane & 15) ^ f) * 16;
      koff[i] = (4 * (y & 3) + (lane >> 4)) * 256 + (lane & 15) * 16;
      vdst[i] = y * 1024 + (lane ^ ((lane >> 5) & 1) << 3) * 16;
      voff[i] = (y & 3) * 1024 + lane * 16;
    }
  }
  // LDS operand addresses.  K: row li of group m is token 8 (li / 4) + 4 m + li % 4, dims 32 c + 8 lj .. + 8;
  // V: row li of group nn is dim 32 (nn / 2) + 8 (li / 4) + 4 (nn % 2) + li % 4, tokens 8 lj .. + 8.
  int kro[4], vro[2];
#pragma unroll
  for (int c = 0; c < 4; ++c) kro[c] = (8 * (li >> 2) + (li & 3)) * 256 + ((4 * c + lj) ^ li) * 16;
#pragma unroll
  for (int h = 0; h < 2; ++h)
    vro[h] = (lj >> 1) * 4096 + (16 * (li >> 2) + 8 * (h ^ (li >> 3)) + 2 * (li & 3) + (lj & 1)) * 16;
  bf16x8 ones;
#pragma unroll
  for (int x = 0; x < 8; ++x) ones[x] = (__bf16)1.0f;

  // ---- the pieces of the slice
  uint64_t u = u_lo;
  for (; u < u_hi; ++s) {
    Seq q = sequence(a, s);
    q.r0 = __builtin_amdgcn_readfirstlane(q.r0);
    q.n = __builtin_amdgcn_readfirstlane(q.n);
    q.T = __builtin_amdgcn_readfirstlane(q.T);
    const uint32_t iu = item_units(q), ni = items(q);
    const uint64_t seq_end = at + (uint64_t)iu * ni;
    for (; u < u_hi && u < seq_end;) {
      const uint32_t it = (uint32_t)((u - at) / iu);
      const uint64_t it0 = at + (uint64_t)it * iu;                // the item's first unit
      const uint64_t piece_end = min(u_hi, it0 + iu);
      const int ncols = q.n * G, nct = (ncols + COLS - 1) / COLS;
      const int nt = (int)iu - kItemCost;
      const int j0 = max((int)(u - it0) - kItemCost, 0), j1 = max((int)(piece_end - it0) - kItemCost, 0);
      u = piece_end;
      if (j0 >= j1) continue;  // (the item's cost units hold no steps)
      const int g = (int)it / nct, c0 = ((int)it - g * nct) * COLS;
      const int pre = q.T - q.n;  // committed tokens
      const int nb = (q.T + kBS - 1) / kBS;
      const int32_t* const bt = a.block_tables + (size_t)s * a.max_blocks;
      const bool active = c0 + 16 * NC * w < ncols;  // this wave has columns

      // copies: two steps in registers, two in LDS
      struct Regs {
        i32x4 k[NP], v[NP];
      };
      Regs rA, rB;
      const auto block_of = [&](int j) __attribute__((always_inline)) {
        return bt[min(KB * min(j, j1 - 1) + blk_w, nb - 1)];
      };
      const auto load = [&](int id, Regs& r) __attribute__((always_inline)) {
        const size_t tile = ((size_t)min(max(__builtin_amdgcn_readfirstlane(id), 0), a.num_blocks_m1) * a.hkv + g) * TB;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          r.k[i] = *(const i32x4*)(a.k + tile + koff[i]);
          r.v[i] = *(const i32x4*)(a.v + tile + voff[i]);
        }
      };
      const auto store = [&](int j, Regs& r) __attribute__((always_inline)) {
        Slot& to = slots[j & 1];
        const int t0 = j * KT + blk_w * kBS;
        if (t0 + kBS > q.T) {  // V of tokens past the end may hold anything: zero
#pragma unroll
          for (int i = 0; i < NP; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              constexpr int N = FP8 ? 4 : 2, BITS = 32 / N;
              const int first = t0 + (FP8 ? 0 : 8 * (lane & 1)) + N * e;
              const int keep = min(max(q.T - first, 0), N);
              r.v[i][e] &= keep == N ? -1 : (1 << (BITS * keep)) - 1;
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if constexpr (FP8) {
            *(i32x4*)(to.k[0] + kdst[i]) = fp8x8_to_bf16(r.k[i][0], r.k[i][1]);
            *(i32x4*)(to.k[0] + (kdst[i] ^ 16)) = fp8x8_to_bf16(r.k[i][2], r.k[i][3]);
            *(i32x4*)(to.v[0] + vdst[i]) = fp8x8_to_bf16(r.v[i][0], r.v[i][1]);
            *(i32x4*)(to.v[0] + vdst[i] + 16) = fp8x8_to_bf16(r.v[i][2], r.v[i][3]);
          } else {
            *(i32x4*)(to.k[0] + kdst[i]) = r.k[i];
            *(i32x4*)(to.v[0] + vdst[i]) = r.v[i];
          }
        }
      };
      int id2;  // block of step j + 2 (in the loop: j + 3) for this wave
      {
        const int a0 = block_of(j0), a1 = block_of(j0 + 1);
        id2 = block_of(j0 + 2);
        load(a0, rA);
        load(a1, rB);
      }

      float cmul = a.scale_log2, vsc = 1.0f;
      if constexpr (FP8) {
        cmul *= a.k_scale[g];
        vsc = a.v_scale[g];
      }
      i32x4 qf[NC][4];
      int tok[NC];
      const auto column = [&](int b, int& t) __attribute__((always_inline)) {  // row (draft, head) of q and out
        const int cc = min(c0 + 16 * (NC * w + b) + li, ncols - 1);  // idle columns repeat the last one
        t = cc / G;
        return (size_t)(q.r0 + t) * a.hq + g * G + (cc - t * G);
      };
#pragma unroll
      for (int b = 0; b < NC; ++b) {
        const uint16_t* const p = a.q + column(b, tok[b]) * kD + 8 * lj;
#pragma unroll
        for (int c = 0; c < 4; ++c) qf[b][c] = *(const i32x4*)(p + 32 * c);
      }
      // the rows' masks as a tile reads them: 64 set bits (committed tokens),
      // the drafts' bits, and clear ones past the last
      const int tok0 = c0 / G, n_rows = (min(c0 + COLS, ncols) - 1) / G - tok0 + 1;
      const int mw = 2 * a.words + 5;
      if (j1 * KT > pre) {
        for (int i = tid; i < n_rows * mw; i += kThreads) {
          const int r = i / mw, k = i - r * mw - 2;
          uint32_t x = k < 0 ? ~0u : 0u;
          if (k >= 0 && 32 * k < q.n) {
            x = a.mask[(size_t)(q.r0 + tok0 + r) * 2 * a.words + k];
            if (q.n < 32 * k + 32) x &= (1u << (q.n - 32 * k)) - 1;
          }
          rows[r][k + 2] = x;
        }
      }

      f32x4 acc[NC][8], lsum[NC];
      float mc[NC], mlim[NC];
#pragma unroll
      for (int b = 0; b < NC; ++b) {
        mc[b] = mlim[b] = kMinusBig;
        lsum[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int nn = 0; nn < 8; ++nn) acc[b][nn] = f32x4{0.f, 0.f, 0.f, 0.f};
      }

      const auto compute = [&](int t0, const char* kt, const char* vt) __attribute__((always_inline)) {
        f32x4 z[NC][2];
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const i32x4 kf = *(const i32x4*)(kt + kro[c] + 1024 * m);
#pragma unroll
            for (int b = 0; b < NC; ++b)
              z[b][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[b][c]),
                  c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : z[b][m], 0, 0, 0);
          }
        i32x4 vf[8];
#pragma unroll
        for (int nn = 0; nn < 8; ++nn) vf[nn] = *(const i32x4*)(vt + vro[nn & 1] + 1024 * (nn >> 1));

        // this lane's tokens: t0 + 8 lj + 4 m + e
        const int tl = t0 + 8 * lj;
        const bool tail = t0 + 32 > pre;
        uint32_t odd = 0;  // this lane's tokens with a V value that is not finite
        uint32_t see[NC];
        if (tail) {
          const int bit = min(tl - pre + 64, 64 * a.words + 96);
#pragma unroll
          for (int b = 0; b < NC; ++b) {
            const uint32_t* const mr = &rows[tok[b] - tok0][bit >> 5];
            see[b] = (uint32_t)(((uint64_t)mr[1] << 32 | mr[0]) >> (bit & 31)) & 0xff;
#pragma unroll
            for (int x = 0; x < 8; ++x)
              if (!((see[b] >> x) & 1)) z[b][x >> 2][x & 3] = -INFINITY;
          }
#pragma unroll
          for (int nn = 0; nn < 8; ++nn)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = (uint32_t)vf[nn][e];
              const bool lo = (x & 0x7f80) == 0x7f80, hi = (x & 0x7f800000) == 0x7f800000;
              odd |= (lo ? 1u : 0u) << (2 * e) | (hi ? 2u : 0u) << (2 * e);
              vf[nn][e] = (int)(x & ((lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u)));
            }
        }
        i32x4 p[NC];
#pragma unroll
        for (int b = 0; b < NC; ++b) {
          float mx = z[b][0][0];
#pragma unroll
          for (int x = 1; x < 8; ++x) mx = fmaxf(mx, z[b][x >> 2][x & 3]);
          if (__builtin_amdgcn_ballot_w64(mx * cmul > mlim[b]) != 0) {
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
          for (int x = 0; x < 8; x += 2) {
            float lo = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][x >> 2][x & 3], cmul, -mc[b]));
            float hi = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][x >> 2][(x & 3) + 1], cmul, -mc[b]));
            if (tail) {  // (a key scale of 0 makes -inf a NaN)
              if (!((see[b] >> x) & 1)) lo = 0.f;
              if (!((see[b] >> (x + 1)) & 1)) hi = 0.f;
            }
            p[b][x >> 1] = pack_bf16(lo, hi);
          }
          lsum[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, p[b]), lsum[b], 0, 0, 0);
        }
#pragma unroll
        for (int nn = 0; nn < 8; ++nn)
#pragma unroll
          for (int b = 0; b < NC; ++b)
            acc[b][nn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8, vf[nn]), __builtin_bit_cast(bf16x8, p[b]), acc[b][nn], 0, 0, 0);

        // the values left out above, for the columns that see them
        if (tail && __builtin_amdgcn_ballot_w64(odd != 0) != 0) {
          for (int x = 0; x < 32; ++x) {
            const int src = x >> 3, bit = x & 7;  // the row of lanes that holds token t0 + x
            if (__ballot(lj == src && ((odd >> bit) & 1)) == 0) continue;
            const char* const col = vt + (x >> 4) * 4096;
#pragma unroll
            for (int b = 0; b < NC; ++b) {
              // this column's probability of the token, from the lane that has it
              const uint32_t sees = __shfl(see[b], 16 * src + li);
              int pw = 0;
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (bit >> 1 == e) pw = p[b][e];
              pw = __shfl(pw, 16 * src + li);
              const float pr = (bit & 1) ? __uint_as_float((uint32_t)pw & 0xffff0000u)
                                         : __uint_as_float((uint32_t)pw << 16);
#pragma unroll
              for (int nn = 0; nn < 8; ++nn)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const int d = 8 * lj + 4 * (nn & 1) + e;  // dim 32 (nn / 2) + d
                  const int piece = (2 * d + ((x >> 3) & 1)) ^ ((d >> 4) & 1) << 3;
                  const uint32_t c = *(const uint16_t*)(col + (nn >> 1) * 1024 + piece * 16 + (x & 7) * 2);
                  if (((sees >> bit) & 1) && (c & 0x7f80) == 0x7f80) acc[b][nn][e] += pr * __uint_as_float(c << 16);
                }
            }
          }
        }
      };

      const auto step = [&](int j, Regs& r) __attribute__((always_inline)) {
        // step j + 1 to LDS (its loads are two steps old), step j + 3 into the registers
        store(j + 1, r);
        const int id = id2;
        id2 = block_of(j + 4);
        load(id, r);
        if (active) {
          const Slot& sl = slots[j & 1];
#pragma unroll
          for (int x = 0; x < SUB; ++x) compute(j * KT + 32 * x, sl.k[x], sl.v[x]);
        }
        lds_barrier();
      };
      store(j0, rA);
      {
        const int id = id2;
        id2 = block_of(j0 + 3);
        load(id, rA);
      }
      lds_barrier();
      int j = j0;
      for (; j + 1 < j1; j += 2) {
        step(j, rB);
        step(j + 1, rA);
      }
      if (j < j1) step(j, rB);

      // ---- results: this lane holds dims 32 (nn / 2) + 8 lj + 4 (nn % 2) + e of its columns
      const bool whole = j0 == 0 && j1 == nt;
      const int slot = 2 * wg + (j0 == 0);
      if (!whole && j0 == 0 && tid == 0) {
        TreePiece d;
        d.s = s;
        d.g = g;
        d.c0 = c0;
        d.last = (int)((it0 + iu - 1) / L);
        a.desc[wg] = d;
      }
#pragma unroll
      for (int b = 0; b < NC; ++b) {
        const int cl = 16 * (NC * w + b) + li;
        if (c0 + cl >= ncols) continue;
        int t;
        const size_t row = column(b, t);
        if (whole) {
          const float l = lsum[b][0];
          const float inv = l == 0.f ? 0.f : vsc / l;  // a row that sees no token: zeros
#pragma unroll
          for (int nn = 0; nn < 8; nn += 2) {
            const f32x4 x = acc[b][nn] * inv, y = acc[b][nn + 1] * inv;
            const i32x4 o = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
            *(i32x4*)(a.out + row * kD + 16 * nn + 8 * lj) = o;
          }
        } else {
          const size_t rec = (size_t)slot * COLS + cl;
          if (lj == 0) {
            a.stat[2 * rec] = mc[b];
            a.stat[2 * rec + 1] = lsum[b][0];
          }
#pragma unroll
          for (int nn = 0; nn < 8; ++nn)
            *(f32x4*)(a.part + rec * kD + 32 * (nn >> 1) + 8 * lj + 4 * (nn & 1)) = acc[b][nn];
        }
      }
      // (the next piece's first writes to LDS follow the last step's barrier; its
      // masks are read only after its first barrier)
    }
    at = seq_end;
  }
}

// Joins the pieces of cut items: out = sum_p o_p 2^(m_p - M) / sum_p l_p 2^(m_p - M).
// One workgroup per 16 columns of one workgroup's unfinished item; sixteen lanes a column.
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int cols) {
  const int wg = blockIdx.x;
  const TreePiece d = a.desc[wg];
  if (d.last < 0) return;
  const int G = a.group;
  const Seq q = sequence(a, d.s);
  const int col = blockIdx.y * 16 + (threadIdx.x >> 4), dim = (threadIdx.x & 15) * 8;
  const int cc = d.c0 + col;
  if (cc >= q.n * G) return;
  const float vsc = a.v_scale ? a.v_scale[d.g] : 1.0f;
  float m = kMinusBig, l = 0.f;
  f32x4 o0 = {0.f, 0.f, 0.f, 0.f}, o1 = o0;
  for (int p = wg; p <= d.last; ++p) {
    const size_t rec = (size_t)(2 * p + (p == wg)) * cols + col;
    const float mp = a.stat[2 * rec], lp = a.stat[2 * rec + 1];
    const f32x4 x = *(const f32x4*)(a.part + rec * kD + dim), y = *(const f32x4*)(a.part + rec * kD + dim + 4);
    const float mn = fmaxf(m, mp);
    const float f = __builtin_amdgcn_exp2f(m - mn), fp = __builtin_amdgcn_exp2f(mp - mn);
    l = l * f + lp * fp;
    o0 = o0 * f + x * fp;
    o1 = o1 * f + y * fp;
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : vsc / l;
  o0 *= inv;
  o1 *= inv;
  const int t = cc / G;
  const i32x4 o = {pack_bf16(o0[0], o0[1]), pack_bf16(o0[2], o0[3]), pack_bf16(o1[0], o1[1]), pack_bf16(o1[2], o1[3])};
  *(i32x4*)(a.out + ((size_t)(q.r0 + t) * a.hq + d.g * G + (cc - t * G)) * kD + dim) = o;
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

// Compute units of the current device (cached per device); 256 without one.
int compute_units() {
  static std::mutex mu;
  static int cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
    (void)hipGetLastError();
    return 256;
  }
  std::lock_guard<std::mutex> lock(mu);
  if (!cached[dev]) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) {
      (void)hipGetLastError();
      n = 256;
    }
    cached[dev] = n;
  }
  return cached[dev];
}

// Which kernel a call takes, and its workspace
struct Plan {
  int waves, blocks;  // of a workgroup; 16-column blocks of a wave
  int workgroups;
  int cols() const { return 16 * waves * blocks; }
  size_t stat_at() const { return ((size_t)workgroups * sizeof(TreePiece) + 255) & ~(size_t)255; }
  size_t part_at() const { return stat_at() + (((size_t)workgroups * 4 * cols() * sizeof(float) + 255) & ~(size_t)255); }
  size_t bytes() const { return part_at() + (size_t)workgroups * 2 * cols() * kD * sizeof(float); }
};

Plan plan(const dp_tree_shape* sh) {
  const int64_t group = sh->n_q_heads / sh->n_kv_heads;
  const int64_t most = std::min<int64_t>(sh->total_q, 64 * sh->mask_words) * group;  // columns of the largest tree
  const int cus = compute_units();
  if (most <= 64) return Plan{4, 1, 2 * cus};
  if (most <= 128) return Plan{4, 2, 2 * cus};
  return Plan{8, 2, cus};
}

template <int NW, int NC>
void launch(const TreeArgs& a, bool fp8, int workgroups, hipStream_t st) {
  if (fp8) hipLaunchKernelGGL((tree_kernel<true, NW, NC>), dim3(workgroups), dim3(NW * 64), 0, st, a);
  else hipLaunchKernelGGL((tree_kernel<false, NW, NC>), dim3(workgroups), dim3(NW * 64), 0, st, a);
}

}  // namespace

extern "C" size_t tree_decode_workspace_size(const dp_tree_shape* sh) {
  if (check_shape(sh) != DP_OK) return 0;
  return plan(sh).bytes();
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
  const Plan pl = plan(sh);
  const size_t need = pl.bytes();
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
  a.desc = (TreePiece*)workspace;
  a.stat = (float*)((char*)workspace + pl.stat_at());
  a.part = (float*)((char*)workspace + pl.part_at());
  (void)hipGetLastError();
  hipStream_t st = (hipStream_t)stream;
  if (pl.waves == 8) launch<8, 2>(a, fp8, pl.workgroups, st);
  else if (pl.blocks == 2) launch<4, 2>(a, fp8, pl.workgroups, st);
  else launch<4, 1>(a, fp8, pl.workgroups, st);
  hipLaunchKernelGGL(tree_merge_kernel, dim3(pl.workgroups, pl.cols() / 16), dim3(256), 0, st, a, pl.cols());
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(DP_EIO, "tree_decode_attention: kernel launch failed: %s", hipGetErrorString(e));
  return DP_OK;
}

// Attention of drafted trees over the block-paged KV cache, for gfx950.
//
// For sequence s with T cached tokens, the last n of them drafted, query row
// i and head h (KV head g = h / G):
//     out = sum_t softmax_t(scale * q . K_t) V_t
// over the T - n committed tokens and the drafts whose bit is set in the
// row's mask.  K tiles are token-major, V tiles dims-major, as for decode.
//
// The (draft, head) pairs of a sequence and KV head form one list of columns,
// draft by draft, and an item is the next 64, 128 or 256 of them: the waves of
// a workgroup share K and V of a tile (16 KiB: 32 tokens of bf16, 64 of e4m3)
// through LDS, 16 or 32 columns each.  Per tile and wave:
//   * S^T = K Q^T with v_mfma_f32_16x16x32_bf16.  The token behind each operand
//     row is chosen so that a lane's scores are the tokens that its operand of
//     O^T += V^T P^T needs: probabilities never move between lanes.
//   * online softmax in base 2 (scale * log2 e folded into one multiply-add);
//     the reference maximum of a column moves only when a score passes it by
//     2^kSlack, so the common path has no rescale.
//   * probabilities are rounded to bf16, the operand's type; the denominator is
//     a product against ones that sums the rounded ones, so that every output
//     is a convex combination of V rows.  All sums are fp32.  That rounding
//     makes the error against 64 bits 2.3e-3 of the norm where rounding the
//     result alone makes 1.7e-3.  A second product with what it takes away gave
//     1.7e-3 and cost 1.5% of the time with 64 columns (181 us -> 183.5), 31%
//     with 256 (424 -> 556) and 33% in e4m3 with 128 (141 -> 188), so it is not
//     made; fp16 holds neither all of V nor the small probabilities of long contexts.
// All tiles of all items are cut into one slice of equal cost per workgroup; an
// item that a cut goes through leaves sums (maximum, denominator, o) that a
// second kernel joins, in order, so results do not depend on timing.
//
// What bounds it, measured on one MI355X (a large read reaches 6.6 TB/s, a
// large bf16 product 1,212 TFLOP/s): 64 columns (eight drafts, GQA 8) memory:
// sixteen contexts of 32,768 tokens, bf16, 411 us, 5.2 TB/s.  The short pool's
// 128 ragged contexts 181 us: 1.4 us a tile and workgroup, 6 us for every end
// of an item, 8 us before the first tile and 13 for the join and its launch.
// 256 columns: neither alone; the matrix cores are busy a third of the time (32
// drafts on sixteen contexts of 65,536 tokens: 1,294 us, 850 TFLOP/s; e4m3,
// sixteen drafts, GQA 16: 977).  Scores, softmax and output products of a tile
// follow each other, and each of K's operands is waited for as it is read from
// LDS (V's eight are read together).  Variants with four tiles on their way, and
// with three tiles' steps interleaved by hand, were within 4% and not kept; they
// read K the same way, so they show no bound.  The 128-column variants spill four
// (bf16) and six (e4m3) registers, stored and loaded at the ends of a piece.
//
// LDS: K's sixteen 16-byte chunks of a token are stored exclusive-or'ed with
// (token % 4, token / 8 % 4), V's with bit 4 of the dimension, so that the
// sixteen lanes one pass of a 16-byte read serves start in distinct banks
// (counted: no conflict cycles in bf16).  e4m3's widened stores go to every
// other 16 bytes, 30% more LDS cycles; half of the lanes in the other order took
// these away and no time (155 us both).
//
// Masks: only tiles that reach past token T - n look at them.  There a value
// of V that is not finite must not leak into rows that do not see its token (0
// times it is not 0): it is made 0 on its way to LDS, and added to the rows
// that see it when they are written.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <mutex>
#include <type_traits>

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
// An item's start and end, in tiles, for equal slices (short pool, us, with 1 / 4 / 16:
// bf16 198 / 186 / 191, e4m3 173 / 153 / 194), and tiles of the smallest slice (three
// contexts of up to 512 tokens, 1 / 4 / 16: 16.3 / 13.6 / 19.5).
constexpr int kItemCost = 4;
constexpr int kMinSlice = 4;

// The item that a workgroup begins and does not finish
struct TreePiece {
  int32_t last;  // the workgroup with its last piece; -1: none
  int32_t s, g, c0, r0, n, T;
  int32_t unused;
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
  float* stat;                  // [2 workgroups, columns, 4] reference maximum, sum, odd
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

// A value that is the same in every lane, in a scalar register
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)x);
}

// Lengths and block tables do not change during a launch: read as constants,
// an entry that the whole wave needs comes through the scalar cache, whose
// loads are counted apart from those of K and V (which return in order: a
// block id among them would hold up every tile behind it).
typedef const __attribute__((address_space(4))) int32_t* ConstInts;
__device__ __forceinline__ ConstInts constants(const int32_t* p) { return (ConstInts)(uintptr_t)p; }

// What an item needs to know of its sequence
struct Seq {
  int r0, n, T;
  int r1;  // the first row of the next sequence
};

// Sequence s, whose rows start at r0, where those of the sequence before end:
// offsets out of order count as the largest so far, so that no row has two
// sequences, whose workgroups would both write it.
__device__ __forceinline__ Seq sequence(const TreeArgs& a, int s, int r0) {
  Seq q;
  q.r0 = r0;
  q.r1 = min(max(constants(a.q_start)[s + 1], r0), a.total_q);
  q.T = min(max(constants(a.context_lens)[s], 0), a.max_ctx);
  q.n = min(min(q.r1 - r0, q.T), 64 * a.words);
  return q;
}

__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// ---- equal slices of all the work
//
// An item is COLS columns of a sequence and KV head; it costs its KV tiles
// and kItemCost more for its start and end.  All items in order (sequence, KV
// head, columns) are cut into one slice of equal cost per workgroup; a piece
// is what a slice holds of an item.

// A piece: tiles j0 .. j1 of nt
struct Piece {
  int s, g, c0, j0, j1, nt;
  Seq q;
  int last;  // the workgroup with the item's last piece
};

template <int COLS, int KT>
struct Walk {
  const TreeArgs& a;
  uint64_t u, u_hi, at, slice;  // next unit, end of the slice, first unit of sequence s
  int s, row, wg;               // row: the first of sequence s

  __device__ __forceinline__ uint32_t units(const Seq& q) const { return (uint32_t)((q.T + KT - 1) / KT + kItemCost); }
  __device__ __forceinline__ uint32_t items(const Seq& q) const {
    return (uint32_t)((q.n * a.group + COLS - 1) / COLS * a.hkv);
  }

  // Finds this workgroup's slice; every thread of the workgroup takes part.
  // Each scans a few sequences; the one that has the slice's first unit says so.
  template <int kThreads>
  __device__ __forceinline__ void begin() {
    __shared__ uint64_t sums[kThreads / 64];
    __shared__ int mixed[kThreads / 64];
    __shared__ uint64_t found_at;
    __shared__ int found, found_row;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, nwg = gridDim.x;
    // consecutive slices on one XCD (workgroups go to the eight in turn)
    wg = nwg % 8 == 0 ? (int)(blockIdx.x % 8) * (nwg / 8) + (int)(blockIdx.x / 8) : (int)blockIdx.x;
    const int per_thread = (a.batch + kThreads - 1) / kThreads;
    const int s_lo = min(tid * per_thread, a.batch), s_hi = min(s_lo + per_thread, a.batch);
    const ConstInts start = constants(a.q_start);
    int row_lo = min(max(start[s_lo], 0), a.total_q);
    uint64_t mine, upto;
    for (bool again = false;; again = true) {
      mine = 0;
      int r = row_lo;
      bool disorder = false;
      for (int i = s_lo; i < s_hi; ++i) {
        const Seq q = sequence(a, i, r);
        mine += (uint64_t)units(q) * items(q);
        disorder |= start[i] > start[i + 1];
        r = q.r1;
      }
      upto = mine;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const uint64_t y = __shfl_up(upto, off);
        if (lane >= off) upto += y;
      }
      const bool any = __builtin_amdgcn_ballot_w64(disorder) != 0;
      if (lane == 63) {
        sums[w] = upto;
        mixed[w] = any;
      }
      __syncthreads();
      bool all_mixed = false;
#pragma unroll
      for (int k = 0; k < kThreads / 64; ++k) all_mixed |= mixed[k] != 0;
      if (again || !all_mixed) break;
      // offsets out of order, a broken promise: the largest so far, slowly
      int most = 0;
      for (int i = 0; i <= s_lo; ++i) most = max(most, start[i]);
      row_lo = min(most, a.total_q);
      __syncthreads();  // (sums and mixed are written again)
    }
    uint64_t total = 0, before = 0;
#pragma unroll
    for (int k = 0; k < kThreads / 64; ++k) {
      if (k < w) before += sums[k];
      total += sums[k];
    }
    slice = uniform(max((total + nwg - 1) / nwg, (uint64_t)kMinSlice));
    u = uniform(min(wg * slice, total));
    u_hi = uniform(min(u + slice, total));
    upto += before;
    if (u < u_hi && mine > 0 && upto - mine <= u && u < upto) {
      uint64_t x = upto - mine;
      int r = row_lo;
      for (int i = s_lo; i < s_hi; ++i) {
        const Seq q = sequence(a, i, r);
        const uint64_t y = (uint64_t)units(q) * items(q);
        if (u < x + y) {
          found = i;
          found_at = x;
          found_row = r;
          break;
        }
        x += y;
        r = q.r1;
      }
    }
    __syncthreads();
    if (u < u_hi) {
      s = uniform(found);
      at = uniform(found_at);
      row = uniform(found_row);
    }
  }

  // The next piece of the slice that holds a tile; false: there is none.
  __device__ __forceinline__ bool next(Piece& p) {
    while (u < u_hi) {
      const Seq q = sequence(a, s, row);
      const uint32_t iu = units(q);
      const uint64_t end = at + (uint64_t)iu * items(q);
      if (u >= end) {
        at = end;
        row = q.r1;
        ++s;
        continue;
      }
      const uint32_t it = (uint32_t)((u - at) / iu);
      const uint64_t it0 = at + (uint64_t)it * iu;
      const uint64_t stop = min(u_hi, it0 + iu);
      p.j0 = max((int)(u - it0) - kItemCost, 0);
      p.j1 = max((int)(stop - it0) - kItemCost, 0);
      u = stop;
      if (p.j0 >= p.j1) continue;  // nothing but the item's cost
      const int nct = (q.n * a.group + COLS - 1) / COLS;
      p.s = s;
      p.g = (int)it / nct;
      p.c0 = ((int)it - p.g * nct) * COLS;
      p.nt = (int)iu - kItemCost;
      p.q = q;
      p.last = (int)((it0 + iu - 1) / slice);
      return true;
    }
    return false;
  }
};

// The masks of a piece's rows as tiles read them: 64 set bits (committed
// tokens), the drafts' bits, and clear ones past the last.
constexpr int kMaskWords = 2 * kMaxWords + 5;
template <int COLS>
struct Masks {
  int words, count;  // words of a row; of all rows
  __device__ __forceinline__ Masks(const TreeArgs& a, const Piece& p) {
    const int tok0 = p.c0 / a.group, n_rows = (min(p.c0 + COLS, p.q.n * a.group) - 1) / a.group - tok0 + 1;
    words = 2 * a.words + 5;
    count = n_rows * words;
  }
  __device__ __forceinline__ uint32_t value(const TreeArgs& a, const Piece& p, int i) const {
    const int r = i / words, k = i - r * words - 2;
    if (k < 0) return ~0u;
    if (32 * k >= p.q.n) return 0;
    const uint32_t x = a.mask[(size_t)(p.q.r0 + p.c0 / a.group + r) * 2 * a.words + k];
    return p.q.n < 32 * k + 32 ? x & ((1u << (p.q.n - 32 * k)) - 1) : x;
  }
};

// ---- one wave's columns
template <int NC>
struct Columns {
  i32x4 qf[NC][4];
  int tok[NC];  // draft of this lane's column, from the piece's first
  f32x4 acc[NC][8], lsum[NC];
  float mc[NC], mlim[NC];

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int b = 0; b < NC; ++b) {
      mc[b] = mlim[b] = kMinusBig;
      lsum[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int nn = 0; nn < 8; ++nn) acc[b][nn] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }

  // Queries of columns first + 16 b + li (idle ones repeat the last).
  __device__ __forceinline__ void load_q(const TreeArgs& a, const Piece& p, int first) {
    const int li = threadIdx.x & 15, lj = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int b = 0; b < NC; ++b) {
      const int cc = min(first + 16 * b + li, p.q.n * a.group - 1), t = cc / a.group;
      tok[b] = t - p.c0 / a.group;
      const uint16_t* const x = a.q + ((size_t)(p.q.r0 + t) * a.hq + p.g * a.group + (cc - t * a.group)) * kD;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        qf[b][c] = *(const i32x4*)(x + 32 * c + 8 * lj);
    }
  }

  // 32 tokens.  kfrag(m, c), vfrag(nn): operands; this lane's tokens are tl .. tl + 8, eight of them for each lj.
  // tail: some may be drafts or lie past the end.
  template <class K, class V>
  __device__ __forceinline__ void attend(const K& kfrag, const V& vfrag, int tl, bool tail, int pre, float cmul, int words,
                                         const uint32_t (*rows)[kMaskWords]) {
    f32x4 z[NC][2];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const i32x4 kf = kfrag(m, c);
#pragma unroll
        for (int b = 0; b < NC; ++b)
          z[b][m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[b][c]),
              c == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : z[b][m], 0, 0, 0);
      }
    __builtin_amdgcn_sched_barrier(0);  // (K's operands are done with before V's are read)
    i32x4 vf[8];
#pragma unroll
    for (int nn = 0; nn < 8; ++nn) vf[nn] = vfrag(nn);

    if (tail) {
      const int bit = min(tl - pre + 64, 64 * words + 96);
#pragma unroll
      for (int b = 0; b < NC; ++b) {
        const uint32_t* const mr = &rows[tok[b]][bit >> 5];
        const uint32_t see = (uint32_t)(((uint64_t)mr[1] << 32 | mr[0]) >> (bit & 31));
#pragma unroll
        for (int x = 0; x < 8; ++x)
          if (!((see >> x) & 1)) z[b][x >> 2][x & 3] = -INFINITY;
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
        const float lo = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][x >> 2][x & 3], cmul, -mc[b]));
        const float hi = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][x >> 2][(x & 3) + 1], cmul, -mc[b]));
        p[b][x >> 1] = pack_bf16(lo, hi);
      }
      bf16x8 ones;
#pragma unroll
      for (int x = 0; x < 8; ++x) ones[x] = (__bf16)1.0f;
      lsum[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, p[b]), lsum[b], 0, 0, 0);
    }
#pragma unroll
    for (int nn = 0; nn < 8; ++nn)
#pragma unroll
      for (int b = 0; b < NC; ++b)
        acc[b][nn] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, vf[nn]), __builtin_bit_cast(bf16x8, p[b]), acc[b][nn], 0, 0, 0);
  }
};

// Eight dimensions of a column.  `odd`: among the tiles that hold drafts is a V
// value that is not finite; the sums left such values out, and here they join
// the rows that see them (their probabilities are not 0, so a NaN or an
// infinity is what they come to).
template <bool FP8>
__device__ __forceinline__ void store_out(const TreeArgs& a, int s, int g, const Seq& q, int cc, int dim, f32x4 x, f32x4 y,
                                          bool odd) {
  constexpr size_t TB = FP8 ? 2048 : 4096;
  const int t = cc / a.group;
  if (odd) {
    const int32_t* const bt = a.block_tables + (size_t)s * a.max_blocks;
    constexpr int KT = FP8 ? 64 : 32;
    const int pre = q.T - q.n;
    for (int tk = pre / KT * KT; tk < q.T; ++tk) {  // from the first tile that holds a draft
      const int j = tk - pre;
      if (j >= 0 && !((a.mask[(size_t)(q.r0 + t) * 2 * a.words + (j >> 5)] >> (j & 31)) & 1)) continue;
      const char* const v = a.v + ((size_t)min(max(bt[tk / kBS], 0), a.num_blocks_m1) * a.hkv + g) * TB;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int i = (dim + e) * kBS + tk % kBS;
        float f;
        if constexpr (FP8) f = (((const uint8_t*)v)[i] & 0x7f) == 0x7f ? NAN : 0.f;
        else f = __uint_as_float((uint32_t)((const uint16_t*)v)[i] << 16);
        if (!((__float_as_uint(f) & 0x7f800000) == 0x7f800000)) continue;
        if (e < 4) x[e] += f;
        else y[e - 4] += f;
      }
    }
  }
  const i32x4 o = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
  *(i32x4*)(a.out + ((size_t)(q.r0 + t) * a.hq + g * a.group + (cc - t * a.group)) * kD + dim) = o;
}

// The record that the join of a cut item starts from
__device__ __forceinline__ void note_start(const TreeArgs& a, const Piece& p, int wg) {
  TreePiece d;
  d.last = p.last;
  d.s = p.s;
  d.g = p.g;
  d.c0 = p.c0;
  d.r0 = p.q.r0;
  d.n = p.q.n;
  d.T = p.q.T;
  d.unused = 0;
  a.desc[wg] = d;
}

// ---- NW waves of 16 NC columns share every tile through LDS
template <bool FP8, int NW, int NC>
__global__ __launch_bounds__(NW * 64, 2) void tree_kernel(TreeArgs a) {
  constexpr int kThreads = NW * 64;
  constexpr int WCOLS = 16 * NC, COLS = WCOLS * NW;
  constexpr int SUB = FP8 ? 2 : 1;    // 32-token parts of a tile
  constexpr int KT = 32 * SUB;        // tokens of a tile: 16 KiB of cache
  constexpr int KB = KT / kBS;        // blocks of a tile
  constexpr int NP = 8 / NW;          // 16-byte pieces of K, and of V, a thread copies per tile
  constexpr size_t TB = FP8 ? 2048 : 4096;  // bytes of a (block, head) tile
  struct Slot {
    char k[SUB][8192], v[SUB][8192];  // bf16: [32 tokens][128], [2 blocks][128 dims][16 tokens]
  };
  __shared__ __attribute__((aligned(16))) Slot slots[2];
  __shared__ uint32_t rows[COLS][kMaskWords];
  __shared__ int odd[2];  // 1: a tile with drafts had a V value that is not finite (two pieces in turn)

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int li = lane & 15, lj = lane >> 4;
  if (tid < 2) odd[tid] = 0;
  Walk<COLS, KT> walk{a};
  walk.template begin<kThreads>();
  if (tid == 0) a.desc[walk.wg].last = -1;

  // geometry of the copies: piece y = NP w + i of a tile
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

  // copies: two tiles in registers, two in LDS
  struct Regs {
    i32x4 k[NP], v[NP];
  };
  Regs rA, rB;
  const auto block_of = [&](const Piece& p, int j) __attribute__((always_inline)) {
    const ConstInts bt = constants(a.block_tables) + (size_t)p.s * a.max_blocks;
    return bt[min(KB * min(j, p.j1 - 1) + blk_w, (p.q.T + kBS - 1) / kBS - 1)];
  };
  const auto load = [&](int id, int g, Regs& x) __attribute__((always_inline)) {
    const size_t tile = ((size_t)min(max(id, 0), a.num_blocks_m1) * a.hkv + g) * TB;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      x.k[i] = *(const i32x4*)(a.k + tile + koff[i]);
      x.v[i] = *(const i32x4*)(a.v + tile + voff[i]);
    }
  };
  // V of drafts that is not finite: 0 times it is not 0, and rows that do not
  // see it must not get it, so it becomes 0 here (store_out() adds it again
  // where it is seen).  V of slots past the end may hold anything: 0 too.
  const auto clean = [&](const Seq& q, int j, Regs& x, int turn) __attribute__((always_inline)) {
    constexpr int N = FP8 ? 4 : 2, BITS = 32 / N;  // values of a word
    constexpr uint32_t EXP = FP8 ? 0x7f : 0x7f80;  // (e4m3 has no infinities: 0x7f and 0xff are NaN)
    bool any = false;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int left = min(max(q.T - (j * KT + blk_w * kBS + (FP8 ? 0 : 8 * (lane & 1)) + N * e), 0), N);
        const uint32_t y = (uint32_t)x.v[i][e] & (left == N ? ~0u : (1u << (BITS * left)) - 1);
        uint32_t keep = 0;
#pragma unroll
        for (int h = 0; h < N; ++h)
          if (((y >> (BITS * h)) & EXP) != EXP) keep |= ((1u << BITS) - 1) << (BITS * h);
        any |= keep != ~0u;
        x.v[i][e] = (int)(y & keep);
      }
    if (any) odd[turn] = 1;
  };
  const auto store = [&](int slot, const Regs& x) __attribute__((always_inline)) {
    Slot& to = slots[slot];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      if constexpr (FP8) {
        *(i32x4*)(to.k[0] + kdst[i]) = fp8x8_to_bf16(x.k[i][0], x.k[i][1]);
        *(i32x4*)(to.k[0] + (kdst[i] ^ 16)) = fp8x8_to_bf16(x.k[i][2], x.k[i][3]);
        *(i32x4*)(to.v[0] + vdst[i]) = fp8x8_to_bf16(x.v[i][0], x.v[i][1]);
        *(i32x4*)(to.v[0] + vdst[i] + 16) = fp8x8_to_bf16(x.v[i][2], x.v[i][3]);
      } else {
        *(i32x4*)(to.k[0] + kdst[i]) = x.k[i];
        *(i32x4*)(to.v[0] + vdst[i]) = x.v[i];
      }
    }
  };

  // The tiles of all pieces form one stream: while tile i is in work, tile i + 1
  // goes to LDS and tile i + 3 is asked for, whichever piece they belong to.
  Piece p, nxt;                  // the piece in work, and the next
  bool more = walk.next(nxt);    // there is a next
  if (!more) return;
  // This wave's blocks of 64 tiles, one a lane, loaded far ahead: loads come
  // back in order, and scalar ones would be waited for with every LDS read.
  constexpr int kChunk = 56;
  int ids, later, first = block_of(nxt, nxt.j0 + lane);  // of tiles base and up, base + kChunk and up; of nxt
  const auto id_at = [&](int v, int i) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(v, i); };
  int j, base, end, turn = 1;  // end: tile j1, or one more, so that pieces start in the same registers
  float cmul, vsc;
  bool active;  // this wave has columns
  Columns<NC> st;

  // The next piece becomes the one in work: its first tile in slot 0, the next
  // two on their way in rB and rA (there already if `linked`).
  const auto enter = [&](bool linked) __attribute__((always_inline)) {
    p = nxt;
    turn ^= 1;
    j = base = p.j0;
    end = p.j0 + (p.j1 - p.j0 + 1) / 2 * 2;
    ids = first;
    if (!linked) {
      load(id_at(ids, 0), p.g, rA);
      load(id_at(ids, 1), p.g, rB);
    }
    st.load_q(a, p, p.c0 + WCOLS * w);
    active = p.c0 + WCOLS * w < p.q.n * a.group;
    later = block_of(p, base + kChunk + lane);
    const Masks<COLS> masks(a, p);
    const uint32_t mask0 = tid < masks.count ? masks.value(a, p, tid) : 0;
    cmul = a.scale_log2;
    vsc = 1.0f;
    if constexpr (FP8) {
      cmul *= a.k_scale[p.g];
      if (cmul == 0.f) cmul = 1e-37f;  // (0 times the -inf of a hidden token is not -inf)
      vsc = a.v_scale[p.g];
    }
    // the next piece is looked up while all that is on its way
    more = walk.next(nxt);
    if (more) first = block_of(nxt, nxt.j0 + lane);
    if (tid < masks.count) rows[tid / masks.words][tid % masks.words] = mask0;
    for (int i = tid + kThreads; i < masks.count; i += kThreads) rows[i / masks.words][i % masks.words] = masks.value(a, p, i);
    st.clear();
    if (!linked) {
      if (p.j0 >= (p.q.T - p.q.n) / KT) clean(p.q, p.j0, rA, turn);
      store(0, rA);
      load(id_at(ids, 2), p.g, rA);
    }
    // Block ids are waited for here, once (the masks' loads behind them were
    // already): else the compiler would wait for all loads in every step.
    __builtin_amdgcn_s_waitcnt(0xf70);  // vmcnt(0)
    if constexpr (FP8) {
      // A scale below 0: the queries change sign instead (-inf hides a token, the largest score leads).
      // A NaN: the queries become NaN instead (the scale would make one of a hidden token's -inf).
      if (!(cmul > 0.f)) {
        const bool nan = cmul != cmul;
        const int flip = nan ? 0 : (int)0x80008000, fill = nan ? 0x7fff7fff : 0;
        cmul = nan ? 1.f : -cmul;
#pragma unroll
        for (int b = 0; b < NC; ++b)
#pragma unroll
          for (int c = 0; c < 4; ++c) st.qf[b][c] = (st.qf[b][c] ^ flip) | fill;
      }
    }
    lds_barrier();
    if (tid == 0) odd[turn ^ 1] = 0;  // (every wave has left the piece before)
  };
  const auto step = [&](int slot, Regs& x) __attribute__((always_inline)) {
    const int pre = p.q.T - p.q.n;  // committed tokens; tiles before pre / KT hold no others
    if (j + 1 < end) {
      if (j + 1 >= pre / KT) clean(p.q, j + 1, x, turn);
    } else if (more && end - p.j0 >= 4 && nxt.j0 >= (nxt.q.T - nxt.q.n) / KT) {
      clean(nxt.q, nxt.j0, x, turn ^ 1);
    }
    store(slot ^ 1, x);
    const bool own = j + 3 < end || !more;
    load(own ? id_at(ids, min(j + 3, end - 1) - base) : id_at(first, j + 3 - end), own ? p.g : nxt.g, x);
    if (active && j < p.j1) {
      const Slot& sl = slots[slot];
#pragma unroll
      for (int y = 0; y < SUB; ++y)
        st.attend([&](int m, int c) __attribute__((always_inline)) { return *(const i32x4*)(sl.k[y] + kro[c] + 1024 * m); },
                  [&](int nn) __attribute__((always_inline)) {
                    return *(const i32x4*)(sl.v[y] + vro[nn & 1] + 1024 * (nn >> 1));
                  },
                  j * KT + 32 * y + 8 * lj, j * KT + 32 * y + 32 > pre, pre, cmul, a.words, rows);
    }
    lds_barrier();
    ++j;
  };
  // Results: this lane holds dims 32 (nn / 2) + 8 lj + 4 (nn % 2) + e of its columns.
  const auto finish = [&]() __attribute__((always_inline)) {
    const bool whole = p.j0 == 0 && p.j1 == p.nt;
    const bool odd_v = odd[turn] != 0;
    if (!whole && p.j0 == 0 && tid == 0) note_start(a, p, walk.wg);
#pragma unroll
    for (int b = 0; b < NC; ++b) {
      const int col = WCOLS * w + 16 * b + li;
      if (p.c0 + col >= p.q.n * a.group) continue;
      if (whole) {
        const float l = st.lsum[b][0];
        const bool none = l == 0.f;  // sees no token, or all its scores are -infinity: zeros, whatever V holds
        const float inv = none ? 0.f : vsc / l;
        if (none) {
#pragma unroll
          for (int nn = 0; nn < 8; ++nn) st.acc[b][nn] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int nn = 0; nn < 8; nn += 2)
          store_out<FP8>(a, p.s, p.g, p.q, p.c0 + col, 16 * nn + 8 * lj, st.acc[b][nn] * inv, st.acc[b][nn + 1] * inv,
                         odd_v && !none);
      } else {
        const size_t rec = (size_t)(2 * walk.wg + (p.j0 == 0)) * COLS + col;
        if (lj == 0) *(f32x4*)(a.stat + 4 * rec) = f32x4{st.mc[b], st.lsum[b][0], odd_v ? 1.f : 0.f, 0.f};
#pragma unroll
        for (int nn = 0; nn < 8; ++nn)
          *(f32x4*)(a.part + rec * kD + 32 * (nn >> 1) + 8 * lj + 4 * (nn & 1)) = st.acc[b][nn];
      }
    }
  };
  for (bool linked = false;;) {
    enter(linked);
    while (true) {
      const int stop = min(base + kChunk, end);
      do {
        step(0, rB);
        step(1, rA);
      } while (j < stop);
      if (j >= end) break;
      ids = later;
      base += kChunk;
      later = block_of(p, base + kChunk + lane);
    }
    finish();
    if (!more) break;
    linked = end - p.j0 >= 4;
  }
}

// Joins the pieces of cut items: out = sum_p o_p 2^(m_p - M) / sum_p l_p 2^(m_p - M).
// One workgroup per 16 columns of one workgroup's unfinished item; sixteen lanes
// a column.  Bound by latency: the first two pieces' places follow from the
// workgroup's index, so they are loaded beside the note that says whether they
// count (they lie inside the workspace whatever it says).
template <bool FP8>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeArgs a, int cols) {
  const int wg = blockIdx.x, next = min(wg + 1, (int)gridDim.x - 1);
  const int col = blockIdx.y * 16 + (threadIdx.x >> 4), dim = (threadIdx.x & 15) * 8;
  struct Sums {
    f32x4 ml, x, y;
  };
  const auto read = [&](int slot) __attribute__((always_inline)) {
    const size_t rec = (size_t)slot * cols + col;
    return Sums{*(const f32x4*)(a.stat + 4 * rec), *(const f32x4*)(a.part + rec * kD + dim),
                *(const f32x4*)(a.part + rec * kD + dim + 4)};
  };
  const Sums s0 = read(2 * wg + 1), s1 = read(2 * next);
  const TreePiece d = a.desc[wg];
  if (d.last < 0) return;
  const Seq q{d.r0, d.n, d.T, d.r0 + d.n};
  const int cc = d.c0 + col;
  if (cc >= q.n * a.group) return;
  const float vsc = FP8 ? a.v_scale[d.g] : 1.0f;
  float m = s0.ml[0], l = s0.ml[1];
  bool odd = s0.ml[2] != 0.f;
  f32x4 o0 = s0.x, o1 = s0.y;
  const auto add = [&](const Sums& s) __attribute__((always_inline)) {
    const float mn = fmaxf(m, s.ml[0]);
    const float f = __builtin_amdgcn_exp2f(m - mn), fs = __builtin_amdgcn_exp2f(s.ml[0] - mn);
    odd |= s.ml[2] != 0.f;
    l = l * f + s.ml[1] * fs;
    o0 = o0 * f + s.x * fs;
    o1 = o1 * f + s.y * fs;
    m = mn;
  };
  add(s1);
#pragma unroll 4
  for (int p = wg + 2; p <= d.last; ++p) add(read(2 * p));
  const bool none = l == 0.f;
  const float inv = none ? 0.f : vsc / l;
  if (none) o0 = o1 = f32x4{0.f, 0.f, 0.f, 0.f};
  store_out<FP8>(a, d.s, d.g, q, cc, dim, o0 * inv, o1 * inv, odd && !none);
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
  int kind;        // columns of an item and how its waves work, see launch_plan()
  int cols;
  int workgroups;
  size_t stat_at() const { return ((size_t)workgroups * sizeof(TreePiece) + 255) & ~(size_t)255; }
  size_t part_at() const { return stat_at() + (((size_t)workgroups * 8 * cols * sizeof(float) + 255) & ~(size_t)255); }
  size_t bytes() const { return part_at() + (size_t)workgroups * 2 * cols * kD * sizeof(float); }
};

Plan plan(const dp_tree_shape* sh) {
  const int64_t group = sh->n_q_heads / sh->n_kv_heads;
  const int64_t per_seq = (sh->total_q * group + std::max(sh->batch, 1) - 1) / std::max(sh->batch, 1);
  const int cus = compute_units();
  // Columns of an item follow the average tree (the host does not know the
  // trees): fewer than a tree has read its cache again for the rest, more leave
  // waves idle.  us with 64 / 128 / 256: 64 columns a tree (short pool, bf16) 186
  // / 192 / 198; 16 to 208 (short pool, e4m3, 112 on average) 170 / 155 / 173; 256
  // (long pool, bf16) 900 / 530 / 440.  Two workgroups of four waves to a compute
  // unit fill each other's gaps (one: 207 for 186, 213 for 162); eight waves of 32
  // columns leave registers for one.  Trees of one size, short pool, bf16, 64 / 72 /
  // 128 / 136 / 256 columns: 181 / 194 / 219 / 241 / 285; e4m3, 64 / 80 / 128 / 144 /
  // 256: 92 / 107 / 128 / 162 / 192.  Trees above the width that the average gives
  // take several items, each of which reads the cache again: one tree of 512 columns
  // on the longest of 128 contexts, the others of 32: 174 for 167.
  if (per_seq <= 64) return Plan{0, 64, 2 * cus};
  if (per_seq <= 128) return Plan{1, 128, 2 * cus};
  return Plan{2, 256, cus};
}

template <bool FP8>
void launch_plan(const Plan& pl, const TreeArgs& a, hipStream_t st) {
  const dim3 grid(pl.workgroups);
  switch (pl.kind) {
    case 0: hipLaunchKernelGGL((tree_kernel<FP8, 4, 1>), grid, dim3(256), 0, st, a); break;
    case 1: hipLaunchKernelGGL((tree_kernel<FP8, 4, 2>), grid, dim3(256), 0, st, a); break;
    default: hipLaunchKernelGGL((tree_kernel<FP8, 8, 2>), grid, dim3(512), 0, st, a); break;
  }
  hipLaunchKernelGGL(tree_merge_kernel<FP8>, dim3(pl.workgroups, pl.cols / 16), dim3(256), 0, st, a, pl.cols);
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
  // (several workgroups read a row of q, and the first may have written its results)
  if (out == q || workspace == q || workspace == out)
    return fail(DP_EINVAL, "tree_decode_attention: q, out and workspace must not be one another");

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
  if (fp8) launch_plan<true>(pl, a, st);
  else launch_plan<false>(pl, a, st);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(DP_EIO, "tree_decode_attention: kernel launch failed: %s", hipGetErrorString(e));
  return DP_OK;
}

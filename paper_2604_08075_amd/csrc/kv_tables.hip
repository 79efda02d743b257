// Block tables and slot maps on the device, for gfx950.
//
// Blocks are handed out on demand (Sec. 3 effect 1).  For a batch of
// sequences with c cached tokens, b blocks and x new tokens this computes, in
// one launch, the blocks each needs, max(0, ceil((c + x) / 16) - b), their
// running sum over the batch, which needs the free ids cover, and for every
// new token its cache slot and position; with parents also its depth and its
// ancestors as bits.  Blocks of sequences that are over go back to the ring.
//
// What bounds it: latency.  A step's 256 sequences are a few kilobytes; the
// chain is load lengths -> scan -> load an id -> store a slot.  So every
// workgroup scans the whole batch by itself (the lengths come from L2, a batch
// of 256 in one go), and then takes its share of the rows: no workgroup waits
// for another, and there is no second launch.  Measured, per call: 256 single
// tokens 6.0 us, 96 trees of up to 32 drafts 6.4, 512 prompts of 722,154 tokens
// (9 MB of slots, positions and tables, 1.0 TB/s) 9.1; with ten barriers a scan
// and wave sums by permutes instead of two and lane shifts 1.2, 0.5 and 1.6 more.
// A row's sequence is found by a binary search over the running sums in LDS.
//
// Nothing that the call reads is written by it (the ring's tail and the table
// entries behind the owned ones are not read), so workgroups need no order.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "common.h"

namespace dpool_tables {

constexpr int kBS = 16;
constexpr int kMaxBatch = 4096;
constexpr int kMaxWords = 4;
constexpr int64_t kMaxCount = (int64_t)1 << 30;  // rows and blocks: two such counts add up in 32 bits
constexpr int kMaxThreads = 512;

struct TablesArgs {
  const int32_t* context;
  const int32_t* owned;
  const int32_t* fresh;    // new tokens, < 0: the sequence is over
  const int32_t* parents;  // [rows] or null
  int32_t* ring;           // [num_blocks]
  const int32_t* state_in;
  int32_t* tables;         // [B, max_blocks]
  int32_t* context_out;
  int32_t* owned_out;
  int32_t* state_out;
  int32_t* q_start;        // [B + 1]
  int64_t* slots;
  int32_t* positions;
  int32_t* granted;
  uint64_t* mask;          // [rows, words]
  int32_t batch, max_blocks, words;
  uint32_t rows, blocks;
};

// Inclusive running sum over a wave, cut at `lim` (a, b <= 2^30 + 1 each, so
// that no sum passes 32 bits; cutting at every step equals cutting the whole
// sum); the wave's last one goes to wsum.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_lanes(uint32_t x, uint32_t lim) {
  return min(x + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, true), lim);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x, uint32_t lim, uint32_t* wsum) {
  x = min(x, lim);
  x = add_lanes<0x111, 0xf>(x, lim);  // from 1, 2, 4 and 8 lanes before, within rows of sixteen
  x = add_lanes<0x112, 0xf>(x, lim);
  x = add_lanes<0x114, 0xf>(x, lim);
  x = add_lanes<0x118, 0xf>(x, lim);
  x = add_lanes<0x142, 0xa>(x, lim);  // the end of row 0 to row 1, of 2 to 3
  x = add_lanes<0x143, 0xc>(x, lim);  // the end of row 1 to rows 2 and 3
  if ((threadIdx.x & 63) == 63) wsum[threadIdx.x >> 6] = x;
  return x;
}

// The same over the workgroup, once all waves' sums are there.  `carry`: the sum of the chunks before, then of this too.
__device__ __forceinline__ uint32_t join_waves(uint32_t x, uint32_t lim, const uint32_t* wsum, uint32_t& carry) {
  const int w = threadIdx.x >> 6, nw = blockDim.x >> 6;
  uint32_t before = carry;
  for (int k = 0; k < nw; ++k) {
    if (k == w) before = carry;
    carry = min(carry + wsum[k], lim);
  }
  return min(x + before, lim);
}

// Largest s with start[s] <= i (start non-decreasing, start[0] = 0 <= i).
__device__ __forceinline__ int find(const uint32_t* start, int n, uint32_t i) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (start[mid] <= i) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__global__ __launch_bounds__(kMaxThreads) void kv_tables_kernel(TablesArgs a) {
  // [B + 1] first row, [B + 1] first released block, [B] first new block of
  // the ring (~0: refused), [threads] + 256 parents of the rows at hand
  extern __shared__ uint32_t lds[];
  __shared__ uint32_t wsum[3][kMaxThreads / 64], took;
  const int B = a.batch, tid = threadIdx.x, nt = blockDim.x;
  uint32_t* const row0 = lds;
  uint32_t* const back0 = row0 + B + 1;
  uint32_t* const take0 = back0 + B + 1;
  int32_t* const par = (int32_t*)(take0 + B);
  const uint32_t nb = a.blocks;
  const int64_t cap = (int64_t)a.max_blocks * kBS;
  uint32_t head = (uint32_t)max(a.state_in[0], 0);
  if (head >= nb) head %= nb;
  const uint32_t free = min((uint32_t)max(a.state_in[1], 0), nb);

  uint32_t rows_c = 0, back_c = 0, need_c = 0;  // sums of the chunks before
  if (tid == 0) row0[0] = back0[0] = took = 0;
  int x1 = 0, c1 = 0, b1 = 0;  // a chunk ahead
  if (tid < B) x1 = a.fresh[tid], c1 = a.context[tid], b1 = a.owned[tid];
  for (int base = 0; base < B; base += nt) {
    const int s = base + tid, x = x1;
    int c = c1, b = b1;
    x1 = 0;
    if (s + nt < B) x1 = a.fresh[s + nt], c1 = a.context[s + nt], b1 = a.owned[s + nt];
    const uint32_t n = (uint32_t)max(x, 0);
    c = (int)min((int64_t)max(c, 0), cap);
    b = max(min(max(b, 0), a.max_blocks), (int)((uint32_t)(c + kBS - 1) / kBS));
    const uint32_t n_upto = wave_scan(n, a.rows + 1, wsum[0]);
    const uint32_t back_upto = wave_scan(x < 0 ? (uint32_t)b : 0, nb, wsum[1]);
    __syncthreads();
    const uint32_t rows_end = join_waves(n_upto, a.rows + 1, wsum[0], rows_c);
    const uint32_t back_end = join_waves(back_upto, nb, wsum[1], back_c);
    const int64_t want = (int64_t)c + n;
    const bool fits = want <= cap && rows_end <= a.rows && !(a.parents && n > 64u * a.words);
    const uint32_t need = fits && x > 0 ? (uint32_t)max((int64_t)0, (want + kBS - 1) / kBS - b) : 0;
    const uint32_t need_upto = wave_scan(need, nb + 1, wsum[2]);
    __syncthreads();  // (what the next chunk writes, everyone has read by then)
    const uint32_t need_end = join_waves(need_upto, nb + 1, wsum[2], need_c);
    const bool ok = fits && (need == 0 || need_end <= free);
    if (s < B) {
      row0[s + 1] = min(rows_end, a.rows);
      back0[s + 1] = back_end;
      take0[s] = ok ? need_end - need : ~0u;
      if (blockIdx.x == 0) {
        a.granted[s] = ok || x < 0;
        a.context_out[s] = x < 0 ? 0 : ok ? (int)want : c;
        a.owned_out[s] = x < 0 ? 0 : ok ? b + (int)need : b;
        a.q_start[s + 1] = (int)min(rows_end, a.rows);
      }
    }
    // the last sum that the free ids still cover is what was taken
    if (blockIdx.x == 0 && ok && need) atomicMax(&took, need_end);
  }
  __syncthreads();
  const uint32_t back = min(back_c, nb - free);  // more would overtake the ring's head: ids that were never handed out
  if (blockIdx.x == 0 && tid == 0) {
    a.q_start[0] = 0;
    a.state_out[0] = (int)((head + took) % nb);  // (both below 2^30 + 1)
    a.state_out[1] = (int)(free - took + back);
  }
  const uint32_t rows_used = row0[B];

  // released blocks
  for (uint32_t f = blockIdx.x * nt + tid; f < back; f += gridDim.x * nt) {
    const int s = find(back0, B, f);
    uint32_t at = head + free + f;  // below 3 * 2^30
    at %= nb;
    a.ring[at] = a.tables[(size_t)s * a.max_blocks + (f - back0[s])];
  }

  // rows, a workgroup's threads a chunk
  for (uint32_t r0 = blockIdx.x * nt; r0 < a.rows; r0 += gridDim.x * nt) {
    const uint32_t r = r0 + tid;
    uint32_t w0 = 0;  // first row whose parent is at hand
    if (a.parents) {
      __syncthreads();  // the previous chunk's are done with
      w0 = r0 < 64u * kMaxWords ? 0 : r0 - 64u * kMaxWords;
      for (uint32_t i = w0 + tid; i < min(r0 + nt, a.rows); i += nt) par[i - w0] = a.parents[i];
      __syncthreads();
    }
    if (r >= a.rows) continue;
    int64_t slot = -1;
    int pos = -1;
    uint64_t bits[kMaxWords] = {0, 0, 0, 0};
    if (r < rows_used) {
      const int s = find(row0, B, r);
      const uint32_t first = row0[s], i = r - first;
      const int c = (int)min((int64_t)max(a.context[s], 0), cap);
      const int64_t t = (int64_t)c + i;
      pos = (int)min(t, (int64_t)INT32_MAX);
      const uint32_t take = take0[s];
      if (take != ~0u) {
        const int b = max(min(max(a.owned[s], 0), a.max_blocks), (c + kBS - 1) / kBS);
        const int blk = (int)(t / kBS);
        int32_t* const entry = a.tables + (size_t)s * a.max_blocks + blk;
        int id;
        if (blk >= b) {
          uint32_t at = head + take + (uint32_t)(blk - b);  // below 3 * 2^30
          at %= nb;
          id = a.ring[at];
          if (t % kBS == 0) *entry = id;  // a new block's first row is this call's
        } else {
          id = *entry;
        }
        if (id >= 0) slot = (int64_t)id * kBS + t % kBS;
      }
      if (a.parents) {
        if (row0[s + 1] - first <= 64u * a.words) {
          // up to the root: every parent comes before its child
          int depth = 0;
          uint32_t at = i;
          for (;;) {
#pragma unroll
            for (int w = 0; w < kMaxWords; ++w)
              if ((int)(at >> 6) == w) bits[w] |= 1ull << (at & 63);
            const int p = par[first + at - w0];
            if (p < 0 || p >= (int)at) break;
            at = (uint32_t)p;
            ++depth;
          }
          pos = (int)min((int64_t)c + depth, (int64_t)INT32_MAX);
        }
      }
    }
    a.slots[r] = slot;
    a.positions[r] = pos;
    if (a.parents) {
#pragma unroll
      for (int w = 0; w < kMaxWords; ++w)
        if (w < a.words) a.mask[(size_t)r * a.words + w] = bits[w];
    }
  }
}

}  // namespace dpool_tables

using namespace dpool_tables;

extern "C" int kv_tables_step(const int32_t* context_lens, const int32_t* n_owned, const int32_t* new_tokens,
                              const int32_t* parents, int32_t* free_ids, const int32_t* free_state_in,
                              int32_t* block_tables, int32_t* context_lens_out, int32_t* n_owned_out,
                              int32_t* free_state_out, int32_t* q_start, int64_t* slots, int32_t* positions,
                              int32_t* granted, uint64_t* tree_mask, const dp_tables_shape* sh, void* stream) {
  using dpool::fail;
  if (!sh) return fail(DP_EINVAL, "kv_tables_step: null shape");
  if (sh->block_size != kBS) return fail(DP_ENOTSUP, "kv_tables_step: block_size %d (only 16)", sh->block_size);
  if (sh->reserved != 0) return fail(DP_EINVAL, "kv_tables_step: reserved must be 0");
  if (sh->batch < 0) return fail(DP_EINVAL, "kv_tables_step: batch < 0");
  if (sh->batch > kMaxBatch) return fail(DP_ENOTSUP, "kv_tables_step: batch above %d", kMaxBatch);
  if (sh->max_blocks_per_seq <= 0 || sh->max_blocks_per_seq > INT32_MAX / kBS)
    return fail(DP_EINVAL, "kv_tables_step: max_blocks_per_seq out of range");
  if (sh->total_rows < 0 || sh->total_rows > kMaxCount || sh->num_blocks <= 0 || sh->num_blocks > kMaxCount)
    return fail(DP_EINVAL, "kv_tables_step: need 0 <= total_rows <= 2^30 and 0 < num_blocks <= 2^30");
  if (sh->mask_words < 0 || sh->mask_words > kMaxWords)
    return fail(DP_ENOTSUP, "kv_tables_step: mask_words %d (0 to %d)", sh->mask_words, kMaxWords);
  if (!free_state_in || !free_state_out || !q_start) return fail(DP_EINVAL, "kv_tables_step: null tensor pointer");
  if (sh->batch > 0 && (!context_lens || !n_owned || !new_tokens || !free_ids || !block_tables || !context_lens_out ||
                        !n_owned_out || !granted))
    return fail(DP_EINVAL, "kv_tables_step: null tensor pointer");
  if (sh->total_rows > 0 && (!slots || !positions)) return fail(DP_EINVAL, "kv_tables_step: null tensor pointer");
  if ((parents != nullptr) != (tree_mask != nullptr) || (parents != nullptr) != (sh->mask_words > 0))
    return fail(DP_EINVAL, "kv_tables_step: parents, tree_mask and mask_words go together");
  if (((uintptr_t)context_lens | (uintptr_t)n_owned | (uintptr_t)new_tokens | (uintptr_t)parents |
       (uintptr_t)free_ids | (uintptr_t)free_state_in | (uintptr_t)block_tables | (uintptr_t)context_lens_out |
       (uintptr_t)n_owned_out | (uintptr_t)free_state_out | (uintptr_t)q_start | (uintptr_t)positions |
       (uintptr_t)granted) & 3 || ((uintptr_t)slots | (uintptr_t)tree_mask) & 7)
    return fail(DP_EINVAL, "kv_tables_step: pointers must be aligned to their elements");
  const void* const in[] = {context_lens, n_owned, new_tokens, free_state_in, parents};
  const void* const out[] = {context_lens_out, n_owned_out, free_state_out, q_start, granted, positions,
                             slots, tree_mask, free_ids, block_tables};
  constexpr int n_out = sizeof(out) / sizeof(out[0]);
  for (const void* i : in)
    for (const void* o : out)
      if (i && i == o) return fail(DP_EINVAL, "kv_tables_step: an output must not be an input");
  for (int i = 0; i < n_out; ++i)
    for (int j = 0; j < i; ++j)
      if (out[i] && out[i] == out[j]) return fail(DP_EINVAL, "kv_tables_step: two outputs are one tensor");

  TablesArgs a;
  a.context = context_lens;
  a.owned = n_owned;
  a.fresh = new_tokens;
  a.parents = parents;
  a.ring = free_ids;
  a.state_in = free_state_in;
  a.tables = block_tables;
  a.context_out = context_lens_out;
  a.owned_out = n_owned_out;
  a.state_out = free_state_out;
  a.q_start = q_start;
  a.slots = slots;
  a.positions = positions;
  a.granted = granted;
  a.mask = tree_mask;
  a.batch = sh->batch;
  a.max_blocks = sh->max_blocks_per_seq;
  a.words = sh->mask_words;
  a.rows = (uint32_t)sh->total_rows;
  a.blocks = (uint32_t)sh->num_blocks;
  const int threads = sh->batch > 256 ? 512 : 256;
  // Threads: the scan takes a batch in as few turns as its size asks for, a small
  // batch with few waves at each barrier (96 trees: 7.4 us with 256, 7.7 with 512;
  // 722,154 rows of 512 prompts 14.2 / 10.9; of 2,048 34.7 / 23.7).  Workgroups:
  // one to as many rows as it has threads, or to 4,096 table entries that may
  // have to go back, at most what fills half of the device's wave slots, as each
  // scans the batch (512 prompts: 13.3 us with half as many, 10.4; 15.8 for 12.0
  // with twice as many, before the scan had two barriers instead of ten).
  const int64_t groups = std::min<int64_t>((1 << 18) / threads, std::max((sh->total_rows + threads - 1) / threads,
                                                         (int64_t)sh->batch * sh->max_blocks_per_seq / 4096));
  const size_t dyn = (size_t)(3 * sh->batch + 2 + (parents ? threads + 64 * kMaxWords : 0)) * sizeof(uint32_t);
  (void)hipGetLastError();
  hipLaunchKernelGGL(kv_tables_kernel, dim3((unsigned)std::max<int64_t>(groups, 1)), dim3(threads), dyn,
                     (hipStream_t)stream, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(DP_EIO, "kv_tables_step: kernel launch failed: %s", hipGetErrorString(e));
  return DP_OK;
}

// Accepted drafts kept in the cache, for gfx950: the K row and V column of
// every accepted draft move to the front of the sequence's drafted slots, in
// the caches of up to 64 layers per launch.
//
// What bounds it: for a step's handful of tokens, latency; one wave takes one
// (layer, sequence, KV head).  For many, the V tiles: a token's V is one column
// of a dims-major tile, 128 values that lie 32 (bf16) or 16 (e4m3) bytes apart,
// so moving 256 bytes touches a whole 4 KB tile twice.  So tiles are read and
// written whole, in 16-byte pieces: a lane holds all tokens of dimensions lane
// and lane + 64, and a moved value passes from one word of its registers to
// another.  Measured: paths of up to eight of sixteen drafts, 128 sequences, 16
// layers, 8 heads, bf16 (56 MB of values; counted 108 MB read, 81 MB written):
// 43 us, 4.4 TB/s (a large copy: 4.8); value by value it was 60.  Paths of up to
// five, five sequences, 6 layers, 4 heads, e4m3: 4.7 us.
//
// Entries are strictly increasing, accepted[j] >= j, and only one wave works
// on a tile.  A target block's moves are read before it is written, and a later
// block's sources lie at or behind it, which nothing has written.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "common.h"

namespace dpool_accept {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kD = 128;
constexpr int kBS = 16;
constexpr int kWaves = 4;
constexpr int kMaxLayers = 64;  // per launch: their addresses are kernel arguments
constexpr int kMaxBatch = 4096;
constexpr int kMaxCall = 1024;  // layers of a call

struct AcceptArgs {
  char* k[kMaxLayers];
  char* v[kMaxLayers];
  const int32_t* tables;
  const int32_t* context;
  const int32_t* q_start;
  const int32_t* accepted;
  const int32_t* n_accepted;
  int32_t* context_out;
  int64_t units;       // layers * batch * hkv
  int64_t num_blocks;
  int32_t batch, hkv, max_blocks, max_ctx, total_q, max_accept, write_context;
};

template <bool FP8>
__global__ __launch_bounds__(kWaves * 64) void kv_accept_kernel(AcceptArgs a) {
  using Code = std::conditional_t<FP8, uint8_t, uint16_t>;
  using Pair = std::conditional_t<FP8, uint16_t, uint32_t>;
  constexpr int kRegs = FP8 ? 1 : 2;  // 16-byte pieces of a dimension's tokens
  constexpr int N = FP8 ? 4 : 2, BITS = 32 / N;  // tokens of a word
  constexpr uint32_t ONES = (1u << BITS) - 1;
  typedef i32x4 Tile[2][kRegs];  // dimensions lane and lane + 64 of a V tile
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (unit >= a.units) return;
  const int per_layer = a.batch * a.hkv;
  const int layer = (int)(unit / per_layer);
  const int s = (int)(unit - (int64_t)layer * per_layer) / a.hkv;
  const int g = (int)(unit - (int64_t)layer * per_layer) - s * a.hkv;
  const int T = min(max(a.context[s], 0), a.max_ctx);
  const int r0 = min(max(a.q_start[s], 0), a.total_q);
  const int n = min(min(max(a.q_start[s + 1], r0), a.total_q) - r0, T);
  const int want = min(min(max(a.n_accepted[s], 0), a.max_accept), n);
  Code* const kl = (Code*)a.k[layer];
  Code* const vl = (Code*)a.v[layer];
  const int32_t* const bt = a.tables + (size_t)s * a.max_blocks;

  const auto load = [&](const Code* p, Tile& x) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < kRegs; ++i) x[h][i] = ((const i32x4*)(p + (lane + 64 * h) * kBS))[i];
  };

  int last = -1, done = 0;  // the last entry so far, and how many were valid
  for (int j0 = 0; j0 < want; j0 += 64) {
    const int j = j0 + lane;
    const int idx = j < want ? a.accepted[(size_t)s * a.max_accept + j] : -1;
    int prev = __shfl_up(idx, 1);
    if (lane == 0) prev = last;
    const uint64_t bad = __ballot(idx <= prev || idx >= n);  // (idx >= 0 follows from idx > prev >= -1)
    const int ok = bad ? __builtin_ctzll(bad) : 64;
    // this lane's move: block and slot that it reads, those that it writes, and their places in the table
    int from = -1, to = -1, s_from = 0, s_to = 0, p_from = -1, p_to = -1;
    if (lane < ok && idx != j) {
      const int ts = T - n + idx, td = T - n + j;
      from = bt[ts / kBS], to = bt[td / kBS];
      if (from >= 0 && from < a.num_blocks && to >= 0 && to < a.num_blocks) {
        p_from = ts / kBS, s_from = ts % kBS;
        p_to = td / kBS, s_to = td % kBS;
      }
    }
    uint64_t todo = __ballot(p_to >= 0);
    while (todo) {
      // the moves into one block: consecutive lanes, consecutive slots
      const int f = __builtin_ctzll(todo), first = __builtin_amdgcn_readlane(s_to, f) - f;  // slot of lane 0
      const uint64_t mine = __ballot(p_to == __builtin_amdgcn_readlane(p_to, f));
      todo &= ~mine;
      uint32_t left = (uint32_t)(mine >> f) << (first + f);  // by slot
      const size_t tile = ((size_t)__builtin_amdgcn_readlane(to, f) * a.hkv + g) * (kBS * kD);
      Tile d, x;
      load(vl + tile, d);
      Pair k[kBS];
#pragma unroll
      for (int t = 0; t < kBS; ++t)
        if (left >> t & 1) {
          const size_t at = ((size_t)__builtin_amdgcn_readlane(from, t - first) * a.hkv + g) * kBS;
          k[t] = *(const Pair*)(kl + (at + __builtin_amdgcn_readlane(s_from, t - first)) * kD + 2 * lane);
        }
#pragma unroll
      for (int t = 0; t < kBS; ++t)
        if (left >> t & 1) *(Pair*)(kl + tile + t * kD + 2 * lane) = k[t];
      while (left) {
        // those that come from one block
        const int e = __builtin_ctz(left) - first, p = __builtin_amdgcn_readlane(p_from, e);
        const uint32_t here = (uint32_t)((__ballot(p_from == p) & mine) >> f) << (first + f);
        left &= ~here;
        if (p == __builtin_amdgcn_readlane(p_to, f)) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < kRegs; ++i) x[h][i] = d[h][i];
        } else load(vl + ((size_t)__builtin_amdgcn_readlane(from, e) * a.hkv + g) * (kBS * kD), x);
#pragma unroll
        for (int t = 0; t < kBS; ++t)
          if (here >> t & 1) {
            const int s0 = __builtin_amdgcn_readlane(s_from, t - first);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t w = (uint32_t)x[h][0][0];
#pragma unroll
              for (int i = 1; i < 4 * kRegs; ++i) w = s0 / N == i ? (uint32_t)x[h][i / 4][i % 4] : w;
              const uint32_t code = w >> (s0 % N * BITS) & ONES;
              const uint32_t rest = (uint32_t)d[h][t / N / 4][t / N % 4] & ~(ONES << (t % N * BITS));
              d[h][t / N / 4][t / N % 4] = (int)(rest | code << (t % N * BITS));
            }
          }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < kRegs; ++i) ((i32x4*)(vl + tile + (lane + 64 * h) * kBS))[i] = d[h][i];
    }
    done += min(ok, want - j0);
    if (bad && ok < want - j0) break;
    last = __shfl(idx, 63);
  }
  if (a.write_context && layer == 0 && g == 0 && lane == 0) a.context_out[s] = a.n_accepted[s] < 0 ? T : T - n + done;
}

}  // namespace dpool_accept

using namespace dpool_accept;

extern "C" int kv_cache_accept(void* const* k_layers, void* const* v_layers, int32_t n_layers,
                               const int32_t* block_tables, const int32_t* context_lens, const int32_t* q_start,
                               const int32_t* accepted, const int32_t* n_accepted, int32_t max_accept,
                               int32_t* context_lens_out, const dp_tree_shape* sh, void* stream) {
  using dpool::fail;
  if (!sh) return fail(DP_EINVAL, "kv_cache_accept: null shape");
  if (sh->head_dim != kD) return fail(DP_ENOTSUP, "kv_cache_accept: head_dim %d (only 128)", sh->head_dim);
  if (sh->block_size != kBS) return fail(DP_ENOTSUP, "kv_cache_accept: block_size %d (only 16)", sh->block_size);
  if (sh->kv_dtype != DP_KV_BF16 && sh->kv_dtype != DP_KV_FP8_E4M3)
    return fail(DP_ENOTSUP, "kv_cache_accept: kv_dtype %d", sh->kv_dtype);
  if (sh->reserved != 0) return fail(DP_EINVAL, "kv_cache_accept: reserved must be 0");
  if (sh->batch < 0) return fail(DP_EINVAL, "kv_cache_accept: batch < 0");
  if (sh->batch > kMaxBatch) return fail(DP_ENOTSUP, "kv_cache_accept: batch above %d", kMaxBatch);
  if (n_layers > kMaxCall) return fail(DP_ENOTSUP, "kv_cache_accept: more than %d layers", kMaxCall);
  if (n_layers <= 0 || max_accept <= 0) return fail(DP_EINVAL, "kv_cache_accept: n_layers and max_accept must be > 0");
  if (sh->n_kv_heads <= 0 || (int64_t)sh->batch * sh->n_kv_heads > INT32_MAX / kMaxLayers)
    return fail(DP_EINVAL, "kv_cache_accept: n_kv_heads out of range");
  if (sh->max_blocks_per_seq <= 0 || sh->max_context_len < 0 ||
      (int64_t)sh->max_blocks_per_seq * kBS < sh->max_context_len || sh->num_blocks <= 0 ||
      sh->num_blocks > INT32_MAX)
    return fail(DP_EINVAL, "kv_cache_accept: need max_blocks_per_seq * 16 >= max_context_len and "
                           "0 < num_blocks <= INT32_MAX");
  if (sh->total_q < 0 || sh->total_q > INT32_MAX / 2) return fail(DP_EINVAL, "kv_cache_accept: total_q out of range");
  if (sh->batch == 0) return DP_OK;
  if (!k_layers || !v_layers || !block_tables || !context_lens || !q_start || !accepted || !n_accepted ||
      !context_lens_out)
    return fail(DP_EINVAL, "kv_cache_accept: null pointer");
  if (context_lens_out == context_lens || context_lens_out == n_accepted || context_lens_out == q_start ||
      context_lens_out == accepted || context_lens_out == block_tables)
    return fail(DP_EINVAL, "kv_cache_accept: context_lens_out must not be an input");
  if (((uintptr_t)block_tables | (uintptr_t)context_lens | (uintptr_t)q_start | (uintptr_t)accepted |
       (uintptr_t)n_accepted | (uintptr_t)context_lens_out) & 3)
    return fail(DP_EINVAL, "kv_cache_accept: pointers must be 4-byte aligned");
  for (int32_t i = 0; i < n_layers; ++i) {
    if (!k_layers[i] || !v_layers[i]) return fail(DP_EINVAL, "kv_cache_accept: null cache of layer %d", i);
    if (((uintptr_t)k_layers[i] | (uintptr_t)v_layers[i]) & 15)
      return fail(DP_EINVAL, "kv_cache_accept: caches must be 16-byte aligned");
    if (k_layers[i] == v_layers[i])
      return fail(DP_EINVAL, "kv_cache_accept: K and V of layer %d are the same cache", i);
    // (a cache given twice would move its tokens twice, in two waves at once)
    bool twice = false;
    for (int32_t j = 0; j < i; ++j)
      twice |= k_layers[j] == k_layers[i] || v_layers[j] == v_layers[i] || k_layers[j] == v_layers[i] ||
               v_layers[j] == k_layers[i];
    if (twice) return fail(DP_EINVAL, "kv_cache_accept: a cache of layer %d was given before", i);
  }

  AcceptArgs a;
  a.tables = block_tables;
  a.context = context_lens;
  a.q_start = q_start;
  a.accepted = accepted;
  a.n_accepted = n_accepted;
  a.context_out = context_lens_out;
  a.num_blocks = sh->num_blocks;
  a.batch = sh->batch;
  a.hkv = sh->n_kv_heads;
  a.max_blocks = sh->max_blocks_per_seq;
  a.max_ctx = sh->max_context_len;
  a.total_q = (int32_t)sh->total_q;
  a.max_accept = max_accept;
  const bool fp8 = sh->kv_dtype == DP_KV_FP8_E4M3;
  (void)hipGetLastError();
  for (int32_t l0 = 0; l0 < n_layers; l0 += kMaxLayers) {
    const int n = std::min(kMaxLayers, n_layers - l0);
    for (int i = 0; i < kMaxLayers; ++i) {
      a.k[i] = i < n ? (char*)k_layers[l0 + i] : nullptr;
      a.v[i] = i < n ? (char*)v_layers[l0 + i] : nullptr;
    }
    a.units = (int64_t)n * sh->batch * sh->n_kv_heads;
    a.write_context = l0 == 0;
    const dim3 grid((unsigned)((a.units + kWaves - 1) / kWaves)), block(kWaves * 64);
    if (fp8) hipLaunchKernelGGL(kv_accept_kernel<true>, grid, block, 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(kv_accept_kernel<false>, grid, block, 0, (hipStream_t)stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(DP_EIO, "kv_cache_accept: kernel launch failed: %s", hipGetErrorString(e));
  }
  return DP_OK;
}

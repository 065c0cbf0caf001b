// Eviction from a cache in pages by accumulated weight (d3tom_cache_evict): which slots of a request stay, and the moves that
// close the gaps.
//
// The kept slots of a request are its `keep` first ones by (weight descending, slot ascending).  Those that lie behind the new
// length move into the gaps before it, the i-th into the i-th: sources are all behind the new length and destinations before
// it, so no move waits for another, and only what has to move does (slots kept in order would all shift from the first gap on).
// Attention does not depend on the order of slots, since keys carry their positions.
//
// plan_kernel: one CTA per request, a radix select of the key of rank `keep` (as select.cu) and one ordered pass that numbers gaps and
// movers.  move_kernel: rows copied by blocks that share all requests' moves.  Bound: latency of the selection, then HBM.
#include "common.cuh"

namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;

struct EvictArgs {
  d3tom_cache cache;
  const int32_t* budget; const int32_t* protect_from; int32_t* length_out;
  int B, cap;                   // cap: slots a request can have in this call
  int32_t* gaps; int32_t* movers;     // [B][cap / 2 + 1] places in the pools; the movers last first
  int32_t* count;               // [B] moves
  int list_stride;
  int* dev_status;
};

// Larger is kept first.  Numbers by their order (-0 as 0), what is not a number and protected slots before all.
__device__ __forceinline__ uint32_t evict_key(float w, bool safe) {
  return safe || w != w ? 0xffffffffu : ordered_key(w + 0.f);
}

__global__ void __launch_bounds__(kThreads) plan_kernel(const EvictArgs a) {
  __shared__ unsigned hist[256], warp_tot[kWarps];
  __shared__ unsigned sh_prefix, sh_remaining, carry, run_gt, run_eq;
  grid_dependency_enter();
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int raw_len = a.cache.length[b];
  const int n = min(max(raw_len, 0), a.cap);
  if (tid == 0 && raw_len != n) atomicExch(a.dev_status, D3TOM_ERR_INVALID_ARG);
  const int keep = min(max(a.budget[b], 0), n);
  __syncthreads();                               // (length_out may be the lengths themselves: everyone has read them)
  if (keep == n || keep == 0) {
    if (tid == 0) { a.length_out[b] = keep; a.count[b] = 0; }
    return;
  }
  const int32_t* table = a.cache.page_table + (size_t)b * a.cache.max_pages;
  const int safe_from = a.protect_from != nullptr ? a.protect_from[b] : 0;
  auto place_of = [&](int slot) -> int {
    const int p = slot / a.cache.page_size, page = table[p];
    return page < 0 || page >= a.cache.pages ? -1 : page * a.cache.page_size + (slot - p * a.cache.page_size);
  };
  auto key_of = [&](int slot) -> uint32_t {
    const int place = place_of(slot);
    if (place < 0) { atomicExch(a.dev_status, D3TOM_ERR_INVALID_ARG); return 0u; }
    return evict_key(a.cache.weight[place], a.protect_from != nullptr && a.cache.token[place] >= safe_from);
  };

  // ---- the key of rank `keep`, eight bits at a time
  if (tid == 0) { sh_prefix = 0u; sh_remaining = (unsigned)keep; run_gt = 0u; run_eq = 0u; }
  uint32_t mask = 0u;
  const int n_round = (n + 31) / 32 * 32;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) hist[tid] = 0u;
    __syncthreads();
    const uint32_t prefix = sh_prefix;
    for (int j = tid; j < n_round; j += kThreads) {
      uint32_t digit = 0xffffffffu;
      if (j < n) {
        const uint32_t key = key_of(j);
        if ((key & mask) == prefix) digit = (key >> shift) & 255u;
      }
      const unsigned peers = __match_any_sync(0xffffffffu, digit);
      if (digit != 0xffffffffu && lane == __ffs(peers) - 1) atomicAdd(&hist[digit], __popc(peers));
    }
    __syncthreads();
    if (warp == 0) {
      unsigned cnt[8], mine = 0u;
#pragma unroll
      for (int i = 0; i < 8; ++i) { cnt[i] = hist[255 - (lane * 8 + i)]; mine += cnt[i]; }
      unsigned incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
      }
      const unsigned excl = incl - mine, rem = sh_remaining;
      __syncwarp();
      if (excl < rem && rem <= incl) {
        unsigned run = excl;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (run < rem && rem <= run + cnt[i]) {
            sh_prefix = prefix | ((uint32_t)(255 - (lane * 8 + i)) << shift);
            sh_remaining = rem - run;
          }
          run += cnt[i];
        }
      }
    }
    mask |= 255u << shift;
    __syncthreads();
  }
  const uint32_t T = sh_prefix;
  const unsigned need_eq = sh_remaining;

  // ---- in order: kept slots counted, gaps before `keep` and movers from `keep` on listed
  int32_t* gaps = a.gaps + (size_t)b * a.list_stride;
  int32_t* movers = a.movers + (size_t)b * a.list_stride;
  for (int base = 0; base < n; base += kThreads) {
    const int j = base + tid;
    bool gt = false, eq = false;
    if (j < n) { const uint32_t key = key_of(j); gt = key > T; eq = key == T; }
    const unsigned val = (gt ? 0x10000u : 0u) | (eq ? 1u : 0u);
    unsigned incl = val;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned t = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += t;
    }
    if (lane == 31) warp_tot[warp] = incl;
    __syncthreads();
    if (warp == 0) {
      const unsigned w = warp_tot[lane];
      unsigned winc = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned t = __shfl_up_sync(0xffffffffu, winc, o);
        if (lane >= o) winc += t;
      }
      warp_tot[lane] = winc - w;
      if (lane == 31) carry = winc;
    }
    __syncthreads();
    const unsigned excl = warp_tot[warp] + incl - val;
    const unsigned gt_before = run_gt + (excl >> 16), eq_before = run_eq + (excl & 0xffffu);
    if (j < n) {
      const bool kept = gt || (eq && eq_before < need_eq);
      const int kept_before = (int)(gt_before + min(eq_before, need_eq));
      if (j < keep && !kept) gaps[j - kept_before] = place_of(j);
      if (j >= keep && kept) movers[keep - 1 - kept_before] = place_of(j);
      if (j == keep) a.count[b] = keep - kept_before;
    }
    __syncthreads();
    if (tid == 0) { run_gt += carry >> 16; run_eq += carry & 0xffffu; }
    __syncthreads();
  }
  if (tid == 0) a.length_out[b] = keep;
}

constexpr int kMoveThreads = 256;

// U: the unit rows are copied in (their length is a multiple of it)
template <typename U>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const EvictArgs a, const int row_units) {
  grid_dependency_enter();
  const int b = blockIdx.x % a.B, first = blockIdx.x / a.B, step = gridDim.x / a.B, n = a.count[b];
  const int32_t* gaps = a.gaps + (size_t)b * a.list_stride;
  const int32_t* movers = a.movers + (size_t)b * a.list_stride;
  for (int i = first; i < n; i += step) {
    const int to = gaps[i], from = movers[n - 1 - i];
    if (to < 0 || from < 0) continue;
    const U* ks = static_cast<const U*>(a.cache.k) + (size_t)from * row_units;
    const U* vs = static_cast<const U*>(a.cache.v) + (size_t)from * row_units;
    U* kd = static_cast<U*>(a.cache.k) + (size_t)to * row_units;
    U* vd = static_cast<U*>(a.cache.v) + (size_t)to * row_units;
    for (int u = threadIdx.x; u < row_units; u += kMoveThreads) {
      const U x = ks[u], y = vs[u];
      kd[u] = x;
      vd[u] = y;
    }
    if (threadIdx.x == 0) {
      a.cache.weight[to] = a.cache.weight[from];
      if (a.cache.token != nullptr) a.cache.token[to] = a.cache.token[from];
    }
  }
}

}  // namespace

int launch_cache_evict(d3tom_ctx* ctx, d3tom_dtype dt, const d3tom_cache& cache, const int32_t* budget,
                       const int32_t* protect_from, int B, int max_length, int32_t* length_out, cudaStream_t s) {
  EvictArgs a = {};
  const long long slots = (long long)cache.max_pages * cache.page_size;
  a.cache = cache; a.budget = budget; a.protect_from = protect_from; a.length_out = length_out; a.B = B;
  a.cap = max_length < slots ? max_length : (int)slots;
  a.list_stride = max_length / 2 + 1;            // moves are at most min(keep, n - keep)
  a.count = static_cast<int32_t*>(ctx->kept_rows);     // (B + 2 B (max_length / 2 + 1) words at most)
  a.gaps = a.count + B;
  a.movers = a.gaps + (size_t)B * a.list_stride;
  a.dev_status = ctx->dev_status;
  D3TOM_CUDA_TRY(ctx, launch_serialized(plan_kernel, B, kThreads, 0, s, a));
  const int row_bytes = cache.kv_heads * ctx->lim.head_dim * (dt == D3TOM_BF16 ? 2 : 4);
  const int per_request = max(1, min(a.list_stride, ceil_div(8 * ctx->sm_count, B)));
  if (row_bytes % 16 == 0) D3TOM_CUDA_TRY(ctx, launch_serialized(move_kernel<uint4>, B * per_request, kMoveThreads, 0, s, a, row_bytes / 16));
  else D3TOM_CUDA_TRY(ctx, launch_serialized(move_kernel<uint2>, B * per_request, kMoveThreads, 0, s, a, row_bytes / 8));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

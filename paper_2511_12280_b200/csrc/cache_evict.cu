// Eviction from a cache in pages by accumulated weight (d3tom_cache_evict): which slots of a request stay, and the moves that
// close the gaps.
//
// The kept slots of a request are its `keep` first ones by (weight descending, slot ascending).  Those that lie behind the new
// length move into the gaps before it, the i-th into the i-th: sources are all behind the new length and destinations before
// it, so no move waits for another, and only what has to move does (slots kept in order would all shift from the first gap on).
// Attention does not depend on the order of slots, since keys carry their positions.
//
// plan_reg_kernel, plan_kernel: one CTA per request, a radix select of the key of rank `keep` (as select.cu) and one ordered pass that
// numbers gaps and movers.  move_kernel: rows copied by blocks that share all requests' moves.  Bound: latency of the selection, then HBM.
#include <type_traits>

#include "common.cuh"

namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;

struct EvictArgs {
  d3tom_cache cache;
  const int32_t* budget; const int32_t* protect_from; int32_t* length_out;
  int B, cap;                   // cap: slots a request can have in this call
  int32_t* gaps; int32_t* movers;     // [B][max_length / 2] places in the pools; the movers last first
  int32_t* count;               // [B] moves
  int list_stride;
  int* dev_status;
};

// Larger is kept first.  Numbers by their order (-0 as 0), what is not a number and protected slots before all.
__device__ __forceinline__ uint32_t evict_key(float w, bool safe) {
  return safe || w != w ? 0xffffffffu : ordered_key(w + 0.f);
}

// A request of this CTA: its length as this call sees it, and how many slots stay.
struct EvictRequest {
  const EvictArgs& a;
  const int32_t* table;
  int n, keep, safe_from;
  __device__ __forceinline__ EvictRequest(const EvictArgs& args, int b) : a(args) {
    const int raw = a.cache.length[b];
    n = min(max(raw, 0), a.cap);
    if (threadIdx.x == 0 && raw != n) report_invalid(a.dev_status);
    keep = min(max(a.budget[b], 0), n);
    table = a.cache.page_table + (size_t)b * a.cache.max_pages;
    safe_from = a.protect_from != nullptr ? a.protect_from[b] : 0;
  }
  __device__ __forceinline__ int place(int slot) const {
    const int p = slot / a.cache.page_size, page = table[p];
    return page < 0 || page >= a.cache.pages ? -1 : page * a.cache.page_size + (slot - p * a.cache.page_size);
  }
  __device__ __forceinline__ uint32_t key_at(int place) const {
    if (place < 0) { report_invalid(a.dev_status); return 0u; }
    return evict_key(a.cache.weight[place], a.protect_from != nullptr && a.cache.token[place] >= safe_from);
  }
};

// inclusive prefix sum over the block in thread order; every warp scans the 32 warp totals itself
__device__ __forceinline__ unsigned block_scan(unsigned val, unsigned* warp_tot) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned incl = val;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned t = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += t;
  }
  if (lane == 31) warp_tot[warp] = incl;
  __syncthreads();
  unsigned w = warp_tot[lane], winc = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned t = __shfl_up_sync(0xffffffffu, winc, o);
    if (lane >= o) winc += t;
  }
  return incl + __shfl_sync(0xffffffffu, winc - w, warp);
}

// Requests of up to 1024 x IPT slots: every thread keeps IPT consecutive slots' keys and places in registers, so pages are looked
// up and weights read once.  Digits from the highest bit of (key - smallest key) on, 12 bits, then 10 and 10, until every
// key that shares the digits so far stays (as select.cu; there is more on it there).
constexpr int kBinsMax = 4096;
template <int IPT>
__global__ void __launch_bounds__(kThreads) plan_reg_kernel(const EvictArgs a) {
  __shared__ unsigned hist[kBinsMax];
  __shared__ unsigned warp_tot[kWarps], warp_lo[kWarps], warp_hi[kWarps];
  __shared__ unsigned sh_prefix, sh_remaining, sh_whole;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, b = blockIdx.x;
  for (int d = tid; d < kBinsMax; d += kThreads) hist[d] = 0u;
  grid_dependency_enter();
  const EvictRequest r(a, b);
  const int n = r.n, keep = r.keep;
  __syncthreads();                               // (length_out may be the lengths themselves: everyone has read them)
  if (tid == 0) a.length_out[b] = keep;
  if (keep == n || keep == 0) {
    if (tid == 0) a.count[b] = 0;
    return;
  }
  const int j0 = tid * IPT;
  int place[IPT];
  uint32_t key[IPT];
#pragma unroll
  for (int i = 0; i < IPT; ++i) place[i] = j0 + i < n ? r.place(j0 + i) : 0;
  uint32_t lo = 0xffffffffu, hi = 0u;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    key[i] = 0u;
    if (j0 + i < n) { key[i] = r.key_at(place[i]); lo = min(lo, key[i]); hi = max(hi, key[i]); }
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lane == 0) { warp_lo[warp] = lo; warp_hi[warp] = hi; }
  __syncthreads();
  lo = __reduce_min_sync(0xffffffffu, warp_lo[lane]);
  hi = __reduce_max_sync(0xffffffffu, warp_hi[lane]);
#pragma unroll
  for (int i = 0; i < IPT; ++i) key[i] -= lo;    // (those past the end are never looked at)
  int top = 32 - __clz((int)(hi - lo));
  uint32_t prefix = 0u;
  unsigned rem = (unsigned)keep;
  bool whole = false;
  auto take_digit = [&](auto first) {
    constexpr bool kFirst = decltype(first)::value;
    constexpr int kBits = kFirst ? 12 : 10, kOwn = kFirst ? 4 : 1;
    const int shift = max(top - kBits, 0);
#pragma unroll
    for (int i = 0; i < IPT; ++i)
      if (j0 + i < n && (kFirst || (key[i] >> top) == (prefix >> top))) atomicAdd(&hist[(key[i] >> shift) & ((1u << kBits) - 1u)], 1u);
    __syncthreads();
    const int top_bin = (1 << kBits) - 1 - kOwn * tid;
    unsigned cnt[kOwn], mine = 0u;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) { cnt[i] = hist[top_bin - i]; hist[top_bin - i] = 0u; mine += cnt[i]; }
    const unsigned incl = block_scan(mine, warp_tot);
    unsigned run = incl - mine;
    if (run < rem && rem <= incl) {              // exactly one thread: the digit of the key of rank `keep`
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (run < rem && rem <= run + cnt[i]) {
          sh_prefix = prefix | ((uint32_t)(top_bin - i) << shift);
          sh_remaining = rem - run;
          sh_whole = rem - run == cnt[i] ? 1u : 0u;
        }
        run += cnt[i];
      }
    }
    __syncthreads();
    prefix = sh_prefix;
    rem = sh_remaining;
    whole = sh_whole != 0u;
    top = shift;
  };
  if (top > 0) take_digit(std::true_type());
  if (top > 0 && !whole) take_digit(std::false_type());
  if (top > 0 && !whole) take_digit(std::false_type());
  uint32_t T = prefix;                           // the key of rank `keep`; or the largest value below all that share its digits
  unsigned need_eq = rem;
  if (whole && T > 0u) { T -= 1u; need_eq = 0u; }

  unsigned val = 0u;
#pragma unroll
  for (int i = 0; i < IPT; ++i)
    if (j0 + i < n) val += (key[i] > T ? 0x10000u : 0u) + (key[i] == T ? 1u : 0u);
  __syncthreads();                               // (warp_tot is written again)
  const unsigned before = block_scan(val, warp_tot) - val;
  unsigned gt_before = before >> 16, eq_before = before & 0xffffu;
  int32_t* gaps = a.gaps + (size_t)b * a.list_stride;
  int32_t* movers = a.movers + (size_t)b * a.list_stride;
#pragma unroll
  for (int i = 0; i < IPT; ++i) {
    const int j = j0 + i;
    if (j < n) {
      const bool gt = key[i] > T, eq = key[i] == T;
      const bool kept = gt || (eq && eq_before < need_eq);
      const int kept_before = (int)(gt_before + min(eq_before, need_eq));
      if (j < keep && !kept) gaps[j - kept_before] = place[i];
      if (j >= keep && kept) movers[keep - 1 - kept_before] = place[i];
      if (j == keep) a.count[b] = keep - kept_before;
      gt_before += gt ? 1u : 0u;
      eq_before += eq ? 1u : 0u;
    }
  }
}

// Longer requests: keys read again for every digit.
__global__ void __launch_bounds__(kThreads) plan_kernel(const EvictArgs a) {
  __shared__ unsigned hist[256], warp_tot[kWarps];
  __shared__ unsigned sh_prefix, sh_remaining, carry, run_gt, run_eq;
  grid_dependency_enter();
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const EvictRequest r(a, b);
  const int n = r.n, keep = r.keep;
  __syncthreads();                               // (length_out may be the lengths themselves: everyone has read them)
  if (tid == 0) a.length_out[b] = keep;
  if (keep == n || keep == 0) {
    if (tid == 0) a.count[b] = 0;
    return;
  }

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
        const uint32_t key = r.key_at(r.place(j));
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
    if (j < n) { const uint32_t key = r.key_at(r.place(j)); gt = key > T; eq = key == T; }
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
      if (j < keep && !kept) gaps[j - kept_before] = r.place(j);
      if (j >= keep && kept) movers[keep - 1 - kept_before] = r.place(j);
      if (j == keep) a.count[b] = keep - kept_before;
    }
    __syncthreads();
    if (tid == 0) { run_gt += carry >> 16; run_eq += carry & 0xffffu; }
    __syncthreads();
  }
}

constexpr int kMoveThreads = 256;

// The blocks share all requests' moves evenly, whatever each request has.  U: the unit rows are copied in (their length is a
// multiple of it).
template <typename U>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const EvictArgs a, const int row_units) {
  grid_dependency_enter();
  const int lane = threadIdx.x & 31;
  long long next = blockIdx.x, base = 0;          // this block's next move among all; the first of request b0
  for (int b0 = 0; b0 < a.B; b0 += 32) {
    const int mine = b0 + lane < a.B ? a.count[b0 + lane] : 0;
    int incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += t;
    }
    const int total = __shfl_sync(0xffffffffu, incl, 31);
    for (; next < base + total; next += gridDim.x) {
      const int at = (int)(next - base), src = __ffs(__ballot_sync(0xffffffffu, incl > at)) - 1;
      const int n = __shfl_sync(0xffffffffu, mine, src), i = at - (__shfl_sync(0xffffffffu, incl, src) - n);
      const size_t list = (size_t)(b0 + src) * a.list_stride;
      const int to = a.gaps[list + i], from = a.movers[list + n - 1 - i];
      if (to < 0 || from < 0) continue;
      const U* ks = static_cast<const U*>(a.cache.k) + (size_t)from * row_units;
      const U* vs = static_cast<const U*>(a.cache.v) + (size_t)from * row_units;
      U* kd = static_cast<U*>(a.cache.k) + (size_t)to * row_units;
      U* vd = static_cast<U*>(a.cache.v) + (size_t)to * row_units;
      int u = threadIdx.x;
      for (; u + kMoveThreads < row_units; u += 2 * kMoveThreads) {
        const U x0 = ks[u], y0 = vs[u], x1 = ks[u + kMoveThreads], y1 = vs[u + kMoveThreads];
        kd[u] = x0; vd[u] = y0; kd[u + kMoveThreads] = x1; vd[u + kMoveThreads] = y1;
      }
      if (u < row_units) {
        const U x0 = ks[u], y0 = vs[u];
        kd[u] = x0; vd[u] = y0;
      }
      if (threadIdx.x == 0) {
        a.cache.weight[to] = a.cache.weight[from];
        if (a.cache.token != nullptr) a.cache.token[to] = a.cache.token[from];
      }
    }
    base += total;
  }
}

}  // namespace

int launch_cache_evict(d3tom_ctx* ctx, d3tom_dtype dt, const d3tom_cache& cache, const int32_t* budget,
                       const int32_t* protect_from, int B, int max_length, int32_t* length_out, cudaStream_t s) {
  EvictArgs a = {};
  const long long slots = (long long)cache.max_pages * cache.page_size;
  a.cache = cache; a.budget = budget; a.protect_from = protect_from; a.length_out = length_out; a.B = B;
  a.cap = max_length < slots ? max_length : (int)slots;
  a.list_stride = max_length / 2;                // moves are at most min(keep, n - keep)
  a.count = static_cast<int32_t*>(ctx->kept_rows);     // (B + 2 B (max_length / 2) words)
  a.gaps = a.count + B;
  a.movers = a.gaps + (size_t)B * a.list_stride;
  a.dev_status = ctx->dev_status;
  auto plan = a.cap <= kThreads ? plan_reg_kernel<1> : a.cap <= 4 * kThreads ? plan_reg_kernel<4> : a.cap <= 8 * kThreads ? plan_reg_kernel<8>
            : a.cap <= 16 * kThreads ? plan_reg_kernel<16> : plan_kernel;
  D3TOM_CUDA_TRY(ctx, launch_serialized(plan, B, kThreads, 0, s, a));
  const int row_bytes = cache.kv_heads * ctx->lim.head_dim * (dt == D3TOM_BF16 ? 2 : 4);
  const long long most = (long long)B * a.list_stride;
  const int blocks = most < 1 ? 1 : most < 8 * ctx->sm_count ? (int)most : 8 * ctx->sm_count;
  if (row_bytes % 16 == 0) D3TOM_CUDA_TRY(ctx, launch_serialized(move_kernel<uint4>, blocks, kMoveThreads, 0, s, a, row_bytes / 16));
  else D3TOM_CUDA_TRY(ctx, launch_serialized(move_kernel<uint2>, blocks, kMoveThreads, 0, s, a, row_bytes / 8));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

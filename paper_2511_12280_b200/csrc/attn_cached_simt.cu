// Attention of a few new rows over a cache in pages on CUDA cores: fp32 caches, and bf16 ones for comparison.
//
// Bound by HBM as long as few rows share a key: a key and its value are read once for up to eight rows x query heads of a key
// head.  A warp takes 32 (key, row) pairs at a time.  Lanes split a key's numbers four each, so its bytes come in one coalesced
// load that needs no shared memory; the partial products of the 32 pairs are summed over the lanes by halving (each step a lane
// hands over the half of its pairs that it does not keep: 31 exchanges for 32 sums), after which a lane has one pair's score and
// takes one exponential.  The probabilities go back to all lanes by shuffles and weight the values, whose loads have been under way
// meanwhile.  Running maximum and sum per row; warps join through shared memory at the end of a segment.
#include "cache_walk.cuh"
#include "ptx.cuh"

namespace {

// Warps per CTA and CTAs per SM for RT rows per tile: one row needs the registers for its loads, eight rows for their sums.
template <int RT> struct SimtShape {
  static constexpr int kWarps = RT == 8 ? 4 : 8;
  static constexpr int kCtas = RT == 8 ? 3 : RT == 1 ? 1 : 2;
};

template <typename T> __device__ __forceinline__ float4 load4(const T* p);
template <> __device__ __forceinline__ float4 load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <> __device__ __forceinline__ float4 load4<__nv_bfloat16>(const __nv_bfloat16* p) {
  const uint2 w = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16),
                     __uint_as_float(w.y & 0xffff0000u));
}

// RT rows per tile; a key's numbers are split over LPK lanes
template <typename T, int RT, int LPK>
__global__ void __launch_bounds__(SimtShape<RT>::kWarps * 32, SimtShape<RT>::kCtas) attn_cached_simt_kernel(const CachedArgs a) {
  constexpr int kWarps = SimtShape<RT>::kWarps, kThreads = kWarps * 32;
  constexpr int kKeys = 32 / RT;                 // keys per warp and step
  constexpr int kSide = 32 / LPK;                // .. side by side
  constexpr int kPasses = kKeys / kSide;         // .. one after the other
  constexpr int kAhead = kPasses < 8 ? kPasses : 8;   // loads in flight per lane
  static_assert(kPasses * RT == LPK, "a lane ends up with one pair");
  __shared__ float o_s[kWarps][RT][LPK * 4];
  __shared__ float2 ml_s[kWarps][RT];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & (LPK - 1), side = lane / LPK;
  const int dh = a.dh, d0 = sub * 4;
  const bool has = d0 < dh;                      // lanes beyond a short head have nothing
  const size_t pitch = (size_t)a.kv_heads * dh;
  grid_dependency_enter();
  const CachedRun run = cached_run(a, blockIdx.x);
  CachedWalk walk;
  walk.start(a, run);
  CachedSegment s = {};
  bool head = true;                              // the run's first segment
  bool missing = false;                          // a slot whose page is not one of the pool's
  while (walk.next(a, s)) {
    if (head && threadIdx.x == kThreads - 1) cached_write_join(a, run, blockIdx.x, s, walk.tiles);
    head = false;
    const int32_t* table = a.page_table + (size_t)s.b * a.max_pages;
    const T* kp = static_cast<const T*>(a.k) + (size_t)s.kv_head * dh + d0;
    const T* vp = static_cast<const T*>(a.v) + (size_t)s.kv_head * dh + d0;
    float4 q[RT], o[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      o[r] = q[r] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < s.rows && has) q[r] = load4(static_cast<const T*>(a.q) + (size_t)cached_row_index(a, s, r) * dh + d0);
    }
    const int my_row = lane % RT;
    const bool scored = a.scores != nullptr && my_row < s.rows;
    float m = -INFINITY, l = 0.f;                // of this lane's row, over its own pairs (l) and all lanes' (m)
    const int end = min(s.len, s.t1 * kKeyTile);
    // lane i: where key i of a step is (slots of a pool are counted in 31 bits); looked up a step ahead
    auto find = [&](int key0) {
      if (lane >= kKeys || key0 + lane >= end) return -1;
      const int at = (int)cached_place(table, key0 + lane, a.page_size, a.pages);
      missing |= at < 0;
      return at;
    };
    int next_at = find(s.t0 * kKeyTile + warp * kKeys);
    for (int key0 = s.t0 * kKeyTile + warp * kKeys; key0 < end; key0 += kWarps * kKeys) {
      float val[LPK];
      float4 vv[kAhead];
      const int at = next_at;
      int place[kPasses];
#pragma unroll
      for (int p = 0; p < kPasses; ++p) place[p] = __shfl_sync(0xffffffffu, at, p * kSide + side);
#pragma unroll
      for (int p0 = 0; p0 < kPasses; p0 += kAhead) {
        float4 kk[kAhead];
        if (p0 == 0)                             // the first values are under way with the first keys
#pragma unroll
          for (int p = 0; p < kAhead; ++p)
            vv[p] = place[p] >= 0 && has ? load4(vp + (size_t)place[p] * pitch) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int p = 0; p < kAhead; ++p)
          kk[p] = place[p0 + p] >= 0 && has ? load4(kp + (size_t)place[p0 + p] * pitch) : make_float4(0.f, 0.f, 0.f, 0.f);
        if (p0 == 0) next_at = find(key0 + kWarps * kKeys);
#pragma unroll
        for (int p = 0; p < kAhead; ++p)
#pragma unroll
          for (int r = 0; r < RT; ++r)
            val[(p0 + p) * RT + r] = q[r].x * kk[p].x + q[r].y * kk[p].y + q[r].z * kk[p].z + q[r].w * kk[p].w;
      }
      // sum over the LPK lanes; lane `sub` keeps pair `sub`
#pragma unroll
      for (int h = LPK / 2; h > 0; h >>= 1) {
        const bool up = (sub & h) != 0;
#pragma unroll
        for (int i = 0; i < h; ++i) {
          const float send = up ? val[i] : val[i + h], keep = up ? val[i + h] : val[i];
          val[i] = keep + __shfl_xor_sync(0xffffffffu, send, h);
        }
      }
      const int key = sub / RT * kSide + side, mine = __shfl_sync(0xffffffffu, at, key);
      const float raw = val[0];
      if (scored && mine >= 0) {
        const int t = (key0 + key) / kKeyTile;
        const CachedScores sc = cached_scores(a, s.lo, s.n, s.len, t);
        sc.tile[(size_t)(s.kv_head * s.n * a.group + s.row0 + my_row) * sc.pitch + (key0 + key - t * kKeyTile)] = raw;
      }
      const float x = mine >= 0 ? raw * a.scale_log2 : -INFINITY;
      float top = x;
#pragma unroll
      for (int h = 16; h >= RT; h >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, h));
      const float m_new = fmaxf(m, top);
      if (__any_sync(0xffffffffu, m_new > m)) {
        const float alpha = m_new > m ? ptx::ex2(m - m_new) : 1.f;
        l *= alpha;
        m = m_new;
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float f = __shfl_sync(0xffffffffu, alpha, r);
          o[r].x *= f; o[r].y *= f; o[r].z *= f; o[r].w *= f;
        }
      }
      const float pr = m == -INFINITY ? (x != x ? x : 0.f) : ptx::ex2(x - m);
      l += pr;
#pragma unroll
      for (int p0 = 0; p0 < kPasses; p0 += kAhead) {
        if (p0 > 0)
#pragma unroll
        for (int p = 0; p < kAhead; ++p)
          vv[p] = place[p0 + p] >= 0 && has ? load4(vp + (size_t)place[p0 + p] * pitch) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int p = 0; p < kAhead; ++p)
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const float f = __shfl_sync(0xffffffffu, pr, side * LPK + (p0 + p) * RT + r);
            o[r].x += f * vv[p].x; o[r].y += f * vv[p].y; o[r].z += f * vv[p].z; o[r].w += f * vv[p].w;
          }
      }
    }
    // ---- the warp's result: sums over the lanes that had other keys
#pragma unroll
    for (int h = 16; h >= RT; h >>= 1) l += __shfl_xor_sync(0xffffffffu, l, h);
#pragma unroll
    for (int r = 0; r < RT; ++r) {
#pragma unroll
      for (int h = 16; h >= LPK; h >>= 1) {
        o[r].x += __shfl_xor_sync(0xffffffffu, o[r].x, h); o[r].y += __shfl_xor_sync(0xffffffffu, o[r].y, h);
        o[r].z += __shfl_xor_sync(0xffffffffu, o[r].z, h); o[r].w += __shfl_xor_sync(0xffffffffu, o[r].w, h);
      }
      if (side == 0) *reinterpret_cast<float4*>(&o_s[warp][r][d0]) = o[r];
    }
    if (lane < RT) ml_s[warp][lane] = make_float2(m, l);
    __syncthreads();
    // ---- the CTA's: into the output, or into this CTA's place for parts
    float* part = a.part + ((size_t)blockIdx.x * 2 + s.slot) * cached_part_stride(a);
    for (int i = threadIdx.x; i < s.rows * dh; i += kThreads) {
      const int r = i / dh, d = i - r * dh;
      float mm = ml_s[0][r].x;
#pragma unroll
      for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, ml_s[w][r].x);
      mm = fmaxf(mm, -1e38f);                    // (a row without keys so far: M stays finite, l is 0)
      float ll = 0.f, oo = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = ptx::ex2(ml_s[w][r].x - mm);
        ll += ml_s[w][r].y * f;
        oo += o_s[w][r][d] * f;
      }
      if (s.whole) {
        const int row = cached_row_index(a, s, r);
        static_cast<T*>(a.out)[(size_t)row * dh + d] = Storage<T>::from_float(ll == 0.f ? 0.f : oo / ll);
        if (d == 0 && a.lse != nullptr) a.lse[row] = make_float2(mm, ll);
      } else {
        part[i] = oo;
        if (d == 0) { part[(size_t)RT * dh + r] = mm; part[(size_t)RT * dh + RT + r] = ll; }
      }
    }
    __syncthreads();
  }
  if (missing) report_invalid(a.dev_status);     // (inside the loop: four requests of 8000 slots x 4 x 128, eight rows 59 -> 63 us)
  if (head && threadIdx.x == 0) cached_write_join(a, run, blockIdx.x, s, 0);
  cached_write_empty<T>(a, threadIdx.x, kThreads);
}

template <typename T, int RT, int LPK>
int launch_rows(d3tom_ctx* ctx, d3tom_dtype dt, CachedArgs a, cudaStream_t s) {
  a.ctas = SimtShape<RT>::kCtas * ctx->sm_count;
  a.tile_rows = RT;
  D3TOM_CUDA_TRY(ctx, launch_serialized(attn_cached_simt_kernel<T, RT, LPK>, a.ctas, SimtShape<RT>::kWarps * 32, 0, s, a));
  D3TOM_LAUNCH_CHECK(ctx);
  return launch_attn_cached_join(ctx, dt, a, s);
}

template <typename T, int LPK>
int launch(d3tom_ctx* ctx, d3tom_dtype dt, const CachedArgs& a, cudaStream_t s) {
  const long long rows = (long long)a.max_rows * a.group;
  if (rows <= 1) return launch_rows<T, 1, LPK>(ctx, dt, a, s);
  if (rows <= 2) return launch_rows<T, 2, LPK>(ctx, dt, a, s);
  // Eight rows share a key's bytes, four make more work items of a small call (us, eight / four: 12 rows x 4 key heads x four
  // requests up to 2177 slots x 64 26.3 / 22.7; 32 rows x 4 x four of 8000 x 128 158 / 185).  Asked with the longest length there can be.
  const long long items = (long long)a.B * a.kv_heads * ((rows + 7) / 8) * ceil_div(a.cap, kKeyTile);
  if (rows <= 4 || items < 6 * ctx->sm_count) return launch_rows<T, 4, LPK>(ctx, dt, a, s);
  return launch_rows<T, 8, LPK>(ctx, dt, a, s);
}

}  // namespace

int launch_attn_cached_simt(d3tom_ctx* ctx, d3tom_dtype dt, const CachedArgs& a, cudaStream_t s) {
  if (dt == D3TOM_BF16) return a.dh <= 64 ? launch<__nv_bfloat16, 16>(ctx, dt, a, s) : launch<__nv_bfloat16, 32>(ctx, dt, a, s);
  return a.dh <= 64 ? launch<float, 16>(ctx, dt, a, s) : launch<float, 32>(ctx, dt, a, s);
}

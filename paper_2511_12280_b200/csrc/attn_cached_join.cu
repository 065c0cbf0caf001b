// What follows the kernels that attend to a cache in pages: the work items that several CTAs shared are joined, and the attention
// mass of every slot goes into its weight.
//
// Join: with (O_i, M_i, l_i) of the segments of an item, M = max M_i, l = sum l_i 2^(M_i - M), O = sum O_i 2^(M_i - M) / l.
// Weight of slot j: sum over the rows i and query heads h of f_i 2^(s_ihj c - M_ih) / l_ih, from the raw scores that the attention
// kernel left (they are 1 / (64 kv_heads / heads) of the keys' bytes).  Both in a fixed order.  Bound: latency, then HBM.
#include "cache_walk.cuh"
#include "ptx.cuh"

namespace {

constexpr int kJoinThreads = 128;

// Block (c, y): if CTA c's run begins inside an item and contains its end, joins rows y, y + gridDim.y, .. of it.
// The blocks also write what no CTA has: zeros for the rows of requests without slots.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const CachedArgs a) {
  grid_dependency_enter();
  const int c = blockIdx.x, tid = threadIdx.x, dh = a.dh;
  for (int b = c; b < a.B; b += gridDim.x) {
    const CachedRequest r = cached_request(a, b);
    const int raw = a.length[b];
    if (tid == 0 && blockIdx.y == 0 && (raw < 0 || raw > a.cap)) atomicExch(a.dev_status, D3TOM_ERR_INVALID_ARG);
    if (r.len > 0) continue;
    T* out = static_cast<T*>(a.out) + (size_t)r.lo * a.H * dh;
    const size_t count = (size_t)r.n * a.H * dh;
    for (size_t i = (size_t)blockIdx.y * kJoinThreads + tid; i < count; i += (size_t)gridDim.y * kJoinThreads)
      out[i] = Storage<T>::from_float(0.f);
  }
  const CachedRun run = cached_run(a, c);
  if (run.w0 >= run.w1) return;
  CachedWalk walk;
  walk.start(a, run);
  CachedSegment s;
  if (!walk.next(a, s) || s.t0 == 0 || s.t1 != walk.tiles) return;      // the run does not begin inside an item, or does not end it
  const long long begin = run.w0 - s.t0;                                 // the item's first tile
  int c0 = (int)(begin * run.ctas / run.total);                          // .. and the CTA that has it
  while (cached_run_begin(run.total, run.ctas, c0) > begin) --c0;
  while (cached_run_begin(run.total, run.ctas, c0 + 1) <= begin) ++c0;
  const size_t stride = (size_t)a.tile_rows * (dh + 2);
  const float* first = a.part + ((size_t)c0 * 2 + (cached_run_begin(run.total, run.ctas, c0) == begin ? 0 : 1)) * stride;
  const float* rest = a.part + (size_t)(c0 + 1) * 2 * stride;
  const int n = c - c0 + 1;
  for (int r = blockIdx.y; r < s.rows; r += gridDim.y) {
    // (O rows, then M of all rows, then l of all rows)
    const size_t at_m = (size_t)a.tile_rows * dh + r, at_l = at_m + a.tile_rows;
    float m = first[at_m];
    for (int i = 1; i < n; ++i) m = fmaxf(m, rest[(size_t)(i - 1) * 2 * stride + at_m]);
    float l = 0.f, o = 0.f;
    for (int i = 0; i < n; ++i) {
      const float* p = i == 0 ? first : rest + (size_t)(i - 1) * 2 * stride;
      const float f = ptx::ex2(p[at_m] - m);
      l += p[at_l] * f;
      if (tid < dh) o += p[(size_t)r * dh + tid] * f;
    }
    const int row = cached_row_index(a, s, r);
    if (tid < dh) static_cast<T*>(a.out)[(size_t)row * dh + tid] = Storage<T>::from_float(l == 0.f ? 0.f : o / l);
    if (tid == 0 && a.lse != nullptr) a.lse[row] = make_float2(m, l);
  }
}

constexpr int kWeightWarps = 8;

// Block (b, x): 128 slots of request b, four per lane; the warps take every eighth row x head.
__global__ void __launch_bounds__(kWeightWarps * 32)
weight_kernel(const CachedArgs a, float* __restrict__ weight, const int add, const float* __restrict__ row_weight,
              const int chunks) {
  __shared__ float4 sum[kWeightWarps][32];
  grid_dependency_enter();
  const int b = blockIdx.x / chunks, first = (blockIdx.x - b * chunks) * 128;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const CachedRequest r = cached_request(a, b);
  const int slot0 = first + lane * 4;
  if (first >= r.len) return;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const int rows = r.n * a.H;
  if (slot0 < r.len) {                          // (the stride is a multiple of four: a float4 ends inside it)
    const float* sc = a.scores + (size_t)r.lo * a.H * a.score_stride + slot0;
    const float2* lse = a.lse + (size_t)r.lo * a.H;
    for (int i = warp; i < rows; i += kWeightWarps) {
      const float2 ml = lse[i];
      const float4 s = *reinterpret_cast<const float4*>(sc + (size_t)i * a.score_stride);
      const float f = ml.y == 0.f ? 0.f : (row_weight != nullptr ? row_weight[r.lo + i / a.H] : 1.f) / ml.y;
      acc.x += f * ptx::ex2(fmaf(s.x, a.scale_log2, -ml.x));
      acc.y += f * ptx::ex2(fmaf(s.y, a.scale_log2, -ml.x));
      acc.z += f * ptx::ex2(fmaf(s.z, a.scale_log2, -ml.x));
      acc.w += f * ptx::ex2(fmaf(s.w, a.scale_log2, -ml.x));
    }
  }
  sum[warp][lane] = acc;
  __syncthreads();
  if (threadIdx.x < 128) {
    const int slot = first + threadIdx.x;
    if (slot < r.len) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < kWeightWarps; ++w) t += reinterpret_cast<const float*>(sum[w])[threadIdx.x];
      const long long place = cached_place(a.page_table + (size_t)b * a.max_pages, slot, a.page_size, a.pages);
      if (place >= 0) weight[place] = add ? weight[place] + t : t;
    }
  }
}

}  // namespace

int launch_attn_cached_join(d3tom_ctx* ctx, d3tom_dtype dt, const CachedArgs& a, cudaStream_t s) {
  const dim3 grid(a.ctas, a.tile_rows < 8 ? a.tile_rows : 8);
  if (dt == D3TOM_BF16) D3TOM_CUDA_TRY(ctx, launch_serialized(join_kernel<__nv_bfloat16>, grid, kJoinThreads, 0, s, a));
  else D3TOM_CUDA_TRY(ctx, launch_serialized(join_kernel<float>, grid, kJoinThreads, 0, s, a));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

int launch_cached_weight(d3tom_ctx* ctx, const CachedArgs& a, float* weight, int add, const float* row_weight,
                         int max_length, cudaStream_t s) {
  const int chunks = ceil_div(max_length, 128);
  if ((long long)chunks * a.B > 0x7fffffffll) return D3TOM_ERR_UNSUPPORTED;
  D3TOM_CUDA_TRY(ctx, launch_serialized(weight_kernel, chunks * a.B, kWeightWarps * 32, 0, s, a, weight, add, row_weight, chunks));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

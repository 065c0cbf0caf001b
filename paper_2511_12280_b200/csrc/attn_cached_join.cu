// What follows the kernels that attend to a cache in pages: the work items that several CTAs shared are joined, and the attention
// mass of every slot goes into its weight.
//
// Join: with (O_i, M_i, l_i) of the segments of an item, M = max M_i, l = sum l_i 2^(M_i - M), O = sum O_i 2^(M_i - M) / l.
// Weight of slot j: sum over the rows i and query heads h of f_i 2^(s_ihj c - M_ih) / l_ih, from the raw scores that the attention
// kernel left (weight_kernel: 88 MB in 20 us, two thirds of what a copy gets, partly from L2; latency where they are few) or from what its
// second pass summed already (mass_kernel: latency).  All in a fixed order.
#include "cache_walk.cuh"
#include "ptx.cuh"

namespace {

constexpr int kJoinWarps = 4;

// Block (c, y), a warp per row: rows y * 4 .. + 3 of the item that ends in CTA c's run, where an earlier CTA began it.
template <typename T>
__global__ void __launch_bounds__(kJoinWarps * 32) join_kernel(const CachedArgs a) {
  grid_dependency_enter();
  const int4 j0 = reinterpret_cast<const int4*>(a.joins)[2 * blockIdx.x];
  const int n = j0.y, r = blockIdx.y * kJoinWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31, d = lane * 4, dh = a.dh;
  if (r >= (n > 0 ? j0.w : 0)) return;
  const int4 j1 = reinterpret_cast<const int4*>(a.joins)[2 * blockIdx.x + 1];
  const size_t stride = cached_part_stride(a);
  // part i: the first at `first`, the others at slot 0 of the CTAs after it
  const size_t first = (size_t)j0.x, rest = (size_t)(j0.x / 2) * 2;
  auto part = [&](int i) { return a.part + (i == 0 ? first : rest + 2 * (size_t)i) * stride; };
  const size_t at_m = (size_t)a.tile_rows * dh + r, at_l = at_m + a.tile_rows;
  // (M, l) of the first 32 parts stay in registers: one round trip to L2 less where there are no more
  float m0 = -INFINITY, l0 = 0.f;
  if (lane < n) { m0 = part(lane)[at_m]; l0 = part(lane)[at_l]; }
  float m = m0;
  for (int i = lane + 32; i < n; i += 32) m = fmaxf(m, part(i)[at_m]);
  m = warp_max(m);
  float l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0; i0 < n; i0 += 32) {
    const int i = i0 + lane;
    if (i0 > 0 && i < n) { m0 = part(i)[at_m]; l0 = part(i)[at_l]; }
    const float f = i < n ? ptx::ex2(m0 - m) : 0.f;
    l += i < n ? l0 * f : 0.f;
    const int many = min(32, n - i0);
#pragma unroll 8
    for (int k = 0; k < many; ++k) {
      const float g = __shfl_sync(0xffffffffu, f, k);
      if (d < dh) {
        const float4 x = *reinterpret_cast<const float4*>(part(i0 + k) + (size_t)r * dh + d);
        o.x += x.x * g; o.y += x.y * g; o.z += x.z * g; o.w += x.w * g;
      }
    }
  }
  l = warp_sum(l);
  const int f = j1.y + r, i = f / a.group, row = (j0.z + i) * a.H + j1.x * a.group + (f - i * a.group);
  if (d < dh) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T* out = static_cast<T*>(a.out) + (size_t)row * dh + d;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(out) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    else *reinterpret_cast<uint2*>(out) = make_uint2(ptx::pack_bf16x2(o.x * inv, o.y * inv), ptx::pack_bf16x2(o.z * inv, o.w * inv));
  }
  if (lane == 0 && a.lse != nullptr) a.lse[row] = make_float2(m, l);
}

// Mass `t` into the weight of a request's slot.  +inf, which keeps a slot from being evicted, stays when weights are set.  (Looked up and
// read ahead of the sums, or between them, it holds back their loads: one block of 64 rows x 32 heads over 1216 slots 31.4 -> 33.4 us.)
__device__ __forceinline__ void put_weight(const CachedArgs& a, float* weight, int b, int slot, float t, int add) {
  const long long place = cached_place(a.page_table + (size_t)b * a.max_pages, slot, a.page_size, a.pages);
  if (place < 0) { report_invalid(a.dev_status); return; }
  const float had = weight[place];
  weight[place] = add ? had + t : had == INFINITY ? had : t;
}

constexpr int kWeightRows = 1024;      // rows x heads whose (M, f / l) are in shared memory at a time

// Block (b, x): 128 slots of request b, four per lane; the warps share its rows x heads.
template <int kWeightWarps>
__global__ void __launch_bounds__(kWeightWarps * 32)
weight_kernel(const CachedArgs a, float* __restrict__ weight, const int add, const int chunks) {
  __shared__ float2 ml[kWeightRows];
  __shared__ float4 sum[kWeightWarps][32];
  grid_dependency_enter();
  const int b = blockIdx.x / chunks, first = (blockIdx.x - b * chunks) * 128;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const CachedRequest r = cached_request(a, b);
  const int slot0 = first + lane * 4;
  if (first >= r.len) return;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  const int rows = r.n * a.H;
  const bool has = slot0 < r.len;               // (the pitch is a multiple of four: a float4 ends inside it)
  const CachedScores scores = cached_scores(a, r.lo, r.n, r.len, first / kKeyTile);
  for (int i0 = 0; i0 < rows; i0 += kWeightRows) {
    const int many = min(kWeightRows, rows - i0);
    if (i0 > 0) __syncthreads();
    for (int i = threadIdx.x; i < many; i += kWeightWarps * 32) {
      const int per_head = r.n * a.group, g = (i0 + i) / per_head, in = i0 + i - g * per_head, row = r.lo + in / a.group;   // (cached_scores)
      const float2 x = a.lse[(size_t)row * a.H + g * a.group + in % a.group];
      const float f = a.row_weight != nullptr ? a.row_weight[row] : 1.f;
      ml[i] = make_float2(-x.x, x.y == 0.f ? 0.f : f / x.y);
    }
    __syncthreads();
    if (has) {
      const float* sc = scores.tile + (size_t)i0 * scores.pitch + lane * 4;
#pragma unroll 8
      for (int i = warp; i < many; i += kWeightWarps) {
        const float2 f = ml[i];
        const float4 s = __ldcs(reinterpret_cast<const float4*>(sc + (size_t)i * scores.pitch));
        acc.x += f.y * ptx::ex2(fmaf(s.x, a.scale_log2, f.x));
        acc.y += f.y * ptx::ex2(fmaf(s.y, a.scale_log2, f.x));
        acc.z += f.y * ptx::ex2(fmaf(s.z, a.scale_log2, f.x));
        acc.w += f.y * ptx::ex2(fmaf(s.w, a.scale_log2, f.x));
      }
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
      put_weight(a, weight, b, slot, t, add);
    }
  }
}

// Block (b, x): 128 slots of request b; adds up what the second pass over the keys left, one number for `columns` rows x heads.
__global__ void __launch_bounds__(128)
mass_kernel(const CachedArgs a, float* __restrict__ weight, const int add, const int chunks, const int columns) {
  grid_dependency_enter();
  const int b = blockIdx.x / chunks, slot = (blockIdx.x - b * chunks) * 128 + threadIdx.x;
  const CachedRequest r = cached_request(a, b);
  if (slot >= r.len) return;
  float t = 0.f;
  for (int f = 0; f < r.n * a.group; f += columns) {
    const int i = f / a.group;
    const float* row = a.mass + ((size_t)(r.lo + i) * a.H + (f - i * a.group)) * a.score_stride + slot;
#pragma unroll 8
    for (int g = 0; g < a.kv_heads; ++g) t += row[(size_t)g * a.group * a.score_stride];
  }
  put_weight(a, weight, b, slot, t, add);
}

}  // namespace

int launch_attn_cached_join(d3tom_ctx* ctx, d3tom_dtype dt, const CachedArgs& a, cudaStream_t s) {
  if (a.cap <= kKeyTile) return D3TOM_OK;        // no item has a second tile
  const dim3 grid(a.ctas, ceil_div(a.tile_rows, kJoinWarps));
  if (dt == D3TOM_BF16) D3TOM_CUDA_TRY(ctx, launch_serialized(join_kernel<__nv_bfloat16>, grid, kJoinWarps * 32, 0, s, a));
  else D3TOM_CUDA_TRY(ctx, launch_serialized(join_kernel<float>, grid, kJoinWarps * 32, 0, s, a));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

int launch_cached_weight(d3tom_ctx* ctx, const CachedArgs& a, float* weight, int add, int mass_columns, cudaStream_t s) {
  const int chunks = ceil_div(a.cap, 128);
  if ((long long)chunks * a.B > 0x7fffffffll) return D3TOM_ERR_UNSUPPORTED;
  // few rows: small blocks, many of them on an SM (64 requests of one row x 32 heads: 14 us with 4 warps, 30 with 16); many rows: the
  // loads of a block side by side (32 rows x 32 heads: 21 us with 16 warps, eight loads each under way; 80 with 8 warps and one)
  if (mass_columns > 0) D3TOM_CUDA_TRY(ctx, launch_serialized(mass_kernel, chunks * a.B, 128, 0, s, a, weight, add, chunks, mass_columns));
  else if ((long long)a.max_rows * a.H <= 256) D3TOM_CUDA_TRY(ctx, launch_serialized(weight_kernel<4>, chunks * a.B, 4 * 32, 0, s, a, weight, add, chunks));
  else D3TOM_CUDA_TRY(ctx, launch_serialized(weight_kernel<16>, chunks * a.B, 16 * 32, 0, s, a, weight, add, chunks));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

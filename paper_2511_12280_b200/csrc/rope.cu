// Rotary positions (d3tom_rope) and the rows that go into a cache in pages (d3tom_cache_append).
//
// A pair (a, b) of a head becomes (a cos t - b sin t, a sin t + b cos t), t = position * theta^-e.  A position step is held as a
// 64-bit fraction of a turn, so position * step is an integer product that wraps around where the angle does: its upper 32
// bits are the angle to 2^-32 of a turn at every position (in fp32 the product itself would be off by radians from a million on),
// and sincospif needs no range reduction.  The angles of a row are shared by its heads: a block computes them once into shared
// memory.  Bound: HBM (every row is read and written once); with few rows, latency.
#include "common.cuh"

namespace {

constexpr int kThreads = 256;

template <typename T> __device__ __forceinline__ T rotated_lo(T x, T y, float c, float s) {
  return Storage<T>::from_float(Storage<T>::to_float(x) * c - Storage<T>::to_float(y) * s);
}
template <typename T> __device__ __forceinline__ T rotated_hi(T x, T y, float c, float s) {
  return Storage<T>::from_float(Storage<T>::to_float(x) * s + Storage<T>::to_float(y) * c);
}

// One block per row (blockIdx.x); gridDim.y blocks share its heads.  kVector: units of 16 bytes (pairs of halves: 2 x 16, where
// the number of pairs is a multiple of the vector); otherwise a pair or a copied number at a time.
template <typename T, bool kVector>
__global__ void __launch_bounds__(kThreads)
rotate_rows_kernel(const RotateArgs a, const __grid_constant__ RopeTable t, const bool to_cache) {
  constexpr int kVec = Storage<T>::kVec;
  __shared__ float2 turn[64];
  const int tid = threadIdx.x, row = blockIdx.x;
  grid_dependency_enter();
  long long place = -1;                          // where the row goes in the pools
  if (to_cache) {
    if (row >= a.cu_rows[a.B]) return;           // (the whole block)
    const int b = find_segment(a.cu_rows, a.B, row);
    const long long slot = (long long)a.cache.length[b] - a.cu_rows[b + 1] + row;
    if (slot >= 0 && slot < (long long)a.cache.max_pages * a.cache.page_size) {
      const int p = (int)slot / a.cache.page_size, page = a.cache.page_table[(size_t)b * a.cache.max_pages + p];
      if (page >= 0 && page < a.cache.pages) place = (long long)page * a.cache.page_size + ((int)slot - p * a.cache.page_size);
    }
    if (place < 0 && tid == 0) atomicExch(a.dev_status, D3TOM_ERR_INVALID_ARG);
    if (tid == 0 && blockIdx.y == 0 && place >= 0) {
      if (a.cache.weight != nullptr) a.cache.weight[place] = a.first_weight != nullptr ? a.first_weight[row] : 0.f;
      if (a.tokens != nullptr) a.cache.token[place] = a.tokens[row];
    }
  }
  if (tid < t.pairs) {
    const long long pos = a.positions[(size_t)row * t.axes + t.axis[tid]];
    const int32_t part = (int32_t)(((unsigned long long)pos * t.turn[tid]) >> 32);   // in 2^-32 of a turn, -1/2 .. 1/2
    float s, c;
    sincospif((float)part * 4.656612873077392578125e-10f, &s, &c);                   // half turns: part * 2^-31
    turn[tid] = make_float2(c, a.inverse ? -s : s);
  }
  __syncthreads();

  const int pairs = t.pairs, dh = a.dh;
  const int pair_units = !kVector ? pairs : t.neighbours ? 0 : pairs / kVec;      // units that rotate two places at once
  const int per_head = !kVector ? dh - pairs : t.neighbours ? dh / kVec : dh / kVec - pair_units;
  const int rot_units = (a.H + a.kv_heads) * per_head, v_units = a.v != nullptr ? a.kv_heads * (dh / kVec) : 0;
  for (int u = blockIdx.y * kThreads + tid; u < rot_units + v_units; u += gridDim.y * kThreads) {
    if (u >= rot_units) {                        // a piece of the value row
      if (place < 0) continue;
      const size_t off = (size_t)(u - rot_units) * kVec;
      *reinterpret_cast<uint4*>(static_cast<T*>(a.cache.v) + (size_t)place * a.kv_heads * dh + off) =
          *reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + (size_t)row * a.kv_heads * dh + off);
      continue;
    }
    const int head = u / per_head, i = u - head * per_head;
    const T* src;
    T* dst;
    if (head < a.H) {
      const size_t off = ((size_t)row * a.H + head) * dh;
      src = static_cast<const T*>(a.q) + off;
      dst = static_cast<T*>(a.q_out) + off;
    } else {
      const size_t off = (size_t)(head - a.H) * dh, width = (size_t)a.kv_heads * dh;
      src = static_cast<const T*>(a.k) + (size_t)row * width + off;
      if (to_cache) {
        if (place < 0) continue;
        dst = static_cast<T*>(a.cache.k) + (size_t)place * width + off;
      } else {
        dst = static_cast<T*>(a.k_out) + (size_t)row * width + off;
      }
    }
    if constexpr (!kVector) {
      if (i < pairs) {
        const int lo = t.neighbours ? 2 * i : i, hi = t.neighbours ? 2 * i + 1 : pairs + i;
        const T x = src[lo], y = src[hi];
        const float2 cs = turn[i];
        dst[lo] = rotated_lo(x, y, cs.x, cs.y);
        dst[hi] = rotated_hi(x, y, cs.x, cs.y);
      } else {
        dst[pairs + i] = src[pairs + i];
      }
    } else if (t.neighbours) {
      float f[kVec];
      const uint4 raw = *reinterpret_cast<const uint4*>(src + i * kVec);
      if (i * kVec >= 2 * pairs) { *reinterpret_cast<uint4*>(dst + i * kVec) = raw; continue; }
      Storage<T>::load(src + i * kVec, f);
#pragma unroll
      for (int e = 0; e < kVec; e += 2) {
        const int pr = (i * kVec + e) >> 1;
        if (pr < pairs) {
          const float2 cs = turn[pr];
          const float x = f[e], y = f[e + 1];
          f[e] = x * cs.x - y * cs.y;
          f[e + 1] = x * cs.y + y * cs.x;
        }
      }
      Storage<T>::store(dst + i * kVec, f);
    } else if (i < pair_units) {
      float x[kVec], y[kVec];
      Storage<T>::load(src + i * kVec, x);
      Storage<T>::load(src + pairs + i * kVec, y);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float2 cs = turn[i * kVec + e];
        const float r = x[e] * cs.x - y[e] * cs.y;
        y[e] = x[e] * cs.y + y[e] * cs.x;
        x[e] = r;
      }
      Storage<T>::store(dst + i * kVec, x);
      Storage<T>::store(dst + pairs + i * kVec, y);
    } else {
      const int at = (pair_units + i) * kVec;
      *reinterpret_cast<uint4*>(dst + at) = *reinterpret_cast<const uint4*>(src + at);
    }
  }
}

template <typename T>
int launch(d3tom_ctx* ctx, const RotateArgs& a, const RopeTable& t, bool to_cache, cudaStream_t s) {
  constexpr int kVec = Storage<T>::kVec;
  const int units = (a.H + 2 * a.kv_heads) * a.dh / kVec;
  const int want = ceil_div(2 * ctx->sm_count, a.rows), most = ceil_div(units, kThreads);
  const dim3 grid(a.rows, want < 1 ? 1 : want < most ? want : most);
  const bool vector = t.neighbours || t.pairs % kVec == 0;
  if (vector) D3TOM_CUDA_TRY(ctx, launch_serialized(rotate_rows_kernel<T, true>, grid, kThreads, 0, s, a, t, to_cache));
  else D3TOM_CUDA_TRY(ctx, launch_serialized(rotate_rows_kernel<T, false>, grid, kThreads, 0, s, a, t, to_cache));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

}  // namespace

int launch_rotate(d3tom_ctx* ctx, d3tom_dtype dt, const RotateArgs& a, const RopeTable& t, bool to_cache, cudaStream_t s) {
  return dt == D3TOM_BF16 ? launch<__nv_bfloat16>(ctx, a, t, to_cache, s) : launch<float>(ctx, a, t, to_cache, s);
}

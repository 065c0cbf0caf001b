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

// Where a row goes in the pools; -1: nowhere.
__device__ __forceinline__ long long row_place(const RotateArgs& a, int row) {
  const int b = find_segment(a.cu_rows, a.B, row);
  const long long slot = (long long)a.cache.length[b] - a.cu_rows[b + 1] + row;
  if (slot < 0 || slot >= (long long)a.cache.max_pages * a.cache.page_size) return -1;
  const int p = (int)slot / a.cache.page_size, page = a.cache.page_table[(size_t)b * a.cache.max_pages + p];
  return page < 0 || page >= a.cache.pages ? -1 : (long long)page * a.cache.page_size + ((int)slot - p * a.cache.page_size);
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
    place = row_place(a, row);
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

// Heads that are rotated whole (2 pairs = dh): a warp takes a row, or a part of its heads where there are few rows.  U lanes have a head, a
// lane always the same pairs of every head, so their cosines and sines stay in registers; 64 bytes of loads per lane are under
// way at a time (with 128 a wave of blocks does not fit the SMs), the first ones before the angles are known.  Heads of 128 bf16, us, with
// the kernel above (angles from shared memory for every unit, a barrier per row) / here: 4288 rows x 64 heads 27.8 / 25.7 (5.5 TB/s),
// 21629 rows x (64 + 32) appended 201 / 171 (6.2 TB/s).
constexpr int kHeadWarps = 4;

template <typename T, bool kNeighbours, int U>
__global__ void __launch_bounds__(kHeadWarps * 32, 8)
rotate_heads_kernel(const RotateArgs a, const __grid_constant__ RopeTable t, const bool to_cache, const int parts) {
  constexpr int kVec = Storage<T>::kVec, kPairs = kNeighbours ? kVec / 2 : kVec, kHeads = 32 / U, kHeadBatch = kNeighbours ? 4 : 2;
  // lanes index the table apart, which the constant bank serves one after the other: once per block (1000 rows: 9.3 -> 6.6 us)
  __shared__ unsigned long long turn[64];
  __shared__ int axis[64];
  if (threadIdx.x < t.pairs) { turn[threadIdx.x] = t.turn[threadIdx.x]; axis[threadIdx.x] = t.axis[threadIdx.x]; }
  __syncthreads();
  const int lane = threadIdx.x & 31, w = blockIdx.x * kHeadWarps + (threadIdx.x >> 5);
  const int row = w / parts, part = w - row * parts;
  if (row >= a.rows) return;
  grid_dependency_enter();
  if (to_cache && row >= a.cu_rows[a.B]) return;
  const int dh = a.dh, heads = a.H + a.kv_heads, step = parts * kHeads, at = (lane % U) * kVec, half = dh / 2;
  const size_t width = (size_t)a.kv_heads * dh;
  const T* q = static_cast<const T*>(a.q) + (size_t)row * a.H * dh + at;
  const T* k = static_cast<const T*>(a.k) + (size_t)row * width + at;
  uint4 lo[kHeadBatch], hi[kHeadBatch];
  auto load = [&](int h0) {
#pragma unroll
    for (int j = 0; j < kHeadBatch; ++j) {
      const int h = h0 + j * step;
      if (h < heads) {
        const T* src = h < a.H ? q + (size_t)h * dh : k + (size_t)(h - a.H) * dh;
        lo[j] = *reinterpret_cast<const uint4*>(src);
        if (!kNeighbours) hi[j] = *reinterpret_cast<const uint4*>(src + half);
      }
    }
  };
  int h = part * kHeads + lane / U;
  load(h);
  // the angles: lane i has pairs i and i + 32, then every lane collects those of its place in a head
  float c[2] = {1.f, 1.f}, s[2] = {0.f, 0.f};
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int pr = lane + j * 32;
    if (pr < t.pairs) {
      const long long pos = a.positions[(size_t)row * t.axes + axis[pr]];
      const int32_t x = (int32_t)(((unsigned long long)pos * turn[pr]) >> 32);
      sincospif((float)x * 4.656612873077392578125e-10f, &s[j], &c[j]);
      if (a.inverse) s[j] = -s[j];
    }
  }
  float cs[kPairs], sn[kPairs];
#pragma unroll
  for (int e = 0; e < kPairs; ++e) {
    const int pr = (lane % U) * kPairs + e;
    const float c0 = __shfl_sync(0xffffffffu, c[0], pr & 31), c1 = __shfl_sync(0xffffffffu, c[1], pr & 31);
    const float s0 = __shfl_sync(0xffffffffu, s[0], pr & 31), s1 = __shfl_sync(0xffffffffu, s[1], pr & 31);
    cs[e] = pr < 32 ? c0 : c1;
    sn[e] = pr < 32 ? s0 : s1;
  }
  long long place = row;                         // of the row in the keys' destination
  if (to_cache) {
    place = row_place(a, row);
    if (part == 0 && lane == 0) {
      if (place < 0) atomicExch(a.dev_status, D3TOM_ERR_INVALID_ARG);
      else {
        if (a.cache.weight != nullptr) a.cache.weight[place] = a.first_weight != nullptr ? a.first_weight[row] : 0.f;
        if (a.tokens != nullptr) a.cache.token[place] = a.tokens[row];
      }
    }
  }
  T* q_out = static_cast<T*>(a.q_out) + (size_t)row * a.H * dh + at;
  T* k_out = static_cast<T*>(to_cache ? a.cache.k : a.k_out) + (size_t)(place < 0 ? 0 : place) * width + at;
  for (; h < heads; h += kHeadBatch * step) {
    if (h != part * kHeads + lane / U) load(h);
#pragma unroll
    for (int j = 0; j < kHeadBatch; ++j) {
      const int hj = h + j * step;
      if (hj >= heads || (hj >= a.H && place < 0)) continue;
      T* dst = hj < a.H ? q_out + (size_t)hj * dh : k_out + (size_t)(hj - a.H) * dh;
      float x[kVec], y[kVec];
      Storage<T>::load(reinterpret_cast<const T*>(&lo[j]), x);
      if constexpr (kNeighbours) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          const float p = x[2 * e], r = x[2 * e + 1];
          y[2 * e] = p * cs[e] - r * sn[e];
          y[2 * e + 1] = p * sn[e] + r * cs[e];
        }
        Storage<T>::store(dst, y);
      } else {
        Storage<T>::load(reinterpret_cast<const T*>(&hi[j]), y);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          const float p = x[e] * cs[e] - y[e] * sn[e];
          y[e] = x[e] * sn[e] + y[e] * cs[e];
          x[e] = p;
        }
        Storage<T>::store(dst, x);
        Storage<T>::store(dst + half, y);
      }
    }
  }
  if (a.v != nullptr && place >= 0) {
    const uint4* src = reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + (size_t)row * width);
    uint4* dst = reinterpret_cast<uint4*>(static_cast<T*>(a.cache.v) + (size_t)place * width);
    const int units = (int)(width / kVec);
    for (int u = part * 32 + lane; u < units; u += kHeadBatch * 32 * parts) {
#pragma unroll
      for (int j = 0; j < kHeadBatch; ++j) if (u + j * 32 * parts < units) lo[j] = src[u + j * 32 * parts];
#pragma unroll
      for (int j = 0; j < kHeadBatch; ++j) if (u + j * 32 * parts < units) dst[u + j * 32 * parts] = lo[j];
    }
  }
}

template <typename T, bool kNeighbours, int U>
int launch_heads(d3tom_ctx* ctx, const RotateArgs& a, const RopeTable& t, bool to_cache, cudaStream_t s) {
  const int steps = ceil_div(a.H + a.kv_heads, 32 / U), want = ceil_div(24 * ctx->sm_count, a.rows);
  const int parts = want < steps ? want : steps;
  D3TOM_CUDA_TRY(ctx, launch_serialized(rotate_heads_kernel<T, kNeighbours, U>, (int)(((long long)a.rows * parts + kHeadWarps - 1) / kHeadWarps),
                                        kHeadWarps * 32, 0, s, a, t, to_cache, parts));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

template <typename T>
int launch(d3tom_ctx* ctx, const RotateArgs& a, const RopeTable& t, bool to_cache, cudaStream_t s) {
  constexpr int kVec = Storage<T>::kVec;
  const int lanes = 2 * t.pairs != a.dh ? 0 : t.neighbours ? a.dh / kVec : t.pairs % kVec == 0 ? t.pairs / kVec : 0;   // of a whole head
  switch (lanes) {
    case 4: if (!t.neighbours) return launch_heads<T, false, 4>(ctx, a, t, to_cache, s); break;
    case 8: return t.neighbours ? launch_heads<T, true, 8>(ctx, a, t, to_cache, s) : launch_heads<T, false, 8>(ctx, a, t, to_cache, s);
    case 16: return t.neighbours ? launch_heads<T, true, 16>(ctx, a, t, to_cache, s) : launch_heads<T, false, 16>(ctx, a, t, to_cache, s);
    case 32: if (t.neighbours) return launch_heads<T, true, 32>(ctx, a, t, to_cache, s); break;
    default: break;
  }
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

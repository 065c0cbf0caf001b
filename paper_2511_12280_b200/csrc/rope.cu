// Rotary positions (d3tom_rope) and the rows that go into a cache in pages (d3tom_cache_append).
//
// A pair (a, b) of a head becomes (a cos t - b sin t, a sin t + b cos t), t = position * theta^-e.  A position step is held as a
// 64-bit fraction of a turn, so position * step is an integer product that wraps around where the angle does, and what it is off by
// at any position is the table's error times the position (in fp32 the product itself would be off by radians from a million on);
// sincospif needs no range reduction.  The angles of a row are shared by its heads: a warp computes them once.  Bound: HBM (every
// row is read and written once); with few rows, latency.
#include "common.cuh"

namespace {

constexpr int kRowWarps = 4;

// Where a row goes in the pools; -1: nowhere.
__device__ __forceinline__ long long row_place(const RotateArgs& a, int row) {
  const int b = find_segment(a.cu_rows, a.B, row);
  const long long slot = (long long)a.cache.length[b] - a.cu_rows[b + 1] + row;
  if (slot < 0 || slot >= (long long)a.cache.max_pages * a.cache.page_size) return -1;
  const int p = (int)slot / a.cache.page_size, page = a.cache.page_table[(size_t)b * a.cache.max_pages + p];
  return page < 0 || page >= a.cache.pages ? -1 : (long long)page * a.cache.page_size + ((int)slot - p * a.cache.page_size);
}

// The angles of a row, for a warp: cosine and sine of pairs lane and lane + 32 (c, s [2]).
template <typename Turn, typename Axis>
__device__ __forceinline__ void row_angles(const RotateArgs& a, const RopeTable& t, const Turn& turn, const Axis& axis, int row,
                                           float (&c)[2], float (&s)[2]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int pr = (threadIdx.x & 31) + j * 32;
    c[j] = 1.f; s[j] = 0.f;
    if (pr < t.pairs) {
      const long long pos = a.positions[(size_t)row * t.axes + axis[pr]];
      // in 2^-64 of a turn, -1/2 .. 1/2: the 25 upper bits, which fp32 holds, and the small rest d (below 2e-7 radians, taken to 2^-48
      // of a turn) by cos(x + d) = cos x - d sin x, sin(x + d) = sin x + d cos x
      const unsigned long long part = (unsigned long long)pos * turn[pr];
      const int32_t upper = (int32_t)(part >> 32) & ~127;
      const float d = (float)(int32_t)((part >> 16) & 0x7fffffu) * (3.14159265358979f * 0x1p-47f);
      sincospif((float)upper * 0x1p-31f, &s[j], &c[j]);                              // in half turns
      const float c0 = c[j];
      c[j] = fmaf(-s[j], d, c0);
      s[j] = fmaf(c0, d, s[j]);
      if (a.inverse) s[j] = -s[j];
    }
  }
}

// Where the row goes, for a warp; its weight and token's number are written by the row's first part.
__device__ __forceinline__ long long row_place_and_marks(const RotateArgs& a, int row, bool first) {
  const long long place = row_place(a, row);
  if (first) {
    if (place < 0) report_invalid(a.dev_status);
    else {
      if (a.cache.weight != nullptr) a.cache.weight[place] = a.first_weight != nullptr ? a.first_weight[row] : 0.f;
      if (a.tokens != nullptr) a.cache.token[place] = a.tokens[row];
    }
  }
  return place;
}

// W numbers of type T as one load or store
template <typename T, int W> struct Pack {
  static constexpr int kBytes = sizeof(T) * W;
  T e[W];
  __device__ __forceinline__ void load(const T* p) { copy(reinterpret_cast<const uint8_t*>(p), reinterpret_cast<uint8_t*>(e)); }
  __device__ __forceinline__ void store(T* p) const { copy(reinterpret_cast<const uint8_t*>(e), reinterpret_cast<uint8_t*>(p)); }
  __device__ static __forceinline__ void copy(const uint8_t* src, uint8_t* dst) {
    if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(src);
    else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(dst) = *reinterpret_cast<const uint32_t*>(src);
    else *reinterpret_cast<uint16_t*>(dst) = *reinterpret_cast<const uint16_t*>(src);
  }
};

// Any rotation: a warp takes a row, or a part of its units where there are few rows.  A unit is W numbers of either half of the pairs (or W
// neighbouring numbers), W the largest power of two up to 16 bytes that divides them; a number between the pairs and the first 16-byte
// boundary after them; or 16 bytes of what is only copied, values included.
template <typename T, int W, bool kNeighbours>
__global__ void __launch_bounds__(kRowWarps * 32)
rotate_rows_kernel(const RotateArgs a, const __grid_constant__ RopeTable t, const bool to_cache, const int parts) {
  constexpr int kVec = Storage<T>::kVec;
  __shared__ unsigned long long turn[64];
  __shared__ int axis[64];
  __shared__ float2 angle[kRowWarps][64];
  if (threadIdx.x < t.pairs) { turn[threadIdx.x] = t.turn[threadIdx.x]; axis[threadIdx.x] = t.axis[threadIdx.x]; }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = blockIdx.x * kRowWarps + warp, row = w / parts, part = w - row * parts;
  if (row >= a.rows) return;
  grid_dependency_enter();
  if (to_cache && row >= a.cu_rows[a.B]) return;
  if (t.pairs > 0) {
    float c[2], s[2];
    row_angles(a, t, turn, axis, row, c, s);
    angle[warp][lane] = make_float2(c[0], s[0]);
    angle[warp][lane + 32] = make_float2(c[1], s[1]);
    __syncwarp();
  }
  const long long place = to_cache ? row_place_and_marks(a, row, part == 0 && lane == 0) : row;
  const int pairs = t.pairs, dh = a.dh, first = (2 * pairs + kVec - 1) / kVec;   // 16-byte pieces of a head that are only copied, from here on
  const int pair_units = kNeighbours ? 2 * pairs / W : pairs / W, single = first * kVec - 2 * pairs;
  const int per_head = pair_units + single + dh / kVec - first;
  const int rot_units = (a.H + a.kv_heads) * per_head, units = rot_units + (a.v != nullptr ? a.kv_heads * (dh / kVec) : 0);
  const size_t width = (size_t)a.kv_heads * dh;
  const float2* cs = angle[warp];
#pragma unroll 2
  for (int u = part * 32 + lane; u < units; u += parts * 32) {
    const T* src;
    T* dst;
    int i = pair_units + single;                 // a copied piece at src
    if (u >= rot_units) {
      if (place < 0) continue;
      const size_t off = (size_t)(u - rot_units) * kVec;
      src = static_cast<const T*>(a.v) + (size_t)row * width + off;
      dst = static_cast<T*>(a.cache.v) + (size_t)place * width + off;
    } else {
      const int head = u / per_head;
      i = u - head * per_head;
      if (head < a.H) {
        const size_t off = ((size_t)row * a.H + head) * dh;
        src = static_cast<const T*>(a.q) + off;
        dst = static_cast<T*>(a.q_out) + off;
      } else {
        if (place < 0) continue;
        const size_t off = (size_t)(head - a.H) * dh;
        src = static_cast<const T*>(a.k) + (size_t)row * width + off;
        dst = static_cast<T*>(to_cache ? a.cache.k : a.k_out) + (size_t)place * width + off;
      }
      if (i >= pair_units + single) {
        const int at = (first + i - pair_units - single) * kVec;
        src += at; dst += at;
        i = pair_units + single;
      }
    }
    if (i >= pair_units + single) {
      *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
    } else if (i >= pair_units) {
      dst[2 * pairs + i - pair_units] = src[2 * pairs + i - pair_units];
    } else if constexpr (kNeighbours) {
      Pack<T, W> x;
      x.load(src + i * W);
#pragma unroll
      for (int e = 0; e < W; e += 2) {
        const float2 f = cs[(i * W + e) >> 1];
        const float p = Storage<T>::to_float(x.e[e]), r = Storage<T>::to_float(x.e[e + 1]);
        x.e[e] = Storage<T>::from_float(p * f.x - r * f.y);
        x.e[e + 1] = Storage<T>::from_float(p * f.y + r * f.x);
      }
      x.store(dst + i * W);
    } else {
      Pack<T, W> x, y;
      x.load(src + i * W);
      y.load(src + pairs + i * W);
#pragma unroll
      for (int e = 0; e < W; ++e) {
        const float2 f = cs[i * W + e];
        const float p = Storage<T>::to_float(x.e[e]), r = Storage<T>::to_float(y.e[e]);
        x.e[e] = Storage<T>::from_float(p * f.x - r * f.y);
        y.e[e] = Storage<T>::from_float(p * f.y + r * f.x);
      }
      x.store(dst + i * W);
      y.store(dst + pairs + i * W);
    }
  }
}

// Heads that are rotated whole (2 pairs = dh): a warp takes a row, or a part of its heads where there are few rows.  U lanes have a head, a
// lane always the same pairs of every head, so their cosines and sines stay in registers; 64 bytes of loads per lane are under
// way at a time (with 128 a wave of blocks does not fit the SMs), the first ones before the angles are known.  Heads of 128 bf16, us, with
// a block per row (angles from shared memory for every unit, a barrier) / here: 4288 rows x 64 heads 27.8 / 25.7 (5.5 TB/s),
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
  float c[2], s[2];
  row_angles(a, t, turn, axis, row, c, s);
  float cs[kPairs], sn[kPairs];
#pragma unroll
  for (int e = 0; e < kPairs; ++e) {
    const int pr = (lane % U) * kPairs + e;
    const float c0 = __shfl_sync(0xffffffffu, c[0], pr & 31), c1 = __shfl_sync(0xffffffffu, c[1], pr & 31);
    const float s0 = __shfl_sync(0xffffffffu, s[0], pr & 31), s1 = __shfl_sync(0xffffffffu, s[1], pr & 31);
    cs[e] = pr < 32 ? c0 : c1;
    sn[e] = pr < 32 ? s0 : s1;
  }
  // of the row in the keys' destination
  const long long place = to_cache ? row_place_and_marks(a, row, part == 0 && lane == 0) : row;
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
  // the widest unit that divides the pairs of a half (or the neighbouring numbers)
  int unit = kVec;
  while (unit > (t.neighbours ? 2 : 1) && (t.neighbours ? 2 * t.pairs : t.pairs) % unit != 0) unit >>= 1;
  auto kernel = t.neighbours ? rotate_rows_kernel<T, 2, true> : rotate_rows_kernel<T, 1, false>;
  if (unit == 8) { if constexpr (kVec == 8) kernel = t.neighbours ? rotate_rows_kernel<T, 8, true> : rotate_rows_kernel<T, 8, false>; }
  else if (unit == 4) kernel = t.neighbours ? rotate_rows_kernel<T, 4, true> : rotate_rows_kernel<T, 4, false>;
  else if (unit == 2) kernel = t.neighbours ? rotate_rows_kernel<T, 2, true> : rotate_rows_kernel<T, 2, false>;
  // warps enough to hide that a lane has one or two loads under way, each with at least four steps after its angles: 4288 rows of
  // 64 heads, 30 of 64 pairs rotated, 89 us with 24 warps per SM, 56 with 48
  const int steps = ceil_div((a.H + 2 * a.kv_heads) * a.dh / unit, 32), want = ceil_div(48 * ctx->sm_count, a.rows);
  const int most = steps < 4 ? 1 : steps / 4, parts = want < most ? want : most;
  D3TOM_CUDA_TRY(ctx, launch_serialized(kernel, (int)(((long long)a.rows * parts + kRowWarps - 1) / kRowWarps), kRowWarps * 32, 0, s, a, t, to_cache, parts));
  D3TOM_LAUNCH_CHECK(ctx);
  return D3TOM_OK;
}

}  // namespace

int launch_rotate(d3tom_ctx* ctx, d3tom_dtype dt, const RotateArgs& a, const RopeTable& t, bool to_cache, cudaStream_t s) {
  return dt == D3TOM_BF16 ? launch<__nv_bfloat16>(ctx, a, t, to_cache, s) : launch<float>(ctx, a, t, to_cache, s);
}

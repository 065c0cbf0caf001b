// Which CTA attends to which keys of a cache in pages, and how the kernels of d3tom_attn_cached find slots.
//
// A work item is (request, key head, up to `tile_rows` of the request's rows x query heads of that key head); its keys
// come in tiles of 128 slots.  The tiles of all items, in order, are dealt to the CTAs in equal runs: CTA c of C has
// tiles [c W / C, (c + 1) W / C) of W, so a batch of very uneven lengths and one very long request load the SMs alike.
// A run covers any number of whole items and at most one item's end at its beginning and one item's beginning at its
// end: two partial results per CTA, kept at part[c][0] (the run's first segment) and part[c][1] (its last).  What each
// CTA does follows from the lengths alone, so results do not depend on timing, and lengths that change between replays
// of a graph are followed without the host.
#pragma once

#include "common.cuh"

constexpr int kKeyTile = 128;

struct CachedRequest {
  int len, n, lo;               // slots, new rows, first packed row
};
__device__ __forceinline__ CachedRequest cached_request(const CachedArgs& a, int b) {
  CachedRequest r;
  const int len = a.length[b];
  const int lo = min(max(a.cu_rows[b], 0), a.total_rows), hi = min(max(a.cu_rows[b + 1], 0), a.total_rows);
  r.len = min(max(len, 0), a.cap);
  r.lo = lo;
  r.n = max(hi - lo, 0);
  return r;
}
__device__ __forceinline__ int cached_row_tiles(const CachedArgs& a, int n) {
  return (n * a.group + a.tile_rows - 1) / a.tile_rows;     // (all rows x heads of a call fit 31 bits, less a tile)
}
__device__ __forceinline__ int cached_key_tiles(int len) { return (len + kKeyTile - 1) / kKeyTile; }
__device__ __forceinline__ long long cached_work(const CachedArgs& a, const CachedRequest& r) {
  return (long long)a.kv_heads * cached_row_tiles(a, r.n) * cached_key_tiles(r.len);
}

// A CTA's run, and the request it begins in.
struct CachedRun {
  long long w0, w1, base, total;   // tiles [w0, w1) of `total`; the first tile of request b
  int b, ctas;                     // ctas that have work
};
// (a 64-bit division is some 300 cycles on the way to a CTA's first load: 32 bits where they do)
__device__ __forceinline__ long long cached_div(long long x, int y) {
  return (x >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}
__device__ __forceinline__ long long cached_run_begin(long long total, int ctas, int c) { return cached_div(total * c, ctas); }

// Whole warp; the same answer in all lanes.  (One pass over the lengths where a warp's lanes have them all: this lies on every
// call's way to its first load.)
__device__ __forceinline__ CachedRun cached_run(const CachedArgs& a, int cta) {
  const int lane = threadIdx.x & 31;
  auto work_of = [&](int b) { return b < a.B ? cached_work(a, cached_request(a, b)) : 0ll; };
  auto scan = [&](long long v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, v, o);
      if (lane >= o) v += t;
    }
    return v;
  };
  const long long mine0 = work_of(lane), incl0 = scan(mine0);
  long long total = __shfl_sync(0xffffffffu, incl0, 31);
  for (int b0 = 32; b0 < a.B; b0 += 32) total += __shfl_sync(0xffffffffu, scan(work_of(b0 + lane)), 31);
  CachedRun run;
  run.total = total;
  run.ctas = total < a.ctas ? (int)total : a.ctas;
  if (a.B == 1 && total > a.ctas) {
    // one request: as many CTAs as its items share evenly, if that is at most a tile more for each; none then ends one item and
    // begins another, which costs it a second first tile and a second result
    const CachedRequest r = cached_request(a, 0);
    const int items = a.kv_heads * cached_row_tiles(a, r.n);
    if (items <= a.ctas) {
      const int even = a.ctas / items * items;
      if (total * (a.ctas - even) <= (long long)a.ctas * even) run.ctas = even;
    }
  }
  run.b = 0; run.base = 0; run.w0 = run.w1 = total;
  if (cta >= run.ctas) return run;
  run.w0 = cached_run_begin(total, run.ctas, cta);
  run.w1 = cached_run_begin(total, run.ctas, cta + 1);
  long long before = 0, mine = mine0, incl = incl0;
  for (int b0 = 0; ; ) {
    const unsigned hit = __ballot_sync(0xffffffffu, before + incl > run.w0);
    if (hit != 0u) {                              // (w0 < total: some request has it)
      const int src = __ffs(hit) - 1;
      run.b = b0 + src;
      run.base = before + __shfl_sync(0xffffffffu, incl - mine, src);
      return run;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
    b0 += 32;
    if (b0 >= a.B) return run;
    mine = work_of(b0 + lane);
    incl = scan(mine);
  }
}

// The segments of a run, one after the other.
struct CachedSegment {
  int b, len, lo, n, rows;      // request, its slots, its first packed row, its rows; rows x query heads of the tile
  int kv_head, row0;            // key head; the tile's first (row x query head)
  int t0, t1;                   // key tiles
  bool whole;                   // the item has no other segment
  int slot;                     // of part[cta] otherwise
};
struct CachedWalk {
  long long w, w_begin, w_end, base, work;
  int b, tiles, row_tiles;
  CachedRequest r;

  __device__ __forceinline__ void enter(const CachedArgs& a) {
    r = cached_request(a, b);
    tiles = cached_key_tiles(r.len);
    row_tiles = cached_row_tiles(a, r.n);
    work = (long long)a.kv_heads * row_tiles * tiles;
  }
  __device__ __forceinline__ void start(const CachedArgs& a, const CachedRun& run) {
    w = w_begin = run.w0; w_end = run.w1; base = run.base; b = run.b;
    if (w < w_end) enter(a);
  }
  __device__ __forceinline__ bool next(const CachedArgs& a, CachedSegment& s) {
    if (w >= w_end) return false;
    while (w >= base + work) { base += work; ++b; enter(a); }
    const long long rel = w - base;
    const int item = (int)cached_div(rel, tiles);
    s.t0 = (int)(rel - (long long)item * tiles);
    s.t1 = (int)min((long long)tiles, s.t0 + (w_end - w));
    s.whole = s.t0 == 0 && s.t1 == tiles;
    s.slot = w == w_begin ? 0 : 1;
    s.b = b; s.len = r.len; s.lo = r.lo; s.n = r.n;
    s.kv_head = item / row_tiles;
    s.row0 = (item - s.kv_head * row_tiles) * a.tile_rows;
    s.rows = (int)min((long long)a.tile_rows, (long long)r.n * a.group - s.row0);
    w += s.t1 - s.t0;
    return true;
  }
};

// Where a CTA keeps its part of an item: O of the tile's rows, then M of all rows, then l.
__device__ __forceinline__ size_t cached_part_stride(const CachedArgs& a) {
  return ((size_t)a.tile_rows * (a.dh + 2) + 3) & ~(size_t)3;
}

// What the join has to do for a run whose first segment is the end of an item: written by one thread per CTA.
struct CachedJoin {
  int first, n;                 // the item's first part (2 * CTA + slot); CTAs that have a part; 0: nothing to join
  int lo, rows, kv_head, row0, pad0, pad1;
};
// s: the run's first segment, of an item of `tiles` key tiles
__device__ __forceinline__ void cached_write_join(const CachedArgs& a, const CachedRun& run, int cta, const CachedSegment& s, int tiles) {
  CachedJoin j = {};
  if (run.w0 < run.w1 && s.t0 > 0 && s.t1 == tiles) {
    const long long begin = run.w0 - s.t0;
    int c0 = (int)(begin * run.ctas / run.total);
    while (cached_run_begin(run.total, run.ctas, c0) > begin) --c0;
    while (cached_run_begin(run.total, run.ctas, c0 + 1) <= begin) ++c0;
    j.first = 2 * c0 + (cached_run_begin(run.total, run.ctas, c0) == begin ? 0 : 1);
    j.n = cta - c0 + 1;
    j.lo = s.lo; j.rows = s.rows; j.kv_head = s.kv_head; j.row0 = s.row0;
  }
  int4* dst = reinterpret_cast<int4*>(a.joins) + 2 * cta;
  dst[0] = make_int4(j.first, j.n, j.lo, j.rows);
  dst[1] = make_int4(j.kv_head, j.row0, 0, 0);
}

// What no run has: zeros for the rows of requests without slots, and the word on lengths that do not fit.  `threads` threads of
// every CTA, this one the `tid`-th of them: whole warps.  All CTAs share such a request's rows, 16 bytes at a time (8 where rows are odd
// multiples of that).  (By one warp of one CTA, a number at a time / so, us: 40 rows x 32 heads x 128 of an empty request 24.4 / 2.9, seven
// blocks of 32 rows over 1088 slots beside one over none 34.8 / 29.6.)
template <typename T>
__device__ __forceinline__ void cached_write_empty(const CachedArgs& a, int tid, int threads) {
  const int lane = threadIdx.x & 31, row_bytes = a.H * a.dh * (int)sizeof(T);
  auto zero = [&](auto unit, const CachedRequest& r) {
    using U = decltype(unit);
    U* out = reinterpret_cast<U*>(static_cast<uint8_t*>(a.out) + (size_t)r.lo * row_bytes);
    const size_t count = (size_t)r.n * (row_bytes / sizeof(U));
    for (size_t i = (size_t)blockIdx.x * threads + tid; i < count; i += (size_t)gridDim.x * threads) out[i] = U{};
  };
  for (int b0 = 0; b0 < a.B; b0 += 32) {
    const int b = b0 + lane;
    bool empty = false;
    if (b < a.B) {
      const CachedRequest r = cached_request(a, b);
      empty = r.len == 0 && r.n > 0;
      const int raw = a.length[b];
      if (blockIdx.x == 0 && (raw < 0 || raw > a.cap)) report_invalid(a.dev_status);
    }
    for (unsigned left = __ballot_sync(0xffffffffu, empty); left != 0u; left &= left - 1u) {
      const CachedRequest r = cached_request(a, b0 + __ffs(left) - 1);
      if (row_bytes % 16 == 0) zero(uint4(), r);
      else zero(uint2(), r);
    }
  }
}

// The rank of row x query head f of a request among all [total_rows * H]: packed row * H + query head.
__device__ __forceinline__ int cached_row_index(const CachedArgs& a, const CachedSegment& s, int r) {
  const int f = s.row0 + r, i = f / a.group;
  return (s.lo + i) * a.H + s.kv_head * a.group + (f - i * a.group);
}

// Where the raw scores of a request (n rows from packed row lo on, `len` slots) are kept: key tile by key tile, in a tile key head by
// key head and row x query head by row x query head, 128 keys each (the last tile as many as it has, rounded up to four).  So what a
// CTA writes per tile is one piece, and what the weights of a tile's slots are summed from is another.  (Row by row of
// all slots, 512 bytes here and there / so, us: eight blocks of 4 rows x 32 heads 79.8 / 73.3, 4 rows x 32 heads on 8 34.4 / 31.7.)
struct CachedScores { float* tile; int pitch; };
__device__ __forceinline__ CachedScores cached_scores(const CachedArgs& a, int lo, int n, int len, int t) {
  const int left = len - t * kKeyTile;
  CachedScores s;
  s.tile = a.scores + (size_t)lo * a.H * a.score_stride + (size_t)t * kKeyTile * (n * a.H);
  s.pitch = left >= kKeyTile ? kKeyTile : (left + 3) & ~3;
  return s;
}

// The slot's place in the pools, -1 where its page is not one of them.
__device__ __forceinline__ long long cached_place(const int32_t* table, int slot, int page_size, int pages) {
  const int p = slot / page_size, page = table[p];
  return page < 0 || page >= pages ? -1 : (long long)page * page_size + (slot - p * page_size);
}

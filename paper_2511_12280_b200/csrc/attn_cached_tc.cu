// Attention of new rows over a cache in pages on the tensor cores, bf16, head_dim 64 or 128 (d3tom_attn_cached).
//
// One token has as many rows per key head as query heads share it, a response block some more: far fewer than the 128 rows of
// a tensor-core tile.  So the products are taken the other way round, with the KEYS as the 128 rows and the new rows x query heads
// as N = 16 .. 128 columns:
//   S^T [128 keys x N] = K Q^T        A = a tile of K as it lies in the cache, B = the rows of Q
//   O^T [dh x N]      += V^T P^T      A = a tile of V, read along dh (its transpose costs nothing), B = P in shared memory
// and no part of a tile is padding but the columns between the rows there are and the next of 16, 32, 64, 128.  The cache is read
// once, by TMA, a page (or its largest power-of-two part) per copy, through a ring of four to ten tiles that runs ahead across work
// items: bound by HBM up to 32 columns at head_dim 128 (one token of 131071 slots x 8 key heads in 89 us, 6.0 TB/s; eight blocks of 32
// rows x 32 heads over up to 4288 slots 62 us of 54) and 16 at 64.  With more it is the softmax warps' way through a tile: the same with
// 64 rows 79 us, with 128 rows 131, some 7000 cycles a tile of which exponentials are a seventh; 64 columns in a thread are more than
// its 168 registers (312 bytes of spills at 128 columns, 72 at 64 x 128, 88 at 32 x 64).
//
// Softmax over the keys is a sum over lanes here.  A thread has one key's scores of all columns; the running maximum is only a
// reference that has to lie within 2^8 of the true one (exact after the final division), so a tile costs one barrier that asks
// whether any score outgrew it, and only a segment's first tile and the rare one that did take maxima over the lanes.  Sums stay
// per lane until the segment ends.  Scores, maxima and sums are fp32; P is rounded to bf16 for the second product (2^-8 of
// each term at most, unbiased), as in the other attention kernels.
//
// The mass per slot.  With few columns the raw scores go out (4 bytes per column, slot and key head, written and read again) and a
// small kernel weighs them once M and l are known.  From some number of columns on that is more than the keys themselves: then the
// same kernel runs a second time over the keys alone (kMass), takes the scores again, the same bits, and sums 2^(s c - M) f / l
// over its columns, one number per slot and tile (launch_attn_cached_tc has the rule and what both take).
//
//   warps 0 .. 3 (or 0 .. 7, a half of the columns each)  softmax and epilogue, a key / a number of O per thread
//   then one warp each: MMA issue, Q rows into shared memory, TMA producer of K, TMA producer of V
// A CTA per SM (two at head_dim 64 up to 32 columns) walks its run of key tiles (cache_walk.cuh).  Every wait is bounded; after one that ran out the softmax
// warps go through the rest of their run without waiting (their barriers need all of them), the other warps stop.
#include "cache_walk.cuh"
#include "ptx.cuh"

namespace {

template <int DH, int N> struct Shape {
  // softmax warpgroups, each with its part of the columns (one / two, us: blocks of 32 rows x 32 heads x 128 68 / 65, of 64 rows 91 /
  // 84; of 32 rows x 64, with two CTAs per SM instead, 49 / 52)
  static constexpr int kGroups = N >= 64 || (N == 32 && DH == 128) ? 2 : 1;
  static constexpr int kCols = N / kGroups;                 // columns per softmax thread
  static constexpr int kSoftmaxWarps = 4 * kGroups;
  static constexpr int kThreads = (kSoftmaxWarps + 4) * 32;
  static constexpr int kSlotBytes = kKeyTile * DH * 2;
  // CTAs per SM: a tile of head_dim 64 has half the bytes but as long a way through softmax (some 1900 cycles, against 1400 for its
  // bytes), so two of them run side by side where their shared memory allows (64 requests, up to 8192 slots, 32 / 16 heads x 64:
  // 249 -> 205 us; blocks of 32 rows 60 -> 51)
  static constexpr int kPerSm = DH == 64 && N <= 32 ? 2 : 1;
  static constexpr bool kScores = DH == 128 ? N <= 64 : N == 16;   // whether raw scores ever go out (attn_cached_mass_columns)
  static constexpr int kQBufs = DH * N >= 128 * 128 ? 1 : 2;
  static constexpr int kSlots = DH == 128 ? (N <= 32 ? 6 : 4) : N == 16 ? 6 : N == 32 ? 4 : N == 64 ? 10 : 8;
  static_assert(kSlots % 2 == 0, "K tiles in the even slots, V tiles in the odd ones: no slot has two producers");
  static constexpr int kQBytes = N * DH * 2;
  static constexpr int kPBytes = N * kKeyTile * 2;
  static constexpr int kFloats = N * 7;                     // reference, factor, four warps' values, row numbers
  static constexpr int kBars = 2 * kSlots + 2 * 2 + 2 + 2 + 1;
  static constexpr int kBytes = 1024 + kSlots * kSlotBytes + kQBufs * kQBytes + kPBytes + kFloats * 4 + kBars * 8 + 64;
  static_assert(kPerSm * (kBytes + 1024) <= 228 * 1024, "shared memory of an SM");
  static constexpr uint32_t kTmemCols = N == 16 ? 64 : 4 * N;   // S twice and O: 3 N, as a power of two
};

// Sums of C values per lane over the warp's lanes: afterwards lane i has the sum of value i (C = 16: i and i + 16 both have it).
template <int C>
__device__ __forceinline__ float lane_sums(float (&v)[C]) {
#pragma unroll
  for (int h = C / 2; h > 0; h >>= 1) {
    const bool up = (threadIdx.x & h) != 0;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float send = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, h);
    }
  }
  if (C == 16) v[0] += __shfl_xor_sync(0xffffffffu, v[0], 16);
  return v[0];
}

template <int DH, int N, bool kMass>
__global__ void __launch_bounds__(Shape<DH, N>::kThreads, Shape<DH, N>::kPerSm)
attn_cached_tc_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v, const CachedArgs a,
                      const int box) {
  using S = Shape<DH, N>;
  constexpr int kCols = S::kCols, kSlots = S::kSlots;
  constexpr int kHalfBytes = kKeyTile * 128;            // 64 numbers of a tile's keys: 128 rows x 128 bytes
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* kv_s = smem;                                 // ring: K_0, V_0, K_1, V_1, ..
  uint8_t* q_s = kv_s + kSlots * S::kSlotBytes;
  uint8_t* p_s = q_s + S::kQBufs * S::kQBytes;
  float* negm_s = reinterpret_cast<float*>(p_s + S::kPBytes);   // [N] minus the reference (log2 domain)
  float* alpha_s = negm_s + N;                          // [N] factor of what was summed before; at the end the sums
  float* red_s = alpha_s + N;                           // [4][N]
  int* row_s = reinterpret_cast<int*>(red_s + 4 * N);   // [N] row number of each column, -1 for none
  uint64_t* bars = reinterpret_cast<uint64_t*>(row_s + N);
  uint64_t* kv_full = bars;                             // [kSlots]
  uint64_t* kv_empty = kv_full + kSlots;                // [kSlots]
  uint64_t* q_full = kv_empty + kSlots;                 // [2]
  uint64_t* q_empty = q_full + 2;                       // [2]
  uint64_t* s_full = q_empty + 2;                       // [2]
  uint64_t* p_full = s_full + 2;                        // [2] (kMass: a tile's scores have been read; otherwise the first alone, P written)
  uint64_t* pv_done = p_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(pv_done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile uint32_t* bad_boxes = tmem_slot + 2;         // [8] per key tile: boxes whose page is not one of the pool's

  const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kSlots; ++i) { ptx::mbar_init(&kv_full[i], 1); ptx::mbar_init(&kv_empty[i], 1); }
    for (int i = 0; i < 2; ++i) { ptx::mbar_init(&q_full[i], 1); ptx::mbar_init(&q_empty[i], 1); ptx::mbar_init(&s_full[i], 1); }
    for (int i = 0; i < 2; ++i) ptx::mbar_init(&p_full[i], S::kSoftmaxWarps);
    ptx::mbar_init(pv_done, 1);
    *abort_flag = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 0) { ptx::tmem_alloc(tmem_slot, S::kTmemCols); ptx::tmem_relinquish(); }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  constexpr uint32_t kColO = 2 * N;
  grid_dependency_enter();
  const CachedRun run = cached_run(a, blockIdx.x);
  CachedWalk walk;
  walk.start(a, run);
  CachedSegment s;

  if (warp >= S::kSoftmaxWarps + 2) {
    // ------------------------------------------------------------ TMA producers, one for K and one for V: a lane per page part
    const int kind = warp - (S::kSoftmaxWarps + 2);     // (kMass: nobody wants V)
    const CUtensorMap* tmap = kind == 0 ? &tmap_k : &tmap_v;
    if (lane == 0) ptx::prefetch_tensormap(tmap);
    const int boxes = kKeyTile / box, outside = a.pages * a.page_size;
    // what is read once need not push the scores out of L2.  (Keeping the keys there for a second pass cost more than it gave:
    // 32 rows x 32 heads 110 -> 119 us.)
    const uint64_t policy = ptx::l2_policy(a.read_once != 0);
    int ring = kind, issued = 0, tile = 0;
    uint32_t phase = 1;                                 // of the ring's `empty` barriers: the first round finds them so
    bool ok = true;
    while (ok && (!kMass || kind == 0) && walk.next(a, s)) {
      const int32_t* table = a.page_table + (size_t)s.b * a.max_pages;
      auto find = [&](int t) -> int {                   // row of this lane's box in the pool; behind its end: nothing, zeros
        const int slot = t * kKeyTile + lane * box;
        if (lane >= boxes || slot >= s.len) return outside;
        const long long at = cached_place(table, slot, a.page_size, a.pages);
        return at < 0 ? -1 : (int)at;
      };
      int row = find(s.t0);
      for (int t = s.t0; t < s.t1; ++t, ++tile) {
        const uint32_t bad = __ballot_sync(0xffffffffu, row < 0);
        if (row < 0) { row = outside; report_invalid(a.dev_status); }
        const int next_row = t + 1 < s.t1 ? find(t + 1) : outside;
        ok = __all_sync(0xffffffffu, ptx::mbar_wait(&kv_empty[ring], phase, abort_flag, a.dev_status));
        if (!ok) break;
        if (lane == 0 && kind == 0) bad_boxes[tile & 7] = bad;   // (at most seven tiles ahead of the softmax warps)
        if (lane == 0) ptx::mbar_arrive_expect_tx(&kv_full[ring], S::kSlotBytes);
        __syncwarp();
        if (lane < boxes)
#pragma unroll
          for (int hf = 0; hf < DH / 64; ++hf)
            ptx::tma_load_2d_hint(kv_s + ring * S::kSlotBytes + hf * kHalfBytes + lane * box * 128, tmap, &kv_full[ring],
                                  s.kv_head * DH + hf * 64, row, policy);
        ++issued;
        ring += 2;
        if (ring >= kSlots) { ring -= kSlots; phase ^= 1u; }
        row = next_row;
      }
    }
    if (!ok) {                                          // copies under way land before the CTA leaves
      for (int i = 0; i < kSlots / 2 && i < issued; ++i) {
        ring -= 2;
        if (ring < 0) { ring += kSlots; phase ^= 1u; }
        ptx::mbar_wait(&kv_full[ring], phase ^ 1u, abort_flag, a.dev_status);
      }
    }
  } else if (warp == S::kSoftmaxWarps) {
    // ------------------------------------------------------------ MMA issue
    if (ptx::elect_one()) {
      constexpr uint32_t idesc_qk = ptx::idesc_bf16_f32(kKeyTile, N, 0, 0);    // both along dh
      constexpr uint32_t idesc_pv = ptx::idesc_bf16_f32(128, N, 1, 0);         // V along dh, which are its rows here
      const ptx::SmemDesc q_desc0 = ptx::smem_desc_kmajor_sw128(ptx::smem_u32(q_s));
      const ptx::SmemDesc p_desc = ptx::smem_desc_kmajor_sw128(ptx::smem_u32(p_s));
      const ptx::SmemDesc k_desc0 = ptx::smem_desc_kmajor_sw128(ptx::smem_u32(kv_s));
      // head_dim 64: the upper 64 rows of the product repeat the lower ones (block distance 0) and are not read
      const ptx::SmemDesc v_desc0 = ptx::smem_desc_mnmajor_sw128(ptx::smem_u32(kv_s), DH == 128 ? kHalfBytes : 0);
      int k_ring = 0, v_ring = 1, tile = 0, seg = 0;
      uint32_t k_phase = 0, v_phase = 0;
      bool ok = true, v_first = false;
      auto advance = [&](int& ring, uint32_t& phase) { ring += 2; if (ring >= kSlots) { ring -= kSlots; phase ^= 1u; } };
      auto issue_pv = [&](int t) {                      // of tile t, whose V is at v_ring
        if constexpr (kMass) {                          // (its scores have been read, that is all)
          ok = ptx::mbar_wait(&p_full[t & 1], (uint32_t)(t >> 1) & 1u, abort_flag, a.dev_status);
          return;
        }
        ok = ptx::mbar_wait(&kv_full[v_ring], v_phase, abort_flag, a.dev_status) &&
             ptx::mbar_wait(p_full, (uint32_t)t & 1u, abort_flag, a.dev_status);
        if (!ok) return;
        ptx::tc_fence_after_sync();
        const ptx::SmemDesc vd = ptx::smem_desc_advance(v_desc0, v_ring * S::kSlotBytes);
#pragma unroll
        for (int kk = 0; kk < kKeyTile / 16; ++kk)
          ptx::mma_ss(tmem + kColO, ptx::smem_desc_advance(vd, kk * 2048),
                      ptx::smem_desc_advance(p_desc, (kk / 4) * (N * 128) + (kk % 4) * 32), idesc_pv, v_first && kk == 0 ? 0u : 1u);
        ptx::mma_commit(&kv_empty[v_ring]);
        ptx::mma_commit(pv_done);
        advance(v_ring, v_phase);
      };
      while (ok && walk.next(a, s)) {
        const int qb = S::kQBufs == 2 ? seg & 1 : 0;
        ok = ptx::mbar_wait(&q_full[qb], (uint32_t)(seg / S::kQBufs) & 1u, abort_flag, a.dev_status);
        const ptx::SmemDesc qd = ptx::smem_desc_advance(q_desc0, qb * S::kQBytes);
        for (int t = s.t0; t < s.t1 && ok; ++t, ++tile) {
          ok = ptx::mbar_wait(&kv_full[k_ring], k_phase, abort_flag, a.dev_status);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const ptx::SmemDesc kd = ptx::smem_desc_advance(k_desc0, k_ring * S::kSlotBytes);
#pragma unroll
          for (int kk = 0; kk < DH / 16; ++kk)          // (S buffer tile & 1: its last reader announced P_(tile-2) since)
            ptx::mma_ss(tmem + (uint32_t)(tile & 1) * N, ptx::smem_desc_advance(kd, (kk / 4) * kHalfBytes + (kk % 4) * 32),
                        ptx::smem_desc_advance(qd, (kk / 4) * (N * 128) + (kk % 4) * 32), idesc_qk, kk > 0 ? 1u : 0u);
          ptx::mma_commit(&s_full[tile & 1]);
          ptx::mma_commit(&kv_empty[k_ring]);
          if (t + 1 == s.t1) ptx::mma_commit(&q_empty[qb]);
          advance(k_ring, k_phase);
          if (tile > 0) issue_pv(tile - 1);
          v_first = t == s.t0;
        }
        ++seg;
      }
      if (ok && tile > 0) issue_pv(tile - 1);
    }
  } else if (warp == S::kSoftmaxWarps + 1) {
    // ------------------------------------------------------------ Q rows, 128-byte swizzle, a segment ahead
    bool ok = true;
    CachedSegment head = {};                            // the run's first segment
    int head_tiles = 0;
    for (int seg = 0; ok && walk.next(a, s); ++seg) {
      const int qb = S::kQBufs == 2 ? seg & 1 : 0;
      if (seg == 0) { head = s; head_tiles = walk.tiles; }
      if (seg >= S::kQBufs)
        ok = __all_sync(0xffffffffu, ptx::mbar_wait(&q_empty[qb], (uint32_t)(seg / S::kQBufs - 1) & 1u, abort_flag, a.dev_status));
      if (!ok) break;
      // asynchronous copies, so that all of a tile's are under way at once; rows that are not there become zeros.  (With loads through
      // registers, eight at a time, and a division per row this was 10 us at 128 columns.)
      constexpr int kChunks = DH / 8, kStep = 32 / kChunks;       // 16-byte pieces of a row; rows per step of the warp
      const int piece = lane % kChunks, di = kStep / a.group, dg = kStep - di * a.group;
      int r = lane / kChunks;
      const int i = (s.row0 + r) / a.group;
      int g = s.row0 + r - i * a.group;
      const size_t token = (size_t)a.H * DH * 2;        // bytes of a packed row, and how far a step goes
      const uint8_t* src = static_cast<const uint8_t*>(a.q) + (size_t)(s.lo + i) * token + (size_t)(s.kv_head * a.group + g) * (DH * 2) + piece * 16;
      const size_t on = di * token + (size_t)dg * (DH * 2), wrap = token - (size_t)a.group * (DH * 2);
      const uint32_t dst = ptx::smem_u32(q_s + qb * S::kQBytes + (piece / 8) * (N * 128));
#pragma unroll 4
      for (; r < N; r += kStep) {
        const bool there = r < s.rows;
        ptx::cp_async_16(dst + r * 128 + (((piece ^ r) & 7) << 4), there ? src : a.q, there);
        src += on;
        g += dg;
        if (g >= a.group) { g -= a.group; src += wrap; }
      }
      ptx::cp_async_wait_all();
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&q_full[qb]);
    }
    if constexpr (!kMass) {
      if (lane == 0) cached_write_join(a, run, blockIdx.x, head, head_tiles);
      cached_write_empty<__nv_bfloat16>(a, lane, 32);
    }
  } else {
    // ------------------------------------------------------------ softmax and epilogue
    const int quarter = warp & 3, group = warp >> 2, col0 = group * kCols;
    const int key = quarter * 32 + lane;                // of the tile; and the number of O this thread writes out
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16;
    const int bar = 1 + group, gt = threadIdx.x & 127;
    const float c = a.scale_log2;
    uint8_t* p_base = p_s + (key >> 6) * (N * 128) + (key & 7) * 2;
    const uint32_t chunk = (uint32_t)(key & 63) >> 3;
    float l[kCols], e[kCols];
    int tile = 0, v_ring = 1;
    uint32_t v_phase = 0;
    auto load_scores = [&](uint32_t buf, bool valid) {
      const uint32_t at = tmem + lane_addr + buf * N + col0;
      if constexpr (kCols == 16) ptx::tmem_ld16(at, reinterpret_cast<uint32_t*>(e));
      else {
#pragma unroll
        for (int i = 0; i < kCols; i += 32) ptx::tmem_ld32(at + i, reinterpret_cast<uint32_t*>(e) + i);
      }
      ptx::tmem_wait_ld();
      if (!valid)
#pragma unroll
        for (int i = 0; i < kCols; ++i) e[i] = -INFINITY;
    };
    if constexpr (kMass) {
      while (walk.next(a, s)) {
        ptx::named_sync(bar, 128);                      // (the last segment's columns are done with)
        const int cols = min(kCols, s.rows - col0);
        if (gt < kCols) {
          float m = 0.f, f = 0.f;
          if (gt < cols) {
            const int row = cached_row_index(a, s, col0 + gt);
            const float2 ml = a.lse[row];
            m = -ml.x;
            f = ml.y == 0.f ? 0.f : (a.row_weight != nullptr ? a.row_weight[row / a.H] : 1.f) / ml.y;
          }
          negm_s[col0 + gt] = m;
          alpha_s[col0 + gt] = f;
        }
        ptx::named_sync(bar, 128);
        float* mass = cols > 0 ? a.mass + (size_t)cached_row_index(a, s, col0) * a.score_stride : nullptr;
        for (int t = s.t0; t < s.t1; ++t, ++tile) {
          const int slot = t * kKeyTile + key;
          ptx::mbar_wait(&s_full[tile & 1], (uint32_t)(tile >> 1) & 1u, abort_flag, a.dev_status);
          ptx::tc_fence_after_sync();
          load_scores(tile & 1, true);
          ptx::tc_fence_before_sync();
          __syncwarp();
          // two barriers: nothing holds a warp back from the next tile's scores, which are there, before the others have read
          // these; the tile after that one waits for all of them
          if (lane == 0) ptx::mbar_arrive(&p_full[tile & 1]);
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < kCols; ++i)
            if (i < cols) sum += alpha_s[col0 + i] * ptx::ex2(fmaf(e[i], c, negm_s[col0 + i]));
          if (mass != nullptr && slot < s.len) mass[slot] = sum;
        }
      }
    }
    while (!kMass && walk.next(a, s)) {
      // (the barrier at the end of the last segment lies behind every use of row_s)
      if (gt < kCols) row_s[col0 + gt] = col0 + gt < s.rows ? cached_row_index(a, s, col0 + gt) : -1;
      const int cols = min(kCols, s.rows - col0);       // columns in use (none or less: padding only)
      for (int t = s.t0; t < s.t1; ++t, ++tile) {
        const int slot = t * kKeyTile + key;
        ptx::mbar_wait(&s_full[tile & 1], (uint32_t)(tile >> 1) & 1u, abort_flag, a.dev_status);
        ptx::tc_fence_after_sync();
        const uint32_t bad = bad_boxes[tile & 7];
        const bool valid = slot < s.len && (bad == 0u || ((bad >> (key / box)) & 1u) == 0u);
        const bool first = t == s.t0;
        load_scores(tile & 1, valid);
        bool grown = false;
        if (first) {
          ptx::named_sync(bar, 128);                    // (row_s)
        }
        // the raw scores leave once P is announced, beside the second product (32 rows x 32 heads 114 -> 110 us)
        float raw[S::kScores ? kCols : 1];
        if constexpr (S::kScores) {
#pragma unroll
          for (int i = 0; i < kCols; ++i) raw[i] = e[i];
        }
        auto put_scores = [&](auto& x) {
          if (!S::kScores || a.scores == nullptr || !valid) return;
          const CachedScores sc = cached_scores(a, s.lo, s.n, s.len, t);
          float* at = sc.tile + (size_t)(s.kv_head * s.n * a.group + s.row0 + col0) * sc.pitch + key;
#pragma unroll
          for (int i = 0; i < kCols; ++i)
            if (i < cols) at[i * sc.pitch] = x[i];
        };
        if (!first) {
          float top = -INFINITY;
#pragma unroll
          for (int i = 0; i < kCols; ++i) { e[i] = fmaf(e[i], c, negm_s[col0 + i]); top = fmaxf(top, e[i]); }
          grown = ptx::named_sync_or(bar, 128, top > 8.f);
        }
        if (first || grown) {
          if (grown) load_scores(tile & 1, valid);
          float mine[(kCols + 31) / 32];
#pragma unroll
          for (int i = 0; i < kCols; ++i) {
            const float top = ptx::warp_max_redux(e[i]);
            if (lane == (i & 31)) mine[i / 32] = top;
          }
#pragma unroll
          for (int i = 0; i < (kCols + 31) / 32; ++i)
            if (i * 32 + lane < kCols) red_s[quarter * N + col0 + i * 32 + lane] = mine[i];
          ptx::named_sync(bar, 128);
          if (gt < kCols) {
            const float* r = red_s + col0 + gt;
            const float top = fmaxf(fmaxf(r[0], r[N]), fmaxf(r[2 * N], r[3 * N])) * c;
            const float old = first ? INFINITY : negm_s[col0 + gt];
            // a column without a score so far gets a reference far below every score: the next tile that has one finds it grown
            const float now = fminf(fminf(old, -top), 1e38f);
            negm_s[col0 + gt] = now;
            alpha_s[col0 + gt] = first ? 0.f : ptx::ex2(now - old);
          }
          ptx::named_sync(bar, 128);
#pragma unroll
          for (int i = 0; i < kCols; ++i) e[i] = fmaf(e[i], c, negm_s[col0 + i]);
          if (grown) {                                  // what was summed so far moves to the new reference
            ptx::mbar_wait(pv_done, (uint32_t)(tile - 1) & 1u, abort_flag, a.dev_status);
            ptx::tc_fence_after_sync();
#pragma unroll 1
            for (int i0 = 0; i0 < kCols; i0 += 16) {
              uint32_t o[16];
              ptx::tmem_ld16(tmem + lane_addr + kColO + col0 + i0, o);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha_s[col0 + i0 + i]);
              ptx::tmem_st16(tmem + lane_addr + kColO + col0 + i0, o);
            }
            ptx::tmem_wait_st();
#pragma unroll
            for (int i = 0; i < kCols; ++i) l[i] *= alpha_s[col0 + i];
          }
        }
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          e[i] = ptx::ex2(e[i]);
          l[i] = first ? e[i] : l[i] + e[i];
        }
        if (tile > 0) ptx::mbar_wait(pv_done, (uint32_t)(tile - 1) & 1u, abort_flag, a.dev_status);   // P has been read
#pragma unroll
        for (int i = 0; i < kCols; ++i)
          *reinterpret_cast<__nv_bfloat16*>(p_base + (col0 + i) * 128 + ((chunk ^ (uint32_t)(i & 7)) << 4)) = __float2bfloat16_rn(e[i]);
        if (s.len - t * kKeyTile < kKeyTile) {
          // the request's last tile: what the pages hold behind its last slot may be anything, and 0 x NaN is not 0
          ptx::mbar_wait(&kv_full[v_ring], v_phase, abort_flag, a.dev_status);
          if (slot >= s.len && group == 0) {
            uint8_t* v = kv_s + v_ring * S::kSlotBytes + key * 128;
#pragma unroll
            for (int hf = 0; hf < DH / 64; ++hf)
#pragma unroll
              for (int i = 0; i < 8; ++i) *reinterpret_cast<uint4*>(v + hf * kHalfBytes + i * 16) = make_uint4(0u, 0u, 0u, 0u);
          }
        }
        v_ring += 2;
        if (v_ring >= kSlots) { v_ring -= kSlots; v_phase ^= 1u; }
        ptx::fence_proxy_async_smem();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(p_full);
        if constexpr (S::kScores) put_scores(raw);
      }
      // ---- the segment's result
      constexpr int kSum = kCols < 32 ? kCols : 32;
#pragma unroll
      for (int i0 = 0; i0 < kCols; i0 += kSum) {
        float v[kSum];
#pragma unroll
        for (int i = 0; i < kSum; ++i) v[i] = l[i0 + i];
        const float sum = lane_sums<kSum>(v);
        if (lane < kSum) red_s[quarter * N + col0 + i0 + lane] = sum;
      }
      ptx::named_sync(bar, 128);
      float* part = a.part + ((size_t)blockIdx.x * 2 + s.slot) * (N * (DH + 2));
      if (gt < kCols) {
        const float* r = red_s + col0 + gt;
        const float sum = (r[0] + r[N]) + (r[2 * N] + r[3 * N]);
        if (gt < cols) {
          if (s.whole) { if (a.lse != nullptr) a.lse[row_s[col0 + gt]] = make_float2(-negm_s[col0 + gt], sum); }
          else { part[N * DH + col0 + gt] = -negm_s[col0 + gt]; part[N * (DH + 1) + col0 + gt] = sum; }
        }
        alpha_s[col0 + gt] = sum == 0.f ? 0.f : 1.f / sum;
      }
      ptx::mbar_wait(pv_done, (uint32_t)(tile - 1) & 1u, abort_flag, a.dev_status);
      ptx::tc_fence_after_sync();
      ptx::named_sync(bar, 128);
      constexpr int kOut = kCols < 32 ? kCols : 32;
#pragma unroll 1
      for (int i0 = 0; i0 < kCols; i0 += kOut) {
        if (i0 >= cols) break;
        uint32_t o[kOut];
        if constexpr (kOut == 16) ptx::tmem_ld16(tmem + lane_addr + kColO + col0 + i0, o);
        else ptx::tmem_ld32(tmem + lane_addr + kColO + col0 + i0, o);
        ptx::tmem_wait_ld();
        if (key < DH) {
          if (s.whole) {
#pragma unroll
            for (int i = 0; i < kOut; ++i) {
              const int col = col0 + i0 + i;
              if (i0 + i < cols)
                static_cast<__nv_bfloat16*>(a.out)[(size_t)row_s[col] * DH + key] = __float2bfloat16_rn(__uint_as_float(o[i]) * alpha_s[col]);
            }
          } else {
            float* to = part + (col0 + i0) * DH + key;
#pragma unroll
            for (int i = 0; i < kOut; ++i)
              if (i0 + i < cols) to[i * DH] = __uint_as_float(o[i]);
          }
        }
      }
      ptx::tc_fence_before_sync();
      ptx::named_sync(bar, 128);                        // shared memory and O may be written again
    }
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) ptx::tmem_dealloc(tmem, S::kTmemCols);
}

// What a launch takes apart from the arguments: the tensor maps and the rows per copy.
struct CacheMaps { CUtensorMap k, v; int box; };
int make_maps(d3tom_ctx* ctx, const CachedArgs& a, CacheMaps* m) {
  m->box = kKeyTile;                                    // rows per copy: a power of two that divides the page
  while (a.page_size % m->box != 0) m->box >>= 1;
  const uint64_t rows = (uint64_t)a.pages * a.page_size, cols = (uint64_t)a.kv_heads * a.dh;
  int r = make_tmap_bf16_2d(&m->k, a.k, rows, cols, cols, (uint32_t)m->box, 64, a.dh == 64);
  if (r == 0) r = make_tmap_bf16_2d(&m->v, a.v, rows, cols, cols, (uint32_t)m->box, 64, a.dh == 64);
  if (r != 0) { ctx->last_cuda_error = r; return D3TOM_ERR_CUDA; }
  return D3TOM_OK;
}

template <int DH, int N>
int launch(d3tom_ctx* ctx, CachedArgs a, bool mass, cudaStream_t s) {
  using Sh = Shape<DH, N>;
  CacheMaps m;
  const int st = make_maps(ctx, a, &m);
  if (st != D3TOM_OK) return st;
  a.tile_rows = N;
  a.read_once = (long long)a.max_rows * a.group <= N;
  a.ctas = Sh::kPerSm * ctx->sm_count;
  if (mass) a.scores = nullptr;
  auto kernel = attn_cached_tc_kernel<DH, N, false>;
  D3TOM_CUDA_TRY(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes));
  D3TOM_CUDA_TRY(ctx, launch_serialized(kernel, a.ctas, Sh::kThreads, Sh::kBytes, s, m.k, m.v, a, m.box));
  D3TOM_LAUNCH_CHECK(ctx);
  const int joined = launch_attn_cached_join(ctx, D3TOM_BF16, a, s);
  if (joined != D3TOM_OK || !mass) return joined;
  if constexpr (N > 16) {                               // (so few columns never ask for a second pass)
    auto again = attn_cached_tc_kernel<DH, N, true>;
    D3TOM_CUDA_TRY(ctx, cudaFuncSetAttribute(again, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kBytes));
    D3TOM_CUDA_TRY(ctx, launch_serialized(again, a.ctas, Sh::kThreads, Sh::kBytes, s, m.k, m.v, a, m.box));
    D3TOM_LAUNCH_CHECK(ctx);
  }
  return D3TOM_OK;
}

template <int DH>
int launch_columns(d3tom_ctx* ctx, const CachedArgs& a, bool mass, cudaStream_t s) {
  const long long rows = (long long)a.max_rows * a.group;
  if (rows <= 16) return launch<DH, 16>(ctx, a, mass, s);
  if (rows <= 32) return launch<DH, 32>(ctx, a, mass, s);
  if (rows <= 64) return launch<DH, 64>(ctx, a, mass, s);
  return launch<DH, 128>(ctx, a, mass, s);
}

}  // namespace

// Whether the mass per slot comes from a second pass over the keys; the columns whose sums are then one number, 0 if not.
// Per slot and key head the scores are 8 bytes a column, written and read, the keys 2 dh bytes and a pass has its own ramp.  us, scores
// out / second pass, eight requests of up to 4288 slots: 32 heads x 128, 24 rows 98 / 112, 32 108 / 112, 40 137 / 123; 32 x 64, 17 rows
// 84 / 76, 24 92 / 78; 32 heads on 8 x 64, 5 rows (20 columns) 39 / 35; ten requests of up to 5345, 8 heads on one x 128, 32 rows 86 / 54.
int attn_cached_mass_columns(const CachedArgs& a) {
  const long long rows = (long long)a.max_rows * a.group;
  if (rows < (a.dh == 128 ? 40 : 17)) return 0;
  if (a.dh == 128) return rows <= 32 ? Shape<128, 32>::kCols : rows <= 64 ? Shape<128, 64>::kCols : Shape<128, 128>::kCols;
  return rows <= 32 ? Shape<64, 32>::kCols : rows <= 64 ? Shape<64, 64>::kCols : Shape<64, 128>::kCols;
}

int launch_attn_cached_tc(d3tom_ctx* ctx, const CachedArgs& a, cudaStream_t s) {
  const bool mass = a.scores != nullptr && attn_cached_mass_columns(a) > 0;
  if (a.dh == 128) return launch_columns<128>(ctx, a, mass, s);
  if (a.dh == 64) return launch_columns<64>(ctx, a, mass, s);
  return D3TOM_ERR_UNSUPPORTED;
}

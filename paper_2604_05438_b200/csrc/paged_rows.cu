// Attention of few query rows over a paged cache: sequences with at most 16 rows (tokens x query heads of a KV head: one
// token of a group of 16, four of a group of 4), and the page-selected form, where every token of a KV head reads a page list
// of its own.
//
//   y = sum_t p_t v_t / sum_t p_t,  p_t = exp(scale * q.k_t - m),  lse = m + log sum_t p_t   over the visible keys t
//
// in one pass with the running maximum m and sum.  A unit is up to 16 query rows of one KV head (tokens x query heads
// of the group), so that the group's heads share every key and value read.  Bound: memory, 2 * 2 * head_dim bytes per
// key against 16 rows of work.  The 16-row mma.sync tile is therefore the right size of matrix instruction (a
// tcgen05 tile has 64 rows at least, and its accumulators would have to come back from tensor memory for every
// tile); what carries the kernel is the TMA ring that keeps copies in flight:
//   - one producer warp: a tile of 64 keys and their values is a handful of page boxes (lane = one box); page ids are
//     read 32 at a time, one batch ahead;
//   - compute warps, each with 16 keys of a tile and a running softmax of its own, so that nothing is exchanged between
//     warps until a unit ends; rows are rescaled only when a maximum moved.
// Probabilities enter the second product as hi + lo pairs of the element type (2^-16 relative for bf16): that costs
// 16 extra matrix instructions per tile, which the kernel has time for, and leaves the output's own rounding as the
// only one of its size.  fp16 has few exponents: there the probabilities are scaled by 2^14 (the largest is then 2^14, since
// m is the maximum), so that a pair holds them to 2^-22 relative down to 2^-17 of the largest and to 2^-39 of the largest
// below that; the sum carries the same factor, and the maximum that is handed on has it taken off.  (Without it terms below
// 2^-25 of the largest vanished from y but stayed in the sum.)
// Work is dealt out in one of two ways.  Long caches: the tiles of all units form one line, cut into as many equal pieces
// as there are resident CTAs; a unit that is cut leaves partial results, joined in a fixed order by a second, dependent
// kernel.  Short ones and short page lists: a unit is cut into up to eight pieces, the CTAs of one cluster, which join
// theirs through distributed shared memory (no second launch, no trip through global memory): 8.7 us against 14.3 for one
// token over 4096 keys of 32 / 8 heads of 64.
// Measured: 32 sequences of 8K-64K tokens, 24 / 8 heads of 128: 638 us = 6.7 TB/s of keys and values, the rate of a copy.
#include "paged.cuh"

namespace tkphi {

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Two floats at shared-memory address p of the cluster's CTA `rank`.
__device__ __forceinline__ float2 ld_cluster_f2(const float* p, int rank) {
  uint32_t a;
  float2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
  return v;
}

// The cluster form has few CTAs, where the time is latency: eight compute warps (four for the even, four for the odd
// tiles) and one CTA per multiprocessor.  Otherwise four warps and two CTAs, so that one works while the other begins or
// ends a unit (page-selected form, 236 tokens x 65 pages of 32: 307 us, with eight warps 383).
template <int D, bool SPLIT>
struct RowCfg {
  static constexpr int WARPS = SPLIT ? 8 : 4;
  static constexpr int THREADS = (WARPS + 1) * 32;
  static constexpr int HALVES = D / 64;
  static constexpr int HALF = kRowKeys * 128;               // bytes of one 64-dim half of a 64-key tile
  static constexpr int TILE = HALVES * HALF;                // keys or values of a tile
  static constexpr int STAGE = 2 * TILE;
  static constexpr int NS = (D == 128 ? 3 : 6) * (SPLIT ? 2 : 1);
  static constexpr size_t red = (size_t)NS * STAGE;         // [warps][16 rows][64 dims] fp32
  static constexpr size_t stat = red + WARPS * kRowTile * 64 * 4;   // [warps][16][2]
  static constexpr size_t bars = stat + WARPS * kRowTile * 2 * 4;
  static constexpr size_t total = bars + (2 * NS) * 8 + 16;
  // cluster form: [16][D] piece of this CTA and [16][2] its statistics, over the ring's first tiles (a CTA has one
  // piece there, and writes it when its warps have read all of them)
  static constexpr size_t keep = 0;
  static_assert(kRowTile * (D + 2) * 4 <= NS * STAGE, "piece");
};

// The pieces of one CTA: (unit, tile range) one after the other.  Every warp runs its own copy.
template <bool BLOCK, bool SPLIT>
struct RowWalk {
  const PagedProblem& p;
  // current piece
  int b, h, tok0, rows, len, pos0;      // sequence, KV head, first token of the unit (global), rows, cache length, position of row 0
  int r_first;                          // first row of the unit within its sequence (0 in the block form)
  int t0, t1, tiles;                    // tile range of the piece, tiles of the unit
  int unit;                             // block form: token * hkv + head
  int n_list;                           // block form: pages of the unit's list
  // line position
  int f, f1, seq_start, seq_end, seq_tiles, seq_rows, seq_tok0, seq_len, seq_q;

  __device__ __forceinline__ void load_seq(int s) {
    seq_tiles = 0; seq_rows = 0; seq_tok0 = 0; seq_len = 0; seq_q = 0;
    if (s < p.batch) {
      seq_tok0 = (int)__ldg(p.cu_q + s);
      seq_q = paged_q_len(p, s);
      seq_len = paged_kv_len(p, s);
      seq_rows = seq_q > 0 ? seq_q * p.group : 0;
      if (seq_rows > p.rows_limit) seq_rows = 0;
      seq_tiles = seq_len > 0 ? (seq_len + kRowKeys - 1) / kRowKeys : 1;
    }
  }
  __device__ __forceinline__ int seq_weight() const { return seq_tiles * p.hkv * ((seq_rows + kRowTile - 1) / kRowTile); }

  __device__ __forceinline__ void split_tiles(int part) {
    const int per = (tiles + p.n_split - 1) / p.n_split;
    t0 = part * per < tiles ? part * per : tiles;
    t1 = t0 + per < tiles ? t0 + per : tiles;
    f1 = t0 < t1 ? 1 : 0;
  }
  __device__ __forceinline__ RowWalk(const PagedProblem& pr, int cta) : p(pr) {
    const int lane = threadIdx.x & 31;
    f = f1 = 0;
    if (BLOCK) {
      unit = cta / p.n_split;
      const int part = cta % p.n_split, tok = unit / p.hkv;
      h = unit % p.hkv;
      b = paged_seq_of(p, tok);
      len = paged_kv_len(p, b);
      tok0 = tok; rows = p.group; r_first = 0;
      pos0 = len - paged_q_len(p, b) + (tok - (int)__ldg(p.cu_q + b));
      if (pos0 < 0) pos0 = 0;                           // (a device length below the new tokens' number)
      const int seen = (pos0 >> p.page_shift) + 1;
      n_list = seen < p.n_keep ? seen : p.n_keep;
      tiles = ((n_list << p.page_shift) + kRowKeys - 1) / kRowKeys;
      split_tiles(part);
      return;
    }
    if (SPLIT) {                                        // sequences of one row tile
      const int u = cta / p.n_split;
      b = u / p.hkv;
      h = u % p.hkv;
      load_seq(b);
      tiles = seq_tiles; r_first = 0; rows = seq_rows; tok0 = seq_tok0; len = seq_len; pos0 = seq_len - seq_q;
      t0 = t1 = 0;
      if (rows > 0) split_tiles(cta % p.n_split);
      return;
    }
    // the line: sequence by sequence, in a sequence row tile by row tile, head by head
    int total = 0;
    for (int s = 0; s < p.batch; s += 32) {
      load_seq(s + lane);
      total += __reduce_add_sync(0xffffffffu, seq_weight());
    }
    const int per = (total + p.row_ctas - 1) / p.row_ctas;
    f = per * cta < total ? per * cta : total;
    f1 = f + per < total ? f + per : total;
    if (f >= f1) return;
    int base = 0;
    b = 0;
    for (int s = 0; s < p.batch; s += 32) {
      load_seq(s + lane);
      const int w = seq_weight(), incl = warp_inclusive_scan(w) + base;
      const unsigned hit = __ballot_sync(0xffffffffu, incl > f);
      if (hit) {
        const int l = __ffs(hit) - 1;
        b = s + l;
        seq_start = __shfl_sync(0xffffffffu, incl - w, l);
        break;
      }
      base = __shfl_sync(0xffffffffu, incl, 31);
    }
    load_seq(b);
    seq_end = seq_start + seq_weight();
  }
  __device__ __forceinline__ bool next() {
    if (f >= f1) return false;
    if (BLOCK || SPLIT) { f = f1; return true; }
    while (f >= seq_end) {
      load_seq(++b);
      seq_start = seq_end;
      seq_end += seq_weight();
    }
    const int local = f - seq_start, u = local / seq_tiles;
    tiles = seq_tiles;
    t0 = local % seq_tiles;
    t1 = t0 + (f1 - f) < tiles ? t0 + (f1 - f) : tiles;
    f += t1 - t0;
    h = u % p.hkv;
    r_first = (u / p.hkv) * kRowTile;
    rows = seq_rows - r_first < kRowTile ? seq_rows - r_first : kRowTile;
    tok0 = seq_tok0;
    len = seq_len;
    pos0 = seq_len - seq_q;
    return true;
  }
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == tiles; }
  __device__ __forceinline__ int slot(int cta) const { return BLOCK ? cta : 2 * cta + (t0 == 0 ? 1 : 0); }
};

template <typename T, int D, bool BLOCK, bool SPLIT>
__global__ void __launch_bounds__(RowCfg<D, SPLIT>::THREADS, SPLIT ? 1 : 2)
paged_rows_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                  const __grid_constant__ PagedProblem p) {
  using C = RowCfg<D, SPLIT>;
  constexpr int kRowWarps = C::WARPS;
  constexpr int NS = C::NS;
  constexpr float kShift = T::kBf16 ? 0.f : 14.f;           // p = 2^kShift exp2(..)
  extern __shared__ __align__(1024) unsigned char smem[];
  float* red = reinterpret_cast<float*>(smem + C::red);
  float* stat = reinterpret_cast<float*>(smem + C::stat);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::bars);
  uint64_t* empty = full + NS;
  volatile int* s_abort = reinterpret_cast<int*>(empty + NS);
  float* keep = reinterpret_cast<float*>(smem + C::keep);
  float* keep_stat = keep + kRowTile * D;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cta = blockIdx.x;

  if (tid == 0) {
    for (int s = 0; s < NS; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 4); }
    mbar_fence_init();
    *s_abort = 0;
  }
  __syncthreads();
  // Inputs of the call may be read once all work before the call is complete.  The block form follows the selection,
  // which begins only then: the page lists alone remain to be waited for, by the producer.
  if (!BLOCK && !p.beside) pdl_wait();
  pdl_launch_next();

  if (warp == kRowWarps) {
    // ================================================================ TMA producer
    RowWalk<BLOCK, SPLIT> w(p, cta);
    if (BLOCK) pdl_wait();
    const int ps = 1 << p.page_shift;
    const int npg = ps < kRowKeys ? kRowKeys >> p.page_shift : 1;             // pages of a tile
    const int box_rows = ps < kRowKeys ? ps : kRowKeys;
    const int copies = 2 * C::HALVES * npg;
    const int which = lane / (C::HALVES * npg), half = (lane / npg) % C::HALVES, pg = lane % npg;
    const CUtensorMap* tm = which ? &tmap_v : &tmap_k;
    const uint64_t pol = BLOCK ? l2_policy_normal() : l2_policy_evict_first();
    const uint32_t dst_off = which * C::TILE + half * C::HALF + pg * box_rows * 128;
    int it = 0;
    bool ok = true;
    int issued[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) issued[s] = -1;
    while (ok && w.next()) {
      const int n_pages_unit = BLOCK ? w.n_list : (w.len + ps - 1) >> p.page_shift;
      const int* list = BLOCK ? p.page_list + (size_t)w.unit * p.n_keep : p.table + (size_t)w.b * p.max_pages;
      int batch0 = ((w.t0 * kRowKeys) >> p.page_shift) & ~31;
      int id = batch0 + lane < n_pages_unit ? (BLOCK ? __ldcg(list + batch0 + lane) : __ldg(list + batch0 + lane)) : p.n_pages;
      int id_next = batch0 + 32 + lane < n_pages_unit ? (BLOCK ? __ldcg(list + batch0 + 32 + lane) : __ldg(list + batch0 + 32 + lane)) : p.n_pages;
      for (int t = w.t0; t < w.t1; ++t, ++it) {
        const int stage = it % NS;
        const int first = (t * kRowKeys) >> p.page_shift;
        if (first >= batch0 + 32) {
          batch0 += 32;
          id = id_next;
          id_next = batch0 + 32 + lane < n_pages_unit ? (BLOCK ? __ldcg(list + batch0 + 32 + lane) : __ldg(list + batch0 + 32 + lane)) : p.n_pages;
        }
        int page = __shfl_sync(0xffffffffu, id, (first + pg) & 31);
        if (page < 0 || page > p.n_pages || (page == p.n_pages && first + pg < n_pages_unit)) {
          if (lane < npg) atomicExch(p.status, kStatusBadPage);
          page = p.n_pages;                     // a box outside the tensor arrives as zeros
        }
        ok = __all_sync(0xffffffffu, mbar_wait(&empty[stage], ((uint32_t)(it / NS) & 1u) ^ 1u, s_abort));
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(&full[stage], C::STAGE);
        __syncwarp();
        if (lane < copies)
          tma_load_4d(smem + (size_t)stage * C::STAGE + dst_off, tm, &full[stage], half * 64,
                      ps > kRowKeys ? (t & 1) * kRowKeys : 0, w.h, page, pol);
#pragma unroll
        for (int s = 0; s < NS; ++s)
          if (s == stage) issued[s] = it;
      }
    }
    if (*s_abort) {
      // every copy that was issued must land before shared memory is released
#pragma unroll
      for (int s = 0; s < NS; ++s)
        for (uint32_t n = 0; issued[s] >= 0 && n < kWaitPolls; ++n) {
          if (mbar_try_wait(&full[s], (uint32_t)(issued[s] / NS) & 1u)) break;
          __nanosleep(64);
        }
    }
  } else {
    // ================================================================ compute
    RowWalk<BLOCK, SPLIT> w(p, cta);
    const int ps = 1 << p.page_shift;
    const int rA = lane >> 2, rB = rA + 8, cc = 2 * (lane & 3);
    bool ok = true;
    int it = 0;
    while (w.next()) {
      // ---- the unit's queries as A operands: row r, dims 16 k ..
      uint32_t qf[D / 16][4];
      {
        const uint32_t* qa = nullptr;
        const uint32_t* qb = nullptr;
        const uint32_t* q = static_cast<const uint32_t*>(p.q);
        if (rA < w.rows) {
          const int r = w.r_first + rA;
          qa = q + ((size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group) * (D / 2);
        }
        if (rB < w.rows) {
          const int r = w.r_first + rB;
          qb = q + ((size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group) * (D / 2);
        }
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          qf[k][0] = qa ? __ldg(qa + k * 8 + (cc >> 1)) : 0u;
          qf[k][1] = qb ? __ldg(qb + k * 8 + (cc >> 1)) : 0u;
          qf[k][2] = qa ? __ldg(qa + k * 8 + 4 + (cc >> 1)) : 0u;
          qf[k][3] = qb ? __ldg(qb + k * 8 + 4 + (cc >> 1)) : 0u;
        }
      }
      // last visible position of this thread's rows; -1: no such row
      int limA = -1, limB = -1;
      if (rA < w.rows) limA = BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + rA) / p.group : w.len - 1;
      if (rB < w.rows) limB = BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + rB) / p.group : w.len - 1;
      // keys up to lim_all are visible to every row of the unit, keys behind lim_last (computed for every tile: there is no
      // register left for it) to none
      const int lim_all = BLOCK ? w.pos0 : p.causal ? w.pos0 + w.r_first / p.group : w.len - 1;
      float o[D / 8][4];
#pragma unroll
      for (int n = 0; n < D / 8; ++n) { o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f; }
      float mA = -INFINITY, mB = -INFINITY, lA = 0.f, lB = 0.f;

      for (int t = w.t0; t < w.t1; ++t, ++it) {
        if (SPLIT && (it & 1) != warp >> 2) continue;
        const int stage = it % NS;
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&full[stage], (uint32_t)(it / NS) & 1u, s_abort));
        if (!ok) continue;                                // the barriers below are still met
        unsigned char* ks = smem + (size_t)stage * C::STAGE;
        unsigned char* vs = ks + C::TILE;
        // position of this warp's first key (its 16 keys never straddle a page); in the block form only the last
        // page of a list can be partly visible, everything before it is
        const int kg = warp & 3;
        int key0 = t * kRowKeys + kg * 16;
        if (BLOCK) {
          const int entry = key0 >> p.page_shift;
          if (entry < w.n_list - 1) key0 = 0 - 16;                          // all visible
          else if (entry == w.n_list - 1) key0 = ((w.pos0 >> p.page_shift) << p.page_shift) + (key0 & (ps - 1));
          else key0 = w.len;                                                // past the list
        }
        const int lim_last = BLOCK ? w.pos0 : p.causal ? w.pos0 + (w.r_first + w.rows - 1) / p.group : w.len - 1;
        if (key0 <= lim_last) {
          bool odd_values = false;                          // a value that is not finite and that not every row sees
          float s[2][4];
#pragma unroll
          for (int n = 0; n < 2; ++n) { s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f; }
          {
            const int row = kg * 16 + ((lane >> 4) << 3) + (lane & 7), sub = (lane >> 3) & 1;
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
              uint32_t bf[4];
              ldmatrix_x4(bf, smem_u32(ks) + (k >> 2) * C::HALF + swz128(row, (2 * k + sub) & 7));
              T::mma(s[0], qf[k], bf[0], bf[1]);
              T::mma(s[1], qf[k], bf[2], bf[3]);
            }
          }
          if (key0 + 15 > lim_all) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int key = key0 + n * 8 + cc + e;
                if (key > limA) s[n][e] = -INFINITY;
                if (key > limB) s[n][2 + e] = -INFINITY;
              }
            // Values that no row sees may be anything (behind the sequence's end they may be left-overs): 0 times them must
            // not reach the product.  Those that some rows see are looked through.
            constexpr int CPR = D / 8;                      // 16-byte pieces of a row
            const int keep = lim_last + 1 - key0;           // >= 1 here
            if (keep < 16) {
              for (int i = lane; i < (16 - keep) * CPR; i += 32) {
                const int row = kg * 16 + keep + i / CPR, c = i % CPR;
                *reinterpret_cast<uint4*>(vs + (c >> 3) * C::HALF + swz128(row, c & 7)) = make_uint4(0, 0, 0, 0);
              }
              fence_proxy_async_smem();                     // before the slot's next copy
              __syncwarp();
            }
            if (!BLOCK && lim_all < lim_last) {
              uint32_t bad = 0;
              for (int i = lane; i < 16 * CPR; i += 32)
                bad |= not_finite<T>(*reinterpret_cast<const uint4*>(vs + ((i % CPR) >> 3) * C::HALF + swz128(kg * 16 + i / CPR, i % CPR & 7)));
              odd_values = __any_sync(0xffffffffu, bad != 0);
            }
          }
          float tA = fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[1][0], s[1][1]));
          float tB = fmaxf(fmaxf(s[0][2], s[0][3]), fmaxf(s[1][2], s[1][3]));
#pragma unroll
          for (int d = 1; d < 4; d <<= 1) {
            tA = fmaxf(tA, __shfl_xor_sync(0xffffffffu, tA, d));
            tB = fmaxf(tB, __shfl_xor_sync(0xffffffffu, tB, d));
          }
          // (maxima are kept as scores, before the scale: the largest score less the maximum is then exactly 0, where
          // scale * score - scaled maximum in one FMA would leave the rounding of the maximum, beyond 2^30 a factor of 2^64)
          const float nA = fmaxf(mA, tA), nB = fmaxf(mB, tB);
          if (__any_sync(0xffffffffu, nA > mA || nB > mB)) {
            const float fA = nA > mA ? ex2_approx((mA - nA) * p.scale_log2) : 1.f, fB = nB > mB ? ex2_approx((mB - nB) * p.scale_log2) : 1.f;
            lA *= fA; lB *= fB;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) { o[n][0] *= fA; o[n][1] *= fA; o[n][2] *= fB; o[n][3] *= fB; }
            mA = nA; mB = nB;
          }
          // a row that has seen nothing yet: every term exp2(-inf - 0) = 0
          const float uA = mA == -INFINITY ? 0.f : mA, uB = mB == -INFINITY ? 0.f : mB;
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              s[n][e] = ex2_approx(fmaf(s[n][e] - uA, p.scale_log2, kShift));
              s[n][2 + e] = ex2_approx(fmaf(s[n][2 + e] - uB, p.scale_log2, kShift));
              lA += s[n][e];
              lB += s[n][2 + e];
            }
          uint32_t ph[4], pl[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {                      // A operand: (row, keys 0-7), (row + 8, 0-7), (row, 8-15), (row + 8, 8-15)
            const float x = s[j >> 1][(j & 1) * 2], y = s[j >> 1][(j & 1) * 2 + 1];
            ph[j] = T::pack(x, y);
            pl[j] = T::pack(x - T::lo(ph[j]), y - T::hi(ph[j]));
          }
          if (!BLOCK && odd_values) {
            // added to the rows that see them, and taken out of the product, where 0 times them would reach the others
#pragma unroll 1
            for (int k = 0; k < 16; ++k) {
              const bool a = key0 + k <= limA, b = key0 + k <= limB;
#pragma unroll
              for (int n = 0; n < D / 8; ++n) {
                const uint32_t x = *reinterpret_cast<const uint32_t*>(vs + (n >> 3) * C::HALF + swz128(kg * 16 + k, n & 7) + cc * 2);
                const uint32_t f = not_finite<T>(x);
                if (f & 0x8000u) { o[n][0] += a ? T::lo(x) : 0.f; o[n][2] += b ? T::lo(x) : 0.f; }
                if (f >> 31) { o[n][1] += a ? T::hi(x) : 0.f; o[n][3] += b ? T::hi(x) : 0.f; }
              }
            }
            __syncwarp();
            for (int i = lane; i < 16 * (D / 2); i += 32) {
              const int d2 = i % (D / 2);
              uint32_t* x = reinterpret_cast<uint32_t*>(vs + (d2 >> 5) * C::HALF + swz128(kg * 16 + i / (D / 2), (d2 >> 2) & 7) + (d2 & 3) * 4);
              *x = finite_part<T>(*x);
            }
            fence_proxy_async_smem();
            __syncwarp();
          }
          {
            const int row = kg * 16 + (((lane >> 3) & 1) << 3) + (lane & 7), sub = lane >> 4;
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
              uint32_t bf[4];
              ldmatrix_x4_trans(bf, smem_u32(vs) + (n >> 2) * C::HALF + swz128(row, (2 * n + sub) & 7));
              T::mma(o[2 * n], ph, bf[0], bf[1]);
              T::mma(o[2 * n + 1], ph, bf[2], bf[3]);
              T::mma(o[2 * n], pl, bf[0], bf[1]);
              T::mma(o[2 * n + 1], pl, bf[2], bf[3]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[stage]);
      }

      // ---- the warps' softmaxes joined; a thread ends up with PER of 64 dims of one row
      mA = mA * p.scale_log2 - kShift; mB = mB * p.scale_log2 - kShift;
#pragma unroll
      for (int d = 1; d < 4; d <<= 1) {
        lA += __shfl_xor_sync(0xffffffffu, lA, d);
        lB += __shfl_xor_sync(0xffffffffu, lB, d);
      }
      if ((lane & 3) == 0) {
        stat[(warp * kRowTile + rA) * 2] = mA; stat[(warp * kRowTile + rA) * 2 + 1] = lA;
        stat[(warp * kRowTile + rB) * 2] = mB; stat[(warp * kRowTile + rB) * 2 + 1] = lB;
      }
      named_barrier(1, kRowWarps * 32);
      float MA = -INFINITY, MB = -INFINITY;
#pragma unroll
      for (int i = 0; i < kRowWarps; ++i) {
        MA = fmaxf(MA, stat[(i * kRowTile + rA) * 2]);
        MB = fmaxf(MB, stat[(i * kRowTile + rB) * 2]);
      }
      // (a warp that has seen nothing has the sum 0; one that has seen no numbers alone has no maximum, but no 0 either)
      const float sA = lA == 0.f ? 0.f : ex2_approx(mA - MA), sB = lB == 0.f ? 0.f : ex2_approx(mB - MB);
      constexpr int PER = 32 / kRowWarps, TPR = 64 / PER;      // dims of a thread, threads of a row
      const int row = tid / TPR, dp = tid % TPR * PER;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int i = 0; i < kRowWarps; ++i) M = fmaxf(M, stat[(i * kRowTile + row) * 2]);
#pragma unroll
      for (int i = 0; i < kRowWarps; ++i) {
        const float l = stat[(i * kRowTile + row) * 2 + 1];
        if (l != 0.f) L += l * ex2_approx(stat[(i * kRowTile + row) * 2] - M);
      }
      const bool fin = w.whole();              // in a cluster: the unit is this CTA's alone
      const int slot = w.slot(cta);
      const int r = w.r_first + row;
      const size_t out_row = (size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group;
#pragma unroll
      for (int x = 0; x < C::HALVES; ++x) {
        // rows of 64 floats, 8-float pieces rotated by the row so that the column accesses spread over the banks
        float* mine = red + warp * kRowTile * 64;
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          const int pa = ((n + rA) & 7) * 8 + cc, pb = ((n + rB) & 7) * 8 + cc;
          *reinterpret_cast<float2*>(mine + rA * 64 + pa) = make_float2(o[x * 8 + n][0] * sA, o[x * 8 + n][1] * sA);
          *reinterpret_cast<float2*>(mine + rB * 64 + pb) = make_float2(o[x * 8 + n][2] * sB, o[x * 8 + n][3] * sB);
        }
        named_barrier(1, kRowWarps * 32);
        float a[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) a[e] = 0.f;
#pragma unroll
        for (int i = 0; i < kRowWarps; ++i)
#pragma unroll
          for (int e = 0; e < PER; e += 4) {
            const float4 u = *reinterpret_cast<const float4*>(red + (i * kRowTile + row) * 64 + (((dp >> 3) + row) & 7) * 8 + (dp & 7) + e);
            a[e] += u.x; a[e + 1] += u.y; a[e + 2] += u.z; a[e + 3] += u.w;
          }
        if (row < w.rows) {
          const float inv = L != 0.f ? 1.f / L : 0.f;
          float* part = (SPLIT ? keep + (size_t)row * D : p.row_part + ((size_t)slot * kRowTile + row) * D) + x * 64 + dp;
#pragma unroll
          for (int e = 0; e < PER; e += 4) {
            if (fin)
              *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.y) + out_row * D + x * 64 + dp + e) =
                  make_uint2(T::pack(a[e] * inv, a[e + 1] * inv), T::pack(a[e + 2] * inv, a[e + 3] * inv));
            else
              *reinterpret_cast<float4*>(part + e) = make_float4(a[e], a[e + 1], a[e + 2], a[e + 3]);
          }
        }
        named_barrier(1, kRowWarps * 32);
      }
      if (tid % TPR == 0 && row < w.rows) {
        if (fin) {
          if (p.lse) p.lse[out_row] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
        } else {
          float* st = SPLIT ? keep_stat + row * 2 : p.row_stat + ((size_t)slot * kRowTile + row) * 2;
          st[0] = M;
          st[1] = L;
        }
      }
    }
  }
  if (SPLIT && p.n_split > 1) {
    // ================================================================ join of the cluster's pieces, rank by rank
    __syncwarp();
    cluster_sync();
    RowWalk<BLOCK, SPLIT> w(p, cta);
    const int rank = cta % p.n_split;
    const int per = (w.tiles + p.n_split - 1) / p.n_split;
    const int pieces = w.rows > 0 && w.tiles > per ? (w.tiles + per - 1) / per : 0;     // 0: nothing to join
    if (pieces > 0 && warp < kRowWarps) {
      // rows in turn over the ranks' warps; a lane owns D / 32 dims
      constexpr int V = D / 32;
      for (int row = rank * kRowWarps + warp; row < w.rows; row += p.n_split * kRowWarps) {
        float2 st[8];
        float2 v[8][V / 2];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int from = i < pieces ? i : 0;
          st[i] = ld_cluster_f2(keep_stat + row * 2, from);
#pragma unroll
          for (int e = 0; e < V / 2; ++e) v[i][e] = ld_cluster_f2(keep + (size_t)row * D + lane * V + 2 * e, from);
        }
        float M = -INFINITY, L = 0.f, a[V];
#pragma unroll
        for (int e = 0; e < V; ++e) a[e] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < pieces) M = fmaxf(M, st[i].x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float f = i < pieces && st[i].y != 0.f ? ex2_approx(st[i].x - M) : 0.f;
          L += st[i].y * f;
#pragma unroll
          for (int e = 0; e < V / 2; ++e) { a[2 * e] += v[i][e].x * f; a[2 * e + 1] += v[i][e].y * f; }
        }
        const float inv = L != 0.f ? 1.f / L : 0.f;
        const int r = w.r_first + row;
        const size_t out_row = (size_t)(w.tok0 + r / p.group) * p.hq + w.h * p.group + r % p.group;
        uint32_t* y = static_cast<uint32_t*>(p.y) + out_row * (D / 2) + lane * (V / 2);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) y[e] = T::pack(a[2 * e] * inv, a[2 * e + 1] * inv);
        if (lane == 0 && p.lse) p.lse[out_row] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
      }
    }
    __syncwarp();
    cluster_sync();                            // shared memory is read by the other ranks until here
  }
  __syncthreads();
  if (*s_abort && tid == 0) atomicExch(p.status, kStatusTimeout);
  // (beside a tile-kernel launch this grid may run next to it: it must not be complete before that one is, because the
  // joins that follow wait for this grid only)
  if (p.beside) pdl_wait();
}

// Joins the partial results of the units that were cut: a CTA per (unit, row), in groups of one thread per pair of dims;
// the parts go to the groups in turn, and everything is added in a fixed order.
constexpr int kMergeThreads = 256;
template <typename T, int D, bool BLOCK>
__global__ void __launch_bounds__(kMergeThreads) paged_rows_merge_kernel(const __grid_constant__ PagedProblem p) {
  constexpr int TPG = D / 2, GROUPS = kMergeThreads / TPG;
  __shared__ float s_stat[GROUPS][2];
  __shared__ float2 s_acc[GROUPS][TPG];
  pdl_wait();
  pdl_launch_next();
  const int lane = threadIdx.x & 31, row = blockIdx.y;
  int first, count, step, rows, tok0, h, r;
  if (BLOCK) {
    const int unit = blockIdx.x, tok = unit / p.hkv;
    h = unit % p.hkv;
    const int b = paged_seq_of(p, tok);
    int pos = paged_kv_len(p, b) - paged_q_len(p, b) + (tok - (int)__ldg(p.cu_q + b));
    if (pos < 0) pos = 0;
    const int seen = (pos >> p.page_shift) + 1, n_list = seen < p.n_keep ? seen : p.n_keep;
    const int tiles = ((n_list << p.page_shift) + kRowKeys - 1) / kRowKeys, per = (tiles + p.n_split - 1) / p.n_split;
    count = (tiles + per - 1) / per;
    first = unit * p.n_split;
    step = 1;
    rows = p.group; tok0 = tok; r = row;
  } else {
    // the line as the row kernel cut it
    const int unit = blockIdx.x, b = unit / p.hkv;
    h = unit % p.hkv;
    int before = 0, total = 0, mine = 0, my_tiles = 1;
    for (int s = 0; s < p.batch; s += 32) {
      int w = 0, tl = 1;
      if (s + lane < p.batch) {
        const int q = paged_q_len(p, s + lane), len = paged_kv_len(p, s + lane);
        int rw = q > 0 ? q * p.group : 0;
        if (rw > p.rows_limit) rw = 0;
        tl = len > 0 ? (len + kRowKeys - 1) / kRowKeys : 1;
        w = tl * p.hkv * ((rw + kRowTile - 1) / kRowTile);
        if (s + lane == b) mine = rw;
      }
      total += __reduce_add_sync(0xffffffffu, w);
      before += __reduce_add_sync(0xffffffffu, s + lane < b ? w : 0);
      if (b >= s && b < s + 32) { mine = __shfl_sync(0xffffffffu, mine, b - s); my_tiles = __shfl_sync(0xffffffffu, tl, b - s); }
    }
    const int rt = row / kRowTile;
    if (row >= mine) return;
    const int per = (total + p.row_ctas - 1) / p.row_ctas;
    const int u0 = before + (rt * p.hkv + h) * my_tiles, u1 = u0 + my_tiles;
    const int c0 = u0 / per, c1 = (u1 - 1) / per;
    count = c1 - c0 + 1;
    first = 2 * c0;                       // the first part starts at the unit's first tile: slot 2 c0 + 1, then 2 (c0 + i)
    step = 2;
    rows = mine; tok0 = (int)__ldg(p.cu_q + b); r = row;
  }
  if (count < 2 || row >= rows) return;   // written by the row kernel itself
  const int rr = r % kRowTile, grp = threadIdx.x / TPG, d = threadIdx.x % TPG;
  float M = -INFINITY, L = 0.f, a0 = 0.f, a1 = 0.f;
  for (int i0 = grp; i0 < count; i0 += 4 * GROUPS) {
    float2 st[4], v[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int i = i0 + x * GROUPS;
      st[x] = make_float2(-INFINITY, 0.f);
      v[x] = make_float2(0.f, 0.f);
      if (i < count) {
        const size_t s = (size_t)(BLOCK ? first + i : i == 0 ? first + 1 : first + step * i) * kRowTile + rr;
        st[x] = __ldcg(reinterpret_cast<const float2*>(p.row_stat) + s);
        v[x] = __ldcg(reinterpret_cast<const float2*>(p.row_part + s * D) + d);
      }
    }
    const float m = fmaxf(fmaxf(fmaxf(st[0].x, st[1].x), fmaxf(st[2].x, st[3].x)), M);
    const float g = M == -INFINITY ? 0.f : ex2_approx(M - m);
    L *= g; a0 *= g; a1 *= g;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float f = st[x].y == 0.f ? 0.f : ex2_approx(st[x].x - m);
      L += st[x].y * f;
      a0 += v[x].x * f;
      a1 += v[x].y * f;
    }
    M = m;
  }
  if (d == 0) { s_stat[grp][0] = M; s_stat[grp][1] = L; }
  s_acc[grp][d] = make_float2(a0, a1);
  __syncthreads();
  if (grp > 0) return;
  M = -INFINITY; L = 0.f; a0 = 0.f; a1 = 0.f;
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) M = fmaxf(M, s_stat[i][0]);
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const float f = s_stat[i][1] == 0.f ? 0.f : ex2_approx(s_stat[i][0] - M);
    const float2 v = s_acc[i][d];
    L += s_stat[i][1] * f;
    a0 += v.x * f;
    a1 += v.y * f;
  }
  const float inv = L != 0.f ? 1.f / L : 0.f;
  const size_t out_row = (size_t)(tok0 + r / p.group) * p.hq + h * p.group + r % p.group;
  reinterpret_cast<uint32_t*>(p.y)[out_row * (D / 2) + d] = T::pack(a0 * inv, a1 * inv);
  if (d == 0 && p.lse) p.lse[out_row] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

template <typename T, int D, bool BLOCK, bool SPLIT>
static cudaError_t launch_rows_s(const PagedProblem& p, const CUtensorMap& tk, const CUtensorMap& tv, int grid, cudaStream_t st) {
  static PerDeviceFlag configured;
  const size_t smem = RowCfg<D, SPLIT>::total;
  const cudaError_t e = set_max_dynamic_smem(configured, reinterpret_cast<const void*>(paged_rows_kernel<T, D, BLOCK, SPLIT>), smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(RowCfg<D, SPLIT>::THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.n_split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = SPLIT && p.n_split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, paged_rows_kernel<T, D, BLOCK, SPLIT>, tk, tv, p);
}

template <typename T, int D, bool BLOCK>
static cudaError_t launch_rows_t(const PagedProblem& p, const CUtensorMap& tk, const CUtensorMap& tv, int grid, bool split,
                                 cudaStream_t st) {
  return split ? launch_rows_s<T, D, BLOCK, true>(p, tk, tv, grid, st) : launch_rows_s<T, D, BLOCK, false>(p, tk, tv, grid, st);
}

template <typename T, int D, bool BLOCK>
static cudaError_t launch_merge_t(const PagedProblem& p, int units, int max_rows, cudaStream_t st) {
  return launch_pdl(paged_rows_merge_kernel<T, D, BLOCK>, dim3(units, max_rows), dim3(kMergeThreads), 0, st, p);
}

#define TKPHI_BY_TYPE(call)                                                          \
  (d == 64 ? (bf16 ? (block ? call(Bf16, 64, true) : call(Bf16, 64, false))           \
                   : (block ? call(Fp16, 64, true) : call(Fp16, 64, false)))          \
           : (bf16 ? (block ? call(Bf16, 128, true) : call(Bf16, 128, false))         \
                   : (block ? call(Fp16, 128, true) : call(Fp16, 128, false))))

cudaError_t launch_paged_rows(const PagedProblem& p, const CUtensorMap& tk, const CUtensorMap& tv, int d, bool bf16,
                              bool block, bool split, int grid, cudaStream_t st) {
#define ROWS(T, D, B) launch_rows_t<T, D, B>(p, tk, tv, grid, split, st)
  return TKPHI_BY_TYPE(ROWS);
#undef ROWS
}

cudaError_t launch_paged_rows_merge(const PagedProblem& p, int d, bool bf16, bool block, int units, int max_rows,
                                    cudaStream_t st) {
#define MERGE(T, D, B) launch_merge_t<T, D, B>(p, units, max_rows, st)
  return TKPHI_BY_TYPE(MERGE);
#undef MERGE
}

}  // namespace tkphi

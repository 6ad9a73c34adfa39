// What the row kernels of 16-bit and of 8-bit caches share: how the work is dealt out (tiles of KEYS keys), the joins.
#pragma once

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

// The pieces of one CTA: (unit, tile range) one after the other.  Every warp runs its own copy.
template <bool BLOCK, bool SPLIT, int KEYS>
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
      seq_tiles = seq_len > 0 ? (seq_len + KEYS - 1) / KEYS : 1;
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
      tiles = ((n_list << p.page_shift) + KEYS - 1) / KEYS;
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

// Join of a cluster's pieces, rank by rank: keep [16][D] and keep_stat [16][2] are every CTA's piece in shared memory.
template <typename T, int D, bool BLOCK, int KEYS, int WARPS>
__device__ __forceinline__ void join_cluster(const PagedProblem& p, int cta, const float* keep, const float* keep_stat) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncwarp();
  cluster_sync();
  RowWalk<BLOCK, true, KEYS> w(p, cta);
  const int rank = cta % p.n_split;
  const int per = (w.tiles + p.n_split - 1) / p.n_split;
  const int pieces = w.rows > 0 && w.tiles > per ? (w.tiles + per - 1) / per : 0;     // 0: nothing to join
  if (pieces > 0 && warp < WARPS) {
    // rows in turn over the ranks' warps; a lane owns D / 32 dims
    constexpr int V = D / 32;
    for (int row = rank * WARPS + warp; row < w.rows; row += p.n_split * WARPS) {
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

// Joins the partial results of the units that were cut: a CTA per (unit, row), in groups of one thread per pair of dims;
// the parts go to the groups in turn, and everything is added in a fixed order.
constexpr int kMergeThreads = 256;
template <typename T, int D, bool BLOCK, int KEYS>
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
    const int tiles = ((n_list << p.page_shift) + KEYS - 1) / KEYS, per = (tiles + p.n_split - 1) / p.n_split;
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
        tl = len > 0 ? (len + KEYS - 1) / KEYS : 1;
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

}  // namespace tkphi

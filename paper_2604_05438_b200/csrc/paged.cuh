// Shared declarations of the paged-cache kernels: the problem as the kernels see it, element types,
// sequence look-ups.  sm_100a only.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"
#include "sm100.cuh"

namespace tkphi {

constexpr int kStatusBadPage = -1;          // a page-table entry outside [0, n_pages) was met
constexpr int kRowTile = 16;                // query rows (tokens x query heads of a KV head) of a row-kernel unit
constexpr int kRowKeys = 64;                // keys of one tile of the row kernel
constexpr int kTileRows = 256;              // rows of a tile-kernel CTA: two 128-row MMA tiles
constexpr int kTileKeys = 128;              // keys of one tile of the tile kernel
constexpr int kMaxSelectPages = 131072;     // pages of a sequence of the page-selected form
constexpr int kMaxKvLen = 1 << 30;          // cache rows of a sequence: a length and a chunk of it add up within 31 bits
constexpr int kMaxGroup = 16;               // query heads per KV head of the paged calls

// One step over a paged cache.  Sequence b brings cu_q[b+1] - cu_q[b] new tokens, the last ones of its
// kv_lens[b] cache rows.  "Rows" of a KV head are its query vectors, token-major: row r is token r / group,
// query head r % group of the group.
struct PagedProblem {
  int batch, hq, hkv, group;
  int page_shift, n_pages, max_pages;
  const int* table;                // [batch][max_pages]
  const long long* kv_lens;        // [batch]
  const long long* cu_q;           // [batch + 1]
  int max_kv;                      // no sequence is read beyond this many rows
  int total_q;
  const void* q; void* y; float* lse;      // [total_q][hq][d], [total_q][hq]
  float scale_log2;                // softmax scale * log2 e
  int causal;
  int* status;
  // row kernel: sequences with at most rows_limit rows
  int rows_limit;
  int row_ctas;                    // CTAs that share the tiles of all units evenly
  int n_split;                     // CTAs per unit where units are cut evenly instead (clusters; the block form)
  int beside;                      // launched beside the tile kernel: does not wait for it before its end
  float* row_part;                 // [2 * row_ctas or units * n_split][16][d] unnormalised partial outputs
  float* row_stat;                 // [..][16][2] their maximum (log2 units) and sum
  // page selection
  int n_keep, n_sink, n_tail, topk;
  int scored;                      // the selection follows a scoring grid
  int held;                        // scores that the selecting CTAs have shared memory for (a multiple of 4)
  const void* bounds;              // [n_pages][hkv][2][d]
  float* page_scores;              // [units][key_stride] 32-bit bounds of the candidate pages
  unsigned long long* page_keys;   // [units][key_stride] their 64-bit bounds as ordered keys, where many are equal
  int key_stride;
  uint4* page_mags;                // [units][mag_parts] per scoring CTA: largest sum of magnitudes behind a bound (bits), smallest
                                   // and largest bound (ordered keys)
  int mag_parts;
  int* page_list;                  // [units][n_keep] physical pages, -1 padded
  int* page_out;                   // [units][n_keep] logical pages, -1 padded, or null
  // tile kernel: sequences with more than rows_limit rows
  int chunk;                       // keys per CTA (a multiple of kTileKeys)
  float* tile_part;                // [CTAs][256][d]
  float* tile_stat;                // [CTAs][256][2]
};

// ---------------------------------------------------------------- 16-bit element types
struct Bf16 {
  static constexpr bool kBf16 = true;
  static constexpr uint32_t kExp = 0x7f807f80u, kExpUnit = 0x00800080u;      // exponent fields of a pair and their lowest bits
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
  static __device__ __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t r; asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r;
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r; asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r;
  }
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};
struct Fp16 {
  static constexpr bool kBf16 = false;
  static constexpr uint32_t kExp = 0x7c007c00u, kExpUnit = 0x04000400u;
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float lo(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xffffu))); }
  static __device__ __forceinline__ float hi(uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w >> 16))); }
  static __device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t r; asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r;
  }
  static __device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t r; asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r;
  }
  static __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
};

// The sign bits of the pair's elements that are infinite or no number (an exponent of ones carries into the sign bit).
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & T::kExp) + T::kExpUnit) & 0x80008000u; }
template <typename T>
__device__ __forceinline__ uint32_t not_finite(const uint4& v) {
  return not_finite<T>(v.x) | not_finite<T>(v.y) | not_finite<T>(v.z) | not_finite<T>(v.w);
}
// The pair with those elements 0.
template <typename T>
__device__ __forceinline__ uint32_t finite_part(uint32_t w) {
  const uint32_t bad = not_finite<T>(w) >> 15;               // 1 in the element's lowest bit
  return w & ~(bad * 0xffffu);
}

// ---------------------------------------------------------------- sequences
__device__ __forceinline__ int paged_kv_len(const PagedProblem& p, int b) {
  const long long n = __ldg(p.kv_lens + b);
  return n < 0 ? 0 : n > p.max_kv ? p.max_kv : (int)n;
}
__device__ __forceinline__ int paged_q_len(const PagedProblem& p, int b) {
  return (int)(__ldg(p.cu_q + b + 1) - __ldg(p.cu_q + b));
}
// Sequence of query token t (whole warp).
__device__ __forceinline__ int paged_seq_of(const PagedProblem& p, int t) {
  const int lane = threadIdx.x & 31;
  int b = 0;
  for (int s = 0; s < p.batch; s += 32) {
    const bool before = s + lane < p.batch && __ldg(p.cu_q + s + lane + 1) <= t;
    const unsigned m = __ballot_sync(0xffffffffu, before);
    b += __popc(m);
    if (m != 0xffffffffu) break;
  }
  return b;
}
__device__ __forceinline__ int warp_inclusive_scan(int v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int n = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += n;
  }
  return v;
}

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* tm, uint64_t* bar, int c0, int c1, int c2,
                                            int c3, uint64_t l2_policy) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%3, %4, %5, %6}], [%2], %7;" ::"r"(smem_u32(dst)),
      "l"(tm), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "l"(l2_policy)
      : "memory");
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t saddr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t saddr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(saddr) : "memory");
}
__device__ __forceinline__ void named_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// Query rows of an MMA tile: whole tokens, so that a tile of queries is one box of the tensor map.
__host__ __device__ inline int tile_rows(int group) { return 128 / group * group; }
// Rows of a scoring tile: tokens of one sequence x the group padded to a power of two.
__host__ __device__ inline int padded_group(int g) { return g <= 1 ? 1 : g <= 2 ? 2 : g <= 4 ? 4 : g <= 8 ? 8 : 16; }

// ---------------------------------------------------------------- launches (host)
struct AppendProblem {
  int batch, hq, hkv, group, d;
  int page_shift, n_pages, max_pages;
  const int* table;
  const long long* kv_lens;
  const long long* cu_q;
  long long max_kv;
  void* k; void* v;
  long long stride_page, stride_head, stride_token;
  const void* k_new; const void* v_new;
  long long k_new_token, k_new_head, v_new_token, v_new_head;
  const void* q; void* q_out;
  long long q_token, q_head, q_out_token, q_out_head;
  const float* inv_freq;           // [rot / 2]
  int rot, pairs;
  const long long* positions;      // [total_q] or null: the cache position of each token
  void* bounds;
  int* status;
  long long total_q;
  int items;                       // CTAs per KV head: spans of 64 positions (or a page of 128) of all sequences, at most
};
cudaError_t launch_paged_append(const AppendProblem& p, bool bf16, cudaStream_t st);
cudaError_t launch_paged_rows(const PagedProblem& p, const CUtensorMap& tk, const CUtensorMap& tv, int d, bool bf16,
                              bool block, bool split, int grid, cudaStream_t st);
int paged_score_parts(int row_tiles, int hkv, int n);        // scoring CTAs per row tile and KV head, for n candidates
cudaError_t launch_paged_select(const PagedProblem& p, int d, bool bf16, int max_pages_seq, int row_tiles, cudaStream_t st);
cudaError_t launch_paged_rows_merge(const PagedProblem& p, int d, bool bf16, bool block, int units, int max_rows, cudaStream_t st);

cudaError_t launch_paged_tiles(const PagedProblem& p, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tq, int d,
                               bool bf16, int grid, cudaStream_t st);
cudaError_t launch_paged_tiles_merge(const PagedProblem& p, int d, bool bf16, cudaStream_t st);

}  // namespace tkphi

// Rows of an 8-bit paged cache back as 16-bit rows: out[cu_rows[b] + i] = codes * 2^(e - 127) of position first[b] + i of
// sequence b, for keys and values, rounded once to the element type (exact in bf16 from 2^-130 to its largest number).
//
// Bound: memory, 2 (d + 1) bytes in and 4 d out per row and head.  A thread has 16 codes of a row's keys and values and writes
// 32 bytes of each; a CTA takes 64 rows and several KV heads, one after the other, so that looking up the rows' places is
// paid once, with the next head's loads in flight while one head is written.
// Measured: 1.6 GB of eight sequences of 8K-64K rows, 24 / 8 heads of 128, 302 us (6.2 TB/s of codes and rows).  What counted:
// 32-byte stores (369 us with two of 16), several heads per CTA; for token-major pages reads that bring 256 bytes into the
// second-level cache (250K rows of 8 heads of 64 expanded to 16 bits: 145 -> 116 us).
#include "held8.cuh"

namespace tkphi {

constexpr int kReadThreads = 256;

// 32 bytes, in one store where they are aligned to that: two of 16 write half sectors.
__device__ __forceinline__ void put32(uint16_t* to, const uint4& a, const uint4& c, bool aligned) {
  if (aligned) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(c.x),
                 "r"(c.y), "r"(c.z), "r"(c.w) : "memory");
  } else {
    reinterpret_cast<uint4*>(to)[0] = a;
    reinterpret_cast<uint4*>(to)[1] = c;
  }
}

// 16 codes.  Token-major pages have a row's heads beside each other, and this CTA's next heads are there.
__device__ __forceinline__ uint4 load_codes(const uint8_t* from) {
  uint4 v;
  asm("ld.global.nc.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(from));
  return v;
}

// What a thread has of one row and head.
struct HeldPiece { uint4 k, v; uint32_t ke, ve; };

// Heads h0 .. h1-1 of ROWS rows: row i * rows-per-pass + tid / lanes-per-row of the CTA is read if ok[i], at `at[i]` of the codes
// and `scale_at[i]` of the scales, and written by put(i, head, keys or values, 32 bytes as two pieces).
template <typename T, int PASSES, typename Put>
__device__ __forceinline__ void copy_heads(const uint8_t* k, const uint8_t* v, const HeldCache& held, long long stride_head, int page_rows,
                                           int h0, int h1, const bool (&ok)[PASSES], const size_t (&at)[PASSES],
                                           const size_t (&scale_at)[PASSES], Put put) {
  HeldPiece now[PASSES], next[PASSES];
  auto load = [&](HeldPiece (&x)[PASSES], int h) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      x[i].k = x[i].v = make_uint4(0, 0, 0, 0);
      x[i].ke = x[i].ve = 0;
      if (!ok[i]) continue;
      const size_t c = at[i] + (size_t)h * stride_head, e = scale_at[i] + (size_t)h * page_rows;
      if (k) { x[i].k = load_codes(k + c); x[i].ke = __ldg(held.k_scales + e); }
      if (v) { x[i].v = load_codes(v + c); x[i].ve = __ldg(held.v_scales + e); }
    }
  };
  load(next, h0);
  for (int h = h0; h < h1; ++h) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) now[i] = next[i];
    if (h + 1 < h1) load(next, h + 1);
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint4 w = s ? now[i].v : now[i].k;
        const float f = held_scale(s ? now[i].ve : now[i].ke);
        const uint2 a = held_values<T>(w.x, f), c = held_values<T>(w.y, f), d = held_values<T>(w.z, f), e = held_values<T>(w.w, f);
        put(i, h, s, make_uint4(a.x, a.y, c.x, c.y), make_uint4(d.x, d.y, e.x, e.y));
      }
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(kReadThreads) paged_read_kernel(const __grid_constant__ ReadProblem p) {
  constexpr int LPR = D / 16, RPP = kReadThreads / LPR, PASSES = kReadRows / RPP;
  static_assert(PASSES >= 1, "rows of a CTA");
  __shared__ int s_seq;
  const int tid = threadIdx.x, lane = tid & 31;
  const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, p.hkv);
  const long long row0 = (long long)blockIdx.x * kReadRows;
  pdl_wait();
  pdl_launch_next();
  if (tid < 32) {
    // the sequence of the first row
    int b = 0;
    for (int s = 0; s < p.batch; s += 32) {
      const bool before = s + lane < p.batch && __ldg(p.cu_rows + s + lane + 1) <= row0;
      const unsigned m = __ballot_sync(0xffffffffu, before);
      b += __popc(m);
      if (m != 0xffffffffu) break;
    }
    if (lane == 0) s_seq = b;
  }
  __syncthreads();
  int b = s_seq;
  const int l = tid % LPR, ps = 1 << p.page_shift;
  bool ok[PASSES];
  size_t at[PASSES], scale_at[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const long long row = row0 + i * RPP + tid / LPR;
    ok[i] = false;
    at[i] = scale_at[i] = 0;
    if (row >= p.total_rows) continue;
    while (b < p.batch && __ldg(p.cu_rows + b + 1) <= row) ++b;
    if (b >= p.batch) continue;
    const long long pos = row - __ldg(p.cu_rows + b) + (p.first ? __ldg(p.first + b) : 0ll);
    if (pos < 0 || pos >= __ldg(p.kv_lens + b) || pos >= p.max_kv) continue;       // (a replay with shorter device lengths: not written)
    const int page = __ldg(p.table + (size_t)b * p.max_pages + (pos >> p.page_shift));
    if (page < 0 || page >= p.n_pages) {
      if (l == 0) atomicExch(p.status, kStatusBadPage);
      continue;
    }
    const int slot = (int)(pos & (ps - 1));
    ok[i] = true;
    at[i] = (size_t)page * p.stride_page + (size_t)slot * p.stride_token + l * 16;
    scale_at[i] = (size_t)page * p.hkv * ps + slot;
  }
  const bool wide = ((reinterpret_cast<uintptr_t>(p.k_out) | reinterpret_cast<uintptr_t>(p.v_out)) & 31u) == 0 &&
                    ((p.k_row | p.k_head | p.v_row | p.v_head) & 15ll) == 0;
  copy_heads<T>(p.k_out ? p.k : nullptr, p.v_out ? p.v : nullptr, p.held, p.stride_head, ps, h0, h1, ok, at, scale_at,
                [&](int i, int h, int s, const uint4& a, const uint4& c) {
                  void* out = s ? p.v_out : p.k_out;
                  if (!ok[i] || !out) return;
                  const size_t row = (size_t)(row0 + i * RPP + tid / LPR);
                  put32(static_cast<uint16_t*>(out) + row * (s ? p.v_row : p.k_row) + (size_t)h * (s ? p.v_head : p.k_head) + l * 16, a, c, wide);
                });
}

// Heads of a CTA: all of them, or fewer where there are not CTAs enough to go round.
static int heads_per_cta(long long blocks, int hkv) {
  int n = hkv;
  while (n > 1 && blocks * ((hkv + n - 1) / n) < 8 * sm_count_current_device()) n = (n + 1) / 2;
  return n;
}

cudaError_t launch_paged_read(const ReadProblem& q, bool bf16, cudaStream_t st) {
  ReadProblem p = q;
  const long long blocks = (p.total_rows + kReadRows - 1) / kReadRows;
  p.heads = heads_per_cta(blocks, p.hkv);
  const dim3 grid((unsigned)blocks, (p.hkv + p.heads - 1) / p.heads), block(kReadThreads);
  if (p.d == 64)
    return bf16 ? launch_pdl(paged_read_kernel<Bf16, 64>, grid, block, 0, st, p) : launch_pdl(paged_read_kernel<Fp16, 64>, grid, block, 0, st, p);
  return bf16 ? launch_pdl(paged_read_kernel<Bf16, 128>, grid, block, 0, st, p) : launch_pdl(paged_read_kernel<Fp16, 128>, grid, block, 0, st, p);
}

// ---------------------------------------------------------------- for attention of many rows
// The caches of the sequences with many rows as 16-bit pages of 128 rows in the workspace, [page][head][slot][dim], one
// sequence's pages behind another's, and a page table of them; rounded as the rows that are read back.  A CTA takes half a page.  Rows at or behind a sequence's length and on bad pages become 0.
template <typename T, int D>
__global__ void __launch_bounds__(kReadThreads) paged_expand_kernel(const __grid_constant__ PagedProblem p, const __grid_constant__ ExpandProblem x) {
  constexpr int LPR = D / 16, RPP = kReadThreads / LPR, PASSES = kReadRows / RPP, PARTS = kExpandRows / kReadRows;
  __shared__ int s_seq, s_page;
  const int tid = threadIdx.x, lane = tid & 31;
  const int out_page = blockIdx.x / PARTS, first = blockIdx.x % PARTS * kReadRows;
  const int h0 = blockIdx.y * x.heads, h1 = min(h0 + x.heads, p.hkv);
  pdl_wait();
  pdl_launch_next();
  if (tid < 32) {
    int base = 0;
    if (lane == 0) s_seq = -1;
    for (int s = 0; s < p.batch; s += 32) {
      int n = 0;
      if (s + lane < p.batch && (long long)paged_q_len(p, s + lane) * p.group > p.rows_limit) n = (paged_kv_len(p, s + lane) + kExpandRows - 1) / kExpandRows;
      const int incl = warp_inclusive_scan(n) + base;
      if (incl > out_page && incl - n <= out_page) {           // one lane
        s_seq = s + lane;
        s_page = out_page - (incl - n);
      }
      base = __shfl_sync(0xffffffffu, incl, 31);
      if (base > out_page) break;
    }
  }
  __syncthreads();
  const int b = s_seq;
  if (b < 0) return;                           // (a replay with shorter lengths)
  const int l = tid % LPR, ps = 1 << p.page_shift, len = paged_kv_len(p, b);
  if (h0 == 0 && first == 0 && tid == 0) x.table[(size_t)b * x.max_pages + s_page] = out_page;
  bool ok[PASSES];
  size_t at[PASSES], scale_at[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int pos = s_page * kExpandRows + first + i * RPP + tid / LPR;
    ok[i] = false;
    at[i] = scale_at[i] = 0;
    if (pos >= len) continue;
    const int page = __ldg(p.table + (size_t)b * p.max_pages + (pos >> p.page_shift));
    if (page < 0 || page >= p.n_pages) {
      if (l == 0) atomicExch(p.status, kStatusBadPage);
      continue;
    }
    const int slot = pos & (ps - 1);
    ok[i] = true;
    at[i] = (size_t)page * x.stride_page + (size_t)slot * x.stride_token + l * 16;
    scale_at[i] = (size_t)page * p.hkv * ps + slot;
  }
  copy_heads<T>(x.k, x.v, x.held, x.stride_head, ps, h0, h1, ok, at, scale_at, [&](int i, int h, int s, const uint4& a, const uint4& c) {
    const size_t row = ((size_t)out_page * p.hkv + h) * kExpandRows + first + i * RPP + tid / LPR;
    put32(static_cast<uint16_t*>(s ? x.v_out : x.k_out) + row * D + l * 16, a, c, true);
  });
}

cudaError_t launch_paged_expand(const PagedProblem& p, const ExpandProblem& q, int d, bool bf16, int pages, cudaStream_t st) {
  ExpandProblem x = q;
  const long long blocks = (long long)pages * (kExpandRows / kReadRows);
  x.heads = heads_per_cta(blocks, p.hkv);
  const dim3 grid((unsigned)blocks, (p.hkv + x.heads - 1) / x.heads), block(kReadThreads);
  if (d == 64)
    return bf16 ? launch_pdl(paged_expand_kernel<Bf16, 64>, grid, block, 0, st, p, x) : launch_pdl(paged_expand_kernel<Fp16, 64>, grid, block, 0, st, p, x);
  return bf16 ? launch_pdl(paged_expand_kernel<Bf16, 128>, grid, block, 0, st, p, x) : launch_pdl(paged_expand_kernel<Fp16, 128>, grid, block, 0, st, p, x);
}

}  // namespace tkphi
